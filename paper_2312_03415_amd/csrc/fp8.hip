// Quantisers of the 8-bit products (see fp8.hpp).  Both are bound by memory: a row quantiser's pass reads 2 bytes and writes 1 per
// element.
#include "fp8.hpp"

#include "gemm.hpp"
#include "gemm_engine.hpp"

namespace rl {
namespace {

constexpr int kThreads = 256;

// from the largest |bits| of a block: scale byte and multiplier 2^-e; not finite: multiplier 0 and byte 127, and *nan set
__device__ __forceinline__ void block_scale(uint32_t top, uint32_t* byte, float* mul, bool* nan) {
  *nan = top >= 0x7F800000u;
  int e = 0;
  if (top != 0u && !*nan) {
    // top = m 2^E, 1 <= m < 2 (denormals too: frexp); 448 = 1.75 * 2^8
    int E;
    const float m = frexpf(__uint_as_float(top), &E);  // m in [0.5, 1)
    e = m > 0.875f ? E - 8 : E - 9;
    if (e < -127) e = -127;
  }
  *byte = (uint32_t)(e + 127);
  *mul = *nan ? 0.f : ldexpf(1.f, -e);
}

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// eight consecutive elements
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[k] = a[k]; v[4 + k] = b[k]; }
  } else {
    const i32x4 a = *reinterpret_cast<const i32x4*>(p);
    const T* t = reinterpret_cast<const T*>(&a);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)t[k];
  }
}

// A wave takes a row's 512 columns at a time, 8 per lane, so that 16 lanes hold a block; a workgroup 4 RW rows.  The scale bytes
// of its rows go through LDS, so that they leave as runs of consecutive bytes.
template <typename T, int RW>
__global__ __launch_bounds__(kThreads) void fp8_rows_kernel(const T* __restrict__ X, int64_t ldx, int n, int K, uint8_t* __restrict__ q, int64_t ldq,
                                                            uint8_t* __restrict__ s, int64_t lds) {
  __shared__ uint8_t sc[4][4 * RW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = (int)blockIdx.y * 512 + lane * 8, r0 = (int)blockIdx.x * (4 * RW) + wave * RW;
  float v[RW][8];
#pragma unroll
  for (int j = 0; j < RW; ++j) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[j][k] = 0.f;
    if (r0 + j < n && col < K) load8(X + (int64_t)(r0 + j) * ldx + col, v[j]);
  }
#pragma unroll
  for (int j = 0; j < RW; ++j) {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t b = __float_as_uint(v[j][k]) & 0x7FFFFFFFu;
      top = top > b ? top : b;
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
      const uint32_t b = (uint32_t)__shfl_xor((int)top, d);
      top = top > b ? top : b;
    }
    uint32_t byte;
    float mul;
    bool nan;
    block_scale(top, &byte, &mul, &nan);
    i32x2 out = {(int)pack4(v[j][0] * mul, v[j][1] * mul, v[j][2] * mul, v[j][3] * mul), (int)pack4(v[j][4] * mul, v[j][5] * mul, v[j][6] * mul, v[j][7] * mul)};
    if (nan) out = i32x2{0x7F7F7F7F, 0x7F7F7F7F};
    if (r0 + j < n && col < ldq) *reinterpret_cast<i32x2*>(q + (int64_t)(r0 + j) * ldq + col) = out;
    if ((lane & 15) == 0) sc[lane >> 4][wave * RW + j] = (uint8_t)byte;
  }
  __syncthreads();
  for (int t = threadIdx.x; t < 16 * RW; t += kThreads) {
    const int b = t / (4 * RW), r = t % (4 * RW), row = (int)blockIdx.x * (4 * RW) + r;
    const int64_t kb = (int64_t)blockIdx.y * 4 + b;
    if (kb * 128 < ldq && row < n) s[kb * lds + row] = sc[b][r];
  }
}

// a workgroup takes a block: 16 threads a row, 16 rows at a time, held in registers between the two uses
template <typename T>
__global__ __launch_bounds__(kThreads) void fp8_blocks_kernel(const T* __restrict__ W, int64_t ldw, int64_t rows, int64_t cols, uint8_t* __restrict__ q,
                                                              int64_t ldq, uint8_t* __restrict__ s) {
  __shared__ uint32_t tops[4];
  const int64_t col = (int64_t)blockIdx.x * 128 + (threadIdx.x & 15) * 8, r0 = (int64_t)blockIdx.y * 128 + (threadIdx.x >> 4);
  float v[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[j][k] = 0.f;
    if (r0 + 16 * j < rows && col < cols) load8(W + (r0 + 16 * j) * ldw + col, v[j]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t b = __float_as_uint(v[j][k]) & 0x7FFFFFFFu;
      top = top > b ? top : b;
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t b = (uint32_t)__shfl_xor((int)top, d);
    top = top > b ? top : b;
  }
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) top = top > tops[k] ? top : tops[k];
  uint32_t byte;
  float mul;
  bool nan;
  block_scale(top, &byte, &mul, &nan);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    i32x2 out = {(int)pack4(v[j][0] * mul, v[j][1] * mul, v[j][2] * mul, v[j][3] * mul), (int)pack4(v[j][4] * mul, v[j][5] * mul, v[j][6] * mul, v[j][7] * mul)};
    if (nan) out = i32x2{0x7F7F7F7F, 0x7F7F7F7F};
    if (r0 + 16 * j < rows && col < cols) *reinterpret_cast<i32x2*>(q + (r0 + 16 * j) * ldq + col) = out;
  }
  if (threadIdx.x == 0) s[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = (uint8_t)byte;
}

template <typename T>
hipError_t rows_run(const void* X, int64_t ldx, int64_t n, int64_t K, void* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream) {
  const unsigned gy = (unsigned)((ldq + 511) / 512);
  if (n >= 2048) {
    launch_timed(fp8_rows_kernel<T, 8>, dim3((unsigned)((n + 31) / 32), gy), dim3(kThreads), 0, stream, static_cast<const T*>(X), ldx, (int)n, (int)K,
                 static_cast<uint8_t*>(q), ldq, s, lds);
  } else {
    launch_timed(fp8_rows_kernel<T, 1>, dim3((unsigned)((n + 3) / 4), gy), dim3(kThreads), 0, stream, static_cast<const T*>(X), ldx, (int)n, (int)K,
                 static_cast<uint8_t*>(q), ldq, s, lds);
  }
  return hipGetLastError();
}
template <typename T>
hipError_t blocks_run(const void* W, int64_t ldw, int64_t rows, int64_t cols, void* q, int64_t ldq, uint8_t* s, hipStream_t stream) {
  launch_timed(fp8_blocks_kernel<T>, dim3((unsigned)((cols + 127) / 128), (unsigned)((rows + 127) / 128)), dim3(kThreads), 0, stream, static_cast<const T*>(W),
               ldw, rows, cols, static_cast<uint8_t*>(q), ldq, s);
  return hipGetLastError();
}

}  // namespace

hipError_t fp8_rows_run(int dtype, const void* X, int64_t ldx, int64_t n, int64_t K, void* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream) {
  return dtype == DT_BF16 ? rows_run<__bf16>(X, ldx, n, K, q, ldq, s, lds, stream) : rows_run<_Float16>(X, ldx, n, K, q, ldq, s, lds, stream);
}

hipError_t fp8_blocks_run(int dtype, const void* W, int64_t ldw, int64_t rows, int64_t cols, void* q, int64_t ldq, uint8_t* s, hipStream_t stream) {
  if (dtype == DT_F32) return blocks_run<float>(W, ldw, rows, cols, q, ldq, s, stream);
  return dtype == DT_BF16 ? blocks_run<__bf16>(W, ldw, rows, cols, q, ldq, s, stream) : blocks_run<_Float16>(W, ldw, rows, cols, q, ldq, s, stream);
}

}  // namespace rl
