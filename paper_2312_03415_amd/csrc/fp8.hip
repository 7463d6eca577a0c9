// Quantisers of the 8-bit products (see fp8.hpp).  Both are bound by memory, 2 bytes read and 1 written per 16-bit element: 8192 x 11008 bf16 in
// blocks of 128 x 128 53 us (5.1 TB/s), its rows 58 us (4.7 TB/s; a layer with an adapter rounds them in its rank products instead).
#include "fp8.hpp"

#include "gemm.hpp"
#include "gemm_engine.hpp"

namespace rl {
namespace {

constexpr int kThreads = 256;

template <typename T, int RW>
__global__ __launch_bounds__(kThreads) void fp8_rows_kernel(const T* __restrict__ X, int64_t ldx, int n, int K, uint8_t* __restrict__ q, int64_t ldq,
                                                            uint8_t* __restrict__ s, int64_t lds) {
  __shared__ uint8_t sc[4][4 * RW];
  fp8_rows_tile<T, RW>(X, ldx, n, K, q, ldq, s, lds, (int)blockIdx.x, (int)blockIdx.y, sc);
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
    if (r0 + 16 * j < rows && col < cols) fp8_load8(W + (r0 + 16 * j) * ldw + col, v[j]);
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
  fp8_block_scale(top, &byte, &mul, &nan);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    i32x2 out = {fp8_pack4(v[j][0] * mul, v[j][1] * mul, v[j][2] * mul, v[j][3] * mul), fp8_pack4(v[j][4] * mul, v[j][5] * mul, v[j][6] * mul, v[j][7] * mul)};
    if (nan) out = i32x2{0x7F7F7F7F, 0x7F7F7F7F};
    if (r0 + 16 * j < rows && col < cols) *reinterpret_cast<i32x2*>(q + (r0 + 16 * j) * ldq + col) = out;
  }
  if (threadIdx.x == 0) s[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = (uint8_t)byte;
}

// a thread takes eight columns of a row
template <typename T>
__global__ __launch_bounds__(kThreads) void fp8_values_kernel(const uint8_t* __restrict__ q, int64_t ldq, const uint8_t* __restrict__ s, int64_t lds, int64_t n,
                                                              int K, T* __restrict__ out, int64_t ldo) {
  const int pieces = K / 8;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n * pieces; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / pieces;
    const int col = (int)(i - row * pieces) * 8;
    const i32x2 b = *reinterpret_cast<const i32x2*>(q + row * ldq + col);
    const int byte = s[(int64_t)(col >> 7) * lds + row];
    T o[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(b[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(b[h], true);
      const float v[4] = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
      for (int k = 0; k < 4; ++k) o[4 * h + k] = from_f32<T>(byte == 255 ? __builtin_nanf("") : ldexpf(v[k], byte - 127));
    }
    typedef __attribute__((__vector_size__(4 * sizeof(int)))) int v4;
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) / 2; ++k) reinterpret_cast<v4*>(out + row * ldo + col)[k] = reinterpret_cast<const v4*>(o)[k];
  }
}
template <typename T>
hipError_t values_run(const void* q, int64_t ldq, const uint8_t* s, int64_t lds, int64_t n, int64_t K, void* out, int64_t ldo, hipStream_t stream) {
  int64_t groups = (n * (K / 8) + kThreads - 1) / kThreads;
  if (groups > (1 << 20)) groups = 1 << 20;
  launch_timed(fp8_values_kernel<T>, dim3((unsigned)groups), dim3(kThreads), 0, stream, static_cast<const uint8_t*>(q), ldq, s, lds, n, (int)K, static_cast<T*>(out), ldo);
  return hipGetLastError();
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

hipError_t fp8_values_run(int dtype, const void* q, int64_t ldq, const uint8_t* s, int64_t lds, int64_t n, int64_t K, void* out, int64_t ldo, hipStream_t stream) {
  if (dtype == DT_F32) return values_run<float>(q, ldq, s, lds, n, K, out, ldo, stream);
  return dtype == DT_BF16 ? values_run<__bf16>(q, ldq, s, lds, n, K, out, ldo, stream) : values_run<_Float16>(q, ldq, s, lds, n, K, out, ldo, stream);
}

hipError_t fp8_blocks_run(int dtype, const void* W, int64_t ldw, int64_t rows, int64_t cols, void* q, int64_t ldq, uint8_t* s, hipStream_t stream) {
  if (dtype == DT_F32) return blocks_run<float>(W, ldw, rows, cols, q, ldq, s, stream);
  return dtype == DT_BF16 ? blocks_run<__bf16>(W, ldw, rows, cols, q, ldq, s, stream) : blocks_run<_Float16>(W, ldw, rows, cols, q, ldq, s, stream);
}

}  // namespace rl
