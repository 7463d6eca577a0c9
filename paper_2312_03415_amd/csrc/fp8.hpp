// e4m3 values with power-of-two block scales: the quantisers (fp8.hip).  Internal to the library.
//
// A block's scale is 2^e, e the smallest integer >= -127 with amax <= 448 * 2^e (448: the largest e4m3 value), stored as the byte
// e + 127; its values are x 2^-e rounded to the nearest e4m3 value, ties to even (the product with a power of two is exact).  An
// all-zero block has scale 1 and zeros; a block that holds an infinity or a NaN has scale 1 and NaNs throughout.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rl {

#if defined(__HIPCC__)
// from the largest |bits| of a block: scale byte and multiplier 2^-e; not finite: multiplier 0 and byte 127, and *nan set
__device__ __forceinline__ void fp8_block_scale(uint32_t top, uint32_t* byte, float* mul, bool* nan) {
  *nan = top >= 0x7F800000u;
  int e = 0;
  if (top != 0u && !*nan) {
    // top = m 2^E, 1/2 <= m < 1 (denormals too: frexp); 448 = 0.875 * 2^9
    int E;
    const float m = frexpf(__uint_as_float(top), &E);
    e = m > 0.875f ? E - 8 : E - 9;
    if (e < -127) e = -127;
  }
  *byte = (uint32_t)(e + 127);
  *mul = *nan ? 0.f : ldexpf(1.f, -e);
}
__device__ __forceinline__ int fp8_pack4(float a, float b, float c, float d) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
// eight consecutive elements
template <typename T>
__device__ __forceinline__ void fp8_load8(const T* p, float (&v)[8]) {
  typedef __attribute__((__vector_size__(4 * sizeof(int)))) int v4;
#pragma unroll
  for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
    const v4 a = reinterpret_cast<const v4*>(p)[q];
    const T* const t = reinterpret_cast<const T*>(&a);
#pragma unroll
    for (int k = 0; k < 16 / (int)sizeof(T); ++k) v[q * (16 / (int)sizeof(T)) + k] = (float)t[k];
  }
}

// Rows of X [n, K] in blocks of 128 columns, a workgroup of 256 threads: a wave takes a row's 512 columns at a time, 8 per lane, so that 16
// lanes hold a block; the workgroup 4 RW rows (tile bx of them, columns 512 by ..).  Their scale bytes go through LDS (`sc`), so that they
// leave as runs of consecutive bytes.
template <typename T, int RW>
__device__ __forceinline__ void fp8_rows_tile(const T* __restrict__ X, int64_t ldx, int n, int K, uint8_t* __restrict__ q, int64_t ldq, uint8_t* __restrict__ s,
                                              int64_t lds, int bx, int by, uint8_t (&sc)[4][4 * RW]) {
  typedef __attribute__((__vector_size__(2 * sizeof(int)))) int v2;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = by * 512 + lane * 8, r0 = bx * (4 * RW) + wave * RW;
  float v[RW][8];
#pragma unroll
  for (int j = 0; j < RW; ++j) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[j][k] = 0.f;
    if (r0 + j < n && col < K) fp8_load8(X + (int64_t)(r0 + j) * ldx + col, v[j]);
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
    fp8_block_scale(top, &byte, &mul, &nan);
    v2 out = {fp8_pack4(v[j][0] * mul, v[j][1] * mul, v[j][2] * mul, v[j][3] * mul), fp8_pack4(v[j][4] * mul, v[j][5] * mul, v[j][6] * mul, v[j][7] * mul)};
    if (nan) out = v2{0x7F7F7F7F, 0x7F7F7F7F};
    if (r0 + j < n && col < ldq) *reinterpret_cast<v2*>(q + (int64_t)(r0 + j) * ldq + col) = out;
    if ((lane & 15) == 0) sc[lane >> 4][wave * RW + j] = (uint8_t)byte;
  }
  __syncthreads();
  for (int t = threadIdx.x; t < 16 * RW; t += 256) {
    const int b = t / (4 * RW), r = t % (4 * RW), row = bx * (4 * RW) + r;
    const int64_t kb = (int64_t)by * 4 + b;
    if (kb * 128 < ldq && row < n) s[kb * lds + row] = sc[b][r];
  }
}
#endif

// rows of X [n, K] in blocks of 128 columns: q [n][ldq] (ldq = K rounded up to 128, zeros behind K), s [ldq / 128][lds]
hipError_t fp8_rows_run(int dtype, const void* X, int64_t ldx, int64_t n, int64_t K, void* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream);
// W [rows, cols] in blocks of 128 x 128: q [rows][ldq], s [ceil(rows / 128)][ceil(cols / 128)]
hipError_t fp8_blocks_run(int dtype, const void* W, int64_t ldw, int64_t rows, int64_t cols, void* q, int64_t ldq, uint8_t* s, hipStream_t stream);

inline int64_t fp8_row_bytes(int64_t K) { return (K + 127) / 128 * 128; }
inline int64_t fp8_scale_ld(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace rl
