// e4m3 values with power-of-two block scales: the quantisers (fp8.hip).  Internal to the library.
//
// A block's scale is 2^e, e the smallest integer >= -127 with amax <= 448 * 2^e (448: the largest e4m3 value), stored as the byte
// e + 127; its values are x 2^-e rounded to the nearest e4m3 value, ties to even (the product with a power of two is exact).  An
// all-zero block has scale 1 and zeros; a block that holds an infinity or a NaN has scale 1 and NaNs throughout.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rl {

// rows of X [n, K] in blocks of 128 columns: q [n][ldq] (ldq = K rounded up to 128, zeros behind K), s [ldq / 128][lds]
hipError_t fp8_rows_run(int dtype, const void* X, int64_t ldx, int64_t n, int64_t K, void* q, int64_t ldq, uint8_t* s, int64_t lds, hipStream_t stream);
// W [rows, cols] in blocks of 128 x 128: q [rows][ldq], s [ceil(rows / 128)][ceil(cols / 128)]
hipError_t fp8_blocks_run(int dtype, const void* W, int64_t ldw, int64_t rows, int64_t cols, void* q, int64_t ldq, uint8_t* s, hipStream_t stream);

inline int64_t fp8_row_bytes(int64_t K) { return (K + 127) / 128 * 128; }
inline int64_t fp8_scale_ld(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace rl
