// Rows of tokens to the rows sorted by expert, and back with weights (rows.hip).  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rl {

// place [n, top]: sorted row of a token's copy j, anything outside [0, n top): none.  source [n top]: negative where no copy stands on a row.
struct RowsDesc {
  int dtype = 0;
  int64_t n = 0, d = 0;
  int top = 1;
  const int32_t *place = nullptr, *source = nullptr;
  const float* weight = nullptr;
  const void* in = nullptr;    // gather: X;  joined: rows;  spread: dY
  int64_t ldin = 0;
  const void* add = nullptr;   // joined: added to the sum, or nullptr
  int64_t ldadd = 0;
  const void* rows = nullptr;  // spread: the rows whose products with dY are wanted, or nullptr
  int64_t ldrows = 0;
  void* out = nullptr;         // spread: nullptr = not wanted
  int64_t ldout = 0;
  float* dweight = nullptr;
  bool stream = false;  // (set by the launches)
};
// a call's 64 x 16 bytes of rows are counted in 32 bits
inline bool rows_fit(int dtype, int64_t n, int64_t d) {
  const int64_t wide = dtype == 0 ? 256 : 512;  // DT_F32
  return (d + wide - 1) / wide <= ((1LL << 32) - 1) / n;
}

// out[place[t, j]] = weight[t, j] in[t] (no weight: the rows as they are), zeros on rows without a copy; dweight[t, j] = <in[t], rows[place[t, j]]>
hipError_t rows_spread(const RowsDesc& d, hipStream_t s);
// out[t] = add[t] + sum over j of weight[t, j] in[place[t, j]]
hipError_t rows_join(const RowsDesc& d, hipStream_t s);

}  // namespace rl
