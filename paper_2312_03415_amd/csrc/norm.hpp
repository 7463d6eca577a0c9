// Root-mean-square norm with the residual's addition, and rows of its output in e4m3 (norm.hip).  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rl {

struct NormDesc {
  int dtype = 0;
  int64_t n = 0, d = 0;
  float eps = 0.f;
  const void *X = nullptr, *R = nullptr, *gain = nullptr;  // forward: h = X (+ R);  backward: X is h
  int64_t ldx = 0, ldr = 0;
  void *Y = nullptr, *H = nullptr;  // H: where h goes, or nullptr
  int64_t ldy = 0, ldh = 0;
  float* rstd = nullptr;  // forward: written unless nullptr;  backward: read
  uint8_t *q = nullptr, *qs = nullptr;  // Y's rows in e4m3, [n][ldq], and their scale bytes [ldq / 128][ldqs], or nullptr
  int64_t ldq = 0, ldqs = 0;
  const void *dY = nullptr, *dH = nullptr;
  int64_t lddy = 0, lddh = 0;
  void *dX = nullptr, *dgain = nullptr;
  int64_t lddx = 0;
  bool stream = false;  // (set by the launches)
};
constexpr int64_t kNormMaxWidth = 32768;  // a row is held in registers

hipError_t norm_forward(const NormDesc& d, hipStream_t s);
size_t norm_backward_workspace(int dtype, int64_t n, int64_t d, bool dgain);
hipError_t norm_backward(const NormDesc& d, void* workspace, hipStream_t s);

}  // namespace rl
