// Products grouped by expert, and products with a frozen weight in 8-bit floating point: host-side interface and kernel arguments.
//
// Row t of X belongs to expert e(t): the rows of an expert are consecutive and end at ends[e] (device memory; the host does not know
// them).  With W, A, B stacks of E matrices (E = 1 and no ends: an ordinary layer)
//     Y_t = X_t W_e + bias_e + s (X_t A_e) B_e,   dX_t = dY_t W_e^T + s (dY_t B_e^T) A_e^T,
//     dA_e = s X_e^T (dY_e B_e^T),   dB_e = s (X_e A_e)^T dY_e,
// and with a W of e4m3 values (one power-of-two scale per 128 x 128 block) X and dY of the two large products are rounded to e4m3 in
// blocks of 128 columns first (fp8.hpp).  Rows behind the last expert's give zeros.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "gemm.hpp"

namespace rl {

struct GroupedArgs {
  // AL = 0: C[n, N] = A[n, K] op(B_e) by rows;  AL = 1: C_e[M, N] = A_e^T B_e over an expert's rows of A [n, M] and B [n, N]
  const void* A;
  int64_t lda;
  const void* B;
  int64_t ldb, sb;  // sb: elements from one expert's B to the next
  void* C;
  int64_t ldc, sc;
  // the adapter's product in the same accumulators: + TA[n, R] TB_e[N, R]^T (R = 0: none)
  const void* TA;
  const void* TB;
  int64_t ldta, ldtb, stb;
  const void* bias;  // [E, N] or nullptr
  // e4m3 operands: scale bytes of A [ceil(K / 128)][ldsa] (row index fastest) and of W [ib, ob], ssb bytes from one expert's to the next
  const uint8_t* SA;
  int64_t ldsa;
  const uint8_t* SB;
  int64_t ssb;
  int scols;  // ob
  float* partial;  // not nullptr: fp32 slices [split][rows][N] instead of C
  const int32_t* ends;
  int experts;
  int n, M, N, K, R;
  int splits, tiles_per_split;
  int band;  // row tiles per band in which the output tiles are walked
  float alpha;  // C = alpha (A B) + TA TB + bias
  // builds that round A on the way (AL = 0, 16-bit): e4m3 bytes [n][ldq], zeros behind K, and scale bytes [ldq / 128][ldqs]
  uint8_t *Q, *QS;
  int64_t ldq, ldqs;
};

// what a launch runs on (T: a rank-r product's)
enum GroupedTile { GT_32x128 = 0, GT_64x128, GT_128x128, GT_64x32, GT_64x64, GT_64x128T, GT_256x256, GT_COUNT };
struct GroupedTileInfo { int bm, bn; };
inline GroupedTileInfo grouped_tile(int t) {
  static const GroupedTileInfo k[GT_COUNT] = {{32, 128}, {64, 128}, {128, 128}, {64, 32}, {64, 64}, {64, 128}, {256, 256}};
  return k[t];
}

// largest number of row tiles that n rows of up to `experts` groups (and the rest behind them) can make; one group without ends: all rows
inline int64_t grouped_row_tiles(int64_t n, int64_t experts, bool ends, int bm, bool f8) {
  if (!ends) return (n + bm - 1) / bm;
  const int64_t groups = (experts + 1 < n ? experts + 1 : n);
  return (n + groups * (bm - 1 + (f8 ? 3 : 0))) / bm;  // (an e4m3 group's first tile starts up to three rows early)
}

// The last round of 256 x 256 tiles, one per compute unit, where it is at most half full, has its tiles' K tiles dealt out to `splits` workgroups
// each, which leave fp32 sums for grouped_mc_join_kernel: (1 - 1 / splits) of a round of nt K tiles of 1.5 us for a round trip of up to
// 64 MB and a launch, together about 40 us; worth it from 60 us saved.  8192 rows of 8 experts, K = 8192 (about 288 tiles), bf16: 257 + 12 us in
// place of 384; 16384 x 11008 -> 4096 e4m3: 735 + 14 in place of 807; where it would save 48 us (K = 4096, bf16) it gains nothing.
struct GroupedSplit {
  int whole, splits, per;  // tiles [0, whole) by themselves; the others' K tiles in `splits` runs of `per`
};
__host__ __device__ inline GroupedSplit grouped_split_round(int total, int nt) {
  const int left = total & 255;
  GroupedSplit s{total, 1, nt};
  if (left == 0 || left > 128) return s;
  int k = 256 / left;
  if (k > 8) k = 8;
  s.per = (nt + k - 1) / k;
  s.splits = (nt + s.per - 1) / s.per;
  if ((nt - s.per) * 3 < 120 || s.per < 4) return GroupedSplit{total, 1, nt};
  s.whole = total - left;
  return s;
}

// rows: A is rounded on the way (GroupedArgs::Q)
hipError_t grouped_rows_launch_bf16(int bl, int tile, const GroupedArgs& a, dim3 grid, hipStream_t s);
hipError_t grouped_rows_launch_f16(int bl, int tile, const GroupedArgs& a, dim3 grid, hipStream_t s);
hipError_t grouped_launch_bf16(bool f8, int bl, int tile, const GroupedArgs& a, dim3 grid, hipStream_t s);
hipError_t grouped_launch_f16(bool f8, int bl, int tile, const GroupedArgs& a, dim3 grid, hipStream_t s);
// tiles of 128 x width of dA and width x 128 of dB: ax and bx of them, in their splits (0: not wanted)
hipError_t grouped_grads_launch_bf16(int width, const GroupedArgs& ga, int ax, const GroupedArgs& gb, int bx, hipStream_t s);
hipError_t grouped_grads_launch_f16(int width, const GroupedArgs& ga, int ax, const GroupedArgs& gb, int bx, hipStream_t s);

// one layer call (experts = 1, ends = nullptr: an ordinary layer)
struct ExpertsDesc {
  int dtype = DT_BF16;
  bool f8 = false;
  int64_t n = 0, experts = 1, i = 0, o = 0, r = 0;
  const int32_t* ends = nullptr;
  bool has_ends = true;  // false: one expert, all rows its (sizes are asked for without ends)
  const void *W = nullptr, *A = nullptr, *B = nullptr, *bias = nullptr;
  int64_t ldw = 0, sw = 0, lda = 0, sa = 0, ldb = 0, sb = 0;
  const uint8_t* w_scales = nullptr;
  int64_t s_scales = 0;
  const void* X = nullptr;   // forward's input; the backward's too
  int64_t ldx = 0;
  const void* dY = nullptr;
  int64_t lddy = 0;
  void *Y = nullptr, *T = nullptr, *dX = nullptr, *dA = nullptr, *dB = nullptr;
  int64_t ldy = 0, ldt = 0, lddx = 0, ldda = 0, sda = 0, lddb = 0, sdb = 0;
  bool has_T = false;  // backward: T holds s X A already
  uint8_t *q = nullptr, *qs = nullptr;  // forward over an e4m3 W: X rounded already (fp8_row_bytes, fp8_scale_ld), or nullptr
  float scale = 1.f;
};
// what a large product of K into N columns runs on: a function of sizes alone, shared by the workspace query and the call.  slices: K in `splits`
// slices that a launch of its own sums (few rows); join: 256 x 256 tiles whose last round may be split
struct GroupedPlan { int tile, splits, per; unsigned gx; bool join; };
GroupedPlan grouped_plan(const ExpertsDesc& d, int64_t N, int64_t K, bool slices);
size_t experts_workspace(const ExpertsDesc& d, bool backward);
hipError_t experts_forward(const ExpertsDesc& d, void* workspace, hipStream_t stream);
hipError_t experts_backward(const ExpertsDesc& d, void* workspace, hipStream_t stream);

}  // namespace rl
