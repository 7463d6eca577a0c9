// Matrix-core kernel of the large grouped and 8-bit products (grouped.hpp): 256 x 256 tiles, one persistent workgroup per compute unit.
//
// What bounds it: the matrix cores, as gemm_mc64.hpp (whose tile, load stream and LDS layouts it takes over): 4 wavefronts with a
// 128 x 128 sub-tile each, 8 x 8 accumulator blocks of 16 x 16 in the 256 accumulation registers, two LDS stages of 64 KB filled by
// LDS-DMA, the load stream running on across output tiles.  What differs:
//  - A K tile is 128 bytes of a row whatever the type: 64 16-bit values or 128 e4m3 values, one scale block.  Both take the matrix
//    cores 32 cycles per block pair (two v_mfma_f32_16x16x32, or one v_mfma_scale_f32_16x16x128_f8f6f4), so that one schedule serves
//    both.  It is cut by columns, not by k: step 0 multiplies B blocks 0..3 and fetches 4..7, step 1 multiplies 4..7 behind the wait
//    and the barrier for the next tile, and fetches the next tile's blocks 0..3 and A blocks 0..5 into registers that are free by
//    then (an A block is dead behind its last product).  128 registers of fragments, none twice.
//  - No LDS read is in flight where the code branches (the end of a K tile): the compiler may copy registers there.
//  - Output tiles are those of the experts' rows; tile counts stay in registers, one expert a lane, so that finding the next tile is
//    a ballot.  Rows and columns outside the operands are fetched from past the buffers' ends, which gives zeros.
//  - The adapter's product is one more run of K tiles in the same stream (T and the other factor, both with the rank in their rows).
//    With its fragments straight from memory behind the K loop, as grouped_mt.hpp has it, an output tile of r = 128 took 20 us more.
// Rates of 8192 x 8192 -> 8192 without adapters: bf16 1.46 (Y) and 1.48 (dX) PFLOP/s, e4m3 2.50 and 2.55 with the rounding of the rows; a library
// product reaches 1.21 / 1.36 and 2.69 on this card.
#pragma once
#include "grouped_mt.hpp"

namespace rl {

#define RL_INLINE __attribute__((always_inline))  // lambdas that hold register arrays by reference

// acc += (rows of W) * (rows of X) with W's scale byte sw (byte 0) and X's scale byte BYTE of sx
template <int BYTE>
__device__ __forceinline__ void mma_f8(f32x4& acc, i32x8 w, i32x8 x, int sw, int sx) {
  if constexpr (BYTE == 0) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(w), "v"(x), "v"(sw), "v"(sx));
  if constexpr (BYTE == 1) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,1,0] op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(w), "v"(x), "v"(sw), "v"(sx));
  if constexpr (BYTE == 2) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,1,0]" : "+a"(acc) : "v"(w), "v"(x), "v"(sw), "v"(sx));
  if constexpr (BYTE == 3) asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,1,0] op_sel_hi:[0,1,0]" : "+a"(acc) : "v"(w), "v"(x), "v"(sw), "v"(sx));
}

// a fragment of 32 bytes: its halves as the LDS reads deliver them, put together behind the wait only
template <bool F8, bool STRIDED> struct McFrag;
template <> struct McFrag<true, false> {
  i32x4 h0, h1;
  __device__ __forceinline__ void touch() { asm volatile("" : "+v"(h0), "+v"(h1)); }
};
template <> struct McFrag<false, false> : McFrag<true, false> {};
template <bool F8> struct McFrag<F8, true> {
  i32x2 q[4];
  __device__ __forceinline__ void touch() { asm volatile("" : "+v"(q[0]), "+v"(q[1]), "+v"(q[2]), "+v"(q[3])); }
};

struct GroupedMcShape {
  static constexpr int BM = 256, BN = 256, A_BYTES = 32768, STAGE_BYTES = 65536, NS = 2;
  static constexpr int SCALES = NS * STAGE_BYTES;            // [stage][wave] 256 scale bytes of the tile's rows
  static constexpr int STAGING = SCALES + NS * 1024;         // epilogue: 4 KB per wave
  static constexpr int LDS_BYTES = STAGING + 4 * 4096;
  static constexpr int kMaxScaleTiles = 128;                 // K tiles whose scales of W two registers hold
};

// Where the output tiles are: the groups' row tiles times nbn, walked in bands of 8 row tiles, a contiguous run per XCD (gemm_mc64.hpp).
// The tile counts of up to 64 experts stay in registers.
template <bool F8>
struct GroupedOrder {
  GroupScan<256, F8> groups;
  int nbm, nbn, total;
  __device__ __forceinline__ void open(const GroupedArgs& g, int lane) {
    nbn = (g.N + 255) >> 8;
    groups.open(g.ends, g.experts, g.n, lane);
    nbm = groups.total;
    total = nbm * nbn;
  }
  template <typename Args>  // (in any address space)
  __device__ __forceinline__ GroupTile at(const Args& g, int lane, int seq, int& n0) const {
    const int x = seq & 7, slot = seq >> 3, q = total >> 3, rem = total & 7;
    const int id = x * q + (x < rem ? x : rem) + slot;
    constexpr int BAND = 8;
    const int per_band = BAND * nbn, band = id / per_band, first_m = band * BAND;
    const int band_rows = (nbm - first_m) < BAND ? (nbm - first_m) : BAND, in_band = id - band * per_band;
    GroupTile out = groups.find(g.ends, g.experts, g.n, lane, first_m + in_band % band_rows);
    // (said to the compiler: with a descriptor that it takes for a lane's own, every load becomes a loop over the lanes)
    out.e = __builtin_amdgcn_readfirstlane(out.e);
    out.lo = __builtin_amdgcn_readfirstlane(out.lo);
    out.hi = __builtin_amdgcn_readfirstlane(out.hi);
    out.m0 = __builtin_amdgcn_readfirstlane(out.m0);
    n0 = __builtin_amdgcn_readfirstlane((in_band / band_rows) * 256);
    return out;
  }
};

// With experts the tile count is the device's to know: the product and the join decide here, where the host has left room for a split.
__device__ __forceinline__ GroupedSplit grouped_split(const GroupedArgs& g, int total, int nt) {
  return g.partial == nullptr ? GroupedSplit{total, 1, nt} : grouped_split_round(total, nt);
}

template <typename T, bool F8, int BL>
__global__ __launch_bounds__(256, 1) void grouped_mc_kernel(GroupedArgs args) {
  // The arguments are read from the kernel's argument segment where they are used: kept in scalar registers across the K loop, they push the
  // loop's own state out of them (17 v_readlane a K tile to fetch it back, e4m3 8 % slower).
  typedef const __attribute__((address_space(4))) GroupedArgs* ArgPtr;
  auto fresh = []() RL_INLINE -> ArgPtr {
#if defined(__HIP_DEVICE_COMPILE__)
    ArgPtr p = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
#else
    return nullptr;
#endif
  };
  using P = GroupedMcShape;
  constexpr int EB = F8 ? 1 : 2, KE = 128 / EB, IPW = 8;
  constexpr bool B_STR = BL == 0;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  unsigned char* const smem = smem_raw;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int s16 = lane & 15, grp = lane >> 4;
  const GroupedArgs& g0 = args;
  const int nt = (g0.K + KE - 1) / KE;
  GroupedOrder<F8> order;
  order.open(g0, lane);
  const GroupedSplit split = grouped_split(g0, order.total, nt);
  const int nwork = split.whole + (order.total - split.whole) * split.splits;
  // work item w: an output tile and its K tiles [u0, u1); the adapter's follow the last of them
  auto item = [&](int w, int& n0, int& u0, int& u1) RL_INLINE -> GroupTile {
    const bool part = w >= split.whole;
    const int j = part ? w - split.whole : 0, tile = j / split.splits, run = j - tile * split.splits;
    u0 = run * split.per;
    u1 = part && u0 + split.per < nt ? u0 + split.per : nt;
    return order.at(*fresh(), lane, part ? split.whole + tile : w, n0);
  };

  // ---- load cursor: the K tile of the output tile that is fetched next.  An output tile's K tiles are the nt of the large product and then
  // the ntail of the adapter's (64 of the rank each, 16-bit, both factors with the rank in their rows).
  constexpr uint32_t OOB = 0x80000000u, kBias = 3 * 1024;  // (four loads share an LDS base and differ in the immediate offset, see gemm_mc64.hpp)
  uint32_t offA[IPW], offB[IPW];
  const unsigned char *pA = nullptr, *pB = nullptr, *pS = nullptr;
  int64_t leftA = 0, leftB = 0, stepB = 0;
  const int ntail = (g0.R + 63) >> 6, experts = g0.experts;
  int cw = blockIdx.x, cu = 0, cnext = 0, cend = 0, leftS = 0, ce = 0, cm0 = 0, cn0 = 0;  // cnext: the K tile at which something changes
  const int64_t ldsa = F8 ? g0.ldsa : 0;
  bool clive = true, in_tail = false;
  const int kpart = g0.K - g0.K / KE * KE, rpart = g0.R & 63;  // what the last K tile of each kind holds, 0: all of it
  // (what follows from the lane alone is not worth registers across the K loop)
  auto opaque_lane = [&]() RL_INLINE {
    int ln = lane;
    asm volatile("" : "+v"(ln));
    return ln;
  };
  auto k_contiguous = [&](uint32_t (&off)[IPW], bool dealt, int rows, int ld, int eb) RL_INLINE {
    const int ln = opaque_lane();
#pragma unroll
    for (int j = 0; j < IPW; ++j) {
      const int p = (wave * IPW + j) * 64 + ln;
      int row = p >> 3;
      const int byte = ((p & 7) ^ ((row >> 1) & 7)) * 16;
      if (dealt) row = (row & 128) + (row & 15) * 8 + ((row & 127) >> 4);  // the wave's rows are dealt out to its blocks
      off[j] = row < rows ? (uint32_t)(row * ld * eb + byte) + (kBias - 1024u * (j & 3)) : OOB;
    }
  };
  auto cut = [&](uint32_t (&off)[IPW], int bytes) RL_INLINE {  // chunks that lie `bytes` or more into the row of a K tile read zeros
    const int ln = opaque_lane();
#pragma unroll
    for (int j = 0; j < IPW; ++j) {
      const int p = (wave * IPW + j) * 64 + ln;
      if (((p & 7) ^ ((p >> 4) & 7)) * 16 >= bytes) off[j] |= OOB;
    }
  };
  auto cursor_main = [&]() RL_INLINE -> int {  // the first K tile of work item cw, or of the next that has any; none left: loads of nothing
    GroupTile t{};
    int u0 = 0, u1 = nt;
    for (;; cw += gridDim.x) {
      if (cw >= nwork) { clive = false; break; }
      t = item(cw, cn0, u0, u1);
      if (t.e < experts) break;
    }
    cend = u1;
    if (!clive) {
      leftA = leftB = 0;
      return u0;
    }
    const ArgPtr ga = fresh();
    ce = t.e;
    cm0 = t.m0;
    const int rows = ga->n - cm0;
    pA = static_cast<const unsigned char*>(ga->A) + (int64_t)cm0 * ga->lda * EB;
    leftA = ((int64_t)(rows - 1) * ga->lda + (F8 ? (int64_t)((ga->K + 127) / 128) * 128 : ga->K)) * EB;
    k_contiguous(offA, F8, rows, (int)ga->lda, EB);
    const unsigned char* const Be = static_cast<const unsigned char*>(ga->B) + (int64_t)ce * ga->sb * EB;
    if constexpr (!B_STR) {
      pB = Be + (int64_t)cn0 * ga->ldb * EB;
      leftB = ((int64_t)(ga->N - cn0 - 1) * ga->ldb + ga->K) * EB;
      stepB = 128;
      k_contiguous(offB, false, ga->N - cn0, (int)ga->ldb, EB);
    } else {
      pB = Be + (int64_t)cn0 * EB;
      leftB = ((int64_t)(ga->K - 1) * ga->ldb + ga->N - cn0) * EB;
      stepB = (int64_t)KE * ga->ldb * EB;
      const int ln = opaque_lane();
#pragma unroll
      for (int j = 0; j < IPW; ++j) {
        const int p = (wave * IPW + j) * 64 + ln, row = F8 ? p >> 4 : p >> 5;
        const int col = F8 ? ((p & 15) ^ grouped_swz<true, 256>(row)) * 16 : ((p & 31) ^ (4 * (row & 3))) * 8;
        offB[j] = cn0 + col < ga->N ? (uint32_t)((row * (int)ga->ldb + col) * EB) + (kBias - 1024u * (j & 3)) : OOB;
      }
    }
    if constexpr (F8) {
      pS = ga->SA + cm0;
      leftS = (int)(ga->ldsa - cm0);
      pS += u0 * ga->ldsa;
    }
    pA += u0 * 128; leftA -= u0 * 128;
    pB += u0 * stepB; leftB -= u0 * stepB;
    in_tail = false;
    return u0;
  };
  auto cursor_tail = [&]() RL_INLINE {  // the first K tile of the adapter's product
    const ArgPtr ga = fresh();
    const int rows = ga->n - cm0;
    pA = static_cast<const unsigned char*>(ga->TA) + (int64_t)cm0 * ga->ldta * 2;
    leftA = ((int64_t)(rows - 1) * ga->ldta + ga->R) * 2;
    k_contiguous(offA, F8, rows, (int)ga->ldta, 2);
    pB = static_cast<const unsigned char*>(ga->TB) + (ce * ga->stb + (int64_t)cn0 * ga->ldtb) * 2;
    leftB = ((int64_t)(ga->N - cn0 - 1) * ga->ldtb + ga->R) * 2;
    stepB = 128;
    k_contiguous(offB, false, ga->N - cn0, (int)ga->ldtb, 2);
    in_tail = true;
  };
  auto cut_main = [&]() RL_INLINE {  // the large product's partial K tile
    if constexpr (!F8) cut(offA, kpart * EB);  // (rows of a rounded A are whole scale blocks, zeros behind K)
    if constexpr (!B_STR) cut(offB, kpart * EB);
  };
  auto cut_tail = [&]() RL_INLINE {
    cut(offA, rpart * 2);
    cut(offB, rpart * 2);
  };
  // The cursor has reached cnext, and it lies ahead of the cursor again afterwards, or nothing is left.  (What several branches would assign
  // is assigned behind them: the compiler folds their stores into one through a choice of addresses, and the variables stay in memory.)
  auto cursor_event = [&]() RL_INLINE {
    int at = cu, next = cend;
    if (cu < cend) {
      cut_main();
    } else if (!in_tail && ntail > 0 && cend == nt) {
      cursor_tail();
      next = nt + ntail - (rpart != 0);
      if (next == at) {
        cut_tail();
        next = nt + ntail;
      }
    } else if (in_tail && cu < nt + ntail) {
      cut_tail();
      next = nt + ntail;
    } else {
      cw += gridDim.x;
      at = cursor_main();
      next = cend - (kpart != 0 && cend == nt);
      if (next == at) {
        if (clive) cut_main();
        next = cend;
      }
    }
    cu = at;
    cnext = next;
  };
  auto rsrc = [&](const unsigned char* base, int64_t left) RL_INLINE {
    const int size = left <= 0 ? 0 : (left > 0x7fff0000 ? 0x7fff0000 : (int)left) + (int)kBias;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base) - kBias, 0, size, 0x00020000);
  };
  __amdgpu_buffer_rsrc_t rsA, rsB;
  auto cursor_point = [&]() RL_INLINE { rsA = rsrc(pA, leftA); rsB = rsrc(pB, leftB); };
  cu = cursor_main();
  cnext = cend - (kpart != 0 && cend == nt);
  if (clive && cnext == cu) {
    cut_main();
    cnext = cend;
  }
  cursor_point();
  // load j of the cursor's K tile into stage `st`: 0..7 the A half, 8..15 the B half, 16 the scales of A
  auto issue_load = [&](int st, auto j_c) RL_INLINE {
    constexpr int j = decltype(j_c)::value;
    if constexpr (j < 16) {
      constexpr bool isB = j >= IPW;
      constexpr int jj = j & (IPW - 1);
      unsigned char* const dst = smem + st * P::STAGE_BYTES + (isB ? P::A_BYTES : 0) + wave * (IPW * 1024) + (jj >> 2) * 4096;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(isB ? rsB : rsA, (mc_lds_void_t*)dst, 16, isB ? offB[jj] : offA[jj], 0, (jj & 3) * 1024, 0);
    } else if constexpr (F8) {
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(pS), 0, clive && !in_tail ? leftS : 0, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (mc_lds_void_t*)(smem + P::SCALES + st * 1024 + wave * 256), 4, 4 * lane, 0, 0, 0);
    }
  };
  // on to the next K tile: the plain step, without a branch (among the products), and what is rare (behind them)
  auto cursor_step = [&]() RL_INLINE {
    ++cu;
    pA += 128; leftA -= 128;
    pB += stepB; leftB -= stepB;
    if constexpr (F8) pS += ldsa;
    cursor_point();
  };
  // ---- fragment addresses inside a stage (half h of a fragment: k 32 h + 8 grp .. + 7, or 64 h + 16 grp .. + 15 for e4m3)
  uint32_t fragA[2], fragB[B_STR ? 8 : 2];
  {
    const int sw = (s16 >> 1) & 7;
#pragma unroll
    for (int h = 0; h < 2; ++h) fragA[h] = (uint32_t)((wm * 128 + s16) * 128 + (((4 * h + grp) ^ sw) << 4));
    if constexpr (!B_STR) {
#pragma unroll
      for (int h = 0; h < 2; ++h) fragB[h] = (uint32_t)(P::A_BYTES + (wn * 128 + s16) * 128 + (((4 * h + grp) ^ sw) << 4));
    } else {
      const int kr = F8 ? 16 * grp + (s16 >> 1) : 8 * grp + (s16 >> 2);
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const int chunk = F8 ? (wn * 8 + b) ^ grouped_swz<true, 256>(kr) : (wn * 16 + 2 * b + ((s16 & 3) >> 1)) ^ (4 * (kr & 3));
        fragB[b] = (uint32_t)(P::A_BYTES + kr * (256 * EB) + chunk * 16 + 8 * (s16 & 1));
      }
    }
  }
  const uint32_t lds_base = (uint32_t)(uintptr_t)((mc_lds_void_t*)smem);
  McFrag<F8, false> fa[8];
  McFrag<F8, B_STR> fb[8];
  i32x2 sa = {0, 0}, san = {0, 0};  // scale bytes of the lane's row of every block: this K tile's, the next's
  auto read_A = [&](auto a_c, uint32_t soff) RL_INLINE {
    constexpr int a = decltype(a_c)::value;
    auto& f = fa[a];
    const uint32_t at0 = lds_base + soff + fragA[0], at1 = lds_base + soff + fragA[1];
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f.h0) : "v"(at0), "i"(a * 2048));
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f.h1) : "v"(at1), "i"(a * 2048));
  };
  auto read_B = [&](auto tail_c, auto b_c, uint32_t soff) RL_INLINE {  // TAIL: a K-contiguous 16-bit tile whatever W's layout
    constexpr int b = decltype(b_c)::value;
    constexpr bool TAIL = decltype(tail_c)::value;
    auto& f = fb[b];
    const uint32_t base = lds_base + soff;
    const auto& fr = fragB;
    [[maybe_unused]] const uint32_t fragT = (uint32_t)(P::A_BYTES + (wn - wm) * 16384);  // the same lanes' rows of the B half
    if constexpr (!B_STR) {
      const uint32_t at0 = base + fr[0], at1 = base + fr[1];
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f.h0) : "v"(at0), "i"(b * 2048));
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f.h1) : "v"(at1), "i"(b * 2048));
    } else if constexpr (TAIL) {
      const uint32_t at0 = base + fragA[0] + fragT, at1 = base + fragA[1] + fragT;
      asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(f.q[0]) : "v"(at0), "i"(b * 2048));
      asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(f.q[1]) : "v"(at0), "i"(b * 2048 + 8));
      asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(f.q[2]) : "v"(at1), "i"(b * 2048));
      asm volatile("ds_read_b64 %0, %1 offset:%2" : "=v"(f.q[3]) : "v"(at1), "i"(b * 2048 + 8));
    } else {
      const uint32_t at = base + fr[b];
      if constexpr (F8) {
        asm volatile("ds_read_b64_tr_b8 %0, %1" : "=v"(f.q[0]) : "v"(at));
        asm volatile("ds_read_b64_tr_b8 %0, %1 offset:2048" : "=v"(f.q[1]) : "v"(at));
        asm volatile("ds_read_b64_tr_b8 %0, %1 offset:16384" : "=v"(f.q[2]) : "v"(at));
        asm volatile("ds_read_b64_tr_b8 %0, %1 offset:18432" : "=v"(f.q[3]) : "v"(at));
      } else {
        asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(f.q[0]) : "v"(at));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:2048" : "=v"(f.q[1]) : "v"(at));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:16384" : "=v"(f.q[2]) : "v"(at));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:18432" : "=v"(f.q[3]) : "v"(at));
      }
    }
  };
  auto read_scales = [&](int st) RL_INLINE {
    if constexpr (F8) asm volatile("ds_read_b64 %0, %1" : "=v"(san) : "v"(lds_base + (uint32_t)(P::SCALES + st * 1024 + wave * 256 + wm * 128 + s16 * 8)));
  };
  auto half = [&](const auto& f, auto h_c) RL_INLINE -> i32x4 {
    constexpr int h = decltype(h_c)::value;
    if constexpr (std::is_same_v<std::decay_t<decltype(f)>, McFrag<F8, true>>) return i32x4{f.q[2 * h][0], f.q[2 * h][1], f.q[2 * h + 1][0], f.q[2 * h + 1][1]};
    else return h == 0 ? f.h0 : f.h1;
  };
  using H0 = std::integral_constant<int, 0>;
  using H1 = std::integral_constant<int, 1>;

  f32x4 acc[8][8];  // lane l: row l % 16 of block a, columns 4 (l / 16) .. + 3 of block b
  int wsc = 0;      // scale byte of W, this K tile
#define MC_FENCE() __builtin_amdgcn_sched_barrier(0)
  // products of A block a with B blocks B0 .. B0 + 3; slot(j) is called behind each quarter of them
  auto row_products = [&](auto tail_c, auto a_c, auto b0_c, auto slot) RL_INLINE {
    constexpr int a = decltype(a_c)::value, B0 = decltype(b0_c)::value;
    constexpr bool TAIL = decltype(tail_c)::value;
    static_for<4>([&](auto j_c) RL_INLINE {
      constexpr int j = decltype(j_c)::value;
      if constexpr (F8 && !TAIL) {
        mma_f8<a & 3>(acc[a][B0 + j], __builtin_shufflevector(half(fb[B0 + j], H0{}), half(fb[B0 + j], H1{}), 0, 1, 2, 3, 4, 5, 6, 7),
                      __builtin_shufflevector(fa[a].h0, fa[a].h1, 0, 1, 2, 3, 4, 5, 6, 7), wsc, sa[a >> 2]);
      } else {
        constexpr int h = j >> 1, b = B0 + 2 * (j & 1);
        Elem16<T>::mma(acc[a][b], half(fb[b], std::integral_constant<int, h>{}), half(fa[a], std::integral_constant<int, h>{}));
        MC_FENCE();
        Elem16<T>::mma(acc[a][b + 1], half(fb[b + 1], std::integral_constant<int, h>{}), half(fa[a], std::integral_constant<int, h>{}));
      }
      MC_FENCE();
      slot(j_c);
      MC_FENCE();
    });
  };

  // ---- prologue: both stages on their way, the first tile landed for everyone, its first fragments in registers
  constexpr int LPT = F8 ? 17 : 16;
#pragma unroll 1
  for (int s = 0; s < 2; ++s) {
    static_for<LPT>([&](auto j) RL_INLINE { issue_load(s, j); });
    cursor_step();
    if (clive && cu >= cnext) {
      cursor_event();
      cursor_point();
    }
  }
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(mc_wait_imm(0, true));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  MC_FENCE();
  static_for<4>([&](auto b) RL_INLINE { read_B(std::false_type{}, b, 0u); });
  static_for<6>([&](auto a) RL_INLINE { read_A(a, 0u); });
  read_scales(0);
  auto wait_next = [&]() RL_INLINE {  // the fragments fetched across the end of a K tile
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    static_for<4>([&](auto b) RL_INLINE { fb[b].touch(); });
    static_for<6>([&](auto a) RL_INLINE { fa[a].touch(); });
    if constexpr (F8) {
      asm volatile("" : "+v"(san));
      sa = san;
    }
    MC_FENCE();
  };
  wait_next();
  int st = 0;

  for (int w = blockIdx.x; w < nwork; w += gridDim.x) {
    int n0, u0, u1;
    const GroupTile t = item(w, n0, u0, u1);
    const bool rest = t.e >= experts;
    ArgPtr ga = fresh();
    [[maybe_unused]] int wscale0 = 127, wscale1 = 127;  // scale bytes of W, a K tile a lane
    if constexpr (F8) {
      if (!rest) {
        const int nb = (n0 >> 7) + wn, blocks = B_STR ? (ga->K + 127) >> 7 : (ga->N + 127) >> 7;
        auto scale = [&](int kb) RL_INLINE {
          kb = kb < nt ? kb : nt - 1;
          const int ib = B_STR ? kb : nb, ob = B_STR ? nb : kb;
          return ib < blocks && ob < ga->scols ? (int)ga->SB[t.e * ga->ssb + (int64_t)ib * ga->scols + ob] : 127;
        };
        wscale0 = scale(lane);
        if (nt > 64) wscale1 = scale(64 + lane);
      }
    }
    f32x4 start[8];  // the accumulators start with the bias
#pragma unroll
    for (int b = 0; b < 8; ++b) start[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (ga->bias != nullptr && !rest && u0 == 0) {
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        int c = n0 + wn * 128 + 16 * b + 4 * grp;
        c = c < ga->N ? c : ga->N - 4;  // (columns beyond N are never stored)
        const i32x2 v = *reinterpret_cast<const i32x2*>(static_cast<const T*>(ga->bias) + (int64_t)t.e * ga->N + c);
        const T* const b4 = reinterpret_cast<const T*>(&v);
#pragma unroll
        for (int e = 0; e < 4; ++e) start[b][e] = (float)b4[e];
      }
    }
    static_for<64>([&](auto e) RL_INLINE { acc[decltype(e)::value >> 3][decltype(e)::value & 7] = start[decltype(e)::value & 7]; });
    if constexpr (F8) {
      __builtin_amdgcn_s_waitcnt(mc_wait_imm(0, false));
      asm volatile("" : "+v"(wscale0), "+v"(wscale1));
      if (u0 > 64) wscale0 = wscale1;
    }

    // A K tile is 64 slots of 32 cycles, two steps.  Its stage is free once every wave has read its last fragments (slot kFree), and the
    // loads of the tile after the next go out from there on, one in two slots, so that the last of them still has three quarters of a K
    // tile to land (issued from the second step on, behind the barrier that hands the next tile over, half: what a compute unit
    // fetches is bound by latency, see below).
    constexpr int kFree = 10, kFirst = kFree + 2, kEarly = (32 - kFirst + 1) / 2;  // kEarly: loads of a refill in front of step 1's wait
    auto refill = [&](auto s_c) RL_INLINE {
      constexpr int s = decltype(s_c)::value, j = (s - kFirst) / 2;
      if constexpr (s >= kFirst && (s - kFirst) % 2 == 0 && j < LPT) issue_load(st, std::integral_constant<int, j>{});
    };
    // one K tile; TAIL, NEXT: it, and the one behind it in the load stream, are of the adapter's product
    auto k_tile = [&](auto tail_c, auto next_c) RL_INLINE {
      const uint32_t soff = (uint32_t)(st * P::STAGE_BYTES), soffn = (uint32_t)((st ^ 1) * P::STAGE_BYTES);
      MC_FENCE();
      // Step 0: B blocks 0..3; A blocks 6, 7 and B blocks 4..7 are fetched, the last reads of this tile's stage.
      static_for<8>([&](auto a_c) RL_INLINE {
        constexpr int a = decltype(a_c)::value;
        row_products(tail_c, a_c, H0{}, [&](auto j_c) RL_INLINE {
          constexpr int s = 4 * a + decltype(j_c)::value;
          if constexpr (s < 2) read_A(std::integral_constant<int, 6 + s>{}, soff);
          if constexpr (s >= 1 && s < 5) read_B(tail_c, std::integral_constant<int, 3 + s>{}, soff);
          if constexpr (s == kFree) {  // everyone has read this tile: its stage may be refilled
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fa[6].touch(); fa[7].touch();
            static_for<4>([&](auto b) RL_INLINE { fb[4 + decltype(b)::value].touch(); });
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
          }
          refill(std::integral_constant<int, s>{});
        });
      });
      // Step 1: B blocks 4..7; behind the first products the next tile has landed, and its first fragments are fetched.
      static_for<8>([&](auto a_c) RL_INLINE {
        constexpr int a = decltype(a_c)::value;
        row_products(tail_c, a_c, std::integral_constant<int, 4>{}, [&](auto j_c) RL_INLINE {
          constexpr int s = 4 * a + decltype(j_c)::value;
          if constexpr (s == 0) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(mc_wait_imm(kEarly, false));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            MC_FENCE();
            read_scales(st ^ 1);
          }
          if constexpr (s >= 1 && s < 5) read_B(next_c, std::integral_constant<int, s - 1>{}, soffn);
          if constexpr (s % 4 == 3 && s < 24) read_A(std::integral_constant<int, s / 4>{}, soffn);
          refill(std::integral_constant<int, 32 + s>{});
          if constexpr (32 + s == kFirst + 2 * LPT) cursor_step();
        });
      });
      wait_next();
    };
    using Main = std::false_type;
    using Tail = std::true_type;
    auto scale_of = [&](int u) RL_INLINE {
      if constexpr (F8) {
        if (__builtin_expect(u == 64, 0)) wscale0 = wscale1;
        wsc = __builtin_amdgcn_readlane(wscale0, u & 63);
        asm volatile("s_nop 4" : "+v"(wsc));  // (in a vector register, ahead of the products that the compiler does not know to guard)
      }
    };
    // (in sequence, and not one loop over kinds: where different products meet, the compiler moves accumulators)
    const bool tail = ntail > 0 && u1 == nt && !rest;
    const int before = rest ? u0 : (tail ? u1 - 1 : u1);  // K tiles with another of the large product's behind them in the stream
    auto next_tile = [&]() RL_INLINE {
      if (__builtin_expect(clive && cu >= cnext, 0)) {
        cursor_event();
        cursor_point();
      }
      st ^= 1;
    };
    for (int u = u0; u < before; ++u) {
      scale_of(u);
      k_tile(Main{}, Main{});
      next_tile();
    }
    if (tail) {
      scale_of(nt - 1);
      k_tile(Main{}, Tail{});
      next_tile();
      for (int u = 1; u < ntail; ++u) {
        k_tile(Tail{}, Tail{});
        next_tile();
      }
      k_tile(Tail{}, Main{});
      next_tile();
    }
    asm volatile("s_nop 7\n\ts_nop 7");  // the last products' results, read by hand below
    ga = fresh();
    if (w >= split.whole) {  // fp32 sums of a run of K tiles, as the accumulators lie
      f32x4* const part = reinterpret_cast<f32x4*>(ga->partial) + ((int64_t)(w - split.whole) * 4 + wave) * 4096 + lane;
      static_for<64>([&](auto e_c) RL_INLINE {
        constexpr int e = decltype(e_c)::value;
        float x0, x1, x2, x3;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x0) : "a"(acc[e >> 3][e & 7][0]));
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x1) : "a"(acc[e >> 3][e & 7][1]));
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x2) : "a"(acc[e >> 3][e & 7][2]));
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x3) : "a"(acc[e >> 3][e & 7][3]));
        part[e * 64] = f32x4{x0, x1, x2, x3};
        MC_FENCE();
      });
      continue;
    }
    // ---- epilogue: 16 rows x 128 columns of the wave at a time through LDS, 16-byte pieces of 4 rows x 256 bytes out (gemm_mc64.hpp)
    const uint32_t stg = lds_base + (uint32_t)(P::STAGING + wave * 4096);
    const int rr = lane >> 4, rc = lane & 15;
    const int ncol = n0 + wn * 128 + rc * 8;
    const bool n_ok = ncol < ga->N;
    T* const C = static_cast<T*>(ga->C) + ncol;
    static_for<8>([&](auto a_c) RL_INLINE {
      constexpr int a = decltype(a_c)::value;
      const uint32_t wr = stg + (uint32_t)s16 * 256u, wsw = 2u * (uint32_t)s16;
      static_for<8>([&](auto b_c) RL_INLINE {
        constexpr int b = decltype(b_c)::value;
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        typedef T tx2_t __attribute__((ext_vector_type(2)));
        float x0, x1, x2, x3;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x0) : "a"(acc[a][b][0]));
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x1) : "a"(acc[a][b][1]));
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x2) : "a"(acc[a][b][2]));
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x3) : "a"(acc[a][b][3]));
        const f32x2_t lo = {x0, x1}, hi2 = {x2, x3};
        const i32x2 v = {(int)__builtin_bit_cast(unsigned, __builtin_convertvector(lo, tx2_t)), (int)__builtin_bit_cast(unsigned, __builtin_convertvector(hi2, tx2_t))};
        const uint32_t slot = ((uint32_t)(4 * b + (grp & 2)) ^ wsw) + (uint32_t)(grp & 1);
        asm volatile("ds_write_b64 %0, %1" : : "v"(wr + slot * 8u), "v"(v) : "memory");
        MC_FENCE();
      });
      i32x4 o[4];
      {
        uint32_t addr[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t row = (uint32_t)(4 * k + rr);
          addr[k] = stg + row * 256u + (((uint32_t)(2 * rc) ^ (2u * row)) * 8u);
        }
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]) : "v"(addr[0]), "v"(addr[1]), "v"(addr[2]), "v"(addr[3]) : "memory");
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = 4 * k + rr, m = t.m0 + wm * 128 + (F8 ? 8 * r + a : 16 * a + r);
        if (n_ok && m >= t.lo && m < t.hi) *reinterpret_cast<i32x4*>(C + (int64_t)m * ga->ldc) = o[k];
      }
      MC_FENCE();
    });
  }
  // the LDS-DMA writes still in flight target this workgroup's LDS: let them land before it is released
  __builtin_amdgcn_s_waitcnt(mc_wait_imm(0, true));
#undef MC_FENCE
}
#undef RL_INLINE

// The split tiles' sums added up in order, rounded and stored: a workgroup takes a sixteenth of a tile (16 of its 256 accumulator blocks).
constexpr int kJoinPieces = 16;
template <typename T, bool F8>
__global__ __launch_bounds__(256) void grouped_mc_join_kernel(GroupedArgs g) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  GroupedOrder<F8> order;
  order.open(g, lane);
  const GroupedSplit split = grouped_split(g, order.total, (g.K + (F8 ? 127 : 63)) / (F8 ? 128 : 64));
  const int tile = (int)blockIdx.x / kJoinPieces, piece = (int)blockIdx.x % kJoinPieces;
  if (tile >= order.total - split.whole) return;
  int n0;
  const GroupTile t = order.at(g, lane, split.whole + tile, n0);
  const f32x4* part = reinterpret_cast<const f32x4*>(g.partial) + (int64_t)tile * split.splits * 16384;
  f32x4 sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < split.splits; ++s, part += 16384) {
#pragma unroll
    for (int k = 0; k < 4; ++k) sum[k] += part[((piece * 4 + wave) * 4 + k) * 64 + lane];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int block = (piece * 4 + wave) * 4 + k;  // [wave of the tile][row block][column block]
    const int w = block >> 6, a = (block >> 3) & 7, b = block & 7, r = lane & 15;
    const int m = t.m0 + (w >> 1) * 128 + (F8 ? 8 * r + a : 16 * a + r), n = n0 + (w & 1) * 128 + 16 * b + 4 * (lane >> 4);
    if (m < t.lo || m >= t.hi || n >= g.N) continue;
    T o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = from_f32<T>(sum[k][e]);
    *reinterpret_cast<i32x2*>(static_cast<T*>(g.C) + (int64_t)m * g.ldc + n) = *reinterpret_cast<const i32x2*>(o);
  }
}

}  // namespace rl
