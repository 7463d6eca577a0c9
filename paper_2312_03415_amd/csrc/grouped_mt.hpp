// Matrix-core kernel of the grouped and 8-bit products (grouped.hpp) on tiles of up to 128 x 128.
//
//  - A workgroup finds its tile itself: the row counts of the experts are in device memory, so the grid is the most tiles that n rows
//    can make and workgroups beyond the last return.  Every wave reads the ends (64 to a load), turns them into tile counts and sums
//    them across its lanes.
//  - 4 waves, K tile of 128 bytes (64 16-bit values, or 128 e4m3 values: one scale block), LDS ring of NS stages filled by 16-byte
//    LDS-DMA loads; what lies outside the operands is fetched from past the buffer's end, which gives zeros.  Layouts and swizzles
//    of the tiles as in gemm_mt.hpp; a K-strided e4m3 tile is read with ds_read_b64_tr_b8.
//  - e4m3: v_mfma_scale_f32_16x16x128_f8f6f4 takes the power-of-two scales with the operands: no vector instruction is spent on
//    them.  A lane wants the scales of row l % 16 of every 16-row block of the wave; the wave's rows are dealt out to the blocks in
//    turn (block a holds rows TM s + a), so that they are consecutive bytes.
//  - The adapter's product runs behind the K loop in the same accumulators, its fragments straight from memory, the first 32 of the rank
//    requested ahead of the loop: T is [n, R] and the other factor is laid out [N, R], both with the contraction in the rows.
//
// What bounds it: what a compute unit fetches through its L1 (33 to 45 B/ns), or memory.  One row tile an expert: 64 rows of 16 experts 4096 ->
// 11008 e4m3, W at 6.2 TB/s (117 us); 16 rows of 8 experts 2048 -> 8192 bf16 39 us, 6.1 TB/s.  More rows: 999 of 12 experts 1032 -> 2744 f16 23 us,
// 2000 x 4096 -> 4096 bf16 68 us (1.0 PFLOP/s).  Two workgroups a compute unit hide each other's waits: one with a ring of four stages took
// 117 us in place of 68 there, and a second set of operand registers, read while the first is multiplied, gained nothing (24.2 us
// against 23.9 and 42.4 against 39.6 at two small shapes, 317 against 306 for 4096 rows of 64 experts 2048 -> 8192 e4m3).
#pragma once
#include <type_traits>
#include <utility>

#include "fp8.hpp"
#include "gemm_mt.hpp"
#include "grouped.hpp"

namespace rl {

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8;

// Tile `t` of the row tiles of all groups: expert, first row of the tile, the group's rows [lo, hi).  e = experts: the rows behind the
// last expert's.  `ends` that are out of range or decrease are clamped, so that no access depends on their values being right.
struct GroupTile {
  int e, m0, lo, hi;
};
template <int BM, bool F8>
__device__ __forceinline__ int group_tiles(int lo, int hi) {
  return hi > lo ? (hi - (F8 ? lo & ~3 : lo) + BM - 1) / BM : 0;
}
// The row tiles of up to 64 experts, one a lane, and of all together; further experts are scanned 64 at a time wherever a tile is looked up.
template <int BM, bool F8>
struct GroupScan {
  int lo, hi, tiles, sum;     // of the first 64: rows, row tiles, row tiles up to and with this one
  int total, rest_lo;         // row tiles of all groups; where the rows behind the last expert's begin
  __device__ __forceinline__ void scan(const int32_t* ends, int experts, int n, int base, int lane) {
    const int e = base + lane;
    auto clamped = [&](int v) { return v < 0 ? 0 : (v > n ? n : v); };
    lo = hi = 0;
    if (e < experts) {
      hi = ends == nullptr ? n : clamped(ends[e]);
      lo = ends == nullptr || e == 0 ? 0 : clamped(ends[e - 1]);
      if (hi < lo) hi = lo;
    }
    tiles = group_tiles<BM, F8>(lo, hi);
    sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(sum, d);
      if (lane >= d) sum += v;
    }
  }
  __device__ __forceinline__ void open(const int32_t* ends, int experts, int n, int lane) {
    if (ends == nullptr) {  // one expert, all rows
      const bool first = lane == 0;
      lo = 0;
      hi = first ? n : 0;
      tiles = first ? (n + BM - 1) / BM : 0;
      sum = total = (n + BM - 1) / BM;
      rest_lo = n;
      return;
    }
    total = 0;
    for (int base = (experts - 1) & ~63; base >= 0; base -= 64) {  // (the first 64 last: theirs stay)
      scan(ends, experts, n, base, lane);
      total += __builtin_amdgcn_readlane(sum, 63);
      if (base == ((experts - 1) & ~63)) rest_lo = __builtin_amdgcn_readlane(hi, (experts - 1) & 63);
    }
    total += group_tiles<BM, F8>(rest_lo, n);
  }
  // row tile t
  __device__ __forceinline__ GroupTile find(const int32_t* ends, int experts, int n, int lane, int t) const {
    GroupScan s = *this;
    GroupTile out{experts, 0, rest_lo, n};
    int before = 0;
    for (int base = 0; base < experts; base += 64) {
      if (base > 0) s.scan(ends, experts, n, base, lane);
      const int all = __builtin_amdgcn_readlane(s.sum, 63);
      if (t < before + all) {
        const int l = __builtin_ctzll(__ballot(s.sum > t - before));
        out.e = base + l;
        out.lo = __builtin_amdgcn_readlane(s.lo, l);
        out.hi = __builtin_amdgcn_readlane(s.hi, l);
        before += __builtin_amdgcn_readlane(s.sum, l) - __builtin_amdgcn_readlane(s.tiles, l);
        break;
      }
      before += all;
    }
    out.m0 = (F8 ? out.lo & ~3 : out.lo) + (t - before) * BM;
    return out;
  }
};

template <bool F8, int AL, int BL, int BM_, int BN_, int WM_, int NS_>
struct GroupedTileShape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = 4 / WM_, NS = NS_;
  static constexpr int EB = F8 ? 1 : 2, KE = 128 / EB;  // bytes of an element, elements of a K tile
  static constexpr bool A_STR = AL == 1, B_STR = BL == 0;
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, S_BYTES = F8 ? 1024 : 0;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + S_BYTES;
  static constexpr int IA = A_BYTES / 4096, IB = B_BYTES / 4096, LPT = IA + IB + (F8 ? 1 : 0);
  static constexpr int EPI_LD = WTN + 4, EPI_BYTES = 4 * 16 * EPI_LD * 4;
  static constexpr int RING_BYTES = NS * STAGE_BYTES, LDS_BYTES = RING_BYTES > EPI_BYTES ? RING_BYTES : EPI_BYTES;
  static_assert(IA >= 1 && IB >= 1 && TM >= 1 && TN >= 1 && LDS_BYTES <= 160 * 1024 && (NS - 1) * LPT < 64, "tile shape");
  static_assert(!F8 || (AL == 0 && BN >= 128 && TM <= 4 && TM != 3), "e4m3 tiles");
};

// chunk (16 bytes) index of k-row q of a K-strided tile with BX columns is XORed with this
template <bool F8, int BX>
__device__ __forceinline__ int grouped_swz(int q) {
  if constexpr (F8) return BX == 128 ? (((q >> 1) & 3) | (((q >> 4) & 1) << 2)) : ((q & 7) | (((q >> 4) & 1) << 3));
  else if constexpr (BX == 32) return 2 * ((q >> 3) & 1);
  else return mt_swz<BX>(q);
}

// ROWS: A, which a rank-r product reads once (X in T = s X A, dY in Z = s dY B^T), is rounded to e4m3 for the large product on the way: a
// thread takes the 16-byte chunks of the tile that it loaded, keeps those of every other K tile, and rounds both halves of a block
// of 128 columns together, the eight lanes of a row agreeing on its largest magnitude.  The pass over A that rounding would take is saved:
// dY of 8192 x 11008 r 32 69 us in place of 58 + 35 in two, of 16384 x 11008 r 128 163 in place of 134 + 102.
template <typename T, bool F8, int AL, int BL, int BM, int BN, int WM, int NS, bool ROWS = false>
__device__ __forceinline__ void grouped_mt_body(const GroupedArgs& g, const int bx, const int by) {
  static_assert(!ROWS || (!F8 && AL == 0), "a 16-bit A by rows");
  using P = GroupedTileShape<F8, AL, BL, BM, BN, WM, NS>;
  constexpr int EB = P::EB, KE = P::KE, TM = P::TM, TN = P::TN;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  unsigned char* const smem = smem_raw;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / P::WN, wn = wave % P::WN;
  const int s16 = lane & 15, grp = lane >> 4;
  const int nbn = (g.N + BN - 1) / BN;

  // ---- this workgroup's tile
  GroupTile gt;
  int m0, n0, u0, u1;
  if constexpr (AL == 0) {
    GroupScan<BM, F8> groups;
    groups.open(g.ends, g.experts, g.n, lane);
    const int nbm = groups.total, total = nbm * nbn;
    if (bx >= total) return;
    const int x = bx & 7, slot = bx >> 3, q = total >> 3, rem = total & 7;
    const int id = x * q + (x < rem ? x : rem) + slot;  // a contiguous run of tiles per XCD, walked in bands of row tiles
    const int per_band = g.band * nbn, band = id / per_band, first_m = band * g.band;
    const int band_rows = (nbm - first_m) < g.band ? (nbm - first_m) : g.band, in_band = id - band * per_band;
    gt = groups.find(g.ends, g.experts, g.n, lane, first_m + in_band % band_rows);
    m0 = gt.m0;
    n0 = (in_band / band_rows) * BN;
    const int nt = gt.e < g.experts ? (g.K + KE - 1) / KE : 0;
    u0 = by * g.tiles_per_split;
    u1 = u0 + g.tiles_per_split < nt ? u0 + g.tiles_per_split : nt;
  } else {
    const int nbm = (g.M + BM - 1) / BM, per = nbm * nbn;
    gt.e = bx / per;
    const int id = bx - gt.e * per;
    auto clamped = [&](int v) { return v < 0 ? 0 : (v > g.n ? g.n : v); };
    gt.hi = g.ends == nullptr ? g.n : clamped(g.ends[gt.e]);
    gt.lo = g.ends == nullptr || gt.e == 0 ? 0 : clamped(g.ends[gt.e - 1]);
    if (gt.hi < gt.lo) gt.hi = gt.lo;
    m0 = (id / nbn) * BM;
    n0 = (id % nbn) * BN;
    const int nt = (gt.hi - gt.lo + KE - 1) / KE, each = (nt + g.splits - 1) / g.splits;
    u0 = by * each;
    u1 = u0 + each < nt ? u0 + each : nt;
  }
  const bool rest = gt.e >= g.experts;
  const int K = AL == 0 ? g.K : gt.hi - gt.lo;

  // ---- loads.  Per-lane byte offsets from a base that moves on by a K tile at a time (64-bit, so that nothing wraps in a long
  // matrix); lanes that must read zeros carry an offset past every buffer's end.
  constexpr uint32_t OOB = 0x80000000u;
  uint32_t offA[P::IA], offB[P::IB], offS = OOB;
  uint32_t tailA = 0, tailB = 0;  // bit j: load j lies beyond K in the last, partial K tile (K-contiguous operands)
  const int ktail = K - (K / KE) * KE;  // != 0: the last K tile holds so many
  auto lane_offset = [&](auto str_c, auto bx_c, int p, int base, int dim, int64_t ld, bool perm) -> uint32_t {
    constexpr bool STR = decltype(str_c)::value;
    constexpr int BX = decltype(bx_c)::value;
    if constexpr (!STR) {
      int row = p >> 3;
      const int col = ((p & 7) ^ ((row >> 1) & 7)) * (16 / EB);
      if (perm) row = (row / P::WTM) * P::WTM + (row % 16) * TM + (row % P::WTM) / 16;
      return base + row < dim ? (uint32_t)(((int64_t)row * ld + col) * EB) : OOB;
    } else {
      constexpr int CPR = BX * EB / 16;
      const int row = p / CPR, col = ((p % CPR) ^ grouped_swz<F8, BX>(row)) * (16 / EB);
      return base + col < dim ? (uint32_t)(((int64_t)row * ld + col) * EB) : OOB;
    }
  };
#pragma unroll
  for (int j = 0; j < P::IA; ++j) {
    const int p = (wave * P::IA + j) * 64 + lane;
    offA[j] = lane_offset(std::bool_constant<P::A_STR>{}, std::integral_constant<int, BM>{}, p, m0, AL == 0 ? g.n : g.M, g.lda, F8);
    if (!P::A_STR && ktail != 0 && ((p & 7) ^ ((p >> 4) & 7)) * (16 / EB) >= ktail) tailA |= 1u << j;
  }
#pragma unroll
  for (int j = 0; j < P::IB; ++j) {
    const int p = (wave * P::IB + j) * 64 + lane;
    offB[j] = lane_offset(std::bool_constant<P::B_STR>{}, std::integral_constant<int, BN>{}, p, n0, g.N, g.ldb, false);
    if (!P::B_STR && ktail != 0 && ((p & 7) ^ ((p >> 4) & 7)) * (16 / EB) >= ktail) tailB |= 1u << j;
  }
  if constexpr (F8) {
    if (lane < BM / 4) offS = 4u * lane;
    tailA = 0;  // rows of A are whole scale blocks, zeros behind K
  }
  // bases of K tile u0 (bytes), and what lies between them and the ends of the operands
  const unsigned char *pA, *pB, *pS = nullptr;
  int64_t leftA, leftB, stepA, stepB;
  {
    const int64_t k0 = (int64_t)u0 * KE;
    if constexpr (AL == 0) {
      const int64_t Ka = F8 ? (int64_t)((K + 127) / 128) * 128 : K, rows = g.n - m0;
      pA = static_cast<const unsigned char*>(g.A) + ((int64_t)m0 * g.lda + k0) * EB;
      leftA = ((rows - 1) * g.lda + Ka - k0) * EB;
      stepA = 128;
    } else {
      pA = static_cast<const unsigned char*>(g.A) + ((gt.lo + k0) * g.lda + m0) * EB;
      leftA = ((K - k0 - 1) * g.lda + g.M - m0) * EB;
      stepA = (int64_t)KE * g.lda * EB;
    }
    const unsigned char* const Be = static_cast<const unsigned char*>(g.B) + (AL == 0 ? (int64_t)(rest ? 0 : gt.e) * g.sb : (int64_t)gt.lo * g.ldb) * EB;
    if constexpr (P::B_STR) {
      pB = Be + (k0 * g.ldb + n0) * EB;
      leftB = ((K - k0 - 1) * g.ldb + g.N - n0) * EB;
      stepB = (int64_t)KE * g.ldb * EB;
    } else {
      pB = Be + ((int64_t)n0 * g.ldb + k0) * EB;
      leftB = ((int64_t)(g.N - n0 - 1) * g.ldb + K - k0) * EB;
      stepB = 128;
    }
    if constexpr (F8) pS = g.SA + u0 * g.ldsa + m0;
  }
  int ul = u0;  // the K tile that is loaded next
  auto rsrc = [&](const unsigned char* base, int64_t left) {
    const int size = ul >= u1 || left <= 0 ? 0 : (left > 0x7fffffff ? 0x7fffffff : (int)left);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, size, 0x00020000);
  };
  auto issue_tile = [&](int st) {
    unsigned char* const dst = smem + st * P::STAGE_BYTES;
    const bool partial = ktail != 0 && ul == K / KE;
    const uint32_t ta = partial ? tailA : 0u, tb = partial ? tailB : 0u;
    const __amdgpu_buffer_rsrc_t ra = rsrc(pA, leftA), rb = rsrc(pB, leftB);
#pragma unroll
    for (int j = 0; j < P::IA; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (mc_lds_void_t*)(dst + (wave * P::IA + j) * 1024), 16, offA[j] | ((ta << (31 - j)) & OOB), 0, 0, 0);
#pragma unroll
    for (int j = 0; j < P::IB; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (mc_lds_void_t*)(dst + P::A_BYTES + (wave * P::IB + j) * 1024), 16, offB[j] | ((tb << (31 - j)) & OOB), 0, 0, 0);
    if constexpr (F8) {
      const __amdgpu_buffer_rsrc_t rs = rsrc(pS, g.ldsa - m0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (mc_lds_void_t*)(dst + P::A_BYTES + P::B_BYTES + wave * 256), 4, offS, 0, 0, 0);
      pS += g.ldsa;
    }
    ++ul;
    pA += stepA; leftA -= stepA;
    pB += stepB; leftB -= stepB;
  };

  // ---- fragment addresses inside a stage
  constexpr int NFA = P::A_STR ? TM : 2, NFB = P::B_STR ? TN : 2;
  uint32_t fragA[NFA], fragB[NFB];
  {
    const int sw = (s16 >> 1) & 7;
    const int kr = F8 ? 16 * grp + (s16 >> 1) : 8 * grp + (s16 >> 2);  // k-row that a transposing read of this lane points at
    const int cb = F8 ? 0 : (s16 & 3) >> 1, half = s16 & 1;             // chunk inside the 16 columns, 8-byte half of it
    if constexpr (!P::A_STR) {
#pragma unroll
      for (int h = 0; h < 2; ++h) fragA[h] = (uint32_t)((wm * P::WTM + s16) * 128 + (((4 * h + grp) ^ sw) << 4));
    } else {
#pragma unroll
      for (int b = 0; b < TM; ++b)
        fragA[b] = (uint32_t)(kr * (BM * EB) + (((wm * P::WTM + 16 * b) * EB / 16 + cb) ^ grouped_swz<F8, BM>(kr)) * 16 + 8 * half);
    }
    if constexpr (!P::B_STR) {
#pragma unroll
      for (int h = 0; h < 2; ++h) fragB[h] = (uint32_t)(P::A_BYTES + (wn * P::WTN + s16) * 128 + (((4 * h + grp) ^ sw) << 4));
    } else {
#pragma unroll
      for (int b = 0; b < TN; ++b)
        fragB[b] = (uint32_t)(P::A_BYTES + kr * (BN * EB) + (((wn * P::WTN + 16 * b) * EB / 16 + cb) ^ grouped_swz<F8, BN>(kr)) * 16 + 8 * half);
    }
  }
  const uint32_t lds_base = (uint32_t)(uintptr_t)((mc_lds_void_t*)smem);
  // half h of a 32-byte fragment: k 32 h + 8 grp .. + 7 (16-bit), 64 h + 16 grp .. + 15 (e4m3)
  auto read_half = [&](auto& out, const auto& fr, uint32_t soff, auto str_c, auto bx_c, auto blk_c, auto h_c) {
    constexpr bool STR = decltype(str_c)::value;
    constexpr int BX = decltype(bx_c)::value, blk = decltype(blk_c)::value, h = decltype(h_c)::value;
    if constexpr (!STR) {
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(out.v) : "v"(lds_base + soff + fr[h]), "i"(blk * 2048));
    } else if constexpr (F8) {
      const uint32_t addr = lds_base + soff + fr[blk];
      asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(out.lo) : "v"(addr), "i"(h * 64 * BX));
      asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(out.hi) : "v"(addr), "i"(h * 64 * BX + 8 * BX));
    } else {
      const uint32_t addr = lds_base + soff + fr[blk];
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(out.lo) : "v"(addr), "i"(h * 64 * BX));
      asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(out.hi) : "v"(addr), "i"(h * 64 * BX + 8 * BX));
    }
  };

  // the adapter's factors, 32 of the rank at a time, straight from memory; the first ones are on their way ahead of the K loop
  constexpr bool TAIL = AL == 0 && !ROWS && BN >= 128;
  const bool has_tail = TAIL && g.R > 0 && !rest;
  // row of the wave's tile that element r of block a is
  auto row_of = [&](int a, int r) { return F8 ? r * TM + a : 16 * a + r; };
  i32x4 tailA_regs[TAIL ? TM : 1], tailB_regs[TAIL ? TN : 1];
  [[maybe_unused]] auto load_tail = [&](int k0) __attribute__((always_inline)) {
    if constexpr (TAIL) {
      const int k = k0 + 8 * grp;
      const i32x4 zero = {0, 0, 0, 0};
      const T* const tb = static_cast<const T*>(g.TB) + gt.e * g.stb;
#pragma unroll
      for (int b = 0; b < TN; ++b) {
        const int c = n0 + wn * P::WTN + 16 * b + s16;
        tailB_regs[b] = k < g.R && c < g.N ? *reinterpret_cast<const i32x4*>(tb + (int64_t)c * g.ldtb + k) : zero;
      }
#pragma unroll
      for (int a = 0; a < TM; ++a) {
        const int m = m0 + wm * P::WTM + row_of(a, s16);
        tailA_regs[a] = k < g.R && m < g.n ? *reinterpret_cast<const i32x4*>(static_cast<const T*>(g.TA) + (int64_t)m * g.ldta + k) : zero;
      }
    }
  };
  if (has_tail) load_tail(0);

  f32x4 acc[TM][TN];  // lane l: row l % 16, columns 4 (l / 16) .. + 3 of each 16x16 block
  static_for<TM * TN>([&](auto e) { acc[decltype(e)::value / TN][decltype(e)::value % TN] = f32x4{0.f, 0.f, 0.f, 0.f}; });

  if (u0 < u1) {
    for (int s = 0; s < NS - 1; ++s) issue_tile(s);
    [[maybe_unused]] i32x4 kept[P::IA];  // ROWS: this thread's chunks of the even K tile of a pair (u0 is even)
    [[maybe_unused]] int wscale = 0;  // scale bytes of W for 64 K tiles, one per lane
    int st = 0, fill = NS - 1;
    for (int u = u0; u < u1; ++u) {
      if constexpr (F8) {
        if (((u - u0) & 63) == 0) {
          const int kb = u + lane < u1 ? u + lane : u1 - 1, nb = (n0 + wn * P::WTN) >> 7;
          const int ob = P::B_STR ? nb : kb, ib = P::B_STR ? kb : nb;
          const int cols = g.scols, rows = P::B_STR ? (K + 127) >> 7 : (g.N + 127) >> 7;
          wscale = ib < rows && ob < cols ? g.SB[gt.e * g.ssb + (int64_t)ib * cols + ob] : 127;
          __builtin_amdgcn_s_waitcnt(mc_wait_imm(0, false));  // here, once in 64 tiles, and not in front of every use
          asm volatile("" : "+v"(wscale));
        }
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(mc_wait_imm((NS - 2) * P::LPT, false));
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      issue_tile(fill);
      fill = fill + 1 == NS ? 0 : fill + 1;
      const uint32_t soff = (uint32_t)(st * P::STAGE_BYTES);
      st = st + 1 == NS ? 0 : st + 1;
      __builtin_amdgcn_sched_barrier(0);
      MtFrag<P::A_STR> fa[TM][2];
      MtFrag<P::B_STR> fb[TN][2];
      [[maybe_unused]] uint32_t sa = 0;
      static_for<2>([&](auto h) {
        static_for<TN>([&](auto b) { read_half(fb[b][h], fragB, soff, std::bool_constant<P::B_STR>{}, std::integral_constant<int, BN>{}, b, h); });
        static_for<TM>([&](auto a) { read_half(fa[a][h], fragA, soff, std::bool_constant<P::A_STR>{}, std::integral_constant<int, BM>{}, a, h); });
      });
      if constexpr (F8) {
        const uint32_t addr = lds_base + soff + (uint32_t)(P::A_BYTES + P::B_BYTES + wave * 256 + wm * P::WTM + s16 * TM);
        if constexpr (TM == 1) asm volatile("ds_read_u8 %0, %1" : "=v"(sa) : "v"(addr));
        else if constexpr (TM == 2) asm volatile("ds_read_u16 %0, %1" : "=v"(sa) : "v"(addr));
        else asm volatile("ds_read_b32 %0, %1" : "=v"(sa) : "v"(addr));
      }
      [[maybe_unused]] i32x4 chunk[P::IA];
      if constexpr (ROWS) {
        const uint32_t at = lds_base + soff + (uint32_t)(wave * (P::IA * 1024) + lane * 16);
        static_for<P::IA>([&](auto j) { auto& c = chunk[j]; const uint32_t a = at; asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(c) : "v"(a), "i"(decltype(j)::value * 1024)); });
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      static_for<2>([&](auto h) {
        static_for<TN>([&](auto b) { fb[b][h].touch(); });
        static_for<TM>([&](auto a) { fa[a][h].touch(); });
      });
      if constexpr (F8) {
        asm volatile("" : "+v"(sa));
        const int wb = __builtin_amdgcn_readlane(wscale, (u - u0) & 63);
        static_for<TM * TN>([&](auto q) {
          constexpr int a = decltype(q)::value / TN, b = decltype(q)::value % TN;
          const i32x4 x0 = fb[b][0].get(), x1 = fb[b][1].get(), y0 = fa[a][0].get(), y1 = fa[a][1].get();
          acc[a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7),
                                                                       __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7), acc[a][b], 0, 0, 0, wb,
                                                                       a, sa);
        });
      } else {
        static_for<2>([&](auto h) {
          static_for<TM * TN>([&](auto q) {
            constexpr int a = decltype(q)::value / TN, b = decltype(q)::value % TN;
            acc[a][b] = Mma16<T>::mma(fb[b][h].get(), fa[a][h].get(), acc[a][b]);
          });
        });
      }
      if constexpr (ROWS) {
        static_for<P::IA>([&](auto j) { auto& c = chunk[j]; asm volatile("" : "+v"(c)); });
        const bool odd = (u & 1) != 0;
        if (odd || u + 1 == u1) {  // the block's second half, or none of it lies inside K
#pragma unroll
          for (int j = 0; j < P::IA; ++j) {
            const i32x4 none = {0, 0, 0, 0}, half[2] = {odd ? kept[j] : chunk[j], odd ? chunk[j] : none};
            float v[16];
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              v[k] = (float)reinterpret_cast<const T*>(&half[k >> 3])[k & 7];
              const uint32_t bits = __float_as_uint(v[k]) & 0x7FFFFFFFu;
              top = top > bits ? top : bits;
            }
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) {
              const uint32_t other = (uint32_t)__shfl_xor((int)top, d);
              top = top > other ? top : other;
            }
            uint32_t byte;
            float mul;
            bool nan;
            fp8_block_scale(top, &byte, &mul, &nan);
            const int p = (wave * P::IA + j) * 64 + lane, row = p >> 3, m = m0 + row, kb = u >> 1;
            const int col = kb * 128 + (((p & 7) ^ ((row >> 1) & 7)) << 3);
            if (n0 == 0 && m >= gt.lo && m < gt.hi) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                i32x2 out = {fp8_pack4(v[8 * h] * mul, v[8 * h + 1] * mul, v[8 * h + 2] * mul, v[8 * h + 3] * mul),
                             fp8_pack4(v[8 * h + 4] * mul, v[8 * h + 5] * mul, v[8 * h + 6] * mul, v[8 * h + 7] * mul)};
                if (nan) out = i32x2{0x7F7F7F7F, 0x7F7F7F7F};
                *reinterpret_cast<i32x2*>(g.Q + (int64_t)m * g.ldq + col + 64 * h) = out;
              }
              if ((lane & 7) == 0) g.QS[(int64_t)kb * g.ldqs + m] = (uint8_t)byte;
            }
          }
        }
#pragma unroll
        for (int j = 0; j < P::IA; ++j) kept[j] = chunk[j];
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // (loads of nothing may still be in flight: the ring becomes the epilogue's staging area behind this)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(mc_wait_imm(0, true));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  // ---- the adapter's product
  if constexpr (TAIL) {
    if (has_tail) {
      for (int k0 = 0;;) {
        static_for<TM * TN>([&](auto q) {
          constexpr int a = decltype(q)::value / TN, b = decltype(q)::value % TN;
          acc[a][b] = Mma16<T>::mma(tailB_regs[b], tailA_regs[a], acc[a][b]);
        });
        if ((k0 += 32) >= g.R) break;
        load_tail(k0);
      }
    }
  }

  // ---- epilogue: 16 rows of the wave at a time through LDS (fp32), then eight columns of a row per lane
  constexpr int LD = P::EPI_LD, LPR = P::WTN / 8, RPP = 64 / LPR;  // lanes per row, rows per pass
  float* const stg = reinterpret_cast<float*>(smem) + wave * (16 * LD);
  const int prow = lane / LPR, pcol = (lane % LPR) * 8;
  const int n = n0 + wn * P::WTN + pcol;
  const bool n_ok = n < g.N;
  const int row_lo = AL == 0 ? gt.lo : 0, row_hi = AL == 0 ? gt.hi : g.M, rows_all = AL == 0 ? g.n : g.M;
  float b8[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) b8[e] = 0.f;
  if (AL == 0 && g.bias != nullptr && n_ok && !rest && g.partial == nullptr) {
    const i32x4 v = *reinterpret_cast<const i32x4*>(static_cast<const T*>(g.bias) + (int64_t)gt.e * g.N + n);
    const T* t8 = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int e = 0; e < 8; ++e) b8[e] = (float)t8[e];
  }
  float* const part = g.partial == nullptr ? nullptr
                      : g.partial + (AL == 0 ? (int64_t)by * g.n : ((int64_t)by * g.experts + gt.e) * g.M) * g.N;
  T* const C = static_cast<T*>(g.C) + (AL == 0 ? 0 : (int64_t)gt.e * g.sc);
#pragma unroll
  for (int a = 0; a < TM; ++a) {
#pragma unroll
    for (int b = 0; b < TN; ++b) *reinterpret_cast<f32x4*>(stg + s16 * LD + 16 * b + 4 * grp) = acc[a][b];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
#pragma unroll
    for (int p = 0; p < (16 + RPP - 1) / RPP; ++p) {
      const int r = p * RPP + prow, m = m0 + wm * P::WTM + row_of(a, r);
      if (r >= 16) continue;
      f32x4 v0 = *reinterpret_cast<const f32x4*>(stg + r * LD + pcol);
      f32x4 v1 = *reinterpret_cast<const f32x4*>(stg + r * LD + pcol + 4);
      if (m >= row_lo && m < row_hi && m < rows_all && n_ok) {
        if (part != nullptr) {
          float* const dst = part + (int64_t)m * g.N + n;
          *reinterpret_cast<f32x4*>(dst) = v0;
          *reinterpret_cast<f32x4*>(dst + 4) = v1;
        } else {
          T o8[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) { o8[e] = from_f32<T>(v0[e] * g.alpha + b8[e]); o8[4 + e] = from_f32<T>(v1[e] * g.alpha + b8[4 + e]); }
          *reinterpret_cast<i32x4*>(C + (int64_t)m * g.ldc + n) = *reinterpret_cast<const i32x4*>(o8);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  }
}

template <typename T, bool F8, int AL, int BL, int BM, int BN, int WM, int NS, bool ROWS>
__global__ __launch_bounds__(256, 2) void grouped_mt_kernel(GroupedArgs g) {
  grouped_mt_body<T, F8, AL, BL, BM, BN, WM, NS, ROWS>(g, (int)blockIdx.x, (int)blockIdx.y);
}

// dA = X^T Z and dB = T^T dY in one launch: the first ax ga.splits workgroups take dA, the others dB.  One of them alone is a launch without the
// other's workgroups.
template <typename T, int R, int WM, int NS, int NS2>
__global__ __launch_bounds__(256, 2) void grouped_mt_grads_kernel(GroupedArgs ga, GroupedArgs gb, int ax, int bx) {
  const int id = (int)blockIdx.x, first = ax * ga.splits;
  if (id < first) grouped_mt_body<T, false, 1, 0, 128, R, WM, NS>(ga, id % ax, id / ax);
  else grouped_mt_body<T, false, 1, 0, R, 128, (R < 64 ? 1 : 2), NS2>(gb, (id - first) % bx, (id - first) / bx);
}

}  // namespace rl
