// Routing of tokens to experts (route.hpp): scores, choice and weights of a token's experts, and the order of the rows sorted by expert.
//
// The choice is decided on the logits themselves where nothing is added to the scores (they have the same order, and scores that round to the same number
// would lose it), otherwise on c = s + bias as 64 bits have it: in 32 bits the two closest of a row's candidates would change places once in some 10^5
// rows.  Groups are ranked by sums of c either way.  c is formed in 32 bits first, with a bound of its error, and only the rows in which two neighbours of
// the choice (or of the groups at its border) are closer than that go through the 64-bit exponentials.
#include "route.hpp"

#include <type_traits>

#include "gemm.hpp"
#include "lanes.hpp"

namespace rl {

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

RoutePlan route_plan(int64_t n, int64_t experts, int64_t top, int64_t groups) {
  RoutePlan p;
  const int64_t more = top < experts ? top + 1 : top;
  p.lanes = experts <= 8 && groups <= 8 ? 8 : 16;
  while (p.lanes < 64 && (p.lanes < more || p.lanes < groups || experts > 16 * p.lanes)) p.lanes *= 2;
  p.per = 1;
  while (p.per * p.lanes < experts) p.per *= 2;
  const int64_t side = 64 / p.lanes;
  // one after the other: its rows' keys (all rows' in 32 bits, or one's in 64), its choices, its counts
  int64_t room = experts * 4 > 256 ? experts * 4 : 256;
  if (groups > 1) {
    const int64_t all = (experts + 3 * p.lanes) * 4 * side, one = (experts + 3 * 64) * 8;
    room = all > room ? all : room;
    room = one > room ? one : room;
  }
  p.room = (unsigned)(ceil_div(room, 16) * 16);
  int most = p.per > 8 ? 8 : 16;  // (the kernel's launch bounds)
  while (most * p.room > (48u << 10)) most /= 2;
  if (n <= 4 * most * side) {
    p.waves = (int)ceil_div(n, side);
    if (p.waves > most) p.waves = most;
    if (p.waves < 4) p.waves = 4;
    p.groups = 1;
    p.each = (int)n;
    return p;
  }
  p.waves = 4;
  while (p.waves < most && ceil_div(n, p.waves * side) > kRouteGroups) p.waves *= 2;
  const int64_t at_once = p.waves * side;
  p.each = (int)(ceil_div(ceil_div(n, kRouteGroups), at_once) * at_once);
  p.groups = (int)ceil_div(n, p.each);
  return p;
}
unsigned route_lds(const RoutePlan& p, int64_t experts, bool wide) {
  return (unsigned)((experts * 4 + 15) / 16 * 16) + (wide ? (p.lanes * p.per > 64 ? p.lanes * p.per : 64) * 4 : 0) + p.room * (unsigned)p.waves;
}

namespace {

constexpr float kNone = -INFINITY;  // the score of an expert that cannot be chosen

template <typename V> __device__ __forceinline__ V ranked(V v) { return v != v ? (V)INFINITY : v + (V)0; }  // a NaN comes before everything; -0 is 0

// value of lane `lane` of a group of L (the same lane for the whole group)
template <int L, typename V>
__device__ __forceinline__ V from_lane(V v, int lane) {
  if constexpr (L == 64) {
    const int s = __builtin_amdgcn_readfirstlane(lane);
    if constexpr (sizeof(V) == 4) {
      return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), s));
    } else {
      const uint64_t u = __builtin_bit_cast(uint64_t, v);
      const uint64_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, s), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), s);
      return __builtin_bit_cast(V, lo | hi << 32);
    }
  } else {
    return __shfl(v, lane, L);
  }
}

// the same number, hidden from the compiler on a path that few calls take: what it gives for each of a lane's places is not worked out ahead of the loop
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+s"(v));
  return v;
}
__device__ __forceinline__ int lane_here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Lane `sub` of the L that share a row holds the experts sub K .. sub K + K - 1, so that the lowest lane has the lowest index.  `fast`: whole rows of
// pieces of 16 bytes, or of K elements, at aligned addresses.
template <typename T, int K>
__device__ __forceinline__ void load_row(const T* row, int sub, int experts, bool there, bool fast, float (&l)[K]) {
  constexpr int B = K * (int)sizeof(T);  // bytes a lane takes
  if constexpr (K > 1 && (B == 4 || B == 8 || B % 16 == 0)) {
    if (fast) {
      constexpr int W = B < 16 ? B / 4 : 4;
      typedef __attribute__((__vector_size__(W * sizeof(int)))) int vec;
      __attribute__((aligned(16))) T t[K];
#pragma unroll
      for (int q = 0; q < B / (4 * W); ++q) {
        vec v = {};
        if (there && sub * K < experts) v = reinterpret_cast<const vec*>(row + sub * K)[q];
        reinterpret_cast<vec*>(t)[q] = v;
      }
#pragma unroll
      for (int k = 0; k < K; ++k) l[k] = there && sub * K < experts ? (float)t[k] : kNone;
      return;
    }
  }
  const int count = here(experts), first = lane_here(sub * K);
#pragma unroll
  for (int k = 0; k < K; ++k) l[k] = there && first + k < count ? (float)row[first + k] : kNone;
}
// (decided on the host: experts a multiple of K, and rows that start where the pieces do)
bool fast_rows(const void* p, int64_t ld, int64_t experts, int K, size_t esz) {
  const size_t b = (size_t)K * esz < 16 ? (size_t)K * esz : 16;
  return experts % K == 0 && reinterpret_cast<uintptr_t>(p) % b == 0 && (size_t)ld * esz % b == 0;
}

// exp by the exponential of 2: off by a unit (2 u) and, through its argument, by 1.5 u |x|
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// exp in 64 bits to 2^-31 of itself, which is what a weight of 32 bits needs: x = n ln 2 + r, |r| <= 0.3466, and the series of exp(r) to r^8 (the rest is
// below r^9 / 9! = 2^-32.2).  0 far below, infinity far above.
__device__ __forceinline__ double exp64_near(double x) {  // (x within 2000 of 0)
  const double n = __builtin_rint(x * 1.4426950408889634074), r = __builtin_fma(n, -0.69314718055994530942, x);
  double p = 1.0 / 40320;
  p = __builtin_fma(p, r, 1.0 / 5040);
  p = __builtin_fma(p, r, 1.0 / 720);
  p = __builtin_fma(p, r, 1.0 / 120);
  p = __builtin_fma(p, r, 1.0 / 24);
  p = __builtin_fma(p, r, 1.0 / 6);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return ldexp(p, (int)n);
}
__device__ __forceinline__ double exp64(double x) { return exp64_near(x < -2000.0 ? -2000.0 : (x > 2000.0 ? 2000.0 : x)); }
// exp(l - base) of l <= base
__device__ __forceinline__ double row_term(float l, float base) { return exp64_near(l - base < -1900.f ? -1900.0 : (double)l - (double)base); }

// row maximum (not counting NaN; 0 where nothing is left) of a row's logits, l = -inf where there is none
template <int L, int K>
__device__ __forceinline__ float row_base(const float (&l)[K]) {
  float m = kNone;
#pragma unroll
  for (int k = 0; k < K; ++k) m = l[k] > m ? l[k] : m;
  m = lanes_max<L>(m);
  return m == kNone ? 0.f : m;
}
// Sum of exp(l - base).  `exact`: the weights are quotients by it, its terms have 2^-31 (us, with them / with those of 32 bits: 1999 x 120 f16 12.2 / 12.0,
// 16384 x 256 f32 20.5 / 19.4; the error of a weight 2.5 / 3.3 10^-8).  Otherwise it serves the ranks of c alone: a term is off by under 3 u of itself, with
// what its argument's product loses put back to first order, and by 1.23 u |l - base| for the difference's rounding and that of log2 e: weighted by
// themselves the terms are off by at most (1.23 ln E + 3) u of the sum.  In 64 bits the additions add nothing to either.
template <int L, int K>
__device__ __forceinline__ double row_sum(const float (&l)[K], float base, bool exact) {
  double s = 0.0;
  if (exact) {
#pragma unroll
    for (int k = 0; k < K; ++k) s += row_term(l[k], base);
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      constexpr float log2e = 1.44269504088896341f;
      const float x = l[k] - base, a = x * log2e, e = __builtin_amdgcn_exp2f(a);
      s += (double)(e != 0.f ? __builtin_fmaf(e, 0.693147181f * __builtin_fmaf(x, log2e, -a), e) : e);  // (x = -inf has no rest)
    }
  }
  return lanes_sum<L>(s);
}

// How far c = s + bias in 32 bits may be off, u = 2^-24: `one` for the score, u |c| for the sum and 30 u |c| for its key's lower four bits.  (By its own
// magnitude: an expert that a bias of -10^9 takes out says nothing about the others.)  As a number, so that infinities stay apart from the rest.
__device__ __forceinline__ float off_by(float one, float c) {
  const float off = __builtin_fmaf(0x1p-19f, fabsf(c), one);
  return off < 3.4028234e38f ? off : 3.4028234e38f;
}

// Which groups are kept, by the sum of their best `group_top` (1 or 2) keys: the keys outside them become -inf.  Where q = 1, 2, .. 16 lanes hold a group
// each looks through its own keys; otherwise a row's keys go through LDS, q lanes to a group whatever its size (groups lie an odd number of q words apart
// there: banks).  BOUND: returns whether what the keys are off by (one: a score, see off_by) can change nothing about it: every sum that is kept is above
// every other by more than both are off by.  All lanes of the wave take part.
struct Groups {
  int size, q, pitch = 0, inverse = 0;
  bool own;
  __device__ __forceinline__ Groups(const RouteDesc& g, int lanes, int per) {
    size = g.experts / g.groups;
    q = size / per;
    own = size % per == 0 && (q & (q - 1)) == 0 && q <= 16;
    if (own) return;
    q = 1;
    while (2 * q * g.groups <= lanes && q < 16) q *= 2;
    pitch = (size + 2 * q - 1) / (2 * q) * (2 * q) + q;
    inverse = ((1 << 21) + size - 1) / size;
  }
  // e / size: e <= 1023
  __device__ __forceinline__ static int of(int e, int inverse) { return (int)(__umul24((unsigned)e, (unsigned)inverse) >> 21); }
};
template <int L, int K, bool BOUND, typename V>
__device__ __forceinline__ bool keep_groups(const RouteDesc& g, const Groups& at, V (&key)[K], V* scratch, int sub, float one = 0.f) {
  const int q = at.q, group = sub / q;
  V a = (V)kNone, b = (V)kNone;  // best and second best
  auto look = [&](V v) {
    const V low = v > a ? a : v;
    a = v > a ? v : a;
    b = low > b ? low : b;
  };
  if (at.own) {
#pragma unroll
    for (int k = 0; k < K; ++k) look(key[k]);
  } else {
    const int inverse = here(at.inverse), experts = here(g.experts), first = lane_here(sub * K);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int e = first + k;
      if (e < experts) scratch[e + at.of(e, inverse) * (at.pitch - at.size)] = key[k];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (group < g.groups)
      for (int i = sub % q; i < at.size; i += q) look(scratch[group * at.pitch + i]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();  // (the scratch is the next row's)
  }
  auto merge = [&](V a2, V b2) {
    const V low = a > a2 ? a2 : a, high = b > b2 ? b : b2;
    a = a > a2 ? a : a2;
    b = low > high ? low : high;
  };
  if (q > 1) { const V a2 = across<1>(a), b2 = across<1>(b); merge(a2, b2); }
  if (q > 2) { const V a2 = across<2>(a), b2 = across<2>(b); merge(a2, b2); }
  if (q > 4) { const V a2 = across<4>(a), b2 = across<4>(b); merge(a2, b2); }
  if (q > 8) { const V a2 = across<8>(a), b2 = across<8>(b); merge(a2, b2); }
  const bool two = g.group_top > 1 && b != (V)kNone;
  const V rank = two ? a + b : a;
  int before = 0;
  for (int o = 0; o < g.groups; ++o) {
    const V r = from_lane<L>(rank, o * q);
    before += r > rank || (r == rank && o < group) ? 1 : 0;
  }
  const bool real = group < g.groups;
  auto mine = [&](bool is) {
    uint64_t m = __ballot(is);
    if constexpr (L < 64) m = (m >> (threadIdx.x & 63 & ~(L - 1))) & ((1ull << L) - 1);
    return m;
  };
  const uint64_t kept = mine(real && before < g.kept);
  bool sure = true;
  if constexpr (BOUND) {
    // (a group that has nothing to choose is no neighbour)
    const float off = off_by(one, a) + (two ? off_by(one, b) : 0.f);
    const bool counts = real && rank != kNone;
    const float low = -lanes_max<L>(counts && before < g.kept ? off - rank : kNone), high = lanes_max<L>(counts && before >= g.kept ? rank + off : kNone);
    sure = low > high;
  }
  if (at.own) {
    const bool out = ((kept >> (group * q & 63)) & 1) == 0;
#pragma unroll
    for (int k = 0; k < K; ++k) key[k] = out ? (V)kNone : key[k];
  } else {
    const int inverse = here(at.inverse), first = lane_here(sub * K);
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (((kept >> (at.of(first + k, inverse) * q & 63)) & 1) == 0) key[k] = (V)kNone;  // (behind the last expert: -inf already)
  }
  return sure;
}

// Keys of one word that no two experts of a lane (K <= 16) share: bits whose order as whole numbers is that of the values (no NaN, no -0), the upper 28 of
// them, then the place, the lower first.  Up to kLeast: -infinity, what cannot be chosen.
constexpr uint32_t kLeast = 0x007FFFFFu;
__device__ __forceinline__ uint32_t lane_key(float v, int k) {
  const uint32_t b = __float_as_uint(v);
  return ((b ^ ((uint32_t)((int)b >> 31) | 0x80000000u)) & ~15u) | (uint32_t)(15 - k);
}
// Of 16-bit logits the whole value and the expert fit: no two of a row are equal.
template <typename T>
__device__ __forceinline__ uint32_t row_key(float v, int e) {
  const uint32_t b = (uint32_t)__builtin_bit_cast(uint16_t, (T)v) << 16;
  return v == kNone ? 0u : ((b ^ ((uint32_t)((int)b >> 31) | 0x80000000u)) & 0xFFFF0000u) | (uint32_t)(1023 - e);
}

// a lane's K different keys in falling order (Batcher's odd-even merging network)
template <int K>
__device__ __forceinline__ void sort_keys(uint32_t (&key)[K]) {
#pragma unroll
  for (int p = 1; p < K; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < K; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < K && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
            const uint32_t a = key[i + j], b = key[i + j + k];
            key[i + j] = a > b ? a : b;
            key[i + j + k] = a > b ? b : a;
          }
}

// The `top` largest keys of a row in falling order, equal ones by index: lane j of the row ends up with choice j (-1: nothing left) and its key.  Each
// lane's keys are sorted first, so that a step is a maximum over the lanes' heads and a shift in the lane that had it.  UNIQUE: row_key, which names the
// expert.  Otherwise lane_key: of the lanes whose heads have the largest value the lowest has the lowest index; it leaves its expert in `list` (64 ints of
// LDS a wave).
template <int L, int K, bool UNIQUE>
__device__ __forceinline__ int choose(int top, uint32_t (&key)[K], int sub, int lane, int* list, uint32_t* mine_key) {
  uint32_t mk = 0u;
  sort_keys<K>(key);
  for (int j = 0; j < top; ++j) {
    bool pop;
    uint32_t m;
    if constexpr (UNIQUE) {
      m = lanes_max<L>(key[0]);
      pop = key[0] == m;
    } else {
      const uint32_t head = key[0] | 15u;
      m = lanes_max<L>(head);
      const uint64_t hit = __ballot(head == m);
      if constexpr (L < 64) pop = sub == __builtin_ctz((uint32_t)(hit >> (lane & ~(L - 1))) & (L < 32 ? (1u << (L & 31)) - 1u : ~0u));
      else pop = sub == __builtin_ctzll(hit);
      if (pop) list[(lane & ~(L - 1)) + j] = sub * K + 15 - (int)(key[0] & 15u);
    }
    mk = sub == j ? m : mk;
    const uint32_t shift = pop ? ~0u : 0u;  // (bit selects: as a condition it becomes a branch around 2 K moves)
    auto pull = [&](auto width) {
      constexpr int W = decltype(width)::value < K ? decltype(width)::value : K;
#pragma unroll
      for (int k = 0; k < W; ++k) key[k] = (shift & (k + 1 < K ? key[k + 1 < K ? k + 1 : 0] : 0u)) | (~shift & key[k]);
    };
    // Of a lane's keys no more are asked for than there are steps left.  (us, with it / without: 16384 x 256 top 8 bf16 16.5 / 17.9, 8192 x 120 top 6 f16
    // 15.7 / 15.5; with lane_key, whose steps wait longer than they work, 16384 x 256 27.2 / 26.9, 8192 x 512 top 10 27.9 / 26.9.)
    const int left = UNIQUE && K > 8 ? top - 1 - j : K;
    if (left > 8) pull(std::integral_constant<int, 16>());
    else if (left > 4) pull(std::integral_constant<int, 8>());
    else pull(std::integral_constant<int, 4>());
  }
  *mine_key = mk;
  if constexpr (UNIQUE) return mk != 0u ? 1023 - (int)(mk & 1023u) : -1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int mine = mk > kLeast ? list[lane] : -1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();  // (the list is the next rows')
  return mine;
}
// the same on 64-bit keys, -inf: cannot be chosen
template <int L, int K>
__device__ __forceinline__ int choose64(int top, double (&key)[K], int sub, int lane) {
  int mine = -1;
  for (int j = 0; j < top; ++j) {
    double head = key[0];
    int place = 0;
#pragma unroll
    for (int k = 1; k < K; ++k) {
      place = key[k] > head ? k : place;
      head = key[k] > head ? key[k] : head;
    }
    const double m = lanes_max<L>(head);
    uint64_t hit = __ballot(head == m);
    if constexpr (L < 64) hit = (hit >> (lane & ~(L - 1))) & ((1ull << L) - 1);
    const int who = __builtin_ctzll(hit);
    const int expert = from_lane<L>(sub * K + place, who);
    if (sub == j) mine = m != (double)kNone ? expert : -1;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (sub == who && k == place) key[k] = (double)kNone;
  }
  return mine;
}
// c of a row in 64 bits, -inf for what cannot be chosen
template <int L, int K>
__device__ __forceinline__ void scores64(const RouteDesc& g, const float (&l)[K], const float* bias, float base, double (&key)[K]) {
  if (!g.sigmoid) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      key[k] = exp((double)l[k] - (double)base);
      s += key[k];
    }
    s = lanes_sum<L>(s);
#pragma unroll
    for (int k = 0; k < K; ++k) key[k] = key[k] / s;
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) key[k] = 1.0 / (1.0 + exp(-(double)l[k]));
  }
#pragma unroll
  for (int k = 0; k < K; ++k) key[k] = l[k] == kNone ? (double)kNone : ranked(key[k] + (double)bias[k]);  // (behind the last expert: -inf)
}

// adds where an expert's rows start, by their counts, to starts; all of them in *total, where an expert's end in `ends` (or nullptr).  All threads.
__device__ __forceinline__ void scan_counts(const int* counts, int* starts, int experts, int* total, int32_t* ends) {
  if (threadIdx.x < 64) {
    const int each = (experts + 63) / 64, lo = (int)threadIdx.x * each;
    int sum = 0;
    for (int k = lo; k < lo + each && k < experts; ++k) sum += counts[k];
    int run = sum;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int v = __shfl_up(run, s);
      if ((int)threadIdx.x >= s) run += v;
    }
    if (threadIdx.x == 63) *total = run;
    run -= sum;
    for (int k = lo; k < lo + each && k < experts; ++k) {
      starts[k] += run;
      run += counts[k];
      if (ends != nullptr) ends[k] = run;
    }
  }
  __syncthreads();
}

// Rows of the entries [lo, hi) of `expert` (an expert's in their order, from starts[e] on): every wave counts a run of them, the counts become
// the waves' first rows, and each wave walks its run, 64 entries at a time, an entry's place among the equal ones before it by ballots over the bits.
// prepare(): the counting, which needs no starts (mine: [waves][experts] ints); finish() after it and a barrier.
struct Placing {
  int64_t first, last;
  int wave, lane;
  int32_t head;  // the wave's first 64 experts
  __device__ __forceinline__ void run(int64_t lo, int64_t hi) {
    lane = threadIdx.x & 63;
    wave = threadIdx.x >> 6;
    const int waves = blockDim.x >> 6;
    const int64_t per = ((hi - lo + waves - 1) / waves + 63) / 64 * 64;
    first = lo + wave * per;
    last = first + per < hi ? first + per : hi;
  }
  __device__ __forceinline__ void prefetch(const RouteDesc& g) { head = first + lane < last ? g.expert[first + lane] : -1; }
  __device__ __forceinline__ int32_t at(const RouteDesc& g, int64_t i0) const { return i0 == first ? head : (i0 + lane < last ? g.expert[i0 + lane] : -1); }
  __device__ __forceinline__ void prepare(const RouteDesc& g, int* mine) const {
    for (int k = threadIdx.x; k < (int)(blockDim.x >> 6) * g.experts; k += blockDim.x) mine[k] = 0;
    __syncthreads();
    for (int64_t i0 = first; i0 < last; i0 += 64) {
      const int e = at(g, i0);
      if (e >= 0) atomicAdd(&mine[wave * g.experts + e], 1);
    }
  }
  __device__ __forceinline__ void finish(const RouteDesc& g, const int* starts, int* mine) const {
    for (int e = threadIdx.x; e < g.experts; e += blockDim.x) {
      int run = starts[e];
      for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
        const int c = mine[w * g.experts + e];
        mine[w * g.experts + e] = run;
        run += c;
      }
    }
    __syncthreads();
    int* const count = mine + wave * g.experts;
    const int bits = 32 - __builtin_clz(g.experts);
    for (int64_t i0 = first; i0 < last; i0 += 64) {
      const int64_t i = i0 + lane;
      const int e = at(g, i0);
      uint64_t same = __ballot(e >= 0);
      for (int b = 0; b < bits; ++b) {
        const bool bit = (e >> b) & 1;
        const uint64_t set = __ballot(bit);
        same &= bit ? set : ~set;
      }
      const int before = __popcll(same & ((1ull << lane) - 1));
      if (e >= 0) {
        const int p = count[e] + before;
        g.place[i] = p;
        g.source[p] = (int32_t)i;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (before == 0) count[e] = p + __popcll(same);
      } else if (i < last) {
        g.place[i] = -1;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// a workgroup's count of an expert's rows is at most its tokens (a token's experts are different ones)
inline __host__ __device__ int count_bytes(int each) { return each < 256 ? 1 : 2; }

// Workgroup b takes the tokens [b each, (b + 1) each), L lanes a token with K experts each, 64 / L tokens side by side in a wave: their experts and weights,
// and how many rows every expert gets (counts [b][experts] in the workspace).  A single workgroup places them too.
// Bound by its instructions and, with one round of waves, by their latency (16384 x 256 in 32 bits, biased sigmoid scores, 8 groups, top 8: 16 MB, 3 us;
// 1400 vector instructions a wave of four tokens, 10 us of them; 18 us): a maximum over 16 lanes serves four tokens at once, where one over 64 serves one
// (38 us).  The scores in 64 bits for every row took 45.
template <typename T, int L, int K, bool WIDE>
__global__ __launch_bounds__(K > 8 ? 512 : 1024, L * K > 256 ? 2 : 4) void route_choose_kernel(RouteDesc g, int each, int fast, int room, void* counts, int single) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  // counts of the workgroup's experts [experts]; the bias [L K, at least 64, zeros behind the last]; then `room` bytes a wave: a list of its
  // choices, its rows' keys (groups), or counts [experts] (Placing)
  int* const count = reinterpret_cast<int*>(lds);
  float* const bias = reinterpret_cast<float*>(lds + (g.experts * 4 + 15) / 16 * 16);
  char* const rest = reinterpret_cast<char*>(bias + (WIDE ? (L * K > 64 ? L * K : 64) : 0));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, sub = lane % L;
  constexpr int SIDE = 64 / L;  // tokens side by side in a wave
  char* const keys = rest + (size_t)wave * room;
  int* const list = reinterpret_cast<int*>(keys);
  for (int k = threadIdx.x; k < g.experts; k += blockDim.x) count[k] = 0;
  if constexpr (WIDE) {
    for (int k = threadIdx.x; k < (L * K > 64 ? L * K : 64); k += blockDim.x) bias[k] = g.bias != nullptr && k < g.experts ? g.bias[k] : 0.f;
  }
  __syncthreads();
  const Groups at(g, L, K);
  const int64_t first = (int64_t)blockIdx.x * each, last = first + each < g.n ? first + each : g.n;
  for (int64_t t0 = first + wave * SIDE; t0 < last; t0 += waves * SIDE) {
    const int64_t t = t0 + lane / L;
    const bool there = t < last;
    const T* const row = static_cast<const T*>(g.logits) + (there ? t : first) * g.ld;
    float l[K];
    load_row<T, K>(row, sub, g.experts, there, fast != 0, l);
    float base = 0.f;
    double sum = 1.0;
    if (!g.sigmoid && (!g.renorm || WIDE)) {
      base = row_base<L, K>(l);
      sum = row_sum<L, K>(l, base, !g.renorm);
    }
    constexpr bool UNIQUE = !WIDE && sizeof(T) == 2;
    const bool added = WIDE && g.bias != nullptr;  // chosen by c, otherwise by the logits of the groups that are left
    // one more than asked for, where there is one and a lane for it: the last of the choice has a neighbour too
    const int more = UNIQUE || g.top == g.experts ? g.top : g.top + 1;
    const float inverse = sum == 0.0 ? 0.f : 1.f / (float)sum;
    float one = 0.f;
    bool close = false;
    uint32_t key[K], mine_key;
    {
      float c[K], odd = 0.f;
      if constexpr (WIDE) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const float s = (g.sigmoid ? __builtin_amdgcn_rcpf(1.f + fast_exp(-l[k])) : fast_exp(l[k] - base) * inverse) + bias[sub * K + k];
          c[k] = l[k] == kNone ? kNone : s;
          odd += s;
        }
        close = odd != odd;  // (a NaN, or infinite biases: 64 bits sort them out)
        // How far a score may be off.  sigmoid: exp is off by 2 u and, through its argument, 1.5 u |l|, of which s (1 - s) keeps under u; 1 + e and the
        // reciprocal by 3 u s: under 2^-21.  softmax: exp by 2 u and 2.5 u |l - max|, of which s keeps under u max s; the sum by (1.23 ln 1024 + 3) u and
        // its rounding; the quotient and the product by 2 u: under 2^-18 max s, max s = 1 / sum.
        one = g.sigmoid ? 0x1p-21f : 0x1p-18f * inverse;
      } else {
#pragma unroll
        for (int k = 0; k < K; ++k) c[k] = ranked(l[k]);
      }
      if (g.groups > 1) {
        if (!keep_groups<L, K, WIDE>(g, at, c, reinterpret_cast<float*>(keys) + (lane / L) * (g.groups * at.pitch), sub, one)) close = true;
      }
      if constexpr (WIDE) {
        if (!added) {  // (read again: held beside c, 16 of them do not fit the registers)
          float again[K];
          asm volatile("" ::: "memory");
          load_row<T, K>(row, sub, g.experts, there, fast != 0, again);
#pragma unroll
          for (int k = 0; k < K; ++k) c[k] = c[k] == kNone ? kNone : ranked(again[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if constexpr (UNIQUE) key[k] = row_key<T>(c[k], sub * K + k);
        else key[k] = lane_key(c[k], k);
      }
    }
    int expert = choose<L, K, UNIQUE>(more <= L ? more : L, key, sub, lane, list, &mine_key);
    float logit = expert >= 0 ? (float)row[expert] : 0.f;
    if constexpr (!UNIQUE) {
      const float mine_b = added && expert >= 0 ? bias[expert] : 0.f;
      const float v = added ? ranked((g.sigmoid ? __builtin_amdgcn_rcpf(1.f + fast_exp(-logit)) : fast_exp(logit - base) * inverse) + mine_b) : 0.f;
      const int from = (lane & ~(L - 1)) | (sub + 1 < L ? sub + 1 : sub);
      const float next = __shfl(v, from), next_l = __shfl(logit, from), next_b = __shfl(mine_b, from);
      const uint32_t next_key = (uint32_t)__shfl((int)mine_key, from);
      if (sub + 1 < more && sub + 1 < L && expert >= 0 && next_key > kLeast) {
        const bool apart = added ? v - next > off_by(one, v) + off_by(one, next) : mine_key >> 4 != next_key >> 4;
        // (equal logits with equal biases are equal in any precision; behind the last pair others may stand that are not)
        if (!apart && !(sub + 2 < more && logit == next_l && mine_b == next_b)) close = true;
      }
      if (more > L) close = true;
      // Rows that 32 bits do not decide: the whole wave takes one after the other, so that its 64-bit keys are few a lane.  (All rows of 16384 x 256 of one
      // value, zero bias: both launches take 41 us, of random ones 24.)
      if (sub >= g.top) expert = -1;
      const uint64_t undecided = __ballot(close && there);
      if (undecided != 0) {
        constexpr int FEW = L * K > 64 ? L * K / 64 : 1;
        const Groups at64(g, 64, FEW);
        for (int r = 0; r < SIDE; ++r) {
          if (L < 64 && ((undecided >> (r * L)) & ((1ull << (L & 63)) - 1)) == 0) continue;
          float l64[FEW];
          double key64[FEW];
          load_row<T, FEW>(static_cast<const T*>(g.logits) + (t0 + r) * g.ld, lane, g.experts, true, fast != 0, l64);
          if constexpr (WIDE) {
            scores64<64, FEW>(g, l64, bias + lane * FEW, from_lane<64>(base, r * L), key64);
          } else {
#pragma unroll
            for (int k = 0; k < FEW; ++k) key64[k] = (double)ranked(l64[k]);
          }
          if (g.groups > 1) keep_groups<64, FEW, false>(g, at64, key64, reinterpret_cast<double*>(keys), lane);
          if constexpr (WIDE) {
            if (!added) {
#pragma unroll
              for (int k = 0; k < FEW; ++k) key64[k] = key64[k] == (double)kNone ? (double)kNone : (double)ranked(l64[k]);
            }
          }
          const int found = __shfl(choose64<64, FEW>(g.top, key64, lane, lane), sub);
          if (lane / L == r) expert = sub < g.top ? found : -1;
        }
        logit = expert >= 0 ? (float)row[expert] : 0.f;
      }
    }
    // Weights: lane j holds choice j.  In 64 bits, rounded once: 2.8 10^-8 of their norm, where a chain of 32-bit operations left 8 10^-8 and took 1 us of
    // 35 less (16384 x 256, with its gradient).
    const bool chosen = sub < g.top && expert >= 0;
    double w = 0.0;
    if (g.renorm) {
      // scores over the largest of the chosen ones: their sum is at least 1 (sigmoid: 1/2), however small they are
      const float a = g.sigmoid ? (logit < 0.f ? logit : (logit != logit ? logit : 0.f)) : logit;
      const float m = lanes_max<L>(chosen ? ranked(a) : kNone);
      if (chosen) {
        w = exp64((double)a - (double)m);
        if (g.sigmoid) w = w / (1.0 + exp64(-fabs((double)logit)));
      }
      const double s = lanes_sum<L>(w);
      if (chosen) w = w / s;
      if (!g.sigmoid && sum != sum) w = sum;  // a NaN in the row
    } else if (chosen) {
      w = g.sigmoid ? 1.0 / (1.0 + exp64(-(double)logit)) : exp64((double)logit - (double)base) / sum;
    }
    if (there && sub < g.top) {
      g.expert[t * g.top + sub] = expert;
      g.weight[t * g.top + sub] = chosen ? (float)((double)g.scale * w) : 0.f;
      if (expert >= 0) atomicAdd(&count[expert], 1);
    }
  }
  __syncthreads();
  if (!single) {
    const bool bytes = count_bytes(each) == 1;
    for (int k = threadIdx.x; k < g.experts; k += blockDim.x) {
      const int64_t at = (int64_t)blockIdx.x * g.experts + k;
      if (bytes) static_cast<uint8_t*>(counts)[at] = (uint8_t)count[k];
      else static_cast<uint16_t*>(counts)[at] = (uint16_t)count[k];
    }
    return;
  }
  __shared__ int total;
  int* const mine = reinterpret_cast<int*>(rest);
  for (int k = threadIdx.x; k < g.experts; k += blockDim.x) {
    mine[k] = count[k];
    count[k] = 0;
  }
  __syncthreads();
  scan_counts(mine, count, g.experts, &total, g.ends);
  for (int64_t p = total + threadIdx.x; p < g.n * g.top; p += blockDim.x) g.source[p] = -1;
  Placing w;
  w.run(0, g.n * g.top);
  w.prefetch(g);
  w.prepare(g, mine);
  __syncthreads();
  w.finish(g, count, mine);
}

// Workgroup b places the rows of the tokens [b each, (b + 1) each), those of `part` workgroups of the choice, behind those of the tokens before: it adds up
// everybody's counts ([groups][experts] of C), W experts a thread and the groups dealt out to the threads that are left.  Reading the counts is what grows
// with both numbers: 512 groups of 256 experts in bytes, read by 256 workgroups, take 7.6 us in all, in 16 bits by 512 17.6; a thread an expert, one group
// after the other, took 15 for 256.
template <typename C>
__global__ __launch_bounds__(512) void route_place_kernel(RouteDesc g, int each, const C* counts, int groups, int part) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ int total;
  int* const starts = reinterpret_cast<int*>(lds);  // [experts]
  int* const all = starts + g.experts;              // [experts]
  int* const mine = all + g.experts;                // [waves][experts]
  const int64_t m = g.n * g.top;
  Placing w;
  const int64_t lo = (int64_t)blockIdx.x * each * g.top, hi = lo + (int64_t)each * g.top;
  w.run(lo, hi < m ? hi : m);
  w.prefetch(g);
  for (int e = threadIdx.x; e < 2 * g.experts; e += blockDim.x) starts[e] = 0;
  w.prepare(g, mine);  // (a barrier inside)
  const int own = (int)blockIdx.x * part;
  auto add = [&](auto width) {
    constexpr int W = decltype(width)::value;
    typedef __attribute__((__vector_size__(W * sizeof(C)))) C vec;
    const int columns = g.experts / W, slices = (int)blockDim.x > columns ? (int)blockDim.x / columns : 1;
    for (int c = (int)threadIdx.x; c < columns * slices; c += (int)blockDim.x) {
      int sum[W], before[W];
#pragma unroll
      for (int k = 0; k < W; ++k) sum[k] = before[k] = 0;
      const int column = c % columns, slice = c / columns;
      const C* const from = counts + column * W;
      if constexpr (W == 4 && sizeof(C) == 1) {
        // two bytes a word at a time: 256 of them do not pass 16 bits
        for (int b0 = slice; b0 < groups; b0 += 256 * slices) {
          uint32_t even = 0, odd = 0, even_b = 0, odd_b = 0;
          const int end = b0 + 256 * slices < groups ? b0 + 256 * slices : groups;
#pragma unroll 16
          for (int b = b0; b < end; b += slices) {
            const uint32_t v = *reinterpret_cast<const uint32_t*>(from + (int64_t)b * g.experts), u = b < own ? v : 0u;
            even += v & 0x00FF00FFu;
            odd += (v >> 8) & 0x00FF00FFu;
            even_b += u & 0x00FF00FFu;
            odd_b += (u >> 8) & 0x00FF00FFu;
          }
          sum[0] += even & 0xFFFF; sum[1] += odd & 0xFFFF; sum[2] += even >> 16; sum[3] += odd >> 16;
          before[0] += even_b & 0xFFFF; before[1] += odd_b & 0xFFFF; before[2] += even_b >> 16; before[3] += odd_b >> 16;
        }
      } else {
#pragma unroll 8
        for (int b = slice; b < groups; b += slices) {
          const vec v = *reinterpret_cast<const vec*>(from + (int64_t)b * g.experts);
#pragma unroll
          for (int k = 0; k < W; ++k) {
            sum[k] += v[k];
            before[k] += b < own ? v[k] : 0;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < W; ++k) {
        atomicAdd(&all[column * W + k], sum[k]);
        if (before[k] != 0) atomicAdd(&starts[column * W + k], before[k]);
      }
    }
  };
  if (g.experts % 4 == 0) {
    add(std::integral_constant<int, 4>());
  } else {
    add(std::integral_constant<int, 1>());
  }
  __syncthreads();
  scan_counts(all, starts, g.experts, &total, blockIdx.x == 0 ? g.ends : nullptr);
  for (int64_t p = total + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; p < m; p += (int64_t)gridDim.x * blockDim.x) g.source[p] = -1;
  w.finish(g, starts, mine);
}

inline __host__ __device__ bool route_wide(const RouteDesc& g) { return g.bias != nullptr || (g.groups > 1 && g.group_top > 1); }

// Gradient of the logits, L lanes a token; p, q as in the forward:
//     softmax:                dl_e = p_e (D_e - sum_j D_j p_j)               D = scale dw, zero off the chosen experts
//     softmax over chosen:    dl_j = q_j (D_j - sum_k D_k q_k)               and zero elsewhere
//     sigmoid:                dl_j = s_j (1 - s_j) D_j;   over the chosen: q_j (1 - s_j) (D_j - sum_k D_k q_k)
// A row is put together in LDS, most of it zeros, and leaves as whole pieces (each lane's own K elements compared with every choice, and stored K apart:
// 12 us for 16384 x 256 top 8 in 32 bits, 7.6 so, 17 MB written).
template <typename T, int L, int K>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteDesc g, int fast, int fast_out) {
  constexpr int SIDE = 64 / L;
  __shared__ __attribute__((aligned(16))) float rows[4][SIDE * L * K];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % L;
  const int64_t t0 = ((int64_t)blockIdx.x * 4 + wave) * SIDE, t = t0 + lane / L;
  const bool there = t < g.n;
  const T* const row = static_cast<const T*>(g.logits) + (there ? t : 0) * g.ld;
  float* const mine = &rows[wave][(lane / L) * (L * K)];
  int expert = -1;
  float logit = 0.f;
  double d = 0.0;  // D: the product's 48 bits
  if (there && sub < g.top) {
    expert = g.expert[t * g.top + sub];
    if (expert >= g.experts) expert = -1;
    if (expert >= 0) {
      d = (double)g.scale * (double)g.dweight[t * g.top + sub];
      logit = (float)row[expert];
    }
  }
  const bool chosen = expert >= 0;
  float out[K], base = 0.f, v = 0.f;
  double sum = 1.0;
#pragma unroll
  for (int k = 0; k < K; ++k) out[k] = 0.f;
  if (!g.sigmoid && (!g.renorm || route_wide(g))) {  // (with a bias a NaN need not be among the chosen: as in the forward)
    float l[K];
    load_row<T, K>(row, sub, g.experts, there, fast != 0, l);
    base = row_base<L, K>(l);
    if (!g.renorm) {
      double e[K], s = 0.0;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        e[k] = row_term(l[k], base);
        s += e[k];
      }
      sum = lanes_sum<L>(s);
      const double p = exp64((double)logit - (double)base) / sum, mean = lanes_sum<L>(chosen ? d * p : 0.0);
      v = (float)(p * (d - mean));
      const double off_chosen = sum == 0.0 ? 0.0 : -mean / sum;
#pragma unroll
      for (int k = 0; k < K; ++k) out[k] = sum == 0.0 ? 0.f : (float)(e[k] * off_chosen);
    } else {
      sum = row_sum<L, K>(l, base, false);
    }
  }
  if (g.renorm || g.sigmoid) {  // (the chosen alone: in 64 bits, as the weights)
    const double far = g.sigmoid ? exp64(-fabs((double)logit)) : 0.0;
    double x = 0.0;
    if (g.renorm) {
      const float a = g.sigmoid ? (logit < 0.f ? logit : (logit != logit ? logit : 0.f)) : logit;
      const float m = lanes_max<L>(chosen ? ranked(a) : kNone);
      double q = 0.0;
      if (chosen) q = exp64((double)a - (double)m) / (1.0 + far);
      const double all = lanes_sum<L>(q);
      if (chosen) q = q / all;
      const double mean = lanes_sum<L>(chosen ? d * q : 0.0);
      if (chosen) x = q * (d - mean);
      if (sum != sum) x = sum;
    } else if (chosen) {
      x = (logit < 0.f ? far : 1.0) / (1.0 + far) * d;
    }
    // 1 - s
    if (g.sigmoid && chosen) x = x * ((logit < 0.f ? 1.0 : far) / (1.0 + far));
    v = (float)x;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) mine[sub * K + k] = out[k];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (chosen) mine[expert] = v;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  constexpr int E = Piece<T>::N;
  for (int r = 0; r < SIDE && t0 + r < g.n; ++r) {
    const float* const from = &rows[wave][r * (L * K)];
    T* const to = static_cast<T*>(g.dlogits) + (t0 + r) * g.lddl;
    if (fast_out) {
      for (int c = lane * E; c < g.experts; c += 64 * E) {
        float f[E];
#pragma unroll
        for (int k = 0; k < E; ++k) f[k] = from[c + k];
        Piece<T>::of(f).store(to + c);
      }
    } else {
      for (int c = lane; c < g.experts; c += 64) to[c] = (T)from[c];
    }
  }
}

template <int L_, int K_> struct Split { static constexpr int L = L_, K = K_; };
template <typename F>
hipError_t by_lanes(int lanes, int per, F&& f) {
  if (lanes == 8) return f(Split<8, 1>());
  if (lanes == 16) {
    if (per == 1) return f(Split<16, 1>());
    if (per == 2) return f(Split<16, 2>());
    if (per == 4) return f(Split<16, 4>());
    return per == 8 ? f(Split<16, 8>()) : f(Split<16, 16>());
  }
  if (lanes == 32) {
    if (per == 1) return f(Split<32, 1>());
    if (per == 2) return f(Split<32, 2>());
    if (per == 4) return f(Split<32, 4>());
    return per == 8 ? f(Split<32, 8>()) : f(Split<32, 16>());
  }
  if (per == 1) return f(Split<64, 1>());
  if (per == 2) return f(Split<64, 2>());
  if (per == 4) return f(Split<64, 4>());
  return per == 8 ? f(Split<64, 8>()) : f(Split<64, 16>());
}

template <typename T>
hipError_t forward_t(const RouteDesc& d, void* workspace, hipStream_t s) {
  const RoutePlan p = route_plan(d.n, d.experts, d.top, d.groups);
  const bool wide = route_wide(d);
  const unsigned lds = route_lds(p, d.experts, wide);
  hipError_t e = by_lanes(p.lanes, p.per, [&](auto split) {
    constexpr int L = decltype(split)::L, K = decltype(split)::K;
    const dim3 grid((unsigned)p.groups), block((unsigned)(p.waves * 64));
    const int fast = fast_rows(d.logits, d.ld, d.experts, K, sizeof(T));
    if (wide) {
      launch_timed(route_choose_kernel<T, L, K, true>, grid, block, lds, s, d, p.each, fast, (int)p.room, workspace, (int)(p.groups == 1));
    } else {
      launch_timed(route_choose_kernel<T, L, K, false>, grid, block, lds, s, d, p.each, fast, (int)p.room, workspace, (int)(p.groups == 1));
    }
    return hipGetLastError();
  });
  if (e != hipSuccess || p.groups == 1) return e;
  // (eight waves: 2000 x 120 top 6 5.7 us, sixteen 6.4, four 7.4; 16384 x 256 top 8 7.6, 8.2, 10.2)
  const int waves = 8, part = (p.groups + 255) / 256;
  const dim3 grid((unsigned)((p.groups + part - 1) / part)), block((unsigned)(waves * 64));
  const unsigned space = (unsigned)((2 + waves) * d.experts * 4);
  if (count_bytes(p.each) == 1) {
    launch_timed(route_place_kernel<uint8_t>, grid, block, space, s, d, p.each * part, static_cast<const uint8_t*>(workspace), p.groups, part);
  } else {
    launch_timed(route_place_kernel<uint16_t>, grid, block, space, s, d, p.each * part, static_cast<const uint16_t*>(workspace), p.groups, part);
  }
  return hipGetLastError();
}
template <typename T>
hipError_t backward_t(const RouteDesc& d, hipStream_t s) {
  const RoutePlan p = route_plan(d.n, d.experts, d.top, 1);
  return by_lanes(p.lanes, p.per, [&](auto split) {
    constexpr int L = decltype(split)::L, K = decltype(split)::K;
    launch_timed(route_backward_kernel<T, L, K>, dim3((unsigned)ceil_div(d.n, 256 / L)), dim3(256), 0, s, d,
                 (int)fast_rows(d.logits, d.ld, d.experts, K, sizeof(T)), (int)fast_rows(d.dlogits, d.lddl, d.experts, Piece<T>::N, sizeof(T)));
    return hipGetLastError();
  });
}

}  // namespace

size_t route_workspace(int64_t n, int64_t experts, int64_t top) {
  // (the counts of the most workgroups there can be: what serves many tokens serves fewer)
  for (int64_t groups : {1, 16, 32, 64})  // (what the groups change of the plan)
    if (route_plan(n, experts, top, groups).groups > 1) return (size_t)kRouteGroups * (size_t)experts * 2;
  return 0;
}
hipError_t route_forward(const RouteDesc& d, void* workspace, hipStream_t s) {
  if (d.dtype == DT_F32) return forward_t<float>(d, workspace, s);
  return d.dtype == DT_BF16 ? forward_t<__bf16>(d, workspace, s) : forward_t<_Float16>(d, workspace, s);
}
hipError_t route_backward(const RouteDesc& d, hipStream_t s) {
  if (d.dtype == DT_F32) return backward_t<float>(d, s);
  return d.dtype == DT_BF16 ? backward_t<__bf16>(d, s) : backward_t<_Float16>(d, s);
}

}  // namespace rl
