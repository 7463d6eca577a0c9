// Routing of tokens to experts (route.hpp): scores, choice and weights of a token's experts, and the order of the rows sorted by expert.
//
// The choice is decided on the logits themselves where nothing is added to the scores (they have the same order), otherwise on scores + bias in
// 64 bits: in 32 bits the two closest of a row's candidates would change places once in some 10^5 rows.
#include "route.hpp"

#include "gemm.hpp"
#include "lanes.hpp"

namespace rl {
namespace {

constexpr float kNone = -INFINITY;  // key of an expert that cannot be chosen

template <typename V> __device__ __forceinline__ V ranked(V v) { return v != v ? (V)INFINITY : v; }  // a NaN comes before everything

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

// row maximum (not counting NaN) and sum of exp(l - max) of a row's logits, l = -inf where there is none; the sum is 0 only where nothing is left
template <int L, int K>
__device__ __forceinline__ void softmax_stats(const float (&l)[K], float* top, float* sum) {
  float m = kNone;
#pragma unroll
  for (int k = 0; k < K; ++k) m = l[k] > m ? l[k] : m;
  m = lanes_max<L>(m);
  const float base = m == kNone ? 0.f : m;
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k) s += expf(l[k] - base);
  *top = base;
  *sum = lanes_sum<L>(s);
}

// best `group_top` (1 or 2) keys of every group, summed, and which groups are kept: the keys outside them become -inf.  The wave's keys go through
// LDS, so that q lanes scan a group whatever its size.
template <int K, typename V>
__device__ __forceinline__ void keep_groups(const RouteDesc& g, V (&key)[K], V* scratch, int lane) {
  const int size = g.experts / g.groups;
  int q = 1;
  while (2 * q * g.groups <= 64 && q < 16) q *= 2;
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (lane + 64 * k < g.experts) scratch[lane + 64 * k] = key[k];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int group = lane / q;
  V a = (V)kNone, b = (V)kNone;  // best and second best
  if (group < g.groups)
    for (int i = lane % q; i < size; i += q) {
      const V v = scratch[group * size + i];
      b = v > a ? a : (v > b ? v : b);
      a = v > a ? v : a;
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
  const V rank = g.group_top > 1 && b != (V)kNone ? a + b : a;
  int before = 0;
  for (int o = 0; o < g.groups; ++o) {
    const V r = from_lane<64>(rank, o * q);
    before += r > rank || (r == rank && o < group) ? 1 : 0;
  }
  const uint64_t kept = __ballot(group < g.groups && before < g.kept);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int e = lane + 64 * k;
    if (e < g.experts && ((kept >> (e / size * q)) & 1) == 0) key[k] = (V)kNone;
  }
  __builtin_amdgcn_wave_barrier();  // (the scratch is the next token's)
}

// the `top` largest keys of a row in falling order, equal ones by index: lane j of the group ends up with choice j and its logit
template <int L, int K, typename V>
__device__ __forceinline__ void choose(int top, V (&key)[K], const float (&l)[K], int sub, int lane, int* expert, float* logit) {
  for (int j = 0; j < top; ++j) {
    V m = key[0];
#pragma unroll
    for (int k = 1; k < K; ++k) m = key[k] > m ? key[k] : m;
    m = lanes_max<L>(m);
    int found = -1, at = 0;
    float v = 0.f;
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      uint64_t hit = __ballot(key[k] == m);
      if constexpr (L < 64) hit = (hit >> (lane & ~(L - 1))) & ((1ull << L) - 1);
      if (hit != 0) {
        found = k;
        at = __builtin_ctzll(hit);
        v = l[k];
      }
    }
    v = from_lane<L>(v, at);
    const bool some = m != (V)kNone;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (k == found && sub == at) key[k] = (V)kNone;
    if (sub == j) {
      *expert = some ? at + L * found : -1;
      *logit = v;
    }
  }
}

// what a workgroup of `waves` waves has in LDS: counts of its experts [experts]; then either a wave's keys [waves][experts] of 8 bytes (groups) or a
// wave's counts [waves][experts] of 4
__device__ __forceinline__ int* lds_counts(char* lds) { return reinterpret_cast<int*>(lds); }

// start of every expert's rows from their counts, in place; returns their sum.  All threads of the workgroup.
__device__ __forceinline__ void scan_counts(const int* counts, int* starts, int experts, int* total) {
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
      const int c = counts[k];
      starts[k] = run;
      run += c;
    }
  }
  __syncthreads();
}

// Rows of the entries [lo, hi) of `expert` (an expert's in their order, from starts[e] on): every wave counts a run of them, the counts become
// the waves' first rows, and each wave walks its run, 64 entries at a time, an entry's place among the equal ones before it by ballots over the bits.
__device__ __forceinline__ void place_entries(const RouteDesc& g, int64_t lo, int64_t hi, const int* starts, int* mine) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int k = threadIdx.x; k < waves * g.experts; k += blockDim.x) mine[k] = 0;
  __syncthreads();
  const int64_t per = ((hi - lo + waves - 1) / waves + 63) / 64 * 64, first = lo + wave * per, last = first + per < hi ? first + per : hi;
  int* const count = mine + wave * g.experts;
  for (int64_t i = first + lane; i < last; i += 64) {
    const int e = g.expert[i];
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < g.experts; e += blockDim.x) {
    int run = starts[e];
    for (int w = 0; w < waves; ++w) {
      const int c = mine[w * g.experts + e];
      mine[w * g.experts + e] = run;
      run += c;
    }
  }
  __syncthreads();
  const int bits = 32 - __builtin_clz(g.experts);
  for (int64_t i0 = first; i0 < last; i0 += 64) {
    const int64_t i = i0 + lane;
    const int e = i < last ? g.expert[i] : -1;
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

// Workgroup b takes the tokens [b each, (b + 1) each), L lanes a token with K experts each: their experts and weights, and how many rows every
// expert gets (counts [b][experts] in the workspace).  A single workgroup places them too.
template <typename T, int L, int K, bool WIDE>
__global__ __launch_bounds__(K > 8 ? 256 : (K > 4 ? 512 : 1024)) void route_choose_kernel(RouteDesc g, int each, uint16_t* counts, int single) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int* const count = lds_counts(lds);
  char* const rest = lds + (g.experts * 4 + 15) / 16 * 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, sub = lane % L;
  for (int k = threadIdx.x; k < g.experts; k += blockDim.x) count[k] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * each, last = first + each < g.n ? first + each : g.n;
  float bias[K];
#pragma unroll
  for (int k = 0; k < K; ++k) bias[k] = g.bias != nullptr && sub + L * k < g.experts ? g.bias[sub + L * k] : 0.f;
  constexpr int SIDE = 64 / L;  // tokens side by side in a wave
  for (int64_t t0 = first + wave * SIDE; t0 < last; t0 += waves * SIDE) {
    const int64_t t = t0 + lane / L;
    const bool there = t < last;
    float l[K];
#pragma unroll
    for (int k = 0; k < K; ++k) l[k] = there && sub + L * k < g.experts ? (float)static_cast<const T*>(g.logits)[t * g.ld + sub + L * k] : kNone;
    float base = 0.f, sum = 1.f;
    if (!g.sigmoid && (!g.renorm || WIDE)) softmax_stats<L, K>(l, &base, &sum);
    int expert = -1;
    float logit = 0.f;
    if constexpr (WIDE) {
      double key[K];
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
      for (int k = 0; k < K; ++k) key[k] = l[k] == kNone ? (double)kNone : ranked(key[k] + (double)bias[k]);
      if (g.groups > 1) keep_groups<K>(g, key, reinterpret_cast<double*>(rest) + wave * g.experts, lane);
      choose<L, K>(g.top, key, l, sub, lane, &expert, &logit);
    } else {
      float key[K];
#pragma unroll
      for (int k = 0; k < K; ++k) key[k] = ranked(l[k]);
      if (g.groups > 1) keep_groups<K>(g, key, reinterpret_cast<float*>(rest) + wave * g.experts, lane);
      choose<L, K>(g.top, key, l, sub, lane, &expert, &logit);
    }
    // weights: lane j holds choice j
    const bool chosen = sub < g.top && expert >= 0;
    float w = 0.f;
    if (g.renorm) {
      // scores over the largest of the chosen ones: their sum is at least 1 (sigmoid: 1/2), however small they are
      const float a = g.sigmoid ? (logit < 0.f ? logit : (logit != logit ? logit : 0.f)) : logit;
      const float m = lanes_max<L>(chosen ? ranked(a) : kNone);
      if (chosen) {
        w = expf(a - m);
        if (g.sigmoid) w = w / (1.f + expf(-fabsf(logit)));
      }
      const float s = lanes_sum<L>(w);
      if (chosen) w = w / s;
      if (!g.sigmoid && sum != sum) w = sum;  // a NaN in the row
    } else if (chosen) {
      w = g.sigmoid ? 1.f / (1.f + expf(-logit)) : expf(logit - base) / sum;
    }
    if (there && sub < g.top) {
      g.expert[t * g.top + sub] = expert;
      g.weight[t * g.top + sub] = chosen ? g.scale * w : 0.f;
      if (expert >= 0) atomicAdd(&count[expert], 1);
    }
  }
  __syncthreads();
  if (!single) {
    for (int k = threadIdx.x; k < g.experts; k += blockDim.x) counts[(int64_t)blockIdx.x * g.experts + k] = (uint16_t)count[k];
    return;
  }
  __shared__ int total;
  int* const mine = reinterpret_cast<int*>(rest);
  for (int k = threadIdx.x; k < g.experts; k += blockDim.x) mine[k] = count[k];
  __syncthreads();
  scan_counts(mine, count, g.experts, &total);
  for (int k = threadIdx.x; k < g.experts; k += blockDim.x) g.ends[k] = count[k] + mine[k];
  for (int64_t p = total + threadIdx.x; p < g.n * g.top; p += blockDim.x) g.source[p] = -1;
  __syncthreads();
  place_entries(g, 0, g.n * g.top, count, mine);
}

// Workgroup b places its tokens' rows behind those of the workgroups before it.
__global__ __launch_bounds__(1024) void route_place_kernel(RouteDesc g, int each, const uint16_t* counts) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ int total;
  int* const starts = reinterpret_cast<int*>(lds);
  int* const mine = starts + g.experts;     // all rows of an expert, then place_entries' own
  int* const before = mine + g.experts;     // (inside place_entries' counts: two waves at least)
  const int groups = (int)gridDim.x;
  for (int e = threadIdx.x; e < g.experts; e += blockDim.x) {
    int all = 0, mark = 0;
#pragma unroll 8
    for (int b = 0; b < groups; ++b) {
      const int c = counts[(int64_t)b * g.experts + e];
      mark += b < (int)blockIdx.x ? c : 0;
      all += c;
    }
    mine[e] = all;
    before[e] = mark;
  }
  __syncthreads();
  scan_counts(mine, starts, g.experts, &total);
  for (int e = threadIdx.x; e < g.experts; e += blockDim.x) {
    if (blockIdx.x == 0) g.ends[e] = starts[e] + mine[e];
    starts[e] += before[e];
  }
  const int64_t m = g.n * g.top;
  for (int64_t p = total + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; p < m; p += (int64_t)groups * blockDim.x) g.source[p] = -1;
  __syncthreads();
  const int64_t lo = (int64_t)blockIdx.x * each * g.top, hi = lo + (int64_t)each * g.top;
  place_entries(g, lo, hi < m ? hi : m, starts, mine);
}

inline __host__ __device__ bool route_wide(const RouteDesc& g) { return g.bias != nullptr || (g.groups > 1 && g.group_top > 1); }

// Gradient of the logits, L lanes a token; p, q as in the forward:
//     softmax:                dl_e = p_e (D_e - sum_j D_j p_j)               D = scale dw, zero off the chosen experts
//     softmax over chosen:    dl_j = q_j (D_j - sum_k D_k q_k)               and zero elsewhere
//     sigmoid:                dl_j = s_j (1 - s_j) D_j;   over the chosen: q_j (1 - s_j) (D_j - sum_k D_k q_k)
template <typename T, int L, int K>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteDesc g) {
  const int lane = threadIdx.x & 63, sub = lane % L;
  const int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  const bool there = t < g.n;
  const T* const row = static_cast<const T*>(g.logits) + (there ? t : 0) * g.ld;
  int expert = -1;
  float d = 0.f, logit = 0.f;
  if (there && sub < g.top) {
    expert = g.expert[t * g.top + sub];
    if (expert >= g.experts) expert = -1;
    if (expert >= 0) {
      d = g.scale * g.dweight[t * g.top + sub];
      logit = (float)row[expert];
    }
  }
  const bool chosen = expert >= 0;
  float out[K], l[K], base = 0.f, sum = 1.f;
  if (!g.sigmoid && (!g.renorm || route_wide(g))) {  // (with a bias a NaN need not be among the chosen: as in the forward)
#pragma unroll
    for (int k = 0; k < K; ++k) l[k] = there && sub + L * k < g.experts ? (float)row[sub + L * k] : kNone;
    softmax_stats<L, K>(l, &base, &sum);
  }
  if (!g.renorm && !g.sigmoid) {
    const float mean = lanes_sum<L>(chosen ? d * (expf(logit - base) / sum) : 0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      l[k] = sum == 0.f ? 0.f : expf(l[k] - base) / sum;
      out[k] = -l[k] * mean;
    }
    for (int j = 0; j < g.top; ++j) {
      const int e = from_lane<L>(expert, j);
      const float x = from_lane<L>(d, j);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (e == sub + L * k) out[k] = l[k] * (x - mean);
    }
  } else {
    const float s = g.sigmoid ? 1.f / (1.f + expf(-logit)) : 1.f, left = g.sigmoid ? 1.f / (1.f + expf(logit)) : 1.f;
    float v = 0.f;
    if (g.renorm) {
      const float a = g.sigmoid ? (logit < 0.f ? logit : (logit != logit ? logit : 0.f)) : logit;
      const float m = lanes_max<L>(chosen ? ranked(a) : kNone);
      float q = 0.f;
      if (chosen) {
        q = expf(a - m);
        if (g.sigmoid) q = q / (1.f + expf(-fabsf(logit)));
      }
      const float all = lanes_sum<L>(q);
      if (chosen) q = q / all;
      const float mean = lanes_sum<L>(chosen ? d * q : 0.f);
      if (chosen) v = q * left * (d - mean);
      if (sum != sum) v = sum;
    } else if (chosen) {
      v = s * left * d;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) out[k] = 0.f;
    for (int j = 0; j < g.top; ++j) {
      const int e = from_lane<L>(expert, j);
      const float x = from_lane<L>(v, j);
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (e == sub + L * k) out[k] = x;
    }
  }
  if (there) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (sub + L * k < g.experts) static_cast<T*>(g.dlogits)[t * g.lddl + sub + L * k] = (T)out[k];
  }
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- plans --------------------------------------------------------------------------------------------

constexpr int64_t kGroups = 256;  // workgroups of a large call; counts of at most 65535 rows an expert in each of them (kRouteMaxTokens)
static_assert(kRouteMaxTokens / kGroups < 65536, "counts are 16 bits");

struct RoutePlan {
  int waves, each, groups, lanes;
};
RoutePlan route_plan(int64_t n, int64_t experts, bool grouped) {
  RoutePlan p;
  p.lanes = grouped || experts > 32 ? 64 : (experts > 16 ? 32 : (experts > 8 ? 16 : 8));
  p.waves = experts > 512 ? 4 : (experts > 256 ? 8 : 16);  // LDS: 8 bytes a wave and expert
  const int64_t at_once = (int64_t)p.waves * (64 / p.lanes);
  if (n <= 8 * at_once) {
    p.groups = 1;
    p.each = (int)n;
    return p;
  }
  p.each = (int)(ceil_div(ceil_div(n, kGroups), at_once) * at_once);
  p.groups = (int)ceil_div(n, p.each);
  return p;
}

template <int L_, int K_> struct Split { static constexpr int L = L_, K = K_; };
template <typename F>
hipError_t by_experts(int lanes, int64_t experts, F&& f) {
  if (lanes == 8) return f(Split<8, 1>());
  if (lanes == 16) return f(Split<16, 1>());
  if (lanes == 32) return f(Split<32, 1>());
  if (experts <= 64) return f(Split<64, 1>());
  if (experts <= 128) return f(Split<64, 2>());
  if (experts <= 256) return f(Split<64, 4>());
  if (experts <= 512) return f(Split<64, 8>());
  return f(Split<64, 16>());
}

template <typename T>
hipError_t forward_t(const RouteDesc& d, void* workspace, hipStream_t s) {
  const RoutePlan p = route_plan(d.n, d.experts, d.groups > 1);
  const unsigned counts = (unsigned)ceil_div(d.experts * 4, 16) * 16, keys = (unsigned)(p.waves * d.experts * 8);
  uint16_t* const space = static_cast<uint16_t*>(workspace);
  const bool wide = route_wide(d);
  hipError_t e = by_experts(p.lanes, d.experts, [&](auto split) {
    constexpr int L = decltype(split)::L, K = decltype(split)::K;
    const dim3 grid((unsigned)p.groups), block((unsigned)(p.waves * 64));
    if (wide) {
      launch_timed(route_choose_kernel<T, L, K, true>, grid, block, counts + keys, s, d, p.each, space, (int)(p.groups == 1));
    } else {
      launch_timed(route_choose_kernel<T, L, K, false>, grid, block, counts + keys, s, d, p.each, space, (int)(p.groups == 1));
    }
    return hipGetLastError();
  });
  if (e != hipSuccess || p.groups == 1) return e;
  launch_timed(route_place_kernel, dim3((unsigned)p.groups), dim3((unsigned)(p.waves * 64)), counts + keys, s, d, p.each, static_cast<const uint16_t*>(space));
  return hipGetLastError();
}
template <typename T>
hipError_t backward_t(const RouteDesc& d, hipStream_t s) {
  const int lanes = route_plan(d.n, d.experts, d.groups > 1).lanes;
  return by_experts(lanes, d.experts, [&](auto split) {
    constexpr int L = decltype(split)::L, K = decltype(split)::K;
    launch_timed(route_backward_kernel<T, L, K>, dim3((unsigned)ceil_div(d.n, 256 / L)), dim3(256), 0, s, d);
    return hipGetLastError();
  });
}

}  // namespace

size_t route_workspace(int64_t n, int64_t experts) {
  size_t need = 0;
  for (int grouped = 0; grouped < 2; ++grouped) {
    const RoutePlan p = route_plan(n, experts, grouped != 0);
    const size_t b = p.groups > 1 ? (size_t)p.groups * (size_t)experts * 2 : 0;
    need = b > need ? b : need;
  }
  return need;
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
