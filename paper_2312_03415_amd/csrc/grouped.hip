// Layers over stacks of expert weights and over an 8-bit weight: launches of a forward and a backward (grouped.hpp), and the small
// kernels between the products.
#include "grouped.hpp"

#include "fp8.hpp"
#include "gemm_engine.hpp"

namespace rl {
namespace {

constexpr int kThreads = 256;
typedef __attribute__((__vector_size__(4 * sizeof(int)))) int v4;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t pad256(int64_t b) { return (b + 255) / 256 * 256; }

// Joins behind rank-r products, in one launch: up to two sets of slices, and a factor turned for the large product.

// out[e][m][0..N) = alpha * sum over slices of partial[slice][e][m][0..N), in slice order; eight columns a thread
struct SliceSum {
  const float* partial;
  void* out;
  int64_t ldo, so, rows;  // rows: of all e
  int splits, M, N, groups;  // groups: its workgroups (0: none)
  float alpha;
};
// out_e[o][k] = in_e[k][o]: the factor B with the contraction in its rows.  From 64 rows a workgroup turns 64 x 64 in LDS, so that loads and
// stores are runs of 128 bytes (8 experts, 128 x 11008, with the slices of 16384 x 128 beside it: 15 us, 28 directly); below that a thread
// takes eight rows of a column (64 experts, 16 x 8192: 9 us, 12 through LDS).
constexpr int kTurnRows = 64;
struct Turn {
  const void* in;
  void* out;
  int64_t ld, stride;
  int R, O, groups;
};
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(SliceSum p, SliceSum q, Turn t) {
  __shared__ __attribute__((aligned(16))) T tile[64][72];
  int id = (int)blockIdx.x;
  if (id < t.groups && t.R < kTurnRows) {
    const int cols = (t.O + kThreads - 1) / kThreads, eights = t.R / 8;
    const int c = id % cols * kThreads + threadIdx.x, k0 = id / cols % eights * 8, e = id / cols / eights;
    if (c >= t.O) return;
    const T* const in = static_cast<const T*>(t.in) + e * t.stride + (int64_t)k0 * t.ld + c;
    T v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = in[k * t.ld];
    *reinterpret_cast<v4*>(static_cast<T*>(t.out) + ((int64_t)e * t.O + c) * t.R + k0) = *reinterpret_cast<const v4*>(v);
    return;
  }
  if (id < t.groups) {
    const int cols = (t.O + 63) / 64, ks = (t.R + 63) / 64;
    const int c0 = id % cols * 64, k0 = id / cols % ks * 64, e = id / cols / ks, kn = t.R - k0 < 64 ? t.R - k0 : 64;
    const T* const in = static_cast<const T*>(t.in) + e * t.stride + (int64_t)k0 * t.ld + c0;
    for (int q = threadIdx.x; q < kn * 8; q += kThreads) {
      const int k = q >> 3, c = (q & 7) * 8;
      if (c0 + c >= t.O) continue;
      const v4 v = *reinterpret_cast<const v4*>(in + k * t.ld + c);
      const T* const w = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int j = 0; j < 8; ++j) tile[c + j][k] = w[j];
    }
    __syncthreads();
    T* const out = static_cast<T*>(t.out) + ((int64_t)e * t.O + c0) * t.R + k0;
    for (int q = threadIdx.x; q < 8 * kn; q += kThreads) {
      const int c = q / (kn / 8), k = q % (kn / 8) * 8;
      if (c0 + c < t.O) *reinterpret_cast<v4*>(out + (int64_t)c * t.R + k) = *reinterpret_cast<const v4*>(&tile[c][k]);
    }
    return;
  }
  id -= t.groups;
  const bool second = id >= p.groups;
  if (second) id -= p.groups;
  const SliceSum& g = second ? q : p;
  const int64_t c = ((int64_t)id * kThreads + threadIdx.x) * 8, row = c / g.N;
  if (row >= g.rows) return;
  const int col = (int)(c - row * g.N);
  const float* part = g.partial + row * g.N + col;
  f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll 4
  for (int k = 0; k < g.splits; ++k) {
    a += *reinterpret_cast<const f32x4*>(part);
    b += *reinterpret_cast<const f32x4*>(part + 4);
    part += g.rows * g.N;
  }
  const int64_t e = row / g.M, m = row - e * g.M;
  T o[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) { o[k] = from_f32<T>(a[k] * g.alpha); o[4 + k] = from_f32<T>(b[k] * g.alpha); }
  *reinterpret_cast<v4*>(static_cast<T*>(g.out) + e * g.so + m * g.ldo + col) = *reinterpret_cast<const v4*>(o);
}

// expert of a row (experts: behind the last one's), the same on every lane
__device__ __forceinline__ int expert_of(const int32_t* ends, int experts, int row, int lane) {
  if (ends == nullptr) return 0;
  int e = 0;
  for (int base = 0; base < experts; base += 64) {
    const bool before = base + lane < experts && ends[base + lane] <= row;
    e += __popcll(__ballot(before));
  }
  return e;
}

struct FewArgs {
  const void *X, *A, *B, *bias;
  int64_t ldx, lda, sa, ldb, sb;
  float *part_t, *part;  // [slices][n][R], [splits][n][N]
  void *Y, *T;
  int64_t ldy, ldt;
  const int32_t* ends;
  int experts, n, K, N, R, slices, splits;
  float scale;
  uint8_t *q, *qs;  // e4m3 W: X rounded
  int64_t ldq, ldqs;
  int qx, qy;       // its workgroups
};

// Few rows, first launch: X rounded to e4m3 (workgroups [0, qx qy), where W is e4m3) and X A in slices of K (the others: one row and one slice
// each, R / 8 threads side by side for eight columns of A each).
template <typename T>
__global__ __launch_bounds__(kThreads) void few_prepare_kernel(FewArgs g) {
  __shared__ union { float sum[kThreads][9]; uint8_t sc[4][4]; } sh;  // (rows of nine: columns of eight would share banks)
  int bx = (int)blockIdx.x;
  if (bx < g.qx * g.qy) {
    fp8_rows_tile<T, 1>(static_cast<const T*>(g.X), g.ldx, g.n, g.K, g.q, g.ldq, g.qs, g.ldqs, bx % g.qx, bx / g.qx, sh.sc);
    return;
  }
  bx -= g.qx * g.qy;
  const int row = bx % g.n, slice = bx / g.n, e = expert_of(g.ends, g.experts, row, threadIdx.x & 63);
  if (e >= g.experts) return;
  const int cg = g.R / 8, kl = kThreads / cg, c = threadIdx.x % cg, k0 = threadIdx.x / cg;
  const int each = (g.K / 8 + g.slices - 1) / g.slices * 8, lo = slice * each, hi = lo + each < g.K ? lo + each : g.K;
  const T* const x = static_cast<const T*>(g.X) + (int64_t)row * g.ldx;
  const T* const a = static_cast<const T*>(g.A) + e * g.sa + c * 8;
  float acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  if (k0 < kl) {
#pragma unroll 4
    for (int k = lo + k0; k < hi; k += kl) {
      const v4 v = *reinterpret_cast<const v4*>(a + (int64_t)k * g.lda);
      const T* const t = reinterpret_cast<const T*>(&v);
      const float xk = (float)x[k];
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += xk * (float)t[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sh.sum[threadIdx.x][j] = acc[j];
  // the kl sums of a column, eight at a time
  for (int left = kl; left > 1; left = (left + 7) / 8) {
    __syncthreads();
    const int next = (left + 7) / 8;
    float s[8];
    if (k0 < next) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = 0.f;
      for (int k = 8 * k0; k < 8 * k0 + 8 && k < left; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += sh.sum[k * cg + c][j];
    }
    __syncthreads();
    if (k0 < next)
#pragma unroll
      for (int j = 0; j < 8; ++j) sh.sum[threadIdx.x][j] = s[j];
  }
  __syncthreads();
  if ((int)threadIdx.x < g.R) g.part_t[((int64_t)slice * g.n + row) * g.R + threadIdx.x] = sh.sum[threadIdx.x / 8][threadIdx.x & 7];
}

// Few rows, last launch: Y = the slices of X W + T B + bias, T = s * the slices of X A rounded to the storage type.  A workgroup takes 512
// columns of a row; slices and rows of B are dealt out to its four waves, so that every trip to memory is on its way at once.
// Bound by latency: a wave a workgroup, walking everything in turn, took 8.8 us for 1 x 4096 -> 4096 r 16 and 6.6 for 48 x 4096 ->
// 11008 r 32.
template <typename T>
__global__ __launch_bounds__(kThreads) void few_finish_kernel(FewArgs g) {
  constexpr int AHEAD = 4;  // rows of B that a wave requests ahead of T
  __shared__ float part[kThreads], t[256];
  __shared__ f32x4 sums[3][2][64];
  const int row = (int)blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, e = expert_of(g.ends, g.experts, row, lane);
  const int col = ((int)blockIdx.x * 64 + lane) * 8;
  const bool rest = e >= g.experts, ok = col < g.N;
  const T* const bp = static_cast<const T*>(g.B) + (rest ? 0 : e * g.sb) + (ok ? col : 0);
  v4 ahead[AHEAD];
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) ahead[j] = wave + 4 * j < g.R ? *reinterpret_cast<const v4*>(bp + (int64_t)(wave + 4 * j) * g.ldb) : v4{0, 0, 0, 0};
  f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
  const float* p = g.part + (int64_t)row * g.N + (ok ? col : 0);
#pragma unroll 4
  for (int j = wave; j < g.splits; j += 4) {
    a += *reinterpret_cast<const f32x4*>(p + (int64_t)j * g.n * g.N);
    b += *reinterpret_cast<const f32x4*>(p + (int64_t)j * g.n * g.N + 4);
  }
  if (g.R > 0) {
    const int groups = kThreads / g.R, k = tid % g.R, q = tid / g.R;
    float s = 0.f;
    if (q < groups && !rest) {
#pragma unroll 8
      for (int j = q; j < g.slices; j += groups) s += g.part_t[((int64_t)j * g.n + row) * g.R + k];
    }
    part[tid] = s;
    __syncthreads();
    if (tid < g.R) {
      for (int j = 1; j < groups; ++j) s += part[j * g.R + tid];
      const T r = from_f32<T>(s * g.scale);
      t[tid] = (float)r;
      if (g.T != nullptr && blockIdx.x == 0) static_cast<T*>(g.T)[(int64_t)row * g.ldt + tid] = r;
    }
    __syncthreads();
    auto add = [&](const v4& v, float x) {
      const T* const w = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int j = 0; j < 4; ++j) { a[j] += x * (float)w[j]; b[j] += x * (float)w[4 + j]; }
    };
    if (!rest) {
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (wave + 4 * j < g.R) add(ahead[j], t[wave + 4 * j]);
#pragma unroll 4
      for (int kk = wave + 4 * AHEAD; kk < g.R; kk += 4) add(*reinterpret_cast<const v4*>(bp + (int64_t)kk * g.ldb), t[kk]);
    }
  }
  if (wave > 0) { sums[wave - 1][0][lane] = a; sums[wave - 1][1][lane] = b; }
  __syncthreads();
  if (wave > 0 || !ok) return;
#pragma unroll
  for (int w = 0; w < 3; ++w) { a += sums[w][0][lane]; b += sums[w][1][lane]; }
  if (g.bias != nullptr && !rest) {
    const v4 v = *reinterpret_cast<const v4*>(static_cast<const T*>(g.bias) + (int64_t)e * g.N + col);
    const T* const w = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int j = 0; j < 4; ++j) { a[j] += (float)w[j]; b[j] += (float)w[4 + j]; }
  }
  T o[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) { o[j] = from_f32<T>(a[j]); o[4 + j] = from_f32<T>(b[j]); }
  *reinterpret_cast<v4*>(static_cast<T*>(g.Y) + (int64_t)row * g.ldy + col) = *reinterpret_cast<const v4*>(o);
}

template <template <typename> class F, typename... Args>
hipError_t by_type(int dtype, Args... args) {
  return dtype == DT_BF16 ? F<__bf16>::run(args...) : F<_Float16>::run(args...);
}
SliceSum slice_sum(const float* partial, int splits, int64_t rows, int64_t M, int64_t N, float alpha, void* out, int64_t ldo, int64_t so) {
  return SliceSum{partial, out, ldo, so, rows, splits, (int)M, (int)N, (int)ceil_div(rows * N / 8, kThreads), alpha};
}
template <typename T>
struct Join {
  static hipError_t run(const SliceSum& p, const SliceSum& q, const Turn& t, hipStream_t s) {
    const unsigned grid = (unsigned)(p.groups + q.groups + t.groups);
    if (grid == 0) return hipSuccess;
    launch_timed(join_kernel<T>, dim3(grid), dim3(kThreads), 0, s, p, q, t);
    return hipGetLastError();
  }
};
template <typename T>
struct FewPrepare {
  static hipError_t run(const FewArgs& g, hipStream_t s) {
    const unsigned grid = (unsigned)(g.qx * g.qy + (g.R > 0 ? g.n * g.slices : 0));
    if (grid == 0) return hipSuccess;
    launch_timed(few_prepare_kernel<T>, dim3(grid), dim3(kThreads), 0, s, g);
    return hipGetLastError();
  }
};
template <typename T>
struct FewFinish {
  static hipError_t run(const FewArgs& g, hipStream_t s) {
    launch_timed(few_finish_kernel<T>, dim3((unsigned)ceil_div(g.N, 512), (unsigned)g.n), dim3(kThreads), 0, s, g);
    return hipGetLastError();
  }
};

hipError_t launch(int dtype, bool f8, int bl, int tile, const GroupedArgs& a, dim3 grid, hipStream_t s) {
  return dtype == DT_BF16 ? grouped_launch_bf16(f8, bl, tile, a, grid, s) : grouped_launch_f16(f8, bl, tile, a, grid, s);
}

// ---- plans: functions of sizes alone, shared by the workspace query and the call ----------------------

constexpr int64_t kUnits = 256;  // compute units
constexpr int64_t kFill = 512;   // workgroups that fill the chip, two to a compute unit

// rows of an expert that gets its share
int64_t share(const ExpertsDesc& d) { return ceil_div(d.n, d.experts < d.n ? d.experts : d.n); }

bool few(const ExpertsDesc& d) { return d.n <= 64 && d.r <= 256; }

}  // namespace

GroupedPlan grouped_plan(const ExpertsDesc& d, int64_t N, int64_t K, bool slices) {
  GroupedPlan p;
  const int64_t rows = share(d), some = d.experts < d.n ? d.experts : d.n;
  auto most = [&](int tile) {  // tiles that there can be: what is launched
    const GroupedTileInfo t = grouped_tile(tile);
    return grouped_row_tiles(d.n, d.experts, d.has_ends, t.bm, d.f8) * ceil_div(N, t.bn);
  };
  auto expected = [&](int tile) {  // tiles that there will be: an expert's last row tile is half full on average
    const GroupedTileInfo t = grouped_tile(tile);
    return (d.has_ends ? (d.n + (some + 1) * (t.bm / 2)) / t.bm : ceil_div(d.n, t.bm)) * ceil_div(N, t.bn);
  };
  // A larger tile costs less a product, as long as it is filled: it is taken where the next smaller ones are more than one round, two to a
  // compute unit (kFill).  Measured without adapters, 16-bit / 8-bit weights, us:
  //  128 x 128 for 64 x 128, K 768 to 8192.  540 to 672 of the smaller (one group, 10 shapes): 14-30 % / 9-31 % saved, Y of 2100 x 4096 -> 2320
  //    56 / 43 in place of 75 / 56.  Fewer than 512 (3 to 8 uneven experts, 6 shapes): 7 % / 3 % saved to 31 % / 24 % lost, dX of 2000 rows of 8
  //    experts 4096 -> 1792 60 / 41 in place of 46 / 33.
  //  256 x 256 for 128 x 128, K 1024 to 8192.  576 to 768 of the smaller (144 to 192 of the larger; one group, 6 shapes): 5-19 % / up to 22 %
  //    saved, 2300 x 4096 -> 4096 93 / 61 in place of 108 / 70; 540 to 672 of 4 to 16 uneven experts: 9-32 % / 1-29 %, 2400 rows of 4 experts
  //    4096 -> 4096 97 / 62 in place of 136 / 73.  Up to 512 of them: 2-34 % lost, 1600 rows of 8 experts 4096 -> 4096 99 / 59 in place of 91 / 54.
  //    A K below 1024 only where they fill a round by themselves: 3000 x 768 -> 4096 (192) 28.7 / 29.6 in place of 28.6 / 27.6.
  //  64 x 128 from about 160: 300 x 4096 -> 4096 (160 tiles) 33 / 24 against 34 / 25 in 32 x 128 tiles, 200 x 2048 -> 2048 (64) 18 / 15
  //    against 15.5 / 13.
  // With 16-bit weights and a long K, up to half a round of 256 x 256 tiles whose K is split over the compute units are faster than one round of
  // smaller ones: 1237 x 5456 -> 2064 (45 tiles, 86 K tiles) 51 against 64, 3000 rows of 8 experts 8192 -> 1024 (60, 128) 79 against 108, 2560 x
  // 8192 -> 2816 (110, 128) 111 against 115; not with 64 K tiles, 2048 x 4096 -> 2048 51 against 43, or with 80, 2048 x 5120 -> 3584 80 against
  // 75; with 8-bit weights 73 against 46 and 70 against 65.
  const int64_t nk = ceil_div(K, d.f8 ? 128 : 64);
  p.tile = GT_32x128;
  // In slices of K (few rows) 64 x 128 tiles pay from 32 K tiles: 64 rows 4096 -> 11008 29 us against 33, 11008 -> 4096 33 against 35, but
  // 2064 -> 5456 19.3 against 18.0.
  if (rows > 32 && (slices ? nk >= 32 : expected(GT_64x128) >= 160)) p.tile = GT_64x128;
  if (!slices && rows > 96 && expected(GT_64x128) > kFill) p.tile = GT_128x128;
  if (!slices && rows > 160 && (!d.f8 || K <= 128 * 128)) {
    const bool few_split = !d.f8 && nk > 80 && expected(GT_64x128) > kUnits && grouped_split_round((int)expected(GT_256x256), (int)nk).splits > 1;
    if ((expected(GT_128x128) > kFill && (K >= 1024 || expected(GT_256x256) >= 208)) || few_split) p.tile = GT_256x256;
  }
  const int64_t tiles = most(p.tile);
  p.gx = (unsigned)(p.tile == GT_256x256 && tiles > kUnits ? kUnits : tiles);
  p.join = false;
  if (p.tile == GT_256x256) {  // the last round of tiles may be worth splitting; how many tiles there are only the device knows, unless all rows are one group's
    p.join = d.has_ends ? 3 * nk >= 160 : grouped_split_round((int)tiles, (int)nk).splits > 1;
    if (p.join) p.gx = (unsigned)kUnits;
    p.splits = 1;
    p.per = (int)nk;
    return p;
  }
  // A workgroup a compute unit: what two would load faster, the sum over twice the slices takes (with the small launches around it, 64 rows
  // 4096 -> 11008 2 slices 28.8 us, 5 30.7; 40 rows 25.0 and 26.1; 5 rows of 8 experts 2048 -> 2048 3 slices 17.2, 6 18.4).
  int64_t s = slices ? kUnits / tiles : 1;
  if (s > nk / 4) s = nk / 4;
  if (s < 1) s = 1;
  p.per = (int)ceil_div(nk, s);
  p.splits = (int)ceil_div(nk, p.per);
  return p;
}

namespace {

// T = s X A, Z = s dY B^T
struct RankPlan { int tile, splits, per; unsigned gx; };
RankPlan rank_plan(const ExpertsDesc& d, int64_t K) {
  RankPlan p;
  p.tile = d.r <= 32 ? GT_64x32 : (d.r <= 64 ? GT_64x64 : (d.n >= 4096 ? GT_128x128 : GT_64x128T));
  const GroupedTileInfo t = grouped_tile(p.tile);
  const int64_t tiles = grouped_row_tiles(d.n, d.experts, d.has_ends, t.bm, false) * ceil_div(d.r, t.bn), nk = ceil_div(K, 128);  // (slices end on a scale block)
  p.gx = (unsigned)tiles;
  int64_t s = kFill / tiles;
  if (s > nk / 2) s = nk / 2;
  if (s < 1) s = 1;
  p.per = 2 * (int)ceil_div(nk, s);
  p.splits = (int)ceil_div(nk * 2, p.per);
  return p;
}
constexpr size_t kJoinBytes = (size_t)kUnits * 256 * 256 * 4;  // a tile's fp32 sums for every compute unit
size_t rank_bytes(const ExpertsDesc& d, const RankPlan& p) { return p.splits > 1 ? (size_t)p.splits * d.n * d.r * 4 : 0; }

// dA = X^T Z (wide = i), dB = T^T dY (wide = o): tiles of 128 by up to 128 of the rank
struct GradPlan { int width, splits, gx; };
GradPlan grad_plan(const ExpertsDesc& d, int64_t wide) {
  GradPlan p;
  p.width = d.r <= 32 ? 32 : (d.r <= 64 ? 64 : 128);
  const int64_t tiles = d.experts * ceil_div(wide, 128) * ceil_div(d.r, p.width);
  p.gx = (int)tiles;
  int64_t s = kFill / tiles;
  const int64_t nk = ceil_div(share(d), 64);
  if (s > nk / 4) s = nk / 4;
  if (s > 16) s = 16;
  p.splits = (int)(s < 1 ? 1 : s);
  return p;
}
size_t grad_bytes(const ExpertsDesc& d, const GradPlan& p, int64_t wide) { return p.splits > 1 ? (size_t)p.splits * d.experts * wide * d.r * 4 : 0; }

// Few rows: slices of K in X A.  A workgroup's threads go around about six times at most (64 rows 11008 -> 4096 r 64 in 8 slices 41 us, in 32 35;
// 48 rows 4096 -> 11008 r 32 in 8 28.6, in 16 27.7; 64 rows 2064 -> 5456 r 16 in 8 18.6, in 32 20.5).
int few_slices(const ExpertsDesc& d) {
  int s = d.n < 32 ? 16 : 8;
  while (s < 32 && d.i * d.r > (int64_t)s * 8 * kThreads * 6) s *= 2;
  return s;
}

// workspace layout
struct Carver {
  char* base;
  size_t used = 0;
  void* take(size_t bytes) {
    void* p = base ? base + used : nullptr;
    used += (size_t)pad256((int64_t)bytes);
    return p;
  }
};
struct Space {
  uint8_t *q = nullptr, *s = nullptr;  // the rounded X or dY
  int64_t ldq = 0, lds = 0;
  void *turned = nullptr, *T = nullptr, *Z = nullptr;
  float *part = nullptr, *part_t = nullptr, *join = nullptr;
  int slices = 0;
  size_t bytes = 0;
};
Space space(const ExpertsDesc& d, bool backward, void* workspace) {
  Carver c{static_cast<char*>(workspace)};
  Space w;
  const int64_t K = backward ? d.o : d.i, N = backward ? d.i : d.o;
  if (d.f8 && (!backward || d.dX != nullptr || workspace == nullptr)) {
    w.ldq = fp8_row_bytes(K);
    w.lds = fp8_scale_ld(d.n);
    w.q = static_cast<uint8_t*>(c.take((size_t)(d.n * w.ldq)));
    w.s = static_cast<uint8_t*>(c.take((size_t)(w.ldq / 128 * w.lds)));
  }
  if (!backward && few(d)) {
    const GroupedPlan m = grouped_plan(d, N, K, true);
    w.part = static_cast<float*>(c.take((size_t)m.splits * d.n * N * 4));
    if (d.r > 0) {
      w.slices = few_slices(d);
      w.part_t = static_cast<float*>(c.take((size_t)w.slices * d.n * d.r * 4));
    }
  } else if (d.r > 0) {
    size_t part = rank_bytes(d, rank_plan(d, d.i));
    w.T = c.take((size_t)(d.n * d.r) * 2);
    if (!backward) {
      w.turned = c.take((size_t)(d.experts * d.o * d.r) * 2);
    } else {
      w.Z = c.take((size_t)(d.n * d.r) * 2);
      const size_t more[2] = {rank_bytes(d, rank_plan(d, d.o)), grad_bytes(d, grad_plan(d, d.i), d.i) + grad_bytes(d, grad_plan(d, d.o), d.o)};
      for (size_t b : more) part = part > b ? part : b;
    }
    w.part = static_cast<float*>(c.take(part));
  }
  if (!(!backward && few(d)) && (!backward || d.dX != nullptr || workspace == nullptr) && grouped_plan(d, N, K, false).join) w.join = static_cast<float*>(c.take(kJoinBytes));
  w.bytes = c.used;
  return w;
}

GroupedArgs rows_args(const ExpertsDesc& d) {
  GroupedArgs a{};
  a.ends = d.ends;
  a.experts = (int)d.experts;
  a.n = (int)d.n;
  a.alpha = 1.f;
  a.splits = 1;
  a.band = 8;
  return a;
}

// T [n, r] = s A_rows F:  F = A [i, r] (X's rows) or B [r, o] read as its transpose (dY's rows)
// `round`: the rows are also rounded to e4m3 into w.q and w.s
hipError_t rank_run(const ExpertsDesc& d, const Space& w, const void* rows, int64_t ldrows, int64_t K, bool backward, bool round, void* out, int64_t ldo, const Turn& turn, hipStream_t stream) {
  float* const part = w.part;
  const RankPlan p = rank_plan(d, K);
  GroupedArgs a = rows_args(d);
  a.A = rows; a.lda = ldrows;
  a.B = backward ? d.B : d.A; a.ldb = backward ? d.ldb : d.lda; a.sb = backward ? d.sb : d.sa;
  a.C = out; a.ldc = ldo;
  a.N = (int)d.r; a.K = (int)K;
  a.alpha = d.scale;
  a.splits = p.splits; a.tiles_per_split = p.per;
  a.partial = p.splits > 1 ? part : nullptr;
  const dim3 grid(p.gx, (unsigned)p.splits);
  hipError_t e;
  if (round) {
    a.Q = w.q; a.ldq = w.ldq; a.QS = w.s; a.ldqs = w.lds;
    e = d.dtype == DT_BF16 ? grouped_rows_launch_bf16(backward ? 1 : 0, p.tile, a, grid, stream) : grouped_rows_launch_f16(backward ? 1 : 0, p.tile, a, grid, stream);
  } else {
    e = launch(d.dtype, false, backward ? 1 : 0, p.tile, a, grid, stream);
  }
  if (e != hipSuccess) return e;
  const SliceSum sum = p.splits > 1 ? slice_sum(part, p.splits, d.n, d.n, d.r, d.scale, out, ldo, 0) : SliceSum{};
  return by_type<Join>(d.dtype, sum, SliceSum{}, turn, stream);
}

// dA and dB, those that are wanted
hipError_t grads_run(const ExpertsDesc& d, const void* T, int64_t ldt, const void* Z, float* part, hipStream_t stream) {
  GroupedArgs a = rows_args(d), b = rows_args(d);
  const GradPlan pa = grad_plan(d, d.i), pb = grad_plan(d, d.o);
  SliceSum sa{}, sb{};
  int ax = 0, bx = 0;
  if (d.dA) {
    a.A = d.X; a.lda = d.ldx; a.B = Z; a.ldb = d.r;
    a.M = (int)d.i; a.N = (int)d.r;
    a.C = d.dA; a.ldc = d.ldda; a.sc = d.sda;
    a.splits = pa.splits;
    ax = pa.gx;
    if (pa.splits > 1) {
      a.partial = part;
      sa = slice_sum(part, pa.splits, d.experts * d.i, d.i, d.r, 1.f, d.dA, d.ldda, d.sda);
      part += pa.splits * d.experts * d.i * d.r;
    }
  }
  if (d.dB) {
    b.A = T; b.lda = ldt; b.B = d.dY; b.ldb = d.lddy;
    b.M = (int)d.r; b.N = (int)d.o;
    b.C = d.dB; b.ldc = d.lddb; b.sc = d.sdb;
    b.splits = pb.splits;
    bx = pb.gx;
    if (pb.splits > 1) {
      b.partial = part;
      sb = slice_sum(part, pb.splits, d.experts * d.r, d.r, d.o, 1.f, d.dB, d.lddb, d.sdb);
    }
  }
  hipError_t e = d.dtype == DT_BF16 ? grouped_grads_launch_bf16(pa.width, a, ax, b, bx, stream) : grouped_grads_launch_f16(pa.width, a, ax, b, bx, stream);
  return e != hipSuccess ? e : by_type<Join>(d.dtype, sa, sb, Turn{}, stream);
}

// the large product: rows (rounded first where W is e4m3 and they are not yet) times W or its transpose, the adapter's product TA TB^T and the bias behind it
hipError_t main_run(const ExpertsDesc& d, bool backward, const Space& w, const void* TA, int64_t ldta, const void* TB, int64_t ldtb, int64_t stb, void* out, int64_t ldo,
                    bool slices, bool rounded, hipStream_t stream) {
  const int64_t K = backward ? d.o : d.i, N = backward ? d.i : d.o;
  const GroupedPlan p = grouped_plan(d, N, K, slices);
  GroupedArgs a = rows_args(d);
  a.A = backward ? d.dY : d.X;
  a.lda = backward ? d.lddy : d.ldx;
  a.B = d.W; a.ldb = d.ldw; a.sb = d.sw;
  if (d.f8) {
    if (!rounded) {
      hipError_t e = fp8_rows_run(d.dtype, a.A, a.lda, d.n, K, w.q, w.ldq, w.s, w.lds, stream);
      if (e != hipSuccess) return e;
    }
    a.A = w.q; a.lda = w.ldq;
    a.SA = w.s; a.ldsa = w.lds;
    a.SB = d.w_scales; a.ssb = d.s_scales;
    a.scols = (int)ceil_div(d.o, 128);
  }
  a.C = out; a.ldc = ldo;
  a.N = (int)N; a.K = (int)K;
  a.splits = p.splits; a.tiles_per_split = p.per;
  // where an expert's rows are one tile, its W is read once, column tiles in order (64 rows of 16 experts 4096 -> 11008: 127 us in bands
  // of 8 experts, 117 so); otherwise bands of row tiles share what they read of it
  if (share(d) <= grouped_tile(p.tile).bm) a.band = 1;
  if (slices) {
    a.partial = w.part;
  } else {
    a.partial = p.join ? w.join : nullptr;
    a.bias = backward ? nullptr : d.bias;
    if (d.r > 0) { a.TA = TA; a.ldta = ldta; a.TB = TB; a.ldtb = ldtb; a.stb = stb; a.R = (int)d.r; }
  }
  return launch(d.dtype, d.f8, backward ? 1 : 0, p.tile, a, dim3(p.gx, (unsigned)p.splits), stream);
}

}  // namespace

size_t experts_workspace(const ExpertsDesc& d, bool backward) { return space(d, backward, nullptr).bytes; }

hipError_t experts_forward(const ExpertsDesc& d, void* workspace, hipStream_t stream) {
  const Space w = space(d, false, workspace);
  hipError_t e;
  if (few(d)) {
    FewArgs f{};
    f.X = d.X; f.A = d.A; f.B = d.B; f.bias = d.bias;
    f.ldx = d.ldx; f.lda = d.lda; f.sa = d.sa; f.ldb = d.ldb; f.sb = d.sb;
    f.part_t = w.part_t; f.part = w.part;
    f.Y = d.Y; f.ldy = d.ldy; f.T = d.T; f.ldt = d.ldt;
    f.ends = d.ends; f.experts = (int)d.experts;
    f.n = (int)d.n; f.K = (int)d.i; f.N = (int)d.o; f.R = (int)d.r;
    f.slices = w.slices; f.splits = grouped_plan(d, d.o, d.i, true).splits;
    f.scale = d.scale;
    if (d.f8) {
      f.q = w.q; f.qs = w.s; f.ldq = w.ldq; f.ldqs = w.lds;
      f.qx = (int)ceil_div(d.n, 4);
      f.qy = (int)ceil_div(w.ldq, 512);
    }
    if ((e = by_type<FewPrepare>(d.dtype, f, stream)) != hipSuccess) return e;
    if ((e = main_run(d, false, w, nullptr, 0, nullptr, 0, 0, nullptr, 0, true, true, stream)) != hipSuccess) return e;
    return by_type<FewFinish>(d.dtype, f, stream);
  }
  void* T = d.T ? d.T : w.T;
  const int64_t ldt = d.T ? d.ldt : d.r;
  if (d.r > 0) {
    const Turn turn{d.B, w.turned, d.ldb, d.sb, (int)d.r, (int)d.o, (int)((d.r < kTurnRows ? ceil_div(d.o, kThreads) * (d.r / 8) : ceil_div(d.o, 64) * ceil_div(d.r, 64)) * d.experts)};
    if ((e = rank_run(d, w, d.X, d.ldx, d.i, false, d.f8, T, ldt, turn, stream)) != hipSuccess) return e;
  }
  return main_run(d, false, w, T, ldt, w.turned, d.r, d.o * d.r, d.Y, d.ldy, false, d.r > 0, stream);
}

hipError_t experts_backward(const ExpertsDesc& d, void* workspace, hipStream_t stream) {
  const Space w = space(d, true, workspace);
  hipError_t e;
  const void* T = d.T;
  int64_t ldt = d.ldt;
  if (d.r > 0) {
    if ((d.dX || d.dA) && (e = rank_run(d, w, d.dY, d.lddy, d.o, true, d.f8 && d.dX != nullptr, w.Z, d.r, Turn{}, stream)) != hipSuccess) return e;
    if (d.dB && !d.has_T) {
      if ((e = rank_run(d, w, d.X, d.ldx, d.i, false, false, w.T, d.r, Turn{}, stream)) != hipSuccess) return e;
      T = w.T;
      ldt = d.r;
    }
    if ((d.dA || d.dB) && (e = grads_run(d, T, ldt, w.Z, w.part, stream)) != hipSuccess) return e;
  }
  if (d.dX) return main_run(d, true, w, w.Z, d.r, d.A, d.lda, d.sa, d.dX, d.lddx, false, d.r > 0, stream);
  return hipSuccess;
}

}  // namespace rl
