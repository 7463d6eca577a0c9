// Rows to the experts and back (rows.hpp).  Nothing is computed that matters: the kernels are bound by memory, and small calls by their launch (48 x 4096
// top 4: 3.6 us).
#include "rows.hpp"

#include "gemm.hpp"
#include "lanes.hpp"

namespace rl {
namespace {

constexpr int kThreads = 256;

// A wave's piece of work: 64 times 16 bytes of a token's row.  (t the same in all lanes, and known to be: its places and weights are scalar loads.)
struct Strip {
  int64_t t;
  int64_t c;  // this lane's column
  __device__ __forceinline__ Strip(int64_t strip, int parts, int piece) {
    const uint32_t s = (uint32_t)__builtin_amdgcn_readfirstlane((int)strip);  // (fewer than 2^32, see strips())
    t = s / (uint32_t)parts;
    c = ((int64_t)(s % (uint32_t)parts) * 64 + (threadIdx.x & 63)) * piece;
  }
};

// Every strip is read once and written to all the token's places (8192 x 4096 top 2 bf16, 201 MB: 31 us, 6.4 TB/s); then the rows without a copy, top of them a token (their zeros keep what reads them
// behind the last expert's rows finite).
template <typename T>
__global__ __launch_bounds__(kThreads) void gather_kernel(RowsDesc g, int parts, uint32_t strips) {
  constexpr int E = Piece<T>::N;
  const int64_t m = g.n * g.top;
  T* const out = static_cast<T*>(g.out);
  for (uint64_t s = (uint64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); s < strips; s += (uint64_t)gridDim.x * (kThreads / 64)) {
    const Strip w((int64_t)s, parts, E);
    const bool in = w.c < g.d;
    const int32_t* const place = g.place + w.t * g.top;
    const int32_t* const source = g.source + w.t * g.top;
    const Piece<T> x = in ? Piece<T>::load(static_cast<const T*>(g.in) + w.t * g.ldin + w.c) : Piece<T>::zero();
    for (int j = 0; j < g.top; ++j) {
      const int64_t p = place[j];
      if (p >= 0 && p < m && in) x.store(out + p * g.ldout + w.c, g.stream);
    }
    for (int j = 0; j < g.top; ++j)
      if (source[j] < 0 && in) Piece<T>::zero().store(out + (w.t * g.top + j) * g.ldout + w.c, g.stream);
  }
}

// out[p] = w in[t] and the products of in[t] with the rows, eight places at a time: P threads a token.  Bound by memory: 8192 x 2048 top 8 bf16 (570 MB)
// 98 us, 5.8 TB/s (129 where a row was loaded, used and stored before the next).
template <typename T, int P>
__global__ __launch_bounds__(kThreads) void spread_kernel(RowsDesc g) {
  constexpr int E = Piece<T>::N, B = 8;
  __shared__ float part[kThreads / 64][B];
  const int64_t t = (int64_t)blockIdx.x * (kThreads / P) + __builtin_amdgcn_readfirstlane((int)threadIdx.x / P);
  const bool in_range = t < g.n;
  const int64_t m = g.n * g.top, row = in_range ? t : 0;
  const int32_t* const place = g.place + row * g.top;
  const T* const in = static_cast<const T*>(g.in) + row * g.ldin;
  const T* const rows = static_cast<const T*>(g.rows);
  T* const out = static_cast<T*>(g.out);
  const int own = threadIdx.x % P;
  for (int j0 = 0; j0 < g.top; j0 += B) {
    int64_t p[B];
    float w[B], dot[B];
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int at = j0 + j < g.top ? j0 + j : g.top - 1;
      p[j] = place[at];
      w[j] = g.weight[row * g.top + at];
    }
#pragma unroll
    for (int j = 0; j < B; ++j) {
      dot[j] = 0.f;
      if (p[j] >= m || j0 + j >= g.top || !in_range) p[j] = -1;
    }
    for (int64_t c = (int64_t)own * E; c < g.d; c += P * E) {
      if (!in_range) break;
      float x[E];
      Piece<T> r[B];
      const Piece<T> xs = Piece<T>::load(in + c);
      if (rows != nullptr) {  // (all of them on their way before the first is used)
#pragma unroll
        for (int j = 0; j < B; ++j) r[j] = p[j] >= 0 ? Piece<T>::load(rows + p[j] * g.ldrows + c) : Piece<T>::zero();
      }
      xs.get(x);
      if (out != nullptr) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
          if (p[j] < 0) continue;
          float o[E];
#pragma unroll
          for (int k = 0; k < E; ++k) o[k] = w[j] * x[k];
          Piece<T>::of(o).store(out + p[j] * g.ldout + c, g.stream);
        }
      }
      if (rows != nullptr) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
          float f[E];
          r[j].get(f);
          // (a copy without a place: its own zeros, whatever dY holds)
#pragma unroll
          for (int k = 0; k < E; ++k) dot[j] += p[j] >= 0 ? x[k] * f[k] : 0.f;
        }
      }
    }
    if (rows != nullptr) {
#pragma unroll
      for (int j = 0; j < B; ++j) dot[j] = lanes_sum<64>(dot[j]);
      if constexpr (P > 64) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
          for (int j = 0; j < B; ++j) part[threadIdx.x >> 6][j] = dot[j];
        }
        __syncthreads();
        if (threadIdx.x < B && in_range && j0 + (int)threadIdx.x < g.top) {
          float s = 0.f;
#pragma unroll
          for (int k = 0; k < P / 64; ++k) s += part[k][threadIdx.x];
          g.dweight[row * g.top + j0 + threadIdx.x] = s;
        }
        __syncthreads();
      } else {
#pragma unroll
        for (int j = 0; j < B; ++j)
          if (own == 0 && in_range && j0 + j < g.top) g.dweight[row * g.top + j0 + j] = dot[j];
      }
    }
  }
  if (out != nullptr && in_range) {
    for (int j = 0; j < g.top; ++j)
      if (g.source[row * g.top + j] < 0)
        for (int64_t c = (int64_t)own * E; c < g.d; c += P * E) Piece<T>::zero().store(out + (row * g.top + j) * g.ldout + c);
  }
}

// A strip of the sum, B copies at a time: their places and weights first (scalar loads), then their rows, all of them on their way before the first is
// used.  Lanes behind the row's end and copies without a place load what is there to load and leave it: without branches around the loads.
// Bound by memory: 8192 x 2048 top 8 bf16 (302 MB) 47 us, 6.4 TB/s, where a copy after the other took 71; 8192 x 4096 top 2 (201 MB) 31 us, with B = 8
// for two copies 38.
template <typename T, int B>
__global__ __launch_bounds__(kThreads) void join_rows_kernel(RowsDesc g, int parts, uint32_t strips) {
  constexpr int E = Piece<T>::N;
  const int64_t m = g.n * g.top;
  for (uint64_t s = (uint64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); s < strips; s += (uint64_t)gridDim.x * (kThreads / 64)) {
    const Strip v((int64_t)s, parts, E);
    const bool there = v.c < g.d;
    const int64_t c = there ? v.c : 0;
    const int32_t* const place = g.place + v.t * g.top;
    const float* const weight = g.weight != nullptr ? g.weight + v.t * g.top : nullptr;
    const T* const in = static_cast<const T*>(g.in) + c;
    float acc[E];
    const Piece<T> add = g.add != nullptr ? Piece<T>::load(static_cast<const T*>(g.add) + v.t * g.ldadd + c) : Piece<T>::zero();
    for (int j0 = 0; j0 < g.top; j0 += B) {
      Piece<T> r[B];
      int64_t p[B];
      float w[B];
      bool ok[B];
#pragma unroll
      for (int j = 0; j < B; ++j) {
        const int at = j0 + j < g.top ? j0 + j : g.top - 1;
        p[j] = place[at];
        w[j] = weight != nullptr ? weight[at] : 1.f;
        ok[j] = j0 + j < g.top && p[j] >= 0 && p[j] < m;
      }
#pragma unroll
      for (int j = 0; j < B; ++j) r[j] = Piece<T>::load(in + (ok[j] ? p[j] : 0) * g.ldin);
      if (j0 == 0) add.get(acc);
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (!ok[j]) continue;  // (whatever the row holds)
        float f[E];
        r[j].get(f);
#pragma unroll
        for (int k = 0; k < E; ++k) acc[k] += w[j] * f[k];
      }
    }
    if (there) Piece<T>::of(acc).store(static_cast<T*>(g.out) + v.t * g.ldout + v.c, g.stream);
  }
}

// strips of all rows, fewer than 2^32 (rows_fit)
template <typename T>
struct Strips {
  int parts;
  uint32_t all;
  dim3 grid;
  explicit Strips(const RowsDesc& d) {
    parts = (int)((d.d + 64 * Piece<T>::N - 1) / (64 * Piece<T>::N));
    all = (uint32_t)(d.n * parts);
    const uint64_t groups = ((uint64_t)all + kThreads / 64 - 1) / (kThreads / 64);
    grid = dim3((unsigned)(groups < (1u << 22) ? groups : (1u << 22)));
  }
};

// A wave a token where there are many and a round of 256 threads over the row would leave a tenth of them idle.  8192 rows, us, wave / workgroup: 1024
// columns top 4 58 / 60, 1536 71 / 83, 2056 102 / 108, 4096 188 / 181, 8192 371 / 357, 2048 top 8 181 / 173.
template <typename T>
bool wave_a_token(const RowsDesc& d) {
  const int64_t pieces = d.d / Piece<T>::N, rounds = (pieces + kThreads - 1) / kThreads;
  return d.n >= 2048 && pieces * 10 < rounds * kThreads * 9;
}

bool streams(int dtype, int64_t rows, int64_t d) { return rows * d * (dtype == DT_F32 ? 4 : 2) >= kStreamBytes; }

template <typename T>
hipError_t spread(const RowsDesc& d, hipStream_t s) {
  if (d.weight == nullptr) {
    const Strips<T> w(d);
    launch_timed(gather_kernel<T>, w.grid, dim3(kThreads), 0, s, d, w.parts, w.all);
  } else if (wave_a_token<T>(d)) {
    launch_timed(spread_kernel<T, 64>, dim3((unsigned)((d.n + 3) / 4)), dim3(kThreads), 0, s, d);
  } else {
    launch_timed(spread_kernel<T, kThreads>, dim3((unsigned)d.n), dim3(kThreads), 0, s, d);
  }
  return hipGetLastError();
}
template <typename T>
hipError_t join(const RowsDesc& d, hipStream_t s) {
  const Strips<T> w(d);
  if (d.top <= 2) {
    launch_timed(join_rows_kernel<T, 2>, w.grid, dim3(kThreads), 0, s, d, w.parts, w.all);
  } else if (d.top <= 4) {
    launch_timed(join_rows_kernel<T, 4>, w.grid, dim3(kThreads), 0, s, d, w.parts, w.all);
  } else {
    launch_timed(join_rows_kernel<T, 8>, w.grid, dim3(kThreads), 0, s, d, w.parts, w.all);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t rows_spread(const RowsDesc& desc, hipStream_t s) {
  RowsDesc d = desc;
  d.stream = streams(d.dtype, d.n * d.top, d.d);
  if (d.dtype == DT_F32) return spread<float>(d, s);
  return d.dtype == DT_BF16 ? spread<__bf16>(d, s) : spread<_Float16>(d, s);
}
hipError_t rows_join(const RowsDesc& desc, hipStream_t s) {
  RowsDesc d = desc;
  d.stream = streams(d.dtype, d.n, d.d);
  if (d.dtype == DT_F32) return join<float>(d, s);
  return d.dtype == DT_BF16 ? join<__bf16>(d, s) : join<_Float16>(d, s);
}

}  // namespace rl
