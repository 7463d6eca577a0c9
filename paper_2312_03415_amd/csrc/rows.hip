// Rows to the experts and back (rows.hpp).  Nothing is computed that matters: both kernels are bound by memory.
#include "rows.hpp"

#include "gemm.hpp"
#include "lanes.hpp"

namespace rl {
namespace {

constexpr int kThreads = 256;

// P threads take a token: 16 bytes of its row each, read once and written to all its places; then the rows without a copy, top of them a token
// (their zeros keep what reads them behind the last expert's rows finite).
template <typename T, int P>
__global__ __launch_bounds__(kThreads) void gather_kernel(RowsDesc g) {
  constexpr int E = Piece<T>::N;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / P) + threadIdx.x / P;
  if (t >= g.n) return;
  const int64_t m = g.n * g.top;
  const int32_t* const place = g.place + t * g.top;
  const int32_t* const source = g.source + t * g.top;
  const T* const in = static_cast<const T*>(g.in) + t * g.ldin;
  T* const out = static_cast<T*>(g.out);
  for (int64_t c = (int64_t)(threadIdx.x % P) * E; c < g.d; c += P * E) {
    const Piece<T> x = Piece<T>::load(in + c);
#pragma unroll 4
    for (int j = 0; j < g.top; ++j) {
      const int64_t p = place[j];
      if (p >= 0 && p < m) x.store(out + p * g.ldout + c);
    }
    for (int j = 0; j < g.top; ++j)
      if (source[j] < 0) Piece<T>::zero().store(out + (t * g.top + j) * g.ldout + c);
  }
}

// out[p] = w in[t] and the products of in[t] with the rows, eight places at a time: P threads a token
template <typename T, int P>
__global__ __launch_bounds__(kThreads) void spread_kernel(RowsDesc g) {
  constexpr int E = Piece<T>::N, B = 8;
  __shared__ float part[kThreads / 64][B];
  const int64_t t = (int64_t)blockIdx.x * (kThreads / P) + threadIdx.x / P;
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
      dot[j] = 0.f;
      p[j] = in_range && j0 + j < g.top ? place[j0 + j] : -1;
      if (p[j] >= m) p[j] = -1;
      w[j] = p[j] >= 0 ? g.weight[row * g.top + j0 + j] : 0.f;
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
          Piece<T>::of(o).store(out + p[j] * g.ldout + c);
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

template <typename T, int P>
__global__ __launch_bounds__(kThreads) void join_rows_kernel(RowsDesc g) {
  constexpr int E = Piece<T>::N, B = 8;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / P) + threadIdx.x / P;
  if (t >= g.n) return;
  const int64_t m = g.n * g.top;
  const int32_t* const place = g.place + t * g.top;
  const float* const weight = g.weight != nullptr ? g.weight + t * g.top : nullptr;
  const T* const in = static_cast<const T*>(g.in);
  for (int64_t c = (int64_t)(threadIdx.x % P) * E; c < g.d; c += P * E) {
    float acc[E];
    if (g.add != nullptr) {
      Piece<T>::load(static_cast<const T*>(g.add) + t * g.ldadd + c).get(acc);
    } else {
#pragma unroll
      for (int k = 0; k < E; ++k) acc[k] = 0.f;
    }
    for (int j0 = 0; j0 < g.top; j0 += B) {
      Piece<T> r[B];
      float w[B];
      bool ok[B];
#pragma unroll
      for (int j = 0; j < B; ++j) {  // (all of them on their way before the first is used)
        const int64_t p = j0 + j < g.top ? place[j0 + j] : -1;
        ok[j] = p >= 0 && p < m;
        w[j] = ok[j] && weight != nullptr ? weight[j0 + j] : 1.f;
        r[j] = ok[j] ? Piece<T>::load(in + p * g.ldin + c) : Piece<T>::zero();
      }
#pragma unroll
      for (int j = 0; j < B; ++j) {
        float f[E];
        r[j].get(f);
#pragma unroll
        for (int k = 0; k < E; ++k) acc[k] = ok[j] ? acc[k] + w[j] * f[k] : acc[k];
      }
    }
    Piece<T>::of(acc).store(static_cast<T*>(g.out) + t * g.ldout + c);
  }
}

template <typename T>
hipError_t spread(const RowsDesc& d, hipStream_t s) {
  if (d.weight == nullptr) {
    launch_timed(gather_kernel<T, kThreads>, dim3((unsigned)d.n), dim3(kThreads), 0, s, d);
  } else {
    launch_timed(spread_kernel<T, kThreads>, dim3((unsigned)d.n), dim3(kThreads), 0, s, d);
  }
  return hipGetLastError();
}
template <typename T>
hipError_t join(const RowsDesc& d, hipStream_t s) {
  launch_timed(join_rows_kernel<T, kThreads>, dim3((unsigned)d.n), dim3(kThreads), 0, s, d);
  return hipGetLastError();
}

}  // namespace

hipError_t rows_spread(const RowsDesc& d, hipStream_t s) {
  if (d.dtype == DT_F32) return spread<float>(d, s);
  return d.dtype == DT_BF16 ? spread<__bf16>(d, s) : spread<_Float16>(d, s);
}
hipError_t rows_join(const RowsDesc& d, hipStream_t s) {
  if (d.dtype == DT_F32) return join<float>(d, s);
  return d.dtype == DT_BF16 ? join<__bf16>(d, s) : join<_Float16>(d, s);
}

}  // namespace rl
