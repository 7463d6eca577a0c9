// Root-mean-square norm (norm.hpp).
//     h = x + r rounded to the storage type (the residual stream is kept in it, and the backward reads it), rho = 1 / sqrt(mean h^2 + eps),
//     y = h rho g;   dh_total = rho (g dy - h rho^2 mean(g dy h)) + dh,   dg = sum over rows of dy h rho.
// Sums are fp32 in a fixed order.  Every tensor passes once: bound by memory.  16384 x 5120 bf16: forward with the residual 110 us (671 MB, 6.1 TB/s),
// backward with dh and dg 134 (5.0 TB/s) and 5 for the sum of dg; 8192 x 4096 with 8-bit rows 55 us (302 MB, 5.5 TB/s); a row of 4096 3.3 us.
#include "norm.hpp"

#include "fp8.hpp"
#include "gemm.hpp"
#include "lanes.hpp"

namespace rl {
namespace {

// A row is held by P threads, V pieces of 16 bytes each: piece k of a thread is the row's piece k P + (its place among the P).
template <int P>
struct Shape {
  static constexpr int kThreads = P > 256 ? P : 256;
  static constexpr int kRows = kThreads / P;  // rows side by side in a workgroup
};

// sum over the P threads of a row
template <int P>
__device__ __forceinline__ float row_sum(float v, float* part) {
  if constexpr (P <= 64) {
    return lanes_sum<P>(v);
  } else {
    v = lanes_sum<64>(v);
    __syncthreads();  // (what was read of the last row's)
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = part[0];
#pragma unroll
    for (int k = 1; k < P / 64; ++k) s += part[k];
    return s;
  }
}

template <typename T, int P, int V, bool Q>
__global__ __launch_bounds__(Shape<P>::kThreads) void norm_forward_kernel(NormDesc g) {
  constexpr int E = Piece<T>::N, ROWS = Shape<P>::kRows;
  __shared__ float part[16];
  const int own = threadIdx.x % P;
  const int pieces = (int)(g.d / E);
  const float scale = 1.f / (float)g.d;
  const T* const gain = static_cast<const T*>(g.gain);
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < g.n; r0 += (int64_t)gridDim.x * ROWS) {
    const int64_t row = r0 + threadIdx.x / P;
    const bool there = row < g.n;
    Piece<T> h[V], w[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int c = k * P + own;
      const bool ok = there && c < pieces;
      h[k] = ok ? Piece<T>::load(static_cast<const T*>(g.X) + row * g.ldx + (uint32_t)(c * E)) : Piece<T>::zero();
      w[k] = ok && g.R != nullptr ? Piece<T>::load(static_cast<const T*>(g.R) + row * g.ldr + (uint32_t)(c * E)) : Piece<T>::zero();
    }
    float sq = 0.f;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float a[E];
      h[k].get(a);
      if (g.R != nullptr) {
        float b[E];
        w[k].get(b);
#pragma unroll
        for (int e = 0; e < E; ++e) a[e] += b[e];
        h[k] = Piece<T>::of(a);
        h[k].get(a);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) sq += a[e] * a[e];
      const int c = k * P + own;
      if (g.H != nullptr && there && c < pieces) h[k].store(static_cast<T*>(g.H) + row * g.ldh + (uint32_t)(c * E), g.stream);
    }
    const float rstd = rsqrtf(row_sum<P>(sq, part) * scale + g.eps);
    if (g.rstd != nullptr && there && own == 0) g.rstd[row] = rstd;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int c = k * P + own;
      const bool ok = there && c < pieces;
      float a[E];
      h[k].get(a);
#pragma unroll
      for (int e = 0; e < E; ++e) a[e] *= rstd;
      if (gain != nullptr) {
        float b[E];
        (ok ? Piece<T>::load(gain + (uint32_t)(c * E)) : Piece<T>::zero()).get(b);
#pragma unroll
        for (int e = 0; e < E; ++e) a[e] *= b[e];
      }
      const Piece<T> y = Piece<T>::of(a);
      if (ok) y.store(static_cast<T*>(g.Y) + row * g.ldy + (uint32_t)(c * E), g.stream);
      if constexpr (Q) {
        // 16 lanes hold a block of 128 columns (E = 8): the rows that the 8-bit layers would make of y
        y.get(a);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint32_t b = __float_as_uint(ok ? a[e] : 0.f) & 0x7FFFFFFFu;
          top = top > b ? top : b;
        }
        top = lanes_max<16>(top);
        uint32_t byte;
        float mul;
        bool nan;
        fp8_block_scale(top, &byte, &mul, &nan);
        typedef __attribute__((__vector_size__(2 * sizeof(int)))) int v2;
        v2 out = {fp8_pack4(a[0] * mul, a[1] * mul, a[2] * mul, a[3] * mul), fp8_pack4(a[4] * mul, a[5] * mul, a[6] * mul, a[7] * mul)};
        if (nan) out = v2{0x7F7F7F7F, 0x7F7F7F7F};
        if (!ok) out = v2{0, 0};
        if (there && (int64_t)c * E < g.ldq) {
          *reinterpret_cast<v2*>(g.q + row * g.ldq + (int64_t)c * E) = out;
          if ((c & 15) == 0) g.qs[(int64_t)(c >> 4) * g.ldqs + row] = (uint8_t)byte;
        }
      }
    }
  }
}

// Workgroups walk over the rows; what a thread adds to dg stays in its registers, and the workgroup leaves one row of sums.  (16384 x 5120, a pass: 255 us,
// without the next row on its way 283.)
template <typename T, int P, int V, bool G>
__global__ __launch_bounds__(Shape<P>::kThreads) void norm_backward_kernel(NormDesc g, float* partial) {
#pragma clang fp contract(off)  // (dx is the same bits with and without dg)
  constexpr int E = Piece<T>::N, ROWS = Shape<P>::kRows;
  __shared__ float part[16];
  __shared__ float cols[G && ROWS > 1 ? ROWS : 1][G && ROWS > 1 ? P * V * E : 1];
  int own = threadIdx.x % P;
  const int pieces = (int)(g.d / E);
  const float scale = 1.f / (float)g.d;
  const T* const gain = static_cast<const T*>(g.gain);
  float dg[G ? V : 1][E];
#pragma unroll
  for (int k = 0; k < (G ? V : 1); ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) dg[k][e] = 0.f;
  // A row's pieces, the next row's on their way while this one's are used; of the widest rows, where both would not fit the registers with dg, this one's
  // alone, in twice the threads (4096 x 32768, a pass over bf16 / f32: 190 / 344 us; by 512 threads that read a row twice 225 / 425).
  constexpr bool AHEAD = V <= 4 && P <= 512;
  static_assert(AHEAD || ROWS == 1);
  auto piece = [&](const void* t, int64_t ld, int64_t row, int k) {
    const int c = k * P + own;
    return t != nullptr && row < g.n && c < pieces ? Piece<T>::load(static_cast<const T*>(t) + row * ld + (uint32_t)(c * E)) : Piece<T>::zero();
  };
  auto fetch = [&](int64_t row, Piece<T> (&h)[V], Piece<T> (&y)[V], Piece<T> (&b)[V], float& rstd) {
    rstd = row < g.n ? g.rstd[row] : 0.f;
    if constexpr (AHEAD) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        h[k] = piece(g.X, g.ldx, row, k);
        y[k] = piece(g.dY, g.lddy, row, k);
        b[k] = piece(g.dH, g.lddh, row, k);
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * ROWS;
  Piece<T> h[V], y[V], b[V], h2[V], y2[V], b2[V];
  float rstd, rstd2 = 0.f;
  int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / P;
  fetch(row, h, y, b, rstd);
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < g.n; r0 += step, row += step) {
    const bool there = row < g.n;
    if (r0 + step < g.n) fetch(row + step, h2, y2, b2, rstd2);
    if constexpr (!AHEAD) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = k * P + own < pieces ? k * P + own : 0;  // (behind the row its first piece, unused: as many zeros would take registers too)
        h[k] = Piece<T>::load(static_cast<const T*>(g.X) + row * g.ldx + (uint32_t)(c * E));
        y[k] = Piece<T>::load(static_cast<const T*>(g.dY) + row * g.lddy + (uint32_t)(c * E));
      }
    }
    auto get_b = [&](int k, float (&f)[E]) { if constexpr (AHEAD) b[k].get(f); else piece(g.dH, g.lddh, row, k).get(f); };
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if constexpr (!AHEAD) asm volatile("" : "+v"(own)::"memory");  // (one piece after the other: addresses and gains of all would not fit)
      const int c = k * P + own;
      if (!AHEAD && c >= pieces) continue;  // (otherwise those behind the row are zero)
      float a[E], u[E], w[E];
      h[k].get(a);
      y[k].get(u);
      (gain != nullptr && c < pieces ? Piece<T>::load(gain + (uint32_t)(c * E)) : Piece<T>::zero()).get(w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xhat = a[e] * rstd;
        if constexpr (G) dg[k][e] = __builtin_fmaf(u[e], xhat, dg[k][e]);
        dot = __builtin_fmaf(gain != nullptr ? u[e] * w[e] : u[e], xhat, dot);
      }
    }
    if (g.dX != nullptr) {
      const float mean = row_sum<P>(dot, part) * scale;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int c = k * P + own;
        if (!there || c >= pieces) continue;
        float a[E], u[E], z[E], w[E];
        h[k].get(a);
        y[k].get(u);
        get_b(k, z);
        (gain != nullptr ? Piece<T>::load(gain + (uint32_t)(c * E)) : Piece<T>::zero()).get(w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float v = __builtin_fmaf(a[e] * rstd, -mean, gain != nullptr ? u[e] * w[e] : u[e]);
          z[e] = g.dH != nullptr ? __builtin_fmaf(rstd, v, z[e]) : rstd * v;
        }
        Piece<T>::of(z).store(static_cast<T*>(g.dX) + row * g.lddx + (uint32_t)(c * E), g.stream);
      }
    }
    rstd = rstd2;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      h[k] = h2[k];
      y[k] = y2[k];
      b[k] = b2[k];
    }
  }
  if constexpr (G) {
    float* const out = partial + (int64_t)blockIdx.x * g.d;
    if constexpr (ROWS == 1) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (k * P + own < pieces)
#pragma unroll
          for (int e = 0; e < E; ++e) out[(int64_t)(k * P + own) * E + e] = dg[k][e];
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) cols[threadIdx.x / P][(k * P + own) * E + e] = dg[k][e];
      __syncthreads();
      for (int c = threadIdx.x; c < (int)g.d; c += Shape<P>::kThreads) {
        float s = cols[0][c];
#pragma unroll
        for (int r = 1; r < ROWS; ++r) s += cols[r][c];
        out[c] = s;
      }
    }
  }
}

// dg = the sum of the partial rows: 32 columns a workgroup, 32 threads a column, which take the rows k, k + 32, .. in order
template <typename T>
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float* __restrict__ partial, int rows, int d, T* __restrict__ out) {
  __shared__ float part[32][33];
  const int c = threadIdx.x & 31, k = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int r = k; r < rows; r += 32) s += partial[(int64_t)r * d + col];
  }
  part[k][c] = s;
  __syncthreads();
  // (threads 32 c .. 32 c + 31 hold column c now)
  s = lanes_sum<32>(part[c][k]);
  if (c == 0 && (int)blockIdx.x * 32 + k < d) out[blockIdx.x * 32 + k] = (T)s;
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// calls f(P, V) as compile-time values: the smallest that holds a row of `pieces`
template <int P_, int V_> struct Hold { static constexpr int P = P_, V = V_; };
template <typename T, typename F>
hipError_t by_width(int64_t pieces, F&& f) {
  if (pieces <= 16) return f(Hold<16, 1>());
  if (pieces <= 32) return f(Hold<32, 1>());
  if (pieces <= 64) return f(Hold<64, 1>());
  if (pieces <= 128) return f(Hold<64, 2>());
  if (pieces <= 256) return f(Hold<256, 1>());
  if (pieces <= 512) return f(Hold<256, 2>());
  if (pieces <= 768) return f(Hold<256, 3>());
  if (pieces <= 1024) return f(Hold<256, 4>());
  if (pieces <= 2048) return f(Hold<512, 4>());
  if constexpr (sizeof(T) == 4) {
    if (pieces > 4096) return f(Hold<1024, 8>());
  }
  return f(Hold<1024, 4>());
}
int64_t rows_at_once(int64_t pieces) { return pieces <= 16 ? 16 : (pieces <= 32 ? 8 : (pieces <= 128 ? 4 : 1)); }

constexpr int64_t kForwardGroups = 1 << 16;  // workgroups; beyond that they walk over rows
// The backward's: as many as are at work at once, four to a compute unit, two where the pieces held ahead fill the registers, one of 1024 threads (16384 x
// 5120: 251 us a pass with 512, 255 with 1024, 279 with 768; 4096 x 32768: 190 us with 256, 202 with 512, whose rows of sums are 64 MB).
int64_t backward_groups(int64_t n, int64_t pieces) {
  const int64_t g = ceil_div(n, rows_at_once(pieces)), most = pieces > 2048 ? 256 : (pieces > 512 ? 512 : 1024);
  return g < most ? g : most;
}

template <typename T>
hipError_t forward_t(const NormDesc& d, hipStream_t s) {
  const int64_t pieces = d.d / Piece<T>::N;
  return by_width<T>(pieces, [&](auto hold) {
    constexpr int P = decltype(hold)::P, V = decltype(hold)::V;
    int64_t groups = ceil_div(d.n, Shape<P>::kRows);
    if (groups > kForwardGroups) groups = kForwardGroups;
    const dim3 grid((unsigned)groups), block(Shape<P>::kThreads);
    if constexpr (sizeof(T) == 2) {
      if (d.q != nullptr) {
        launch_timed(norm_forward_kernel<T, P, V, true>, grid, block, 0, s, d);
        return hipGetLastError();
      }
    }
    launch_timed(norm_forward_kernel<T, P, V, false>, grid, block, 0, s, d);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t backward_t(const NormDesc& d, float* partial, hipStream_t s) {
  const int64_t pieces = d.d / Piece<T>::N, groups = backward_groups(d.n, pieces);
  hipError_t e = by_width<T>(pieces, [&](auto hold) {
    constexpr int P = decltype(hold)::P, V = decltype(hold)::V;
    const dim3 grid((unsigned)groups), block(Shape<P>::kThreads);
    if (d.dgain != nullptr) {
      launch_timed(norm_backward_kernel<T, P, V, true>, grid, block, 0, s, d, partial);
    } else {
      launch_timed(norm_backward_kernel<T, P, V, false>, grid, block, 0, s, d, partial);
    }
    return hipGetLastError();
  });
  if (e != hipSuccess || d.dgain == nullptr) return e;
  launch_timed(norm_gain_kernel<T>, dim3((unsigned)ceil_div(d.d, 32)), dim3(1024), 0, s, static_cast<const float*>(partial), (int)groups, (int)d.d,
               static_cast<T*>(d.dgain));
  return hipGetLastError();
}

bool streams(const NormDesc& d) { return d.n * d.d * (d.dtype == DT_F32 ? 4 : 2) >= kStreamBytes; }

}  // namespace

hipError_t norm_forward(const NormDesc& desc, hipStream_t s) {
  NormDesc d = desc;
  d.stream = streams(d);
  if (d.dtype == DT_F32) return forward_t<float>(d, s);
  return d.dtype == DT_BF16 ? forward_t<__bf16>(d, s) : forward_t<_Float16>(d, s);
}
size_t norm_backward_workspace(int dtype, int64_t n, int64_t d, bool dgain) {
  return dgain ? (size_t)(backward_groups(n, d / (dtype == DT_F32 ? 4 : 8)) * d) * 4 : 0;
}
hipError_t norm_backward(const NormDesc& desc, void* workspace, hipStream_t s) {
  NormDesc d = desc;
  d.stream = streams(d);
  float* const partial = static_cast<float*>(workspace);
  if (d.dtype == DT_F32) return backward_t<float>(d, partial, s);
  return d.dtype == DT_BF16 ? backward_t<__bf16>(d, partial, s) : backward_t<_Float16>(d, partial, s);
}

}  // namespace rl
