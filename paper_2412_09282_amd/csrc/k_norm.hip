// The norm after a block, its gate and scale, the residual sum, and the norm before the next block, in one pass over the rows:
//   u = x, or n(x) w_post + b_post;   r' = r + alpha (g u);   h = n(r') w_pre + b_pre, as it is or in 8 bits
// with n(x) = x / sqrt(mean x^2 + eps), or (x - mean x) / sqrt(mean (x - mean x)^2 + eps).
// A row stays in the registers of its threads between its sums, so that x, r and g are read and r' and h written once: memory
// bounds it.  Sums, means and the root are fp64: no finite row overflows or loses what is left of a large mean, and
// the vector units have room for them beside the memory.  h is of r' before its rounding to its stored type.
#include "row_tile.h"

namespace crvq {
namespace {

struct NormArgs {
  NormDesc d;
  int64_t T;
};

// Long rows fill the registers: the work of a vector ends before the next one's begins.
template <int V>
__device__ __forceinline__ void one_by_one(float (&x)[8]) {
  if constexpr (V > 2) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(x[e]));  // nor is its fp64 form kept for later
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <typename Tile, int V>
__device__ __forceinline__ void normed(const Tile& tile, float (&x)[V][8], bool layer, const void* w, const void* b, bool w_f32,
                                       double eps, double* red) {
  const double n = static_cast<double>(tile.N);
  double s = 0.0, by = 1.0;
  if (layer) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      one_by_one<V>(x[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += static_cast<double>(x[v][e]);  // past N they are 0
    }
    // x - mean leaves fp32's range only where the mean is near it, and is then held by halves; a mean that large leaves no
    // difference so small that half of it is not fp32's
    const double mean = tile.sum(s, red) / n;
    by = fabs(mean) >= 0x1p100 ? 0.5 : 1.0;
    const double from = -mean * by;
    s = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      one_by_one<V>(x[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double y = tile.has(v, e) ? fma(static_cast<double>(x[v][e]), by, from) : 0.0;
        s = fma(y, y, s);
        x[v][e] = static_cast<float>(y);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      one_by_one<V>(x[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fma(static_cast<double>(x[v][e]), static_cast<double>(x[v][e]), s);
    }
  }
  const double inv = 1.0 / (sqrt(tile.sum(s, red + 16) / (n * by * by) + eps) * by);
  // |x| inv is at most sqrt(N) whatever the row's size, but inv itself may leave fp32's range where eps is 0
  const float f = static_cast<float>(inv);
  if (f < __builtin_inff() && f >= 0x1p-126f) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= f;
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      one_by_one<V>(x[v]);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] = static_cast<float>(static_cast<double>(x[v][e]) * inv);
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    one_by_one<V>(x[v]);
    float y[8];
    if (w) {
      tile.load(w, w_f32, v, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= y[e];
    }
    if (b) {
      tile.load(b, w_f32, v, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] += y[e];
    }
  }
}

template <typename X, typename R, typename Tile>
__global__ __launch_bounds__(Tile::kBlock) void norm_kernel(const NormArgs a) {
  constexpr int V = Tile::kVectors;
  __shared__ double red_all[Tile::kRows][4 * 16];  // an array of its own for every sum
  __shared__ uint32_t red_max[Tile::kRows][16];
  const NormDesc& d = a.d;
  Tile tile;
  tile.N = static_cast<int>(d.N);
  tile.t = threadIdx.x % Tile::kThreads;
  const int mine = threadIdx.x / Tile::kThreads;
  double* red = red_all[mine];
  // rows past the last one repeat it and store nothing, since rows of two waves share barriers
  const int64_t at = static_cast<int64_t>(blockIdx.x) * Tile::kRows + mine, row = at < a.T ? at : a.T - 1;
  const bool there = at < a.T;
  float x[V][8], y[V <= 2 ? V : 1][8];
  const R* r = static_cast<const R*>(d.r) + row * d.ldr;
#pragma unroll
  for (int v = 0; v < V; ++v) tile.load(static_cast<const X*>(d.x) + row * d.ldx, v, x[v]);
  if (V <= 2 && d.r) {  // on its way while x is summed
#pragma unroll
    for (int v = 0; v < V; ++v) tile.load(r, v, y[v % 2]);
  }
  if (d.post) normed(tile, x, d.layer, d.w_post, d.b_post, d.w_f32, d.eps, red);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    one_by_one<V>(x[v]);
    if (d.gate) {
      float g[8];
      tile.load(static_cast<const X*>(d.gate) + row * d.ldg, v, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= g[e];
    }
    float z[8];
    if (V > 2 && d.r) tile.load(r, v, z);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[v][e] *= d.alpha;
      if (d.r) x[v][e] += V <= 2 ? y[v % 2][e] : z[e];
      if (!tile.has(v, e)) x[v][e] = 0.f;
    }
    if (d.r_out && there) tile.store(static_cast<R*>(d.r_out) + row * d.ldro, v, x[v]);
  }
  if (!d.h) return;
  normed(tile, x, d.layer, d.w_pre, d.b_pre, d.w_f32, d.eps, red + 32);
  if (d.h_scale) {
    tile.quantize(x, static_cast<int8_t*>(d.h) + row * d.ldh, d.h_scale + row, red_max[mine], there);
  } else if (there) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      one_by_one<V>(x[v]);
      tile.store(static_cast<X*>(d.h) + row * d.ldh, v, x[v]);
    }
  }
}

template <typename X, typename R>
hipError_t norm_as(const NormArgs& a, hipStream_t stream) {
  return with_row_tile(a.d.N, [&](auto tile) {
    using Tile = decltype(tile);
    norm_kernel<X, R, Tile><<<dim3(static_cast<uint32_t>(cdiv(a.T, Tile::kRows))), Tile::kBlock, 0, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_norm(const NormDesc& d, int64_t T, int x_type, int r_type, hipStream_t stream) {
  const NormArgs a = {d, T};
  const bool xf = x_type == ET_F32, rf = r_type == ET_F32;
  if (xf) return rf ? norm_as<uint32_t, uint32_t>(a, stream) : norm_as<uint32_t, uint16_t>(a, stream);
  return rf ? norm_as<uint16_t, uint32_t>(a, stream) : norm_as<uint16_t, uint16_t>(a, stream);
}

}  // namespace crvq
