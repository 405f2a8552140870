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

template <typename Tile, int V>
__device__ __forceinline__ void normed(const Tile& tile, float (&x)[V][8], bool layer, const void* w, const void* b, bool w_f32,
                                       double eps, double* red) {
  const double n = static_cast<double>(tile.N);
  double s = 0.0;
  if (layer) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += static_cast<double>(x[v][e]);  // past N they are 0
    const double mean = tile.sum(s, red) / n;
    s = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double y = tile.has(v, e) ? static_cast<double>(x[v][e]) - mean : 0.0;
        s = fma(y, y, s);
        x[v][e] = static_cast<float>(y);
      }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fma(static_cast<double>(x[v][e]), static_cast<double>(x[v][e]), s);
  }
  const double inv = 1.0 / sqrt(tile.sum(s, red + 16) / n + eps);
  // |x| inv is at most sqrt(N) whatever the row's size, but inv itself may pass fp32's range where eps is 0
  const float f = static_cast<float>(inv);
  const bool far = !(f < __builtin_inff()) || f < 0x1p-126f;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[v][e] = far ? static_cast<float>(static_cast<double>(x[v][e]) * inv) : x[v][e] * f;
  if (w) {
    float y[V][8];
    tile.load(w, w_f32, y);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= y[v][e];
  }
  if (b) {
    float y[V][8];
    tile.load(b, w_f32, y);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] += y[v][e];
  }
}

template <typename X, typename R, typename Tile>
__global__ __launch_bounds__(Tile::kBlock) void norm_kernel(const NormArgs a) {
  constexpr int V = Tile::kVectors;
  __shared__ double red[4 * 16];  // an array of its own for every sum
  __shared__ uint32_t red_max[16];
  const NormDesc& d = a.d;
  Tile tile;
  tile.N = static_cast<int>(d.N);
  tile.t = threadIdx.x % Tile::kThreads;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * Tile::kRows + threadIdx.x / Tile::kThreads;
  if (row >= a.T) return;  // whole waves
  float x[V][8], y[V][8];
  tile.load(static_cast<const X*>(d.x) + row * d.ldx, x);
  if (d.r) tile.load(static_cast<const R*>(d.r) + row * d.ldr, y);
  if (d.post) normed(tile, x, d.layer, d.w_post, d.b_post, d.w_f32, d.eps, red);
  if (d.gate) {
    float g[V][8];
    tile.load(static_cast<const X*>(d.gate) + row * d.ldg, g);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= g[v][e];
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[v][e] *= d.alpha;
      if (d.r) x[v][e] += y[v][e];
      if (!tile.has(v, e)) x[v][e] = 0.f;
    }
  if (d.r_out) tile.store(static_cast<R*>(d.r_out) + row * d.ldro, x);
  if (!d.h) return;
  normed(tile, x, d.layer, d.w_pre, d.b_pre, d.w_f32, d.eps, red + 32);
  if (d.h_scale) tile.quantize(x, static_cast<int8_t*>(d.h) + row * d.ldh, d.h_scale + row, red_max);
  else tile.store(static_cast<X*>(d.h) + row * d.ldh, x);
}

template <typename X, typename R, bool VEC>
hipError_t norm_as(const NormArgs& a, hipStream_t stream) {
  return with_row_tile<VEC>(a.d.N, [&](auto tile) {
    using Tile = decltype(tile);
    norm_kernel<X, R, Tile><<<dim3(static_cast<uint32_t>(cdiv(a.T, Tile::kRows))), Tile::kBlock, 0, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_norm(const NormDesc& d, int64_t T, int x_type, int r_type, hipStream_t stream) {
  const NormArgs a = {d, T};
  // 16-byte loads: rows of whole vectors whose first elements are aligned
  auto fits = [&](const void* p, int64_t ld, int es) { return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * es % 16 == 0); };
  const int xs = x_type == ET_F32 ? 4 : 2, rs = r_type == ET_F32 ? 4 : 2;
  const bool vec = d.N % 8 == 0 && fits(d.x, d.ldx, xs) && fits(d.gate, d.ldg, xs) && fits(d.r, d.ldr, rs) &&
                   fits(d.r_out, d.ldro, rs) && fits(d.h, d.ldh, d.h_scale ? 2 : xs) && fits(d.w_post, 0, 4) &&
                   fits(d.b_post, 0, 4) && fits(d.w_pre, 0, 4) && fits(d.b_pre, 0, 4);
  const bool xf = x_type == ET_F32, rf = r_type == ET_F32;
  if (xf) {
    if (rf) return vec ? norm_as<uint32_t, uint32_t, true>(a, stream) : norm_as<uint32_t, uint32_t, false>(a, stream);
    return vec ? norm_as<uint32_t, uint16_t, true>(a, stream) : norm_as<uint32_t, uint16_t, false>(a, stream);
  }
  if (rf) return vec ? norm_as<uint16_t, uint32_t, true>(a, stream) : norm_as<uint16_t, uint32_t, false>(a, stream);
  return vec ? norm_as<uint16_t, uint16_t, true>(a, stream) : norm_as<uint16_t, uint16_t, false>(a, stream);
}

}  // namespace crvq
