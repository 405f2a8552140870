// Matrices in 8 bits with a scale for each row, and the product y[t][r] = sx[t] sw[r] sum_j cx[t][j] cw[r][j] of two of
// them (activations by tokens, weights by output channels).  The sums are exact integers of 32 bits, so neither the order
// of their terms nor how they are divided changes a result.
#include "row_tile.h"

namespace crvq {
namespace {

typedef int w8_i4 __attribute__((ext_vector_type(4)));

// A row to its codes: one pass over the data, the row in registers between its largest magnitude and its codes.
template <typename X, typename Tile>
__global__ __launch_bounds__(Tile::kBlock) void w8_quantize_kernel(const X* X_, int64_t ldx, int64_t rows, int N, int8_t* codes,
                                                                   int64_t ld, float* scales) {
  __shared__ uint32_t red[16];
  Tile tile;
  tile.N = N;
  tile.t = threadIdx.x % Tile::kThreads;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * Tile::kRows + threadIdx.x / Tile::kThreads;
  if (row >= rows) return;  // whole waves
  float x[Tile::kVectors][8];
  tile.load(X_ + row * ldx, x);
  tile.quantize(x, codes + row * ld, scales + row, red);
}

struct W8Args {
  W8 w, x;
  void* y;
  int64_t ldy;
  int N, y_f32;
};

__device__ __forceinline__ void put(const W8Args& a, int64_t t, int64_t r, int sum) {
  const float v = static_cast<float>(sum) * (a.x.scales[t] * a.w.scales[r]);
  if (a.y_f32) static_cast<float*>(a.y)[t * a.ldy + r] = v;
  else static_cast<uint16_t*>(a.y)[t * a.ldy + r] =
      static_cast<uint16_t>(__builtin_bit_cast(uint32_t, __builtin_convertvector((row_f2{v, 0.f}), row_b2)));
}

// 16 columns of a row from column k on as they are in memory (k a multiple of 16), zeros from column N on.
__device__ __forceinline__ w8_i4 piece(const int8_t* row, int k, int N) {
  if (k >= N) return w8_i4{0, 0, 0, 0};
  w8_i4 v = *reinterpret_cast<const w8_i4*>(row + k);
  const int n = N - k;  // columns that there are
  if (n < 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = min(max(n - 4 * i, 0), 4);
      v[i] = b == 4 ? v[i] : v[i] & static_cast<int>((1u << (8 * b)) - 1u);
    }
  }
  return v;
}

// Few tokens: a workgroup has 16 RT rows of the matrix and 16 TT tokens, and its waves share the columns, 256 at a time; the
// matrix is read once per 16 TT tokens, straight into the operands of the matrix instructions.  Memory bounds it.
template <int RT, int TT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void w8_few_kernel(const W8Args a) {
  constexpr int kTiles = RT * TT;
  __shared__ __align__(16) w8_i4 join[WAVES][kTiles][64];
  const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4, wave = threadIdx.x >> 6;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * (16 * RT), tok0 = static_cast<int64_t>(blockIdx.y) * (16 * TT);
  const int8_t *w[RT], *x[TT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t row = row0 + i * 16 + r;
    w[i] = a.w.codes + (row < a.w.rows ? row : a.w.rows - 1) * a.w.ld;  // rows past the last one repeat it
  }
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    const int64_t tok = tok0 + i * 16 + r;
    x[i] = a.x.codes + (tok < a.x.rows ? tok : a.x.rows - 1) * a.x.ld;
  }
  w8_i4 acc[RT][TT] = {};
  const int whole = a.N / 256 * 256;
  for (int k0 = wave * 256; k0 < a.N; k0 += WAVES * 256) {
    w8_i4 wv[4][RT], xv[4][TT];
    if (k0 < whole) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int i = 0; i < RT; ++i) wv[u][i] = *reinterpret_cast<const w8_i4*>(w[i] + k0 + u * 64 + c * 16);
#pragma unroll
        for (int i = 0; i < TT; ++i) xv[u][i] = *reinterpret_cast<const w8_i4*>(x[i] + k0 + u * 64 + c * 16);
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int i = 0; i < RT; ++i) wv[u][i] = piece(w[i], k0 + u * 64 + c * 16, a.N);
#pragma unroll
        for (int i = 0; i < TT; ++i) xv[u][i] = piece(x[i], k0 + u * 64 + c * 16, a.N);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][i], xv[u][j], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) join[wave][i * TT + j][lane] = acc[i][j];
  __syncthreads();
  // element e: row e % (16 RT) of token e / (16 RT), so that neighbours write neighbouring rows
  for (int e = threadIdx.x; e < kTiles * 256; e += WAVES * 64) {
    const int row = e % (16 * RT), tok = e / (16 * RT), tile = (row >> 4) * TT + (tok >> 4);
    const int at = ((row & 15) >> 2) * 16 + (tok & 15);
    int sum = 0;
#pragma unroll
    for (int v = 0; v < WAVES; ++v) sum += join[v][tile][at][row & 3];
    if (row0 + row < a.w.rows && tok0 + tok < a.x.rows) put(a, tok0 + tok, row0 + row, sum);
  }
}

template <int RT, int TT, int WAVES>
hipError_t few(const W8Args& a, hipStream_t stream) {
  const int64_t gx = cdiv(a.w.rows, 16 * RT), gy = cdiv(a.x.rows, 16 * TT);
  if (gx > 0x7fffffffLL || gy > 65535) return hipErrorInvalidConfiguration;
  w8_few_kernel<RT, TT, WAVES><<<dim3(static_cast<uint32_t>(gx), static_cast<uint32_t>(gy)), WAVES * 64, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w8_quantize(const void* X, int64_t ldx, int type, int64_t rows, int64_t N, int8_t* codes, int64_t ld,
                              float* scales, hipStream_t stream) {
  const int es = type == ET_F32 ? 4 : 2;
  auto as = [&](auto* p, auto vec) {
    using X_ = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
    return with_row_tile<decltype(vec)::value>(N, [&](auto tile) {
      using Tile = decltype(tile);
      w8_quantize_kernel<X_, Tile><<<dim3(static_cast<uint32_t>(cdiv(rows, Tile::kRows))), Tile::kBlock, 0, stream>>>(
          p, ldx, rows, static_cast<int>(N), codes, ld, scales);
      return hipGetLastError();
    });
  };
  const bool vec = N % 8 == 0 && reinterpret_cast<uintptr_t>(X) % 16 == 0 && ldx * es % 16 == 0;
  if (type == ET_F32) {
    const auto* p = static_cast<const uint32_t*>(X);
    return vec ? as(p, std::true_type{}) : as(p, std::false_type{});
  }
  const auto* p = static_cast<const uint16_t*>(X);
  return vec ? as(p, std::true_type{}) : as(p, std::false_type{});
}

size_t w8_gemm_ws_bytes(int64_t M, int64_t N, int64_t T) { return 0; }

hipError_t launch_w8_gemm(const W8& w, const W8& x, int64_t N, void* y, int64_t ldy, int y_type, void* ws, hipStream_t stream) {
  const W8Args a = {w, x, y, ldy, static_cast<int>(N), y_type == ET_F32};
  if (x.rows <= 16) return few<1, 1, 8>(a, stream);
  if (x.rows <= 32) return few<1, 2, 8>(a, stream);
  return few<1, 4, 8>(a, stream);
}

}  // namespace crvq
