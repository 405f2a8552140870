// Matrices in 8 bits with a scale for each row, and the product y[t][r] = sx[t] sw[r] sum_j cx[t][j] cw[r][j] of two of
// them (activations by tokens, weights by output channels).  The sums are exact integers of 32 bits, so neither the order
// of their terms nor how they are divided changes a result.
#include "row_tile.h"

namespace crvq {
namespace {

typedef int w8_i4 __attribute__((ext_vector_type(4)));
typedef int w8_i16 __attribute__((ext_vector_type(16)));

// A row to its codes: one pass over the data, the row in registers between its largest magnitude and its codes.
template <typename X, typename Tile>
__global__ __launch_bounds__(Tile::kBlock) void w8_quantize_kernel(const X* X_, int64_t ldx, int64_t rows, int N, int8_t* codes,
                                                                   int64_t ld, float* scales) {
  __shared__ uint32_t red[Tile::kRows][16];
  Tile tile;
  tile.N = N;
  tile.t = threadIdx.x % Tile::kThreads;
  const int mine = threadIdx.x / Tile::kThreads;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * Tile::kRows + mine, row = at < rows ? at : rows - 1;
  float x[Tile::kVectors][8];
#pragma unroll
  for (int v = 0; v < Tile::kVectors; ++v) tile.load(X_ + row * ldx, v, x[v]);
  tile.quantize(x, codes + row * ld, scales + row, red[mine], at < rows);
}

constexpr int64_t kMostLd = int64_t{1} << 22;

struct W8Args {
  W8 w, x;
  void* y;
  int64_t ldy;
  int N, y_f32, y_vec;  // y_vec: rows of y take stores of four elements
  int splits;           // of the columns; more than one: sums go to part[split][T][M]
  int* part;
};

__device__ __forceinline__ uint32_t pair(float a, float b) {  // to bf16, nearest even; a NaN stays one
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((row_f2{a, b}), row_b2));
}

__device__ __forceinline__ void put(const W8Args& a, int64_t t, int64_t r, int sum) {
  const float v = static_cast<float>(sum) * (a.x.scales[t] * a.w.scales[r]);
  if (a.y_f32) static_cast<float*>(a.y)[t * a.ldy + r] = v;
  else static_cast<uint16_t*>(a.y)[t * a.ldy + r] =
      static_cast<uint16_t>(pair(v, 0.f));
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

// Many tokens: a workgroup has BM rows of the matrix by BT tokens, its waves 32 x 32 tiles of them in registers.  128 columns of
// both operands lie in LDS, and the next 128 are on their way there, straight from memory (buffer loads to LDS) while
// the matrix instructions run.  A row's eight pieces of 16 columns are stored at piece ^ (row / 2 % 8), so that the 16 rows that are
// read at once lie in different banks.
template <int BM, int BT, int WM, int WT, int STAGES>
__global__ __launch_bounds__(WM * WT * 64) void w8_tile_kernel(const W8Args a, int tiles_m, int tiles_t) {
  constexpr int kWaves = WM * WT, MI = BM / WM / 32, TI = BT / WT / 32;  // 32 x 32 tiles of a wave
  constexpr int kBuffer = (BM + BT) * 128, kLoads = (BM + BT) / 8 / kWaves;  // a wave's loads of 8 rows
  static_assert(BM / 8 % kWaves == 0 && BT / 8 % kWaves == 0, "a wave's loads are of one operand each");
  extern __shared__ __align__(16) uint8_t lds[];  // [STAGES][BM + BT][128]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroups go round the eight dies: each die gets a run of tiles, four token tiles wide, whose operands its cache holds.
  int id = blockIdx.x;
  {
    const int n = gridDim.x, per = n >> 3, rest = n & 7, die = id & 7;
    id = die * per + min(die, rest) + (id >> 3);
  }
  const int wide = 4 * tiles_m, band = id / wide, in_band = min(4, tiles_t - band * 4);
  id -= band * wide;
  const int tm = id / in_band, tt = band * 4 + id - tm * in_band;
  const int64_t row0 = static_cast<int64_t>(tm) * BM, tok0 = static_cast<int64_t>(tt) * BT;
  const int rows = static_cast<int>(min<int64_t>(BM, a.w.rows - row0)), toks = static_cast<int>(min<int64_t>(BT, a.x.rows - tok0));
  const int end = (a.N + 15) & ~15;
  const auto rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(a.w.codes + row0 * a.w.ld), 0,
                                                    static_cast<int>((rows - 1) * a.w.ld) + end, 0x00027000);
  const auto rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(a.x.codes + tok0 * a.x.ld), 0,
                                                    static_cast<int>((toks - 1) * a.x.ld) + end, 0x00027000);
  // the lane's place in each load; rows past the last one repeat it
  uint32_t from[kLoads];
  int chunk[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (i * kWaves + wave) * 8 + (lane >> 3), in = row < BM ? row : row - BM;
    chunk[i] = ((lane & 7) ^ ((in >> 1) & 7)) * 16;
    from[i] = static_cast<uint32_t>(row < BM ? min(in, rows - 1) * a.w.ld : min(in, toks - 1) * a.x.ld) + chunk[i];
  }
  auto fetch = [&](int k0, int buffer) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      // pieces past the row's end: past the buffer's end, which reads zeros
      const uint32_t at = k0 + chunk[i] < end ? from[i] : 0x80000000u;
      auto* to = reinterpret_cast<__attribute__((address_space(3))) void*>(
          static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds + buffer * kBuffer + (i * kWaves + wave) * 1024)));
      if (i < BM / 8 / kWaves) __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, to, 16, at, k0, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, to, 16, at, k0, 0, 0);
    }
  };
  const int wm = wave / WT, wt = wave % WT, r = lane & 31, half = lane >> 5;
  w8_i16 acc[MI][TI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < TI; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
  const int swz = (r >> 1) & 7;
  auto compute = [&](const uint8_t* from_lds, int k0, auto tail) {
    const uint8_t* w = from_lds + (wm * (BM / WM) + r) * 128;
    const uint8_t* x = from_lds + (BM + wt * (BT / WT) + r) * 128;
    w8_i4 wv[2][MI], xv[2][TI];
    auto read = [&](int s) {
      const int at = ((2 * s + half) ^ swz) * 16;
#pragma unroll
      for (int j = 0; j < TI; ++j) xv[s & 1][j] = *reinterpret_cast<const w8_i4*>(x + j * 4096 + at);
#pragma unroll
      for (int i = 0; i < MI; ++i) wv[s & 1][i] = *reinterpret_cast<const w8_i4*>(w + i * 4096 + at);
      if constexpr (decltype(tail)::value) {  // columns from N on: zeros in one operand
        const int n = a.N - (k0 + (2 * s + half) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int b = min(max(n - 4 * e, 0), 4);
          const int keep = b == 4 ? -1 : static_cast<int>((1u << (8 * b)) - 1u);
#pragma unroll
          for (int i = 0; i < MI; ++i) wv[s & 1][i][e] &= keep;
        }
      }
    };
    // operands are asked for one step of 32 columns before they are used
    read(0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) read(s + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < TI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv[s & 1][i], xv[s & 1][j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // A step's loads to LDS have arrived (those of the STAGES - 2 steps after it may be on their way), for every wave, and
  // every wave has read what it asked for: by hand, since __syncthreads waits for all loads.
  auto arrived = [&] {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * kLoads) : "memory");
  };
  // this split's steps: first .. last
  const int steps = ((a.N - 1) >> 7) + 1, each = (steps + a.splits - 1) / a.splits, split = blockIdx.y;
  const int first = split * each, last = min(first + each, steps) - 1;
#pragma unroll
  for (int k = 0; k < STAGES - 1; ++k) fetch((first + k) * 128, k);
  int now = 0, next = STAGES - 1;  // the buffers of this step and of the one that is asked for
  for (int k = first; k < last; ++k) {
    arrived();  // this buffer is there, and nobody reads the one before any more
    fetch((k + STAGES - 1) * 128, next);  // past the last step too, zeros: what is waited for stays the same
    compute(lds + now * kBuffer, k * 128, std::false_type{});
    next = now;
    now = now + 1 == STAGES ? 0 : now + 1;
  }
  arrived();
  compute(lds + now * kBuffer, last * 128, std::true_type{});
  // lane (r, half) has token r and rows 8 g + 4 half + 0 .. 3 of a tile
#pragma unroll
  for (int j = 0; j < TI; ++j) {
    const int tok = wt * (BT / WT) + j * 32 + r;
    if (tok >= toks) continue;
    if (a.splits > 1) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int row = wm * (BM / WM) + i * 32 + 8 * g + 4 * half;
          int* to = a.part + (split * a.x.rows + tok0 + tok) * a.w.rows + row0 + row;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (row + e < rows) to[e] = acc[i][j][4 * g + e];
        }
      continue;
    }
    const float sx = a.x.scales[tok0 + tok];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int row = wm * (BM / WM) + i * 32 + 8 * g + 4 * half;
        if (row >= rows) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = static_cast<float>(acc[i][j][4 * g + e]) * (sx * a.w.scales[row0 + min(row + e, rows - 1)]);
        const int64_t at = (tok0 + tok) * a.ldy + row0 + row;
        if (a.y_f32) {
          float* y = static_cast<float*>(a.y) + at;
          if (a.y_vec && row + 4 <= rows) {
            *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
          } else {
            for (int e = 0; e < 4 && row + e < rows; ++e) y[e] = v[e];
          }
        } else {
          uint16_t* y = static_cast<uint16_t*>(a.y) + at;
          const uint32_t p = pair(v[0], v[1]), q = pair(v[2], v[3]);
          if (a.y_vec && row + 4 <= rows) {
            *reinterpret_cast<uint2*>(y) = make_uint2(p, q);
          } else {
            for (int e = 0; e < 4 && row + e < rows; ++e) y[e] = static_cast<uint16_t>((e < 2 ? p : q) >> (16 * (e & 1)));
          }
        }
      }
  }
}

__global__ __launch_bounds__(256) void w8_join_kernel(const W8Args a) {
  const int64_t r = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, t = blockIdx.y;
  if (r >= a.w.rows) return;
  int sum = 0;
  for (int s = 0; s < a.splits; ++s) sum += a.part[(s * a.x.rows + t) * a.w.rows + r];
  put(a, t, r, sum);
}

template <int BM, int BT, int WM, int WT, int STAGES>
hipError_t tile(const W8Args& a, hipStream_t stream) {
  const int64_t tm = cdiv(a.w.rows, BM), tt = cdiv(a.x.rows, BT);
  if (tm * tt > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(tm * tt), static_cast<uint32_t>(a.splits));
  w8_tile_kernel<BM, BT, WM, WT, STAGES><<<grid, WM * WT * 64, STAGES * (BM + BT) * 128, stream>>>(
      a, static_cast<int>(tm), static_cast<int>(tt));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w8_quantize(const void* X, int64_t ldx, int type, int64_t rows, int64_t N, int8_t* codes, int64_t ld,
                              float* scales, hipStream_t stream) {
  auto as = [&](auto* p) {
    using X_ = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
    return with_row_tile(N, [&](auto tile) {
      using Tile = decltype(tile);
      w8_quantize_kernel<X_, Tile><<<dim3(static_cast<uint32_t>(cdiv(rows, Tile::kRows))), Tile::kBlock, 0, stream>>>(
          p, ldx, rows, static_cast<int>(N), codes, ld, scales);
      return hipGetLastError();
    });
  };
  return type == ET_F32 ? as(static_cast<const uint32_t*>(X)) : as(static_cast<const uint16_t*>(X));
}

// How a product is divided.  Up to 64 tokens: 16 or 32 rows a workgroup, the columns over its waves; where there are rows for
// tiles of 64 or 128 on most CUs, these, which read x less often (us, 28672 x 8192 by 16 tokens: 48 with tiles of 64, 58 with 32 rows
// a workgroup; by 32 tokens 48, 69; 8192 x 8192 by 32: 24, 21, and with 16 rows 25; 4096 x 4096 by 32: 12, 11, 8; by
// 64 tokens 28672 x 8192 52 with tiles of 128 and 56 of 64 rows, 13824 x 5120 31, 24 and 42 with 32 rows a workgroup).
// More tokens: the tiles whose rounds on 256 CUs cost least, with the time of a step of 128 columns that each was
// measured to take on a full chip; few of the smallest ones are split along the columns, eight steps at least, and
// joined by a second launch (1000 x 14336 by 100: 14.7 us, unsplit 32).
enum { kFew1, kFew2, kFew12, kFew22, kTile64x32, kTile128x64, kTile64, kTile128, kTile256x128, kTile256 };
constexpr int64_t kRows32 = 6144, kRows64 = 12288, kRows128 = 20480;  // from these on: 32, 64, 128 rows
W8Plan plan_w8(int64_t M, int64_t N, int64_t T, bool far) {
  if (far) return {T <= 16 ? kFew1 : kFew22, 1};
  if (T <= 8) return {kFew1, 1};
  if (T <= 32 && M >= kRows64) return {kTile64x32, 1};
  if (T <= 16) return {M >= kRows32 ? kFew2 : kFew1, 1};
  if (T <= 32) return {M >= kRows32 ? kFew22 : kFew12, 1};
  if (T <= 64 && M >= kRows128) return {kTile128x64, 1};
  if (T <= 64 && M < kRows32) return {kFew22, 1};
  const auto tiles = [&](int64_t m, int64_t t) { return cdiv(M, m) * cdiv(T, t); };
  const int64_t n64 = tiles(64, 64);
  int form = kTile64;
  double best = n64 <= 256 ? 0.42 : 0.65 * cdiv(n64, 512);
  auto consider = [&](int f, int64_t n, double us) {
    if (us * cdiv(n, 256) < best) best = us * cdiv(n, 256), form = f;
  };
  consider(kTile128, tiles(128, 128), 0.78);
  consider(kTile256x128, tiles(256, 128), 1.3);
  consider(kTile256, tiles(256, 256), 2.0);
  const int64_t room = 256 / n64, long_enough = cdiv(N, 128) / 8, n = room < long_enough ? room : long_enough;
  return {form, form == kTile64 && n > 1 ? static_cast<int>(n) : 1};
}

size_t w8_gemm_ws_bytes(int64_t M, int64_t N, int64_t T) {
  const W8Plan p = plan_w8(M, N, T, false);
  WsCursor c(nullptr);
  if (p.splits > 1) c.take<int>(static_cast<size_t>(p.splits) * M * T);
  return c.used;
}

hipError_t launch_w8_gemm(const W8& w, const W8& x, int64_t N, void* y, int64_t ldy, int y_type, void* ws, hipStream_t stream) {
  // a tile's rows lie within 2^31 bytes of its first one
  W8Plan p = plan_w8(w.rows, N, x.rows, w.ld > kMostLd || x.ld > kMostLd);
  WsCursor c(ws);
  W8Args a = {w, x, y, ldy, static_cast<int>(N), y_type == ET_F32, 0, p.splits, nullptr};
  if (p.splits > 1) a.part = c.take<int>(static_cast<size_t>(p.splits) * w.rows * x.rows);
  const int es = a.y_f32 ? 4 : 2;
  a.y_vec = reinterpret_cast<uintptr_t>(y) % (4 * es) == 0 && ldy % 4 == 0;
  hipError_t e = hipSuccess;
  switch (p.form) {
    case kFew1: return few<1, 1, 8>(a, stream);
    case kFew2: return few<2, 1, 8>(a, stream);
    case kFew12: return few<1, 2, 8>(a, stream);
    case kFew22: return few<2, 2, 8>(a, stream);
    case kTile64x32: return tile<64, 32, 2, 1, 4>(a, stream);
    case kTile128x64: return tile<128, 64, 2, 2, 6>(a, stream);
    case kTile128: return tile<128, 128, 4, 2, 4>(a, stream);
    case kTile256x128: return tile<256, 128, 4, 2, 3>(a, stream);
    case kTile256: return tile<256, 256, 4, 4, 2>(a, stream);
    default: e = tile<64, 64, 2, 2, 4>(a, stream);
  }
  if (e != hipSuccess || p.splits == 1) return e;
  w8_join_kernel<<<dim3(static_cast<uint32_t>(cdiv(w.rows, 256)), static_cast<uint32_t>(x.rows)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace crvq
