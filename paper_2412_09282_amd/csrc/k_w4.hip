// 4-bit matrices with a scale (and a zero point) per group of consecutive columns: quantization,
// reconstruction and the product with a few vectors.
#include "kv_common.h"

namespace crvq {
namespace {

constexpr float kMinScale = 7.888609052210118e-31f;  // 2^-100

template <typename T>
__device__ __forceinline__ float ld1(const T* p) {
  if constexpr (sizeof(T) == 4)
    return *reinterpret_cast<const float*>(p);
  else
    return bf16_f(*p);
}
template <typename T>
__device__ __forceinline__ void st1(T* p, float x) {
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<float*>(p) = x;
  else
    *p = static_cast<T>(f_bf16(x));
}

template <typename TS>
__device__ __forceinline__ float scale_at(const W4& w, int64_t r, int64_t g) {
  return ld1(static_cast<const TS*>(w.scales) + r * w.ld_s + g);
}
__device__ __forceinline__ float zero_at(const W4& w, int64_t r, int64_t g) {
  return w.zeros ? static_cast<float>(w.zeros[r * w.ld_z + g]) : 8.f;
}

// A workgroup's threads are 256 / L rows of L lanes, L a power of two, and L lanes walk a row in blocks of L: no
// division.
struct Lanes {
  int log2;         // of L
  int64_t blocks;   // of L units in a row
};

// ---- quantization: a lane owns eight columns (four bytes of codes), group / 8 lanes share a group -------
template <typename T, typename TS>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const T* W, int64_t ldw, const W4 w, int vec, const Lanes ln,
                                                          int64_t stored) {
  const uint32_t rows = 256u >> ln.log2;
  const int64_t band = blockIdx.x / static_cast<uint32_t>(ln.blocks), part = blockIdx.x % static_cast<uint32_t>(ln.blocks);
  const int64_t r = band * rows + (threadIdx.x >> ln.log2);
  const int64_t j0 = ((part << ln.log2) + (threadIdx.x & ((1 << ln.log2) - 1))) * 8;
  const bool in = r < w.M;
  float x[8];
  float lo = 0.f, hi = 0.f;
  bool finite = true;
  const T* p = W + r * ldw + j0;
  if (vec && in && j0 + 8 <= w.N) {
    if constexpr (sizeof(T) == 4) {
      const uint4 u = ld_stream(p), v = ld_stream(p + 4);
      x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
      x[4] = __uint_as_float(v.x); x[5] = __uint_as_float(v.y); x[6] = __uint_as_float(v.z); x[7] = __uint_as_float(v.w);
    } else {
      const uint4 u = ld_stream(p);
      const uint32_t e[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(e[i] << 16);
        x[2 * i + 1] = __uint_as_float(e[i] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = in && j0 + i < w.N ? ld1(p + i) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    finite &= fabsf(x[i]) < __uint_as_float(0x7f800000u);
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
  if (!finite) hi = __uint_as_float(0x7f800000u);  // and so the scale is not finite
  for (int o = 1; o < 1 << (w.group_log2 - 3); o <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, o));
    hi = fmaxf(hi, __shfl_xor(hi, o));
  }
  if (!in) return;
  float s = fmaxf(w.zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f, kMinScale);
  if (!(s < __uint_as_float(0x7f800000u))) s = __uint_as_float(0x7fc00000u);
  if (sizeof(TS) == 2) s = bf16_f(f_bf16(s));
  const bool number = s == s;
  const float z = !w.zeros ? 8.f : number ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = number && j0 + i < w.N ? fminf(fmaxf(rintf(x[i] / s) + z, 0.f), 15.f) : 0.f;
    c |= static_cast<uint32_t>(static_cast<int>(q)) << (4 * i);
  }
  if (j0 < stored) *reinterpret_cast<uint32_t*>(w.codes + r * w.ld + (j0 >> 1)) = c;
  if ((j0 & ((1 << w.group_log2) - 1)) == 0 && j0 < w.N) {
    const int64_t g = j0 >> w.group_log2;
    st1(static_cast<TS*>(w.scales) + r * w.ld_s + g, s);
    if (w.zeros) w.zeros[r * w.ld_z + g] = static_cast<uint8_t>(z);
  }
}

// ---- reconstruction: a lane owns 16 bytes of the output, so that a wave stores 1 KB at once -------------------
template <typename T, typename TS>
__global__ __launch_bounds__(256) void w4_dequant_kernel(const W4 w, T* out, int64_t ldo, int vec, const Lanes ln) {
  constexpr int E = 16 / sizeof(T);
  const uint32_t rows = 256u >> ln.log2;
  const int64_t band = blockIdx.x / static_cast<uint32_t>(ln.blocks), part = blockIdx.x % static_cast<uint32_t>(ln.blocks);
  const int64_t r = band * rows + (threadIdx.x >> ln.log2);
  const int64_t j0 = ((part << ln.log2) + (threadIdx.x & ((1 << ln.log2) - 1))) * E;
  if (r >= w.M || j0 >= w.N) return;
  const uint8_t* p = w.codes + r * w.ld + (j0 >> 1);
  const uint32_t c = E == 8 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
  const float s = scale_at<TS>(w, r, j0 >> w.group_log2), z = zero_at(w, r, j0 >> w.group_log2);
  float x[E];
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = (static_cast<float>((c >> (4 * i)) & 15) - z) * s;
  T* o = out + r * ldo + j0;
  if (vec && j0 + E <= w.N) {
    if constexpr (E == 4)
      st_stream(o, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])));
    else
      st_stream(o, make_uint4(f_bf16x2(x[0], x[1]), f_bf16x2(x[2], x[3]), f_bf16x2(x[4], x[5]), f_bf16x2(x[6], x[7])));
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (j0 + i < w.N) st1(o + i, x[i]);
  }
}

// ---- product ----------------------------------------------------------------------------------------------
// A step is 16 rows of W by 128 columns: lane l = 16 c + r loads the 16 bytes of row r's columns 32 c .. 32 c + 31,
// so a wave reads 1 KB with one load and every lane's codes belong to one group.  Each of the four words is
// turned into eight bf16 numbers 16 + code (code in the upper mantissa bits of 16: a shift and an and-or for two), the
// right operand of one v_mfma_f32_16x16x32_bf16; the left one holds x.  What that instruction would add up over the four
// quarters c, different groups when group < 128, is kept apart by its 16 left rows: they are 16 / TB segments of
// TB vectors, and the row of (segment, vector) holds x in the segment's quarters and zeros elsewhere.  TB = 4, 8,
// 16 gives segments of 32, 64, 128 columns.  A fifth to eighth instruction with ones on the right gives the
// segment's sum X of x, and a row's total takes  s (acc - (16 + z) X),  where acc and X are fp32.
// Waves of a workgroup share the rows and take every waves-th step of the columns; x (fp32: three bf16 terms, which
// hold all of its 24 bits, as three vectors) waits in LDS in the order of the codes, all of it or a chunk of columns
// at a time.
typedef __bf16 w4_bf8 __attribute__((ext_vector_type(8)));
typedef float w4_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t w4_u4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 128;    // columns of a step
constexpr int kXPad = 8;      // elements between rows of x in LDS
constexpr int kXBytes = 68 << 10;  // two workgroups a CU

struct GemvArgs {
  W4 w;
  const void* x;
  void* y;
  int64_t ldx, ldy, T;
  int x_f32, y_f32, x_vec;
  int per_pass;  // vectors of one workgroup (grid y passes)
  int steps;     // steps of a wave within a chunk of columns
  int chunks;
};

// Two bf16 of x in the order of the codes' halves: (u.lo, v.lo) and (u.hi, v.hi).
__device__ __forceinline__ uint32_t lo2(uint32_t u, uint32_t v) { return __builtin_amdgcn_perm(v, u, 0x05040100u); }
__device__ __forceinline__ uint32_t hi2(uint32_t u, uint32_t v) { return __builtin_amdgcn_perm(v, u, 0x07060302u); }

// Eight codes of a word as bf16 16 + code, columns 0 4 1 5 2 6 3 7.
__device__ __forceinline__ w4_bf8 widen8(uint32_t c) {
  constexpr uint32_t mask = 0x00780078u, base = 0x41804180u;
  const w4_u4 v = {((c << 3) & mask) | base, ((c >> 1) & mask) | base, ((c >> 5) & mask) | base, ((c >> 9) & mask) | base};
  return __builtin_bit_cast(w4_bf8, v);
}

// x[t][j .. j+7] to LDS, in the codes' order; zero past column N.
__device__ __forceinline__ void stage8(const GemvArgs& a, int64_t t, int64_t j, uint16_t* xs, int ld, int row, int rows) {
  if (a.x_f32) {
    const float* p = static_cast<const float*>(a.x) + t * a.ldx + j;
    float x[8];
    if (a.x_vec && j + 8 <= a.w.N) {
      const float4 u = reinterpret_cast<const float4*>(p)[0], v = reinterpret_cast<const float4*>(p)[1];
      x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = j + i < a.w.N ? p[i] : 0.f;
    }
#pragma unroll
    for (int term = 0; term < 3; ++term) {  // the upper halves, then what they leave
      uint4 o;
      o.x = hi2(__float_as_uint(x[0]), __float_as_uint(x[4]));
      o.y = hi2(__float_as_uint(x[1]), __float_as_uint(x[5]));
      o.z = hi2(__float_as_uint(x[2]), __float_as_uint(x[6]));
      o.w = hi2(__float_as_uint(x[3]), __float_as_uint(x[7]));
      *reinterpret_cast<uint4*>(xs + (row + term * rows) * ld) = o;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(a.x) + t * a.ldx + j;
    uint4 u;
    if (a.x_vec && j + 8 <= a.w.N) {
      u = *reinterpret_cast<const uint4*>(p);
    } else {
      uint32_t e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = j + i < a.w.N ? p[i] : 0u;
      u = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    }
    *reinterpret_cast<uint4*>(xs + row * ld) = make_uint4(lo2(u.x, u.z), hi2(u.x, u.z), lo2(u.y, u.w), hi2(u.y, u.w));
  }
}

// NB blocks of TB vectors; NR of a lane's four sums of a block in use; RB blocks of 16 rows; U steps loaded at once.
template <int TB, int NB, int NR, int RB, int U, typename TS>
__global__ __launch_bounds__(1024) void w4_gemv_kernel(const GemvArgs a) {
  extern __shared__ __align__(16) uint16_t xs[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
  const int r = lane & 15, c = lane >> 4;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * (16 * RB);
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * a.per_pass;
  const int nt = static_cast<int>(min(a.T - t0, static_cast<int64_t>(a.per_pass)));
  const int held = a.x_f32 ? 3 * nt : nt;  // rows of x in LDS
  const int chunk_cols = a.steps * waves * kStep, ld = chunk_cols + kXPad;
  uint16_t* zero = xs + held * ld;         // eight zeros, for rows of other segments

  // weights: this lane's row of every block, its 32 columns
  const uint8_t* codes[RB];
  const TS* scales[RB];
  const uint8_t* zeros[RB];
  const int64_t stored = (a.w.N + 31) & ~int64_t{31}, last_group = (a.w.N - 1) >> a.w.group_log2;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int64_t row = min(row0 + b * 16 + r, a.w.M - 1);
    codes[b] = a.w.codes + row * a.w.ld;
    scales[b] = static_cast<const TS*>(a.w.scales) + row * a.w.ld_s;
    zeros[b] = a.w.zeros ? a.w.zeros + row * a.w.ld_z : nullptr;
  }
  const int seg_col = ((c * 4) / TB) * (8 * TB);  // first column of the segment whose sums this lane holds
  uint4 wq[U][RB];
  float sc[U][RB], zp[U][RB];
  auto column = [&](int n) {  // first column of this wave's n-th step
    const int chunk = n / a.steps;
    return static_cast<int64_t>(chunk) * chunk_cols + static_cast<int64_t>((n - chunk * a.steps) * waves + wave) * kStep;
  };
  auto load = [&](int n) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t kb = column(n + u);
      if (kb >= a.w.N) break;
      const int64_t col = kb + 32 * c, g = min((kb + seg_col) >> a.w.group_log2, last_group);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        wq[u][b] = ld_stream(codes[b] + (col < stored ? col >> 1 : 0));
        sc[u][b] = ld1(scales[b] + g);
        zp[u][b] = zeros[b] ? static_cast<float>(zeros[b][g]) : 8.f;
      }
    }
  };

  w4_f4 tot[RB][NB];
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n) tot[b][n] = w4_f4{0.f, 0.f, 0.f, 0.f};
  // left operand: this lane's row is a vector of a segment; it reads x where the segment has this lane's columns
  const uint16_t* xp[NB];
  int xstep[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int v = n * TB + (r & (TB - 1));
    const bool live = r / TB == (c * 4) / TB && v < held;
    xp[n] = live ? xs + v * ld + 32 * c : zero;
    xstep[n] = live ? 1 : 0;
  }
  const w4_bf8 ones = __builtin_bit_cast(w4_bf8, w4_u4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});

  load(0);
  const int total = a.chunks * a.steps;
  for (int n0 = 0; n0 < total; n0 += U) {
    if (n0 % a.steps == 0) {  // the next chunk of x
      const int64_t k0 = static_cast<int64_t>(n0 / a.steps) * chunk_cols;
      if (n0) __syncthreads();
      const int per = chunk_cols >> 3;
      for (int i = tid; i < nt * per; i += blockDim.x) {
        const int t = i / per, j = (i - t * per) * 8;
        stage8(a, t0 + t, k0 + j, xs + j, ld, t, nt);
      }
      if (tid < 2) reinterpret_cast<uint2*>(zero)[tid] = make_uint2(0u, 0u);
      __syncthreads();
    }
    uint4 cur[U][RB];
    float cs[U][RB], cz[U][RB];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < RB; ++b) cur[u][b] = wq[u][b], cs[u][b] = sc[u][b], cz[u][b] = zp[u][b];
    if (n0 + U < total) load(n0 + U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (column(n0 + u) >= a.w.N) break;
      const int at = ((n0 + u) % a.steps * waves + wave) * kStep;
      w4_f4 acc[RB][NB], sum[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        sum[n] = w4_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[b][n] = sum[n];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w4_bf8 right[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const uint32_t word = i == 0 ? cur[u][b].x : i == 1 ? cur[u][b].y : i == 2 ? cur[u][b].z : cur[u][b].w;
          right[b] = widen8(word);
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const w4_bf8 left = *reinterpret_cast<const w4_bf8*>(xp[n] + xstep[n] * (at + 8 * i));
          sum[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(left, ones, sum[n], 0, 0, 0);
#pragma unroll
          for (int b = 0; b < RB; ++b)
            acc[b][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(left, right[b], acc[b][n], 0, 0, 0);
        }
      }
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < NR; ++i)
            tot[b][n][i] = fmaf(cs[u][b], fmaf(-16.f - cz[u][b], sum[n][i], acc[b][n][i]), tot[b][n][i]);
    }
  }

  // joined over waves, segments and terms, in that order
  __syncthreads();
  float* part = reinterpret_cast<float*>(xs);  // [wave][RB][NB][16 left rows][16 rows of W]
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < NR; ++i) part[(((wave * RB + b) * NB + n) * 16 + 4 * c + i) * 16 + r] = tot[b][n][i];
  __syncthreads();
  for (int o = tid; o < nt * 16 * RB; o += blockDim.x) {
    const int t = o / (16 * RB), rr = o - t * (16 * RB), b = rr >> 4;
    if (row0 + rr >= a.w.M) continue;
    float y = 0.f;
    for (int v = t; v < held; v += nt) {
      const int n = v / TB, at = v - n * TB;
      for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int s = 0; s < 16 / TB; ++s) y += part[(((w * RB + b) * NB + n) * 16 + s * TB + at) * 16 + (rr & 15)];
    }
    const int64_t to = (t0 + t) * a.ldy + row0 + rr;
    if (a.y_f32)
      static_cast<float*>(a.y)[to] = y;
    else
      static_cast<uint16_t*>(a.y)[to] = static_cast<uint16_t>(f_bf16(y));
  }
}

// L lanes for rows of `units`, at least `least` of them (a power of two), and the grid for M rows.
hipError_t lanes_of(int64_t M, int64_t units, int least, Lanes* ln, dim3* grid) {
  ln->log2 = 0;
  while ((1 << ln->log2) < least || (ln->log2 < 8 && (int64_t{1} << ln->log2) < units)) ++ln->log2;
  ln->blocks = cdiv(units, int64_t{1} << ln->log2);
  const int64_t n = cdiv(M, 256 >> ln->log2) * ln->blocks;
  if (n > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  *grid = dim3(static_cast<uint32_t>(n));
  return hipSuccess;
}

bool aligned16(const void* p, int64_t ld, int es) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * es % 16 == 0; }

template <typename T, typename TS>
hipError_t quantize_as(const void* W, int64_t ldw, const W4& w, hipStream_t stream) {
  // codes are stored up to a multiple of 16 bytes, which every row stride holds; the lanes of a group stay together
  const int64_t stored = cdiv(w.N, 32) * 32;
  Lanes ln;
  dim3 grid;
  const hipError_t e = lanes_of(w.M, stored / 8, 1 << (w.group_log2 - 3), &ln, &grid);
  if (e != hipSuccess) return e;
  w4_quantize_kernel<T, TS><<<grid, 256, 0, stream>>>(static_cast<const T*>(W), ldw, w, aligned16(W, ldw, sizeof(T)), ln, stored);
  return hipGetLastError();
}

template <typename T, typename TS>
hipError_t dequant_as(const W4& w, void* out, int64_t ldo, hipStream_t stream) {
  Lanes ln;
  dim3 grid;
  const hipError_t e = lanes_of(w.M, cdiv(w.N, 16 / sizeof(T)), 1, &ln, &grid);
  if (e != hipSuccess) return e;
  w4_dequant_kernel<T, TS><<<grid, 256, 0, stream>>>(w, static_cast<T*>(out), ldo, aligned16(out, ldo, sizeof(T)), ln);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w4_quantize(const void* W, int64_t ldw, int type, const W4& w, hipStream_t stream) {
  if (type == ET_F32)
    return w.s_type == ET_F32 ? quantize_as<uint32_t, uint32_t>(W, ldw, w, stream) : quantize_as<uint32_t, uint16_t>(W, ldw, w, stream);
  return w.s_type == ET_F32 ? quantize_as<uint16_t, uint32_t>(W, ldw, w, stream) : quantize_as<uint16_t, uint16_t>(W, ldw, w, stream);
}

hipError_t launch_w4_dequant(const W4& w, void* out, int64_t ldo, int type, hipStream_t stream) {
  if (type == ET_F32)
    return w.s_type == ET_F32 ? dequant_as<uint32_t, uint32_t>(w, out, ldo, stream) : dequant_as<uint32_t, uint16_t>(w, out, ldo, stream);
  return w.s_type == ET_F32 ? dequant_as<uint16_t, uint32_t>(w, out, ldo, stream) : dequant_as<uint16_t, uint16_t>(w, out, ldo, stream);
}

size_t w4_gemv_ws_bytes(int64_t, int64_t, int64_t) { return 0; }

template <int TB, int NB, int NR, int RB, int U>
static hipError_t gemv_as(GemvArgs a, int waves, hipStream_t stream) {
  const int rows = a.x_f32 ? 3 * a.per_pass : a.per_pass;
  // all of x in LDS, or chunks of whole batches of steps; rows <= 64 leaves at least one batch of four waves
  const int64_t fit = (kXBytes - 16) / 2 / rows - kXPad;
  while (waves > 1 && static_cast<int64_t>(U) * waves * kStep > fit) waves >>= 1;
  const int64_t all = cdiv(cdiv(a.w.N, static_cast<int64_t>(kStep) * waves), U);  // batches of a wave
  const int64_t most = fit / (static_cast<int64_t>(U) * waves * kStep);
  a.steps = static_cast<int>((all < most ? all : most) * U);
  a.chunks = static_cast<int>(cdiv(all * U, a.steps));
  const size_t x_bytes = static_cast<size_t>(rows) * (a.steps * waves * kStep + kXPad) * 2 + 16;
  const size_t part = static_cast<size_t>(waves) * RB * NB * 256 * 4;
  const size_t lds = x_bytes > part ? x_bytes : part;
  const dim3 grid(static_cast<uint32_t>(cdiv(a.w.M, 16 * RB)), static_cast<uint32_t>(cdiv(a.T, a.per_pass)));
  if (a.w.s_type == ET_F32)
    w4_gemv_kernel<TB, NB, NR, RB, U, uint32_t><<<grid, waves * 64, lds, stream>>>(a);
  else
    w4_gemv_kernel<TB, NB, NR, RB, U, uint16_t><<<grid, waves * 64, lds, stream>>>(a);
  return hipGetLastError();
}

template <int TB>
static hipError_t gemv_blocks(int nb, const GemvArgs& a, int waves, hipStream_t stream) {
  switch (nb) {
    case 1: return gemv_as<TB, 1, 4, 1, 2>(a, waves, stream);
    case 2: return gemv_as<TB, 2, 4, 1, 2>(a, waves, stream);
    case 3: return gemv_as<TB, 3, 4, 1, 1>(a, waves, stream);
    default: return gemv_as<TB, 4, 4, 1, 1>(a, waves, stream);
  }
}

hipError_t launch_w4_gemv(const W4& w, int64_t T, const void* x, int64_t ldx, int x_type, void* y, int64_t ldy, int y_type,
                          void*, hipStream_t stream) {
  GemvArgs a = {};
  a.w = w;
  a.x = x;
  a.y = y;
  a.ldx = ldx;
  a.ldy = ldy;
  a.T = T;
  a.x_f32 = x_type == ET_F32;
  a.y_f32 = y_type == ET_F32;
  a.x_vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (ldx * (a.x_f32 ? 4 : 2)) % 16 == 0;
  const int terms = a.x_f32 ? 3 : 1;
  // the widest segments that stay within a group and are needed: fewer instructions a vector
  const int widest = w.group_log2 >= 7 ? 16 : 1 << (w.group_log2 - 3);
  const int64_t rows = T * terms;
  const int tb = rows <= 4 || widest == 4 ? 4 : rows <= 8 || widest == 8 ? 8 : 16;
  const int most = 4 * tb / terms;  // vectors of a pass
  a.per_pass = static_cast<int>(T < most ? T : most);
  const int nb = static_cast<int>(cdiv(a.per_pass * terms, tb));
  if (cdiv(T, a.per_pass) > 65535) return hipErrorInvalidConfiguration;
  const int64_t steps = cdiv(w.N, kStep);
  const int waves = steps >= 16 ? 8 : steps >= 8 ? 4 : steps >= 2 ? 2 : 1;
  if (tb == 4 && rows == 1) return gemv_as<4, 1, 1, 1, 4>(a, waves, stream);
  if (tb == 4) return gemv_blocks<4>(nb, a, waves, stream);
  if (tb == 8) return gemv_blocks<8>(nb, a, waves, stream);
  return gemv_blocks<16>(nb, a, waves, stream);
}

}  // namespace crvq
