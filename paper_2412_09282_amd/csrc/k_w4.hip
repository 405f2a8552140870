// 4-bit matrices with a scale (and a zero point) per group of consecutive columns: quantization,
// reconstruction and the product with a few vectors.
#include "kv_common.h"

#include <algorithm>

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

// ---- quantization: a lane owns eight columns (four bytes of codes), group / 8 lanes share a group.  5120 x 5120 from bf16:
// 31 us; four rows a lane (35) and products with the scale's reciprocal in place of divisions (30) were measured ----
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
  // (hi - lo) / 15 as half of each, which rounds the same and stays within fp32's range
  float s = fmaxf(w.zeros ? (0.5f * hi - 0.5f * lo) / 7.5f : fmaxf(hi, -lo) / 7.f, kMinScale);
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

// ---- reconstruction: a lane owns 16 bytes of the output, so that a wave stores 1 KB at once.  5120 x 5120 to fp32: 19 us
// (118 MB) ----
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
// turned into eight bf16 numbers 2^-12 (16 + code) (code in the upper mantissa bits of 2^-8: a shift and an and-or for two), the
// right operand of one v_mfma_f32_16x16x32_bf16; the left one holds x.  What that instruction would add up over the four
// quarters c, different groups when group < 128, is kept apart by its 16 left rows: they are 16 / TB segments of
// TB vectors, and the row of (segment, vector) holds x in the segment's quarters and zeros elsewhere.  TB = 4, 8,
// 16 gives segments of 32, 64, 128 columns.  A row's total takes  s (acc - (16 + z) X),  X 2^-12 times the sum of x over the
// segment (the same instruction with 2^-12 on the right, once for all rows); acc and X are fp32, and the factor, which the end takes
// back, keeps them finite for every finite x (31 x 128 < 2^12).
// A workgroup keeps a chunk of the columns of x in LDS, in the order of the codes (fp32: three bf16 terms, which hold
// all of its 24 bits, as three vectors), and walks blocks of 16 rows, the next block's codes on their way while one is
// computed; its waves share the rows and take every waves-th step of the columns.  Chunks are joined by a second
// launch.  Reading the codes bounds one vector (28672 x 8192: 121 MB in 32 us, 3.8 TB/s); with more of them the vector units
// and LDS share it (5120 x 13824, eleven vectors: 22.5 us, and 4.2 for the join of seven chunks).  Segments of 32 and 64 columns
// pay for staying apart: three quarters or half of the left operand are zeros.
typedef __bf16 w4_bf8 __attribute__((ext_vector_type(8)));
typedef float w4_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t w4_u4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 128;             // columns of a step
constexpr float kBack = 4096.f;        // from the sums' unit to y's
constexpr int kXPad = 8;               // elements between rows of x in LDS
constexpr int kStaging = 4;            // of the plan: what staging x costs a workgroup, in blocks of rows (1 and 16 measure the same)
constexpr int64_t kMostPasses = 65535;   // grid z
constexpr int64_t kPartBytes = 64 << 20;  // of the chunks' parts: many vectors go in several launches, whose parts stay in the cache
constexpr int kXBytes = 73 << 10;      // of x in LDS at most

struct GemvArgs {
  W4 w;
  const void* x;
  void* y;
  float* part;  // [chunk][T][M] when there are several
  int64_t ldx, ldy, T;
  int x_f32, y_f32, x_vec;
  int per_pass, batches, chunks;
  int s_vec;  // the scales of a step (and its zero points) can be read with one load
};
constexpr int batch_steps(int nb) { return nb == 1 ? 4 : 2; }
constexpr int groups_of_step(int group_log2) { return group_log2 >= 7 ? 1 : kStep >> group_log2; }
constexpr int sums_of(int64_t T, bool x_f32, int tb) { return tb == 4 && T == 1 && !x_f32 ? 1 : 4; }  // of a lane's four, in use

// Two bf16 of x in the order of the codes' halves: (u.lo, v.lo) and (u.hi, v.hi).
__device__ __forceinline__ uint32_t lo2(uint32_t u, uint32_t v) { return __builtin_amdgcn_perm(v, u, 0x05040100u); }
__device__ __forceinline__ uint32_t hi2(uint32_t u, uint32_t v) { return __builtin_amdgcn_perm(v, u, 0x07060302u); }

// Eight codes of a word as bf16 2^-12 (16 + code), columns 0 4 1 5 2 6 3 7; mask and base in registers, for one and-or.
__device__ __forceinline__ w4_bf8 widen8(uint32_t c, uint32_t mask, uint32_t base) {
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

// E scales that lie next to each other, and their zero points, from group g on.
template <int E, typename TS>
struct RawScales {
  float s[E], z[E];
  __device__ __forceinline__ void load(const TS* scale, const uint8_t* zero, int64_t g, int64_t last, bool vec) {
    if (E > 1 && vec && g + E - 1 <= last) {
      if constexpr (sizeof(TS) == 4) {
        typedef float V __attribute__((ext_vector_type(E)));
        const V v = *reinterpret_cast<const V*>(scale + g);
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] = v[e];
      } else {
        typedef uint16_t V __attribute__((ext_vector_type(E)));
        const V v = *reinterpret_cast<const V*>(scale + g);
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] = bf16_f(v[e]);
      }
      if (zero) {
        typedef uint8_t Z __attribute__((ext_vector_type(E)));
        const Z v = *reinterpret_cast<const Z*>(zero + g);
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = static_cast<float>(v[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int64_t at = min(g + e, last);
        s[e] = ld1(scale + at);
        if (zero) z[e] = static_cast<float>(zero[at]);
      }
    }
    if (!zero) {
#pragma unroll
      for (int e = 0; e < E; ++e) z[e] = 8.f;
    }
  }
};

// Between stores to LDS and the loads of other lanes of the same wave: a wave's LDS instructions execute in order, the
// compiler has to keep them so.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// NB blocks of TB vectors; NR of a lane's four sums of a block in use; E groups in a step (1 for groups of 128 and
// more).  The scales of a batch are 16 rows times U E groups: a lane reads E of one row, all with one load, and
// hands them on through LDS (one load of a scale for every step made the kernel 40 % slower).
template <int TB, int NB, int NR, int E, typename TS>
__global__ __launch_bounds__(1024) void w4_gemv_kernel(const GemvArgs a) {
  constexpr int U = batch_steps(NB);
  extern __shared__ __align__(16) uint16_t xs[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
  const int r = lane & 15, c = lane >> 4;
  const int64_t t0 = static_cast<int64_t>(blockIdx.z) * a.per_pass;
  const int nt = static_cast<int>(min(a.T - t0, static_cast<int64_t>(a.per_pass)));
  const int held = a.x_f32 ? 3 * nt : nt;  // rows of x in LDS
  const int steps = a.batches * U * waves, cols = steps * kStep, ld = cols + kXPad;
  const int64_t k0 = static_cast<int64_t>(blockIdx.y) * cols;
  uint16_t* zero = xs + held * ld;                               // eight zeros, for rows of other segments
  float* sums = reinterpret_cast<float*>(zero + 8);              // X: [step][block][quarter][NR]
  float2* held_scales = reinterpret_cast<float2*>(sums + steps * (NB * 4 * NR)) + wave * (16 * U * E);  // [row][step][group]
  float* part = reinterpret_cast<float*>(held_scales + (waves - wave) * (16 * U * E));  // [2][wave][block][vector][16 rows]

  // this lane's codes and scales: row r of a block of 16, columns 32 c of a step
  const int64_t stored = (a.w.N + 31) & ~int64_t{31}, last_group = (a.w.N - 1) >> a.w.group_log2;
  const int64_t blocks = (a.w.M + 15) >> 4;
  const int seg_group = ((c * 4) / TB) * (8 * TB) * E / kStep;  // the group in a step of the segment whose sums this lane holds
  const TS* const scales = static_cast<const TS*>(a.w.scales);
  uint4 wq[U];
  RawScales<E, TS> raw;
  const int sr = lane >> 2, su = lane & 3;  // the row and step whose scales this lane reads
  auto load = [&](int64_t block, int batch) {
    const uint8_t* codes = a.w.codes + min(block * 16 + r, a.w.M - 1) * a.w.ld;
    const int64_t kb = k0 + static_cast<int64_t>((batch * waves + wave) * U) * kStep;
    if (su < U) {
      const int64_t row = min(block * 16 + sr, a.w.M - 1), g = min((kb + su * kStep) >> a.w.group_log2, last_group);
      raw.load(scales + row * a.w.ld_s, a.w.zeros ? a.w.zeros + row * a.w.ld_z : nullptr, g, last_group, a.s_vec);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t col = kb + u * kStep + 32 * c;
      wq[u] = *reinterpret_cast<const uint4*>(codes + (col < stored ? col >> 1 : 0));  // past the row: x is zero there
    }
  };
  int64_t block = blockIdx.x;
  load(block, 0);

  const int per = cols >> 3;
  for (int i = tid; i < nt * per; i += blockDim.x) {
    const int t = i / per, j = (i - t * per) * 8;
    stage8(a, t0 + t, k0 + j, xs + j, ld, t, nt);
  }
  if (tid < 2) reinterpret_cast<uint2*>(zero)[tid] = make_uint2(0u, 0u);
  __syncthreads();

  // left operand: this lane's row is a vector of a segment; it reads x where the segment has this lane's columns
  const uint16_t* xp[NB];
  int live[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int v = n * TB + (r & (TB - 1));
    live[n] = r / TB == (c * 4) / TB && v < held;
    xp[n] = live[n] ? xs + v * ld + 32 * c : zero;
  }
  const w4_bf8 ones = __builtin_bit_cast(w4_bf8, w4_u4{0x39803980u, 0x39803980u, 0x39803980u, 0x39803980u});  // of 2^-12
  for (int s = wave; s < steps; s += waves) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      w4_f4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const w4_bf8*>(xp[n] + live[n] * (s * kStep + 8 * i)), ones,
                                                      sum, 0, 0, 0);
      if (r == 0) {
#pragma unroll
        for (int i = 0; i < NR; ++i) sums[((s * NB + n) * 4 + c) * NR + i] = sum[i];
      }
    }
  }
  __syncthreads();

  uint32_t mask = 0x00780078u, base = 0x3b803b80u;
  asm volatile("" : "+s"(mask), "+v"(base));
  w4_f4 tot[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) tot[n] = w4_f4{0.f, 0.f, 0.f, 0.f};
  int batch = 0, buffer = 0;
  while (block < blocks) {
    uint4 cur[U];
    float2 scale[U];
    wave_lds_order();
    if (su < U) {
#pragma unroll
      for (int e = 0; e < E; ++e) held_scales[(sr * U + su) * E + e] = make_float2(raw.s[e], -16.f - raw.z[e]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) cur[u] = wq[u];
    wave_lds_order();
#pragma unroll
    for (int u = 0; u < U; ++u) scale[u] = held_scales[(r * U + u) * E + seg_group];
    const bool last = batch + 1 == a.batches;
    const int64_t next = last ? block + gridDim.x : block;
    if (next < blocks) load(next, last ? 0 : batch + 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = (batch * waves + wave) * U + u;
      w4_f4 acc[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[n] = w4_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const w4_bf8 right = widen8(i == 0 ? cur[u].x : i == 1 ? cur[u].y : i == 2 ? cur[u].z : cur[u].w, mask, base);
#pragma unroll
        for (int n = 0; n < NB; ++n)
          acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const w4_bf8*>(xp[n] + live[n] * (s * kStep + 8 * i)),
                                                           right, acc[n], 0, 0, 0);
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < NR; ++i)
          tot[n][i] = fmaf(scale[u].x, fmaf(scale[u].y, sums[((s * NB + n) * 4 + c) * NR + i], acc[n][i]), tot[n][i]);
    }
    if (!last) {
      ++batch;
      continue;
    }
    // joined over the segments in the wave, then over waves and terms, in that order
    float* mine = part + (buffer * waves + wave) * (NB * TB * 16);
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        float x = tot[n][i];
        if (TB <= 8) {
          const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
          x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        }
        if (TB == 4) {
          const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
          x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        }
        if (4 * c < TB) mine[(n * TB + 4 * c + i) * 16 + r] = x;
        tot[n][i] = 0.f;
      }
    __syncthreads();
    const float* all = part + buffer * waves * (NB * TB * 16);
    for (int o = tid; o < nt * 16; o += blockDim.x) {
      const int t = o >> 4;
      const int64_t row = block * 16 + (o & 15);
      if (row >= a.w.M) continue;
      float y = 0.f;
      for (int v = t; v < held; v += nt)
#pragma unroll 4
        for (int w = 0; w < waves; ++w) y += all[(w * (NB * TB) + v) * 16 + (o & 15)];
      if (a.chunks > 1)
        a.part[(static_cast<int64_t>(blockIdx.y) * a.T + t0 + t) * a.w.M + row] = y;
      else if (a.y_f32)
        static_cast<float*>(a.y)[(t0 + t) * a.ldy + row] = y * kBack;
      else
        static_cast<uint16_t*>(a.y)[(t0 + t) * a.ldy + row] = static_cast<uint16_t>(f_bf16(y * kBack));
    }
    buffer ^= 1;
    batch = 0;
    block = next;
  }
}

// y = the sum of the chunks' parts, in order.
__global__ __launch_bounds__(256) void w4_join_kernel(const GemvArgs a) {
  const int64_t n = a.T * a.w.M, i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n) return;
  float y = 0.f;
#pragma unroll 4
  for (int s = 0; s < a.chunks; ++s) y += a.part[s * n + i];
  const int64_t t = i / a.w.M, at = t * a.ldy + i - t * a.w.M;
  if (a.y_f32)
    static_cast<float*>(a.y)[at] = y * kBack;
  else
    static_cast<uint16_t*>(a.y)[at] = static_cast<uint16_t>(f_bf16(y * kBack));
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

// What a workgroup holds in LDS: x and eight zeros, its sums, the scales of a batch, and the parts of y.
size_t w4_gemv_lds(const W4Plan& p, int64_t T, bool x_f32, int group_log2) {
  const int U = batch_steps(p.nb), held = p.per_pass * (x_f32 ? 3 : 1);
  const size_t steps = static_cast<size_t>(p.waves) * p.batches * U;
  return held * (steps * kStep + kXPad) * 2 + 16 + steps * p.nb * 4 * sums_of(T, x_f32, p.tb) * sizeof(float) +
         static_cast<size_t>(p.waves) * 16 * U * groups_of_step(group_log2) * sizeof(float2) +
         size_t{2} * p.waves * p.nb * p.tb * 16 * sizeof(float);
}

// The widest segments that stay within a group and are needed take the fewest instructions; the columns are cut where
// x does not fit into LDS, and, where there are few rows, until the chip is filled.
static W4Plan plan_columns(int64_t M, int64_t N, int64_t T, bool x_f32, int group_log2) {
  W4Plan p;
  const int terms = x_f32 ? 3 : 1, widest = group_log2 >= 7 ? 16 : 1 << (group_log2 - 3);
  const int64_t rows = T * terms;
  p.tb = rows <= 4 || widest == 4 ? 4 : rows <= 8 || widest == 8 ? 8 : 16;
  const int most = (p.tb == 4 ? 4 : 2) * p.tb / terms;
  p.per_pass = static_cast<int>(T < most ? T : most);
  p.nb = static_cast<int>(cdiv(static_cast<int64_t>(p.per_pass) * terms, p.tb));
  // One row of x: workgroups of 8 waves, three a CU (28672 x 8192: 32.8 us; 16 waves, one a CU: 35.7); a few rows: of 16
  // (four vectors, groups of 32: 45 us; 8: 62), several blocks: of 8, for the sums' LDS.
  const int U = batch_steps(p.nb), most_waves = rows > 1 && p.nb == 1 ? 16 : 8;
  const int64_t fit = (kXBytes / 2 / (p.per_pass * terms) - kXPad) / kStep;  // steps of x in LDS: at least 8
  const int64_t steps = cdiv(N, kStep), blocks = cdiv(M, 16), passes = cdiv(T, p.per_pass);
  int64_t chunk = steps < fit ? steps : fit;
  if (blocks * passes < 64 && steps > 32) {  // few rows: chunks of at least 8 steps
    const int64_t want = cdiv(256, blocks * passes), c = cdiv(steps, want);
    if (c < chunk) chunk = c < 8 ? 8 : c;
  }
  const int64_t w = cdiv(chunk, U);
  p.waves = static_cast<int>(w < most_waves ? w : most_waves);
  int64_t batches = cdiv(chunk, p.waves * U);
  if (batches * p.waves * U > fit) {
    if (batches > 1) --batches;
    else p.waves = static_cast<int>(fit / U);
  }
  p.batches = static_cast<int>(batches);
  p.chunks = static_cast<int>(cdiv(steps, static_cast<int64_t>(p.waves) * p.batches * U));
  p.groups = 0;
  return p;
}

W4Plan plan_w4_gemv(int64_t M, int64_t N, int64_t T, bool x_f32, int group_log2) {
  W4Plan p = plan_columns(M, N, T, x_f32, group_log2);
  // A round of workgroups is what the CUs hold at once, by waves and by LDS; the rows are divided so that whole rounds walk
  // them (4096 x 4096, sixteen vectors, groups of 32: 16.2 us; twice as many workgroups, half a round too many: 22.4).  Several
  // rounds are taken where one would leave CUs idle (5120 x 13824, 300 vectors, groups of 64: 424 us, one round of 171: 755).
  const int64_t lds = static_cast<int64_t>(w4_gemv_lds(p, T, x_f32, group_log2));
  const int waves = T * (x_f32 ? 3 : 1) > 1 && p.nb == 1 ? 16 : 24;  // of a CU
  const int64_t per_cu = std::min<int64_t>(std::max<int64_t>(1, waves / p.waves), std::max<int64_t>(1, (160 << 10) / lds));
  const int64_t blocks = cdiv(M, 16), round = 256 * per_cu, each = p.chunks * cdiv(T, p.per_pass);
  int64_t least = INT64_MAX;
  for (int r = 1; r <= 4 && p.groups < blocks; ++r) {
    const int64_t g = std::min(blocks, std::max<int64_t>(1, r * round / each));
    const int64_t cost = cdiv(g * each, round) * (cdiv(blocks, g) + kStaging);
    if (cost < least) least = cost, p.groups = g;
  }
  return p;
}

static size_t part_bytes(const W4Plan& p, int64_t M, int64_t T) {
  return p.chunks > 1 ? align256(static_cast<size_t>(p.chunks) * T * M * sizeof(float)) : 0;
}

// Vectors of one launch of T that are planned as p: whole passes whose parts fit kPartBytes, and at least one pass.
static int64_t launch_vectors(const W4Plan& p, int64_t M, int64_t T) {
  int64_t passes = kMostPasses;
  if (p.chunks > 1) passes = std::min(passes, kPartBytes / (p.chunks * M * static_cast<int64_t>(sizeof(float)) * p.per_pass));
  return std::min(T, std::max<int64_t>(1, passes) * p.per_pass);
}

size_t w4_gemv_ws_bytes(int64_t M, int64_t N, int64_t T) {
  size_t most = 0;
  for (int f32 = 0; f32 < 2; ++f32)
    for (int g = 5; g <= 7; ++g) {
      W4Plan p = plan_columns(M, N, T, f32, g);
      const int64_t each = launch_vectors(p, M, T), rest = T % each;
      if (each < T) p = plan_columns(M, N, each, f32, g);
      most = std::max(most, part_bytes(p, M, each));
      if (rest) most = std::max(most, part_bytes(plan_columns(M, N, rest, f32, g), M, rest));
    }
  return most;
}

template <int TB, int NB, int NR, int E>
static hipError_t gemv_as(const W4Plan& p, const GemvArgs& a, hipStream_t stream) {
  const size_t lds = w4_gemv_lds(p, a.T, a.x_f32, a.w.group_log2);
  const int64_t passes = cdiv(a.T, p.per_pass);
  if (p.chunks > 65535) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(p.groups), static_cast<uint32_t>(p.chunks), static_cast<uint32_t>(passes));
  if (a.w.s_type == ET_F32)
    w4_gemv_kernel<TB, NB, NR, E, uint32_t><<<grid, p.waves * 64, lds, stream>>>(a);
  else
    w4_gemv_kernel<TB, NB, NR, E, uint16_t><<<grid, p.waves * 64, lds, stream>>>(a);
  return hipGetLastError();
}

template <int E>
static hipError_t gemv_groups(const W4Plan& p, const GemvArgs& a, hipStream_t stream) {
  if (p.tb == 4) {
    if (sums_of(a.T, a.x_f32, p.tb) == 1) return gemv_as<4, 1, 1, E>(p, a, stream);
    if (p.nb == 1) return gemv_as<4, 1, 4, E>(p, a, stream);
    if (p.nb == 2) return gemv_as<4, 2, 4, E>(p, a, stream);
    return p.nb == 3 ? gemv_as<4, 3, 4, E>(p, a, stream) : gemv_as<4, 4, 4, E>(p, a, stream);
  }
  if constexpr (E <= 2)
    if (p.tb == 8) return p.nb == 1 ? gemv_as<8, 1, 4, E>(p, a, stream) : gemv_as<8, 2, 4, E>(p, a, stream);
  if constexpr (E == 1)
    if (p.tb == 16) return p.nb == 1 ? gemv_as<16, 1, 4, E>(p, a, stream) : gemv_as<16, 2, 4, E>(p, a, stream);
  return hipErrorInvalidValue;  // a segment wider than a group: the plan gives none
}

hipError_t launch_w4_gemv(const W4& w, int64_t T, const void* x, int64_t ldx, int x_type, void* y, int64_t ldy, int y_type,
                          void* ws, hipStream_t stream) {
  GemvArgs a = {};
  a.w = w;
  a.ldx = ldx;
  a.ldy = ldy;
  a.x_f32 = x_type == ET_F32;
  a.y_f32 = y_type == ET_F32;
  a.x_vec = aligned16(x, ldx, a.x_f32 ? 4 : 2);
  a.part = static_cast<float*>(ws);
  const int groups = groups_of_step(w.group_log2), es = w.s_type == ET_F32 ? 4 : 2;
  a.s_vec = reinterpret_cast<uintptr_t>(w.scales) % (groups * es) == 0 && w.ld_s % groups == 0 &&
            reinterpret_cast<uintptr_t>(w.zeros) % groups == 0 && w.ld_z % groups == 0;
  W4Plan p = plan_w4_gemv(w.M, w.N, T, a.x_f32, w.group_log2);
  const int64_t each = launch_vectors(p, w.M, T);
  for (int64_t t = 0; t < T; t += each) {
    a.T = std::min(each, T - t);
    a.x = static_cast<const char*>(x) + t * ldx * (a.x_f32 ? 4 : 2);
    a.y = static_cast<char*>(y) + t * ldy * (a.y_f32 ? 4 : 2);
    if (a.T < T) p = plan_w4_gemv(w.M, w.N, a.T, a.x_f32, w.group_log2);
    a.per_pass = p.per_pass;
    a.batches = p.batches;
    a.chunks = p.chunks;
    const hipError_t e = groups == 1 ? gemv_groups<1>(p, a, stream)
                         : groups == 2 ? gemv_groups<2>(p, a, stream) : gemv_groups<4>(p, a, stream);
    if (e != hipSuccess) return e;
    if (p.chunks == 1) continue;
    const int64_t n = cdiv(a.T * w.M, 256);
    if (n > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    w4_join_kernel<<<dim3(static_cast<uint32_t>(n)), 256, 0, stream>>>(a);
    const hipError_t joined = hipGetLastError();
    if (joined != hipSuccess) return joined;
  }
  return hipSuccess;
}

}  // namespace crvq
