// Attention of new tokens over the paged 8-bit cache, out_i = sum_t p_t V_t with p = softmax(scale q_i . K_t).
//
// A wave owns 16 QB query rows ("columns": column c of a sequence and key head is new token c / G, query head
// c % G of the G that share the key head) and walks a range of tokens 64 at a time, with the running
// maximum m and sum l of the softmax in registers; nothing of size rows x tokens exists.
//   S^T = K Q^T on v_mfma_i32_16x16x64_i8: the key codes are the left operand as they lie in the cache, a query row is a
//     fixed-point number of 2 (bf16) or 3 (fp32) signed 8-bit digits, so the products are exact integers and no
//     code is widened.  The score is the integer times alpha = (query step) (key scale) |scale| log2(e).
//   O^T += V^T P^T on v_mfma_f32_16x16x32_f16: the value codes lie transposed in the cache, 16 tokens of an
//     element in 16 bytes, and are widened to fp16 in registers (exact); the weights are rounded to fp16.  The page's
//     value scale goes into the weights, relative to a power of two 2^e that follows the largest scale met so far.
//     A step with a weight below fp16's normal numbers (2^-21 of the row's largest) takes its weights as
//     two bf16 terms, whose range is fp32's, and so keeps 16 bits of every weight; fp32 queries take three terms always.
// The token in row 4 c + i of tile u is 16 c + 4 u + i: a lane (column r = lane % 16, quarter c = lane / 16) then
// holds the scores of 16 consecutive tokens, which are exactly its operands of the second product and, pages being
// multiples of 16, belong to one page.  Operands go from the cache to registers without LDS.
#include "kv_common.h"

namespace crvq {
namespace {

typedef int at_i4 __attribute__((ext_vector_type(4)));
typedef float at_f4 __attribute__((ext_vector_type(4)));
typedef float at_f2 __attribute__((ext_vector_type(2)));
typedef _Float16 at_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 at_h2 __attribute__((ext_vector_type(2)));
typedef __bf16 at_b8 __attribute__((ext_vector_type(8)));
typedef uint32_t at_u4 __attribute__((ext_vector_type(4)));
typedef uint16_t at_s2 __attribute__((ext_vector_type(2)));

constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTokens = 64;     // tokens of a step
// The maximum is renewed when a score passes it by more than 2^kSlack, so weights reach 2^kSlack; with the
// scale's factor at most 2^kLift they stay below fp16's 2^16 and keep 11 bits down to 2^-21 of the maximum.
constexpr float kSlack = 8.f;
constexpr int kLift = 7;

struct AttnArgs {
  KvCache c;
  KvBatch bt;
  KvRows q, out;
  float* lse;
  float *po, *pm, *pl;  // partial results [split][b][i][h][D], and their maxima and sums
  float scale;
  int Hq, G, causal, window, splits, tiles, o_vec;
};

__device__ __forceinline__ float quarters_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quarters_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ int wave_min(int x) {
  for (int o = 32; o; o >>= 1) x = min(x, __shfl_xor(x, o));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x) { return -wave_min(-x); }

// Eight value codes (two words) as fp16: byte + 128 under fp16's 1024, less 1152.
__device__ __forceinline__ at_h8 widen8(uint32_t a, uint32_t b) {
  a ^= 0x80808080u;
  b ^= 0x80808080u;
  const uint32_t k = 0x64646464u;
  const at_u4 v = {__builtin_amdgcn_perm(k, a, 0x04010400u), __builtin_amdgcn_perm(k, a, 0x04030402u),
                   __builtin_amdgcn_perm(k, b, 0x04010400u), __builtin_amdgcn_perm(k, b, 0x04030402u)};
  return __builtin_bit_cast(at_h8, v) - static_cast<_Float16>(1152.f);
}

// Eight value codes as bf16: integers of eight bits are the upper halves of their fp32.
__device__ __forceinline__ at_b8 widen8_bf16(uint32_t a, uint32_t b) {
  at_u4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? a : b;
    const float x = static_cast<float>(static_cast<int8_t>(w >> (16 * (i & 1))));
    const float y = static_cast<float>(static_cast<int8_t>(w >> (16 * (i & 1) + 8)));
    v[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
  }
  return __builtin_bit_cast(at_b8, v);
}

// One element of a query row as signed digits, the highest first, in byte `at` of each digit's word.
template <int NT>
__device__ __forceinline__ void digits(int v, int at, uint32_t (&w)[NT]) {
#pragma unroll
  for (int n = NT - 1; n > 0; --n) {
    const int low = static_cast<int8_t>(v);
    w[n] |= (static_cast<uint32_t>(low) & 255u) << (8 * at);
    v = (v - low) >> 8;
  }
  w[0] |= (static_cast<uint32_t>(v) & 255u) << (8 * at);
}

template <typename T>
__device__ __forceinline__ float elem(const T* p, int i) {
  if constexpr (sizeof(T) == 4)
    return reinterpret_cast<const float*>(p)[i];
  else
    return bf16_f(p[i]);
}

// DT tiles of 16 elements hold a head; a wave has 16 QB columns; WK waves of a workgroup share their columns and
// take turns at the tokens, the others (4 / WK) have columns of their own.  SMALL: pages below 64 tokens.
template <typename T, int DT, int QB, int WK, bool SMALL>
__global__ __launch_bounds__(256) void kv_attention_kernel(const AttnArgs a) {
  constexpr int DC = (DT + 3) / 4;                // 64-element chunks of a head
  constexpr int NT = sizeof(T) == 4 ? 3 : 2;      // digits of a query element
  constexpr int PT = sizeof(T) == 4 ? 3 : 2;      // bf16 terms of a weight
  constexpr double kSteps = NT == 3 ? 8355711.0 : 32639.0;  // 127 in every digit
  constexpr int kRow = DT * 16 + 4;               // floats of a column in LDS
  __shared__ __align__(16) float join[WK > 1 ? WK * 16 * QB * kRow : 4];
  __shared__ float join_m[WK > 1 ? WK * 16 * QB : 1], join_l[WK > 1 ? WK * 16 * QB : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r = lane & 15, c = lane >> 4;
  const int D = a.c.D, pl2 = a.c.page_log2;

  // which columns: tiles of a sequence last to first, so that the longest rows of a causal prompt start first
  int64_t item = blockIdx.x;
  const int hk = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  const int b = static_cast<int>(item % a.bt.B);
  item /= a.bt.B;
  const int split = static_cast<int>(item % a.splits);
  const int tile = a.tiles - 1 - static_cast<int>(item / a.splits);
  const KvSeq sq = kv_seq(a.bt, b, pl2);
  const int cols = min(sq.n, a.bt.max_new) * a.G;
  const int col0 = (tile * (4 / WK) + (WK == 1 ? wave : 0)) * (16 * QB);
  if (col0 >= cols) return;  // with WK > 1 all waves of the workgroup
  const bool ok = sq.ok && (sq.len == 0 || a.c.n_pages > 0);

  // queries: fixed point, 16 elements of a column and chunk in a lane
  at_i4 q[QB][DC][NT];
  float step[QB];
  int lo[QB], hi[QB];
#pragma unroll
  for (int n = 0; n < QB; ++n) {
    const int col = min(col0 + n * 16 + r, cols - 1);  // columns past the last one repeat it
    const int i = col / a.G, h = hk * a.G + col - i * a.G;
    const T* row = static_cast<const T*>(a.q.p) + (sq.row0 + i) * a.q.tok + h * a.q.head;
    uint32_t most = 0;
#pragma unroll
    for (int ch = 0; ch < DC; ++ch)
      if (ch * 64 + c * 16 < D)
        for (int e = 0; e < 16; ++e)
          most = max(most, __float_as_uint(elem(row, ch * 64 + c * 16 + e)) & 0x7fffffffu);
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 16)));
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 32)));
    const bool finite = most < 0x7f800000u;
    const double inv = finite && most ? (a.scale < 0.f ? -kSteps : kSteps) / static_cast<double>(__uint_as_float(most)) : 0.0;
    step[n] = finite ? static_cast<float>(static_cast<double>(__uint_as_float(most)) / kSteps * fabs(static_cast<double>(a.scale)) *
                                          static_cast<double>(kLog2e))
                     : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int ch = 0; ch < DC; ++ch) {
      uint32_t w[4][NT] = {};
      if (finite && ch * 64 + c * 16 < D) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          digits<NT>(static_cast<int>(rint(static_cast<double>(elem(row, ch * 64 + c * 16 + e)) * inv)), e & 3, w[e >> 2]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
        q[n][ch][t] = at_i4{static_cast<int>(w[0][t]), static_cast<int>(w[1][t]), static_cast<int>(w[2][t]), static_cast<int>(w[3][t])};
    }
    hi[n] = ok ? sq.len : 0;
    lo[n] = 0;
    if (a.causal) {
      const int place = sq.len - sq.n + i;
      hi[n] = min(hi[n], max(place + 1, 0));
      if (a.window) lo[n] = max(place + 1 - a.window, 0);
    }
    if (lo[n] >= hi[n]) lo[n] = hi[n] = 0;
  }
  // the wave's tokens, and those that all of its columns see
  int first = 0x7fffffff, last = 0, all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
  for (int n = 0; n < QB; ++n) {
    if (hi[n] > 0) first = min(first, lo[n]);
    last = max(last, hi[n]);
    all_lo = max(all_lo, lo[n]);
    all_hi = min(all_hi, hi[n]);
  }
  first = wave_min(first);
  last = wave_max(last);
  all_lo = wave_max(all_lo);
  all_hi = wave_min(all_hi);
  first = min(first, last) & ~(kTokens - 1);
  if (a.splits > 1) {  // an equal share of the tokens, in whole rounds of the waves
    const int span = (last - first + a.splits - 1) / a.splits, round = kTokens * WK;
    const int share = (span + round - 1) / round * round;
    const int64_t from = first + static_cast<int64_t>(split) * share;
    first = static_cast<int>(from < last ? from : last);
    last = min(last, first + share);
  }
  const int from = first + (WK > 1 ? wave * kTokens : 0);

  at_f4 o[QB][DT];
  float m[QB], l[QB];
  int e = -126;  // exponent that value scales are taken relative to
#pragma unroll
  for (int n = 0; n < QB; ++n) {
    m[n] = -kInf;
    l[n] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[n][d] = at_f4{0.f, 0.f, 0.f, 0.f};
  }

  const int32_t* table = a.bt.table + static_cast<int64_t>(b) * a.bt.ld_table;
  // the page of the 16 tokens from t on: uniform unless pages are small; past the length that of token t0
  auto page_of = [&](int t, int t0) { return table[(t < sq.len ? t : t0) >> pl2]; };
  auto there = [&](int p) { return static_cast<uint32_t>(p) < static_cast<uint32_t>(a.c.n_pages); };
  const int k_group = r >> 2;  // the 16 tokens of a step that this lane's row of a key tile belongs to
  const int64_t head_bytes = static_cast<int64_t>(D) << pl2;

  at_i4 kreg[4][DC];
  auto load_keys = [&](int t0) {
    const int g = SMALL ? t0 + 16 * k_group : t0;
    const int p = page_of(g, t0);
    const int64_t head = static_cast<int64_t>(there(p) ? p : 0) * a.c.Hkv + hk;
    const int slot = (SMALL ? g & ((1 << pl2) - 1) : (t0 & ((1 << pl2) - 1)) + 16 * k_group) + (r & 3);
    const int8_t* k = a.c.k + head * head_bytes + slot * D;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int ch = 0; ch < DC; ++ch) {
        const int d = ch * 64 + c * 16;
        kreg[u][ch] = *reinterpret_cast<const at_i4*>(k + 4 * u * D + (d < D ? d : 0));  // past D the digits are 0
      }
  };

  if (from < last) load_keys(from);
  for (int t0 = from; t0 < last; t0 += kTokens * WK) {
    // values, and the scales of this lane's 16 tokens
    const int g = SMALL ? t0 + 16 * c : t0;
    const int p = page_of(g, t0);
    const bool have = there(p);
    const int64_t head = static_cast<int64_t>(have ? p : 0) * a.c.Hkv + hk;
    const int slot = SMALL ? g & ((1 << pl2) - 1) : (t0 & ((1 << pl2) - 1)) + 16 * c;
    const int8_t* v = a.c.v + head * head_bytes + slot;
    at_u4 vreg[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
      vreg[d] = *reinterpret_cast<const at_u4*>(v + (static_cast<int64_t>(min(d * 16 + r, D - 1)) << pl2));
    const float ks = a.c.k_scale[head];
    float vs = a.c.v_scale[head];
    const bool good = have && ks >= 0.f && ks < kInf && vs >= 0.f && vs < kInf;
    if (!good) vs = 0.f;

    // scores
    at_f4 s[QB][4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int n = 0; n < QB; ++n) {
        at_i4 acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[t] = at_i4{0, 0, 0, 0};
#pragma unroll
          for (int ch = 0; ch < DC; ++ch) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kreg[u][ch], q[n][ch][t], acc[t], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float low = static_cast<float>((acc[NT - 2][i] << 8) + acc[NT - 1][i]);
          s[n][u][i] = NT == 3 ? fmaf(static_cast<float>(acc[0][i]), 65536.f, low) : low;
        }
      }
    if (t0 + kTokens * WK < last) load_keys(t0 + kTokens * WK);

    // the power of two that value scales are relative to
    const int ve = SMALL ? wave_max((static_cast<int>(__float_as_uint(vs)) >> 23) - 126)
                         : __builtin_amdgcn_readfirstlane((static_cast<int>(__float_as_uint(vs)) >> 23) - 126);
    float fall = 1.f;
    if (ve > e) {
      fall = ldexpf(1.f, max(e - ve, -126));
      e = ve;
    }
    const float weight = fmaxf(ldexpf(vs, -e), 0x1p-40f) * static_cast<float>(1 << kLift);
    const float unweight = 1.f / weight;
    const bool whole = t0 >= all_lo && t0 + kTokens <= all_hi;

#pragma unroll
    for (int n = 0; n < QB; ++n) {
      const float alpha = good ? step[n] * ks : __uint_as_float(0x7fc00000u);
      uint32_t seen = 0xffffu;  // which of the lane's 16 tokens its column sees
      if (!whole) {
        const int base = t0 + 16 * c;
        const int x = min(max(lo[n] - base, 0), 16), y = min(max(hi[n] - base, 0), 16);
        seen = ((1u << y) - 1u) & ~((1u << x) - 1u);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (!(seen >> j & 1)) s[n][j >> 2][j & 3] = -3e38f;
      }
      float top = fmaxf(fmaxf(s[n][0][0], s[n][0][1]), s[n][0][2]);
#pragma unroll
      for (int j = 3; j < 16; ++j) top = fmaxf(top, s[n][j >> 2][j & 3]);
      top *= alpha;
      float keep = fall;
      if (__any(top > m[n] + kSlack || fall != 1.f)) {
        const float now = fmaxf(m[n], quarters_max(top));
        const float f = m[n] > -kInf ? __builtin_amdgcn_exp2f(m[n] - now) : 0.f;
        m[n] = now;
        l[n] *= f;
        keep *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[n][d] *= keep;
      }
      // weights p 2^.. = exp2(score - m) weight, as exp2 of one fused multiply-add
      float sum = 0.f;
      const float shift = __builtin_amdgcn_logf(weight) - m[n];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        float pj = __builtin_amdgcn_exp2f(fmaf(s[n][j >> 2][j & 3], alpha, shift));
        if (!whole && !(seen >> j & 1)) pj = 0.f;
        sum += pj;
        s[n][j >> 2][j & 3] = pj;
      }
      l[n] = fmaf(sum, unweight, l[n]);
    }
    // values
    bool wide = sizeof(T) == 4;
    at_h8 pw[QB][2];
    if constexpr (sizeof(T) == 2) {
      at_s2 least = {0x7fff, 0x7fff};
#pragma unroll
      for (int n = 0; n < QB; ++n)
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const at_h2 h = __builtin_convertvector((at_f2{s[n][j >> 2][j & 3], s[n][j >> 2][(j & 3) + 1]}), at_h2);
          least = __builtin_elementwise_min(least, __builtin_bit_cast(at_s2, h));
          pw[n][j >> 3][j & 7] = h[0];
          pw[n][j >> 3][(j & 7) + 1] = h[1];
        }
      wide = __any(least[0] < 0x0400 || least[1] < 0x0400);
    }
    if (!wide) {
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const at_h8 v0 = widen8(vreg[d][0], vreg[d][1]), v1 = widen8(vreg[d][2], vreg[d][3]);
#pragma unroll
        for (int n = 0; n < QB; ++n) {
          o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pw[n][0], o[n][d], 0, 0, 0);
          o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pw[n][1], o[n][d], 0, 0, 0);
        }
      }
    } else {
      at_b8 pb[QB][2][PT];
#pragma unroll
      for (int n = 0; n < QB; ++n)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = s[n][2 * w + (j >> 2)][j & 3];
#pragma unroll
          for (int t = 0; t < PT; ++t) {  // the upper halves, then what they leave
            at_u4 x;
#pragma unroll
            for (int j = 0; j < 8; j += 2)
              x[j >> 1] = __builtin_amdgcn_perm(__float_as_uint(p[j + 1]), __float_as_uint(p[j]), 0x07060302u);
            pb[n][w][t] = __builtin_bit_cast(at_b8, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] -= __uint_as_float(__float_as_uint(p[j]) & 0xffff0000u);
          }
        }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const at_b8 v0 = widen8_bf16(vreg[d][0], vreg[d][1]), v1 = widen8_bf16(vreg[d][2], vreg[d][3]);
#pragma unroll
        for (int n = 0; n < QB; ++n)
#pragma unroll
          for (int t = PT - 1; t >= 0; --t) {
            o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pb[n][0][t], o[n][d], 0, 0, 0);
            o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pb[n][1][t], o[n][d], 0, 0, 0);
          }
      }
    }
  }

  const float back = ldexpf(1.f, e - kLift);
#pragma unroll
  for (int n = 0; n < QB; ++n) {
    l[n] = quarters_sum(l[n]);
#pragma unroll
    for (int d = 0; d < DT; ++d) o[n][d] *= back;
  }
  const float nan = __uint_as_float(0x7fc00000u);

  // a column's result: to the output, or to the partial results of this split
  auto row_of = [&](int col, int& i, int& h) {
    i = col / a.G;
    h = hk * a.G + col - i * a.G;
  };
  auto stats = [&](int col, float mm, float ll) {
    int i, h;
    row_of(col, i, h);
    if (a.splits > 1) {
      const int64_t at = ((static_cast<int64_t>(split) * a.bt.B + b) * a.bt.max_new + i) * a.Hq + h;
      a.pm[at] = mm;
      a.pl[at] = ok ? ll : nan;
    } else if (a.lse) {
      a.lse[static_cast<int64_t>(sq.row0 + i) * a.Hq + h] = !ok ? nan : ll == 0.f ? -kInf : (mm + __builtin_amdgcn_logf(ll)) * kLn2;
    }
  };
  auto put = [&](int col, int d, at_f4 x, float ll) {
    if (d >= D) return;
    int i, h;
    row_of(col, i, h);
    if (a.splits > 1) {
      const int64_t at = ((static_cast<int64_t>(split) * a.bt.B + b) * a.bt.max_new + i) * a.Hq + h;
      if (ll != 0.f) *reinterpret_cast<at_f4*>(a.po + at * D + d) = x;
      return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = !ok ? nan : ll == 0.f ? 0.f : x[k] / ll;
    T* out = static_cast<T*>(a.out.p) + (sq.row0 + i) * a.out.tok + h * a.out.head + d;
    if constexpr (sizeof(T) == 4) {
      float* f = reinterpret_cast<float*>(out);
      if (a.o_vec) {
        *reinterpret_cast<at_f4*>(f) = x;
      } else {
        for (int k = 0; k < 4; ++k) f[k] = x[k];
      }
    } else {
      if (a.o_vec) {
        *reinterpret_cast<uint2*>(out) = make_uint2(f_bf16x2(x[0], x[1]), f_bf16x2(x[2], x[3]));
      } else {
        for (int k = 0; k < 4; ++k) out[k] = static_cast<T>(f_bf16(x[k]));
      }
    }
  };

  if constexpr (WK == 1) {
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      const int col = col0 + n * 16 + r;
      if (col >= cols) continue;
      if (c == 0) stats(col, m[n], l[n]);
#pragma unroll
      for (int d = 0; d < DT; ++d) put(col, d * 16 + 4 * c, o[n][d], l[n]);
    }
  } else {
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      const int at = (wave * QB + n) * 16 + r;
      if (c == 0) {
        join_m[at] = m[n];
        join_l[at] = l[n];
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<at_f4*>(join + at * kRow + d * 16 + 4 * c) = o[n][d];
    }
    __syncthreads();
    for (int x = threadIdx.x; x < 16 * QB * DT * 4; x += 256) {
      const int col = x / (DT * 4), d = (x - col * (DT * 4)) * 4;
      if (col0 + col >= cols) break;
      float mm = -kInf;
#pragma unroll
      for (int w = 0; w < WK; ++w) mm = fmaxf(mm, join_m[w * QB * 16 + col]);
      float ll = 0.f;
      at_f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        const int at = w * QB * 16 + col;
        const float f = join_m[at] == -kInf ? 0.f : __builtin_amdgcn_exp2f(join_m[at] - mm);
        ll = fmaf(f, join_l[at], ll);
        y += f * *reinterpret_cast<const at_f4*>(join + at * kRow + d);
      }
      if (d == 0) stats(col0 + col, mm, ll);
      put(col0 + col, d, y, ll);
    }
  }
}

// Joins the splits of one (row, head): the factors of the splits first, a thread each, then 4 elements a thread in
// groups that share the splits.
constexpr int kSplits = 256;
template <typename T>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(const AttnArgs a) {
  __shared__ __align__(16) at_f4 part[256];
  __shared__ float factor[kSplits], red[8];
  const int tid = threadIdx.x;
  uint32_t item = blockIdx.x;
  const int h = static_cast<int>(item % a.Hq);
  item /= a.Hq;
  const int i = static_cast<int>(item % a.bt.max_new), b = static_cast<int>(item / a.bt.max_new);
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  if (i >= sq.n) return;
  const int64_t stride = static_cast<int64_t>(a.bt.B) * a.bt.max_new * a.Hq;
  const int64_t at = (static_cast<int64_t>(b) * a.bt.max_new + i) * a.Hq + h;
  // a split that saw nothing has l = 0 and stored no output; a NaN goes on into l
  const float ms = tid < a.splits ? a.pm[tid * stride + at] : -kInf, ls = tid < a.splits ? a.pl[tid * stride + at] : 0.f;
  float m = ls == 0.f ? -kInf : ms;
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float f = ls == 0.f ? 0.f : ls == ls ? __builtin_amdgcn_exp2f(ms - m) : ls;
  float l = f == f ? f * ls : f;
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
  if ((tid & 63) == 0) red[4 + (tid >> 6)] = l;
  if (tid < kSplits) factor[tid] = f == f ? f : 0.f;
  __syncthreads();
  l = (red[4] + red[5]) + (red[6] + red[7]);
  const int per = a.c.D >> 2, groups = 256 / per, g = tid / per, d = (tid - g * per) * 4;
  at_f4 y = {0.f, 0.f, 0.f, 0.f};
  if (g < groups) {
#pragma unroll 4
    for (int s = g; s < a.splits; s += groups)
      if (factor[s] != 0.f) y += factor[s] * *reinterpret_cast<const at_f4*>(a.po + (s * stride + at) * a.c.D + d);
  }
  part[tid] = y;
  __syncthreads();
  if (g != 0) return;
  for (int s = 1; s < groups; ++s) y += part[s * per + tid];
  const float bad = l - l;  // 0, or NaN
  const int64_t row = sq.row0 + i;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float x = l == 0.f ? 0.f : y[k] / l + bad;
    T* out = static_cast<T*>(a.out.p) + row * a.out.tok + h * a.out.head + d + k;
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<float*>(out) = x;
    else
      *out = static_cast<T>(f_bf16(x));
  }
  if (a.lse && d == 0) a.lse[row * a.Hq + h] = l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2 + bad;
}

// How a call is divided.  One tile of columns: its workgroups' four waves share the columns (16) and take turns at the
// tokens; more: every wave has 16 kPromptBlocks columns of its own.  Tokens are split over workgroups until
// kWorkgroups are at work, a share being at least kShare tokens.
struct AttnPlan {
  bool prompt;
  int tiles, splits;
};
constexpr int kPromptBlocks = 2;
constexpr int64_t kWorkgroups = 1024;
constexpr int kShare = 512;
AttnPlan plan_attention(int B, int Hq, int Hkv, int max_new, int max_kv) {
  AttnPlan p;
  const int64_t cols = static_cast<int64_t>(max_new) * (Hq / Hkv);
  p.prompt = cols > 16;
  p.tiles = static_cast<int>(cdiv(cols, p.prompt ? 64 * kPromptBlocks : 16));
  const int64_t groups = static_cast<int64_t>(B) * Hkv * p.tiles;
  const int64_t most = cdiv(max_kv, kShare), want = cdiv(kWorkgroups, groups);
  const int64_t n = want < most ? want : most;
  p.splits = static_cast<int>(n < 1 ? 1 : n > kSplits ? kSplits : n);
  return p;
}

struct AttnWs {
  float *po, *pm, *pl;
};
AttnWs carve_attention(WsCursor& c, const AttnPlan& p, int B, int Hq, int D, int max_new) {
  AttnWs w = {nullptr, nullptr, nullptr};
  if (p.splits == 1) return w;
  const size_t rows = static_cast<size_t>(p.splits) * B * max_new * Hq;
  w.po = c.take<float>(rows * D);
  w.pm = c.take<float>(rows);
  w.pl = c.take<float>(rows);
  return w;
}

template <typename T, int DT>
hipError_t attend_as(const AttnPlan& p, const AttnArgs& a, hipStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(p.tiles) * p.splits * a.bt.B * a.c.Hkv;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(blocks));
  const bool small = a.c.page_log2 < 6;
  if (p.prompt) {
    if (small) kv_attention_kernel<T, DT, kPromptBlocks, 1, true><<<grid, 256, 0, stream>>>(a);
    else kv_attention_kernel<T, DT, kPromptBlocks, 1, false><<<grid, 256, 0, stream>>>(a);
  } else {
    if (small) kv_attention_kernel<T, DT, 1, 4, true><<<grid, 256, 0, stream>>>(a);
    else kv_attention_kernel<T, DT, 1, 4, false><<<grid, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t attend(const AttnPlan& p, const AttnArgs& a, hipStream_t stream) {
  const int D = a.c.D;
  hipError_t e = D <= 64 ? attend_as<T, 4>(p, a, stream)
                 : D <= 128 ? attend_as<T, 8>(p, a, stream) : attend_as<T, 16>(p, a, stream);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t rows = static_cast<int64_t>(a.bt.B) * a.bt.max_new * a.Hq;
  if (rows > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  kv_attention_join_kernel<T><<<dim3(static_cast<uint32_t>(rows)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t kv_attention_ws_bytes(int B, int Hq, int Hkv, int D, int max_new, int max_kv) {
  WsCursor c(nullptr);
  carve_attention(c, plan_attention(B, Hq, Hkv, max_new, max_kv), B, Hq, D, max_new);
  return c.used;
}

hipError_t launch_kv_attention(const KvCache& c, const KvBatch& bt, int max_kv, int type, int Hq, const KvRows& q,
                               const KvRows& out, float scale, int causal, int window, float* lse, void* ws,
                               hipStream_t stream) {
  const AttnPlan p = plan_attention(bt.B, Hq, c.Hkv, bt.max_new, max_kv);
  WsCursor cur(ws);
  const AttnWs w = carve_attention(cur, p, bt.B, Hq, c.D, bt.max_new);
  AttnArgs a = {c, bt, q, out, lse, w.po, w.pm, w.pl, scale, Hq, Hq / c.Hkv, causal, window, p.splits, p.tiles, 0};
  const int es = type == ET_F32 ? 4 : 2;
  a.o_vec = (reinterpret_cast<uintptr_t>(out.p) % (4 * es)) == 0 && out.tok % 4 == 0 && out.head % 4 == 0;
  return type == ET_F32 ? attend<uint32_t>(p, a, stream) : attend<uint16_t>(p, a, stream);
}

}  // namespace crvq
