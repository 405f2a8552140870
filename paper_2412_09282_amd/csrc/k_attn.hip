// Attention of new tokens over the paged 8-bit cache, out_i = sum_t p_t V_t with p = softmax(scale q_i . K_t).
//
// A wave owns 16 QB query rows ("columns": column c of a sequence and key head is new token c / G, query head
// c % G of the G that share the key head) and walks a range of tokens 64 at a time, with the running
// maximum m and sum l of the softmax in registers; nothing of size rows x tokens exists.
//   S^T = K Q^T on v_mfma_i32_16x16x64_i8: the key codes are the left operand as they lie in the cache, a query row is a
//     fixed-point number of 3 signed 8-bit digits, so the products are exact integers and no code is widened.  The score is the integer times alpha = (query step) (key scale) |scale| log2(e).
//   O^T += V^T P^T on v_mfma_f32_16x16x32_f16: the value codes lie transposed in the cache, 16 tokens of an
//     element in 16 bytes, and are widened to fp16 in registers (exact); the weights are rounded to fp16, once where every
//     wave has columns of its own (11 bits), else to two terms (22 bits).  Decoding steps wait for memory and take the second
//     term at no cost (one run: 32 sequences of up to 4096 tokens 138 us with it and without, heads of 256 elements 69 for 65);
//     prompts are bound by these instructions (with two 596 us for 384), and their error against 64 bits is that of
//     rounding the output to bf16 with either (1.67e-3 and 1.66e-3).  The page's
//     value scale goes into the weights, relative to a power of two 2^e of each column that follows the largest of its weights
//     times scale: scales of any size then add up as in fp32, and a page that a column does not see does not matter to it.
//     Weights below fp16's normal numbers (2^-21 of the row's largest) are added in further passes over the step, 2^14
//     times as large each, so that they keep their 11 bits too, down to fp32's smallest normal number; a pass is taken only
//     where there are any.  For fp32 queries the weights are three bf16 terms, which hold all of their 24 bits.
// The token in row 4 c + i of tile u is 16 c + 4 u + i: a lane (column r = lane % 16, quarter c = lane / 16) then
// holds the scores of 16 consecutive tokens, which are exactly its operands of the second product and, pages being
// multiples of 16, belong to one page.
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
// The maximum is renewed when a score, or a score with its page's value scale, passes it by more than 2^kSlack, so
// weights reach 2^kSlack; with a factor of at most 2^kLift they stay below fp16's 2^16 and keep 11 bits down to 2^-21 of the maximum.
constexpr float kSlack = 8.f;
constexpr int kLift = 7;
constexpr int kFaint = -64;    // pages whose scales are this far below 2^e: the softmax's sum is taken of weights of its own
constexpr float kFar = 0x1p23f;  // maxima from here on are whole numbers or coarser
constexpr int kNothing = -1024;  // exponent of a value scale of 0

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

// Which sequence, key head, split and tile of columns a workgroup has.  Key heads are neighbours, so that with a
// multiple of eight of them a chip's die reads few heads; the tiles of a sequence go last to first, so that the longest
// rows of a causal prompt start first; sequences come one after the other: the workgroups that a short one has no work for
// are then a run (as every second one they left half of the CUs idle: 556 against 404 us for two prompts of 2048
// and about 300, when that was changed).
struct Place {
  int hk, b, split, tile;
};
__device__ __forceinline__ Place place_of(const AttnArgs& a) {
  uint32_t item = blockIdx.x;
  Place p;
  p.hk = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  p.split = static_cast<int>(item % a.splits);
  item /= a.splits;
  p.tile = a.tiles - 1 - static_cast<int>(item % a.tiles);
  p.b = static_cast<int>(item / a.tiles);
  return p;
}

// The sequence that is `rank`-th by the mean length of its rows, len - n / 2, longest first, so that a call does not end
// with long rows on few CUs (one run: two prompts, 2048 rows over 4000 tokens and 393 over 3469: 392 us, in their own order 424).
// Up to 64 sequences, a lane each; more keep their order.
__device__ __forceinline__ int ranked(const KvBatch& bt, int rank) {
  if (bt.B > 64 || bt.B == 1) return rank;
  const int lane = threadIdx.x & 63;
  int64_t key = INT64_MIN;  // past the last sequence: after all of them
  if (lane < bt.B) key = 2 * static_cast<int64_t>(bt.kv_len[lane]) - bt.start[lane + 1] + bt.start[lane];
  int before = 0;
  for (int j = 0; j < bt.B; ++j) {
    const int64_t other = __shfl(key, j);
    before += other > key || (other == key && j < lane);
  }
  return __ffsll(static_cast<unsigned long long>(__ballot(lane < bt.B && before == rank))) - 1;
}

// The state of a wave's 16 QB columns; DT tiles of 16 elements hold a head.  HALF: keys come widened to fp16, and a
// query row is fp16 relative to a power of two (a bf16 element keeps its 8 bits down to 2^-28 of the row's largest).
// SMALL: the 16 tokens of a lane may have a page, and scales, of their own.
template <typename T, int DT, int QB, bool HALF, bool SMALL>
struct Columns {
  static constexpr int DC = HALF ? (DT + 1) / 2 : (DT + 3) / 4;      // chunks of a head: 32 (HALF) or 64 elements
  static constexpr int NT = HALF ? 1 : 3;                            // digits of a query element
  static constexpr double kSteps = 8355711.0;                        // 127 in every digit
  at_i4 q[QB][DC][NT];
  float step[QB], m[QB], l[QB];
  int e[QB];                          // exponents that value scales are taken relative to
  int lo[QB], hi[QB];                 // the tokens a column sees
  float slack;                        // kSlack; once a maximum has passed kFar, so low that every step renews it
  int first, last, all_lo, all_hi;    // the tokens any of them sees, and those that all of them see
  at_f4 o[QB][DT];                    // in units of 2^(m + e - kLift)

  // Queries: fixed point, 16 elements of a column and chunk in a lane; HALF: 8 of them.
  __device__ __forceinline__ void begin(const AttnArgs& a, const KvSeq& sq, bool ok, int hk, int col0, int cols) {
    const int r = threadIdx.x & 15, c = (threadIdx.x >> 4) & 3, D = a.c.D;
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      const int col = min(col0 + n * 16 + r, cols - 1);  // columns past the last one repeat it
      const int i = col / a.G, h = hk * a.G + col - i * a.G;
      const T* row = static_cast<const T*>(a.q.p) + (sq.row0 + i) * a.q.tok + h * a.q.head;
      constexpr int E = HALF ? 8 : 16;
      uint32_t most = 0;
#pragma unroll
      for (int ch = 0; ch < DC; ++ch)
        if ((ch * 4 + c) * E < D)
          for (int x = 0; x < E; ++x) most = max(most, __float_as_uint(elem(row, (ch * 4 + c) * E + x)) & 0x7fffffffu);
      most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 16)));
      most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 32)));
      const bool finite = most < 0x7f800000u;
      const double size = static_cast<double>(__uint_as_float(most)), slope = fabs(static_cast<double>(a.scale)) * kLog2e;
      const int up = 14 - (static_cast<int>(most >> 23) - 127);  // HALF: elements below 2^15
      const double inv = finite && most ? (a.scale < 0.f ? -kSteps : kSteps) / size : 0.0;
      step[n] = !finite ? __uint_as_float(0x7fc00000u) : static_cast<float>(HALF ? ldexp(slope, -up) : size / kSteps * slope);
#pragma unroll
      for (int ch = 0; ch < DC; ++ch) {
        const int at = (ch * 4 + c) * E;
        if constexpr (HALF) {
          at_h8 h = {};
          if (finite && at < D) {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              const float v = ldexpf(elem(row, at + x), up);
              h[x] = static_cast<_Float16>(a.scale < 0.f ? -v : v);
            }
          }
          q[n][ch][0] = __builtin_bit_cast(at_i4, h);
          continue;
        }
        uint32_t w[4][NT] = {};
        if (finite && at < D) {
#pragma unroll
          for (int x = 0; x < 16; ++x)
            digits<NT>(static_cast<int>(rint(static_cast<double>(elem(row, at + x)) * inv)), x & 3, w[x >> 2]);
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
      m[n] = -kInf;
      l[n] = 0.f;
      e[n] = 0;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[n][d] = at_f4{0.f, 0.f, 0.f, 0.f};
    }
    slack = kSlack;
    first = 0x7fffffff, last = 0, all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      if (hi[n] > 0) first = min(first, lo[n]);
      last = max(last, hi[n]);
      all_lo = max(all_lo, lo[n]);
      all_hi = min(all_hi, hi[n]);
    }
    last = wave_max(last);
    first = min(wave_min(first), last) & ~(kTokens - 1);
    all_lo = wave_max(all_lo);
    all_hi = wave_min(all_hi);
  }

  // The scores of 64 tokens, in query steps: key(u, ch) is the left operand of tile u and chunk ch.
  // LDS: operands come from LDS, and are asked for a tile before they are used.
  template <bool LDS, class Key>
  __device__ __forceinline__ void scores(at_f4 (&s)[QB][4], Key&& key) {
    at_i4 ahead[2][DC];
#pragma unroll
    for (int ch = 0; ch < DC; ++ch) ahead[0][ch] = key(0, ch);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const at_i4 (&k)[DC] = ahead[u & 1];
      if (u < 3) {
#pragma unroll
        for (int ch = 0; ch < DC; ++ch) ahead[(u + 1) & 1][ch] = key(u + 1, ch);
      }
      if constexpr (LDS) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < QB; ++n) {
        if constexpr (HALF) {
          at_f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ch = 0; ch < DC; ++ch)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(at_h8, k[ch]), __builtin_bit_cast(at_h8, q[n][ch][0]),
                                                         acc, 0, 0, 0);
          s[n][u] = acc;
          continue;
        }
        at_i4 acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[t] = at_i4{0, 0, 0, 0};
#pragma unroll
          for (int ch = 0; ch < DC; ++ch) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k[ch], q[n][ch][t], acc[t], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float low = static_cast<float>((acc[NT > 1 ? NT - 2 : 0][i] << 8) + acc[NT - 1][i]);
          s[n][u][i] = fmaf(static_cast<float>(acc[0][i]), 65536.f, low);
        }
      }
    }
  }

  // Scores to weights; ks and vs are the scales of this lane's 16 tokens, `good` whether they can be used.
  __device__ __forceinline__ void weigh(at_f4 (&s)[QB][4], int t0, float ks, float vs, bool good) {
    const int c = (threadIdx.x >> 4) & 3;
    // the value scale as 2^ve times a number in [1/2, 1)
    const bool some = good && vs > 0.f;
    const int ve = some ? __builtin_amdgcn_frexp_expf(vs) : kNothing;
    const float lift = (some ? __builtin_amdgcn_frexp_mantf(vs) : 1.f) * static_cast<float>(1 << kLift);
    const float lift_log = __builtin_amdgcn_logf(lift), unlift = __builtin_amdgcn_rcpf(lift);
    const bool whole = t0 >= all_lo && t0 + kTokens <= all_hi;
    uint32_t seen[QB];  // which of the lane's 16 tokens its column sees
    float by[QB], shift[QB];  // a weight, with its value scale, is exp2(score by + shift)
    float undo[QB];     // from the sum of the weights that enter the second product to that of the softmax
    if (!whole) {
      asm volatile("; a branch, not selections");
      const int base = t0 + 16 * c;
#pragma unroll
      for (int n = 0; n < QB; ++n) {
        const int x = min(max(lo[n] - base, 0), 16), y = min(max(hi[n] - base, 0), 16);
        seen[n] = ((1u << y) - 1u) & ~((1u << x) - 1u);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (!(seen[n] >> j & 1)) s[n][j >> 2][j & 3] = -kInf;  // stays below every score whatever its page's scale is
      }
    }
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      by[n] = good ? step[n] * ks : __uint_as_float(0x7fc00000u);
      float top = fmaxf(fmaxf(s[n][0][0], s[n][0][1]), s[n][0][2]);
#pragma unroll
      for (int j = 3; j < 16; ++j) top = fmaxf(top, s[n][j >> 2][j & 3]);
      top *= by[n];  // -infinity where the column sees none of them, or (alpha 0) NaN, which no comparison and no maximum takes
      float from = m[n];
      if (__builtin_expect(__any(top > m[n] + (slack - static_cast<float>(max(ve - e[n], 0)))), 0)) {
        asm volatile("; a branch, not selections");
        const float now = fmaxf(m[n], quarters_max(top));
        const float fall = m[n] > -kInf ? m[n] - now : -kInf;
        // the largest with its value scale, relative to `now` before exponents are added: scores may be past 2^24
        const float reach = fmaxf(fall + static_cast<float>(e[n]), quarters_max((top - now) + static_cast<float>(ve)));
        const int at = now > -kInf && reach > -kInf ? static_cast<int>(rintf(reach)) : 0;
        l[n] *= __builtin_amdgcn_exp2f(fall);
        const float keep = __builtin_amdgcn_exp2f(fall + static_cast<float>(e[n] - at));
        m[n] = now;
        e[n] = at;
        if (__any(now > -kInf && fabsf(now) >= kFar)) slack = -3e38f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[n][d] *= keep;
        from = now;
        if (__builtin_expect(slack < 0.f, 0)) {  // scores are rounded before the maximum is taken off, as it is: fused they would differ by 1 and more
#pragma unroll
          for (int j = 0; j < 16; ++j) s[n][j >> 2][j & 3] = s[n][j >> 2][j & 3] * by[n] - now;
          by[n] = 1.f;
          from = 0.f;
        }
      }
      const int rel = ve - e[n];
      undo[n] = ldexpf(unlift, -rel);
      if (__builtin_expect(__any(rel < kFaint), 0)) {  // their products with the value scale may vanish where they themselves do not
        asm volatile("; a branch, not selections");
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (whole || (seen[n] >> j & 1)) sum += __builtin_amdgcn_exp2f(fmaf(s[n][j >> 2][j & 3], by[n], -from));
        l[n] += sum;
        undo[n] = 0.f;
      }
      // weights p 2^.. = exp2(score - m) times the scale's factor, as exp2 of one fused multiply-add
      shift[n] = (lift_log + static_cast<float>(rel)) - from;
    }
#pragma unroll
    for (int n = 0; n < QB; ++n)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        s[n][j >> 2][j & 3] = __builtin_amdgcn_exp2f(fmaf(s[n][j >> 2][j & 3], by[n], shift[n]));
    if (!whole) {
      asm volatile("; a branch, not selections");
#pragma unroll
      for (int n = 0; n < QB; ++n)
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (!(seen[n] >> j & 1)) s[n][j >> 2][j & 3] = 0.f;
    }
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 16; ++j) sum += s[n][j >> 2][j & 3];
      l[n] = fmaf(sum, undo[n], l[n]);
    }
  }

  // Adds the values of 64 tokens: value(d, w) is the left operand (fp16; bf16 for fp32 queries) of tile d and half w.
  template <bool LDS, class Value>
  __device__ __forceinline__ void add(at_f4 (&s)[QB][4], Value&& value) {
    if constexpr (sizeof(T) == 2) {
      at_h8 pw[QB][2], pl[QB][2];  // the weights as fp16, and what that leaves of them
      at_s2 least = {0x7fff, 0x7fff};
      auto round = [&]() {
#pragma unroll
        for (int n = 0; n < QB; ++n)
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            const at_h2 h = __builtin_convertvector((at_f2{s[n][j >> 2][j & 3], s[n][j >> 2][(j & 3) + 1]}), at_h2);
            least = __builtin_elementwise_min(least, __builtin_bit_cast(at_s2, h));
            pw[n][j >> 3][j & 7] = h[0];
            pw[n][j >> 3][(j & 7) + 1] = h[1];
            if constexpr (!HALF) {
              pl[n][j >> 3][j & 7] = static_cast<_Float16>(s[n][j >> 2][j & 3] - static_cast<float>(h[0]));
              pl[n][j >> 3][(j & 7) + 1] = static_cast<_Float16>(s[n][j >> 2][(j & 3) + 1] - static_cast<float>(h[1]));
            }
          }
      };
      round();
      at_u4 ahead[2][2] = {{value(0, 0), value(0, 1)}};
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        if constexpr (LDS) {
          if (d + 1 < DT) ahead[(d + 1) & 1][0] = value(d + 1, 0), ahead[(d + 1) & 1][1] = value(d + 1, 1);
          __builtin_amdgcn_sched_barrier(0);
        } else if (d > 0) {
          ahead[d & 1][0] = value(d, 0);
          ahead[d & 1][1] = value(d, 1);
        }
        const at_h8 v0 = __builtin_bit_cast(at_h8, ahead[d & 1][0]), v1 = __builtin_bit_cast(at_h8, ahead[d & 1][1]);
#pragma unroll
        for (int n = 0; n < QB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pw[n][0], o[n][d], 0, 0, 0);
#pragma unroll
        for (int n = 0; n < QB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pw[n][1], o[n][d], 0, 0, 0);
        if constexpr (!HALF) {
#pragma unroll
          for (int n = 0; n < QB; ++n) {
            o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pl[n][0], o[n][d], 0, 0, 0);
            o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pl[n][1], o[n][d], 0, 0, 0);
          }
        }
      }
      // weights below fp16's normal numbers: what the rounding left of them, 2^14 times as large in every pass; nine of them reach
      // fp32's smallest normal number
      if (!__any(least[0] < 0x0400 || least[1] < 0x0400)) return;
      asm volatile("; a branch, not selections");
      float by = 1.f;
#pragma unroll 1
      for (int pass = 1; pass < 10; ++pass) {
        bool more = false;
#pragma unroll
        for (int n = 0; n < QB; ++n)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float x = s[n][j >> 2][j & 3];
            const float rest = fabsf(x) < 0x1p-14f ? (x - static_cast<float>(pw[n][j >> 3][j & 7])) * 0x1p14f : 0.f;
            s[n][j >> 2][j & 3] = rest;
            more |= rest != 0.f;
          }
        if (!__any(more)) return;
        by *= 0x1p-14f;
        round();
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const at_h8 v0 = __builtin_bit_cast(at_h8, value(d, 0)), v1 = __builtin_bit_cast(at_h8, value(d, 1));
#pragma unroll
          for (int n = 0; n < QB; ++n) {
            at_f4 part = {0.f, 0.f, 0.f, 0.f};
            part = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pw[n][0], part, 0, 0, 0);
            part = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pw[n][1], part, 0, 0, 0);
            if constexpr (!HALF) {
              part = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pl[n][0], part, 0, 0, 0);
              part = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pl[n][1], part, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][d][i] = fmaf(part[i], by, o[n][d][i]);
          }
        }
      }
    } else {
      at_b8 pb[QB][2][3];
#pragma unroll
      for (int n = 0; n < QB; ++n)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = s[n][2 * w + (j >> 2)][j & 3];
#pragma unroll
          for (int t = 0; t < 3; ++t) {  // the upper halves, then what they leave
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
        const at_b8 v0 = __builtin_bit_cast(at_b8, value(d, 0)), v1 = __builtin_bit_cast(at_b8, value(d, 1));
#pragma unroll
        for (int n = 0; n < QB; ++n)
#pragma unroll
          for (int t = 2; t >= 0; --t) {
            o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pb[n][0][t], o[n][d], 0, 0, 0);
            o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pb[n][1][t], o[n][d], 0, 0, 0);
          }
      }
    }
  }

  // Sums over the quarters, and o back from its power of two.
  __device__ __forceinline__ void end() {
#pragma unroll
    for (int n = 0; n < QB; ++n) {
      l[n] = quarters_sum(l[n]);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][d][i] = ldexpf(o[n][d][i], e[n] - kLift);
    }
  }
};

// Eight value codes as the second product takes them.
template <typename T>
__device__ __forceinline__ at_u4 widen(uint32_t a, uint32_t b) {
  if constexpr (sizeof(T) == 4)
    return __builtin_bit_cast(at_u4, widen8_bf16(a, b));
  else
    return __builtin_bit_cast(at_u4, widen8(a, b));
}

// A column's result, to the output or to the partial results of a split.
template <typename T>
struct Results {
  const AttnArgs& a;
  const KvSeq& sq;
  const Place& p;
  bool ok;
  __device__ __forceinline__ void row_of(int col, int& i, int& h) const {
    i = col / a.G;
    h = p.hk * a.G + col - i * a.G;
  }
  __device__ __forceinline__ int64_t part(int i, int h) const {
    return ((static_cast<int64_t>(p.split) * a.bt.B + p.b) * a.bt.max_new + i) * a.Hq + h;
  }
  __device__ __forceinline__ void stats(int col, float m, float l) const {
    int i, h;
    row_of(col, i, h);
    const float nan = __uint_as_float(0x7fc00000u);
    if (a.splits > 1) {
      a.pm[part(i, h)] = m;
      a.pl[part(i, h)] = ok ? l : nan;
    } else if (a.lse) {
      a.lse[static_cast<int64_t>(sq.row0 + i) * a.Hq + h] = !ok ? nan : l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
  }
  __device__ __forceinline__ void put(int col, int d, at_f4 x, float l) const {
    if (d >= a.c.D) return;
    int i, h;
    row_of(col, i, h);
    if (a.splits > 1) {
      if (l != 0.f) *reinterpret_cast<at_f4*>(a.po + part(i, h) * a.c.D + d) = x;
      return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = !ok ? __uint_as_float(0x7fc00000u) : l == 0.f ? 0.f : x[k] / l;
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
  }
};

// What the tokens of a step need from the block table and the scales.
struct Pages {
  const int32_t* table;
  int64_t n_pages;
  int len, log2;
  // the page of the 16 tokens from t on in the step at t0; past the length that of t0, whose codes are as good as any
  __device__ __forceinline__ int of(int t, int t0) const { return table[(t < len ? t : t0) >> log2]; }
  __device__ __forceinline__ bool there(int p) const { return static_cast<uint32_t>(p) < static_cast<uint32_t>(n_pages); }
};
__device__ __forceinline__ bool usable(float ks, float vs) { return ks >= 0.f && ks < kInf && vs >= 0.f && vs < kInf; }

// An equal share of the tokens first .. last for a split, in whole rounds.
__device__ __forceinline__ void share_of(const AttnArgs& a, int split, int round, int& first, int& last) {
  if (a.splits == 1) return;
  const int span = (last - first + a.splits - 1) / a.splits, share = (span + round - 1) / round * round;
  const int64_t from = first + static_cast<int64_t>(split) * share;
  first = static_cast<int>(from < last ? from : last);
  last = min(last, first + share);
}

// Few columns: the four waves of a workgroup share 16 and take turns at the tokens; the cache is read once, from
// memory into the operands' registers, a step's keys while the step before is computed.  Reads bound it: 32 sequences
// of 2048 to 4096 tokens (682 MB) take 133 us, 5.1 TB/s (a device copy, which writes as much as it reads, moves 4.9); one
// sequence of 131001 tokens (268 MB) in 64 shares of 8 heads 62.5 us, 4.3 TB/s, 8 us of it the join.
template <typename T, int DT, bool SMALL>
__global__ __launch_bounds__(256, DT <= 8 ? 2 : 1) void kv_attention_step_kernel(const AttnArgs a) {
  constexpr int kRow = DT * 16 + 4, kStride = 4 * kTokens;
  __shared__ __align__(16) float join[4 * 16 * kRow];
  __shared__ float join_m[64], join_l[64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = threadIdx.x & 15, c = (threadIdx.x >> 4) & 3;
  const int D = a.c.D, pl2 = a.c.page_log2, in_page = (1 << pl2) - 1;
  const Place pc = place_of(a);
  const KvSeq sq = kv_seq(a.bt, pc.b, pl2);
  const int cols = min(sq.n, a.bt.max_new) * a.G, col0 = pc.tile * 16;
  if (col0 >= cols) return;
  const bool ok = sq.ok && (sq.len == 0 || a.c.n_pages > 0);
  Columns<T, DT, 1, false, SMALL> w;
  w.begin(a, sq, ok, pc.hk, col0, cols);
  int first = w.first, last = w.last;
  share_of(a, pc.split, kStride, first, last);
  const int from = first + wave * kTokens;

  // addresses: the page's (uniform; SMALL: of this lane's 16 tokens) plus a lane's constant offset
  const Pages pages = {a.bt.table + static_cast<int64_t>(pc.b) * a.bt.ld_table, a.c.n_pages, sq.len, pl2};
  const int group = r >> 2;  // the 16 tokens of a step that this lane's row of a key tile belongs to
  auto uniform = [](int x) { return SMALL ? x : __builtin_amdgcn_readfirstlane(x); };
  auto head_of = [&](int p) { return static_cast<int64_t>(pages.there(p) ? p : 0) * a.c.Hkv + pc.hk; };
  auto key_page = [&](int t0) { return t0 < last ? uniform(pages.of(SMALL ? t0 + 16 * group : t0, t0)) : 0; };
  auto value_page = [&](int t0) { return t0 < last ? uniform(pages.of(SMALL ? t0 + 16 * c : t0, t0)) : 0; };
  const int64_t head_bytes = static_cast<int64_t>(D) << pl2;
  uint32_t koff[(DT + 3) / 4];
#pragma unroll
  for (int ch = 0; ch < (DT + 3) / 4; ++ch)  // past D the digits are 0, and any codes will do
    koff[ch] = ((SMALL ? 0 : 16 * group) + (r & 3)) * D + (ch * 64 + c * 16 < D ? ch * 64 + c * 16 : 0);
  const uint32_t voff = (static_cast<uint32_t>(r) << pl2) + (SMALL ? 0 : 16 * c);
  const int tiles = D >> 4;
  at_i4 kreg[4][(DT + 3) / 4];
  auto load_keys = [&](int t0, int p) {
    const int8_t* k = a.c.k + head_of(p) * head_bytes + ((SMALL ? t0 + 16 * group : t0) & in_page) * D;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int ch = 0; ch < (DT + 3) / 4; ++ch) kreg[u][ch] = *reinterpret_cast<const at_i4*>(k + (koff[ch] + 4 * u * D));
  };

  int kp = key_page(from), vp = SMALL ? value_page(from) : kp;
  if (from < last) load_keys(from, kp);
  kp = key_page(from + kStride);
  for (int t0 = from; t0 < last; t0 += kStride) {
    const int64_t head = head_of(vp);
    const int8_t* v = a.c.v + head * head_bytes + ((SMALL ? t0 + 16 * c : t0) & in_page);
    at_u4 vreg[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
      vreg[d] = *reinterpret_cast<const at_u4*>(v + (static_cast<int64_t>(min(d, tiles - 1) * 16) << pl2) + voff);
    const float ks = a.c.k_scale[head], vs = a.c.v_scale[head];
    const bool good = pages.there(vp) && usable(ks, vs);
    at_f4 s[1][4];
    w.template scores<false>(s, [&](int u, int ch) { return kreg[u][ch]; });
    if (t0 + kStride < last) load_keys(t0 + kStride, kp);
    vp = SMALL ? value_page(t0 + kStride) : kp;
    kp = key_page(t0 + 2 * kStride);
    w.weigh(s, t0, ks, vs, good);
    w.template add<false>(s, [&](int d, int half) {
      asm volatile("" : "+v"(vreg[d]));  // widened where it is used, in every pass
      return widen<T>(vreg[d][2 * half], vreg[d][2 * half + 1]);
    });
  }
  w.end();

  const int at0 = wave * 16 + r;
  if (c == 0) {
    join_m[at0] = w.m[0];
    join_l[at0] = w.l[0];
  }
#pragma unroll
  for (int d = 0; d < DT; ++d) *reinterpret_cast<at_f4*>(join + at0 * kRow + d * 16 + 4 * c) = w.o[0][d];
  __syncthreads();
  const Results<T> out = {a, sq, pc, ok};
  for (int x = threadIdx.x; x < 16 * DT * 4; x += 256) {
    const int col = x / (DT * 4), d = (x - col * (DT * 4)) * 4;
    if (col0 + col >= cols) break;
    float mm = -kInf;
#pragma unroll
    for (int k = 0; k < 4; ++k) mm = fmaxf(mm, join_m[k * 16 + col]);
    float ll = 0.f;
    at_f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = k * 16 + col;
      const float f = join_m[at] == -kInf ? 0.f : __builtin_amdgcn_exp2f(join_m[at] - mm);
      ll = fmaf(f, join_l[at], ll);
      y += f * *reinterpret_cast<const at_f4*>(join + at * kRow + d);
    }
    if (d == 0) out.stats(col0 + col, mm, ll);
    out.put(col0 + col, d, y, ll);
  }
}

// Many columns: every wave has 16 QB of its own, and the four of a workgroup walk the same tokens.  A step's keys
// and values pass through LDS, two steps of them, widened once for all four waves (keys of fp32 queries as they are).  Rows of
// LDS are padded by 16 bytes, and a key's row is u * 16 + r for the token that is row r of tile u, so that the 16 rows
// an instruction reads lie in different banks.  4096 tokens over 8192, 64 heads over 8, take
// 1.41 ms without a mask (780 TFLOP/s, of 1360 that a large library product of bf16 reaches).  A wave reads a step's keys and
// values, 32 KB, for 32 columns: 128 KB a workgroup and step, as many cycles of LDS as the products take of the matrix cores, and
// in one wave they come one after the other, as do scores, weights and values.  Two waves a SIMD hide a part of that (one: 1.95 for
// 1.33 ms, when that was measured).  Smaller calls lose at their end, when the last workgroups run alone: two prompts of 2048 and
// 393, 348 us (696 TFLOP/s; 360 to 382 with the calls in a graph, from one card to another).
template <typename T, int DT, int QB, bool SMALL>
__global__ __launch_bounds__(256, DT <= 8 ? 2 : 1) void kv_attention_prompt_kernel(const AttnArgs a) {
  constexpr bool HALF = sizeof(T) == 2;
  constexpr int kKeyRow = DT * 16 * (HALF ? 2 : 1) + 16, kValueRow = kTokens * 2 + 16;
  constexpr int kKeyBytes = kTokens * kKeyRow, kBuffer = kKeyBytes + DT * 16 * kValueRow;
  constexpr int kPer = (DT * 16 * 4 + 255) / 256;  // 16-byte pieces of keys, and of values, that a thread moves
  extern __shared__ __align__(16) uint8_t lds[];   // [2][kBuffer]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = threadIdx.x, r = tid & 15, c = (tid >> 4) & 3;
  const int D = a.c.D, pl2 = a.c.page_log2, in_page = (1 << pl2) - 1;
  Place pc = place_of(a);
  pc.b = __builtin_amdgcn_readfirstlane(ranked(a.bt, pc.b));
  const KvSeq sq = kv_seq(a.bt, pc.b, pl2);
  const int cols = min(sq.n, a.bt.max_new) * a.G, tile0 = pc.tile * (64 * QB), col0 = tile0 + wave * (16 * QB);
  if (tile0 >= cols) return;
  const bool ok = sq.ok && (sq.len == 0 || a.c.n_pages > 0), mine = col0 < cols;
  Columns<T, DT, QB, HALF, SMALL> w;
  w.begin(a, sq, ok, pc.hk, min(col0, cols - 1), cols);
  // the workgroup's tokens
  int* shared = reinterpret_cast<int*>(lds);
  if ((tid & 63) == 0) {
    shared[2 * wave] = w.first;
    shared[2 * wave + 1] = w.last;
  }
  __syncthreads();
  int first = 0x7fffffff, last = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (shared[2 * k + 1] > 0) first = min(first, shared[2 * k]);
    last = max(last, shared[2 * k + 1]);
  }
  last = __builtin_amdgcn_readfirstlane(last);
  first = min(__builtin_amdgcn_readfirstlane(first), last);
  __syncthreads();
  share_of(a, pc.split, kTokens, first, last);

  const Pages pages = {a.bt.table + static_cast<int64_t>(pc.b) * a.bt.ld_table, a.c.n_pages, sq.len, pl2};
  auto head_of = [&](int p) { return static_cast<int64_t>(pages.there(p) ? p : 0) * a.c.Hkv + pc.hk; };
  const int64_t head_bytes = static_cast<int64_t>(D) << pl2;
  // the pieces this thread moves: of keys, 16 elements of a token; of values, 16 tokens of an element
  const int pieces = 4 * D, d16 = D >> 4;
  int kt[kPer], ke[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int x = min(tid + i * 256, pieces - 1);
    kt[i] = x / d16;
    ke[i] = x - kt[i] * d16;
  }
  // A step's pages are looked up two steps ahead, its keys, values and scales are read one step ahead.
  int kp[SMALL ? kPer : 1], vp[SMALL ? kPer : 1], sp = 0;
  auto look_up = [&](int t0) {
    if (t0 >= last) return;
    if constexpr (SMALL) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        kp[i] = pages.of(t0 + (kt[i] & ~15), t0);
        vp[i] = pages.of(t0 + (min(tid + i * 256, pieces - 1) & 3) * 16, t0);
      }
      sp = pages.of(t0 + 16 * c, t0);
    } else {
      sp = __builtin_amdgcn_readfirstlane(pages.of(t0, t0));
    }
  };
  at_u4 kreg[kPer], vreg[kPer];
  float ks_next = 0.f, vs_next = 0.f;
  bool good_next = false;
  auto fetch = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int8_t* k = a.c.k + head_of(SMALL ? kp[SMALL ? i : 0] : sp) * head_bytes;
      kreg[i] = *reinterpret_cast<const at_u4*>(k + (((t0 + kt[i]) & in_page) * D + ke[i] * 16));
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int x = min(tid + i * 256, pieces - 1), g = (x & 3) * 16;
      const int8_t* v = a.c.v + head_of(SMALL ? vp[SMALL ? i : 0] : sp) * head_bytes;
      vreg[i] = *reinterpret_cast<const at_u4*>(v + (((x >> 2) << pl2) + ((t0 + g) & in_page)));
    }
    const int64_t head = head_of(sp);
    ks_next = a.c.k_scale[head];
    vs_next = a.c.v_scale[head];
    good_next = pages.there(sp);
  };
  auto settle = [&](uint8_t* to) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int x = min(tid + i * 256, pieces - 1);
      const int row = ((kt[i] >> 2) & 3) * 16 + (kt[i] >> 4) * 4 + (kt[i] & 3);
      if constexpr (HALF) {
        uint8_t* k = to + row * kKeyRow + ke[i] * 32;
        *reinterpret_cast<at_u4*>(k) = widen<T>(kreg[i][0], kreg[i][1]);
        *reinterpret_cast<at_u4*>(k + 16) = widen<T>(kreg[i][2], kreg[i][3]);
      } else {
        *reinterpret_cast<at_u4*>(to + row * kKeyRow + ke[i] * 16) = kreg[i];
      }
      uint8_t* v = to + kKeyBytes + (x >> 2) * kValueRow + (x & 3) * 32;
      *reinterpret_cast<at_u4*>(v) = widen<T>(vreg[i][0], vreg[i][1]);
      *reinterpret_cast<at_u4*>(v + 16) = widen<T>(vreg[i][2], vreg[i][3]);
    }
  };
  // what no piece fills: elements past D of the keys (their digits are 0) and value rows past D (their sums are
  // not stored) may hold anything that is finite, and are cleared once
  if (D < DT * 16) {
    for (int x = tid * 16; x < 2 * kBuffer; x += 256 * 16) *reinterpret_cast<at_u4*>(lds + x) = at_u4{0, 0, 0, 0};
    __syncthreads();
  }

  look_up(first);
  if (first < last) {
    fetch(first);
    settle(lds);
  }
  look_up(first + kTokens);
  __syncthreads();
  int buffer = 0;
  for (int t0 = first; t0 < last; t0 += kTokens) {
    const uint8_t* from = lds + buffer * kBuffer;
    const float ks = ks_next, vs = vs_next;
    const bool good = good_next && usable(ks, vs);
    if (t0 + kTokens < last) fetch(t0 + kTokens);
    look_up(t0 + 2 * kTokens);
    if (t0 + kTokens > w.first && t0 < w.last) {
      at_f4 s[QB][4];
      __builtin_amdgcn_s_setprio(1);
      w.template scores<true>(s, [&](int u, int ch) { return *reinterpret_cast<const at_i4*>(from + (u * 16 + r) * kKeyRow + ch * 64 + c * 16); });
      __builtin_amdgcn_s_setprio(0);
      w.weigh(s, t0, ks, vs, good);
      __builtin_amdgcn_s_setprio(1);
      const uint8_t* v = from + kKeyBytes + r * kValueRow + c * 32;
      w.template add<true>(s, [&](int d, int half) { return *reinterpret_cast<const at_u4*>(v + d * 16 * kValueRow + half * 16); });
      __builtin_amdgcn_s_setprio(0);
    }
    buffer ^= 1;
    if (t0 + kTokens < last) settle(lds + buffer * kBuffer);
    __syncthreads();
  }
  w.end();
  if (!mine) return;
  const Results<T> out = {a, sq, pc, ok};
#pragma unroll
  for (int n = 0; n < QB; ++n) {
    const int col = col0 + n * 16 + r;
    if (col >= cols) continue;
    if (c == 0) out.stats(col, w.m[n], w.l[n]);
#pragma unroll
    for (int d = 0; d < DT; ++d) out.put(col, d * 16 + 4 * c, w.o[n][d], w.l[n]);
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

// The same for few splits and many rows: D / 4 threads a (row, head), which walk the splits.
template <typename T>
__global__ __launch_bounds__(256) void kv_attention_join_rows_kernel(const AttnArgs a, int64_t items) {
  const int per = a.c.D >> 2, g = threadIdx.x / per, d = (threadIdx.x - g * per) * 4;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (256 / per) + g;
  if (g >= 256 / per || item >= items) return;
  const uint32_t row_of = static_cast<uint32_t>(item / a.Hq);
  const int h = static_cast<int>(item - static_cast<int64_t>(row_of) * a.Hq), b = static_cast<int>(row_of / a.bt.max_new);
  const int i = static_cast<int>(row_of - static_cast<uint32_t>(b) * a.bt.max_new);
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  if (i >= sq.n) return;
  float m = -kInf, l = 0.f;
  at_f4 y = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; ++s) {
    const int64_t at = s * items + item;
    const float ls = a.pl[at], ms = a.pm[at];
    if (ls == 0.f) continue;  // saw nothing and stored no output; a NaN goes on into l
    const float now = fmaxf(m, ms), keep = m == -kInf ? 0.f : __builtin_amdgcn_exp2f(m - now);
    const float f = ls == ls ? __builtin_amdgcn_exp2f(ms - now) : 0.f;
    l = fmaf(l, keep, ls == ls ? f * ls : ls);
    y = y * keep;
    if (f != 0.f) y += f * *reinterpret_cast<const at_f4*>(a.po + at * a.c.D + d);
    m = now;
  }
  const float bad = l - l;  // 0, or NaN
  const int64_t row = sq.row0 + i;
  T* out = static_cast<T*>(a.out.p) + row * a.out.tok + h * a.out.head + d;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float x = l == 0.f ? 0.f : y[k] / l + bad;
    if constexpr (sizeof(T) == 4)
      reinterpret_cast<float*>(out)[k] = x;
    else
      out[k] = static_cast<T>(f_bf16(x));
  }
  if (a.lse && d == 0) a.lse[row * a.Hq + h] = l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2 + bad;
}

// How a call is divided.  Shares are joined by a second launch; 512 workgroups are two a CU (256 to 2048 were measured: 1024
// cost a long sequence 68 us instead of 64 and prompts with heads of 192 elements 437 instead of 318).  One tile of columns: its workgroups' four waves share the columns (16) and take turns at the
// tokens; more: every wave has 16 prompt_blocks columns of its own.  Tokens are split over workgroups until
// kWorkgroups are at work, a share being at least kShare tokens.
struct AttnPlan {
  bool prompt;
  int tiles, splits;
};
constexpr int prompt_blocks(int D) { return D <= 128 ? 2 : 1; }  // what the registers hold
constexpr int64_t kWorkgroups = 512;
constexpr int kFewSplits = 8;
constexpr int kShare = 512;
AttnPlan plan_attention(int B, int Hq, int Hkv, int D, int max_new, int max_kv) {
  AttnPlan p;
  const int64_t cols = static_cast<int64_t>(max_new) * (Hq / Hkv);
  p.prompt = cols > 16;
  p.tiles = static_cast<int>(cdiv(cols, p.prompt ? 64 * prompt_blocks(D) : 16));
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
  constexpr int QB = prompt_blocks(DT * 16);
  const int64_t blocks = static_cast<int64_t>(p.tiles) * p.splits * a.bt.B * a.c.Hkv;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(blocks));
  const bool small = a.c.page_log2 < 6;
  const size_t lds = 2 * (kTokens * (DT * 16 * (sizeof(T) == 2 ? 2 : 1) + 16) + DT * 16 * (kTokens * 2 + 16));
  if (p.prompt) {
    if (small) kv_attention_prompt_kernel<T, DT, QB, true><<<grid, 256, lds, stream>>>(a);
    else kv_attention_prompt_kernel<T, DT, QB, false><<<grid, 256, lds, stream>>>(a);
  } else {
    if (small) kv_attention_step_kernel<T, DT, true><<<grid, 256, 0, stream>>>(a);
    else kv_attention_step_kernel<T, DT, false><<<grid, 256, 0, stream>>>(a);
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
  if (p.prompt && p.splits <= kFewSplits) {
    const int64_t each = 256 / (D >> 2);
    kv_attention_join_rows_kernel<T><<<dim3(static_cast<uint32_t>(cdiv(rows, each))), 256, 0, stream>>>(a, rows);
    return hipGetLastError();
  }
  kv_attention_join_kernel<T><<<dim3(static_cast<uint32_t>(rows)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t kv_attention_ws_bytes(int B, int Hq, int Hkv, int D, int max_new, int max_kv) {
  WsCursor c(nullptr);
  carve_attention(c, plan_attention(B, Hq, Hkv, D, max_new, max_kv), B, Hq, D, max_new);
  return c.used;
}

hipError_t launch_kv_attention(const KvCache& c, const KvBatch& bt, int max_kv, int type, int Hq, const KvRows& q,
                               const KvRows& out, float scale, int causal, int window, float* lse, void* ws,
                               hipStream_t stream) {
  const AttnPlan p = plan_attention(bt.B, Hq, c.Hkv, c.D, bt.max_new, max_kv);
  WsCursor cur(ws);
  const AttnWs w = carve_attention(cur, p, bt.B, Hq, c.D, bt.max_new);
  AttnArgs a = {c, bt, q, out, lse, w.po, w.pm, w.pl, scale, Hq, Hq / c.Hkv, causal, window, p.splits, p.tiles, 0};
  const int es = type == ET_F32 ? 4 : 2;
  a.o_vec = (reinterpret_cast<uintptr_t>(out.p) % (4 * es)) == 0 && out.tok % 4 == 0 && out.head % 4 == 0;
  return type == ET_F32 ? attend<uint32_t>(p, a, stream) : attend<uint16_t>(p, a, stream);
}

}  // namespace crvq
