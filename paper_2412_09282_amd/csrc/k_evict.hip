// Drafted tokens over the paged 8-bit cache, and the cache within a budget: the masks of a tree of drafts, the attention weight
// that every cached token received, the tokens that a budget keeps by it, and their move to other pages.
#include "kv_common.h"

namespace crvq {
namespace {

typedef int ev_i4 __attribute__((ext_vector_type(4)));
typedef float ev_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t ev_u4 __attribute__((ext_vector_type(4)));
typedef uint16_t ev_s2 __attribute__((ext_vector_type(2)));
typedef __bf16 ev_b8 __attribute__((ext_vector_type(8)));

constexpr float kInf = __builtin_inff();
constexpr float kMost = 0x1.fffffep127f;
constexpr float kLog2e = 1.4426950408889634f;

// ---- masks of a tree of drafted tokens --------------------------------------------------------------

// A thread walks from its token to the root: a handful of steps, read from the cache's nearest level.
__global__ __launch_bounds__(64) void tree_mask_kernel(const int32_t* parents, const int32_t* start, const int32_t* kv_len, int max_new,
                                                       int64_t n_tokens, int window, uint64_t* mask, int64_t ld, int32_t* places) {
  const int b = blockIdx.y, i = blockIdx.x * 64 + threadIdx.x;
  const int r0 = start[b], r1 = start[b + 1], len = kv_len[b];
  if (r0 < 0 || r1 < r0 || r1 > n_tokens || r1 - r0 > max_new || i >= r1 - r0) return;
  const int32_t* parent = parents + r0;
  // parents come before their children, so that every walk ends
  int depth = 0;
  bool good = true;
  for (int j = i; j >= 0; ++depth) {
    const int p = parent[j];
    good = good && p >= -1 && p < j;
    j = good ? p : -1;
  }
  const int64_t place = static_cast<int64_t>(len) - (r1 - r0) + depth - 1;
  if (places) places[r0 + i] = good && place >= 0 ? static_cast<int>(place) : -1;
  if (!mask) return;
  int j = i, left = good ? (window ? min(window, depth) : depth) : 0;
  for (int64_t w = ld - 1; w >= 0; --w) {
    uint64_t bits = 0;
    while (left > 0 && (j >> 6) >= w) {
      bits |= uint64_t{1} << (j & 63);
      j = parent[j];
      --left;
    }
    mask[(r0 + i) * ld + w] = bits;
  }
}

// ---- the attention weight of every cached token -------------------------------------------------------
//
// w_t = decay w_t + sum over the rows i and heads h that see t of exp(scale q_ih . K_t - lse_ih): the scores of a tile of 16
// tokens by 16 columns (column c of a sequence and key head is new token c / G, query head c % G of the G that share the
// key head) come from v_mfma_f32_16x16x32_bf16 with the key codes, which bf16 holds exactly, as left operand; fp32 queries are
// three bf16 terms.  A lane has one column and four tokens of a tile; sums go over the columns last.

struct WeightArgs {
  KvCache c;
  KvBatch bt;
  KvRows q;
  KvWeights w;
  float* part;  // [share][b][hk][max_kv], where shares > 1
  int Hq, G, shares, tiles, max_kv, q_vec;
};

// Eight codes as bf16, `by` (a power of two) times: integers of eight bits are the upper halves of their fp32.
__device__ __forceinline__ ev_b8 widen8(int a, int b, float by = 1.f) {
  ev_u4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? a : b;
    const float x = static_cast<float>(static_cast<int8_t>(w >> (16 * (i & 1)))) * by;
    const float y = static_cast<float>(static_cast<int8_t>(w >> (16 * (i & 1) + 8))) * by;
    v[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
  }
  return __builtin_bit_cast(ev_b8, v);
}

// A load from a place that is the same for the whole wave, on the scalar unit.
template <typename V>
__device__ __forceinline__ V scalar_load(const V* p) {
  const uint64_t at = reinterpret_cast<uintptr_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
  return *reinterpret_cast<const __attribute__((address_space(4))) V*>(static_cast<uint64_t>(hi) << 32 | lo);
}

// 16 or 4 bytes of every lane to LDS, one lane's after the other's from `to` on, which is the same for the whole wave.
typedef const __attribute__((address_space(1))) void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;
__device__ __forceinline__ void load_lds16(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds(reinterpret_cast<global_ptr>(reinterpret_cast<uintptr_t>(from)),
                                   reinterpret_cast<lds_ptr>(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(to))), 16, 0, 0);
}
__device__ __forceinline__ void load_lds4(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds(reinterpret_cast<global_ptr>(reinterpret_cast<uintptr_t>(from)),
                                   reinterpret_cast<lds_ptr>(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(to))), 4, 0, 0);
}

// Sums over the 16 lanes of a row, in every one of them.
__device__ __forceinline__ float row_sum(float x) {
  auto add = [&](auto ror) {
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ror)::value, 0xf, 0xf, false));
  };
  add(std::integral_constant<int, 0x128>{});  // rotated by 8, 4, 2, 1 lanes
  add(std::integral_constant<int, 0x124>{});
  add(std::integral_constant<int, 0x122>{});
  add(std::integral_constant<int, 0x121>{});
  return x;
}

// What a lane reads of a column's query: 16 elements of a chunk of 64, as it has 16 code bytes of a token.
template <typename T, int DC>
struct RawQuery {
  static constexpr int NV = sizeof(T) == 4 ? 4 : 2;
  ev_u4 x[DC][NV];
  float lse;

  // query row i, head g of the key head; always one that there is
  __device__ __forceinline__ void load(const WeightArgs& a, const KvSeq& sq, int hk, int i, int g) {
    const int c = (threadIdx.x >> 4) & 3, h = hk * a.G + g;
    const int64_t row = sq.row0 + i;
    lse = a.w.lse[row * a.Hq + h];
    const T* p = static_cast<const T*>(a.q.p) + row * a.q.tok + h * a.q.head;
#pragma unroll
    for (int ch = 0; ch < DC; ++ch) {
      const T* e = p + (ch * 64 + c * 16 < a.c.D ? ch * 64 + c * 16 : 0);  // past D the codes are 0
      if (a.q_vec) {
#pragma unroll
        for (int v = 0; v < NV; ++v) x[ch][v] = *reinterpret_cast<const ev_u4*>(e + v * (16 / NV));
      } else {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if constexpr (NV == 4) x[ch][v][k] = e[v * 4 + k];
            else x[ch][v][k] = e[v * 8 + 2 * k] | static_cast<uint32_t>(e[v * 8 + 2 * k + 1]) << 16;
          }
      }
    }
  }

  // Whether any of this lane's elements is 2^100 or more.
  __device__ __forceinline__ bool far() const {
    if constexpr (NV == 4) {
      uint32_t most = 0;
#pragma unroll
      for (int ch = 0; ch < DC; ++ch)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int k = 0; k < 4; ++k) most = max(most, x[ch][v][k] & 0x7fffffffu);
      return most >= 0x71800000u;
    } else {
      ev_s2 most = {0, 0};
#pragma unroll
      for (int ch = 0; ch < DC; ++ch)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int k = 0; k < 4; ++k) most = __builtin_elementwise_max(most, __builtin_bit_cast(ev_s2, x[ch][v][k] & 0x7fff7fffu));
      return max(most[0], most[1]) >= 0x7180;
    }
  }
};

// 16 columns: their queries as right operands, what they see, and their log-sum-exps in powers of two.  DC chunks of 64 elements hold a
// head; the first eight of a lane's 16 elements of a chunk are of one instruction, the others of the next.
template <typename T, int DC>
struct Queries {
  static constexpr int NT = sizeof(T) == 4 ? 3 : 1;
  ev_b8 q[DC][2][NT];
  float lse2;
  int lo, hi;
  const uint64_t* bits;

  // The operands; `ok`: of a row that has weights.
  __device__ __forceinline__ void operands(const RawQuery<T, DC>& raw, bool ok) {
    lse2 = ok ? raw.lse * kLog2e : 0.f;
#pragma unroll
    for (int ch = 0; ch < DC; ++ch) {
      if constexpr (NT == 1) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          ev_u4 v = raw.x[ch][half];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = ok ? v[k] : 0u;
          q[ch][half][0] = __builtin_bit_cast(ev_b8, v);
        }
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = ok ? __uint_as_float(raw.x[ch][2 * half + (e >> 2)][e & 3]) : 0.f;
#pragma unroll
          for (int t = 0; t < 3; ++t) {  // the upper halves, then what they leave
            ev_u4 v;
#pragma unroll
            for (int e = 0; e < 8; e += 2) v[e >> 1] = __builtin_amdgcn_perm(__float_as_uint(x[e + 1]), __float_as_uint(x[e]), 0x07060302u);
            q[ch][half][t] = __builtin_bit_cast(ev_b8, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] -= __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
          }
        }
      }
    }
  }
  // 2^-16 of them.
  __device__ __forceinline__ void bring_down() {
#pragma unroll
    for (int ch = 0; ch < DC; ++ch)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          ev_u4 v = __builtin_bit_cast(ev_u4, q[ch][half][t]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[e] = __builtin_amdgcn_perm(__float_as_uint(__uint_as_float(v[e] & 0xffff0000u) * 0x1p-16f),
                                         __float_as_uint(__uint_as_float(v[e] << 16) * 0x1p-16f), 0x07060302u);
          q[ch][half][t] = __builtin_bit_cast(ev_b8, v);
        }
  }
  __device__ __forceinline__ void set_plain(const RawQuery<T, DC>& raw) { operands(raw, true); }
  __device__ __forceinline__ void set(const WeightArgs& a, const KvSeq& sq, const RawQuery<T, DC>& raw, int i, bool there) {
    const bool ok = there && fabsf(raw.lse) < kInf;  // neither a row that sees nothing nor one that is NaN has weights
    operands(raw, ok);
    lo = hi = 0;
    bits = nullptr;
    if (!ok) return;
    const int context = sq.len - sq.n;
    hi = sq.len;
    if (a.w.tree.mask) {
      const int64_t row = sq.row0 + i;
      bits = a.w.tree.mask + row * a.w.tree.ld;
      if (a.w.window) {
        const int64_t from = static_cast<int64_t>(a.w.tree.places ? a.w.tree.places[row] : context + i) + 1 - a.w.window;
        lo = static_cast<int>(from < 0 ? 0 : from < context ? from : max(context, 0));
      }
    } else if (a.w.causal) {
      hi = min(hi, max(context + i + 1, 0));
      if (a.w.window) lo = max(context + i + 1 - a.w.window, 0);
    }
  }

  // Which of the tokens t .. t + 3 this lane's column sees; context: tokens before the new ones.
  __device__ __forceinline__ uint32_t sees(int t, int context) const {
    const int x = min(max(lo - t, 0), 4), y = min(max(hi - t, 0), 4);
    uint32_t m = ((1u << y) - 1u) & ~((1u << x) - 1u);
    if (bits && t + 3 >= context && m) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = t + i - context;
        if (j >= 0 && (m >> i & 1) && !(bits[j >> 6] >> (j & 63) & 1)) m &= ~(1u << i);
      }
    }
    return m;
  }
};

// 64 tokens of a wave, in four tiles of 16 that each lie in one page: their codes as they are in memory, and their scales.
template <int DC>
struct RawTokens {
  ev_i4 k[4][DC];
  float ks[4];  // times `slope`; 0 where `good` is not
  uint32_t good;  // tiles whose page and scale can be used

  __device__ __forceinline__ void load(const WeightArgs& a, const KvSeq& sq, int b, int hk, int t0, float slope) {
    const int r = threadIdx.x & 15, c = (threadIdx.x >> 4) & 3, D = a.c.D, pl2 = a.c.page_log2;
    const int32_t* table = a.bt.table + b * a.bt.ld_table;
    int64_t head[4];
    good = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = t0 + 16 * u, page = t < sq.len ? scalar_load(table + (t >> pl2)) : -1;
      const bool there = static_cast<uint32_t>(page) < static_cast<uint32_t>(a.c.n_pages);
      good |= there ? 1u << u : 0u;
      head[u] = static_cast<int64_t>(there ? page : 0) * a.c.Hkv + hk;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = t0 + 16 * u;
      const int8_t* p = a.c.k + ((head[u] << pl2) + ((t & ((1 << pl2) - 1)) + r)) * D + c * 16;
#pragma unroll
      for (int ch = 0; ch < DC; ++ch) {
        k[u][ch] = ev_i4{0, 0, 0, 0};
        if ((good >> u & 1) && ch * 64 + c * 16 < D) k[u][ch] = *reinterpret_cast<const ev_i4*>(p + ch * 64);
      }
      ks[u] = 0.f;
      if (good >> u & 1) ks[u] = scalar_load(a.c.k_scale + head[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (!(ks[u] >= 0.f && ks[u] < kInf)) good &= ~(1u << u);
      ks[u] = (good >> u & 1) ? __builtin_amdgcn_fmed3f(ks[u] * slope, -kMost, kMost) : 0.f;  // a number, for sums of 0
    }
  }
};

// Adds the weights of 16 columns to the sums of a tile of 16 tokens from t on: k are its left operands.
template <typename T, int DC>
__device__ __forceinline__ void add_weights(const ev_b8 (&k)[DC][2], float ks, bool good, const Queries<T, DC>& q, int t, int context,
                                            bool whole, ev_f4& sum) {
  ev_f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int n = Queries<T, DC>::NT - 1; n >= 0; --n)
#pragma unroll
    for (int ch = 0; ch < DC; ++ch) {
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[ch][0], q.q[ch][0][n], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[ch][1], q.q[ch][1][n], s, 0, 0, 0);
    }
  if (whole) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += __builtin_amdgcn_exp2f(fmaf(s[i], ks, -q.lse2));
  } else {
    asm volatile("; a branch, not selections");
    const uint32_t m = good ? q.sees(t + 4 * ((threadIdx.x >> 4) & 3), context) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[i], ks, -q.lse2));
      sum[i] += m >> i & 1 ? p : 0.f;
    }
  }
}

// The sums of 64 tokens over the columns: lane (r, c) takes the token of tile r / 4 that is element r % 4 of its quarter.
__device__ __forceinline__ float over_columns(const ev_f4 (&sum)[4]) {
  const int r = threadIdx.x & 15;
  float mine = 0.f;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = row_sum(sum[u][i]);
      mine = r == 4 * u + i ? x : mine;
    }
  return mine;
}
__device__ __forceinline__ int token_of(int t0) {
  const int r = threadIdx.x & 15, c = (threadIdx.x >> 4) & 3;
  return t0 + 16 * (r >> 2) + 4 * c + (r & 3);
}

// Up to 16 NB columns: their queries stay in registers and every wave walks 64 tokens at a time, the next ones' codes on their way.
// Memory bounds it: a token of 32 sequences of up to 4096, 32 heads of 128 (384 MB), 88 us, 4.3 TB/s, of fp32 queries 96;
// with 24 tokens each (two blocks of columns) 101 us, with 40 135.  Two waves a SIMD where the registers do: products then end in
// registers that the vector unit reads (40 tokens 136 us for 146).
template <typename T, int DC, int NB>
__global__ __launch_bounds__(256, DC * sizeof(T) <= 4 || (DC * NB <= 4 && DC * sizeof(T) <= 8) ? 2 : 1) void kv_weights_step_kernel(const WeightArgs a) {
  const int lane = threadIdx.x & 63, r = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t item = blockIdx.x;
  const int hk = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  const int part = static_cast<int>(item % a.shares), b = static_cast<int>(item / a.shares);
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  if (!sq.ok || sq.n == 0 || sq.len > a.max_kv) return;
  const int cols = sq.n * a.G, context = sq.len - sq.n, stride = a.shares * 256;
  int t0 = (part * 4 + wave) * 64;
  if (t0 >= sq.len) return;
  RawTokens<DC> next;
  float slope = a.w.scale * kLog2e;  // scores in powers of two
  next.load(a, sq, b, hk, t0, slope);
  Queries<T, DC> q[NB];
  bool far = false;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int col = min(n * 16 + r, cols - 1), i = col / a.G;
    RawQuery<T, DC> raw;
    raw.load(a, sq, hk, i, col - i * a.G);
    far = far || raw.far();
    q[n].set(a, sq, raw, i, n * 16 + r < cols);
  }
  // 2^-16 times, no sum of codes times queries leaves fp32; what products below 2^-126 lose by it is nothing beside them.
  if (__any(far)) {
    slope *= 0x1p16f;
#pragma unroll
    for (int u = 0; u < 4; ++u) next.ks[u] = __builtin_amdgcn_fmed3f(next.ks[u] * 0x1p16f, -kMost, kMost);
#pragma unroll
    for (int n = 0; n < NB; ++n) q[n].bring_down();
  }
  const int64_t head = static_cast<int64_t>(b) * a.c.Hkv + hk;
  for (; t0 < sq.len; t0 += stride) {
    const RawTokens<DC> now = next;
    const int t = token_of(t0);
    const int64_t at = head * a.w.ld + t;
    const float old = a.w.before && t < context ? a.w.before[at] : 0.f;
    if (t0 + stride < sq.len) next.load(a, sq, b, hk, t0 + stride, slope);
    bool whole[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
      whole[n] = now.good == 15u && __all(n * 16 + r >= cols || (q[n].lo <= t0 && q[n].hi >= t0 + 64 && (!q[n].bits || t0 + 64 <= context)));
    ev_f4 sum[4] = {};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      ev_b8 k[DC][2];
#pragma unroll
      for (int ch = 0; ch < DC; ++ch) {
        k[ch][0] = widen8(now.k[u][ch][0], now.k[u][ch][1]);
        k[ch][1] = widen8(now.k[u][ch][2], now.k[u][ch][3]);
      }
#pragma unroll
      for (int n = NB - 1; n >= 0; --n) {
        add_weights(k, now.ks[u], now.good >> u & 1, q[n], t0 + 16 * u, context, whole[n], sum[u]);
        if (whole[n] && n * 16 + r >= cols) sum[u] = ev_f4{0.f, 0.f, 0.f, 0.f};  // columns past the last one
      }
    }
    const float mine = over_columns(sum);
    if (t < sq.len) a.w.after[at] = a.w.before && t < context ? fmaf(a.w.decay, old, mine) : mine;
  }
}

// More columns: every wave keeps 64 tokens in registers, and the four of a workgroup walk the columns that see any of theirs, 32 at a
// time, whose queries lie in LDS for all of them, two steps ahead, put there by the loads themselves (16 bytes of a lane
// where it reads them).  The vector units bound it, with 16 exponentials, products and sums of a lane for a tile of 64 tokens by 16
// columns (over half of the cycles; the matrix instructions a third beside them): two prompts of up to 2048 rows over
// 4000 tokens, 64 heads over 8, take 221 us (841 TFLOP/s; 244 in a short run of a graph, as the figures below); one of 2048
// over 8192, 32 heads with keys of their own, 153 us (788 TFLOP/s); the two prompts in fp32, with three times the matrix
// instructions and one wave a SIMD, 785.
constexpr int weights_step_bytes(int dc, int nv) { return 2 * dc * nv * 1024 + 4 * 256; }
template <typename T, int DC, bool VEC>
__global__ __launch_bounds__(256, DC * sizeof(T) <= 4 ? 2 : 1) void kv_weights_kernel(const WeightArgs a) {
  constexpr int NV = RawQuery<T, DC>::NV, kPieces = DC * NV, kBlock = kPieces * 1024, kStage = weights_step_bytes(DC, NV);
  constexpr int kLoads = kPieces / 2 + 1;  // of a wave in a step
  extern __shared__ __align__(16) uint8_t lds[];  // [3 steps]([2 blocks of 16 columns][DC][NV][64 lanes][16], [4 waves][64 lanes] lse)
  const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t item = blockIdx.x;
  const int hk = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  const int share = static_cast<int>(item % a.shares);
  item /= a.shares;
  const int tile = static_cast<int>(item % a.tiles), b = static_cast<int>(item / a.tiles);
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  const int tile0 = tile * 256, t0 = tile0 + wave * 64;
  if (!sq.ok || sq.n == 0 || sq.len > a.max_kv || tile0 >= sq.len) return;
  const int cols = sq.n * a.G, context = sq.len - sq.n;
  // the columns that see any of the tokens from `from` to `to`
  auto first_of = [&](int from) { return a.w.causal && from > context ? (from - context) * a.G : 0; };
  auto last_of = [&](int to) {
    if (!a.w.causal || !a.w.window) return cols;
    return static_cast<int>(max<int64_t>(min<int64_t>(cols, (static_cast<int64_t>(to) + a.w.window - context) * a.G), 0));
  };
  int first = first_of(tile0) & ~31, last = last_of(tile0 + 255);
  // Every shares'-th step: those that need masks lie next to each other, and all shares read neighbouring queries at a time
  // (the two prompts 265 us for 300 with shares that lie one after the other).
  const int stride = 32 * a.shares;
  first += share * 32;
  const int my_first = first_of(t0), my_last = t0 < sq.len ? last_of(t0 + 63) : 0;
  ev_b8 k[4][DC][2];
  float ks[4];
  uint32_t good;
  {
    RawTokens<DC> raw;
    raw.load(a, sq, b, hk, t0, a.w.scale * kLog2e);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      // 2^-16 times, no sum of codes times queries leaves fp32.  What products below 2^-126 lose by it is below 2^-42 of a score
      // with scales below 2^60; with larger ones a score is out of fp32 before its sum is.
      const bool near = fabsf(raw.ks[u]) < 0x1p60f;
      const float by = near ? 0x1p-16f : 1.f;
#pragma unroll
      for (int ch = 0; ch < DC; ++ch) {
        k[u][ch][0] = widen8(raw.k[u][ch][0], raw.k[u][ch][1], by);
        k[u][ch][1] = widen8(raw.k[u][ch][2], raw.k[u][ch][3], by);
      }
      ks[u] = raw.ks[u] * (near ? 0x1p16f : 1.f);
    }
    good = raw.good;
  }
  // Columns between these two see every token of the wave: they need no masks, nor selections where no row is out.
  int plain_from = 0, plain_to = cols & ~31;
  if (a.w.tree.mask) {
    if (t0 + 64 > context || a.w.window) plain_to = 0;
  } else if (a.w.causal) {
    plain_from = max(t0 + 63 - context, 0) * a.G;
    if (a.w.window) plain_to = static_cast<int>(min<int64_t>(plain_to, (static_cast<int64_t>(t0) - context + a.w.window) * a.G) & ~int64_t{31});
  }
  if (good != 15u || t0 + 64 > sq.len) plain_to = 0;

  // Two waves fetch a block of a step's two.  This lane's column of the next one: its row and head, where its query and log-sum-exp
  // are, and how far these move in a step (`up` rows and `over` heads, a row more and G heads less where the heads end).
  const int blk_of = wave >> 1, half = wave & 1, up = stride / a.G, over = stride - up * a.G;
  int i = (first + blk_of * 16 + r) / a.G, g = first + blk_of * 16 + r - i * a.G;
  const T* q_at = static_cast<const T*>(a.q.p) + (sq.row0 + i) * a.q.tok + (hk * a.G + g) * a.q.head;
  const float* lse_at = a.w.lse + static_cast<int64_t>(sq.row0 + i) * a.Hq + hk * a.G + g;
  int64_t q_on = up * a.q.tok + over * a.q.head, q_wrap = a.q.tok - a.G * a.q.head;
  int64_t lse_on = up * a.Hq + over, lse_wrap = a.Hq - a.G;
  // what is there past the last column: the key head's first query
  const T* q_first = static_cast<const T*>(a.q.p) + sq.row0 * a.q.tok + hk * a.G * a.q.head;
  const float* lse_first = a.w.lse + static_cast<int64_t>(sq.row0) * a.Hq + hk * a.G;
  // In vector registers, as they are added to lanes' places: there are too few scalar ones
  // (252 us with them there, 244 now).
  asm("" : "+v"(q_on), "+v"(q_wrap), "+v"(lse_on), "+v"(lse_wrap), "+v"(q_first), "+v"(lse_first));
  int element[DC];  // past D the codes are 0
#pragma unroll
  for (int ch = 0; ch < DC; ++ch) element[ch] = (ch * 64 + c * 16 < a.c.D ? ch * 64 + c * 16 : 0) + half * (16 / NV);
  // Queries of 32 columns to LDS, and their log-sum-exps; past the last column those of one that there is.  Every wave has as
  // many loads as any other: every second piece of its block, and the block's log-sum-exps.
  auto fetch = [&](uint8_t* to) {
    const bool there = i < sq.n;
    const T* p = there ? q_at : q_first;
#pragma unroll
    for (int x = 0; x < kPieces / 2; ++x) {  // piece 2 x + half: chunk (2 x + half) / NV, part (2 x + half) % NV of a lane's elements
      const T* e = p + element[2 * x / NV] + 2 * x % NV * (16 / NV);
      uint8_t* at = to + blk_of * kBlock + (2 * x + half) * 1024;
      if constexpr (VEC) {
        load_lds16(e, at);
      } else {
        ev_u4 y;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          if constexpr (NV == 4) y[n] = e[n];
          else y[n] = e[2 * n] | static_cast<uint32_t>(e[2 * n + 1]) << 16;
        }
        *reinterpret_cast<ev_u4*>(at + lane * 16) = y;
      }
    }
    load_lds4(there ? lse_at : lse_first, to + 2 * kBlock + wave * 256);
    i += up;
    g += over;
    q_at += q_on;
    lse_at += lse_on;
    if (g >= a.G) {
      g -= a.G;
      ++i;
      q_at += q_wrap;
      lse_at += lse_wrap;
    }
  };
  ev_f4 total[4] = {}, sum[4] = {};
  int buffer = 0, n = 0;
  if (first < last) {
    fetch(lds);
    fetch(lds + kStage);
  }
  for (; first < last; first += stride) {
    // this step's loads have arrived (the next one's may be on their way), for every wave, and every wave has read
    // what the step after the next one takes the place of
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(VEC ? kLoads : 0) : "memory");
    const uint8_t* step = lds + buffer * kStage + lane * 16;
    auto read = [&](int blk, RawQuery<T, DC>& raw) {
#pragma unroll
      for (int ch = 0; ch < DC; ++ch)
#pragma unroll
        for (int v = 0; v < NV; ++v) raw.x[ch][v] = *reinterpret_cast<const ev_u4*>(step + blk * kBlock + (ch * NV + v) * 1024);
      raw.lse = *reinterpret_cast<const float*>(lds + buffer * kStage + 2 * kBlock + blk * 512 + lane * 4);
    };
    RawQuery<T, DC> raw[2];
    read(0, raw[0]);
    read(1, raw[1]);
    fetch(lds + (buffer == 0 ? 2 : buffer - 1) * kStage);  // while these are read (264 us after it, 252 now)
    if (first >= plain_from && first + 32 <= plain_to && __all(fabsf(raw[0].lse) < kInf && fabsf(raw[1].lse) < kInf)) {
      Queries<T, DC> q[2];
      q[0].set_plain(raw[0]);
      q[1].set_plain(raw[1]);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) add_weights(k[u], ks[u], true, q[blk], t0 + 16 * u, context, true, sum[u]);
    } else {
      asm volatile("; a branch, not selections");
#pragma unroll 1
      for (int blk = 0; blk < 2; ++blk) {
        const int col0 = first + blk * 16;
        if (col0 + 16 <= my_first || col0 >= min(last, my_last)) continue;
        RawQuery<T, DC> one;
        read(blk, one);
        Queries<T, DC> q;
        q.set(a, sq, one, min((col0 + r) / a.G, sq.n - 1), col0 + r < cols);
#pragma unroll
        for (int u = 0; u < 4; ++u) add_weights(k[u], ks[u], good >> u & 1, q, t0 + 16 * u, context, false, sum[u]);
      }
    }
    if (++n == 16) {  // sums of sums: the error of long ones grows with their root
      asm volatile("; a branch, not selections");
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        total[u] += sum[u];
        sum[u] = ev_f4{0.f, 0.f, 0.f, 0.f};
      }
      n = 0;
    }
    buffer = buffer == 2 ? 0 : buffer + 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing comes to LDS any more
#pragma unroll
  for (int u = 0; u < 4; ++u) sum[u] += total[u];
  const float mine = over_columns(sum);
  const int t = token_of(t0);
  if (t >= sq.len) return;
  const int64_t head = static_cast<int64_t>(b) * a.c.Hkv + hk;
  if (a.shares > 1) {
    a.part[((static_cast<int64_t>(share) * a.bt.B) * a.c.Hkv + head) * a.max_kv + t] = mine;
    return;
  }
  const int64_t at = head * a.w.ld + t;
  a.w.after[at] = a.w.before && t < context ? fmaf(a.w.decay, a.w.before[at], mine) : mine;
}

__global__ __launch_bounds__(256) void kv_weights_join_kernel(const WeightArgs a) {
  const int hk = blockIdx.y % a.c.Hkv, b = blockIdx.y / a.c.Hkv, t = blockIdx.x * 256 + threadIdx.x;
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  if (!sq.ok || sq.n == 0 || sq.len > a.max_kv || t >= sq.len) return;
  const int64_t head = static_cast<int64_t>(b) * a.c.Hkv + hk, at = head * a.w.ld + t;
  float x = 0.f;
  for (int s = 0; s < a.shares; ++s) x += a.part[((static_cast<int64_t>(s) * a.bt.B) * a.c.Hkv + head) * a.max_kv + t];
  a.w.after[at] = a.w.before && t < sq.len - sq.n ? fmaf(a.w.decay, a.w.before[at], x) : x;
}

// How a call is divided.  Columns that fit four blocks stay in registers (us, 32 sequences of up to 4096 tokens, 32 heads: 24 columns 106
// for 179 when they are walked, 40 147 for 200), the tokens over 2048 workgroups.  More are walked, in shares of 512 columns and more
// until 2048 workgroups are at work, of 128 until each CU has one, which a second launch joins in order (us, 300 rows over 1500 tokens, 12
// heads over 4: 24 in shares of 128 columns, 48 of 512; four sequences of 512 rows, heads of 256: 77 and 48).
struct WeightPlan {
  int blocks;  // of 16 columns in a wave's registers; 0: the columns are walked
  int shares, parts;  // parts: shares that are joined by a second launch
};
WeightPlan plan_weights(int B, int Hq, int Hkv, int max_new, int max_kv) {
  const int64_t cols = static_cast<int64_t>(max_new) * (Hq / Hkv), heads = static_cast<int64_t>(B) * Hkv, tiles = cdiv(max_kv, 256);
  auto shares = [](int64_t want, int64_t most) { return static_cast<int>(want < 1 || most < 1 ? 1 : want < most ? want : most); };
  if (cols <= 64) return {cols <= 16 ? 1 : cols <= 32 ? 2 : 4, shares(cdiv(2048, heads), tiles), 1};
  auto of = [&](int64_t workgroups, int64_t columns) {
    const int64_t want = cdiv(workgroups, heads * tiles);
    return shares(want < 16 ? want : 16, cdiv(cols, columns));
  };
  const int n = of(2048, 512), few = of(256, 128);
  return {0, n > few ? n : few, n > few ? n : few};
}

// ---- the tokens that a budget keeps ---------------------------------------------------------------------
//
// Keys of 32 bits order the weights; three passes of a radix select (11, 11 and 10 bits) find the smallest key that is kept and how many
// equal to it are, then the kept tokens are written in order.  Up to kSelectMost tokens one workgroup has a head's keys in
// its registers; beyond, a head's tokens are divided over workgroups, whose counts meet in the workspace between four launches.

// Orders weights as numbers: NaN below all, then from -infinity to infinity; 0 and -0 are equal.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 0u;
  const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct SelectArgs {
  const int32_t* kv_len;
  const float* weights;
  int64_t ld;
  KvKeep k;
  float* kept;  // [B][Hkv][k.ld], or NULL
  int Hkv, budget, sinks, recent;
  // of the divided form: `per` tokens a workgroup, `chunks` of them a head
  int64_t per;
  int chunks;
  uint32_t *bins[3], *above, *found;  // [heads][chunks][2048 / 2048 / 1024], [heads][chunks][2], [heads][4]
};

constexpr int kSelectThreads = 1024, kSelectMost = 16384;
__device__ constexpr int select_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ constexpr uint32_t select_mask(int pass) { return pass == 2 ? 1023u : 2047u; }

// What a head keeps.
struct SelectHead {
  int64_t row;
  int len, n, left;  // tokens, kept ones, and those among them that are kept for their weight
  const float* w;
  __device__ __forceinline__ SelectHead(const SelectArgs& a, int head, bool first) {
    const int b = head / a.Hkv, given = a.kv_len[b];
    row = head;
    len = given < 0 || given > a.ld ? 0 : given;
    n = min(len, a.budget);
    left = n < len ? n - a.sinks - a.recent : 0;  // where some are not kept, sinks and recent ones are so many
    w = a.weights + row * a.ld;
    if (first && head % a.Hkv == 0) a.k.len[b] = n;
  }
  __device__ __forceinline__ bool always(const SelectArgs& a, int t) const { return n == len || t < a.sinks || t >= len - a.recent; }
};

// Inclusive sums over a wave's lanes: within rows of 16, then a row's last lane to the rows after it.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes below
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 to the second row, 47 to the fourth
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
  return x;
}
// Inclusive sums over the workgroup's threads, and the total; `waves`: 16 entries that nobody else uses until the next barrier.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* waves, uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_scan(x);
  __syncthreads();
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int v = 0; v < kSelectThreads / 64; ++v) {
    const uint32_t y = waves[v];
    if (v < wave) x += y;
    total += y;
  }
  return x;
}

// The bin that the left-th largest key lies in, counts x0 and x1 being those of bins 2 t and 2 t + 1 of thread t, and what is left
// of `left` within it.
__device__ __forceinline__ void find_bin(uint32_t x0, uint32_t x1, uint32_t& left, uint32_t& bin, uint32_t* waves, uint32_t* pick) {
  uint32_t total;
  const uint32_t up_to = block_scan(x0 + x1, waves, total), above1 = total - up_to, above0 = above1 + x1;  // keys in higher bins
  if (above1 < left && left <= above1 + x1) pick[0] = 2 * threadIdx.x + 1, pick[1] = left - above1;
  if (above0 < left && left <= above0 + x0) pick[0] = 2 * threadIdx.x, pick[1] = left - above0;
  __syncthreads();
  bin = pick[0];
  left = pick[1];
}

// The weights of tokens t .. t + K - 1, 0 from `to` on.
struct __attribute__((packed, aligned(4))) FourWeights {
  float x[4];
};
template <int K>
__device__ __forceinline__ void load_weights(const float* from, int t, int to, float (&w)[K]) {
#pragma unroll
  for (int k = 0; k < K; k += 4) {
    if (t + k + 3 < to) {
      const FourWeights f = *reinterpret_cast<const FourWeights*>(from + t + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[k + e] = f.x[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[k + e] = t + k + e < to ? from[t + k + e] : 0.f;
    }
  }
}

// Writes those of a thread's K tokens from t on that are kept: with keys above `least`, and the first `equal` ones equal to it.
// before: how many of either kind there are in the tokens before the workgroup's, (above << 32) + equal; counted on.
template <int K>
__device__ __forceinline__ void write_kept(const SelectArgs& a, const SelectHead& h, const float (&w)[K], int t, int to, uint32_t least,
                                           uint32_t equal, uint64_t& before, uint32_t* waves) {
  uint32_t gt = 0, eq = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const bool there = t + k < to, always = there && h.always(a, t + k);
    const uint32_t x = key_of(w[k]);
    gt += always || (there && h.left > 0 && x > least);
    eq += there && !always && h.left > 0 && x == least;
  }
  static_assert(K * kSelectThreads < 65536, "both counts fit 32 bits");
  uint32_t total;
  const uint32_t up_to = block_scan(gt << 16 | eq, waves, total);
  uint32_t g = static_cast<uint32_t>(before >> 32) + (up_to >> 16) - gt, e = static_cast<uint32_t>(before) + (up_to & 65535u) - eq;  // before this thread's tokens
  before += static_cast<uint64_t>(total >> 16) << 32 | (total & 65535u);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const bool there = t + k < to, always = there && h.always(a, t + k);
    const uint32_t x = key_of(w[k]);
    const bool more = always || (there && h.left > 0 && x > least), same = there && !always && h.left > 0 && x == least;
    if (more || (same && e < equal)) {
      const int64_t at = h.row * a.k.ld + g + min(e, equal);
      a.k.keep[at] = t + k;
      if (a.kept) a.kept[at] = w[k];
    }
    g += more;
    e += same;
  }
}

// A head in one workgroup: thread t has tokens t K .. t K + K - 1.
template <int K>
__global__ __launch_bounds__(kSelectThreads) void kv_select_kernel(const SelectArgs a) {
  __shared__ uint32_t hist[2048], pick[2];
  __shared__ __align__(16) uint32_t waves[kSelectThreads / 64];
  const int tid = threadIdx.x, at = tid * K;
  const SelectHead h(a, blockIdx.x, tid == 0);
  float w[K];
  load_weights<K>(h.w, at, h.len, w);
  uint32_t least = 0xffffffffu, equal = 0, left = h.left;
  if (left > 0) {
    least = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = select_shift(pass);
      for (int x = tid; x < 2048; x += kSelectThreads) hist[x] = 0;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const uint32_t x = key_of(w[k]);
        const bool in = pass == 0 || x >> select_shift(pass == 0 ? 0 : pass - 1) == least >> select_shift(pass == 0 ? 0 : pass - 1);
        if (in && at + k < h.len && !h.always(a, at + k)) atomicAdd(&hist[x >> shift & select_mask(pass)], 1u);
      }
      __syncthreads();
      uint32_t bin;
      find_bin(hist[2 * tid], hist[2 * tid + 1], left, bin, waves, pick);
      least |= bin << shift;
    }
    equal = left;
  }
  uint64_t before = 0;
  write_kept<K>(a, h, w, at, h.len, least, equal, before, waves);
}

// Always kept tokens before token t.
__device__ __forceinline__ int n_always_before(const SelectArgs& a, const SelectHead& h, int t) {
  if (h.n == h.len) return t;
  return min(a.sinks, t) + max(t - (h.len - a.recent), 0);
}

// A head's chunk in one workgroup, launch PASS of four: counts of the chunk's keys by 11, 11 and 10 bits, each of those that share the
// higher bits of the smallest kept key, which the chunks' counts of the launch before give; then the kept tokens.
template <int PASS>
__global__ __launch_bounds__(kSelectThreads) void kv_select_chunk_kernel(const SelectArgs a) {
  __shared__ uint32_t hist[2048], pick[2];
  __shared__ __align__(16) uint32_t waves[kSelectThreads / 64];
  const int tid = threadIdx.x;
  const int head = blockIdx.x / a.chunks, chunk = blockIdx.x - head * a.chunks;
  const SelectHead h(a, head, PASS == 0 && chunk == 0 && tid == 0);
  const int64_t from = chunk * a.per;
  const int to = static_cast<int>(from + a.per < h.len ? from + a.per : h.len), chunks = static_cast<int>((h.len + a.per - 1) / a.per);
  if (from >= h.len || (PASS < 3 && h.left <= 0)) return;
  const int64_t mine = static_cast<int64_t>(head) * a.chunks + chunk;
  constexpr int kBins[3] = {2048, 2048, 1024};
  // rounds of 8 neighbouring tokens a thread; the first one's weights, and what the chunks before keep for their higher bits, are on
  // their way while the bin is found (four launches over 131001 tokens of 8 heads 31 us, one load after the other 35)
  constexpr int K = 8, kRound = K * kSelectThreads;
  float w[K];
  load_weights<K>(h.w, static_cast<int>(from) + tid * K, to, w);
  uint32_t above = 0, same = 0;
  if (PASS == 3 && h.left > 0)
    for (int x = tid; x < 2 * chunk; x += kSelectThreads) above += a.above[static_cast<int64_t>(head) * a.chunks * 2 + x];
  uint32_t* found = a.found + static_cast<int64_t>(head) * 4;  // the first two bins, and what is left within the second
  uint32_t least = 0xffffffffu, left = h.left, bin = 0;
  if (PASS > 0 && h.left > 0) {
    if (PASS > 1) {
      least = found[0] << 21;
      left = found[1];
    } else {
      least = 0;
    }
    if (PASS > 2) {
      least |= found[2] << 10;
      left = found[3];
    }
    // all chunks' counts of the launch before; this chunk's keys above the bin that they give are kept
    constexpr int kOf = PASS > 0 ? PASS - 1 : 0, kCount = kBins[kOf];
    uint32_t x[2] = {0, 0}, own[2] = {0, 0}, below[2] = {0, 0};
    if (2 * tid < kCount)
#pragma unroll 8
      for (int c = 0; c < chunks; ++c) {
        const uint2 y = *reinterpret_cast<const uint2*>(a.bins[kOf] + (static_cast<int64_t>(head) * a.chunks + c) * kCount + 2 * tid);
        x[0] += y.x, x[1] += y.y;
        if (c == chunk) own[0] = y.x, own[1] = y.y;
        if (c < chunk) below[0] += y.x, below[1] += y.y;
      }
    find_bin(x[0], x[1], left, bin, waves, pick);
    least |= bin << select_shift(kOf);
    if (PASS < 3) {
      uint32_t total;
      block_scan((2 * tid > static_cast<int>(bin) ? own[0] : 0u) + (2 * tid + 1 > static_cast<int>(bin) ? own[1] : 0u), waves, total);
      if (tid == 0) {
        a.above[mine * 2 + kOf] = total;
        if (chunk == 0) {
          found[2 * kOf] = bin;
          found[2 * kOf + 1] = left;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (2 * tid + e > static_cast<int>(bin)) above += below[e];
        if (2 * tid + e == static_cast<int>(bin)) same = below[e];
      }
    }
  }
  if constexpr (PASS < 3) {
    constexpr int kHigher = PASS > 0 ? select_shift(PASS - 1) : 0;
    for (int x = tid; x < kBins[PASS]; x += kSelectThreads) hist[x] = 0;
    __syncthreads();
    for (int64_t t0 = from; t0 < to; t0 += kRound) {
      const int t = static_cast<int>(t0) + tid * K;
      if (t0 != from) load_weights<K>(h.w, t, to, w);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const uint32_t x = key_of(w[k]);
        if ((PASS == 0 || x >> kHigher == least >> kHigher) && t + k < to && !h.always(a, t + k))
          atomicAdd(&hist[x >> select_shift(PASS) & select_mask(PASS)], 1u);
      }
    }
    __syncthreads();
    for (int x = tid; x < kBins[PASS]; x += kSelectThreads) a.bins[PASS][mine * kBins[PASS] + x] = hist[x];
  } else {
    const uint32_t equal = h.left > 0 ? left : 0;
    // kept tokens of the chunks before: those above the bins, those above the key in the last bins, and the always kept ones
    uint32_t all_above, all_same;
    block_scan(above, waves, all_above);
    block_scan(same, waves, all_same);
    uint64_t before = (static_cast<uint64_t>(all_above) + n_always_before(a, h, static_cast<int>(from))) << 32 | all_same;
    for (int64_t t0 = from; t0 < to; t0 += kRound) {
      const int t = static_cast<int>(t0) + tid * K;
      if (t0 != from) load_weights<K>(h.w, t, to, w);
      write_kept<K>(a, h, w, t, to, least, equal, before, waves);
    }
  }
}

// ---- kept tokens to other pages -------------------------------------------------------------------------

struct GatherArgs {
  KvCache c;
  const int32_t *table, *to, *kv_len;
  int64_t ld_table, ld_to;
  KvKeep k;
  int B, pages;  // pages: grid's bound of a sequence's new ones
  int slices;    // 0: a workgroup moves a page's keys and values; else the first one the keys, the others slices of the values
};

// Four codes times a factor each, rounded to the nearest integer: the product's last places under 1.5 * 2^23.
__device__ __forceinline__ uint32_t moved4(uint32_t codes, const float (&f)[4]) {
  uint32_t z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y = static_cast<float>(static_cast<int8_t>(codes >> (8 * i))) * f[i];
    z[i] = __float_as_uint(y + 12582912.f);
  }
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(z[3], z[2], 0x0c0c0400u), __builtin_amdgcn_perm(z[1], z[0], 0x0c0c0400u), 0x05040100u);
}

// A new page's scale is the largest of its tokens' old ones; a code becomes rint(c (old / new)).  Keys move 16 bytes at a time.  Values
// lie transposed, so that a kept one is a byte among others that are not kept: neighbouring tokens of one old page are a run,
// and the runs' rows pass through LDS whole, some elements at a time, where they are few enough; otherwise byte by byte (one
// sequence of 131001 tokens to 16000, 8 heads, pages of 128: 57 us, most of it the 134 MB of values that the kept eighth lies in;
// 32 sequences of up to 4096 tokens to 1024, 32 heads, pages of 64: 174 us, byte by byte 249; with pages of 32, which go byte by
// byte, 265, of 16 318).
constexpr int kGatherLds = 16384;
__global__ __launch_bounds__(256) void kv_gather_kernel(const GatherArgs a) {
  __shared__ int64_t from[256];     // the token's head and slot: (page * Hkv + hk) * page size + slot
  __shared__ float by[2][256];      // old scale over new
  __shared__ float red[2][4];
  __shared__ int64_t run_head[256];  // the old page's head of a run
  __shared__ int runs_of[4];
  extern __shared__ __align__(16) uint8_t rows[];  // kGatherLds bytes where pages are of 64 tokens or more: [run][element][slot]
  const int tid = threadIdx.x, D = a.c.D, pl2 = a.c.page_log2, P = 1 << pl2;
  uint32_t item = blockIdx.x;
  const int slice = static_cast<int>(item % (a.slices + 1));
  item /= a.slices + 1;
  const int hk = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  const int p = static_cast<int>(item % a.pages), b = static_cast<int>(item / a.pages);
  const int len = a.kv_len[b], count = a.k.len[b], at0 = p << pl2;
  if (count <= at0 || count > a.k.ld || count > a.ld_to << pl2) return;
  const int dest = a.to[b * a.ld_to + p];
  if (static_cast<uint32_t>(dest) >= static_cast<uint32_t>(a.c.n_pages)) return;
  const int n = min(P, count - at0);
  // the tokens' places and scales
  const float nan = __uint_as_float(0x7fc00000u);
  float ks = 0.f, vs = 0.f;
  if (tid < n) {
    const int t = a.k.keep[(static_cast<int64_t>(b) * a.k.heads + (a.k.heads > 1 ? hk : 0)) * a.k.ld + at0 + tid];
    int page = -1;
    if (t >= 0 && t < len && len <= a.ld_table << pl2) page = a.table[b * a.ld_table + (t >> pl2)];
    const bool good = static_cast<uint32_t>(page) < static_cast<uint32_t>(a.c.n_pages);
    const int64_t head = static_cast<int64_t>(good ? page : 0) * a.c.Hkv + hk;
    from[tid] = (head << pl2) + (t & (P - 1));
    ks = good ? a.c.k_scale[head] : nan;
    vs = good ? a.c.v_scale[head] : nan;
    // -0 is 0, whose bits lie below all others
    ks = ks > 0.f && ks < kInf ? ks : ks == 0.f ? 0.f : nan;
    vs = vs > 0.f && vs < kInf ? vs : vs == 0.f ? 0.f : nan;
  }
  // the largest as bits: NaN lies above all
  uint32_t mk = __float_as_uint(ks), mv = __float_as_uint(vs);
  for (int o = 32; o; o >>= 1) {
    mk = max(mk, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mk), o)));
    mv = max(mv, static_cast<uint32_t>(__shfl_xor(static_cast<int>(mv), o)));
  }
  if ((tid & 63) == 0) red[0][tid >> 6] = __uint_as_float(mk), red[1][tid >> 6] = __uint_as_float(mv);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    mk = max(mk, __float_as_uint(red[0][i]));
    mv = max(mv, __float_as_uint(red[1][i]));
  }
  const float k_new = __uint_as_float(mk), v_new = __uint_as_float(mv);
  if (tid < n) {
    by[0][tid] = ks == k_new ? 1.f : ks / k_new;  // 0 / 0 among them
    by[1][tid] = vs == v_new ? 1.f : vs / v_new;
  }
  const bool k_ok = k_new == k_new, v_ok = v_new == v_new;
  // runs, and which one each token is of
  const bool begins = tid < n && (tid == 0 || from[tid] >> pl2 != from[tid - 1] >> pl2);
  const unsigned long long begun = __ballot(begins);
  if ((tid & 63) == 0) runs_of[tid >> 6] = __popcll(begun);
  __syncthreads();
  int run = __popcll(begun & ((2ull << (tid & 63)) - 1)) - 1, runs = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < tid >> 6) run += runs_of[i];
    runs += runs_of[i];
  }
  if (begins) run_head[run] = from[tid] >> pl2;
  const int64_t head = static_cast<int64_t>(dest) * a.c.Hkv + hk;
  if (tid == 0 && slice == 0) {
    a.c.k_scale[head] = k_new;
    a.c.v_scale[head] = v_new;
  }
  auto moved = [](int8_t c, float f) { return static_cast<int8_t>(rintf(static_cast<float>(c) * f)); };
  const int d16 = D >> 4;
  int8_t* k_to = a.c.k + (head << pl2) * D;
  for (int x = tid; x < P * d16 && slice == 0; x += 256) {
    const int j = x / d16, e = (x - j * d16) * 16;
    ev_i4 y = {0, 0, 0, 0};
    if (j < n && k_ok) {
      y = *reinterpret_cast<const ev_i4*>(a.c.k + from[j] * D + e);
      const float f = by[0][j];
      if (f != 1.f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = static_cast<int>(moved4(static_cast<uint32_t>(y[i]), {f, f, f, f}));
      }
    }
    *reinterpret_cast<ev_i4*>(k_to + j * D + e) = y;
  }
  // the elements of the values that are this workgroup's
  const int per = a.slices ? (D / 16 + a.slices - 1) / a.slices * 16 : D, first = a.slices ? (slice - 1) * per : 0, last = min(D, first + per);
  if (slice == 0 ? a.slices > 0 : first >= last) return;
  int8_t* v_to = a.c.v + (head << pl2) * D;
  if (!v_ok || P < 64 || runs << pl2 > kGatherLds / 4) {
    for (int x = (first << pl2) + tid; x < last << pl2; x += 256) {
      const int e = x >> pl2, j = x & (P - 1);
      int8_t y = 0;
      if (j < n && v_ok) {
        const int64_t head_from = from[j] >> pl2;
        y = moved(a.c.v[((head_from * D + e) << pl2) + (from[j] & (P - 1))], by[1][j]);
      }
      v_to[x] = y;
    }
    return;
  }
  // this thread's four tokens of an element: where they are in their run's row, and their factors
  __shared__ int place[256];
  const int lanes = P >> 2, j0 = (tid & (lanes - 1)) * 4, each = min(D, kGatherLds / (runs << pl2));  // elements at a time
  if (tid < n) place[tid] = ((run * each) << pl2) + static_cast<int>(from[tid] & (P - 1));
  __syncthreads();
  int at[4];
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at[i] = j0 + i < n ? place[j0 + i] : 0;
    f[i] = j0 + i < n ? by[1][j0 + i] : 0.f;
  }
  // the rows of the next elements are on their way while these are written (the 32 sequences 174 us for 177, 30000 of 32768
  // tokens 61 for 65; 4000 of 16000, whose runs are short, 27 for 26)
  constexpr int kHeld = kGatherLds / 16 / 256;
  ev_i4 held[kHeld];
  auto rows_of = [&](int e0, auto&& use) {  // this thread's 16-byte pieces: of run u, y pieces into its elements from e0 on
    const int row_pieces = min(each, last - e0) << pl2 >> 4;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int x = tid + i * 256, u = x / row_pieces;
      if (u < runs) use(i, u, x - u * row_pieces);
    }
  };
  auto fetch = [&](int e0) {
    rows_of(e0, [&](int i, int u, int y) {
      held[i] = *reinterpret_cast<const ev_i4*>(a.c.v + ((run_head[u] * D + e0) << pl2) + y * 16);
    });
  };
  // all waves' LDS accesses are over; loads and stores to memory go on
  auto barrier = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  fetch(first);
  for (int e0 = first; e0 < last; e0 += each) {
    const int count = min(each, last - e0);
    barrier();
    rows_of(e0, [&](int i, int u, int y) { *reinterpret_cast<ev_i4*>(rows + ((u * each) << pl2) + y * 16) = held[i]; });
    barrier();
    if (e0 + each < last) fetch(e0 + each);
    for (int x = tid; x < count * lanes; x += 256) {
      const int e = x / lanes;
      const uint8_t* row = rows + (e << pl2);
      const uint32_t word = row[at[0]] | static_cast<uint32_t>(row[at[1]]) << 8 | static_cast<uint32_t>(row[at[2]]) << 16 |
                            static_cast<uint32_t>(row[at[3]]) << 24;
      *reinterpret_cast<uint32_t*>(v_to + (static_cast<int64_t>(e0 + e) << pl2) + j0) = moved4(word, f);
    }
  }
}

}  // namespace

hipError_t launch_tree_mask(int B, const int32_t* parents, const int32_t* start, const int32_t* kv_len, int max_new,
                            int64_t n_tokens, int window, uint64_t* mask, int64_t ld, int32_t* places, hipStream_t stream) {
  if (B > 65535) return hipErrorInvalidConfiguration;
  tree_mask_kernel<<<dim3(static_cast<uint32_t>(cdiv(max_new, 64)), static_cast<uint32_t>(B)), 64, 0, stream>>>(
      parents, start, kv_len, max_new, n_tokens, window, mask, ld, places);
  return hipGetLastError();
}

size_t kv_weights_ws_bytes(int B, int Hq, int Hkv, int D, int max_new, int max_kv) {
  const WeightPlan p = plan_weights(B, Hq, Hkv, max_new, max_kv);
  WsCursor c(nullptr);
  if (p.parts > 1) c.take<float>(static_cast<size_t>(p.parts) * B * Hkv * max_kv);
  return c.used;
}

hipError_t launch_kv_weights(const KvCache& c, const KvBatch& bt, int max_kv, int type, int Hq, const KvRows& q,
                             const KvWeights& w, void* ws, hipStream_t stream) {
  const WeightPlan p = plan_weights(bt.B, Hq, c.Hkv, bt.max_new, max_kv);
  const int es = type == ET_F32 ? 4 : 2, tiles = static_cast<int>(cdiv(max_kv, 256));
  WsCursor cur(ws);
  float* part = p.parts > 1 ? cur.take<float>(static_cast<size_t>(p.parts) * bt.B * c.Hkv * max_kv) : nullptr;
  WeightArgs a = {c, bt, q, w, part, Hq, Hq / c.Hkv, p.shares, tiles, max_kv, 0};
  a.q_vec = reinterpret_cast<uintptr_t>(q.p) % 16 == 0 && q.tok * es % 16 == 0 && q.head * es % 16 == 0;
  const int64_t blocks = static_cast<int64_t>(bt.B) * c.Hkv * p.shares * (p.blocks ? 1 : tiles);
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffffLL || static_cast<int64_t>(bt.B) * c.Hkv > 65535) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(blocks));
  auto as = [&](auto t, auto dc) {
    using T = decltype(t);
    constexpr size_t lds = 3 * weights_step_bytes(decltype(dc)::value, sizeof(T) == 4 ? 4 : 2);
    if (p.blocks == 1) kv_weights_step_kernel<T, decltype(dc)::value, 1><<<grid, 256, 0, stream>>>(a);
    else if (p.blocks == 2) kv_weights_step_kernel<T, decltype(dc)::value, 2><<<grid, 256, 0, stream>>>(a);
    else if (p.blocks == 4) kv_weights_step_kernel<T, decltype(dc)::value, 4><<<grid, 256, 0, stream>>>(a);
    else if (a.q_vec) kv_weights_kernel<T, decltype(dc)::value, true><<<grid, 256, lds, stream>>>(a);
    else kv_weights_kernel<T, decltype(dc)::value, false><<<grid, 256, lds, stream>>>(a);
    return hipGetLastError();
  };
  auto of = [&](auto t) {
    return c.D <= 64 ? as(t, std::integral_constant<int, 1>{}) : c.D <= 128 ? as(t, std::integral_constant<int, 2>{})
                                                                              : as(t, std::integral_constant<int, 4>{});
  };
  const hipError_t e = type == ET_F32 ? of(uint32_t{}) : of(uint16_t{});
  if (e != hipSuccess || p.parts == 1) return e;
  kv_weights_join_kernel<<<dim3(static_cast<uint32_t>(tiles), static_cast<uint32_t>(bt.B * c.Hkv)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

namespace {
// Chunks of the divided form: of 8192 tokens, or what leaves about 1024 of them for all heads.
int select_chunks(int64_t heads, int64_t ld) {
  if (ld <= kSelectMost) return 0;
  const int64_t most = cdiv(ld, 8192), want = cdiv(1024, heads);
  return static_cast<int>(want < most ? want : most);
}
void carve_select(WsCursor& c, int64_t heads, int chunks, SelectArgs& a) {
  if (!chunks) return;
  const size_t n = static_cast<size_t>(heads) * chunks;
  a.bins[0] = c.take<uint32_t>(n * 2048);
  a.bins[1] = c.take<uint32_t>(n * 2048);
  a.bins[2] = c.take<uint32_t>(n * 1024);
  a.above = c.take<uint32_t>(n * 2);
  a.found = c.take<uint32_t>(static_cast<size_t>(heads) * 4);
}
}  // namespace

size_t kv_select_ws_bytes(int B, int Hkv, int64_t ld) {
  const int64_t heads = static_cast<int64_t>(B) * Hkv;
  SelectArgs a = {};
  WsCursor c(nullptr);
  carve_select(c, heads, select_chunks(heads, ld), a);
  return c.used;
}

hipError_t launch_kv_select(int B, int Hkv, const int32_t* kv_len, const float* weights, int64_t ld, int budget, int sinks,
                            int recent, const KvKeep& k, float* kept_weights, void* ws, hipStream_t stream) {
  const int64_t heads = static_cast<int64_t>(B) * Hkv;
  const int chunks = select_chunks(heads, ld);
  if (heads * (chunks > 0 ? chunks : 1) > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  SelectArgs a = {kv_len, weights, ld, k, kept_weights, Hkv, budget, sinks, recent, 0, chunks, {}, nullptr, nullptr};
  const dim3 grid(static_cast<uint32_t>(heads * (chunks > 0 ? chunks : 1)));
  if (!chunks) {
    if (ld <= 4096) kv_select_kernel<4><<<grid, kSelectThreads, 0, stream>>>(a);
    else if (ld <= 8192) kv_select_kernel<8><<<grid, kSelectThreads, 0, stream>>>(a);
    else kv_select_kernel<16><<<grid, kSelectThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  a.per = cdiv(cdiv(ld, chunks), kSelectThreads) * kSelectThreads;
  WsCursor cur(ws);
  carve_select(cur, heads, chunks, a);
  kv_select_chunk_kernel<0><<<grid, kSelectThreads, 0, stream>>>(a);
  kv_select_chunk_kernel<1><<<grid, kSelectThreads, 0, stream>>>(a);
  kv_select_chunk_kernel<2><<<grid, kSelectThreads, 0, stream>>>(a);
  kv_select_chunk_kernel<3><<<grid, kSelectThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_gather(const KvCache& c, int B, const int32_t* table, int64_t ld_table, const int32_t* kv_len, const KvKeep& k,
                            int max_keep, const int32_t* to, int64_t ld_to, hipStream_t stream) {
  const int64_t pages = cdiv(max_keep, int64_t{1} << c.page_log2), heads = pages * B * c.Hkv;
  // fewer pages than CUs are divided over three workgroups each (40 pages 10 us for 14)
  const int slices = heads < 256 ? 2 : 0;
  const int64_t blocks = heads * (slices + 1);
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const GatherArgs a = {c, table, to, kv_len, ld_table, ld_to, k, B, static_cast<int>(pages), slices};
  kv_gather_kernel<<<dim3(static_cast<uint32_t>(blocks)), 256, c.page_log2 >= 6 ? kGatherLds : 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace crvq
