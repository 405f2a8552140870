// Drafted tokens over the paged 8-bit cache, and the cache within a budget: the masks of a tree of drafts, the attention weight
// that every cached token received, the tokens that a budget keeps by it, and their move to other pages.
#include "kv_common.h"

namespace crvq {
namespace {

typedef int ev_i4 __attribute__((ext_vector_type(4)));
typedef float ev_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t ev_u4 __attribute__((ext_vector_type(4)));
typedef __bf16 ev_b8 __attribute__((ext_vector_type(8)));

constexpr float kInf = __builtin_inff();
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

// Eight codes as bf16: integers of eight bits are the upper halves of their fp32.
__device__ __forceinline__ ev_b8 widen8(int a, int b) {
  ev_u4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? a : b;
    const float x = static_cast<float>(static_cast<int8_t>(w >> (16 * (i & 1))));
    const float y = static_cast<float>(static_cast<int8_t>(w >> (16 * (i & 1) + 8)));
    v[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
  }
  return __builtin_bit_cast(ev_b8, v);
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

// 16 columns: their queries as right operands, what they see, and their log-sum-exps in powers of two.  DC chunks of 64 elements hold a head; a lane's 16
// elements of a chunk lie as the 16 code bytes it has of a token, the first eight in one instruction, the others in the next.
template <typename T, int DC>
struct Queries {
  static constexpr int NT = sizeof(T) == 4 ? 3 : 1;
  ev_b8 q[DC][2][NT];
  float lse2;
  int lo, hi;
  const uint64_t* bits;

  __device__ __forceinline__ void load(const WeightArgs& a, const KvSeq& sq, int hk, int col, int cols) {
    const int c = (threadIdx.x >> 4) & 3, i = col / a.G, h = hk * a.G + col - i * a.G;
    const int64_t row = sq.row0 + i;
    float lse = -kInf;
    if (col < cols) lse = a.w.lse[row * a.Hq + h];
    const bool ok = fabsf(lse) < kInf;  // neither a row that sees nothing nor one that is NaN has weights
    lse2 = lse * kLog2e;
    lo = hi = 0;
    bits = nullptr;
    const T* p = static_cast<const T*>(a.q.p) + row * a.q.tok + h * a.q.head + c * 16;
#pragma unroll
    for (int ch = 0; ch < DC; ++ch) {
      const bool there = ok && ch * 64 + c * 16 < a.c.D;
      if constexpr (sizeof(T) == 2) {
        ev_u4 x[2] = {};
        if (there) {
          if (a.q_vec) {
            x[0] = *reinterpret_cast<const ev_u4*>(p + ch * 64);
            x[1] = *reinterpret_cast<const ev_u4*>(p + ch * 64 + 8);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e >> 3][(e >> 1) & 3] |= static_cast<uint32_t>(p[ch * 64 + e]) << (16 * (e & 1));
          }
        }
        q[ch][0][0] = __builtin_bit_cast(ev_b8, x[0]);
        q[ch][1][0] = __builtin_bit_cast(ev_b8, x[1]);
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float x[8] = {};
          if (there) {
            const float* f = reinterpret_cast<const float*>(p) + ch * 64 + half * 8;
            if (a.q_vec) {
              const float4 u = *reinterpret_cast<const float4*>(f), v = *reinterpret_cast<const float4*>(f + 4);
              x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = f[e];
            }
          }
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
    if (!ok) return;
    const int context = sq.len - sq.n;
    hi = sq.len;
    if (a.w.tree.mask) {
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

  // whether this lane's column sees token t; context: tokens before the new ones
  __device__ __forceinline__ bool sees(int t, int context) const {
    if (t < lo || t >= hi) return false;
    const int j = t - context;
    return !bits || j < 0 || (bits[j >> 6] >> (j & 63) & 1);
  }
};

// 64 tokens of a wave: their codes as left operands, their scales, and the sums so far.
template <int DC>
struct Tokens {
  ev_b8 k[4][DC][2];
  float ks[4];
  bool good[4];
  ev_f4 sum[4];

  __device__ __forceinline__ void load(const WeightArgs& a, const KvSeq& sq, int b, int hk, int t0) {
    const int r = threadIdx.x & 15, c = (threadIdx.x >> 4) & 3, D = a.c.D, pl2 = a.c.page_log2;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int t = t0 + 16 * u;  // the tile's tokens lie in one page
      const int page = t < sq.len ? a.bt.table[b * a.bt.ld_table + (t >> pl2)] : -1;
      good[u] = static_cast<uint32_t>(page) < static_cast<uint32_t>(a.c.n_pages);
      const int64_t head = static_cast<int64_t>(good[u] ? page : 0) * a.c.Hkv + hk;
      ks[u] = good[u] ? a.c.k_scale[head] : 0.f;
      good[u] = good[u] && ks[u] >= 0.f && ks[u] < kInf;
      const int8_t* p = a.c.k + ((head << pl2) + ((t & ((1 << pl2) - 1)) + r)) * D + c * 16;
      sum[u] = ev_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ch = 0; ch < DC; ++ch) {
        ev_i4 x = {0, 0, 0, 0};
        if (good[u] && ch * 64 + c * 16 < D) x = *reinterpret_cast<const ev_i4*>(p + ch * 64);
        k[u][ch][0] = widen8(x[0], x[1]);
        k[u][ch][1] = widen8(x[2], x[3]);
      }
      ks[u] = good[u] ? ks[u] * (a.w.scale * kLog2e) : 0.f;
    }
  }

  // Adds the weights of 16 columns; whole: every column sees every token.
  template <typename T>
  __device__ __forceinline__ void add(const Queries<T, DC>& q, int t0, int context, bool whole) {
    const int c = (threadIdx.x >> 4) & 3;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      ev_f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = Queries<T, DC>::NT - 1; t >= 0; --t)
#pragma unroll
        for (int ch = 0; ch < DC; ++ch) {
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[u][ch][0], q.q[ch][0][t], s, 0, 0, 0);
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[u][ch][1], q.q[ch][1][t], s, 0, 0, 0);
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[i], ks[u], -q.lse2));
        sum[u][i] += (whole || (good[u] && q.sees(t0 + 16 * u + 4 * c + i, context))) ? p : 0.f;
      }
    }
  }
};

template <typename T, int DC>
__global__ __launch_bounds__(256) void kv_weights_kernel(const WeightArgs a) {
  const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4, wave = threadIdx.x >> 6;
  uint32_t item = blockIdx.x;
  const int hk = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  const int share = static_cast<int>(item % a.shares);
  item /= a.shares;
  const int tile = static_cast<int>(item % a.tiles), b = static_cast<int>(item / a.tiles);
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  const int t0 = (tile * 4 + wave) * 64;
  if (!sq.ok || sq.n == 0 || sq.len > a.max_kv || t0 >= sq.len) return;
  const int cols = sq.n * a.G, context = sq.len - sq.n;
  int first = 0, last = cols;  // the columns that see any of the tokens
  if (a.w.causal) {
    if (t0 > context) first = (t0 - context) * a.G;
    if (a.w.window) last = static_cast<int>(min<int64_t>(last, (static_cast<int64_t>(t0) + 63 + a.w.window - context) * a.G));
  }
  first &= ~15;
  if (a.shares > 1) {  // an equal share of the column blocks
    const int blocks = (max(last - first, 0) + 15) >> 4, each = (blocks + a.shares - 1) / a.shares;
    first += share * each * 16;
    last = min(last, first + each * 16);
  }
  Tokens<DC> k;
  k.load(a, sq, b, hk, t0);
  ev_f4 total[4] = {};
  int n = 0;
  for (int col = first; col < last; col += 16) {
    Queries<T, DC> q;
    q.load(a, sq, hk, col + r, cols);
    const bool sees_all = q.lo <= t0 && q.hi >= t0 + 64 && (!q.bits || t0 + 64 <= context);
    const bool whole = __all(sees_all && k.good[0] && k.good[1] && k.good[2] && k.good[3]);
    k.add(q, t0, context, whole);
    if (++n == 32) {  // sums of sums: the error of long ones grows with their root
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        total[u] += k.sum[u];
        k.sum[u] = ev_f4{0.f, 0.f, 0.f, 0.f};
      }
      n = 0;
    }
  }
  // lane (r, c) takes the token of tile r / 4 that is element r % 4 of its quarter
  float mine = 0.f;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = row_sum(total[u][i] + k.sum[u][i]);
      mine = r == 4 * u + i ? x : mine;
    }
  const int t = t0 + 16 * (r >> 2) + 4 * c + (r & 3);
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

int weight_shares(int B, int Hq, int Hkv, int max_new, int max_kv) {
  const int64_t groups = static_cast<int64_t>(B) * Hkv * cdiv(max_kv, 256), blocks = cdiv(static_cast<int64_t>(max_new) * (Hq / Hkv), 16);
  const int64_t want = cdiv(2048, groups > 0 ? groups : 1), most = cdiv(blocks, 32);
  const int64_t n = want < most ? want : most;
  return static_cast<int>(n < 1 ? 1 : n > 16 ? 16 : n);
}

// ---- the tokens that a budget keeps ---------------------------------------------------------------------
//
// One workgroup has a head's weights: four passes of a radix select find the smallest key that is kept and how many equal to
// it are, a last one writes the kept tokens in order.

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
};

__global__ __launch_bounds__(1024) void kv_select_kernel(const SelectArgs a) {
  __shared__ uint32_t hist[256], pick[2];
  __shared__ uint32_t scan[2][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
  const int64_t row = static_cast<int64_t>(b) * a.Hkv + hk;
  const int given = a.kv_len[b], len = given < 0 || given > a.ld ? 0 : given, n = min(len, a.budget);
  if (hk == 0 && tid == 0) a.k.len[b] = n;
  const float* w = a.weights + row * a.ld;
  auto key = [&](int t) { return t < a.sinks || t >= len - a.recent ? 0xffffffffu : key_of(w[t]); };
  // the n-th largest key, and how many of those equal to it are kept
  uint32_t least = 0, equal = 0;
  if (n < len) {
    uint32_t left = n;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int t = tid; t < len; t += 1024) {
        const uint32_t x = key(t);
        if (shift == 24 || (x >> (shift + 8)) == (least >> (shift + 8))) atomicAdd(&hist[(x >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        int d = 255;
        while (d > 0 && hist[d] < left) left -= hist[d--];
        pick[0] = static_cast<uint32_t>(d) << shift;
        pick[1] = left;
      }
      __syncthreads();
      least |= pick[0];
      left = pick[1];
    }
    equal = left;
  }
  // in order: those above it, and the first `equal` ones equal to it
  uint32_t above = 0, same = 0;  // of the tokens before this round
  for (int t0 = 0; t0 < len; t0 += 1024) {
    const int t = t0 + tid;
    const uint32_t x = t < len ? key(t) : 0;
    const bool gt = t < len && (n == len || x > least), eq = n < len && t < len && x == least;
    const unsigned long long bg = __ballot(gt), be = __ballot(eq), before = (1ull << lane) - 1;
    __syncthreads();
    if (lane == 0) {
      scan[0][wave] = __popcll(bg);
      scan[1][wave] = __popcll(be);
    }
    __syncthreads();
    uint32_t g = above + __popcll(bg & before), e = same + __popcll(be & before);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const uint32_t p = scan[0][v], q = scan[1][v];
      if (v < wave) g += p, e += q;
      above += p, same += q;
    }
    if (gt || (eq && e < equal)) {
      const int64_t at = row * a.k.ld + g + min(e, equal);
      a.k.keep[at] = t;
      if (a.kept) a.kept[at] = w[t];
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
};

// A new page's scale is the largest of its tokens' old ones; a code becomes rint(c (old / new)).
__global__ __launch_bounds__(256) void kv_gather_kernel(const GatherArgs a) {
  __shared__ int64_t from[256];     // the token's head and slot: (page * Hkv + hk) * page size + slot
  __shared__ float by[2][256];      // old scale over new
  __shared__ float red[2][4];
  const int tid = threadIdx.x, D = a.c.D, pl2 = a.c.page_log2, P = 1 << pl2;
  uint32_t item = blockIdx.x;
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
    if (!(ks >= 0.f && ks < kInf)) ks = nan;
    if (!(vs >= 0.f && vs < kInf)) vs = nan;
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
  __syncthreads();
  const int64_t head = static_cast<int64_t>(dest) * a.c.Hkv + hk;
  if (tid == 0) {
    a.c.k_scale[head] = k_new;
    a.c.v_scale[head] = v_new;
  }
  auto moved = [](int8_t c, float f) { return static_cast<int8_t>(rintf(static_cast<float>(c) * f)); };
  const int d16 = D >> 4;
  int8_t* k_to = a.c.k + (head << pl2) * D;
  for (int x = tid; x < P * d16; x += 256) {
    const int j = x / d16, e = (x - j * d16) * 16;
    ev_i4 y = {0, 0, 0, 0};
    if (j < n && k_ok) {
      y = *reinterpret_cast<const ev_i4*>(a.c.k + from[j] * D + e);
      const float f = by[0][j];
      if (f != 1.f) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int v = moved(static_cast<int8_t>(y[i >> 2] >> (8 * (i & 3))), f);
          y[i >> 2] = (y[i >> 2] & ~(255 << (8 * (i & 3)))) | ((v & 255) << (8 * (i & 3)));
        }
      }
    }
    *reinterpret_cast<ev_i4*>(k_to + j * D + e) = y;
  }
  int8_t* v_to = a.c.v + (head << pl2) * D;
  for (int x = tid; x < P * D; x += 256) {
    const int e = x >> pl2, j = x & (P - 1);
    int8_t y = 0;
    if (j < n && v_ok) {
      const int64_t head_from = from[j] >> pl2;
      y = moved(a.c.v[((head_from * D + e) << pl2) + (from[j] & (P - 1))], by[1][j]);
    }
    v_to[x] = y;
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
  const int shares = weight_shares(B, Hq, Hkv, max_new, max_kv);
  WsCursor c(nullptr);
  if (shares > 1) c.take<float>(static_cast<size_t>(shares) * B * Hkv * max_kv);
  return c.used;
}

hipError_t launch_kv_weights(const KvCache& c, const KvBatch& bt, int max_kv, int type, int Hq, const KvRows& q,
                             const KvWeights& w, void* ws, hipStream_t stream) {
  const int shares = weight_shares(bt.B, Hq, c.Hkv, bt.max_new, max_kv), es = type == ET_F32 ? 4 : 2;
  WsCursor cur(ws);
  float* part = shares > 1 ? cur.take<float>(static_cast<size_t>(shares) * bt.B * c.Hkv * max_kv) : nullptr;
  const int tiles = static_cast<int>(cdiv(max_kv, 256));
  WeightArgs a = {c, bt, q, w, part, Hq, Hq / c.Hkv, shares, tiles, max_kv, 0};
  a.q_vec = reinterpret_cast<uintptr_t>(q.p) % 16 == 0 && q.tok * es % 16 == 0 && q.head * es % 16 == 0;
  const int64_t blocks = static_cast<int64_t>(bt.B) * c.Hkv * tiles * shares;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffffLL || static_cast<int64_t>(bt.B) * c.Hkv > 65535) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(blocks));
  auto as = [&](auto t) {
    using T = decltype(t);
    if (c.D <= 64) kv_weights_kernel<T, 1><<<grid, 256, 0, stream>>>(a);
    else if (c.D <= 128) kv_weights_kernel<T, 2><<<grid, 256, 0, stream>>>(a);
    else kv_weights_kernel<T, 4><<<grid, 256, 0, stream>>>(a);
  };
  if (type == ET_F32) as(uint32_t{});
  else as(uint16_t{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || shares == 1) return e;
  kv_weights_join_kernel<<<dim3(static_cast<uint32_t>(cdiv(max_kv, 256)), static_cast<uint32_t>(bt.B * c.Hkv)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_select(int B, int Hkv, const int32_t* kv_len, const float* weights, int64_t ld, int budget, int sinks,
                            int recent, const KvKeep& k, float* kept_weights, hipStream_t stream) {
  const int64_t blocks = static_cast<int64_t>(B) * Hkv;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const SelectArgs a = {kv_len, weights, ld, k, kept_weights, Hkv, budget, sinks, recent};
  kv_select_kernel<<<dim3(static_cast<uint32_t>(blocks)), 1024, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_gather(const KvCache& c, int B, const int32_t* table, int64_t ld_table, const int32_t* kv_len, const KvKeep& k,
                            int max_keep, const int32_t* to, int64_t ld_to, hipStream_t stream) {
  const int64_t pages = cdiv(max_keep, int64_t{1} << c.page_log2), blocks = pages * B * c.Hkv;
  if (blocks == 0) return hipSuccess;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const GatherArgs a = {c, table, to, kv_len, ld_table, ld_to, k, B, static_cast<int>(pages)};
  kv_gather_kernel<<<dim3(static_cast<uint32_t>(blocks)), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace crvq
