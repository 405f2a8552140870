// The paged 8-bit cache of keys and values: appending (rotation, quantization, storage) and reading back.
//
// Append: one workgroup owns one head of one page of keys or of values and the new tokens that fall into
// it, so the page's scale has one writer.  It takes the largest magnitude of its rotated elements, settles
// the scale, brings older codes to it if it grew, and stores the new codes; the elements stay in registers meanwhile
// (those of long pages past the first kKept chunks of a thread are read again).  Values are stored transposed: the
// new tokens go through an LDS tile and leave as 16-byte runs of slots, a few of them as bytes.  The same launch
// rotates the queries, a workgroup a row.  Memory bounds prompts (three of up to 2048 tokens, 64 query and 8 key heads:
// 47 us for 196 MB, 4.2 TB/s).  A decoding step, 9.8 us for the 1.2 MB of 32 sequences of 32 heads, is latency: a workgroup
// looks up lengths, page and scale before it reads one token's 128 elements, for which 16 of its 256 threads have work.  So is
// reading back, 25 MB in 10.6 us (2.3 TB/s): look-ups, one read and one store a thread.
#include "kv_common.h"

namespace crvq {
namespace {

constexpr float kMinScale = 7.888609052210118e-31f;  // 2^-100
constexpr int kSeg = 64;                             // slots of the LDS tile of a page of values
constexpr int kTileLd = kSeg + 4;

template <typename T>
__device__ __forceinline__ float ld1(const T* p) {
  if constexpr (sizeof(T) == 4)
    return *reinterpret_cast<const float*>(p);
  else
    return bf16_f(*p);
}

// Eight consecutive elements; VEC: 16-byte aligned.
template <typename T, bool VEC>
__device__ __forceinline__ void ld8(const T* p, float (&x)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = ld1(p + i);
  } else if constexpr (sizeof(T) == 4) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
}

template <typename T>
__device__ __forceinline__ void st1(T* p, float x) {
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<float*>(p) = x;
  else
    *p = static_cast<T>(f_bf16(x));
}

template <typename T, bool VEC>
__device__ __forceinline__ void st8(T* p, const float (&x)[8]) {
  if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i) st1(p + i, x[i]);
  } else if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint4 a;
    a.x = f_bf16x2(x[0], x[1]);
    a.y = f_bf16x2(x[2], x[3]);
    a.z = f_bf16x2(x[4], x[5]);
    a.w = f_bf16x2(x[6], x[7]);
    *reinterpret_cast<uint4*>(p) = a;
  }
}

// The angles of one row; ok = 0: its place lies outside the table.
struct Angles {
  const float *c, *s;
  int ok;
};
__device__ __forceinline__ Angles angles(const KvRotation& rt, int row, int place) {
  const int64_t p = rt.positions ? rt.positions[row] : place;
  Angles a;
  a.ok = p >= 0 && p < rt.n_angles;
  const int64_t at = a.ok ? p * (rt.rot >> 1) : 0;
  a.c = rt.cos + at;
  a.s = rt.sin + at;
  return a;
}

// The angles of pairs j .. j + 7 (j a multiple of 8).  A table may have no rows at all: outside it nothing is read.
__device__ __forceinline__ void angles8(const KvRotation& rt, const Angles& an, int j, float (&c)[8], float (&s)[8]) {
  if (!an.ok) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = __uint_as_float(0x7fc00000u), s[i] = 0.f;
  } else if (rt.vec) {
    const float4 c0 = reinterpret_cast<const float4*>(an.c + j)[0], c1 = reinterpret_cast<const float4*>(an.c + j)[1];
    const float4 s0 = reinterpret_cast<const float4*>(an.s + j)[0], s1 = reinterpret_cast<const float4*>(an.s + j)[1];
    c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
    s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = an.c[j + i], s[i] = an.s[j + i];
  }
}

// Pair j of a row, (a, b) -> (a c - b s, b c + a s).
__device__ __forceinline__ void turn(const Angles& an, int j, float& a, float& b) {
  const float c = an.ok ? an.c[j] : __uint_as_float(0x7fc00000u), s = an.ok ? an.s[j] : 0.f;
  const float u = a * c - b * s, w = b * c + a * s;
  a = u;
  b = w;
}

// Elements e0 .. e0 + 7 of a head's row, rotated.
template <typename T, bool VEC>
__device__ __forceinline__ void rotated8(const T* row, int e0, const KvRotation& rt, const Angles& an, float (&x)[8]) {
  ld8<T, VEC>(row + e0, x);
  if (!rt.cos || e0 >= rt.rot) return;
  const int r = rt.rot >> 1;
  if (rt.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      if (e0 + i < rt.rot) turn(an, (e0 + i) >> 1, x[i], x[i + 1]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = e0 + i;
    if (e < r) {
      float y = ld1(row + e + r);
      turn(an, e, x[i], y);
    } else if (e < rt.rot) {
      float y = ld1(row + e - r);
      turn(an, e - r, y, x[i]);
    }
  }
}

// How a head's row is cut into units, each read by one thread before it writes (so q_out may be q): chunks of eight
// elements; the first chunks of a rotation by halves together with their partner chunks; or, where chunks are not
// aligned or the halves are not whole chunks, single pairs and elements.
enum Units : int { kChunks, kPairs, kSingle };
__host__ __device__ inline int units_of(int kind, int D, int r) {
  return kind == kSingle ? D - r : kind == kPairs ? (D - r) >> 3 : D >> 3;
}

__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o)));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
  __syncthreads();
  return max(max(lds[0], lds[1]), max(lds[2], lds[3]));
}

__device__ __forceinline__ uint32_t rescale4(uint32_t c, float f) {
  uint32_t o = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = rintf(static_cast<float>(static_cast<int8_t>(c >> (8 * i))) * f);
    o |= (static_cast<uint32_t>(static_cast<int>(x)) & 255u) << (8 * i);
  }
  return o;
}

__device__ __forceinline__ uint32_t quantize1(float x, float scale) {
  const float q = fminf(fmaxf(rintf(x / scale), -127.f), 127.f);
  return static_cast<uint32_t>(static_cast<int>(q)) & 255u;
}

constexpr int kThreads = 256;
constexpr int kKept = 4;   // chunks of new elements a thread keeps between the two uses: pages of 64 x 128 in registers
constexpr int kFew = 16;   // new tokens below which values are stored as bytes

struct AppendArgs {
  KvCache c;
  KvBatch bt;
  KvRows k, v, q, q_out;
  KvRotation rt;
  int Hq;
  int64_t kv_blocks;  // B * pages * Hkv * 2 workgroups of pages; one a row of queries follows
  int pages;          // pages a sequence's new tokens may touch
  int units, key_units;  // of the queries, of the keys
};

// One row of queries: a thread's unit is the same for all of its heads where it can be, and so are its angles.
template <typename T, bool VEC>
__device__ __forceinline__ void rotate_queries(const AppendArgs& a, int row) {
  const int D = a.c.D, r = a.rt.cos ? a.rt.rot >> 1 : 0;
  Angles an = {nullptr, nullptr, 0};
  if (r) {
    int place = 0;
    if (!a.rt.positions) {  // the sequence of this row
      int lo = 0, hi = a.bt.B;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.bt.start[mid + 1] > row) hi = mid; else lo = mid + 1;
      }
      if (lo >= a.bt.B) return;
      const KvSeq s = kv_seq(a.bt, lo, a.c.page_log2);
      if (!s.ok || s.n > s.len || row < s.row0) return;
      place = s.len - s.n + row - s.row0;
    }
    an = angles(a.rt, row, place);
  }
  const int per = units_of(a.units, D, r);
  const T* in0 = static_cast<const T*>(a.q.p) + row * a.q.tok;
  T* out0 = static_cast<T*>(a.q_out.p) + row * a.q_out.tok;
  if (a.units == kPairs && kThreads % per == 0 && (kThreads / per) * 4 >= a.Hq) {  // angles once, up to four heads
    const int unit = threadIdx.x % per, e0 = unit * 8 + (unit * 8 >= r ? r : 0);
    const bool pair = e0 < r;
    float cs[8], sn[8];
    if (pair) angles8(a.rt, an, e0, cs, sn);
    for (int h = threadIdx.x / per; h < a.Hq; h += kThreads / per) {
      const T* in = in0 + h * a.q.head;
      T* out = out0 + h * a.q_out.head;
      float x[8], y[8];
      ld8<T, VEC>(in + e0, x);
      if (pair) {
        ld8<T, VEC>(in + e0 + r, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float u = x[i] * cs[i] - y[i] * sn[i], w = y[i] * cs[i] + x[i] * sn[i];
          x[i] = u;
          y[i] = w;
        }
        st8<T, VEC>(out + e0 + r, y);
      }
      st8<T, VEC>(out + e0, x);
    }
    return;
  }
  for (int u = threadIdx.x; u < a.Hq * per; u += kThreads) {
    const int h = u / per, unit = u - h * per;
    const T* in = in0 + h * a.q.head;
    T* out = out0 + h * a.q_out.head;
    if (a.units == kSingle) {
      if (unit < r) {
        const int e = a.rt.interleaved ? 2 * unit : unit, f = a.rt.interleaved ? e + 1 : e + r;
        float x = ld1(in + e), y = ld1(in + f);
        turn(an, unit, x, y);
        st1(out + e, x);
        st1(out + f, y);
      } else {
        out[unit + r] = in[unit + r];
      }
      continue;
    }
    const int e0 = unit * 8 + (a.units == kPairs && unit * 8 >= r ? r : 0);
    float x[8], y[8];
    if (a.units == kPairs && e0 < r) {
      ld8<T, VEC>(in + e0, x);
      ld8<T, VEC>(in + e0 + r, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) turn(an, e0 + i, x[i], y[i]);
      st8<T, VEC>(out + e0, x);
      st8<T, VEC>(out + e0 + r, y);
    } else {
      rotated8<T, VEC>(in, e0, a.rt, an, x);
      st8<T, VEC>(out + e0, x);
    }
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const AppendArgs a) {
  __shared__ uint32_t red[4];
  extern __shared__ __align__(16) uint8_t tile[];  // [D][page + 4]
  if (blockIdx.x >= a.kv_blocks) {
    rotate_queries<T, VEC>(a, static_cast<int>(blockIdx.x - a.kv_blocks));
    return;
  }
  const int tid = threadIdx.x, D = a.c.D, P = 1 << a.c.page_log2;
  uint32_t item = blockIdx.x;
  const bool values = item & 1;
  item >>= 1;
  const int h = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  const int j = static_cast<int>(item % a.pages), b = static_cast<int>(item / a.pages);
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  if (!sq.ok || sq.n == 0 || sq.n > sq.len) return;
  const int first = sq.len - sq.n, p = (first >> a.c.page_log2) + j;
  if ((static_cast<int64_t>(p) << a.c.page_log2) >= sq.len) return;
  const int64_t page = a.bt.table[b * a.bt.ld_table + p];
  if (page < 0 || page >= a.c.n_pages) return;
  const int t0 = p << a.c.page_log2;
  const int lo = max(first, t0) - t0, hi = min(sq.len - t0, P);  // its new slots; older ones before lo
  const KvRows src = values ? a.v : a.k;
  const T* base = static_cast<const T*>(src.p) + h * src.head;
  const int cpr = D >> 3, chunks = (hi - lo) * cpr;
  const int row_lo = sq.row0 + t0 + lo - first;
  float* sp = (values ? a.c.v_scale : a.c.k_scale) + page * a.c.Hkv + h;
  const float old = *sp;

  auto load = [&](int c, int& slot, int& e0, float (&x)[8]) {
    const int i = c / cpr;
    e0 = (c - i * cpr) * 8;
    slot = lo + i;
    const int row = row_lo + i;
    const T* r = base + row * src.tok;
    if (values)
      ld8<T, VEC>(r + e0, x);
    else
      rotated8<T, VEC>(r, e0, a.rt, a.rt.cos ? angles(a.rt, row, t0 + slot) : Angles{nullptr, nullptr, 0}, x);
  };
  // a unit of keys rotated by halves: two chunks, or one that is not rotated (e1 < 0)
  const bool pairs = !values && a.key_units == kPairs;
  const int r = pairs ? a.rt.rot >> 1 : 0, upt = units_of(kPairs, D, r), units = (hi - lo) * upt;
  auto load_pair = [&](int u, int& slot, int& e0, int& e1, float (&x)[8], float (&y)[8]) {
    const int i = u / upt, unit = u - i * upt;
    e0 = unit * 8 + (unit * 8 >= r ? r : 0);
    e1 = e0 < r ? e0 + r : -1;
    slot = lo + i;
    const T* row = base + (row_lo + i) * src.tok;
    ld8<T, VEC>(row + e0, x);
    if (e1 < 0) return;
    ld8<T, VEC>(row + e1, y);
    float cs[8], sn[8];
    angles8(a.rt, angles(a.rt, row_lo + i, t0 + slot), e0, cs, sn);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float u2 = x[k] * cs[k] - y[k] * sn[k], w2 = y[k] * cs[k] + x[k] * sn[k];
      x[k] = u2;
      y[k] = w2;
    }
  };
  auto largest = [](const float (&x)[8], uint32_t m) {  // magnitude as bits: a NaN is larger than every number
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
  };

  uint32_t m = 0;
  float kept[kKept][8];
  int slots[kKept], at[kKept];
#pragma unroll
  for (int i = 0; i < kKept; ++i) at[i] = -1;
  if (pairs) {
#pragma unroll
    for (int i = 0; i < kKept; i += 2)
      if (tid + (i >> 1) * kThreads < units) {
        load_pair(tid + (i >> 1) * kThreads, slots[i], at[i], at[i + 1], kept[i], kept[i + 1]);
        slots[i + 1] = slots[i];
        m = largest(kept[i], m);
        if (at[i + 1] >= 0) m = largest(kept[i + 1], m);
      }
    for (int u = tid + kKept / 2 * kThreads; u < units; u += kThreads) {
      int slot, e0, e1;
      float x[8], y[8];
      load_pair(u, slot, e0, e1, x, y);
      m = largest(x, m);
      if (e1 >= 0) m = largest(y, m);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kKept; ++i)
      if (tid + i * kThreads < chunks) {
        load(tid + i * kThreads, slots[i], at[i], kept[i]);
        m = largest(kept[i], m);
      }
    for (int c = tid + kKept * kThreads; c < chunks; c += kThreads) {
      int slot, e0;
      float x[8];
      load(c, slot, e0, x);
      m = largest(x, m);
    }
  }
  m = block_max(m, red);
  const int64_t head_at = (page * a.c.Hkv + h) * (static_cast<int64_t>(D) << a.c.page_log2);
  int8_t* codes = (values ? a.c.v : a.c.k) + head_at;
  const bool finite = m < 0x7f800000u;
  float scale = finite ? fmaxf(__uint_as_float(m) / 127.f, kMinScale) : __uint_as_float(0x7fc00000u);
  if (lo > 0) {
    if (finite && !(scale > old)) scale = old;
    if (scale > old) {  // the older codes move to the larger scale, 16 at a time
      const float f = old / scale;
      const int per = values ? (lo + 15) >> 4 : D >> 4, n = (values ? D : lo) * per;
#pragma unroll 4
      for (int u = tid; u < n; u += kThreads) {
        const int r = u / per;
        uint4* to = reinterpret_cast<uint4*>(codes + (values ? r << a.c.page_log2 : r * D)) + (u - r * per);
        uint4 w = *to;
        w.x = rescale4(w.x, f);
        w.y = rescale4(w.y, f);
        w.z = rescale4(w.z, f);
        w.w = rescale4(w.w, f);
        *to = w;
      }
      __syncthreads();  // before new codes go into the words rewritten here
    }
  }
  if (tid == 0) *sp = scale;  // every thread read the old one before block_max
  const bool number = scale == scale;
  const bool tiled = values && hi - lo >= kFew;
  const int tile_ld = P + 4;

  auto store = [&](int slot, int e0, const float (&x)[8]) {
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = number ? quantize1(x[i], scale) : 0u;
    if (!values) {
      uint2 w;
      w.x = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
      w.y = q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24;
      *reinterpret_cast<uint2*>(codes + slot * D + e0) = w;
    } else if (tiled) {
#pragma unroll
      for (int i = 0; i < 8; ++i) tile[(e0 + i) * tile_ld + slot] = static_cast<uint8_t>(q[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) codes[((e0 + i) << a.c.page_log2) + slot] = static_cast<int8_t>(q[i]);
    }
  };
#pragma unroll
  for (int i = 0; i < kKept; ++i)
    if (at[i] >= 0) store(slots[i], at[i], kept[i]);
  if (pairs) {
    for (int u = tid + kKept / 2 * kThreads; u < units; u += kThreads) {
      int slot, e0, e1;
      float x[8], y[8];
      load_pair(u, slot, e0, e1, x, y);
      store(slot, e0, x);
      if (e1 >= 0) store(slot, e1, y);
    }
  } else {
    for (int c = tid + kKept * kThreads; c < chunks; c += kThreads) {
      int slot, e0;
      float x[8];
      load(c, slot, e0, x);
      store(slot, e0, x);
    }
  }
  if (!tiled) return;
  __syncthreads();
  const int run0 = lo >> 4, runs = ((hi + 15) >> 4) - run0;  // of 16 slots
  for (int u = tid; u < D * runs; u += kThreads) {
    const int d = u / runs, g = (run0 + u - d * runs) * 16;
    const uint8_t* t = tile + d * tile_ld + g;
    int8_t* out = codes + (d << a.c.page_log2) + g;
    if (g >= lo && g + 16 <= hi) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(t);
      *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      for (int i = 0; i < 16; ++i)
        if (g + i >= lo && g + i < hi) out[i] = static_cast<int8_t>(t[i]);
    }
  }
}

struct ReadArgs {
  KvCache c;
  KvBatch bt;
  KvRows k, v;
  int segs, seg_log2;  // segments a sequence's tokens may touch; slots of one (min(page, kSeg))
};

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void kv_read_kernel(const ReadArgs a) {
  __shared__ __align__(16) uint8_t tile[CRVQ_KV_MAX_D * kTileLd];
  const int tid = threadIdx.x, D = a.c.D;
  int64_t item = blockIdx.x;
  const bool values = item & 1;
  item >>= 1;
  const int h = static_cast<int>(item % a.c.Hkv);
  item /= a.c.Hkv;
  const int j = static_cast<int>(item % a.segs), b = static_cast<int>(item / a.segs);
  const KvRows dst = values ? a.v : a.k;
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  if (!dst.p || !sq.ok || sq.n == 0 || sq.n > sq.len) return;
  const int first = sq.len - sq.n, S = 1 << a.seg_log2, t0 = ((first >> a.seg_log2) + j) << a.seg_log2;
  if (t0 >= sq.len) return;
  const int64_t page = a.bt.table[b * a.bt.ld_table + (t0 >> a.c.page_log2)];
  const bool there = page >= 0 && page < a.c.n_pages;
  const int slot0 = t0 & ((1 << a.c.page_log2) - 1);
  const int64_t head = (there ? page : 0) * a.c.Hkv + h;
  const int8_t* codes = (values ? a.c.v : a.c.k) + head * (static_cast<int64_t>(D) << a.c.page_log2);
  const float scale = there ? (values ? a.c.v_scale : a.c.k_scale)[head] : __uint_as_float(0x7fc00000u);
  const int lo = max(first - t0, 0), hi = min(sq.len - t0, S), cpr = D >> 3;
  if (values && there) {  // the segment of every d, 16 slots at a time
    const int runs = S >> 4;
    for (int u = tid; u < D * runs; u += 256) {
      const int d = u / runs, g = (u - d * runs) * 16;
      const uint4 w = *reinterpret_cast<const uint4*>(codes + (d << a.c.page_log2) + slot0 + g);
      uint32_t* t = reinterpret_cast<uint32_t*>(tile + d * kTileLd + g);
      t[0] = w.x; t[1] = w.y; t[2] = w.z; t[3] = w.w;
    }
    __syncthreads();
  }
  T* base = static_cast<T*>(dst.p) + h * dst.head;
  for (int c = tid; c < (hi - lo) * cpr; c += 256) {
    const int i = lo + c / cpr, e0 = (c % cpr) * 8;
    float x[8];
    if (!there) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = scale;
    } else if (values) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(static_cast<int8_t>(tile[(e0 + e) * kTileLd + i])) * scale;
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(codes + (slot0 + i) * D + e0);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[e] = static_cast<float>(static_cast<int8_t>((e < 4 ? w.x : w.y) >> (8 * (e & 3)))) * scale;
    }
    st8<T, VEC>(base + (sq.row0 + t0 + i - first) * dst.tok + e0, x);
  }
}

// Rows whose chunks of eight elements are 16-byte aligned.
bool aligned_rows(const KvRows& r, int type) {
  const int64_t per = type == ET_F32 ? 4 : 8;
  return !r.p || ((reinterpret_cast<uintptr_t>(r.p) & 15) == 0 && r.tok % per == 0 && r.head % per == 0);
}

}  // namespace

hipError_t launch_kv_append(const KvCache& c, const KvBatch& bt, int type, const KvRows& k, const KvRows& v, int Hq,
                            const KvRows& q, const KvRows& q_out, const KvRotation& rt, hipStream_t stream) {
  AppendArgs a = {c, bt, k, v, q, q_out, rt, Hq, 0, 0, 0, 0};
  const int P = 1 << c.page_log2;
  a.pages = static_cast<int>((static_cast<int64_t>(bt.max_new) + P - 2) / P + 1);
  a.kv_blocks = static_cast<int64_t>(bt.B) * a.pages * c.Hkv * 2;
  const bool vec = aligned_rows(k, type) && aligned_rows(v, type) && aligned_rows(q, type) && aligned_rows(q_out, type);
  const int r = rt.cos ? rt.rot >> 1 : 0;
  const bool halves = r && !rt.interleaved;
  a.units = !vec || (halves && (r & 7)) ? kSingle : halves ? kPairs : kChunks;
  a.key_units = a.units == kPairs ? kPairs : kChunks;
  a.rt.vec = (r & 3) == 0 && ((reinterpret_cast<uintptr_t>(rt.cos) | reinterpret_cast<uintptr_t>(rt.sin)) & 15) == 0;
  const int64_t blocks = a.kv_blocks + (q.p ? bt.n_tokens : 0);
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const dim3 grid(static_cast<uint32_t>(blocks));
  const size_t lds = bt.max_new < kFew ? 0 : static_cast<size_t>(c.D) * (P + 4);
  if (type == ET_F32) {
    if (vec) kv_append_kernel<uint32_t, true><<<grid, kThreads, lds, stream>>>(a);
    else kv_append_kernel<uint32_t, false><<<grid, kThreads, lds, stream>>>(a);
  } else {
    if (vec) kv_append_kernel<uint16_t, true><<<grid, kThreads, lds, stream>>>(a);
    else kv_append_kernel<uint16_t, false><<<grid, kThreads, lds, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvCache& c, const KvBatch& bt, int type, const KvRows& k_out, const KvRows& v_out,
                          hipStream_t stream) {
  ReadArgs a = {c, bt, k_out, v_out, 0, 0};
  a.seg_log2 = c.page_log2 < 6 ? c.page_log2 : 6;
  const int S = 1 << a.seg_log2;
  a.segs = static_cast<int>((static_cast<int64_t>(bt.max_new) + S - 2) / S + 1);
  const int64_t blocks = static_cast<int64_t>(bt.B) * a.segs * c.Hkv * 2;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  const bool vec = aligned_rows(k_out, type) && aligned_rows(v_out, type);
  const dim3 grid(static_cast<uint32_t>(blocks));
  if (type == ET_F32) {
    if (vec) kv_read_kernel<uint32_t, true><<<grid, 256, 0, stream>>>(a);
    else kv_read_kernel<uint32_t, false><<<grid, 256, 0, stream>>>(a);
  } else {
    if (vec) kv_read_kernel<uint16_t, true><<<grid, 256, 0, stream>>>(a);
    else kv_read_kernel<uint16_t, false><<<grid, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace crvq
