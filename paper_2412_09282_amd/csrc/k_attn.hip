// Attention of new tokens over the paged 8-bit cache.
//
// One wave owns one query row and walks the row's visible tokens 64 at a time: a lane takes the dot product of
// one token, the wave settles the running maximum and sum of the softmax, and the weights go through LDS to
// the lanes that own the elements of the output.
#include "kv_common.h"

namespace crvq {
namespace {

struct AttnArgs {
  KvCache c;
  KvBatch bt;
  KvRows q, out;
  float* lse;
  float scale;
  int Hq, causal, window;
};

template <typename T>
__global__ __launch_bounds__(64) void kv_attention_rows_kernel(const AttnArgs a) {
  __shared__ float qs[CRVQ_KV_MAX_D], ps[64];
  const int lane = threadIdx.x, D = a.c.D, P = 1 << a.c.page_log2;
  int64_t item = blockIdx.x;
  const int h = static_cast<int>(item % a.Hq);
  item /= a.Hq;
  const int i = static_cast<int>(item % a.bt.max_new), b = static_cast<int>(item / a.bt.max_new);
  const KvSeq sq = kv_seq(a.bt, b, a.c.page_log2);
  if (i >= sq.n) return;
  const int hk = h / (a.Hq / a.c.Hkv), row = sq.row0 + i;
  const T* q = static_cast<const T*>(a.q.p) + row * a.q.tok + h * a.q.head;
  bool bad = !sq.ok;
  for (int e = lane; e < D; e += 64) {
    const float x = sizeof(T) == 4 ? reinterpret_cast<const float*>(q)[e] : bf16_f(q[e]);
    if (!(fabsf(x) < __uint_as_float(0x7f800000u))) bad = true;
    qs[e] = x;
  }
  bad = __any(bad);
  __syncthreads();
  int from = 0, to = bad ? 0 : sq.len;
  if (a.causal) {
    const int place = sq.len - sq.n + i;
    to = min(to, place + 1);
    if (a.window) from = max(0, place + 1 - a.window);
  }
  float m = -__uint_as_float(0x7f800000u), l = 0.f, o[CRVQ_KV_MAX_D / 64] = {0.f, 0.f, 0.f, 0.f};
  for (int t0 = from & ~63; t0 < to; t0 += 64) {
    const int t = t0 + lane;
    float s = -__uint_as_float(0x7f800000u), vs = 0.f;
    if (t >= from && t < to) {
      const int64_t page = a.bt.table[b * a.bt.ld_table + (t >> a.c.page_log2)];
      if (page < 0 || page >= a.c.n_pages) {
        bad = true;
      } else {
        const int64_t head = page * a.c.Hkv + hk;
        const int8_t* k = a.c.k + ((head << a.c.page_log2) + (t & (P - 1))) * D;
        float dot = 0.f;
        for (int e = 0; e < D; ++e) dot += qs[e] * static_cast<float>(k[e]);
        const float ks = a.c.k_scale[head];
        vs = a.c.v_scale[head];
        if (!(fabsf(ks) < __uint_as_float(0x7f800000u)) || !(fabsf(vs) < __uint_as_float(0x7f800000u))) bad = true;
        s = dot * ks * a.scale;
      }
    }
    bad = __any(bad);
    if (bad) break;
    float top = s;
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float nm = fmaxf(m, top), keep = expf(m - nm);
    const float p = expf(s - nm);
    float sum = p;
    for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
    l = l * keep + sum;
    m = nm;
    __syncthreads();
    ps[lane] = p * vs;
    __syncthreads();
#pragma unroll
    for (int g = 0; g < CRVQ_KV_MAX_D / 64; ++g) {
      const int d = g * 64 + lane;
      if (d >= D) break;
      float acc = o[g] * keep;
      for (int u = 0; u < 64; ++u) {
        const int tt = t0 + u;
        if (tt < from || tt >= to) continue;
        const int64_t head = static_cast<int64_t>(a.bt.table[b * a.bt.ld_table + (tt >> a.c.page_log2)]) * a.c.Hkv + hk;
        acc += ps[u] * static_cast<float>(a.c.v[((head * D + d) << a.c.page_log2) + (tt & (P - 1))]);
      }
      o[g] = acc;
    }
  }
  const float nan = __uint_as_float(0x7fc00000u);
  T* out = static_cast<T*>(a.out.p) + row * a.out.tok + h * a.out.head;
  for (int g = 0; g < CRVQ_KV_MAX_D / 64; ++g) {
    const int d = g * 64 + lane;
    if (d >= D) break;
    const float x = bad ? nan : (l > 0.f ? o[g] / l : 0.f);
    if (sizeof(T) == 4)
      reinterpret_cast<float*>(out)[d] = x;
    else
      out[d] = static_cast<T>(f_bf16(x));
  }
  if (a.lse && lane == 0)
    a.lse[static_cast<int64_t>(row) * a.Hq + h] = bad ? nan : (l > 0.f ? m + logf(l) : -__uint_as_float(0x7f800000u));
}

}  // namespace

size_t kv_attention_ws_bytes(int, int, int, int, int, int) { return 0; }

hipError_t launch_kv_attention(const KvCache& c, const KvBatch& bt, int, int type, int Hq, const KvRows& q,
                               const KvRows& out, float scale, int causal, int window, float* lse, void*,
                               hipStream_t stream) {
  const AttnArgs a = {c, bt, q, out, lse, scale, Hq, causal, window};
  const int64_t blocks = static_cast<int64_t>(bt.B) * bt.max_new * Hq;
  if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  if (type == ET_F32)
    kv_attention_rows_kernel<uint32_t><<<dim3(static_cast<uint32_t>(blocks)), 64, 0, stream>>>(a);
  else
    kv_attention_rows_kernel<uint16_t><<<dim3(static_cast<uint32_t>(blocks)), 64, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace crvq
