// Shared by the kernels of the 8-bit key / value cache (k_kv.hip, k_attn.hip): the cache and batch
// descriptions and the device-side checks of the indices they hold.
#pragma once

#include "crvq.h"
#include "crvq_internal.h"

namespace crvq {

// One sequence's new rows and length, as far as the device arrays describe them.
struct KvSeq {
  int row0;  // first row
  int n;     // rows
  int len;   // tokens in the cache, the new ones included
  bool in_rows;  // its rows lie within [0, n_tokens]
  bool ok;       // and there are at most max_new, and its length fits its block table
};

__device__ __forceinline__ KvSeq kv_seq(const KvBatch& bt, int b, int page_log2) {
  KvSeq s;
  const int r0 = bt.start[b], r1 = bt.start[b + 1];
  s.row0 = r0;
  s.len = bt.kv_len[b];
  s.in_rows = r0 >= 0 && r1 >= r0 && r1 <= bt.n_tokens;
  s.n = s.in_rows ? r1 - r0 : 0;
  s.ok = s.in_rows && s.n <= bt.max_new && s.len >= 0 && s.len <= CRVQ_KV_MAX_LEN && s.len <= (bt.ld_table << page_log2);
  return s;
}

__device__ __forceinline__ float bf16_f(uint32_t bits16) { return __uint_as_float(bits16 << 16); }

// fp32 to bf16, round to nearest even (a NaN stays one): two at a time, and one.
typedef float kv_f2 __attribute__((ext_vector_type(2)));
typedef __bf16 kv_b2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t f_bf16x2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((kv_f2{a, b}), kv_b2));
}
__device__ __forceinline__ uint32_t f_bf16(float f) { return f_bf16x2(f, 0.f) & 0xffffu; }

}  // namespace crvq
