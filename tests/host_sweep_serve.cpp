// Host-side sweep of the quantized attention block's planners and launch arithmetic over degenerate shapes, built
// with the library's sources compiled for the host only under -fsanitize=undefined.  No GPU is used: device pointers are
// fake addresses that are never dereferenced on the host, and every launch fails for lack of a device, after the
// host has computed its grid and workspace layout.
#include <cstdio>

#include "crvq.h"

static void* fake(size_t i) { return reinterpret_cast<void*>((static_cast<uintptr_t>(i) + 1) << 40); }
static long long g_calls = 0, g_hip = 0;
static int g_bad = 0;

static void expect_ok_or_hip(int status, const char* what) {
  ++g_calls;
  if (status == CRVQ_ERR_HIP) ++g_hip;
  if (status != CRVQ_OK && status != CRVQ_ERR_HIP) {
    std::fprintf(stderr, "unexpected status %d from %s: %s\n", status, what, crvq_last_error());
    ++g_bad;
  }
}

int main() {
  const size_t big = size_t{1} << 40;
  int8_t* k = static_cast<int8_t*>(fake(1));
  int8_t* v = static_cast<int8_t*>(fake(2));
  float* ks = static_cast<float*>(fake(3));
  float* vs = static_cast<float*>(fake(4));
  const int32_t* table = static_cast<const int32_t*>(fake(5));
  const int32_t* start = static_cast<const int32_t*>(fake(6));
  const int32_t* len = static_cast<const int32_t*>(fake(7));
  for (int B : {1, 2, 33})
    for (int Hkv : {1, 5, 32})
      for (int G : {1, 3, 8, 20})
        for (int D : {16, 64, 80, 128, 192, 256})
          for (int page : {16, 64, 256})
            for (int new_tokens : {1, 4, 17, 300, 5000})
              for (int kv : {0, 1, 513, 140000, 1 << 30})
                for (int dt : {CRVQ_F32, CRVQ_BF16}) {
                  const int Hq = Hkv * G;
                  const int64_t n = static_cast<int64_t>(B) * new_tokens;
                  const size_t ws = crvq_kv_attention_workspace_size(B, Hq, Hkv, D, new_tokens, kv);
                  if (ws % 256) ++g_bad;
                  expect_ok_or_hip(crvq_kv_attention(B, Hq, Hkv, D, page, 100, k, v, ks, vs, table, 50, start, len, new_tokens, kv,
                                                     n, dt, fake(8), Hq * D, D, fake(9), Hq * D, D, 0.1f, 1, kv % 7,
                                                     static_cast<float*>(fake(10)), fake(11), ws > big ? ws : big, nullptr),
                                   "crvq_kv_attention");
                  if (kv > 1) continue;
                  expect_ok_or_hip(crvq_kv_append(B, Hq, Hkv, D, page, 100, k, v, ks, vs, table, 50, start, len, new_tokens, n, dt,
                                                  fake(12), Hkv * D, D, fake(13), Hkv * D + 1, D, fake(8), Hq * D, D, fake(9),
                                                  Hq * D, D, static_cast<float*>(fake(14)), static_cast<float*>(fake(15)), 1000,
                                                  kv ? D : D / 2, nullptr, kv, nullptr),
                                   "crvq_kv_append");
                  expect_ok_or_hip(crvq_kv_read(B, Hkv, D, page, 100, k, v, ks, vs, table, 50, start, len, new_tokens, n, dt,
                                                fake(12), Hkv * D, D, kv ? nullptr : fake(13), Hkv * D, D, nullptr),
                                   "crvq_kv_read");
                }
  for (int64_t M : {1, 15, 16, 17, 64, 1031, 28672, 1 << 20})
    for (int64_t N : {1, 2, 31, 32, 33, 127, 128, 129, 3000, 8192, 13824, 100000, 1 << 20})
      for (int group : {32, 64, 128, 256})
        for (int dt : {CRVQ_F32, CRVQ_BF16}) {
          const int64_t ld = (N + 31) / 32 * 16, G = (N + group - 1) / group;
          uint8_t* codes = static_cast<uint8_t*>(fake(20));
          uint8_t* zeros = group == 64 ? nullptr : static_cast<uint8_t*>(fake(22));
          expect_ok_or_hip(crvq_w4_quantize(M, N, group, fake(23), N, dt, codes, ld, fake(21), dt, G, zeros, G, nullptr),
                           "crvq_w4_quantize");
          expect_ok_or_hip(crvq_w4_dequant(M, N, group, codes, ld, fake(21), dt, G, zeros, G, fake(24), N, dt, nullptr),
                           "crvq_w4_dequant");
          for (int64_t T : {1, 2, 3, 5, 8, 11, 16, 17, 64, 1000}) {
            const size_t ws = crvq_w4_gemv_workspace_size(M, N, T);
            expect_ok_or_hip(crvq_w4_gemv(M, N, T, group, codes, ld, fake(21), dt, G, zeros, G, fake(25), N, dt, fake(26), M, dt,
                                          fake(27), ws, nullptr),
                             "crvq_w4_gemv");
          }
        }
  if (g_bad) {
    std::fprintf(stderr, "host sweep: %d failures\n", g_bad);
    return 1;
  }
  std::printf("host sweep ok: %lld calls, %lld of them reached a launch\n", g_calls, g_hip);
  return 0;
}
