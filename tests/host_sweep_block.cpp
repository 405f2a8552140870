// Host-side sweep of the planners and launch arithmetic of drafts, budgets, 8-bit products and norms over degenerate shapes, built
// with the library's sources compiled for the host only under -fsanitize=undefined.  No GPU is used: device pointers are
// fake addresses that are never dereferenced on the host, and every launch fails for lack of a device, after the
// host has computed its grid and workspace layout.
#include <cstdio>

#include "crvq.h"

static void* fake(size_t i) { return reinterpret_cast<void*>((static_cast<uintptr_t>(i) + 1) << 42); }
template <typename T>
static T* of(size_t i) { return static_cast<T*>(fake(i)); }
static long long g_calls = 0, g_hip = 0;
static int g_bad = 0;

static void expect(int status, const char* what, bool unsupported = false) {
  ++g_calls;
  if (status == CRVQ_ERR_HIP) ++g_hip;
  if (status != CRVQ_OK && status != CRVQ_ERR_HIP && !(unsupported && status == CRVQ_ERR_UNSUPPORTED)) {
    std::fprintf(stderr, "unexpected status %d from %s: %s\n", status, what, crvq_last_error());
    ++g_bad;
  }
}

int main() {
  const size_t big = size_t{1} << 41;
  for (int B : {1, 2, 33})
    for (int Hkv : {1, 5, 32})
      for (int G : {1, 3, 20})
        for (int D : {16, 80, 128, 256})
          for (int page : {16, 64, 256})
            for (int n_new : {1, 17, 65, 300, 5000})
              for (int kv : {1, 513, 140000, 1 << 30})
                for (int dt : {CRVQ_F32, CRVQ_BF16}) {
                  const int Hq = Hkv * G;
                  const int64_t n = static_cast<int64_t>(B) * n_new, words = (n_new + 63) / 64;
                  size_t ws = crvq_kv_tree_attention_workspace_size(B, Hq, Hkv, D, n_new, kv);
                  if (ws % 256) ++g_bad;
                  expect(crvq_kv_tree_attention(B, Hq, Hkv, D, page, 100, of<int8_t>(1), of<int8_t>(2), of<float>(3), of<float>(4),
                                                of<int32_t>(5), 50, of<int32_t>(6), of<int32_t>(7), n_new, kv, n, dt, fake(8), Hq * D, D,
                                                fake(9), Hq * D, D, 0.1f, of<uint64_t>(10), words, kv % 7, of<int32_t>(11), of<float>(12),
                                                fake(20), ws > big ? ws : big, nullptr),
                         "crvq_kv_tree_attention");
                  ws = crvq_kv_weights_workspace_size(B, Hq, Hkv, D, n_new, kv);
                  if (ws % 256) ++g_bad;
                  expect(crvq_kv_weights(B, Hq, Hkv, D, page, 100, of<int8_t>(1), of<float>(3), of<int32_t>(5), 50, of<int32_t>(6), of<int32_t>(7),
                                         n_new, kv, n, dt, fake(8), Hq * D + kv % 2, D, of<float>(12), 0.1f, 1, kv % 7,
                                         n_new % 2 ? of<uint64_t>(10) : nullptr, words, nullptr, 0.5f, of<float>(14), of<float>(16), kv, fake(20),
                                         ws > big ? ws : big, nullptr),
                         "crvq_kv_weights");
                }
  for (int B : {1, 3, 700})
    for (int n : {1, 64, 65, 4000}) expect(crvq_tree_mask(B, of<int32_t>(1), of<int32_t>(2), of<int32_t>(3), n, n * 2, n % 3, of<uint64_t>(4), 63, of<int32_t>(5), nullptr), "crvq_tree_mask");
  for (int B : {1, 9, 1000})
    for (int Hkv : {1, 8, 33})
      for (int64_t ld : {0, 1, 5, 4096, 4097, 16384, 16385, 131001, 1 << 24, 1 << 30})
        for (int budget : {0, 1, 100, 1 << 30}) {
          const int64_t most = budget < ld ? budget : ld;
          const size_t ws = crvq_kv_select_workspace_size(B, Hkv, ld);
          if (ws % 256) ++g_bad;
          expect(crvq_kv_select(B, Hkv, of<int32_t>(1), of<float>(30), ld, budget, budget / 3, budget / 2, of<int32_t>(90), most + 3, of<int32_t>(3),
                                of<float>(150), fake(20), ws > big ? ws : big, nullptr),
                 "crvq_kv_select");
        }
  for (int D : {16, 80, 256})
    for (int page : {16, 64, 256})
      for (int keep : {1, 15, 64, 100000})
        for (int heads : {1, 8})
          expect(crvq_kv_gather(7, 8, D, page, 1000, of<int8_t>(1), of<int8_t>(2), of<float>(3), of<float>(4), of<int32_t>(5), 50, of<int32_t>(6),
                                of<int32_t>(7), keep + 1, heads, of<int32_t>(8), keep, of<int32_t>(9), 40, nullptr),
                 "crvq_kv_gather");
  for (int64_t M : {1, 15, 64, 1031, 6144, 12288, 28672, 1 << 20})
    for (int64_t N : {1, 15, 16, 17, 127, 128, 129, 3000, 14336, 65536})
      for (int64_t T : {1, 8, 9, 16, 17, 32, 33, 64, 65, 200, 4096, 100000})
        for (int64_t pad : {0, 1 << 23}) {
          const int64_t ld = (N + 15) / 16 * 16 + pad;
          const size_t ws = crvq_w8_gemm_workspace_size(M, N, T);
          if (ws % 256) ++g_bad;
          expect(crvq_w8_gemm(M, N, T, of<int8_t>(1), ld, of<float>(100), of<int8_t>(200), ld, of<float>(300), fake(400), M, T % 2 ? CRVQ_F32 : CRVQ_BF16,
                              fake(20), ws > big ? ws : big, nullptr),
                 "crvq_w8_gemm", T > 65535 * 16);
          if (T < 64 && !pad)
            expect(crvq_w8_quantize(M, N, fake(1), N + 1, T % 2 ? CRVQ_F32 : CRVQ_BF16, of<int8_t>(100), ld, of<float>(200), nullptr), "crvq_w8_quantize");
        }
  for (int64_t N : {1, 8, 511, 512, 513, 1024, 1025, 2048, 4096, 8192, 8193, 16384, 32768, 65535, 65536})
    for (int64_t T : {1, 3, 4, 5, 100000})
      for (int dt : {CRVQ_F32, CRVQ_BF16})
        for (int rd : {CRVQ_F32, CRVQ_BF16})
          expect(crvq_norm(T, N, T % 2, fake(1), N, dt, 1, fake(2), nullptr, fake(3), T % 2 ? N : 0, 0.5, fake(40), N, fake(80), N, rd, fake(5), nullptr,
                           CRVQ_F32, 1e-5, of<int8_t>(120), (N + 15) / 16 * 16, of<float>(7), nullptr),
                 "crvq_norm");
  std::printf("host sweep %s: %lld calls, %lld reached a launch\n", g_bad ? "FAILED" : "ok", g_calls, g_hip);
  return g_bad ? 1 : 0;
}
