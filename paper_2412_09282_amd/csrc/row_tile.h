// Shared by the kernels that hold whole rows in registers (k_norm.hip, k_w8.hip): how a row's elements lie in the threads
// that share it, its loads and stores, its sums and largest magnitude, and its 8-bit codes.
#pragma once

#include "crvq.h"
#include "crvq_internal.h"

namespace crvq {

typedef float row_f2 __attribute__((ext_vector_type(2)));
typedef __bf16 row_b2 __attribute__((ext_vector_type(2)));

// THREADS threads (a wave, or a workgroup of its own) hold a row of up to THREADS * V * 8 elements.  VEC: thread t holds
// the 8 elements from (v THREADS + t) 8 on, in loads of 16 bytes; otherwise element (v 8 + e) THREADS + t, one by one.
template <int THREADS, int V, bool VEC>
struct RowTile {
  static constexpr int kThreads = THREADS, kVectors = V, kBlock = THREADS < 256 ? 256 : THREADS, kRows = kBlock / THREADS;
  int t, N;
  __device__ __forceinline__ int at(int v, int e) const { return VEC ? (v * THREADS + t) * 8 + e : (v * 8 + e) * THREADS + t; }
  __device__ __forceinline__ bool has(int v, int e) const { return at(v, VEC ? 0 : e) < N; }

  template <typename T>
  __device__ __forceinline__ void load(const T* row, float (&x)[V][8]) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (VEC) {
        if (!has(v, 0)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[v][e] = 0.f;
        } else if constexpr (sizeof(T) == 4) {
          const float4 a = *reinterpret_cast<const float4*>(row + at(v, 0)), b = *reinterpret_cast<const float4*>(row + at(v, 4));
          x[v][0] = a.x, x[v][1] = a.y, x[v][2] = a.z, x[v][3] = a.w;
          x[v][4] = b.x, x[v][5] = b.y, x[v][6] = b.z, x[v][7] = b.w;
        } else {
          const uint4 a = *reinterpret_cast<const uint4*>(row + at(v, 0));
          const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[v][2 * e] = __uint_as_float(w[e] << 16);
            x[v][2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[v][e] = 0.f;
          if (has(v, e)) {
            if constexpr (sizeof(T) == 4) x[v][e] = reinterpret_cast<const float*>(row)[at(v, e)];
            else x[v][e] = __uint_as_float(static_cast<uint32_t>(row[at(v, e)]) << 16);
          }
        }
      }
    }
  }
  // a row of a type that is known at run time
  __device__ __forceinline__ void load(const void* row, bool f32, float (&x)[V][8]) const {
    if (f32) load(static_cast<const uint32_t*>(row), x);
    else load(static_cast<const uint16_t*>(row), x);
  }

  static __device__ __forceinline__ uint32_t pair(float a, float b) {  // rounded to nearest even; a NaN stays one
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((row_f2{a, b}), row_b2));
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (&x)[V][8]) const {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (VEC) {
        if (!has(v, 0)) continue;
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(row + at(v, 0)) = make_float4(x[v][0], x[v][1], x[v][2], x[v][3]);
          *reinterpret_cast<float4*>(row + at(v, 4)) = make_float4(x[v][4], x[v][5], x[v][6], x[v][7]);
        } else {
          *reinterpret_cast<uint4*>(row + at(v, 0)) = make_uint4(pair(x[v][0], x[v][1]), pair(x[v][2], x[v][3]),
                                                                 pair(x[v][4], x[v][5]), pair(x[v][6], x[v][7]));
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (has(v, e)) {
            if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(row)[at(v, e)] = x[v][e];
            else row[at(v, e)] = static_cast<T>(pair(x[v][e], 0.f));
          }
      }
    }
  }

  // The sum over the row's threads, in an order that the row's size alone sets.  `red`: kBlock / 64 entries that no other
  // sum or maximum of the row uses.
  __device__ __forceinline__ double sum(double x, double* red) const {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    if constexpr (THREADS > 64) {
      if ((t & 63) == 0) red[t >> 6] = x;
      __syncthreads();
      x = red[0];
#pragma unroll
      for (int w = 1; w < THREADS / 64; ++w) x += red[w];
    }
    return x;
  }
  __device__ __forceinline__ uint32_t max_bits(uint32_t x, uint32_t* red) const {
#pragma unroll
    for (int o = 32; o; o >>= 1) x = max(x, static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), o)));
    if constexpr (THREADS > 64) {
      if ((t & 63) == 0) red[t >> 6] = x;
      __syncthreads();
      x = red[0];
#pragma unroll
      for (int w = 1; w < THREADS / 64; ++w) x = max(x, red[w]);
    }
    return x;
  }

  // The row in 8 bits: s = max(max|x| / 127, 2^-100), c = min(max(rint(x / s), -127), 127), each operation rounded on its
  // own; a NaN or infinity makes s NaN and the codes 0.  Codes past N up to a multiple of 16 are 0.
  __device__ __forceinline__ void quantize(const float (&x)[V][8], int8_t* row, float* scale, uint32_t* red) const {
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[v][e]) & 0x7fffffffu);  // orders magnitudes, NaN last
    most = max_bits(most, red);
    const bool finite = most < 0x7f800000u;
    const float s = fmaxf(__uint_as_float(most) / 127.f, 0x1p-100f);
    if (t == 0) *scale = finite ? s : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      int c[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = finite ? static_cast<int>(fminf(fmaxf(rintf(x[v][e] / s), -127.f), 127.f)) : 0;
      if constexpr (VEC) {
        if (!has(v, 0)) continue;
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= (static_cast<uint32_t>(c[e]) & 255u) << (8 * (e & 3));
        *reinterpret_cast<uint2*>(row + at(v, 0)) = make_uint2(w[0], w[1]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (has(v, e)) row[at(v, e)] = static_cast<int8_t>(c[e]);
      }
    }
    const int end = (N + 15) & ~15;
    if (t < end - N) row[N + t] = 0;
  }
};

// Calls f with the tile that a row of N elements takes: a wave up to 1024 elements, 256 threads up to 8192, 1024 above.
// What bounds it: registers hold 32 elements of a thread (64 for the longest rows), so a row is read once.
template <bool VEC, class F>
hipError_t with_row_tile(int64_t N, F&& f) {
  if (N <= 512) return f(RowTile<64, 1, VEC>{});
  if (N <= 1024) return f(RowTile<64, 2, VEC>{});
  if (N <= 2048) return f(RowTile<256, 1, VEC>{});
  if (N <= 4096) return f(RowTile<256, 2, VEC>{});
  if (N <= 8192) return f(RowTile<256, 4, VEC>{});
  if (N <= 16384) return f(RowTile<1024, 2, VEC>{});
  if (N <= 32768) return f(RowTile<1024, 4, VEC>{});
  return f(RowTile<1024, 8, VEC>{});
}

}  // namespace crvq
