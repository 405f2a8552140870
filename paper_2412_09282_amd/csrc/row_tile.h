// Shared by the kernels that hold whole rows in registers (k_norm.hip, k_w8.hip): how a row's elements lie in the threads
// that share it, its loads and stores, its sums and largest magnitude, and its 8-bit codes.
#pragma once

#include "crvq.h"
#include "crvq_internal.h"

namespace crvq {

typedef float row_f2 __attribute__((ext_vector_type(2)));
typedef __bf16 row_b2 __attribute__((ext_vector_type(2)));

// THREADS threads (a wave, or up to a workgroup of its own) hold a row of up to THREADS * V * 8 elements: thread t the 8 from
// (v THREADS + t) 8 on, in loads of 16 bytes, which may start at any element.  WHOLE: N is a multiple of 8; otherwise the row's
// last few elements go one by one.
template <typename T>
struct RowPiece;
template <>
struct __attribute__((packed, aligned(4))) RowPiece<uint32_t> {
  float x[8];
};
template <>
struct __attribute__((packed, aligned(2))) RowPiece<uint16_t> {
  uint32_t x[4];
};

template <int THREADS, int V, bool WHOLE>
struct RowTile {
  static constexpr int kThreads = THREADS, kVectors = V, kBlock = THREADS < 256 ? 256 : THREADS, kRows = kBlock / THREADS;
  int t, N;
  __device__ __forceinline__ int at(int v, int e) const { return (v * THREADS + t) * 8 + e; }
  __device__ __forceinline__ bool has(int v, int e) const { return at(v, WHOLE ? 0 : e) < N; }

  template <typename T>
  __device__ __forceinline__ void load(const T* row, int v, float (&x)[8]) const {
    if (has(v, 7)) {
      const RowPiece<T> p = *reinterpret_cast<const RowPiece<T>*>(row + at(v, 0));
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p.x[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = __uint_as_float(p.x[e] << 16);
          x[2 * e + 1] = __uint_as_float(p.x[e] & 0xffff0000u);
        }
      }
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if constexpr (!WHOLE) {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (has(v, e)) {
          if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(row[at(v, e)]);
          else x[e] = __uint_as_float(static_cast<uint32_t>(row[at(v, e)]) << 16);
        }
    }
  }
  // a row of a type that is known at run time
  __device__ __forceinline__ void load(const void* row, bool f32, int v, float (&x)[8]) const {
    if (f32) load(static_cast<const uint32_t*>(row), v, x);
    else load(static_cast<const uint16_t*>(row), v, x);
  }

  static __device__ __forceinline__ uint32_t pair(float a, float b) {  // rounded to nearest even; a NaN stays one
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((row_f2{a, b}), row_b2));
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, int v, const float (&x)[8]) const {
    RowPiece<T> p;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p.x[e] = x[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) p.x[e] = pair(x[2 * e], x[2 * e + 1]);
    }
    if (has(v, 7)) {
      *reinterpret_cast<RowPiece<T>*>(row + at(v, 0)) = p;
    } else if constexpr (!WHOLE) {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (has(v, e)) {
          if constexpr (sizeof(T) == 4) row[at(v, e)] = __float_as_uint(x[e]);
          else row[at(v, e)] = static_cast<T>(p.x[e >> 1] >> (16 * (e & 1)));
        }
    }
  }

  // The sum over the row's threads, in an order that the row's size alone sets.  `red`: THREADS / 64 entries that no other
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
  // own; a NaN or infinity makes s NaN and the codes 0.  Codes past N up to a multiple of 16 are 0.  Nothing is stored unless `there`.
  __device__ __forceinline__ void quantize(const float (&x)[V][8], int8_t* row, float* scale, uint32_t* red, bool there) const {
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[v][e]) & 0x7fffffffu);  // orders magnitudes, NaN last
    most = max_bits(most, red);
    if (!there) return;
    const bool finite = most < 0x7f800000u;
    const float s = fmaxf(__uint_as_float(most) / 127.f, 0x1p-100f);
    const int end = (N + 15) & ~15;  // past N the elements are 0
    if (t == 0) *scale = finite ? s : __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      int c[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = finite ? static_cast<int>(fminf(fmaxf(rintf(x[v][e] / s), -127.f), 127.f)) : 0;
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e >> 2] |= (static_cast<uint32_t>(c[e]) & 255u) << (8 * (e & 3));
      if (at(v, 0) < end) *reinterpret_cast<uint2*>(row + at(v, 0)) = make_uint2(w[0], w[1]);
    }
  }
};

// Calls f with the tile that a row of N elements takes: 8 elements a thread up to 2048, 16 up to 16384 (32 of them cost
// registers that other rows' loads need: 8192 rows of 8192 in the norm 258 us, with 16 196 when that was measured and 178
// now), more only where a workgroup ends.
template <class F>
hipError_t with_row_tile(int64_t N, F&& f) {
  auto as = [&](auto threads, auto v) {
    constexpr int kT = decltype(threads)::value, kV = decltype(v)::value;
    return N % 8 == 0 ? f(RowTile<kT, kV, true>{}) : f(RowTile<kT, kV, false>{});
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  if (N <= 512) return as(std::integral_constant<int, 64>{}, One{});
  if (N <= 1024) return as(std::integral_constant<int, 128>{}, One{});
  if (N <= 2048) return as(std::integral_constant<int, 256>{}, One{});
  if (N <= 4096) return as(std::integral_constant<int, 256>{}, Two{});
  if (N <= 8192) return as(std::integral_constant<int, 512>{}, Two{});
  if (N <= 16384) return as(std::integral_constant<int, 1024>{}, Two{});
  if (N <= 32768) return as(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
  return as(std::integral_constant<int, 1024>{}, std::integral_constant<int, 8>{});
}

}  // namespace crvq
