// 4-bit matrices with a scale (and a zero point) per group of consecutive columns: quantization,
// reconstruction and the product with a few vectors.
#include "kv_common.h"

namespace crvq {
namespace {

constexpr float kMinScale = 7.888609052210118e-31f;  // 2^-100

template <typename T>
__device__ __forceinline__ float ld1(const T* p) {
  if constexpr (sizeof(T) == 4)
    return *reinterpret_cast<const float*>(p);
  else
    return bf16_f(*p);
}
template <typename T>
__device__ __forceinline__ void st1(T* p, float x) {
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<float*>(p) = x;
  else
    *p = static_cast<T>(f_bf16(x));
}

template <typename TS>
__device__ __forceinline__ float scale_at(const W4& w, int64_t r, int64_t g) {
  return ld1(static_cast<const TS*>(w.scales) + r * w.ld_s + g);
}
__device__ __forceinline__ float zero_at(const W4& w, int64_t r, int64_t g) {
  return w.zeros ? static_cast<float>(w.zeros[r * w.ld_z + g]) : 8.f;
}

// ---- quantization: a lane owns eight columns (four bytes of codes), group / 8 lanes share a group -------
template <typename T, typename TS>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const T* W, int64_t ldw, const W4 w, int64_t units, int64_t stored) {
  const int64_t u = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;  // eight columns of a row
  const int64_t r = u / units, j0 = (u - r * units) * 8;
  const bool in = r < w.M;
  float x[8];
  float lo = 0.f, hi = 0.f;
  bool finite = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = in && j0 + i < w.N ? ld1(W + r * ldw + j0 + i) : 0.f;
    finite &= fabsf(x[i]) < __uint_as_float(0x7f800000u);
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
  int bad = !finite;
  for (int o = 1; o < 1 << (w.group_log2 - 3); o <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, o));
    hi = fmaxf(hi, __shfl_xor(hi, o));
    bad |= __shfl_xor(bad, o);
  }
  if (!in) return;
  float s = fmaxf(w.zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f, kMinScale);
  if (bad || !(s < __uint_as_float(0x7f800000u))) s = __uint_as_float(0x7fc00000u);
  if (sizeof(TS) == 2) s = bf16_f(f_bf16(s));
  const bool number = s == s;
  const float z = !w.zeros ? 8.f : number ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = number && j0 + i < w.N ? fminf(fmaxf(rintf(x[i] / s) + z, 0.f), 15.f) : 0.f;
    c |= static_cast<uint32_t>(static_cast<int>(q)) << (4 * i);
  }
  if (j0 < stored) *reinterpret_cast<uint32_t*>(w.codes + r * w.ld + (j0 >> 1)) = c;
  if ((j0 & ((1 << w.group_log2) - 1)) == 0 && j0 < w.N) {
    const int64_t g = j0 >> w.group_log2;
    st1(static_cast<TS*>(w.scales) + r * w.ld_s + g, s);
    if (w.zeros) w.zeros[r * w.ld_z + g] = static_cast<uint8_t>(z);
  }
}

template <typename T, typename TS>
__global__ __launch_bounds__(256) void w4_dequant_kernel(const W4 w, T* out, int64_t ldo, int64_t units) {
  const int64_t u = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t r = u / units, j0 = (u - r * units) * 8;
  if (r >= w.M) return;
  const uint32_t c = *reinterpret_cast<const uint32_t*>(w.codes + r * w.ld + (j0 >> 1));
  const float s = scale_at<TS>(w, r, j0 >> w.group_log2), z = zero_at(w, r, j0 >> w.group_log2);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (j0 + i < w.N) st1(out + r * ldo + j0 + i, (static_cast<float>((c >> (4 * i)) & 15) - z) * s);
}

// ---- product: a wave per row and vector -------------------------------------------------------------------
template <typename TX, typename TY, typename TS>
__global__ __launch_bounds__(256) void w4_gemv_kernel(const W4 w, int64_t T, const TX* x, int64_t ldx, TY* y, int64_t ldy) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (item >= w.M * T) return;
  const int64_t t = item / w.M, r = item - t * w.M;
  const int lane = threadIdx.x & 63;
  float acc = 0.f;
  for (int64_t j0 = lane * 8; j0 < w.N; j0 += 512) {
    const uint32_t c = *reinterpret_cast<const uint32_t*>(w.codes + r * w.ld + (j0 >> 1));
    const float s = scale_at<TS>(w, r, j0 >> w.group_log2), z = zero_at(w, r, j0 >> w.group_log2);
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (j0 + i < w.N) {
        const float xv = ld1(x + t * ldx + j0 + i);
        part = fmaf(static_cast<float>((c >> (4 * i)) & 15) - z, xv, part) + (xv - xv);  // an infinity becomes NaN
      }
    acc = fmaf(s, part, acc);
  }
  for (int o = 32; o; o >>= 1) acc += __shfl_xor(acc, o);
  if (lane == 0) st1(y + t * ldy + r, acc);
}

hipError_t blocks_of(int64_t items, int per, dim3* grid) {
  const int64_t n = cdiv(items, per);
  if (n > 0x7fffffffLL) return hipErrorInvalidConfiguration;
  *grid = dim3(static_cast<uint32_t>(n));
  return hipSuccess;
}

}  // namespace

hipError_t launch_w4_quantize(const void* W, int64_t ldw, int type, const W4& w, hipStream_t stream) {
  // the units of a row are padded to whole groups of lanes, so that no group straddles two waves; codes are
  // stored up to a multiple of 16 bytes, which every row stride holds
  const int64_t span = w.group_log2 > 5 ? int64_t{1} << w.group_log2 : 32, stored = cdiv(w.N, 32) * 32;
  const int64_t units = cdiv(w.N, span) * span / 8;
  dim3 grid;
  const hipError_t e = blocks_of(w.M * units, 256, &grid);
  if (e != hipSuccess) return e;
  if (type == ET_F32) {
    if (w.s_type == ET_F32) w4_quantize_kernel<uint32_t, uint32_t><<<grid, 256, 0, stream>>>(static_cast<const uint32_t*>(W), ldw, w, units, stored);
    else w4_quantize_kernel<uint32_t, uint16_t><<<grid, 256, 0, stream>>>(static_cast<const uint32_t*>(W), ldw, w, units, stored);
  } else {
    if (w.s_type == ET_F32) w4_quantize_kernel<uint16_t, uint32_t><<<grid, 256, 0, stream>>>(static_cast<const uint16_t*>(W), ldw, w, units, stored);
    else w4_quantize_kernel<uint16_t, uint16_t><<<grid, 256, 0, stream>>>(static_cast<const uint16_t*>(W), ldw, w, units, stored);
  }
  return hipGetLastError();
}

hipError_t launch_w4_dequant(const W4& w, void* out, int64_t ldo, int type, hipStream_t stream) {
  const int64_t units = cdiv(w.N, 8);
  dim3 grid;
  const hipError_t e = blocks_of(w.M * units, 256, &grid);
  if (e != hipSuccess) return e;
  if (type == ET_F32) {
    if (w.s_type == ET_F32) w4_dequant_kernel<uint32_t, uint32_t><<<grid, 256, 0, stream>>>(w, static_cast<uint32_t*>(out), ldo, units);
    else w4_dequant_kernel<uint32_t, uint16_t><<<grid, 256, 0, stream>>>(w, static_cast<uint32_t*>(out), ldo, units);
  } else {
    if (w.s_type == ET_F32) w4_dequant_kernel<uint16_t, uint32_t><<<grid, 256, 0, stream>>>(w, static_cast<uint16_t*>(out), ldo, units);
    else w4_dequant_kernel<uint16_t, uint16_t><<<grid, 256, 0, stream>>>(w, static_cast<uint16_t*>(out), ldo, units);
  }
  return hipGetLastError();
}

size_t w4_gemv_ws_bytes(int64_t, int64_t, int64_t) { return 0; }

template <typename TX, typename TY>
static hipError_t gemv_as(const W4& w, int64_t T, const void* x, int64_t ldx, void* y, int64_t ldy, hipStream_t stream) {
  dim3 grid;
  const hipError_t e = blocks_of(w.M * T, 4, &grid);
  if (e != hipSuccess) return e;
  const TX* xt = static_cast<const TX*>(x);
  TY* yt = static_cast<TY*>(y);
  if (w.s_type == ET_F32)
    w4_gemv_kernel<TX, TY, uint32_t><<<grid, 256, 0, stream>>>(w, T, xt, ldx, yt, ldy);
  else
    w4_gemv_kernel<TX, TY, uint16_t><<<grid, 256, 0, stream>>>(w, T, xt, ldx, yt, ldy);
  return hipGetLastError();
}

hipError_t launch_w4_gemv(const W4& w, int64_t T, const void* x, int64_t ldx, int x_type, void* y, int64_t ldy, int y_type,
                          void*, hipStream_t stream) {
  if (x_type == ET_F32)
    return y_type == ET_F32 ? gemv_as<uint32_t, uint32_t>(w, T, x, ldx, y, ldy, stream)
                            : gemv_as<uint32_t, uint16_t>(w, T, x, ldx, y, ldy, stream);
  return y_type == ET_F32 ? gemv_as<uint16_t, uint32_t>(w, T, x, ldx, y, ldy, stream)
                          : gemv_as<uint16_t, uint16_t>(w, T, x, ldx, y, ldy, stream);
}

}  // namespace crvq
