// What the sequence-model operators share: element types, pairs of neighbouring values, and the 8-bit format of kept
// activations.
//
// 8-bit format.  The last axis is cut into groups of 64 values (the last one may be shorter).  A group has one scale
// byte c, standing for 2^(c - 127), and a code byte per value.  The scale is the smallest power of two, not
// below 2^-127, at which the largest magnitude of the group is below 128 for int8 (codes are rounded to nearest, ties to
// even, and end at 127) or no more than 448 for e4m3.
// A power of two costs int8 up to one of its seven bits against a free scale; in return scaling is exact, decoding
// needs one multiplication, and codes do not depend on how a quotient is rounded.  c = 255 marks a group that holds an
// infinity or a NaN: all of it decodes to NaN.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/snn.h"

namespace snnk {

constexpr int KEEP_GROUP = SNN_KEEP_GROUP;
// The bounds-checked build can let bounded waits run out (snn_selftest_scan_wait, snn_selftest_vocab_loss_wait); in the other
// one their limits are constants (as parameters they cost the recurrence 2 %: 2048 x 16 x 2048 bf16/int8 training 326 -> 332 us).
#if defined(SNN_DEBUG_CHECKS) && SNN_DEBUG_CHECKS
constexpr bool WAIT_TESTS = true;
#else
constexpr bool WAIT_TESTS = false;
#endif

template <typename IO> struct Pair;
template <> struct Pair<float> { using raw = float2; };
template <> struct Pair<__nv_bfloat16> { using raw = __nv_bfloat162; };
template <> struct Pair<__half> { using raw = __half2; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float2 to_f32(float2 v) { return v; }
__device__ __forceinline__ float2 to_f32(__nv_bfloat162 v) { return __bfloat1622float2(v); }
__device__ __forceinline__ float2 to_f32(__half2 v) { return __half22float2(v); }
template <typename IO> __device__ __forceinline__ IO from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
__device__ __forceinline__ void set_raw(float2& r, float2 v) { r = v; }
__device__ __forceinline__ void set_raw(__nv_bfloat162& r, float2 v) { r = __float22bfloat162_rn(v); }
__device__ __forceinline__ void set_raw(__half2& r, float2 v) { r = __float22half2_rn(v); }

// Values c and c + 1 of a row, of which n_ok (0, 1 or 2) exist.  The loads are unconditional, so that many of them are in
// flight at once: a value that does not exist is read from another place of the row and means nothing.  PAIRS: an access
// of two values is aligned, and rows have an even number of them.
template <bool PAIRS, typename IO>
__device__ __forceinline__ float2 load_pair(const IO* row, int c, int n_ok) {
  if (PAIRS) return to_f32(*reinterpret_cast<const typename Pair<IO>::raw*>(row + (n_ok ? c : 0)));
  return make_float2(to_f32(row[n_ok ? c : 0]), to_f32(row[n_ok == 2 ? c + 1 : 0]));
}
// The same in the values' own type.
template <bool PAIRS, typename IO>
__device__ __forceinline__ typename Pair<IO>::raw load_raw(const IO* row, int c, int n_ok) {
  if (PAIRS) return *reinterpret_cast<const typename Pair<IO>::raw*>(row + (n_ok ? c : 0));
  typename Pair<IO>::raw r;
  r.x = row[n_ok ? c : 0];
  r.y = row[n_ok == 2 ? c + 1 : 0];
  return r;
}
template <bool PAIRS, typename IO>
__device__ __forceinline__ void store_pair(IO* row, int c, int n_ok, float2 v) {
  if (PAIRS) {
    typename Pair<IO>::raw r;
    set_raw(r, v);
    if (n_ok) *reinterpret_cast<typename Pair<IO>::raw*>(row + c) = r;
    return;
  }
  if (n_ok > 0) row[c] = from_f32<IO>(v.x);
  if (n_ok > 1) row[c + 1] = from_f32<IO>(v.y);
}

// ---- pairs of fp32 values --------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t bits2(float2 v) { return (uint64_t)__float_as_uint(v.y) << 32 | __float_as_uint(v.x); }
__device__ __forceinline__ float2 from_bits2(uint64_t u) { return make_float2(__uint_as_float((uint32_t)u), __uint_as_float((uint32_t)(u >> 32))); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
  return from_bits2(d);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// ---- 8-bit codes -------------------------------------------------------------------------------------------
// Scale byte of a group whose largest magnitude has the bit pattern `top` (NaN sorts above infinity above the rest).
template <int FORMAT> __device__ __forceinline__ uint32_t keep_scale_byte(uint32_t top) {
  const int exponent = (int)(top >> 23);
  const uint32_t fraction = top & 0x7fffffu;
  if (exponent == 255) return 255u;
  // top = 1.f x 2^(exponent - 127).  int8: 1.f x 64 is below 128.  e4m3: 1.f x 256 is at most 448 while 1.f <= 1.75, one
  // scale up beyond that.
  const int c = FORMAT == SNN_KEEP_INT8 ? exponent - 6 : exponent - 8 + (fraction > 0x600000u);
  return (uint32_t)max(c, 0);
}
__device__ __forceinline__ float keep_scale_inverse(uint32_t c) { return __uint_as_float((254u - min(c, 253u)) << 23); }
__device__ __forceinline__ float keep_scale_value(uint32_t c) {
  return __uint_as_float(c == 0u ? 0x00400000u : c == 255u ? 0x7fc00000u : c << 23);
}
// Whether an int8 code of a group could round to 128 and has to be cut.
template <int FORMAT> __device__ __forceinline__ bool keep_needs_cut(uint32_t top) {
  return FORMAT == SNN_KEEP_INT8 && (top & 0x7fffffu) >= 0x7f0000u;
}
// Two code bytes, low first.
template <int FORMAT> __device__ __forceinline__ uint32_t keep_encode2(float2 v, float inverse, bool cut) {
  const float2 u = mul2(v, both(inverse));
  if (FORMAT == SNN_KEEP_INT8) {
    // adding 1.5 x 2^23 rounds to an integer (nearest even) and leaves it in the low bits: no conversion instructions,
    // which run at a quarter of the rate
    const float magic = 12582912.f;
    float2 r = add2(u, both(magic));
    if (cut) r = make_float2(fminf(fmaxf(r.x, magic - 127.f), magic + 127.f), fminf(fmaxf(r.y, magic - 127.f), magic + 127.f));
    return __byte_perm(__float_as_uint(r.x), __float_as_uint(r.y), 0x0040) & 0xffffu;
  }
  return (uint32_t)__nv_cvt_float2_to_fp8x2(u, __NV_SATFINITE, __NV_E4M3);
}
template <typename IO> __device__ __forceinline__ float largest_finite();
template <> __device__ __forceinline__ float largest_finite<float>() { return __uint_as_float(0x7f7fffffu); }
template <> __device__ __forceinline__ float largest_finite<__nv_bfloat16>() { return __uint_as_float(0x7f7f0000u); }
template <> __device__ __forceinline__ float largest_finite<__half>() { return 65504.f; }
// The values of two codes, within the range of type IO.
template <typename IO> __device__ __forceinline__ float within(float v) {   // NaN stays
  const float top = largest_finite<IO>();
  return fabsf(v) > top ? copysignf(top, v) : v;
}
template <typename IO, int FORMAT> __device__ __forceinline__ float2 keep_decode2(uint32_t codes, float scale) {
  float a, b;
  if (FORMAT == SNN_KEEP_INT8) {   // code + 128 in the low bits of 2^23: again no conversion instructions
    const uint32_t u = codes ^ 0x8080u;
    a = __fmul_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7650)) - 8388736.f, scale);
    b = __fmul_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7651)) - 8388736.f, scale);
    // (an int8 code stays below the largest value of the type that was packed: only fp16 can be too narrow for it)
    if (largest_finite<IO>() > 65504.f) return make_float2(a, b);
  } else {
    const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3)));
    a = __fmul_rn(v.x, scale);
    b = __fmul_rn(v.y, scale);
  }
  return make_float2(within<IO>(a), within<IO>(b));
}
// The larger magnitude of two values; NaN if one of them is.
__device__ __forceinline__ float larger_magnitude(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(fabsf(a)), "f"(fabsf(b)));
  return m;
}

// ---- host side -----------------------------------------------------------------------------------------------
inline size_t dtype_size(int dtype) { return dtype == SNN_DTYPE_FP32 ? 4 : 2; }
inline bool dtype_known(int dtype) { return dtype >= SNN_DTYPE_FP32 && dtype <= SNN_DTYPE_FP16; }
inline snn_status launched() { return cudaGetLastError() == cudaSuccess ? SNN_OK : SNN_ERR_CUDA; }

}  // namespace snnk
