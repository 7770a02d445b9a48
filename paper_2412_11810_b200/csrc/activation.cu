// Activations in 8 bits (include/snn.h, "sequence-model operators"; the format stands in seq_common.cuh).
//
// Bound by HBM (bytes of a value + 1 each way).  FAST: eight lanes share a group, eight neighbouring values each, so that
// loads and stores are 8 to 32 bytes per lane, and a warp has PACK_UNROLL x 4 groups in flight; it needs rows that are
// multiples of 8 values and aligned to them.  Otherwise a warp takes one group at a time, two values per lane.
#include <algorithm>
#include <type_traits>

#include "seq_common.cuh"

using namespace snnk;

namespace {

constexpr int PACK_WARPS = 8, PACK_UNROLL = 4;
template <typename IO> struct Eight;   // eight neighbouring values, in 16-byte accesses
template <> struct Eight<float> {
  float4 a, b;
  __device__ float2 pair(int j) const { return j == 0 ? make_float2(a.x, a.y) : j == 1 ? make_float2(a.z, a.w) : j == 2 ? make_float2(b.x, b.y) : make_float2(b.z, b.w); }
  __device__ void set(int j, float2 v) { if (j == 0) a.x = v.x, a.y = v.y; else if (j == 1) a.z = v.x, a.w = v.y; else if (j == 2) b.x = v.x, b.y = v.y; else b.z = v.x, b.w = v.y; }
};
template <typename IO> struct alignas(16) EightHalves {
  typename Pair<IO>::raw v[4];
  __device__ float2 pair(int j) const { return to_f32(v[j]); }
  __device__ void set(int j, float2 x) { set_raw(v[j], x); }
};
template <> struct Eight<__nv_bfloat16> : EightHalves<__nv_bfloat16> {};
template <> struct Eight<__half> : EightHalves<__half> {};

template <typename IO, int FORMAT, bool FAST>
__global__ void __launch_bounds__(32 * PACK_WARPS) activation_pack_kernel(const IO* values, int64_t n_rows, int n_cols, int64_t stride,
                                                                          uint8_t* codes, uint8_t* scales) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int groups = (n_cols + KEEP_GROUP - 1) / KEEP_GROUP;
  const int64_t n = n_rows * groups;
  if constexpr (FAST) {
    const int64_t step = (int64_t)gridDim.x * PACK_WARPS * 4 * PACK_UNROLL;
    for (int64_t g0 = ((int64_t)blockIdx.x * PACK_WARPS + warp) * 4 * PACK_UNROLL + (lane >> 3); g0 - (lane >> 3) < n; g0 += step) {
      Eight<IO> v[PACK_UNROLL];
#pragma unroll
      for (int u = 0; u < PACK_UNROLL; ++u) {   // (groups that do not exist: another one, not stored)
        const int64_t g = min(g0 + 4 * u, n - 1), row = g / groups;
        const int c = (int)(g - row * groups) * KEEP_GROUP + (lane & 7) * 8;
        v[u] = *reinterpret_cast<const Eight<IO>*>(values + row * stride + (c < n_cols ? c : 0));
      }
#pragma unroll
      for (int u = 0; u < PACK_UNROLL; ++u) {
        const int64_t g = min(g0 + 4 * u, n - 1), row = g / groups;
        const int group = (int)(g - row * groups), c = group * KEEP_GROUP + (lane & 7) * 8;
        const bool on = c < n_cols;
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = larger_magnitude(m, larger_magnitude(v[u].pair(j).x, v[u].pair(j).y));
        uint32_t top = on ? __float_as_uint(m) : 0u;
#pragma unroll
        for (int o = 1; o < 8; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const uint32_t byte = keep_scale_byte<FORMAT>(top);
        const float inverse = keep_scale_inverse(byte);
        uint2 q = make_uint2(0u, 0u);
        if (byte != 255u) {
          q.x = keep_encode2<FORMAT>(v[u].pair(0), inverse, top) | keep_encode2<FORMAT>(v[u].pair(1), inverse, top) << 16;
          q.y = keep_encode2<FORMAT>(v[u].pair(2), inverse, top) | keep_encode2<FORMAT>(v[u].pair(3), inverse, top) << 16;
        }
        if (g0 + 4 * u < n) {
          if (on) *reinterpret_cast<uint2*>(codes + row * n_cols + c) = q;
          if ((lane & 7) == 0) scales[g] = (uint8_t)byte;
        }
      }
    }
  } else for (int64_t i = (int64_t)blockIdx.x * PACK_WARPS + warp; i < n; i += (int64_t)gridDim.x * PACK_WARPS) {
    const int64_t row = i / groups;
    const int c = (int)(i % groups) * KEEP_GROUP + 2 * lane, n_ok = min(max(n_cols - c, 0), 2);
    uint32_t byte;
    const uint32_t pair = encode_row<FORMAT>(load_pair<false>(values + row * stride, c, n_ok), n_ok, byte);
    if (n_ok > 0) codes[row * n_cols + c] = (uint8_t)(pair & 255u);
    if (n_ok > 1) codes[row * n_cols + c + 1] = (uint8_t)(pair >> 8);
    if (lane == 0) scales[i] = (uint8_t)byte;
  }
}
template <typename IO, int FORMAT, bool FAST>
__global__ void __launch_bounds__(32 * PACK_WARPS) activation_unpack_kernel(const uint8_t* codes, const uint8_t* scales, int64_t n_rows,
                                                                            int n_cols, IO* values, int64_t stride) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int groups = (n_cols + KEEP_GROUP - 1) / KEEP_GROUP;
  const int64_t n = n_rows * groups;
  if constexpr (FAST) {
    const int64_t step = (int64_t)gridDim.x * PACK_WARPS * 4 * PACK_UNROLL;
    for (int64_t g0 = ((int64_t)blockIdx.x * PACK_WARPS + warp) * 4 * PACK_UNROLL + (lane >> 3); g0 - (lane >> 3) < n; g0 += step) {
      uint2 q[PACK_UNROLL];
      uint32_t byte[PACK_UNROLL];
#pragma unroll
      for (int u = 0; u < PACK_UNROLL; ++u) {
        const int64_t g = min(g0 + 4 * u, n - 1), row = g / groups;
        const int c = (int)(g - row * groups) * KEEP_GROUP + (lane & 7) * 8;
        q[u] = *reinterpret_cast<const uint2*>(codes + row * n_cols + (c < n_cols ? c : 0));
        byte[u] = scales[g];
      }
#pragma unroll
      for (int u = 0; u < PACK_UNROLL; ++u) {
        const int64_t g = min(g0 + 4 * u, n - 1), row = g / groups;
        const int c = (int)(g - row * groups) * KEEP_GROUP + (lane & 7) * 8;
        const float scale = keep_scale_value(byte[u]);
        Eight<IO> v;
        v.set(0, keep_decode2<IO, FORMAT>(q[u].x & 0xffffu, scale));
        v.set(1, keep_decode2<IO, FORMAT>(q[u].x >> 16, scale));
        v.set(2, keep_decode2<IO, FORMAT>(q[u].y & 0xffffu, scale));
        v.set(3, keep_decode2<IO, FORMAT>(q[u].y >> 16, scale));
        if (g0 + 4 * u < n && c < n_cols) *reinterpret_cast<Eight<IO>*>(values + row * stride + c) = v;
      }
    }
  } else for (int64_t i = (int64_t)blockIdx.x * PACK_WARPS + warp; i < n; i += (int64_t)gridDim.x * PACK_WARPS) {
    const int64_t row = i / groups;
    const int c = (int)(i % groups) * KEEP_GROUP + 2 * lane, n_ok = min(max(n_cols - c, 0), 2);
    store_pair<false>(values + row * stride, c, n_ok, decode_pair<IO>(codes + row * n_cols, scales[i], c, n_ok, FORMAT));
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
// the kernels' template arguments: the value type, and whether the fast path's alignment holds
template <typename F> snn_status by_dtype(int dtype, bool pairs, F&& f) {
  if (dtype == SNN_DTYPE_FP32) return pairs ? f(float(), std::true_type()) : f(float(), std::false_type());
  if (dtype == SNN_DTYPE_BF16) return pairs ? f(__nv_bfloat16(), std::true_type()) : f(__nv_bfloat16(), std::false_type());
  return pairs ? f(__half(), std::true_type()) : f(__half(), std::false_type());
}

// whether rows can be accessed eight values at a time
bool rows_of_eight(const void* values, int n_cols, int64_t row_stride, const uint8_t* codes) {
  return n_cols % 8 == 0 && row_stride % 8 == 0 && (uintptr_t)values % 16 == 0 && (uintptr_t)codes % 8 == 0;
}
unsigned pack_blocks(int64_t n_rows, int n_cols, bool fast) {
  const int64_t groups = n_rows * ((n_cols + KEEP_GROUP - 1) / KEEP_GROUP), per_block = PACK_WARPS * (fast ? 4 * PACK_UNROLL : 1);
  return (unsigned)std::min<int64_t>((groups + per_block - 1) / per_block, 148 * 8);
}
}  // namespace

extern "C" snn_status snn_activation_pack(const void* values, int32_t dtype, int64_t n_rows, int32_t n_cols, int64_t row_stride,
                                          int32_t format, uint8_t* codes, uint8_t* scales, void* stream) {
  if (n_rows < 0 || n_cols < 0 || !dtype_known(dtype) || (format != SNN_KEEP_INT8 && format != SNN_KEEP_E4M3)) return SNN_ERR_INVALID_ARG;
  if (n_rows == 0 || n_cols == 0) return SNN_OK;
  if (!values || !codes || !scales) return SNN_ERR_INVALID_ARG;
  return by_dtype(dtype, rows_of_eight(values, n_cols, row_stride, codes), [&](auto io, auto is_fast) {
    using IO = decltype(io);
    constexpr bool FAST = decltype(is_fast)::value;
    const auto kernel = format == SNN_KEEP_INT8 ? activation_pack_kernel<IO, SNN_KEEP_INT8, FAST> : activation_pack_kernel<IO, SNN_KEEP_E4M3, FAST>;
    kernel<<<pack_blocks(n_rows, n_cols, FAST), 32 * PACK_WARPS, 0, (cudaStream_t)stream>>>((const IO*)values, n_rows, n_cols, row_stride, codes, scales);
    return launched();
  });
}

extern "C" snn_status snn_activation_unpack(const uint8_t* codes, const uint8_t* scales, int32_t format, int64_t n_rows, int32_t n_cols,
                                            void* values, int32_t dtype, int64_t row_stride, void* stream) {
  if (n_rows < 0 || n_cols < 0 || !dtype_known(dtype) || (format != SNN_KEEP_INT8 && format != SNN_KEEP_E4M3)) return SNN_ERR_INVALID_ARG;
  if (n_rows == 0 || n_cols == 0) return SNN_OK;
  if (!values || !codes || !scales) return SNN_ERR_INVALID_ARG;
  return by_dtype(dtype, rows_of_eight(values, n_cols, row_stride, codes), [&](auto io, auto is_fast) {
    using IO = decltype(io);
    constexpr bool FAST = decltype(is_fast)::value;
    const auto kernel = format == SNN_KEEP_INT8 ? activation_unpack_kernel<IO, SNN_KEEP_INT8, FAST> : activation_unpack_kernel<IO, SNN_KEEP_E4M3, FAST>;
    kernel<<<pack_blocks(n_rows, n_cols, FAST), 32 * PACK_WARPS, 0, (cudaStream_t)stream>>>(codes, scales, n_rows, n_cols, (IO*)values, row_stride);
    return launched();
  });
}
