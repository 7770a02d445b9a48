// Activations in 8 bits (include/snn.h, "sequence-model operators"; the format stands in seq_common.cuh).
//
// Bound by HBM (bytes of a value + 1 each way) as long as a value costs few instructions: eight lanes share a group, eight
// values each, and a warp has PACK_UNROLL x 4 groups in flight.  FAST: 16 bytes of values per access, neighbouring lanes at
// neighbouring addresses; it needs rows that are multiples of 8 values and aligned.  Otherwise value by value, eight
// neighbouring ones per group and access.
#include <algorithm>
#include <type_traits>

#include "seq_common.cuh"

using namespace snnk;

namespace {

constexpr int PACK_WARPS = 8, PACK_UNROLL = 4;
// Quotients by the groups of a row: a multiplication with ceil(2^64 / d) is exact while the dividend times d is below 2^64.
struct Divisor {
  uint64_t inverse;   // 0: the divisor is 1
  int d;
  __device__ __forceinline__ int64_t quotient(int64_t n) const { return inverse ? (int64_t)__umul64hi((uint64_t)n, inverse) : n; }
};
// Place in its group of the j-th value of lane s (of eight).
template <typename IO, bool FAST> __device__ __forceinline__ constexpr int place(int s, int j) {
  constexpr int V = 16 / sizeof(IO);   // values per access
  return FAST ? j / V * (8 * V) + s * V + j % V : s + 8 * j;
}
template <typename IO> struct alignas(16) Sixteen {
  typename Pair<IO>::raw v[8 / sizeof(IO)];
};
// The eight values of a lane as fp32 pairs, and back; `row`: the group's first value, of which n exist.
template <typename IO, bool FAST> struct Values {
  Sixteen<IO> q[sizeof(IO) / 2];
  __device__ __forceinline__ void load(const IO* row, int s, int n) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(IO) / 2; ++i) {
      const int at = place<IO, true>(s, i * (16 / (int)sizeof(IO)));
      q[i] = *reinterpret_cast<const Sixteen<IO>*>(row + (at < n ? at : 0));
    }
  }
  __device__ __forceinline__ float2 pair(int j) const { return to_f32(q[2 * j / (16 / (int)sizeof(IO))].v[j % (8 / (int)sizeof(IO))]); }
};
template <typename IO> struct Values<IO, false> {
  IO v[8];
  __device__ __forceinline__ void load(const IO* row, int s, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = row[min(s + 8 * j, n - 1)];
  }
  __device__ __forceinline__ float2 pair(int j) const { return make_float2(to_f32(v[2 * j]), to_f32(v[2 * j + 1])); }
};

template <typename IO, int FORMAT, bool FAST>
__global__ void __launch_bounds__(32 * PACK_WARPS, 3) activation_pack_kernel(const IO* values, int64_t n_rows, int n_cols, int64_t stride,
                                                                             Divisor by, uint8_t* codes, uint8_t* scales) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = lane % 8;
  const int64_t n = n_rows * by.d, step = (int64_t)gridDim.x * PACK_WARPS * 4 * PACK_UNROLL;
  for (int64_t first = ((int64_t)blockIdx.x * PACK_WARPS + warp) * 4 * PACK_UNROLL; first < n; first += step) {
    Values<IO, FAST> v[PACK_UNROLL];
#pragma unroll
    for (int u = 0; u < PACK_UNROLL; ++u) {   // (groups that do not exist: the last one again, not stored)
      const int64_t g = min(first + 4 * u + lane / 8, n - 1), row = by.quotient(g);
      const int c0 = (int)(g - row * by.d) * KEEP_GROUP;
      v[u].load(values + row * stride + c0, s, n_cols - c0);
    }
#pragma unroll
    for (int u = 0; u < PACK_UNROLL; ++u) {
      const int64_t wanted = first + 4 * u + lane / 8, g = min(wanted, n - 1), row = by.quotient(g);
      const int c0 = (int)(g - row * by.d) * KEEP_GROUP, here = min(n_cols - c0, KEEP_GROUP);
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {   // (values that do not exist are copies of others of the group)
        const float2 f = v[u].pair(j);
        m = larger_magnitude(m, larger_magnitude(f.x, f.y));
      }
      uint32_t top = __float_as_uint(m);
#pragma unroll
      for (int o = 1; o < 8; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const uint32_t byte = keep_scale_byte<FORMAT>(top);
      const float inverse = keep_scale_inverse(byte);
      const bool cut = __any_sync(0xffffffffu, keep_needs_cut<FORMAT>(top));
      uint32_t q[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = byte == 255u ? 0u : keep_encode2<FORMAT>(v[u].pair(j), inverse, cut);
      if (wanted >= n) continue;
      uint8_t* const out = codes + row * n_cols + c0;
      if constexpr (!FAST) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (s + 8 * j < here) out[s + 8 * j] = (uint8_t)(q[j / 2] >> (8 * (j % 2)));
      } else if constexpr (sizeof(IO) == 2) {
        if (8 * s < here) *reinterpret_cast<uint2*>(out + 8 * s) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
      } else {
        if (4 * s < here) *reinterpret_cast<uint32_t*>(out + 4 * s) = q[0] | q[1] << 16;
        if (32 + 4 * s < here) *reinterpret_cast<uint32_t*>(out + 32 + 4 * s) = q[2] | q[3] << 16;
      }
      if (s == 0) scales[g] = (uint8_t)byte;
    }
  }
}
template <typename IO, int FORMAT, bool FAST>
__global__ void __launch_bounds__(32 * PACK_WARPS, 3) activation_unpack_kernel(const uint8_t* codes, const uint8_t* scales, int64_t n_rows,
                                                                               int n_cols, Divisor by, IO* values, int64_t stride) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = lane % 8;
  const int64_t n = n_rows * by.d, step = (int64_t)gridDim.x * PACK_WARPS * 4 * PACK_UNROLL;
  for (int64_t first = ((int64_t)blockIdx.x * PACK_WARPS + warp) * 4 * PACK_UNROLL; first < n; first += step) {
    uint32_t q[PACK_UNROLL][4], byte[PACK_UNROLL];
#pragma unroll
    for (int u = 0; u < PACK_UNROLL; ++u) {
      const int64_t g = min(first + 4 * u + lane / 8, n - 1), row = by.quotient(g);
      const int c0 = (int)(g - row * by.d) * KEEP_GROUP, here = min(n_cols - c0, KEEP_GROUP);
      const uint8_t* const in = codes + row * n_cols + c0;
      if constexpr (!FAST) {
#pragma unroll
        for (int j = 0; j < 4; ++j) q[u][j] = (uint32_t)in[min(s + 16 * j, here - 1)] | (uint32_t)in[min(s + 16 * j + 8, here - 1)] << 8;
      } else {
        uint2 w;
        if constexpr (sizeof(IO) == 2) {
          w = *reinterpret_cast<const uint2*>(in + (8 * s < here ? 8 * s : 0));
        } else {
          w.x = *reinterpret_cast<const uint32_t*>(in + (4 * s < here ? 4 * s : 0));
          w.y = *reinterpret_cast<const uint32_t*>(in + (32 + 4 * s < here ? 32 + 4 * s : 0));
        }
        q[u][0] = w.x & 0xffffu, q[u][1] = w.x >> 16, q[u][2] = w.y & 0xffffu, q[u][3] = w.y >> 16;
      }
      byte[u] = scales[g];
    }
#pragma unroll
    for (int u = 0; u < PACK_UNROLL; ++u) {
      const int64_t wanted = first + 4 * u + lane / 8, g = min(wanted, n - 1), row = by.quotient(g);
      const int c0 = (int)(g - row * by.d) * KEEP_GROUP, here = min(n_cols - c0, KEEP_GROUP);
      const float scale = keep_scale_value(byte[u]);
      if (wanted >= n) continue;
      IO* const out = values + row * stride + c0;
      float2 f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = keep_decode2<IO, FORMAT>(q[u][j], scale);
      if constexpr (!FAST) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (s + 8 * j < here) out[s + 8 * j] = from_f32<IO>(j % 2 ? f[j / 2].y : f[j / 2].x);
      } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(IO) / 2; ++i) {
          Sixteen<IO> r;
#pragma unroll
          for (int h = 0; h < 8 / (int)sizeof(IO); ++h) set_raw(r.v[h], f[i * (8 / (int)sizeof(IO)) + h]);
          const int at = place<IO, true>(s, i * (16 / (int)sizeof(IO)));
          if (at < here) *reinterpret_cast<Sixteen<IO>*>(out + at) = r;
        }
      }
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
// the kernels' template arguments: the value type, and whether the fast path's alignment holds
template <typename F> snn_status by_dtype(int dtype, bool pairs, F&& f) {
  if (dtype == SNN_DTYPE_FP32) return pairs ? f(float(), std::true_type()) : f(float(), std::false_type());
  if (dtype == SNN_DTYPE_BF16) return pairs ? f(__nv_bfloat16(), std::true_type()) : f(__nv_bfloat16(), std::false_type());
  return pairs ? f(__half(), std::true_type()) : f(__half(), std::false_type());
}

constexpr int32_t WIDEST = INT32_MAX - (KEEP_GROUP - 1);   // a row's last group ends within 32 bits
// whether rows can be accessed 16 bytes of values, or eight codes, at a time
bool rows_of_sixteen(const void* values, int n_cols, int64_t row_stride, const uint8_t* codes) {
  return n_cols % 8 == 0 && row_stride % 8 == 0 && (uintptr_t)values % 16 == 0 && (uintptr_t)codes % 8 == 0;
}
Divisor divisor_of(int n_cols) {
  const int d = (n_cols + KEEP_GROUP - 1) / KEEP_GROUP;
  return {d == 1 ? 0 : ~(uint64_t)0 / d + 1, d};
}
// three blocks fit an SM
unsigned pack_blocks(int64_t n_rows, int n_cols) {
  const int64_t groups = n_rows * ((n_cols + KEEP_GROUP - 1) / KEEP_GROUP), per_block = PACK_WARPS * PACK_UNROLL * 4;
  return (unsigned)std::min<int64_t>((groups + per_block - 1) / per_block, 148 * 3);
}
}  // namespace

extern "C" snn_status snn_activation_pack(const void* values, int32_t dtype, int64_t n_rows, int32_t n_cols, int64_t row_stride,
                                          int32_t format, uint8_t* codes, uint8_t* scales, void* stream) {
  if (n_rows < 0 || n_cols < 0 || !dtype_known(dtype) || (format != SNN_KEEP_INT8 && format != SNN_KEEP_E4M3)) return SNN_ERR_INVALID_ARG;
  if (n_cols > WIDEST) return SNN_ERR_UNSUPPORTED;
  if (n_rows == 0 || n_cols == 0) return SNN_OK;
  if (!values || !codes || !scales) return SNN_ERR_INVALID_ARG;
  return by_dtype(dtype, rows_of_sixteen(values, n_cols, row_stride, codes), [&](auto io, auto is_fast) {
    using IO = decltype(io);
    constexpr bool FAST = decltype(is_fast)::value;
    const auto kernel = format == SNN_KEEP_INT8 ? activation_pack_kernel<IO, SNN_KEEP_INT8, FAST> : activation_pack_kernel<IO, SNN_KEEP_E4M3, FAST>;
    kernel<<<pack_blocks(n_rows, n_cols), 32 * PACK_WARPS, 0, (cudaStream_t)stream>>>((const IO*)values, n_rows, n_cols, row_stride, divisor_of(n_cols), codes, scales);
    return launched();
  });
}

extern "C" snn_status snn_activation_unpack(const uint8_t* codes, const uint8_t* scales, int32_t format, int64_t n_rows, int32_t n_cols,
                                            void* values, int32_t dtype, int64_t row_stride, void* stream) {
  if (n_rows < 0 || n_cols < 0 || !dtype_known(dtype) || (format != SNN_KEEP_INT8 && format != SNN_KEEP_E4M3)) return SNN_ERR_INVALID_ARG;
  if (n_cols > WIDEST) return SNN_ERR_UNSUPPORTED;
  if (n_rows == 0 || n_cols == 0) return SNN_OK;
  if (!values || !codes || !scales) return SNN_ERR_INVALID_ARG;
  return by_dtype(dtype, rows_of_sixteen(values, n_cols, row_stride, codes), [&](auto io, auto is_fast) {
    using IO = decltype(io);
    constexpr bool FAST = decltype(is_fast)::value;
    const auto kernel = format == SNN_KEEP_INT8 ? activation_unpack_kernel<IO, SNN_KEEP_INT8, FAST> : activation_unpack_kernel<IO, SNN_KEEP_E4M3, FAST>;
    kernel<<<pack_blocks(n_rows, n_cols), 32 * PACK_WARPS, 0, (cudaStream_t)stream>>>(codes, scales, n_rows, n_cols, divisor_of(n_cols), (IO*)values, row_stride);
    return launched();
  });
}
