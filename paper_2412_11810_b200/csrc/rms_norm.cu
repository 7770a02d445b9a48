// Root-mean-square norm with the residual's addition (include/snn.h, "sequence-model operators").
//
//   h = x + residual, rounded to the type;  s = 1 / sqrt(mean(h^2) + eps);  y = h s w
//   with g = dy w, c = mean(g h s):  dx = s (g - h s c) + dh,  dw = sum over the rows of dy h s
//
// Bound by HBM: every value is read and written once.  A row belongs to `lanes` threads (8, 16, 32, or whole warps) that hold
// one or two octets each in registers, so that the second use of h costs no second read.  Up to 32 lanes a warp handles whole
// rows and nothing waits for a block.  Rows that do not fit (16384 columns forward, 8192 backward, where dy, dh and the sums
// for dw are held as well) are read a second time, from L2.
#include <algorithm>
#include <type_traits>

#include "octet.cuh"

using namespace snnk;

namespace {

constexpr int RMS_THREADS = 256;      // of a block whose rows need no more than a warp
constexpr int RMS_MOST_LANES = 1024, RMS_MOST_LANES_BACK = 512;

struct RmsParams {
  int64_t rows;
  int n, lanes, keep_format;
  float eps, inverse_n;
  const void *x, *residual, *weight, *dy, *dh;
  int64_t x_stride, residual_stride, h_stride, y_stride, dy_stride, dh_stride, dx_stride;
  void *h, *y, *dx;
  float* rstd;
  uint8_t *codes, *scales;
  float* partial;                     // [blocks][n]: each block's share of dw
};

// The sum over the lanes of a row, the same bits for all of them.  `turn` counts the calls: two buffers take turns, so that
// one barrier a call is enough.
__device__ __forceinline__ float row_sum(float v, int lanes, int turn, float (*shared)[32]) {
  for (int o = 1; o < min(lanes, 32); o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lanes <= 32) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) shared[turn & 1][warp] = v;
  __syncthreads();
  v = lane < lanes / 32 ? shared[turn & 1][lane] : 0.f;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float scale_of(float sum, const RmsParams& p) { return rsqrtf(sum * p.inverse_n + p.eps); }
// Where squares leave the range of fp32 they are summed again of values times 2^-80: that of the largest row is finite, and
// eps, at most one, is nothing beside it.  An infinity in the row leaves a scale of zero, NaN a NaN.
constexpr float RMS_DOWN = 0x1p-80f;
__device__ __forceinline__ float scale_of_far(float sum, const RmsParams& p) { return rsqrtf(sum * p.inverse_n) * RMS_DOWN; }

// The 8-bit codes of an octet y of the group at column c0 of a row.
template <int FORMAT, bool FAST>
__device__ __forceinline__ void keep_octet(const float2 y[4], int64_t row, int c0, int s, const RmsParams& p, bool store) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = larger_magnitude(m, larger_magnitude(y[i].x, y[i].y));
  const uint32_t top = group_top(m), byte = keep_scale_byte<FORMAT>(top);
  const float inverse = keep_scale_inverse(byte);
  const bool cut = __any_sync(0xffffffffu, keep_needs_cut<FORMAT>(top));
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = byte == 255u ? 0u : keep_encode2<FORMAT>(y[i], inverse, cut);
  if (!store) return;
  store_codes<FAST>(p.codes + row * p.n, c0, s, p.n, q);
  if (s == 0 && c0 < p.n) p.scales[row * ((p.n + KEEP_GROUP - 1) / KEEP_GROUP) + c0 / KEEP_GROUP] = (uint8_t)byte;
}

// y of one octet of h, as values, as codes, or both.
template <typename IO, typename WT, bool FAST>
__device__ __forceinline__ void finish_octet(const Octet<IO, FAST>& h, float scale, int64_t row, int c0, int s, const RmsParams& p, bool store) {
  float2 y[4];
  if (p.weight) {
    Octet<WT, FAST> w;
    w.load((const WT*)p.weight, c0, s, p.n);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = mul2(mul2(h.pair(i), both(scale)), w.pair(i));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = mul2(h.pair(i), both(scale));
  }
  if (p.y) {
    Octet<IO, FAST> out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out.set(i, y[i]);
    if (store) out.store((IO*)p.y + row * p.y_stride, c0, s, p.n);
  }
  if (p.keep_format == SNN_KEEP_INT8) keep_octet<SNN_KEEP_INT8, FAST>(y, row, c0, s, p, store);
  if (p.keep_format == SNN_KEEP_E4M3) keep_octet<SNN_KEEP_E4M3, FAST>(y, row, c0, s, p, store);
}
// An octet of h: that of x, or its sum with the residual's, which is stored.
template <typename IO, bool FAST>
__device__ __forceinline__ void sum_octet(Octet<IO, FAST>& h, const Octet<IO, FAST>& r, int64_t row, int c0, int s, const RmsParams& p, bool store) {
  if (!p.residual) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) h.set(i, add2(h.pair(i), r.pair(i)));
  if (store) h.store((IO*)p.h + row * p.h_stride, c0, s, p.n);
}

template <typename IO, typename WT, bool FAST, int OCTETS>
__global__ void __launch_bounds__(RMS_MOST_LANES) rms_forward_kernel(const RmsParams p) {
  __shared__ float shared[2][32];
  const int slot = threadIdx.x / p.lanes, t = threadIdx.x % p.lanes, s = t & 7, per_block = blockDim.x / p.lanes;
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * per_block; base < p.rows; base += (int64_t)gridDim.x * per_block) {
    const bool store = base + slot < p.rows;   // (a slot without a row repeats the last one and stores nothing)
    const int64_t row = min(base + slot, p.rows - 1);
    Octet<IO, FAST> h[OCTETS], r[OCTETS];
#pragma unroll
    for (int o = 0; o < OCTETS; ++o) h[o].load((const IO*)p.x + row * p.x_stride, (t / 8 + o * (p.lanes / 8)) * KEEP_GROUP, s, p.n);
    if (p.residual) {
#pragma unroll
      for (int o = 0; o < OCTETS; ++o) r[o].load((const IO*)p.residual + row * p.residual_stride, (t / 8 + o * (p.lanes / 8)) * KEEP_GROUP, s, p.n);
    }
    float2 sum = both(0.f);
#pragma unroll
    for (int o = 0; o < OCTETS; ++o) {
      sum_octet<IO, FAST>(h[o], r[o], row, (t / 8 + o * (p.lanes / 8)) * KEEP_GROUP, s, p, store);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = fma2(h[o].pair(i), h[o].pair(i), sum);
    }
    float total = row_sum(sum.x + sum.y, p.lanes, turn++, shared), scale = scale_of(total, p);
    // (lanes of one warp may hold different rows: they all go the same way, as do all threads of a row's warps)
    const bool far = !(total <= largest_finite<float>());
    if (p.lanes > 32 ? far : __any_sync(0xffffffffu, far)) {
      sum = both(0.f);
#pragma unroll
      for (int o = 0; o < OCTETS; ++o) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 v = mul2(h[o].pair(i), both(RMS_DOWN));
          sum = fma2(v, v, sum);
        }
      }
      total = row_sum(sum.x + sum.y, p.lanes, turn++, shared);
      if (far) scale = scale_of_far(total, p);
    }
    if (p.rstd && t == 0 && store) p.rstd[row] = scale;
#pragma unroll
    for (int o = 0; o < OCTETS; ++o) finish_octet<IO, WT, FAST>(h[o], scale, row, (t / 8 + o * (p.lanes / 8)) * KEEP_GROUP, s, p, store);
  }
}
// A block per row, which is read twice.
template <typename IO, typename WT, bool FAST>
__global__ void __launch_bounds__(RMS_MOST_LANES) rms_forward_wide_kernel(const RmsParams p) {
  __shared__ float shared[2][32];
  const int t = threadIdx.x, s = t & 7, groups = (p.n + KEEP_GROUP - 1) / KEEP_GROUP, rounds = (groups + RMS_MOST_LANES / 8 - 1) / (RMS_MOST_LANES / 8);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const IO* const from = (const IO*)p.x + row * p.x_stride;
    const IO* const again = p.residual ? (const IO*)p.h + row * p.h_stride : from;
    float2 sum = both(0.f);
    for (int o = 0; o < rounds; ++o) {
      const int64_t c = (int64_t)(t / 8 + o * (RMS_MOST_LANES / 8)) * KEEP_GROUP;
      const int c0 = (int)min(c, (int64_t)p.n);
      Octet<IO, FAST> h, r;
      h.load(from, c0, s, p.n);
      if (p.residual) r.load((const IO*)p.residual + row * p.residual_stride, c0, s, p.n);
      sum_octet<IO, FAST>(h, r, row, c0, s, p, true);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = fma2(h.pair(i), h.pair(i), sum);
    }
    float total = row_sum(sum.x + sum.y, RMS_MOST_LANES, turn++, shared), scale = scale_of(total, p);
    if (!(total <= largest_finite<float>())) {
      sum = both(0.f);
      for (int o = 0; o < rounds; ++o) {
        const int c0 = (int)min((int64_t)(t / 8 + o * (RMS_MOST_LANES / 8)) * KEEP_GROUP, (int64_t)p.n);
        Octet<IO, FAST> h;
        h.load(again, c0, s, p.n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 v = mul2(h.pair(i), both(RMS_DOWN));
          sum = fma2(v, v, sum);
        }
      }
      scale = scale_of_far(row_sum(sum.x + sum.y, RMS_MOST_LANES, turn++, shared), p);
    }
    if (p.rstd && t == 0) p.rstd[row] = scale;
    for (int o = 0; o < rounds; ++o) {   // (a thread reads back what it stored itself)
      const int c0 = (int)min((int64_t)(t / 8 + o * (RMS_MOST_LANES / 8)) * KEEP_GROUP, (int64_t)p.n);
      Octet<IO, FAST> h;
      h.load(again, c0, s, p.n);
      finish_octet<IO, WT, FAST>(h, scale, row, c0, s, p, true);
    }
  }
}

// n = h s and g = dy w of pair i of an octet.
template <typename IO, typename WT, bool FAST>
__device__ __forceinline__ float2 weighted(const Octet<IO, FAST>& dy, const Octet<WT, FAST>& w, bool has_weight, int i) {
  return has_weight ? mul2(dy.pair(i), w.pair(i)) : dy.pair(i);
}

template <typename IO, typename WT, bool FAST, int OCTETS>
__global__ void __launch_bounds__(RMS_MOST_LANES_BACK) rms_backward_kernel(const RmsParams p) {
  __shared__ float shared[2][32];
  __shared__ float dw_shared[32 * OCTETS * 8];   // rows within a warp only
  let_next_kernel_start();
  const int slot = threadIdx.x / p.lanes, t = threadIdx.x % p.lanes, s = t & 7, per_block = blockDim.x / p.lanes;
  const int64_t step = (int64_t)gridDim.x * per_block;
  int turn = 0;
  float2 dw[OCTETS][4];
#pragma unroll
  for (int o = 0; o < OCTETS; ++o)
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[o][i] = both(0.f);
  auto column = [&](int o) { return (t / 8 + o * (p.lanes / 8)) * KEEP_GROUP; };
  for (int64_t base = (int64_t)blockIdx.x * per_block; base < p.rows; base += step) {
    const bool mine = base + slot < p.rows;
    const int64_t row = min(base + slot, p.rows - 1);
    Octet<IO, FAST> h[OCTETS], dy[OCTETS], dh[OCTETS];
#pragma unroll
    for (int o = 0; o < OCTETS; ++o) {
      h[o].load((const IO*)p.h + row * p.h_stride, column(o), s, p.n);
      dy[o].load((const IO*)p.dy + row * p.dy_stride, column(o), s, p.n);
      if (p.dh) dh[o].load((const IO*)p.dh + row * p.dh_stride, column(o), s, p.n);
    }
    const float scale = p.rstd[row];
    float2 sum = both(0.f);
#pragma unroll
    for (int o = 0; o < OCTETS; ++o) {
      Octet<WT, FAST> w;
      if (p.weight) w.load((const WT*)p.weight, column(o), s, p.n);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 n = mul2(h[o].pair(i), both(scale));
        sum = fma2(weighted(dy[o], w, p.weight != nullptr, i), n, sum);
        if (mine) dw[o][i] = fma2(dy[o].pair(i), n, dw[o][i]);
      }
    }
    const float c = row_sum(sum.x + sum.y, p.lanes, turn++, shared) * p.inverse_n;
#pragma unroll
    for (int o = 0; o < OCTETS; ++o) {
      Octet<WT, FAST> w;
      if (p.weight) w.load((const WT*)p.weight, column(o), s, p.n);
      Octet<IO, FAST> out;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 n = mul2(h[o].pair(i), both(scale));
        float2 v = mul2(fma2(n, both(-c), weighted(dy[o], w, p.weight != nullptr, i)), both(scale));
        if (p.dh) v = add2(v, dh[o].pair(i));
        out.set(i, v);
      }
      if (mine) out.store((IO*)p.dx + row * p.dx_stride, column(o), s, p.n);
    }
  }
  if (!p.partial) return;
  float* const to = p.partial + (int64_t)blockIdx.x * p.n;
  if (p.lanes > 32) {
#pragma unroll
    for (int o = 0; o < OCTETS; ++o)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = column(o) + octet_place<FAST>(s, j);
        if (at < p.n) to[at] = j % 2 ? dw[o][j / 2].y : dw[o][j / 2].x;
      }
    return;
  }
  // the rows of a block one behind the other
  for (int k = 0; k < per_block; ++k) {
    if (slot == k) {
#pragma unroll
      for (int o = 0; o < OCTETS; ++o)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = column(o) + octet_place<FAST>(s, j);
          const float v = j % 2 ? dw[o][j / 2].y : dw[o][j / 2].x;
          dw_shared[at] = k == 0 ? v : dw_shared[at] + v;
        }
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < p.n; i += blockDim.x) to[i] = dw_shared[i];
}
template <typename IO, typename WT, bool FAST>
__global__ void __launch_bounds__(RMS_MOST_LANES) rms_backward_wide_kernel(const RmsParams p) {
  __shared__ float shared[2][32];
  const int t = threadIdx.x, s = t & 7, groups = (p.n + KEEP_GROUP - 1) / KEEP_GROUP, rounds = (groups + RMS_MOST_LANES / 8 - 1) / (RMS_MOST_LANES / 8);
  int turn = 0;
  float* const to = p.partial ? p.partial + (int64_t)blockIdx.x * p.n : nullptr;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const float scale = p.rstd[row];
    float2 sum = both(0.f);
    float c = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int o = 0; o < rounds; ++o) {
        const int c0 = (int)min((int64_t)(t / 8 + o * (RMS_MOST_LANES / 8)) * KEEP_GROUP, (int64_t)p.n);
        Octet<IO, FAST> h, dy, dh, out;
        Octet<WT, FAST> w;
        h.load((const IO*)p.h + row * p.h_stride, c0, s, p.n);
        dy.load((const IO*)p.dy + row * p.dy_stride, c0, s, p.n);
        if (p.weight) w.load((const WT*)p.weight, c0, s, p.n);
        if (p.dh && pass) dh.load((const IO*)p.dh + row * p.dh_stride, c0, s, p.n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 n = mul2(h.pair(i), both(scale)), g = weighted(dy, w, p.weight != nullptr, i);
          if (!pass) {
            sum = fma2(g, n, sum);
            continue;
          }
          float2 v = mul2(fma2(n, both(-c), g), both(scale));
          if (p.dh) v = add2(v, dh.pair(i));
          out.set(i, v);
          if (!to) continue;
          const float2 d = mul2(dy.pair(i), n);   // (every place of a block's share belongs to one thread)
          const int at = c0 + octet_place<FAST>(s, 2 * i), next = c0 + octet_place<FAST>(s, 2 * i + 1);
          if (at < p.n) to[at] = row == blockIdx.x ? d.x : to[at] + d.x;
          if (next < p.n) to[next] = row == blockIdx.x ? d.y : to[next] + d.y;
        }
        if (pass) out.store((IO*)p.dx + row * p.dx_stride, c0, s, p.n);
      }
      if (!pass) c = row_sum(sum.x + sum.y, RMS_MOST_LANES, turn++, shared) * p.inverse_n;
    }
  }
}
// dw from the blocks' shares, in their order: 32 columns a block, eight rows of shares at a time.
template <typename WT> __global__ void __launch_bounds__(256) rms_dweight_kernel(const float* partial, int blocks, int n, WT* dw) {
  __shared__ float shared[8][32];
  wait_for_kernel_before();
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  float sum = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int b = y; b < blocks; b += 8) sum += partial[(int64_t)b * n + c];
  }
  shared[y][x] = sum;
  __syncthreads();
  if (y > 0 || c >= n) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) sum += shared[k][x];
  dw[c] = from_f32<WT>(sum);
}

// ---- host ----------------------------------------------------------------------------------------------------
struct Shape {
  int lanes, octets, threads;   // octets 0: rows that do not fit registers
};
Shape shape_of(int n, int most_lanes) {
  const int groups = (n + KEEP_GROUP - 1) / KEEP_GROUP;
  for (int octets = 1; octets <= 2; ++octets) {
    const int need = 8 * ((groups + octets - 1) / octets);
    const int lanes = need > 32 ? (need + 31) / 32 * 32 : need > 16 ? 32 : need;
    if (lanes <= (octets == 1 ? 256 : most_lanes)) return {lanes, octets, lanes > 32 ? lanes : RMS_THREADS};
  }
  return {RMS_MOST_LANES, 0, RMS_MOST_LANES};
}
unsigned blocks_of(const Shape& s, int64_t rows, int per_sm) {
  const int64_t per_block = s.threads / s.lanes, want = (rows + per_block - 1) / per_block;
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(want, (int64_t)148 * per_sm));
}
// blocks of the backward pass: two thousand threads of an SM at most, and no more than rows
unsigned backward_blocks(int n, int64_t rows) {
  const Shape s = shape_of(n, RMS_MOST_LANES_BACK);
  return blocks_of(s, rows, std::max(1, 1024 / s.threads));
}
snn_status check(const snn_rms_norm_args* a) {
  if (!a || a->rows < 0 || a->n < 1 || !dtype_known(a->dtype)) return SNN_ERR_INVALID_ARG;
  if (a->weight_dtype != a->dtype && a->weight_dtype != SNN_DTYPE_FP32) return SNN_ERR_INVALID_ARG;
  if (a->n > INT32_MAX - (KEEP_GROUP - 1)) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}
bool no_overlap(const snn_rms_norm_args* a, int64_t stride) { return a->rows < 2 || stride >= a->n; }
template <typename F> snn_status by_types(int dtype, int weight_dtype, bool fast, F&& f) {
  auto with = [&](auto io, auto wt) { return fast ? f(io, wt, std::true_type()) : f(io, wt, std::false_type()); };
  if (dtype == SNN_DTYPE_FP32) return with(float(), float());
  if (dtype == SNN_DTYPE_BF16) return weight_dtype == SNN_DTYPE_FP32 ? with(__nv_bfloat16(), float()) : with(__nv_bfloat16(), __nv_bfloat16());
  return weight_dtype == SNN_DTYPE_FP32 ? with(__half(), float()) : with(__half(), __half());
}
}  // namespace

extern "C" snn_status snn_rms_norm_workspace(const snn_rms_norm_args* a, size_t* bytes) {
  const snn_status st = check(a);
  if (st != SNN_OK) return st;
  if (!bytes) return SNN_ERR_INVALID_ARG;
  *bytes = a->rows == 0 ? 0 : ((size_t)backward_blocks(a->n, a->rows) * a->n * 4 + 255) / 256 * 256;
  return SNN_OK;
}

extern "C" snn_status snn_rms_norm_forward(const snn_rms_norm_args* a, void* stream) {
  const snn_status st = check(a);
  if (st != SNN_OK) return st;
  if (!(a->eps >= 1e-30f && a->eps <= 1.f)) return SNN_ERR_INVALID_ARG;
  if (a->keep_format != SNN_KEEP_RAW && a->keep_format != SNN_KEEP_INT8 && a->keep_format != SNN_KEEP_E4M3) return SNN_ERR_INVALID_ARG;
  if (a->rows == 0) return SNN_OK;
  const bool keeps = a->keep_format != SNN_KEEP_RAW;
  if (!a->x || (a->residual && !a->h) || (!a->y && !keeps) || (keeps && (!a->codes || !a->scales))) return SNN_ERR_INVALID_ARG;
  if ((a->residual && !no_overlap(a, a->h_stride)) || (a->y && !no_overlap(a, a->y_stride))) return SNN_ERR_INVALID_ARG;
  RmsParams p{};
  const Shape s = shape_of(a->n, RMS_MOST_LANES);
  p.rows = a->rows, p.n = a->n, p.lanes = s.lanes, p.keep_format = a->keep_format, p.eps = a->eps, p.inverse_n = 1.f / (float)a->n;
  p.x = a->x, p.x_stride = a->x_stride, p.residual = a->residual, p.residual_stride = a->residual_stride, p.weight = a->weight;
  p.h = a->h, p.h_stride = a->h_stride, p.y = a->y, p.y_stride = a->y_stride, p.rstd = a->rstd, p.codes = a->codes, p.scales = a->scales;
  const bool fast = a->n % 8 == 0 && octet_rows(a->x, a->x_stride, a->dtype) && octet_rows(a->residual, a->residual_stride, a->dtype) &&
                    octet_rows(a->residual ? a->h : nullptr, a->h_stride, a->dtype) && octet_rows(a->y, a->y_stride, a->dtype) &&
                    octet_rows(a->weight, 0, a->weight_dtype) && (!keeps || aligned_to(a->codes, 8));
  return by_types(a->dtype, a->weight_dtype, fast, [&](auto io, auto wt, auto is_fast) {
    using IO = decltype(io);
    using WT = decltype(wt);
    constexpr bool FAST = decltype(is_fast)::value;
    const auto kernel = s.octets == 0   ? rms_forward_wide_kernel<IO, WT, FAST>
                        : s.octets == 1 ? rms_forward_kernel<IO, WT, FAST, 1>
                        : rms_forward_kernel<IO, WT, FAST, 2>;
    return launch_behind(kernel, blocks_of(s, a->rows, 1 << 16), s.threads, 0, (cudaStream_t)stream, false, p);
  });
}

extern "C" snn_status snn_rms_norm_backward(const snn_rms_norm_args* a, void* stream) {
  const snn_status st = check(a);
  if (st != SNN_OK) return st;
  const cudaStream_t on = (cudaStream_t)stream;
  if (a->rows == 0) {
    if (!a->dweight) return SNN_OK;
    return cudaMemsetAsync(a->dweight, 0, (size_t)a->n * dtype_size(a->weight_dtype), on) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
  }
  if (!a->h || !a->rstd || !a->dy || !a->dx || !no_overlap(a, a->dx_stride)) return SNN_ERR_INVALID_ARG;
  const unsigned blocks = backward_blocks(a->n, a->rows);
  if (a->dweight) {
    if (!a->workspace || !aligned_to(a->workspace, 256)) return SNN_ERR_INVALID_ARG;
    if (a->workspace_bytes < (size_t)blocks * a->n * 4) return SNN_ERR_WORKSPACE_TOO_SMALL;
  }
  RmsParams p{};
  const Shape s = shape_of(a->n, RMS_MOST_LANES_BACK);
  p.rows = a->rows, p.n = a->n, p.lanes = s.lanes, p.inverse_n = 1.f / (float)a->n, p.weight = a->weight;
  p.h = a->h, p.h_stride = a->h_stride, p.rstd = a->rstd, p.dy = a->dy, p.dy_stride = a->dy_stride, p.dh = a->dh, p.dh_stride = a->dh_stride;
  p.dx = a->dx, p.dx_stride = a->dx_stride, p.partial = a->dweight ? (float*)a->workspace : nullptr;
  const bool fast = a->n % 8 == 0 && octet_rows(a->h, a->h_stride, a->dtype) && octet_rows(a->dy, a->dy_stride, a->dtype) &&
                    octet_rows(a->dh, a->dh_stride, a->dtype) && octet_rows(a->dx, a->dx_stride, a->dtype) && octet_rows(a->weight, 0, a->weight_dtype);
  const snn_status done = by_types(a->dtype, a->weight_dtype, fast, [&](auto io, auto wt, auto is_fast) {
    using IO = decltype(io);
    using WT = decltype(wt);
    constexpr bool FAST = decltype(is_fast)::value;
    const auto kernel = s.octets == 0   ? rms_backward_wide_kernel<IO, WT, FAST>
                        : s.octets == 1 ? rms_backward_kernel<IO, WT, FAST, 1>
                        : rms_backward_kernel<IO, WT, FAST, 2>;
    return launch_behind(kernel, blocks, s.threads, 0, on, false, p);
  });
  if (done != SNN_OK || !a->dweight) return done;
  const unsigned tiles = (unsigned)((a->n + 31) / 32);
  if (a->weight_dtype == SNN_DTYPE_FP32) return launch_behind(rms_dweight_kernel<float>, tiles, 256, 0, on, true, p.partial, (int)blocks, a->n, (float*)a->dweight);
  if (a->weight_dtype == SNN_DTYPE_BF16)
    return launch_behind(rms_dweight_kernel<__nv_bfloat16>, tiles, 256, 0, on, true, p.partial, (int)blocks, a->n, (__nv_bfloat16*)a->dweight);
  return launch_behind(rms_dweight_kernel<__half>, tiles, 256, 0, on, true, p.partial, (int)blocks, a->n, (__half*)a->dweight);
}
