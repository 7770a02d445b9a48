// The gated linear recurrence with its backward pass, and activations in 8 bits (include/snn.h, "sequence-model
// operators").
//
// A step is an affine map of the state, h -> a h + b, and maps compose: (a2, b2) o (a1, b1) = (a2 a1, a2 b1 + b2).  So a
// run of steps can be summarised before its start is known, and time is split three ways: a thread takes 8 steps of two
// neighbouring channels in registers, the 8 warps of a thread block a chunk of 64 steps, the blocks of a cluster (1..8)
// neighbouring chunks.  Warps exchange their summaries through shared memory, blocks through distributed shared memory
// behind one hardware cluster barrier per turn; the state at the end of a turn is carried to the next one in registers.
// Every input is read once, every output written once, nothing waits on a flag in memory, and the order of the
// arithmetic is fixed by the sizes alone.  The kernels are bound by HBM; the cluster size only has to supply enough
// blocks for it when there are few channels.
#include <cooperative_groups.h>

#include <algorithm>

#include "seq_common.cuh"

namespace cg = cooperative_groups;
using namespace snnk;

namespace {

constexpr int SCAN_K = 8;                       // steps per thread
constexpr int SCAN_WARPS = 8;
constexpr int SCAN_THREADS = 32 * SCAN_WARPS;
constexpr int SCAN_COLS = 64;                   // channels per thread block, two per lane: one group of the 8-bit format
constexpr int SCAN_MAX_CLUSTER = 8;
constexpr int SCAN_SHORT = 16;                  // up to so many steps a thread simply walks through them
static_assert(SCAN_K * SCAN_WARPS == SNN_SCAN_CHUNK, "a thread block's run of steps is a chunk");
static_assert(SCAN_COLS == KEEP_GROUP, "a warp encodes one group at a time");

struct ScanParams {
  int T, B, N, n_tiles;      // n_tiles: column tiles per sample
  int mode, x_format, gate_format;
  bool vec_in, vec_dh, vec_out, vec_codes, vec_x, vec_gate;
  const void *x, *gate, *dh;
  void *h, *dx, *dgate;
  int64_t xs[2], gs[2], hs[2], dhs[2], dxs[2], dgs[2];
  const int32_t* lengths;
  const float *state, *dlast;
  float *last, *states, *dstate;
  uint8_t *x_codes, *x_scales, *gate_codes, *gate_scales;
};

// a and the factor i of x.  sigmoid(g) and 1 - sigmoid(g) both without cancellation: with e = exp(-|g|), the larger of
// the two is 1 / (1 + e) and the smaller e / (1 + e).
__device__ __forceinline__ void coefficients(float g, int mode, float& a, float& i) {
  if (mode == SNN_SCAN_DIRECT) { a = g; i = 1.f; return; }
  const float e = __expf(-fabsf(g));
  const float large = __fdividef(1.f, 1.f + e), small = e * large;
  a = g >= 0.f ? large : small;
  i = g >= 0.f ? small : large;
  if (g != g) { a = g; i = g; }
}

struct Map2 {   // the affine maps of two channels
  float a0, b0, a1, b1;
};
__device__ __forceinline__ Map2 identity2() { return {1.f, 0.f, 1.f, 0.f}; }
__device__ __forceinline__ float2 apply(const Map2& m, float2 h) { return make_float2(fmaf(m.a0, h.x, m.b0), fmaf(m.a1, h.y, m.b1)); }
__device__ __forceinline__ float4 as4(const Map2& m) { return make_float4(m.a0, m.b0, m.a1, m.b1); }
__device__ __forceinline__ Map2 as_map(float4 v) { return {v.x, v.y, v.z, v.w}; }
__device__ __forceinline__ Map2 then(const Map2& first, const Map2& second) {
  return {first.a0 * second.a0, fmaf(second.a0, first.b0, second.b0), first.a1 * second.a1, fmaf(second.a1, first.b1, second.b1)};
}

__device__ __forceinline__ float2 load_state(const float* p, int64_t row, int N, int c, int n_ok) {
  float2 v = make_float2(0.f, 0.f);
  if (p && n_ok > 0) v.x = p[row * N + c];
  if (p && n_ok > 1) v.y = p[row * N + c + 1];
  return v;
}
__device__ __forceinline__ void store_state(float* p, int64_t row, int N, int c, int n_ok, float2 v) {
  if (p && n_ok > 0) p[row * N + c] = v.x;
  if (p && n_ok > 1) p[row * N + c + 1] = v.y;
}

// Encodes the warp's 64 values of row `row` (two per lane) and stores codes and scale.  Called by whole warps.
__device__ __forceinline__ void keep_row(float2 v, int64_t row, int N, int c, int n_ok, int format, bool vec, uint8_t* codes,
                                         uint8_t* scales) {
  uint32_t top = 0;
  if (n_ok > 0) top = magnitude_bits(v.x);
  if (n_ok > 1) top = max(top, magnitude_bits(v.y));
  top = __reduce_max_sync(0xffffffffu, top);
  const uint32_t byte = keep_scale_byte(top, format);
  const uint32_t pair = byte == 255u ? 0u : keep_encode2(v, keep_scale_inverse(byte), format);
  uint8_t* const at = codes + row * N + c;
  if (n_ok == 2 && vec) {
    *reinterpret_cast<uint16_t*>(at) = (uint16_t)pair;
  } else {
    if (n_ok > 0) at[0] = (uint8_t)(pair & 255u);
    if (n_ok > 1) at[1] = (uint8_t)(pair >> 8);
  }
  if ((threadIdx.x & 31) == 0) scales[row * ((N + KEEP_GROUP - 1) / KEEP_GROUP) + c / KEEP_GROUP] = (uint8_t)byte;
}
template <typename IO>
__device__ __forceinline__ float2 kept_pair(const uint8_t* codes, const uint8_t* scales, int64_t row, int N, int c, int n_ok,
                                            int format, bool vec) {
  if (n_ok == 0) return make_float2(0.f, 0.f);
  const float scale = keep_scale_value(scales[row * ((N + KEEP_GROUP - 1) / KEEP_GROUP) + c / KEEP_GROUP]);
  const uint8_t* const at = codes + row * N + c;
  uint32_t pair;
  if (n_ok == 2 && vec) pair = *reinterpret_cast<const uint16_t*>(at);
  else pair = (uint32_t)at[0] | (n_ok > 1 ? (uint32_t)at[1] << 8 : 0u);
  return keep_decode2<IO>(pair, scale, format);
}

__device__ __forceinline__ int length_of(const ScanParams& p, int b) {
  return p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
}

// Zeros at the steps [t0, T) of two channels, one step per warp of the cluster.
template <typename IO>
__device__ __forceinline__ void zero_steps(const ScanParams& p, IO* out, const int64_t* stride, int b, int c, int n_ok, int t0, int first,
                                           int step) {
  for (int64_t t = (int64_t)t0 + first; t < p.T; t += step)
    store_pair<IO>(out + t * stride[0] + b * stride[1], c, n_ok, p.vec_out, make_float2(0.f, 0.f));
}

// ---- forward -----------------------------------------------------------------------------------------------
template <typename IO, bool KEEP>
__global__ void __launch_bounds__(SCAN_THREADS) scan_forward_kernel(const ScanParams p) {
  __shared__ float4 s_warp[2][SCAN_WARPS][32];
  __shared__ float4 s_block[2][SCAN_MAX_CLUSTER][32];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tile = (int)blockIdx.x / S, b = tile / p.n_tiles, c = (tile % p.n_tiles) * SCAN_COLS + 2 * lane;
  const int n_ok = min(max(p.N - c, 0), 2);
  const int len = length_of(p, b);
  const IO* const x = (const IO*)p.x + b * p.xs[1];
  const IO* const gate = (const IO*)p.gate + b * p.gs[1];
  IO* const h_out = (IO*)p.h + b * p.hs[1];
  float2 carry = load_state(p.state, b, p.N, c, n_ok);
  int buf = 0;
  int64_t turn = 0;
  for (; turn < len; turn += (int64_t)S * SNN_SCAN_CHUNK, buf ^= 1) {
    const int64_t chunk0 = turn + (int64_t)rank * SNN_SCAN_CHUNK, t0 = chunk0 + warp * SCAN_K;
    float2 xv[SCAN_K], gv[SCAN_K];
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      const bool on = t0 + k < len;
      xv[k] = on ? load_pair<IO>(x + (t0 + k) * p.xs[0], c, n_ok, p.vec_in) : make_float2(0.f, 0.f);
      gv[k] = on ? load_pair<IO>(gate + (t0 + k) * p.gs[0], c, n_ok, p.vec_in) : make_float2(0.f, 0.f);
    }
    if (KEEP) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) {
        if (t0 + k < len) {   // the same for the whole warp
          const int64_t row = (t0 + k) * p.B + b;
          if (p.x_format != SNN_KEEP_RAW) keep_row(xv[k], row, p.N, c, n_ok, p.x_format, p.vec_codes, p.x_codes, p.x_scales);
          if (p.gate_format != SNN_KEEP_RAW)
            keep_row(gv[k], row, p.N, c, n_ok, p.gate_format, p.vec_codes, p.gate_codes, p.gate_scales);
        }
      }
    }
    Map2 mine = identity2();
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {   // xv becomes b, gv becomes a
      float a0 = 1.f, a1 = 1.f, i0 = 0.f, i1 = 0.f;
      if (t0 + k < len) {
        coefficients(gv[k].x, p.mode, a0, i0);
        coefficients(gv[k].y, p.mode, a1, i1);
      }
      gv[k] = make_float2(a0, a1);
      xv[k] = make_float2(i0 * xv[k].x, i1 * xv[k].y);
      mine = then(mine, Map2{gv[k].x, xv[k].x, gv[k].y, xv[k].y});
    }
    s_warp[buf][warp][lane] = as4(mine);
    __syncthreads();
    Map2 before = identity2();   // the warps before this one
    for (int w = 0; w < warp; ++w) before = then(before, as_map(s_warp[buf][w][lane]));
    float2 start = carry;        // the state before this block's chunk
    if (S > 1) {
      if (warp == SCAN_WARPS - 1) {
        const float4 all = as4(then(before, mine));
        for (int r = 0; r < S; ++r) cluster.map_shared_rank(&s_block[buf][rank][0], r)[lane] = all;
      }
      cluster.sync();
      for (int r = 0; r < S; ++r) {
        if (r == rank) start = carry;
        carry = apply(as_map(s_block[buf][r][lane]), carry);
      }
    } else {
      Map2 all = before;
      for (int w = warp; w < SCAN_WARPS; ++w) all = then(all, as_map(s_warp[buf][w][lane]));
      carry = apply(all, carry);
    }
    if (KEEP && warp == 0 && chunk0 < len)
      store_state(p.states, (chunk0 / SNN_SCAN_CHUNK) * p.B + b, p.N, c, n_ok, start);
    float2 h = apply(before, start);
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      h.x = fmaf(gv[k].x, h.x, xv[k].x);
      h.y = fmaf(gv[k].y, h.y, xv[k].y);
      if (t0 + k < len) store_pair<IO>(h_out + (t0 + k) * p.hs[0], c, n_ok, p.vec_out, h);
    }
  }
  if (rank == 0 && warp == 0) store_state(p.last, b, p.N, c, n_ok, carry);
  zero_steps<IO>(p, (IO*)p.h, p.hs, b, c, n_ok, len, rank * SCAN_WARPS + warp, S * SCAN_WARPS);
}

// Few steps (the token of a serving loop): a thread takes two channels of one sample through all of them.
template <typename IO>
__global__ void __launch_bounds__(128) scan_short_kernel(const ScanParams p) {
  const int pairs = (p.N + 1) / 2;
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (int64_t)p.B * pairs) return;
  const int b = (int)(i / pairs), c = (int)(i % pairs) * 2, n_ok = min(p.N - c, 2);
  const int len = length_of(p, b);
  const IO* const x = (const IO*)p.x + b * p.xs[1];
  const IO* const gate = (const IO*)p.gate + b * p.gs[1];
  IO* const h_out = (IO*)p.h + b * p.hs[1];
  float2 h = load_state(p.state, b, p.N, c, n_ok);
#pragma unroll 1
  for (int64_t t = 0; t < p.T; ++t) {
    float2 shown = make_float2(0.f, 0.f);
    if (t < len) {
      const float2 xv = load_pair<IO>(x + t * p.xs[0], c, n_ok, p.vec_in), gv = load_pair<IO>(gate + t * p.gs[0], c, n_ok, p.vec_in);
      float a0, a1, i0, i1;
      coefficients(gv.x, p.mode, a0, i0);
      coefficients(gv.y, p.mode, a1, i1);
      h = shown = make_float2(fmaf(a0, h.x, i0 * xv.x), fmaf(a1, h.y, i1 * xv.y));
    }
    store_pair<IO>(h_out + t * p.hs[0], c, n_ok, p.vec_out, shown);
  }
  store_state(p.last, b, p.N, c, n_ok, h);
}

// ---- backward ----------------------------------------------------------------------------------------------
// The quantity handed from step to step is e_t = a_t D_t = a_t (dh_t + e_{t+1}), again an affine map, composed from the
// last step to the first; the states of the chunk are recomputed from its checkpoint by the forward maps.  A block's
// chunk starts at a checkpoint, so only e crosses blocks.
template <typename IO>
__global__ void __launch_bounds__(SCAN_THREADS) scan_backward_kernel(const ScanParams p) {
  __shared__ float4 s_fwd[2][SCAN_WARPS][32];
  __shared__ float4 s_bwd[2][SCAN_WARPS][32];
  __shared__ float4 s_block[2][SCAN_MAX_CLUSTER][32];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tile = (int)blockIdx.x / S, b = tile / p.n_tiles, c = (tile % p.n_tiles) * SCAN_COLS + 2 * lane;
  const int n_ok = min(max(p.N - c, 0), 2);
  const int len = length_of(p, b);
  const IO* const x = (const IO*)p.x + b * p.xs[1];
  const IO* const gate = (const IO*)p.gate + b * p.gs[1];
  const IO* const dh = (const IO*)p.dh + b * p.dhs[1];
  IO* const dx = (IO*)p.dx + b * p.dxs[1];
  IO* const dgate = (IO*)p.dgate + b * p.dgs[1];
  float2 carry = load_state(p.dlast, b, p.N, c, n_ok);   // e behind the turn's last step
  const int64_t per_turn = (int64_t)S * SNN_SCAN_CHUNK;
  int buf = 0;
  for (int64_t turn = (len + per_turn - 1) / per_turn * per_turn - per_turn; turn >= 0; turn -= per_turn, buf ^= 1) {
    const int64_t chunk0 = turn + (int64_t)rank * SNN_SCAN_CHUNK, t0 = chunk0 + warp * SCAN_K;
    float2 xv[SCAN_K], a[SCAN_K], in[SCAN_K], d[SCAN_K];
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      const bool on = t0 + k < len;
      const int64_t row = (t0 + k) * p.B + b;
      const float2 zero = make_float2(0.f, 0.f);
      xv[k] = !on ? zero
              : p.x_format == SNN_KEEP_RAW ? load_pair<IO>(x + (t0 + k) * p.xs[0], c, n_ok, p.vec_x)
                                           : kept_pair<IO>(p.x_codes, p.x_scales, row, p.N, c, n_ok, p.x_format, p.vec_codes);
      a[k] = !on ? zero
             : p.gate_format == SNN_KEEP_RAW ? load_pair<IO>(gate + (t0 + k) * p.gs[0], c, n_ok, p.vec_gate)
                                             : kept_pair<IO>(p.gate_codes, p.gate_scales, row, p.N, c, n_ok, p.gate_format, p.vec_codes);
      d[k] = on ? load_pair<IO>(dh + (t0 + k) * p.dhs[0], c, n_ok, p.vec_dh) : zero;
    }
    const float2 kept = chunk0 < len ? load_state(p.states, (chunk0 / SNN_SCAN_CHUNK) * p.B + b, p.N, c, n_ok) : make_float2(0.f, 0.f);
    Map2 forth = identity2(), back = identity2();
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      float a0 = 1.f, a1 = 1.f, i0 = 0.f, i1 = 0.f;
      if (t0 + k < len) {
        coefficients(a[k].x, p.mode, a0, i0);
        coefficients(a[k].y, p.mode, a1, i1);
      }
      a[k] = make_float2(a0, a1);
      in[k] = make_float2(i0, i1);
      forth = then(forth, Map2{a0, i0 * xv[k].x, a1, i1 * xv[k].y});
    }
#pragma unroll
    for (int k = SCAN_K - 1; k >= 0; --k) back = then(back, Map2{a[k].x, a[k].x * d[k].x, a[k].y, a[k].y * d[k].y});
    s_fwd[buf][warp][lane] = as4(forth);
    s_bwd[buf][warp][lane] = as4(back);
    __syncthreads();
    float2 h = kept;
    for (int w = 0; w < warp; ++w) h = apply(as_map(s_fwd[buf][w][lane]), h);
    Map2 behind = identity2();   // the later warps of this block
    for (int w = SCAN_WARPS - 1; w > warp; --w) behind = then(behind, as_map(s_bwd[buf][w][lane]));
    float2 start = carry;        // e behind this block's chunk
    if (S > 1) {
      if (warp == 0) {
        const float4 all = as4(then(behind, back));
        for (int r = 0; r < S; ++r) cluster.map_shared_rank(&s_block[buf][rank][0], r)[lane] = all;
      }
      cluster.sync();
      for (int r = S - 1; r >= 0; --r) {
        if (r == rank) start = carry;
        carry = apply(as_map(s_block[buf][r][lane]), carry);
      }
    } else {
      Map2 all = behind;
      for (int w = warp; w >= 0; --w) all = then(all, as_map(s_bwd[buf][w][lane]));
      carry = apply(all, carry);
    }
    float2 e = apply(behind, start);
#pragma unroll
    for (int k = SCAN_K - 1; k >= 0; --k) {   // d becomes D
      d[k] = make_float2(d[k].x + e.x, d[k].y + e.y);
      e = make_float2(a[k].x * d[k].x, a[k].y * d[k].y);
    }
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      if (t0 + k < len) {
        float2 gx = d[k], gg;
        if (p.mode == SNN_SCAN_DIRECT) {
          gg = make_float2(d[k].x * h.x, d[k].y * h.y);
        } else {
          gx = make_float2(d[k].x * in[k].x, d[k].y * in[k].y);
          gg = make_float2(gx.x * a[k].x * (h.x - xv[k].x), gx.y * a[k].y * (h.y - xv[k].y));
        }
        store_pair<IO>(dx + (t0 + k) * p.dxs[0], c, n_ok, p.vec_out, gx);
        store_pair<IO>(dgate + (t0 + k) * p.dgs[0], c, n_ok, p.vec_out, gg);
        h = make_float2(fmaf(a[k].x, h.x, in[k].x * xv[k].x), fmaf(a[k].y, h.y, in[k].y * xv[k].y));
      }
    }
  }
  if (rank == 0 && warp == 0) store_state(p.dstate, b, p.N, c, n_ok, carry);
  zero_steps<IO>(p, (IO*)p.dx, p.dxs, b, c, n_ok, len, rank * SCAN_WARPS + warp, S * SCAN_WARPS);
  zero_steps<IO>(p, (IO*)p.dgate, p.dgs, b, c, n_ok, len, rank * SCAN_WARPS + warp, S * SCAN_WARPS);
}

// ---- 8-bit activations on their own --------------------------------------------------------------------------
// A warp takes one group of 64 values at a time; bound by HBM (bytes of a value + 1).
constexpr int PACK_WARPS = 8;
template <typename IO>
__global__ void __launch_bounds__(32 * PACK_WARPS) activation_pack_kernel(const IO* values, int64_t n_rows, int n_cols, int64_t stride,
                                                                          int format, bool vec, bool vec_codes, uint8_t* codes,
                                                                          uint8_t* scales) {
  const int lane = threadIdx.x & 31;
  const int groups = (n_cols + KEEP_GROUP - 1) / KEEP_GROUP;
  const int64_t n = n_rows * groups, step = (int64_t)gridDim.x * PACK_WARPS;
  for (int64_t i = (int64_t)blockIdx.x * PACK_WARPS + (threadIdx.x >> 5); i < n; i += step) {
    const int64_t row = i / groups;
    const int c = (int)(i % groups) * KEEP_GROUP + 2 * lane, n_ok = min(max(n_cols - c, 0), 2);
    keep_row(load_pair<IO>(values + row * stride, c, n_ok, vec), row, n_cols, c, n_ok, format, vec_codes, codes, scales);
  }
}
template <typename IO>
__global__ void __launch_bounds__(32 * PACK_WARPS) activation_unpack_kernel(const uint8_t* codes, const uint8_t* scales, int format,
                                                                            int64_t n_rows, int n_cols, IO* values, int64_t stride,
                                                                            bool vec, bool vec_codes) {
  const int lane = threadIdx.x & 31;
  const int groups = (n_cols + KEEP_GROUP - 1) / KEEP_GROUP;
  const int64_t n = n_rows * groups, step = (int64_t)gridDim.x * PACK_WARPS;
  for (int64_t i = (int64_t)blockIdx.x * PACK_WARPS + (threadIdx.x >> 5); i < n; i += step) {
    const int64_t row = i / groups;
    const int c = (int)(i % groups) * KEEP_GROUP + 2 * lane, n_ok = min(max(n_cols - c, 0), 2);
    store_pair<IO>(values + row * stride, c, n_ok, vec, kept_pair<IO>(codes, scales, row, n_cols, c, n_ok, format, vec_codes));
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
size_t dtype_size(int dtype) { return dtype == SNN_DTYPE_FP32 ? 4 : 2; }
bool dtype_known(int dtype) { return dtype >= SNN_DTYPE_FP32 && dtype <= SNN_DTYPE_FP16; }
// whether pairs of values can be accessed at once: even offsets everywhere
bool pairs_aligned(const void* p, int dtype, int64_t s0, int64_t s1) {
  return (uintptr_t)p % (2 * dtype_size(dtype)) == 0 && s0 % 2 == 0 && s1 % 2 == 0;
}
bool aligned2(const void* p) { return (uintptr_t)p % 2 == 0; }
// a value type for the kernels' templates
template <typename F> snn_status by_dtype(int dtype, F&& f) {
  if (dtype == SNN_DTYPE_FP32) return f(float());
  if (dtype == SNN_DTYPE_BF16) return f(__nv_bfloat16());
  return f(__half());
}

snn_status check_common(const snn_scan_args* a) {
  if (!a || a->T < 0 || a->B < 0 || a->N < 0 || a->T >= (1 << 30) || !dtype_known(a->dtype)) return SNN_ERR_INVALID_ARG;
  if (a->mode != SNN_SCAN_SIGMOID && a->mode != SNN_SCAN_DIRECT) return SNN_ERR_INVALID_ARG;
  for (int f : {a->x_format, a->gate_format})
    if (f < SNN_KEEP_RAW || f > SNN_KEEP_E4M3) return SNN_ERR_INVALID_ARG;
  if (a->mode == SNN_SCAN_DIRECT && a->gate_format != SNN_KEEP_RAW) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}
ScanParams params_of(const snn_scan_args* a) {
  ScanParams p{};
  p.T = a->T; p.B = a->B; p.N = a->N;
  p.n_tiles = (a->N + SCAN_COLS - 1) / SCAN_COLS;
  p.mode = a->mode; p.x_format = a->x_format; p.gate_format = a->gate_format;
  p.x = a->x; p.gate = a->gate; p.dh = a->dh; p.h = a->h; p.dx = a->dx; p.dgate = a->dgate;
  for (int i = 0; i < 2; ++i) {
    p.xs[i] = a->x_stride[i]; p.gs[i] = a->gate_stride[i]; p.hs[i] = a->h_stride[i];
    p.dhs[i] = a->dh_stride[i]; p.dxs[i] = a->dx_stride[i]; p.dgs[i] = a->dgate_stride[i];
  }
  p.lengths = a->lengths; p.state = a->state; p.dlast = a->dlast; p.last = a->last; p.states = a->states; p.dstate = a->dstate;
  p.x_codes = a->x_codes; p.x_scales = a->x_scales; p.gate_codes = a->gate_codes; p.gate_scales = a->gate_scales;
  p.vec_x = pairs_aligned(p.x, a->dtype, p.xs[0], p.xs[1]);
  p.vec_gate = pairs_aligned(p.gate, a->dtype, p.gs[0], p.gs[1]);
  p.vec_in = p.vec_x && p.vec_gate;
  p.vec_dh = pairs_aligned(p.dh, a->dtype, p.dhs[0], p.dhs[1]);
  p.vec_codes = a->N % 2 == 0 && aligned2(p.x_codes) && aligned2(p.gate_codes);
  return p;
}
// Blocks per column tile: enough for four blocks on each of 148 SMs, no more than there are chunks.
int cluster_of(int64_t tiles, int T) {
  int S = 1;
  while (S < SCAN_MAX_CLUSTER && tiles * S < 4 * 148 && (int64_t)S * SNN_SCAN_CHUNK < T) S *= 2;
  return S;
}
template <typename K> snn_status launch_clusters(K kernel, const ScanParams& p, cudaStream_t stream) {
  const int64_t tiles = (int64_t)p.B * p.n_tiles;
  const int S = cluster_of(tiles, p.T);
  if (tiles * S > INT32_MAX) return SNN_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(tiles * S));
  cfg.blockDim = dim3(SCAN_THREADS);
  cfg.stream = stream;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = (unsigned)S;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
}
snn_status launched() { return cudaGetLastError() == cudaSuccess ? SNN_OK : SNN_ERR_CUDA; }

}  // namespace

extern "C" snn_status snn_scan_forward(const snn_scan_args* a, void* stream) {
  const snn_status st = check_common(a);
  if (st != SNN_OK) return st;
  const bool keep = a->states != nullptr && a->T > 0;
  if (a->B == 0 || a->N == 0) return SNN_OK;
  if (a->T > 0) {
    if (!keep && (a->x_format != SNN_KEEP_RAW || a->gate_format != SNN_KEEP_RAW)) return SNN_ERR_INVALID_ARG;
    if (!a->x || !a->gate || !a->h) return SNN_ERR_INVALID_ARG;
    if (a->x_format != SNN_KEEP_RAW && (!a->x_codes || !a->x_scales)) return SNN_ERR_INVALID_ARG;
    if (a->gate_format != SNN_KEEP_RAW && (!a->gate_codes || !a->gate_scales)) return SNN_ERR_INVALID_ARG;
  }
  ScanParams p = params_of(a);
  p.vec_out = pairs_aligned(p.h, a->dtype, p.hs[0], p.hs[1]);
  const cudaStream_t s = (cudaStream_t)stream;
  return by_dtype(a->dtype, [&](auto io) {
    using IO = decltype(io);
    if (!keep && p.T <= SCAN_SHORT) {
      const int64_t blocks = ((int64_t)p.B * ((p.N + 1) / 2) + 127) / 128;
      if (blocks > INT32_MAX) return SNN_ERR_UNSUPPORTED;
      scan_short_kernel<IO><<<(unsigned)blocks, 128, 0, s>>>(p);
      return launched();
    }
    return keep ? launch_clusters(scan_forward_kernel<IO, true>, p, s) : launch_clusters(scan_forward_kernel<IO, false>, p, s);
  });
}

extern "C" snn_status snn_scan_backward(const snn_scan_args* a, void* stream) {
  const snn_status st = check_common(a);
  if (st != SNN_OK) return st;
  if (a->B == 0 || a->N == 0) return SNN_OK;
  if (a->T > 0) {
    if (!a->dh || !a->dx || !a->dgate || !a->states) return SNN_ERR_INVALID_ARG;
    if (a->x_format == SNN_KEEP_RAW ? !a->x : !a->x_codes || !a->x_scales) return SNN_ERR_INVALID_ARG;
    if (a->gate_format == SNN_KEEP_RAW ? !a->gate : !a->gate_codes || !a->gate_scales) return SNN_ERR_INVALID_ARG;
  }
  ScanParams p = params_of(a);
  p.vec_out = pairs_aligned(p.dx, a->dtype, p.dxs[0], p.dxs[1]) && pairs_aligned(p.dgate, a->dtype, p.dgs[0], p.dgs[1]);
  return by_dtype(a->dtype, [&](auto io) { return launch_clusters(scan_backward_kernel<decltype(io)>, p, (cudaStream_t)stream); });
}

extern "C" snn_status snn_activation_pack(const void* values, int32_t dtype, int64_t n_rows, int32_t n_cols, int64_t row_stride,
                                          int32_t format, uint8_t* codes, uint8_t* scales, void* stream) {
  if (n_rows < 0 || n_cols < 0 || !dtype_known(dtype) || (format != SNN_KEEP_INT8 && format != SNN_KEEP_E4M3)) return SNN_ERR_INVALID_ARG;
  if (n_rows == 0 || n_cols == 0) return SNN_OK;
  if (!values || !codes || !scales) return SNN_ERR_INVALID_ARG;
  const int64_t groups = n_rows * ((n_cols + KEEP_GROUP - 1) / KEEP_GROUP);
  const unsigned blocks = (unsigned)std::min<int64_t>((groups + PACK_WARPS - 1) / PACK_WARPS, 148 * 8);
  return by_dtype(dtype, [&](auto io) {
    using IO = decltype(io);
    activation_pack_kernel<IO><<<blocks, 32 * PACK_WARPS, 0, (cudaStream_t)stream>>>(
        (const IO*)values, n_rows, n_cols, row_stride, format, pairs_aligned(values, dtype, row_stride, 0),
        n_cols % 2 == 0 && aligned2(codes), codes, scales);
    return launched();
  });
}

extern "C" snn_status snn_activation_unpack(const uint8_t* codes, const uint8_t* scales, int32_t format, int64_t n_rows, int32_t n_cols,
                                            void* values, int32_t dtype, int64_t row_stride, void* stream) {
  if (n_rows < 0 || n_cols < 0 || !dtype_known(dtype) || (format != SNN_KEEP_INT8 && format != SNN_KEEP_E4M3)) return SNN_ERR_INVALID_ARG;
  if (n_rows == 0 || n_cols == 0) return SNN_OK;
  if (!values || !codes || !scales) return SNN_ERR_INVALID_ARG;
  const int64_t groups = n_rows * ((n_cols + KEEP_GROUP - 1) / KEEP_GROUP);
  const unsigned blocks = (unsigned)std::min<int64_t>((groups + PACK_WARPS - 1) / PACK_WARPS, 148 * 8);
  return by_dtype(dtype, [&](auto io) {
    using IO = decltype(io);
    activation_unpack_kernel<IO><<<blocks, 32 * PACK_WARPS, 0, (cudaStream_t)stream>>>(
        codes, scales, format, n_rows, n_cols, (IO*)values, row_stride, pairs_aligned(values, dtype, row_stride, 0),
        n_cols % 2 == 0 && aligned2(codes));
    return launched();
  });
}
