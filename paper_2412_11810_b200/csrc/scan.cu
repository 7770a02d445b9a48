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
#include <type_traits>

#include "seq_common.cuh"
#include "tma.cuh"

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
  const void *x, *gate, *dh;
  void *h, *dx, *dgate;
  int64_t xs[2], gs[2], hs[2], dhs[2], dxs[2], dgs[2];
  const int32_t* lengths;
  const float *state, *dlast;
  float *last, *states, *dstate;
  uint8_t *x_codes, *x_scales, *gate_codes, *gate_scales;
};

// a and the factor i of x.  sigmoid(g) and 1 - sigmoid(g) both without cancellation: with e = exp(-|g|), the larger of
// the two is 1 / (1 + e) and the smaller e / (1 + e).  (1 + e lies in [1, 2]: the hardware's reciprocal needs no care for
// the ends of the range; an e below 2^-126 counts as zero.)
__device__ __forceinline__ void sigmoids(float g, float& a, float& i) {
  float e, large;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(g) * -1.44269504f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(large) : "f"(1.f + e));
  const float small = e * large;
  a = g >= 0.f ? large : small;
  i = g >= 0.f ? small : large;
}
// gv becomes a, in becomes i, for all steps of a thread
__device__ __forceinline__ void coefficients(float2 (&gv)[SCAN_K], float2 (&in)[SCAN_K], int mode) {
  if (mode == SNN_SCAN_DIRECT) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) in[k] = make_float2(1.f, 1.f);
  } else {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      sigmoids(gv[k].x, gv[k].x, in[k].x);
      sigmoids(gv[k].y, gv[k].y, in[k].y);
    }
  }
}

struct Map2 {   // the affine maps of two channels
  float a0, b0, a1, b1;
};
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

// ---- kept rows in 8 bits ------------------------------------------------------------------------------------
// The scale and this lane's two codes of a row of 64 values, two per lane.  Called by whole warps.
template <int FORMAT> __device__ __forceinline__ uint32_t encode_row(float2 v, int n_ok, uint32_t& byte) {
  const float m = larger_magnitude(n_ok > 0 ? v.x : 0.f, n_ok > 1 ? v.y : 0.f);
  const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(m));   // bit patterns of magnitudes sort as they do
  byte = keep_scale_byte<FORMAT>(top);
  return byte == 255u ? 0u : keep_encode2<FORMAT>(v, keep_scale_inverse(byte), top);
}
// Encodes the warp's steps t0.. (those before `len`) and stores codes and scales.  FAST: rows of codes are multiples of 16
// bytes and aligned to them; they go through the warp's 512 bytes of shared memory, to be stored 16 bytes at a time.
template <int FORMAT, bool FAST>
__device__ __forceinline__ void keep_steps(const float2 (&v)[SCAN_K], const ScanParams& p, int b, int c, int n_ok, int t0, int len,
                                           uint8_t* codes, uint8_t* scales, unsigned char* s_codes) {
  const int lane = threadIdx.x & 31, groups = (p.N + KEEP_GROUP - 1) / KEEP_GROUP;
  uint32_t mine = 0;
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) {
    uint32_t byte;
    const uint32_t pair = encode_row<FORMAT>(v[k], n_ok, byte);
    if (lane == k) mine = byte;
    if (FAST) {
      *reinterpret_cast<uint16_t*>(s_codes + k * SCAN_COLS + 2 * lane) = (uint16_t)pair;
    } else if (t0 + k < len) {
      uint8_t* const at = codes + ((int64_t)(t0 + k) * p.B + b) * p.N + c;
      if (n_ok > 0) at[0] = (uint8_t)(pair & 255u);
      if (n_ok > 1) at[1] = (uint8_t)(pair >> 8);
    }
  }
  if (lane < SCAN_K && t0 + lane < len) scales[((int64_t)(t0 + lane) * p.B + b) * groups + c / KEEP_GROUP] = (uint8_t)mine;
  if (FAST) {
    __syncwarp();
    const int k = lane >> 2, col = c / SCAN_COLS * SCAN_COLS + (lane & 3) * 16;
    const uint4 row = *reinterpret_cast<const uint4*>(s_codes + lane * 16);
    if (t0 + k < len && col < p.N) *reinterpret_cast<uint4*>(codes + ((int64_t)(t0 + k) * p.B + b) * p.N + col) = row;
    __syncwarp();
  }
}

__device__ __forceinline__ int length_of(const ScanParams& p, int b) {
  return p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
}

// Zeros at the steps [t0, T) of two channels, one step per warp of the cluster.
template <bool PAIRS, typename IO>
__device__ __forceinline__ void zero_steps(const ScanParams& p, IO* out, const int64_t* stride, int b, int c, int n_ok, int t0, int first,
                                           int step) {
  for (int64_t t = (int64_t)t0 + first; t < p.T; t += step)
    store_pair<PAIRS>(out + t * stride[0] + b * stride[1], c, n_ok, make_float2(0.f, 0.f));
}

// ---- staging ------------------------------------------------------------------------------------------------
// Pairs on their way from HBM: every thread copies its own pairs of the coming turns to shared memory (cp.async, 4 or 8
// bytes), as many turns ahead as the ring is deep, and reads back only what it copied itself: no barrier, and the loads of
// a turn are in flight while the ones before it are computed and handed on.
template <typename IO> struct Ring { static constexpr int DEPTH = sizeof(IO) == 4 ? 2 : 3; };
template <int BYTES> __device__ __forceinline__ void copy_async(void* smem, const void* gmem) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem), "n"(BYTES)
                 : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

constexpr int PIECE = SCAN_K * SCAN_THREADS;          // pairs of one tensor that a block needs for a turn
constexpr int CODE_PIECE = SCAN_K * SCAN_WARPS * SCAN_COLS;   // bytes, if they are 8-bit codes

// Copies this thread's SCAN_K steps from t0 on to smem[k * SCAN_THREADS]; behind the sequence's end the last step again.
template <typename IO>
__device__ __forceinline__ void stage(typename Pair<IO>::raw* smem, const IO* column, int64_t stride, int t0, int len) {
  if (t0 + SCAN_K <= len) {
    const IO* at = column + t0 * stride;
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k, at += stride) copy_async<2 * sizeof(IO)>(smem + k * SCAN_THREADS, at);
  } else {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) copy_async<2 * sizeof(IO)>(smem + k * SCAN_THREADS, column + min(t0 + k, len - 1) * stride);
  }
}
// The codes of the warp's steps, 16 bytes per lane, to the warp's 512 bytes at smem.
__device__ __forceinline__ void stage_codes(unsigned char* smem, const uint8_t* codes, const ScanParams& p, int b, int col0, int t0, int len) {
  const int lane = threadIdx.x & 31, col = col0 + (lane & 3) * 16;
  const int64_t row = (int64_t)min(t0 + (lane >> 2), len - 1) * p.B + b;
  if (col < p.N) copy_async<16>(smem + lane * 16, codes + row * p.N + col);
}

// ---- between the blocks of a cluster --------------------------------------------------------------------------
// Every turn each block sends the summary of its chunk to all blocks: asynchronous stores to their shared memory that
// count towards an mbarrier there.  Two buffers are enough: a block sends the summary of turn i + 2 only after it has all of
// turn i + 1, and a block sends that one only after its warps have read those of turn i.
struct ClusterExchange {
  float4 slot[2][SCAN_MAX_CLUSTER][32];
  uint64_t full[2];
};
__device__ __forceinline__ void exchange_init(ClusterExchange& x, cg::cluster_group& cluster) {
  if (threadIdx.x == 0) {
    mbar_init(&x.full[0], 1);
    mbar_init(&x.full[1], 1);
    mbar_fence_init();
  }
  cluster.sync();
}
// by one whole warp
__device__ __forceinline__ void exchange_send(ClusterExchange& x, int i, int S, int rank, float4 v) {
  const int lane = threadIdx.x & 31;
  const uint32_t slot = smem_u32(&x.slot[i & 1][rank][lane]), bar = smem_u32(&x.full[i & 1]);
  if (lane == 0) mbar_arrive_expect_tx(&x.full[i & 1], (uint32_t)S * 32u * sizeof(float4));
  for (int r = 0; r < S; ++r) {
    uint32_t to, signal;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(slot), "r"(r));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(signal) : "r"(bar), "r"(r));
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to),
                 "r"(__float_as_uint(v.x)), "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)), "r"(__float_as_uint(v.w)), "r"(signal)
                 : "memory");
  }
}
// by all threads; false if the summaries did not come (then the caller makes its results NaN)
__device__ __forceinline__ bool exchange_wait(ClusterExchange& x, int i) { return mbar_wait(&x.full[i & 1], (uint32_t)(i >> 1) & 1u); }

// ---- forward -----------------------------------------------------------------------------------------------
template <typename IO, bool KEEP, bool FAST>
__global__ void __launch_bounds__(SCAN_THREADS, 3) scan_forward_kernel(const ScanParams p) {
  using raw = typename Pair<IO>::raw;
  constexpr int DEPTH = Ring<IO>::DEPTH;
  extern __shared__ __align__(16) unsigned char s_ring[];   // FAST: [DEPTH][x, gate][SCAN_K][SCAN_THREADS] pairs
  __shared__ float4 s_warp[2][SCAN_WARPS][32];
  __shared__ ClusterExchange s_exchange;
  __shared__ __align__(16) unsigned char s_codes[KEEP ? SCAN_WARPS : 1][SCAN_K * SCAN_COLS];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tile = (int)blockIdx.x / S, b = tile / p.n_tiles, c = (tile % p.n_tiles) * SCAN_COLS + 2 * lane;
  const int n_ok = min(max(p.N - c, 0), 2);
  const int len = length_of(p, b);
  const IO* const x = (const IO*)p.x + b * p.xs[1];
  const IO* const gate = (const IO*)p.gate + b * p.gs[1];
  IO* const h_out = (IO*)p.h + b * p.hs[1] + c;
  const int per_turn = S * SNN_SCAN_CHUNK, ahead = rank * SNN_SCAN_CHUNK + warp * SCAN_K;
  raw* const ring = reinterpret_cast<raw*>(s_ring) + threadIdx.x;
  auto issue = [&](int turn, int slot) {
    if (FAST && turn < len) {
      stage<IO>(ring + slot * (2 * PIECE), x + (n_ok ? c : 0), p.xs[0], turn + ahead, len);
      stage<IO>(ring + slot * (2 * PIECE) + PIECE, gate + (n_ok ? c : 0), p.gs[0], turn + ahead, len);
    }
    if (FAST) copies_issued();
  };
  float2 carry = load_state(p.state, b, p.N, c, n_ok);
  int slot = 0;
  for (int d = 0; d < DEPTH - 1; ++d) issue(d * per_turn, d);
  if (S > 1) exchange_init(s_exchange, cluster);
  for (int turn = 0, i = 0; turn < len; turn += per_turn, ++i) {
    const int buf = i & 1, chunk0 = turn + rank * SNN_SCAN_CHUNK, t0 = turn + ahead;
    const bool full = t0 + SCAN_K <= len;
    float2 xv[SCAN_K], gv[SCAN_K];
    if (FAST) {
      issue(turn + (DEPTH - 1) * per_turn, slot == 0 ? DEPTH - 1 : slot - 1);
      copies_landed<DEPTH - 1>();
      const raw* const at = ring + slot * (2 * PIECE);
      slot = slot == DEPTH - 1 ? 0 : slot + 1;
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) {
        xv[k] = to_f32(at[k * SCAN_THREADS]);
        gv[k] = to_f32(at[PIECE + k * SCAN_THREADS]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) {
        xv[k] = load_pair<FAST>(x + min(t0 + k, len - 1) * p.xs[0], c, n_ok);
        gv[k] = load_pair<FAST>(gate + min(t0 + k, len - 1) * p.gs[0], c, n_ok);
      }
    }
    if (KEEP) {
      if (p.x_format == SNN_KEEP_INT8) keep_steps<SNN_KEEP_INT8, FAST>(xv, p, b, c, n_ok, t0, len, p.x_codes, p.x_scales, s_codes[warp]);
      if (p.x_format == SNN_KEEP_E4M3) keep_steps<SNN_KEEP_E4M3, FAST>(xv, p, b, c, n_ok, t0, len, p.x_codes, p.x_scales, s_codes[warp]);
      if (p.gate_format == SNN_KEEP_INT8)
        keep_steps<SNN_KEEP_INT8, FAST>(gv, p, b, c, n_ok, t0, len, p.gate_codes, p.gate_scales, s_codes[warp]);
      if (p.gate_format == SNN_KEEP_E4M3)
        keep_steps<SNN_KEEP_E4M3, FAST>(gv, p, b, c, n_ok, t0, len, p.gate_codes, p.gate_scales, s_codes[warp]);
    }
    float2 in[SCAN_K];
    coefficients(gv, in, p.mode);   // gv becomes a, and xv b
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) xv[k] = make_float2(in[k].x * xv[k].x, in[k].y * xv[k].y);
    if (!full) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (t0 + k >= len) gv[k] = make_float2(1.f, 1.f), xv[k] = make_float2(0.f, 0.f);
    }
    Map2 mine{gv[0].x, xv[0].x, gv[0].y, xv[0].y};
#pragma unroll
    for (int k = 1; k < SCAN_K; ++k) mine = then(mine, Map2{gv[k].x, xv[k].x, gv[k].y, xv[k].y});
    s_warp[buf][warp][lane] = as4(mine);
    __syncthreads();
    float2 h;                // the state before this warp's steps
    float2 start = carry;    // ... before this block's chunk
    if (S > 1) {
      if (warp == 0) {
        Map2 all = mine;
        for (int w = 1; w < SCAN_WARPS; ++w) all = then(all, as_map(s_warp[buf][w][lane]));
        exchange_send(s_exchange, i, S, rank, as4(all));
      }
      const bool came = exchange_wait(s_exchange, i);
      for (int r = 0; r < S; ++r) {
        if (r == rank) start = carry;
        carry = apply(as_map(s_exchange.slot[buf][r][lane]), carry);
      }
      if (!came) carry.x = carry.y = start.x = start.y = __uint_as_float(0x7fc00000u);
      h = start;
      for (int w = 0; w < warp; ++w) h = apply(as_map(s_warp[buf][w][lane]), h);
    } else {
#pragma unroll
      for (int w = 0; w < SCAN_WARPS; ++w) {
        if (w == warp) h = carry;
        carry = apply(as_map(s_warp[buf][w][lane]), carry);
      }
    }
    if (KEEP && warp == 0 && chunk0 < len)
      store_state(p.states, (int64_t)(chunk0 / SNN_SCAN_CHUNK) * p.B + b, p.N, c, n_ok, start);
    IO* at = h_out + t0 * p.hs[0];
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k, at += p.hs[0]) {
      h.x = fmaf(gv[k].x, h.x, xv[k].x);
      h.y = fmaf(gv[k].y, h.y, xv[k].y);
      if (full || t0 + k < len) store_pair<FAST>(at, 0, n_ok, h);
    }
  }
  if (rank == 0 && warp == 0) store_state(p.last, b, p.N, c, n_ok, carry);
  zero_steps<FAST>(p, (IO*)p.h, p.hs, b, c, n_ok, len, rank * SCAN_WARPS + warp, S * SCAN_WARPS);
  if (S > 1) cluster.sync();   // no block leaves while another may still write to its shared memory
}

// Few steps (the token of a serving loop): a thread takes two channels of one sample through all of them.
template <typename IO, bool PAIRS>
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
      const float2 xv = load_pair<PAIRS>(x + t * p.xs[0], c, n_ok), gv = load_pair<PAIRS>(gate + t * p.gs[0], c, n_ok);
      float a0 = gv.x, a1 = gv.y, i0 = 1.f, i1 = 1.f;
      if (p.mode != SNN_SCAN_DIRECT) {
        sigmoids(gv.x, a0, i0);
        sigmoids(gv.y, a1, i1);
      }
      h = shown = make_float2(fmaf(a0, h.x, i0 * xv.x), fmaf(a1, h.y, i1 * xv.y));
    }
    store_pair<PAIRS>(h_out + t * p.hs[0], c, n_ok, shown);
  }
  store_state(p.last, b, p.N, c, n_ok, h);
}

// ---- backward ----------------------------------------------------------------------------------------------
// The quantity handed from step to step is e_t = a_t D_t = a_t (dh_t + e_{t+1}), again an affine map, composed from the
// last step to the first; the states of the chunk are recomputed from its checkpoint by the forward maps.  A block's
// chunk starts at a checkpoint, so only e crosses blocks.
template <typename IO>
__device__ __forceinline__ float2 decode_pair(const uint8_t* row, uint32_t scale, int c, int n_ok, int format) {
  const uint32_t pair = (uint32_t)row[n_ok ? c : 0] | (uint32_t)row[n_ok == 2 ? c + 1 : 0] << 8;
  return format == SNN_KEEP_INT8 ? keep_decode2<IO, SNN_KEEP_INT8>(pair, keep_scale_value(scale))
                                 : keep_decode2<IO, SNN_KEEP_E4M3>(pair, keep_scale_value(scale));
}
template <int FORMAT, typename IO>
__device__ __forceinline__ void decode_steps(float2 (&v)[SCAN_K], const unsigned char* s_codes, uint32_t scales, int from) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) {
    const float scale = keep_scale_value(__shfl_sync(0xffffffffu, scales, from + k));
    v[k] = keep_decode2<IO, FORMAT>(*reinterpret_cast<const uint16_t*>(s_codes + k * SCAN_COLS + 2 * lane), scale);
  }
}

template <typename IO, bool FAST>
__global__ void __launch_bounds__(SCAN_THREADS, 2) scan_backward_kernel(const ScanParams p) {
  using raw = typename Pair<IO>::raw;
  constexpr int DEPTH = Ring<IO>::DEPTH;
  extern __shared__ __align__(16) unsigned char s_ring[];   // FAST: [DEPTH] of dh pairs, x and gate (pairs or codes)
  __shared__ float4 s_fwd[2][SCAN_WARPS][32];
  __shared__ float4 s_bwd[2][SCAN_WARPS][32];
  __shared__ ClusterExchange s_exchange;
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tile = (int)blockIdx.x / S, b = tile / p.n_tiles, col0 = (tile % p.n_tiles) * SCAN_COLS, c = col0 + 2 * lane;
  const int n_ok = min(max(p.N - c, 0), 2), groups = p.n_tiles;
  const int len = length_of(p, b);
  const IO* const x = (const IO*)p.x + b * p.xs[1];
  const IO* const gate = (const IO*)p.gate + b * p.gs[1];
  const IO* const dh = (const IO*)p.dh + b * p.dhs[1];
  IO* const dx = (IO*)p.dx + b * p.dxs[1] + c;
  IO* const dgate = (IO*)p.dgate + b * p.dgs[1] + c;
  const bool raw_x = p.x_format == SNN_KEEP_RAW, raw_gate = p.gate_format == SNN_KEEP_RAW;
  const int per_turn = S * SNN_SCAN_CHUNK, ahead = rank * SNN_SCAN_CHUNK + warp * SCAN_K;
  const int x_at = PIECE * (int)sizeof(raw), gate_at = x_at + (raw_x ? PIECE * (int)sizeof(raw) : CODE_PIECE);
  const int slot_bytes = gate_at + (raw_gate ? PIECE * (int)sizeof(raw) : CODE_PIECE);
  const int code_off = warp * SCAN_K * SCAN_COLS;
  auto pairs_of = [&](int at) { return reinterpret_cast<raw*>(s_ring + at) + threadIdx.x; };
  auto issue = [&](int turn, int slot) {
    if (FAST && turn >= 0) {
      const int at = slot * slot_bytes, t0 = turn + ahead;
      stage<IO>(pairs_of(at), dh + (n_ok ? c : 0), p.dhs[0], t0, len);
      if (raw_x) stage<IO>(pairs_of(at + x_at), x + (n_ok ? c : 0), p.xs[0], t0, len);
      else stage_codes(s_ring + at + x_at + code_off, p.x_codes, p, b, col0, t0, len);
      if (raw_gate) stage<IO>(pairs_of(at + gate_at), gate + (n_ok ? c : 0), p.gs[0], t0, len);
      else stage_codes(s_ring + at + gate_at + code_off, p.gate_codes, p, b, col0, t0, len);
    }
    if (FAST) copies_issued();
  };
  // scale bytes: of x in lanes 0..7 (one per step), of the gate in lanes 8..15, read one turn ahead
  auto load_scales = [&](int turn) -> uint32_t {
    const int64_t row = (int64_t)max(min(turn + ahead + (lane & 7), len - 1), 0) * p.B + b;
    if (turn < 0) return 0;
    if (lane < 8) return raw_x ? 0 : p.x_scales[row * groups + col0 / KEEP_GROUP];
    if (lane < 16) return raw_gate ? 0 : p.gate_scales[row * groups + col0 / KEEP_GROUP];
    return 0;
  };
  auto load_start = [&](int turn) {   // the kept state of this block's chunk
    if (turn < 0) return make_float2(0.f, 0.f);
    return load_state(p.states, (int64_t)(min(turn + rank * SNN_SCAN_CHUNK, len - 1) / SNN_SCAN_CHUNK) * p.B + b, p.N, c, n_ok);
  };
  float2 carry = load_state(p.dlast, b, p.N, c, n_ok);   // e behind the turn's last step
  int slot = 0;
  const int last_turn = (len + per_turn - 1) / per_turn * per_turn - per_turn;
  for (int d = 0; d < DEPTH - 1; ++d) issue(last_turn - d * per_turn, d);
  uint32_t next_scales = load_scales(last_turn);
  float2 next_start = load_start(last_turn);
  if (S > 1) exchange_init(s_exchange, cluster);
  for (int turn = last_turn, i = 0; turn >= 0; turn -= per_turn, ++i) {
    const int buf = i & 1, t0 = turn + ahead;
    const bool full = t0 + SCAN_K <= len;
    float2 xv[SCAN_K], a[SCAN_K], in[SCAN_K], d[SCAN_K];
    const uint32_t scales = next_scales;
    float2 h = next_start;
    next_scales = load_scales(turn - per_turn);
    next_start = load_start(turn - per_turn);
    if (FAST) {
      issue(turn - (DEPTH - 1) * per_turn, slot == 0 ? DEPTH - 1 : slot - 1);
      copies_landed<DEPTH - 1>();
      __syncwarp();   // codes were copied by other lanes
      const int at = slot * slot_bytes;
      slot = slot == DEPTH - 1 ? 0 : slot + 1;
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) d[k] = to_f32(pairs_of(at)[k * SCAN_THREADS]);
      if (raw_x) {
#pragma unroll
        for (int k = 0; k < SCAN_K; ++k) xv[k] = to_f32(pairs_of(at + x_at)[k * SCAN_THREADS]);
      } else if (p.x_format == SNN_KEEP_INT8) {
        decode_steps<SNN_KEEP_INT8, IO>(xv, s_ring + at + x_at + code_off, scales, 0);
      } else {
        decode_steps<SNN_KEEP_E4M3, IO>(xv, s_ring + at + x_at + code_off, scales, 0);
      }
      if (raw_gate) {
#pragma unroll
        for (int k = 0; k < SCAN_K; ++k) a[k] = to_f32(pairs_of(at + gate_at)[k * SCAN_THREADS]);
      } else if (p.gate_format == SNN_KEEP_INT8) {
        decode_steps<SNN_KEEP_INT8, IO>(a, s_ring + at + gate_at + code_off, scales, 8);
      } else {
        decode_steps<SNN_KEEP_E4M3, IO>(a, s_ring + at + gate_at + code_off, scales, 8);
      }
      __syncwarp();   // all lanes have read their codes before the slot is filled again
    } else {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) {
        const int64_t t = min(t0 + k, len - 1);
        d[k] = load_pair<FAST>(dh + t * p.dhs[0], c, n_ok);
        xv[k] = raw_x ? load_pair<FAST>(x + t * p.xs[0], c, n_ok)
                      : decode_pair<IO>(p.x_codes + (t * p.B + b) * p.N, __shfl_sync(0xffffffffu, scales, k), c, n_ok, p.x_format);
        a[k] = raw_gate ? load_pair<FAST>(gate + t * p.gs[0], c, n_ok)
                        : decode_pair<IO>(p.gate_codes + (t * p.B + b) * p.N, __shfl_sync(0xffffffffu, scales, 8 + k), c, n_ok, p.gate_format);
      }
    }
    coefficients(a, in, p.mode);
    if (!full) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (t0 + k >= len) a[k] = make_float2(1.f, 1.f), xv[k] = d[k] = in[k] = make_float2(0.f, 0.f);
    }
    Map2 forth{a[0].x, in[0].x * xv[0].x, a[0].y, in[0].y * xv[0].y};
#pragma unroll
    for (int k = 1; k < SCAN_K; ++k) forth = then(forth, Map2{a[k].x, in[k].x * xv[k].x, a[k].y, in[k].y * xv[k].y});
    // the way back has the same product of decays; its other part is e before the warp's steps if none came in
    float2 e0 = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = SCAN_K - 1; k >= 0; --k) e0 = make_float2(a[k].x * (d[k].x + e0.x), a[k].y * (d[k].y + e0.y));
    const Map2 back{forth.a0, e0.x, forth.a1, e0.y};
    s_fwd[buf][warp][lane] = as4(forth);
    s_bwd[buf][warp][lane] = as4(back);
    __syncthreads();
    for (int w = 0; w < warp; ++w) h = apply(as_map(s_fwd[buf][w][lane]), h);
    float2 e;   // behind this warp's steps
    if (S > 1) {
      if (warp == 0) {
        Map2 all = as_map(s_bwd[buf][SCAN_WARPS - 1][lane]);
        for (int w = SCAN_WARPS - 2; w >= 0; --w) all = then(all, as_map(s_bwd[buf][w][lane]));
        exchange_send(s_exchange, i, S, rank, as4(all));
      }
      const bool came = exchange_wait(s_exchange, i);
      e = carry;
      for (int r = S - 1; r >= 0; --r) {
        if (r == rank) e = carry;
        carry = apply(as_map(s_exchange.slot[buf][r][lane]), carry);
      }
      if (!came) carry.x = carry.y = e.x = e.y = __uint_as_float(0x7fc00000u);
      for (int w = SCAN_WARPS - 1; w > warp; --w) e = apply(as_map(s_bwd[buf][w][lane]), e);
    } else {
#pragma unroll
      for (int w = SCAN_WARPS - 1; w >= 0; --w) {
        if (w == warp) e = carry;
        carry = apply(as_map(s_bwd[buf][w][lane]), carry);
      }
    }
#pragma unroll
    for (int k = SCAN_K - 1; k >= 0; --k) {   // d becomes D
      d[k] = make_float2(d[k].x + e.x, d[k].y + e.y);
      e = make_float2(a[k].x * d[k].x, a[k].y * d[k].y);
    }
    IO *dx_at = dx + t0 * p.dxs[0], *dg_at = dgate + t0 * p.dgs[0];
    const bool direct = p.mode == SNN_SCAN_DIRECT;
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k, dx_at += p.dxs[0], dg_at += p.dgs[0]) {
      // DIRECT: dx = D, dgate = D h; SIGMOID: dx = D i, dgate = D i a (h - x)
      const float2 gx = make_float2(d[k].x * in[k].x, d[k].y * in[k].y);
      const float2 gg = direct ? make_float2(d[k].x * h.x, d[k].y * h.y)
                               : make_float2(gx.x * a[k].x * (h.x - xv[k].x), gx.y * a[k].y * (h.y - xv[k].y));
      if (full || t0 + k < len) {
        store_pair<FAST>(dx_at, 0, n_ok, gx);
        store_pair<FAST>(dg_at, 0, n_ok, gg);
      }
      h = make_float2(fmaf(a[k].x, h.x, in[k].x * xv[k].x), fmaf(a[k].y, h.y, in[k].y * xv[k].y));
    }
  }
  if (rank == 0 && warp == 0) store_state(p.dstate, b, p.N, c, n_ok, carry);
  zero_steps<FAST>(p, (IO*)p.dx, p.dxs, b, c, n_ok, len, rank * SCAN_WARPS + warp, S * SCAN_WARPS);
  zero_steps<FAST>(p, (IO*)p.dgate, p.dgs, b, c, n_ok, len, rank * SCAN_WARPS + warp, S * SCAN_WARPS);
  if (S > 1) cluster.sync();
}

// ---- 8-bit activations on their own --------------------------------------------------------------------------
// Bound by HBM (bytes of a value + 1 each way).  FAST: eight lanes share a group, eight neighbouring values each, so that
// loads and stores are 8 to 32 bytes per lane, and a warp has PACK_UNROLL x 4 groups in flight; it needs rows that are
// multiples of 8 values and aligned to them.  Otherwise a warp takes one group at a time, two values per lane.
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
size_t dtype_size(int dtype) { return dtype == SNN_DTYPE_FP32 ? 4 : 2; }
bool dtype_known(int dtype) { return dtype >= SNN_DTYPE_FP32 && dtype <= SNN_DTYPE_FP16; }
// whether pairs of values can be accessed at once: even offsets everywhere
bool pairs_aligned(const void* p, size_t size, int64_t s0, int64_t s1 = 0) {
  return (uintptr_t)p % (2 * size) == 0 && s0 % 2 == 0 && s1 % 2 == 0;
}
// the kernels' template arguments: the value type, and whether the fast path's alignment holds
template <typename F> snn_status by_dtype(int dtype, bool pairs, F&& f) {
  if (dtype == SNN_DTYPE_FP32) return pairs ? f(float(), std::true_type()) : f(float(), std::false_type());
  if (dtype == SNN_DTYPE_BF16) return pairs ? f(__nv_bfloat16(), std::true_type()) : f(__nv_bfloat16(), std::false_type());
  return pairs ? f(__half(), std::true_type()) : f(__half(), std::false_type());
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
  return p;
}
// rows of 8-bit codes that can be accessed 16 bytes at a time
bool codes_aligned(const ScanParams& p) {
  bool ok = true;
  if (p.x_format != SNN_KEEP_RAW) ok = ok && p.N % 16 == 0 && (uintptr_t)p.x_codes % 16 == 0;
  if (p.gate_format != SNN_KEEP_RAW) ok = ok && p.N % 16 == 0 && (uintptr_t)p.gate_codes % 16 == 0;
  return ok;
}
// Blocks per column tile: enough for four blocks on each of 148 SMs, no more than there are chunks.
int cluster_of(int64_t tiles, int T) {
  int S = 1;
  while (S < SCAN_MAX_CLUSTER && tiles * S < 4 * 148 && (int64_t)S * SNN_SCAN_CHUNK < T) S *= 2;
  return S;
}
template <typename K> snn_status launch_clusters(K kernel, size_t ring_bytes, const ScanParams& p, cudaStream_t stream) {
  const int64_t tiles = (int64_t)p.B * p.n_tiles;
  const int S = cluster_of(tiles, p.T);
  if (tiles * S > INT32_MAX) return SNN_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(tiles * S));
  cfg.blockDim = dim3(SCAN_THREADS);
  cfg.stream = stream;
  cfg.dynamicSmemBytes = ring_bytes;
  if (ring_bytes && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ring_bytes) != cudaSuccess)
    return cudaGetLastError(), SNN_ERR_CUDA;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = (unsigned)S;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
}
// whether rows can be accessed eight values at a time
bool rows_of_eight(const void* values, int n_cols, int64_t row_stride, const uint8_t* codes) {
  return n_cols % 8 == 0 && row_stride % 8 == 0 && (uintptr_t)values % 16 == 0 && (uintptr_t)codes % 8 == 0;
}
unsigned pack_blocks(int64_t n_rows, int n_cols, bool fast) {
  const int64_t groups = n_rows * ((n_cols + KEEP_GROUP - 1) / KEEP_GROUP), per_block = PACK_WARPS * (fast ? 4 * PACK_UNROLL : 1);
  return (unsigned)std::min<int64_t>((groups + per_block - 1) / per_block, 148 * 8);
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
  const size_t size = dtype_size(a->dtype);
  const bool fast = p.N % 2 == 0 && pairs_aligned(p.x, size, p.xs[0], p.xs[1]) && pairs_aligned(p.gate, size, p.gs[0], p.gs[1]) &&
                    pairs_aligned(p.h, size, p.hs[0], p.hs[1]) && codes_aligned(p);
  const cudaStream_t s = (cudaStream_t)stream;
  return by_dtype(a->dtype, fast, [&](auto io, auto is_fast) {
    using IO = decltype(io);
    constexpr bool FAST = decltype(is_fast)::value;
    if (!keep && p.T <= SCAN_SHORT) {
      const int64_t blocks = ((int64_t)p.B * ((p.N + 1) / 2) + 127) / 128;
      if (blocks > INT32_MAX) return SNN_ERR_UNSUPPORTED;
      scan_short_kernel<IO, FAST><<<(unsigned)blocks, 128, 0, s>>>(p);
      return launched();
    }
    const size_t ring = FAST ? Ring<IO>::DEPTH * 2 * PIECE * 2 * sizeof(IO) : 0;
    return keep ? launch_clusters(scan_forward_kernel<IO, true, FAST>, ring, p, s)
                : launch_clusters(scan_forward_kernel<IO, false, FAST>, ring, p, s);
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
  const size_t size = dtype_size(a->dtype);
  const bool fast = p.N % 2 == 0 && pairs_aligned(p.dh, size, p.dhs[0], p.dhs[1]) && pairs_aligned(p.dx, size, p.dxs[0], p.dxs[1]) &&
                    pairs_aligned(p.dgate, size, p.dgs[0], p.dgs[1]) && codes_aligned(p) &&
                    (p.x_format != SNN_KEEP_RAW || pairs_aligned(p.x, size, p.xs[0], p.xs[1])) &&
                    (p.gate_format != SNN_KEEP_RAW || pairs_aligned(p.gate, size, p.gs[0], p.gs[1]));
  return by_dtype(a->dtype, fast, [&](auto io, auto is_fast) {
    using IO = decltype(io);
    constexpr bool FAST = decltype(is_fast)::value;
    const size_t piece = PIECE * 2 * sizeof(IO);
    const size_t slot = piece + (p.x_format == SNN_KEEP_RAW ? piece : CODE_PIECE) + (p.gate_format == SNN_KEEP_RAW ? piece : CODE_PIECE);
    return launch_clusters(scan_backward_kernel<IO, FAST>, FAST ? Ring<IO>::DEPTH * slot : 0, p, (cudaStream_t)stream);
  });
}

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
