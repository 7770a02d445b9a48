// The gated linear recurrence with its backward pass (include/snn.h, "sequence-model operators").
//
// A step is an affine map of the state, h -> a h + b, and maps compose: (a2, b2) o (a1, b1) = (a2 a1, a2 b1 + b2).  So a
// run of steps can be summarised before its start is known.  A thread takes 8 steps of two neighbouring channels in
// registers, the 8 warps of a thread block a chunk of 64 steps, and the block walks through the chunks of its 64 channels;
// each turn one warp chains the summaries of the others.  Every input is read once, every output written once.
// Where there are fewer tiles of channels than SMs the time axis is cut into segments as well: a first kernel summarises
// every segment (it reads the inputs once more, without a barrier in its loop), and the blocks of the second one chain the
// summaries of the segments before their own.  (Blocks in a cluster that hand summaries on every turn read the inputs only
// once, but wait for one another: 65536 x 1024 bf16 forward took 235 us that way.)  The order of the arithmetic is fixed
// by the sizes and by what is kept.
//
// The kernels are bound by HBM as long as a step costs few instructions: channels are handled in pairs (f32x2 arithmetic),
// tiles of 64 steps x 64 channels arrive by TMA a turn or two ahead and leave by TMA, so that the threads compute no
// addresses.  Data that TMA cannot describe (rows that are not multiples of 16 bytes) takes one of two other paths: plain
// loads of pairs, or of single values.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "seq_common.cuh"
#include "tma.cuh"

using namespace snnk;

namespace {

constexpr int SCAN_K = 8;                       // steps per thread
constexpr int WARPS = SNN_SCAN_CHUNK / SCAN_K;  // a thread block's turn is a chunk
constexpr int SCAN_COLS = 64;                   // channels per thread block, two per lane: one group of the 8-bit format
constexpr int SCAN_SHORT = 16;                  // up to so many steps a thread simply walks through them
constexpr int SCAN_DEPTH = 2;                   // turns whose inputs are in shared memory or on their way
constexpr int PIECE = SNN_SCAN_CHUNK * SCAN_COLS;   // values of one tensor that a block needs for a turn
constexpr int WARP_PIECE = SCAN_K * SCAN_COLS;      // ... that a warp does
static_assert(SCAN_COLS == KEEP_GROUP, "a warp encodes one group at a time");

// How data comes and goes: TILES by TMA (rows of the tensors are multiples of 16 bytes), PAIRS two values at a time,
// SCALAR one at a time.
enum Path { SCALAR, PAIRS, TILES };

struct ScanParams {
  CUtensorMap in[3], out[4];   // TILES.  forward: x, gate -> h, -, codes of x, codes of gate; backward: dh, x, gate -> dx, dgate
  int T, B, N, n_tiles;        // n_tiles: column tiles per sample
  int segments, segment_steps; // of the time axis; a multiple of a chunk each
  int parts;                   // of a segment, summarised by a block each
  float4* summaries;           // [segments][parts][B][n_tiles][32] maps of pairs of channels, if there are several segments
  float2* start;               // forward, several segments: the summary kernel's copy of `state`, [B][n_tiles][32].  The blocks of
                               // the last segment write `last`, which may be the same buffer, while others still start
  int mode, x_format, gate_format;
  const void *x, *gate, *dh;
  void *h, *dx, *dgate;
  int64_t xs[2], gs[2], hs[2], dhs[2], dxs[2], dgs[2];
  const int32_t* lengths;
  const float *state, *dlast;
  float *last, *states, *dstate;
  uint8_t *x_codes, *x_scales, *gate_codes, *gate_scales;
  // TILES, WAIT_TESTS: limits of the waits.  The self-test lets them run out: no loads of the turns from this step on (in the
  // order in which the pass goes), or a warp that does not wait for them
  uint32_t polls;
  int loads_end, quits_at;
};

struct Map2 {   // the affine maps of two channels
  float2 a, b;
};
__device__ __forceinline__ float2 apply(const Map2& m, float2 h) { return fma2(m.a, h, m.b); }
__device__ __forceinline__ float4 as4(const Map2& m) { return make_float4(m.a.x, m.a.y, m.b.x, m.b.y); }
__device__ __forceinline__ Map2 as_map(float4 v) { return {make_float2(v.x, v.y), make_float2(v.z, v.w)}; }
__device__ __forceinline__ Map2 then(const Map2& first, const Map2& second) { return {mul2(first.a, second.a), fma2(second.a, first.b, second.b)}; }

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// a and the factor i of x: sigmoid(g) and 1 - sigmoid(g), both without cancellation.
// For any g: with e = exp(-|g|), the larger of the two is 1 / (1 + e) and the smaller e / (1 + e).  (1 + e lies in [1, 2]; an
// e below 2^-126 counts as zero.)
__device__ __forceinline__ void sigmoids(float2 g, float2& a, float2& i) {
  const float2 e = make_float2(exp2_fast(fabsf(g.x) * -1.44269504f), exp2_fast(fabsf(g.y) * -1.44269504f));
  const float2 d = add2(e, both(1.f)), large = make_float2(reciprocal(d.x), reciprocal(d.y)), small = mul2(e, large);
  a = make_float2(g.x >= 0.f ? large.x : small.x, g.y >= 0.f ? large.y : small.y);
  i = make_float2(g.x >= 0.f ? small.x : large.x, g.y >= 0.f ? small.y : large.y);
}
// For g >= LOWEST_GATE: with e = exp(-g), a = 1 / (1 + e) and i = e a; nothing leaves the range of fp32.
constexpr float LOWEST_GATE = -80.f;
__device__ __forceinline__ void ordinary_sigmoids(float2 g, float2& a, float2& i) {
  const float2 t = mul2(g, both(-1.44269504f)), e = make_float2(exp2_fast(t.x), exp2_fast(t.y)), d = add2(e, both(1.f));
  a = make_float2(reciprocal(d.x), reciprocal(d.y));
  i = mul2(e, a);
}
// gv becomes a, in becomes i, for all steps of a thread
__device__ __forceinline__ void coefficients(float2 (&gv)[SCAN_K], float2 (&in)[SCAN_K], int mode) {
  if (mode == SNN_SCAN_DIRECT) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) in[k] = both(1.f);
    return;
  }
  float lowest = 0.f;
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) lowest = fminf(lowest, fminf(gv[k].x, gv[k].y));
  if (lowest >= LOWEST_GATE) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) ordinary_sigmoids(gv[k], gv[k], in[k]);
  } else {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) sigmoids(gv[k], gv[k], in[k]);
  }
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
__device__ __forceinline__ int length_of(const ScanParams& p, int b) {
  return p.lengths ? min(max(p.lengths[b], 0), p.T) : p.T;
}

// Where a thread stands: its block's segment [from, to) of one sample's steps, of which those before `end` exist, its
// warp's steps within a turn, its two channels.
struct Place {
  int lane, warp, b, col0, c, n_ok, len, segment, from, to, end, ahead;
  int64_t map;   // of its pair of channels in a segment's summaries
};
__device__ __forceinline__ Place place_of(const ScanParams& p) {
  Place w;
  w.lane = threadIdx.x & 31;
  w.warp = threadIdx.x >> 5;
  // neighbouring blocks: neighbouring channels of the same steps, which lie in the same DRAM pages
  const int tiles = p.B * p.n_tiles, tile = (int)(blockIdx.x % (unsigned)tiles);
  w.segment = (int)(blockIdx.x / (unsigned)tiles);
  w.b = tile / p.n_tiles;
  w.col0 = (tile % p.n_tiles) * SCAN_COLS;
  w.c = w.col0 + 2 * w.lane;
  w.n_ok = min(max(p.N - w.c, 0), 2);
  w.len = length_of(p, w.b);
  w.from = w.segment * p.segment_steps;
  w.to = w.segment == p.segments - 1 ? p.T : w.from + p.segment_steps;
  w.end = min(w.to, w.len);
  w.ahead = w.warp * SCAN_K;
  w.map = (int64_t)tile * 32 + w.lane;
  return w;
}
__device__ __forceinline__ int64_t maps_per_part(const ScanParams& p) { return (int64_t)p.B * p.n_tiles * 32; }
// The state before a segment (REVERSE: e behind it), from that before the first (behind the last).
template <bool REVERSE> __device__ __forceinline__ float2 enter_segment(const ScanParams& p, const Place& w, float2 h) {
  const int n = (REVERSE ? p.segments - 1 - w.segment : w.segment) * p.parts;
  const float4* at = p.summaries + (REVERSE ? p.segments * p.parts - 1 : 0) * maps_per_part(p) + w.map;
  const int64_t step = REVERSE ? -maps_per_part(p) : maps_per_part(p);
#pragma unroll 16
  for (int q = 0; q < n; ++q, at += step) h = apply(as_map(*at), h);
  return h;
}

// Zeros at the steps of the segment from `first` on, two channels, one step per warp.
template <bool IN_PAIRS, typename IO>
__device__ __forceinline__ void zero_steps(const Place& w, IO* out, const int64_t* stride, int first) {
  for (int64_t t = (int64_t)first + w.warp; t < w.to; t += WARPS)
    store_pair<IN_PAIRS>(out + t * stride[0] + w.b * stride[1], w.c, w.n_ok, make_float2(0.f, 0.f));
}

// ---- inputs and outputs of a turn -----------------------------------------------------------------------------
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, const void* smem_src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z),
               "r"(smem_u32(smem_src)) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void bulk_read_done() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory"); }

// This thread's pairs out of a staged tile.
template <typename IO>
__device__ __forceinline__ void read_pairs(float2 (&v)[SCAN_K], const void* tile, const Place& w) {
  using raw = typename Pair<IO>::raw;
  const raw* const at = reinterpret_cast<const raw*>(reinterpret_cast<const IO*>(tile) + w.warp * WARP_PIECE) + w.lane;
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) v[k] = to_f32(at[k * (SCAN_COLS / 2)]);
}
// The same as they are.
template <typename IO>
__device__ __forceinline__ void read_raw(typename Pair<IO>::raw (&v)[SCAN_K], const void* tile, const Place& w) {
  using raw = typename Pair<IO>::raw;
  const raw* const at = reinterpret_cast<const raw*>(reinterpret_cast<const IO*>(tile) + w.warp * WARP_PIECE) + w.lane;
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) v[k] = at[k * (SCAN_COLS / 2)];
}
template <typename IO> __device__ __forceinline__ void to_raw(typename Pair<IO>::raw (&r)[SCAN_K], const float2 (&v)[SCAN_K]) {
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) set_raw(r[k], v[k]);
}
// This thread's values straight from memory.
template <bool IN_PAIRS, typename IO>
__device__ __forceinline__ void load_values(float2 (&v)[SCAN_K], const IO* sample, int64_t stride, const Place& w, int t0) {
  if (t0 + SCAN_K <= w.len) {
    const IO* at = sample + t0 * stride;
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k, at += stride) v[k] = load_pair<IN_PAIRS>(at, w.c, w.n_ok);
  } else {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) v[k] = load_pair<IN_PAIRS>(sample + min(t0 + k, w.len - 1) * stride, w.c, w.n_ok);
  }
}

// ---- kept rows in 8 bits ------------------------------------------------------------------------------------
// Encodes the warp's steps t0.. (those before the sequence's end); codes to s_codes (TILES: they leave by TMA, and channels
// that do not exist are zeros) or to memory.
template <int FORMAT, int PATH>
__device__ __forceinline__ void keep_steps(const float2 (&v)[SCAN_K], const ScanParams& p, const Place& w, int t0, uint8_t* codes,
                                           uint8_t* scales, unsigned char* s_codes) {
  uint32_t top[SCAN_K], worst = 0, fraction = 0;   // magnitudes' bit patterns sort as they do
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) {
    const float m = PATH == TILES ? larger_magnitude(v[k].x, v[k].y) : larger_magnitude(w.n_ok > 0 ? v[k].x : 0.f, w.n_ok > 1 ? v[k].y : 0.f);
    top[k] = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
    worst = max(worst, top[k]);
    fraction = max(fraction, top[k] & 0x7fffffu);
  }
  uint32_t pair[SCAN_K];
  if (worst < 0x7f800000u && (FORMAT == SNN_KEEP_E4M3 || fraction < 0x7f0000u)) {
    // all finite, and no int8 code beyond 127: 1 / scale from the exponent alone (see keep_scale_byte)
    constexpr uint32_t add = FORMAT == SNN_KEEP_INT8 ? 0u : 0x1fffffu, from = (FORMAT == SNN_KEEP_INT8 ? 260u : 262u) << 23;
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      const float2 u = mul2(v[k], both(__uint_as_float(min(from - ((top[k] + add) & 0x7f800000u), 254u << 23))));
      if (FORMAT == SNN_KEEP_INT8) {
        const float2 r = add2(u, both(12582912.f));
        pair[k] = __byte_perm(__float_as_uint(r.x), __float_as_uint(r.y), 0x0040);
      } else {
        pair[k] = (uint32_t)__nv_cvt_float2_to_fp8x2(u, __NV_SATFINITE, __NV_E4M3);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) {
      const uint32_t byte = keep_scale_byte<FORMAT>(top[k]);
      pair[k] = byte == 255u ? 0u : keep_encode2<FORMAT>(v[k], keep_scale_inverse(byte), keep_needs_cut<FORMAT>(top[k]));
    }
  }
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) {
    if (PATH == TILES) {
      *reinterpret_cast<uint16_t*>(s_codes + k * SCAN_COLS + 2 * w.lane) = (uint16_t)pair[k];
    } else if (t0 + k < w.len) {
      uint8_t* const at = codes + ((int64_t)(t0 + k) * p.B + w.b) * p.N + w.c;
      if (PATH == PAIRS) {
        if (w.n_ok) *reinterpret_cast<uint16_t*>(at) = (uint16_t)pair[k];
      } else {
        if (w.n_ok > 0) at[0] = (uint8_t)(pair[k] & 255u);
        if (w.n_ok > 1) at[1] = (uint8_t)(pair[k] >> 8);
      }
    }
  }
  // lane k writes the scale of step k
  static_assert(SCAN_K == 8, "three bits select a step");
  const bool b0 = w.lane & 1, b1 = w.lane & 2, b2 = w.lane & 4;
  const uint32_t lo = b1 ? (b0 ? top[3] : top[2]) : (b0 ? top[1] : top[0]), hi = b1 ? (b0 ? top[7] : top[6]) : (b0 ? top[5] : top[4]);
  if (w.lane < SCAN_K && t0 + w.lane < w.len)
    scales[((int64_t)(t0 + w.lane) * p.B + w.b) * p.n_tiles + w.col0 / KEEP_GROUP] = (uint8_t)keep_scale_byte<FORMAT>(b2 ? hi : lo);
}
template <int PATH>
__device__ __forceinline__ void keep_steps(int format, const float2 (&v)[SCAN_K], const ScanParams& p, const Place& w, int t0, uint8_t* codes,
                                           uint8_t* scales, unsigned char* s_codes) {
  if (format == SNN_KEEP_INT8) keep_steps<SNN_KEEP_INT8, PATH>(v, p, w, t0, codes, scales, s_codes);
  if (format == SNN_KEEP_E4M3) keep_steps<SNN_KEEP_E4M3, PATH>(v, p, w, t0, codes, scales, s_codes);
}
// The warp's steps kept as no numbers (by the lanes that wrote the scales).
__device__ __forceinline__ void void_kept(const ScanParams& p, const Place& w, int t0) {
  if (w.lane >= SCAN_K || t0 + w.lane >= w.len) return;
  const int64_t at = ((int64_t)(t0 + w.lane) * p.B + w.b) * p.n_tiles + w.col0 / KEEP_GROUP;
  if (p.x_format != SNN_KEEP_RAW) p.x_scales[at] = 255;
  if (p.gate_format != SNN_KEEP_RAW) p.gate_scales[at] = 255;
}
// The kept values of this thread's steps; the scales' bytes lie in lanes from, from + 1, ...
template <int FORMAT, typename IO>
__device__ __forceinline__ void decode_steps(float2 (&v)[SCAN_K], const void* tile, const Place& w, uint32_t bytes, int from) {
  const uint16_t* const at = reinterpret_cast<const uint16_t*>(reinterpret_cast<const unsigned char*>(tile) + w.warp * WARP_PIECE) + w.lane;
  const float scale = keep_scale_value(bytes);
  if (FORMAT == SNN_KEEP_INT8) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) v[k] = keep_decode2<IO, FORMAT>(at[k * (SCAN_COLS / 2)], __shfl_sync(0xffffffffu, scale, from + k));
    return;
  }
  // no e4m3 value beyond the type's range at these scales: nothing to cut
  const bool within = __all_sync(0xffffffffu, !(448.f * scale > largest_finite<IO>()));
  if (within) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k)
      v[k] = mul2(__half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)at[k * (SCAN_COLS / 2)], __NV_E4M3))),
                  both(__shfl_sync(0xffffffffu, scale, from + k)));
  } else {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) v[k] = keep_decode2<IO, FORMAT>(at[k * (SCAN_COLS / 2)], __shfl_sync(0xffffffffu, scale, from + k));
  }
}
// The same straight from memory, all loads before the first use.
template <bool IN_PAIRS>
__device__ __forceinline__ void load_codes(uint32_t (&q)[SCAN_K], const uint8_t* codes, const ScanParams& p, const Place& w, int t0) {
#pragma unroll
  for (int k = 0; k < SCAN_K; ++k) {
    const uint8_t* const row = codes + ((int64_t)min(t0 + k, w.len - 1) * p.B + w.b) * p.N;
    if (IN_PAIRS) q[k] = *reinterpret_cast<const uint16_t*>(row + (w.n_ok ? w.c : 0));
    else q[k] = (uint32_t)row[w.n_ok ? w.c : 0] | (uint32_t)row[w.n_ok == 2 ? w.c + 1 : 0] << 8;
  }
}
template <typename IO>
__device__ __forceinline__ void decode_loaded(float2 (&v)[SCAN_K], const uint32_t (&q)[SCAN_K], uint32_t bytes, int from, int format) {
  const float scale = keep_scale_value(bytes);
  if (format == SNN_KEEP_INT8) {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) v[k] = keep_decode2<IO, SNN_KEEP_INT8>(q[k], __shfl_sync(0xffffffffu, scale, from + k));
  } else {
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) v[k] = keep_decode2<IO, SNN_KEEP_E4M3>(q[k], __shfl_sync(0xffffffffu, scale, from + k));
  }
}
// The barriers that count the bytes of the ring's slots (TILES).
__device__ __forceinline__ void barriers_init(uint64_t* landed) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < SCAN_DEPTH; ++i) mbar_init(&landed[i], 1);
    mbar_fence_init();
  }
  __syncthreads();
}
__device__ __forceinline__ uint32_t polls_of(const ScanParams& p, const Place& w, bool quits) {
  return !WAIT_TESTS ? MBAR_WAIT_LIMIT : quits && w.warp == 5 ? 0u : p.polls;
}
__device__ __forceinline__ float2 nan2() { return both(__uint_as_float(0x7fc00000u)); }

// ---- forward -----------------------------------------------------------------------------------------------
template <typename IO> __host__ __device__ constexpr int forward_slot() { return 2 * PIECE * (int)sizeof(IO); }
template <typename IO, bool KEEP> __host__ __device__ constexpr int forward_out() { return WARP_PIECE * ((int)sizeof(IO) + (KEEP ? 2 : 0)); }   // per warp and buffer

template <typename IO, bool KEEP, int PATH>
__global__ void __launch_bounds__(32 * WARPS, KEEP || sizeof(IO) == 4 ? 3 : 4) scan_forward_kernel(const __grid_constant__ ScanParams p) {
  constexpr int SLOT = forward_slot<IO>(), OUT = forward_out<IO, KEEP>();
  extern __shared__ __align__(128) unsigned char s_dyn[];   // ring [SCAN_DEPTH][x, gate]; TILES: then out [WARPS][2][h, codes]
  __shared__ float4 s_sum[WARPS][32];
  __shared__ float2 s_start[WARPS][32];
  __shared__ uint64_t s_landed[SCAN_DEPTH];
  const Place w = place_of(p);
  const IO* const x = (const IO*)p.x + w.b * p.xs[1];
  const IO* const gate = (const IO*)p.gate + w.b * p.gs[1];
  IO* const h_out = (IO*)p.h + w.b * p.hs[1];
  auto issue = [&](int turn, int slot) {   // by one thread
    unsigned char* const at = s_dyn + slot * SLOT;
    if constexpr (PATH == TILES) {
      if (turn < w.end && !(WAIT_TESTS && turn >= p.loads_end)) {
        mbar_arrive_expect_tx(&s_landed[slot], SLOT);
        tma_load_3d(at, &p.in[0], w.col0, w.b, turn, &s_landed[slot]);
        tma_load_3d(at + SLOT / 2, &p.in[1], w.col0, w.b, turn, &s_landed[slot]);
      }
    }
  };
  barriers_init(s_landed);
  const bool loader = PATH == TILES && threadIdx.x == 32 * (WARPS - 1);
  if (loader)
    for (int d = 0; d < SCAN_DEPTH; ++d) issue(w.from + d * SNN_SCAN_CHUNK, d);
  float2 carry = both(0.f);   // warp 0 chains the summaries
  if (w.warp == 0) carry = enter_segment<false>(p, w, p.segments > 1 ? p.start[w.map] : load_state(p.state, w.b, p.N, w.c, w.n_ok));
  bool alive = true;
  int turn = w.from;
  for (int i = 0; turn < w.end; turn += SNN_SCAN_CHUNK, ++i) {
    const int slot = i % SCAN_DEPTH, t0 = turn + w.ahead;
    const bool full = t0 + SCAN_K <= w.len;
    unsigned char* const out = s_dyn + SCAN_DEPTH * SLOT + (w.warp * 2 + (i & 1)) * OUT;
    float2 xv[SCAN_K], gv[SCAN_K];
    if constexpr (PATH != TILES) {
      load_values<PATH == PAIRS>(xv, x, p.xs[0], w, t0);
      load_values<PATH == PAIRS>(gv, gate, p.gs[0], w, t0);
    } else {
      if (alive) alive = mbar_wait(&s_landed[slot], (uint32_t)(i / SCAN_DEPTH) & 1u, polls_of(p, w, turn >= p.quits_at));
      if (w.lane == 0) bulk_read_done<1>();   // the out buffer used two turns ago has been read
      __syncwarp();
      read_pairs<IO>(xv, s_dyn + slot * SLOT, w);
      read_pairs<IO>(gv, s_dyn + slot * SLOT + SLOT / 2, w);
      if (!alive) gv[0] = nan2();
    }
    if constexpr (KEEP) {
      unsigned char* const codes = out + WARP_PIECE * sizeof(IO);
      keep_steps<PATH>(p.x_format, xv, p, w, t0, p.x_codes, p.x_scales, codes);
      keep_steps<PATH>(p.gate_format, gv, p, w, t0, p.gate_codes, p.gate_scales, codes + WARP_PIECE);
      if (!alive) void_kept(p, w, t0);
    }
    float2 in[SCAN_K];
    coefficients(gv, in, p.mode);   // gv becomes a, and xv b
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) xv[k] = mul2(in[k], xv[k]);
    if (!full) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (t0 + k >= w.len) gv[k] = both(1.f), xv[k] = both(0.f);
    }
    Map2 mine{gv[0], xv[0]};
#pragma unroll
    for (int k = 1; k < SCAN_K; ++k) mine = then(mine, Map2{gv[k], xv[k]});
    s_sum[w.warp][w.lane] = as4(mine);
    __syncthreads();
    if (loader) issue(turn + SCAN_DEPTH * SNN_SCAN_CHUNK, slot);   // all warps have read the slot
    if (w.warp == 0) {
      float2 h = carry;
      if (!alive) h = nan2();
      if (KEEP) store_state(p.states, (int64_t)(turn / SNN_SCAN_CHUNK) * p.B + w.b, p.N, w.c, w.n_ok, h);
#pragma unroll
      for (int v = 0; v < WARPS; ++v) {
        s_start[v][w.lane] = h;
        h = apply(as_map(s_sum[v][w.lane]), h);
      }
      carry = h;
    }
    __syncthreads();
    float2 h = s_start[w.warp][w.lane];
    if constexpr (PATH == TILES) {
      IO* const to = reinterpret_cast<IO*>(out) + 2 * w.lane;
      if (full) {
#pragma unroll
        for (int k = 0; k < SCAN_K; ++k) store_pair<true>(to + k * SCAN_COLS, 0, 2, h = fma2(gv[k], h, xv[k]));
      } else {
#pragma unroll
        for (int k = 0; k < SCAN_K; ++k) {
          h = fma2(gv[k], h, xv[k]);
          store_pair<true>(to + k * SCAN_COLS, 0, 2, t0 + k < w.len ? h : both(0.f));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (w.lane == 0) {
        if (t0 < w.to) {
          tma_store_3d(&p.out[0], w.col0, w.b, t0, out);
          if (KEEP && p.x_format != SNN_KEEP_RAW) tma_store_3d(&p.out[2], w.col0, w.b, t0, out + WARP_PIECE * sizeof(IO));
          if (KEEP && p.gate_format != SNN_KEEP_RAW) tma_store_3d(&p.out[3], w.col0, w.b, t0, out + WARP_PIECE * (sizeof(IO) + 1));
        }
        bulk_commit();
      }
    } else {
      IO* at = h_out + t0 * p.hs[0];
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k, at += p.hs[0]) {
        h = fma2(gv[k], h, xv[k]);
        if (full || t0 + k < w.len) store_pair<PATH == PAIRS>(at, w.c, w.n_ok, h);
      }
    }
  }
  if (w.segment == p.segments - 1 && w.warp == 0) store_state(p.last, w.b, p.N, w.c, w.n_ok, carry);
  zero_steps<PATH != SCALAR>(w, (IO*)p.h, p.hs, PATH == TILES ? turn : max(w.end, w.from));
  if (PATH == TILES && w.lane == 0) bulk_read_done<0>();
  if (!alive)
    for (int i = 0; i < 100; ++i) __nanosleep(20000);   // copies that did not come in time may still be under way
}

// Few steps (the token of a serving loop): a thread takes two channels of one sample through all of them.
template <typename IO, bool IN_PAIRS>
__global__ void __launch_bounds__(128) scan_short_kernel(const __grid_constant__ ScanParams p) {
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
      float2 xv = load_pair<IN_PAIRS>(x + t * p.xs[0], c, n_ok), a = load_pair<IN_PAIRS>(gate + t * p.gs[0], c, n_ok);
      if (p.mode != SNN_SCAN_DIRECT) {
        float2 in;
        sigmoids(a, a, in);
        xv = mul2(in, xv);
      }
      h = shown = fma2(a, h, xv);
    }
    store_pair<IN_PAIRS>(h_out + t * p.hs[0], c, n_ok, shown);
  }
  store_state(p.last, b, p.N, c, n_ok, h);
}

// ---- backward ----------------------------------------------------------------------------------------------
// The quantity handed from step to step is e_t = a_t D_t = a_t (dh_t + e_{t+1}), again an affine map, composed from the
// last step to the first; the states of the chunk are recomputed from its checkpoint by the forward maps.  A block's
// chunk starts at a checkpoint, so only e crosses blocks.  Warp 0 chains the states, warp 1 the e.
// NaN in place of the gradients of a warp's steps.
template <typename IO> __device__ __forceinline__ void void_steps(unsigned char* out, const Place& w, int t0) {
  IO* const to = reinterpret_cast<IO*>(out) + 2 * w.lane;
  for (int k = 0; k < 2 * SCAN_K; ++k) store_pair<true>(to + k * SCAN_COLS, 0, 2, t0 + k % SCAN_K < w.len ? nan2() : both(0.f));
}

template <typename IO, int PATH>
__global__ void __launch_bounds__(32 * WARPS, 2) scan_backward_kernel(const __grid_constant__ ScanParams p) {
  using raw = typename Pair<IO>::raw;
  constexpr int VALUES = PIECE * (int)sizeof(IO), OUT = 2 * WARP_PIECE * (int)sizeof(IO);
  extern __shared__ __align__(128) unsigned char s_dyn[];   // ring [SCAN_DEPTH] of dh, x, gate (values or codes); TILES: out
  __shared__ float4 s_forth[WARPS][32];
  __shared__ float2 s_back[WARPS][32];
  __shared__ float2 s_h[WARPS][32], s_e[WARPS][32];
  __shared__ uint64_t s_landed[SCAN_DEPTH];
  const Place w = place_of(p);
  const IO* const x = (const IO*)p.x + w.b * p.xs[1];
  const IO* const gate = (const IO*)p.gate + w.b * p.gs[1];
  const IO* const dh = (const IO*)p.dh + w.b * p.dhs[1];
  const bool raw_x = p.x_format == SNN_KEEP_RAW, raw_gate = p.gate_format == SNN_KEEP_RAW;
  const int x_at = VALUES, gate_at = x_at + (raw_x ? VALUES : PIECE), slot_bytes = gate_at + (raw_gate ? VALUES : PIECE);
  auto issue = [&](int turn, int slot) {
    unsigned char* const at = s_dyn + slot * slot_bytes;
    if constexpr (PATH == TILES) {
      if (turn >= w.from && !(WAIT_TESTS && turn <= p.loads_end)) {
        mbar_arrive_expect_tx(&s_landed[slot], slot_bytes);
        tma_load_3d(at, &p.in[0], w.col0, w.b, turn, &s_landed[slot]);
        tma_load_3d(at + x_at, &p.in[1], w.col0, w.b, turn, &s_landed[slot]);
        tma_load_3d(at + gate_at, &p.in[2], w.col0, w.b, turn, &s_landed[slot]);
      }
    }
  };
  // scale bytes: of x in lanes 0..7 (one per step), of the gate in lanes 8..15, read one turn ahead
  auto load_scales = [&](int turn) -> uint32_t {
    if (turn < w.from || w.lane >= 16 || (w.lane < 8 ? raw_x : raw_gate)) return 0u;
    const int64_t row = (int64_t)min(turn + w.ahead + (w.lane & 7), w.len - 1) * p.B + w.b;
    return (w.lane < 8 ? p.x_scales : p.gate_scales)[row * p.n_tiles + w.col0 / KEEP_GROUP];
  };
  auto load_start = [&](int turn) {   // the kept state of the turn's chunk
    if (turn < w.from || w.warp != 0) return both(0.f);
    return load_state(p.states, (int64_t)(turn / SNN_SCAN_CHUNK) * p.B + w.b, p.N, w.c, w.n_ok);
  };
  barriers_init(s_landed);
  const bool loader = PATH == TILES && threadIdx.x == 32 * (WARPS - 1);
  const int turns = (max(w.end - w.from, 0) + SNN_SCAN_CHUNK - 1) / SNN_SCAN_CHUNK, last_turn = w.from + (turns - 1) * SNN_SCAN_CHUNK;
  if (loader)
    for (int d = 0; d < SCAN_DEPTH; ++d) issue(last_turn - d * SNN_SCAN_CHUNK, d);
  float2 carry = both(0.f);   // e behind the turn's last step, chained by warp 1
  if (w.warp == 1) carry = enter_segment<true>(p, w, load_state(p.dlast, w.b, p.N, w.c, w.n_ok));
  uint32_t next_scales = load_scales(last_turn);
  float2 next_start = load_start(last_turn);
  bool alive = true;
  for (int turn = last_turn, i = 0; turn >= w.from; turn -= SNN_SCAN_CHUNK, ++i) {
    const int slot = i % SCAN_DEPTH, t0 = turn + w.ahead;
    const bool full = t0 + SCAN_K <= w.len;
    unsigned char* const out = s_dyn + SCAN_DEPTH * slot_bytes + (w.warp * 2 + (i & 1)) * OUT;
    // x and dh stay in their own type (a register per pair if it has 16 bits); kept values fit it (see keep_decode2)
    raw xr[SCAN_K], dr[SCAN_K];
    float2 a[SCAN_K], in[SCAN_K];
    const uint32_t scales = next_scales;
    const float2 start = next_start;
    next_scales = load_scales(turn - SNN_SCAN_CHUNK);
    next_start = load_start(turn - SNN_SCAN_CHUNK);
    unsigned char* const at = s_dyn + slot * slot_bytes;
    if (PATH == TILES) {
      if (alive) alive = mbar_wait(&s_landed[slot], (uint32_t)(i / SCAN_DEPTH) & 1u, polls_of(p, w, turn <= p.quits_at));
      if (w.lane == 0) bulk_read_done<1>();
      __syncwarp();
    }
    uint32_t xq[SCAN_K], gq[SCAN_K];   // codes, where they do not come by TMA
    if constexpr (PATH != TILES) {
      if (!raw_x) load_codes<PATH == PAIRS>(xq, p.x_codes, p, w, t0);
      if (!raw_gate) load_codes<PATH == PAIRS>(gq, p.gate_codes, p, w, t0);
      float2 v[SCAN_K];
      load_values<PATH == PAIRS>(v, dh, p.dhs[0], w, t0);
      to_raw<IO>(dr, v);
    } else {
      read_raw<IO>(dr, at, w);
    }
    if (raw_x && PATH == TILES) {
      read_raw<IO>(xr, at + x_at, w);
    } else {
      float2 v[SCAN_K];
      if (raw_x) load_values<PATH == PAIRS>(v, x, p.xs[0], w, t0);
      else if (PATH != TILES) decode_loaded<IO>(v, xq, scales, 0, p.x_format);
      else if (p.x_format == SNN_KEEP_INT8) decode_steps<SNN_KEEP_INT8, IO>(v, at + x_at, w, scales, 0);
      else decode_steps<SNN_KEEP_E4M3, IO>(v, at + x_at, w, scales, 0);
      to_raw<IO>(xr, v);
    }
    if (raw_gate) {
      if constexpr (PATH != TILES) load_values<PATH == PAIRS>(a, gate, p.gs[0], w, t0);
      else read_pairs<IO>(a, at + gate_at, w);
    } else if constexpr (PATH == TILES) {
      if (p.gate_format == SNN_KEEP_INT8) decode_steps<SNN_KEEP_INT8, IO>(a, at + gate_at, w, scales, 8);
      else decode_steps<SNN_KEEP_E4M3, IO>(a, at + gate_at, w, scales, 8);
    } else {
      decode_loaded<IO>(a, gq, scales, 8, p.gate_format);
    }
    if (!alive) a[0] = nan2();
    coefficients(a, in, p.mode);
    if (!full) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        if (t0 + k >= w.len) {
          a[k] = both(1.f);
          in[k] = both(0.f);
          set_raw(xr[k], both(0.f));
          set_raw(dr[k], both(0.f));
        }
    }
    Map2 forth{a[0], mul2(in[0], to_f32(xr[0]))};
#pragma unroll
    for (int k = 1; k < SCAN_K; ++k) forth = then(forth, Map2{a[k], mul2(in[k], to_f32(xr[k]))});
    // the way back has the same product of decays; its other part is e before the warp's steps if none came in
    float2 e0 = mul2(a[SCAN_K - 1], to_f32(dr[SCAN_K - 1]));
#pragma unroll
    for (int k = SCAN_K - 2; k >= 0; --k) e0 = mul2(a[k], add2(to_f32(dr[k]), e0));
    s_forth[w.warp][w.lane] = as4(forth);
    s_back[w.warp][w.lane] = e0;
    __syncthreads();
    if (loader) issue(turn - SCAN_DEPTH * SNN_SCAN_CHUNK, slot);
    if (w.warp == 0) {
      float2 h = alive ? start : nan2();
#pragma unroll
      for (int v = 0; v < WARPS; ++v) {
        s_h[v][w.lane] = h;
        h = apply(as_map(s_forth[v][w.lane]), h);
      }
    } else if (w.warp == 1) {
      auto back = [&](int v) { return Map2{as_map(s_forth[v][w.lane]).a, s_back[v][w.lane]}; };
      float2 e = carry;
      if (!alive) e = nan2();
#pragma unroll
      for (int v = WARPS - 1; v >= 0; --v) {
        s_e[v][w.lane] = e;
        e = apply(back(v), e);
      }
      carry = e;
    }
    __syncthreads();
    float2 h = s_h[w.warp][w.lane], e = s_e[w.warp][w.lane];
    // u_k = dgate_k / D_k from the first step to the last, then D and the results from the last to the first.
    // DIRECT: u = h, dx = D; SIGMOID: u = i a (h - x), dx = D i
    auto outputs = [&](auto is_direct, auto is_full) {
      constexpr bool DIRECT = decltype(is_direct)::value, FULL = decltype(is_full)::value;
      float2 u[SCAN_K];
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) {
        const float2 xv = to_f32(xr[k]);
        u[k] = DIRECT ? h : mul2(mul2(in[k], a[k]), fma2(xv, both(-1.f), h));
        h = fma2(a[k], h, DIRECT ? xv : mul2(in[k], xv));
      }
      IO *dx_to, *dg_to;
      if (PATH == TILES) {
        dx_to = reinterpret_cast<IO*>(out) + (SCAN_K - 1) * SCAN_COLS + 2 * w.lane;
        dg_to = dx_to + WARP_PIECE;
      } else {
        dx_to = (IO*)p.dx + w.b * p.dxs[1] + (t0 + SCAN_K - 1) * p.dxs[0];
        dg_to = (IO*)p.dgate + w.b * p.dgs[1] + (t0 + SCAN_K - 1) * p.dgs[0];
      }
#pragma unroll
      for (int k = SCAN_K - 1; k >= 0; --k) {
        const float2 D = add2(to_f32(dr[k]), e), gx = DIRECT ? D : mul2(D, in[k]), gg = mul2(D, u[k]);
        e = mul2(a[k], D);
        const bool on = FULL || t0 + k < w.len;
        if (PATH == TILES) {
          store_pair<true>(dx_to, 0, 2, on ? gx : both(0.f));
          store_pair<true>(dg_to, 0, 2, on ? gg : both(0.f));
          dx_to -= SCAN_COLS;
          dg_to -= SCAN_COLS;
        } else {
          if (on) store_pair<PATH == PAIRS>(dx_to, w.c, w.n_ok, gx);
          if (on) store_pair<PATH == PAIRS>(dg_to, w.c, w.n_ok, gg);
          dx_to -= p.dxs[0];
          dg_to -= p.dgs[0];
        }
      }
    };
    if (p.mode == SNN_SCAN_DIRECT) full ? outputs(std::true_type(), std::true_type()) : outputs(std::true_type(), std::false_type());
    else full ? outputs(std::false_type(), std::true_type()) : outputs(std::false_type(), std::false_type());
    if (PATH == TILES) {
      if (!alive) void_steps<IO>(out, w, t0);
      fence_proxy_async_smem();
      __syncwarp();
      if (w.lane == 0) {
        if (t0 < w.to) {
          tma_store_3d(&p.out[0], w.col0, w.b, t0, out);
          tma_store_3d(&p.out[1], w.col0, w.b, t0, out + OUT / 2);
        }
        bulk_commit();
      }
    }
  }
  if (w.segment == 0 && w.warp == 1) store_state(p.dstate, w.b, p.N, w.c, w.n_ok, carry);
  const int first = PATH == TILES ? w.from + turns * SNN_SCAN_CHUNK : max(w.end, w.from);
  zero_steps<PATH != SCALAR>(w, (IO*)p.dx, p.dxs, first);
  zero_steps<PATH != SCALAR>(w, (IO*)p.dgate, p.dgs, first);
  if (PATH == TILES && w.lane == 0) bulk_read_done<0>();
  if (!alive)
    for (int i = 0; i < 100; ++i) __nanosleep(20000);
}

// ---- segments ------------------------------------------------------------------------------------------------
// The maps of the parts of every segment but the last (REVERSE, the backward pass: but the first).  A warp takes an eighth of
// a part's steps on its own, so nothing waits inside the loop; plain loads, 8 steps at a time.
template <typename IO, bool IN_PAIRS, bool REVERSE>
__global__ void __launch_bounds__(32 * WARPS, sizeof(IO) == 2 ? 4 : 3) scan_summary_kernel(const __grid_constant__ ScanParams p) {
  __shared__ float4 s_sum[WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned tiles = (unsigned)(p.B * p.n_tiles);
  const int tile = (int)(blockIdx.x % tiles), part = (int)(blockIdx.x / tiles) + (REVERSE ? p.parts : 0);   // counted from the first segment's first
  const int b = tile / p.n_tiles, c = (tile % p.n_tiles) * SCAN_COLS + 2 * lane, n_ok = min(max(p.N - c, 0), 2);
  const int len = length_of(p, b), steps = p.segment_steps / p.parts, share = steps / WARPS, first = part * steps + warp * share;
  const int end = min(first + share, len);
  const IO* const from = REVERSE ? (const IO*)p.dh + b * p.dhs[1] : (const IO*)p.x + b * p.xs[1];
  const int64_t from_stride = REVERSE ? p.dhs[0] : p.xs[0];
  const IO* const gate = (const IO*)p.gate + b * p.gs[1];
  const bool raw_gate = !REVERSE || p.gate_format == SNN_KEEP_RAW;
  using raw = typename Pair<IO>::raw;
  Map2 m{both(1.f), both(0.f)};
  const int turns = (max(end - first, 0) + SCAN_K - 1) / SCAN_K;
  for (int i = 0; i < turns; ++i) {
    const int t0 = first + (REVERSE ? turns - 1 - i : i) * SCAN_K;
    const bool full = t0 + SCAN_K <= end;
    // values stay in their own type until their step: registers for a fourth block per SM
    raw v[SCAN_K], g[SCAN_K];
#pragma unroll
    for (int k = 0; k < SCAN_K; ++k) v[k] = load_raw<IN_PAIRS>(from + min(t0 + k, end - 1) * from_stride, c, n_ok);
    if (raw_gate) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) g[k] = load_raw<IN_PAIRS>(gate + min(t0 + k, end - 1) * p.gs[0], c, n_ok);
    } else {
      uint32_t codes[SCAN_K], bytes[SCAN_K];
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) {
        const int64_t row = (int64_t)min(t0 + k, end - 1) * p.B + b;
        const uint8_t* const at = p.gate_codes + row * p.N;
        if (IN_PAIRS) codes[k] = *reinterpret_cast<const uint16_t*>(at + (n_ok ? c : 0));
        else codes[k] = (uint32_t)at[n_ok ? c : 0] | (uint32_t)at[n_ok == 2 ? c + 1 : 0] << 8;
        bytes[k] = p.gate_scales[row * p.n_tiles + (c - 2 * lane) / KEEP_GROUP];
      }
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k)
        set_raw(g[k], p.gate_format == SNN_KEEP_INT8 ? keep_decode2<IO, SNN_KEEP_INT8>(codes[k], keep_scale_value(bytes[k]))
                                                     : keep_decode2<IO, SNN_KEEP_E4M3>(codes[k], keep_scale_value(bytes[k])));
    }
    float lowest = 0.f;
    if (p.mode != SNN_SCAN_DIRECT) {
#pragma unroll
      for (int k = 0; k < SCAN_K; ++k) lowest = fminf(lowest, fminf(to_f32(g[k]).x, to_f32(g[k]).y));
    }
    auto compose = [&](auto kind) {   // 0: direct, 1: ordinary gates, 2: any
#pragma unroll
      for (int j = 0; j < SCAN_K; ++j) {
        const int k = REVERSE ? SCAN_K - 1 - j : j;
        float2 a = to_f32(g[k]), in = both(1.f), x = to_f32(v[k]);
        if constexpr (decltype(kind)::value == 1) ordinary_sigmoids(a, a, in);
        if constexpr (decltype(kind)::value == 2) sigmoids(a, a, in);
        float2 added = mul2(REVERSE ? a : in, x);
        if (!full && t0 + k >= end) a = both(1.f), added = both(0.f);
        m = then(m, Map2{a, added});
      }
    };
    if (p.mode == SNN_SCAN_DIRECT) compose(std::integral_constant<int, 0>());
    else if (lowest >= LOWEST_GATE) compose(std::integral_constant<int, 1>());
    else compose(std::integral_constant<int, 2>());
  }
  s_sum[warp][lane] = as4(m);
  __syncthreads();
  if (warp == 0) {
    m = as_map(s_sum[REVERSE ? WARPS - 1 : 0][lane]);
#pragma unroll
    for (int v = 1; v < WARPS; ++v) m = then(m, as_map(s_sum[REVERSE ? WARPS - 1 - v : v][lane]));
    p.summaries[part * maps_per_part(p) + (int64_t)tile * 32 + lane] = as4(m);
    if (!REVERSE && part == 0) p.start[(int64_t)tile * 32 + lane] = load_state(p.state, b, p.N, c, n_ok);
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
// whether pairs of values can be accessed at once: even offsets everywhere
bool pairs_aligned(const void* p, size_t size, const int64_t* s) {
  return (uintptr_t)p % (2 * size) == 0 && s[0] % 2 == 0 && s[1] % 2 == 0;
}
// A tensor map over [T][B][N] with boxes of `steps` x 64 channels of one sample; false if TMA cannot describe it.
bool tile_map(CUtensorMap* out, const void* base, int dtype_bytes, int dtype, int T, int B, int N, int64_t st, int64_t sb, int steps) {
  tensor_map_encode_fn encode = tensor_map_encoder();
  if (!encode || (uintptr_t)base % 16 != 0) return false;
  // (a stride that is never used may be anything: take one that fits)
  const int64_t row = ((int64_t)N * dtype_bytes + 15) / 16 * 16;
  const int64_t b_bytes = B > 1 ? sb * dtype_bytes : row, t_bytes = T > 1 ? st * dtype_bytes : row * B;
  if (b_bytes % 16 != 0 || t_bytes % 16 != 0 || b_bytes <= 0 || t_bytes <= 0 || b_bytes >= ((int64_t)1 << 40) || t_bytes >= ((int64_t)1 << 40))
    return false;
  const cuuint64_t dims[3] = {(cuuint64_t)N, (cuuint64_t)B, (cuuint64_t)T}, strides[2] = {(cuuint64_t)b_bytes, (cuuint64_t)t_bytes};
  const cuuint32_t box[3] = {SCAN_COLS, 1, (cuuint32_t)steps}, elem[3] = {1, 1, 1};
  const CUtensorMapDataType type = dtype < 0                     ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                   : dtype == SNN_DTYPE_FP32     ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == SNN_DTYPE_BF16     ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                                 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encode(out, type, 3, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool value_map(CUtensorMap* out, const void* base, const snn_scan_args* a, const int64_t* s, int steps) {
  return tile_map(out, base, (int)dtype_size(a->dtype), a->dtype, a->T, a->B, a->N, s[0], s[1], steps);
}
bool code_map(CUtensorMap* out, const uint8_t* base, const snn_scan_args* a, int steps) {
  return tile_map(out, base, 1, -1, a->T, a->B, a->N, (int64_t)a->B * a->N, a->N, steps);
}
// the kernels' template arguments: the value type and the path
template <typename F> snn_status by_path(int path, F&& f) {
  if (path == TILES) return f(std::integral_constant<int, TILES>());
  return path == PAIRS ? f(std::integral_constant<int, PAIRS>()) : f(std::integral_constant<int, SCALAR>());
}
template <typename F> snn_status by_type(int dtype, int path, F&& f) {
  return by_path(path, [&](auto is_path) {
    if (dtype == SNN_DTYPE_FP32) return f(float(), is_path);
    return dtype == SNN_DTYPE_BF16 ? f(__nv_bfloat16(), is_path) : f(__half(), is_path);
  });
}

snn_status check_common(const snn_scan_args* a) {
  if (!a || a->T < 0 || a->B < 0 || a->N < 0 || a->T >= (1 << 30) || !dtype_known(a->dtype)) return SNN_ERR_INVALID_ARG;
  if (a->mode != SNN_SCAN_SIGMOID && a->mode != SNN_SCAN_DIRECT) return SNN_ERR_INVALID_ARG;
  for (int f : {a->x_format, a->gate_format})
    if (f < SNN_KEEP_RAW || f > SNN_KEEP_E4M3) return SNN_ERR_INVALID_ARG;
  if (a->mode == SNN_SCAN_DIRECT && a->gate_format != SNN_KEEP_RAW) return SNN_ERR_UNSUPPORTED;
  if (a->N > INT32_MAX - (SCAN_COLS - 1)) return SNN_ERR_UNSUPPORTED;   // (the last tile of channels ends within 32 bits)
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
  p.polls = MBAR_WAIT_LIMIT;
  return p;
}
// Segments of the time axis: as many as fill the device once (`resident` blocks fit an SM), each with two turns at least.
// Below four segments one is as fast: what the SMs left idle would win goes into reading the inputs twice and into a second
// launch (2048 x 2 x 4096 bf16, 128 tiles: 43 us with one segment, 42 with three, 41 with four; 4096 x 2 x 512, 16 tiles: 80 and 18).
void cut_time(ScanParams& p, int resident) {
  const int64_t tiles = std::max<int64_t>((int64_t)p.B * p.n_tiles, 1);
  int64_t n = std::min<int64_t>(148 * resident / tiles, p.T / (2 * SNN_SCAN_CHUNK));
  if (n < 4) n = 1;
  p.segment_steps = (int)((((int64_t)p.T + n - 1) / n + SNN_SCAN_CHUNK - 1) / SNN_SCAN_CHUNK * SNN_SCAN_CHUNK);
  p.segments = p.segment_steps ? (p.T + p.segment_steps - 1) / p.segment_steps : 1;
  // the summary's blocks wait for their loads, and more than fit at once share the work more evenly: parts as long as a
  // warp has 128 steps (65536 x 1 x 2048 bf16 backward, 912 steps per warp with one part: 516, 493, 469, 470 us with 1, 2,
  // 4, 8; 65536 x 1 x 1024, 456 steps: 211, 195, 196, 196; forward, 304 steps: 144, 142, 145, 150)
  p.parts = 1;
  while (p.parts < 4 && p.segment_steps >= 2 * p.parts * WARPS * 128) p.parts *= 2;
}
// Blocks per SM: a forward pass that keeps nothing fits a fourth one of 16-bit values (65536 x 1 x 1024 bf16: 142 us with
// segments for three, 133 for four).  fp32: two, but one where states are kept (the tiles and the room for two copies in 8 bits
// take 119 KB); it is cut as for two all the same, and its segments take two turns on the device.
int resident_blocks(int dtype, bool backward, bool keep) {
  if (dtype == SNN_DTYPE_FP32) return backward ? 1 : 2;
  return backward ? 2 : keep ? 3 : 4;
}
size_t map_bytes(const ScanParams& p) { return sizeof(float4) * 32 * (size_t)p.segments * p.parts * p.B * p.n_tiles; }
size_t summary_bytes(const ScanParams& p) { return p.segments > 1 ? map_bytes(p) + sizeof(float2) * 32 * (size_t)p.B * p.n_tiles : 0; }

snn_status set_segments(ScanParams& p, const snn_scan_args* a, bool backward) {
  cut_time(p, resident_blocks(a->dtype, backward, a->states != nullptr));
  if (p.segments == 1) return SNN_OK;
  if (a->workspace_bytes < summary_bytes(p)) return SNN_ERR_WORKSPACE_TOO_SMALL;
  if (!a->workspace || (uintptr_t)a->workspace % 256 != 0) return SNN_ERR_INVALID_ARG;
  p.summaries = (float4*)a->workspace;
  p.start = (float2*)((char*)a->workspace + map_bytes(p));
  return SNN_OK;
}
template <typename K> snn_status launch(K kernel, size_t smem, int64_t blocks, const ScanParams& p, cudaStream_t stream) {
  if (blocks > INT32_MAX) return SNN_ERR_UNSUPPORTED;
  if (smem && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
    return cudaGetLastError(), SNN_ERR_CUDA;
  kernel<<<(unsigned)blocks, 32 * WARPS, smem, stream>>>(p);
  return launched();
}

struct WaitTest {   // of snn_selftest_scan_wait
  int step;
  bool quits;
  uint32_t polls;
};
void set_limits(ScanParams& p, const WaitTest* test, int never) {
  p.loads_end = p.quits_at = never;
  if (!test) return;
  p.polls = test->polls;
  (test->quits ? p.quits_at : p.loads_end) = test->step;
}

}  // namespace

extern "C" snn_status snn_scan_workspace(const snn_scan_args* a, int32_t backward, size_t* bytes) {
  const snn_status st = check_common(a);
  if (st != SNN_OK) return st;
  if (!bytes) return SNN_ERR_INVALID_ARG;
  ScanParams p = params_of(a);
  *bytes = 0;
  for (bool keep : {false, true}) {   // enough for either forward pass
    cut_time(p, resident_blocks(a->dtype, backward != 0, keep));
    *bytes = std::max(*bytes, summary_bytes(p));
  }
  return SNN_OK;
}

namespace {
snn_status forward(const snn_scan_args* a, const WaitTest* test, void* stream) {
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
  const bool pairs = a->N % 2 == 0 && pairs_aligned(p.x, size, p.xs) && pairs_aligned(p.gate, size, p.gs) && pairs_aligned(p.h, size, p.hs) &&
                     (uintptr_t)p.x_codes % 2 == 0 && (uintptr_t)p.gate_codes % 2 == 0;
  const cudaStream_t s = (cudaStream_t)stream;
  if (!keep && a->T <= SCAN_SHORT) {
    const int64_t blocks = ((int64_t)p.B * ((p.N + 1) / 2) + 127) / 128;
    if (blocks > INT32_MAX) return SNN_ERR_UNSUPPORTED;
    return by_type(a->dtype, pairs ? PAIRS : SCALAR, [&](auto io, auto path) {
      scan_short_kernel<decltype(io), decltype(path)::value == PAIRS><<<(unsigned)blocks, 128, 0, s>>>(p);
      return launched();
    });
  }
  set_limits(p, test, INT32_MAX);
  const snn_status cut = set_segments(p, a, false);
  if (cut != SNN_OK) return cut;
  const bool tiles = pairs && value_map(&p.in[0], p.x, a, p.xs, SNN_SCAN_CHUNK) && value_map(&p.in[1], p.gate, a, p.gs, SNN_SCAN_CHUNK) &&
                     value_map(&p.out[0], p.h, a, p.hs, SCAN_K) && (p.x_format == SNN_KEEP_RAW || code_map(&p.out[2], p.x_codes, a, SCAN_K)) &&
                     (p.gate_format == SNN_KEEP_RAW || code_map(&p.out[3], p.gate_codes, a, SCAN_K));
  return by_type(a->dtype, tiles ? TILES : pairs ? PAIRS : SCALAR, [&](auto io, auto path) {
    using IO = decltype(io);
    constexpr int PATH = decltype(path)::value;
    const int64_t blocks = (int64_t)p.B * p.n_tiles;
    auto go = [&](auto is_keep) {
      constexpr bool KEEP = decltype(is_keep)::value;
      const size_t ring = PATH != TILES ? 0 : SCAN_DEPTH * forward_slot<IO>(), out = PATH == TILES ? 2 * WARPS * forward_out<IO, KEEP>() : 0;
      return launch(scan_forward_kernel<IO, KEEP, PATH>, ring + out, blocks * p.segments, p, s);
    };
    if (p.segments > 1) {
      const snn_status st = launch(scan_summary_kernel<IO, PATH != SCALAR, false>, 0, blocks * (p.segments - 1) * p.parts, p, s);
      if (st != SNN_OK) return st;
    }
    return keep ? go(std::true_type()) : go(std::false_type());
  });
}

snn_status backward(const snn_scan_args* a, const WaitTest* test, void* stream) {
  const snn_status st = check_common(a);
  if (st != SNN_OK) return st;
  if (a->B == 0 || a->N == 0) return SNN_OK;
  const bool raw_x = a->x_format == SNN_KEEP_RAW, raw_gate = a->gate_format == SNN_KEEP_RAW;
  if (a->T > 0) {
    if (!a->dh || !a->dx || !a->dgate || !a->states) return SNN_ERR_INVALID_ARG;
    if (raw_x ? !a->x : !a->x_codes || !a->x_scales) return SNN_ERR_INVALID_ARG;
    if (raw_gate ? !a->gate : !a->gate_codes || !a->gate_scales) return SNN_ERR_INVALID_ARG;
  }
  ScanParams p = params_of(a);
  const size_t size = dtype_size(a->dtype);
  const bool pairs = a->N % 2 == 0 && pairs_aligned(p.dh, size, p.dhs) && pairs_aligned(p.dx, size, p.dxs) && pairs_aligned(p.dgate, size, p.dgs) &&
                     (!raw_x || pairs_aligned(p.x, size, p.xs)) && (!raw_gate || pairs_aligned(p.gate, size, p.gs)) &&
                     (uintptr_t)p.x_codes % 2 == 0 && (uintptr_t)p.gate_codes % 2 == 0;
  set_limits(p, test, -1);
  const snn_status cut = set_segments(p, a, true);
  if (cut != SNN_OK) return cut;
  const bool tiles = pairs && a->T > 0 && value_map(&p.in[0], p.dh, a, p.dhs, SNN_SCAN_CHUNK) &&
                     (raw_x ? value_map(&p.in[1], p.x, a, p.xs, SNN_SCAN_CHUNK) : code_map(&p.in[1], p.x_codes, a, SNN_SCAN_CHUNK)) &&
                     (raw_gate ? value_map(&p.in[2], p.gate, a, p.gs, SNN_SCAN_CHUNK) : code_map(&p.in[2], p.gate_codes, a, SNN_SCAN_CHUNK)) &&
                     value_map(&p.out[0], p.dx, a, p.dxs, SCAN_K) && value_map(&p.out[1], p.dgate, a, p.dgs, SCAN_K);
  return by_type(a->dtype, tiles ? TILES : pairs ? PAIRS : SCALAR, [&](auto io, auto path) {
    using IO = decltype(io);
    constexpr int PATH = decltype(path)::value;
    const size_t values = PIECE * sizeof(IO), slot = values + (raw_x ? values : PIECE) + (raw_gate ? values : PIECE);
    const size_t ring = PATH != TILES ? 0 : SCAN_DEPTH * slot, out = PATH == TILES ? 2 * WARPS * 2 * WARP_PIECE * sizeof(IO) : 0;
    const int64_t blocks = (int64_t)p.B * p.n_tiles;
    if (p.segments > 1) {
      const snn_status st = launch(scan_summary_kernel<IO, PATH != SCALAR, true>, 0, blocks * (p.segments - 1) * p.parts, p, (cudaStream_t)stream);
      if (st != SNN_OK) return st;
    }
    return launch(scan_backward_kernel<IO, PATH>, ring + out, blocks * p.segments, p, (cudaStream_t)stream);
  });
}
}  // namespace

extern "C" snn_status snn_scan_forward(const snn_scan_args* a, void* stream) { return forward(a, nullptr, stream); }
extern "C" snn_status snn_scan_backward(const snn_scan_args* a, void* stream) { return backward(a, nullptr, stream); }

extern "C" snn_status snn_selftest_scan_wait(const snn_scan_args* a, int32_t is_backward, int32_t step, int32_t quits, uint32_t poll_limit,
                                             void* stream) {
  if (step < 0 || poll_limit == 0 || poll_limit > MBAR_WAIT_LIMIT) return SNN_ERR_INVALID_ARG;
  if (!WAIT_TESTS) return SNN_ERR_UNSUPPORTED;
  const WaitTest test{step, quits != 0, poll_limit};
  return is_backward ? backward(a, &test, stream) : forward(a, &test, stream);
}
