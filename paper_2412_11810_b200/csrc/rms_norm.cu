// Root-mean-square norm with the residual's addition (include/snn.h, "sequence-model operators").
//
//   h = x + residual, rounded to the type;  s = 1 / sqrt(mean(h^2) + eps);  y = h s w
//   with g = dy w, c = mean(g h s):  dx = s (g - h s c) + dh,  dw = sum over the rows of dy h s
//
// Bound by HBM: every value is read and written once.  A row belongs to `lanes` threads (part of a warp, or whole warps) that
// hold one or two units each (unit.cuh) in registers, so that the second use of h costs no second read; the loads of the next row
// are on their way while one is finished.  Within a warp nothing waits for a block.  Rows that do not fit (16384 values of a
// 16-bit type, 8192 of fp32) are read a second time, from L2.
//
// Measured, bf16 with residual: 32768 x 2048 forward 80 us (6.7 TB/s), backward 84 us (6.4 TB/s) and 6 us for dw from the blocks'
// shares; 16384 x 4096 to int8 alone 77 us (6.1 TB/s; 68 with codes that were rounded twice, 73 with ties and limits of scales left to
// chance).  Units of 16 bytes and a row per block and launch, without the next row's loads, took 112, 115 and 108 us: they were bound by
// instructions (42 a value).  Rows that vectors do not fit: 16384 x 4090
// 190 us (pairs; 359 us with eight lanes a group, whose accesses spread over as many lines).
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "unit.cuh"

using namespace snnk;

namespace {

constexpr int RMS_THREADS = 256;      // of a block whose rows need no more than a warp
constexpr int RMS_MOST_LANES = 512, RMS_WIDE = 1024;   // threads of a row; of one that does not fit registers
constexpr size_t RMS_SUMS = 192 * 1024;                // bytes of such a row's sums for dw in shared memory

struct RmsParams {
  int64_t rows;
  int n, groups, lanes, keep_format;
  float eps, inverse_n;
  double inverse;                     // 1 / n
  const void *x, *residual, *weight, *dy, *dh;
  int64_t x_stride, residual_stride, h_stride, y_stride, dy_stride, dh_stride, dx_stride;
  void *h, *y, *dx;
  float* rstd;
  uint8_t *codes, *scales;
  float* partial;                     // [blocks][n]: each block's share of dw
};

// The sum over the lanes of a row, the same bits for all of them, of type T.  `turn` counts the calls: two buffers take turns, so
// that one barrier a call is enough.
struct Sums {
  double in64;
  float in32;
};
template <bool BLOCK, typename T> __device__ __forceinline__ T row_sum(T v, int lanes, int turn, Sums (*shared)[32]) {
  for (int o = 1; o < (BLOCK ? 32 : lanes); o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  if constexpr (BLOCK) {
    T* const buffer = reinterpret_cast<T*>(shared[turn & 1]);
    if ((threadIdx.x & 31) == 0) buffer[threadIdx.x >> 5] = v;
    __syncthreads();
    v = buffer[0];
    for (int k = 1; k < lanes / 32; ++k) v += buffer[k];
  }
  return v;
}
// The same of both at once: that in 32 bits has the bits of the one above.
template <bool BLOCK> __device__ __forceinline__ Sums row_sums(Sums s, int lanes, int turn, Sums (*shared)[32]) {
  for (int o = 1; o < (BLOCK ? 32 : lanes); o *= 2) s.in64 += __shfl_xor_sync(0xffffffffu, s.in64, o), s.in32 += __shfl_xor_sync(0xffffffffu, s.in32, o);
  if constexpr (BLOCK) {
    Sums* const buffer = shared[turn & 1];
    if ((threadIdx.x & 31) == 0) buffer[threadIdx.x >> 5] = s;
    __syncthreads();
    s = buffer[0];   // (two at a time: four take 15 registers more, and with 104 fp32 rows by pairs have three blocks an SM instead of four)
#pragma unroll 2
    for (int k = 1; k < lanes / 32; ++k) s.in64 += buffer[k].in64, s.in32 += buffer[k].in32;
  }
  return s;
}
__device__ __forceinline__ float scale_of(float sum, const RmsParams& p) { return rsqrtf(sum * p.inverse_n + p.eps); }
// A row's scale and what it is off by: with a copy in 8 bits the lanes' sums are joined in 64 bits, and two steps of Newton's iteration
// leave 1 / sqrt of them in 64 bits, so that codes are those of the formula.  (Of the scale in fp32 alone, and y rounded before it was
// coded, one code in a million was the one beside it.)  Where mean and root are numbers of few bits, they are found: the quotient has
// its remainder added, and the second step ends at such a root, which the first one passes by 2^-44.
// The values and rstd take a scale from sums in 32 bits, with a copy in 8 bits as without one: they have the same bits in both calls.
// (Sums in 64 bits for all calls cost 1 % of 32768 x 2048, and 4 % where a row's threads wait for one another, 16384 x 4090.)
struct Scale {
  float rounded;             // that of the values
  float value, rest, down;   // 1 / sqrt(mean + eps) = (value + rest) down
};
__device__ __forceinline__ double root_inverse(double m) {
  double s = (double)rsqrtf((float)m);
#pragma unroll
  for (int k = 0; k < 2; ++k) s = fma(s * 0.5, fma(-(m * s), s, 1.0), s);
  return s;
}
__device__ __forceinline__ double mean_of(double sum, const RmsParams& p) {
  const double q = sum * p.inverse;
  return fma(fma(-q, (double)p.n, sum), p.inverse, q);
}
__device__ __forceinline__ Scale scale_of(double sum, const RmsParams& p) {
  const double s = root_inverse(mean_of(sum, p) + (double)p.eps);
  const float value = (float)s;
  return {value, value, (float)(s - (double)value), 1.f};
}
// Where squares leave the range of fp32 they are summed again of values times 2^-80: that of the largest row is finite, and
// eps, at most one, is nothing beside it.  The scale, down to 2^-128, is held times 2^32: as it is it would be subnormal.  An infinity
// in the row leaves a scale of zero, NaN a NaN.
constexpr float RMS_DOWN = 0x1p-80f, RMS_SCALE_DOWN = 0x1p-32f;
__device__ __forceinline__ Scale scale_of_far(double sum, const RmsParams& p) {
  if (!(sum <= (double)largest_finite<float>())) return {rsqrtf((float)sum), rsqrtf((float)sum), 0.f, 1.f};
  const double s = root_inverse(mean_of(sum, p)) * 0x1p-48;
  const float value = (float)s;
  return {value * RMS_SCALE_DOWN, value, (float)(s - (double)value), RMS_SCALE_DOWN};
}

// Which row of a turn of its block a thread works at, which of the row's threads it is, and its columns.  (Less than a warp a row: by
// vectors only.)
template <bool BLOCK, int ACCESS, int N> struct Place {
  int slot, t, lanes, n;
  __device__ __forceinline__ explicit Place(const RmsParams& p) : lanes(p.lanes), n(p.n) {
    slot = BLOCK ? 0 : threadIdx.x / p.lanes;
    t = BLOCK ? threadIdx.x : threadIdx.x % p.lanes;
  }
  __device__ __forceinline__ int per_block() const { return BLOCK ? 1 : RMS_THREADS / lanes; }
  __device__ __forceinline__ Columns<ACCESS, N> columns(int i) const {   // of the thread's i-th unit
    return {((t & ~31) + i * lanes) * N + Columns<ACCESS, N>::of_lane(t & 31), n};
  }
};
// A number that is not exact has its lowest bit set, where y has been rounded toward zero: it lies neither on a border between two codes
// nor on that between two scales then, and is rounded but once.
__device__ __forceinline__ float2 inexact(float2 v) { return make_float2(__uint_as_float(__float_as_uint(v.x) | 1u), __uint_as_float(__float_as_uint(v.y) | 1u)); }
// (what left fp32 was cut to its largest value)
__device__ __forceinline__ uint32_t top_of_cut(uint32_t top) { return top == 0x7f7fffffu ? 0x7f800000u : top; }
// The 8-bit codes of a unit y, rounded as above; the lanes of a warp do this together.
template <int FORMAT, int ACCESS, int N> __device__ __forceinline__ void keep_unit(const float2 y[N / 2], int64_t row, Columns<ACCESS, N> at, const RmsParams& p, bool store) {
  uint8_t* const codes = p.codes + row * p.n + at.first;
  uint8_t* const scales = p.scales + row * p.groups;
  if constexpr (ACCESS == VECTORS) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) m = larger_of(m, y[i]);
    const uint32_t top = top_of_cut(group_top<KEEP_GROUP / N>(m)), byte = keep_scale_byte<FORMAT>(top);
    const float inverse = keep_scale_inverse(byte);
    // (rarely: a group whose largest value could round up to 128, or one that is not finite)
    const bool rare = __any_sync(0xffffffffu, byte == 255u || keep_needs_cut<FORMAT>(top));
    uint32_t q[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) q[i] = __byte_perm(encode_pair<FORMAT>(y[2 * i], inverse, rare), encode_pair<FORMAT>(y[2 * i + 1], inverse, rare), 0x5410);
    if (rare && byte == 255u) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) q[i] = 0u;
    }
    if (!store || !at.exists(0)) return;
    if constexpr (N == 16)
      *reinterpret_cast<uint4*>(codes) = make_uint4(q[0], q[1], q[2], q[3]);
    else
      *reinterpret_cast<uint2*>(codes) = make_uint2(q[0], q[1]);
    if (at.first % KEEP_GROUP == 0) scales[at.first / KEEP_GROUP] = (uint8_t)byte;
  } else {
    // group k of the unit: a pair of each lane, or two values 32 places apart.  All lanes know its scale; lane k keeps it.
    const int lane = threadIdx.x & 31, start = at.first - Columns<ACCESS, N>::of_lane(lane);
    uint32_t mine = 0u;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      if (start + k * KEEP_GROUP >= p.n) break;
      const uint32_t top = top_of_cut(__reduce_max_sync(0xffffffffu, __float_as_uint(larger_of(0.f, y[k])))), byte = keep_scale_byte<FORMAT>(top);
      const uint32_t q = byte == 255u ? 0u : encode_pair<FORMAT>(y[k], keep_scale_inverse(byte), keep_needs_cut<FORMAT>(top));
      if (lane == k) mine = byte;
      if (!store) continue;
      if (ACCESS == PAIRS) {
        if (at.exists(2 * k)) *reinterpret_cast<uint16_t*>(codes + at.behind(2 * k)) = (uint16_t)q;
      } else {
        if (at.exists(2 * k)) codes[at.behind(2 * k)] = (uint8_t)q;
        if (at.exists(2 * k + 1)) codes[at.behind(2 * k + 1)] = (uint8_t)(q >> 8);
      }
    }
    if (store && lane < N / 2 && start + lane * KEEP_GROUP < p.n) scales[start / KEEP_GROUP + lane] = (uint8_t)mine;
  }
}
// y of one unit of h, as values, as codes, or both.  For codes, h s w is computed with what h s and the scale are off by, and
// rounded toward zero.  With h of 16 bits the upper 12 bits of s have an exact product, and the others are a correction.
template <typename IO, typename WT, int ACCESS, int N>
__device__ __forceinline__ void finish_unit(const Unit<IO, N>& h, const Unit<WT, N>& w, Scale scale, int64_t row, Columns<ACCESS, N> at, const RmsParams& p, bool store) {
  if (p.y && store) {
    Unit<IO, N> out;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 y = mul_pair(h.pair(i), both(scale.rounded));
      out.set(i, p.weight ? mul_pair(y, w.pair(i)) : y);
    }
    at.store(out, (IO*)p.y + row * p.y_stride);
  }
  if (p.keep_format == SNN_KEEP_RAW) return;
  const float upper = sizeof(IO) == 2 ? __uint_as_float(__float_as_uint(scale.value) & 0xfffff000u) : scale.value;
  const float lower = scale.value - upper + scale.rest;
  // v s = first + rest
  auto product = [&](float2 v, float2& first, float2& rest) {
    first = mul_pair(v, both(upper));
    if constexpr (sizeof(IO) == 2)
      rest = mul_pair(v, both(lower));
    else
      rest = fma_pair(v, both(lower), fma_pair(v, both(upper), mul_pair(v, both(-upper))));
  };
  float2 y[N / 2];
  if (scale.rest != 0.f && scale.down == 1.f) {
    // A scale of more than 24 bits: so has every product with it, since that of two odd numbers is at least as long as each.
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      float2 first, rest;
      product(h.pair(i), first, rest);
      const float2 weight = p.weight ? w.pair(i) : both(1.f);
      y[i] = inexact(fma_pair_down(first, weight, mul_pair(rest, weight)));
    }
  } else {
    const bool exact = scale.rest == 0.f;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      float2 first, rest;
      product(mul_pair(h.pair(i), both(scale.down)), first, rest);
      const float2 weight = p.weight ? w.pair(i) : both(1.f);
      rest = mul_pair(rest, weight);
      const float2 v = fma_pair_down(first, weight, rest), off = add_pair(fma_pair(first, weight, make_float2(-v.x, -v.y)), rest), up = inexact(v);
      y[i] = make_float2(off.x == 0.f && exact ? v.x : up.x, off.y == 0.f && exact ? v.y : up.y);
    }
  }
  if (p.keep_format == SNN_KEEP_INT8)
    keep_unit<SNN_KEEP_INT8, ACCESS, N>(y, row, at, p, store);
  else
    keep_unit<SNN_KEEP_E4M3, ACCESS, N>(y, row, at, p, store);
}
// Sums of squares of a lane: in 32 bits, and what 64 bits need beside them, so that rows of one magnitude, whose largest y is next to a
// border, come out on the right side of it.  bf16: squares have 16 bits, and a lane adds up few enough of them.  fp16: they have 22 bits, of
// which fp32 holds the sums of four.  fp32: what roundings leave out (all of it where no square is larger than the sum before it).
template <typename IO, int UNITS> struct Squares {
  static constexpr bool FOURS = std::is_same<IO, __half>::value;
  float2 in32{0.f, 0.f}, lost{0.f, 0.f}, fours[UNITS][2];
  __device__ __forceinline__ double in64() const {
    double sum = 0.0;
    if constexpr (FOURS) {
#pragma unroll
      for (int i = 0; i < UNITS; ++i) sum += (double)fours[i][0].x + (double)fours[i][0].y + ((double)fours[i][1].x + (double)fours[i][1].y);
    } else {
      sum = (double)in32.x + (double)in32.y + (double)(lost.x + lost.y);
    }
    return sum;
  }
};
// Unit i of h: that of x, or its sum with the residual's; and its squares, in 64 bits as well where that is asked for.
template <typename IO, int N, int UNITS>
__device__ __forceinline__ void sum_unit(Unit<IO, N>& h, const Unit<IO, N>& r, bool residual, Squares<IO, UNITS>& s, int i, bool in64) {
  if (residual) {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) h.set(k, add_pair(h.pair(k), r.pair(k)));
  }
  if constexpr (Squares<IO, UNITS>::FOURS) {
    static_assert(N == 16, "two times four pairs");
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float2 four = mul_pair(h.pair(4 * j), h.pair(4 * j));
#pragma unroll
      for (int k = 1; k < 4; ++k) four = fma_pair(h.pair(4 * j + k), h.pair(4 * j + k), four);
      s.in32 = add_pair(s.in32, four);
      s.fours[i][j] = four;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      const float2 v = h.pair(k), before = s.in32;
      s.in32 = fma_pair(v, v, before);
      if (std::is_same<IO, float>::value && in64) s.lost = add_pair(s.lost, fma_pair(v, v, fma_pair(s.in32, both(-1.f), before)));
    }
  }
}
template <typename IO, int N> __device__ __forceinline__ void sum_unit_far(const Unit<IO, N>& h, float2& sum) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const float2 v = mul_pair(h.pair(i), both(RMS_DOWN));
    sum = fma_pair(v, v, sum);
  }
}

// BLOCK: a row per block and turn; otherwise a warp holds whole rows.  The loads of the next row are on their way while a row
// is finished; the weight stays in registers.
template <typename IO, typename WT, int ACCESS, int UNITS, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? RMS_MOST_LANES : RMS_THREADS, BLOCK && ACCESS == VECTORS && UNITS == 1 ? 2 : 1) rms_forward_kernel(const RmsParams p) {
  constexpr int N = UNIT<IO>;
  __shared__ Sums shared[2][32];
  const Place<BLOCK, ACCESS, N> at(p);
  const int64_t step = (int64_t)gridDim.x * at.per_block();
  const bool residual = p.residual != nullptr;
  int turn = 0;
  Unit<WT, N> w[UNITS];
  Unit<IO, N> x[UNITS], r[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    x[i].zero(), r[i].zero();   // (and stay so behind the row's end)
    if (!p.weight) continue;
    w[i].zero();
    at.columns(i).load(w[i], (const WT*)p.weight);
  }
  auto load = [&](int64_t row) {
    const IO* const from = (const IO*)p.x + row * p.x_stride;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) at.columns(i).load(x[i], from);
    if (!residual) return;
    const IO* const other = (const IO*)p.residual + row * p.residual_stride;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) at.columns(i).load(r[i], other);
  };
  const int64_t first = (int64_t)blockIdx.x * at.per_block();
  if (first < p.rows) load(min(first + at.slot, p.rows - 1));
  for (int64_t base = first; base < p.rows; base += step) {
    const bool store = base + at.slot < p.rows;   // (a slot without a row repeats the last one and stores nothing)
    const int64_t row = min(base + at.slot, p.rows - 1);
    Unit<IO, N> h[UNITS];
    Squares<IO, UNITS> squares;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      h[i] = x[i];
      sum_unit(h[i], r[i], residual, squares, i, p.keep_format != SNN_KEEP_RAW);
      if (residual && store) at.columns(i).store(h[i], (IO*)p.h + row * p.h_stride);
    }
    if (base + step < p.rows) load(min(base + step + at.slot, p.rows - 1));
    Scale scale;
    float total;
    if (p.keep_format != SNN_KEEP_RAW) {
      const Sums sums = row_sums<BLOCK>({squares.in64(), squares.in32.x + squares.in32.y}, at.lanes, turn++, shared);
      scale = scale_of(sums.in64, p), total = sums.in32;
    } else {
      scale = {}, total = row_sum<BLOCK>(squares.in32.x + squares.in32.y, at.lanes, turn++, shared);
    }
    scale.rounded = scale_of(total, p);
    const bool far = !(total <= largest_finite<float>());
    // (lanes of one warp may hold different rows: they all go the same way, as do all threads of a row's warps)
    if (BLOCK ? far : __any_sync(0xffffffffu, far)) {
      float2 sum = both(0.f);
#pragma unroll
      for (int i = 0; i < UNITS; ++i) sum_unit_far(h[i], sum);
      const double again = row_sum<BLOCK>((double)sum.x + (double)sum.y, at.lanes, turn++, shared);
      if (far) scale = scale_of_far(again, p);
    }
    if (p.rstd && at.t == 0 && store) p.rstd[row] = scale.rounded;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) finish_unit<IO, WT, ACCESS, N>(h[i], w[i], scale, row, at.columns(i), p, store);
  }
}
// A block per row, which is read twice.
template <typename IO, typename WT, int ACCESS> __global__ void __launch_bounds__(RMS_WIDE) rms_forward_wide_kernel(const RmsParams p) {
  constexpr int N = UNIT<IO>;
  using At = Columns<ACCESS, N>;
  __shared__ Sums shared[2][32];
  const int t = threadIdx.x;
  const bool residual = p.residual != nullptr;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const IO* const from = (const IO*)p.x + row * p.x_stride;
    const IO* const again = residual ? (const IO*)p.h + row * p.h_stride : from;
    Squares<IO, 1> squares;
    double fours = 0.0;
    // (a warp whose columns begin behind the last one has nothing to do: its lanes go the same way)
    auto each = [&](auto&& f) {
      for (int64_t start = (t & ~31) * N; start < p.n; start += RMS_WIDE * N) f(At{(int)start + At::of_lane(t & 31), p.n});
    };
    each([&](At at) {
      Unit<IO, N> h, r;
      h.zero(), r.zero();
      at.load(h, from);
      if (residual) at.load(r, (const IO*)p.residual + row * p.residual_stride);
      sum_unit(h, r, residual, squares, 0, true);
      if (Squares<IO, 1>::FOURS) fours += squares.in64();
      if (residual) at.store(h, (IO*)p.h + row * p.h_stride);
    });
    const double total = row_sum<true>(Squares<IO, 1>::FOURS ? fours : squares.in64(), RMS_WIDE, turn++, shared);
    Scale scale = scale_of(total, p);
    if (!(total <= largest_finite<float>())) {
      float2 sum = both(0.f);
      each([&](At at) {
        Unit<IO, N> h;
        h.zero();
        at.load(h, again);
        sum_unit_far(h, sum);
      });
      scale = scale_of_far(row_sum<true>((double)sum.x + (double)sum.y, RMS_WIDE, turn++, shared), p);
    }
    if (p.rstd && t == 0) p.rstd[row] = scale.rounded;
    each([&](At at) {   // (a thread reads back what it stored itself)
      Unit<IO, N> h;
      Unit<WT, N> w;
      h.zero(), w.zero();
      at.load(h, again);
      if (p.weight) at.load(w, (const WT*)p.weight);
      finish_unit<IO, WT, ACCESS, N>(h, w, scale, row, at, p, true);
    });
  }
}

// g = dy w of pair i of a unit.
template <typename IO, typename WT, int N> __device__ __forceinline__ float2 weighted(const Unit<IO, N>& dy, const Unit<WT, N>& w, bool has_weight, int i) {
  return has_weight ? mul_pair(dy.pair(i), w.pair(i)) : dy.pair(i);
}
template <typename IO, typename WT, int ACCESS, int UNITS, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? RMS_MOST_LANES : RMS_THREADS) rms_backward_kernel(const RmsParams p) {
  constexpr int N = UNIT<IO>;
  __shared__ Sums shared[2][32];
  __shared__ float dw_shared[BLOCK ? 1 : 32 * N];
  let_next_kernel_start();
  const Place<BLOCK, ACCESS, N> at(p);
  const int64_t step = (int64_t)gridDim.x * at.per_block();
  const bool has_weight = p.weight != nullptr;
  int turn = 0;
  // the loads of the next row are on their way while a row is worked at, where registers hold both
  constexpr bool AHEAD = ACCESS == VECTORS && UNITS == 1;
  struct Inputs {
    Unit<IO, N> h[UNITS], dy[UNITS], dh[UNITS];
    float scale;
  } now, next;
  float2 dw[UNITS][N / 2];
  Unit<WT, N> w[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    now.h[i].zero(), now.dy[i].zero(), now.dh[i].zero(), w[i].zero();   // (and stay so behind the row's end)
    if (has_weight) at.columns(i).load(w[i], (const WT*)p.weight);
#pragma unroll
    for (int k = 0; k < N / 2; ++k) dw[i][k] = both(0.f);
  }
  auto load = [&](Inputs& in, int64_t row) {
    const IO *const from = (const IO*)p.h + row * p.h_stride, *const from_dy = (const IO*)p.dy + row * p.dy_stride;
    in.scale = p.rstd[row];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) at.columns(i).load(in.h[i], from);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) at.columns(i).load(in.dy[i], from_dy);
    if (!p.dh) return;
    const IO* const from_dh = (const IO*)p.dh + row * p.dh_stride;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) at.columns(i).load(in.dh[i], from_dh);
  };
  next = now;
  if (AHEAD && (int64_t)blockIdx.x * at.per_block() < p.rows) load(next, min((int64_t)blockIdx.x * at.per_block() + at.slot, p.rows - 1));
  for (int64_t base = (int64_t)blockIdx.x * at.per_block(); base < p.rows; base += step) {
    const bool mine = base + at.slot < p.rows;
    const int64_t row = min(base + at.slot, p.rows - 1);
    if (AHEAD) {
      now = next;
      if (base + step < p.rows) load(next, min(base + step + at.slot, p.rows - 1));
    } else {
      load(now, row);
    }
    const float scale = now.scale;
    float2 sum = both(0.f);
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        const float2 n = mul_pair(now.h[i].pair(k), both(scale));
        sum = fma_pair(weighted(now.dy[i], w[i], has_weight, k), n, sum);
        if (BLOCK || mine) dw[i][k] = fma_pair(now.dy[i].pair(k), n, dw[i][k]);
      }
    const float c = row_sum<BLOCK>(sum.x + sum.y, at.lanes, turn++, shared) * p.inverse_n;
    IO* const to = (IO*)p.dx + row * p.dx_stride;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      Unit<IO, N> out;
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        const float2 n = mul_pair(now.h[i].pair(k), both(scale));
        float2 v = mul_pair(fma_pair(n, both(-c), weighted(now.dy[i], w[i], has_weight, k)), both(scale));
        if (p.dh) v = add_pair(v, now.dh[i].pair(k));
        out.set(k, v);
      }
      if (mine) at.columns(i).store(out, to);
    }
  }
  if (!p.partial) return;
  float* const to = p.partial + (int64_t)blockIdx.x * p.n;
  auto each = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) f(at.columns(i).first + Columns<ACCESS, N>::behind(j), j % 2 ? dw[i][j / 2].y : dw[i][j / 2].x);
  };
  if constexpr (BLOCK) {
    each([&](int c, float v) {
      if (c < p.n) to[c] = v;
    });
  } else {   // the rows of a block one behind the other
    for (int k = 0; k < at.per_block(); ++k) {
      if (at.slot == k) each([&](int c, float v) { dw_shared[c] = k == 0 ? v : dw_shared[c] + v; });
      __syncthreads();
    }
    for (int i = threadIdx.x; i < p.n; i += blockDim.x) to[i] = dw_shared[i];
  }
}
// A block per row, which is read twice.  Its share of dw lies in shared memory, each thread's sums at places of its own, or where that
// is too small (in_shared false) in the workspace itself.
template <typename IO, typename WT, int ACCESS> __global__ void __launch_bounds__(RMS_WIDE) rms_backward_wide_kernel(const RmsParams p, bool in_shared) {
  constexpr int N = UNIT<IO>;
  using At = Columns<ACCESS, N>;
  __shared__ Sums shared[2][32];
  extern __shared__ float sums[];
  let_next_kernel_start();
  const int t = threadIdx.x;
  const bool has_weight = p.weight != nullptr;
  int turn = 0;
  float* const to = p.partial ? p.partial + (int64_t)blockIdx.x * p.n : nullptr;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const bool first = row == blockIdx.x;
    const float scale = p.rstd[row];
    float2 sum = both(0.f);
    float c = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      float* mine = sums + t;   // value v of round r: RMS_WIDE (N r + v) on
      for (int64_t start = (t & ~31) * N; start < p.n; start += RMS_WIDE * N, mine += RMS_WIDE * N) {
        const At at{(int)start + At::of_lane(t & 31), p.n};
        Unit<IO, N> h, dy, dh, out;
        Unit<WT, N> w;
        h.zero(), dy.zero(), dh.zero(), w.zero();
        at.load(h, (const IO*)p.h + row * p.h_stride);
        at.load(dy, (const IO*)p.dy + row * p.dy_stride);
        if (has_weight) at.load(w, (const WT*)p.weight);
        if (p.dh && pass) at.load(dh, (const IO*)p.dh + row * p.dh_stride);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) {
          const float2 n = mul_pair(h.pair(k), both(scale)), gw = weighted(dy, w, has_weight, k);
          if (!pass) {
            sum = fma_pair(gw, n, sum);
            continue;
          }
          float2 v = mul_pair(fma_pair(n, both(-c), gw), both(scale));
          if (p.dh) v = add_pair(v, dh.pair(k));
          out.set(k, v);
          if (!to) continue;
          const float2 d = mul_pair(dy.pair(k), n);
          if (in_shared) {
            mine[RMS_WIDE * 2 * k] = first ? d.x : mine[RMS_WIDE * 2 * k] + d.x;
            mine[RMS_WIDE * (2 * k + 1)] = first ? d.y : mine[RMS_WIDE * (2 * k + 1)] + d.y;
          } else {   // (every place of a block's share belongs to one thread)
            const int a = at.first + At::behind(2 * k), b = at.first + At::behind(2 * k + 1);
            if (at.exists(2 * k)) to[a] = first ? d.x : to[a] + d.x;
            if (at.exists(2 * k + 1)) to[b] = first ? d.y : to[b] + d.y;
          }
        }
        if (pass) at.store(out, (IO*)p.dx + row * p.dx_stride);
      }
      if (!pass) c = row_sum<true>(sum.x + sum.y, RMS_WIDE, turn++, shared) * p.inverse_n;
    }
  }
  if (!to || !in_shared) return;
  const float* mine = sums + t;
  for (int64_t start = (t & ~31) * N; start < p.n; start += RMS_WIDE * N, mine += RMS_WIDE * N) {
    const At at{(int)start + At::of_lane(t & 31), p.n};
#pragma unroll
    for (int v = 0; v < N; ++v)
      if (at.exists(v)) to[at.first + At::behind(v)] = mine[RMS_WIDE * v];
  }
}
// dw from the blocks' shares, in an order of its own: 32 columns a block, 32 rows of shares at a time.
template <typename WT> __global__ void __launch_bounds__(1024) rms_dweight_kernel(const float* partial, int blocks, int n, WT* dw) {
  __shared__ float shared[32][33];
  wait_for_kernel_before();
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  float sum = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int b = y; b < blocks; b += 32) sum += partial[(int64_t)b * n + c];
  }
  shared[y][x] = sum;
  __syncthreads();
  sum = shared[x][y];   // column y of the block, share x
#pragma unroll
  for (int o = 1; o < 32; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (x == 0 && blockIdx.x * 32 + y < n) dw[blockIdx.x * 32 + y] = from_f32<WT>(sum);
}

// ---- host ----------------------------------------------------------------------------------------------------
int unit_of(int dtype) { return 32 / (int)dtype_size(dtype); }
struct Shape {
  int lanes, units, threads, blocks;   // units 0: rows that do not fit registers
  bool block;                          // a row per block
};
// One unit a thread where rows are few, so that a row is spread over many threads; two where the rows fill the device with half
// the threads each, so that what a row costs beside its values is shared by more of them.  (Without vectors a second unit only
// means more registers, and a row has a warp at least.)
Shape shape_of(const snn_rms_norm_args* a, int access, bool two, int resident) {
  const int unit = unit_of(a->dtype), groups = (a->n + KEEP_GROUP - 1) / KEEP_GROUP, per_group = KEEP_GROUP / unit;
  Shape s{RMS_WIDE, 0, RMS_WIDE, 0, true};
  for (int units = 1; units <= 2; ++units) {
    const int64_t need = (int64_t)per_group * ((groups + units - 1) / units);
    int lanes = access == VECTORS ? per_group : 32;
    while (lanes < need && lanes < 32) lanes *= 2;
    if (need > 32) lanes = (int)std::min<int64_t>((need + 31) / 32 * 32, INT32_MAX - 31);
    if (lanes > RMS_MOST_LANES) continue;
    if (s.units && (access != VECTORS || !two || need < 32 || a->rows * lanes < 148 * 512)) break;
    const bool block = units > 1 || lanes > 32;
    s = {lanes, units, block ? lanes : RMS_THREADS, 0, block};
  }
  const int64_t per_block = s.threads / s.lanes, turns = (a->rows + per_block - 1) / per_block;
  s.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(turns, (int64_t)148 * std::max(1, (s.units == 2 ? 512 : resident) / s.threads)));
  return s;
}
Shape shape_forward(const snn_rms_norm_args* a, int access) { return shape_of(a, access, true, 1024); }
Shape shape_back(const snn_rms_norm_args* a, int access) { return shape_of(a, access, false, 512); }

snn_status check(const snn_rms_norm_args* a) {
  if (!a || a->rows < 0 || a->n < 1 || !dtype_known(a->dtype)) return SNN_ERR_INVALID_ARG;
  if (a->weight_dtype != a->dtype && a->weight_dtype != SNN_DTYPE_FP32) return SNN_ERR_INVALID_ARG;
  if (a->n > INT32_MAX - (KEEP_GROUP - 1)) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}
bool no_overlap(const snn_rms_norm_args* a, int64_t stride) { return a->rows < 2 || stride >= a->n; }
template <typename F> snn_status by_types(int dtype, int weight_dtype, int access, F&& f) {
  auto with = [&](auto io, auto wt) {
    return access == VECTORS ? f(io, wt, std::integral_constant<int, VECTORS>())
           : access == PAIRS ? f(io, wt, std::integral_constant<int, PAIRS>())
                             : f(io, wt, std::integral_constant<int, SINGLE>());
  };
  if (dtype == SNN_DTYPE_FP32) return with(float(), float());
  if (dtype == SNN_DTYPE_BF16) return weight_dtype == SNN_DTYPE_FP32 ? with(__nv_bfloat16(), float()) : with(__nv_bfloat16(), __nv_bfloat16());
  return weight_dtype == SNN_DTYPE_FP32 ? with(__half(), float()) : with(__half(), __half());
}
// The widest access that all of the rows allow.
struct Rows {
  const void* p;
  int64_t stride;
  int dtype;
};
int access_of(const snn_rms_norm_args* a, std::initializer_list<Rows> all) {
  int access = VECTORS;
  for (const Rows& r : all) access = std::min(access, row_access(r.p, r.stride, a->n, r.dtype, unit_of(a->dtype)));
  return access;
}
}  // namespace

extern "C" snn_status snn_rms_norm_workspace(const snn_rms_norm_args* a, size_t* bytes) {
  const snn_status st = check(a);
  if (st != SNN_OK) return st;
  if (!bytes) return SNN_ERR_INVALID_ARG;
  // (whether rows can be accessed by vectors is not asked here)
  const int blocks = std::max(shape_back(a, VECTORS).blocks, shape_back(a, SINGLE).blocks);
  *bytes = a->rows == 0 ? 0 : ((size_t)blocks * a->n * 4 + 255) / 256 * 256;
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
  p.rows = a->rows, p.n = a->n, p.groups = (a->n + KEEP_GROUP - 1) / KEEP_GROUP, p.keep_format = a->keep_format, p.eps = a->eps, p.inverse_n = 1.f / (float)a->n, p.inverse = 1.0 / a->n;
  p.x = a->x, p.x_stride = a->x_stride, p.residual = a->residual, p.residual_stride = a->residual_stride, p.weight = a->weight;
  p.h = a->h, p.h_stride = a->h_stride, p.y = a->y, p.y_stride = a->y_stride, p.rstd = a->rstd, p.codes = a->codes, p.scales = a->scales;
  int access = access_of(a, {{a->x, a->x_stride, a->dtype}, {a->residual, a->residual_stride, a->dtype}, {a->residual ? a->h : nullptr, a->h_stride, a->dtype},
                             {a->y, a->y_stride, a->dtype}, {a->weight, 0, a->weight_dtype}});
  if (keeps && !aligned_to(a->codes, 16)) access = std::min(access, aligned_to(a->codes, 2) ? (int)PAIRS : (int)SINGLE);
  const Shape s = shape_forward(a, access);
  p.lanes = s.lanes;
  return by_types(a->dtype, a->weight_dtype, access, [&](auto io, auto wt, auto with) {
    using IO = decltype(io);
    using WT = decltype(wt);
    constexpr int ACCESS = decltype(with)::value;
    const auto kernel = s.units == 0   ? rms_forward_wide_kernel<IO, WT, ACCESS>
                        : !s.block     ? rms_forward_kernel<IO, WT, ACCESS, 1, false>
                        : s.units == 1 ? rms_forward_kernel<IO, WT, ACCESS, 1, true>
                                       : rms_forward_kernel<IO, WT, ACCESS, 2, true>;
    return launch_behind(kernel, (unsigned)s.blocks, s.threads, 0, (cudaStream_t)stream, false, p);
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
  const int access = access_of(a, {{a->h, a->h_stride, a->dtype}, {a->dy, a->dy_stride, a->dtype}, {a->dh, a->dh_stride, a->dtype}, {a->dx, a->dx_stride, a->dtype},
                                   {a->weight, 0, a->weight_dtype}});
  const Shape s = shape_back(a, access);
  if (a->dweight) {
    if (!a->workspace || !aligned_to(a->workspace, 256)) return SNN_ERR_INVALID_ARG;
    if (a->workspace_bytes < (size_t)s.blocks * a->n * 4) return SNN_ERR_WORKSPACE_TOO_SMALL;
  }
  RmsParams p{};
  p.rows = a->rows, p.n = a->n, p.groups = (a->n + KEEP_GROUP - 1) / KEEP_GROUP, p.lanes = s.lanes, p.inverse_n = 1.f / (float)a->n, p.weight = a->weight;
  p.h = a->h, p.h_stride = a->h_stride, p.rstd = a->rstd, p.dy = a->dy, p.dy_stride = a->dy_stride, p.dh = a->dh, p.dh_stride = a->dh_stride;
  p.dx = a->dx, p.dx_stride = a->dx_stride, p.partial = a->dweight ? (float*)a->workspace : nullptr;
  const snn_status done = by_types(a->dtype, a->weight_dtype, access, [&](auto io, auto wt, auto with) {
    using IO = decltype(io);
    using WT = decltype(wt);
    constexpr int ACCESS = decltype(with)::value;
    if (s.units == 0) {
      const size_t round = (size_t)RMS_WIDE * UNIT<IO> * 4, sums = (a->n * (size_t)4 + round - 1) / round * round;
      const bool in_shared = a->dweight && sums <= RMS_SUMS;
      if (in_shared && !allow_shared<rms_backward_wide_kernel<IO, WT, ACCESS>>((int)RMS_SUMS)) return SNN_ERR_CUDA;
      return launch_behind(rms_backward_wide_kernel<IO, WT, ACCESS>, (unsigned)s.blocks, s.threads, in_shared ? sums : 0, on, false, p, in_shared);
    }
    const auto kernel = !s.block       ? rms_backward_kernel<IO, WT, ACCESS, 1, false>
                        : s.units == 1 ? rms_backward_kernel<IO, WT, ACCESS, 1, true>
                                       : rms_backward_kernel<IO, WT, ACCESS, 2, true>;
    return launch_behind(kernel, (unsigned)s.blocks, s.threads, 0, on, false, p);
  });
  if (done != SNN_OK || !a->dweight) return done;
  const unsigned tiles = (unsigned)((a->n + 31) / 32);
  if (a->weight_dtype == SNN_DTYPE_FP32) return launch_behind(rms_dweight_kernel<float>, tiles, 1024, 0, on, true, p.partial, s.blocks, a->n, (float*)a->dweight);
  if (a->weight_dtype == SNN_DTYPE_BF16)
    return launch_behind(rms_dweight_kernel<__nv_bfloat16>, tiles, 1024, 0, on, true, p.partial, s.blocks, a->n, (__nv_bfloat16*)a->dweight);
  return launch_behind(rms_dweight_kernel<__half>, tiles, 1024, 0, on, true, p.partial, s.blocks, a->n, (__half*)a->dweight);
}
