// One step of beam search over a vocabulary, and the beams' states in their new order (include/snn.h, "sequence-model operators").
//
//   score(k, v) = s_k + (z_kv - m_k) - log sum_v exp(z_kv - m_k),  m_k = max_v z_kv;  the best `width` of a sample, lower k V + v first
//
// Bound by HBM: the logits are read once.  A warp walks through a part of a beam's row, segment by segment of 2 KB, and leaves
// behind its maximum, its sum of exponentials and its `width` best classes; a second kernel, a block per sample, joins the parts
// of each row and the rows of the sample; a third moves the states.  Each is set up while the one before it runs.
//
// The best of a part: maxima that lanes have seen give a bound that at least `width` values of the row reach, and few more do.
// What reaches it is put aside; where that gets too much, the best of it are kept and are the bound.
//
// Measured, the best 8 of 64 x 8 rows of 131072 (a fifth of them ended): fp32 45 us (4.8 TB/s of what is read); bf16, none ended,
// 42 us, bound by instructions (12 a value, and what each waits for the one before it).  The best 32: 71 and 61 to 79 us; with
// a bound from 32 maxima instead of 64, and the best taken one after the other, 104 and 111.  Blocks of eight warps at segments of
// 16 KB waited for one another (fp32 76 us); warps that did not share their bound put more aside (53 and 71 us).
//
// Keys hold the value above the complement of the class, so that no two are the same and ties go to the lower class.
#include <algorithm>

#include "unit.cuh"

using namespace snnk;

namespace {

constexpr int BM_WARPS = 8, BM_STAGES = 3, BM_CANDIDATES = 88, BM_HELD = 64;   // of a block; of a warp, and between segments
constexpr int BM_MOST = 32;          // beams of a sample, and survivors
constexpr int BM_JOIN_WARPS = 8;
constexpr int BM_TABLE = 64;         // states of one launch
constexpr int BM_COPY_THREADS = 256;
constexpr int BM_PIECE = 16 * 1024, BM_PIECE_IN_PLACE = 1024;   // bytes of a row at a time

struct BeamParams {
  int64_t rows, parts;
  int K, W, V, splits, length;        // a row is cut into `splits` parts of `length` segments
  int64_t sample_stride, beam_stride, end;
  const void* logits;
  const float* scores;
  const uint8_t* ended;
  uint64_t* keys;                    // [rows][splits][W], falling; 0: none
  float2* stats;                     // [rows][splits]: maximum, sum of exp(z - maximum)
  int64_t *tokens, *parents;         // [B][W]
  float* new_scores;
  uint8_t* new_ended;
};

__device__ __forceinline__ uint32_t rising(float v) {   // unsigned numbers that order as finite values do; -0 is 0
  const uint32_t u = __float_as_uint(v + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_rising(uint32_t r) { return __uint_as_float(r & 0x80000000u ? r ^ 0x80000000u : ~r); }
__device__ __forceinline__ uint64_t key_of(float v, uint32_t c) { return (uint64_t)rising(v) << 32 | (0xffffffffu - c); }
__device__ __forceinline__ uint32_t class_of(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
  const uint32_t high = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
  const uint32_t low = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32) == high ? (uint32_t)v : 0u);
  return (uint64_t)high << 32 | low;
}
// Whether a beam goes on to other classes than the end's: it has not ended, and its score is a number.
__device__ __forceinline__ bool goes_on(const BeamParams& p, int64_t row) {
  return !(p.ended && p.ended[row]) && fabsf(p.scores[row]) <= largest_finite<float>();
}

// The largest of m and a pair, without notice of NaN.
__device__ __forceinline__ float larger_number(float m, float2 v) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(m), "f"(v.x), "f"(v.y));
  return d;
}
// A segment's place in shared memory, and the values of a lane: fp32 classes lane + 32 j, 16-bit ones 2 lane + 64 j and the next,
// whatever the address of the row (so that equal rows have equal sums).  The bytes lie as in the row, 16 by 16: class 0 of the
// segment stands `lead` values behind the start.
template <typename IO> struct Segment {
  static constexpr int VALUES = 64 / sizeof(IO), CLASSES = 32 * VALUES, PER_COPY = 16 / sizeof(IO), BYTES = CLASSES * sizeof(IO) + 16;
  // Starts the copies of classes c0 .. of a row of V; 16 bytes that reach beyond the row's ends are read value by value.
  static __device__ __forceinline__ void fetch(uint8_t* to, const IO* z, int64_t c0, int V) {
    const int lead = (int)((uintptr_t)(z + c0) % 16 / sizeof(IO)), lane = threadIdx.x & 31;
    if (c0 >= lead && c0 + CLASSES + PER_COPY <= V) {   // all of them lie within the row
      const uint32_t at = (uint32_t)__cvta_generic_to_shared(to) + 16 * lane;
      const IO* const from = z + c0 - lead + PER_COPY * lane;
#pragma unroll
      for (int i = 0; i < CLASSES / PER_COPY / 32; ++i) copy_16(at + 16 * 32 * i, from + PER_COPY * 32 * i);
      if (lead && lane == 0) copy_16(at + 16 * (CLASSES / PER_COPY), from + CLASSES);
      return;
    }
    const int here = (int)min((int64_t)CLASSES, V - c0), copies = (lead + here + PER_COPY - 1) / PER_COPY;
    for (int i = lane; i < copies; i += 32) {
      const int64_t c = c0 + i * PER_COPY - lead;
      if (c >= 0 && c + PER_COPY <= V) {
        copy_16((uint32_t)__cvta_generic_to_shared(to + 16 * i), z + c);
      } else {
        for (int j = 0; j < PER_COPY; ++j)
          if (c + j >= 0 && c + j < V) reinterpret_cast<IO*>(to)[i * PER_COPY + j] = z[c + j];
      }
    }
  }
  using Raw = typename Pair<IO>::raw;
  Raw raw[VALUES / 2];    // what does not exist is -infinity: never a candidate, as what is masked
  const IO* at;           // class 0 of the segment in shared memory
  int here;               // classes that exist
  __device__ __forceinline__ void read(const uint8_t* from, const IO* z, int64_t c0, int V) {
    const int lead = (int)((uintptr_t)(z + c0) % 16 / sizeof(IO));
    const IO none = from_f32<IO>(__uint_as_float(0xff800000u));
    here = (int)min((int64_t)CLASSES, V - c0);
    at = reinterpret_cast<const IO*>(from) + lead;
    if (here == CLASSES) {
      if (sizeof(IO) == 2 && lead % 2 == 0) {
#pragma unroll
        for (int i = 0; i < VALUES / 2; ++i) raw[i] = *reinterpret_cast<const Raw*>(at + place(2 * i));
      } else {
#pragma unroll
        for (int i = 0; i < VALUES / 2; ++i) raw[i].x = at[place(2 * i)], raw[i].y = at[place(2 * i + 1)];
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < VALUES / 2; ++i) {
      const int a = place(2 * i), b = place(2 * i + 1);
      raw[i].x = a < here ? at[a] : none;
      raw[i].y = b < here ? at[b] : none;
    }
  }
  static __device__ __forceinline__ int place(int j) { return place(j, threadIdx.x & 31); }
  static __device__ __forceinline__ int place(int j, int lane) {
    return sizeof(IO) == 2 ? 2 * lane + j / 2 * 64 + j % 2 : lane + j * 32;
  }
  __device__ __forceinline__ float2 pair(int i) const { return to_f32(raw[i]); }
  // without notice of NaN, but where there is nothing else
  __device__ __forceinline__ float most_of_eight(int q) const {
    if constexpr (sizeof(IO) == 4) {
      return larger_number(larger_number(larger_number(fmaxf(raw[4 * q].x, raw[4 * q].y), raw[4 * q + 1]), raw[4 * q + 2]), raw[4 * q + 3]);
    } else {
      const float2 m = to_f32(__hmax2(__hmax2(raw[4 * q], raw[4 * q + 1]), __hmax2(raw[4 * q + 2], raw[4 * q + 3])));
      return fmaxf(m.x, m.y);
    }
  }
  // Value j of a lane once more, from shared memory: few are looked at again, and registers are worth more than they.
  __device__ __forceinline__ float again(int j, int lane) const {
    const int c = place(j, lane);
    return c < here ? to_f32(at[c]) : __uint_as_float(0xff800000u);
  }
};
__device__ __forceinline__ float exp2_of(float v) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
  return e;
}
constexpr float LOG2_E = 1.4426950408889634f;

// The best `width` of a warp's first n candidates, falling, to their beginning: each to the place that the number of larger ones
// gives it.  (Taking the largest of all `width` times waits for one result after the other.)
template <int EACH> __device__ __forceinline__ int best_candidates(uint64_t* candidates, int n, int width) {
  const int lane = threadIdx.x & 31;
  uint64_t mine[EACH];
  int before[EACH];
  __syncwarp();
#pragma unroll
  for (int k = 0; k < EACH; ++k) mine[k] = lane + 32 * k < n ? candidates[lane + 32 * k] : 0, before[k] = 0;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const uint64_t key = candidates[i];
#pragma unroll
    for (int k = 0; k < EACH; ++k) before[k] += key > mine[k];
  }
  __syncwarp();
#pragma unroll
  for (int k = 0; k < EACH; ++k)
    if (mine[k] && before[k] < width) candidates[before[k]] = mine[k];
  __syncwarp();
  return min(n, width);
}
__device__ __forceinline__ int best_candidates(uint64_t* candidates, int n, int width) {
  return n <= 32 ? best_candidates<1>(candidates, n, width) : best_candidates<(BM_CANDIDATES + 31) / 32>(candidates, n, width);
}
// A number that the width-th largest of the lanes' numbers, two of each, reaches, and is close to: it is built bit by bit from the
// highest one in which they differ, nine of them, or the upper half where the signs or much of the exponents differ.
__device__ __forceinline__ uint32_t largest_of_lanes(uint32_t a, uint32_t b, int width) {
  const uint32_t most = __reduce_max_sync(0xffffffffu, max(a, b)), least = __reduce_min_sync(0xffffffffu, min(a, b));
  if (most == least) return most;
  const int top = 31 - __clz(most ^ least);
  uint32_t found = most & ~(0xffffffffu >> (31 - top));
  for (int bit = top, last = min(16, max(top - 8, 0)); bit >= last; --bit) {
    const uint32_t next = found | 1u << bit;
    if (__popc(__ballot_sync(0xffffffffu, a >= next)) + __popc(__ballot_sync(0xffffffffu, b >= next)) >= width) found = next;
  }
  return found;
}

// (Four blocks an SM for 16-bit types, 38 to 43 us against 42 to 45; fp32 with as many took 49 to 51 instead of 43, its registers spilled.)
// A warp: `length` segments of a row, one behind the other through a ring of BM_STAGES places of its own in shared memory.
template <typename IO> __global__ void __launch_bounds__(32 * BM_WARPS, sizeof(IO) == 2 ? 4 : 3) beam_rows_kernel(const BeamParams p) {
  using Seg = Segment<IO>;
  constexpr int VALUES = Seg::VALUES;
  extern __shared__ __align__(16) uint8_t ring_of_all[];
  __shared__ uint64_t candidates_of_all[BM_WARPS][BM_CANDIDATES];
  __shared__ float most_of_all[BM_WARPS][2][32];   // the lanes' maxima so far, of two halves of their values
  let_next_kernel_start();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t part = (int64_t)blockIdx.x * BM_WARPS + warp, row = part / p.splits;
  most_of_all[warp][0][lane] = most_of_all[warp][1][lane] = __uint_as_float(0xff800000u);
  __syncthreads();
  if (part >= p.parts || !goes_on(p, row)) return;
  uint8_t* const ring = ring_of_all + warp * (BM_STAGES * Seg::BYTES);
  uint64_t* const candidates = candidates_of_all[warp];
  const IO* const z = (const IO*)p.logits + row / p.K * p.sample_stride + row % p.K * p.beam_stride;
  const int64_t first = (part - row * p.splits) * p.length * Seg::CLASSES;
  // the warps of the block that work at the same row
  const int from = (int)max((int64_t)0, warp - (part - row * p.splits)), to = (int)min((int64_t)BM_WARPS, warp + (row + 1) * p.splits - part);
  const int segments = (int)min((int64_t)p.length, (p.V - first + Seg::CLASSES - 1) / Seg::CLASSES);
  auto fetch = [&](int s) {
    if (s < segments) Seg::fetch(ring + s % BM_STAGES * Seg::BYTES, z, first + (int64_t)s * Seg::CLASSES, p.V);
    close_group();
  };
#pragma unroll
  for (int s = 0; s < BM_STAGES - 1; ++s) fetch(s);
  const float none = __uint_as_float(0xff800000u);
  float most = none, sum = 0.f;        // of this lane's values: the maximum, and the sum of exp(v - maximum)
  float half[2] = {none, none};        // maxima of values 0 .. 7, 16 .. 23 of the segments, and of the others
  float bound = none;                  // candidates are values at or above it, all of them finite
  int count = 0;                       // candidates so far
  for (int s = 0; s < segments; ++s) {
    wait_groups<BM_STAGES - 2>();
    __syncwarp();                      // the segment is there for all lanes, and the one before it has been read by all
    fetch(s + BM_STAGES - 1);
    const int64_t c0 = first + (int64_t)s * Seg::CLASSES;
    Seg g;
    g.read(ring + s % BM_STAGES * Seg::BYTES, z, c0, p.V);
    float now[2] = {none, none};
#pragma unroll
    for (int q = 0; q < VALUES / 8; ++q) now[q % 2] = fmaxf(now[q % 2], g.most_of_eight(q));
    const float here = fmaxf(now[0], now[1]);
    if (here > most) {
      sum *= exp2_of((most - here) * LOG2_E);   // (0 of a sum that is 0)
      most = here;
    }
    if (most > none) {
      // (the difference first: it is exact where the values are near one another, which is where it counts)
      float2 more = both(0.f);
#pragma unroll
      for (int i = 0; i < VALUES / 2; ++i) {
        const float2 d = mul_pair(add_pair(g.pair(i), both(-most)), both(LOG2_E));
        more = add_pair(more, make_float2(exp2_of(d.x), exp2_of(d.y)));
      }
      sum += more.x + more.y;
    } else {   // masked places alone, or NaN, of which the maximum takes no notice
#pragma unroll
      for (int i = 0; i < VALUES / 2; ++i)
        if (g.pair(i).x != g.pair(i).x || g.pair(i).y != g.pair(i).y) sum = __uint_as_float(0x7fc00000u);
    }
    // The largest of what a half of lane l of each of the row's warps has seen: the width-th largest of these 64 is a bound that at
    // least `width` values of the row reach (and 44 of a row in any order, where width is 32; of 32 numbers the least had 130).
    // It is taken again when the part that has been read has doubled.  (Another warp's maximum may be an older one: the bound is
    // lower then, not wrong.)
#pragma unroll
    for (int h = 0; h < 2; ++h) half[h] = fmaxf(half[h], now[h]);
    if ((s & (s + 1)) == 0) {
      float m[2] = {half[0], half[1]};
#pragma unroll
      for (int h = 0; h < 2; ++h) *(volatile float*)&most_of_all[warp][h][lane] = half[h];
      for (int w = from; w < to; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) m[h] = fmaxf(m[h], *(const volatile float*)&most_of_all[w][h][lane]);
      const float least = from_rising(largest_of_lanes(rising(m[0]), rising(m[1]), p.W));
      bound = fmaxf(bound, fmaxf(least, -largest_finite<float>()));
    }
    // Lanes that have seen a value at or above the bound are few, mostly one: all lanes look at the values of one such lane (two of
    // fp32) again, a value each.
    uint32_t passing = __ballot_sync(0xffffffffu, here >= bound);
    if (!passing) continue;
    const int held = count;
    while (passing) {
      int from_lane = __ffs(passing) - 1;
      passing &= passing - 1u;
      if (VALUES == 16) {
        if (lane >= 16) from_lane = __ffs(passing) - 1;   // (-1: no second one)
        passing &= passing - 1u;
      }
      const int j = lane % VALUES;
      const float v = from_lane >= 0 ? g.again(j, from_lane) : none;
      const uint32_t passed = __ballot_sync(0xffffffffu, v >= bound);
      const int at = count + __popc(passed & ((1u << lane) - 1u));
      if (v >= bound && at < BM_CANDIDATES) candidates[at] = key_of(v, (uint32_t)(c0 + Seg::place(j, from_lane)));
      count += __popc(passed);
    }
    if (count <= BM_HELD) continue;
    if (count <= BM_CANDIDATES) {
      count = best_candidates(candidates, count, p.W);
    } else {
      // too many at or above the bound (equal values, or rising ones): the next best of the candidates that were there before and of
      // all values of the segment, one after the other
      __syncwarp();
      const uint64_t old[2] = {lane < held ? candidates[lane] : 0, lane + 32 < held ? candidates[lane + 32] : 0};
      __syncwarp();
      uint64_t last = ~(uint64_t)0;
      for (count = 0; count < p.W; ++count) {
        uint64_t best = old[0] < last ? old[0] : 0;
        if (old[1] < last && old[1] > best) best = old[1];
        for (int j = 0; j < VALUES; ++j) {
          const float v = g.again(j, lane);
          const uint64_t key = v >= bound ? key_of(v, (uint32_t)(c0 + Seg::place(j))) : 0;
          if (key < last && key > best) best = key;
        }
        last = warp_max(best);
        if (!last) break;
        if (lane == 0) candidates[count] = last;
      }
      __syncwarp();
    }
    // a later class has to be larger, not equal
    if (count == p.W) bound = fmaxf(from_rising((uint32_t)(candidates[p.W - 1] >> 32) + 1), -largest_finite<float>());
  }
  count = best_candidates(candidates, count, p.W);
  uint64_t* const out = p.keys + part * p.W;
  if (lane < p.W) out[lane] = lane < count ? candidates[lane] : 0;
  float m = most;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float total = most > none ? sum * exp2_of((most - m) * LOG2_E) : sum;
#pragma unroll
  for (int o = 16; o > 0; o /= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) p.stats[part] = make_float2(m, total);
}

// A block per sample: the rows of its beams from their segments, a warp each, then the sample from its rows.
__global__ void __launch_bounds__(32 * BM_JOIN_WARPS) beam_join_kernel(const BeamParams p) {
  __shared__ uint64_t keys_of[BM_MOST * BM_MOST];   // the best of each beam, [K][W]
  __shared__ uint64_t scores_of[BM_MOST * BM_MOST]; // their scores, as whole numbers that order alike; 0: none
  __shared__ float row_max[BM_MOST];
  __shared__ double row_base[BM_MOST];              // score less log sum
  __shared__ int64_t found[BM_MOST];
  __shared__ int valid;
  extern __shared__ uint8_t heads_of_all[];
  let_next_kernel_start();
  wait_for_kernel_before();
  const int64_t b = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  uint8_t* const heads = heads_of_all + warp * p.splits;
  for (int k = warp; k < p.K; k += warps) {
    const int64_t row = b * p.K + k;
    if (!goes_on(p, row)) {
      // an ended beam goes on with the end alone, at its own score
      const bool stays = p.ended && p.ended[row] && fabsf(p.scores[row]) <= largest_finite<float>();
      for (int r = lane; r < p.W; r += 32) keys_of[k * p.W + r] = r == 0 && stays ? key_of(0.f, (uint32_t)p.end) : 0;
      if (lane == 0) row_max[k] = 0.f, row_base[k] = (double)p.scores[row];
      continue;
    }
    float m = __uint_as_float(0xff800000u);
    for (int l = lane; l < p.splits; l += 32) m = fmaxf(m, p.stats[row * p.splits + l].x);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    double total = 0.0;
    for (int l = lane; l < p.splits; l += 32) {
      const float2 s = p.stats[row * p.splits + l];
      if (s.y != 0.f) total += (double)s.y * (double)exp2_of((s.x - m) * LOG2_E);   // (a segment without a value has a sum of zero)
      heads[l] = 0;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
    const bool alive = total > 0.0 && total < INFINITY;   // (not where it is NaN)
    if (lane == 0) {
      // log(2^e f) with f from 0.7 to 1.4, where the logarithm in fp32 is off by 2^-25 at most
      int e;
      double f = frexp(total, &e);
      if (f < 0.70710678) f *= 2.0, --e;
      row_max[k] = m, row_base[k] = (double)p.scores[row] - (e * 0.6931471805599453 + (double)logf((float)f) + (f - (double)(float)f) / f);
    }
    __syncwarp();
    const uint64_t* const keys = p.keys + row * p.splits * p.W;
    // a lane looks after the lists lane, lane + 32, ..; the largest of their first keys is taken, `width` times.  Where it has
    // one list, the key behind the first one is already here when that is taken.
    uint64_t here = 0, behind = 0;
    int from = 0;
    const bool one = p.splits <= 32;
    auto key_at = [&](int l, int at) { return at < p.W ? keys[(int64_t)l * p.W + at] : 0; };
    auto look = [&]() {
      here = 0;
      for (int l = lane; l < p.splits; l += 32) {
        const uint64_t key = key_at(l, heads[l]);
        if (key > here) here = key, from = l;
      }
    };
    if (one) {
      if (lane < p.splits) here = key_at(lane, 0), behind = key_at(lane, 1);
      from = 1;
    } else {
      look();
    }
    for (int r = 0; r < p.W; ++r) {
      const uint64_t best = alive ? warp_max(here) : 0;
      if (lane == 0) keys_of[k * p.W + r] = best;
      if (best && best == here) {
        if (one) {
          here = behind;
          behind = key_at(lane, ++from);
        } else {
          ++heads[from];
          look();
        }
      }
      __syncwarp();
    }
  }
  if (threadIdx.x == 0) valid = 0;
  __syncthreads();
  const int all = p.K * p.W;
  for (int i = threadIdx.x; i < all; i += blockDim.x) {
    const uint64_t key = keys_of[i];
    const int k = i / p.W;
    uint64_t order = 0;
    if (key) {
      const double score = row_base[k] + ((double)from_rising((uint32_t)(key >> 32)) - (double)row_max[k]) + 0.0;
      const uint64_t u = (uint64_t)__double_as_longlong(score);
      order = u ^ ((uint64_t)((int64_t)u >> 63) | (uint64_t)1 << 63);
      atomicAdd(&valid, 1);
    }
    scores_of[i] = order;
  }
  __syncthreads();
  auto write = [&](int at, int64_t flat, float score) {
    const int64_t k = flat / p.V, c = flat % p.V, to = b * p.W + at;
    p.tokens[to] = c;
    p.parents[to] = k;
    p.new_scores[to] = score;
    if (p.new_ended) p.new_ended[to] = (p.ended && p.ended[b * p.K + k]) || c == p.end;
    found[at] = flat;
  };
  // each to the place that the number of better ones gives it; of equal scores the lower beam's is first, and a beam's own list
  // is in its order
  for (int i = threadIdx.x; i < all; i += blockDim.x) {
    const uint64_t order = scores_of[i];
    if (!order) continue;
    int before = 0;
    for (int j = 0; j < all; ++j) before += scores_of[j] > order || (scores_of[j] == order && j < i);
    if (before >= p.W) continue;
    const uint64_t u = order & (uint64_t)1 << 63 ? order ^ (uint64_t)1 << 63 : ~order;
    write(before, (int64_t)(i / p.W) * p.V + class_of(keys_of[i]), (float)__longlong_as_double((int64_t)u));
  }
  if (valid >= p.W) return;
  __syncthreads();
  if (threadIdx.x > 0) return;
  // fewer continuations than survivors: all of them are here, and the others, at -infinity, follow in their order
  int n = valid;
  for (int64_t flat = 0; n < p.W; ++flat) {
    bool taken = false;
    for (int i = 0; i < n; ++i) taken = taken || found[i] == flat;
    if (!taken) write(n++, flat, __uint_as_float(0xff800000u));
  }
}

// ---- rows in the order of their parents ------------------------------------------------------------------------
struct RowsOf {
  const uint8_t* from;
  uint8_t* to;
  int64_t bytes;                // of a row
  int64_t tile;                 // number of its first tile
  int64_t pieces;               // of a row
  int32_t unit, in_place;       // bytes of an access; from == to
};
struct ReorderParams {
  int count, K, W;
  int64_t tiles;
  const int64_t* parents;       // [B][W]
  RowsOf t[BM_TABLE];
};
// A piece of one row.
template <typename U> __device__ __forceinline__ void copy_piece(const RowsOf& t, const ReorderParams& p, int64_t row, int64_t begin) {
  const int64_t sample = row / p.W, parent = p.parents[row];
  const int units = (int)(min((int64_t)BM_PIECE, t.bytes - begin) / sizeof(U));
  const bool exists = parent >= 0 && parent < p.K;
  const U* const from = reinterpret_cast<const U*>(t.from + (sample * p.K + (exists ? parent : 0)) * t.bytes + begin);
  U* const to = reinterpret_cast<U*>(t.to + row * t.bytes + begin);
#pragma unroll 4
  for (int i = threadIdx.x; i < units; i += BM_COPY_THREADS) to[i] = exists ? from[i] : U{};
}
// A piece of all rows of a sample, through shared memory: all of them are read before one is written.
template <typename U> __device__ __forceinline__ void exchange_piece(const RowsOf& t, const ReorderParams& p, int64_t sample, int64_t begin, U* held) {
  const int units = (int)(min((int64_t)BM_PIECE_IN_PLACE, t.bytes - begin) / sizeof(U));
  uint8_t* const rows = t.to + sample * p.K * t.bytes + begin;
  for (int k = 0; k < p.K; ++k)
    for (int i = threadIdx.x; i < units; i += BM_COPY_THREADS) held[k * units + i] = reinterpret_cast<const U*>(rows + k * t.bytes)[i];
  __syncthreads();
  for (int w = 0; w < p.W; ++w) {
    const int64_t k = p.parents[sample * p.W + w];
    if (k == w) continue;
    for (int i = threadIdx.x; i < units; i += BM_COPY_THREADS) reinterpret_cast<U*>(rows + w * t.bytes)[i] = k >= 0 && k < p.K ? held[k * units + i] : U{};
  }
  __syncthreads();
}
template <typename U> __device__ __forceinline__ void reorder_piece(const RowsOf& t, const ReorderParams& p, int64_t tile, void* stage) {
  if (t.in_place)
    exchange_piece<U>(t, p, tile / t.pieces, tile % t.pieces * BM_PIECE_IN_PLACE, (U*)stage);
  else
    copy_piece<U>(t, p, tile / t.pieces, tile % t.pieces * BM_PIECE);
}
__global__ void __launch_bounds__(BM_COPY_THREADS) reorder_rows_kernel(const __grid_constant__ ReorderParams p) {
  extern __shared__ uint4 stage[];
  wait_for_kernel_before();
  for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
    int low = 0, high = p.count;
    while (high - low > 1) {
      const int mid = (low + high) / 2;
      if (p.t[mid].tile <= tile)
        low = mid;
      else
        high = mid;
    }
    const RowsOf& t = p.t[low];
    if (t.unit == 16)
      reorder_piece<uint4>(t, p, tile - t.tile, stage);
    else if (t.unit == 4)
      reorder_piece<uint32_t>(t, p, tile - t.tile, stage);
    else
      reorder_piece<uint8_t>(t, p, tile - t.tile, stage);
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
struct Split {
  int length, splits;
};
// Parts of as many segments as still give every warp that the device holds one of them, and no more than 32 (one list of the best for
// each lane that joins them) where that leaves at least half of them one.
Split split_of(int64_t rows, int V, int dtype) {
  const int64_t classes = 32 * 64 / (int64_t)dtype_size(dtype), segments = (V + classes - 1) / classes;
  int64_t length = 32;
  while (length > 1 && rows * ((segments + length - 1) / length) < 148 * 24) length /= 2;
  while ((segments + length - 1) / length > 32 && rows * ((segments + 2 * length - 1) / (2 * length)) >= 148 * 8) length *= 2;
  while ((segments + length - 1) / length > 1024) length *= 2;   // (whose heads the joining kernel keeps in shared memory)
  return {(int)length, (int)((segments + length - 1) / length)};
}
snn_status check(const snn_beam_args* a) {
  if (!a || a->B < 0 || a->K < 1 || a->W < 1 || a->V < 1 || !dtype_known(a->dtype)) return SNN_ERR_INVALID_ARG;
  if ((int64_t)a->K * a->V < a->W || a->end < -1 || a->end >= a->V || (a->end < 0 && (a->ended || a->new_ended))) return SNN_ERR_INVALID_ARG;
  if (a->K > BM_MOST || a->W > BM_MOST || a->V > 1 << 22) return SNN_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)a->B * a->K;
  if (rows * split_of(rows, a->V, a->dtype).splits > INT32_MAX) return SNN_ERR_UNSUPPORTED;
  return SNN_OK;
}
struct Layout {
  size_t stats, total;
};
Layout layout_of(const snn_beam_args* a) {
  const int64_t rows = (int64_t)a->B * a->K;
  const size_t lists = (size_t)rows * split_of(rows, a->V, a->dtype).splits;
  const size_t keys = (lists * a->W * 8 + 255) / 256 * 256;
  return {keys, keys + (lists * 8 + 255) / 256 * 256};
}
snn_status check_rows(const snn_state_rows* t, int32_t count, int32_t K, int32_t W) {
  if (count < 0 || (count > 0 && !t)) return SNN_ERR_INVALID_ARG;
  for (int k = 0; k < count; ++k) {
    if (t[k].row_bytes < 0 || t[k].row_bytes > (int64_t)1 << 50) return SNN_ERR_INVALID_ARG;
    if (t[k].row_bytes > 0 && (!t[k].from || !t[k].to || (t[k].from == t[k].to && K != W))) return SNN_ERR_INVALID_ARG;
  }
  return SNN_OK;
}
snn_status reorder(const snn_state_rows* t, int32_t count, const int64_t* parents, int64_t B, int K, int W, cudaStream_t stream, bool behind) {
  ReorderParams p{};
  p.K = K, p.W = W, p.parents = parents;
  for (int k = 0; k < count;) {
    p.count = 0, p.tiles = 0;
    bool staged = false;
    for (; k < count && p.count < BM_TABLE; ++k) {
      if (t[k].row_bytes == 0) continue;
      const uintptr_t all = (uintptr_t)t[k].from | (uintptr_t)t[k].to | (uintptr_t)t[k].row_bytes;
      const bool in_place = t[k].from == t[k].to;
      staged = staged || in_place;
      const int64_t piece = in_place ? BM_PIECE_IN_PLACE : BM_PIECE, pieces = (t[k].row_bytes + piece - 1) / piece;
      p.t[p.count++] = {(const uint8_t*)t[k].from, (uint8_t*)t[k].to, t[k].row_bytes, p.tiles, pieces, all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1, in_place};
      p.tiles += pieces * B * (in_place ? 1 : W);
    }
    if (p.tiles == 0) continue;
    const snn_status st = launch_behind(reorder_rows_kernel, (unsigned)std::min<int64_t>(p.tiles, 148 * 8), BM_COPY_THREADS, staged ? (size_t)K * BM_PIECE_IN_PLACE : 0, stream, behind, p);
    if (st != SNN_OK) return st;
    behind = false;
  }
  return SNN_OK;
}
template <typename IO> snn_status launch_rows(const BeamParams& p, cudaStream_t stream) {
  constexpr int SMEM = BM_WARPS * BM_STAGES * Segment<IO>::BYTES;
  if (!allow_shared<beam_rows_kernel<IO>>(SMEM)) return SNN_ERR_CUDA;
  return launch_behind(beam_rows_kernel<IO>, (unsigned)((p.parts + BM_WARPS - 1) / BM_WARPS), 32 * BM_WARPS, SMEM, stream, false, p);
}
}  // namespace

extern "C" snn_status snn_beam_workspace(const snn_beam_args* a, size_t* bytes) {
  const snn_status st = check(a);
  if (st != SNN_OK) return st;
  if (!bytes) return SNN_ERR_INVALID_ARG;
  *bytes = layout_of(a).total;
  return SNN_OK;
}

extern "C" snn_status snn_beam_step(const snn_beam_args* a, void* stream) {
  snn_status st = check(a);
  if (st == SNN_OK) st = check_rows(a->states, a->n_states, a->K, a->W);
  if (st != SNN_OK) return st;
  if (a->B == 0) return SNN_OK;
  if (!a->logits || !a->scores || !a->tokens || !a->parents || !a->new_scores || !aligned_to(a->logits, dtype_size(a->dtype))) return SNN_ERR_INVALID_ARG;
  if (!a->workspace || !aligned_to(a->workspace, 256)) return SNN_ERR_INVALID_ARG;
  const Layout l = layout_of(a);
  if (a->workspace_bytes < l.total) return SNN_ERR_WORKSPACE_TOO_SMALL;
  BeamParams p{};
  p.rows = (int64_t)a->B * a->K;
  const Split s = split_of(p.rows, a->V, a->dtype);
  p.K = a->K, p.W = a->W, p.V = a->V, p.splits = s.splits, p.length = s.length, p.parts = p.rows * s.splits, p.sample_stride = a->sample_stride, p.beam_stride = a->beam_stride, p.end = a->end;
  p.logits = a->logits, p.scores = a->scores, p.ended = a->ended;
  p.keys = (uint64_t*)a->workspace, p.stats = (float2*)((char*)a->workspace + l.stats);
  p.tokens = a->tokens, p.parents = a->parents, p.new_scores = a->new_scores, p.new_ended = a->new_ended;
  const cudaStream_t on = (cudaStream_t)stream;
  st = a->dtype == SNN_DTYPE_FP32   ? launch_rows<float>(p, on)
       : a->dtype == SNN_DTYPE_BF16 ? launch_rows<__nv_bfloat16>(p, on)
                                    : launch_rows<__half>(p, on);
  if (st != SNN_OK) return st;
  const int warps = std::min(a->K, BM_JOIN_WARPS);
  st = launch_behind(beam_join_kernel, (unsigned)a->B, 32 * warps, (size_t)warps * s.splits, on, true, p);
  if (st != SNN_OK) return st;
  return reorder(a->states, a->n_states, a->parents, a->B, a->K, a->W, on, true);
}

extern "C" snn_status snn_reorder_rows(const snn_state_rows* states, int32_t count, const int64_t* parents, int32_t B, int32_t K, int32_t W, void* stream) {
  const snn_status st = check_rows(states, count, K, W);
  if (st != SNN_OK) return st;
  if (B < 0 || K < 1 || W < 1 || (B > 0 && count > 0 && !parents)) return SNN_ERR_INVALID_ARG;
  if (K > BM_MOST || W > BM_MOST) return SNN_ERR_UNSUPPORTED;
  return B == 0 ? SNN_OK : reorder(states, count, parents, B, K, W, (cudaStream_t)stream, false);
}
