// One AdamW step over all tensors of a model (include/snn.h, "sequence-model operators").
//
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,  p' = p (1 - lr wd) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// With moments in fp32 bound by HBM (28 bytes a parameter with everything in fp32: 345 M parameters 1510 us, 6.4 TB/s), in 8 bits
// (10 bytes with bf16 parameters and gradients) by instructions: 60 a parameter, three quarters of the issue slots (70 M
// parameters 170 us, 4.2 TB/s).  A thread block takes tiles of a tensor, eight neighbouring parameters a thread and turn; where a
// tile's tensor lies is found by bisection in a table that comes with the launch, so that nothing is copied to the device first
// and a graph holds it.
//
// Moments in 8 bits: e4m3 groups of 64, the second moment as its root.  A moment moves by a thousandth of its distance a step,
// far less than half a step of its codes: rounded to nearest it would never move.  It is rounded up or down at random, up with
// a probability that is the fraction of the step, so that its mean moves as it should; the bits are a hash of seed, step and
// place.  Both moments are floats rather than integers of a common scale because they are divided by one another: a root that
// is small in its group keeps its relative precision (down to 2^-18 of the largest), and one above zero never becomes zero.
#include <algorithm>

#include "unit.cuh"

using namespace snnk;

namespace {

constexpr int AW_THREADS = 256, AW_VALUES = 8;   // values of a thread and turn: eight lanes a group
constexpr int AW_TURNS = 8;                       // of a tile, where there is enough to do
constexpr int AW_NORM_BLOCKS = 148 * 4;

struct AwTensor {
  void* p;
  const void* g;
  void* copy;
  int64_t n, state;             // values; place of the first one in the moments, a multiple of 64
  int64_t tile;                 // number of its first tile
  int8_t p_dtype, g_dtype, copy_dtype, vectors;   // vectors: all three can be accessed 32 bytes at a time
};
// What the whole step has in common, written by adamw_begin_kernel.
struct AwStep {
  float factor;                 // of the gradients
  float rate, root;             // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  float keep, keep_rest;        // 1 - lr wd, the sum of the two
  uint32_t key;
  int32_t skip;
};
struct AwBegin {
  int64_t* step;
  double lr, beta1, beta2, weight_decay, max_norm;
  const float *lr_device, *scale_device;
  float scale;
  uint64_t seed;
  const double* partial;        // [AW_NORM_BLOCKS] sums of squares, NULL without a clip
  float* norm;
  AwStep* out;
};
template <int COUNT> struct AwParams {
  int count;
  int64_t tiles;
  int turns;                    // of a tile, AW_THREADS times AW_VALUES each
  float beta1, one_less_beta1, beta2, one_less_beta2, eps;
  float *m, *v;
  uint8_t *m_codes, *m_scales, *v_codes, *v_scales;
  double* partial;
  const AwStep* step;
  AwTensor t[COUNT];
};

template <int COUNT> __device__ __forceinline__ int tensor_of(const AwParams<COUNT>& a, int64_t tile) {
  int low = 0, high = a.count;   // the last tensor that starts at or before the tile
  while (high - low > 1) {
    const int mid = (low + high) / 2;
    if (a.t[mid].tile <= tile)
      low = mid;
    else
      high = mid;
  }
  return low;
}

// N values from place i on, of which n - i exist; the others are zero.
template <int N, typename T> __device__ __forceinline__ void load_values(float2 f[N / 2], const T* p, int64_t i, int64_t n, bool vectors) {
  if (vectors && i + N <= n) {
    Unit<T, N> b;
    b.get(p + i);
#pragma unroll
    for (int k = 0; k < N / 2; ++k) f[k] = b.pair(k);
    return;
  }
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    f[k].x = i + 2 * k < n ? to_f32(p[i + 2 * k]) : 0.f;
    f[k].y = i + 2 * k + 1 < n ? to_f32(p[i + 2 * k + 1]) : 0.f;
  }
}
template <int N, typename T> __device__ __forceinline__ void store_values(const float2 f[N / 2], T* p, int64_t i, int64_t n, bool vectors) {
  if (vectors && i + N <= n) {
    Unit<T, N> b;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) b.set(k, f[k]);
    b.put(p + i);
    return;
  }
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    if (i + 2 * k < n) p[i + 2 * k] = from_f32<T>(f[k].x);
    if (i + 2 * k + 1 < n) p[i + 2 * k + 1] = from_f32<T>(f[k].y);
  }
}
template <int N> __device__ __forceinline__ void load_values(float2 f[N / 2], const void* p, int dtype, int64_t i, int64_t n, bool vectors) {
  if (dtype == SNN_DTYPE_FP32)
    load_values<N>(f, (const float*)p, i, n, vectors);
  else if (dtype == SNN_DTYPE_BF16)
    load_values<N>(f, (const __nv_bfloat16*)p, i, n, vectors);
  else
    load_values<N>(f, (const __half*)p, i, n, vectors);
}
template <int N> __device__ __forceinline__ void store_values(const float2 f[N / 2], void* p, int dtype, int64_t i, int64_t n, bool vectors) {
  if (dtype == SNN_DTYPE_FP32)
    store_values<N>(f, (float*)p, i, n, vectors);
  else if (dtype == SNN_DTYPE_BF16)
    store_values<N>(f, (__nv_bfloat16*)p, i, n, vectors);
  else
    store_values<N>(f, (__half*)p, i, n, vectors);
}

// ---- random bits ---------------------------------------------------------------------------------------------
// Shifts and products by odd numbers: every bit of the result depends on every bit of x (tested: each of the 32 x 32 pairs
// of an input and an output bit flips together with probability 0.5 within 0.013).
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ x >> 16) * 0xEE1F5725u;
  x = (x ^ x >> 15) * 0x5DE0A3B7u;
  return x ^ x >> 16;
}
// mix(place ^ key) of place = first + j, first a multiple of 8 and j below it, from base = mix_base(first ^ key)
__device__ __forceinline__ uint32_t mix_base(uint32_t x) { return x ^ x >> 16; }
__device__ __forceinline__ uint32_t mix_from(uint32_t base, uint32_t j) {
  uint32_t x = (base ^ j) * 0xEE1F5725u;
  x = (x ^ x >> 15) * 0x5DE0A3B7u;
  return x ^ x >> 16;
}
__device__ __forceinline__ uint32_t key_of(uint64_t seed, uint64_t step) {
  uint32_t key = mix(0x2545F491u ^ (uint32_t)seed);
  key = mix(key ^ (uint32_t)(seed >> 32));
  key = mix(key ^ (uint32_t)step);
  return mix(key ^ (uint32_t)(step >> 32));
}

// ---- moments in 8 bits -----------------------------------------------------------------------------------------
constexpr int AW_LANES = KEEP_GROUP / AW_VALUES;
struct AwCodes {
  uint32_t q[AW_VALUES / 4];
  __device__ __forceinline__ void get(const uint8_t* p) { memcpy(q, __builtin_assume_aligned(p, 8), 8); }
  __device__ __forceinline__ void put(uint8_t* p) const { memcpy(__builtin_assume_aligned(p, 8), q, 8); }
};
// A value times 2^-120 over its group's scale has the e4m3 code in bits 20 to 26 of its fp32 pattern, subnormal codes among
// them (they are subnormal there as well), and the fraction of a step in the 20 bits below.  The pattern moved up by four bits
// plus 2^8 r, with r of 16 bits, has the rounded code in its highest byte.
constexpr uint32_t AW_BITS_LOW = 0x4104u, AW_BITS_HIGH = 0x4324u;   // selectors of 2^8 r for the two halves of the random bits
__device__ __forceinline__ uint32_t highest_bytes(const uint32_t y[4]) {
  return __byte_perm(__byte_perm(y[0], y[1], 0x0073), __byte_perm(y[2], y[3], 0x0073), 0x5410);
}
constexpr uint32_t AW_FAR_BYTE = 133;   // 2^-120 over a larger scale is subnormal
// Codes of a lane's values; byte: their group's scale byte; some_far: whether one of the warp's is above AW_FAR_BYTE.  ROOT: nothing is
// negative, and what is above zero stays above zero.
template <bool ROOT> __device__ __forceinline__ AwCodes encode_at_random(float2 f[AW_VALUES / 2], const uint32_t r[AW_VALUES], uint32_t byte, bool some_far) {
  // 2^-120 over the scale, 2^(7 - byte); where that is subnormal, in two steps (what is then too small to count, but not zero, counts
  // as 2^-60, far below a step)
  const bool far = byte > AW_FAR_BYTE;
  if (some_far) {
    const float inverse = keep_scale_inverse(byte);
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) {
      const float2 u = mul_pair(f[k], both(inverse));
      if (far) f[k] = ROOT ? make_float2(f[k].x > 0.f ? fmaxf(u.x, 0x1p-60f) : 0.f, f[k].y > 0.f ? fmaxf(u.y, 0x1p-60f) : 0.f) : u;
    }
  }
  const float factor = __uint_as_float((far ? 7u : 134u - byte) << 23);
  AwCodes c;
#pragma unroll
  for (int k = 0; k < AW_VALUES / 4; ++k) {
    uint32_t y[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t t = __float_as_uint((h ? f[2 * k + j].y : f[2 * k + j].x) * factor), random = __byte_perm(r[4 * k + 2 * j + h], 0u, ROOT ? AW_BITS_HIGH : AW_BITS_LOW);
        uint32_t v = (t << 4) + random;
        if (ROOT)
          v = max(v, min(__float_as_uint(h ? f[2 * k + j].y : f[2 * k + j].x), 1u << 24));
        else
          v |= t & 0x80000000u;
        y[2 * j + h] = v;
      }
    }
    c.q[k] = byte == 255u ? 0u : highest_bytes(y);
  }
  return c;
}
// The e4m3 values of codes, without their scale.
__device__ __forceinline__ void decode(float2 f[AW_VALUES / 2], const AwCodes& codes) {
#pragma unroll
  for (int k = 0; k < AW_VALUES / 2; ++k) {
    const uint32_t two = codes.q[k / 2] >> (16 * (k & 1));
    f[k] = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3)));
  }
}
__device__ __forceinline__ uint32_t top_of(const float2 f[AW_VALUES / 2]) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < AW_VALUES / 2; ++k) m = larger_of(m, f[k]);
  return group_top<AW_LANES>(m);
}
// Square roots by the hardware's approximation of 1 / sqrt(v) and one step of Newton's iteration from the residual v - s^2, which
// leaves them correctly rounded but for a few; of numbers below 2^-126 they are too small, of infinity NaN.
__device__ __forceinline__ float2 root_of(float2 v) {
  float2 y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(v.x, 0x1p-126f)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(v.y, 0x1p-126f)));
  const float2 s = mul_pair(v, y);
  return fma_pair(make_float2(fmaf(-s.x, s.x, v.x) * 0.5f, fmaf(-s.y, s.y, v.y) * 0.5f), y, s);
}
__device__ __forceinline__ float at_least(float v, float least) {   // NaN stays
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(v), "f"(least));
  return d;
}
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// ---- kernels -------------------------------------------------------------------------------------------------
// Where a block's values lie: tiles of tensors, the turns of each.
template <int COUNT> struct AwWalk {
  int64_t tile, first;   // first place of the tile
  int turn, tensor;
  __device__ __forceinline__ void seek(const AwParams<COUNT>& a) {
    if (tile < 0 || tile >= a.tiles) return;
    tensor = tensor_of(a, tile);
    first = (tile - a.t[tensor].tile) * a.turns * (AW_THREADS * AW_VALUES);
    turn = 0;
  }
  __device__ __forceinline__ AwWalk(const AwParams<COUNT>& a, int64_t from) : tile(from), first(0), turn(0), tensor(0) { seek(a); }
  __device__ __forceinline__ int64_t place() const { return first + (turn * AW_THREADS + (int)threadIdx.x) * AW_VALUES; }
  // (a turn in which the warp has no values ends the tile)
  __device__ __forceinline__ void go_on(const AwParams<COUNT>& a, int64_t step) {
    if (++turn < a.turns && first + (turn * AW_THREADS + (int)(threadIdx.x & ~31u)) * AW_VALUES < a.t[tensor].n) return;
    tile += step;
    seek(a);
  }
};

// The sum of squares of a thread's values of a tile of type T, from place i on; four turns at a time, so that as many loads are on
// their way.
template <typename T> __device__ __forceinline__ double squares_of(const T* g, int64_t i, int64_t n, int turns, bool vectors) {
  constexpr int AHEAD = 4, STEP = AW_THREADS * AW_VALUES;
  double sum = 0.0;
  for (int turn = 0; turn < turns && i < n; turn += AHEAD, i += AHEAD * STEP) {
    Unit<T, AW_VALUES> u[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int64_t at = i + k * STEP, left = turn + k < turns ? n - at : 0;
      if (vectors && left >= AW_VALUES) {
        u[k].get(g + at);
      } else {
        T v[AW_VALUES];
#pragma unroll
        for (int j = 0; j < AW_VALUES; ++j) v[j] = j < left ? g[at + j] : from_f32<T>(0.f);
        memcpy(u[k].u, v, sizeof(v));
      }
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      float2 s = both(0.f);
#pragma unroll
      for (int j = 0; j < AW_VALUES / 2; ++j) s = fma_pair(u[k].pair(j), u[k].pair(j), s);
      const float here = s.x + s.y;
      if (here >= 0x1p-100f && here <= 0x1p126f) {
        sum += (double)here;
      } else {   // squares beyond the range of fp32
#pragma unroll
        for (int j = 0; j < AW_VALUES / 2; ++j) sum += (double)u[k].pair(j).x * u[k].pair(j).x + (double)u[k].pair(j).y * u[k].pair(j).y;
      }
    }
  }
  return sum;
}
// Sums of squares of the gradients, a block's share in 64 bits.
template <int COUNT> __global__ void __launch_bounds__(AW_THREADS) adamw_norm_kernel(const __grid_constant__ AwParams<COUNT> a, int first) {
  let_next_kernel_start();
  double sum = 0.0;
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const AwTensor& t = a.t[tensor_of(a, tile)];
    const int64_t i = ((tile - t.tile) * a.turns * AW_THREADS + threadIdx.x) * AW_VALUES;
    sum += t.g_dtype == SNN_DTYPE_FP32   ? squares_of((const float*)t.g, i, t.n, a.turns, t.vectors)
           : t.g_dtype == SNN_DTYPE_BF16 ? squares_of((const __nv_bfloat16*)t.g, i, t.n, a.turns, t.vectors)
                                         : squares_of((const __half*)t.g, i, t.n, a.turns, t.vectors);
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  __shared__ double shared[AW_THREADS / 32];
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int k = 1; k < AW_THREADS / 32; ++k) sum += shared[k];
  a.partial[blockIdx.x] = first ? sum : a.partial[blockIdx.x] + sum;
}
// One block: the norm, the step's number, and the factors that follow from it.  The powers take longer than all else: a warp each
// raises them, beside the one that waits for the sums.
__global__ void __launch_bounds__(AW_THREADS) adamw_begin_kernel(const AwBegin b) {
  let_next_kernel_start();
  __shared__ double shared[AW_THREADS], left[2];   // 1 - beta^t
  // (the kernel before it, if any, is that of the norm: it does not write the step's number)
  const int64_t t = *b.step + 1;
  if (threadIdx.x == 32) left[0] = 1.0 - pow(b.beta1, (double)t);
  if (threadIdx.x == 64) left[1] = 1.0 - pow(b.beta2, (double)t);
  wait_for_kernel_before();
  double sum = 0.0;
  if (b.partial) {
    for (int k = threadIdx.x; k < AW_NORM_BLOCKS; k += AW_THREADS) sum += b.partial[k];
    shared[threadIdx.x] = sum;
    __syncthreads();
    for (int o = AW_THREADS / 2; o > 0; o /= 2) {
      if (threadIdx.x < o) shared[threadIdx.x] += shared[threadIdx.x + o];
      __syncthreads();
    }
    sum = shared[0];
  } else {
    __syncthreads();
  }
  if (threadIdx.x > 0) return;
  const double scale = (double)b.scale * (b.scale_device ? (double)*b.scale_device : 1.0);
  AwStep s{(float)scale, 0.f, 0.f, 0.f, 0.f, 0u, 0};
  if (b.partial) {
    const double norm = sqrt(sum) * fabs(scale);
    if (b.norm) *b.norm = (float)norm;
    if (!(norm < INFINITY)) s.skip = 1;
    if (norm > b.max_norm) s.factor = (float)(scale * (b.max_norm / norm));
  }
  if (!s.skip) {
    *b.step = t;
    const double lr = b.lr_device ? (double)*b.lr_device : b.lr;
    s.rate = (float)(lr / left[0]);
    s.root = (float)(1.0 / sqrt(left[1]));
    // In one float a decay of 2e-7 would be 1.8e-7.  Two of the same sign, of which the second is never zero, leave an infinite
    // parameter infinite.
    const double keep = 1.0 - lr * b.weight_decay;
    s.keep = (float)keep;
    if (keep != 0.0 && fabs((double)s.keep) >= fabs(keep)) s.keep = __uint_as_float(__float_as_uint(s.keep) - 1u);
    s.keep_rest = (float)(keep - (double)s.keep);
    s.key = key_of(b.seed, (uint64_t)t);
  }
  *b.out = s;
}

__device__ __forceinline__ float2 times(float2 v, float factor) { return mul_pair(v, both(factor)); }

// The step of a thread's parameters and their moments, of which b1 m and b2 v are at hand; g is spent.  On return v holds roots where
// EIGHT.  Products and sums are rounded one by one: what is rounded at random afterwards is then what tensor operations, one after
// the other, give as well.
template <bool EIGHT, int N, int COUNT>
__device__ __forceinline__ void step_values(const AwParams<COUNT>& a, const AwStep& step, float2 p[N / 2], float2 g[N / 2], float2 m[N / 2], float2 v[N / 2]) {
  float2 root[N / 2];
  if (step.factor != 1.f) {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) g[k] = times(g[k], step.factor);
  }
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    m[k] = add_pair(m[k], times(g[k], a.one_less_beta1));
    v[k] = add_pair(v[k], times(mul_pair(g[k], g[k]), a.one_less_beta2));
    root[k] = EIGHT ? root_of(v[k]) : make_float2(__fsqrt_rn(v[k].x), __fsqrt_rn(v[k].y));
  }
  if constexpr (EIGHT) {
    // Where all of a thread's roots are below 2^-44, squares may be subnormal (one that is beside a larger root has the smallest
    // code or none either way); where one is NaN, a square may be infinite.
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) top = larger_of(top, root[k]);
    if (top != 0.f && !(top >= 0x1p-44f)) {
#pragma unroll
      for (int k = 0; k < N / 2; ++k) root[k] = make_float2(__fsqrt_rn(v[k].x), __fsqrt_rn(v[k].y));
    }
  }
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    // (a root of a subnormal square may be too small here: it counts as the smallest of a normal one)
    const float2 counts = EIGHT ? make_float2(at_least(root[k].x, 0x1p-63f), at_least(root[k].y, 0x1p-63f)) : root[k];
    const float2 below = fma_pair(counts, both(step.root), both(a.eps)), up = times(m[k], -step.rate);
    const float2 update = EIGHT ? mul_pair(up, make_float2(reciprocal(below.x), reciprocal(below.y)))
                                : make_float2(__fdividef(up.x, below.x), __fdividef(up.y, below.y));
    p[k] = fma_pair(p[k], both(step.keep), fma_pair(p[k], both(step.keep_rest), update));
    if (EIGHT) v[k] = root[k];
  }
}

// Moments in fp32.
template <int COUNT> __global__ void __launch_bounds__(AW_THREADS, 4) adamw_update_kernel(const __grid_constant__ AwParams<COUNT> a) {
  wait_for_kernel_before();
  const AwStep step = *a.step;
  if (step.skip) return;
  // from the last tile to the first: where the gradients have just been read for their norm, the last of them are in L2
  for (AwWalk<COUNT> at(a, a.tiles - 1 - blockIdx.x); at.tile >= 0; at.go_on(a, -(int64_t)gridDim.x)) {
    const AwTensor& t = a.t[at.tensor];
    const int64_t i = at.place(), state = t.state + i, n = t.n;
    if (i >= n) continue;
    float2 p[AW_VALUES / 2], g[AW_VALUES / 2], m[AW_VALUES / 2], v[AW_VALUES / 2];
    load_values<AW_VALUES>(p, t.p, t.p_dtype, i, n, t.vectors);
    load_values<AW_VALUES>(g, t.g, t.g_dtype, i, n, t.vectors);
    Unit<float, AW_VALUES> b;
    b.get(a.m + state);
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) m[k] = times(b.pair(k), a.beta1);
    b.get(a.v + state);
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) v[k] = times(b.pair(k), a.beta2);
    step_values<false, AW_VALUES>(a, step, p, g, m, v);
    store_values<AW_VALUES>(p, t.p, t.p_dtype, i, n, t.vectors);
    if (t.copy) store_values<AW_VALUES>(p, t.copy, t.copy_dtype, i, n, t.vectors);
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) b.set(k, m[k]);
    b.put(a.m + state);
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) b.set(k, v[k]);
    b.put(a.v + state);
  }
}

// b1 m and b2 v from their codes.  The scale is a power of two, so that it can be multiplied by b1 or b2 first: the product with a
// value (or with its square, which is exact) is rounded once either way.  Where the square of a scale leaves the range, one
// by one.
template <int COUNT>
__device__ __forceinline__ void read_moments(const AwParams<COUNT>& a, float2 m[AW_VALUES / 2], float2 v[AW_VALUES / 2], const AwCodes& m_codes, const AwCodes& v_codes, uint32_t m_byte, uint32_t v_byte) {
  decode(m, m_codes);
  decode(v, v_codes);
  const float m_scale = keep_scale_value(m_byte) * a.beta1, v_scale = keep_scale_value(v_byte);
#pragma unroll
  for (int k = 0; k < AW_VALUES / 2; ++k) m[k] = times(m[k], m_scale), v[k] = mul_pair(v[k], v[k]);
  if (v_byte - 80u < 96u) {   // scales from 2^-47 to 2^48
    const float square = v_scale * v_scale * a.beta2;
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) v[k] = times(v[k], square);
  } else {
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) v[k] = times(times(times(v[k], v_scale), v_scale), a.beta2);
  }
}
// The largest root that is kept, the last code of its scale: squares of what it is rounded to are finite.
constexpr float AW_LARGEST = 0x1.cp63f;   // 448 x 2^55
constexpr uint32_t AW_LARGEST_BYTE = 55 + 127;
// A moment pair that is about to be coded.  Of a finite gradient whose square is infinite the step has been none (m / infinity); the
// largest root and no first moment stand for that from now on, since a group that holds an infinity is lost.  (NaN and infinite
// gradients are.)
__device__ __forceinline__ void keep_finite(float& m, float& root) {
  if (!(root > AW_LARGEST && fabsf(m) <= largest_finite<float>())) return;
  if (root > largest_finite<float>()) m = 0.f;
  root = AW_LARGEST;
}
// The moments back to codes and scale bytes; the lanes of a warp do this together.
struct AwPacked {
  AwCodes m, v;
  uint32_t m_byte, v_byte;
};
__device__ __forceinline__ AwPacked pack_moments(const AwStep& step, int64_t at, float2 m[AW_VALUES / 2], float2 root[AW_VALUES / 2]) {
  AwPacked k;
  k.v_byte = keep_scale_byte<SNN_KEEP_E4M3>(top_of(root)), k.m_byte = keep_scale_byte<SNN_KEEP_E4M3>(top_of(m));
  const bool far = __any_sync(0xffffffffu, k.v_byte > AW_FAR_BYTE);
  if (far && __any_sync(0xffffffffu, k.v_byte > AW_LARGEST_BYTE)) {
#pragma unroll
    for (int j = 0; j < AW_VALUES / 2; ++j) keep_finite(m[j].x, root[j].x), keep_finite(m[j].y, root[j].y);
    k.v_byte = keep_scale_byte<SNN_KEEP_E4M3>(top_of(root)), k.m_byte = keep_scale_byte<SNN_KEEP_E4M3>(top_of(m));
  }
  uint32_t r[AW_VALUES];
  const uint32_t base = mix_base((uint32_t)at ^ step.key ^ mix((uint32_t)(at >> 32)));
#pragma unroll
  for (int j = 0; j < AW_VALUES; ++j) r[j] = mix_from(base, j);
  k.m = encode_at_random<false>(m, r, k.m_byte, __any_sync(0xffffffffu, k.m_byte > AW_FAR_BYTE)), k.v = encode_at_random<true>(root, r, k.v_byte, far);
  return k;
}
constexpr int AW_STEP = 32 * AW_VALUES;   // of a warp and turn
static_assert(AW_TURNS * AW_STEP == 32 * KEEP_GROUP, "a scale byte of a part for each lane");
// A warp's part of a tile: 2048 values one behind the other (AW_TURNS a tile, where there are that many turns), or what a tensor's
// end leaves of them.  types: those of parameters and gradients where all values exist and vectors fit them, otherwise -1.
template <int COUNT> struct AwPart {
  const AwTensor* t;
  int64_t tile, first;
  int types;
  __device__ __forceinline__ AwPart(const AwParams<COUNT>& a, int64_t at) : t(nullptr), tile(at), first(0), types(-1) {
    if (tile < 0) return;
    t = &a.t[tensor_of(a, tile)];
    const int64_t part = (int64_t)a.turns * AW_STEP;
    first = ((tile - t->tile) * (AW_THREADS / 32) + (threadIdx.x >> 5)) * part;
    if (a.turns == AW_TURNS && t->vectors && first + part <= t->n) types = t->p_dtype * 3 + t->g_dtype;
  }
  __device__ __forceinline__ static constexpr int of(int p, int g) { return p * 3 + g; }
};
// A whole part in these types.  The 32 scale bytes are read and written at once, lane by lane: stores of parts of a 32-byte sector
// cost L2 so much that 70 M parameters took 199 us instead of 166 with four bytes a warp and turn (351 against 119 us where nothing was
// computed).  Sixteen values a thread need a fifth fewer instructions and as long, since fewer warps find room; so do copies to shared
// memory a turn ahead.
template <typename PT, typename GT, int COUNT>
__device__ __forceinline__ void update_part(const AwParams<COUNT>& a, const AwStep& step, const AwPart<COUNT>& part) {
  const AwTensor& t = *part.t;
  const int lane = threadIdx.x & 31;
  const int64_t begin = part.first + lane * AW_VALUES, group0 = (t.state + part.first) / KEEP_GROUP + lane;
  PT* to = (PT*)t.p + begin;
  const GT* from = (const GT*)t.g + begin;
  int64_t at = t.state + begin;
  const uint32_t m_bytes = a.m_scales[group0], v_bytes = a.v_scales[group0];
  uint32_t m_new = 0u, v_new = 0u;
#pragma unroll 1
  for (int turn = 0; turn < AW_TURNS; ++turn) {
    constexpr int GROUPS = 32 / AW_LANES;   // of a turn
    Unit<PT, AW_VALUES> up;
    Unit<GT, AW_VALUES> ug;
    AwCodes m_codes, v_codes;
    up.get(to);
    ug.get(from);
    m_codes.get(a.m_codes + at);
    v_codes.get(a.v_codes + at);
    float2 p[AW_VALUES / 2], g[AW_VALUES / 2], m[AW_VALUES / 2], v[AW_VALUES / 2];
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) p[k] = up.pair(k), g[k] = ug.pair(k);
    const int group = turn * GROUPS + lane / AW_LANES;
    read_moments(a, m, v, m_codes, v_codes, __shfl_sync(0xffffffffu, m_bytes, group), __shfl_sync(0xffffffffu, v_bytes, group));
    step_values<true, AW_VALUES>(a, step, p, g, m, v);
#pragma unroll
    for (int k = 0; k < AW_VALUES / 2; ++k) up.set(k, p[k]);
    up.put(to);
    if (t.copy) store_values<AW_VALUES>(p, t.copy, t.copy_dtype, begin + turn * AW_STEP, t.n, true);
    const AwPacked k = pack_moments(step, at, m, v);
    k.m.put(a.m_codes + at);
    k.v.put(a.v_codes + at);
    const uint32_t m_here = __shfl_sync(0xffffffffu, k.m_byte, lane % GROUPS * AW_LANES), v_here = __shfl_sync(0xffffffffu, k.v_byte, lane % GROUPS * AW_LANES);
    if (lane / GROUPS == turn) m_new = m_here, v_new = v_here;
    to += AW_STEP, from += AW_STEP, at += AW_STEP;
  }
  a.m_scales[group0] = (uint8_t)m_new;
  a.v_scales[group0] = (uint8_t)v_new;
}
// A thread's values up to place n: at a tensor's end, or where vectors do not fit, or another mixture of types.  What lies behind
// n is zero, also to the group.
template <int COUNT> __device__ __noinline__ void update_any(const AwParams<COUNT>& a, const AwStep& step, const AwTensor& t, int64_t i, int64_t n) {
  const int64_t at = t.state + i;
  float2 p[AW_VALUES / 2], g[AW_VALUES / 2], m[AW_VALUES / 2], v[AW_VALUES / 2];
#pragma unroll
  for (int k = 0; k < AW_VALUES / 2; ++k) m[k] = v[k] = both(0.f);
  if (i < n) {
    load_values<AW_VALUES>(p, t.p, t.p_dtype, i, n, t.vectors);
    load_values<AW_VALUES>(g, t.g, t.g_dtype, i, n, t.vectors);
    AwCodes m_codes, v_codes;
    m_codes.get(a.m_codes + at);
    v_codes.get(a.v_codes + at);
    read_moments(a, m, v, m_codes, v_codes, a.m_scales[at / KEEP_GROUP], a.v_scales[at / KEEP_GROUP]);
    step_values<true, AW_VALUES>(a, step, p, g, m, v);
    store_values<AW_VALUES>(p, t.p, t.p_dtype, i, n, t.vectors);
    if (t.copy) store_values<AW_VALUES>(p, t.copy, t.copy_dtype, i, n, t.vectors);
  }
#pragma unroll
  for (int k = 0; k < AW_VALUES / 2; ++k) {
    if (i + 2 * k >= n) m[k].x = v[k].x = 0.f;
    if (i + 2 * k + 1 >= n) m[k].y = v[k].y = 0.f;
  }
  const AwPacked k = pack_moments(step, at, m, v);
  if ((i & ~(int64_t)(KEEP_GROUP - 1)) >= n) return;
  k.m.put(a.m_codes + at);
  k.v.put(a.v_codes + at);
  if (threadIdx.x % AW_LANES == 0) a.m_scales[at / KEEP_GROUP] = (uint8_t)k.m_byte, a.v_scales[at / KEEP_GROUP] = (uint8_t)k.v_byte;
}
template <int COUNT> __global__ void __launch_bounds__(AW_THREADS, 4) adamw_update_packed_kernel(const __grid_constant__ AwParams<COUNT> a) {
  using BF = __nv_bfloat16;
  using Part = AwPart<COUNT>;
  wait_for_kernel_before();
  const AwStep step = *a.step;
  if (step.skip) return;
  for (int64_t tile = a.tiles - 1 - blockIdx.x; tile >= 0; tile -= gridDim.x) {
    const Part part(a, tile);
    if (part.types == Part::of(SNN_DTYPE_BF16, SNN_DTYPE_BF16)) {
      update_part<BF, BF>(a, step, part);
    } else if (part.types == Part::of(SNN_DTYPE_FP32, SNN_DTYPE_FP32)) {
      update_part<float, float>(a, step, part);
    } else if (part.types == Part::of(SNN_DTYPE_FP32, SNN_DTYPE_BF16)) {
      update_part<float, BF>(a, step, part);
    } else if (part.types == Part::of(SNN_DTYPE_FP16, SNN_DTYPE_FP16)) {
      update_part<__half, __half>(a, step, part);
    } else {
      const int64_t n = min(part.first + (int64_t)a.turns * AW_STEP, part.t->n);
      for (int64_t i = part.first; i < n; i += AW_STEP) update_any(a, step, *part.t, i + (threadIdx.x & 31) * AW_VALUES, n);
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
snn_status check(const snn_adamw_args* a) {
  if (!a || a->count < 0 || (a->count > 0 && !a->tensors)) return SNN_ERR_INVALID_ARG;
  if (a->moment_format != SNN_KEEP_RAW && a->moment_format != SNN_KEEP_E4M3) return SNN_ERR_INVALID_ARG;
  for (int k = 0; k < a->count; ++k) {
    const snn_adamw_tensor& t = a->tensors[k];
    if (t.n < 0 || t.n >= (int64_t)1 << 50 || !dtype_known(t.param_dtype) || !dtype_known(t.grad_dtype)) return SNN_ERR_INVALID_ARG;
    if (t.n > 0 && (!t.param || !t.grad || (t.copy && !dtype_known(t.copy_dtype)))) return SNN_ERR_INVALID_ARG;
  }
  auto fraction = [](double v) { return v >= 0.0 && v < 1.0; };
  auto finite = [](double v) { return v >= 0.0 && v <= 3e38; };
  if (!fraction(a->beta1) || !fraction(a->beta2) || !finite(a->lr) || !finite(a->weight_decay) || !(a->eps >= 1e-30 && a->eps <= 1.0)) return SNN_ERR_INVALID_ARG;
  if (!(a->scale >= -3e38f && a->scale <= 3e38f) || !(a->max_norm >= 0.0)) return SNN_ERR_INVALID_ARG;
  return SNN_OK;
}
constexpr size_t AW_WORKSPACE = SNN_ADAMW_WORKSPACE;
static_assert(256 + AW_NORM_BLOCKS * 8 <= AW_WORKSPACE && sizeof(AwStep) <= 256, "the workspace holds what is laid out in it");

// The launches of one list of tensors, as many at a time as the table holds.
template <int COUNT, typename F> snn_status in_tables(const snn_adamw_args* a, const AwParams<COUNT>& common, F&& launch) {
  AwParams<COUNT> p = common;
  const int64_t tile = (int64_t)AW_THREADS * AW_VALUES * p.turns;
  int64_t state = 0;
  bool first = true;
  for (int k = 0; k < a->count;) {
    p.count = 0, p.tiles = 0;
    for (; k < a->count && p.count < COUNT; ++k) {
      const snn_adamw_tensor& t = a->tensors[k];
      if (t.n == 0) continue;
      const bool vectors = aligned_to(t.param, 32) && aligned_to(t.grad, 32) && (!t.copy || aligned_to(t.copy, 32));
      p.t[p.count++] = {t.param, t.grad, t.copy, t.n, state, p.tiles, (int8_t)t.param_dtype, (int8_t)t.grad_dtype, (int8_t)t.copy_dtype, (int8_t)vectors};
      p.tiles += (t.n + tile - 1) / tile;
      state += (t.n + KEEP_GROUP - 1) / KEEP_GROUP * KEEP_GROUP;
    }
    if (p.count == 0) break;
    const snn_status st = launch(p, first);
    if (st != SNN_OK) return st;
    first = false;
  }
  return SNN_OK;
}
template <int COUNT> snn_status step_of(const snn_adamw_args* a, cudaStream_t stream) {
  AwParams<COUNT> p{};
  p.beta1 = (float)a->beta1, p.one_less_beta1 = (float)(1.0 - a->beta1), p.beta2 = (float)a->beta2, p.one_less_beta2 = (float)(1.0 - a->beta2);
  p.eps = (float)a->eps, p.m = a->m, p.v = a->v;
  p.m_codes = a->m_codes, p.m_scales = a->m_scales, p.v_codes = a->v_codes, p.v_scales = a->v_scales;
  AwStep* const step = (AwStep*)a->workspace;
  p.step = step;
  p.partial = (double*)((char*)a->workspace + 256);
  const bool clips = a->max_norm > 0.0, eight = a->moment_format == SNN_KEEP_E4M3;
  // tiles of several turns share what it takes to find them, where there are enough of them for every SM
  int64_t values = 0;
  for (int k = 0; k < a->count; ++k) values += a->tensors[k].n;
  p.turns = values >= (int64_t)148 * 4 * AW_TURNS * AW_THREADS * AW_VALUES ? AW_TURNS : 1;
  bool normed = false;
  if (clips) {
    bool any = false;
    const snn_status st = in_tables(a, p, [&](const AwParams<COUNT>& q, bool first) {
      any = true;
      return launch_behind(adamw_norm_kernel<COUNT>, AW_NORM_BLOCKS, AW_THREADS, 0, stream, false, q, (int)first);
    });
    if (st != SNN_OK) return st;
    normed = any;
    if (!any && cudaMemsetAsync(p.partial, 0, AW_NORM_BLOCKS * 8, stream) != cudaSuccess) return cudaGetLastError(), SNN_ERR_CUDA;
  }
  const AwBegin b{a->step, a->lr, a->beta1, a->beta2, a->weight_decay, a->max_norm, a->lr_device, a->scale_device, a->scale, a->seed,
                  clips ? p.partial : nullptr, a->norm, step};
  snn_status st = launch_behind(adamw_begin_kernel, 1, AW_THREADS, 0, stream, clips && normed, b);
  if (st != SNN_OK) return st;
  return in_tables(a, p, [&](const AwParams<COUNT>& q, bool first) {
    if (eight) return launch_behind(adamw_update_packed_kernel<COUNT>, (unsigned)std::min<int64_t>(q.tiles, 148 * 4), AW_THREADS, 0, stream, first, q);
    return launch_behind(adamw_update_kernel<COUNT>, (unsigned)std::min<int64_t>(q.tiles, 148 * 8), AW_THREADS, 0, stream, first, q);
  });
}
}  // namespace

extern "C" snn_status snn_adamw_workspace(const snn_adamw_args* a, size_t* bytes) {
  const snn_status st = check(a);
  if (st != SNN_OK) return st;
  if (!bytes) return SNN_ERR_INVALID_ARG;
  *bytes = AW_WORKSPACE;
  return SNN_OK;
}

extern "C" snn_status snn_adamw_step(const snn_adamw_args* a, void* stream) {
  const snn_status st = check(a);
  if (st != SNN_OK) return st;
  if (!a->step || !a->workspace || !aligned_to(a->workspace, 256)) return SNN_ERR_INVALID_ARG;
  bool any = false;
  for (int k = 0; k < a->count; ++k) any = any || a->tensors[k].n > 0;
  if (any && a->moment_format == SNN_KEEP_RAW && (!a->m || !a->v || !aligned_to(a->m, 32) || !aligned_to(a->v, 32))) return SNN_ERR_INVALID_ARG;
  if (any && a->moment_format == SNN_KEEP_E4M3 &&
      (!a->m_codes || !a->v_codes || !a->m_scales || !a->v_scales || !aligned_to(a->m_codes, 8) || !aligned_to(a->v_codes, 8)))
    return SNN_ERR_INVALID_ARG;
  if (a->workspace_bytes < AW_WORKSPACE) return SNN_ERR_WORKSPACE_TOO_SMALL;
  // a launch carries its table of tensors: a small one for the usual lists, a large one for long lists
  return a->count <= 64 ? step_of<64>(a, (cudaStream_t)stream) : step_of<512>(a, (cudaStream_t)stream);
}
