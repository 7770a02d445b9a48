// One AdamW step over all tensors of a model (include/snn.h, "sequence-model operators").
//
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,  p' = p (1 - lr wd) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// Bound by HBM (28 bytes a parameter with everything in fp32, 10 with bf16 parameters and gradients and moments in 8 bits).
// A thread block takes tiles of a tensor, eight (16 with moments in 8 bits) neighbouring parameters a thread and turn; where a
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

constexpr int AW_THREADS = 256, AW_MOST_TURNS = 4;   // of a tile
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
  float keep;                   // 1 - lr wd
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
  int turns;                    // of a tile: AW_THREADS times 8 or 16 values each
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
__device__ __forceinline__ uint32_t key_of(uint64_t seed, uint64_t step) {
  uint32_t key = mix(0x2545F491u ^ (uint32_t)seed);
  key = mix(key ^ (uint32_t)(seed >> 32));
  key = mix(key ^ (uint32_t)step);
  return mix(key ^ (uint32_t)(step >> 32));
}

// ---- moments in 8 bits -----------------------------------------------------------------------------------------
constexpr int AW_PACKED = 16;   // values of a lane: four lanes a group
// A value times 2^-120 over its group's scale has the e4m3 code in bits 20 to 26 of its fp32 pattern, subnormal codes among
// them (they are subnormal there as well), and the fraction of a step in the 20 bits below.  The pattern moved up by four bits
// plus 2^8 r, with r of 16 bits, has the rounded code in its highest byte.
constexpr uint32_t AW_BITS_LOW = 0x4104u, AW_BITS_HIGH = 0x4324u;   // selectors of 2^8 r for the two halves of the random bits
__device__ __forceinline__ uint32_t highest_bytes(const uint32_t y[4]) {
  return __byte_perm(__byte_perm(y[0], y[1], 0x0073), __byte_perm(y[2], y[3], 0x0073), 0x5410);
}
// Codes of a lane's 16 values; byte: their group's scale byte.  ROOT: nothing is negative, and what is above zero stays above zero.
template <bool ROOT> __device__ __forceinline__ uint4 encode_at_random(float2 f[AW_PACKED / 2], const uint32_t r[AW_PACKED], uint32_t byte) {
  // 2^-120 over the scale, 2^(7 - byte); where that is subnormal, 2^-126 of it beforehand
  const bool far = byte > 133u;
  if (__any_sync(0xffffffffu, far)) {
#pragma unroll
    for (int k = 0; k < AW_PACKED / 2; ++k) {
      const float2 down = mul_pair(f[k], both(0x1p-126f));
      const float2 least = ROOT ? make_float2(f[k].x > 0.f ? 0x1p-100f : 0.f, f[k].y > 0.f ? 0x1p-100f : 0.f) : both(0.f);
      if (far) f[k] = ROOT ? make_float2(fmaxf(down.x, least.x), fmaxf(down.y, least.y)) : down;
    }
  }
  const float factor = __uint_as_float((far ? 260u - byte : 134u - byte) << 23);
  uint32_t q[AW_PACKED / 4];
#pragma unroll
  for (int k = 0; k < AW_PACKED / 4; ++k) {
    uint32_t y[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float2 u = mul_pair(f[2 * k + j], both(factor));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t t = __float_as_uint(h ? u.y : u.x), random = __byte_perm(r[4 * k + 2 * j + h], 0u, ROOT ? AW_BITS_HIGH : AW_BITS_LOW);
        uint32_t v = (t << 4) + random;
        if (ROOT)
          v = max(v, min(__float_as_uint(h ? f[2 * k + j].y : f[2 * k + j].x), 1u << 24));
        else
          v |= t & 0x80000000u;
        y[2 * j + h] = v;
      }
    }
    q[k] = highest_bytes(y);
  }
  return byte == 255u ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(q[0], q[1], q[2], q[3]);
}
__device__ __forceinline__ void decode(float2 f[AW_PACKED / 2], const uint32_t codes[AW_PACKED / 4], uint32_t byte) {
  const float scale = keep_scale_value(byte);
#pragma unroll
  for (int k = 0; k < AW_PACKED / 2; ++k) {
    const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(codes[k / 2] >> (16 * (k & 1))), __NV_E4M3)));
    f[k] = mul_pair(v, both(scale));
  }
}
__device__ __forceinline__ uint32_t top_of(const float2 f[AW_PACKED / 2]) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < AW_PACKED / 2; ++k) m = larger_of(m, f[k]);
  return group_top<KEEP_GROUP / AW_PACKED>(m);
}
// Square roots by the hardware's approximation of 1 / sqrt(v) and one step of Newton's iteration from the residual v - s^2, which
// leaves them correctly rounded but for a few; of numbers below 2^-126 they are too small.
__device__ __forceinline__ float2 root_of(float2 v) {
  float2 y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(v.x, 0x1p-126f)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(v.y, 0x1p-126f)));
  const float2 s = mul_pair(v, y), off = fma_pair(make_float2(-s.x, -s.y), s, v);
  return fma_pair(mul_pair(off, both(0.5f)), y, s);
}
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// ---- kernels -------------------------------------------------------------------------------------------------
// Sums of squares of the gradients, a block's share in 64 bits.
template <int COUNT, int N> __global__ void __launch_bounds__(AW_THREADS) adamw_norm_kernel(const __grid_constant__ AwParams<COUNT> a, int first) {
  let_next_kernel_start();
  double sum = 0.0;
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const AwTensor& t = a.t[tensor_of(a, tile)];
    const int64_t n = t.n;
    int64_t i = ((tile - t.tile) * a.turns * AW_THREADS + threadIdx.x) * N;
    for (int turn = 0; turn < a.turns && i < n; ++turn, i += AW_THREADS * N) {
      float2 g[N / 2];
      load_values<N>(g, t.g, t.g_dtype, i, n, t.vectors);
      float2 s = both(0.f);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) s = fma_pair(g[k], g[k], s);
      const float here = s.x + s.y;
      if (here >= 0x1p-100f && here <= 0x1p126f) {
        sum += (double)here;
        continue;
      }
#pragma unroll
      for (int k = 0; k < N / 2; ++k) sum += (double)g[k].x * g[k].x + (double)g[k].y * g[k].y;   // squares beyond the range of fp32
    }
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
// One block: the norm, the step's number, and the factors that follow from it.
__global__ void __launch_bounds__(AW_THREADS) adamw_begin_kernel(const AwBegin b) {
  let_next_kernel_start();
  wait_for_kernel_before();
  __shared__ double shared[AW_THREADS];
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
  }
  if (threadIdx.x > 0) return;
  const double scale = (double)b.scale * (b.scale_device ? (double)*b.scale_device : 1.0);
  AwStep s{(float)scale, 0.f, 0.f, 0.f, 0u, 0};
  if (b.partial) {
    const double norm = sqrt(sum) * fabs(scale);
    if (b.norm) *b.norm = (float)norm;
    if (!(norm < INFINITY)) s.skip = 1;
    if (norm > b.max_norm) s.factor = (float)(scale * (b.max_norm / norm));
  }
  if (!s.skip) {
    const int64_t t = *b.step + 1;
    *b.step = t;
    const double lr = b.lr_device ? (double)*b.lr_device : b.lr;
    s.rate = (float)(lr / (1.0 - pow(b.beta1, (double)t)));
    s.root = (float)(1.0 / sqrt(1.0 - pow(b.beta2, (double)t)));
    s.keep = (float)(1.0 - lr * b.weight_decay);
    s.key = key_of(b.seed, (uint64_t)t);
  }
  *b.out = s;
}

// EIGHT: moments in 8 bits.
template <int COUNT, bool EIGHT> __global__ void __launch_bounds__(AW_THREADS) adamw_update_kernel(const __grid_constant__ AwParams<COUNT> a) {
  constexpr int N = EIGHT ? AW_PACKED : 8;
  wait_for_kernel_before();
  const AwStep step = *a.step;
  if (step.skip) return;
  // from the last tile to the first: where the gradients have just been read for their norm, the last of them are in L2
  for (int64_t tile = a.tiles - 1 - blockIdx.x; tile >= 0; tile -= gridDim.x) {
    const AwTensor& t = a.t[tensor_of(a, tile)];
    const int64_t n = t.n, first = (tile - t.tile) * a.turns * (AW_THREADS * N), state = t.state;
    for (int turn = 0; turn < a.turns; ++turn) {
      const int64_t i = first + (turn * AW_THREADS + (int)threadIdx.x) * N, at = state + i;
      // (in 8 bits the lanes of a group work together: those behind the tensor's end hold zeros)
      const bool here = i < n, group = (i & ~(int64_t)(KEEP_GROUP - 1)) < n;
      if (!__any_sync(0xffffffffu, group)) break;
      float2 p[N / 2], g[N / 2], m[N / 2], v[N / 2];
#pragma unroll
      for (int k = 0; k < N / 2; ++k) p[k] = g[k] = m[k] = v[k] = both(0.f);
      if (here) {
        load_values<N>(p, t.p, t.p_dtype, i, n, t.vectors);
        load_values<N>(g, t.g, t.g_dtype, i, n, t.vectors);
      }
      if constexpr (EIGHT) {
        if (group) {
          uint32_t m_codes[4], v_codes[4];
          get_16(m_codes, a.m_codes + at);
          get_16(v_codes, a.v_codes + at);
          const uint32_t m_byte = a.m_scales[at / KEEP_GROUP], v_byte = a.v_scales[at / KEEP_GROUP];
          decode(m, m_codes, m_byte);
          decode(v, v_codes, v_byte);
        }
      } else if (here) {
        Unit<float, N> b;
        b.get(a.m + at);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) m[k] = b.pair(k);
        b.get(a.v + at);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) v[k] = b.pair(k);
      }
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        g[k] = mul_pair(g[k], both(step.factor));
        // (products and sums are rounded one by one: what is rounded at random afterwards is then what tensor operations, one
        // after the other, give as well)
        m[k] = add_pair(mul_pair(m[k], both(a.beta1)), mul_pair(g[k], both(a.one_less_beta1)));
        if (EIGHT) v[k] = mul_pair(v[k], v[k]);
        v[k] = add_pair(mul_pair(v[k], both(a.beta2)), mul_pair(mul_pair(g[k], g[k]), both(a.one_less_beta2)));
        const float2 root = EIGHT ? root_of(v[k]) : make_float2(__fsqrt_rn(v[k].x), __fsqrt_rn(v[k].y));
        const float2 below = fma_pair(root, both(step.root), both(a.eps)), up = mul_pair(m[k], both(-step.rate));
        const float2 update = EIGHT ? mul_pair(up, make_float2(reciprocal(below.x), reciprocal(below.y)))
                                    : make_float2(__fdividef(up.x, below.x), __fdividef(up.y, below.y));
        p[k] = fma_pair(p[k], both(step.keep), update);
        if (EIGHT) g[k] = v[k], v[k] = root;   // (the root is what is kept)
      }
      if (here) {
        store_values<N>(p, t.p, t.p_dtype, i, n, t.vectors);
        if (t.copy) store_values<N>(p, t.copy, t.copy_dtype, i, n, t.vectors);
      }
      if constexpr (EIGHT) {
        if (i + N > n) {   // what lies behind the tensor's end is nothing to its group
#pragma unroll
          for (int k = 0; k < N / 2; ++k) {
            if (i + 2 * k >= n) m[k].x = v[k].x = 0.f;
            if (i + 2 * k + 1 >= n) m[k].y = v[k].y = 0.f;
          }
        }
        uint32_t top = top_of(v);
        if (__any_sync(0xffffffffu, top - 1u < (83u << 23) - 1u)) {   // roots below 2^-44, but not zero: squares may be subnormal
#pragma unroll
          for (int k = 0; k < N / 2; ++k) {
            if (v[k].x > 0.f) v[k].x = __fsqrt_rn(g[k].x);
            if (v[k].y > 0.f) v[k].y = __fsqrt_rn(g[k].y);
          }
          top = top_of(v);
        }
        const uint32_t v_byte = keep_scale_byte<SNN_KEEP_E4M3>(top), m_byte = keep_scale_byte<SNN_KEEP_E4M3>(top_of(m));
        uint32_t r[N];
        const uint32_t key = step.key ^ mix((uint32_t)(at >> 32));
#pragma unroll
        for (int j = 0; j < N; ++j) r[j] = mix((uint32_t)(at + j) ^ key);
        const uint4 m_codes = encode_at_random<false>(m, r, m_byte), v_codes = encode_at_random<true>(v, r, v_byte);
        if (group) {
          *reinterpret_cast<uint4*>(a.m_codes + at) = m_codes;
          *reinterpret_cast<uint4*>(a.v_codes + at) = v_codes;
          if ((threadIdx.x & 3) == 0) a.m_scales[at / KEEP_GROUP] = (uint8_t)m_byte, a.v_scales[at / KEEP_GROUP] = (uint8_t)v_byte;
        }
      } else if (here) {
        Unit<float, N> b;
#pragma unroll
        for (int k = 0; k < N / 2; ++k) b.set(k, m[k]);
        b.put(a.m + at);
#pragma unroll
        for (int k = 0; k < N / 2; ++k) b.set(k, v[k]);
        b.put(a.v + at);
      }
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
  const int64_t tile = (int64_t)AW_THREADS * (a->moment_format == SNN_KEEP_RAW ? 8 : AW_PACKED) * p.turns;
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
  p.turns = values >= (int64_t)148 * 8 * AW_MOST_TURNS * AW_THREADS * AW_PACKED ? AW_MOST_TURNS : 1;
  if (clips) {
    bool any = false;
    const snn_status st = in_tables(a, p, [&](const AwParams<COUNT>& q, bool first) {
      any = true;
      return launch_behind(eight ? adamw_norm_kernel<COUNT, AW_PACKED> : adamw_norm_kernel<COUNT, 8>, AW_NORM_BLOCKS, AW_THREADS, 0, stream, false, q, (int)first);
    });
    if (st != SNN_OK) return st;
    if (!any && cudaMemsetAsync(p.partial, 0, AW_NORM_BLOCKS * 8, stream) != cudaSuccess) return cudaGetLastError(), SNN_ERR_CUDA;
  }
  const AwBegin b{a->step, a->lr, a->beta1, a->beta2, a->weight_decay, a->max_norm, a->lr_device, a->scale_device, a->scale, a->seed,
                  clips ? p.partial : nullptr, a->norm, step};
  snn_status st = launch_behind(adamw_begin_kernel, 1, AW_THREADS, 0, stream, false, b);
  if (st != SNN_OK) return st;
  return in_tables(a, p, [&](const AwParams<COUNT>& q, bool first) {
    const unsigned blocks = (unsigned)std::min<int64_t>(q.tiles, 148 * 8);
    return eight ? launch_behind(adamw_update_kernel<COUNT, true>, blocks, AW_THREADS, 0, stream, first, q)
                                             : launch_behind(adamw_update_kernel<COUNT, false>, blocks, AW_THREADS, 0, stream, first, q);
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
      (!a->m_codes || !a->v_codes || !a->m_scales || !a->v_scales || !aligned_to(a->m_codes, 16) || !aligned_to(a->v_codes, 16)))
    return SNN_ERR_INVALID_ARG;
  if (a->workspace_bytes < AW_WORKSPACE) return SNN_ERR_WORKSPACE_TOO_SMALL;
  // a launch carries its table of tensors: a small one for the usual lists, a large one for long lists
  return a->count <= 64 ? step_of<64>(a, (cudaStream_t)stream) : step_of<512>(a, (cudaStream_t)stream);
}
