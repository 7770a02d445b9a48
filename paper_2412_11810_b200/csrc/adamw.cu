// One AdamW step over all tensors of a model (include/snn.h, "sequence-model operators").
//
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,  p' = p (1 - lr wd) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// Bound by HBM (28 bytes a parameter with everything in fp32, 10 with bf16 parameters and gradients and moments in 8 bits).
// A thread block takes tiles of 2048 parameters, eight neighbouring ones a thread; where a tile's tensor lies is found by
// bisection in a table that comes with the launch, so that nothing is copied to the device first and a graph holds it.
//
// Moments in 8 bits: e4m3 groups of 64, the second moment as its root.  A moment moves by a thousandth of its distance a step,
// far less than half a step of its codes: rounded to nearest it would never move.  It is rounded up or down at random, up with
// a probability that is the fraction of the step, so that its mean moves as it should; the bits are a hash of seed, step and
// place.  Both moments are floats rather than integers of a common scale because they are divided by one another: a root that
// is small in its group keeps its relative precision (down to 2^-18 of the largest), and one above zero never becomes zero.
#include <algorithm>

#include "octet.cuh"

using namespace snnk;

namespace {

constexpr int AW_THREADS = 256, AW_TILE = 8 * AW_THREADS;
constexpr int AW_NORM_BLOCKS = 148 * 4;

struct AwTensor {
  void* p;
  const void* g;
  void* copy;
  int64_t n, state;             // values; place of the first one in the moments, a multiple of 64
  int64_t tile;                 // number of its first tile
  int8_t p_dtype, g_dtype, copy_dtype, vectors;   // vectors: all three can be accessed eight values at a time
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

// Eight values from place i on, of which n - i exist; the others are zero.
template <typename T> __device__ __forceinline__ void load_eight(float2 f[4], const T* p, int64_t i, int64_t n, bool vectors) {
  if (vectors && i + 8 <= n) {
    Bits<T> b;
    b.get(p + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = b.pair(k);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    f[k].x = i + 2 * k < n ? to_f32(p[i + 2 * k]) : 0.f;
    f[k].y = i + 2 * k + 1 < n ? to_f32(p[i + 2 * k + 1]) : 0.f;
  }
}
template <typename T> __device__ __forceinline__ void store_eight(const float2 f[4], T* p, int64_t i, int64_t n, bool vectors) {
  if (vectors && i + 8 <= n) {
    Bits<T> b;
#pragma unroll
    for (int k = 0; k < 4; ++k) b.set(k, f[k]);
    b.put(p + i);
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (i + 2 * k < n) p[i + 2 * k] = from_f32<T>(f[k].x);
    if (i + 2 * k + 1 < n) p[i + 2 * k + 1] = from_f32<T>(f[k].y);
  }
}
__device__ __forceinline__ void load_eight(float2 f[4], const void* p, int dtype, int64_t i, int64_t n, bool vectors) {
  if (dtype == SNN_DTYPE_FP32)
    load_eight(f, (const float*)p, i, n, vectors);
  else if (dtype == SNN_DTYPE_BF16)
    load_eight(f, (const __nv_bfloat16*)p, i, n, vectors);
  else
    load_eight(f, (const __half*)p, i, n, vectors);
}
__device__ __forceinline__ void store_eight(const float2 f[4], void* p, int dtype, int64_t i, int64_t n, bool vectors) {
  if (dtype == SNN_DTYPE_FP32)
    store_eight(f, (float*)p, i, n, vectors);
  else if (dtype == SNN_DTYPE_BF16)
    store_eight(f, (__nv_bfloat16*)p, i, n, vectors);
  else
    store_eight(f, (__half*)p, i, n, vectors);
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
// The e4m3 code of u, at most 448 in magnitude, rounded away from zero where the fraction of a step and r / 2^16 reach one.
// A normal e4m3 value keeps three fraction bits: r is added to the first 16 of the 20 that are cut.  Below 2^-6 the step is
// 2^-9, that of values in [2^-6, 2^-5): 2^-6 is added first and taken off again.
__device__ __forceinline__ float round_at_random(float u, uint32_t r) {
  const float a = fabsf(u);
  const float shift = a < 0x1p-6f ? 0x1p-6f : 0.f;
  const uint32_t bits = (__float_as_uint(a + shift) + (r << 4)) & 0xfff00000u;
  return copysignf(fminf(__uint_as_float(bits) - shift, 448.f), u);
}
// Eight values of a lane to codes; top: the group's largest magnitude.  ROOT: what is above zero stays above zero.
template <bool ROOT> __device__ __forceinline__ uint2 encode_eight(const float2 f[4], const uint32_t r[8], uint32_t byte) {
  if (byte == 255u) return make_uint2(0u, 0u);
  const float inverse = keep_scale_inverse(byte);
  uint32_t q[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 u = mul2(f[k], both(inverse));
    float2 c = make_float2(round_at_random(u.x, ROOT ? r[2 * k] >> 16 : r[2 * k] & 0xffffu),
                           round_at_random(u.y, ROOT ? r[2 * k + 1] >> 16 : r[2 * k + 1] & 0xffffu));
    if (ROOT) c = make_float2(u.x > 0.f ? fmaxf(c.x, 0x1p-9f) : c.x, u.y > 0.f ? fmaxf(c.y, 0x1p-9f) : c.y);
    q[k] = (uint32_t)__nv_cvt_float2_to_fp8x2(c, __NV_SATFINITE, __NV_E4M3);
  }
  return make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
}
__device__ __forceinline__ void decode_eight(float2 f[4], uint2 codes, uint32_t byte) {
  const float scale = keep_scale_value(byte);
#pragma unroll
  for (int k = 0; k < 4; ++k) f[k] = keep_decode2<float, SNN_KEEP_E4M3>((k < 2 ? codes.x : codes.y) >> (16 * (k & 1)) & 0xffffu, scale);
}
__device__ __forceinline__ uint32_t scale_byte_of(const float2 f[4]) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) m = larger_magnitude(m, larger_magnitude(f[k].x, f[k].y));
  return keep_scale_byte<SNN_KEEP_E4M3>(group_top(m));
}

// ---- kernels -------------------------------------------------------------------------------------------------
// Sums of squares of the gradients, a block's share in 64 bits.
template <int COUNT> __global__ void __launch_bounds__(AW_THREADS) adamw_norm_kernel(const __grid_constant__ AwParams<COUNT> a, int first) {
  let_next_kernel_start();
  double sum = 0.0;
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const AwTensor& t = a.t[tensor_of(a, tile)];
    const int64_t i = (tile - t.tile) * AW_TILE + threadIdx.x * 8;
    if (i >= t.n) continue;
    float2 g[4];
    load_eight(g, t.g, t.g_dtype, i, t.n, t.vectors);
    float2 s = both(0.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) s = fma2(g[k], g[k], s);
    const float here = s.x + s.y;
    if (here >= 0x1p-100f && here <= 0x1p126f) {
      sum += (double)here;
      continue;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sum += (double)g[k].x * g[k].x + (double)g[k].y * g[k].y;   // squares beyond the range of fp32
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

__device__ __forceinline__ float root_of(float v) { return __fsqrt_rn(v); }

template <int COUNT, bool EIGHT> __global__ void __launch_bounds__(AW_THREADS) adamw_update_kernel(const __grid_constant__ AwParams<COUNT> a) {
  wait_for_kernel_before();
  const AwStep step = *a.step;
  if (step.skip) return;
  // from the last tile to the first: where the gradients have just been read for their norm, the last of them are in L2
  for (int64_t tile = a.tiles - 1 - blockIdx.x; tile >= 0; tile -= gridDim.x) {
    const AwTensor& t = a.t[tensor_of(a, tile)];
    const int64_t n = t.n, i = (tile - t.tile) * AW_TILE + threadIdx.x * 8, at = t.state + i;
    // (in 8 bits the lanes of a group work together: those behind the tensor's end hold zeros; a group has a lane before it,
    // or is skipped by all of its lanes)
    const bool here = i < n, group = (i & ~(int64_t)(KEEP_GROUP - 1)) < n;
    if (EIGHT ? !__any_sync(0xffffffffu, group) : !here) continue;
    float2 p[4], g[4], m[4], v[4];
    uint32_t m_byte = 0, v_byte = 0;
    uint2 m_codes = make_uint2(0u, 0u), v_codes = m_codes;
    if (here) {
      load_eight(p, t.p, t.p_dtype, i, n, t.vectors);
      load_eight(g, t.g, t.g_dtype, i, n, t.vectors);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) p[k] = g[k] = both(0.f);
    }
    if (EIGHT) {
      if (group) {
        m_codes = *reinterpret_cast<const uint2*>(a.m_codes + at);
        v_codes = *reinterpret_cast<const uint2*>(a.v_codes + at);
        m_byte = a.m_scales[at / KEEP_GROUP], v_byte = a.v_scales[at / KEEP_GROUP];
      }
      decode_eight(m, m_codes, m_byte);
      decode_eight(v, v_codes, v_byte);
    } else {
      Bits<float> b;
      b.get(a.m + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) m[k] = b.pair(k);
      b.get(a.v + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = b.pair(k);
    }
    float2 root[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      g[k] = mul2(g[k], both(step.factor));
      // (products and sums are rounded one by one: what is rounded at random afterwards is then what tensor operations, one
      // after the other, give as well)
      m[k] = add2(mul2(m[k], both(a.beta1)), mul2(g[k], both(a.one_less_beta1)));
      if (EIGHT) v[k] = mul2(v[k], v[k]);
      v[k] = add2(mul2(v[k], both(a.beta2)), mul2(mul2(g[k], g[k]), both(a.one_less_beta2)));
      root[k] = make_float2(root_of(v[k].x), root_of(v[k].y));
      const float2 below = fma2(root[k], both(step.root), both(a.eps)), up = mul2(m[k], both(step.rate));
      p[k] = fma2(p[k], both(step.keep), make_float2(-__fdividef(up.x, below.x), -__fdividef(up.y, below.y)));
    }
    if (EIGHT && i + 8 > n) {   // what lies behind the tensor's end is nothing to its group
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i + 2 * k >= n) m[k].x = root[k].x = 0.f;
        if (i + 2 * k + 1 >= n) m[k].y = root[k].y = 0.f;
      }
    }
    if (here) {
      store_eight(p, t.p, t.p_dtype, i, n, t.vectors);
      if (t.copy) store_eight(p, t.copy, t.copy_dtype, i, n, t.vectors);
    }
    if (EIGHT) {
      uint32_t r[8];
      const uint32_t key = step.key ^ mix((uint32_t)(at >> 32));
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] = mix((uint32_t)(at + j) ^ key);
      m_byte = scale_byte_of(m), v_byte = scale_byte_of(root);
      if (!group) continue;
      *reinterpret_cast<uint2*>(a.m_codes + at) = encode_eight<false>(m, r, m_byte);
      *reinterpret_cast<uint2*>(a.v_codes + at) = encode_eight<true>(root, r, v_byte);
      if ((threadIdx.x & 7) == 0) a.m_scales[at / KEEP_GROUP] = (uint8_t)m_byte, a.v_scales[at / KEEP_GROUP] = (uint8_t)v_byte;
    } else {
      Bits<float> b;
#pragma unroll
      for (int k = 0; k < 4; ++k) b.set(k, m[k]);
      b.put(a.m + at);
#pragma unroll
      for (int k = 0; k < 4; ++k) b.set(k, v[k]);
      b.put(a.v + at);
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
  int64_t state = 0;
  bool first = true;
  for (int k = 0; k < a->count;) {
    p.count = 0, p.tiles = 0;
    for (; k < a->count && p.count < COUNT; ++k) {
      const snn_adamw_tensor& t = a->tensors[k];
      if (t.n == 0) continue;
      const bool vectors = aligned_to(t.param, 8 * dtype_size(t.param_dtype)) && aligned_to(t.grad, 8 * dtype_size(t.grad_dtype)) &&
                           (!t.copy || aligned_to(t.copy, 8 * dtype_size(t.copy_dtype)));
      p.t[p.count++] = {t.param, t.grad, t.copy, t.n, state, p.tiles, (int8_t)t.param_dtype, (int8_t)t.grad_dtype, (int8_t)t.copy_dtype, (int8_t)vectors};
      p.tiles += (t.n + AW_TILE - 1) / AW_TILE;
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
  const bool clips = a->max_norm > 0.0;
  if (clips) {
    bool any = false;
    const snn_status st = in_tables(a, p, [&](const AwParams<COUNT>& q, bool first) {
      any = true;
      return launch_behind(adamw_norm_kernel<COUNT>, AW_NORM_BLOCKS, AW_THREADS, 0, stream, false, q, (int)first);
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
    return a->moment_format == SNN_KEEP_E4M3 ? launch_behind(adamw_update_kernel<COUNT, true>, blocks, AW_THREADS, 0, stream, first, q)
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
      (!a->m_codes || !a->v_codes || !a->m_scales || !a->v_scales || !aligned_to(a->m_codes, 8) || !aligned_to(a->v_codes, 8)))
    return SNN_ERR_INVALID_ARG;
  if (a->workspace_bytes < AW_WORKSPACE) return SNN_ERR_WORKSPACE_TOO_SMALL;
  // a launch carries its table of tensors: a small one for the usual lists, a large one for long lists
  return a->count <= 64 ? step_of<64>(a, (cudaStream_t)stream) : step_of<512>(a, (cudaStream_t)stream);
}
