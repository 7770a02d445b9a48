// 32 bytes of a row per thread, and what kernels that move such units share.
//
// A unit is N values of a lane: 8 of fp32, 16 of a 16-bit type.  By VECTORS they are neighbours and one 256-bit access, so that the
// lanes of a warp cover whole lines with it; a group of 64 values (KEEP_GROUP) belongs to 64 / N lanes.  It needs rows of
// multiples of N values at addresses of multiples of 32 bytes.  Otherwise the lanes of a warp take neighbouring PAIRS, where rows
// are even and pairs aligned, or SINGLE values, and a unit has every 32nd of them: an access of a warp is 64 to 256 bytes without a
// gap, and a group is one pair of each lane or two values.
#pragma once
#include <string.h>

#include <atomic>
#include <type_traits>

#include "seq_common.cuh"

namespace snnk {

template <typename T> constexpr int UNIT = 32 / (int)sizeof(T);

// ---- pairs of fp32 values in two registers -------------------------------------------------------------------
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 fma_pair_down(float2 a, float2 b, float2 c) {   // rounded toward zero
  float2 d;
  asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rz.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// The largest magnitude of m and a pair; NaN if one of them is.
__device__ __forceinline__ float larger_of(float m, float2 v) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(m), "f"(fabsf(v.x)), "f"(fabsf(v.y)));
  return d;
}

// ---- units -----------------------------------------------------------------------------------------------------
// (volatile keeps the order of these accesses among one another; a store that depends on a load comes behind it anyway)
__device__ __forceinline__ void get_32(uint32_t* u, const void* p) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
               : "l"(p));
}
__device__ __forceinline__ void put_32(void* p, const uint32_t* u) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]),
               "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}
__device__ __forceinline__ void get_16(uint32_t* u, const void* p) {
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "l"(p));
}
__device__ __forceinline__ void put_16(void* p, const uint32_t* u) {
  asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]) : "memory");
}
template <typename T> __device__ __forceinline__ float2 pair_of(const uint32_t* u, int i) {
  if constexpr (sizeof(T) == 4) {
    return make_float2(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
  } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {   // the upper half of an fp32 value
    return make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
  } else {
    __half2 r;
    memcpy(&r, &u[i], 4);
    return __half22float2(r);
  }
}
template <typename T> __device__ __forceinline__ void set_pair(uint32_t* u, int i, float2 v) {
  if constexpr (sizeof(T) == 4) {
    u[2 * i] = __float_as_uint(v.x), u[2 * i + 1] = __float_as_uint(v.y);
  } else {
    typename Pair<T>::raw r;
    set_raw(r, v);
    memcpy(&u[i], &r, 4);
  }
}
// N values of type T: 16 or 32 bytes, or a multiple of that.
template <typename T, int N> struct Unit {
  static constexpr int WORDS = N * (int)sizeof(T) / 4, LANES = KEEP_GROUP / N;
  uint32_t u[WORDS];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) u[i] = 0u;
  }
  __device__ __forceinline__ float2 pair(int i) const { return pair_of<T>(u, i); }
  __device__ __forceinline__ void set(int i, float2 v) { set_pair<T>(u, i, v); }
  __device__ __forceinline__ void get(const T* p) {
    if constexpr (WORDS == 4) {
      get_16(u, p);
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; i += 8) get_32(u + i, (const uint32_t*)p + i);
    }
  }
  __device__ __forceinline__ void put(T* p) const {
    if constexpr (WORDS == 4) {
      put_16(p, u);
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; i += 8) put_32((uint32_t*)p + i, u + i);
    }
  }
};
enum Access { SINGLE, PAIRS, VECTORS };
// Where the values of a unit stand in a row of n: `first` is the lane's first one.
template <int ACCESS, int N> struct Columns {
  int first, n;
  static __device__ __forceinline__ constexpr int behind(int v) { return ACCESS == VECTORS ? v : ACCESS == PAIRS ? 64 * (v / 2) + v % 2 : 32 * v; }
  // the columns from `start` on, of which a lane's share is N
  static __device__ __forceinline__ constexpr int of_lane(int lane) { return ACCESS == VECTORS ? N * lane : ACCESS == PAIRS ? 2 * lane : lane; }
  // (by vectors all values of a unit exist or none does, by pairs both of a pair)
  __device__ __forceinline__ bool exists(int v) const { return ACCESS == VECTORS ? first < n : behind(v) < n - first; }
  // Values that do not exist: by vectors what the unit held before, otherwise zero.
  template <typename T> __device__ __forceinline__ void load(Unit<T, N>& u, const T* row) const {
    if constexpr (ACCESS == VECTORS) {
      if (first < n) u.get(row + first);
    } else if constexpr (ACCESS == PAIRS) {
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        typename Pair<T>::raw r{};
        if (exists(2 * k)) r = *reinterpret_cast<const typename Pair<T>::raw*>(row + first + behind(2 * k));
        memcpy(u.u + k * (int)sizeof(T) / 2, &r, sizeof(r));
      }
    } else {
      T v[N];
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = exists(j) ? row[first + behind(j)] : from_f32<T>(0.f);
      memcpy(u.u, v, sizeof(v));
    }
  }
  template <typename T> __device__ __forceinline__ void store(const Unit<T, N>& u, T* row) const {
    if constexpr (ACCESS == VECTORS) {
      if (first < n) u.put(row + first);
    } else if constexpr (ACCESS == PAIRS) {
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        typename Pair<T>::raw r;
        memcpy(&r, u.u + k * (int)sizeof(T) / 2, sizeof(r));
        if (exists(2 * k)) *reinterpret_cast<typename Pair<T>::raw*>(row + first + behind(2 * k)) = r;
      }
    } else {
      T v[N];
      memcpy(v, u.u, sizeof(v));
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (exists(j)) row[first + behind(j)] = v[j];
    }
  }
};

// ---- copies to shared memory ----------------------------------------------------------------------------------
// Copies of 16 bytes from global to shared memory that the thread does not wait for.
__device__ __forceinline__ void copy_16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void close_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int OPEN> __device__ __forceinline__ void wait_groups() { asm volatile("cp.async.wait_group %0;" ::"n"(OPEN) : "memory"); }

// ---- 8-bit codes of a group ------------------------------------------------------------------------------------
// Largest magnitude of a group as a bit pattern, from that of its lanes; NaN sorts above infinity above the rest.
template <int LANES> __device__ __forceinline__ uint32_t group_top(float m) {
  uint32_t top = __float_as_uint(m);
#pragma unroll
  for (int o = 1; o < LANES; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  return top;
}
// The codes of two values, low first, rounded to nearest.  rare: whether a code of the warp could round up to 128.
template <int FORMAT> __device__ __forceinline__ uint32_t encode_pair(float2 v, float inverse, bool rare) {
  if (FORMAT == SNN_KEEP_INT8) {
    // 1.5 x 2^23 + v / scale, rounded once: the integer stands in the low bits
    const float magic = 12582912.f;
    float2 a = fma_pair(v, both(inverse), both(magic));
    if (rare) a = make_float2(fminf(fmaxf(a.x, magic - 127.f), magic + 127.f), fminf(fmaxf(a.y, magic - 127.f), magic + 127.f));
    return __byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040);   // (the upper half is not used)
  }
  return (uint32_t)__nv_cvt_float2_to_fp8x2(mul_pair(v, both(inverse)), __NV_SATFINITE, __NV_E4M3);
}

// ---- launches behind one another's start ---------------------------------------------------------------------
__device__ __forceinline__ void wait_for_kernel_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;"); }

// behind: the kernel may be set up while the one before it in the stream runs; it calls wait_for_kernel_before() before it
// touches anything that one writes or reads.
template <typename... P, typename... A>
snn_status launch_behind(void (*kernel)(P...), unsigned grid, int threads, size_t smem, cudaStream_t stream, bool behind, const A&... args) {
  if (!behind) {
    kernel<<<grid, threads, smem, stream>>>(P(args)...);
    return launched();
  }
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
}
// Lets a kernel have more than 48 KB of shared memory, once for each device.
template <auto KERNEL> bool allow_shared(int bytes) {
  static std::atomic<uint64_t> done{0};
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return cudaGetLastError(), false;
  if (device < 64 && done.load() >> device & 1) return true;
  if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return cudaGetLastError(), false;
  if (device < 64) done.fetch_or((uint64_t)1 << device);
  return true;
}

inline bool aligned_to(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }
// The widest access that rows of n values allow (rows that do not exist do not stand in the way).
inline int row_access(const void* p, int64_t stride, int n, int dtype, int unit) {
  const size_t size = dtype_size(dtype);
  if (!p || (n % unit == 0 && stride * (int64_t)size % 32 == 0 && aligned_to(p, 32))) return VECTORS;
  return n % 2 == 0 && stride % 2 == 0 && aligned_to(p, 2 * size) ? PAIRS : SINGLE;
}

}  // namespace snnk
