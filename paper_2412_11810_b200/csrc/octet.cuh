// Eight values of a row per thread, and what kernels that move such octets share.
//
// A group of 64 values (KEEP_GROUP) belongs to eight neighbouring lanes.  FAST: lane s holds values 8s .. 8s + 7, which are
// one access of 16 bytes (16-bit types) or 32 bytes (fp32: one 256-bit load or store, so that the lanes of a warp cover whole
// lines either way); it needs rows of multiples of 8 values at addresses of multiples of 16 resp. 32 bytes.  Otherwise lane s
// holds s, s + 8, ..: single values, neighbouring lanes at neighbouring addresses.
#pragma once
#include "seq_common.cuh"

namespace snnk {

template <bool FAST> __device__ __forceinline__ constexpr int octet_place(int s, int j) { return FAST ? 8 * s + j : s + 8 * j; }

// (volatile keeps the order of these accesses among one another; a store that depends on a load comes behind it anyway)
template <typename T> struct Bits;   // eight values as they lie in memory
template <> struct Bits<float> {
  uint32_t u[8];
  __device__ __forceinline__ void get(const float* p) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
                 : "l"(p));
  }
  __device__ __forceinline__ void put(float* p) const {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]),
                 "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
                 : "memory");
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = 0u;
  }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1])); }
  __device__ __forceinline__ void set(int i, float2 v) { u[2 * i] = __float_as_uint(v.x), u[2 * i + 1] = __float_as_uint(v.y); }
};
template <typename T> struct Bits16 {
  uint32_t u[4];
  __device__ __forceinline__ void get(const T* p) {
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "l"(p));
  }
  __device__ __forceinline__ void put(T* p) const {
    asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]) : "memory");
  }
  __device__ __forceinline__ void zero() { u[0] = u[1] = u[2] = u[3] = 0u; }
  __device__ __forceinline__ float2 pair(int i) const {
    typename Pair<T>::raw r;
    memcpy(&r, &u[i], 4);
    return to_f32(r);
  }
  __device__ __forceinline__ void set(int i, float2 v) {
    typename Pair<T>::raw r;
    set_raw(r, v);
    memcpy(&u[i], &r, 4);
  }
};
template <> struct Bits<__nv_bfloat16> : Bits16<__nv_bfloat16> {};
template <> struct Bits<__half> : Bits16<__half> {};

// The octet of lane s of the group that starts at column c0 of a row of n values; places behind the row's end hold zero.
template <typename T, bool FAST> struct Octet : Bits<T> {
  __device__ __forceinline__ void load(const T* row, int c0, int s, int n) {
    if (FAST) {
      if (c0 + 8 * s < n)
        this->get(row + c0 + 8 * s);
      else
        this->zero();
      return;
    }
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c0 + s + 8 * j < n ? row[c0 + s + 8 * j] : from_f32<T>(0.f);
    memcpy(this->u, v, sizeof(v));
  }
  __device__ __forceinline__ void store(T* row, int c0, int s, int n) const {
    if (FAST) {
      if (c0 + 8 * s < n) this->put(row + c0 + 8 * s);
      return;
    }
    T v[8];
    memcpy(v, this->u, sizeof(v));
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c0 + s + 8 * j < n) row[c0 + s + 8 * j] = v[j];
  }
};

// Eight codes (two per word of q, low first) of lane s of the group at column c0.
template <bool FAST> __device__ __forceinline__ void store_codes(uint8_t* row, int c0, int s, int n, const uint32_t q[4]) {
  if (FAST) {
    if (c0 + 8 * s < n) *reinterpret_cast<uint2*>(row + c0 + 8 * s) = make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (c0 + s + 8 * j < n) row[c0 + s + 8 * j] = (uint8_t)(q[j / 2] >> (8 * (j % 2)));
}
// Largest magnitude of a group as a bit pattern, from that of its eight lanes; NaN sorts above infinity above the rest.
__device__ __forceinline__ uint32_t group_top(float m) {
  uint32_t top = __float_as_uint(m);
#pragma unroll
  for (int o = 1; o < 8; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  return top;
}

// ---- launches behind one another's start ---------------------------------------------------------------------
__device__ __forceinline__ void wait_for_kernel_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;"); }

// behind: the kernel may be set up while the one before it in the stream runs; it calls wait_for_kernel_before() before it
// touches anything that one writes or reads.
template <typename... P, typename... A>
snn_status launch_behind(void (*kernel)(P...), unsigned grid, int threads, size_t smem, cudaStream_t stream, bool behind, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = &at;
  cfg.numAttrs = behind ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
}

inline bool aligned_to(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }
// whether rows can be accessed eight values at a time (a row that does not exist does not stand in the way)
inline bool octet_rows(const void* p, int64_t stride, int dtype) { return !p || (stride % 8 == 0 && aligned_to(p, 8 * dtype_size(dtype))); }

}  // namespace snnk
