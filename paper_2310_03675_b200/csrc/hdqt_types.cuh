// Element types of the floating-point operators: conversions to and from fp32 and vector accesses.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "hdqt_common.cuh"

namespace hdqt {

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

// one rounding, ties to even
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N elements of T as one access; the address must be aligned to sizeof(Vec)
template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// all N elements to and from fp32, two at a time where there are two
template <typename T, int N>
__device__ __forceinline__ void unpack(const Vec<T, N>& v, float (&f)[N]) {
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(&v.v[i]);   // bf16 is the upper half of an fp32
        f[i] = __uint_as_float(w << 16);
        f[i + 1] = __uint_as_float(w & 0xFFFF0000u);
      } else {
        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&v.v[i]));
        f[i] = t.x;
        f[i + 1] = t.y;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f32(v.v[i]);
  }
}
template <typename T, int N>
__device__ __forceinline__ Vec<T, N> pack(const float (&f)[N]) {
  Vec<T, N> v;
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      if constexpr (std::is_same_v<T, __nv_bfloat16>) *reinterpret_cast<__nv_bfloat162*>(&v.v[i]) = __floats2bfloat162_rn(f[i], f[i + 1]);
      else *reinterpret_cast<__half2*>(&v.v[i]) = __floats2half2_rn(f[i], f[i + 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v.v[i] = from_f32<T>(f[i]);
  }
  return v;
}

// hardware approximations (2 units in the last place or better; results below 2^-126 become 0)
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;

// Element i of a parameter vector whose type is known at run time only.  Plain loads: the 16-bit forms of __ldg are
// inline assembly that the compiler may execute ahead of the test that guards it, and a pointer may be null behind such a test.
__device__ __forceinline__ float load_param(const void* p, int32_t dtype, int64_t i) {
  if (dtype == HDQT_DTYPE_F32) return reinterpret_cast<const float*>(p)[i];
  if (dtype == HDQT_DTYPE_BF16) return to_f32(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
  return to_f32(reinterpret_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_param(void* p, int32_t dtype, int64_t i, float v) {
  if (dtype == HDQT_DTYPE_F32) reinterpret_cast<float*>(p)[i] = v;
  else if (dtype == HDQT_DTYPE_BF16) reinterpret_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(v);
  else reinterpret_cast<__half*>(p)[i] = from_f32<__half>(v);
}

// Programmatic dependent launch: the kernels of one call start while their predecessor runs and wait here for its results, so that
// launch latency is paid once per call.  The first kernel of a call is launched the ordinary way (behind everything
// before it); nothing may be read or written ahead of the wait.
__device__ __forceinline__ void chain_wait() {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
template <typename... P, typename... A>
inline void launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);      // (a failure is left for cudaGetLastError)
}

inline int dtype_size(int64_t dtype) {   // 0 = unknown type
  return dtype == HDQT_DTYPE_F32 ? 4 : (dtype == HDQT_DTYPE_BF16 || dtype == HDQT_DTYPE_F16) ? 2 : 0;
}

}  // namespace hdqt
