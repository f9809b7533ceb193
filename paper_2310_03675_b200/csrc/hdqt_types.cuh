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

// Sixteen bytes of elements held as four words.  A Vec of 16-bit elements that lives across a branch or a loop turn is taken apart
// into eight half-word registers by the compiler, which costs more instructions than the arithmetic on them.
struct alignas(16) Words {
  uint32_t w[4];
};
template <typename T>
__device__ __forceinline__ void unpack(const Words& v, float (&f)[16 / sizeof(T)]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      f[i] = __uint_as_float(v.w[i]);
    } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
      f[2 * i] = __uint_as_float(v.w[i] << 16);
      f[2 * i + 1] = __uint_as_float(v.w[i] & 0xFFFF0000u);
    } else {
      const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&v.w[i]));
      f[2 * i] = t.x;
      f[2 * i + 1] = t.y;
    }
  }
}
template <typename T>
__device__ __forceinline__ Words pack_words(const float (&f)[16 / sizeof(T)]) {
  Words v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) v.w[i] = __float_as_uint(f[i]);
    else if constexpr (std::is_same_v<T, __nv_bfloat16>) *reinterpret_cast<__nv_bfloat162*>(&v.w[i]) = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    else *reinterpret_cast<__half2*>(&v.w[i]) = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
  }
  return v;
}

// ---- pairs of fp32 operations as one instruction ----------------------------------------------------------------

__device__ __forceinline__ void add2(float& a0, float& a1, float b0, float b1) {
  asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %3};\nadd.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
      : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1));
}
__device__ __forceinline__ void mul2(float& a0, float& a1, float b0, float b1) {
  asm("{\n.reg .b64 a, b;\nmov.b64 a, {%0, %1};\nmov.b64 b, {%2, %3};\nmul.rn.f32x2 a, a, b;\nmov.b64 {%0, %1}, a;\n}"
      : "+f"(a0), "+f"(a1) : "f"(b0), "f"(b1));
}
// o = a b + c
__device__ __forceinline__ void fma2(float& o0, float& o1, float a0, float a1, float b0, float b1, float c0, float c1) {
  asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 a, a, b, c;\nmov.b64 {%0, %1}, a;\n}"
      : "=f"(o0), "=f"(o1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}

// ---- activations and what they are made of ----

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
// in the first kernel of a call: the next one may be set up while this one ends
__device__ __forceinline__ void chain_next() { asm volatile("griddepcontrol.launch_dependents;"); }
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

// 1 / (1 + exp(-z)); exp overflows to infinity for z < -88, where the reciprocal is the correct 0
__device__ __forceinline__ float sigmoid(float z) { return rcp(1.0f + ex2(z * -kLog2e)); }

template <int kAct>
__device__ __forceinline__ float act_fwd(float z) {
  if constexpr (kAct == HDQT_ACT_RELU) {      // (a NaN stays)
    float r;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(z));
    return r;
  }
  if constexpr (kAct == HDQT_ACT_SILU) return z * sigmoid(z);
  return z;
}
// dy * act'(z)
template <int kAct>
__device__ __forceinline__ float act_bwd(float dy, float z) {
  if constexpr (kAct == HDQT_ACT_RELU) return z > 0.0f ? dy : 0.0f;
  if constexpr (kAct == HDQT_ACT_SILU) {
    const float s = sigmoid(z);
    return dy * fmaf(s * (1.0f - s), z, s);
  }
  return dy;
}
// f<activation>() for the call's activation: the loops inside know it at compile time
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == HDQT_ACT_SILU) f.template operator()<HDQT_ACT_SILU>();
  else if (act == HDQT_ACT_RELU) f.template operator()<HDQT_ACT_RELU>();
  else f.template operator()<HDQT_ACT_NONE>();
}

// ---- host side ----

inline int dtype_size(int64_t dtype) {   // 0 = unknown type
  return dtype == HDQT_DTYPE_F32 ? 4 : (dtype == HDQT_DTYPE_BF16 || dtype == HDQT_DTYPE_F16) ? 2 : 0;
}

// widest access (16 bytes, or down to one element) that `align` (bases and strides in bytes, or-ed together) allows
inline int vector_width(int64_t channels, int elem, uintptr_t align) {
  int v = 16 / elem;
  while (v > 1 && (channels % v != 0 || (align & (uintptr_t)(v * elem - 1)) != 0)) v >>= 1;
  return v;
}

template <typename F>
hdqt_status_t with_type_and_width(int dtype, int vec, F&& f) {
  if (dtype == HDQT_DTYPE_F32) {
    if (vec == 4) return f.template operator()<float, 4>();
    if (vec == 2) return f.template operator()<float, 2>();
    return f.template operator()<float, 1>();
  }
  if (dtype == HDQT_DTYPE_BF16) {
    if (vec == 8) return f.template operator()<__nv_bfloat16, 8>();
    if (vec == 4) return f.template operator()<__nv_bfloat16, 4>();
    if (vec == 2) return f.template operator()<__nv_bfloat16, 2>();
    return f.template operator()<__nv_bfloat16, 1>();
  }
  if (vec == 8) return f.template operator()<__half, 8>();
  if (vec == 4) return f.template operator()<__half, 4>();
  if (vec == 2) return f.template operator()<__half, 2>();
  return f.template operator()<__half, 1>();
}

inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

inline hdqt_status_t last_error(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? HDQT_OK : cuda_failure(e, what);
}

// dgamma (y) and dbeta (x): sums of the parts [parts, channels] of a backward pass, in a fixed order; NULL = not needed
void launch_param_grad(const float2* part, int64_t parts, int channels, void* dgamma, void* dbeta, int32_t param_dtype, bool chained,
                       cudaStream_t s);

}  // namespace hdqt
