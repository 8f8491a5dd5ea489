// Element types of the operators that take more than fp32: their numbers at the C boundary (those of idkm_set_wq_dtype) and
// the conversions to and from fp32, which all of them compute in.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace idkm {

enum ElemType { ELEM_F32 = 0, ELEM_BF16 = 1, ELEM_F16 = 2 };

inline int elem_bytes(int type) { return type == ELEM_F32 ? 4 : 2; }
inline bool elem_known(int type) { return type >= ELEM_F32 && type <= ELEM_F16; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

template <class T>
__device__ __forceinline__ T from_f32(float x);   // to nearest even
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// 16 bytes of elements, as they lie in memory.
template <class T>
struct Vec16 {
  static constexpr int N = 16 / (int)sizeof(T);
  union {
    uint4 raw;
    T e[N];
  };
  __device__ __forceinline__ Vec16() {}
};

// Calls f with a null pointer of the element type's C++ type.
template <class F>
inline int with_type(int type, F f) {
  switch (type) {
    case ELEM_F32: return f((float*)nullptr);
    case ELEM_BF16: return f((__nv_bfloat16*)nullptr);
    default: return f((__half*)nullptr);
  }
}

}  // namespace idkm
