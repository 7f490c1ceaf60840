// nf_types.h - element types of the training-step operators (nf_orthogonal.hip, nf_embedding.hip).
#ifndef NF_TYPES_H
#define NF_TYPES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "nf.h"

namespace nf {

struct Bf16 {
  uint16_t u;
};

inline bool known_type(int32_t t) { return t == NF_TYPE_F32 || t == NF_TYPE_BF16 || t == NF_TYPE_F16; }
// Whether `stride` is less than what rows x cols elements take, rows `ld` apart (a product that may pass 64 bits).
inline bool overlaps(int64_t stride, int64_t rows, int64_t ld, int64_t cols) {
  return (__int128)stride < (__int128)(rows - 1) * ld + cols;
}
inline size_t type_bytes(int32_t t) { return t == NF_TYPE_F32 ? 4 : 2; }

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(_Float16 x) { return (float)x; }
__device__ __forceinline__ float to_f32(Bf16 x) { return __uint_as_float((uint32_t)x.u << 16); }

// FP32 to a type, to nearest, ties to even; NaN stays NaN.
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ _Float16 from_f32<_Float16>(float x) {
  asm("" : "+v"(x));  // else a product before it becomes one instruction that rounds to FP16 only, not to FP32 first
  return (_Float16)x;
}
template <>
__device__ __forceinline__ Bf16 from_f32<Bf16>(float x) {
  return __builtin_bit_cast(Bf16, (__bf16)x);
}

// N adjacent elements at any element's address: the card reads and writes
// whole registers across alignment.
template <typename T, int N>
struct __attribute__((packed)) Near {
  T v[N];
};

// Calls f with a null pointer of the type's element.
template <typename F>
inline void with_type(int32_t t, F f) {
  if (t == NF_TYPE_F32)
    f((float*)nullptr);
  else if (t == NF_TYPE_BF16)
    f((Bf16*)nullptr);
  else
    f((_Float16*)nullptr);
}

}  // namespace nf
#endif  // NF_TYPES_H
