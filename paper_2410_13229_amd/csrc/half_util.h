// Device-side helpers of the 16-bit operators: element types, conversions, matrix instructions.
#pragma once

#include <hip/hip_runtime.h>

namespace quamba {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

template <typename T>
struct Half;  // T = _Float16 or __bf16

template <>
struct Half<_Float16> {
  typedef _Float16 v4 __attribute__((ext_vector_type(4)));
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  // lane l holds 8 consecutive k (8 (l / 32) ..) of row l % 32; result as for every 32 x 32 product
  static __device__ __forceinline__ v16f mfma32(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  // lane l holds 8 consecutive k (8 (l / 16) ..) of row l % 16; result register r = row 4 (l / 16) + r, column l % 16
  static __device__ __forceinline__ v4f mfma16(v8 a, v8 b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

template <>
struct Half<__bf16> {
  typedef __bf16 v4 __attribute__((ext_vector_type(4)));
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ v16f mfma32(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ v4f mfma16(v8 a, v8 b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

template <typename T>
__device__ __forceinline__ float to_f32(T v) {
  return static_cast<float>(v);
}
// round to nearest, ties to even
template <typename T>
__device__ __forceinline__ T from_f32(float v) {
  return static_cast<T>(v);
}

// 16 bytes a lane from the buffer's offset off (lane) + soff (wave) to consecutive LDS from `to` on; zeros where off is past the
// buffer's end (the test looks at off alone)
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t buffer, int off, int soff, char *to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (void __attribute__((address_space(3))) *)to, 16, off, soff, 0, 0);
}

// Eight consecutive elements of a row from element k on, zeros past K.  A 16-byte load at any element's address.
template <typename T>
__device__ __forceinline__ typename Half<T>::v8 row8(const T *row, int k, int K) {
  typename Half<T>::v8 v;
  if (k + 8 <= K) {
    __builtin_memcpy(&v, row + k, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < K ? row[k + e] : static_cast<T>(0.f);
  }
  return v;
}

}  // namespace quamba
