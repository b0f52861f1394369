// Elements of rows as 32-bit values, eight neighbours at a time (loads and stores of 16 bytes, which have to lie at multiples of 16) or one.
#pragma once
#include "common.hpp"

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

template <typename T, int N> struct Elems;
template <> struct Elems<bf16_t, 8> {
  u32x4_t w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *(const u32x4_t*)p; }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); }
};
template <> struct Elems<float, 8> {
  u32x4_t lo, hi;
  __device__ __forceinline__ void load(const float* p) {
    lo = *(const u32x4_t*)p;
    hi = *(const u32x4_t*)(p + 4);
  }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i < 4 ? lo[i & 3] : hi[i & 3]); }
};
template <typename T> struct Elems<T, 1> {
  T w;
  __device__ __forceinline__ void load(const T* p) { w = *p; }
  __device__ __forceinline__ float at(int) const { return load_f32(&w, 0); }
};

template <int N> __device__ __forceinline__ void store_elems(bf16_t* p, const float* f) {
  if constexpr (N == 1) {
    *p = f32_to_bf16(f[0]);
  } else {
    *(u32x4_t*)p = u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  }
}
template <int N> __device__ __forceinline__ void store_elems(float* p, const float* f) {
  if constexpr (N == 1) {
    *p = f[0];
  } else {
    *(floatx4*)p = floatx4{f[0], f[1], f[2], f[3]};
    *(floatx4*)(p + 4) = floatx4{f[4], f[5], f[6], f[7]};
  }
}

// rows of `stride` elements of `size` bytes, all at multiples of 16 bytes
inline bool rows_at_16(const void* p, long long stride, int size) { return (((uintptr_t)p | (uintptr_t)(stride * size)) & 15) == 0; }
