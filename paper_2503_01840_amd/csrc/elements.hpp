// Rows of elements as pieces of eight, in 32 bits each.  Where every row starts at a multiple of 16 bytes and has whole pieces, a piece is loads and stores of 16 bytes.
// ODD: rows that do not (the same loads and stores, which this GPU also does at multiples of two bytes), the last piece of a row maybe shorter: an element at a time.
#pragma once
#include "common.hpp"

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_anywhere __attribute__((aligned(2)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x2_t u32x2_anywhere __attribute__((aligned(1)));

constexpr int PIECE = 8;
__host__ __device__ __forceinline__ int pieces_of(int n) { return (n + PIECE - 1) / PIECE; }

template <bool ODD> __device__ __forceinline__ u32x4_t load16(const void* p) {
  if constexpr (ODD) return *(const u32x4_anywhere*)p;
  else return *(const u32x4_t*)p;
}
template <bool ODD> __device__ __forceinline__ void store16(void* p, u32x4_t v) {
  if constexpr (ODD) *(u32x4_anywhere*)p = v;
  else *(u32x4_t*)p = v;
}

template <typename T> struct Piece8;
template <> struct Piece8<bf16_t> {
  u32x4_t w;
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); }
  // `left`: elements from p to the end of the row
  template <bool ODD> __device__ __forceinline__ void load(const bf16_t* p, int left) {
    if (!ODD || left >= PIECE) {
      w = load16<ODD>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (2 * i < left ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
  }
};
template <> struct Piece8<float> {
  u32x4_t lo, hi;
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i < 4 ? lo[i & 3] : hi[i & 3]); }
  template <bool ODD> __device__ __forceinline__ void load(const float* p, int left) {
    if (!ODD || left >= PIECE) {
      lo = load16<ODD>(p);
      hi = load16<ODD>(p + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = i < left ? __float_as_uint(p[i]) : 0u;
        hi[i] = i + 4 < left ? __float_as_uint(p[i + 4]) : 0u;
      }
    }
  }
};

template <bool ODD> __device__ __forceinline__ void store_piece(bf16_t* p, const float* f, int left) {
  if (!ODD || left >= PIECE) {
    store16<ODD>(p, u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])});
  } else {
#pragma unroll
    for (int i = 0; i < PIECE; ++i)
      if (i < left) p[i] = f32_to_bf16(f[i]);
  }
}
template <bool ODD> __device__ __forceinline__ void store_piece(float* p, const float* f, int left) {
  if (!ODD || left >= PIECE) {
    store16<ODD>(p, u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])});
    store16<ODD>(p + 4, u32x4_t{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])});
  } else {
#pragma unroll
    for (int i = 0; i < PIECE; ++i)
      if (i < left) p[i] = f[i];
  }
}

// rows of `stride` elements of `size` bytes, all at multiples of 16 bytes
inline bool rows_at_16(const void* p, long long stride, int size) { return (((uintptr_t)p | (uintptr_t)(stride * size)) & 15) == 0; }
