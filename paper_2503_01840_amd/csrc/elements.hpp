// Rows of elements as pieces of N (8 or 4), in 32 bits each, a piece one load or store of at most 16 bytes, neighbouring lanes' pieces one behind the other: 8 bf16 elements, or 4
// where an fp32 row is among a kernel's (two stores of 16 bytes 32 apart for 8 of them take 1.5 times as long).  ODD: rows that do not start at multiples of a piece's
// bytes (the same loads and stores, which this GPU also does at multiples of an element's), or whose last piece is shorter: loaded as the row's last N elements and shifted when they are there
// where elements have 16 bits (element by element each would be waited for: the gradient of 16384 rows of 4095 241 us instead of 149), element by element where they
// have 32, and stored 4, 2 and 1 at a time.
#pragma once
#include "common.hpp"

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x4_t u32x4_anywhere __attribute__((aligned(2)));
typedef u32x2_t u32x2_anywhere __attribute__((aligned(1)));
typedef uint32_t u32_anywhere __attribute__((aligned(1)));

__host__ __device__ __forceinline__ int pieces_of(int n, int N) { return (n + N - 1) / N; }

// words of 4, 8 or 16 bytes
template <int BYTES> struct Words;
template <> struct Words<4> { typedef uint32_t type; typedef u32_anywhere anywhere; };
template <> struct Words<8> { typedef u32x2_t type; typedef u32x2_anywhere anywhere; };
template <> struct Words<16> { typedef u32x4_t type; typedef u32x4_anywhere anywhere; };

template <typename T, int N> struct Piece {
  static constexpr int BYTES = N * sizeof(T);
  typedef typename Words<BYTES>::type words;
  words w;
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
  // `left`: elements from p to the end of the row of `dim`; settle() follows, once, before the elements are used
  template <bool ODD> __device__ __forceinline__ void load(const T* p, int left, int dim) {
    if constexpr (!ODD) {
      w = *(const words*)p;
    } else if constexpr (sizeof(T) == 4) {
      if (left >= N) {
        w = *(const typename Words<BYTES>::anywhere*)p;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = i < left ? __float_as_uint(p[i]) : 0u;
      }
    } else if (dim >= N) {
      w = *(const typename Words<BYTES>::anywhere*)(p - max(N - left, 0));
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w[i] = (2 * i < left ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
  }
  // bf16: the elements that there are to the front, zeros behind them.
  template <bool ODD> __device__ __forceinline__ void settle(int left, int dim) {
    if constexpr (ODD && sizeof(T) == 2) {
      constexpr int W = BYTES / 4;
      if (left >= N || dim < N) return;
      int k = N - left;
      if (k & 1) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = i + 1 < W ? w[i] >> 16 | w[i + 1] << 16 : w[i] >> 16;
      }
      k >>= 1;
      if (k & 1) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = i + 1 < W ? w[i + 1] : 0u;
      }
      if (k & 2) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = i + 2 < W ? w[i + 2] : 0u;
      }
    }
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    }
  }
};

// STREAM: past the caches, for results that are larger than these
template <int N, bool ODD, bool STREAM = false, typename T> __device__ __forceinline__ void store_piece(T* p, const float* f, int left) {
  Piece<T, N> v;
  v.set(f);
  if constexpr (!ODD) {
    typedef typename Piece<T, N>::words words;
    if constexpr (STREAM) __builtin_nontemporal_store(v.w, (words*)p);
    else *(words*)p = v.w;
  } else if (left >= N) {
    *(typename Words<Piece<T, N>::BYTES>::anywhere*)p = v.w;
  } else if constexpr (sizeof(T) == 4) {                      // N = 4: 2 elements and 1
    if (left & 2) *(u32x2_anywhere*)p = u32x2_t{v.w[0], v.w[1]};
    if (left & 1) p[left & 2] = __uint_as_float(left & 2 ? v.w[2] : v.w[0]);
  } else {                                                    // 4 elements, 2 and 1
    if constexpr (N == 8)
      if (left & 4) *(u32x2_anywhere*)p = u32x2_t{v.w[0], v.w[1]};
    const uint32_t next = N == 8 && (left & 4) ? v.w[N / 2 - 2] : v.w[0], behind = N == 8 && (left & 4) ? v.w[N / 2 - 1] : v.w[1];
    if (left & 2) *(u32_anywhere*)(p + (left & 4)) = next;
    if (left & 1) p[left & 6] = (T)(left & 2 ? behind : next);
  }
}

// rows of `stride` elements of `size` bytes, all at multiples of 16 bytes
inline bool rows_at_16(const void* p, long long stride, int size) { return (((uintptr_t)p | (uintptr_t)(stride * size)) & 15) == 0; }
