// Rotary positions of queries and keys, and their gradient.
//
// A wavefront has one row (or a part of its heads): each lane forms the sine and cosine of one pair's angle and puts them into LDS; then the lanes take
// 16-byte pieces of the heads, in the half layout two pieces that belong together, four of them in flight.  The angle is a fraction of
// a turn, position times turns per position in 64 bits less its whole part, so that the 32-bit sine and cosine of it are as good at position
// 131071 as at position 1.  Bound by bytes, every row read and written once: 16384 rows of 64 + 8 heads of 128 in bf16 124.5 us, 4.85 TB/s, a large copy's rate (239 with one
// pair to a thread and round); 2047 rows of 32 + 8 heads in fp32, half of each head rotated, 16.8 us, 5.0 TB/s.  Sizes and addresses that do not fill 16 bytes go an element at a time, bound
// by instructions and requests in bf16: the prompt above with 122 of 128 dimensions rotated 197 us, 3.1 TB/s (neighbours 234), 5512 rows 79 us, in fp32 99 us, 4.1 TB/s.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int MAX_PAIRS = 512;

// cosine and signed sine of pair i at this position, times the amplitude
__device__ __forceinline__ void angle(const RopeAngles& a, double pos, int i, float* cs, float* sn) {
  const double f = a.turns[i];
  float s, c;
  sincospif(2.f * (float)fma(pos, f, -rint(pos * f)), &s, &c);
  cs[i] = a.amplitude * c;
  sn[i] = a.sign * a.amplitude * s;
}

// One pair, rotated: the same bits in every kernel.
__device__ __forceinline__ void turn(float xa, float xb, float c, float s, float& ya, float& yb) {
  ya = fmaf(xa, c, -(xb * s));
  yb = fmaf(xb, c, xa * s);
}

// N elements, as one load or store
template <int BYTES> struct Bits;
template <> struct Bits<2> { typedef uint16_t type; };
template <> struct Bits<4> { typedef uint32_t type; };
template <> struct Bits<16> { typedef u32x4 type; };
template <typename T, int N> struct Piece {
  typename Bits<N * sizeof(T)>::type w;
  __device__ __forceinline__ float at(int i) const {
    if constexpr (N == 1) return load_f32((const T*)&w, 0);
    else if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (N == 1) {
      store_from_f32((T*)&w, 0, f[0]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
        else w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
      }
    }
  }
};

// A task is a piece of a head, the first `turning` ones to be rotated.  N > 1: pieces of 16 bytes; neighbours as pairs within a piece (INSIDE), else with the piece
// `apart` elements on.  N = 1, for any sizes and addresses: the first element of a pair, `step` elements behind the one of the task before.  Tasks of a row go over
// `share` each of gridDim.y wavefronts.
template <typename T, int N, bool INSIDE>
__global__ __launch_bounds__(256) void rope_kernel(RopeTensor q, RopeTensor k, RopeAngles a, int rows, int d, Divisor per_head, int turning, int apart, int step, int share) {
  constexpr int U = N == 1 ? 8 : 4;
  typedef Piece<T, N> P;
  __shared__ __attribute__((aligned(16))) float cs[4][MAX_PAIRS], sn[4][MAX_PAIRS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = blockIdx.x * 4 + wave, half = a.rot >> 1;
  if (r >= rows) return;
  const int tasks = (q.heads + k.heads) * per_head.d, first = blockIdx.y * share, last = min(tasks, first + share);
  const T* qx = (const T*)q.x + (size_t)r * q.stride;
  const T* kx = (const T*)k.x + (size_t)r * k.stride;
  T* qy = (T*)q.y + (size_t)r * q.y_stride;
  T* ky = (T*)k.y + (size_t)r * k.y_stride;
  bool ready = false;
  for (int u0 = first; u0 < last; u0 += 64 * U) {
    P lo[U], hi[U];
    int task[U];
    T* to[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = u0 + 64 * j + lane;
      task[j] = -1;
      if (u < last) {
        const int h = u / per_head, t = u % per_head;
        const bool is_k = h >= q.heads;
        const size_t off = (size_t)(is_k ? h - q.heads : h) * d + (t < turning ? t * step : a.rot + (t - turning) * N);
        const T* x = (is_k ? kx : qx) + off;
        to[j] = (is_k ? ky : qy) + off;
        task[j] = t;
        lo[j] = *(const P*)x;
        if (!INSIDE && t < turning) hi[j] = *(const P*)(x + apart);
      }
    }
    if (!ready) {
      const double pos = (double)a.positions[r];
      for (int i = lane; i < half; i += 64) angle(a, pos, i, cs[wave], sn[wave]);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      ready = true;
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int t = task[j];
      if (t < 0) continue;
      if (t >= turning) {
        *(P*)to[j] = lo[j];
      } else if constexpr (INSIDE) {
        float f[N];
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
          turn(lo[j].at(2 * i), lo[j].at(2 * i + 1), cs[wave][t * (N / 2) + i], sn[wave][t * (N / 2) + i], f[2 * i], f[2 * i + 1]);
        lo[j].set(f);
        *(P*)to[j] = lo[j];
      } else {
        float fa[N], fb[N];
#pragma unroll
        for (int i = 0; i < N; ++i) turn(lo[j].at(i), hi[j].at(i), cs[wave][t * N + i], sn[wave][t * N + i], fa[i], fb[i]);
        lo[j].set(fa);
        hi[j].set(fb);
        *(P*)to[j] = lo[j];
        *(P*)(to[j] + apart) = hi[j];
      }
    }
  }
}

bool aligned(const RopeTensor& t, int size) {
  return !t.x || ((((uintptr_t)t.x | (uintptr_t)t.y) & 15) == 0 && t.stride * size % 16 == 0 && t.y_stride * size % 16 == 0);
}

template <typename T>
hipError_t launch(const RopeTensor& q, const RopeTensor& k, const RopeAngles& a, int rows, int d, hipStream_t st) {
  constexpr int WIDE = 16 / sizeof(T);
  const int half = a.rot / 2, unit = a.interleaved ? a.rot : half;                  // what pieces to be rotated have to fill
  const bool wide = d % WIDE == 0 && unit % WIDE == 0 && aligned(q, sizeof(T)) && aligned(k, sizeof(T));
  const int n = wide ? WIDE : 1, turning = wide ? unit / WIDE : half;
  const bool in_place = q.x == q.y && (!k.x || k.x == k.y);         // then the rest of a head stays as it is
  const int per_head = turning + (in_place ? 0 : (d - a.rot) / n), tasks = (q.heads + k.heads) * per_head;
  // up to some thousand rows: a row over several wavefronts, each with the row's angles of its own (one / several, us: 4 rows of 72 heads 5.8 / 2.5, of 512 30.0 / 2.6, 1000 rows
  // of 72 9.2 / 6.6, 2047 fp32 rows of 40, half of each head 18.1 / 14.8 out of the last-level cache; an empty launch takes 2.2)
  const int most = (tasks + 63) / 64, want = std::max(1, std::min(most, 8192 / rows));
  const int share = (most + want - 1) / want * 64;
  const dim3 grid((rows + 3) / 4, (tasks + share - 1) / share);
  const Divisor by = divisor(per_head);
  if (!wide)
    hipLaunchKernelGGL((rope_kernel<T, 1, false>), grid, dim3(256), 0, st, q, k, a, rows, d, by, turning, a.interleaved ? 1 : half, a.interleaved ? 2 : 1, share);
  else if (a.interleaved)
    hipLaunchKernelGGL((rope_kernel<T, WIDE, true>), grid, dim3(256), 0, st, q, k, a, rows, d, by, turning, 0, WIDE, share);
  else
    hipLaunchKernelGGL((rope_kernel<T, WIDE, false>), grid, dim3(256), 0, st, q, k, a, rows, d, by, turning, half, WIDE, share);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(bool bf16, const RopeTensor& q, const RopeTensor& k, const RopeAngles& a, int rows, int d, hipStream_t st) {
  return bf16 ? launch<bf16_t>(q, k, a, rows, d, st) : launch<float>(q, k, a, rows, d, st);
}
