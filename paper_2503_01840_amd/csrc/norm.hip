// The residual stream and its root-mean-square norm, the norm in 8 bits, and the gradient of both.
//
// A row h = x + residual is read once into the registers of its 8 to 1024 threads, its squares are summed by exchanges within the wavefronts and through LDS between
// them, and the row is written as h and as gain * h / sqrt(mean + eps).  The gradient's rows go to at most 512 workgroups in turn, which keep the gains' gradient in
// registers; their parts are added by a second launch (4.8 us).  Bound by bytes, at a large copy's rate and above where rows are many: 16384 rows of 8192 in bf16 180 to 182 us
// (5.9 TB/s), 8192 of 4096 onto an fp32 stream 72 (5.6), 2048 of 8192 in 8 bits 25.2 (4.7), the gradient of 8191 rows of 4096 on an fp32 stream 102 (5.3).
// Measured and not kept: an eighth of the rows to each XCD (2 to 17 % slower); the gradient's next row asked for while one is worked on (0 to 8 % slower); results stored past the
// caches (2 to 10 % faster alone, but with an addition behind it that reads them 4096 rows of 8192 in bf16 72 -> 79 us).
// 1024 threads have 128 registers each.  A gradient with an fp32 type among more than 8192 columns, four pieces to a thread, wants more: up to 12 to a thread are spilled where rows are whole, up
// to 40 where they are odd.
#include <algorithm>

#include "elements.hpp"
#include "kernels.hpp"

namespace {

constexpr float CODE_MOST = 448.f, LEAST_SCALE = 0x1p-100f;
__host__ __device__ __forceinline__ int padded(int dim) { return (dim + 7) & ~7; }
constexpr int MANY_ROWS = 1024;
template <typename X, typename H, typename Y> constexpr int piece_size() { return sizeof(X) == 4 || sizeof(H) == 4 || sizeof(Y) == 4 ? 4 : 8; }

// The sum over the 2^lg threads of a row (8 to 1024, neighbours), the same on each; wavefronts in order, `red` a place for each of the workgroup's.
__device__ __forceinline__ float wave_part_sum(float v, int lg) {
  v = xlane_sum_step<2>(xlane_sum_step<1>(xlane_sum_step<0>(v)));
  if (lg > 3) v = xlane_sum_step<3>(v);
  if (lg > 4) v = xlane_sum_step<4>(v);
  if (lg > 5) v = xlane_sum_step<5>(v);
  return v;
}
__device__ __forceinline__ float row_sum(float v, int lg, float* red) {
  v = wave_part_sum(v, lg);
  if (lg <= 6) return v;
  const int wave = threadIdx.x >> 6, W = 1 << (lg - 6);
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  const float* mine = red + (wave & -W);
  v = mine[0];
  for (int i = 1; i < W; ++i) v += mine[i];
  return v;
}

template <bool ODD, int N> __device__ __forceinline__ void load_gains(const NormRows& a, int p, float* g) {
  const int left = a.dim - p * N;
  if (a.gain_bf16) {
    Piece<bf16_t, N> w;
    w.template load<ODD>((const bf16_t*)a.gain + p * N, left, a.dim);
    w.template settle<ODD>(left, a.dim);
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = w.at(i);
  } else {
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      Piece<float, 4> w;
      w.template load<ODD>((const float*)a.gain + p * N + k, left - k, a.dim);
      w.template settle<ODD>(left - k, a.dim);
#pragma unroll
      for (int i = 0; i < 4; ++i) g[k + i] = w.at(i);
    }
  }
}

__device__ __forceinline__ float finite_magnitude(float x) {
  const float a = fabsf(x);
  return a < __builtin_huge_valf() ? a : 0.f;
}
__device__ __forceinline__ float scale_of(float amax) { return fmaxf(amax / CODE_MOST, LEAST_SCALE); }

// Values under a scale: the product with its reciprocal and one step from there, which around every border between two codes is the nearest fp32 of the quotient, so that each code is
// the one that a division gives (the product alone, off by up to two last places, took a neighbour's now and then).  Scales below 2^-64 are raised, or what the step multiplies would leave
// fp32's range.  2048 bf16 rows of 8192 take 25.2 us, by products alone 24.1.
struct Quotient {
  float raise, scale, inv;
  __device__ __forceinline__ Quotient(float s) : raise(s < 0x1p-64f ? 0x1p64f : 1.f), scale(s * raise), inv(1.f / scale) {}
  __device__ __forceinline__ float operator()(float x) const {
    x *= raise;
    const float q = x * inv;
    return fmaf(fmaf(-q, scale, x), inv, q);
  }
};
// Two values under a scale as codes; what is not finite as NaN.
__device__ __forceinline__ uint32_t to_codes(float a, float b, const Quotient& under) {
  const float ya = fminf(fmaxf(under(a), -CODE_MOST), CODE_MOST), yb = fminf(fmaxf(under(b), -CODE_MOST), CODE_MOST);
  uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(ya, yb, 0, false) & 0xFFFFu;
  if (!(fabsf(a) < __builtin_huge_valf())) c = (c & 0xFF00u) | 0x7Fu;
  if (!(fabsf(b) < __builtin_huge_valf())) c = (c & 0x00FFu) | 0x7F00u;
  return c;
}

// Y: type of the norm; uint8_t: codes, a.group columns to a scale (0: a row).  2^lg threads to a row, P pieces to a thread.
template <typename X, typename H, typename Y, bool ADDED, bool ODD, int P>
__global__ __launch_bounds__(1024) void add_norm_kernel(NormRows a, int lg) {
  constexpr bool CODES = sizeof(Y) == 1;
  constexpr int N = piece_size<X, H, Y>();
  __shared__ float red[16], most[CODES ? 16 : 1];
  const int per = blockDim.x >> lg, t = threadIdx.x & ((1 << lg) - 1);
  const long long row = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * per + (threadIdx.x >> lg);
  const int pieces = row < a.rows ? pieces_of(a.dim, N) : 0;
  Piece<X, N> x[P];
  Piece<H, N> res[P];
  float h[P][N];
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int p = t + (j << lg);
    if (p < pieces) {
      x[j].template load<ODD>((const X*)a.x + row * a.x_stride + (long long)p * N, a.dim - p * N, a.dim);
      if constexpr (ADDED) res[j].template load<ODD>((const H*)a.residual + row * a.residual_stride + (long long)p * N, a.dim - p * N, a.dim);
    }
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int p = t + (j << lg);
    if (p < pieces) {
      x[j].template settle<ODD>(a.dim - p * N, a.dim);
      if constexpr (ADDED) res[j].template settle<ODD>(a.dim - p * N, a.dim);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        h[j][i] = x[j].at(i);
        if constexpr (ADDED) h[j][i] += res[j].at(i);
        sum = fmaf(h[j][i], h[j][i], sum);
      }
      if constexpr (ADDED) store_piece<N, ODD>((H*)a.sum_out + row * a.sum_stride + (long long)p * N, h[j], a.dim - p * N);
    }
  }
  const float r = 1.f / sqrtf(row_sum(sum, lg, red) / (float)a.dim + a.eps);
  if constexpr (!CODES) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + (j << lg);
      if (p < pieces) {
        float g[N];
        load_gains<ODD, N>(a, p, g);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] *= h[j][i] * r;
        store_piece<N, ODD>((Y*)a.out + row * a.out_stride + (long long)p * N, g, a.dim - p * N);
      }
    }
  } else {
    const int n_scales = a.group ? (a.dim + a.group - 1) / a.group : 1;
    float amax = 0.f, part[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + (j << lg);
      part[j] = 0.f;
      if (p < pieces) {
        float g[N];
        load_gains<ODD, N>(a, p, g);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          h[j][i] = g[i] * (h[j][i] * r);
          if (!ODD || i < a.dim - p * N) part[j] = fmaxf(part[j], finite_magnitude(h[j][i]));
        }
      }
      if (a.group) {                                          // 128 / N lanes have a group
        part[j] = xlane_max_step<3>(xlane_max_step<2>(xlane_max_step<1>(xlane_max_step<0>(part[j]))));
        if constexpr (N == 4) part[j] = xlane_max_step<4>(part[j]);
      } else {
        amax = fmaxf(amax, part[j]);
      }
    }
    if (!a.group) {
      amax = xlane_max_step<3>(xlane_max_step<2>(xlane_max_step<1>(xlane_max_step<0>(amax))));
      if (lg > 4) amax = xlane_max_step<4>(amax);
      if (lg > 5) amax = xlane_max_step<5>(amax);
      if (lg > 6) {
        const int wave = threadIdx.x >> 6, W = 1 << (lg - 6);
        if ((threadIdx.x & 63) == 0) most[wave] = amax;
        __syncthreads();
        for (int i = 0; i < W; ++i) amax = fmaxf(amax, most[(wave & -W) + i]);
      }
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + (j << lg);
      if (p >= pieces) continue;
      const float scale = scale_of(a.group ? part[j] : amax);
      const Quotient under(scale);
      if (a.group ? p * N % 128 == 0 : p == 0) a.scales[row * n_scales + (a.group ? p * N / 128 : 0)] = scale;
      uint8_t* to = (uint8_t*)a.out + row * a.out_stride + (long long)p * N;
      typename Words<N>::type c;
      if constexpr (N == 8) c = u32x2_t{to_codes(h[j][0], h[j][1], under) | to_codes(h[j][2], h[j][3], under) << 16, to_codes(h[j][4], h[j][5], under) | to_codes(h[j][6], h[j][7], under) << 16};
      else c = to_codes(h[j][0], h[j][1], under) | to_codes(h[j][2], h[j][3], under) << 16;
      if constexpr (!ODD) {
        *(typename Words<N>::type*)to = c;
      } else if (a.dim - p * N >= N) {
        *(typename Words<N>::anywhere*)to = c;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i < a.dim - p * N) to[i] = (uint8_t)(((const uint32_t*)&c)[i / 4] >> 8 * (i & 3));
      }
    }
  }
}

// Gradient of the sum, rows dealt out in turn; the gains' gradient of a workgroup's rows to its part of the workspace, padded(dim) apart.  dynamic LDS: that many floats
// where a workgroup has several rows at a time.
template <typename X, typename H, typename Y, bool ODD, int P>
__global__ __launch_bounds__(1024) void add_norm_grad_kernel(NormGradRows b, int lg) {
  constexpr int N = piece_size<X, H, Y>();
  extern __shared__ float gains[];
  __shared__ float red[2][2][16];
  const NormRows& a = b.fwd;
  const int wave = threadIdx.x >> 6, per = blockDim.x >> lg, group = threadIdx.x >> lg, t = threadIdx.x & ((1 << lg) - 1), all = pieces_of(a.dim, N);
  float g[P][N], dg[P][N];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int p = t + (j << lg);
#pragma unroll
    for (int i = 0; i < N; ++i) g[j][i] = dg[j][i] = 0.f;
    if (p < all) load_gains<ODD, N>(a, p, g[j]);
  }
  int turn = 0;
  for (long long r0 = (long long)blockIdx.x * per; r0 < a.rows; r0 += (long long)gridDim.x * per, turn ^= 1) {
    const long long row = r0 + group;
    const int pieces = row < a.rows ? all : 0;
    Piece<Y, N> dy[P];
    Piece<H, N> h[P], dh[P];
    float hh = 0.f, gh = 0.f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + (j << lg);
      if (p < pieces) {
        dy[j].template load<ODD>((const Y*)b.dy + row * b.dy_stride + (long long)p * N, a.dim - p * N, a.dim);
        h[j].template load<ODD>((const H*)b.h + row * b.h_stride + (long long)p * N, a.dim - p * N, a.dim);
        if (b.dh) dh[j].template load<ODD>((const H*)b.dh + row * b.dh_stride + (long long)p * N, a.dim - p * N, a.dim);
      }
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + (j << lg);
      if (p < pieces) {
        dy[j].template settle<ODD>(a.dim - p * N, a.dim);
        h[j].template settle<ODD>(a.dim - p * N, a.dim);
        if (b.dh) dh[j].template settle<ODD>(a.dim - p * N, a.dim);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          hh = fmaf(h[j].at(i), h[j].at(i), hh);
          gh = fmaf(g[j][i] * dy[j].at(i), h[j].at(i), gh);
        }
      }
    }
    hh = wave_part_sum(hh, lg);
    gh = wave_part_sum(gh, lg);
    if (lg > 6) {                                             // two places in turn: one barrier a row
      const int W = 1 << (lg - 6);
      if ((threadIdx.x & 63) == 0) {
        red[turn][0][wave] = hh;
        red[turn][1][wave] = gh;
      }
      __syncthreads();
      hh = red[turn][0][wave & -W];
      gh = red[turn][1][wave & -W];
      for (int i = 1; i < W; ++i) {
        hh += red[turn][0][(wave & -W) + i];
        gh += red[turn][1][(wave & -W) + i];
      }
    }
    const float r = 1.f / sqrtf(hh / (float)a.dim + a.eps), c = r * (gh / (float)a.dim);       // of the normalised row: r's cube leaves fp32 where a row is small
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + (j << lg);
      if (p < pieces) {
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float d = dy[j].at(i), v = h[j].at(i) * r;
          y[i] = r * fmaf(-v, c, g[j][i] * d);
          if (b.dh) y[i] += dh[j].at(i);
          dg[j][i] = fmaf(d, v, dg[j][i]);
        }
        if (b.d_sum) store_piece<N, ODD>((H*)b.d_sum + row * b.d_sum_stride + (long long)p * N, y, a.dim - p * N);
        if (b.dx) store_piece<N, ODD>((X*)b.dx + row * b.dx_stride + (long long)p * N, y, a.dim - p * N);
      }
    }
  }
  if (!b.partial) return;
  float* to = b.partial + (size_t)blockIdx.x * padded(a.dim);
  if (per > 1) {                                              // rows of a wavefront by exchanges, of a workgroup one after the other
    if (lg < 6) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (lg <= 3) dg[j][i] += __shfl_xor(dg[j][i], 8, 64);     // step 3 is a mirror: lanes of other columns
          if (lg <= 4) dg[j][i] = xlane_sum_step<4>(dg[j][i]);
          dg[j][i] = xlane_sum_step<5>(dg[j][i]);
        }
      }
    }
    const int turns = lg < 6 ? blockDim.x >> 6 : per, own_turn = lg < 6 ? ((threadIdx.x & 63) >> lg ? -1 : wave) : group;
    for (int w = 0; w < turns; ++w) {
      if (w == own_turn) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const int p = t + (j << lg);
          if (p < all) {
#pragma unroll
            for (int i = 0; i < N; ++i) gains[p * N + i] = (w ? gains[p * N + i] : 0.f) + dg[j][i];
          }
        }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < a.dim; i += blockDim.x) to[i] = gains[i];
    return;
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int p = t + (j << lg);
    if (p < all) {
#pragma unroll
      for (int i = 0; i < N; i += 4) store_piece<4, false>(to + p * N + i, dg[j] + i, 4);
    }
  }
}

// d_gain = the sum of the workgroups' parts, 64 columns to a workgroup of 16 wavefronts.
__global__ __launch_bounds__(1024) void gain_sum_kernel(const float* partial, int parts, int dim, bool bf16, void* d_gain) {
  __shared__ float red[16][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, at = blockIdx.x * 64 + lane, apart = padded(dim);
  float s = 0.f;
  if (at < dim) {
#pragma unroll 8
    for (int i = wave; i < parts; i += 16) s += partial[(size_t)i * apart + at];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && at < dim) {
    for (int i = 1; i < 16; ++i) s += red[i][lane];
    if (bf16) store_from_f32((bf16_t*)d_gain, at, s);
    else ((float*)d_gain)[at] = s;
  }
}

// Threads to a row, as a power of two: a piece each up to a wavefront's 64, and where rows are few; up to `most` pieces each where they are many.  One and two, us:
// 16384 bf16 rows of 8192 179 and 186, but 4096 of 2048 12.4 and 10.8, and without a residual 16384 of 4096 53 and 46; 2048 rows of 8192 in 8 bits, by products alone, 27.5 and 24.1; 8192 fp32 rows of
// 4096 90 and 93, onto an fp32 stream 71 and 69.  The gradient: 16384 rows of 2048 62 and 54, four pieces in fp32 8191 rows of 4096 134 and 99.
int threads_of(int pieces, int most, int rows, int least) {
  const int share = rows >= MANY_ROWS ? most : 1;
  int lg = least;
  while (lg < 10 && (lg < 6 ? 1 << lg : share << lg) < pieces) ++lg;
  return lg;
}

template <typename X, typename H, typename Y, bool ADDED, bool ODD, int P>
hipError_t launch_forward(const NormRows& a, int lg, hipStream_t st) {
  const int threads = std::max(256, 1 << lg), per = threads >> lg;
  const int blocks = (a.rows + per - 1) / per, x = std::min(blocks, 1 << 20);      // a grid has less than 2^32 threads in one direction
  hipLaunchKernelGGL((add_norm_kernel<X, H, Y, ADDED, ODD, P>), dim3(x, (blocks + x - 1) / x), dim3(threads), 0, st, a, lg);
  return hipGetLastError();
}

template <typename X, typename H, typename Y, bool ADDED, bool ODD>
hipError_t forward(const NormRows& a, hipStream_t st) {
  constexpr int N = piece_size<X, H, Y>();
  const int pieces = pieces_of(a.dim, N), lg = threads_of(pieces, N == 8 && ADDED && sizeof(Y) > 1 && pieces >= 1024 ? 1 : 2, a.rows, sizeof(Y) > 1 ? 3 : N == 8 ? 4 : 5), P = (pieces + (1 << lg) - 1) >> lg;
  if (P <= 1) return launch_forward<X, H, Y, ADDED, ODD, 1>(a, lg, st);
  if constexpr (N == 4)
    if (P > 2) return launch_forward<X, H, Y, ADDED, ODD, 4>(a, lg, st);
  return launch_forward<X, H, Y, ADDED, ODD, 2>(a, lg, st);                        // 2048 pieces of 8 at most
}

template <typename X, typename H, typename Y>
hipError_t forward_rows(const NormRows& a, bool wide, hipStream_t st) {
  if (a.residual) return wide ? forward<X, H, Y, true, false>(a, st) : forward<X, H, Y, true, true>(a, st);
  if constexpr (sizeof(X) == sizeof(H)) return wide ? forward<X, H, Y, false, false>(a, st) : forward<X, H, Y, false, true>(a, st);
  return hipErrorInvalidValue;
}

template <typename X, typename H>
hipError_t forward_types(const NormRows& a, int out_type, bool wide, hipStream_t st) {
  if (out_type == NORM_BF16) return forward_rows<X, H, bf16_t>(a, wide, st);
  if (out_type == NORM_FP32) return forward_rows<X, H, float>(a, wide, st);
  return forward_rows<X, H, uint8_t>(a, wide, st);
}

int type_size(int t) { return t == NORM_FP32 ? 4 : t == NORM_BF16 ? 2 : 1; }

template <typename X, typename H, typename Y, bool ODD, int P>
hipError_t launch_backward(const NormGradRows& b, int lg, hipStream_t st) {
  // Rows that take longer by what each thread does want more threads at a time: us with 256 and 512, 65536 fp32 rows of 257 97 and 65, of 1000 on an fp32 stream 241 and 194, 16384 bf16 rows
  // of 4095 149 and 110; but whole bf16 rows, of 1000 104 and 112, 16384 of 4096 102 and 110.
  const int threads = std::max(piece_size<X, H, Y>() == 4 || ODD ? 512 : 256, 1 << lg), per = threads >> lg;
  // A workgroup to a CU where it has 1024 threads, else two; one also where a single round of them would leave as many parts as there are rows.  us in 512, 256, 128 parts: 512 bf16 rows
  // of 8192 20.0, 15.7, 17.9; 1024 rows 21.1, 22.1, 26.3; 8191 rows of 4096 on an fp32 stream 102, 121, 215; 2048 of 16384 138, 128
  const int blocks = (b.fwd.rows + per - 1) / per, grid = std::min(blocks, threads == 1024 || blocks <= NORM_GRAD_PARTS ? NORM_GRAD_PARTS / 2 : NORM_GRAD_PARTS);
  hipLaunchKernelGGL((add_norm_grad_kernel<X, H, Y, ODD, P>), dim3(grid), dim3(threads), per > 1 ? padded(b.fwd.dim) * sizeof(float) : 0, st, b, lg);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !b.partial) return e;
  hipLaunchKernelGGL(gain_sum_kernel, dim3((b.fwd.dim + 63) / 64), dim3(1024), 0, st, b.partial, grid, b.fwd.dim, b.fwd.gain_bf16, b.d_gain);
  return hipGetLastError();
}

template <typename X, typename H, typename Y, bool ODD>
hipError_t backward(const NormGradRows& b, hipStream_t st) {
  constexpr int N = piece_size<X, H, Y>();
  const int pieces = pieces_of(b.fwd.dim, N), lg = threads_of(pieces, 2, b.fwd.rows, 3), P = (pieces + (1 << lg) - 1) >> lg;
  if (P <= 1) return launch_backward<X, H, Y, ODD, 1>(b, lg, st);
  if constexpr (N == 4)
    if (P > 2) return launch_backward<X, H, Y, ODD, 4>(b, lg, st);
  return launch_backward<X, H, Y, ODD, 2>(b, lg, st);
}

template <typename X, typename H, typename Y>
hipError_t backward_as(const NormGradRows& b, bool wide, hipStream_t st) {
  return wide ? backward<X, H, Y, false>(b, st) : backward<X, H, Y, true>(b, st);
}

template <typename X, typename H>
hipError_t backward_types(const NormGradRows& b, int dy_type, bool wide, hipStream_t st) {
  return dy_type == NORM_BF16 ? backward_as<X, H, bf16_t>(b, wide, st) : backward_as<X, H, float>(b, wide, st);
}

}  // namespace

hipError_t launch_norm_rows(const NormRows& a, int x_type, int sum_type, int out_type, hipStream_t st) {
  const bool wide = a.dim % 8 == 0 && rows_at_16(a.x, a.x_stride, type_size(x_type)) && rows_at_16(a.gain, 0, 1) &&
                    (!a.residual || (rows_at_16(a.residual, a.residual_stride, type_size(sum_type)) && rows_at_16(a.sum_out, a.sum_stride, type_size(sum_type)))) &&
                    (out_type == NORM_CODES ? ((uintptr_t)a.out | (uintptr_t)a.out_stride) % 8 == 0 : rows_at_16(a.out, a.out_stride, type_size(out_type)));
  if (x_type == NORM_FP32) return forward_types<float, float>(a, out_type, wide, st);
  return sum_type == NORM_FP32 ? forward_types<bf16_t, float>(a, out_type, wide, st) : forward_types<bf16_t, bf16_t>(a, out_type, wide, st);
}

hipError_t launch_norm_rows_grad(const NormGradRows& b, int dy_type, int sum_type, int x_type, hipStream_t st) {
  const NormRows& a = b.fwd;
  const int sum_size = type_size(sum_type);
  const bool wide = a.dim % 8 == 0 && rows_at_16(a.gain, 0, 1) && rows_at_16(b.dy, b.dy_stride, type_size(dy_type)) && rows_at_16(b.h, b.h_stride, sum_size) &&
                    (!b.dh || rows_at_16(b.dh, b.dh_stride, sum_size)) && (!b.d_sum || rows_at_16(b.d_sum, b.d_sum_stride, sum_size)) &&
                    (!b.dx || rows_at_16(b.dx, b.dx_stride, type_size(x_type)));
  if (x_type == NORM_FP32) return backward_types<float, float>(b, dy_type, wide, st);
  return sum_type == NORM_FP32 ? backward_types<bf16_t, float>(b, dy_type, wide, st) : backward_types<bf16_t, bf16_t>(b, dy_type, wide, st);
}

size_t norm_grad_workspace(int rows, int dim) { return ((size_t)std::min(rows, NORM_GRAD_PARTS) * padded(dim) * sizeof(float) + 255) / 256 * 256; }
