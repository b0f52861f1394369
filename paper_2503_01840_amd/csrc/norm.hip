// The residual stream and its root-mean-square norm, the norm in 8 bits, and the gradient of both.
//
// A row h = x + residual is read once into registers, 64 W threads to a row, its squares summed by exchanges within the wavefronts and through LDS between
// them, and the row written as h and as gain * h * rsqrt(mean + eps).  Bound by bytes.
#include <algorithm>

#include "elements.hpp"
#include "kernels.hpp"

namespace {

constexpr float CODE_MOST = 448.f, LEAST_SCALE = 0x1p-100f;

// The sum over the 64 W threads of a row, the same on each; waves of a workgroup in order, `red` a wavefront's place each.
__device__ __forceinline__ float row_sum(float v, int W, float* red) {
  v = wave_sum_butterfly(v);
  if (W == 1) return v;
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  const float* mine = red + wave / W * W;
  v = mine[0];
  for (int i = 1; i < W; ++i) v += mine[i];
  return v;
}

__device__ __forceinline__ float load_gain(const NormRows& a, int i) {
  return a.gain_bf16 ? load_f32((const bf16_t*)a.gain, i) : load_f32((const float*)a.gain, i);
}
template <int N> __device__ __forceinline__ void load_gains(const NormRows& a, int at, float* g) {
  if constexpr (N == 1) {
    g[0] = load_gain(a, at);
  } else if (a.gain_bf16) {
    Elems<bf16_t, N> w;
    w.load((const bf16_t*)a.gain + at);
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = w.at(i);
  } else {
    Elems<float, N> w;
    w.load((const float*)a.gain + at);
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = w.at(i);
  }
}

__device__ __forceinline__ float finite_magnitude(float x) {
  const float a = fabsf(x);
  return a < __builtin_huge_valf() ? a : 0.f;
}
__device__ __forceinline__ float scale_of(float amax) { return fmaxf(amax / CODE_MOST, LEAST_SCALE); }

// Two values under a scale's reciprocal as codes; what is not finite as NaN.  The product instead of a quotient moves a value by 2^-24 of it, against a
// code's 2^-4.
__device__ __forceinline__ uint32_t to_codes(float a, float b, float inv) {
  const float ya = fminf(fmaxf(a * inv, -CODE_MOST), CODE_MOST), yb = fminf(fmaxf(b * inv, -CODE_MOST), CODE_MOST);
  uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(ya, yb, 0, false) & 0xFFFFu;
  if (!(fabsf(a) < __builtin_huge_valf())) c = (c & 0xFF00u) | 0x7Fu;
  if (!(fabsf(b) < __builtin_huge_valf())) c = (c & 0x00FFu) | 0x7F00u;
  return c;
}

// Y: type of the norm; uint8_t: codes, a.group columns to a scale (0: a row).  P pieces of N columns to a thread.
template <typename X, typename H, typename Y, bool ADDED, int N, int P>
__global__ __launch_bounds__(1024) void add_norm_kernel(NormRows a, int W) {
  constexpr bool CODES = sizeof(Y) == 1;
  __shared__ float red[16];
  __shared__ uint32_t most[CODES ? 16 * 16 + 128 : 1];       // largest magnitudes (bits) of a row's groups, or of its wavefronts
  const int wave = threadIdx.x >> 6, per = blockDim.x / (64 * W), group = wave / W;
  const int t = threadIdx.x - group * 64 * W, step = 64 * W;
  const long long row = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * per + group;
  const bool live = row < a.rows;
  const int pieces = a.dim / N;
  Elems<X, N> x[P];
  Elems<H, N> res[P];
  float h[P][N];
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int p = t + j * step;
    if (live && p < pieces) {
      x[j].load((const X*)a.x + row * a.x_stride + (long long)p * N);
      if constexpr (ADDED) res[j].load((const H*)a.residual + row * a.residual_stride + (long long)p * N);
    }
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int p = t + j * step;
    if (live && p < pieces) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        h[j][i] = x[j].at(i);
        if constexpr (ADDED) h[j][i] += res[j].at(i);
        sum = fmaf(h[j][i], h[j][i], sum);
      }
      if constexpr (ADDED) store_elems<N>((H*)a.sum_out + row * a.sum_stride + (long long)p * N, h[j]);
    }
  }
  const float r = 1.f / sqrtf(row_sum(sum, W, red) / (float)a.dim + a.eps);
  if constexpr (!CODES) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + j * step;
      if (live && p < pieces) {
        float g[N];
        load_gains<N>(a, p * N, g);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] *= h[j][i] * r;
        store_elems<N>((Y*)a.out + row * a.out_stride + (long long)p * N, g);
      }
    }
  } else {
    const int n_scales = a.group ? (a.dim + a.group - 1) / a.group : 1;
    uint32_t* mine = most + (N == 1 ? group * n_scales : 0);
    if constexpr (N == 1) {                                   // groups may lie across wavefronts
      for (int i = threadIdx.x; i < per * n_scales; i += blockDim.x) most[i] = 0;
      __syncthreads();
    }
    float amax = 0.f, part[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + j * step;
      part[j] = 0.f;
      if (live && p < pieces) {
        float g[N];
        load_gains<N>(a, p * N, g);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          h[j][i] = g[i] * (h[j][i] * r);
          part[j] = fmaxf(part[j], finite_magnitude(h[j][i]));
        }
      }
      if constexpr (N == 8) {
        if (a.group) part[j] = xlane_max_step<3>(xlane_max_step<2>(xlane_max_step<1>(xlane_max_step<0>(part[j]))));    // 16 lanes have a group
        else amax = fmaxf(amax, part[j]);
      } else {
        part[j] = wave_max(part[j]);                          // 64 columns: half a group
        const int p0 = p & ~63;
        if ((threadIdx.x & 63) == 0 && p0 < pieces) atomicMax(&mine[a.group ? p0 / 128 : 0], __float_as_uint(part[j]));
      }
    }
    if constexpr (N == 8) {
      if (!a.group) {
        amax = wave_max(amax);
        if (W > 1) {
          if ((threadIdx.x & 63) == 0) most[wave] = __float_as_uint(amax);
          __syncthreads();
          for (int i = 0; i < W; ++i) amax = fmaxf(amax, __uint_as_float(most[group * W + i]));
        }
      }
    } else {
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + j * step;
      if (!(live && p < pieces)) continue;
      const int s = a.group ? p * N / 128 : 0;
      const float scale = scale_of(N == 1 ? __uint_as_float(mine[s]) : a.group ? part[j] : amax), inv = 1.f / scale;
      if (a.group ? p * N % 128 == 0 : p == 0) a.scales[row * n_scales + s] = scale;
      uint8_t* to = (uint8_t*)a.out + row * a.out_stride + (long long)p * N;
      if constexpr (N == 8) {
        uint2 c;
        c.x = to_codes(h[j][0], h[j][1], inv) | to_codes(h[j][2], h[j][3], inv) << 16;
        c.y = to_codes(h[j][4], h[j][5], inv) | to_codes(h[j][6], h[j][7], inv) << 16;
        *(uint2*)to = c;
      } else {
        *to = (uint8_t)to_codes(h[j][0], 0.f, inv);
      }
    }
  }
}

// Gradient of the sum, rows dealt out in turn; the gains' gradient of a workgroup's rows to its part of the workspace.  dynamic LDS: a.dim floats where a workgroup has
// several rows at a time.
template <typename X, typename H, typename Y, int N, int P>
__global__ __launch_bounds__(1024) void add_norm_grad_kernel(NormGradRows b, int W) {
  extern __shared__ float gains[];
  __shared__ float red[2][2][16];
  const NormRows& a = b.fwd;
  const int wave = threadIdx.x >> 6, per = blockDim.x / (64 * W), group = wave / W;
  const int t = threadIdx.x - group * 64 * W, step = 64 * W;
  const int pieces = a.dim / N;
  float g[P][N], dg[P][N];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const int p = t + j * step;
#pragma unroll
    for (int i = 0; i < N; ++i) g[j][i] = dg[j][i] = 0.f;
    if (p < pieces) load_gains<N>(a, p * N, g[j]);
  }
  int turn = 0;
  for (long long r0 = (long long)blockIdx.x * per; r0 < a.rows; r0 += (long long)gridDim.x * per, turn ^= 1) {
    const long long row = r0 + group;
    const bool live = row < a.rows;
    Elems<Y, N> dy[P];
    Elems<H, N> h[P], dh[P];
    float hh = 0.f, gh = 0.f;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + j * step;
      if (live && p < pieces) {
        dy[j].load((const Y*)b.dy + row * b.dy_stride + (long long)p * N);
        h[j].load((const H*)b.h + row * b.h_stride + (long long)p * N);
        if (b.dh) dh[j].load((const H*)b.dh + row * b.dh_stride + (long long)p * N);
      }
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + j * step;
      if (live && p < pieces) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          hh = fmaf(h[j].at(i), h[j].at(i), hh);
          gh = fmaf(g[j][i] * dy[j].at(i), h[j].at(i), gh);
        }
      }
    }
    // two places in turn: one barrier a row
    hh = wave_sum_butterfly(hh);
    gh = wave_sum_butterfly(gh);
    if (W > 1) {
      if ((threadIdx.x & 63) == 0) {
        red[turn][0][wave] = hh;
        red[turn][1][wave] = gh;
      }
      __syncthreads();
      hh = red[turn][0][group * W];
      gh = red[turn][1][group * W];
      for (int i = 1; i < W; ++i) {
        hh += red[turn][0][group * W + i];
        gh += red[turn][1][group * W + i];
      }
    }
    const float r = 1.f / sqrtf(hh / (float)a.dim + a.eps), c = r * r * r * (gh / (float)a.dim);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const int p = t + j * step;
      if (live && p < pieces) {
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float d = dy[j].at(i), v = h[j].at(i);
          y[i] = fmaf(g[j][i] * d, r, -(v * c));
          if (b.dh) y[i] += dh[j].at(i);
          dg[j][i] = fmaf(d, v * r, dg[j][i]);
        }
        if (b.d_sum) store_elems<N>((H*)b.d_sum + row * b.d_sum_stride + (long long)p * N, y);
        if (b.dx) store_elems<N>((X*)b.dx + row * b.dx_stride + (long long)p * N, y);
      }
    }
  }
  if (!b.partial) return;
  float* to = b.partial + (size_t)blockIdx.x * a.dim;
  if (per > 1) {                                              // rows of a workgroup one after the other
    for (int w = 0; w < per; ++w) {
      if (w == group) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const int p = t + j * step;
          if (p < pieces) {
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
    const int p = t + j * step;
    if (p < pieces) {
#pragma unroll
      for (int i = 0; i < N; ++i) to[p * N + i] = dg[j][i];
    }
  }
}

// d_gain = the sum of the workgroups' parts, 64 columns to a workgroup of 16 wavefronts.
__global__ __launch_bounds__(1024) void gain_sum_kernel(const float* partial, int parts, int dim, bool bf16, void* d_gain) {
  __shared__ float red[16][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, at = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (at < dim) {
#pragma unroll 8
    for (int i = wave; i < parts; i += 16) s += partial[(size_t)i * dim + at];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && at < dim) {
    for (int i = 1; i < 16; ++i) s += red[i][lane];
    if (bf16) store_from_f32((bf16_t*)d_gain, at, s);
    else ((float*)d_gain)[at] = s;
  }
}

template <typename X, typename H, typename Y, bool ADDED, int N, int P>
hipError_t launch_forward(const NormRows& a, int W, hipStream_t st) {
  const int threads = std::max(256, 64 * W), per = threads / (64 * W);
  const int blocks = (a.rows + per - 1) / per, x = std::min(blocks, 1 << 20);      // a grid has less than 2^32 threads in one direction
  hipLaunchKernelGGL((add_norm_kernel<X, H, Y, ADDED, N, P>), dim3(x, (blocks + x - 1) / x), dim3(threads), 0, st, a, W);
  return hipGetLastError();
}

// Threads to a row: one piece each where rows are few, up to four where there are many.
int wavefronts_of(int pieces, int most, int rows) {
  const int share = rows >= 1024 ? std::min(4, most) : 1;
  int W = 1;
  while (W < 16 && 64 * W * share < pieces) W *= 2;
  return W;
}

template <typename X, typename H, typename Y, bool ADDED>
hipError_t forward(const NormRows& a, bool wide, hipStream_t st) {
  if (wide) {
    const int pieces = a.dim / 8, W = wavefronts_of(pieces, 4, a.rows), P = (pieces + 64 * W - 1) / (64 * W);
    if (P <= 1) return launch_forward<X, H, Y, ADDED, 8, 1>(a, W, st);
    if (P <= 2) return launch_forward<X, H, Y, ADDED, 8, 2>(a, W, st);
    return launch_forward<X, H, Y, ADDED, 8, 4>(a, W, st);
  }
  const int W = wavefronts_of(a.dim, 4, a.rows), P = (a.dim + 64 * W - 1) / (64 * W);
  if (P <= 4) return launch_forward<X, H, Y, ADDED, 1, 4>(a, W, st);
  return launch_forward<X, H, Y, ADDED, 1, 16>(a, W, st);
}

template <typename X, typename H>
hipError_t forward_types(const NormRows& a, int out_type, bool wide, hipStream_t st) {
  if (a.residual) {
    if (out_type == NORM_BF16) return forward<X, H, bf16_t, true>(a, wide, st);
    if (out_type == NORM_FP32) return forward<X, H, float, true>(a, wide, st);
    return forward<X, H, uint8_t, true>(a, wide, st);
  }
  if constexpr (sizeof(X) == sizeof(H)) {
    if (out_type == NORM_BF16) return forward<X, H, bf16_t, false>(a, wide, st);
    if (out_type == NORM_FP32) return forward<X, H, float, false>(a, wide, st);
    return forward<X, H, uint8_t, false>(a, wide, st);
  }
  return hipErrorInvalidValue;
}

int type_size(int t) { return t == NORM_FP32 ? 4 : t == NORM_BF16 ? 2 : 1; }

template <typename X, typename H, typename Y, int N, int P>
hipError_t launch_backward(const NormGradRows& b, int W, hipStream_t st) {
  const int threads = std::max(256, 64 * W), per = threads / (64 * W);
  const int grid = std::min((b.fwd.rows + per - 1) / per, NORM_GRAD_PARTS);
  hipLaunchKernelGGL((add_norm_grad_kernel<X, H, Y, N, P>), dim3(grid), dim3(threads), per > 1 ? b.fwd.dim * sizeof(float) : 0, st, b, W);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !b.partial) return e;
  hipLaunchKernelGGL(gain_sum_kernel, dim3((b.fwd.dim + 63) / 64), dim3(1024), 0, st, b.partial, grid, b.fwd.dim, b.fwd.gain_bf16, b.d_gain);
  return hipGetLastError();
}

template <typename X, typename H, typename Y>
hipError_t backward(const NormGradRows& b, bool wide, hipStream_t st) {
  const int rows = b.fwd.rows, dim = b.fwd.dim;
  if (wide) {
    const int pieces = dim / 8, W = wavefronts_of(pieces, 2, rows), P = (pieces + 64 * W - 1) / (64 * W);
    if (P <= 1) return launch_backward<X, H, Y, 8, 1>(b, W, st);
    return launch_backward<X, H, Y, 8, 2>(b, W, st);
  }
  const int W = wavefronts_of(dim, 4, rows), P = (dim + 64 * W - 1) / (64 * W);
  if (P <= 4) return launch_backward<X, H, Y, 1, 4>(b, W, st);
  return launch_backward<X, H, Y, 1, 16>(b, W, st);
}

template <typename X, typename H>
hipError_t backward_types(const NormGradRows& b, int dy_type, bool wide, hipStream_t st) {
  return dy_type == NORM_BF16 ? backward<X, H, bf16_t>(b, wide, st) : backward<X, H, float>(b, wide, st);
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

size_t norm_grad_workspace(int rows, int dim) { return ((size_t)std::min(rows, NORM_GRAD_PARTS) * dim * sizeof(float) + 255) / 256 * 256; }
