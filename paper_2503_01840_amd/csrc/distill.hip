// Cross entropy of a student's logits against the weights of a teacher's largest ones, and its gradient.
//
// loss = P log(sum_v e^((x_v - m) / T)) + sum_j p_j (m - x_j) / T with m the row's largest logit: differences from m, not from the log-sum, keep what a large m would round
// away.  A workgroup takes a row; where rows are few, parts of it, each with its own m and sum, joined by the next launch.  The gradient's
// entries of the teacher's tokens are written a second time, once the row is written: a token's weights are summed by its first entry, so no atomics.
// Bound by bytes: the logits read, the gradient written.
#include <algorithm>

#include "elements.hpp"
#include "kernels.hpp"

namespace {

constexpr int MOST_K = 1024;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
constexpr float NONE = -__builtin_huge_valf();

// A row's 16-byte pieces from the multiple of 16 at or below its start on; elements outside the row as -infinity.
template <typename T> struct RowPieces {
  static constexpr int N = 16 / sizeof(T);
  const T* row;
  int head, vocab, pieces;                    // elements that the first piece has in front of the row

  __device__ __forceinline__ RowPieces(const T* p, int v) : row(p), vocab(v) {
    head = (int)(((uintptr_t)p & 15) / sizeof(T));
    pieces = (head + v + N - 1) / N;
  }
  __device__ __forceinline__ bool whole(int p) const { return p * N >= head && p * N - head + N <= vocab; }
  __device__ __forceinline__ u32x4_t load(int p) const {
    const int e = p * N - head;
    if (whole(p)) return *(const u32x4_t*)(row + e);
    u32x4_t w;
    if constexpr (N == 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = e + 2 * i >= 0 && e + 2 * i < vocab ? row[e + 2 * i] : 0xFF80u;
        const uint32_t hi = e + 2 * i + 1 >= 0 && e + 2 * i + 1 < vocab ? row[e + 2 * i + 1] : 0xFF80u;
        w[i] = lo | hi << 16;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = e + i >= 0 && e + i < vocab ? __float_as_uint(row[e + i]) : 0xFF800000u;
    }
    return w;
  }
  static __device__ __forceinline__ u32x4_t none() {
    const uint32_t x = N == 8 ? 0xFF80FF80u : 0xFF800000u;
    return u32x4_t{x, x, x, x};
  }
  static __device__ __forceinline__ float at(const u32x4_t& w, int i) {
    if constexpr (N == 8) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    else return __uint_as_float(w[i]);
  }
  // to a row that starts at the same place within 16 bytes (`even`), or anywhere
  __device__ __forceinline__ void store(T* out, int p, const float* f, bool even) const {
    const int e = p * N - head;
    if (even && whole(p)) {
      if constexpr (N == 8) *(u32x4_t*)(out + e) = u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
      else *(floatx4*)(out + e) = floatx4{f[0], f[1], f[2], f[3]};
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e + i >= 0 && e + i < vocab) store_from_f32(out, e + i, f[i]);
  }
};

// A largest logit and the sum of exp2(c (x - it)).
struct Stat {
  float m, s;
};
__device__ __forceinline__ float finite_or_zero(float m) { return m == NONE ? 0.f : m; }
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float c) {
  const float m = fmaxf(a.m, b.m), at = finite_or_zero(m);
  return {m, a.s * exp2_fast((a.m - at) * c) + b.s * exp2_fast((b.m - at) * c)};
}
template <typename T, int U> __device__ __forceinline__ void add_pieces(Stat& st, const u32x4_t* w, float c) {
  typedef RowPieces<T> R;
  float m = st.m;
#pragma unroll
  for (int j = 0; j < U; ++j) {
#pragma unroll
    for (int i = 0; i < R::N; ++i) m = fmaxf(m, R::at(w[j], i));
  }
  const float at = finite_or_zero(m);
  float s = st.s * exp2_fast((st.m - at) * c), more = 0.f;
#pragma unroll
  for (int j = 0; j < U; ++j) {
#pragma unroll
    for (int i = 0; i < R::N; i += 2) {
      s += exp2_fast((R::at(w[j], i) - at) * c);
      more += exp2_fast((R::at(w[j], i + 1) - at) * c);
    }
  }
  st = {m, s + more};
}
template <int STEP> __device__ __forceinline__ Stat join_step(const Stat& a, float c) {
  uint32_t m0, m1, s0, s1;
  xlane_partners<STEP>(__float_as_uint(a.m), m0, m1);
  xlane_partners<STEP>(__float_as_uint(a.s), s0, s1);
  return join({__uint_as_float(m0), __uint_as_float(s0)}, {__uint_as_float(m1), __uint_as_float(s1)}, c);
}
// The workgroup's, the same on every thread.  red: 2 * 16 floats
template <int THREADS> __device__ __forceinline__ Stat join_workgroup(Stat a, float c, float (*red)[16]) {
  a = join_step<5>(join_step<4>(join_step<3>(join_step<2>(join_step<1>(join_step<0>(a, c), c), c), c), c), c);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[0][wave] = a.m;
    red[1][wave] = a.s;
  }
  __syncthreads();
  a = {red[0][0], red[1][0]};
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) a = join(a, {red[0][i], red[1][i]}, c);
  return a;
}

// Of pieces first..last-1 of a row, by all threads of the workgroup.
template <typename T, int THREADS> __device__ __forceinline__ Stat pieces_stat(const RowPieces<T>& r, int first, int last, float c, float (*red)[16]) {
  constexpr int U = 4;
  Stat st = {NONE, 0.f};
  for (int p0 = first + threadIdx.x; p0 < last; p0 += U * THREADS) {
    u32x4_t w[U];
#pragma unroll
    for (int j = 0; j < U; ++j) w[j] = p0 + j * THREADS < last ? r.load(p0 + j * THREADS) : r.none();
    add_pieces<T, U>(st, w, c);
  }
  return join_workgroup<THREADS>(st, c, red);
}

// ---------------------------------------------------------------- the teacher's weights of a row
struct Teacher {
  int32_t id[MOST_K];       // of the student, -1: none
  float p[MOST_K];
  float x[MOST_K];          // the student's logit of it
};
// Weights and logits of the tokens among elements lo..hi-1 of the row (of the others: weights); returns P.
template <typename T, int THREADS>
__device__ __forceinline__ float weights(const DistillRows& a, long long r, const T* row, int lo, int hi, Teacher& t, float* red) {
  float most = NONE;
  for (int j = threadIdx.x; j < a.k; j += THREADS) {
    int id = a.ids[r * a.k + j];
    if (a.t2d) id = id >= 0 && id < a.n_t2d ? a.t2d[id] : -1;
    if (id < 0 || id >= a.vocab) id = -1;
    const float z = id < 0 ? NONE : a.values[r * a.k + j];
    t.id[j] = id;
    t.p[j] = z;
    t.x[j] = id >= lo && id < hi ? load_f32(row, id) : 0.f;
    most = fmaxf(most, z);
  }
  if (!a.lse) most = block_max(most, red);
  const float lse = a.lse ? a.lse[r] : 0.f;
  float sum = 0.f;
  for (int j = threadIdx.x; j < a.k; j += THREADS) {
    const float z = t.p[j];
    const float p = z == NONE ? 0.f : a.lse ? expf(z / a.temperature - lse) : expf((z - most) / a.temperature);
    t.p[j] = p;
    sum += p;
  }
  sum = block_sum(sum, red);                                  // a barrier too: the arrays are whole behind it
  if (a.lse || sum == 0.f) return sum;
  for (int j = threadIdx.x; j < a.k; j += THREADS) t.p[j] /= sum;
  return sum / sum;
}

template <int THREADS> __device__ __forceinline__ float loss_of(const DistillRows& a, const Teacher& t, float P, const Stat& st, float* red) {
  float v = 0.f;
  for (int j = threadIdx.x; j < a.k; j += THREADS) {
    const float p = t.p[j];
    if (p != 0.f) v = fmaf(p, (st.m - t.x[j]) / a.temperature, v);
  }
  v = block_sum(v, red);
  return P == 0.f ? 0.f : fmaf(P, logf(st.s), v);
}

// ---------------------------------------------------------------- kernels
// Largest logit and sum of a part of a row: grid (rows, 1 / more, parts).
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_part_kernel(DistillRows a, float c, int share, float* partial) {
  __shared__ float red[2][16];
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  const int first = blockIdx.z * share;
  const Stat st = pieces_stat<T, THREADS>(row, min(first, row.pieces), min(first + share, row.pieces), c, red);
  if (threadIdx.x == 0) *(float2*)(partial + ((size_t)r * gridDim.z + blockIdx.z) * 2) = make_float2(st.m, st.s);
}

// Loss and stats of a row, from the row itself or (parts > 0) from those of its parts.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_loss_kernel(DistillRows a, float c, const float* partial, int parts) {
  __shared__ Teacher t;
  __shared__ float red[2][16], red1[17];
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  const float P = weights<T, THREADS>(a, r, row.row, 0, a.vocab, t, red1);
  Stat st;
  if (parts) {
    st = {NONE, 0.f};
    for (int i = threadIdx.x; i < parts; i += THREADS) {
      const float2 v = *(const float2*)(partial + ((size_t)r * parts + i) * 2);
      st = join(st, {v.x, v.y}, c);
    }
    st = join_workgroup<THREADS>(st, c, red);
  } else {
    st = pieces_stat<T, THREADS>(row, 0, row.pieces, c, red);
  }
  const float loss = loss_of<THREADS>(a, t, P, st, red1);
  if (threadIdx.x == 0) {
    a.loss[r] = loss;
    if (a.stats) *(float2*)(a.stats + 2 * r) = make_float2(st.m, st.s);
  }
}

// The gradient's entries of the teacher's tokens among elements lo..hi-1: g (P q - p) with q = softmax of the student's logit, k = g P / sum.
template <typename T, int THREADS>
__device__ __forceinline__ void write_tokens(const DistillRows& a, const Teacher& t, T* out, int lo, int hi, const Stat& st, float c, float k, float g) {
  __syncthreads();                                            // the row is written
  for (int j = threadIdx.x; j < a.k; j += THREADS) {
    const int id = t.id[j];
    if (id < lo || id >= hi) continue;
    float p = 0.f;
    bool first = true;
    for (int i = 0; i < a.k; ++i) {
      if (t.id[i] != id) continue;
      p += t.p[i];
      first = first && i >= j;
    }
    if (first) store_from_f32(out, id, fmaf(k, exp2_fast((t.x[j] - st.m) * c), -(g * p)));
  }
}

template <typename T, int THREADS, int U>
__device__ __forceinline__ void write_pieces(const RowPieces<T>& r, T* out, bool even, int first, int last, const Stat& st, float c, float k) {
  for (int p0 = first + threadIdx.x; p0 < last; p0 += U * THREADS) {
    u32x4_t w[U];
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (p0 + j * THREADS < last) w[j] = r.load(p0 + j * THREADS);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (p0 + j * THREADS >= last) break;
      float f[RowPieces<T>::N];
#pragma unroll
      for (int i = 0; i < RowPieces<T>::N; ++i) f[i] = k * exp2_fast((r.at(w[j], i) - st.m) * c);
      r.store(out, p0 + j * THREADS, f, even);
    }
  }
}
template <typename T, int THREADS>
__device__ __forceinline__ void write_zeros(const RowPieces<T>& r, T* out, bool even, int first, int last) {
  const float zero[RowPieces<T>::N] = {};
  for (int p = first + threadIdx.x; p < last; p += THREADS) r.store(out, p, zero, even);
}

// grid (rows, 1 / more, parts): the gradient of a part of a row
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(DistillRows a, float c, int share) {
  __shared__ Teacher t;
  __shared__ float red1[17];
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  T* out = (T*)a.d_logits + r * a.d_stride;
  const bool even = (((uintptr_t)out ^ (uintptr_t)row.row) & 15) == 0;
  const int first = min((int)blockIdx.z * share, row.pieces), last = min(first + share, row.pieces);
  const int lo = max(0, first * row.N - row.head), hi = min(a.vocab, last * row.N - row.head);
  const float dloss = a.dloss[r];
  float P = 0.f;
  if (dloss != 0.f) P = weights<T, THREADS>(a, r, row.row, lo, hi, t, red1);
  if (P == 0.f) {
    write_zeros<T, THREADS>(row, out, even, first, last);
    return;
  }
  const Stat st = {a.stats[2 * r], a.stats[2 * r + 1]};
  const float g = dloss / a.temperature, k = g * P / st.s;
  write_pieces<T, THREADS, 4>(row, out, even, first, last, st, c, k);
  write_tokens<T, THREADS>(a, t, out, lo, hi, st, c, k, g);
}

// Loss and gradient of a row.  R > 0: its pieces stay in R registers of 16 bytes a thread between the two.
template <typename T, int THREADS, int R>
__global__ __launch_bounds__(THREADS) void distill_step_kernel(DistillRows a, float c) {
  __shared__ Teacher t;
  __shared__ float red[2][16], red1[17];
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  T* out = (T*)a.d_logits + r * a.d_stride;
  const bool even = (((uintptr_t)out ^ (uintptr_t)row.row) & 15) == 0;
  const float dloss = a.dloss[r];
  const float P = weights<T, THREADS>(a, r, row.row, 0, a.vocab, t, red1);
  if (P == 0.f) {
    write_zeros<T, THREADS>(row, out, even, 0, row.pieces);
    if (threadIdx.x == 0) a.loss[r] = 0.f;
    return;
  }
  u32x4_t w[R ? R : 1];
  Stat st;
  if constexpr (R > 0) {
#pragma unroll
    for (int j = 0; j < R; ++j) w[j] = (int)threadIdx.x + j * THREADS < row.pieces ? row.load(threadIdx.x + j * THREADS) : row.none();
    st = {NONE, 0.f};
    constexpr int U = R < 4 ? R : 4;
#pragma unroll
    for (int j = 0; j < R; j += U) add_pieces<T, U>(st, w + j, c);
    st = join_workgroup<THREADS>(st, c, red);
  } else {
    st = pieces_stat<T, THREADS>(row, 0, row.pieces, c, red);
  }
  const float loss = loss_of<THREADS>(a, t, P, st, red1);
  if (threadIdx.x == 0) a.loss[r] = loss;
  if (dloss == 0.f) {
    write_zeros<T, THREADS>(row, out, even, 0, row.pieces);
    return;
  }
  const float g = dloss / a.temperature, k = g * P / st.s;
  if constexpr (R > 0) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int p = threadIdx.x + j * THREADS;
      if (p >= row.pieces) break;
      float f[RowPieces<T>::N];
#pragma unroll
      for (int i = 0; i < RowPieces<T>::N; ++i) f[i] = k * exp2_fast((row.at(w[j], i) - st.m) * c);
      row.store(out, p, f, even);
    }
  } else {
    write_pieces<T, THREADS, 4>(row, out, even, 0, row.pieces, st, c, k);
  }
  write_tokens<T, THREADS>(a, t, out, 0, a.vocab, st, c, k, g);
}

// ---------------------------------------------------------------- launches
float factor_of(const DistillRows& a) { return (float)(1.4426950408889634074 / (double)a.temperature); }
int most_pieces(const DistillRows& a, int size) { return (int)(((long long)a.vocab * size + 15) / 16 + 1); }       // of a row wherever it starts

// Parts of a row, so that few rows fill the chip: of at least 1024 pieces
int parts_of(int rows, int pieces) { return std::max(1, std::min((pieces + 1023) / 1024, 1024 / std::min(rows, 1024))); }
dim3 grid_of(int rows, int parts) {
  const int x = std::min(rows, 1 << 20);                      // a grid has less than 2^32 threads in one direction
  return dim3(x, (rows + x - 1) / x, parts);
}

template <typename T> hipError_t loss_rows(const DistillRows& a, void* ws, hipStream_t st) {
  const int pieces = most_pieces(a, sizeof(T)), parts = parts_of(a.rows, pieces);
  const float c = factor_of(a);
  if (parts > 1) {
    const int share = (pieces + parts - 1) / parts;
    hipLaunchKernelGGL((distill_part_kernel<T, 256>), grid_of(a.rows, parts), dim3(256), 0, st, a, c, share, (float*)ws);
    hipLaunchKernelGGL((distill_loss_kernel<T, 256>), grid_of(a.rows, 1), dim3(256), 0, st, a, c, (const float*)ws, parts);
  } else {
    hipLaunchKernelGGL((distill_loss_kernel<T, 256>), grid_of(a.rows, 1), dim3(256), 0, st, a, c, (const float*)nullptr, 0);
  }
  return hipGetLastError();
}

template <typename T> hipError_t grad_rows(const DistillRows& a, hipStream_t st) {
  const int pieces = most_pieces(a, sizeof(T)), parts = parts_of(a.rows, pieces), share = (pieces + parts - 1) / parts;
  hipLaunchKernelGGL((distill_grad_kernel<T, 256>), grid_of(a.rows, parts), dim3(256), 0, st, a, factor_of(a), share);
  return hipGetLastError();
}

template <typename T> hipError_t step_rows(const DistillRows& a, void* ws, hipStream_t st) {
  const int pieces = most_pieces(a, sizeof(T));
  if (parts_of(a.rows, pieces) > 1) {                         // the stats behind the parts'
    DistillRows b = a;
    b.stats = (float*)ws + 2 * (size_t)a.rows * parts_of(a.rows, pieces);
    const hipError_t e = loss_rows<T>(b, ws, st);
    return e != hipSuccess ? e : grad_rows<T>(b, st);
  }
  const float c = factor_of(a);
  hipLaunchKernelGGL((distill_step_kernel<T, 1024, 0>), grid_of(a.rows, 1), dim3(1024), 0, st, a, c);
  return hipGetLastError();
}

}  // namespace

size_t distill_workspace(int rows, int vocab) {
  DistillRows a = {};
  a.vocab = vocab;
  const int parts = parts_of(rows, most_pieces(a, 4));        // no fewer than of bf16 rows
  return parts > 1 ? ((size_t)rows * (parts + 1) * 2 * sizeof(float) + 255) / 256 * 256 : 0;
}
hipError_t launch_distill(const DistillRows& a, bool bf16, void* ws, hipStream_t st) { return bf16 ? loss_rows<bf16_t>(a, ws, st) : loss_rows<float>(a, ws, st); }
hipError_t launch_distill_grad(const DistillRows& a, bool bf16, hipStream_t st) { return bf16 ? grad_rows<bf16_t>(a, st) : grad_rows<float>(a, st); }
hipError_t launch_distill_step(const DistillRows& a, bool bf16, void* ws, hipStream_t st) { return bf16 ? step_rows<bf16_t>(a, ws, st) : step_rows<float>(a, ws, st); }
