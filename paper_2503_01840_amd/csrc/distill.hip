// Cross entropy of a student's logits against the weights of a teacher's largest ones, and its gradient.
//
// loss = P log(sum_v e^((x_v - m) / T)) + sum_j p_j (m - x_j) / T with m the row's largest logit: differences from m, not from the log-sum, keep what a large m would round
// away.  A workgroup takes a row; where rows are few, parts of it, each with its own m and sum, joined by the next launch.  Loss and gradient in one call read the
// logits once: a row of up to 16384 pieces of 16 bytes stays in the registers of its workgroup between the two (read twice, the second time out of the caches: 2048 rows of
// 32000 in fp32 163 us instead of 107, 2047 of 128256 in bf16 312 instead of 223).  The teacher's weights are one wavefront's work while the row is on its way;
// the gradient's entries of its tokens are written a second time, once the row is written.  A token's weights go to its first entry, found by a hash (by comparing
// all entries 345 us instead of 233, with 128 of them), in the order of entries: results do not change from call to call.
// Bound by bytes, the logits read, the gradient written, at 4.3 to 5.2 TB/s where rows are many; in bf16 the exponentials take half of that time under the loads.
#include <algorithm>

#include "elements.hpp"
#include "kernels.hpp"

namespace {

constexpr float NONE = -__builtin_huge_valf();
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row as 16-byte pieces from its first multiple of 16 bytes on, and the few elements in front of them and behind, one to each of a workgroup's first threads.
template <typename T> struct RowPieces {
  static constexpr int N = 16 / sizeof(T);
  const T* row;
  int head, vocab, pieces;                    // head: elements in front of the pieces

  __device__ __forceinline__ RowPieces(const T* p, int v) : row(p), vocab(v) {
    head = min((int)((-(uintptr_t)p & 15) / sizeof(T)), v);
    pieces = (v - head) / N;
  }
  // piece at + lane's: with `at` the same for a wavefront its address takes no vector registers
  __device__ __forceinline__ u32x4_t load(int at, uint32_t lane = 0) const { return *(const u32x4_t*)((const char*)(row + head) + (size_t)(uint32_t)at * 16 + lane * 16u); }
  static __device__ __forceinline__ u32x4_t none() {
    const uint32_t x = N == 8 ? 0xFF80FF80u : 0xFF800000u;
    return u32x4_t{x, x, x, x};
  }
  static __device__ __forceinline__ float at(const u32x4_t& w, int i) {
    if constexpr (N == 8) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    else return __uint_as_float(w[i]);
  }
  // this thread's element outside the pieces, -1: none
  __device__ __forceinline__ int single() const {
    const int i = threadIdx.x, e = i < head ? i : i + pieces * N;
    return e < vocab && i < 2 * N ? e : -1;
  }
  // EVEN: every row of the result starts at the same place within 16 bytes as its logits
  template <bool EVEN> __device__ __forceinline__ void store(T* out, int at, uint32_t lane, const float* f) const {
    if constexpr (EVEN) {
      void* to = (char*)(out + head) + (size_t)(uint32_t)at * 16 + lane * 16u;
      if constexpr (N == 8) *(u32x4_t*)to = u32x4_t{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
      else *(floatx4*)to = floatx4{f[0], f[1], f[2], f[3]};
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) store_from_f32(out, head + (at + (int)lane) * N + i, f[i]);
    }
  }
  // k exp2(c (x - m)) of a piece
  template <bool EVEN> __device__ __forceinline__ void store_gradient(T* out, int at, uint32_t lane, const u32x4_t& w, float m, float c, float k) const {
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = k * exp2_fast((RowPieces::at(w, i) - m) * c);
    store<EVEN>(out, at, lane, f);
  }
  template <bool EVEN> __device__ __forceinline__ void store_zeros(T* out, int p) const {
    const float zero[N] = {};
    store<EVEN>(out, p, 0, zero);
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
template <typename T> __device__ __forceinline__ void add_single(Stat& st, const RowPieces<T>& r, float c) {
  const int e = r.single();
  if (e >= 0) st = join(st, {load_f32(r.row, e), 1.f}, c);
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

// Of pieces first..last-1 of a row, this thread's share.  KEEP: they are left in `keep`, which has a place for piece `first` and each behind it.
template <typename T, int THREADS, bool KEEP = false>
__device__ __forceinline__ Stat pieces_stat(const RowPieces<T>& r, int first, int last, float c, Stat st = {NONE, 0.f}, u32x4_t* keep = nullptr) {
  constexpr int U = 8;
  for (int p0 = first + threadIdx.x; p0 < last; p0 += U * THREADS) {
    u32x4_t w[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      w[j] = p0 + j * THREADS < last ? r.load(p0 + j * THREADS) : r.none();
      if (KEEP && p0 + j * THREADS < last) keep[p0 - first + j * THREADS] = w[j];
    }
    constexpr int A = 16 / RowPieces<T>::N;                   // 16 values at a time
#pragma unroll
    for (int j = 0; j < U; j += A) add_pieces<T, A>(st, w + j, c);
  }
  return st;
}

// ---------------------------------------------------------------- the teacher's weights of a row
// In LDS, k of each and a table: the power of two from 4 k on, at least 64 and at most 2048 places; the first wavefront of a workgroup writes and reads them, while the others' logits are on
// their way.
struct Teacher {
  int32_t* id;              // of the student; -1: none, or a token that occurred before
  float* p;
  float* x;                 // the student's logit of it
  float* all;               // the weights of all entries of its token
  int32_t* first;           // by a hash of tokens: the tokens, then each one's first entry
  __device__ __forceinline__ Teacher(void* lds, int k) : id((int32_t*)lds), p((float*)lds + k), x((float*)lds + 2 * k), all((float*)lds + 3 * k), first((int32_t*)lds + 4 * k) {}
};
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ bool mine(int id, int lo, int hi, int front, int back) { return (id >= lo && id < hi) || (id >= 0 && id < front) || id >= back; }
// Weights, and logits of the tokens among elements lo..hi-1, below `front` and from `back` on; returns P.
template <typename T>
__device__ __forceinline__ float weights(const DistillRows& a, long long r, const T* row, int lo, int hi, int front, int back, const Teacher& t) {
  constexpr int U = 4;                                        // entries a lane asks for at a time
  const int lane = threadIdx.x & 63;
  const int32_t* ids = a.ids + r * a.k;
  const float* values = a.values + r * a.k;
  float most = NONE;
#pragma unroll 1
  for (int j0 = lane; j0 < a.k; j0 += 64 * U) {
    int id[U];
    float z[U], x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool entry = j0 + 64 * u < a.k;
      id[u] = entry ? ids[j0 + 64 * u] : -1;
      z[u] = entry ? values[j0 + 64 * u] : NONE;
    }
    if (a.t2d) {
#pragma unroll
      for (int u = 0; u < U; ++u) id[u] = id[u] >= 0 && id[u] < a.n_t2d ? a.t2d[id[u]] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (id[u] < 0 || id[u] >= a.vocab) id[u] = -1, z[u] = NONE;
      x[u] = mine(id[u], lo, hi, front, back) ? load_f32(row, id[u]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      most = fmaxf(most, z[u]);
      const int j = j0 + 64 * u;
      if (j < a.k) t.id[j] = id[u], t.p[j] = z[u], t.x[j] = x[u];
    }
  }
  most = wave_max(most);
  const float lse = a.lse ? a.lse[r] : 0.f;
  float sum = 0.f;
#pragma unroll 1
  for (int j = lane; j < a.k; j += 64) {
    const float z = t.p[j];
    const float p = z == NONE ? 0.f : a.lse ? expf(z / a.temperature - lse) : expf((z - most) / a.temperature);
    t.p[j] = p;
    sum += p;
  }
  sum = wave_sum_butterfly(sum);
  if (a.lse || sum == 0.f) return sum;
#pragma unroll 1
  for (int j = lane; j < a.k; j += 64) t.p[j] /= sum;
  return sum / sum;
}
// For the gradient: a token's weights to its first entry, added in the order of entries.  A chain of LDS round trips, and where rows are few what the call waits for (16 rows of 128256, 512
// entries: 15 us; with 2 k places that hold entries, whose tokens are compared, 21).
__device__ __forceinline__ void gather_tokens(const DistillRows& a, const Teacher& t) {
  const int lane = threadIdx.x & 63, mask = a.table - 1;
#pragma unroll 1
  for (int i = lane * 4; i < a.table; i += 256) *(int4*)(t.first + i) = make_int4(-1, -1, -1, -1);
  wave_fence();
  // a place for each token: the first from its hash on that is free or the token's already; t.all: the entry's place
#pragma unroll 1
  for (int j = lane; j < a.k; j += 64) {
    const int id = t.id[j];
    uint32_t at = (uint32_t)id * 0x9E3779B1u >> 7 & mask;     // Fibonacci hashing
    while (id >= 0) {
      const int other = atomicCAS(&t.first[at], -1, id);
      if (other < 0 || other == id) break;
      at = (at + 1) & mask;
    }
    t.all[j] = __int_as_float((int)at);
  }
  wave_fence();
  // the token's first entry in its place
#pragma unroll 1
  for (int j = lane; j < a.k; j += 64) t.first[__float_as_int(t.all[j])] = 0x7FFFFFFF;
  wave_fence();
#pragma unroll 1
  for (int j = lane; j < a.k; j += 64)
    if (t.id[j] >= 0) atomicMin(&t.first[__float_as_int(t.all[j])], j);
  wave_fence();
#pragma unroll 1
  for (int j0 = 0; j0 < a.k; j0 += 64) {
    const int j = j0 + lane;
    const bool token = j < a.k && t.id[j] >= 0;
    const int first = token ? t.first[__float_as_int(t.all[j])] : j;
    wave_fence();
    if (j < a.k) t.all[j] = t.p[j];
    uint64_t again = __ballot(first != j);
    if (first != j) t.id[j] = -1;
    wave_fence();
    while (again) {
      const int l = __builtin_ctzll(again), to = __builtin_amdgcn_readlane(first, l);
      again &= again - 1;
      if (lane == 0) t.all[to] += t.p[j0 + l];
      wave_fence();
    }
  }
}
__device__ __forceinline__ void write_loss(const DistillRows& a, long long r, const Teacher& t, float P, const Stat& st) {
  float v = 0.f;
#pragma unroll 1
  for (int j = threadIdx.x & 63; j < a.k; j += 64) {
    const float p = t.p[j];
    if (p != 0.f) v = fmaf(p, (st.m - t.x[j]) / a.temperature, v);
  }
  v = wave_sum_butterfly(v);
  if ((threadIdx.x & 63) == 0) a.loss[r] = P == 0.f ? 0.f : fmaf(P, logf(st.s), v);
}
// The gradient's entries of these tokens: g (P q - p) with q = softmax of the student's logit, k = g P / sum.
template <typename T>
__device__ __forceinline__ void write_tokens(const DistillRows& a, const Teacher& t, T* out, int lo, int hi, int front, int back, const Stat& st, float c, float k, float g) {
#pragma unroll 1
  for (int j = threadIdx.x & 63; j < a.k; j += 64) {
    const int id = t.id[j];
    if (mine(id, lo, hi, front, back)) store_from_f32(out, id, fmaf(k, exp2_fast((t.x[j] - st.m) * c), -(g * t.all[j])));
  }
}

// ---------------------------------------------------------------- kernels
// Largest logit and sum of a part of a row: grid (rows, 1 / more, parts); the single elements belong to part 0.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_part_kernel(DistillRows a, float c, int share, float* partial) {
  __shared__ float red[2][16];
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  const int first = blockIdx.z * share;
  Stat st = pieces_stat<T, THREADS>(row, min(first, row.pieces), min(first + share, row.pieces), c);
  if (blockIdx.z == 0) add_single(st, row, c);
  st = join_workgroup<THREADS>(st, c, red);
  if (threadIdx.x == 0) *(float2*)(partial + ((size_t)r * gridDim.z + blockIdx.z) * 2) = make_float2(st.m, st.s);
}

// Loss and stats of a row, from the row itself or (parts > 0) from those of its parts.  dynamic LDS here and below: the teacher's, at a multiple of 16 bytes, by which it is cleared
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_loss_kernel(DistillRows a, float c, const float* partial, int parts) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ float red[2][16];
  const Teacher t(lds, a.k);
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  float P = 0.f;
  if (threadIdx.x < 64) P = weights<T>(a, r, row.row, 0, a.vocab, a.vocab, a.vocab, t);
  Stat st = {NONE, 0.f};
  if (parts) {
    for (int i = threadIdx.x; i < parts; i += THREADS) {
      const float2 v = *(const float2*)(partial + ((size_t)r * parts + i) * 2);
      st = join(st, {v.x, v.y}, c);
    }
  } else {
    st = pieces_stat<T, THREADS>(row, 0, row.pieces, c);
    add_single(st, row, c);
  }
  st = join_workgroup<THREADS>(st, c, red);
  if (threadIdx.x >= 64) return;
  write_loss(a, r, t, P, st);
  if (threadIdx.x == 0 && a.stats) *(float2*)(a.stats + 2 * r) = make_float2(st.m, st.s);
}

template <typename T, int THREADS, bool EVEN>
__device__ __forceinline__ void write_pieces(const RowPieces<T>& r, T* out, int first, int last, const Stat& st, float c, float k) {
  constexpr int U = 8;
  for (int p0 = first + threadIdx.x; p0 < last; p0 += U * THREADS) {
    u32x4_t w[U];
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (p0 + j * THREADS < last) w[j] = r.load(p0 + j * THREADS);
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (p0 + j * THREADS < last) r.template store_gradient<EVEN>(out, p0 + j * THREADS, 0, w[j], st.m, c, k);
  }
}
template <typename T, int THREADS, bool EVEN>
__device__ __forceinline__ void write_zeros(const RowPieces<T>& r, T* out, int first, int last) {
  for (int p = first + threadIdx.x; p < last; p += THREADS) r.template store_zeros<EVEN>(out, p);
}
// any: k exp2(c (x - m)), else 0
template <typename T> __device__ __forceinline__ void write_single(const RowPieces<T>& r, T* out, bool any, const Stat& st, float c, float k) {
  const int e = r.single();
  if (e >= 0) store_from_f32(out, e, any ? k * exp2_fast((load_f32(r.row, e) - st.m) * c) : 0.f);
}

// grid (rows, 1 / more, parts): the gradient of a part of a row, the single elements with part 0.  The first R THREADS pieces are on their way while the
// teacher's weights are formed.
template <typename T, int THREADS, int R, bool EVEN>
__global__ __launch_bounds__(THREADS) void distill_grad_kernel(DistillRows a, float c, int share) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ float sum_of_weights;
  const Teacher t(lds, a.k);
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  T* out = (T*)a.d_logits + r * a.d_stride;
  const int first = min((int)blockIdx.z * share, row.pieces), last = min(first + share, row.pieces);
  // elements of this workgroup: those of its pieces and, for part 0, those in front and behind
  const int lo = row.head + first * row.N, hi = row.head + last * row.N, front = blockIdx.z == 0 ? row.head : 0, back = blockIdx.z == 0 ? row.head + row.pieces * row.N : a.vocab;
  const float dloss = a.dloss[r];
  if (dloss == 0.f) {
    write_zeros<T, THREADS, EVEN>(row, out, first, last);
    if (blockIdx.z == 0) write_single(row, out, false, {}, c, 0.f);
    return;
  }
  u32x4_t w[R];
#pragma unroll
  for (int j = 0; j < R; ++j)
    if ((int)threadIdx.x < last - first - j * THREADS) w[j] = row.load(first + j * THREADS, threadIdx.x);
  if (threadIdx.x < 64) {
    const float P = weights<T>(a, r, row.row, lo, hi, front, back, t);
    gather_tokens(a, t);
    if (threadIdx.x == 0) sum_of_weights = P;
  }
  __syncthreads();
  const float P = sum_of_weights;
  if (P == 0.f) {
    write_zeros<T, THREADS, EVEN>(row, out, first, last);
    if (blockIdx.z == 0) write_single(row, out, false, {}, c, 0.f);
    return;
  }
  const Stat st = {a.stats[2 * r], a.stats[2 * r + 1]};
  const float g = dloss / a.temperature, k = g * P / st.s;
#pragma unroll
  for (int j = 0; j < R; ++j)
    if ((int)threadIdx.x < last - first - j * THREADS) row.template store_gradient<EVEN>(out, first + j * THREADS, threadIdx.x, w[j], st.m, c, k);
  write_pieces<T, THREADS, EVEN>(row, out, first + R * THREADS, last, st, c, k);
  if (blockIdx.z == 0) write_single(row, out, true, st, c, k);
  __syncthreads();                                            // the tokens' entries behind everybody's
  if (threadIdx.x < 64) write_tokens<T>(a, t, out, lo, hi, front, back, st, c, k, g);
}

// Loss and gradient of a row: its first R THREADS pieces stay in registers between the two, the next Q THREADS in LDS (behind the teacher's), what is behind
// them is read twice.
template <typename T, int THREADS, int R, int Q, int WAVES, bool EVEN>
__global__ __launch_bounds__(THREADS, WAVES) void distill_step_kernel(DistillRows a, float c) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ float red[2][16], sum_of_weights;
  const Teacher t(lds, a.k);
  const long long r = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (r >= a.rows) return;
  const RowPieces<T> row((const T*)a.logits + r * a.stride, a.vocab);
  T* out = (T*)a.d_logits + r * a.d_stride;
  u32x4_t w[R];
#pragma unroll
  for (int j = 0; j < R; ++j) w[j] = (int)threadIdx.x < row.pieces - j * THREADS ? row.load(j * THREADS, threadIdx.x) : row.none();
  const float dloss = a.dloss[r];
  float P = 0.f;
  if (threadIdx.x < 64) {
    P = weights<T>(a, r, row.row, 0, a.vocab, a.vocab, a.vocab, t);
    gather_tokens(a, t);
    if (threadIdx.x == 0) sum_of_weights = P;
  }
  Stat st = {NONE, 0.f};
  constexpr int U = R < 16 / RowPieces<T>::N ? R : 16 / RowPieces<T>::N;      // 16 values at a time: more take more registers than there are
#pragma unroll
  for (int j = 0; j < R; j += U) {
    add_pieces<T, U>(st, w + j, c);
    __builtin_amdgcn_sched_barrier(0);
  }
  u32x4_t* kept = (u32x4_t*)lds + a.k + a.table / 4;         // each place its thread's own
  const int in_lds = min((R + Q) * THREADS, row.pieces);
  if constexpr (Q > 0) st = pieces_stat<T, THREADS, true>(row, R * THREADS, in_lds, c, st, kept);
  st = pieces_stat<T, THREADS>(row, (R + Q) * THREADS, row.pieces, c, st);
  add_single(st, row, c);
#pragma unroll
  for (int j = 0; j < R; ++j) asm volatile("" : "+v"(w[j]));          // packed until the gradient: bf16 values unpacked above would take twice the registers
  st = join_workgroup<THREADS>(st, c, red);                   // a barrier: sum_of_weights too
  P = sum_of_weights;
  const bool any = dloss != 0.f && P != 0.f;
  const float g = dloss / a.temperature, k = g * P / st.s;
  write_single(row, out, any, st, c, k);
  if (threadIdx.x >= THREADS - 64) write_loss(a, r, t, P, st);
  if (!any) {
    write_zeros<T, THREADS, EVEN>(row, out, 0, row.pieces);
    return;
  }
#pragma unroll
  for (int j = 0; j < R; ++j)
    if ((int)threadIdx.x < row.pieces - j * THREADS) row.template store_gradient<EVEN>(out, j * THREADS, threadIdx.x, w[j], st.m, c, k);
  if constexpr (Q > 0)
    for (int p = R * THREADS + threadIdx.x; p < in_lds; p += THREADS) row.template store_gradient<EVEN>(out, p, 0, kept[p - R * THREADS], st.m, c, k);
  write_pieces<T, THREADS, EVEN>(row, out, (R + Q) * THREADS, row.pieces, st, c, k);
  __syncthreads();                                            // the tokens' entries behind everybody's
  if (threadIdx.x < 64) write_tokens<T>(a, t, out, 0, a.vocab, a.vocab, a.vocab, st, c, k, g);
}

// ---------------------------------------------------------------- launches
size_t lds_of(const DistillRows& a) { return ((size_t)a.k * 16 + (size_t)a.table * 4 + 15) / 16 * 16; }
float factor_of(const DistillRows& a) { return (float)(1.4426950408889634074 / (double)a.temperature); }
int most_pieces(const DistillRows& a, int size) { return std::max(1, a.vocab / (16 / size)); }       // of a row, wherever it starts

// Parts of a row, where few rows would leave most of the chip idle.  Gradient: its workgroups are one launch in any case (us, 16384 pieces: 16 rows 6.3 in 16 parts, 12.2 in one;
// 128 rows 15.4 in four, 16.7; 256 rows 29.8 in four, 23.0 in one).
int grad_parts(int rows, int pieces) { return rows >= 256 ? 1 : std::max(1, std::min(pieces / 1024, 512 / rows)); }
// Loss, and loss and gradient in one call: in parts they are two and three launches, which cost the host 3 us each.  16 rows of 16384 pieces: loss 6.6 us in parts and 10.2
// in one, a call of it 14 and 10; step 12.6 and 17.2; of 32768 pieces 6.7 and 10.2, 14.5 and 19.4; 64 rows 11.6 and 11.5, 23.4 and 22.5.
int loss_parts(int rows, int pieces) { return rows >= 64 || pieces <= 32768 ? 1 : std::min((pieces + 1023) / 1024, 1024 / rows); }
int step_parts(int rows, int pieces) { return rows >= 64 || pieces <= 16384 ? 1 : std::min((pieces + 1023) / 1024, 1024 / rows); }
dim3 grid_of(int rows, int parts) {
  const int x = std::min(rows, 1 << 20);                      // a grid has less than 2^32 threads in one direction
  return dim3(x, (rows + x - 1) / x, parts);
}

template <typename T, int THREADS> void loss_kernel(const DistillRows& a, const float* partial, int parts, hipStream_t st) {
  hipLaunchKernelGGL((distill_loss_kernel<T, THREADS>), grid_of(a.rows, 1), dim3(THREADS), lds_of(a), st, a, factor_of(a), partial, parts);
}
template <typename T> hipError_t loss_rows(const DistillRows& a, int parts, void* ws, hipStream_t st) {
  const int pieces = most_pieces(a, sizeof(T));
  if (parts > 1) {
    hipLaunchKernelGGL((distill_part_kernel<T, 256>), grid_of(a.rows, parts), dim3(256), 0, st, a, factor_of(a), (pieces + parts - 1) / parts, (float*)ws);
    loss_kernel<T, 64>(a, (const float*)ws, parts, st);
  } else if (pieces <= 512) {                                 // eight pieces to a thread: fewer take longer where rows are many, and no less where they are few
    loss_kernel<T, 64>(a, nullptr, 0, st);                    // 16384 bf16 rows of 4000 29 us, with 128 threads 40 (64 rows 5.0, 5.0)
  } else if (pieces <= 1024) {
    loss_kernel<T, 128>(a, nullptr, 0, st);                   // 8192 of 8000 28, with 256 37 (64 rows 5.1, 5.0)
  } else if (pieces <= 2048) {                                // 3000 of 16000 19.9, with 128 20.6, with 512 26.5
    loss_kernel<T, 256>(a, nullptr, 0, st);
  } else {
    loss_kernel<T, 512>(a, nullptr, 0, st);
  }
  return hipGetLastError();
}

bool rows_even(const DistillRows& a, int size) {
  return ((((uintptr_t)a.logits - (uintptr_t)a.d_logits) | (uintptr_t)((a.stride - a.d_stride) * size)) & 15) == 0;
}

template <typename T, int THREADS, int R> hipError_t grad_kernel(const DistillRows& a, int parts, int share, hipStream_t st) {
  if (rows_even(a, sizeof(T)))
    hipLaunchKernelGGL((distill_grad_kernel<T, THREADS, R, true>), grid_of(a.rows, parts), dim3(THREADS), lds_of(a), st, a, factor_of(a), share);
  else
    hipLaunchKernelGGL((distill_grad_kernel<T, THREADS, R, false>), grid_of(a.rows, parts), dim3(THREADS), lds_of(a), st, a, factor_of(a), share);
  return hipGetLastError();
}
// Threads and pieces that each asks for ahead.  us, many rows: 500 pieces 128 x 4 51.8 (64 x 4 61.5, 256 x 4 59.3), 1000 256 x 4 53.2 (128 x 4 56.9, 256 x 16 57.1), 2000 256 x 16 55.7
// (256 x 4 60.7, 512 x 16 65.6), 4000 512 x 16 104.3 (256 x 16 108.6), 16000 1024 x 16 203.2 (512 x 16 204.4).
template <typename T> hipError_t grad_rows(const DistillRows& a, hipStream_t st) {
  const int pieces = most_pieces(a, sizeof(T)), parts = grad_parts(a.rows, pieces), share = (pieces + parts - 1) / parts;
  if (share <= 256) return grad_kernel<T, 64, 4>(a, parts, share, st);
  if (share <= 512) return grad_kernel<T, 128, 4>(a, parts, share, st);
  if (share <= 1024) return grad_kernel<T, 256, 4>(a, parts, share, st);
  if (share <= 2048) return grad_kernel<T, 256, 16>(a, parts, share, st);
  if (share <= 8192) return grad_kernel<T, 512, 16>(a, parts, share, st);
  return grad_kernel<T, 1024, 16>(a, parts, share, st);
}

template <typename T, int THREADS, int R, int Q, int WAVES, bool EVEN = true> hipError_t step_kernel(const DistillRows& a, hipStream_t st) {
  const auto kernel = distill_step_kernel<T, THREADS, R, Q, WAVES, EVEN>;
  if constexpr (Q > 0) {
    static DeviceOnce once;
    const hipError_t e = once.run([&] { return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, Q * THREADS * 16 + 24 * 1024); });
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid_of(a.rows, 1), dim3(THREADS), lds_of(a) + (size_t)Q * THREADS * 16, st, a, factor_of(a));
  return hipGetLastError();
}

// The fewest threads whose registers hold a row.  us, many rows: 500 pieces 128 x 4 53.9 (64 x 4, half of the row read twice, 64.7; 256 x 4 65.5), 1000 256 x 4 54.2 (256 x 8 57.5),
// 2000 256 x 8 55.8 (512 x 8 64.4), 4000 512 x 8 103.5 (512 x 16 105.1, 1024 x 16 202), 8000 512 x 16 106 (1024 x 16 140), 31250 1024 x 16 and 8 in LDS 115 (without these 133).
template <typename T> hipError_t step_rows(const DistillRows& a, void* ws, hipStream_t st) {
  const int pieces = most_pieces(a, sizeof(T)), parts = step_parts(a.rows, pieces);
  if (parts > 1) {                                            // one after the other, with the stats behind the parts'
    DistillRows b = a;
    b.stats = (float*)ws + 2 * (size_t)a.rows * parts;
    const hipError_t e = loss_rows<T>(b, parts, ws, st);
    return e != hipSuccess ? e : grad_rows<T>(b, st);
  }
  if (!rows_even(a, sizeof(T))) return step_kernel<T, 512, 16, 0, 4, false>(a, st);
  if (pieces <= 256) return step_kernel<T, 64, 4, 0, 4>(a, st);
  if (pieces <= 512) return step_kernel<T, 128, 4, 0, 4>(a, st);
  if (pieces <= 1024) return step_kernel<T, 256, 4, 0, 4>(a, st);
  if (pieces <= 2048) return step_kernel<T, 256, 8, 0, 4>(a, st);
  if (pieces <= 4096) return step_kernel<T, 512, 8, 0, 4>(a, st);
  if (pieces <= 8192) return step_kernel<T, 512, 16, 0, 4>(a, st);
  if (pieces <= 16384) return step_kernel<T, 1024, 16, 0, 4>(a, st);
  return step_kernel<T, 1024, 16, 8, 4>(a, st);
}

}  // namespace

size_t distill_workspace(int rows, int vocab) {
  DistillRows a = {};
  a.vocab = vocab;
  const int parts = step_parts(rows, most_pieces(a, 4));      // no fewer than of bf16 rows, or of a loss
  return parts > 1 ? ((size_t)rows * (parts + 1) * 2 * sizeof(float) + 255) / 256 * 256 : 0;
}
template <typename T> static hipError_t loss_as(const DistillRows& a, void* ws, hipStream_t st) { return loss_rows<T>(a, loss_parts(a.rows, most_pieces(a, sizeof(T))), ws, st); }
hipError_t launch_distill(const DistillRows& a, bool bf16, void* ws, hipStream_t st) { return bf16 ? loss_as<bf16_t>(a, ws, st) : loss_as<float>(a, ws, st); }
hipError_t launch_distill_grad(const DistillRows& a, bool bf16, hipStream_t st) { return bf16 ? grad_rows<bf16_t>(a, st) : grad_rows<float>(a, st); }
hipError_t launch_distill_step(const DistillRows& a, bool bf16, void* ws, hipStream_t st) { return bf16 ? step_rows<bf16_t>(a, ws, st) : step_rows<float>(a, ws, st); }
