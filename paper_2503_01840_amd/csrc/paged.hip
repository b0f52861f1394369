// Rows written into the pages of their sequences, as they are or in 8 bits, and read back.
//
// A thread has 16 bytes of a dense key row and the same of the value row; CH = head_dim * element size / 16 neighbouring lanes have a head, whose
// largest magnitude they find by exchanges within 16 lanes.  A power of two as the scale makes the scaling and the way back exact: a
// value is rounded once, to a code.  Where a wavefront lies within one row (a row of 64 pieces and more), its place is looked up with
// scalar loads (40954 rows of 8 heads into 8 bits 54 us, by every lane for itself 68).  Bound by bytes; a thread has 32 of them in flight and nothing else waits, so eight wavefronts a SIMD cover the latency: 20480 rows of 8 heads of 128 read
// back from 8 bits in 26.5 us (4.8 TB/s, a large copy's rate; 106 by a wavefront to a head and two bytes to a lane), 8960 written in 12.6 (4.4 TB/s; 45).
#include "paged.hpp"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int LEAST_EXP = 127 - 110, MOST_EXP = 127 + 120;
// 256 * 2^120 is behind bf16's range: a row of that exponent takes 240 for what is nearer to 256 (still within 2^-4 of the value).
__device__ __forceinline__ float largest_code(int x) { return x == MOST_EXP ? 240.f : 448.f; }

struct PagedRows {
  const int32_t* start;
  const int32_t* n;
  const int32_t* row_start;
  char* k;                  // dense rows
  char* v;
  long long n_rows, row_bytes;
  Divisor rows;             // of a sequence, at most
};

// Slot of row j of sequence b, -1 where there is none; *row: its dense row
__device__ __forceinline__ int place_of_row(const PagedView& c, const PagedRows& r, int b, int j, long long* row) {
  *row = r.row_start != nullptr ? (long long)r.row_start[b] + j : (long long)b * r.rows.d + j;
  const long long pos = (r.start != nullptr ? (long long)r.start[b] : 0) + j;
  if ((r.n != nullptr && j >= r.n[b]) || *row < 0 || *row >= r.n_rows || pos < 0 || pos >= c.tokens) return -1;
  const int page = c.table[(size_t)b * c.max_pages + (int)pos / c.page];
  if (page < 0 || page >= c.n_pages) return -1;
  return page * c.page.d + (int)pos % c.page;
}

// The exponent byte of a row whose largest finite magnitude is amax: the smallest e with amax <= 448 * 2^e, at least -110.
__device__ __forceinline__ int exp_of(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  return max((int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), LEAST_EXP);
}

__device__ __forceinline__ float finite_magnitude(float x) {
  const float a = fabsf(x);
  return a < __builtin_huge_valf() ? a : 0.f;
}

// Eight bf16 values to codes, under the scale of the CH lanes that have their row.
template <int CH> __device__ __forceinline__ u32x2 to_codes(const u32x4& w, int* x) {
  float f[8], amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    amax = fmaxf(amax, finite_magnitude(f[i]));
  }
  amax = xlane_max_step<2>(xlane_max_step<1>(xlane_max_step<0>(amax)));
  if constexpr (CH == 16) amax = xlane_max_step<3>(amax);
  *x = exp_of(amax);
  const float inv = __uint_as_float((uint32_t)(254 - *x) << 23), most = largest_code(*x);
  u32x2 codes;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = fminf(fmaxf(f[4 * i + j] * inv, -most), most);
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (!(fabsf(f[4 * i + j]) < __builtin_huge_valf())) c = (c & ~(0xFF << 8 * j)) | 0x7F << 8 * j;
    codes[i] = (uint32_t)c;
  }
  return codes;
}

__device__ __forceinline__ u32x4 from_codes(const u32x2& c, float scale) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[i], scale, false));
    w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c[i], scale, true));
  }
  return w;
}

// per_row: pieces of a row (KV heads * CH); WITHIN: a multiple of 64, so that a wavefront has pieces of one row
template <int CH, bool FP8, bool READ, bool WITHIN>
__global__ __launch_bounds__(256) void paged_rows_kernel(int pieces, Divisor per_row, Divisor rows, const int32_t* start, const int32_t* n, const int32_t* row_start,
                                                         PagedView c, PagedRows r) {
  r.rows = rows, r.start = start, r.n = n, r.row_start = row_start;       // in registers when the kernel starts: 2 to 6 % less time
  const int at = blockIdx.x * 256 + threadIdx.x;
  if (at >= pieces) return;
  int line = at / per_row;
  if constexpr (WITHIN) line = __builtin_amdgcn_readfirstlane(line);
  const int piece = at - line * per_row.d;
  long long row;
  const int slot = place_of_row(c, r, line / r.rows, line % r.rows, &row);
  if (slot < 0) return;
  const size_t dense = (size_t)row * r.row_bytes + (size_t)piece * 16;
  const size_t cached = ((size_t)slot * per_row.d + piece) * (FP8 ? 8 : 16);
  const size_t exps = (size_t)slot * c.Hkv + piece / CH;
  if constexpr (READ) {
    if constexpr (FP8) {
      const u32x2 k = *(const u32x2*)(c.k + cached), v = *(const u32x2*)(c.v + cached);
      const float ks = exp_scale(c.k_exp[exps]), vs = exp_scale(c.v_exp[exps]);
      *(u32x4*)(r.k + dense) = from_codes(k, ks);
      *(u32x4*)(r.v + dense) = from_codes(v, vs);
    } else {
      const u32x4 k = *(const u32x4*)(c.k + cached), v = *(const u32x4*)(c.v + cached);
      *(u32x4*)(r.k + dense) = k;
      *(u32x4*)(r.v + dense) = v;
    }
  } else {
    const u32x4 k = *(const u32x4*)(r.k + dense), v = *(const u32x4*)(r.v + dense);
    if constexpr (FP8) {
      int kx, vx;
      *(u32x2*)(c.k + cached) = to_codes<CH>(k, &kx);
      *(u32x2*)(c.v + cached) = to_codes<CH>(v, &vx);
      if (piece % CH == 0) {
        c.k_exp[exps] = (uint8_t)kx;
        c.v_exp[exps] = (uint8_t)vx;
      }
    } else {
      *(u32x4*)(c.k + cached) = k;
      *(u32x4*)(c.v + cached) = v;
    }
  }
}

template <int CH, bool FP8, bool READ>
hipError_t launch(const PagedView& c, const PagedRows& r, int B, hipStream_t st) {
  const int per_row = c.Hkv * CH, pieces = B * r.rows.d * per_row;
  const dim3 grid((pieces + 255) / 256);
  if (per_row % 64 == 0) hipLaunchKernelGGL((paged_rows_kernel<CH, FP8, READ, true>), grid, dim3(256), 0, st, pieces, divisor(per_row), r.rows, r.start, r.n, r.row_start, c, r);
  else hipLaunchKernelGGL((paged_rows_kernel<CH, FP8, READ, false>), grid, dim3(256), 0, st, pieces, divisor(per_row), r.rows, r.start, r.n, r.row_start, c, r);
  return hipGetLastError();
}

template <bool READ>
hipError_t launch_rows(const PagedView& c, int dtype, const PagedRows& r, int B, hipStream_t st) {
  if (dtype == PAGED_FP8) return c.d == 128 ? launch<16, true, READ>(c, r, B, st) : launch<8, true, READ>(c, r, B, st);
  // copies: what the pieces are does not matter
  return dtype == PAGED_BF16 ? (c.d == 128 ? launch<16, false, READ>(c, r, B, st) : launch<8, false, READ>(c, r, B, st))
                             : (c.d == 128 ? launch<32, false, READ>(c, r, B, st) : launch<16, false, READ>(c, r, B, st));
}

}  // namespace

hipError_t launch_paged_rows(const PagedView& c, int dtype, bool read, int B, int rows, const int32_t* start, const int32_t* n,
                             const int32_t* row_start, void* k, void* v, long long n_rows, long long row_bytes, hipStream_t st) {
  const PagedRows r = {start, n, row_start, (char*)k, (char*)v, n_rows, row_bytes, divisor(rows)};
  return read ? launch_rows<true>(c, dtype, r, B, st) : launch_rows<false>(c, dtype, r, B, st);
}
