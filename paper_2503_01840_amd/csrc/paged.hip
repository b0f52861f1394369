// Rows written into the pages of their sequences, as they are or in 8 bits, and read back.
#include "paged.hpp"

namespace {

constexpr int LEAST_EXP = 127 - 110, MOST_EXP = 127 + 120;
// 256 * 2^120 is behind bf16's range: a row of that exponent takes 240 for what is nearer to 256 (still within 2^-4 of the value).
__device__ __forceinline__ float largest_code(int x) { return x == MOST_EXP ? 240.f : 448.f; }

struct PagedRows {
  const int32_t* start;
  const int32_t* n;
  const int32_t* row_start;
  char* k;                  // dense rows
  char* v;
  long long n_rows, row_stride;     // stride in bytes
  Divisor rows;
};

// Slot of row j of sequence b, -1 where there is none; *row: its dense row
template <bool READ>
__device__ __forceinline__ long long place_of_row(const PagedView& c, const PagedRows& r, int b, int j, long long* row) {
  if (r.n != nullptr && j >= r.n[b]) return -1;
  *row = r.row_start != nullptr ? (long long)r.row_start[b] + j : (long long)b * r.rows.d + j;
  const long long pos = (r.start != nullptr ? (long long)r.start[b] : 0) + j;
  if (*row < 0 || *row >= r.n_rows || pos < 0 || pos >= c.tokens) return -1;
  const int page = c.table[(size_t)b * c.max_pages + (int)pos / c.page];
  if (page < 0 || page >= c.n_pages) return -1;
  return (long long)page * c.page.d + (int)pos % c.page;
}

// The exponent byte of a row whose largest finite magnitude is amax: the smallest e with amax <= 448 * 2^e, at least -110.
__device__ __forceinline__ int exp_of(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  return max((int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), LEAST_EXP);
}

// One wavefront per (row, head): k, then v.
template <typename T, bool FP8, bool READ>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedView c, PagedRows r, int units, Divisor heads) {
  const int unit = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (unit >= units) return;
  const int row_of = unit / heads, h = unit % heads, b = row_of / r.rows, j = row_of % r.rows;
  long long row;
  const long long slot = place_of_row<READ>(c, r, b, j, &row);
  if (slot < 0) return;
  for (int kv = 0; kv < 2; ++kv) {
    T* dense = (T*)((kv ? r.v : r.k) + row * r.row_stride) + (size_t)h * c.d;
    const size_t at = (size_t)slot * c.Hkv + h;
    if constexpr (!FP8) {
      T* cached = (T*)(kv ? c.v : c.k) + at * c.d;
      for (int i = lane; i < c.d; i += 64) {
        if (READ) dense[i] = cached[i];
        else cached[i] = dense[i];
      }
    } else {
      uint8_t* codes = (uint8_t*)(kv ? c.v : c.k) + at * c.d;
      uint8_t* xp = (kv ? c.v_exp : c.k_exp) + at;
      if (READ) {
        const float scale = exp_scale(*xp);
        for (int i = lane; i < c.d; i += 64) dense[i] = f32_to_bf16(__builtin_amdgcn_cvt_f32_fp8((int)codes[i], 0) * scale);
      } else {
        float amax = 0.f;
        for (int i = lane; i < c.d; i += 64) {
          const float a = fabsf(bf16_to_f32(dense[i]));
          if (a < __builtin_huge_valf()) amax = fmaxf(amax, a);
        }
        const int x = exp_of(wave_max(amax));
        const float inv = __uint_as_float((uint32_t)(254 - x) << 23), most = largest_code(x);
        for (int i = lane; i < c.d; i += 64) {
          const float a = bf16_to_f32(dense[i]);
          const uint32_t code = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(a * inv, -most), most), 0.f, 0, false) & 0xFFu;
          codes[i] = fabsf(a) < __builtin_huge_valf() ? (uint8_t)code : (uint8_t)0x7F;
        }
        if (lane == 0) *xp = (uint8_t)x;
      }
    }
  }
}

template <bool READ>
hipError_t launch_rows(const PagedView& c, int dtype, const PagedRows& r, int B, hipStream_t st) {
  const int units = B * r.rows.d * c.Hkv;
  const dim3 grid((units + 3) / 4);
  const Divisor heads = divisor(c.Hkv);
  if (dtype == PAGED_FP8) hipLaunchKernelGGL((paged_rows_kernel<bf16_t, true, READ>), grid, dim3(256), 0, st, c, r, units, heads);
  else if (dtype == PAGED_BF16) hipLaunchKernelGGL((paged_rows_kernel<bf16_t, false, READ>), grid, dim3(256), 0, st, c, r, units, heads);
  else hipLaunchKernelGGL((paged_rows_kernel<float, false, READ>), grid, dim3(256), 0, st, c, r, units, heads);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_rows(const PagedView& c, int dtype, bool read, int B, int rows, const int32_t* start, const int32_t* n,
                             const int32_t* row_start, void* k, void* v, long long n_rows, long long row_bytes, hipStream_t st) {
  const PagedRows r = {start, n, row_start, (char*)k, (char*)v, n_rows, row_bytes, divisor(rows)};
  return read ? launch_rows<true>(c, dtype, r, B, st) : launch_rows<false>(c, dtype, r, B, st);
}
