// Attention of one new token of every sequence over its paged keys and values (bf16, fp32, or 8 bits with a scale per row).
//
// A workgroup has the (up to 16) query heads of one KV head and one part of a sequence; its wavefronts take tiles of 16 or 32 keys in turn, each
// with a running maximum, sum and output of its own, and are joined through LDS at the end; parts of a sequence are joined by a second launch.
// Everything a wavefront multiplies comes from global memory straight into the registers where the matrix units want it:
//   scores  S^T = K Q^T: lane (g, m) = (lane / 16, lane % 16) holds key m of a block of 16, of whose row the four lanes g load 64 contiguous bytes at a time;
//           which dimensions these are does not matter as long as Q's operand has the same.
//           The result has for query m the keys 4 g + i of both blocks: eight keys in a lane, which is an operand of the next product as it stands.
//   values  O^T = V^T P^T: lane (g, m) loads of each of its eight keys' rows the dimensions m D / 16 ... (16 lanes: the whole row), and
//           turns eight keys by two bytes or one around in registers; product i has the i-th dimension of every lane.
// No tile passes through LDS, no wavefront waits for another, and a page may end anywhere: the lanes look up 16 or 32 keys' pages one tile
// ahead of the loads, which are one tile ahead of the products.
#include <cfloat>

#include "paged.hpp"
#include "paged_rules.hpp"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int WAVES = 4;
constexpr float SLACK = 8.f;              // the running maximum moves when a score exceeds it by more than 2^8

struct AttnArgs {
  PagedView c;
  const char* q;
  long long q_stride;                     // in bytes
  const int32_t* kv_len;
  int max_len, H, G, chunk, parts;
  Divisor by_units;                       // KV heads x row tiles
  Divisor by_heads;
  float scale_log2;
  void* out;
  float* lse;
  float* part_o;                          // [B, H, parts, D]
  float* part_ml;                         // [B, H, parts, 2]
};

template <int I, int N, typename F> __device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

// Lane E of every 16 lanes, to all of them.
template <int E> __device__ __forceinline__ uint32_t bcast16(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x150 + E, 0xF, 0xF, true); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Two codes of a dword (low or high half) as bf16: times 2^k, exact.
template <bool HIGH> __device__ __forceinline__ uint32_t bf16_of_codes(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, HIGH));
}

template <int TYPE> struct CacheType;
template <> struct CacheType<PAGED_FP32> { static constexpr int SIZE = 4, BLOCKS = 1; typedef float row; };
template <> struct CacheType<PAGED_BF16> { static constexpr int SIZE = 2, BLOCKS = 2; typedef bf16_t row; };
template <> struct CacheType<PAGED_FP8> { static constexpr int SIZE = 1, BLOCKS = 2; typedef bf16_t row; };

template <int TYPE, int D>
struct Tile {                             // one tile's keys and values, as loaded
  static constexpr int SIZE = CacheType<TYPE>::SIZE, BLOCKS = CacheType<TYPE>::BLOCKS;
  static constexpr int KL = D * SIZE / 64, E = 4 * BLOCKS, VD = D * SIZE / 64;      // loads of a key row, value rows, dwords of a value row
  u32x4 k[BLOCKS][KL];
  uint32_t v[E][VD];
  uint32_t exps;                          // 8 bits: lane (g, m): of key (g, m % 8), its key row's (m < 8) or value row's
};

template <int TYPE, int D>
__global__ __launch_bounds__(64 * WAVES) void paged_attn_kernel(AttnArgs p) {
#pragma clang fp contract(off)            // a score and the maximum that it may be have to be the same number, however large
  typedef Tile<TYPE, D> T;
  typedef typename CacheType<TYPE>::row Row;
  constexpr bool FP8 = TYPE == PAGED_FP8, F32 = TYPE == PAGED_FP32;
  constexpr int BLOCKS = T::BLOCKS, E = T::E, KEYS = 16 * BLOCKS, NF = D / 16;      // NF: products over the values
  constexpr int LDS_ROW = D + 4;
  __shared__ float so[WAVES][PAGED_ROWS][LDS_ROW], sml[WAVES][PAGED_ROWS][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int b = blockIdx.y, part = (int)blockIdx.x / p.by_units, unit = (int)blockIdx.x % p.by_units, hk = unit % p.by_heads, rt = unit / p.by_heads;
  const int n = min(max(p.kv_len[b], 0), p.max_len);
  const int begin = part * p.chunk, end = min(n, begin + p.chunk);
  if (begin >= n && part > 0) return;
  const int head0 = hk * p.G + rt * PAGED_ROWS, rows = min(PAGED_ROWS, p.G - rt * PAGED_ROWS);
  const int n_tiles = (end - begin + KEYS - 1) / KEYS;

  // queries, in the order of the keys' dimensions
  u32x4 q[T::SIZE == 1 ? 2 * T::KL : T::KL];
  {
    const char* qrow = p.q + (long long)b * p.q_stride + (size_t)(head0 + min(m, rows - 1)) * (D * sizeof(Row));
#pragma unroll
    for (int j = 0; j < (int)(sizeof(q) / 16); ++j) {
      const int at = FP8 ? 64 * (j >> 1) + 16 * g + 8 * (j & 1) : F32 ? 16 * j + 4 * g : 32 * j + 8 * g;
      q[j] = *(const u32x4*)(qrow + at * sizeof(Row));
      if (m >= rows) q[j] = u32x4{0, 0, 0, 0};
    }
  }

  const int32_t* table = p.c.table + (size_t)b * p.c.max_pages;
  const uint32_t row_bytes = (uint32_t)p.c.Hkv * (D * T::SIZE);
  const char* kbase = p.c.k + (size_t)hk * (D * T::SIZE) + 16 * g;
  const char* vbase = p.c.v + (size_t)hk * (D * T::SIZE) + m * (D * T::SIZE / 16);
  const uint8_t* xbase = FP8 ? (m < 8 ? p.c.k_exp : p.c.v_exp) + hk : nullptr;
  const int my_e = m % E, my_key = 16 * (my_e >> 2) + 4 * g + (my_e & 3);           // the key of a tile whose page this lane looks up
  const int from_lane = 4 * (16 * (m >> 2) + (m & 3));                              // the lane that has key m of block 0 (of block 1: 4 lanes on), in bytes

  auto slot_of = [&](int tile) {          // of this lane's key; keys behind the end repeat the last one
    const int key = min(begin + tile * KEYS + my_key, end - 1);
    const int page = min(max(table[key / p.c.page], 0), p.c.n_pages - 1);
    return page * p.c.page.d + key % p.c.page;
  };
  auto load = [&](T& t, int slot) {
    if constexpr (FP8) t.exps = xbase[(size_t)(uint32_t)slot * (uint32_t)p.c.Hkv];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      const uint32_t s = (uint32_t)__builtin_amdgcn_ds_bpermute(from_lane + 16 * i, slot);
      const char* row = kbase + (uint64_t)s * row_bytes;
#pragma unroll
      for (int j = 0; j < T::KL; ++j) t.k[i][j] = *(const u32x4*)(row + 64 * j);
    }
    static_for<0, E>([&](auto e) {
      const char* row = vbase + (uint64_t)bcast16<e>((uint32_t)slot) * row_bytes;
      if constexpr (T::VD == 1) t.v[e][0] = *(const uint32_t*)row;
      else if constexpr (T::VD == 2) *(u32x2*)t.v[e] = *(const u32x2*)row;
      else
#pragma unroll
        for (int j = 0; j < T::VD; j += 4) *(u32x4*)(t.v[e] + j) = *(const u32x4*)(row + 4 * j);
    });
  };

  floatx4 o[NF];
#pragma unroll
  for (int i = 0; i < NF; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
  float mx = -FLT_MAX, l = 0.f;           // of query m; l: over this lane's keys

  auto work = [&](T& t, int tile) {
    // scores of keys (g, e), e = 4 block + i
    float x[E];
    float kscale[BLOCKS];
    if constexpr (FP8)
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) kscale[i] = exp_scale((uint32_t)__builtin_amdgcn_ds_bpermute(from_lane + 16 * i, (int)t.exps));
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < T::KL; ++j) {
        if constexpr (F32) {
#pragma unroll
          for (int h = 0; h < 4; ++h) s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[i][j][h]), __uint_as_float(q[j][h]), s, 0, 0, 0);
        } else if constexpr (FP8) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t w0 = t.k[i][j][2 * h], w1 = t.k[i][j][2 * h + 1];
            const u32x4 a = {bf16_of_codes<false>(w0, kscale[i]), bf16_of_codes<true>(w0, kscale[i]), bf16_of_codes<false>(w1, kscale[i]),
                             bf16_of_codes<true>(w1, kscale[i])};
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, q[2 * j + h]), s, 0, 0, 0);
          }
        } else {
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[i][j]), __builtin_bit_cast(bf16x8, q[j]), s, 0, 0, 0);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) x[4 * i + r] = s[r] * p.scale_log2;
    }
    const int left = end - begin - tile * KEYS;             // keys of this tile; uniform
    if (left < KEYS) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool seen = 16 * (e >> 2) + 4 * g + (e & 3) < left;
        if (!seen) x[e] = -__builtin_huge_valf();
#pragma unroll
        for (int j = 0; j < T::VD; ++j) t.v[e][j] = seen ? t.v[e][j] : 0u;          // a weight of zero does not silence an infinity
      }
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < E; ++e) top = fmaxf(top, x[e]);
    top = xlane_max_step<5>(xlane_max_step<4>(top));
    if (__any(top > mx + SLACK)) {
      const float to = fmaxf(mx, top), a = exp2_fast(mx - to);
      mx = to;
      l *= a;
#pragma unroll
      for (int i = 0; i < NF; ++i) o[i] *= a;
    }
    float w[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      w[e] = exp2_fast(x[e] - mx);
      l += w[e];
    }
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < NF; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[e][i]), w[e], o[i], 0, 0, 0);
    } else {
      if constexpr (FP8) static_for<0, E>([&](auto e) { w[e] *= exp_scale(bcast16<8 + e>(t.exps)); });
      // a weight as a head of 8 bits and a tail of 8 more; the tail of a weight above zero is above zero, so that an infinity stays one
      u32x4 head, tail;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w0 = __float_as_uint(w[2 * j]), w1 = __float_as_uint(w[2 * j + 1]);
        head[j] = __builtin_amdgcn_perm(w1, w0, 0x07060302u);
        tail[j] = pack_bf16x2(fmaf(__uint_as_float(w0 & 0xFFFF0000u), -0x1.fffffep-1f, w[2 * j]), fmaf(__uint_as_float(w1 & 0xFFFF0000u), -0x1.fffffep-1f, w[2 * j + 1]));
      }
      auto product = [&](int i, const u32x4& a) {
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, head), o[i], 0, 0, 0);
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, tail), o[i], 0, 0, 0);
      };
      if constexpr (FP8) {
#pragma unroll
        for (int c = 0; c < T::VD; ++c)                      // four dimensions of a dword
#pragma unroll
          for (int hi = 0; hi < 2; ++hi) {
            u32x4 a0, a1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t two = __builtin_amdgcn_perm(t.v[2 * j + 1][c], t.v[2 * j][c], hi ? 0x07030602u : 0x05010400u);
              a0[j] = bf16_of_codes<false>(two, 1.f);
              a1[j] = bf16_of_codes<true>(two, 1.f);
            }
            product(4 * c + 2 * hi, a0);
            product(4 * c + 2 * hi + 1, a1);
          }
      } else {
#pragma unroll
        for (int c = 0; c < T::VD; ++c) {
          u32x4 a0, a1;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            a0[j] = __builtin_amdgcn_perm(t.v[2 * j + 1][c], t.v[2 * j][c], 0x05040100u);
            a1[j] = __builtin_amdgcn_perm(t.v[2 * j + 1][c], t.v[2 * j][c], 0x07060302u);
          }
          product(2 * c, a0);
          product(2 * c + 1, a1);
        }
      }
    }
  };

  if (wave < n_tiles) {
    T ta, tb;
    int slot = slot_of(wave), next = slot_of(wave + WAVES);
    load(ta, slot);
    for (int t = wave;;) {
      if (t + WAVES < n_tiles) load(tb, next);
      next = slot_of(t + 2 * WAVES);
      __builtin_amdgcn_sched_barrier(0);
      work(ta, t);
      if ((t += WAVES) >= n_tiles) break;
      if (t + WAVES < n_tiles) load(ta, next);
      next = slot_of(t + 2 * WAVES);
      __builtin_amdgcn_sched_barrier(0);
      work(tb, t);
      if ((t += WAVES) >= n_tiles) break;
    }
  }
  l = xlane_sum_step<5>(xlane_sum_step<4>(l));

  // the wavefronts' results, joined
  if (m < rows) {
    if (g == 0) { sml[wave][m][0] = mx; sml[wave][m][1] = l; }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < NF; ++i) so[wave][m][NF * (4 * g + r) + i] = o[i][r];
  }
  __syncthreads();
  const bool whole = n <= p.chunk;
  for (int u = threadIdx.x; u < rows * (D / 4); u += 64 * WAVES) {
    const int row = u / (D / 4), d4 = u % (D / 4) * 4;
    float M = sml[0][row][0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sml[w][row][0]);
    float L = 0.f;
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w < n_tiles) {
        const float a = exp2_fast(sml[w][row][0] - M);
        L += a * sml[w][row][1];
        sum += a * *(const floatx4*)&so[w][row][d4];
      }
    }
    const size_t bh = (size_t)b * p.H + head0 + row;
    if (whole) {
      if (n == 0) sum = floatx4{0.f, 0.f, 0.f, 0.f};
      else sum /= L;
      if constexpr (F32) *(floatx4*)((float*)p.out + bh * D + d4) = sum;
      else store4_plain((bf16_t*)p.out, bh * D + d4, sum[0], sum[1], sum[2], sum[3]);
      if (d4 == 0 && p.lse != nullptr) p.lse[bh] = n == 0 ? -__builtin_huge_valf() : (M + log2f(L)) * 0.69314718055994531f;
    } else {
      *(floatx4*)(p.part_o + (bh * p.parts + part) * D + d4) = sum;
      if (d4 == 0) *(float2*)(p.part_ml + (bh * p.parts + part) * 2) = make_float2(M, L);
    }
  }
}

// One workgroup per (sequence, query head): its parts, D / 4 lanes to each.
template <bool F32, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(AttnArgs p) {
  constexpr int LANES = D / 4, PER = 256 / LANES;
  __shared__ float so[PER][D], sml[PER][2];
  const int h = blockIdx.x, b = blockIdx.y, n = min(max(p.kv_len[b], 0), p.max_len);
  const int parts = (n + p.chunk - 1) / p.chunk;
  if (parts <= 1) return;
  const size_t bh = (size_t)b * p.H + h;
  const int at = threadIdx.x / LANES, d4 = threadIdx.x % LANES * 4;
  float M = -FLT_MAX, L = 0.f;
  floatx4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int i = at; i < parts; i += PER) {
    const float2 ml = *(const float2*)(p.part_ml + (bh * p.parts + i) * 2);
    const floatx4 v = *(const floatx4*)(p.part_o + (bh * p.parts + i) * D + d4);
    const float to = fmaxf(M, ml.x), a = exp2_fast(M - to), c = exp2_fast(ml.x - to);
    M = to;
    L = L * a + ml.y * c;
    sum = sum * a + v * c;
  }
  *(floatx4*)&so[at][d4] = sum;
  if (d4 == 0) { sml[at][0] = M; sml[at][1] = L; }
  __syncthreads();
  if (at > 0) return;
  for (int i = 1; i < min(PER, parts); ++i) {
    const float to = fmaxf(M, sml[i][0]), a = exp2_fast(M - to), c = exp2_fast(sml[i][0] - to);
    M = to;
    L = L * a + sml[i][1] * c;
    sum = sum * a + *(const floatx4*)&so[i][d4] * c;
  }
  sum /= L;
  if constexpr (F32) *(floatx4*)((float*)p.out + bh * D + d4) = sum;
  else store4_plain((bf16_t*)p.out, bh * D + d4, sum[0], sum[1], sum[2], sum[3]);
  if (d4 == 0 && p.lse != nullptr) p.lse[bh] = (M + log2f(L)) * 0.69314718055994531f;
}

template <int TYPE, int D>
hipError_t launch(const AttnArgs& a, int B, int units, hipStream_t st) {
  hipLaunchKernelGGL((paged_attn_kernel<TYPE, D>), dim3(units * a.parts, B), dim3(64 * WAVES), 0, st, a);
  if (a.parts > 1) hipLaunchKernelGGL((paged_join_kernel<TYPE == PAGED_FP32, D>), dim3(a.H, B), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t paged_attention_workspace(int B, int H, int Hkv, int d, int max_len) {
  return paged_partial_floats(B, H, d, paged_split(B, H, Hkv, max_len).parts) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedView& c, int dtype, int B, int H, const void* q, long long q_bytes, const int32_t* kv_len, int max_len,
                                  float scale, void* out, float* lse, void* workspace, hipStream_t st) {
  const PagedSplit s = paged_split(B, H, c.Hkv, max_len);
  float* part_o = (float*)workspace;
  const AttnArgs a = {c, (const char*)q, q_bytes, kv_len, max_len, H, H / c.Hkv, s.chunk, s.parts, divisor(c.Hkv * s.row_tiles), divisor(c.Hkv),
                      scale * 1.4426950408889634f, out, lse, part_o, part_o ? part_o + (size_t)B * H * s.parts * c.d : nullptr};
  const int units = c.Hkv * s.row_tiles;
  if (dtype == PAGED_FP8) return c.d == 128 ? launch<PAGED_FP8, 128>(a, B, units, st) : launch<PAGED_FP8, 64>(a, B, units, st);
  if (dtype == PAGED_BF16) return c.d == 128 ? launch<PAGED_BF16, 128>(a, B, units, st) : launch<PAGED_BF16, 64>(a, B, units, st);
  return c.d == 128 ? launch<PAGED_FP32, 128>(a, B, units, st) : launch<PAGED_FP32, 64>(a, B, units, st);
}
