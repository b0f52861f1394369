// Attention of one new token of every sequence over its paged keys and values (bf16, fp32, or 8 bits with a scale per row):
// o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), s_j = scale q.k_j, in one pass with a running maximum m.
//
// A wavefront has up to 16 or 32 query heads of one KV head and walks over tiles of 32 keys (fp32: 16), with a maximum, a sum and an output of its
// own; what wavefronts have of one sequence is joined at the end, through LDS within a workgroup, by a second launch between workgroups (paged_rules.hpp says which).
// Everything a wavefront multiplies comes from global memory straight into the registers where the matrix units want it:
//   scores  S^T = K Q^T: lane (g, m) = (lane / 16, lane % 16) holds key m of a block of 16, of whose row the four lanes g load 64 contiguous bytes at a time;
//           which dimensions these are does not matter as long as Q's operand has the same.
//           The result has for query m the keys 4 g + i of both blocks: eight keys in a lane, which is an operand of the next product as it stands.
//   values  O^T = V^T P^T: lane (g, m) loads of each of its eight keys' rows the dimensions m D / 16 ... (16 lanes: the whole row), and
//           turns eight keys by two bytes or one around in registers; product i has the i-th dimension of every lane.
// No tile passes through LDS, no wavefront waits for another while it walks, and a page may end anywhere: pages are looked up one tile ahead of the loads, which are one
// tile ahead of the products.  8-bit rows become bf16 by an exact conversion (a value row's scale multiplies its weight instead: a conversion takes two keys).
//
// Bound by bytes: 64 sequences of 512..2048 tokens, 32 heads of 128 over 8, bf16: 64.0 us, 5.2 TB/s (8 bits: 40.0 us, of which 5 join); one of 131071
// under 64 heads in 8 bits 56.9 us, 5.2 TB/s and 5.2 us of joining; 256 of 1300 in bf16 237 to 253 us by box, 5.4 to 5.7 TB/s.  A tile of 128 dimensions is 8 score and 24 value products and some
// 200 (bf16) or 250 (8 bits) vector instructions, 11 and 23 % of the time that its bytes take.  Two tiles of registers in flight in turn took 211 registers and 4 % longer than
// one whose halves are asked for again as soon as they are used (150).
#include <cfloat>

#include "paged.hpp"
#include "paged_rules.hpp"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int WAVES = PAGED_WAVES;
constexpr float SLACK = 8.f;              // the running maximum moves when a score exceeds it by more than 2^8
constexpr int PARTS = 3;                  // bf16 terms of a weight

// What a kernel needs for its first loads comes in arguments of its own as well, which are in registers when it starts (one sequence of 4096 tokens 10.2 -> 9.8 us, of 128
// 4.55 -> 4.46).
struct AttnArgs {
  PagedView c;
  const char* q;
  long long q_stride;                     // in bytes
  const int32_t* kv_len;
  int max_len, H, G, B, units;            // units: KV heads x row tiles
  int ranges;                             // a launch over ranges: into how many all sequences' tiles are divided
  Divisor by_units, by_heads;
  float scale_log2;
  void* out;
  float* lse;
  float* part_o;                          // [ranges + B, H, D]: of range r and sequence b at r + b
  float* part_ml;                         // [ranges + B, H, 2]
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

// An address that every lane has, kept in scalar registers: a load then adds a lane's 32 bits to it by itself.
typedef const char __attribute__((address_space(1)))* GlobalBytes;
__device__ __forceinline__ GlobalBytes uniform(const char* p) {
  GlobalBytes g = (GlobalBytes)(uintptr_t)p;
  asm("" : "+s"(g));
  return g;
}
__device__ __forceinline__ uint32_t in_place(uint32_t offset) {      // keeps the widening to 64 bits, and so the scalar base, at the load
  asm("" : "+v"(offset));
  return offset;
}
template <typename T> __device__ __forceinline__ T load_at(GlobalBytes p) { return *(const T __attribute__((address_space(1)))*)p; }

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
  uint32_t exps;                          // 8 bits: see load_exps
};

// One (KV head, row tile) of one sequence: queries in registers, the running maximum, sum and output of the tiles that this wavefront has taken.
// BLOCKED: pages are whole blocks of 16 keys, so that a block's page is looked up once, by scalar loads, and rows lie at fixed distances.
// TILES: of 16 query heads each.
template <int TYPE, int D, bool BLOCKED, int TILES>
struct Walk {
  typedef Tile<TYPE, D> T;
  typedef typename CacheType<TYPE>::row Row;
  static constexpr bool FP8 = TYPE == PAGED_FP8, F32 = TYPE == PAGED_FP32;
  static constexpr int BLOCKS = T::BLOCKS, E = T::E, KEYS = 16 * BLOCKS, NF = D / 16, ROWS = 16 * TILES;      // NF: products over the values
  static constexpr int KB = D * T::SIZE, VB = KB / 16;                                       // bytes of a row, and of a lane's part of a value row

  const AttnArgs& p;
  const int lane, m, g;
  int b, n, hk, head0, rows;
  static constexpr int QL = FP8 ? 2 * T::KL : T::KL;
  u32x4 q[TILES][QL];
  floatx4 o[TILES][NF];
  float mx[TILES], l[TILES];              // of queries m, 16 + m; l: over this lane's keys
  const int32_t* table;
  uint32_t row_bytes;

  __device__ __forceinline__ Walk(const AttnArgs& args) : p(args), lane(threadIdx.x & 63), m(threadIdx.x & 15), g((threadIdx.x & 63) >> 4) {
    row_bytes = (uint32_t)p.c.Hkv * KB;
  }

  __device__ __forceinline__ void begin(int seq, int unit) {
    b = seq;
    hk = unit % p.by_heads;
    const int rt = unit / p.by_heads;
    head0 = hk * p.G + rt * ROWS;
    rows = min(ROWS, p.G - rt * ROWS);
    table = p.c.table + (size_t)b * p.c.max_pages;
    // in the order of the keys' dimensions
#pragma unroll
    for (int r = 0; r < TILES; ++r) {
      const char* qrow = p.q + (long long)b * p.q_stride + (size_t)(head0 + min(16 * r + m, rows - 1)) * (D * sizeof(Row));
#pragma unroll
      for (int j = 0; j < QL; ++j) {
        const int at = FP8 ? 64 * (j >> 1) + 16 * g + 8 * (j & 1) : F32 ? 16 * j + 4 * g : 32 * j + 8 * g;
        q[r][j] = *(const u32x4*)(qrow + at * sizeof(Row));
        if (16 * r + m >= rows) q[r][j] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < NF; ++i) o[r][i] = floatx4{0.f, 0.f, 0.f, 0.f};
      mx[r] = -FLT_MAX;
      l[r] = 0.f;
    }
  }

  // ---- where a tile's rows lie.  BLOCKED: the slots of the first keys of its blocks (uniform); else the slot of one key in every lane.
  struct Place { int slot[BLOCKED ? BLOCKS : 1]; };
  struct Entry { int page[BLOCKED ? BLOCKS : 1]; };
  // Keys behind a sequence's end are looked up like any other: in the table's bounds, on a page within the pool, and never counted.  So the first tile is
  // asked for before the length is known.
  __device__ __forceinline__ int clamped(int key) const { return min(key, p.c.tokens - 1); }
  __device__ __forceinline__ int lane_key(int tile) const {         // the key that this lane looks up
    const int e = m % E;
    return clamped(tile * KEYS + 16 * (e >> 2) + 4 * g + (e & 3));
  }
  __device__ __forceinline__ Entry entry_of(int tile) const {
    Entry x;
    if constexpr (BLOCKED) {
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i)
        x.page[i] = ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)table)[clamped(tile * KEYS + 16 * i) / p.c.page];
    } else {
      x.page[0] = table[lane_key(tile) / p.c.page];
    }
    return x;
  }
  __device__ __forceinline__ Place place_of(int tile, const Entry& x) const {
    Place s;
    if constexpr (BLOCKED) {
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i)
        s.slot[i] = min(max(x.page[i], 0), p.c.n_pages - 1) * p.c.page.d + (clamped(tile * KEYS + 16 * i) & ~15) % p.c.page;
    } else {
      s.slot[0] = min(max(x.page[0], 0), p.c.n_pages - 1) * p.c.page.d + lane_key(tile) % p.c.page;
    }
    return s;
  }

  // ---- loads
  __device__ __forceinline__ int from_lane(int block) const { return 4 * (16 * (m >> 2) + (m & 3) + 4 * block); }     // of the lane that has key m of a block, in bytes
  __device__ __forceinline__ uint32_t load_exps(const Place& s) const {      // lane (g, m): of key (g, m % 8), its key row's (m < 8) or value row's
    if constexpr (!FP8) return 0;
    const uint8_t* x = (m < 8 ? p.c.k_exp : p.c.v_exp) + hk;
    if constexpr (BLOCKED) {
      const int s0 = s.slot[0], s1 = s.slot[BLOCKS - 1];
      const uint32_t slot = (uint32_t)(m & 4 ? s1 : s0) + (uint32_t)(4 * g + (m & 3));
      return x[(uint64_t)slot * (uint32_t)p.c.Hkv];
    } else {
      return x[(uint64_t)(uint32_t)s.slot[0] * (uint32_t)p.c.Hkv];
    }
  }
  __device__ __forceinline__ void load_k(T& t, const Place& s) const {
    const uint32_t at = BLOCKED ? in_place((uint32_t)m * row_bytes + 16 * g) : 0;
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      GlobalBytes row;
      if constexpr (BLOCKED) row = uniform(p.c.k + (uint64_t)(uint32_t)s.slot[i] * row_bytes + (size_t)hk * KB) + at;
      else row = (GlobalBytes)(uintptr_t)(p.c.k + (size_t)hk * KB + 16 * g + (uint64_t)(uint32_t)__builtin_amdgcn_ds_bpermute(from_lane(i), s.slot[0]) * row_bytes);
#pragma unroll
      for (int j = 0; j < T::KL; ++j) t.k[i][j] = load_at<u32x4>(row + 64 * j);
    }
  }
  __device__ __forceinline__ void load_v(T& t, const Place& s) const {
    const uint32_t at = BLOCKED ? in_place(4 * (uint32_t)g * row_bytes + m * VB) : 0;
    static_for<0, E>([&](auto e) {
      GlobalBytes row;
      if constexpr (BLOCKED)
        row = uniform(p.c.v + (uint64_t)((uint32_t)s.slot[e / 4] + e % 4) * row_bytes + (size_t)hk * KB) + at;
      else row = (GlobalBytes)(uintptr_t)(p.c.v + (size_t)hk * KB + m * VB + (uint64_t)bcast16<e>((uint32_t)s.slot[0]) * row_bytes);
      if constexpr (T::VD == 1) t.v[e][0] = load_at<uint32_t>(row);
      else if constexpr (T::VD == 2) *(u32x2*)t.v[e] = load_at<u32x2>(row);
      else
#pragma unroll
        for (int j = 0; j < T::VD; j += 4) *(u32x4*)(t.v[e] + j) = load_at<u32x4>(row + 4 * j);
    });
  }

  // ---- products
  template <typename F> __device__ __forceinline__ void work(T& t, int tile, F&& keys_are_used) {
#pragma clang fp contract(off)            // a score and the maximum that it may be have to be the same number, however large
    float x[TILES][E];                    // scores of keys (g, e), e = 4 block + i
    float kscale[BLOCKS];
    if constexpr (FP8)
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) kscale[i] = exp_scale((uint32_t)__builtin_amdgcn_ds_bpermute(from_lane(i), (int)t.exps));
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      // fp32: four sums of a quarter of the products each, for shorter chains of roundings and of instructions
      constexpr int SUMS = F32 ? 4 : 1;
      floatx4 s[TILES][SUMS];
#pragma unroll
      for (int r = 0; r < TILES; ++r)
#pragma unroll
        for (int h = 0; h < SUMS; ++h) s[r][h] = floatx4{0.f, 0.f, 0.f, 0.f};
      auto product = [&](const u32x4& a, int j) {
#pragma unroll
        for (int r = 0; r < TILES; ++r) s[r][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, q[r][j]), s[r][0], 0, 0, 0);
      };
#pragma unroll
      for (int j = 0; j < T::KL; ++j) {
        if constexpr (F32) {
#pragma unroll
          for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int r = 0; r < TILES; ++r)
              s[r][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.k[i][j][h]), __uint_as_float(q[r][j][h]), s[r][h], 0, 0, 0);
        } else if constexpr (FP8) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t w0 = t.k[i][j][2 * h], w1 = t.k[i][j][2 * h + 1];
            product(u32x4{bf16_of_codes<false>(w0, kscale[i]), bf16_of_codes<true>(w0, kscale[i]), bf16_of_codes<false>(w1, kscale[i]),
                          bf16_of_codes<true>(w1, kscale[i])}, 2 * j + h);
          }
        } else {
          product(t.k[i][j], j);
        }
      }
#pragma unroll
      for (int r = 0; r < TILES; ++r) {
        if constexpr (F32) s[r][0] = (s[r][0] + s[r][1]) + (s[r][2] + s[r][3]);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[r][4 * i + c] = s[r][0][c] * p.scale_log2;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    keys_are_used();
    __builtin_amdgcn_sched_barrier(0);
    const int left = n - tile * KEYS;     // keys of this tile; uniform
    if (left < KEYS) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool seen = 16 * (e >> 2) + 4 * g + (e & 3) < left;
#pragma unroll
        for (int r = 0; r < TILES; ++r)
          if (!seen) x[r][e] = -__builtin_huge_valf();
#pragma unroll
        for (int j = 0; j < T::VD; ++j) t.v[e][j] = seen ? t.v[e][j] : 0u;          // a weight of zero does not silence an infinity
      }
      if (16 * (m >> 2 & 1) + 4 * g + (m & 3) >= left) t.exps = 127;                // nor what lies in the place of an exponent
    }
    u32x4 part[TILES][PARTS];
    float w[TILES][E];
#pragma unroll
    for (int r = 0; r < TILES; ++r) {
      float top = x[r][0];
#pragma unroll
      for (int e = 1; e < E; ++e) top = fmaxf(top, x[r][e]);
      top = xlane_max_step<5>(xlane_max_step<4>(top));
      if (__any(top > mx[r] + SLACK)) {
        const float to = fmaxf(mx[r], top), a = exp2_fast(mx[r] - to);
        mx[r] = to;
        l[r] *= a;
#pragma unroll
        for (int i = 0; i < NF; ++i) o[r][i] *= a;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        w[r][e] = exp2_fast(x[r][e] - mx[r]);
        l[r] += w[r][e];
      }
      if constexpr (FP8) static_for<0, E>([&](auto e) { w[r][e] *= exp_scale(bcast16<8 + e>(t.exps)); });
      // a weight as three bf16 terms of 8 bits each, all 24 of it.  With two, outputs were off by 3e-6 of their norm before they are rounded to bf16, and the difference of
      // two equal weights by 2e-5 of them; with three 4e-7 and 1e-6, as any sum in 32 bits, in the same time where keys come from memory (the cases above: 63.9 / 64.0, 39.5 / 39.5, 56.6 / 56.8 us; 8 bits of 64
      // dimensions 26.4 / 27.8, 32 heads over one, 100 sequences of 300..700 in 8 bits 12.8 / 13.6).
      // What is left behind a term is kept above zero, by 2^-24 of the term, so that an infinity times it stays one.
      if constexpr (!F32)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float a = w[r][2 * j], b = w[r][2 * j + 1];
#pragma unroll
          for (int c = 0; c + 1 < PARTS; ++c) {
            const uint32_t wa = __float_as_uint(a), wb = __float_as_uint(b);
            part[r][c][j] = __builtin_amdgcn_perm(wb, wa, 0x07060302u);
            a = fmaf(__uint_as_float(wa & 0xFFFF0000u), -0x1.fffffep-1f, a);
            b = fmaf(__uint_as_float(wb & 0xFFFF0000u), -0x1.fffffep-1f, b);
          }
          part[r][PARTS - 1][j] = pack_bf16x2(a, b);
        }
    }
    auto product = [&](int i, const u32x4& a) {
#pragma unroll
      for (int r = 0; r < TILES; ++r)
#pragma unroll
        for (int c = 0; c < PARTS; ++c)
          o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, part[r][c]), o[r][i], 0, 0, 0);
    };
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
          for (int r = 0; r < TILES; ++r) o[r][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[e][i]), w[r][e], o[r][i], 0, 0, 0);
    } else if constexpr (FP8) {
#pragma unroll
      for (int c = 0; c < T::VD; ++c)                        // four dimensions of a dword
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

  // Tiles first, first + STEP, ... below last, of a sequence of len keys.  A tile's keys are asked for as soon as those of the one before are multiplied,
  // its values likewise, and its table entries one tile earlier; ask() begins.
  T t;
  Entry next;
  template <int STEP> __device__ __forceinline__ void ask(int first) {
    const Place s = place_of(first, entry_of(first));
    next = entry_of(first + STEP);
    t.exps = load_exps(s);
    load_k(t, s);
    load_v(t, s);
  }
  template <int STEP> __device__ __forceinline__ void tiles(int first, int last, int len) {
    n = len;
    if (first >= last) return;
    int i = first;
    for (; i + STEP < last; i += STEP) {
      const Place s = place_of(i + STEP, next);
      next = entry_of(i + 2 * STEP);
      uint32_t exps;
      work(t, i, [&] {
        exps = load_exps(s);
        load_k(t, s);
      });
      load_v(t, s);
      t.exps = exps;
    }
    work(t, i, [] {});
#pragma unroll
    for (int r = 0; r < TILES; ++r) l[r] = xlane_sum_step<5>(xlane_sum_step<4>(l[r]));
  }

  // f(query, tile, first of four dimensions, their sums): of query m of a tile this lane has the dimensions NF * (4 g + c) + i
  template <typename F> __device__ __forceinline__ void each4(F&& f) const {
#pragma unroll
    for (int r = 0; r < TILES; ++r)
      if (16 * r + m < rows)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < NF; i += 4) f(16 * r + m, r, NF * (4 * g + c) + i, floatx4{o[r][i][c], o[r][i + 1][c], o[r][i + 2][c], o[r][i + 3][c]});
  }
};

template <bool F32> __device__ __forceinline__ void store_out(const AttnArgs& p, size_t at, const floatx4& v) {
  if constexpr (F32) *(floatx4*)((float*)p.out + at) = v;
  else store4_plain((bf16_t*)p.out, at, v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ float lse_of(float mx, float l) { return (mx + log2f(l)) * 0.69314718055994531f; }
__device__ __forceinline__ int length_of(const AttnArgs& p, int b) { return min(max(p.kv_len[b], 0), p.max_len); }

// The results of a workgroup's wavefronts, joined: f(row, first of four dimensions, their sums, maximum, sum of weights).
template <typename W, int D, typename F>
__device__ __forceinline__ void join_team(const W& w, int wave, int active, F&& f) {
  __shared__ __attribute__((aligned(16))) float so[WAVES][W::ROWS][D + 4], sml[WAVES][W::ROWS][2];
  if (wave < active)
    w.each4([&](int row, int r, int d, const floatx4& v) {
      *(floatx4*)&so[wave][row][d] = v;
      if (d == 0) { sml[wave][row][0] = w.mx[r]; sml[wave][row][1] = w.l[r]; }
    });
  __syncthreads();
  for (int u = threadIdx.x; u < w.rows * (D / 4); u += 64 * WAVES) {
    const int row = u / (D / 4), d = u % (D / 4) * 4;
    float M = -FLT_MAX, L = 0.f;
    for (int i = 0; i < active; ++i) M = fmaxf(M, sml[i][row][0]);
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < active; ++i) {
      const float a = exp2_fast(sml[i][row][0] - M);
      L += a * sml[i][row][1];
      sum += a * *(const floatx4*)&so[i][row][d];
    }
    f(row, d, sum, M, L);
  }
}

template <int D>
__device__ __forceinline__ void store_part(const AttnArgs& p, int range, int b, int h, int d, const floatx4& sum, float M, float L) {
  const size_t part = (size_t)(range + b) * p.H + h;
  *(floatx4*)(p.part_o + part * D + d) = sum;
  if (d == 0) *(float2*)(p.part_ml + part * 2) = make_float2(M, L);
}
template <bool F32, int D>
__device__ __forceinline__ void store_result(const AttnArgs& p, int b, int h, int d, const floatx4& sum, float M, float L) {
  const size_t bh = (size_t)b * p.H + h;
  store_out<F32>(p, bh * D + d, sum / L);
  if (d == 0 && p.lse != nullptr) p.lse[bh] = lse_of(M, L);
}
template <bool F32, int D>
__device__ __forceinline__ void store_nothing(const AttnArgs& p, int b, int h, int d) {            // of a sequence without a token
  const size_t bh = (size_t)b * p.H + h;
  store_out<F32>(p, bh * D + d, floatx4{0.f, 0.f, 0.f, 0.f});
  if (d == 0 && p.lse != nullptr) p.lse[bh] = -__builtin_huge_valf();
}

// The sequence in place `at` when of every 64, those behind the last whole 64 before the others, the longest comes first: every lane counts the longer ones for its
// sequence, a wavefront an eighth of them.
__device__ __forceinline__ int longest_first(const AttnArgs& p, int wave, int at) {
  __shared__ int ranks[WAVES][64];
  const int lane = threadIdx.x & 63, rest = p.B & 63, b0 = at < rest ? p.B - rest : (at - rest) & ~63, place = at < rest ? at : (at - rest) & 63;
  const long long key = b0 + lane < p.B ? (long long)length_of(p, b0 + lane) * 64 + 63 - lane : -1ll - lane;
  const int hi = (int)(key >> 32), lo = (int)key;
  int rank = 0;
#pragma unroll
  for (int j = 0; j < 64 / WAVES; ++j) {
    const long long other = (long long)__builtin_amdgcn_readlane(hi, wave * (64 / WAVES) + j) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, wave * (64 / WAVES) + j);
    rank += other > key ? 1 : 0;
  }
  ranks[wave][lane] = rank;
  __syncthreads();
  rank = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) rank += ranks[i][lane];
  return b0 + __builtin_ctzll(__ballot(rank == place));
}

// Short contexts, or very many: a workgroup per sequence and unit; one launch.  Where there are more workgroups than CUs, those of long sequences
// begin first: 64 of 512..2048 tokens, 32 heads over 8, bf16 76.6 -> 65.2 us.
template <int TYPE, int D, bool BLOCKED, int TILES>
__global__ __launch_bounds__(64 * WAVES) void paged_whole_kernel(const int32_t* kv_len, const int32_t* table, int B, int max_len, int max_pages, int tokens, Divisor page,
                                                             int n_pages, AttnArgs p) {
  p.kv_len = kv_len, p.B = B, p.max_len = max_len, p.c.table = table, p.c.max_pages = max_pages, p.c.tokens = tokens, p.c.page = page, p.c.n_pages = n_pages;
  typedef Walk<TYPE, D, BLOCKED, TILES> W;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = p.B > 1 && (long long)p.B * p.units > 256 ? longest_first(p, wave, blockIdx.y) : (int)blockIdx.y;
  W w(p);
  w.begin(b, blockIdx.x);
  w.template ask<WAVES>(wave);
  const int n = length_of(p, b), n_tiles = (n + W::KEYS - 1) / W::KEYS;
  w.template tiles<WAVES>(wave, n_tiles, n);
  join_team<W, D>(w, wave, min(n_tiles, WAVES), [&](int row, int d, const floatx4& sum, float M, float L) {
    if (n > 0) store_result<W::F32, D>(p, b, w.head0 + row, d, sum, M, L);
    else store_nothing<W::F32, D>(p, b, w.head0 + row, d);
  });
}

// Tiles of the sequences b0 .. b0 + 63, up to and with this lane's.
template <int KEYS> __device__ __forceinline__ int scan_tiles(const AttnArgs& p, int b0) {
  const int lane = threadIdx.x & 63;
  int v = b0 + lane < p.B ? (length_of(p, b0 + lane) + KEYS - 1) / KEYS : 0;
  // within 16 lanes from 1, 2, 4, 8 lanes below, then the sums of the 16 and 32 lanes before
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}
// Longer contexts: all sequences' tiles in equal ranges; the parts of sequences that do not lie within one range are joined by the next kernel.
// TEAM: a workgroup has a range of one unit.  Else a wavefront has, and the wavefronts of a workgroup have the units of one range after the other, so that together
// they read whole rows.
template <int TYPE, int D, bool BLOCKED, int TILES, bool TEAM>
__global__ __launch_bounds__(64 * WAVES) void paged_ranges_kernel(const int32_t* kv_len, int B, int max_len, int ranges, Divisor by_units, AttnArgs p) {
  p.kv_len = kv_len, p.B = B, p.max_len = max_len, p.ranges = ranges, p.by_units = by_units;
  typedef Walk<TYPE, D, BLOCKED, TILES> W;
  constexpr int STEP = TEAM ? WAVES : 1;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = TEAM ? blockIdx.x : (int)blockIdx.x * WAVES + wave;
  const int range = at / p.by_units, unit = at % p.by_units, offset = TEAM ? wave : 0;
  if (range >= p.ranges) return;
  int scanned = scan_tiles<W::KEYS>(p, 0), total = __builtin_amdgcn_readlane(scanned, 63), b0 = 0;
  for (int c = 64; c < p.B; c += 64) total += __builtin_amdgcn_readlane(scan_tiles<W::KEYS>(p, c), 63);
  const int per = paged_tiles_of_range(total, p.ranges);
  int x = range * per;                    // next tile, counted over all sequences
  const int last = min(total, x + per);
  W w(p);
  while (x < last) {
    for (int end; x >= (end = __builtin_amdgcn_readlane(scanned, 63));) scanned = end + scan_tiles<W::KEYS>(p, b0 += 64);
    const int i = __builtin_ctzll(__ballot(scanned > x));    // the first sequence of these 64 that ends behind x
    const int b = b0 + i, n = length_of(p, b), n_tiles = (n + W::KEYS - 1) / W::KEYS, ends = __builtin_amdgcn_readlane(scanned, i), starts = ends - n_tiles;
    const int stop = min(ends, last), first = x - starts + offset, behind = stop - starts;
    const bool whole = x == starts && stop == ends;
    w.begin(b, unit);
    if (first < behind) {
      w.template ask<STEP>(first);
      w.template tiles<STEP>(first, behind, n);
    }
    if constexpr (TEAM) {
      join_team<W, D>(w, wave, min(stop - x, WAVES), [&](int row, int d, const floatx4& sum, float M, float L) {
        if (whole) store_result<W::F32, D>(p, b, w.head0 + row, d, sum, M, L);
        else store_part<D>(p, range, b, w.head0 + row, d, sum, M, L);
      });
      if (stop < last) __syncthreads();
    } else if (whole) {
      w.each4([&](int row, int r, int d, const floatx4& v) { store_result<W::F32, D>(p, b, w.head0 + row, d, v, w.mx[r], w.l[r]); });
    } else {
      w.each4([&](int row, int r, int d, const floatx4& v) { store_part<D>(p, range, b, w.head0 + row, d, v, w.mx[r], w.l[r]); });
    }
    x = stop;
  }
}

// What is joined: a maximum, a sum of weights and four sums of values.
struct Joint {
  float M, L;
  floatx4 sum;
  __device__ __forceinline__ void add(float m, float l, const floatx4& v) {
    const float to = fmaxf(M, m), a = exp2_fast(M - to), c = exp2_fast(m - to);
    M = to;
    L = L * a + l * c;
    sum = sum * a + v * c;
  }
};

// The parts of a (sequence, query head), and the sequences without a token.  DL lanes have DL * 4 dimensions of a part, a head's WAVES_PER wavefronts as many
// parts at a time as they have such groups, four of them in flight; groups are joined by exchanges within a wavefront, then through LDS.
// Few parts: a wavefront to a head with all its dimensions.  Many (131072 tokens under 64 heads: 256 parts): eight, with 32 dimensions, 8.1 -> 5.8 us.
template <int KEYS, bool F32, int D, int DL, int WAVES_PER>
__global__ __launch_bounds__(512) void paged_join_kernel(const int32_t* kv_len, int B, int max_len, int ranges, int H, float* part_ml, float* part_o, AttnArgs p) {
  p.kv_len = kv_len, p.B = B, p.max_len = max_len, p.ranges = ranges, p.H = H, p.part_ml = part_ml, p.part_o = part_o;
  constexpr int PER = 64 * WAVES_PER / DL, HEADS = 8 / WAVES_PER;
  __shared__ __attribute__((aligned(16))) float so[8][4 * DL], sml[8][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.x * HEADS + wave / WAVES_PER, b = blockIdx.y, n = length_of(p, b);
  const int at = threadIdx.x % (64 * WAVES_PER) / DL, d = blockIdx.z * (4 * DL) + lane % DL * 4;
  int total = 0, ends = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int scanned = scan_tiles<KEYS>(p, b0);
    if (b >= b0 && b < b0 + 64) ends = total + __builtin_amdgcn_readlane(scanned, b - b0);
    total += __builtin_amdgcn_readlane(scanned, 63);
  }
  if (n == 0) {
    if (at == 0 && h < p.H) store_nothing<F32, D>(p, b, h, d);
    return;
  }
  const int per = paged_tiles_of_range(total, p.ranges), starts = ends - (n + KEYS - 1) / KEYS;
  const int first = paged_first_range(starts, per), parts = paged_last_range(ends, per) - first + 1;
  if (parts <= 1) return;
  const size_t part0 = (size_t)(first + b) * p.H + min(h, p.H - 1);
  Joint j = {-FLT_MAX, 0.f, {0.f, 0.f, 0.f, 0.f}};
  for (int i0 = at; i0 < parts; i0 += 4 * PER) {
    float2 ml[4];
    floatx4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const size_t part = part0 + (size_t)min(i0 + i * PER, parts - 1) * p.H;
      ml[i] = *(const float2*)(p.part_ml + part * 2);
      v[i] = *(const floatx4*)(p.part_o + part * D + d);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i0 + i * PER < parts) j.add(ml[i].x, ml[i].y, v[i]);
  }
#pragma unroll
  for (int o = DL; o < 64; o *= 2) {
    const float m = __shfl_xor(j.M, o, 64), l = __shfl_xor(j.L, o, 64);
    j.add(m, l, floatx4{__shfl_xor(j.sum[0], o, 64), __shfl_xor(j.sum[1], o, 64), __shfl_xor(j.sum[2], o, 64), __shfl_xor(j.sum[3], o, 64)});
  }
  if constexpr (WAVES_PER > 1) {
    if (lane < DL) {
      *(floatx4*)&so[wave][4 * lane] = j.sum;
      if (lane == 0) { sml[wave][0] = j.M; sml[wave][1] = j.L; }
    }
    __syncthreads();
    if (threadIdx.x >= DL) return;
    for (int i = 1; i < WAVES_PER; ++i) j.add(sml[i][0], sml[i][1], *(const floatx4*)&so[i][4 * lane]);
  }
  if (lane < DL && h < p.H) store_result<F32, D>(p, b, h, d, j.sum, j.M, j.L);
}

template <int TYPE, int D, bool BLOCKED, int TILES>
hipError_t launch(const AttnArgs& a, const PagedSplit& s, hipStream_t st) {
  constexpr int KEYS = 16 * CacheType<TYPE>::BLOCKS;
  constexpr bool F32 = TYPE == PAGED_FP32;
  const dim3 team(64 * WAVES);
  if (s.ranges == 0) {
    hipLaunchKernelGGL((paged_whole_kernel<TYPE, D, BLOCKED, TILES>), dim3(a.units, a.B), team, 0, st, a.kv_len, a.c.table, a.B, a.max_len, a.c.max_pages, a.c.tokens,
                       a.c.page, a.c.n_pages, a);
    return hipGetLastError();
  }
  auto ranges = [&](auto kernel, int workgroups) { hipLaunchKernelGGL(kernel, dim3(workgroups), team, 0, st, a.kv_len, a.B, a.max_len, a.ranges, a.by_units, a); };
  auto join = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(512), 0, st, a.kv_len, a.B, a.max_len, a.ranges, a.H, a.part_ml, a.part_o, a); };
  const int n = s.ranges * a.units;
  if (s.team) ranges(paged_ranges_kernel<TYPE, D, BLOCKED, TILES, true>, n);
  else ranges(paged_ranges_kernel<TYPE, D, BLOCKED, TILES, false>, (n + WAVES - 1) / WAVES);
  if (s.ranges / a.B > 16) join(paged_join_kernel<KEYS, F32, D, 8, 8>, dim3(a.H, a.B, D / 32));
  else join(paged_join_kernel<KEYS, F32, D, D / 4, 1>, dim3((a.H + 7) / 8, a.B));
  return hipGetLastError();
}
// Pages of whole blocks of 16 keys against any others, the sizes above: 64.7 against 67.1 us (pages of 16, of 100 tokens), 8 bits 42.9 against 43.7, fp32 (16 sequences of
// 1000..2048) 42.7 against 45.5.
template <int TYPE, int D>
hipError_t launch(const AttnArgs& a, const PagedSplit& s, hipStream_t st) {
  if constexpr (TYPE != PAGED_FP32)
    if (s.rows == 32) return a.c.page.d % 16 == 0 ? launch<TYPE, D, true, 2>(a, s, st) : launch<TYPE, D, false, 2>(a, s, st);
  return a.c.page.d % 16 == 0 ? launch<TYPE, D, true, 1>(a, s, st) : launch<TYPE, D, false, 1>(a, s, st);
}

PagedSplit split_of(const PagedView& c, int dtype, int B, int H, int max_len) {
  return paged_split(B, H, c.Hkv, c.d * (dtype == PAGED_FP32 ? 4 : dtype == PAGED_BF16 ? 2 : 1), dtype == PAGED_FP32, max_len);
}

}  // namespace

size_t paged_attention_workspace(const PagedView& c, int dtype, int B, int H, int max_len) {
  return paged_partial_floats(B, H, c.d, split_of(c, dtype, B, H, max_len).ranges) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedView& c, int dtype, int B, int H, const void* q, long long q_bytes, const int32_t* kv_len, int max_len,
                                  float scale, void* out, float* lse, void* workspace, hipStream_t st) {
  const PagedSplit s = split_of(c, dtype, B, H, max_len);
  float* part_o = (float*)workspace;
  const AttnArgs a = {c, (const char*)q, q_bytes, kv_len, max_len, H, H / c.Hkv, B, s.units, s.ranges, divisor(s.units), divisor(c.Hkv),
                      scale * 1.4426950408889634f, out, lse, part_o, part_o ? part_o + (size_t)(s.ranges + B) * H * c.d : nullptr};
  if (dtype == PAGED_FP8) return c.d == 128 ? launch<PAGED_FP8, 128>(a, s, st) : launch<PAGED_FP8, 64>(a, s, st);
  if (dtype == PAGED_BF16) return c.d == 128 ? launch<PAGED_BF16, 128>(a, s, st) : launch<PAGED_BF16, 64>(a, s, st);
  return c.d == 128 ? launch<PAGED_FP32, 128>(a, s, st) : launch<PAGED_FP32, 64>(a, s, st);
}
