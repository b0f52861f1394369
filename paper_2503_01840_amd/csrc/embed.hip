// Rows of an embedding table, and the table's gradient.
//
// Rows: a wavefront takes a row or a part of it, the token once for all its lanes, 16 bytes to a lane and load, four of them on their way at a time.  Bound by bytes: 16384 rows of 8192 in
// bf16 77 us (268 MB written, 165 read); 60 rows of 4096 onto fp32 2.4, an empty launch's time.
//
// Gradient: the rows' tokens are sorted first, so that a token's rows are neighbours and their sum has an order of its own: up to 12288 rows by counting smaller ones in one launch, beyond by
// digits of at most 9 bits in two launches each.  Workgroups behind those that sort write zeros to the table meanwhile.  Then CHUNK sorted places at a time are summed by a wavefront for 64
// pieces of columns, all CHUNK rows on their way at once; a token's sum that lies within them is written at once, the ends of one that does not go to the workspace and are added by the
// last launch; few rows are summed in one launch, token by token.  Bound by bytes, of which a large table's zeros are nearly all: 8192 rows of 4096 into 128256 in bf16 158 us for tokens and zeros (1051 MB, 6.7 TB/s), 17 and 6 for the sums;
// 1021 fp32 rows of 251 into 2048 6.3, 7.9 and 3.6, three launches that wait for memory.  Added to a table that is there: 8192 rows of 4096 47 us, where the sort has no zeros above it, 16384 rows 79,
// of 256 columns 35, of which sorting by two digits is 23 (counts 3.0 each, places 8.6).
// Measured and not kept: one launch without sorted tokens for up to 1024 rows, each workgroup looking through all tokens for its part of the table (1021 rows of 251: 16.8 -> 15.4 us, but
// 33 where half of the rows have one token, 61 where all have; tables of 1 GB 168 -> 171); zeros by the launch that sums; a token's rows 8 or 32 at a time.
#include <algorithm>

#include "elements.hpp"
#include "kernels.hpp"

namespace {

// Bytes of a result from which it is stored past the caches, which it would fill: 16384 rows of 4096 in fp32 (256 MiB) 76 -> 51 us, with an addition behind them that reads them
// 176 -> 169; 64 MiB in bf16 20 -> 17, but with the addition 41 -> 43.
constexpr size_t STREAMED = (size_t)128 << 20;

// ---------------------------------------------------------------- rows
template <typename T, typename O, bool ODD, bool STREAM>
__global__ __launch_bounds__(256) void embed_kernel(const int32_t* tokens, const T* table, int rows, int dim, int vocab, float scale, O* out, long long stride, int share) {
  constexpr int N = sizeof(T) + sizeof(O) == 4 ? 8 : 4, U = 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = blockIdx.x * 4 + wave;
  if (r >= rows) return;
  const int token = tokens[r], first = blockIdx.y * share, last = min(pieces_of(dim, N), first + share);
  const bool seen = token >= 0 && token < vocab;
  const T* from = table + (size_t)(seen ? token : 0) * dim;
  O* to = out + (size_t)r * stride;
  for (int p0 = first; p0 < last; p0 += 64 * U) {
    Piece<T, N> e[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int p = p0 + 64 * j + lane;
      if (seen && p < last) e[j].template load<ODD>(from + (size_t)p * N, dim - p * N, dim);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int p = p0 + 64 * j + lane;
      if (p < last) {
        float f[N];
        e[j].template settle<ODD>(dim - p * N, dim);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = seen ? scale * e[j].at(i) : 0.f;
        store_piece<N, ODD, STREAM>(to + (size_t)p * N, f, dim - p * N);
      }
    }
  }
}

// Pieces to a wavefront: 64 where rows are few, up to 256 where they are many (us; by 64 in any case, by 256 in any case: 60 rows of 4096 onto fp32 2.5, 2.9; 1000 rows 7.0, 6.7, by
// this rule 5.8; 16384 rows 82, 74).
template <typename T, typename O, bool ODD, bool STREAM>
hipError_t rows_of(const EmbedRows& a, hipStream_t st) {
  constexpr int N = sizeof(T) + sizeof(O) == 4 ? 8 : 4;
  const int pieces = pieces_of(a.dim, N), most = (pieces + 63) / 64, want = std::max(1, std::min(most, 8192 / a.rows));
  const int share = 64 * std::min(4, (most + want - 1) / want);
  const dim3 grid((a.rows + 3) / 4, (pieces + share - 1) / share);
  hipLaunchKernelGGL((embed_kernel<T, O, ODD, STREAM>), grid, dim3(256), 0, st, a.tokens, (const T*)a.table, a.rows, a.dim, a.vocab, a.scale, (O*)a.out, a.stride, share);
  return hipGetLastError();
}

// ---------------------------------------------------------------- zeros
// The workgroups behind the first `sorting` ones of every launch that sorts write zeros to the table's blocks from first_block on: sorting keeps few of the chip's
// units busy.  A table's bytes are pieces of 16 from its first multiple of 16 on, a block's 1024 of them, one to a thread, and less than 16 bytes in front and behind.
// Workgroups go to the XCDs in turn; each XCD has an eighth of a launch's blocks one behind the other (6.9 TB/s; blocks in turn 6.1, 8192 pieces to a block 5.6).
constexpr int FILL_PIECES = 1024;
struct Fill {
  char* table;
  size_t bytes;
  int sorting, first_block, blocks;                           // of this launch: blocks a multiple of 8
};
__device__ __forceinline__ void fill(const Fill& f) {
  const int head = (int)min(f.bytes, (size_t)(-(uintptr_t)f.table & 15)), b = blockIdx.x - f.sorting;
  const size_t pieces = (f.bytes - head) / 16, block = (size_t)f.first_block + (b & 7) * (f.blocks >> 3) + (b >> 3), p = block * FILL_PIECES + threadIdx.x;
  const u32x4_t zero = {0, 0, 0, 0};
  u32x4_t* body = (u32x4_t*)(f.table + head);
  if (p < pieces) __builtin_nontemporal_store(zero, body + p);
  if (block == 0) {
    const int tail = (int)(f.bytes - head - pieces * 16), i = threadIdx.x;
    if (i < head) f.table[i] = 0;
    if (i < tail) ((char*)(body + pieces))[i] = 0;
  }
}
// The share of launch number `launch` of `launches`
void share_out(Fill& f, int launch, int launches) {
  const size_t eights = f.bytes ? (f.bytes / 16 + 8 * FILL_PIECES - 1) / (8 * FILL_PIECES) + (f.bytes < 16) : 0;
  const size_t from = eights * launch / launches, to = eights * (launch + 1) / launches;
  f.first_block = (int)(8 * from);
  f.blocks = (int)(8 * (to - from));
}

// ---------------------------------------------------------------- tokens in order
// A tile of 4096 places to a workgroup of 16 wavefronts: wavefront w has places 256 w + 64 r + lane, r < 4, so that the order of places is that of (w, r, lane).
constexpr int TILE = 4096, DIGITS = 512;

__device__ __forceinline__ uint32_t key_of(const int32_t* tokens, int i, int n, int vocab) {
  if (i >= n) return 0xFFFFFFFFu;                             // behind everything
  const int t = tokens[i];
  return t >= 0 && t < vocab ? (uint32_t)t : (uint32_t)vocab; // padding behind the vocabulary
}

// The place that each of a tile's keys takes by one digit, in order among equal ones, from base[digit] on.
__device__ __forceinline__ void ranks(const uint32_t* key, int shift, int bits, uint16_t (*count)[DIGITS], const uint32_t* base, int* to) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const uint32_t mask = (1u << bits) - 1;
  for (int i = threadIdx.x; i < 16 * DIGITS; i += 1024) count[i / DIGITS][i % DIGITS] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint32_t d = (key[r] >> shift) & mask;
    uint64_t same = ~0ull;
    for (int b = 0; b < bits; ++b) {
      const bool one = (d >> b) & 1;
      const uint64_t vote = __ballot(one);
      same &= one ? vote : ~vote;
    }
    const int before = __popcll(same & ((1ull << lane) - 1)), so_far = count[wave][d];
    to[r] = so_far + before;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // every lane has read its count
    __builtin_amdgcn_wave_barrier();
    if (before == 0) count[wave][d] = (uint16_t)(so_far + __popcll(same));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  if (threadIdx.x < DIGITS) {                                 // counts of the wavefronts before
    uint32_t total = 0;
    for (int w = 0; w < 16; ++w) {
      const uint32_t c = count[w][threadIdx.x];
      count[w][threadIdx.x] = (uint16_t)total;
      total += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint32_t d = (key[r] >> shift) & mask;
    to[r] += base[d] + count[wave][d];
  }
}

// Up to RANKED places: the place of a key is the number of smaller ones and of equal ones in front of it.  A workgroup counts for 64 keys, each of its 16
// wavefronts a 16th of all others, which it has in scalar registers.  By digits, in four to six launches, us of the whole gradient of 256 columns: 2048 rows 16.8 and 24.9, 8192 26.6 and
// 31.3, 16384 44.4 and 37.0.
constexpr int RANKED = 12288;
__global__ __launch_bounds__(1024) void sort_ranks_kernel(const int32_t* __restrict__ tokens, int n, int vocab, int share, int32_t* token_out, int32_t* row_out, Fill f) {
  if ((int)blockIdx.x >= f.sorting) return fill(f);
  __shared__ int counts[16][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, i0 = blockIdx.x * 64, i = i0 + lane;
  const uint32_t key = key_of(tokens, i, n, vocab);
  const int first = min(n, wave * share), last = min(n, first + share);
  uint32_t before = 0;
  // padding has a key of its own behind the others; as an unsigned number it is at least that
  auto count = [&](int from, int to, uint32_t below) {
    int j = from;
    for (; j + 16 <= to; j += 16) {
#pragma unroll
      for (int u = 0; u < 16; ++u) before += min((uint32_t)tokens[j + u], (uint32_t)vocab) < below;
    }
    for (; j < to; ++j) before += min((uint32_t)tokens[j], (uint32_t)vocab) < below;
  };
  count(first, min(last, i0), key + 1);
  for (int j = max(first, i0); j < min(last, i0 + 64); ++j) before += min((uint32_t)tokens[j], (uint32_t)vocab) < (j < i ? key + 1 : key);
  count(max(first, i0 + 64), last, key);
  counts[wave][lane] = (int)before;
  __syncthreads();
  if (threadIdx.x < 64 && i < n) {
    int at = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) at += counts[w][lane];
    token_out[at] = (int32_t)key;
    row_out[at] = i;
  }
}

// One digit of more places: a tile's counts, then each tile's places.
__global__ __launch_bounds__(1024) void sort_count_kernel(const int32_t* tokens, int n, int vocab, int shift, int bits, uint32_t* hist, Fill f) {
  if ((int)blockIdx.x >= f.sorting) return fill(f);
  __shared__ uint32_t count[DIGITS];
  if (threadIdx.x < DIGITS) count[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = blockIdx.x * TILE + r * 1024 + threadIdx.x;
    if (i < n) atomicAdd(&count[(key_of(tokens, i, n, vocab) >> shift) & ((1u << bits) - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < DIGITS) hist[(size_t)blockIdx.x * DIGITS + threadIdx.x] = count[threadIdx.x];
}
__global__ __launch_bounds__(1024) void sort_place_kernel(const int32_t* tokens, const int32_t* rows, int n, int vocab, int shift, int bits, const uint32_t* hist, int tiles,
                                                          int32_t* token_out, int32_t* row_out, Fill f) {
  if ((int)blockIdx.x >= f.sorting) return fill(f);
  __shared__ uint16_t count[16][DIGITS];
  __shared__ uint32_t base[DIGITS], wave_sums[DIGITS / 64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  uint32_t key[4];
  int row[4], to[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = blockIdx.x * TILE + 256 * wave + 64 * r + lane;
    key[r] = key_of(tokens, i, n, vocab);
    row[r] = i < n && rows ? rows[i] : i;
  }
  // base = the count of smaller digits in all tiles, and of this one in the tiles before
  uint32_t all = 0, before = 0;
  if (threadIdx.x < DIGITS) {
    const uint32_t* h = hist + threadIdx.x;
#pragma unroll 8
    for (int t = 0; t < tiles; ++t) {
      const uint32_t c = h[(size_t)t * DIGITS];
      all += c;
      before += t < (int)blockIdx.x ? c : 0;
    }
  }
  uint32_t sum = all;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t v = __shfl_up(sum, o, 64);
    if (lane >= o) sum += v;
  }
  if (lane == 63 && wave < DIGITS / 64) wave_sums[wave] = sum;
  __syncthreads();
  if (threadIdx.x < DIGITS) {
    for (int w = 0; w < wave; ++w) sum += wave_sums[w];
    base[threadIdx.x] = sum - all + before;
  }
  ranks(key, shift, bits, count, base, to);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = blockIdx.x * TILE + 256 * wave + 64 * r + lane;
    if (i < n) {                                              // those behind the end have the largest digit and are its last ones
      token_out[to[r]] = (int32_t)key[r];
      row_out[to[r]] = row[r];
    }
  }
}

// ---------------------------------------------------------------- sums
constexpr int CHUNK = 16;
__host__ __device__ __forceinline__ int padded(int dim) { return (dim + 7) & ~7; }

// A wavefront sums a chunk's rows for 64 pieces of columns.
// partial: [chunk][2][padded(dim)]: sums of a chunk's first token that began before it, and of its last one that goes on behind it.
template <typename T, typename O, bool ODD, bool ADD>
__global__ __launch_bounds__(256) void embed_sum_kernel(const int32_t* __restrict__ token, const int32_t* __restrict__ row_of, int n, int dim, int vocab, int slabs, int sums, EmbedGrad g) {
  constexpr int N = sizeof(T) + sizeof(O) == 4 ? 8 : 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int task = blockIdx.x * 4 + wave, pieces = pieces_of(dim, N);
  if (task >= sums) return;
  O* table = (O*)g.d_table;
  const int chunk = task / slabs, p = (task - chunk * slabs) * 64 + lane, first = chunk * CHUNK, count = min(n - first, CHUNK);
  // lane j has the token and row of place first + j; lane CHUNK the token before, the next one that behind, padding (vocab) where there is none
  int tokens = vocab, rows = 0;
  if (lane < count) {
    tokens = token[first + lane];
    rows = row_of[first + lane];
  } else if (lane == CHUNK && first > 0) {
    tokens = token[first - 1];
  } else if (lane == CHUNK + 1 && first + CHUNK < n) {
    tokens = token[first + CHUNK];
  }
  const bool has = p < pieces;
  int current = __builtin_amdgcn_readlane(tokens, 0);
  if (current >= vocab) return;                               // padding only
  bool began_before = __builtin_amdgcn_readlane(tokens, CHUNK) == current;
  const int left = dim - p * N;
  const T* dy = (const T*)g.dy + (size_t)p * N;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  // what is left of `current` goes to the table, or to the workspace
  auto leave = [&](bool goes_on) {
    if (!has) return;
    if (began_before || goes_on) {
      float* to = g.partial + ((size_t)chunk * 2 + (began_before ? 0 : 1)) * padded(dim) + (size_t)p * N;
#pragma unroll
      for (int i = 0; i < N; i += 4) store_piece<4, false>(to + i, sum + i, 4);
      return;
    }
    O* to = table + (size_t)current * dim + (size_t)p * N;
    float f[N];
    if constexpr (ADD) {
      Piece<O, N> old;
      old.template load<ODD>(to, left, dim);
      old.template settle<ODD>(left, dim);
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = fmaf(g.scale, sum[i], old.at(i));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = g.scale * sum[i];
    }
    store_piece<N, ODD>(to, f, left);
  };
  Piece<T, N> e[CHUNK];
#pragma unroll
  for (int j = 0; j < CHUNK; ++j)                             // places behind the last have row 0, which is not added
    if (has) e[j].template load<ODD>(dy + (size_t)__builtin_amdgcn_readlane(rows, j) * g.stride, left, dim);
#pragma unroll
  for (int j = 0; j < CHUNK; ++j) {
    const int next = __builtin_amdgcn_readlane(tokens, j);
    if (next != current) {
      leave(false);
      if (next >= vocab) return;                              // padding, or behind the last place
      current = next;
      began_before = false;
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] = 0.f;
    }
    e[j].template settle<ODD>(left, dim);
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += has ? e[j].at(i) : 0.f;
  }
  leave(__builtin_amdgcn_readlane(tokens, CHUNK + 1) == current);
}

// Tokens whose rows lie in several chunks: workgroup (chunk, 64 pieces of columns) adds the parts of the one that begins in this chunk and goes on behind it, a quarter of
// them to each wavefront.
template <typename O, bool ODD, bool ADD>
__global__ __launch_bounds__(256) void embed_join_kernel(const int32_t* __restrict__ token, int n, int dim, int vocab, EmbedGrad g) {
  constexpr int N = 4;
  __shared__ float part[4][64 * N];
  const int chunk = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, p = blockIdx.y * 64 + lane;
  const int first = chunk * CHUNK, end = first + CHUNK;
  if (end >= n) return;
  const int v = token[end - 1], before = token[max(first, 1) - 1], start = token[first], behind = token[end];
  if (v >= vocab || behind != v || (start == v && first > 0 && before == v)) return;
  int parts = 1;                                              // chunks that begin with this token follow each other
  for (;;) {
    const long long at = (long long)(chunk + parts + lane) * CHUNK;
    const uint64_t same = __ballot(at < n && token[at] == v);
    parts += __popcll(same);
    if (~same) break;
  }
  const int share = (parts + 3) / 4;
  const bool has = p < pieces_of(dim, N);
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  if (has) {
#pragma unroll 4
    for (int c = wave * share; c < min(parts, (wave + 1) * share); ++c) {
      Piece<float, N> e;
      e.template load<false>(g.partial + ((size_t)(chunk + c) * 2 + (c ? 0 : 1)) * padded(dim) + (size_t)p * N, N, N);
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += e.at(i);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) part[wave][lane * N + i] = sum[i];
  __syncthreads();
  if (wave || !has) return;
  float f[N];
  O* to = (O*)g.d_table + (size_t)v * dim + (size_t)p * N;
  Piece<O, N> old;
  if constexpr (ADD) {
    old.template load<ODD>(to, dim - p * N, dim);
    old.template settle<ODD>(dim - p * N, dim);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float s = (part[0][lane * N + i] + part[1][lane * N + i]) + (part[2][lane * N + i] + part[3][lane * N + i]);
    f[i] = ADD ? fmaf(g.scale, s, old.at(i)) : g.scale * s;
  }
  store_piece<N, ODD>(to, f, dim - p * N);
}

// Few rows: no parts and no second launch.  A workgroup has the tokens whose first place is one of CHUNK, a wavefront each; one with more than 64 rows, the last, is summed by all wavefronts, a
// 16th of its places each.  With one token in many rows a CU draws them alone, so this is for few: us, sums and parts in two launches against this, tokens of a log-uniform rank and one token
// in all rows: 300 rows of 4096 20.4 and 16.3, 19.9 and 19.3; 400 20.5 and 17.2, 20.4 and 21.0; 512 20.6 and 17.2, 21.2 and 26.8; 2048 25.5 and 28.2, 32.1 and 66.9.
// 16 registers of a thread are spilled where odd bf16 rows are added to a bf16 table.
constexpr int RUN_ROWS = 384;
template <typename T, typename O, bool ODD, bool ADD>
__global__ __launch_bounds__(1024) void embed_runs_kernel(const int32_t* __restrict__ token, const int32_t* __restrict__ row_of, int n, int dim, int vocab, EmbedGrad g) {
  constexpr int N = sizeof(T) + sizeof(O) == 4 ? 8 : 4, U = 16;
  __shared__ float part[16][64 * N];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = blockIdx.x * CHUNK, p = blockIdx.y * 64 + lane, left = dim - p * N;
  const bool has = p < pieces_of(dim, N);
  const int before = first ? token[first - 1] : -1, mine = first + lane < n ? token[first + lane] : vocab;       // padding, and what is behind the end: vocab
  const int row = first + lane < n ? row_of[first + lane] : 0;
  const int previous = __shfl_up(mine, 1, 64);
  const uint64_t ends = __ballot(mine != (lane ? previous : before));             // places where another token begins
  const uint64_t starts = __ballot(mine < vocab) & ends & ((1ull << CHUNK) - 1);
  if (!starts) return;
  const T* dy = (const T*)g.dy + (size_t)p * N;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  auto add_rows = [&](int rows, int from, int to) {           // of lanes from..to-1
    for (int l = from; l < to; l += U) {
      Piece<T, N> e[U];
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (l + j < to && has) e[j].template load<ODD>(dy + (size_t)__builtin_amdgcn_readlane(rows, l + j) * g.stride, left, dim);
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (l + j < to) {
          e[j].template settle<ODD>(left, dim);
#pragma unroll
          for (int i = 0; i < N; ++i) sum[i] += has ? e[j].at(i) : 0.f;
        }
      }
    }
  };
  auto leave = [&](int v) {
    if (!has) return;
    O* to = (O*)g.d_table + (size_t)v * dim + (size_t)p * N;
    float f[N];
    Piece<O, N> old;
    if constexpr (ADD) {
      old.template load<ODD>(to, left, dim);
      old.template settle<ODD>(left, dim);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = ADD ? fmaf(g.scale, sum[i], old.at(i)) : g.scale * sum[i];
    store_piece<N, ODD>(to, f, left);
  };
  const int last = 63 - __builtin_clzll(starts);              // the last start: its token may go on behind these 64 places
  const bool is_long = ends >> (last + 1) == 0;
  uint64_t left_starts = starts;
  for (int w = 0; w < wave && left_starts; ++w) left_starts &= left_starts - 1;
  if (left_starts) {
    const int at = __builtin_ctzll(left_starts);
    if (at != last || !is_long) {
      add_rows(row, at, at + 1 + __builtin_ctzll(ends >> (at + 1)));
      leave(__builtin_amdgcn_readlane(mine, at));
    }
  }
  if (!is_long) return;
  const int v = __builtin_amdgcn_readlane(mine, last);
  int length = 64 - last;
  for (;;) {
    const int i = first + last + length + lane;
    const uint64_t same = __ballot(i < n && token[i] == v);
    length += __popcll(same);
    if (~same) break;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  const int from = first + last + (int)((long long)length * wave / 16), to = first + last + (int)((long long)length * (wave + 1) / 16);
  for (int l = from; l < to; l += 64) {
    const int rows = l + lane < to ? row_of[l + lane] : 0;
    add_rows(rows, 0, min(64, to - l));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) part[wave][lane * N + i] = sum[i];
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sum[i] = part[0][lane * N + i];
#pragma unroll
    for (int w = 1; w < 16; ++w) sum[i] += part[w][lane * N + i];
  }
  leave(v);
}

// ---------------------------------------------------------------- the workspace: keys and rows, twice, counts, parts
size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }
int chunks_of(int rows) { return (rows + CHUNK - 1) / CHUNK; }

// Sorted tokens and their rows, in *token and *row, and zeros in the table (f.bytes > 0).
hipError_t sort_tokens(const EmbedGrad& g, Fill f, char* ws, const int32_t** token, const int32_t** row, hipStream_t st) {
  const int n = g.rows;
  const size_t array = aligned((size_t)n * sizeof(int32_t));
  int32_t* key[2] = {(int32_t*)ws, (int32_t*)(ws + array)};
  int32_t* rows[2] = {(int32_t*)(ws + 2 * array), (int32_t*)(ws + 3 * array)};
  if (n <= RANKED) {
    f.sorting = (n + 63) / 64;
    share_out(f, 0, 1);
    hipLaunchKernelGGL(sort_ranks_kernel, dim3(f.sorting + f.blocks), dim3(1024), 0, st, g.tokens, n, g.vocab, (n + 255) / 256 * 16, key[0], rows[0], f);
    *token = key[0], *row = rows[0];
    return hipGetLastError();
  }
  int bits = 1;                                               // of the largest key, the vocabulary's size
  while (bits < 31 && g.vocab >> bits) ++bits;
  const int passes = (bits + 8) / 9, each = (bits + passes - 1) / passes;
  uint32_t* hist = (uint32_t*)(ws + 4 * array);
  f.sorting = (n + TILE - 1) / TILE;
  const int32_t* from = g.tokens;
  const int32_t* from_rows = nullptr;
  for (int pass = 0; pass < passes; ++pass) {
    share_out(f, 2 * pass, 2 * passes);
    hipLaunchKernelGGL(sort_count_kernel, dim3(f.sorting + f.blocks), dim3(1024), 0, st, from, n, g.vocab, pass * each, each, hist, f);
    share_out(f, 2 * pass + 1, 2 * passes);
    hipLaunchKernelGGL(sort_place_kernel, dim3(f.sorting + f.blocks), dim3(1024), 0, st, from, from_rows, n, g.vocab, pass * each, each, hist, f.sorting, key[pass & 1], rows[pass & 1], f);
    from = key[pass & 1], from_rows = rows[pass & 1];
  }
  *token = from, *row = from_rows;
  return hipGetLastError();
}

template <typename T, typename O, bool ODD, bool ADD>
hipError_t sums_of(EmbedGrad g, char* ws, hipStream_t st) {
  const int32_t *token, *row;
  hipError_t e = sort_tokens(g, {(char*)g.d_table, ADD ? 0 : (size_t)g.vocab * g.dim * sizeof(O), 0, 0, 0}, ws, &token, &row, st);
  if (e != hipSuccess) return e;
  g.partial = (float*)(ws + 4 * aligned((size_t)g.rows * sizeof(int32_t)) + aligned((size_t)((g.rows + TILE - 1) / TILE) * DIGITS * sizeof(uint32_t)));
  constexpr int N = sizeof(T) + sizeof(O) == 4 ? 8 : 4;
  if (g.rows <= RUN_ROWS) {
    hipLaunchKernelGGL((embed_runs_kernel<T, O, ODD, ADD>), dim3(chunks_of(g.rows), (pieces_of(g.dim, N) + 63) / 64), dim3(1024), 0, st, token, row, g.rows, g.dim, g.vocab, g);
    return hipGetLastError();
  }
  const int slabs = (pieces_of(g.dim, N) + 63) / 64, sums = chunks_of(g.rows) * slabs;
  hipLaunchKernelGGL((embed_sum_kernel<T, O, ODD, ADD>), dim3((sums + 3) / 4), dim3(256), 0, st, token, row, g.rows, g.dim, g.vocab, slabs, sums, g);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((embed_join_kernel<O, ODD, ADD>), dim3(chunks_of(g.rows), (g.dim + 255) / 256), dim3(256), 0, st, token, g.rows, g.dim, g.vocab, g);
  return hipGetLastError();
}

template <typename T, typename O>
hipError_t sums_as(const EmbedGrad& g, bool add, char* ws, hipStream_t st) {
  const bool wide = g.dim % 8 == 0 && rows_at_16(g.dy, g.stride, sizeof(T)) && rows_at_16(g.d_table, g.dim, sizeof(O));
  if (wide) return add ? sums_of<T, O, false, true>(g, ws, st) : sums_of<T, O, false, false>(g, ws, st);
  return add ? sums_of<T, O, true, true>(g, ws, st) : sums_of<T, O, true, false>(g, ws, st);
}

template <typename T, typename O> hipError_t rows_as(const EmbedRows& a, hipStream_t st) {
  const bool wide = a.dim % 8 == 0 && rows_at_16(a.table, a.dim, sizeof(T)) && rows_at_16(a.out, a.stride, sizeof(O));
  if (!wide) return rows_of<T, O, true, false>(a, st);
  return (size_t)a.rows * a.dim * sizeof(O) >= STREAMED ? rows_of<T, O, false, true>(a, st) : rows_of<T, O, false, false>(a, st);
}

}  // namespace

hipError_t launch_embed(const EmbedRows& a, bool table_bf16, bool out_bf16, hipStream_t st) {
  if (table_bf16) return out_bf16 ? rows_as<bf16_t, bf16_t>(a, st) : rows_as<bf16_t, float>(a, st);
  return out_bf16 ? rows_as<float, bf16_t>(a, st) : rows_as<float, float>(a, st);
}

size_t embed_grad_workspace(int rows, int dim) {
  return 4 * aligned((size_t)rows * sizeof(int32_t)) + aligned((size_t)((rows + TILE - 1) / TILE) * DIGITS * sizeof(uint32_t)) +
         (rows > RUN_ROWS ? aligned((size_t)chunks_of(rows) * 2 * padded(dim) * sizeof(float)) : 0);
}

hipError_t launch_embed_grad(const EmbedGrad& g, bool dy_bf16, bool out_bf16, bool add, void* ws, hipStream_t st) {
  if (dy_bf16) return out_bf16 ? sums_as<bf16_t, bf16_t>(g, add, (char*)ws, st) : sums_as<bf16_t, float>(g, add, (char*)ws, st);
  return out_bf16 ? sums_as<float, bf16_t>(g, add, (char*)ws, st) : sums_as<float, float>(g, add, (char*)ws, st);
}
