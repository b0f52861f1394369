// How the attention of single tokens over pages divides its work: the rule by sizes (host code), and the division itself (host and device).
#pragma once
#include <algorithm>
#include <cstddef>

#include "divisor.hpp"

constexpr int PAGED_WAVES = 8;            // wavefronts of a workgroup

struct PagedSplit {
  int rows;                               // query heads of one KV head that a wavefront has: 16 or 32
  int units;                              // what wavefronts share a sequence out by: its KV heads, each as often as its query heads need wavefronts
  int ranges;                             // into how many all sequences' keys are divided; 0: a workgroup per sequence and unit, one launch
  bool team;                              // a range of a unit to a workgroup, else to a wavefront
};
// A launch that knows only a bound of the lengths.  Times in us, in captured graphs, whole / team / wavefronts, 32 heads of 128 over 8:
//   A CU draws some 50 GB/s, so a whole context goes to one workgroup where it is short: one sequence of 256 tokens 5.7 / 6.8 / 11.0, of 512
//   7.9 / 7.0 / 11.3, of 768 10.7 / 8.4 / 12.9, of 2048 23.0 / 8.6 / 12.6 (bf16).  The second launch that parts need costs the host 4 us more, so up to 768 (a graph
//   pays no such cost, and is up to 2.4 us slower than in parts from 513 on).
//   Where sequences fill the chip (the longest begin first) the second launch costs more than uneven lengths: 32 of 500..1024 tokens 24.7 / 27.4 / 28.6, 64 of
//   300..1024 38.3 / 42.3 / 41.9, 48 of 512..2048 53.5 / 55.7 / 54.5, 64 of them 65.1 / 71.3 / 70.9, in fp32 117 / 119 / 127; but 32 of 500..4096 75.4 / 64.1 / 63.7,
//   and where a head's row is one memory line only, 64 of 512..2048 in 8 bits 46.5 / 45.7 / 41.6, in bf16 with 64 dimensions 43.3 / 44.2 / 38.7.
//   Beyond 2048 tokens it depends on the lengths: 40 (320 groups) of 512..3000 62.3 / 59.9 / 60.7, of 512..4096 84.2 / 78.0 / 75.9; 48 (384) of 512..4096 90.9 / 91.4 / 91.3, in fp32 of
//   512..3000 123 / 123 / 131; 64 (512) of 512..3000 89.1 / 93.2 / 93.4, of 512..4096 115 / 119 / 118; 128 of them 225 / 229 / 225.
//   A wavefront with a range of its own has no exchange at the end and, with eight units, reads whole rows together with its neighbours, but needs a long range and
//   leaves more parts to join: 131071 tokens in 8 bits under 64 heads 63.0 (team) / 57.2, 256 of 1300 in bf16 255 / 245; 8 of 4000..8192 44.0 / 46.1, 16 of
//   1000..2048 in fp32 42.5 / 46.8, one of 16384 under 64 heads 19.8 / 22.8; 24 heads over one, 19 of up to 103066 in 8 bits 61.7 / 70.2.
//   Beyond 1024 sequences every wavefront would look through them all: 1025 of 100..2000 823 / 858 / 808, 1500 of up to 1500 under 8 heads over 2 226 / 247 / 249, 2000 of 100..3000
//   so in 8 bits with 64 dimensions 226 / 267 / 207.
// More than 16 query heads to a KV head: 32 of them to a wavefront, as two products of each operand, but for few keys, which leave CUs idle (16 / 32 heads, us, beside what a copy of as many
// bytes takes: that case 79.2 / 60.1, 50.9; 64 over one, 16 of 4096..8192 in bf16 35.9 / 28.0, 10.2; 64 of 512..2048 under 24 21.3 / 19.5, 8.6; 4 of 100..700 10.4 / 12.9, 0.2), and not with
// fp32 caches, whose operands leave no registers for it.
// row_bytes: of a head's row in the cache.
inline PagedSplit paged_split(int B, int H, int Hkv, int row_bytes, bool fp32, int max_len) {
  const int G = H / Hkv;
  const long keys = (long)B * max_len;
  const int rows = !fp32 && G > 16 && keys * Hkv >= 65536 ? 32 : 16;
  const long units = (long)Hkv * ((G + rows - 1) / rows), groups = B * units;
  PagedSplit s = {rows, (int)units, 0, false};
  if (max_len <= 768 || (max_len <= 1024 && groups >= 256) || (max_len <= 2048 && groups >= 320 && row_bytes >= 256)) return s;
  if (B > 1024 || keys >= 1l << 33) return s;                // what a wavefront looks through, and counts in 32 bits
  s.team = units < 8 || keys * units < 2048l * 384;
  s.ranges = (int)std::max(1l, std::min((s.team ? 256 : 256 * PAGED_WAVES) / units, keys / 64));
  return s;
}

// fp32 elements of the parts' results: D sums, the maximum and the sum of weights, for every head
inline size_t paged_partial_floats(int B, int H, int D, int ranges) { return ranges > 0 ? (size_t)(ranges + B) * H * (D + 2) : 0; }

// Tiles of a range, of `total`.  Range r has tiles r * per .. (r + 1) * per - 1, counted over all sequences, some ranges none.
HOST_AND_DEVICE int paged_tiles_of_range(int total, int ranges) {
  const int per = (int)((total + (long long)ranges - 1) / ranges);
  return per > 1 ? per : 1;
}
// The ranges that a sequence with tiles starts .. ends - 1 lies in.  Its part of range r is kept in place r + b: from one part to the next in the order of the
// tiles either r or b grows, so that no two share a place, and there are fewer than ranges + B.
HOST_AND_DEVICE int paged_first_range(int starts, int per) { return starts / per; }
HOST_AND_DEVICE int paged_last_range(int ends, int per) { return (ends - 1) / per; }
