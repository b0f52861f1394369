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
// A launch that knows only a bound of the lengths.  Times in us, whole / team / wavefronts, 32 heads of 128 over 8:
//   A CU draws some 50 GB/s, so a whole context goes to one workgroup where it is short: one sequence of 256 tokens 5.7 / 6.9 / 9.1, of 512
//   7.8 / 7.1 / 9.7, of 768 10.8 / 8.2 / 10.5, of 2048 23.5 / 9.7 / 11.6 (bf16).  The second launch that parts need costs the host 4 us more, so up to 768.
//   Where sequences fill the chip (the longest begin first) the second launch costs more than uneven lengths: 32 of 500..1024 tokens 24.9 / 28.3 / 29.1, 64 of
//   300..1024 38.1 / 42.9 / 42.5, 48 of 512..2048 53.6 / 56.0 / 55.8, 64 of them 65.2 / 70.1 / 69.4, in fp32 117 / 120 / 128; but 32 of 500..4096 75.2 / 64.5 / 62.8,
//   and where a head's row is one memory line only, 64 of 512..2048 in 8 bits 45.9 / 45.9 / 42.0, in bf16 with 64 dimensions 43.3 / 44.7 / 37.8.
//   A wavefront with a range of its own has no exchange at the end and, with eight units, reads whole rows together with its neighbours, but needs a long range and
//   leaves more parts to join: 131071 tokens in 8 bits under 64 heads 62.4 (team) / 57.3, 256 of 1300 in bf16 259 / 237; 8 of 4000..8192 44.6 / 45.1, 16 of
//   1000..2048 in fp32 41.9 / 46.2, one of 16384 under 64 heads 19.8 / 22.7; 24 heads over one, 19 of up to 103066 in 8 bits 60.1 / 68.6.
// More than 16 query heads to a KV head: 32 of them to a wavefront, as two products of each operand, but for few keys, which leave CUs idle (16 / 32 heads, us: that case
// 79.1 / 60.1, 64 over one, 16 of 4096..8192 in bf16 35.9 / 28.2, 64 of 512..2048 under 24 22.4 / 21.9; 4 of 100..700 10.2 / 12.4), and not with fp32 caches,
// whose operands leave no registers for it.
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
