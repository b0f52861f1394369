// Into how many parts the attention of single tokens over pages splits a context (host code).
#pragma once
#include <algorithm>
#include <cstddef>

constexpr int PAGED_ROWS = 16;            // query heads of one KV head that a workgroup has

struct PagedSplit {
  int chunk;                              // keys of a part
  int parts;                              // of the longest context that a launch has to expect
  int row_tiles;                          // workgroups that a KV head's query heads take
};

inline PagedSplit paged_split(int B, int H, int Hkv, int max_len) {
  const int tiles = (H / Hkv + PAGED_ROWS - 1) / PAGED_ROWS;
  const long units = (long)B * Hkv * tiles, target = 2048;
  const long parts = std::max(1l, std::min((target + units - 1) / units, (max_len + 255l) / 256));
  const int chunk = (int)(((max_len + parts - 1) / parts + 127) / 128 * 128);
  return {chunk, (max_len + chunk - 1) / chunk, tiles};
}

// fp32 elements of the parts' results: D sums, the maximum and the sum of weights, for every head and part
inline size_t paged_partial_floats(int B, int H, int D, int parts) { return parts > 1 ? (size_t)B * H * parts * (D + 2) : 0; }
