// A cache in pages as the kernels see it (include/eagle3.h: eagle3_paged_kv): slots of [Hkv, d] elements, found through a table of pages.
#pragma once
#include "common.hpp"
#include "kernels.hpp"

struct PagedView {
  char* k;
  char* v;
  uint8_t* k_exp;           // fp8: a scale exponent per (slot, head)
  uint8_t* v_exp;
  const int32_t* table;     // [B, max_pages]
  int n_pages, max_pages, Hkv, d, tokens;     // tokens: max_pages * page_size
  Divisor page;             // page size
};

// An e4m3 row's scale 2^(x - 127) as a float, x >= 1
__device__ __forceinline__ float exp_scale(uint32_t x) { return __uint_as_float(x << 23); }
