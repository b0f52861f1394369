// Attention of one new token of every sequence over its paged keys and values.
#include <cfloat>

#include "paged.hpp"

namespace {

template <typename T> __device__ __forceinline__ float cached(const T* p, size_t i, float) { return load_f32(p, i); }
template <> __device__ __forceinline__ float cached<uint8_t>(const uint8_t* p, size_t i, float scale) {
  return __builtin_amdgcn_cvt_f32_fp8((int)p[i], 0) * scale;
}

// One workgroup per (sequence, query head): four wavefronts take every fourth key, a lane D / 64 dimensions.
template <typename Q, typename C, int D>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedView c, const Q* __restrict__ q, long long q_stride, const int32_t* __restrict__ kv_len,
                                                         int max_len, int H, float scale, Q* __restrict__ out, float* __restrict__ lse) {
#pragma clang fp contract(off)     // a score and the maximum that it may be have to be the same number, however large
  constexpr int E = D / 64;
  constexpr bool FP8 = sizeof(C) == 1;
  __shared__ float sm[4], sl[4], so[4][D];
  const int b = blockIdx.y, h = blockIdx.x, hk = h / (H / c.Hkv), lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int n = min(max(kv_len[b], 0), max_len);
  float qv[E], o[E], m = -FLT_MAX, l = 0.f;
  for (int e = 0; e < E; ++e) {
    qv[e] = load_f32(q, (size_t)b * q_stride + (size_t)h * D + lane * E + e);
    o[e] = 0.f;
  }
  for (int p = w; p < n; p += 4) {
    const int page = min(max(c.table[(size_t)b * c.max_pages + p / c.page], 0), c.n_pages - 1);
    const size_t at = ((size_t)page * c.page.d + p % c.page) * c.Hkv + hk;
    const float ks = FP8 ? exp_scale(c.k_exp[at]) : 1.f, vs = FP8 ? exp_scale(c.v_exp[at]) : 1.f;
    float s = 0.f;
    for (int e = 0; e < E; ++e) s = fmaf(qv[e], cached((const C*)c.k, at * D + lane * E + e, ks), s);
    s = wave_sum(s) * scale;
    const float mn = fmaxf(m, s), a = expf(m - mn), w8 = expf(s - mn);
    m = mn;
    l = l * a + w8;
    for (int e = 0; e < E; ++e) o[e] = o[e] * a + w8 * cached((const C*)c.v, at * D + lane * E + e, vs);
  }
  if (lane == 0) { sm[w] = m; sl[w] = l; }
  for (int e = 0; e < E; ++e) so[w][lane * E + e] = o[e];
  __syncthreads();
  const float M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  float L = 0.f;
  for (int i = 0; i < 4; ++i) L += sl[i] * expf(sm[i] - M);
  const int t = threadIdx.x;
  if (t < D) {
    float v = 0.f;
    for (int i = 0; i < 4; ++i) v += so[i][t] * expf(sm[i] - M);
    store_from_f32(out, ((size_t)b * H + h) * D + t, n > 0 ? v / L : 0.f);
  }
  if (t == 0 && lse != nullptr) lse[(size_t)b * H + h] = n > 0 ? M + logf(L) : -__builtin_huge_valf();
}

template <typename Q, typename C>
hipError_t launch(const PagedView& c, int B, int H, const void* q, long long q_stride, const int32_t* kv_len, int max_len, float scale, void* out,
                  float* lse, hipStream_t st) {
  if (c.d == 128)
    hipLaunchKernelGGL((paged_attn_kernel<Q, C, 128>), dim3(H, B), dim3(256), 0, st, c, (const Q*)q, q_stride, kv_len, max_len, H, scale, (Q*)out, lse);
  else
    hipLaunchKernelGGL((paged_attn_kernel<Q, C, 64>), dim3(H, B), dim3(256), 0, st, c, (const Q*)q, q_stride, kv_len, max_len, H, scale, (Q*)out, lse);
  return hipGetLastError();
}

}  // namespace

size_t paged_attention_workspace(int, int, int, int, int) { return 0; }

hipError_t launch_paged_attention(const PagedView& c, int dtype, int B, int H, const void* q, long long q_stride, const int32_t* kv_len, int max_len,
                                  float scale, void* out, float* lse, void*, hipStream_t st) {
  if (dtype == PAGED_FP8) return launch<bf16_t, uint8_t>(c, B, H, q, q_stride, kv_len, max_len, scale, out, lse, st);
  if (dtype == PAGED_BF16) return launch<bf16_t, bf16_t>(c, B, H, q, q_stride, kv_len, max_len, scale, out, lse, st);
  return launch<float, float>(c, B, H, q, q_stride, kv_len, max_len, scale, out, lse, st);
}
