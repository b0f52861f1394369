// Rotary positions of queries and keys, and their gradient.
#include "common.hpp"
#include "kernels.hpp"

namespace {

// One workgroup per row: the row's sines and cosines first, then every pair of every head.
template <typename T>
__global__ __launch_bounds__(256) void rope_kernel(RopeTensor q, RopeTensor k, RopeAngles a, int d) {
  __shared__ float cs[512], sn[512];
  const int r = blockIdx.x, half = a.rot >> 1;
  const double pos = (double)a.positions[r];
  for (int i = threadIdx.x; i < half; i += 256) {
    const double t = pos * a.turns[i];
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    cs[i] = a.amplitude * c;
    sn[i] = a.sign * a.amplitude * s;
  }
  __syncthreads();
  const int per_head = half + d - a.rot;            // pairs, then dimensions that stay
  for (int u = threadIdx.x; u < (q.heads + k.heads) * per_head; u += 256) {
    const int h = u / per_head, i = u % per_head;
    const bool is_k = h >= q.heads;
    const RopeTensor& t = is_k ? k : q;
    const T* x = (const T*)t.x + (size_t)r * t.stride + (size_t)(is_k ? h - q.heads : h) * d;
    T* y = (T*)t.y + (size_t)r * t.y_stride + (size_t)(is_k ? h - q.heads : h) * d;
    if (i < half) {
      const int ia = a.interleaved ? 2 * i : i, ib = a.interleaved ? 2 * i + 1 : i + half;
      const float xa = load_f32(x, ia), xb = load_f32(x, ib);
      store_from_f32(y, ia, xa * cs[i] - xb * sn[i]);
      store_from_f32(y, ib, xb * cs[i] + xa * sn[i]);
    } else {
      y[i + half] = x[i + half];
    }
  }
}

}  // namespace

hipError_t launch_rope(bool bf16, const RopeTensor& q, const RopeTensor& k, const RopeAngles& a, int rows, int d, hipStream_t st) {
  if (bf16) hipLaunchKernelGGL(rope_kernel<bf16_t>, dim3(rows), dim3(256), 0, st, q, k, a, d);
  else hipLaunchKernelGGL(rope_kernel<float>, dim3(rows), dim3(256), 0, st, q, k, a, d);
  return hipGetLastError();
}
