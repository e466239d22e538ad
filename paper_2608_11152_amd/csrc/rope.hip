// kvp_rope_apply: rotary positions on rows of heads, [tokens, heads, head_dim] with strides.
//   y_a = m (x_a cos - x_b sin),  y_b = m (x_a sin + x_b cos)   for the pair (a, b) of dims, angle = position * f
// in fp32, rounded once to the element type; the transpose (the gradient) takes -sin.  Dims from rotary_dim on are
// copied.  Bandwidth bound: 6 flops and one read and write per pair.
#include <algorithm>

#include "rope_dev.h"

namespace kvp {
namespace {

__device__ __forceinline__ float load(const uint16_t* p) { return widen(*p); }
__device__ __forceinline__ float load(const float* p) { return *p; }
__device__ __forceinline__ void store(uint16_t* p, float v) { *p = narrow(v); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }

// One thread per pair, or per dim that is not rotated.  A pair is read whole before it is written, so y may be x.
template <class T>
__global__ __launch_bounds__(256) void rope_pair_kernel(RopeArgs a) {
  const int R = a.table.rotary_dim, units = a.D - R / 2;
  const int64_t n = a.tokens * a.heads * units;
  const int64_t step = (int64_t)gridDim.x * 256;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += step) {
    const int64_t th = e / units;
    const int u = (int)(e - th * units);
    const int64_t t = th / a.heads;
    const int h = (int)(th - t * a.heads);
    const T* x = reinterpret_cast<const T*>(a.x) + t * a.x_token + h * a.x_head;
    T* y = reinterpret_cast<T*>(a.y) + t * a.y_token + h * a.y_head;
    if (u >= R / 2) {
      y[u + R / 2] = x[u + R / 2];
      continue;
    }
    float sn, cs;
    pair_turn(a.table, u, a.pos[t], &sn, &cs);
    if (a.grad) sn = -sn;
    const int i0 = a.table.interleaved ? 2 * u : u, i1 = a.table.interleaved ? 2 * u + 1 : u + R / 2;
    const float p = load(x + i0), q = load(x + i1);
    float y0, y1;
    turn(p, q, sn, cs, &y0, &y1);
    store(y + i0, y0);
    store(y + i1, y1);
  }
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, bool f32, hipStream_t s) {
  const int64_t n = a.tokens * a.heads * (a.D - a.table.rotary_dim / 2);
  if (n == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, 1 << 20));
  if (f32) hipLaunchKernelGGL(rope_pair_kernel<float>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rope_pair_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace kvp
