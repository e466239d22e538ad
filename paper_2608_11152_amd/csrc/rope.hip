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

// Any sizes, strides and alignment: one thread per pair, or per dim that is not rotated.  A pair is read whole before it
// is written, so y may be x.
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

// A head in units of 8 dims, 16 bytes of bf16 a load: in the half layout a unit and the one R / 2 further, in the
// interleaved one a unit alone; dims that are not rotated follow.  A thread holds one unit of up to N heads of a token,
// whose sines and cosines (32 instructions a pair) it computes once, while the loads are under way.  16384 tokens of 36
// heads of 128, bf16 (302 MB): 55 us, 5.5 TB/s where a copy reaches 5.1; 5003 tokens of 32 heads, fp32, half of each head
// rotated (164 MB): 31 us, 5.2 TB/s.
template <class T, bool IL, int N, bool Stream>
__global__ __launch_bounds__(256) void rope_unit_kernel(RopeArgs a) {
  const int R = a.table.rotary_dim, turned = IL ? R / 8 : R / 16;
  const unsigned e = blockIdx.x * 256u + threadIdx.x;
  const unsigned th = a.by_units.quotient(e), t = a.by_heads.quotient(th);
  const int u = (int)(e - th * a.by_units.d), h0 = (int)(th - t * a.by_heads.d), step = (int)a.by_heads.d;
  if (t >= a.tokens) return;
  const bool pass = u >= turned;
  const int i0 = pass ? R + (u - turned) * 8 : u * 8, i1 = i0 + R / 2;  // i1: half layout
  const T* x = reinterpret_cast<const T*>(a.x) + t * a.x_token + h0 * a.x_head;
  T* y = reinterpret_cast<T*>(a.y) + t * a.y_token + h0 * a.y_head;
  Eight p[N], q[IL ? 1 : N];
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (h0 + n * step < a.heads) {
      p[n].template load<Stream>(x + n * step * a.x_head + i0);
      if (!IL && !pass) q[n].template load<Stream>(x + n * step * a.x_head + i1);
    }
  if (!pass) {
    Turns<IL ? 4 : 8> w;
    w.set(a.table, IL ? u * 4 : u * 8, a.pos[t]);
    if (a.grad)
#pragma unroll
      for (float& s : w.sn) s = -s;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if constexpr (IL) turn_neighbours(p[n], w);
      else turn_halves(p[n], q[n], w);
    }
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (h0 + n * step < a.heads) {
      p[n].template store<Stream>(y + n * step * a.y_head + i0);
      if (!IL && !pass) q[n].template store<Stream>(y + n * step * a.y_head + i1);
    }
}

template <class T>
bool in_units(const RopeArgs& a) {
  const int64_t per = 16 / sizeof(T);  // elements of 16 bytes
  return a.D % 8 == 0 && a.table.rotary_dim % (a.table.interleaved ? 8 : 16) == 0 &&
         (a.x_token | a.x_head | a.y_token | a.y_head) % per == 0 &&
         (reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y)) % 16 == 0;
}

template <class T, bool IL, int N, bool Stream = false>
void launch_units(RopeArgs a, unsigned units, hipStream_t s) {
  a.by_units = FastDiv(units);
  a.by_heads = FastDiv((a.heads + N - 1) / N);
  const int64_t per = (int64_t)a.by_units.d * a.by_heads.d;
  const int64_t most = std::max<int64_t>(1, (1ll << 30) / per);  // tokens of a launch: 31-bit thread indices
  for (int64_t t = 0; t < a.tokens; t += most) {
    RopeArgs b = a;
    b.tokens = std::min(most, a.tokens - t);
    b.x = reinterpret_cast<const T*>(a.x) + t * a.x_token;
    b.y = reinterpret_cast<T*>(a.y) + t * a.y_token;
    b.pos = a.pos + t;
    hipLaunchKernelGGL((rope_unit_kernel<T, IL, N, Stream>), dim3((unsigned)((b.tokens * per + 255) / 256)), dim3(256), 0, s, b);
  }
}

template <class T, bool IL>
void launch_layout(const RopeArgs& a, hipStream_t s) {
  const unsigned units = (IL ? a.table.rotary_dim / 8 : a.table.rotary_dim / 16) + (a.D - a.table.rotary_dim) / 8;
  // More heads a thread where that leaves waves enough, one where there is little to do; four of fp32 hold too many
  // registers.  36 heads of 128, with 1 / 2 / 4 heads a thread: bf16, 512 tokens (147456 units) 4.9 / 5.1 / 5.8 us, 1024
  // 7.3 / 6.9 / 7.2 us, 16384 interleaved 65 / 57 / 55 us; fp32, 16384 106 / 107 / 113 us.
  const int64_t threads = a.tokens * a.heads * units;
  // Streaming a large call's rows: those 16384 tokens 64 -> 55 us, in a chain with a copy before and one behind 181 -> 156 us
  // (8192 tokens, 75 MB: 78 -> 81 us; fp32, whose lanes write half of their 32 bytes at a time, 107 -> 132 us).
  if constexpr (sizeof(T) == 2) {
    if (threads >= 1 << 21 && a.heads >= 4) {
      if (a.tokens * a.heads * a.D * (int64_t)sizeof(T) >= kStreamBytes) launch_units<T, IL, 4, true>(a, units, s);
      else launch_units<T, IL, 4>(a, units, s);
      return;
    }
  }
  if (threads >= 1 << 18 && a.heads >= 2) launch_units<T, IL, 2>(a, units, s);
  else launch_units<T, IL, 1>(a, units, s);
}

template <class T>
bool launch_in_units(const RopeArgs& a, hipStream_t s) {
  if (!in_units<T>(a)) return false;
  if (a.table.interleaved) launch_layout<T, true>(a, s);
  else launch_layout<T, false>(a, s);
  return true;
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, bool f32, hipStream_t s) {
  if (f32 ? launch_in_units<float>(a, s) : launch_in_units<uint16_t>(a, s)) return hipGetLastError();
  const int64_t n = a.tokens * a.heads * (a.D - a.table.rotary_dim / 2);
  if (n == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((n + 255) / 256, 1 << 20));
  if (f32) hipLaunchKernelGGL(rope_pair_kernel<float>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rope_pair_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace kvp
