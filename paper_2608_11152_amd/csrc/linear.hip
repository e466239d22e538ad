// Linear attention with a decay per head over a state per session:
//   S_t = decay S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t
// q, k, v bf16, the state and every sum fp32; the output is rounded once.  The recurrence itself: one workgroup per
// (item, KV head), thread c holds column c of the state in registers and walks the item's tokens.
#include "rope_dev.h"

namespace kvp {
namespace {

template <int D, class List>
__global__ __launch_bounds__(D) void linear_step_kernel(LinearArgs a, List list) {
  __shared__ float ks[D], qs[16][D];
  const LinearItem it = list.items[blockIdx.x];
  const int h = blockIdx.y, c = threadIdx.x, G = a.Hq / a.Hkv;
  const float decay = list.decay[h];
  float S[D];
  const float* from = a.state + ((int64_t)it.src * a.Hkv + h) * D * D + c;
#pragma unroll
  for (int r = 0; r < D; ++r) S[r] = it.src >= 0 ? from[r * D] : 0.0f;
  for (int i = 0; i < it.n; ++i) {
    const int64_t t = (int64_t)it.t0 + i;
    __syncthreads();
    ks[c] = widen(a.k[t * a.k_stride + h * D + c]);
    for (int g = 0; g < G; ++g) qs[g][c] = widen(a.q[t * a.q_stride + (h * G + g) * D + c]);
    const float v = widen(a.v[t * a.v_stride + h * D + c]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < D; ++r) S[r] = fmaf(ks[r], v, decay * S[r]);
    for (int g = 0; g < G; ++g) {
      float o = 0.0f;
#pragma unroll
      for (int r = 0; r < D; ++r) o = fmaf(qs[g][r], S[r], o);
      const int64_t at = (t * a.Hq + h * G + g) * D + c;
      if (a.out_f32) reinterpret_cast<float*>(a.out)[at] = o * a.scale;
      else reinterpret_cast<uint16_t*>(a.out)[at] = narrow(o * a.scale);
    }
  }
  if (it.dst < 0) return;
  float* to = a.state + ((int64_t)it.dst * a.Hkv + h) * D * D + c;
#pragma unroll
  for (int r = 0; r < D; ++r) to[r * D] = S[r];
}

}  // namespace

hipError_t launch_linear_decode(const LinearArgs& a, const LinearList& list, int n_items, int D, hipStream_t s) {
  if (n_items == 0) return hipSuccess;
  const dim3 grid(n_items, a.Hkv);
  if (D == 128) hipLaunchKernelGGL((linear_step_kernel<128, LinearList>), grid, dim3(128), 0, s, a, list);
  else hipLaunchKernelGGL((linear_step_kernel<64, LinearList>), grid, dim3(64), 0, s, a, list);
  return hipGetLastError();
}

hipError_t launch_linear_chunk(const LinearArgs& a, const LinearItems& list, int n_items, int D, hipStream_t s) {
  if (n_items == 0) return hipSuccess;
  const dim3 grid(n_items, a.Hkv);
  if (D == 128) hipLaunchKernelGGL((linear_step_kernel<128, LinearItems>), grid, dim3(128), 0, s, a, list);
  else hipLaunchKernelGGL((linear_step_kernel<64, LinearItems>), grid, dim3(64), 0, s, a, list);
  return hipGetLastError();
}

}  // namespace kvp
