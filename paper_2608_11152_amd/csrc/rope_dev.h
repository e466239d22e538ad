// Rotary positions on the device: the angle of a pair, its sine and cosine, and where a pair sits in a head.
//
// Pair i of a token at position p is turned by p * f_i radians.  The host passes f_i as the fraction of a turn per
// position, 2^64 f_i / (2 pi) rounded to an integer (kvp_rope.turns), so the product with p modulo 2^64 is the angle
// modulo one turn with hardly a loss at far positions: the table's half step times 2^31 positions is 2^-34 of a turn.  The
// sine takes the angle rounded to 2^-32 of a turn, at any position.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "kvp_kernels.h"

namespace kvp {

// sin and cos of phase / 2^64 turns.  The phase is rounded to 2^-32 of a turn, 2^-33 (7.3e-10 radian) off at most.  The
// nearest quarter turn is taken out in integers; what remains, |x| <= pi / 4, goes into the Taylor series (first terms left
// out: x^11 / 11! = 2e-9, x^12 / 12! = 1e-10, under half a step of fp32).
__device__ __forceinline__ void sincos_turns(uint64_t phase, float* sn, float* cs) {
  const unsigned top = (unsigned)((phase + (1ull << 31)) >> 32), quad = (top + (1u << 29)) >> 30;
  const int r = (int)(top - (quad << 30));
  const float x = (float)r * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float y = x * x;
  const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), x);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f),
                                       1.0f / 24.0f), -0.5f), 1.0f);
  const bool odd = quad & 1;
  const float a = odd ? c : s, b = odd ? s : c;
  *sn = quad & 2 ? -a : a;
  *cs = (quad == 1 || quad == 2) ? -b : b;
}

__device__ __forceinline__ void pair_turn(const RopeTable& t, int pair, int pos, float* sn, float* cs) {
  sincos_turns((uint64_t)(int64_t)pos * t.turns[pair], sn, cs);
  *sn *= t.magnitude;
  *cs *= t.magnitude;
}

// The pair (p, q) turned.  Written with its fused steps, so every kernel rounds it alike.
__device__ __forceinline__ void turn(float p, float q, float sn, float cs, float* y0, float* y1) {
  *y0 = fmaf(p, cs, -(q * sn));
  *y1 = fmaf(p, sn, q * cs);
}

// sin and cos of N consecutive pairs.
template <int N>
struct Turns {
  float sn[N], cs[N];
  __device__ __forceinline__ void set(const RopeTable& t, int first, int pos) {
#pragma unroll
    for (int i = 0; i < N; ++i) pair_turn(t, first + i, pos, &sn[i], &cs[i]);
  }
};

// Calls whose rows read are half of the last-level cache (256 MB) or more stream them past the caches.
constexpr int64_t kStreamBytes = 128ll << 20;

__device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float((unsigned)b << 16); }
__device__ __forceinline__ uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }  // to nearest even

// 8 consecutive elements of a head, as bf16 or fp32.
struct Eight {
  float x[8];
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  template <bool Stream = false>  // past the caches
  __device__ __forceinline__ void load(const uint16_t* p) {
    const u32x4* const at = reinterpret_cast<const u32x4*>(p);
    const u32x4 v = Stream ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(v[j] << 16);
      x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
    }
  }
  template <bool Stream = false>
  __device__ __forceinline__ void load(const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
  __device__ __forceinline__ uint4 bf16() const {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__bf16)x[j];
    return __builtin_bit_cast(uint4, v);
  }
  template <bool Stream = false>
  __device__ __forceinline__ void store(uint16_t* p) const {
    const u32x4 v = __builtin_bit_cast(u32x4, bf16());
    if (Stream) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = v;
  }
  template <bool Stream = false>
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
};

// Pairs (a[j], b[j]): two runs of 8 dims of the half layout.
__device__ __forceinline__ void turn_halves(Eight& a, Eight& b, const Turns<8>& t) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float y0, y1;
    turn(a.x[j], b.x[j], t.sn[j], t.cs[j], &y0, &y1);
    a.x[j] = y0;
    b.x[j] = y1;
  }
}

// Pairs (a[2 j], a[2 j + 1]): 8 dims of the interleaved layout.
__device__ __forceinline__ void turn_neighbours(Eight& a, const Turns<4>& t) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float y0, y1;
    turn(a.x[2 * j], a.x[2 * j + 1], t.sn[j], t.cs[j], &y0, &y1);
    a.x[2 * j] = y0;
    a.x[2 * j + 1] = y1;
  }
}

}  // namespace kvp
