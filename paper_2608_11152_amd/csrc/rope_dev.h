// Rotary positions on the device: the angle of a pair, its sine and cosine, and where a pair sits in a head.
//
// Pair i of a token at position p is turned by p * f_i radians.  The host passes f_i as the fraction of a turn per
// position, 2^64 f_i / (2 pi) rounded to an integer (kvp_rope.turns), so the product with p modulo 2^64 is the angle
// modulo one turn with no loss at far positions: the table's half step times 2^31 positions is 2^-34 of a turn.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "kvp_kernels.h"

namespace kvp {

// sin and cos of phase / 2^64 turns.  The nearest quarter turn is taken out in integers; what remains, |x| <= pi / 4,
// goes into the Taylor series (first terms left out: x^11 / 11! = 2e-9, x^12 / 12! = 1e-10, under half a step of fp32).
__device__ __forceinline__ void sincos_turns(uint64_t phase, float* sn, float* cs) {
  const unsigned quad = (unsigned)((phase + (1ull << 61)) >> 62);
  const int r = (int)((int64_t)(phase - ((uint64_t)quad << 62)) >> 32);
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

__device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float((unsigned)b << 16); }
__device__ __forceinline__ uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }  // to nearest even

}  // namespace kvp
