// Linear attention with a decay per head over a state per session:
//   S_t = decay S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t
// q, k, v bf16, the state and every sum fp32; the output is rounded once.
//
// linear_token_kernel: single tokens.
//
// linear_chunk_kernel: chunks of 64 tokens, from the state S before the chunk (rows i, j of the chunk, l = decay):
//   O = (l^(i+1) Q) S + (Q K^T . l^(i-j) for j <= i) V          S' = l^64 S + (l^(63-j) K)^T V
// One workgroup of 2 D threads per (item, KV head) walks an item's tokens; each of its D / 32 waves holds 32 columns of
// S in registers (fp32, 2 D registers' worth per 4 rows) from the first chunk to the last, so a chunk reads q, k, v and
// writes o, once.  Bandwidth is what bounds it: 8 D bytes and 6 D^2 .. 10 D^2 flops a token and head.
//
// All products run as v_mfma_f32_16x16x32_bf16.  Its result tile gives a lane 4 rows (4 g + r) of one column; its
// operand wants 8 consecutive k of one row or column.  Two stacked result tiles are such an operand if k is read in the
// order  slot(8 g + b) = 4 g + b, slot(8 g + 4 + b) = 16 + 4 g + b  (b < 4): the sum over k does not mind.  So the
// dims of Q and K and the tokens of K^T and V^T lie in that order in LDS, and the state and the weights of a chunk go
// from one product's result into the next one's operand without leaving their registers:
//   P^T (keys x rows)   = K Q^T           O^T (columns x rows) = S^T Q^T + V^T P^T           S (dims x columns) = K^T V
// A sequence that would leave compute units without work is cut into parts (plan_linear): linear_chunk_kernel without its
// outputs sums each part from zeros, linear_scan_kernel turns the sums into the states before the parts, and the parts are
// items.  The parts' keys and values are read twice.
//
// Each wave computes all of P^T (a tenth of its matrix work) rather than share it through LDS and a barrier.
//
// Operands that are not bf16 are carried as sums of bf16 parts: S and P as two (2^-18 left: far inside a bf16 output's
// half step 2^-9), the decayed V that goes into the state as three (2^-26: the state is fp32).
#include <algorithm>

#include "rope_dev.h"

namespace kvp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ unsigned pack2(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(unsigned, v);
}
__device__ __forceinline__ float low(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(unsigned w) { return __uint_as_float(w & 0xffff0000u); }

// The bf16 of x and y, packed; x and y become what is left of them.
__device__ __forceinline__ unsigned part(float& x, float& y) {
  const unsigned w = pack2(x, y);
  x -= low(w);
  y -= high(w);
  return w;
}

// x, as a value that the compiler does not know: reads at it are made again instead of held in registers.
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Position of element x of a 32 block in the order of the operands above.
__device__ __forceinline__ int slot_of(int x) { return ((x >> 2) & 3) * 8 + ((x >> 4) & 1) * 4 + (x & 3); }

__device__ double power(double x, unsigned n) {
  double y = 1.0;
  for (; n; n >>= 1, x *= x)
    if (n & 1) y *= x;
  return y;
}

constexpr int kChunk = 64;  // tokens

template <int D>
struct Tiles {
  uint16_t q[kChunk][D + 8];   // rows of tokens, dims in slot order.  The 16 bytes behind each row spread the 16 rows
  uint16_t k[kChunk][D + 8];   // that a wave reads at a time over all banks
  uint16_t kt[D][kChunk + 8];  // rows of dims, tokens in slot order
  uint16_t vt[D][kChunk + 8];
  float pw[kChunk + 1];        // decay^n
};

// Where piece p (8 tokens) of a row of K^T or V^T lies in its row.  Rows are 36 words apart: a wave writes one piece of
// rows 8 apart (32 words: two bank groups without this), and reads rows m, or 8 (m / 4) + m % 4, of one tile.
__device__ __forceinline__ int piece_at(int row, int p) { return 8 * (p ^ ((row >> 2) & 4) ^ ((row >> 5) & 3)); }

// 8 rows (tokens) of 8 elements become 8 rows (dims) of 8 tokens, and go to LDS.
template <int P>
__device__ __forceinline__ void store_transposed(uint16_t (*dst)[P], int dim, int piece, const u32x4* row) {
  const int at = piece_at(dim, piece);  // dim is a multiple of 8: the same for all 8 rows
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = __builtin_amdgcn_perm(row[2 * j + 1][d >> 1], row[2 * j][d >> 1], d & 1 ? 0x07060302u : 0x05040100u);
    *reinterpret_cast<u32x4*>(&dst[dim + d][at]) = w;
  }
}

// 8 dims of one token, in slot order: two pieces of 4.
template <int P>
__device__ __forceinline__ void store_row(uint16_t (*dst)[P], int token, int dim, u32x4 v) {
  uint16_t* p = &dst[token][(dim & ~31) + slot_of(dim & 31)];
  *reinterpret_cast<u32x2*>(p) = u32x2{v[0], v[1]};
  *reinterpret_cast<u32x2*>(p + 8) = u32x2{v[2], v[3]};
}

__device__ __forceinline__ u32x4 ld16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }

// Up to a chunk's rows of one head, as a buffer: reads behind the last row give zeros, writes there are dropped.
struct Rows {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ Rows(const void* p, int64_t stride, int rows, int D, int bytes = 2)
      : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0,
                                               rows > 0 ? ((min(rows, kChunk) - 1) * (int)stride + D) * bytes : 0,
                                               0x00020000)) {}
  __device__ __forceinline__ u32x4 load(int at) const { return __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0); }
  __device__ __forceinline__ void store(int at, u32x4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, at, 0, 0);
  }
};

// State of an item: a slot of the caller's, a part of the workspace (-2, -3, ..), or none (-1).
__device__ __forceinline__ float* state_at(const LinearArgs& a, int slot, int h, int D) {
  float* base = slot >= 0 ? a.state : a.parts;
  return base + ((int64_t)(slot >= 0 ? slot : -2 - slot) * a.Hkv + h) * D * D;
}

// kAttend: outputs and state; otherwise only the state, from zeros (the sum of a part of a long sequence).
template <int D, bool kAttend>
__global__ __launch_bounds__(2 * D, 2) void linear_chunk_kernel(LinearArgs a, LinearItems list) {
  __shared__ Tiles<D> L;
  constexpr int KS = D / 32, MT = D / 16;  // k-steps and row tiles over the dims of k
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, m = lane & 15, g = lane >> 4;
  const int item = blockIdx.x / a.Hkv, h = blockIdx.x - item * a.Hkv, G = kAttend ? a.Hq / a.Hkv : 1;
  const LinearItem it = list.items[item];
  const double l1 = (double)list.decay[h];
  if (tid <= kChunk) L.pw[tid] = (float)power(l1, tid);

  // Column n of the wave's 16-wide tile nt is column 8 (n / 4) + 4 nt + n % 4 of its 32: a lane's rows of O^T from
  // both tiles are then 8 consecutive columns.
  const int col = 32 * w + 8 * (m >> 2) + (m & 3);
  f32x4 S[MT][2] = {};
  if (it.src != -1) {
    const float* from = state_at(a, it.src, h, D) + 4 * g * D + col;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[mt][nt][r] = from[(16 * mt + r) * D + 4 * nt];
  }

  // What a thread brings: an 8 x 8 block of k (the first D threads) or v, and 4 pieces of q.  Rows behind the item's
  // last are outside their buffer and read as zeros.
  const int c8 = (tid % (D / 8)) * 8, tg = (tid % D) / (D / 8), first = 32 * (tg >> 2) + 4 * (tg & 3);
  const bool keys = w < D / 64;
  const uint16_t* const kv = keys ? a.k : a.v;
  const int64_t kv_stride = keys ? a.k_stride : a.v_stride;
  const int qrow = tid / (D / 8);
  u32x4 rkv[8], rq[4];
  auto fetch_kv = [&](int c) {
    const Rows rows(kv + (it.t0 + (int64_t)c) * kv_stride + h * D, kv_stride, it.n - c, D);
    const int at = again(2 * (first * (int)kv_stride + c8));
#pragma unroll
    for (int j = 0; j < 8; ++j) rkv[j] = rows.load(at + 2 * ((j & 3) + 4 * (j & 4)) * (int)kv_stride);
  };
  auto fetch_q = [&](int c, int gq) {
    const Rows rows(a.q + (it.t0 + (int64_t)c) * a.q_stride + (h * G + gq) * D, a.q_stride, it.n - c, D);
    const int at = again(2 * (qrow * (int)a.q_stride + c8));
#pragma unroll
    for (int j = 0; j < 4; ++j) rq[j] = rows.load(at + 32 * j * (int)a.q_stride);
  };
  fetch_kv(0);
  if (kAttend) fetch_q(0, 0);

  // The state's decay over a chunk, l^64 rounded to fp32, would be off the same way at every chunk.  `off` is the
  // product of the factors so far over the true one, within a step of fp32 of 1; each factor takes it back.
  const double l64 = power(l1, kChunk), back = 1.0 / l64;
  const bool track = l64 > 1e-30;
  double off = 1.0;

  for (int c = 0; c < it.n; c += kChunk) {
    const int n = min(kChunk, it.n - c);
    __syncthreads();
    if (keys) {
      store_transposed(L.kt, c8, tg, rkv);
      if (kAttend)
#pragma unroll
        for (int j = 0; j < 8; ++j) store_row(L.k, first + (j & 3) + 4 * (j & 4), c8, rkv[j]);
    } else {
      store_transposed(L.vt, c8, tg, rkv);
    }
    if (kAttend) {
      for (int gq = 0; gq < G; ++gq) {
        if (gq > 0) __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) store_row(L.q, qrow + 16 * j, c8, rq[j]);
        __syncthreads();
        if (gq + 1 < G) fetch_q(c, gq + 1);
        // O^T = S^T Q^T for the chunk's four row tiles
        f32x4 O[4][2] = {};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          __builtin_amdgcn_sched_barrier(0);
          u32x4 qf[4];
#pragma unroll
          for (int rt = 0; rt < 4; ++rt) qf[rt] = ld16(&L.q[16 * rt + m][32 * ks + 8 * g]);
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            u32x4 hi, lo;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              float x = S[2 * ks + (b >> 1)][nt][2 * (b & 1)], y = S[2 * ks + (b >> 1)][nt][2 * (b & 1) + 1];
              hi[b] = part(x, y);
              lo[b] = pack2(x, y);
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) O[rt][nt] = mfma16(hi, qf[rt], O[rt][nt]);
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) O[rt][nt] = mfma16(lo, qf[rt], O[rt][nt]);
          }
        }
        const int es = a.out_f32 ? 4 : 2;
        const Rows out(reinterpret_cast<char*>(a.out) + ((it.t0 + (int64_t)c) * a.Hq + h * G + gq) * D * es, a.Hq * D,
                       n, D, es);
        bool bad = false;
#pragma unroll
        for (int rt = 3; rt >= 0; --rt) {
          __builtin_amdgcn_sched_barrier(0);
          // P^T: lane column m is row i = 16 rt + m, its rows are keys j = 16 jt + 4 g + r
          const int g8 = again(8 * g), m4 = again(m - 4 * g);
          f32x4 P[4] = {};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const u32x4 qf = ld16(&L.q[16 * rt + m][32 * ks + g8]);
#pragma unroll
            for (int jt = 0; jt <= rt; ++jt) P[jt] = mfma16(ld16(&L.k[16 * jt + m][32 * ks + g8]), qf, P[jt]);
          }
#pragma unroll
          for (int jt = 0; jt <= rt; ++jt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int e = m4 + 16 * (rt - jt) - r;
              P[jt][r] *= a.scale * L.pw[jt < rt ? e : max(e, 0)];
              if (jt == rt && e < 0) P[jt][r] = 0.0f;
            }
          f32x4 V[2] = {};
#pragma unroll
          for (int s = 0; s <= rt / 2; ++s) {
            u32x4 hi, lo;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              float x = P[2 * s + (b >> 1)][2 * (b & 1)], y = P[2 * s + (b >> 1)][2 * (b & 1) + 1];
              hi[b] = part(x, y);
              lo[b] = pack2(x, y);
            }
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
              const u32x4 vf = ld16(&L.vt[col + 4 * nt][piece_at(col, 4 * s + (g8 >> 3))]);
              V[nt] = mfma16(vf, hi, V[nt]);
              V[nt] = mfma16(vf, lo, V[nt]);
            }
          }
          if (rt == 3) {
            // A value of v that is not finite gives no number in the chunk's last row, and, as 0 times it, in earlier
            // rows that must not see it.
            float z = 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) z += (V[0][r] - V[0][r]) + (V[1][r] - V[1][r]);
            if (__any(z != 0.0f)) {
              float y = 0.0f;
#pragma unroll 1
              for (int s = 0; s < 4; ++s) {
                const u32x4 v = ld16(&L.vt[32 * w + (lane >> 1)][32 * (lane & 1) + 8 * s]);  // any order will do
#pragma unroll
                for (int b = 0; b < 4; ++b) y += (low(v[b]) - low(v[b])) + (high(v[b]) - high(v[b]));
              }
              bad = __any(y != 0.0f);
            }
          }
          const int i = 16 * rt + m;
          if (bad) {  // key by key: only keys up to the row are multiplied at all
            V[0] = V[1] = f32x4{};
#pragma unroll 1
            for (int j = 0; j < 16 * rt + 16; ++j) {
              float p = 0.0f;
#pragma unroll 1
              for (int d = 0; d < D; d += 8) {
                const u32x4 x = ld16(&L.q[i][d]), y = ld16(&L.k[j][d]);
#pragma unroll
                for (int b = 0; b < 4; ++b) p = fmaf(high(x[b]), high(y[b]), fmaf(low(x[b]), low(y[b]), p));
              }
              p *= a.scale * L.pw[max(i - j, 0)];
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                const int row = 32 * w + 8 * g + x, at = (j & 32) + slot_of(j & 31);
                const float v = widen(L.vt[row][piece_at(row, at >> 3) + (at & 7)]);
                if (j <= i) V[x >> 2][x & 3] = fmaf(p, v, V[x >> 2][x & 3]);
              }
            }
          }
          const float f = a.scale * L.pw[again(i + 1)];
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int r = 0; r < 4; ++r) V[nt][r] = fmaf(O[rt][nt][r], f, V[nt][r]);
          const int at = again(i) * a.Hq * D + 32 * w + 8 * g;
          if (a.out_f32) {
            out.store(4 * at, __builtin_bit_cast(u32x4, V[0]));
            out.store(4 * at + 16, __builtin_bit_cast(u32x4, V[1]));
          } else {
            out.store(2 * at, u32x4{pack2(V[0][0], V[0][1]), pack2(V[0][2], V[0][3]), pack2(V[1][0], V[1][1]),
                                    pack2(V[1][2], V[1][3])});
          }
        }
      }
    } else {
      __syncthreads();
    }
    // The next chunk's rows, which arrive during the update of the state.
    fetch_kv(c + kChunk);
    if (kAttend) fetch_q(c + kChunk, 0);
    __builtin_amdgcn_sched_barrier(0);
    const int g8 = again(8 * g);
    // S = l^n S + (l^(n-1-j) V's rows times K^T); rows from n on are zeros
    float keep = L.pw[n];
    if (n == kChunk && track) {
      keep = (float)(l64 * (2.0 - off));
      off *= (double)keep * back;
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) S[mt][nt] *= keep;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      __builtin_amdgcn_sched_barrier(0);
      float d[8];
#pragma unroll
      for (int b = 0; b < 8; ++b) d[b] = L.pw[max(n - 1 - (32 * s + (g8 >> 1) + (b & 3) + 4 * (b & 4)), 0)];
      u32x4 vp[2][3];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
        const u32x4 vf = ld16(&L.vt[col + 4 * nt][piece_at(col, 4 * s + (g8 >> 3))]);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          float x = low(vf[b]) * d[2 * b], y = high(vf[b]) * d[2 * b + 1];
          vp[nt][0][b] = part(x, y);
          vp[nt][1][b] = part(x, y);
          vp[nt][2][b] = pack2(x, y);
        }
      }
      // Four independent sums at a time: one product's result is the next but three's summand.
#pragma unroll
      for (int mt = 0; mt < MT; mt += 2) {
        const u32x4 kf[2] = {ld16(&L.kt[16 * mt + m][piece_at(16 * mt, 4 * s + (g8 >> 3))]),
                             ld16(&L.kt[16 * mt + 16 + m][piece_at(16 * mt + 16, 4 * s + (g8 >> 3))])};
#pragma unroll
        for (int x = 2; x >= 0; --x)
#pragma unroll
          for (int y = 0; y < 4; ++y) S[mt + (y >> 1)][y & 1] = mfma16(kf[y >> 1], vp[y & 1][x], S[mt + (y >> 1)][y & 1]);
      }
    }
  }
  if (it.dst == -1) return;
  float* to = state_at(a, it.dst, h, D) + 4 * g * D + col;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) to[(16 * mt + r) * D + 4 * nt] = S[mt][nt][r];
}

// States before each part of the long sequences, from the parts' own sums: S_0 = source, S_i = l^len S_(i-1) + sum_(i-1).
// Slot i of a sequence's parts holds sum_(i-1) before and S_i afterwards.  One thread per element, in 64 bits: the decay
// of one part meets that of hundreds.
__global__ __launch_bounds__(256) void linear_scan_kernel(LinearArgs a, LinearItems list, int D) {
  const int per = D * D / 256, e = (blockIdx.x % per) * 256 + threadIdx.x;
  const int h = blockIdx.x / per % a.Hkv;
  const LinearScan sc = list.scans[blockIdx.x / per / a.Hkv];
  const double f = power((double)list.decay[h], sc.len);
  float* p = state_at(a, -2 - sc.part, h, D) + e;
  const int64_t step = (int64_t)a.Hkv * D * D;
  double S = 0.0;
  if (sc.src >= 0) {
    const float x = state_at(a, sc.src, h, D)[e];
    p[0] = x;
    S = x;
  }
  constexpr int U = 16;  // loads in flight
  for (int i = 1; i < sc.n; i += U) {
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = i + u < sc.n ? p[(i + u) * step] : 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      S = fma(S, f, (double)x[u]);
      if (i + u < sc.n) p[(i + u) * step] = (float)S;
    }
  }
}

// Single tokens: one workgroup per (sequence, KV head).  A thread holds 4 columns of D / R rows of the state, R apart, all
// loads issued before the first is used; the rows' sums for the output meet in the wave and then in LDS.  Bandwidth is
// what bounds it: the state is read and written once, past the caches.
template <int D>
__global__ __launch_bounds__(256) void linear_token_kernel(LinearArgs a, LinearBatch batch) {
  constexpr int C = D / 4, R = 256 / C, N = D / R;  // threads per row, rows at a time, rows per thread
  extern __shared__ float lds[];  // k, then per query head q and the waves' sums: (1 + 5 G) D
  float* const ks = lds;
  float* const qs = ks + D;
  const int tid = threadIdx.x, w = tid >> 6, c = 4 * (tid % C), r0 = tid / C;
  const int i = blockIdx.x / a.Hkv, h = blockIdx.x - i * a.Hkv, G = a.Hq / a.Hkv;
  float* const part = qs + G * D;  // [G][4][D]
  const int src = batch.slots[i].x, dst = batch.slots[i].y;
  const int64_t t = batch.first + i;
  f32x4 S[N] = {};
  if (src >= 0) {
    const float* from = state_at(a, src, h, D) + r0 * D + c;
#pragma unroll
    for (int n = 0; n < N; ++n) S[n] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(from + n * R * D));
  }
  if (tid < D) ks[tid] = widen(a.k[t * a.k_stride + h * D + tid]);
  for (int e = tid; e < G * D; e += 256) qs[e] = widen(a.q[t * a.q_stride + h * G * D + e]);
  const u32x2 vw = *reinterpret_cast<const u32x2*>(a.v + t * a.v_stride + h * D + c);
  const f32x4 v{low(vw[0]), high(vw[0]), low(vw[1]), high(vw[1])};
  const float decay = batch.decay[h];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const float k = ks[r0 + n * R];
#pragma unroll
    for (int x = 0; x < 4; ++x) S[n][x] = fmaf(k, v[x], decay * S[n][x]);
  }
  if (dst >= 0) {
    float* to = state_at(a, dst, h, D) + r0 * D + c;
#pragma unroll
    for (int n = 0; n < N; ++n) __builtin_nontemporal_store(S[n], reinterpret_cast<f32x4*>(to + n * R * D));
  }
  for (int g = 0; g < G; ++g) {
    f32x4 o = {};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float q = qs[g * D + r0 + n * R];
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x] = fmaf(q, S[n][x], o[x]);
    }
#pragma unroll
    for (int d = C; d < 64; d *= 2)
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x] += __shfl_xor(o[x], d);
    if ((tid & 63) < C) *reinterpret_cast<f32x4*>(part + (4 * g + w) * D + c) = o;
  }
  __syncthreads();
  for (int e = tid; e < G * D; e += 256) {
    const float* p = part + 4 * (e / D) * D + e % D;
    const float o = a.scale * (p[0] + p[D] + (p[2 * D] + p[3 * D]));
    const int64_t at = (t * a.Hq + h * G) * D + e;
    if (a.out_f32) reinterpret_cast<float*>(a.out)[at] = o;
    else reinterpret_cast<uint16_t*>(a.out)[at] = narrow(o);
  }
}

}  // namespace

hipError_t launch_linear_decode(const LinearArgs& a, const LinearBatch& batch, int n, int D, hipStream_t s) {
  if (n == 0) return hipSuccess;
  const dim3 grid(n * a.Hkv);
  const size_t lds = (size_t)(1 + 5 * (a.Hq / a.Hkv)) * D * sizeof(float);
  if (D == 128) hipLaunchKernelGGL(linear_token_kernel<128>, grid, dim3(256), lds, s, a, batch);
  else hipLaunchKernelGGL(linear_token_kernel<64>, grid, dim3(256), lds, s, a, batch);
  return hipGetLastError();
}

template <int D>
static void launch_chunk(const LinearArgs& a, const LinearItems& list, hipStream_t s) {
  if (list.n_scans > 0) {
    LinearItems sums = list;
    sums.items = list.sums;
    hipLaunchKernelGGL((linear_chunk_kernel<D, false>), dim3(list.n_sums * a.Hkv), dim3(2 * D), 0, s, a, sums);
    hipLaunchKernelGGL(linear_scan_kernel, dim3(list.n_scans * a.Hkv * (D * D / 256)), dim3(256), 0, s, a, list, D);
  }
  hipLaunchKernelGGL((linear_chunk_kernel<D, true>), dim3(list.n_items * a.Hkv), dim3(2 * D), 0, s, a, list);
}

hipError_t launch_linear_chunk(const LinearArgs& a, const LinearItems& list, int D, hipStream_t s) {
  if (list.n_items == 0) return hipSuccess;
  if (D == 128) launch_chunk<128>(a, list, s);
  else launch_chunk<64>(a, list, s);
  return hipGetLastError();
}

}  // namespace kvp
