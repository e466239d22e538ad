// Linear attention with a decay per head over a state per session:
//   S_t = decay S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t
// q, k, v bf16, the state and every sum fp32; the output is rounded once.  How the matrix products take fp32 operands
// stands at linear_chunk_kernel below.
//
// linear_token_kernel: single tokens.
//
// linear_chunk_kernel: chunks of 64 tokens, from the state S before the chunk (rows i, j of the chunk, l = decay):
//   O = (l^(i+1) Q) S + (Q K^T . l^(i-j) for j <= i) V          S' = l^64 S + (l^(63-j) K)^T V
// One workgroup of 2 D threads per (item, KV head) walks an item's tokens; each of its D / 32 waves holds 32 columns of
// S in registers (fp32, D / 2 of them) from the first chunk to the last, so a chunk reads q, k and v and writes o, once:
// 8 D bytes a token and head, and 12 D^2 flops as matrix products of bf16 parts (below).
//
// All products run as v_mfma_f32_16x16x32_bf16.  Its result tile gives a lane 4 rows (4 g + r) of one column; its
// operand wants 8 consecutive k (8 g ..) of one row or column.  Which dim or token a row of a tile stands for is free: row
// m of an even tile is 8 (m / 4) + m % 4 of its 32, of the odd tile 4 more, so a lane's rows of both are 8 consecutive
// ones, and the state and the weights of a chunk are the next product's operand as they come out of the last one's result:
//   P^T (keys x rows)   = K Q^T           O^T (columns x rows) = S^T Q^T + V^T P^T           S (dims x columns) = K^T V
// The waves share P's tiles (each wave needs all of them) through the place of q in LDS, which is done with by then.
// Rows of q, k and v go from memory straight to LDS, past the caches (165 -> 163 and 799 -> 776 us below); K^T and V^T
// come from there through its transposing reads.
//
// Operands that are not bf16 are carried as sums of bf16 parts.  The decayed V that goes into the state is three (2^-26
// left: the state is fp32).  S and P are three for fp32 outputs, which are then 2^-23 off (2-norm, relative), 2^-18.6 with
// two; the prompts below take 195 us with three, 185 with two.  For bf16 outputs they are two (2^-18 left, far inside the
// output's half step 2^-9): three take 178 us instead of 159, and with two one output in 500 is rounded to the other
// neighbour.  One part for S and P would take 6% less time, with 2^-9 of the state in every output.
//
// Three workgroups fit a compute unit (50 KB of LDS; 149 VGPRs, which the sched_barriers and Lane keep them at).  64
// prompts of 128 .. 1024 tokens with 16 heads of 128, 663 MB: 158 us, 4.2 TB/s of the 5.1 that a copy reaches.  A SIMD has
// a matrix instruction under way in 35% of the cycles, a vector instruction in 42%, either in 66%; its waves wait for loads,
// LDS and barriers 29% of their time and for their turn to issue 39%.
//
// A sequence that would leave compute units without work is cut into parts (plan_linear): linear_sum_kernel sums each part
// from zeros, linear_scan_kernel turns the sums into the states before the parts, and the parts are items.  The parts'
// keys and values are read twice: 131071 tokens with 16 heads of 128 take 765 us, 225 of them the sums (1.1 GB, 4.9 TB/s;
// 206 GFLOP: V in 3 parts), 18 the scan, 514 the chunks (2.2 GB, 4.3 TB/s; the SIMDs have an instruction under way in 73% of
// the cycles).
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

// The bf16 of x and y, packed; x and y become what is left of them.  Of an infinity, NaN is left.
__device__ __forceinline__ unsigned part(float& x, float& y) {
  unsigned w = pack2(x, y);
  asm("" : "+v"(w));  // (or x is converted a second time, alone)
  x -= low(w);
  y -= high(w);
  return w;
}

__device__ double power(double x, unsigned n) {
  double y = 1.0;
  for (; n; n >>= 1, x *= x)
    if (n & 1) y *= x;
  return y;
}

constexpr int kChunk = 64;  // tokens

// A tile in LDS: 64 rows (tokens) of D elements.  The 16-byte pieces of a row are keyed by an exclusive or with the row,
// so that the reads of a tile hit all banks: one piece of 16 rows (16 in a row, or m / 4 of 8 apart), where the hardware
// serves lanes of two neighbouring pieces together; or halves of 4 pieces of 8 rows (two rows share their banks then).
template <int D>
__device__ __forceinline__ int tile_key(int row) {
  const int b = row ^ (row >> 2);  // bit 2: bits 2 and 4 of the row
  return D == 128 ? (row & 1) + 2 * ((b >> 2) & 1) + 4 * ((row >> 1) & 1) + (row & 8)
                  : ((row >> 1) & 1) + 2 * ((b >> 2) & 1) + 4 * ((row >> 3) & 1);
}
template <int D>
__device__ __forceinline__ int tile_at(int row, int piece) {  // in bytes
  return 2 * D * row + 16 * (piece ^ tile_key<D>(row));
}
// tile_at of a row 4 y + 16 x + 32 z further (y and x 0 or 1, the row's bits 2 and 4 clear), from the row's own
template <int D>
__device__ __forceinline__ int later(int at, int y, int x, int z) {
  return (at ^ (32 * (x ^ y))) + 2 * D * (4 * y + 16 * x + 32 * z);
}

// Row tile rt (16 rows) sees keys of the halves s <= rt / 2 of a chunk.
__host__ __device__ constexpr int pair_of(int rt, int s) { return rt < 2 ? rt : 2 * rt - 2 + s; }
constexpr int kPwsBase = 31;
constexpr int weights(int parts) { return 6 * parts * 1024; }  // bf16 parts of 6 operands, 16 bytes a lane

template <int D, int Parts>
struct Tiles {
  unsigned char q[std::max(2 * D * kChunk, weights(Parts))];  // later the weights
  unsigned char k[2 * D * kChunk], v[2 * D * kChunk];
  float pw[2 * kChunk];              // decay^(e - 63), 0 below
  float pws[kChunk + 1 + kPwsBase];  // scale decay^(e - kPwsBase), 0 below
};

template <int D>
struct SumTiles {
  unsigned char k[2][2 * D * kChunk], v[2 * D * kChunk];
  float pw[2 * kChunk];
};

__device__ __forceinline__ u32x4 ld16(const unsigned char* p) { return *reinterpret_cast<const u32x4*>(p); }
// The LDS's transposing read: of every 16 lanes, lanes 4 r .. 4 r + 3 name 4 elements each of a row r, and lane l gets
// element l of the 4 rows.  Here the rows are tokens 32 z + 8 g .. + 3 and .. + 7, so a lane gets an operand of 8 tokens.
__device__ __forceinline__ u32x2 ld_turned(const unsigned char* p) {
  typedef short i16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) i16x4 lds4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p));
}
template <int D>
__device__ __forceinline__ u32x4 ld_column(const unsigned char* tile, int at, int z) {
  const u32x2 x = ld_turned(tile + later<D>(at, 0, 0, z)), y = ld_turned(tile + later<D>(at, 1, 0, z));
  return u32x4{x[0], x[1], y[0], y[1]};
}

// A wave's share of a tile from memory straight to LDS, 1 KB at a time: with W waves, rows 1024 / (2 D) (w + W j) ..,
// 16 bytes a lane.  The last rows of an item may end inside the tile: rows from n on repeat row n - 1 and are cleared later.
template <int D>
__device__ __forceinline__ void fetch_tile(unsigned char* tile, const uint16_t* head, int stride, int n, int w, int lane) {
  constexpr int PL = D / 8, RW = 64 / PL;  // lanes of a row, rows of a wave
  const int row = RW * w + lane / PL, src = 16 * ((lane % PL) ^ tile_key<D>(row));
  const uint64_t base = reinterpret_cast<uint64_t>(head);
  const u32x4 rsrc{(unsigned)base, (unsigned)(base >> 32) & 0xffffu, (unsigned)(2 * ((kChunk - 1) * stride + D)), 0x00020000u};
  const unsigned dst = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)(tile) + 1024 * w;
  // In assembly: after the builtin the compiler makes every transposing read wait for all tiles under way.  The kernel
  // waits itself, at its barriers; loads of the compiler's own are waited for behind these, or with them.  (The wait
  // states cover m0, and scalar registers that a vector instruction wrote just before.)
  auto put = [&](int j, int from, int uniform) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst + 32 * D * j)), "v"(from), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(uniform))
                 : "memory", "m0");
  };
  if (n == kChunk) {
    const int even = 2 * stride * row + src, odd = 2 * stride * row + (src ^ 32);
#pragma unroll
    for (int j = 0; j < 4; ++j) put(j, j & 1 ? odd : even, 32 * stride * j);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) put(j, 2 * stride * min(row + 16 * j, n - 1) + (src ^ (32 * (j & 1))), 0);
  }
}

// State of an item: a slot of the caller's, a part of the workspace (-2, -3, ..), or none (-1).
__device__ __forceinline__ float* state_at(const LinearArgs& a, int slot, int h, int D) {
  float* base = slot >= 0 ? a.state : a.parts;
  return base + ((int64_t)(slot >= 0 ? slot : -2 - slot) * a.Hkv + h) * D * D;
}

#define KVP_ASM_BARRIER(loads) asm volatile("s_waitcnt vmcnt(" #loads ") lgkmcnt(0)\n\ts_barrier" ::: "memory")
// Every wave's loads have arrived; all but its last four (one fetch_tile); its LDS reads and writes are done.
__device__ __forceinline__ void arrived() { KVP_ASM_BARRIER(0); }
__device__ __forceinline__ void arrived_but_4() { KVP_ASM_BARRIER(4); }
__device__ __forceinline__ void all_read() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
#undef KVP_ASM_BARRIER

__device__ __forceinline__ double uniform(double x) {  // of a value that all lanes have: in scalar registers
  const u32x2 u = __builtin_bit_cast(u32x2, x);
  return __builtin_bit_cast(double, u32x2{(unsigned)__builtin_amdgcn_readfirstlane((int)u[0]),
                                          (unsigned)__builtin_amdgcn_readfirstlane((int)u[1])});
}

// A lane's number, asked for again: two instructions instead of registers held through the chunk.
struct Lane {
  int lane, m, g;
  __device__ __forceinline__ Lane() {
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
    m = lane & 15;
    g = lane >> 4;
  }
};

// What a wave of a chunk kernel is, and the parts that both kernels share.
template <int D>
struct Wave {
  static constexpr int MT = D / 16;  // row tiles over the dims of k
  int w, item, h;
  __device__ __forceinline__ explicit Wave(int Hkv)
      : w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), item(blockIdx.x / Hkv), h(blockIdx.x - item * Hkv) {}

  __device__ __forceinline__ void fetch(unsigned char* tile, const uint16_t* x, int64_t stride, int head, const LinearItem& it,
                                        int c) const {
    if (c < it.n)
      fetch_tile<D>(tile, x + (it.t0 + (int64_t)c) * stride + head * D, (int)stride, min(kChunk, it.n - c), w, Lane().lane);
  }

  // Rows of a tile that stand in for those behind the item's last: v's must not count.
  __device__ __forceinline__ void clear_behind(unsigned char* v, int n) const {
    for (int e = 64 * w + Lane().lane; e < (kChunk - n) * (D / 8); e += 2 * D)
      *reinterpret_cast<u32x4*>(v + 2 * D * n + 16 * e) = u32x4{0, 0, 0, 0};
  }

  // The wave's 32 columns of the state: tiles [row tile][column tile], element offsets of a lane's 4 rows.
  __device__ __forceinline__ int state_lane() const {
    const Lane l;
    return 8 * l.g * D + 32 * w + 8 * (l.m >> 2) + (l.m & 3);
  }
  __device__ __forceinline__ static constexpr int state_off(int mt, int nt, int r) {
    return (32 * (mt >> 1) + 4 * (mt & 1) + r) * D + 4 * nt;
  }

  // V^T: operands of [32 tokens][16 columns]
  __device__ __forceinline__ void load_v(const unsigned char* v, u32x4 vf[2][2]) const {
    const Lane l;
    const int at = tile_at<D>(8 * l.g + (l.m >> 2), 4 * w + (l.m & 3));
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) vf[s][nt] = ld_column<D>(v + 8 * nt, at, s);
  }

  // S = keep S + K^T (l^(n-1-j) v_j); v's rows from n on are zeros
  __device__ __forceinline__ void update(f32x4 S[MT][2], const unsigned char* k, const u32x4 vf[2][2], const float* pw, int n,
                                         float keep) const {
    const Lane l;
    const int last = n - 1 - 8 * l.g, at = tile_at<D>(8 * l.g + (l.m >> 2), l.m & 3);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) S[mt][nt] *= keep;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      __builtin_amdgcn_sched_barrier(0);
      float d[8];
#pragma unroll
      for (int b = 0; b < 8; ++b) d[b] = pw[last - (32 * s + b) + 63];
      u32x4 vp[2][3];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          float x = low(vf[s][nt][b]) * d[2 * b], y = high(vf[s][nt][b]) * d[2 * b + 1];
          vp[nt][0][b] = part(x, y);
          vp[nt][1][b] = part(x, y);
          vp[nt][2][b] = pack2(x, y);
        }
      }
      // Four independent sums at a time: one product's result is the next but three's summand.
#pragma unroll
      for (int mt = 0; mt < MT; mt += 2) {
        if (mt % 4 == 0) __builtin_amdgcn_sched_barrier(0);
        const u32x4 kf[2] = {ld_column<D>(k, at ^ (32 * mt), s), ld_column<D>(k + 8, at ^ (32 * mt), s)};
#pragma unroll
        for (int x = 2; x >= 0; --x)
#pragma unroll
          for (int y = 0; y < 4; ++y) S[mt + (y >> 1)][y & 1] = mfma16(kf[y >> 1], vp[y & 1][x], S[mt + (y >> 1)][y & 1]);
      }
    }
  }
};

// The state's decay over a chunk, l^64 rounded to fp32, would be off the same way at every chunk.  `off` is the product of
// the factors so far over the true one, within a step of fp32 of 1; each factor takes it back.
struct ChunkDecay {
  double whole, back, off = 1.0;
  __device__ __forceinline__ explicit ChunkDecay(double l) : whole(uniform(power(l, kChunk))), back(uniform(1.0 / whole)) {}
  __device__ __forceinline__ float next(float table, int n) {
    if (n < kChunk || whole < 1e-30) return table;  // the last chunk; or nothing is left of the state
    const float f = (float)(whole * (2.0 - off));
    off = uniform(off * ((double)f * back));
    return f;
  }
};

// The sum of a part of a long sequence: its state from zeros, for linear_scan_kernel.
template <int D>
__global__ __launch_bounds__(2 * D, 3) void linear_sum_kernel(LinearArgs a, LinearItems list) {
  __shared__ SumTiles<D> L;
  const Wave<D> me(a.Hkv);
  const LinearItem it = list.sums[me.item];
  ChunkDecay decay((double)list.decay[me.h]);
  for (int e = threadIdx.x; e < 2 * kChunk; e += 2 * D)
    L.pw[e] = e < 63 ? 0.0f : (float)power((double)list.decay[me.h], e - 63);
  f32x4 S[Wave<D>::MT][2] = {};
  me.fetch(L.k[0], a.k, a.k_stride, me.h, it, 0);
  me.fetch(L.v, a.v, a.v_stride, me.h, it, 0);
  for (int c = 0, odd = 0; c < it.n; c += kChunk, odd ^= 1) {
    const int n = min(kChunk, it.n - c);
    arrived();
    if (n < kChunk) {
      me.clear_behind(L.v, n);
      all_read();
    }
    me.fetch(L.k[odd ^ 1], a.k, a.k_stride, me.h, it, c + kChunk);
    u32x4 vf[2][2];
    me.load_v(L.v, vf);
    all_read();
    me.fetch(L.v, a.v, a.v_stride, me.h, it, c + kChunk);
    me.update(S, L.k[odd], vf, L.pw, n, decay.next(L.pw[n + 63], n));
  }
  float* to = state_at(a, it.dst, me.h, D) + me.state_lane();
#pragma unroll
  for (int mt = 0; mt < Wave<D>::MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) to[Wave<D>::state_off(mt, nt, r)] = S[mt][nt][r];
}

// F32: fp32 outputs.
template <int D, bool F32>
__global__ __launch_bounds__(2 * D, 3) void linear_chunk_kernel(LinearArgs a, LinearItems list) {
  constexpr int Parts = F32 ? 3 : 2;  // bf16 parts of the state and the weights
  __shared__ Tiles<D, Parts> L;
  constexpr int KS = D / 32, MT = Wave<D>::MT;  // k-steps and row tiles over the dims of k
  const Wave<D> me(a.Hkv);
  const int w = me.w, h = me.h, G = a.Hq / a.Hkv, tid = threadIdx.x;
  const LinearItem it = list.items[me.item];
  const int first = h * G + it.g0;
  ChunkDecay decay((double)list.decay[h]);
  if (tid <= kChunk) {
    const double x = power((double)list.decay[h], tid);
    L.pw[tid + 63] = (float)x;
    L.pws[tid + kPwsBase] = (float)(a.scale * x);
  }
  if (tid < 63) L.pw[tid] = 0.0f;
  if (tid < kPwsBase) L.pws[tid] = 0.0f;

  // Loads are under way while there is work that does not need them: the next q and v during the update of the state, the
  // next k (its tile is the update's) and still v during the state's product with q.
  me.fetch(L.q, a.q, a.q_stride, first, it, 0);
  me.fetch(L.v, a.v, a.v_stride, h, it, 0);
  f32x4 S[MT][2] = {};
  if (it.src != -1) {
    const float* from = state_at(a, it.src, h, D) + me.state_lane();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[mt][nt][r] = from[Wave<D>::state_off(mt, nt, r)];
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) asm volatile("" : "+v"(S[mt][0]), "+v"(S[mt][1]));  // waits for it here, not in the loop

  for (int c = 0; c < it.n; c += kChunk) {
    const int n = min(kChunk, it.n - c);
    arrived_but_4();  // q (not yet v); and the update is done with k
    me.fetch(L.k, a.k, a.k_stride, h, it, c);
    u32x4 vf[2][2];
    for (int gq = 0; gq < it.gn; ++gq) {
      if (gq > 0) arrived();
      // O^T = S^T Q^T for the chunk's four row tiles, lane column m being row i = 16 rt + m
      const Lane l0;
      const int q_at = tile_at<D>(l0.m, l0.g);
      f32x4 O[4][2] = {};
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) asm volatile("" : "+v"(S[mt][0]), "+v"(S[mt][1]));  // (not split once for all heads)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        __builtin_amdgcn_sched_barrier(0);
        u32x4 qf[4];
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) qf[rt] = ld16(L.q + later<D>(q_at ^ (64 * ks), 0, rt & 1, rt >> 1));
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          u32x4 sp[Parts];
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            float x = S[2 * ks + (b >> 1)][nt][2 * (b & 1)], y = S[2 * ks + (b >> 1)][nt][2 * (b & 1) + 1];
#pragma unroll
            for (int p = 0; p + 1 < Parts; ++p) sp[p][b] = part(x, y);
            sp[Parts - 1][b] = pack2(x, y);
          }
#pragma unroll
          for (int p = 0; p < Parts; ++p)
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) O[rt][nt] = mfma16(sp[p], qf[rt], O[rt][nt]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (gq == 0) {
        arrived();  // k and v
        if (n < kChunk) me.clear_behind(L.v, n);  // (before the next barrier but one, after which v is read)
      }
      // The wave's share of the tiles (rt, jt) of P^T = K Q^T; its rows are keys j = 32 (jt / 2) + 4 (jt % 2) + 8 g + r.
      constexpr int W = D / 32, N = 12 / W;
      u32x2 weight[N][Parts];
      {
        const Lane l;
        const int k_at = tile_at<D>(8 * (l.m >> 2) + (l.m & 3), l.g), q_at = tile_at<D>(l.m, l.g);
        f32x4 P[N] = {};
        int qa[N], ka[N];
#pragma unroll
        for (int x = 0; x < N; ++x) {
          const int t = w + W * x, rt = t < 4 ? t >> 1 : 2 + ((t - 4) >> 2), jt = t < 4 ? t & 1 : t & 3;
          qa[x] = later<D>(q_at, 0, rt & 1, rt >> 1);
          ka[x] = later<D>(k_at, jt & 1, 0, jt >> 1);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int x = 0; x < N; ++x) P[x] = mfma16(ld16(L.k + (ka[x] ^ (64 * ks))), ld16(L.q + (qa[x] ^ (64 * ks))), P[x]);
#pragma unroll
        for (int x = 0; x < N; ++x) {
          const int t = w + W * x, rt = t < 4 ? t >> 1 : 2 + ((t - 4) >> 2), jt = t < 4 ? t & 1 : t & 3;
          const int e = l.m - 8 * l.g + 16 * rt - 32 * (jt >> 1) - 4 * (jt & 1);  // i - j for r = 0
#pragma unroll
          for (int r = 0; r < 4; ++r) P[x][r] = e - r >= 0 ? P[x][r] * L.pws[e - r + kPwsBase] : 0.0f;
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            float y0 = P[x][2 * b], y1 = P[x][2 * b + 1];
#pragma unroll
            for (int p = 0; p + 1 < Parts; ++p) weight[x][p][b] = part(y0, y1);
            weight[x][Parts - 1][b] = pack2(y0, y1);
          }
        }
      }
      all_read();  // q, whose place the weights take: by pair_of, part and lane
#pragma unroll
      for (int x = 0; x < N; ++x) {
        const int t = w + W * x, rt = t < 4 ? t >> 1 : 2 + ((t - 4) >> 2), jt = t < 4 ? t & 1 : t & 3;
        unsigned char* const to = L.q + 1024 * Parts * pair_of(rt, jt >> 1) + 16 * Lane().lane + 8 * (jt & 1);
#pragma unroll
        for (int p = 0; p < Parts; ++p) *reinterpret_cast<u32x2*>(to + 1024 * p) = weight[x][p];
      }
      all_read();
      me.load_v(L.v, vf);
      const int es = F32 ? 4 : 2;
      char* const out = reinterpret_cast<char*>(a.out) + ((it.t0 + (int64_t)c) * a.Hq + first + gq) * D * es;
      bool bad = false;
#pragma unroll
      for (int rt = 3; rt >= 0; --rt) {
        __builtin_amdgcn_sched_barrier(0);
        const Lane l;
        f32x4 V[2] = {};
#pragma unroll
        for (int s = 0; s <= rt / 2; ++s) {
          const unsigned char* const from = L.q + 1024 * Parts * pair_of(rt, s) + 16 * l.lane;
          u32x4 wp[Parts];
#pragma unroll
          for (int p = 0; p < Parts; ++p) wp[p] = ld16(from + 1024 * p);
#pragma unroll
          for (int p = 0; p < Parts; ++p)
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) V[nt] = mfma16(vf[s][nt], wp[p], V[nt]);
        }
        if (rt == 3) {
          // A value of v that is not finite gives no number in the chunk's last row, and, as 0 times it, in earlier
          // rows that must not see it.
          float z = 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r) z = fmaf(V[0][r], 0.0f, fmaf(V[1][r], 0.0f, z));
          if (__any(z != 0.0f)) {
            float y = 0.0f;
#pragma unroll 1
            for (int s = 0; s < 4; ++s) {
              const u32x4 v = ld16(L.v + tile_at<D>(l.lane, 4 * w + s));
#pragma unroll
              for (int b = 0; b < 4; ++b) y += (low(v[b]) - low(v[b])) + (high(v[b]) - high(v[b]));
            }
            bad = __any(y != 0.0f);
          }
        }
        const int i = 16 * rt + l.m;
        if (bad) {  // key by key: only keys up to the row are multiplied at all
          const uint16_t* const qi = a.q + (it.t0 + (int64_t)(c + min(i, n - 1))) * a.q_stride + (first + gq) * D;
          V[0] = V[1] = f32x4{};
#pragma unroll 1
          for (int j = 0; j < 16 * rt + 16; ++j) {
            float p = 0.0f;
#pragma unroll 1
            for (int d = 0; d < D / 8; ++d) {
              const u32x4 x = *reinterpret_cast<const u32x4*>(qi + 8 * d), y = ld16(L.k + tile_at<D>(j, d));
#pragma unroll
              for (int b = 0; b < 4; ++b) p = fmaf(high(x[b]), high(y[b]), fmaf(low(x[b]), low(y[b]), p));
            }
            p *= L.pws[max(i - j, 0) + kPwsBase];
            const u32x4 v = ld16(L.v + tile_at<D>(j, 4 * w + l.g));
#pragma unroll
            for (int x = 0; x < 8; ++x)
              if (j <= i) V[x >> 2][x & 3] = fmaf(p, x & 1 ? high(v[x >> 1]) : low(v[x >> 1]), V[x >> 2][x & 3]);
          }
        }
        const float f = L.pws[i + 1 + kPwsBase];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int r = 0; r < 4; ++r) V[nt][r] = fmaf(O[rt][nt][r], f, V[nt][r]);
        if (i < n) {
          const int at = i * a.Hq * D + 32 * w + 8 * l.g;
          if constexpr (F32) {
            f32x4* o = reinterpret_cast<f32x4*>(out + 4 * (int64_t)at);
            o[0] = V[0];
            o[1] = V[1];
          } else {
            *reinterpret_cast<u32x4*>(out + 2 * (int64_t)at) =
                u32x4{pack2(V[0][0], V[0][1]), pack2(V[0][2], V[0][3]), pack2(V[1][0], V[1][1]), pack2(V[1][2], V[1][3])};
          }
        }
      }
      all_read();  // the weights and v
      if (gq + 1 < it.gn) me.fetch(L.q, a.q, a.q_stride, first + gq + 1, it, c);
    }
    if (it.dst == -1 && c + kChunk >= it.n) return;  // nobody asks for the state
    me.fetch(L.q, a.q, a.q_stride, first, it, c + kChunk);
    me.fetch(L.v, a.v, a.v_stride, h, it, c + kChunk);
    me.update(S, L.k, vf, L.pw, n, decay.next(L.pw[n + 63], n));
  }
  if (it.dst == -1) return;
  float* to = state_at(a, it.dst, h, D) + me.state_lane();
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) to[Wave<D>::state_off(mt, nt, r)] = S[mt][nt][r];
}

// States before each part of the long sequences, from the parts' own sums: S_0 = source, S_i = l^len S_(i-1) + sum_(i-1).
// Slot i of a sequence's parts holds sum_(i-1) before and S_i afterwards.  In 64 bits: the decay of one part meets that of
// hundreds.  A thread takes 4 elements; `Ways` of them share out the parts of an element, meet, and go on from the sum of
// those before.  The chain of loads is what bounds it, or where there are few parts, the powers of the decay that each
// thread takes: up to Ways * U parts every load is issued before the first is used, and kept; beyond that the parts are
// read twice, U at a time.  1 head of 64, 25000 tokens in 390 parts, with 2 / 4 / 16 ways (U = 8, 16, 8): 65 / 36 / 16 us
// (a thread an element: 103); 16 heads of 128, 131071 tokens in 47: 27 / 19 / 28 us; 9 sequences of 3500 tokens in 5 parts
// each: 22 / 39 / 106 us.
template <int Ways, int U>
__global__ __launch_bounds__(256) void linear_scan_kernel(LinearArgs a, LinearItems list, int D) {
  constexpr int kScanLanes = 256 / Ways, kScanElements = 4 * kScanLanes;
  __shared__ double sums[Ways][kScanElements];
  const int lane = threadIdx.x % kScanLanes, way = threadIdx.x / kScanLanes;
  const int per = D * D / kScanElements, e = (blockIdx.x % per) * kScanElements + 4 * lane;
  const int h = blockIdx.x / per % a.Hkv;
  const LinearScan sc = list.scans[blockIdx.x / per / a.Hkv];
  f32x4* const p = reinterpret_cast<f32x4*>(state_at(a, -2 - sc.part, h, D) + e);
  const int64_t step = (int64_t)a.Hkv * D * D / 4;
  f32x4 source{};
  if (sc.src >= 0) source = *reinterpret_cast<const f32x4*>(state_at(a, sc.src, h, D) + e);
  const int m = (sc.n - 1 + Ways - 1) / Ways, lo = 1 + way * m, hi = min(lo + m, sc.n);
  f32x4 x[U];
  auto load = [&](int i) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < hi) x[u] = p[(i + u) * step];
  };
  if (m <= U) load(lo);
  const double f = power((double)list.decay[h], sc.len);
  double S[4] = {};
  for (int i = lo; i < hi; i += U) {
    if (m > U) load(i);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < hi)
#pragma unroll
        for (int b = 0; b < 4; ++b) S[b] = fma(S[b], f, (double)x[u][b]);
  }
#pragma unroll
  for (int b = 0; b < 4; ++b) sums[way][4 * lane + b] = S[b];
  __syncthreads();
  const double over = power(f, m);
#pragma unroll
  for (int b = 0; b < 4; ++b) S[b] = source[b];
  for (int w = 0; w < way; ++w)
#pragma unroll
    for (int b = 0; b < 4; ++b) S[b] = fma(S[b], over, sums[w][4 * lane + b]);
  for (int i = lo; i < hi; i += U) {
    if (m > U) load(i);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < hi) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          S[b] = fma(S[b], f, (double)x[u][b]);
          x[u][b] = (float)S[b];
        }
        p[(i + u) * step] = x[u];
      }
  }
  if (way == 0 && sc.src >= 0) p[0] = source;
}

// Single tokens: one workgroup per (sequence, KV head).  A thread holds 4 columns of D / R rows of the state, R apart, all
// loads issued before the first is used; the rows' sums for the output meet in the wave and then in LDS.  Bandwidth is
// what bounds it: the state is read once and written once, past the caches (ordinary stores: 142 us below).  512 samples
// of 64 prompts with 16 heads of 128 (612 MB, 537 of them written; a prompt's states are read by its samples from the
// caches): 106 us, 5.8 TB/s; with streaming loads 128, as 320 + 192 sequences 133.  512 sequences in place (1.07 GB): 182
// us, 5.9 TB/s; with streaming loads 201.  4 sequences: 4.5 us of a call's 13.5.
template <int D>
__global__ __launch_bounds__(256) void linear_token_kernel(LinearArgs a, LinearBatch batch) {
  constexpr int C = D / 4, R = 256 / C, N = D / R;  // threads per row, rows at a time, rows per thread
  extern __shared__ float lds[];  // k, then per query head q and the waves' sums: (1 + 5 G) D
  float* const ks = lds;
  float* const qs = ks + D;
  const int tid = threadIdx.x, w = tid >> 6, c = 4 * (tid % C), r0 = tid / C;
  const int i = blockIdx.x / a.Hkv, h = blockIdx.x - i * a.Hkv, G = a.Hq / a.Hkv;
  float* const part = qs + G * D;  // [G][4][D]
  const int src = batch.few ? batch.few_slots[i].x : batch.slots[i].x, dst = batch.few ? batch.few_slots[i].y : batch.slots[i].y;
  const int64_t t = batch.first + i;
  f32x4 S[N] = {};
  if (src >= 0) {
    const float* from = state_at(a, src, h, D) + r0 * D + c;
#pragma unroll
    for (int n = 0; n < N; ++n) S[n] = *reinterpret_cast<const f32x4*>(from + n * R * D);
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

template <int Ways, int U>
static void launch_scan(const LinearArgs& a, const LinearItems& list, int D, hipStream_t s) {
  const dim3 grid(list.n_scans * a.Hkv * (D * D * Ways / 1024));
  hipLaunchKernelGGL((linear_scan_kernel<Ways, U>), grid, dim3(256), 0, s, a, list, D);
}

template <int D, bool F32>
static void launch_chunk(const LinearArgs& a, const LinearItems& list, hipStream_t s) {
  if (list.n_sums > 0) hipLaunchKernelGGL(linear_sum_kernel<D>, dim3(list.n_sums * a.Hkv), dim3(2 * D), 0, s, a, list);
  if (list.most_parts > 64) launch_scan<16, 8>(a, list, D, s);
  else if (list.most_parts > 32) launch_scan<4, 16>(a, list, D, s);
  else if (list.most_parts > 0) launch_scan<2, 8>(a, list, D, s);
  LinearItems some = list;
  const int most = (1 << 23) / a.Hkv;  // a launch has fewer than 2^32 threads
  for (int i = 0; i < list.n_items; i += most) {
    some.items = list.items + i;
    some.n_items = std::min(most, list.n_items - i);
    hipLaunchKernelGGL((linear_chunk_kernel<D, F32>), dim3(some.n_items * a.Hkv), dim3(2 * D), 0, s, a, some);
  }
}

hipError_t launch_linear_chunk(const LinearArgs& a, const LinearItems& list, int D, hipStream_t s) {
  if (list.n_items == 0) return hipSuccess;
  if (D == 128) a.out_f32 ? launch_chunk<128, true>(a, list, s) : launch_chunk<128, false>(a, list, s);
  else a.out_f32 ? launch_chunk<64, true>(a, list, s) : launch_chunk<64, false>(a, list, s);
  return hipGetLastError();
}

}  // namespace kvp
