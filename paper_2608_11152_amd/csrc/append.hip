// kv_append / kv_gather / pool fill kernels.
//
// kv_append writes new tokens' K/V into their paged slots (a session's retained KV blocks grow, Sec. 3.2
// of the paper); kv_gather reads tokens back in logical order.  Both work on (page run, kv head) units:
// one wave moves every token of one sequence that lands in one page, for one KV head, so each unit's
// writes are whole 16-byte chunks of a single 8 KB page block.
#include <algorithm>

#include "kvp_kernels.h"
#include "kvp_layout.h"
#include "rope_dev.h"

namespace kvp {

namespace {

// Pool writes are streaming stores: left as ordinary dirty lines in the caches, the scattered page
// blocks of a large append slow the next decode's streaming reads when they are evicted.
__device__ __forceinline__ void store_stream(uint16_t* p, uint4 v) {
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p));
}

// A wave writes the V block's slots of run r from its tokens' rows in vs [slot][dim]: 2*D chunks, chunk (dt, h, c) holds
// slots 8h..8h+7 of dim 16*dt + c.
template <int D>
__device__ __forceinline__ void put_v(const PageRun& r, const uint16_t* vs, uint16_t* vblk, int lane) {
  for (int e = lane; e < 2 * D; e += 64) {
    const int c = e & 15, h = (e >> 4) & 1, dt = e >> 5;
    const int dim = dt * 16 + c;
    uint16_t* dst = vblk + v_index<D>(/*token of slot 8h*/ slot_token(8 * h), dim);
    bool any = false, all = true;
    for (int j = 0; j < 8; ++j) {
      const int t = slot_token(8 * h + j);
      const bool in = t >= r.s_lo && t < r.s_hi;
      any |= in;
      all &= in;
    }
    if (!any) continue;
    union { uint4 u; uint16_t s[8]; } val;
    if (!all) val.u = *reinterpret_cast<const uint4*>(dst);
    for (int j = 0; j < 8; ++j) {
      const int t = slot_token(8 * h + j);
      if (t >= r.s_lo && t < r.s_hi) val.s[j] = vs[t * D + dim];
    }
    store_stream(dst, val.u);
  }
}

template <int D>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  __shared__ uint16_t vstage[4][16 * D];  // one page of V tokens per wave, [slot][dim]
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + w;
  const int run = unit / a.Hkv, head = unit - run * a.Hkv;
  if (run >= a.n_runs) return;
  const PageRun r = a.runs[run];
  const int id = a.bt[(int64_t)r.row * a.maxp + r.lpage];
  if ((unsigned)id >= (unsigned)a.num_pages) {
    if (lane == 0) atomicCAS(a.err, 0, KVP_ERANGE);
    return;
  }
  uint16_t* kblk = a.layer + ((int64_t)id * a.Hkv + head) * (2 * 16 * D);
  uint16_t* vblk = kblk + 16 * D;
  constexpr int CH = D / 8;  // 16-byte chunks per token row
  const int ntok = r.s_hi - r.s_lo;
  uint16_t* vs = vstage[w];
  for (int e = lane; e < ntok * CH; e += 64) {
    const int tt = e / CH, c8 = e - tt * CH;
    const int64_t src = ((r.src0 + tt) * a.Hkv + head) * D + c8 * 8;
    const uint4 kk = *reinterpret_cast<const uint4*>(a.k + src);
    const uint4 vv = *reinterpret_cast<const uint4*>(a.v + src);
    const int s = r.s_lo + tt;
    store_stream(kblk + k_index<D>(s, c8 * 8), kk);
    *reinterpret_cast<uint4*>(vs + s * D + c8 * 8) = vv;
  }
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  put_v<D>(r, vs, vblk, lane);
}

// ---------------------------------------------------------------------------------------------------
// FP8 (OCP E4M3) pools: y = fp32(x) * inv_scale is rounded to the nearest E4M3 value, ties to the even
// mantissa, saturating at +-448; NaN stays NaN and keeps its sign.  The conversion instruction rounds so;
// it does not saturate, and sets the sign of every NaN.
// ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned e4m3_pair(float x, float y) {  // codes of x and y in the low two bytes
  const float a = x != x ? x : __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f);
  const float b = y != y ? y : __builtin_amdgcn_fmed3f(y, -448.0f, 448.0f);
  const unsigned sign = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x0c0c0703u);  // their top bytes
  return ((unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0x7f7fu) | (sign & 0x8080u);
}
__device__ __forceinline__ unsigned e4m3_code(float y) { return e4m3_pair(y, y) & 0xffu; }

__device__ __forceinline__ float bf16_to_f32(uint16_t b) { return __uint_as_float((unsigned)b << 16); }

// Quantised codes of 8 bf16 elements, packed little-endian into two words.
__device__ __forceinline__ uint2 quant8(uint4 x, float inv) {
  const uint16_t* h = reinterpret_cast<const uint16_t*>(&x);
  unsigned w[2] = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 8; j += 2)
    w[j >> 2] |= e4m3_pair(bf16_to_f32(h[j]) * inv, bf16_to_f32(h[j + 1]) * inv) << (8 * (j & 3));
  return make_uint2(w[0], w[1]);
}

// As put_v, quantised.  D pieces of 16 bytes; piece (Y, h, cc) holds slots 8h..8h+7 of dims 32Y + cc and 32Y + 16 + cc.
template <int D>
__device__ __forceinline__ void put_v_fp8(const PageRun& r, const uint16_t* vs, uint8_t* vblk, float inv_scale, int lane) {
  for (int e = lane; e < D; e += 64) {
    const int cc = e & 15, h = (e >> 4) & 1, Y = e >> 5;
    uint8_t* dst = vblk + ((Y * 2 + h) * 16 + cc) * 16;
    bool any = false, all = true;
    for (int j = 0; j < 8; ++j) {
      const int t = slot_token(8 * h + j);
      const bool in = t >= r.s_lo && t < r.s_hi;
      any |= in;
      all &= in;
    }
    if (!any) continue;
    union { uint4 u; uint8_t b[16]; } val;
    if (!all) val.u = *reinterpret_cast<const uint4*>(dst);
    for (int dh = 0; dh < 2; ++dh)
      for (int j = 0; j < 8; j += 2) {
        const int dim = 32 * Y + 16 * dh + cc, t0 = slot_token(8 * h + j), t1 = slot_token(8 * h + j + 1);
        const unsigned codes = e4m3_pair(bf16_to_f32(vs[t0 * D + dim]) * inv_scale, bf16_to_f32(vs[t1 * D + dim]) * inv_scale);
        if (t0 >= r.s_lo && t0 < r.s_hi) val.b[dh * 8 + j] = (uint8_t)codes;
        if (t1 >= r.s_lo && t1 < r.s_hi) val.b[dh * 8 + j + 1] = (uint8_t)(codes >> 8);
      }
    store_stream(reinterpret_cast<uint16_t*>(dst), val.u);
  }
}

template <int D>
__global__ __launch_bounds__(256) void append_fp8_kernel(AppendArgs a) {
  __shared__ uint16_t vstage[4][16 * D];  // one page of V tokens per wave, [token][dim] bf16
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + w;
  const int run = unit / a.Hkv, head = unit - run * a.Hkv;
  if (run >= a.n_runs) return;
  const PageRun r = a.runs[run];
  const int id = a.bt[(int64_t)r.row * a.maxp + r.lpage];
  if ((unsigned)id >= (unsigned)a.num_pages) {
    if (lane == 0) atomicCAS(a.err, 0, KVP_ERANGE);
    return;
  }
  uint8_t* kblk = reinterpret_cast<uint8_t*>(a.layer) + ((int64_t)id * a.Hkv + head) * (2 * 16 * D);
  uint8_t* vblk = kblk + 16 * D;
  const int ntok = r.s_hi - r.s_lo;
  // K: one 16-byte piece per (token, X): dims 64(X/4) + 8(X%4) + j, then the same + 32.
  constexpr int NX = D / 16;
  for (int e = lane; e < ntok * NX; e += 64) {
    const int tt = e / NX, X = e - tt * NX;
    const int c0 = 64 * (X >> 2) + 8 * (X & 3);
    const int64_t src = ((r.src0 + tt) * a.Hkv + head) * D;
    const uint2 lo = quant8(*reinterpret_cast<const uint4*>(a.k + src + c0), a.inv_scale_k);
    const uint2 hi = quant8(*reinterpret_cast<const uint4*>(a.k + src + c0 + 32), a.inv_scale_k);
    store_stream(reinterpret_cast<uint16_t*>(kblk + (X * 16 + r.s_lo + tt) * 16), make_uint4(lo.x, lo.y, hi.x, hi.y));
  }
  uint16_t* vs = vstage[w];
  constexpr int CH = D / 8;
  for (int e = lane; e < ntok * CH; e += 64) {
    const int tt = e / CH, c8 = e - tt * CH;
    const int64_t src = ((r.src0 + tt) * a.Hkv + head) * D + c8 * 8;
    *reinterpret_cast<uint4*>(vs + (r.s_lo + tt) * D + c8 * 8) = *reinterpret_cast<const uint4*>(a.v + src);
  }
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  put_v_fp8<D>(r, vs, vblk, a.inv_scale_v, lane);
}

// bf16(fp32(code value) * scale) of the two codes in half `hi` of w.
__device__ __forceinline__ unsigned dequant2(unsigned w, bool hi, float scale) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 v = hi ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  bf2 b;
  b[0] = (__bf16)(v[0] * scale);
  b[1] = (__bf16)(v[1] * scale);
  return __builtin_bit_cast(unsigned, b);
}

template <int D>
__global__ __launch_bounds__(256) void gather_fp8_kernel(GatherArgs a) {
  __shared__ uint8_t vblock[4][16 * D];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + w;
  const int run = unit / a.Hkv, head = unit - run * a.Hkv;
  if (run >= a.n_runs) return;
  const PageRun r = a.runs[run];
  const int id = a.bt[(int64_t)r.row * a.maxp + r.lpage];
  const bool ok = (unsigned)id < (unsigned)a.num_pages;
  if (!ok && lane == 0) atomicCAS(a.err, 0, KVP_ERANGE);
  const uint8_t* kblk = reinterpret_cast<const uint8_t*>(a.layer) + ((int64_t)(ok ? id : 0) * a.Hkv + head) * (2 * 16 * D);
  const uint8_t* vblk = kblk + 16 * D;
  uint8_t* vb = vblock[w];
  for (int e = lane; e < D; e += 64)
    *reinterpret_cast<uint4*>(vb + e * 16) = *reinterpret_cast<const uint4*>(vblk + e * 16);
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  constexpr int CH = D / 8;
  const int ntok = r.s_hi - r.s_lo;
  for (int e = lane; e < ntok * CH; e += 64) {
    const int tt = e / CH, c8 = e - tt * CH;
    const int s = r.s_lo + tt;
    const int64_t dst = ((r.src0 + tt) * a.Hkv + head) * D + c8 * 8;
    uint4 kk = make_uint4(0, 0, 0, 0), vv = make_uint4(0, 0, 0, 0);
    if (ok) {
      const uint2 kc = *reinterpret_cast<const uint2*>(kblk + k8_index<D>(s, c8 * 8));  // 8 consecutive dims
      kk = make_uint4(dequant2(kc.x, false, a.scale_k), dequant2(kc.x, true, a.scale_k),
                      dequant2(kc.y, false, a.scale_k), dequant2(kc.y, true, a.scale_k));
      unsigned vw[2] = {0u, 0u};
      for (int j = 0; j < 8; ++j) vw[j >> 2] |= (unsigned)vb[v8_index<D>(s, c8 * 8 + j)] << (8 * (j & 3));
      vv = make_uint4(dequant2(vw[0], false, a.scale_v), dequant2(vw[0], true, a.scale_v),
                      dequant2(vw[1], false, a.scale_v), dequant2(vw[1], true, a.scale_v));
    }
    *reinterpret_cast<uint4*>(a.k + dst) = kk;
    *reinterpret_cast<uint4*>(a.v + dst) = vv;
  }
}

template <int D>
__global__ __launch_bounds__(256) void gather_kernel(GatherArgs a) {
  __shared__ uint16_t vblock[4][16 * D];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + w;
  const int run = unit / a.Hkv, head = unit - run * a.Hkv;
  if (run >= a.n_runs) return;
  const PageRun r = a.runs[run];
  const int id = a.bt[(int64_t)r.row * a.maxp + r.lpage];
  const bool ok = (unsigned)id < (unsigned)a.num_pages;
  if (!ok && lane == 0) atomicCAS(a.err, 0, KVP_ERANGE);
  const uint16_t* kblk = a.layer + ((int64_t)(ok ? id : 0) * a.Hkv + head) * (2 * 16 * D);
  const uint16_t* vblk = kblk + 16 * D;
  uint16_t* vb = vblock[w];
  for (int e = lane; e < 2 * D; e += 64)
    *reinterpret_cast<uint4*>(vb + e * 8) = *reinterpret_cast<const uint4*>(vblk + e * 8);
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  constexpr int CH = D / 8;
  const int ntok = r.s_hi - r.s_lo;
  for (int e = lane; e < ntok * CH; e += 64) {
    const int tt = e / CH, c8 = e - tt * CH;
    const int s = r.s_lo + tt;
    const int64_t dst = ((r.src0 + tt) * a.Hkv + head) * D + c8 * 8;
    uint4 kk = ok ? *reinterpret_cast<const uint4*>(kblk + k_index<D>(s, c8 * 8)) : make_uint4(0, 0, 0, 0);
    union { uint4 u; uint16_t s[8]; } vv;
    for (int j = 0; j < 8; ++j) vv.s[j] = ok ? vb[v_index<D>(s, c8 * 8 + j)] : 0;
    *reinterpret_cast<uint4*>(a.k + dst) = kk;
    *reinterpret_cast<uint4*>(a.v + dst) = vv.u;
  }
}

// kv_append_rope.  One wave per (page run, KV head) turns the keys and writes both blocks; one per (page run, some query
// heads) turns the queries of the same tokens.  A lane holds a unit of 8 dims of one token (in the half layout 8 more,
// R / 2 further or the next ones that are not rotated), computes its sines and cosines once and uses them for all of the
// wave's heads; a run of few tokens spreads the heads over the lanes.  Bandwidth is what bounds it: 16416 tokens of 32 + 4
// heads of 128 (336 MB) take 64 us, 5.3 TB/s where a copy reaches 5.1; 3567 tokens into FP8 pages 15.4 us, 4.5 TB/s.
// A step of 512 single tokens (11 us for 10.5 MB) is a chain of waits: a key wave's for its run record in pinned host memory
// (in two trips), the page id, the row of v, the row of k, the rotation's table, then put_v's D / 32 rounds of pieces, which
// are read, changed and written one round after the other (with one token in the page 2 bytes of each 16: 9.7 MB read and 9.4
// written in all).
//
// Query heads of a wave: 8, or 4 in the interleaved layout (whose waves take twice the passes over a run) where the waves
// of a call have room beside each other.  4160 tokens with 8 / 4: 32 + 2 heads interleaved 18.1 / 17.0 us, 8 + 8 17.0 /
// 15.0; 32 + 8 heads 19.8 / 21.3, not interleaved 20.9 / 23.9; FP8 with 2 for the 3567 tokens 17.2.
constexpr int kQueryHeads = 8, kFewQueryHeads = 4, kFewWaves = 4096;

template <int D, bool F8, bool IL, bool Stream>
__global__ __launch_bounds__(256) void append_rope_kernel(AppendRopeArgs r) {
  __shared__ uint16_t vstage[4][16 * D];
  const AppendArgs& a = r.kv;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  // The waves for queries first, then those for keys: taken in turn, workgroups of one kind met on every other XCD.
  unsigned unit = blockIdx.x * 4u + w;
  const bool key = unit >= r.q_units;
  if (key) unit -= r.q_units;
  const FastDiv& by = key ? r.by_keys : r.by_queries;
  const unsigned run = by.quotient(unit);
  const int slot = (int)(unit - run * by.d);
  if (run >= (unsigned)a.n_runs) return;
  const PageRun pr = a.runs[run];
  const int ntok = pr.s_hi - pr.s_lo;
  // Units of a token and head: 8 dims; in the half layout 8 and 8 more, `next` further.
  constexpr int units = IL ? D / 8 : D / 16;
  const int R = r.table.rotary_dim, turned = IL ? R / 8 : R / 16;
  const int width = ntok * units > 32 ? 64 : ntok * units > 16 ? 32 : ntok * units > 8 ? 16 : 8;

  if (!key) {
    const int h_lo = slot * r.q_heads, h_hi = min(h_lo + r.q_heads, r.Hq);
    const int across = 64 / width;  // heads at a time
    for (int e = lane & (width - 1); e < ntok * units; e += width) {
      const int tt = e / units, u = e % units;
      const int64_t tok = pr.src0 + tt;
      const bool pass = u >= turned;
      const int i0 = IL ? 8 * u : pass ? 16 * u : 8 * u, next = pass ? 8 : R / 2;
      const uint16_t* x = r.q + tok * r.q_stride + i0;
      uint16_t* y = r.q_out + tok * r.q_out_stride + i0;
      Turns<IL ? 4 : 8> t;
      if (!pass) t.set(r.table, IL ? u * 4 : u * 8, pr.lpage * 16 + pr.s_lo + tt);
      constexpr int N = 2;  // heads whose loads are under way together
      for (int h = h_lo + lane / width; h < h_hi; h += N * across) {
        Eight p[N], q[N];
#pragma unroll
        for (int n = 0; n < N; ++n)
          if (h + n * across < h_hi) {
            p[n].template load<Stream>(x + (h + n * across) * D);
            if (!IL) q[n].template load<Stream>(x + (h + n * across) * D + next);
          }
#pragma unroll
        for (int n = 0; n < N; ++n)
          if (h + n * across < h_hi) {
            if (!pass) {
              if constexpr (IL) turn_neighbours(p[n], t);
              else turn_halves(p[n], q[n], t);
            }
            p[n].store(y + (h + n * across) * D);
            if (!IL) q[n].store(y + (h + n * across) * D + next);
          }
      }
    }
    return;
  }

  const int id = a.bt[(int64_t)pr.row * a.maxp + pr.lpage];
  if ((unsigned)id >= (unsigned)a.num_pages) {
    if (lane == 0) atomicCAS(a.err, 0, KVP_ERANGE);
    return;
  }
  const int64_t block = ((int64_t)id * a.Hkv + slot) * (2 * 16 * D);
  uint8_t* const b8 = reinterpret_cast<uint8_t*>(a.layer) + block;
  uint16_t* const b16 = a.layer + block;
  auto put_k = [&](int s, int c, const Eight& v) {  // 8 dims of a token: 16 bytes, or 8 codes
    if (F8) {
      unsigned code[2] = {0u, 0u};
#pragma unroll
      for (int j = 0; j < 8; j += 2)
        code[j >> 2] |= e4m3_pair(v.x[j] * a.inv_scale_k, v.x[j + 1] * a.inv_scale_k) << (8 * (j & 3));
      *reinterpret_cast<uint2*>(b8 + k8_index<D>(s, c)) = make_uint2(code[0], code[1]);
    } else {
      store_stream(b16 + k_index<D>(s, c), v.bf16());
    }
  };
  uint16_t* vs = vstage[w];
  constexpr int CH = D / 8;
  for (int e = lane; e < ntok * CH; e += 64) {
    const int tt = e / CH, c8 = e - tt * CH;
    const Eight::u32x4* const at =
        reinterpret_cast<const Eight::u32x4*>(a.v + (pr.src0 + tt) * r.v_stride + slot * D + c8 * 8);
    *reinterpret_cast<Eight::u32x4*>(vs + (pr.s_lo + tt) * D + c8 * 8) = Stream ? __builtin_nontemporal_load(at) : *at;
  }
  for (int e = lane; e < ntok * units; e += 64) {
    const int tt = e / units, u = e % units, s = pr.s_lo + tt;
    const uint16_t* x = a.k + (pr.src0 + tt) * r.k_stride + slot * D;
    const bool pass = u >= turned;
    const int i0 = IL ? 8 * u : pass ? 16 * u : 8 * u, next = pass ? 8 : R / 2;
    Eight p, q;
    p.template load<Stream>(x + i0);
    if (!IL) q.template load<Stream>(x + i0 + next);
    if (!pass) {
      Turns<IL ? 4 : 8> t;
      t.set(r.table, IL ? u * 4 : u * 8, pr.lpage * 16 + s);
      if constexpr (IL) turn_neighbours(p, t);
      else turn_halves(p, q, t);
    }
    put_k(s, i0, p);
    if (!IL) put_k(s, i0 + next, q);
  }
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  if (F8) put_v_fp8<D>(pr, vs, b8 + 16 * D, a.inv_scale_v, lane);
  else put_v<D>(pr, vs, b16 + 16 * D, lane);
}

// kv_append_rope of a rotary_dim that is not made of whole units: one wave per (page run, head), the KV heads first, then
// the query heads of the same tokens.  A lane turns pairs of one head's dims; a dim that is not rotated is a unit too.
template <int D, bool F8>
__global__ __launch_bounds__(256) void append_rope_pair_kernel(AppendRopeArgs r) {
  const AppendArgs& a = r.kv;
  const int lane = threadIdx.x & 63;
  const unsigned unit = blockIdx.x * 4u + (threadIdx.x >> 6), run = r.by_slots.quotient(unit);
  const int h = (int)(unit - run * r.by_slots.d);
  if (run >= (unsigned)a.n_runs) return;
  const PageRun pr = a.runs[run];
  const int ntok = pr.s_hi - pr.s_lo;
  const bool key = h < a.Hkv;
  int64_t block = 0;
  if (key) {
    const int id = a.bt[(int64_t)pr.row * a.maxp + pr.lpage];
    if ((unsigned)id >= (unsigned)a.num_pages) {
      if (lane == 0) atomicCAS(a.err, 0, KVP_ERANGE);
      return;
    }
    block = ((int64_t)id * a.Hkv + h) * (2 * 16 * D);
  }
  uint8_t* const b8 = reinterpret_cast<uint8_t*>(a.layer) + block;
  uint16_t* const b16 = a.layer + block;
  const int R = r.table.rotary_dim, units = D - R / 2;
  for (int e = lane; e < ntok * units; e += 64) {
    const int tt = e / units, u = e - tt * units, s = pr.s_lo + tt;
    const int64_t tok = pr.src0 + tt;
    const uint16_t* x = key ? a.k + tok * r.k_stride + h * D : r.q + tok * r.q_stride + (h - a.Hkv) * D;
    const bool pair = u < R / 2;
    const int i0 = !pair ? u + R / 2 : r.table.interleaved ? 2 * u : u;
    const int i1 = !pair ? i0 : r.table.interleaved ? 2 * u + 1 : u + R / 2;
    float y0 = widen(x[i0]), y1 = y0;
    if (pair) {
      float sn, cs;
      pair_turn(r.table, u, pr.lpage * 16 + s, &sn, &cs);
      turn(y0, widen(x[i1]), sn, cs, &y0, &y1);
    }
    if (!key) {
      uint16_t* o = r.q_out + tok * r.q_out_stride + (h - a.Hkv) * D;
      o[i0] = narrow(y0);
      o[i1] = narrow(y1);
    } else if (F8) {
      b8[k8_index<D>(s, i0)] = (uint8_t)e4m3_code(y0 * a.inv_scale_k);
      b8[k8_index<D>(s, i1)] = (uint8_t)e4m3_code(y1 * a.inv_scale_k);
    } else {
      b16[k_index<D>(s, i0)] = narrow(y0);
      b16[k_index<D>(s, i1)] = narrow(y1);
    }
  }
  if (!key) return;
  for (int e = lane; e < ntok * D; e += 64) {
    const int tt = e / D, c = e - tt * D, s = pr.s_lo + tt;
    const uint16_t v = a.v[(pr.src0 + tt) * r.v_stride + h * D + c];
    if (F8) b8[16 * D + v8_index<D>(s, c)] = (uint8_t)e4m3_code(widen(v) * a.inv_scale_v);
    else b16[16 * D + v_index<D>(s, c)] = v;
  }
}

__global__ void fill_zero_kernel(uint4* p, size_t n16) {
  const size_t stride = (size_t)gridDim.x * blockDim.x;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += stride) p[i] = make_uint4(0, 0, 0, 0);
}

// Copy n bytes from pinned host memory to device memory: 16-byte pieces read over the host link by the
// threads of the grid, the last n mod 16 bytes by one thread.  It runs on the compute queue in stream
// order, so the kernel after it needs no hand-off from the copy engine.
__global__ __launch_bounds__(256) void copy_from_host_kernel(unsigned char* dst, const unsigned char* src, size_t n) {
  const size_t n16 = n / 16;
  const size_t stride = (size_t)gridDim.x * blockDim.x;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += stride)
    reinterpret_cast<uint4*>(dst)[i] = reinterpret_cast<const uint4*>(src)[i];
  if (blockIdx.x == 0 && threadIdx.x == 0)
    for (size_t i = n16 * 16; i < n; ++i) dst[i] = src[i];
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, int D, hipStream_t s) {
  const int64_t units = (int64_t)a.n_runs * a.Hkv;
  if (units == 0) return hipSuccess;
  const dim3 grid((unsigned)((units + 3) / 4));
  if (a.fp8) {
    if (D == 128) hipLaunchKernelGGL(append_fp8_kernel<128>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(append_fp8_kernel<64>, grid, dim3(256), 0, s, a);
  } else if (D == 128) {
    hipLaunchKernelGGL(append_kernel<128>, grid, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(append_kernel<64>, grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

template <int D, bool F8>
static void launch_append_rope(const AppendRopeArgs& a, hipStream_t s) {
  const bool whole = a.table.rotary_dim % (a.table.interleaved ? 8 : 16) == 0;
  const int64_t waves = (int64_t)a.kv.n_runs * (a.kv.Hkv + (a.Hq + kFewQueryHeads - 1) / kFewQueryHeads);
  const int q_heads = !whole ? 1 : a.table.interleaved && waves <= kFewWaves ? kFewQueryHeads : kQueryHeads;
  const int q_slots = (a.Hq + q_heads - 1) / q_heads, slots = a.kv.Hkv + q_slots;
  const int most = std::max(1, ((1 << 26) - 4) / slots);  // runs of a launch, which has fewer than 2^32 threads
  AppendRopeArgs b = a;
  // Rows read streamed: 201 MB of them 86 -> 77 us, 151 MB 57 -> 57, 100 MB 40 -> 44 us.
  const bool stream = a.tokens * (a.Hq + 2 * a.kv.Hkv) * D * 2 >= kStreamBytes;
  b.q_heads = q_heads;
  b.by_slots = FastDiv(slots);
  b.by_keys = FastDiv(a.kv.Hkv);
  b.by_queries = FastDiv(std::max(1, q_slots));
  for (int r = 0; r < a.kv.n_runs; r += most) {
    b.kv.runs = a.kv.runs + r;
    b.kv.n_runs = std::min(most, a.kv.n_runs - r);
    b.q_units = (unsigned)b.kv.n_runs * q_slots;
    const dim3 grid((unsigned)(((int64_t)b.kv.n_runs * slots + 3) / 4));
    if (!whole) hipLaunchKernelGGL((append_rope_pair_kernel<D, F8>), grid, dim3(256), 0, s, b);
    else if (stream && a.table.interleaved) hipLaunchKernelGGL((append_rope_kernel<D, F8, true, true>), grid, dim3(256), 0, s, b);
    else if (stream) hipLaunchKernelGGL((append_rope_kernel<D, F8, false, true>), grid, dim3(256), 0, s, b);
    else if (a.table.interleaved) hipLaunchKernelGGL((append_rope_kernel<D, F8, true, false>), grid, dim3(256), 0, s, b);
    else hipLaunchKernelGGL((append_rope_kernel<D, F8, false, false>), grid, dim3(256), 0, s, b);
  }
}

hipError_t launch_append_rope(const AppendRopeArgs& a, int D, hipStream_t s) {
  if (a.kv.n_runs == 0) return hipSuccess;
  if (D == 128) a.kv.fp8 ? launch_append_rope<128, true>(a, s) : launch_append_rope<128, false>(a, s);
  else a.kv.fp8 ? launch_append_rope<64, true>(a, s) : launch_append_rope<64, false>(a, s);
  return hipGetLastError();
}

hipError_t launch_gather(const GatherArgs& a, int D, hipStream_t s) {
  const int64_t units = (int64_t)a.n_runs * a.Hkv;
  if (units == 0) return hipSuccess;
  const dim3 grid((unsigned)((units + 3) / 4));
  if (a.fp8) {
    if (D == 128) hipLaunchKernelGGL(gather_fp8_kernel<128>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(gather_fp8_kernel<64>, grid, dim3(256), 0, s, a);
  } else if (D == 128) {
    hipLaunchKernelGGL(gather_kernel<128>, grid, dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(gather_kernel<64>, grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_copy_from_host(void* dst, const void* src, size_t n, hipStream_t s) {
  if (n == 0) return hipSuccess;
  const unsigned blocks = (unsigned)std::min<size_t>(256, (n / 16 + 255) / 256 + 1);
  hipLaunchKernelGGL(copy_from_host_kernel, dim3(blocks), dim3(256), 0, s, reinterpret_cast<unsigned char*>(dst),
                     reinterpret_cast<const unsigned char*>(src), n);
  return hipGetLastError();
}

hipError_t launch_fill_zero(void* p, size_t bytes, hipStream_t s) {
  const size_t n16 = bytes / 16;
  if (n16 == 0) return hipSuccess;
  const unsigned blocks = (unsigned)std::min<size_t>(8192, (n16 + 255) / 256);
  hipLaunchKernelGGL(fill_zero_kernel, dim3(blocks), dim3(256), 0, s, reinterpret_cast<uint4*>(p), n16);
  return hipGetLastError();
}

}  // namespace kvp
