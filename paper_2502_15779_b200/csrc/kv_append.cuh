// Appending keys and values to the paged 8-bit cache, with the rotation by position on the way (rcp_kv_append).
//
//   rotation   pair (a, b) of a head, pair i of token at position p: (a c - b s, b c + a s), c = cos, s = sin of rope[p][i];
//              fp32, every product and sum rounded once (no fused multiply-add), so that the codes do not depend on a compiler
//   codes      e4m3(x / 2^e), round to nearest even; e as in kv_common.cuh over the block's new tokens, never below the exponent
//              the block has where it holds older tokens, which are rescaled when it grows
//
// Work. One CTA per block that gets new tokens, key head and half (keys, values): the block's scale needs a maximum over its tokens, so
// the new values stay in registers between the maximum and the codes. Blocks are found on the device: a sequence with n new
// tokens touches at most floor(n / page) + 2 of them, so candidate floor(starts[b] / page) + 2 b + j is its j-th, and
// a binary search over starts turns a candidate into its sequence; where max_new is small, seqs * (blocks of max_new tokens) are
// fewer and need no search. Further CTAs rotate queries: a thread takes eight pairs of a token through several heads, so that the
// 64 bytes of cosines are read once for all of them.
#pragma once
#include "common.cuh"
#include "kv_common.cuh"

namespace rcp {

constexpr int kAppendThreads = 128;
constexpr int kQueryHeads = 8;   // heads a thread takes its cosines through

struct AppendParams {
  const __half *q, *k, *v;
  long long q_stride, k_stride, v_stride;   // elements between tokens
  const float2* rope;                       // [positions][rot / 2]
  int rot, interleaved;
  int heads, kv_heads, dim;
  KvSeqs s;
  uint8_t *k_cache, *v_cache;               // [pages][kv_heads][page][dim]
  float *k_scale, *v_scale;                 // [pages][kv_heads]
  __half* q_out;                            // [tokens][heads][dim]
  int candidates, direct;                   // blocks to look at; direct: so many to a sequence (0: by search)
  int query_tokens, query_splits;           // tokens of a query CTA, CTAs that share its heads
};

// sixteen values of a head: a rotation unit is eight pairs (a and b), a plain one sixteen consecutive elements
struct Unit { uint4 a, b; };
// where unit u of a head lies: first elements of its halves and of its pairs (pair < 0: not rotated)
struct UnitAt { int a, b, pair; };
__device__ __forceinline__ UnitAt unit_at(int u, int rot, int interleaved) {
  if (16 * u >= rot) return {16 * u, 16 * u + 8, -1};
  if (interleaved) return {16 * u, 16 * u + 8, 8 * u};
  return {8 * u, rot / 2 + 8 * u, 8 * u};
}
__device__ __forceinline__ void unpack8(uint4 v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
// the unit's sixteen values in the order of its two halves, rotated by cs (eight pairs) if it is a rotation unit
__device__ __forceinline__ void unit_values(const Unit& in, bool rotated, int interleaved, const float2 (&cs)[8], float (&x)[8], float (&y)[8]) {
  unpack8(in.a, x);
  unpack8(in.b, y);
  if (!rotated) return;
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      float& p = i < 4 ? x[2 * i] : y[2 * i - 8];
      float& r = i < 4 ? x[2 * i + 1] : y[2 * i - 7];
      const float a = p, b = r;
      p = __fsub_rn(__fmul_rn(a, cs[i].x), __fmul_rn(b, cs[i].y));
      r = __fadd_rn(__fmul_rn(b, cs[i].x), __fmul_rn(a, cs[i].y));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float a = x[i], b = y[i];
      x[i] = __fsub_rn(__fmul_rn(a, cs[i].x), __fmul_rn(b, cs[i].y));
      y[i] = __fadd_rn(__fmul_rn(b, cs[i].x), __fmul_rn(a, cs[i].y));
    }
  }
}
__device__ __forceinline__ void load_pairs(const float2* at, float2 (&cs)[8]) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(at) + i);
    cs[2 * i] = make_float2(v.x, v.y);
    cs[2 * i + 1] = make_float2(v.z, v.w);
  }
}
// finite, NaN as zero: one bad number does not spoil its block
__device__ __forceinline__ float kv_finite(float x) { return x == x ? fminf(fmaxf(x, -kKvCap), kKvCap) : 0.f; }
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float inv) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; i++) w[i] = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i] * inv, x[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}
// four codes times a power of two
__device__ __forceinline__ uint32_t rescale4(uint32_t c, float f) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c >> (16 * i)), __NV_E4M3);
    const float2 v = __half22float2(__half2(h));
    r |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v.x * f, v.y * f), __NV_SATFINITE, __NV_E4M3) << (16 * i);
  }
  return r;
}

__device__ __forceinline__ void rotate_queries(const AppendParams& p, int cta) {
  const int upt = p.dim / 16;   // units of a head
  const int split = cta % p.query_splits;
  const int h0 = (int)((long long)p.heads * split / p.query_splits), h1 = (int)((long long)p.heads * (split + 1) / p.query_splits);
  const int t = (cta / p.query_splits) * p.query_tokens + (int)threadIdx.x / upt, u = (int)threadIdx.x % upt;
  if ((int)threadIdx.x >= p.query_tokens * upt || t >= p.s.tokens || t >= p.s.starts[p.s.seqs] || t < p.s.starts[0]) return;
  const KvSeq sq = kv_seq(p.s, kv_find(p.s.starts, p.s.seqs, t));
  const int i = t - sq.t0, pos = sq.first + i;
  if (i < 0 || i >= sq.n) return;
  const bool known = pos >= 0 && pos < sq.end;
  const UnitAt at = unit_at(u, p.rot, p.interleaved);
  float2 cs[8];
  if (known && at.pair >= 0) load_pairs(p.rope + (long long)pos * (p.rot / 2) + at.pair, cs);
  const __half* src = p.q + (long long)t * p.q_stride;
  __half* dst = p.q_out + (long long)t * p.heads * p.dim;
#pragma unroll 4
  for (int h = h0; h < h1; h++) {
    const Unit in{*reinterpret_cast<const uint4*>(src + h * p.dim + at.a), *reinterpret_cast<const uint4*>(src + h * p.dim + at.b)};
    float x[8], y[8];
    unit_values(in, known && at.pair >= 0, p.interleaved, cs, x, y);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const __half2 lo = __floats2half2_rn(x[2 * j], x[2 * j + 1]), hi = __floats2half2_rn(y[2 * j], y[2 * j + 1]);
      w[j] = known ? *reinterpret_cast<const uint32_t*>(&lo) : 0u;
      w[4 + j] = known ? *reinterpret_cast<const uint32_t*>(&hi) : 0u;
    }
    *reinterpret_cast<uint4*>(dst + h * p.dim + at.a) = make_uint4(w[0], w[1], w[2], w[3]);
    *reinterpret_cast<uint4*>(dst + h * p.dim + at.b) = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// UNITS: units of sixteen values a thread holds of a block, page * dim / 16 / kAppendThreads
template <int UNITS>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const AppendParams p) {
  __shared__ uint32_t s_max[kAppendThreads / 32];
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int per = 2 * p.kv_heads, cand = (int)blockIdx.x / per;
  if (cand >= p.candidates) {
    rotate_queries(p, (int)blockIdx.x - p.candidates * per);
    return;
  }
  const int which = (int)blockIdx.x - cand * per, head = which >> 1, tid = (int)threadIdx.x;
  const bool keys = (which & 1) == 0;
  int b, j;
  if (p.direct) {
    b = cand / p.direct;
    j = cand - b * p.direct;
  } else {
    int lo = 0, hi = p.s.seqs;   // the last sequence whose candidates start at or in front of this one
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((p.s.starts[mid] >> p.s.lg_page) + 2 * mid <= cand) lo = mid; else hi = mid;
    }
    b = lo;
    j = cand - ((p.s.starts[b] >> p.s.lg_page) + 2 * b);
  }
  const KvSeq sq = kv_seq(p.s, b);
  // positions of the sequence's new tokens that exist, and the part of them in this block
  const int lo = max(sq.first, 0), hi = min(sq.first + sq.n, sq.end);
  if (j < 0 || lo >= hi) return;
  const int blk = (lo >> p.s.lg_page) + j, base = blk << p.s.lg_page;
  if (blk >= p.s.width || base >= hi) return;
  const int from = max(lo, base) - base, to = min(hi - base, p.s.page);   // new slots
  const int pg = p.s.table[(long long)b * p.s.width + blk];
  if (pg < 0 || pg >= p.s.pages) return;
  const long long block = (long long)pg * p.kv_heads + head;
  uint8_t* const codes = (keys ? p.k_cache : p.v_cache) + block * p.s.page * p.dim;
  float* const scale = (keys ? p.k_scale : p.v_scale) + block;
  const int e_old = from > 0 ? kv_stored_exponent(*scale) : kKvExpMin;
  const long long stride = keys ? p.k_stride : p.v_stride;
  const __half* const src = (keys ? p.k : p.v) + (long long)head * p.dim;
  const int rot = keys && p.rope ? p.rot : 0, lg_upt = p.dim == 64 ? 2 : 3, total = (to - from) << lg_upt;
  Unit in[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; i++) {
    const int n = tid + i * kAppendThreads, slot = from + (n >> lg_upt);
    const UnitAt at = unit_at(n & ((1 << lg_upt) - 1), rot, p.interleaved);
    if (n < total) {
      const __half* const row = src + (long long)(sq.t0 + base + slot - sq.first) * stride;
      in[i] = {*reinterpret_cast<const uint4*>(row + at.a), *reinterpret_cast<const uint4*>(row + at.b)};
    }
  }
  // once for the largest magnitude, once for the codes: the rotation is cheaper to repeat than 32 registers a unit are to keep
  auto values = [&](int i, float (&x)[8], float (&y)[8], UnitAt& at, int& slot) {
    const int n = tid + i * kAppendThreads;
    slot = from + (n >> lg_upt);
    at = unit_at(n & ((1 << lg_upt) - 1), rot, p.interleaved);
    float2 cs[8];
    if (at.pair >= 0) load_pairs(p.rope + (long long)(base + slot) * (p.rot / 2) + at.pair, cs);
    unit_values(in[i], at.pair >= 0, p.interleaved, cs, x, y);
#pragma unroll
    for (int k = 0; k < 8; k++) {
      x[k] = kv_finite(x[k]);
      y[k] = kv_finite(y[k]);
    }
  };
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < UNITS; i++) {
    if (tid + i * kAppendThreads >= total) break;
    float x[8], y[8];
    UnitAt at;
    int slot;
    values(i, x, y, at, slot);
#pragma unroll
    for (int k = 0; k < 8; k++) amax = fmaxf(amax, fmaxf(fabsf(x[k]), fabsf(y[k])));
  }
  const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(amax));
  if ((tid & 31) == 0) s_max[tid >> 5] = top;
  __syncthreads();
  uint32_t all = s_max[0];
#pragma unroll
  for (int w = 1; w < kAppendThreads / 32; w++) all = max(all, s_max[w]);
  const int e_new = max(kv_exponent(__uint_as_float(all)), e_old);
  const float inv = kv_pow2(-e_new);
#pragma unroll
  for (int i = 0; i < UNITS; i++) {
    if (tid + i * kAppendThreads >= total) break;
    float x[8], y[8];
    UnitAt at;
    int slot;
    values(i, x, y, at, slot);
    uint8_t* const row = codes + slot * p.dim;
    *reinterpret_cast<uint2*>(row + at.a) = codes8(x, inv);
    *reinterpret_cast<uint2*>(row + at.b) = codes8(y, inv);
  }
  if (from > 0 && e_new > e_old) {   // the older tokens of the block, to its new scale
    const float f = kv_pow2(e_old - e_new);
    for (int n = tid; n < from * p.dim / 16; n += kAppendThreads) {
      uint4 c = reinterpret_cast<const uint4*>(codes)[n];
      c.x = rescale4(c.x, f); c.y = rescale4(c.y, f); c.z = rescale4(c.z, f); c.w = rescale4(c.w, f);
      reinterpret_cast<uint4*>(codes)[n] = c;
    }
  }
  if (tid == 0 && (from == 0 || e_new > e_old)) *scale = kv_pow2(e_new);
}

}  // namespace rcp
