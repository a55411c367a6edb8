// Appending keys and values to the paged 8-bit cache, with the rotation by position on the way (rcp_kv_append).
//
//   rotation   pair (a, b) of a head, pair i of token at position p: (a c - b s, b c + a s), c = cos, s = sin of rope[p][i];
//              fp32, every product and sum rounded once (no fused multiply-add), so that the codes do not depend on a compiler
//   codes      e4m3(x / 2^e), round to nearest even; e as in kv_common.cuh over the block's new tokens, never below the exponent
//              the block has where it holds older tokens, which are rescaled when it grows
//
// kv_append_kernel: one CTA per block that gets new tokens, key head and half (keys, values). The block's scale needs a maximum over its
// tokens, so the values, rotated, stay in registers between the maximum and the codes. Blocks are found on the device: a sequence with n
// new tokens touches at most floor(n / page) + 2 of them, so candidate floor(starts[b] / page) + 2 b + j is its j-th, and
// a binary search over starts turns a candidate into its sequence; where max_new is small, seqs * (blocks of max_new tokens) are
// fewer and need no search. Prompts of 6100 tokens in all, 32 heads on 8 of 128: 36 us with the queries (3.8 TB/s), 14.6 without (2.6): latency and
// what is in flight (a chain of five loads a CTA, 24 warps an SM). Rotating twice, for the maximum and for the codes, instead of keeping the
// values: 40 us.
// kv_append_one_kernel: one new token a sequence at most (max_new 1), as in decoding. Bound by latency: three loads that depend on one another. A
// warp has four (dim 128) or eight (64) blocks of a sequence, sixteen values a lane; a block whose scale grows is rescaled by the
// whole warp. One sequence 2.3 us, 128 sequences with 64 heads on 8 of 128 4.3 (one CTA of the other kernel a block: 10.4).
// In both, further CTAs rotate queries: a thread takes eight pairs of a token through several heads, so that the 64 bytes of
// cosines are read once for all of them.
// Numbers that are not finite or above kKvCap are looked for with the maximum (which keeps NaN); only where there are some the values
// are cut off one by one.
#pragma once
#include "common.cuh"
#include "kv_common.cuh"

namespace rcp {

constexpr int kAppendThreads = 128;   // (of kv_append_one_kernel, and of query CTAs in it)

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
  int query_splits;                         // CTAs that share the heads of a query CTA's tokens
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
// Two fp32 products at a time, each rounded. (Sums and differences of them one by one: a packed addition behind a packed product is
// made one operation with one rounding, although both say .rn.)
__device__ __forceinline__ float2 mul2_rn(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
// the unit's sixteen values in the order of its two halves, rotated by cs (eight pairs) if it is a rotation unit
__device__ __forceinline__ void unit_values(const Unit& in, bool rotated, int interleaved, const float2 (&cs)[8], float (&x)[8], float (&y)[8]) {
  unpack8(in.a, x);
  unpack8(in.b, y);
  if (!rotated) return;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {   // two pairs (a, b) at a time
    float &a0 = interleaved ? (i < 4 ? x[2 * i] : y[2 * i - 8]) : x[i], &b0 = interleaved ? (i < 4 ? x[2 * i + 1] : y[2 * i - 7]) : y[i];
    float &a1 = interleaved ? (i < 4 ? x[2 * i + 2] : y[2 * i - 6]) : x[i + 1], &b1 = interleaved ? (i < 4 ? x[2 * i + 3] : y[2 * i - 5]) : y[i + 1];
    const float2 a = make_float2(a0, a1), b = make_float2(b0, b1), c = make_float2(cs[i].x, cs[i + 1].x), s = make_float2(cs[i].y, cs[i + 1].y);
    const float2 ac = mul2_rn(a, c), bs = mul2_rn(b, s), bc = mul2_rn(b, c), as = mul2_rn(a, s);
    a0 = __fsub_rn(ac.x, bs.x); a1 = __fsub_rn(ac.y, bs.y);
    b0 = __fadd_rn(bc.x, as.x); b1 = __fadd_rn(bc.y, as.y);
  }
}
// largest magnitude, NaN if there is one
__device__ __forceinline__ float max_abs(float top, const float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float a = fabsf(x[i]), b = fabsf(x[i + 1]);
    asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(a), "f"(b));
  }
  return top;
}
__device__ __forceinline__ void load_pairs(const float2* at, float2 (&cs)[8]) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(at) + i);
    cs[2 * i] = make_float2(v.x, v.y);
    cs[2 * i + 1] = make_float2(v.z, v.w);
  }
}
// kKvCap at most, NaN as zero: one bad number does not spoil its block
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

// cuts values that are not finite or too large off; returns the largest magnitude then
__device__ __forceinline__ float make_finite(float (&x)[8], float (&y)[8], float top) {
#pragma unroll
  for (int k = 0; k < 8; k++) {
    x[k] = kv_finite(x[k]);
    y[k] = kv_finite(y[k]);
    top = fmaxf(top, fmaxf(fabsf(x[k]), fabsf(y[k])));
  }
  return top;
}

__device__ __forceinline__ void rotate_queries(const AppendParams& p, int cta) {
  const int upt = p.dim / 16;   // units of a head
  const int split = cta % p.query_splits;
  const int h0 = (int)((long long)p.heads * split / p.query_splits), h1 = (int)((long long)p.heads * (split + 1) / p.query_splits);
  const int t = (cta / p.query_splits) * ((int)blockDim.x / upt) + (int)threadIdx.x / upt, u = (int)threadIdx.x % upt;
  if (t >= p.s.tokens || t >= p.s.starts[p.s.seqs] || t < p.s.starts[0]) return;
  // with one token a sequence row t is sequence t, as a rule
  int b = min(t, p.s.seqs - 1);
  KvSeq sq = kv_seq(p.s, b);
  if (t < sq.t0 || t >= sq.t0 + sq.n) {
    b = kv_find(p.s.starts, p.s.seqs, t);
    sq = kv_seq(p.s, b);
  }
  const int i = t - sq.t0, pos = sq.first + i;
  if (i < 0 || i >= sq.n) return;
  const bool known = pos >= 0 && pos < sq.end;
  const UnitAt at = unit_at(u, p.rot, p.interleaved);
  float2 cs[8];
  if (known && at.pair >= 0) load_pairs(p.rope + (long long)pos * (p.rot / 2) + at.pair, cs);
  const __half* src = p.q + (long long)t * p.q_stride;
  __half* dst = p.q_out + (long long)t * p.heads * p.dim;
  if (!known) {
    for (int h = h0; h < h1; h++) {
      *reinterpret_cast<uint4*>(dst + h * p.dim + at.a) = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(dst + h * p.dim + at.b) = make_uint4(0, 0, 0, 0);
    }
    return;
  }
#pragma unroll 4
  for (int h = h0; h < h1; h++) {
    const Unit in{*reinterpret_cast<const uint4*>(src + h * p.dim + at.a), *reinterpret_cast<const uint4*>(src + h * p.dim + at.b)};
    float x[8], y[8];
    unit_values(in, at.pair >= 0, p.interleaved, cs, x, y);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const __half2 lo = __floats2half2_rn(x[2 * j], x[2 * j + 1]), hi = __floats2half2_rn(y[2 * j], y[2 * j + 1]);
      w[j] = *reinterpret_cast<const uint32_t*>(&lo);
      w[4 + j] = *reinterpret_cast<const uint32_t*>(&hi);
    }
    *reinterpret_cast<uint4*>(dst + h * p.dim + at.a) = make_uint4(w[0], w[1], w[2], w[3]);
    *reinterpret_cast<uint4*>(dst + h * p.dim + at.b) = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// UNITS: units of sixteen values a thread holds of a block, page * dim / 16 / THREADS
template <int UNITS, int THREADS>
__global__ void __launch_bounds__(THREADS) kv_append_kernel(const AppendParams p) {
  __shared__ uint32_t s_max[THREADS / 32];
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
  // a thread's units are of the same place in their heads (THREADS is a multiple of the units of a head)
  const UnitAt at = unit_at(tid & ((1 << lg_upt) - 1), rot, p.interleaved);
  const int slot0 = from + (tid >> lg_upt);
  constexpr int LG_THREADS = THREADS == 128 ? 7 : 8;
  float x[UNITS][8], y[UNITS][8];
  float amax = 0.f;
  {
    Unit in[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; i++) {
      in[i] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
      if (tid + i * THREADS < total) {
        const __half* const row = src + (long long)(sq.t0 + base + slot0 + (i << (LG_THREADS - lg_upt)) - sq.first) * stride;
        in[i] = {*reinterpret_cast<const uint4*>(row + at.a), *reinterpret_cast<const uint4*>(row + at.b)};
      }
    }
#pragma unroll
    for (int i = 0; i < UNITS; i++) {
      const bool live = tid + i * THREADS < total, rotated = live && at.pair >= 0;
      float2 cs[8];
      if (rotated) load_pairs(p.rope + (long long)(base + slot0 + (i << (LG_THREADS - lg_upt))) * (p.rot / 2) + at.pair, cs);
      unit_values(in[i], rotated, p.interleaved, cs, x[i], y[i]);
      amax = max_abs(max_abs(amax, x[i]), y[i]);
    }
  }
  if (!(amax <= kKvCap)) {
    amax = 0.f;
#pragma unroll
    for (int i = 0; i < UNITS; i++) amax = make_finite(x[i], y[i], amax);
  }
  const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(amax));
  if ((tid & 31) == 0) s_max[tid >> 5] = top;
  __syncthreads();
  uint32_t all = s_max[0];
#pragma unroll
  for (int w = 1; w < THREADS / 32; w++) all = max(all, s_max[w]);
  const int e_new = max(kv_exponent(__uint_as_float(all)), e_old);
  const float inv = kv_pow2(-e_new);
#pragma unroll
  for (int i = 0; i < UNITS; i++) {
    if (tid + i * THREADS >= total) break;
    uint8_t* const row = codes + (slot0 + (i << (LG_THREADS - lg_upt))) * p.dim;
    *reinterpret_cast<uint2*>(row + at.a) = codes8(x[i], inv);
    *reinterpret_cast<uint2*>(row + at.b) = codes8(y[i], inv);
  }
  if (from > 0 && e_new > e_old) {   // the older tokens of the block, to its new scale
    const float f = kv_pow2(e_old - e_new);
    for (int n = tid; n < from * p.dim / 16; n += THREADS) {
      uint4 c = reinterpret_cast<const uint4*>(codes)[n];
      c.x = rescale4(c.x, f); c.y = rescale4(c.y, f); c.z = rescale4(c.z, f); c.w = rescale4(c.w, f);
      reinterpret_cast<uint4*>(codes)[n] = c;
    }
  }
  if (tid == 0 && (from == 0 || e_new > e_old)) *scale = kv_pow2(e_new);
}

__global__ void __launch_bounds__(kAppendThreads) kv_append_one_kernel(const AppendParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if ((int)blockIdx.x >= p.candidates) {
    rotate_queries(p, (int)blockIdx.x - p.candidates);
    return;
  }
  const int lg_upt = p.dim == 64 ? 2 : 3, lg_per = 5 - lg_upt;   // units of a block's token, blocks of a warp
  const int lane = (int)threadIdx.x & 31, w = (int)blockIdx.x * (kAppendThreads / 32) + ((int)threadIdx.x >> 5);
  const int per_seq = (2 * p.kv_heads + (1 << lg_per) - 1) >> lg_per, b = w / per_seq;
  if (b >= p.s.seqs) return;
  const KvSeq sq = kv_seq(p.s, b);
  if (sq.n < 1 || sq.first < 0 || sq.first >= sq.end) return;
  const int which = ((w - b * per_seq) << lg_per) + (lane >> lg_upt), u = lane & ((1 << lg_upt) - 1);
  const bool have = which < 2 * p.kv_heads, keys = which < p.kv_heads;
  const int head = keys ? which : which - p.kv_heads, slot = sq.first & (p.s.page - 1);
  const int pg = p.s.table[(long long)b * p.s.width + (sq.first >> p.s.lg_page)];
  const int rot = keys && p.rope ? p.rot : 0;
  const UnitAt at = unit_at(u, rot, p.interleaved);
  Unit in{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  float2 cs[8];
  if (have) {
    const __half* const row = (keys ? p.k : p.v) + (long long)sq.t0 * (keys ? p.k_stride : p.v_stride) + (long long)head * p.dim;
    in = {*reinterpret_cast<const uint4*>(row + at.a), *reinterpret_cast<const uint4*>(row + at.b)};
    if (at.pair >= 0) load_pairs(p.rope + (long long)sq.first * (p.rot / 2) + at.pair, cs);
  }
  if (pg < 0 || pg >= p.s.pages) return;
  const long long block = (long long)pg * p.kv_heads + (have ? head : 0);
  uint8_t* const codes = (keys ? p.k_cache : p.v_cache) + block * p.s.page * p.dim;
  float* const scale = (keys ? p.k_scale : p.v_scale) + block;
  const int e_old = slot > 0 ? kv_stored_exponent(*scale) : kKvExpMin;
  float x[8], y[8];
  unit_values(in, have && at.pair >= 0, p.interleaved, cs, x, y);
  float amax = max_abs(max_abs(0.f, x), y);
  if (!(amax <= kKvCap)) amax = make_finite(x, y, 0.f);
  uint32_t top = __float_as_uint(amax);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  if (p.dim == 128) top = max(top, __shfl_xor_sync(0xffffffffu, top, 4));
  const int e_new = max(kv_exponent(__uint_as_float(top)), e_old);
  if (have) {
    const float inv = kv_pow2(-e_new);
    uint8_t* const row = codes + slot * p.dim;
    *reinterpret_cast<uint2*>(row + at.a) = codes8(x, inv);
    *reinterpret_cast<uint2*>(row + at.b) = codes8(y, inv);
    if (u == 0 && (slot == 0 || e_new > e_old)) *scale = kv_pow2(e_new);
  }
  // blocks whose scale grows: their older tokens, one block after the other, the whole warp at each
  uint32_t grow = __ballot_sync(0xffffffffu, have && u == 0 && slot > 0 && e_new > e_old);
  while (grow) {
    const int from = __ffs((int)grow) - 1;
    grow &= grow - 1;
    uint4* const c0 = reinterpret_cast<uint4*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(codes), from));
    const float f = kv_pow2(__shfl_sync(0xffffffffu, e_old - e_new, from));
#pragma unroll 4
    for (int n = lane; n < slot * p.dim / 16; n += 32) {
      uint4 c = c0[n];
      c.x = rescale4(c.x, f); c.y = rescale4(c.y, f); c.z = rescale4(c.z, f); c.w = rescale4(c.w, f);
      c0[n] = c;
    }
  }
}

}  // namespace rcp
