// Softmax attention of new tokens over the paged 8-bit cache (rcp_kv_attention).
//
//   out[t][h] = sum_j p_j v_j / sum_j p_j,  p_j = exp(sm_scale (q[t][h] . k_j)),  j over the positions 0 .. position of t
//   k_j, v_j: code times the scale of its block; a page outside the cache holds no keys; a row without keys is zero.
#pragma once
#include "common.cuh"
#include "kv_common.cuh"

namespace rcp {

struct AttnParams {
  const __half* q;
  long long q_stride;        // elements between tokens
  int heads, kv_heads, dim;
  float scale_log2;          // sm_scale * log2(e)
  KvSeqs s;
  const uint8_t *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  __half* out;               // [tokens][heads][dim]
};

constexpr int kAttnWarps = 4;
template <int DIM>
__global__ void __launch_bounds__(kAttnWarps * 32) kv_attention_rows_kernel(const AttnParams p) {
  constexpr int PER = DIM / 32;
  __shared__ float s_m[kAttnWarps], s_l[kAttnWarps], s_o[kAttnWarps][DIM];
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (t >= p.s.starts[p.s.seqs] || t < p.s.starts[0]) return;
  const int b = kv_find(p.s.starts, p.s.seqs, t);
  const KvSeq sq = kv_seq(p.s, b);
  const int i = t - sq.t0;
  if (i >= sq.n) return;
  const int pos = sq.first + i, end = pos < sq.end ? pos + 1 : 0, kv = h / (p.heads / p.kv_heads);
  float q[PER], o[PER] = {}, m = -1e30f, l = 0.f;
#pragma unroll
  for (int e = 0; e < PER; e++) q[e] = __half2float(p.q[t * p.q_stride + h * DIM + lane * PER + e]);
  for (int j = warp; j < end; j += kAttnWarps) {
    const int pg = p.s.table[(long long)b * p.s.width + (j >> p.s.lg_page)];
    if (pg < 0 || pg >= p.s.pages) continue;
    const long long block = (long long)pg * p.kv_heads + kv;
    const long long at = (block * p.s.page + (j & (p.s.page - 1))) * DIM + lane * PER;
    float dot = 0.f;
#pragma unroll
    for (int e = 0; e < PER; e++) dot = fmaf(q[e], __half2float(__half(__nv_cvt_fp8_to_halfraw(p.k_cache[at + e], __NV_E4M3))), dot);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, x);
    const float s = dot * (p.k_scale[block] * p.scale_log2), mn = fmaxf(m, s), f = exp2f(m - mn), w = exp2f(s - mn);
    l = l * f + w;
    const float wv = w * p.v_scale[block];
#pragma unroll
    for (int e = 0; e < PER; e++) o[e] = fmaf(wv, __half2float(__half(__nv_cvt_fp8_to_halfraw(p.v_cache[at + e], __NV_E4M3))), o[e] * f);
    m = mn;
  }
  if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
#pragma unroll
  for (int e = 0; e < PER; e++) s_o[warp][lane * PER + e] = o[e];
  __syncthreads();
  if (threadIdx.x < DIM) {
    float top = s_m[0], sum = 0.f, acc = 0.f;
    for (int w = 1; w < kAttnWarps; w++) top = fmaxf(top, s_m[w]);
    for (int w = 0; w < kAttnWarps; w++) {
      const float f = exp2f(s_m[w] - top);
      sum += s_l[w] * f;
      acc += s_o[w][threadIdx.x] * f;
    }
    p.out[((long long)t * p.heads + h) * DIM + threadIdx.x] = __float2half_rn(sum > 0.f ? acc / sum : 0.f);
  }
}

}  // namespace rcp
