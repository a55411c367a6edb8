// Low-rank adapters of many requests beside a shared projection (rcp_lora_add):
//   z[m][r] = sum_k a[i][r][k] x[m][k],  y[m][n] = base[m][n] + scaling[i] sum_r b[i][n][r] z[m][r],  i = adapter[m]
#pragma once
#include "common.cuh"

namespace rcp {

struct LoraParams {
  const __half* x;
  long long x_stride;
  const __half *a, *b;       // [adapters][rank][K], [adapters][N][rank]
  const int32_t* adapter;    // [M]
  const float* scaling;      // [adapters]
  const __half* base;        // [M][N] or null
  __half* y;                 // [M][N]
  float* z;                  // [M][rank]
  int M, N, K, rank, adapters;
};

__global__ void __launch_bounds__(256) lora_down_kernel(const LoraParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < (long long)p.M * p.rank; w += (long long)gridDim.x * 8) {
    const int m = (int)(w / p.rank), r = (int)(w % p.rank), i = p.adapter[m];
    if (i < 0 || i >= p.adapters) continue;
    const __half *x = p.x + m * p.x_stride, *a = p.a + ((long long)i * p.rank + r) * p.K;
    float sum = 0.f;
    for (int k = lane; k < p.K; k += 32) sum = fmaf(__half2float(a[k]), __half2float(x[k]), sum);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if (lane == 0) p.z[w] = sum * p.scaling[i];
  }
}
__global__ void __launch_bounds__(256) lora_up_kernel(const LoraParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int m = blockIdx.y, n = blockIdx.x * 256 + threadIdx.x, i = p.adapter[m];
  if (n >= p.N) return;
  const long long at = (long long)m * p.N + n;
  float y = p.base ? __half2float(p.base[at]) : 0.f;
  if (i >= 0 && i < p.adapters) {
    const __half* b = p.b + ((long long)i * p.N + n) * p.rank;
    for (int r = 0; r < p.rank; r++) y = fmaf(__half2float(b[r]), p.z[(long long)m * p.rank + r], y);
  }
  p.y[at] = __float2half_rn(y);
}

}  // namespace rcp
