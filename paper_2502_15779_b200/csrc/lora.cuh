// Low-rank adapters of many requests beside a shared projection (rcp_lora_add):
//   z[m][r] = sum_k a[i][r][k] x[m][k],  y[m][n] = base[m][n] + scaling[i] sum_r b[i][n][r] z[m][r],  i = adapter[m]
//
// lora_few_kernel: up to kLoraFew tokens, as in decoding. Bound by latency, and by the adapters' bytes where every token has its own. One
// launch: a cluster of eight CTAs takes the tokens of one adapter (eight at most), each CTA a part of K for z; the parts of z go to
// all eight through distributed shared memory, and behind the cluster's barrier each CTA takes a part of the rows of b.
// lora_down_kernel, lora_up_kernel: more tokens, as in prompts, in tiles; bound by x, base and y (with hundreds of tokens an
// adapter is read from L2). Both products on the tensor cores, fragments straight from memory: the order of the inner index
// is free as long as both operands share it, so a thread reads 16 (z) or 8 (y) contiguous bytes. z is a sum in fp32; for the second
// product each token's row is scaled by a power of two and split into two fp16 numbers, 22 bits of it. A tile goes once
// through for each adapter that its tokens have, and rows of other adapters are dropped, not multiplied by zero: what is not a number in
// one request's adapter stays there.
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
  int parts;                 // CTAs of a cluster of lora_down_kernel: parts of K
  int wide;                  // rows of base and y start on 16 bytes
};

constexpr int kLoraThreads = 256, kLoraWarps = kLoraThreads / 32;
constexpr int kLoraFew = 64, kLoraCluster = 8, kLoraGroup = 8;
constexpr int kLoraMaxRank = 128;

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// stores to the same place of CTA `cta` of the cluster
__device__ __forceinline__ void st_cluster(const void* at, uint32_t cta, float v) {
  const uint32_t here = (uint32_t)__cvta_generic_to_shared(at);
  asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f32 [a], %2;\n\t}" ::"r"(here), "r"(cta), "f"(v) : "memory");
}
__device__ __forceinline__ void halves8(uint4 v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

struct LoraFewShared {
  float part[kLoraCluster][kLoraGroup][kLoraMaxRank];   // parts of z, one from each CTA of the cluster
  float z[kLoraGroup][kLoraMaxRank];
  int token[kLoraGroup];
};

// the cluster's tokens (count of them, the same adapter i): G is how many the registers are for
template <int G>
__device__ __forceinline__ void lora_few(const LoraParams& p, LoraFewShared& s, int i, int count, uint32_t cta) {
  constexpr int RB = G == 1 ? 4 : 2;   // rows of a at a time
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, R = p.rank;
  const int units = p.K / 8, u0 = (int)((long long)units * cta / kLoraCluster), u1 = (int)((long long)units * (cta + 1) / kLoraCluster);
  const uint4* const a = reinterpret_cast<const uint4*>(p.a + (long long)i * R * p.K);
  const uint4* x[G];
#pragma unroll
  for (int t = 0; t < G; t++) x[t] = reinterpret_cast<const uint4*>(p.x + (long long)s.token[min(t, count - 1)] * p.x_stride);
  for (int r0 = warp * RB; r0 < R; r0 += kLoraWarps * RB) {
    float acc[RB][G] = {};
    const uint4* row[RB];
#pragma unroll
    for (int r = 0; r < RB; r++) row[r] = a + (long long)min(r0 + r, R - 1) * units;
#pragma unroll(G == 1 ? 4 : 1)
    for (int u = u0 + lane; u < u1; u += 32) {
      float av[RB][8];
#pragma unroll
      for (int r = 0; r < RB; r++) halves8(__ldg(row[r] + u), av[r]);
#pragma unroll
      for (int t = 0; t < G; t++) {
        float xv[8];
        halves8(ld_input(x[t] + u), xv);
#pragma unroll
        for (int r = 0; r < RB; r++)
#pragma unroll
          for (int e = 0; e < 8; e++) acc[r][t] = fmaf(av[r][e], xv[e], acc[r][t]);
      }
    }
#pragma unroll
    for (int r = 0; r < RB; r++)
#pragma unroll
      for (int t = 0; t < G; t++) {
        float v = acc[r][t];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (r0 + r < R && t < count && lane < kLoraCluster) st_cluster(&s.part[cta][t][r0 + r], lane, v);
      }
  }
  // rows of b on their way (at most 32 columns of the first rows), and what they are added to
  const int n0 = (int)((long long)p.N * cta / kLoraCluster), n1 = (int)((long long)p.N * (cta + 1) / kLoraCluster), V = R / 8;
  const uint4* const b = reinterpret_cast<const uint4*>(p.b + (long long)i * p.N * R);
  constexpr int PF = 4;
  uint4 pre[PF];
#pragma unroll
  for (int v = 0; v < PF; v++)
    if (n0 + tid < n1 && v < V) pre[v] = __ldg(b + (long long)(n0 + tid) * V + v);
  cluster_barrier();
  const float scale = p.scaling[i];
  for (int e = tid; e < count * R; e += kLoraThreads) {
    const int t = e / R, r = e - t * R;
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < kLoraCluster; c++) sum += s.part[c][t][r];
    s.z[t][r] = sum * scale;
  }
  __syncthreads();
  for (int n = n0 + tid; n < n1; n += kLoraThreads) {
    float y[G] = {};
    const uint4* const row = b + (long long)n * V;
#pragma unroll 4
    for (int v = 0; v < V; v++) {
      float bv[8];
      if (n == n0 + tid && v < PF) halves8(v == 0 ? pre[0] : v == 1 ? pre[1] : v == 2 ? pre[2] : pre[3], bv);
      else halves8(__ldg(row + v), bv);
#pragma unroll
      for (int t = 0; t < G; t++)
        if (t < count) {
          const float4 z0 = *reinterpret_cast<const float4*>(&s.z[t][8 * v]), z1 = *reinterpret_cast<const float4*>(&s.z[t][8 * v + 4]);
          y[t] = fmaf(bv[0], z0.x, y[t]); y[t] = fmaf(bv[1], z0.y, y[t]); y[t] = fmaf(bv[2], z0.z, y[t]); y[t] = fmaf(bv[3], z0.w, y[t]);
          y[t] = fmaf(bv[4], z1.x, y[t]); y[t] = fmaf(bv[5], z1.y, y[t]); y[t] = fmaf(bv[6], z1.z, y[t]); y[t] = fmaf(bv[7], z1.w, y[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < G; t++)
      if (t < count) {
        const long long at = (long long)s.token[t] * p.N + n;
        p.y[at] = __float2half_rn(p.base ? __half2float(p.base[at]) + y[t] : y[t]);
      }
  }
}

// One cluster a token. The cluster of the first, ninth, ... token of an adapter takes that one and the next seven of the adapter; the
// others have nothing to do.
__global__ void __cluster_dims__(kLoraCluster, 1, 1) __launch_bounds__(kLoraThreads) lora_few_kernel(const LoraParams p) {
  __shared__ __align__(16) LoraFewShared s;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int m = (int)blockIdx.x / kLoraCluster, lane = threadIdx.x & 31;
  const uint32_t cta = cluster_rank();
  // tokens of the same adapter in front of this one, and it and those behind it (every warp for itself: kLoraFew is two votes)
  const int i = p.adapter[m];
  const uint32_t lo = __ballot_sync(0xffffffffu, lane < p.M && p.adapter[min(lane, p.M - 1)] == i);
  const uint32_t hi = __ballot_sync(0xffffffffu, lane + 32 < p.M && p.adapter[min(lane + 32, p.M - 1)] == i);
  const unsigned long long same = (unsigned long long)hi << 32 | lo;
  if (i < 0 || i >= p.adapters) {   // none: the cluster copies its token's row
    for (int n = (int)cta * kLoraThreads + (int)threadIdx.x; n < p.N; n += kLoraCluster * kLoraThreads) {
      const long long at = (long long)m * p.N + n;
      p.y[at] = p.base ? p.base[at] : __float2half_rn(0.f);
    }
    return;
  }
  const int rank = __popcll(same & ((1ull << m) - 1));
  if (rank % kLoraGroup) return;
  unsigned long long mine = same & ~((1ull << m) - 1);
  const int count = min(__popcll(mine), kLoraGroup);
  if (threadIdx.x == 0)
    for (int t = 0; t < count; t++) {
      s.token[t] = __ffsll((long long)mine) - 1;
      mine &= mine - 1;
    }
  // every CTA of the cluster runs before its shared memory is written to from the others
  cluster_barrier();
  if (count == 1) lora_few<1>(p, s, i, count, cta);
  else lora_few<kLoraGroup>(p, s, i, count, cta);
}

__device__ __forceinline__ void lora_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// the different adapters of a tile's tokens, in the order of their first token; returns how many (adapters[t] of the tokens: -1 none)
template <int TILE>
__device__ __forceinline__ int tile_adapters(const LoraParams& p, int m0, int (&adapter)[TILE], int (&list)[TILE], int& count) {
  const int tid = threadIdx.x;
  if (tid < TILE) {
    const int i = m0 + tid < p.M ? p.adapter[m0 + tid] : -1;
    adapter[tid] = i >= 0 && i < p.adapters ? i : -1;
  }
  __syncthreads();
  if (tid == 0) {
    int n = 0;
    for (int t = 0; t < TILE; t++) {
      const int i = adapter[t];
      if (i < 0 || (t > 0 && adapter[t - 1] == i)) continue;
      bool known = false;
      for (int k = 0; k < n; k++) known |= list[k] == i;
      if (!known) list[n++] = i;
    }
    count = n;
  }
  __syncthreads();
  return count;
}

constexpr int kDownTokens = 32;
// z of kDownTokens tokens: two groups of 16 tokens x four quarters of the rank among the warps; the CTAs of a cluster have a part of K each
__global__ void __launch_bounds__(kLoraThreads) lora_down_kernel(const LoraParams p) {
  __shared__ __align__(16) float s_part[kDownTokens][kLoraMaxRank];   // this CTA's part of the sums
  __shared__ int s_adapter[kDownTokens], s_list[kDownTokens], s_count;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3;
  const uint32_t part = cluster_rank();
  const int m0 = (int)blockIdx.x / p.parts * kDownTokens, R = p.rank;
  const int chunks = p.K / 64, c0 = chunks * (int)part / p.parts, c1 = chunks * ((int)part + 1) / p.parts;
  const int mt = warp & 1, tiles = R / 8, n0 = tiles * (warp >> 1) / 4, nn = tiles * ((warp >> 1) + 1) / 4 - n0;   // at most four
  const int different = tile_adapters(p, m0, s_adapter, s_list, s_count);
  for (int e = 0; e < different; e++) {
    const int i = s_list[e];
    const __half* xr[2];
#pragma unroll
    for (int h = 0; h < 2; h++) xr[h] = p.x + (long long)min(m0 + mt * 16 + h * 8 + g, p.M - 1) * p.x_stride + 8 * j;
    const __half* ar = p.a + ((long long)i * R + n0 * 8 + g) * p.K + 8 * j;
    float acc[4][4] = {};
#pragma unroll 2
    for (int c = c0; c < c1; c++) {
      uint4 xv[2][2], av[2][4];
#pragma unroll
      for (int q = 0; q < 2; q++) {
#pragma unroll
        for (int h = 0; h < 2; h++) xv[q][h] = ld_input(reinterpret_cast<const uint4*>(xr[h] + c * 64 + q * 32));
#pragma unroll
        for (int n = 0; n < 4; n++)
          if (n < nn) av[q][n] = __ldg(reinterpret_cast<const uint4*>(ar + (long long)n * 8 * p.K + c * 64 + q * 32));
      }
#pragma unroll
      for (int q = 0; q < 2; q++)
#pragma unroll
        for (int n = 0; n < 4; n++)
          if (n < nn) {
            lora_mma(acc[n], xv[q][0].x, xv[q][1].x, xv[q][0].y, xv[q][1].y, av[q][n].x, av[q][n].y);
            lora_mma(acc[n], xv[q][0].z, xv[q][1].z, xv[q][0].w, xv[q][1].w, av[q][n].z, av[q][n].w);
          }
    }
#pragma unroll
    for (int n = 0; n < 4; n++)
      if (n < nn)
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const int t = mt * 16 + h * 8 + g;
          if (s_adapter[t] == i) *reinterpret_cast<float2*>(&s_part[t][(n0 + n) * 8 + 2 * j]) = make_float2(acc[n][2 * h], acc[n][2 * h + 1]);
        }
  }
  // the parts of the cluster's CTAs, each CTA a share of the sums
  cluster_barrier();
  const int all = kDownTokens * R;
  for (int v = all * (int)part / p.parts + tid; v < all * ((int)part + 1) / p.parts; v += kLoraThreads) {
    const int t = v / R, r = v - t * R, i = s_adapter[t];
    if (i < 0) continue;
    float sum = 0.f;
    for (int c = 0; c < p.parts; c++) {
      float w;
      const uint32_t here = (uint32_t)__cvta_generic_to_shared(&s_part[t][r]);
      asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(w) : "r"(here), "r"(c) : "memory");
      sum += w;
    }
    p.z[(long long)(m0 + t) * R + r] = sum * p.scaling[i];
  }
  cluster_barrier();   // no CTA ends while others read its shared memory
}

constexpr int kUpTokens = 64, kUpCols = 128, kUpTiles = 4;   // columns of a tile, tiles of a CTA
struct LoraUpShared {
  __half z[2][kUpTokens][kLoraMaxRank + 16];   // upper and lower part of z / 2^exponent
  float stage[kLoraWarps][16][64 + 4];
  float unit[kUpTokens];
  int adapter[kUpTokens], list[kUpTokens], count;
};
// y of kUpTokens tokens x kUpTiles * kUpCols columns: four groups of 16 tokens x two halves of a tile's columns among the warps
__global__ void __launch_bounds__(kLoraThreads) lora_up_kernel(const LoraParams p) {
  extern __shared__ __align__(16) uint8_t lora_shared[];
  LoraUpShared& s = *reinterpret_cast<LoraUpShared*>(lora_shared);
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3, R = p.rank;
  const int m0 = (int)blockIdx.y * kUpTokens;
  const int different = tile_adapters(p, m0, s.adapter, s.list, s.count);
  // four threads a token: its largest |z|, then z / 2^exponent in two parts, zeroes behind the rank (up to a multiple of 16)
  {
    const int t = tid >> 2, q = tid & 3;
    const bool have = s.adapter[t] >= 0;
    const float* const z = p.z + (long long)(m0 + t) * R;
    float top = 0.f;
    if (have)
      for (int r = 4 * q; r < R; r += 16) {
        const float4 v = *reinterpret_cast<const float4*>(z + r);
        top = fmaxf(fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))), top);
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = min(max((int)(__float_as_uint(top) >> 23) - 126, -100), 126);   // |z| < 2^e
    const float inv = __int_as_float((127 - e) << 23);
    if (q == 0) s.unit[t] = __int_as_float((e + 127) << 23);
    for (int r = 4 * q; r < (R + 15) / 16 * 16; r += 16) {
      float4 v = have && r < R ? *reinterpret_cast<const float4*>(z + r) : make_float4(0.f, 0.f, 0.f, 0.f);
      v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
      const __half2 h0 = __floats2half2_rn(v.x, v.y), h1 = __floats2half2_rn(v.z, v.w);
      const float2 f0 = __half22float2(h0), f1 = __half22float2(h1);
      const __half2 l0 = __floats2half2_rn(v.x - f0.x, v.y - f0.y), l1 = __floats2half2_rn(v.z - f1.x, v.w - f1.y);
      *reinterpret_cast<uint2*>(&s.z[0][t][r]) = make_uint2(*reinterpret_cast<const uint32_t*>(&h0), *reinterpret_cast<const uint32_t*>(&h1));
      *reinterpret_cast<uint2*>(&s.z[1][t][r]) = make_uint2(*reinterpret_cast<const uint32_t*>(&l0), *reinterpret_cast<const uint32_t*>(&l1));
    }
  }
  __syncthreads();
  const int mt = warp & 3, half = warp >> 2, steps = (R + 15) / 16;
  float(*const stage)[64 + 4] = s.stage[warp];
  for (int tile = 0; tile < kUpTiles; tile++) {
    const int n0 = ((int)blockIdx.x * kUpTiles + tile) * kUpCols + half * 64;
    if (n0 >= p.N) break;
    // adapter by adapter, the rows that have it; last the rows without any
    for (int e = 0; e <= different; e++) {
      const int i = e < different ? s.list[e] : -1;
      const bool mine = __any_sync(0xffffffffu, lane < 16 && m0 + mt * 16 + lane < p.M && s.adapter[mt * 16 + lane] == i);
      if (!mine) continue;
      if (i >= 0) {
        float acc[8][4] = {};
        const __half* const b = p.b + ((long long)i * p.N + n0 + g) * R + 4 * j;
        for (int k = 0; k < steps; k++) {
          uint2 bv[8];
#pragma unroll
          for (int n = 0; n < 8; n++)
            bv[n] = n0 + n * 8 + g < p.N && 16 * k + 4 * j < R ? __ldg(reinterpret_cast<const uint2*>(b + (long long)n * 8 * R + 16 * k)) : make_uint2(0, 0);
#pragma unroll
          for (int h = 0; h < 2; h++) {
            const uint2 u = *reinterpret_cast<const uint2*>(&s.z[h][mt * 16 + g][16 * k + 4 * j]);
            const uint2 v = *reinterpret_cast<const uint2*>(&s.z[h][mt * 16 + 8 + g][16 * k + 4 * j]);
#pragma unroll
            for (int n = 0; n < 8; n++) lora_mma(acc[n], u.x, v.x, u.y, v.y, bv[n].x, bv[n].y);
          }
        }
        __syncwarp();
        const float u0 = s.unit[mt * 16 + g], u1 = s.unit[mt * 16 + 8 + g];
#pragma unroll
        for (int n = 0; n < 8; n++) {
          *reinterpret_cast<float2*>(&stage[g][n * 8 + 2 * j]) = make_float2(acc[n][0] * u0, acc[n][1] * u0);
          *reinterpret_cast<float2*>(&stage[g + 8][n * 8 + 2 * j]) = make_float2(acc[n][2] * u1, acc[n][3] * u1);
        }
        __syncwarp();
      }
      if (p.wide) {
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const int row = q * 4 + (lane >> 3), c = (lane & 7) * 8, m = m0 + mt * 16 + row;
          if (m >= p.M || s.adapter[mt * 16 + row] != i || n0 + c >= p.N) continue;
          const long long at = (long long)m * p.N + n0 + c;
          float v[8] = {};
          if (p.base) halves8(*reinterpret_cast<const uint4*>(p.base + at), v);
          if (i >= 0)
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] += stage[row][c + k];
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; k++) {
            const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&h);
          }
          *reinterpret_cast<uint4*>(p.y + at) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else {
        for (int q = 0; q < 32; q++) {
          const int row = q >> 1, c = (q & 1) * 32 + lane, m = m0 + mt * 16 + row;
          if (m >= p.M || s.adapter[mt * 16 + row] != i || n0 + c >= p.N) continue;
          const long long at = (long long)m * p.N + n0 + c;
          float v = p.base ? __half2float(p.base[at]) : 0.f;
          if (i >= 0) v += stage[row][c];
          p.y[at] = __float2half_rn(v);
        }
      }
      __syncwarp();
    }
  }
}

}  // namespace rcp
