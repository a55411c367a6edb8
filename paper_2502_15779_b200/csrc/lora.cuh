// Low-rank adapters of many requests beside a shared projection (rcp_lora_add):
//   z[m][r] = sum_k a[i][r][k] x[m][k],  y[m][n] = base[m][n] + scaling[i] sum_r b[i][n][r] z[m][r],  i = adapter[m]
//
// lora_few_kernel: up to kLoraFew tokens, as in decoding. Bound by latency, and by the adapters' bytes where every token has its own. One
// launch: a cluster of eight CTAs takes the tokens of one adapter (eight at most), each CTA a part of K for z; the parts of z go to
// all eight through distributed shared memory, and behind the cluster's barrier each CTA takes a part of the rows of b. One token, 10240 x 8192, rank
// 16: 4.4 us (two launches: 15 with a plain loop a row); sixteen tokens of up to sixteen adapters, 6144 x 4096, rank 32: 6.7 us, 1.6 TB/s.
// lora_down_kernel, lora_up_kernel: more tokens, as in prompts, in tiles; bound by x, base and y (with hundreds of tokens an
// adapter is read from L2). Both products on the tensor cores, fragments straight from memory: the order of the inner index
// is free as long as both operands share it, so a thread reads 16 (z) or 8 (y) contiguous bytes. z is a sum in fp32; for the second
// product each token's row is scaled by a power of two and split into two fp16 numbers: 22 bits of each z down to 2^-18 of the row's largest. A tile goes once
// through for each adapter that its tokens have, and rows of other adapters are dropped, not multiplied by zero: what is not a number in
// one request's adapter stays there. 2011 tokens of five requests and some without, 28672 x 4096, rank 64: 90 us, 15 of them the first
// product; the second moves 250 MB in 75 us (3.3 TB/s). Bound by instructions (500 a warp and 32 x 32 results; beside products on mma.sync the others go
// two a clock, which makes 66 us of them): with neither base nor stores it took 81 us of 93. Steps: fragments and base straight from memory 113 us;
// operands through shared memory 106; z in two parts and in the tensor core's order made by the first kernel, not by every CTA of the second, and the
// first one's columns known to the compiler 93; a kernel of their own for rows that do not start on 16 bytes 90.
#pragma once
#include <cstddef>

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
  uint8_t* z;                // a record of lora_record_bytes() for each tile of tokens
  int M, N, K, rank, adapters;
  int parts;                 // CTAs of a cluster of lora_down_kernel: parts of K
  int up_tiles;              // column tiles of a CTA of lora_up_kernel
};

constexpr int kLoraThreads = 256, kLoraWarps = kLoraThreads / 32;
constexpr int kLoraFew = 64, kLoraCluster = 8, kLoraGroup = 8;
constexpr int kLoraMaxRank = 128;
// A token's z are scaled to below 2^15, as large as fp16 holds them: the two parts' steps then end at 2^-24 beside a largest of 2^15, so that z down to 2^-18 of the
// token's largest keep 22 bits, and what is lost of smaller ones is 2^-40 of it.
constexpr int kLoraRoom = 15;

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
  constexpr int RB = G <= 2 ? 4 : 2;   // rows of a at a time
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
#pragma unroll(G == 1 ? 4 : G == 2 ? 2 : 1)
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
  // Rows of b a few at a time, sixteen bytes of each asked for together with what they are added to (one row at a time, each waited for, took
  // half of the call); the first of them in front of the barrier.
  const int n0 = (int)((long long)p.N * cta / kLoraCluster), n1 = (int)((long long)p.N * (cta + 1) / kLoraCluster), V = R / 8;
  const uint4* const b = reinterpret_cast<const uint4*>(p.b + (long long)i * p.N * R);
  constexpr int ROWS = G == 1 ? 4 : 2, VB = 2;   // rows at a time, 16-byte pieces of each at a time
  uint4 bv[ROWS][VB];
  __half base[ROWS][G];
  auto ask_b = [&](int n, int v0) {
#pragma unroll
    for (int r = 0; r < ROWS; r++)
#pragma unroll
      for (int v = 0; v < VB; v++)
        bv[r][v] = n + r * kLoraThreads < n1 && v0 + v < V ? __ldg(b + (long long)(n + r * kLoraThreads) * V + v0 + v) : make_uint4(0, 0, 0, 0);
  };
  auto ask_base = [&](int n) {
#pragma unroll
    for (int r = 0; r < ROWS; r++)
#pragma unroll
      for (int t = 0; t < G; t++)
        base[r][t] = p.base && t < count && n + r * kLoraThreads < n1 ? p.base[(long long)s.token[t] * p.N + n + r * kLoraThreads] : __float2half_rn(0.f);
  };
  int n = n0 + tid;
  ask_b(n, 0);
  ask_base(n);
  cluster_barrier();
  const float scale = p.scaling[i];
  for (int e = tid; e < kLoraGroup * kLoraMaxRank; e += kLoraThreads) {
    const int t = e / kLoraMaxRank, r = e % kLoraMaxRank;
    if (t >= count || r >= R) continue;
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < kLoraCluster; c++) sum += s.part[c][t][r];
    s.z[t][r] = sum * scale;
  }
  __syncthreads();
  for (; n < n1; n += ROWS * kLoraThreads) {
    float y[ROWS][G] = {};
    for (int v0 = 0; v0 < V; v0 += VB) {
      float w[ROWS][VB][8];
#pragma unroll
      for (int r = 0; r < ROWS; r++)
#pragma unroll
        for (int v = 0; v < VB; v++) halves8(bv[r][v], w[r][v]);
      if (v0 + VB < V) ask_b(n, v0 + VB);
#pragma unroll
      for (int v = 0; v < VB; v++) {
        if (v0 + v >= V) break;
#pragma unroll
        for (int t = 0; t < G; t++)
          if (t < count) {
            const float4 z0 = *reinterpret_cast<const float4*>(&s.z[t][8 * (v0 + v)]), z1 = *reinterpret_cast<const float4*>(&s.z[t][8 * (v0 + v) + 4]);
            const float z[8] = {z0.x, z0.y, z0.z, z0.w, z1.x, z1.y, z1.z, z1.w};
#pragma unroll
            for (int r = 0; r < ROWS; r++)
#pragma unroll
              for (int k = 0; k < 8; k++) y[r][t] = fmaf(w[r][v][k], z[k], y[r][t]);
          }
      }
    }
    __half out[ROWS][G];
#pragma unroll
    for (int r = 0; r < ROWS; r++)
#pragma unroll
      for (int t = 0; t < G; t++) out[r][t] = __float2half_rn(__half2float(base[r][t]) + y[r][t]);
    // the next rows before these are stored
    const int now = n;
    if (n + ROWS * kLoraThreads < n1) {
      ask_b(n + ROWS * kLoraThreads, 0);
      ask_base(n + ROWS * kLoraThreads);
    }
#pragma unroll
    for (int r = 0; r < ROWS; r++)
#pragma unroll
      for (int t = 0; t < G; t++)
        if (t < count && now + r * kLoraThreads < n1) p.y[(long long)s.token[t] * p.N + now + r * kLoraThreads] = out[r][t];
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
  else if (count == 2) lora_few<2>(p, s, i, count, cta);
  else if (count <= 4) lora_few<4>(p, s, i, count, cta);
  else lora_few<kLoraGroup>(p, s, i, count, cta);
}

__device__ __forceinline__ void lora_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// the same with sums of zero in front
__device__ __forceinline__ void lora_mma_first(float (&c)[4], uint4 a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1), "f"(0.f));
}

constexpr int kLoraTile = 64;   // tokens of a tile
struct alignas(16) LoraTokens {
  int adapter[kLoraTile];   // of the tile's tokens, -1: none, -2: no such token
  int list[kLoraTile];      // the different ones
  int count;
  int none;                 // whether there are tokens without one
  int pad[2];
  float unit[kLoraTile];    // what a token's z in the record is to be multiplied by, a power of two
};
// What lora_down_kernel leaves for lora_up_kernel, a tile: its tokens, then z as the tensor core wants it: [upper, lower parts][16 tokens][step
// of 16 r] of 512 bytes, a lane's 16 bytes side by side.
constexpr int kLoraRecordZ = 1024;
static_assert(sizeof(LoraTokens) <= kLoraRecordZ, "");
__host__ __device__ inline int lora_record_bytes(int rank) { return kLoraRecordZ + (rank + 15) / 16 * 4096; }
// Fills s; returns how many adapters there are. By one warp in a few votes (one thread with a loop took 4 us).
__device__ __forceinline__ int tile_adapters(const LoraParams& p, int m0, LoraTokens& s) {
  const int tid = threadIdx.x;
  if (tid < 32) {
    int i[2], n = 0;
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int m = m0 + 32 * h + tid;
      i[h] = m < p.M ? p.adapter[m] : -2;
      if (m < p.M && (i[h] < 0 || i[h] >= p.adapters)) i[h] = -1;
      s.adapter[32 * h + tid] = i[h];
    }
    const bool none = __any_sync(0xffffffffu, i[0] == -1 || i[1] == -1);
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const uint32_t alike = __match_any_sync(0xffffffffu, i[h]);   // every lane has to come here, those without an adapter too
      bool lead = i[h] >= 0 && __ffs((int)alike) - 1 == tid;
      for (int k = 0; k < n; k++) lead = lead && s.list[k] != i[h];   // n: those of the first half
      const uint32_t leads = __ballot_sync(0xffffffffu, lead);
      __syncwarp();
      if (lead) s.list[n + __popc(leads & ((1u << tid) - 1))] = i[h];
      __syncwarp();
      n += __popc(leads);
    }
    if (tid == 0) { s.count = n; s.none = none; }
  }
  __syncthreads();
  return s.count;
}

__device__ __forceinline__ void lora_copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 lora_lds(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

constexpr int kDownStages = 4;  // of 64 elements of K: the tile's tokens, then the adapter's rows, 128 bytes each
inline size_t lora_down_smem(int rank) { return (size_t)kDownStages * (kLoraTile + rank) * 128; }   // >= kLoraTile * rank * 4

// z of a tile: four groups of 16 tokens x two halves of the rank among the warps; the CTAs of a cluster have a part of K each, through a
// ring of asynchronous copies (fragments straight from memory took 31 us for 2011 tokens, 4096 elements, rank 64, bound by the cache's
// ports: every row is wanted by two or four warps). Odd rows have their 64-byte halves exchanged, which keeps the reads of the fragments free
// of bank conflicts.
// STEPS: the rank in steps of 16, rounded up (eight columns a warp has at most STEPS times)
template <int STEPS>
__global__ void __launch_bounds__(kLoraThreads, 2) lora_down_kernel(const LoraParams p) {
  extern __shared__ __align__(128) uint8_t lora_shared[];
  __shared__ LoraTokens s;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3;
  const uint32_t part = cluster_rank(), base = (uint32_t)__cvta_generic_to_shared(lora_shared);
  const int m0 = (int)blockIdx.x / p.parts * kLoraTile, R = p.rank;
  const int chunks = p.K / 64, c0 = chunks * (int)part / p.parts, c1 = chunks * ((int)part + 1) / p.parts;
  const int mt = warp & 3, tiles = R / 8, n0 = warp < 4 ? 0 : tiles / 2, nn = warp < 4 ? tiles / 2 : tiles - tiles / 2;
  const int stage_bytes = (kLoraTile + R) * 128;
  const int different = tile_adapters(p, m0, s);
  uint8_t* const record = p.z + (long long)(m0 / kLoraTile) * lora_record_bytes(R);
  if (part == 0 && blockIdx.y == 0)
    for (int v = tid; v < (int)(offsetof(LoraTokens, unit) / 16); v += kLoraThreads) reinterpret_cast<uint4*>(record)[v] = reinterpret_cast<const uint4*>(&s)[v];
  float acc[STEPS][4];
  for (int e = (int)blockIdx.y; e < different; e += (int)gridDim.y) {
    const int i = s.list[e];
    // this thread's copies: 16 bytes of every 32nd row, two of tokens, up to four of the adapter
    const int copy_row = tid >> 3, copy_to = copy_row * 128 + (((tid & 7) ^ ((copy_row & 1) << 2)) << 4);
    const __half* from_x[2];
#pragma unroll
    for (int k = 0; k < 2; k++) from_x[k] = p.x + (long long)min(m0 + copy_row + 32 * k, p.M - 1) * p.x_stride + c0 * 64 + (tid & 7) * 8;
    const __half* from_a = p.a + ((long long)i * R + copy_row) * p.K + c0 * 64 + (tid & 7) * 8;
    int asked = c0, stage_to = 0;
    auto load = [&]() {
      if (asked < c1) {
        const uint32_t dst = base + (uint32_t)(stage_to * stage_bytes + copy_to);
#pragma unroll
        for (int k = 0; k < 2; k++) { lora_copy16(dst + 32 * 128 * k, from_x[k]); from_x[k] += 64; }
#pragma unroll
        for (int k = 0; k < (STEPS + 1) / 2; k++)
          if (copy_row + 32 * k < R) lora_copy16(dst + (kLoraTile + 32 * k) * 128, from_a + (long long)32 * k * p.K);
        from_a += 64;
        asked++;
      }
      if (++stage_to == kDownStages) stage_to = 0;
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int n = 0; n < STEPS; n++)
#pragma unroll
      for (int k = 0; k < 4; k++) acc[n][k] = 0.f;
#pragma unroll
    for (int c = 0; c < kDownStages - 1; c++) load();
    int stage = 0;
    for (int c = c0; c < c1; c++) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kDownStages - 2) : "memory");
      __syncthreads();
      load();
      const uint32_t xs = base + (uint32_t)(stage * stage_bytes), as = xs + kLoraTile * 128;
      if (++stage == kDownStages) stage = 0;
#pragma unroll
      for (int q = 0; q < 2; q++) {
        const uint32_t at = (uint32_t)(((4 * q + j) ^ ((g & 1) << 2)) << 4);
        const uint4 u = lora_lds(xs + (mt * 16 + g) * 128 + at), v = lora_lds(xs + (mt * 16 + 8 + g) * 128 + at);
#pragma unroll
        for (int n = 0; n < STEPS; n++)
          if (n < STEPS - 1 || n < nn) {
            const uint4 w = lora_lds(as + ((n0 + n) * 8 + g) * 128 + at);
            lora_mma(acc[n], u.x, v.x, u.y, v.y, w.x, w.y);
            lora_mma(acc[n], u.z, v.z, u.w, v.w, w.z, w.w);
          }
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    float* const out = reinterpret_cast<float*>(lora_shared);   // [tokens][rank]: no more than the ring
#pragma unroll
    for (int n = 0; n < STEPS; n++)
      if (n < nn)
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const int t = mt * 16 + h * 8 + g;
          if (s.adapter[t] == i) *reinterpret_cast<float2*>(out + t * R + (n0 + n) * 8 + 2 * j) = make_float2(acc[n][2 * h], acc[n][2 * h + 1]);
        }
    // the parts of the cluster's CTAs, each CTA a share of the sums
    cluster_barrier();
    const int share = kLoraTile / p.parts;
    const float scaling = p.scaling[i];
    for (int t = share * (int)part + warp; t < share * ((int)part + 1); t += kLoraWarps) {   // a warp a token, a lane four of its z
      if (s.adapter[t] != i) continue;
      const int r = 4 * lane;
      float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < R) {
        const uint32_t here = base + (uint32_t)((t * R + r) * 4);
        float4 w[8];
#pragma unroll
        for (int c = 0; c < 8; c++) {
          w[c] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (c < p.parts)
            asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [a];\n\t}"
                         : "=f"(w[c].x), "=f"(w[c].y), "=f"(w[c].z), "=f"(w[c].w) : "r"(here), "r"(c) : "memory");
        }
#pragma unroll
        for (int c = 0; c < 8; c++) { z.x += w[c].x; z.y += w[c].y; z.z += w[c].z; z.w += w[c].w; }
        z.x *= scaling; z.y *= scaling; z.z *= scaling; z.w *= scaling;
      }
      // z / 2^exponent, below 2^15, in two fp16 numbers, zeroes behind the rank (up to a multiple of 16)
      const float top = fmaxf(fmaxf(fabsf(z.x), fabsf(z.y)), fmaxf(fabsf(z.z), fabsf(z.w)));
      const int exponent = min(max((int)(__reduce_max_sync(0xffffffffu, __float_as_uint(top)) >> 23) - 126 - kLoraRoom, -100), 126);   // |z| < 2^(exponent + kLoraRoom)
      const float inv = __int_as_float((127 - exponent) << 23);
      if (lane == 0) reinterpret_cast<LoraTokens*>(record)->unit[t] = __int_as_float((exponent + 127) << 23);
      if (r < 16 * STEPS) {
        z.x *= inv; z.y *= inv; z.z *= inv; z.w *= inv;
        const __half2 h0 = __floats2half2_rn(z.x, z.y), h1 = __floats2half2_rn(z.z, z.w);
        const float2 f0 = __half22float2(h0), f1 = __half22float2(h1);
        const __half2 l0 = __floats2half2_rn(z.x - f0.x, z.y - f0.y), l1 = __floats2half2_rn(z.z - f1.x, z.w - f1.y);
        // row t % 16 of its 16 tokens, inner elements 4 q .. 4 q + 3 of a step: registers 0 and 2 of lane (t % 8) 4 + q, 1 and 3 for the lower eight rows
        uint32_t* const to = reinterpret_cast<uint32_t*>(record + kLoraRecordZ + ((t >> 4) * STEPS + (r >> 4)) * 512 + ((t & 7) * 4 + (lane & 3)) * 16) + (t >> 3 & 1);
        constexpr int lower = kLoraTile / 16 * STEPS * 128;   // in words
        to[0] = *reinterpret_cast<const uint32_t*>(&h0);
        to[2] = *reinterpret_cast<const uint32_t*>(&h1);
        to[lower] = *reinterpret_cast<const uint32_t*>(&l0);
        to[lower + 2] = *reinterpret_cast<const uint32_t*>(&l1);
      }
    }
    cluster_barrier();   // nobody overwrites its ring, or ends, while others read from it
  }
}

constexpr int kUpCols = 128;   // columns of a tile (32 a warp); a CTA has p.up_tiles of them: a few short waves of CTAs (lora_many)
// shared memory of lora_up_kernel: z, two stages of a tile's rows of b, three of what is added to; rows with gaps against bank conflicts
template <int STEPS>
struct UpLayout {
  static constexpr int row = STEPS * 16 + 16;                       // halves of a row of b
  static constexpr int z = 0, stage0 = STEPS * 4096;                // z as in the record
  static constexpr int b_bytes = kUpCols * row * 2, base_row = kUpCols * 2 + 16, add_bytes = kLoraTile * base_row;
  static constexpr int add0 = stage0 + 2 * b_bytes, bytes = add0 + 3 * add_bytes;   // (what comes from far away is asked for one tile earlier)
};
// y of kLoraTile tokens x p.up_tiles * kUpCols columns; a warp has half of the tile's tokens and 32 columns. Column c of n-tile n is column
// 8 (c / 2) + 2 n + c % 2 of the 32, so that a thread's sums of a row are eight columns side by side and meet base and y in 16 bytes.
// The next tile's rows of b and of base are on their way to shared memory meanwhile.
// STEPS: the rank in steps of 16, rounded up; WIDE: rows of base and y start on 16 bytes
template <int STEPS, bool WIDE>
__global__ void __launch_bounds__(kLoraThreads, STEPS <= 4 ? 2 : 1) lora_up_kernel(const LoraParams p) {
  using L = UpLayout<STEPS>;
  extern __shared__ __align__(128) uint8_t lora_shared[];
  __shared__ LoraTokens s;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3, R = p.rank;
  const uint32_t base = (uint32_t)__cvta_generic_to_shared(lora_shared);
  const int m0 = (int)blockIdx.y * kLoraTile;
  const uint8_t* const record = p.z + (long long)blockIdx.y * lora_record_bytes(R);
  if (tid < (int)(sizeof(LoraTokens) / 16)) reinterpret_cast<uint4*>(&s)[tid] = reinterpret_cast<const uint4*>(record)[tid];
#pragma unroll
  for (int k = 0; k < STEPS; k++) lora_copy16(base + 16 * (tid + k * kLoraThreads), record + kLoraRecordZ + 16 * (tid + k * kLoraThreads));
  __syncthreads();
  // passes of a tile: the adapters, and the rows without any if there are some; this CTA has every splits-th
  const int different = s.count, split = (int)blockIdx.z, splits = (int)gridDim.z, passes = (different + (s.none ? 1 : 0) - split + splits - 1) / splits;
  const int first = (int)blockIdx.x * p.up_tiles, tiles = min(p.up_tiles, (p.N + kUpCols - 1) / kUpCols - first);
  // Copies of a thread, 16 bytes each: of b every second piece of one row, of base a piece of every sixteenth row.
  const int b_row = tid >> 1, b_odd = tid & 1, add_row = tid >> 4, add_col = 8 * (tid & 15);
  const uint32_t b_to = base + (uint32_t)(L::stage0 + b_row * L::row * 2 + b_odd * 16);
  const uint32_t add_to = base + (uint32_t)(L::add0 + add_row * L::base_row + add_col * 2);
  if (passes <= 0) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  int add_adapter[4];
  const __half* add_from[4];
#pragma unroll
  for (int k = 0; k < 4; k++) {
    const int row = add_row + 16 * k;
    add_adapter[k] = p.base && WIDE ? s.adapter[row] : -2;
    add_from[k] = p.base + (long long)(m0 + row) * p.N + first * kUpCols + add_col;
  }
  int b_tile = 0, b_pass = 0, add_tile = 0, add_pass = 0, b_stage = 0, add_stage = 0;
  auto load_b = [&]() {   // of the next pass
    if (b_tile < tiles) {
      const int e = split + b_pass * splits, i = e < different ? s.list[e] : -1, n0 = (first + b_tile) * kUpCols;
      if (i >= 0 && n0 + b_row < p.N) {
        const __half* const from = p.b + ((long long)i * p.N + n0 + b_row) * R + 8 * b_odd;
#pragma unroll
        for (int q = 0; q < STEPS; q++)
          if (q < STEPS - 1 || 16 * (STEPS - 1) + 8 * b_odd < R) lora_copy16(b_to + b_stage * L::b_bytes + 32 * q, from + 16 * q);
      }
      if (++b_pass == passes) { b_pass = 0; b_tile++; }
    }
    b_stage ^= 1;
  };
  auto load_add = [&]() {
    if (add_tile < tiles) {
      const int e = split + add_pass * splits, i = e < different ? s.list[e] : -1;
      if ((first + add_tile) * kUpCols + add_col < p.N)
#pragma unroll
        for (int k = 0; k < 4; k++)
          if (add_adapter[k] == i) lora_copy16(add_to + add_stage * L::add_bytes + 16 * k * L::base_row, add_from[k] + add_tile * kUpCols);
      if (++add_pass == passes) { add_pass = 0; add_tile++; }
    }
    if (++add_stage == 3) add_stage = 0;
  };
  const int all = tiles * passes;
  // the rest of an odd number of pieces: never written again
  for (int v = tid; v < 2 * kUpCols; v += kLoraThreads)
    *reinterpret_cast<uint4*>(lora_shared + L::stage0 + (v / kUpCols) * L::b_bytes + (v % kUpCols) * L::row * 2 + (STEPS * 16 - 8) * 2) = make_uint4(0, 0, 0, 0);
  __syncthreads();
  load_b();
  load_add();
  asm volatile("cp.async.commit_group;" ::: "memory");
  load_b();
  load_add();
  load_add();
  asm volatile("cp.async.commit_group;" ::: "memory");
  // this thread's four rows: their adapters (-2: no such row), units and places
  const int t0 = (warp >> 2) * 32;
  int adapter[2][2];
  float unit[2][2];
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int t = t0 + m * 16 + h * 8 + g;
      adapter[m][h] = s.adapter[t];
      unit[m][h] = s.unit[t];
    }
  __half* to[2][2];
#pragma unroll
  for (int m = 0; m < 2; m++)
#pragma unroll
    for (int h = 0; h < 2; h++) to[m][h] = p.y + (long long)(m0 + t0 + m * 16 + h * 8 + g) * p.N;
  const uint8_t* const z0 = lora_shared + (t0 >> 4) * STEPS * 512 + lane * 16;
  const int b_at = ((warp & 3) * 32 + 8 * (g >> 1) + (g & 1)) * L::row * 2 + 8 * j;                 // column of n-tile 0, and 2 n rows on
  const int base_at = (t0 + g) * L::base_row + ((warp & 3) * 32 + 8 * j) * 2;
  int tile = 0, pass = 0, add_now = 0;
  for (int k = 0; k < all; k++) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();
    const uint8_t *const st = lora_shared + L::stage0 + (k & 1) * L::b_bytes, *const add_st = lora_shared + L::add0 + add_now * L::add_bytes;
    const int e = split + pass * splits, i = e < different ? s.list[e] : -1, col = (first + tile) * kUpCols + (warp & 3) * 32 + 8 * j;
    bool mine[2][2], any = false;
#pragma unroll
    for (int m = 0; m < 2; m++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        mine[m][h] = adapter[m][h] == i && col < p.N;
        any |= mine[m][h];
      }
    if (__any_sync(0xffffffffu, any)) {
      float acc[2][4][4];
      if (i >= 0) {
        // fragments of four steps at a time, all asked for in front of the products
        constexpr int AHEAD = STEPS < 4 ? STEPS : 4;
#pragma unroll
        for (int x0 = 0; x0 < STEPS; x0 += AHEAD) {
          uint2 bv[AHEAD][4];
          uint4 a[AHEAD][2];
#pragma unroll
          for (int x = 0; x < AHEAD; x++)
#pragma unroll
            for (int n = 0; n < 4; n++)
              if (x0 + x < STEPS) bv[x][n] = *reinterpret_cast<const uint2*>(st + b_at + 2 * n * L::row * 2 + 32 * (x0 + x));
#pragma unroll
          for (int mh = 0; mh < 4; mh++) {   // (upper, lower parts) x (tokens 0 .. 15, 16 .. 31)
            const int m = mh & 1, h = mh >> 1;
#pragma unroll
            for (int x = 0; x < AHEAD; x++)
              if (x0 + x < STEPS) a[x][mh & 1] = *reinterpret_cast<const uint4*>(z0 + ((h * (kLoraTile / 16) + m) * STEPS + x0 + x) * 512);
#pragma unroll
            for (int x = 0; x < AHEAD; x++)
              if (x0 + x < STEPS)
#pragma unroll
                for (int n = 0; n < 4; n++) {
                  const uint4 u = a[x][mh & 1];
                  if (x0 + x == 0 && h == 0) lora_mma_first(acc[m][n], u, bv[x][n].x, bv[x][n].y);
                  else lora_mma(acc[m][n], u.x, u.y, u.z, u.w, bv[x][n].x, bv[x][n].y);
                }
          }
        }
      }
      if constexpr (WIDE) {
#pragma unroll
        for (int m = 0; m < 2; m++)
#pragma unroll
          for (int h = 0; h < 2; h++) {
            if (!mine[m][h]) continue;
            const uint4 add = p.base ? *reinterpret_cast<const uint4*>(add_st + base_at + (m * 16 + h * 8) * L::base_row) : make_uint4(0, 0, 0, 0);
            float v[8];
            halves8(add, v);
            uint32_t w[4];
#pragma unroll
            for (int n = 0; n < 4; n++) {
              const __half2 y = __floats2half2_rn(fmaf(acc[m][n][2 * h], unit[m][h], v[2 * n]), fmaf(acc[m][n][2 * h + 1], unit[m][h], v[2 * n + 1]));
              w[n] = *reinterpret_cast<const uint32_t*>(&y);
            }
            // (without an adapter the row as it is, the signs of its zeroes too)
            *reinterpret_cast<uint4*>(to[m][h] + col) = i < 0 ? add : make_uint4(w[0], w[1], w[2], w[3]);
          }
      } else {
        // Rows that do not start on 16 bytes: the sums through shared memory (where base would be), so that a warp has 32 columns of one row at a time
        // (1743 tokens, 21607 columns, rank 56: 234 us with each thread's own eight columns, two bytes a time; 133 so).
        constexpr int pitch = 36;
        static_assert(kLoraWarps * 32 * pitch * 4 <= 3 * L::add_bytes, "");
        float* const sums = reinterpret_cast<float*>(lora_shared + L::add0) + warp * 32 * pitch;
        if (i >= 0) {
#pragma unroll
          for (int m = 0; m < 2; m++)
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
              for (int n = 0; n < 4; n += 2)
                *reinterpret_cast<float4*>(sums + (m * 16 + h * 8 + g) * pitch + 8 * j + 2 * n) =
                    make_float4(acc[m][n][2 * h], acc[m][n][2 * h + 1], acc[m][n + 1][2 * h], acc[m][n + 1][2 * h + 1]);
        }
        __syncwarp();
        const int c = col - 8 * j + lane;
        const long long at = (long long)(m0 + t0) * p.N + c;
        for (int r0 = 0; r0 < 32; r0 += 16) {
          __half add[16];
#pragma unroll
          for (int r = 0; r < 16; r++)
            add[r] = p.base && c < p.N && s.adapter[t0 + r0 + r] == i ? p.base[at + (long long)(r0 + r) * p.N] : __float2half_rn(0.f);
#pragma unroll
          for (int r = 0; r < 16; r++)
            if (c < p.N && s.adapter[t0 + r0 + r] == i)
              p.y[at + (long long)(r0 + r) * p.N] =
                  i < 0 ? add[r] : __float2half_rn(fmaf(sums[(r0 + r) * pitch + lane], s.unit[t0 + r0 + r], __half2float(add[r])));
        }
      }
    }
    __syncthreads();
    load_b();
    load_add();
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (++add_now == 3) add_now = 0;
    if (++pass == passes) { pass = 0; tile++; }
  }
}

}  // namespace rcp
