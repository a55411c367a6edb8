// Attention of many rows of a sequence (prompts, long guesses) over the paged 8-bit cache on tcgen05; the operator is that of
// kv_attention.cuh, for the sequences whose new tokens times query heads of a key head are more than p.few.
//
// Work. One CTA a key head and 256 rows of a sequence (tokens x query heads that share the key head, token by token), two row tiles of 128.
// For each tile of 64 keys: S_t = Q_t K^T (both operands in shared memory), weights to tensor memory as fp16 in the place of the scores,
// O_t += P_t V (weights from tensor memory). Tensor memory is full: for each row tile two tiles of scores and the sums, 2 x 64 + dim columns.
// Warps. Four that turn codes into fp16, once for all 256 rows, from memory through registers into shared memory (128-byte
// swizzle; values keep their order, keys along the rows, and are read as a transposed operand); two that issue, one a row tile, so that neither
// waits for the other's softmax; eight for the softmax, one thread a row. The next tile's scores are made while the softmax works on these.
// Softmax as in kv_attention.cuh: a row's reference moves only when a score is more than kAttnSlack above it, the sums in tensor memory
// are rescaled then. (The sum of the weights is of fp32 ones here, before they are rounded to fp16 for the product: tensor memory has no column left for
// it, and adding the rounded ones again would be 64 conversions more in a chain that is what bounds the kernel. So their roundings do not cancel: off by
// 2.5e-4 of the results' norm, 2.2e-4 in the kernel of few rows, 2.1e-4 for the rounding of the result alone.) The scales of the values' blocks
// are folded into the fp16 values relative to a power of two, the unit of the sums, which stays while the exponents of a tile's one or two blocks are
// within -15 .. 7 of it (fp16 holds codes of 2^-9 .. 448 exactly there) and otherwise moves to four above the larger one, less where the smaller one
// would be out of that range; converters and softmax warps follow the same rule on the same scales, so nothing has to be handed over. (Of two blocks
// in the same 64 keys, which only pages of 32 have, one whose scale is more than 2^22 below the other's loses low bits of its smallest codes, one 2^32
// below all of them.)
// Bound by the softmax warps' chain of a tile: of 2250 clocks factors and masks take 380, the wait for the scores 195, reading them 87, their
// maximum 470, exponentials, sums and fp16 1090; the tensor pipe is at work 1280 of them (64 keys of both row tiles; the scores' products are
// bound by shared memory, 48 clocks each instead of 32), the exponentials' unit 1024. 32 heads on 8, prompts of 2000, 1790 and 1190 tokens behind
// 3000, 2506 and 2154: 336 us, 848 TFLOP/s; 17 % of it is the last wave of CTAs. 64 wide the softmax has as much to do for half the products: 294 us, 483
// TFLOP/s (12 bytes of registers are spilled there). Steps: tiles of 128 keys with one tile of scores 446 us; with the 128
// scores of a row in registers at once (spilled) 529; the next scores read between the exponentials 429 (they are waited for a whole chain too
// early: the place they go to is free only when the weights in it have been multiplied); two threads a row, sixteen softmax warps, 381.
#pragma once
#include "kv_attention.cuh"
#include "ptx.cuh"

namespace rcp {

constexpr int kPromptThreads = 512, kPromptRows = 256, kPromptKeys = 64, kPromptStages = 4;

constexpr uint32_t kPromptPolls = 1u << 18;   // a wait of this kernel is a few microseconds

template <int DIM>
struct PromptLayout {
  static constexpr int q_bytes = 128 * DIM * 2, tile_bytes = kPromptKeys * DIM * 2;   // fp16, in blocks of 64 elements: 128 bytes a row
  static constexpr int q = 0, k = 2 * q_bytes, v = k + kPromptStages * tile_bytes, bars = v + kPromptStages * tile_bytes;
  static constexpr int bytes = bars + 256 + 1024;            // the swizzle wants 1024-byte alignment
};

__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
        "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
               "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void tmem_st32w(uint32_t at, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// fp32 += fp16 x fp16; A from shared memory or from tensor memory (at `a`)
__device__ __forceinline__ void umma_ss(uint32_t elected, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 ad, bd;\n\tmov.b64 ad, {%1, %3};\n\tmov.b64 bd, {%2, %3};\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], ad, bd, %4, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(elected), "r"(acc)
               : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t elected, uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 bd;\n\tmov.b64 bd, {%2, %3};\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], bd, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(elected), "r"(acc)
               : "memory");
}


// two fp32 numbers at a time
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Pages and scales of a sequence's keys in units of 32, one unit a lane, 32 units (sixteen tiles) at a time; the next 32 are asked for ahead.
struct PromptBlocks {
  const KvSeqs* s;
  const int32_t* row;                 // the sequence's row of the table
  const float *k_scale, *v_scale;
  int kv, kv_heads, end, lane;
  int page, next_page;                // -1: none
  float ks, next_ks;
  int ve, next_ve;                    // exponent of the values' scale
  int range;                          // in which the unit may stay with a tile's one or two blocks: from (even lanes), to (odd lanes)
  int unit;                           // exponent of the unit of the sums; kNoUnit in front of the first tile
  static constexpr int kNone = -1000, kNoUnit = 1000;   // of a block that is not there

  __device__ __forceinline__ int find(int at) const {   // page of keys 32 at ..
    if (at * 32 >= end) return -1;
    const int pg = row[at * 32 >> s->lg_page];
    return pg >= 0 && pg < s->pages ? pg : -1;
  }
  __device__ __forceinline__ void scales(int pg, float& k, int& v) const {
    k = pg >= 0 ? k_scale[(long long)pg * kv_heads + kv] : 1.f;
    v = pg >= 0 ? kv_stored_exponent(v_scale[(long long)pg * kv_heads + kv]) : kNone;
  }
  __device__ __forceinline__ void start() {
    next_page = find(lane);
    scales(next_page, next_ks, next_ve);
    unit = kNoUnit;
  }
  // to be called for every tile in turn; returns by how many powers of two the sums' unit grows with it (0 as a rule)
  __device__ __forceinline__ int step(int tile) {
    if ((tile & 15) == 0) {
      page = next_page; ks = next_ks; ve = next_ve;
      const int other = __shfl_xor_sync(0xffffffffu, ve, 1), top = max(ve, other), low = min(ve, other) == kNone ? top : min(ve, other);
      range = top == kNone ? (lane & 1 ? kNoUnit : -kNoUnit) : lane & 1 ? max(low + 15, top - 7) : top - 7;
      next_page = find((tile + 16) * 2 + lane);
    }
    if ((tile & 15) == 8) scales(next_page, next_ks, next_ve);
    // (a vote on sixteen tiles at once instead, without these shuffles as a rule: 348 us against 337, the branch keeps other instructions from between them)
    const int from = __shfl_sync(0xffffffffu, range, (tile & 15) * 2), to = __shfl_sync(0xffffffffu, range, (tile & 15) * 2 + 1);
    if (unit >= from && unit <= to) return 0;
    const int now = min(from + 11, to), grow = unit == kNoUnit ? 0 : now - unit;
    unit = now;
    return grow;
  }
};

// LIMITED: waits of p.polls polls, for tests of giving up (with them for all, 28 bytes of registers are spilled and prompts take 2 us more)
template <int DIM, bool LIMITED>
__global__ void __launch_bounds__(kPromptThreads, 1) kv_attention_prompt_kernel(const AttnParams p) {
  using L = PromptLayout<DIM>;
  constexpr int BLOCK_Q = 128 * 128, BLOCK = kPromptKeys * 128;   // bytes of a 64-element block of 128 queries, of a tile's keys
  extern __shared__ uint8_t prompt_raw[];
  __shared__ uint32_t s_tmem;
  const uint32_t raw = smem_u32(prompt_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const gen = prompt_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // which sequence and rows: candidate floor(starts[b] group / 256) + b + j is tile j of sequence b; the last ones first, they have most keys
  const int kv = (int)blockIdx.x % p.kv_heads, cand = (int)(gridDim.x / p.kv_heads) - 1 - (int)blockIdx.x / p.kv_heads;
  int lo = 0, hi = p.s.seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((int)((long long)p.s.starts[mid] * p.group / kPromptRows) + mid <= cand) lo = mid; else hi = mid;
  }
  const KvSeq sq = kv_seq(p.s, lo);
  const int b = lo, tile_row = (cand - (int)((long long)p.s.starts[b] * p.group / kPromptRows) - b) * kPromptRows;
  const int total_rows = sq.n * p.group, rows = min(total_rows - tile_row, kPromptRows);
  // Few rows are the other kernel's, which is launched behind this one unless there is but one sequence. Behind a wait that gave up nothing
  // more is waited for: the rows are NaN until the status is cleared.
  const int gave_up = __syncthreads_or(tid == 0 && *reinterpret_cast<volatile int32_t*>(p.status) != 0);
  const bool mine = tile_row >= 0 && rows > 0 && total_rows > p.few;
  constexpr uint32_t kNoResult = 0x7FFF7FFFu;   // NaN
  if (gave_up || !mine) {
    asm volatile("griddepcontrol.launch_dependents;");
    if (mine)
      for (int x = tid; x < rows * (DIM / 8); x += kPromptThreads) {
        const int r = tile_row + x / (DIM / 8), i = r / p.group;
        *reinterpret_cast<uint4*>(p.out + ((long long)(sq.t0 + i) * p.heads + (long long)kv * p.group + (r - i * p.group)) * DIM + x % (DIM / 8) * 8) =
            make_uint4(kNoResult, kNoResult, kNoResult, kNoResult);
      }
    return;
  }
  const int last_pos = sq.first + (tile_row + rows - 1) / p.group;
  const int keys = min(max(last_pos + 1, 0), sq.end), tiles = (keys + kPromptKeys - 1) / kPromptKeys;
  const int halves = rows > 128 ? 2 : 1;

  const uint32_t bar = base + L::bars;
  constexpr uint32_t STAGES = kPromptStages;
  const uint32_t k_full = bar, k_empty = k_full + 8 * STAGES, v_full = k_empty + 8 * STAGES, v_empty = v_full + 8 * STAGES;
  const uint32_t s_full = v_empty + 8 * STAGES;                                      // [row tile][buffer]
  const uint32_t p_full = s_full + 32;                                               // [row tile][buffer]: a warp may be a tile ahead of the others
  const uint32_t o_done = p_full + 32, drained = o_done + 16;                        // [row tile]
  if (tid == 0) {
    for (uint32_t i = 0; i < STAGES; i++) {
      mbar_init(k_full + 8 * i, 128);
      mbar_init(k_empty + 8 * i, halves);
      mbar_init(v_full + 8 * i, 128);
      mbar_init(v_empty + 8 * i, halves);
    }
    for (int i = 0; i < 2; i++) {
      mbar_init(s_full + 16 * i, 1);
      mbar_init(s_full + 16 * i + 8, 1);
      mbar_init(p_full + 16 * i, 128);
      mbar_init(p_full + 16 * i + 8, 128);
      mbar_init(o_done + 8 * i, 1);
      mbar_init(drained + 8 * i, 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 15) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // queries, 16 bytes at a time; rows that do not exist are zeroes
  for (int x = tid; x < halves * 128 * (DIM / 8); x += kPromptThreads) {
    const int row = x / (DIM / 8), c = x % (DIM / 8), r = tile_row + row, i = r / p.group;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (row < rows)
      v = *reinterpret_cast<const uint4*>(p.q + (long long)(sq.t0 + i) * p.q_stride + (long long)(kv * p.group + r - i * p.group) * DIM + 8 * c);
    *reinterpret_cast<uint4*>(gen + L::q + (row >> 7) * L::q_bytes + (c >> 3) * BLOCK_Q + (row & 127) * 128 + (((c & 7) ^ (row & 7)) << 4)) = v;
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  // the next kernel may start when every CTA has its tensor memory: one that waits for this one must not hold what this one wants
  asm volatile("griddepcontrol.launch_dependents;");

  PromptBlocks blocks;
  blocks.s = &p.s;
  blocks.row = p.s.table + (long long)b * p.s.width;
  blocks.k_scale = p.k_scale; blocks.v_scale = p.v_scale;
  blocks.kv = kv; blocks.kv_heads = p.kv_heads; blocks.end = sq.end; blocks.lane = lane;
  constexpr uint32_t kS = 0, kO = 256;   // tensor memory: scores (and weights) of the row tiles, then their sums
  bool ok = true;
  auto prompt_wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_warp(bar, parity, LIMITED ? p.polls : kPromptPolls); };

  if (warp < 8) {
    // ---------------------------------------------------------------- softmax: a thread a row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    const int half = warp >> 2;
    if (half < halves) {
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, at_s = kS + 128u * half + lanes, at_o = kO + (uint32_t)(DIM * half) + lanes;
      const int r = tile_row + half * 128 + (warp & 3) * 32 + lane;
      const bool have = r < total_rows;
      const int i = r / p.group, pos = sq.first + i;
      const int lim = !have ? INT_MAX : pos >= 0 && pos < sq.end ? pos + 1 : 0;   // keys the row sees
      const int least = (int)__reduce_min_sync(0xffffffffu, lim);
      float m = kAttnNoMax, l = 0.f;
      blocks.start();
      for (int t = 0; t < tiles; t++) {
        const int grow = blocks.step(t);
        float c[2];
        bool some = true;
#pragma unroll
        for (int k = 0; k < 2; k++) {
          const int from = (t & 15) * 2 + k;
          c[k] = fmaxf(__shfl_sync(0xffffffffu, blocks.ks, from) * p.scale_log2, 1e-37f);   // above zero: a score of -inf stays one
          some = some && __shfl_sync(0xffffffffu, blocks.page, from) >= 0;
        }
        const uint32_t at = at_s + 64u * (t & 1);
        ok = prompt_wait(s_full + 16 * half + 8 * (t & 1), (uint32_t)(t >> 1) & 1u);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        uint32_t s[2][32];
        tmem_ld32(at, s[0]);
        tmem_ld32(at + 32u, s[1]);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        if (!some || (t + 1) * kPromptKeys > least) {   // keys that some row of the warp does not see, or that are not there
#pragma unroll
          for (int k = 0; k < 2; k++) {
            const int left = __shfl_sync(0xffffffffu, blocks.page, (t & 15) * 2 + k) >= 0 ? lim - t * kPromptKeys - 32 * k : 0;
#pragma unroll
            for (int x = 0; x < 32; x++)
              if (x >= left) s[k][x] = 0xFF800000u;
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 2; k++) {
          float a[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int x = 0; x < 16; x++) a[x & 3] = max3(a[x & 3], __uint_as_float(s[k][2 * x]), __uint_as_float(s[k][2 * x + 1]));
          top = fmaxf(top, max3(fmaxf(a[0], a[1]), a[2], a[3]) * c[k]);
        }
        if (__any_sync(0xffffffffu, top > m + kAttnSlack || grow != 0)) {
          const float mn = fmaxf(m, top), f = exp2_fast(m - mn);
          m = mn;
          l *= f;
          const float fu = f * kv_pow2(min(max(-grow, -100), 100));
          if (t > 0) {
            ok = prompt_wait(o_done + 8 * half, (t - 1) & 1);   // the product of the tile in front is in the sums
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int d = 0; d < DIM / 32; d++) {
              uint32_t o[32];
              tmem_ld32(at_o + 32u * d, o);
              asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
              for (int x = 0; x < 32; x++) o[x] = __float_as_uint(__uint_as_float(o[x]) * fu);
              tmem_st32w(at_o + 32u * d, o);
            }
          }
        }
        const float ref = m - kAttnLift;
        float2 sum[2] = {};
#pragma unroll
        for (int k = 0; k < 2; k++) {
          uint32_t w[16];
#pragma unroll
          for (int x = 0; x < 16; x++) {
            const float2 y = fma2(make_float2(__uint_as_float(s[k][2 * x]), __uint_as_float(s[k][2 * x + 1])), make_float2(c[k], c[k]), make_float2(-ref, -ref));
            const float2 e = make_float2(exp2_fast(y.x), exp2_fast(y.y));
            const __half2 h = __float22half2_rn(e);
            w[x] = *reinterpret_cast<const uint32_t*>(&h);
            sum[x & 1] = add2(sum[x & 1], e);
          }
          tmem_st16(at + 16u * k, w);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        mbar_arrive(p_full + 16 * half + 8 * (t & 1));
      }
      if (ok) ok = prompt_wait(drained + 8 * half, 0);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      __half* const to = p.out + ((long long)(sq.t0 + i) * p.heads + (long long)kv * p.group + (r - i * p.group)) * DIM;
      if (!ok && have) {
#pragma unroll
        for (int d = 0; d < DIM / 8; d++) reinterpret_cast<uint4*>(to)[d] = make_uint4(kNoResult, kNoResult, kNoResult, kNoResult);
      }
      if (ok) {
        const float f = l > 0.f ? kv_pow2(min(max(blocks.unit, -100), 100)) / l : l;
#pragma unroll
        for (int d = 0; d < DIM / 32; d++) {
          uint32_t o[32];
          if (tiles > 0) {
            tmem_ld32(at_o + 32u * d, o);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          }
          if (have) {
#pragma unroll
            for (int x = 0; x < 4; x++) {
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 4; k++) {
                const __half2 h = tiles > 0 && l != 0.f ? __floats2half2_rn(__uint_as_float(o[8 * x + 2 * k]) * f, __uint_as_float(o[8 * x + 2 * k + 1]) * f)
                                                        : __floats2half2_rn(0.f, 0.f);
                w[k] = *reinterpret_cast<const uint32_t*>(&h);
              }
              *reinterpret_cast<uint4*>(to + 32 * d + 8 * x) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
      }
    }
  } else if (warp < 12) {
    // ---------------------------------------------------------------- converters
    asm volatile("setmaxnreg.dec.sync.aligned.u32 112;");
    // A thread has row `me / 4` of each unit of 32 keys and a quarter of each of its 64-element blocks, 16 codes: 64 bytes of a row to four
    // lanes, and no two lanes of eight that store together in the same banks (rows side by side differ in the swizzle).
    constexpr int BLOCKS = DIM / 64, UNITS = kPromptKeys / 32, COPIES = UNITS * BLOCKS;
    const int me = tid - 256, row = me >> 2, quarter = me & 3;
    blocks.start();
    uint4 codes[2][COPIES];   // keys, values: asked for a tile ahead
    long long from[UNITS];    // the row's place in the cache, below zero: none
    auto ask = [&](uint4 (&to)[COPIES], const uint8_t* cache) {
#pragma unroll
      for (int u = 0; u < UNITS; u++)
#pragma unroll
        for (int k = 0; k < BLOCKS; k++) {
          to[u * BLOCKS + k] = make_uint4(0, 0, 0, 0);
          if (from[u] >= 0) to[u * BLOCKS + k] = __ldcg(reinterpret_cast<const uint4*>(cache + from[u] + 64 * k));
        }
    };
    const uint32_t to0 = (uint32_t)(row * 128) + (((uint32_t)(2 * quarter) ^ ((uint32_t)row & 7u)) << 4);
    auto put = [&](const uint4 (&codes)[COPIES], uint32_t dst, bool values, const int (&shift)[UNITS]) {
#pragma unroll
      for (int u = 0; u < UNITS; u++) {
        const __half2 f = __float2half2_rn(kv_pow2(min(max(shift[u], -30), 7)));
#pragma unroll
        for (int k = 0; k < BLOCKS; k++) {
          const uint4 c = codes[u * BLOCKS + k];
          uint32_t h[8];
          e4m3_halves(c.x, h[0], h[1]);
          e4m3_halves(c.y, h[2], h[3]);
          e4m3_halves(c.z, h[4], h[5]);
          e4m3_halves(c.w, h[6], h[7]);
          if (values) {
#pragma unroll
            for (int x = 0; x < 8; x++) {
              const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&h[x]), f);
              h[x] = *reinterpret_cast<const uint32_t*>(&y);
            }
          }
          const uint32_t at = dst + to0 + (uint32_t)(k * BLOCK + u * 32 * 128);
          asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
          asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at ^ 16u), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
        }
      }
    };
    int shift[UNITS];
    // where the thread's rows of tile t are, and how far the values' exponents are from the unit of the sums
    auto step = [&](int t) {
      blocks.step(t);
#pragma unroll
      for (int k = 0; k < UNITS; k++) {
        const int page = __shfl_sync(0xffffffffu, blocks.page, (t & 15) * 2 + k), ve = __shfl_sync(0xffffffffu, blocks.ve, (t & 15) * 2 + k);
        const int j = t * kPromptKeys + 32 * k + row;
        shift[k] = page >= 0 ? ve - blocks.unit : 0;
        from[k] = page >= 0 && j < sq.end ? (((long long)page * p.kv_heads + kv) * p.s.page + (j & (p.s.page - 1))) * DIM + 16 * quarter : -1;
      }
    };
    if (tiles > 0) {
      step(0);
      ask(codes[0], p.k_cache);
      ask(codes[1], p.v_cache);
    }
    for (int t = 0; t < tiles; t++) {
      const int stage = t % kPromptStages;
      const uint32_t parity = (uint32_t)(t / kPromptStages) & 1u;
      int now[UNITS];
#pragma unroll
      for (int k = 0; k < UNITS; k++) now[k] = shift[k];
      if (t + 1 < tiles) step(t + 1);
      ok = prompt_wait(k_empty + 8 * stage, parity ^ 1u);
      if (!ok) break;
      put(codes[0], base + L::k + stage * L::tile_bytes, false, now);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(k_full + 8 * stage);
      if (t + 1 < tiles) ask(codes[0], p.k_cache);
      ok = prompt_wait(v_empty + 8 * stage, parity ^ 1u);
      if (!ok) break;
      put(codes[1], base + L::v + stage * L::tile_bytes, true, now);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(v_full + 8 * stage);
      if (t + 1 < tiles) ask(codes[1], p.v_cache);
    }
  } else {
    // ---------------------------------------------------------------- issuers, one a row tile
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    const int half = warp - 12;
    if (half < halves) {
      const uint32_t elected = elect_one() ? 1u : 0u;
      // 128-byte swizzle, eight rows 1024 bytes; values: 64 elements and 64 keys on, a block on
      const uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
      const uint32_t q0 = (base + L::q + half * L::q_bytes) >> 4 | 1u << 16;
      const uint32_t k0 = (base + L::k) >> 4 | 1u << 16, v0 = (base + L::v) >> 4 | (uint32_t)(BLOCK >> 4) << 16;
      const uint32_t idesc_s = (1u << 4) | (uint32_t)(kPromptKeys >> 3) << 17 | 8u << 24;
      const uint32_t idesc_o = (1u << 4) | 1u << 16 | (uint32_t)(DIM >> 3) << 17 | 8u << 24;
      const uint32_t at_s = kS + 128u * half, at_o = kO + (uint32_t)(DIM * half);
      auto scores = [&](int t) {
        const int stage = t % kPromptStages;
        ok = prompt_wait(k_full + 8 * stage, (uint32_t)(t / kPromptStages) & 1u);
        if (!ok) return;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t kb = k0 + (uint32_t)(stage * (L::tile_bytes >> 4));
#pragma unroll
        for (int x = 0; x < DIM / 16; x++)
          umma_ss(elected, at_s + 64u * (t & 1), q0 + (uint32_t)((x >> 2) * (BLOCK_Q >> 4) + (x & 3) * 2),
                  kb + (uint32_t)((x >> 2) * (BLOCK >> 4) + (x & 3) * 2), desc_hi, idesc_s, x > 0 ? 1u : 0u);
        umma_commit(elected, s_full + 16 * half + 8 * (t & 1));
        umma_commit(elected, k_empty + 8 * stage);
      };
      if (tiles > 0) scores(0);
      for (int t = 0; t < tiles && ok; t++) {
        // the next scores, while the softmax works on these: they take the place of weights that have been multiplied
        if (t + 1 < tiles) {
          if (t > 0) ok = prompt_wait(o_done + 8 * half, (t - 1) & 1);
          if (ok) scores(t + 1);
          if (!ok) break;
        }
        const int stage = t % kPromptStages;
        ok = prompt_wait(v_full + 8 * stage, (uint32_t)(t / kPromptStages) & 1u) &&
             prompt_wait(p_full + 16 * half + 8 * (t & 1), (uint32_t)(t >> 1) & 1u);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t vb = v0 + (uint32_t)(stage * (L::tile_bytes >> 4));
#pragma unroll
        for (int x = 0; x < kPromptKeys / 16; x++)
          umma_ts(elected, at_o, at_s + 64u * (t & 1) + 8u * x, vb + 128u * x, desc_hi, idesc_o, t > 0 || x > 0 ? 1u : 0u);
        umma_commit(elected, o_done + 8 * half);
        umma_commit(elected, v_empty + 8 * stage);
      }
      // nothing of this warp is at work any more when tensor and shared memory are given back (waited for with the full limit whatever p.polls is)
      umma_commit(elected, drained + 8 * half);
      __syncwarp();
      mbar_wait_warp(drained + 8 * half, 0, kPromptPolls);
    }
  }
  if (!ok && lane == 0) atomicExch(p.status, warp < 8 ? 3 : warp < 12 ? 4 : 5);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 15) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(0), "r"(512) : "memory");
  }
}

}  // namespace rcp
