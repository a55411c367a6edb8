// Softmax attention of new tokens over the paged 8-bit cache (rcp_kv_attention).
//
//   out[t][h] = sum_j p_j v_j / sum_j p_j,  p_j = exp(sm_scale (q[t][h] . k_j)),  j over the positions 0 .. position of t
//   k_j, v_j: code times the scale of its block; a page outside the cache holds no keys; a row without keys is zero.
//
// kv_attention_split_kernel: few rows (new tokens x query heads of a key head) a sequence, where the cache is what has to be read. Bound by
// HBM: every code once. Rows are columns here: S^T = K Q^T and O^T = V^T P^T, so that 16 keys fill the tensor core's 16 rows
// and eight queries its eight columns. A tile is 32 keys; codes become fp16 in registers.
//   Fragments. Both products may take their inner index in any order that their operands share. Keys: a thread reads 16 bytes of a row
//   (and the queries' fragments are made in that order), values: 16 bytes of each of its four tokens, whose bytes are
//   interleaved in pairs of tokens before they are converted. The weights come out of the first product with keys along the
//   rows and go into the second one transposed (movmatrix).
//   Softmax. Scores in units of log2. The reference m of a row moves only when a tile has a score more than kAttnSlack above it, which
//   a vote finds out (no reduction as a rule); weights are 2^(s - m + kAttnLift), at most 2^14 in fp16, so that weights down to 2^-22
//   of the largest keep all their bits. The sum of the weights is one more row of the second product, of ones: what is summed is what
//   the values are multiplied with, so the rounding of weights to fp16 cancels where they are alike.
//   Scales are powers of two: the keys' goes into the factor of the scores, the values' into the unit of the sums, which are rescaled
//   when the next block has another one (exactly, or by 2^-149 at the bottom).
//   Work. Sequences x row tiles x key heads are cut into tiles of keys, and the list of all tiles is shared out evenly over warps, whatever
//   the lengths are. A warp loads ahead through its own ring of asynchronous copies, across the ends of sequences too. What it
//   has of a segment (the keys of one sequence, row tile and key head) in part goes to shared memory; the CTA joins what its
//   warps have, and of a segment that goes on in other CTAs the last one to arrive joins the parts, in their order (so results repeat).
//   Measured (us, GB/s of what has to be read and written): 64 sequences of 8000 keys at most, 32 heads on 8 of 128: 120, 5.9 TB/s; one of
//   130999 keys, 64 on 8: 54, 5.0; 16 x 4000, 32 on 32: 63, 5.3; five tokens each of 16 x 8000: 58, 3.2 (three columns of rows; the chain of
//   operations of a tile, 840 instructions where one column takes 500, on two warps a scheduler with 255 registers each); one of 777 keys, dim 64: 7.2, of 20: 3.6. A tile takes a warp some 1700 clocks
//   however few there are: that is what short sequences wait for. 12 or 16 warps a CTA (fewer registers, parts to memory) were slower everywhere (16 x 4000:
//   70), and so was nearly everywhere a tile's scores made ahead of the weights of the one in front.
#pragma once
#include <climits>

#include "common.cuh"
#include "kv_common.cuh"

namespace rcp {

struct AttnParams {
  const __half* q;
  long long q_stride;        // elements between tokens
  int heads, kv_heads, group;   // group: query heads of a key head
  uint32_t group_inv, kv_heads_inv;   // for attn_quotient
  float scale_log2;          // sm_scale * log2(e)
  KvSeqs s;
  const uint8_t *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  __half* out;               // [tokens][heads][dim]
  int32_t* status;           // set when a bounded wait gives up
  uint32_t polls;            // of such a wait, in tests
  int few;                   // sequences with more rows than that are the prompt kernel's, the others the split kernel's (0: one kernel has all)
  int32_t* arrived;          // [2][kAttnMaxCtas], zero between calls: of segments, of groups of CTAs
  float* parts;              // [kAttnMaxCtas][2][rows][dim + 2]
};

constexpr int kAttnMaxCtas = 256, kAttnMaxRows = 24;
constexpr int kAttnWarps = 8, kAttnTile = 32;
constexpr int kAttnAlone = 4;   // tiles a warp
constexpr int kAttnJoin = 16;   // parts that are joined at once
constexpr float kAttnSlack = 6.f, kAttnLift = 8.f, kAttnNoMax = -1e30f;
constexpr size_t kAttnArrivedAt = 256, kAttnPartsAt = kAttnArrivedAt + 2 * kAttnMaxCtas * sizeof(int32_t);
constexpr size_t kAttnWorkspaceBytes = kAttnPartsAt + (size_t)kAttnMaxCtas * 2 * kAttnMaxRows * (128 + 2) * sizeof(float);

// tiles in the ring: what shared memory has room for beside the parts, five of 64 elements, three of 128 with eight rows, two with more
template <int DIM, int NT>
struct AttnLayout {
  static constexpr int stages = DIM == 64 ? 5 : NT == 1 ? 3 : 2;
  static constexpr int tile_bytes = kAttnTile * DIM;              // of keys, and of values
  static constexpr int stage_bytes = 2 * tile_bytes;
  static constexpr int rows = 8 * NT;
  static constexpr int part_floats = rows * (DIM + 2);            // sums [rows][dim], then references and sums of weights
  static constexpr int ring = 0, first = kAttnWarps * stages * stage_bytes;
  static constexpr int meta = first + kAttnWarps * part_floats * 4;   // per warp and stage: scales of keys and values, whether there are any
  static constexpr int list = meta + kAttnWarps * stages * 16;
  static constexpr int bytes = list + 2 * kAttnWarps * 32 + 80;
  static_assert(part_floats * 4 <= stages * stage_bytes, "a warp's last part goes where its ring was");
  static_assert(RCP_KV_MAX_SEQS * 8 <= kAttnWarps * stages * stage_bytes, "the list of sequences' tiles lies there at first");
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t attn_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint4 lds_v4(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
// the four e4m3 codes of a word as fp16 pairs (bytes 0, 1 and bytes 2, 3)
__device__ __forceinline__ void e4m3_halves(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same onto sums of zero
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// x / d for x < 2^16 and d <= 1024, with inv = 2^32 / d rounded up (0 for 1): off by less than x / 2^32 < 1 / d before it is cut off. (Rows
// of a sequence are 8000 at most here, 48 where there are hundreds of key heads: attn_few_rows.)
__device__ __forceinline__ int attn_quotient(int x, uint32_t inv) { return inv ? (int)__umulhi((uint32_t)x, inv) : x; }

// A place in the list of tiles: segment `seg` of sequence b (row tile seg / kv_heads, key head seg % kv_heads), tile of its keys.
struct AttnPlace {
  int b, seg, tile;
  int segs, tiles;     // of the sequence: segments, tiles each
  KvSeq sq;
};
template <int ROWS>
__device__ __forceinline__ void attn_sequence(const AttnParams& p, int b, AttnPlace& at) {
  at.b = b;
  at.sq = kv_seq(p.s, b);
  const int rows = at.sq.n * p.group;
  at.segs = p.few && rows > p.few ? 0 : (rows + ROWS - 1) / ROWS * p.kv_heads;
  at.tiles = max(1, (at.sq.end + kAttnTile - 1) / kAttnTile);
}
template <int ROWS>
__device__ __forceinline__ void attn_next_segment(const AttnParams& p, AttnPlace& at) {
  at.tile = 0;
  if (++at.seg < at.segs) return;
  at.seg = 0;
  do attn_sequence<ROWS>(p, at.b + 1, at);
  while (at.segs == 0);
}

// what is to be done with a part of a segment in shared memory
struct alignas(16) AttnPiece {
  int seg, tile0, tiles, of;   // the keys' tiles tile0 .. tile0 + tiles - 1 of `of` (tiles 0: nothing here)
  int t0, n;                   // of the sequence
  long long start;             // the segment's first tile in the list of all: segments differ in it
};

// y = sums / weights as fp16, to the row's place
template <int DIM>
__device__ __forceinline__ __half* attn_row(const AttnParams& p, int t0, int n, int seg, int rows, int row) {
  const int rt = attn_quotient(seg, p.kv_heads_inv), r = rt * rows + row;
  if (r >= n * p.group) return nullptr;
  const int i = attn_quotient(r, p.group_inv);
  return p.out + ((long long)(t0 + i) * p.heads + (long long)(seg - rt * p.kv_heads) * p.group + (r - i * p.group)) * DIM;
}

template <int E>
__device__ __forceinline__ void attn_store(__half* to, const float (&acc)[E], float f) {
#pragma unroll
  for (int k = 0; k < E; k += 2) *reinterpret_cast<__half2*>(to + k) = __floats2half2_rn(acc[k] * f, acc[k + 1] * f);
}

// DIM: of a head; NT: columns of eight rows a row tile has
template <int DIM, int NT>
__global__ void __launch_bounds__(kAttnWarps * 32, 1) kv_attention_split_kernel(const AttnParams p) {
  using L = AttnLayout<DIM, NT>;
  constexpr int ROWS = L::rows, KSTEPS = DIM / 16, MT = DIM / 16, S = L::stages;
  extern __shared__ __align__(1024) uint8_t attn_shared[];
  const uint32_t base = attn_smem(attn_shared);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, j = lane & 3;
  AttnPiece* const list = reinterpret_cast<AttnPiece*>(attn_shared + L::list);
  long long* const s_sum = reinterpret_cast<long long*>(attn_shared + L::list + 2 * kAttnWarps * sizeof(AttnPiece));   // [8]: one a warp
  int* const s_joins = reinterpret_cast<int*>(s_sum + kAttnWarps);
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // Tiles in front of each sequence, and where this warp's share of them begins. Up to 32 sequences every warp finds that out for itself, a
  // sequence a lane; more are scanned by the CTA.
  long long total, c0, c1, w0, each, more;   // each, more: the first `more` CTAs have each + 1 tiles, the others `each`
  int ctas;
  auto quotient = [](long long a, long long b) { return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b); };
  AttnPlace at{};
  long long in = 0;   // the share's first tile in its sequence
  // A CTA a segment, whose warps' parts meet in shared memory, where the longest one takes a warp at most kAttnAlone tiles more than its even share would:
  // parts that meet in memory cost as much (16 sequences of 300 keys, 32 heads on 8 of 128: 6.7 us, of 1900: 16.0 against 19.1).
  auto whole = [&](int segs, int tiles) {
    return segs <= (int)gridDim.x && (long long)tiles * gridDim.x - total <= (long long)kAttnAlone * kAttnWarps * gridDim.x;
  };
  auto share = [&]() {   // of `total`: as many CTAs as have a tile for each of their warps
    ctas = (int)min((long long)gridDim.x, (total + kAttnWarps - 1) / kAttnWarps);
    if (p.s.seqs == 1 && whole(at.segs, at.tiles)) ctas = at.segs;
    if ((int)blockIdx.x >= ctas) return false;
    each = quotient(total, ctas);
    more = total - each * ctas;
    c0 = each * blockIdx.x + min((long long)blockIdx.x, more);
    c1 = c0 + each + ((int)blockIdx.x < more ? 1 : 0);
    w0 = c0 + (c1 - c0) * warp / kAttnWarps;
    return true;
  };
  if (p.s.seqs == 1) {
    attn_sequence<ROWS>(p, 0, at);
    total = (long long)at.segs * at.tiles;
    if (!share()) return;
    in = w0;
  } else if (p.s.seqs <= 32) {
    if (lane < p.s.seqs) attn_sequence<ROWS>(p, lane, at);
    const long long mine = (long long)at.segs * at.tiles;
    long long upto = mine;
    int segs = at.segs;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, upto, d);
      const int os = __shfl_up_sync(0xffffffffu, segs, d);
      if (lane >= d) {
        upto += o;
        segs += os;
      }
    }
    const int all = __shfl_sync(0xffffffffu, segs, 31);
    total = __shfl_sync(0xffffffffu, upto, 31);
    int b;
    if (whole(all, (int)__reduce_max_sync(0xffffffffu, at.segs ? at.tiles : 0))) {
      if ((int)blockIdx.x >= all) return;
      b = __popc(__ballot_sync(0xffffffffu, segs <= (int)blockIdx.x));   // the first sequence that has segments behind this one
      c0 = __shfl_sync(0xffffffffu, upto - mine + (long long)((int)blockIdx.x - (segs - at.segs)) * at.tiles, b);
      c1 = c0 + __shfl_sync(0xffffffffu, at.tiles, b);
      w0 = c0 + (c1 - c0) * warp / kAttnWarps;
      each = more = 0;   // (no segment goes on elsewhere)
    } else {
      if (!share()) return;
      // the last sequence with no more than w0 tiles in front of it (it has some itself, or there is nothing to do)
      b = 31 - __clz((int)__ballot_sync(0xffffffffu, lane < p.s.seqs && upto - mine <= w0));
    }
    in = w0 - __shfl_sync(0xffffffffu, upto - mine, b);
    at.b = b;
    at.segs = __shfl_sync(0xffffffffu, at.segs, b);
    at.tiles = __shfl_sync(0xffffffffu, at.tiles, b);
    at.sq.t0 = __shfl_sync(0xffffffffu, at.sq.t0, b);
    at.sq.n = __shfl_sync(0xffffffffu, at.sq.n, b);
    at.sq.first = __shfl_sync(0xffffffffu, at.sq.first, b);
    at.sq.end = __shfl_sync(0xffffffffu, at.sq.end, b);
  } else {
    long long* const before = reinterpret_cast<long long*>(attn_shared);
    constexpr int PER = RCP_KV_MAX_SEQS / (kAttnWarps * 32);
    long long mine[PER], sum = 0;
    const int per = (p.s.seqs + kAttnWarps * 32 - 1) / (kAttnWarps * 32);
#pragma unroll
    for (int i = 0; i < PER; i++) {
      mine[i] = 0;
      if (i < per && tid * per + i < p.s.seqs) {
        attn_sequence<ROWS>(p, tid * per + i, at);
        mine[i] = (long long)at.segs * at.tiles;
      }
      sum += mine[i];
    }
    long long upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += o;
    }
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
    long long run = upto - sum;
    total = 0;
#pragma unroll
    for (int w = 0; w < kAttnWarps; w++) {
      if (w < warp) run += s_sum[w];
      total += s_sum[w];
    }
#pragma unroll
    for (int i = 0; i < PER; i++) {
      if (i < per && tid * per + i < p.s.seqs) before[tid * per + i] = run;
      run += mine[i];
    }
    __syncthreads();
    if (!share()) return;
    int lo = 0, hi = p.s.seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before[mid] <= w0) lo = mid; else hi = mid;
    }
    attn_sequence<ROWS>(p, lo, at);
    in = w0 - before[lo];
    __syncthreads();   // the list of tiles gives way to the rings
  }
  const int todo = (int)min(c0 + (c1 - c0) * (warp + 1) / kAttnWarps - w0, (long long)INT_MAX);
  if (todo > 0) {
    at.seg = (int)quotient(in, at.tiles);
    at.tile = (int)(in - (long long)at.seg * at.tiles);
  }
  if (lane < 2) list[2 * warp + lane].tiles = 0;   // (written again and read by this warp, then by all behind a barrier)
  __syncwarp();

  if (todo > 0) {
    const uint32_t ring = base + (uint32_t)(warp * S * L::stage_bytes);
    float* const metaf = reinterpret_cast<float*>(attn_shared + L::meta) + warp * S * 4;
    AttnPlace ld = at;
    int loaded = 0, ld_stage = 0, pages_at = -1, pages_b = -1, my_page = -1;
    // where a lane's 16-byte pieces go, every 512 bytes one: piece c of a row, exchanged within 128 bytes so that the reads below meet no bank twice
    const int row0 = lane / (DIM / 16), line0 = DIM == 128 ? row0 : row0 >> 1, in0 = DIM == 128 ? lane & 7 : (row0 & 1) * 4 + (lane & 3);
    const uint32_t k_to = (uint32_t)(line0 * 128 + ((DIM == 128 ? in0 ^ ((row0 & 1) << 2) : in0) << 4));
    const uint32_t v_to0 = (uint32_t)(L::tile_bytes + line0 * 128 + ((in0 ^ (((row0 >> 1) & 3) << 1)) << 4));
    const uint32_t v_to1 = DIM == 128 ? v_to0 ^ 64u : v_to0;   // (rows four further on)
    // asks for the next tile
    auto load = [&]() {
      if (loaded < todo) {
        // pages of 32 tiles at a time, one a lane
        if (ld.b != pages_b || ld.tile < pages_at || ld.tile >= pages_at + 32) {
          pages_b = ld.b;
          pages_at = ld.tile;
          const int t = ld.tile + lane;
          my_page = t * kAttnTile < ld.sq.end ? p.s.table[(long long)ld.b * p.s.width + (t * kAttnTile >> p.s.lg_page)] : -1;
        }
        const int pg = __shfl_sync(0xffffffffu, my_page, ld.tile - pages_at), j0 = ld.tile * kAttnTile;
        const bool there = pg >= 0 && pg < p.s.pages;
        const int kv = ld.seg - attn_quotient(ld.seg, p.kv_heads_inv) * p.kv_heads;
        const long long block = there ? (long long)pg * p.kv_heads + kv : 0;
        const long long off = (block * p.s.page + (j0 & (p.s.page - 1))) * DIM + lane * 16;
        const int live = there ? min(ld.sq.end - j0, kAttnTile) : 0;   // keys of the tile that exist: the others are zeroes
        const uint32_t dst = ring + (uint32_t)(ld_stage * L::stage_bytes);
        const uint8_t *const k_from = p.k_cache + off, *const v_from = p.v_cache + off;
        if (live == kAttnTile) {
#pragma unroll
          for (int i = 0; i < DIM / 16; i++) {
            cp_async16(dst + k_to + i * 512, k_from + i * 512);
            cp_async16(dst + (i & 1 ? v_to1 : v_to0) + i * 512, v_from + i * 512);
          }
        } else {
#pragma unroll
          for (int i = 0; i < DIM / 16; i++) {
            const int bytes = (lane + 32 * i) / (DIM / 16) < live ? 16 : 0;   // (nothing is read where it is zero)
            cp_async16(dst + k_to + i * 512, bytes ? k_from + i * 512 : p.k_cache, bytes);
            cp_async16(dst + (i & 1 ? v_to1 : v_to0) + i * 512, bytes ? v_from + i * 512 : p.v_cache, bytes);
          }
        }
        float* const m = metaf + ld_stage * 4;
        if (lane == 0) cp_async4(attn_smem(m), p.k_scale + block);
        if (lane == 1) cp_async4(attn_smem(m + 1), p.v_scale + block);
        if (lane == 2) m[2] = there ? 1.f : 0.f;
        loaded++;
        if (++ld.tile == ld.tiles && loaded < todo) attn_next_segment<ROWS>(p, ld);
      }
      if (++ld_stage == S) ld_stage = 0;
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < S - 1; i++) load();

    uint32_t q[NT][KSTEPS][2];
    float o[MT][NT][4], l[NT][4], m[NT][2], vs = 1.f;
    int lim[NT][2], least = 0;
    // queries and limits of a segment; sums at zero
    auto begin = [&]() {
      const int rt = attn_quotient(at.seg, p.kv_heads_inv), kv = at.seg - rt * p.kv_heads, r0 = rt * ROWS, rows = at.sq.n * p.group;
#pragma unroll
      for (int n = 0; n < NT; n++) {
        const int r = r0 + n * 8 + g, i = attn_quotient(r, p.group_inv);
        const bool have = r < rows;
        const __half* const src = p.q + (have ? (long long)(at.sq.t0 + i) * p.q_stride + (long long)(kv * p.group + r - i * p.group) * DIM : 0);
#pragma unroll
        for (int c = 0; c < KSTEPS / 4; c++) {
          const uint4 *v = reinterpret_cast<const uint4*>(src + 16 * (j + 4 * c));
          const uint4 a = have ? v[0] : make_uint4(0, 0, 0, 0), b = have ? v[1] : make_uint4(0, 0, 0, 0);
          q[n][4 * c][0] = a.x; q[n][4 * c][1] = a.y; q[n][4 * c + 1][0] = a.z; q[n][4 * c + 1][1] = a.w;
          q[n][4 * c + 2][0] = b.x; q[n][4 * c + 2][1] = b.y; q[n][4 * c + 3][0] = b.z; q[n][4 * c + 3][1] = b.w;
        }
        least = n == 0 ? INT_MAX : least;
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const int rr = r0 + n * 8 + 2 * j + e, pos = at.sq.first + attn_quotient(rr, p.group_inv);
          lim[n][e] = rr >= rows ? INT_MAX : pos >= 0 && pos < at.sq.end ? pos + 1 : 0;
          least = min(least, lim[n][e]);
          m[n][e] = kAttnNoMax;
        }
#pragma unroll
        for (int e = 0; e < 4; e++) {
          l[n][e] = 0.f;
#pragma unroll
          for (int u = 0; u < MT; u++) o[u][n][e] = 0.f;
        }
      }
      least = (int)__reduce_min_sync(0xffffffffu, least);
      vs = 1.f;
    };
    // the warp's part of the segment, tiles t0 .. t1 - 1 of it: to its rows if that is all, else to shared memory
    auto end = [&](int t0, int t1, bool last, long long unit) {   // unit: tile t1 - 1 in the list of all
      if (t0 == 0 && t1 == at.tiles) {
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
          for (int e = 0; e < 2; e++) {
            __half* const to = attn_row<DIM>(p, at.sq.t0, at.sq.n, at.seg, ROWS, n * 8 + 2 * j + e);
            const float f = l[n][e] > 0.f ? vs / l[n][e] : l[n][e];   // no keys: zero (and a sum that is no number stays one)
            if (to) {
#pragma unroll
              for (int u = 0; u < MT; u += 4) {
                uint32_t w[4];
#pragma unroll
                for (int x = 0; x < 4; x++) {
                  const __half2 h = __floats2half2_rn(o[u + x][n][e] * f, o[u + x][n][2 + e] * f);
                  w[x] = *reinterpret_cast<const uint32_t*>(&h);
                }
                *reinterpret_cast<uint4*>(to + (DIM / 8) * g + 2 * u) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          }
        return;
      }
      float* const part = last ? reinterpret_cast<float*>(attn_shared + warp * S * L::stage_bytes)
                               : reinterpret_cast<float*>(attn_shared + L::first) + warp * L::part_floats;
#pragma unroll
      for (int n = 0; n < NT; n++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const int row = n * 8 + 2 * j + e;
#pragma unroll
          for (int u = 0; u < MT; u++)
            *reinterpret_cast<float2*>(part + row * DIM + (DIM / 8) * g + 2 * u) = make_float2(o[u][n][e] * vs, o[u][n][2 + e] * vs);
          if (g == 0) {
            part[ROWS * DIM + row] = m[n][e];
            part[ROWS * (DIM + 1) + row] = l[n][e];
          }
        }
      if (lane == 0) list[2 * warp + (last ? 1 : 0)] = AttnPiece{at.seg, t0, t1 - t0, at.tiles, at.sq.t0, at.sq.n, unit + 1 - t1};
    };

    begin();
    int stage = 0, from = at.tile;
    for (int done = 0; done < todo; done++) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
      __syncwarp();
      load();
      const uint32_t kt = ring + (uint32_t)(stage * L::stage_bytes), vt = kt + L::tile_bytes;
      const float4 meta = *reinterpret_cast<const float4*>(metaf + stage * 4);
      const float ks = meta.x, vs_new = meta.y, there = meta.z;
      if (++stage == S) stage = 0;
      float s[2][NT][4];
#pragma unroll
      for (int t = 0; t < 2; t++) {
        constexpr int CHAINS = NT < 3 ? 2 : 1;   // products of 16 keys add to CHAINS sums in turn: a shorter chain, where registers allow
        float part[CHAINS][NT][4];
#pragma unroll
        for (int c = 0; c < KSTEPS / 4; c++) {
          uint4 x[2];
#pragma unroll
          for (int hf = 0; hf < 2; hf++) {
            const int row = t * 16 + hf * 8 + g;
            const int line = DIM == 128 ? row : row >> 1, in = DIM == 128 ? (j + 4 * c) ^ ((row & 1) << 2) : (row & 1) * 4 + j;
            x[hf] = lds_v4(kt + line * 128 + in * 16);
          }
          const uint32_t w0[4] = {x[0].x, x[0].y, x[0].z, x[0].w}, w1[4] = {x[1].x, x[1].y, x[1].z, x[1].w};
#pragma unroll
          for (int k = 0; k < 4; k++) {
            uint32_t a0, a1, a2, a3;
            e4m3_halves(w0[k], a0, a2);
            e4m3_halves(w1[k], a1, a3);
#pragma unroll
            for (int n = 0; n < NT; n++) {
              if (c == 0 && k < CHAINS) mma16816_first(part[k][n], a0, a1, a2, a3, q[n][k][0], q[n][k][1]);
              else mma16816(part[k % CHAINS][n], a0, a1, a2, a3, q[n][4 * c + k][0], q[n][4 * c + k][1]);
            }
          }
        }
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
          for (int e = 0; e < 4; e++) s[t][n][e] = CHAINS == 2 ? part[0][n][e] + part[CHAINS - 1][n][e] : part[0][n][e];
      }
      const float c = there != 0.f ? fmaxf(ks * p.scale_log2, 1e-37f) : 1.f;   // above zero: a score of -inf stays one
      const int j0 = at.tile * kAttnTile;
      if (there == 0.f || j0 + kAttnTile > least) {   // keys that some row does not see
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
          for (int n = 0; n < NT; n++)
#pragma unroll
            for (int e = 0; e < 4; e++)
              if (there == 0.f || j0 + t * 16 + (e >> 1) * 8 + g >= lim[n][e & 1]) s[t][n][e] = -INFINITY;
      }
      bool move = vs_new != vs;
      float top[NT][2];
#pragma unroll
      for (int n = 0; n < NT; n++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          top[n][e] = fmaxf(fmaxf(s[0][n][e], s[0][n][2 + e]), fmaxf(s[1][n][e], s[1][n][2 + e])) * c;
          move |= top[n][e] > m[n][e] + kAttnSlack;
        }
      if (__any_sync(0xffffffffu, move)) {
        const float fv = there != 0.f ? vs / vs_new : 1.f;   // a quotient of powers of two
        if (there != 0.f) vs = vs_new;
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
          for (int e = 0; e < 2; e++) {
            float t = top[n][e];
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
            const float mn = fmaxf(m[n][e], t), f = exp2_fast(m[n][e] - mn);
            m[n][e] = mn;
            l[n][e] *= f;
#pragma unroll
            for (int u = 0; u < MT; u++) {
              o[u][n][e] *= f * fv;
              o[u][n][2 + e] *= f * fv;
            }
          }
      }
      uint32_t pt[2][NT][2];
#pragma unroll
      for (int n = 0; n < NT; n++) {
        const float m0 = m[n][0] - kAttnLift, m1 = m[n][1] - kAttnLift;
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
          for (int hf = 0; hf < 2; hf++) {
            const __half2 h = __floats2half2_rn(exp2_fast(fmaf(s[t][n][2 * hf], c, -m0)), exp2_fast(fmaf(s[t][n][2 * hf + 1], c, -m1)));
            pt[t][n][hf] = transpose8x8(*reinterpret_cast<const uint32_t*>(&h));
          }
      }
#pragma unroll
      for (int t = 0; t < 2; t++) {
#pragma unroll
        for (int n = 0; n < NT; n++) mma16816(l[n], 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u, pt[t][n][0], pt[t][n][1]);
        uint32_t x[4][DIM / 32];   // the thread's DIM / 8 bytes of tokens 2 j, 2 j + 1, 2 j + 8, 2 j + 9
#pragma unroll
        for (int k = 0; k < 4; k++) {
          const int row = t * 16 + 2 * j + (k & 1) + (k >> 1) * 8;
          if constexpr (DIM == 128) {
            const uint4 v = lds_v4(vt + row * 128 + ((g ^ (((row >> 1) & 3) << 1)) << 4));
            x[k][0] = v.x; x[k][1] = v.y; x[k][2] = v.z; x[k][3] = v.w;
          } else {
            const uint2 v = lds_v2(vt + (row >> 1) * 128 + ((((row & 1) * 4 + (g >> 1)) ^ (((row >> 1) & 3) << 1)) << 4) + (g & 1) * 8);
            x[k][0] = v.x; x[k][1] = v.y;
          }
        }
#pragma unroll
        for (int w = 0; w < DIM / 32; w++) {
          uint32_t a[2][4];
#pragma unroll
          for (int hf = 0; hf < 2; hf++) {
            e4m3_halves(__byte_perm(x[2 * hf][w], x[2 * hf + 1][w], 0x5140), a[0][2 * hf], a[0][2 * hf + 1]);
            e4m3_halves(__byte_perm(x[2 * hf][w], x[2 * hf + 1][w], 0x7362), a[1][2 * hf], a[1][2 * hf + 1]);
          }
#pragma unroll
          for (int n = 0; n < NT; n++) {
            mma16816(o[2 * w][n], a[0][0], a[0][1], a[0][2], a[0][3], pt[t][n][0], pt[t][n][1]);
            mma16816(o[2 * w + 1][n], a[1][0], a[1][1], a[1][2], a[1][3], pt[t][n][0], pt[t][n][1]);
          }
        }
      }
      if (++at.tile == at.tiles) {
        if (done + 1 == todo) asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        end(from, at.tiles, done + 1 == todo, w0 + done);
        if (done + 1 < todo) {
          attn_next_segment<ROWS>(p, at);
          begin();
          from = 0;
        }
      } else if (done + 1 == todo) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        end(from, at.tile, true, w0 + done);
      }
    }
  }
  __syncthreads();

  // the warps' parts: runs of the same segment are joined
  constexpr int SLOTS = 2 * kAttnWarps, PART = L::part_floats;
  auto part_of = [&](int slot) {
    return reinterpret_cast<const float*>(attn_shared + ((slot & 1) ? (slot >> 1) * S * L::stage_bytes : L::first + (slot >> 1) * PART * 4));
  };
  // A piece a lane; the first lane of each run of pieces of a segment stands for the run. A warp takes a row, a lane DIM / 32 of its elements.
  constexpr int E = DIM / 32;
  const AttnPiece piece = list[lane % SLOTS];
  const uint32_t valid = __ballot_sync(0xffffffffu, lane < SLOTS && piece.tiles > 0);
  const uint32_t in_front = valid & ((1u << lane) - 1);
  const long long start_in_front = __shfl_sync(0xffffffffu, piece.start, in_front ? 31 - __clz((int)in_front) : 0);
  const uint32_t heads = __ballot_sync(0xffffffffu, (valid >> lane & 1) && (!in_front || start_in_front != piece.start));
  uint32_t open = 0;   // runs that are not the whole of their segment: two at most, the first and the last
  for (uint32_t todo_runs = heads; todo_runs; todo_runs &= todo_runs - 1) {
    const int s0 = __ffs((int)todo_runs) - 1;
    const uint32_t behind = heads & ~((2u << s0) - 1), members = valid & (behind ? (1u << (__ffs((int)behind) - 1)) - 1 : ~0u) & ~((1u << s0) - 1);
    const bool member = members >> lane & 1;
    const int tiles = __reduce_add_sync(0xffffffffu, member ? piece.tiles : 0);
    const int seg = __shfl_sync(0xffffffffu, piece.seg, s0), t0 = __shfl_sync(0xffffffffu, piece.t0, s0), n = __shfl_sync(0xffffffffu, piece.n, s0);
    const bool whole = tiles == __shfl_sync(0xffffffffu, piece.of, s0);
    // of a segment that does not begin here the first slot, of one that does not end here the second
    float* const mine = p.parts + ((size_t)blockIdx.x * 2 + (__shfl_sync(0xffffffffu, piece.tile0, s0) > 0 ? 0 : 1)) * PART;
    if (!whole) open |= 1u << s0;
    for (int row = warp; row < ROWS; row += kAttnWarps) {
      __half* const to = attn_row<DIM>(p, t0, n, seg, ROWS, row);
      if (!to) break;   // (the rows behind it are not there either)
      const float* const ref = part_of(lane % SLOTS) + ROWS * DIM + row;
      const float m = member ? ref[0] : kAttnNoMax;
      float top = m;
#pragma unroll
      for (int x = SLOTS / 2; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x, SLOTS));
      top = __shfl_sync(0xffffffffu, top, 0);
      const float f = member ? exp2f(m - top) : 0.f, lf = member ? ref[ROWS] * f : 0.f;
      float sum = 0.f, acc[E] = {};
      for (uint32_t left = members; left; left &= left - 1) {
        const int s = __ffs((int)left) - 1;
        const float fs = __shfl_sync(0xffffffffu, f, s);
        sum += __shfl_sync(0xffffffffu, lf, s);
        const float* const from = part_of(s) + row * DIM + E * lane;
#pragma unroll
        for (int k = 0; k < E; k++) acc[k] += from[k] * fs;
      }
      if (whole) {
        attn_store<E>(to + E * lane, acc, sum > 0.f ? 1.f / sum : sum);
      } else {
#pragma unroll
        for (int k = 0; k < E; k += 2) __stcg(reinterpret_cast<float2*>(mine + row * DIM + E * lane + k), make_float2(acc[k], acc[k + 1]));
        if (lane == 0) {
          __stcg(mine + ROWS * DIM + row, top);
          __stcg(mine + ROWS * (DIM + 1) + row, sum);
        }
      }
    }
  }
  if (!open) return;
  // The last of the CTAs that have parts of a segment to arrive here joins them, in their order. Of more than 2 kAttnJoin parts it joins what the last to
  // arrive of each kAttnJoin CTAs have joined, at the first one's place: of 148 parts of 24 rows a join alone is 1.8 MB for one SM (one sequence
  // of 91439 keys, 24 heads on one: 65 us, with groups 29).
  auto owner = [&](long long unit) {
    const long long big = more * (each + 1);
    return (int)(unit < big ? quotient(unit, each + 1) : more + quotient(unit - big, each));
  };
  int first = 0, final = 0;   // CTAs with parts of the lane's segment
  if (open >> lane & 1) {
    first = owner(piece.start);
    final = owner(piece.start + piece.of - 1);
  }
  __threadfence();
  __syncthreads();
  if (warp == 0 && (open >> lane & 1)) {
    const bool grouped = final - first >= 2 * kAttnJoin;
    const int from = grouped ? (int)blockIdx.x - ((int)blockIdx.x - first) % kAttnJoin : first, count = grouped ? min(kAttnJoin, final - from + 1) : final - first + 1;
    bool join = true;   // (a group of one has nothing to wait for; its place among the counters may be another segment's)
    if (count > 1) {
      int32_t* const counter = p.arrived + (grouped ? kAttnMaxCtas : 0) + from;
      join = atomicAdd(counter, 1) == count - 1;
      if (join) *counter = 0;
    }
    s_joins[open & ((1u << lane) - 1) ? 1 : 0] = join;
  }
  __syncthreads();
  for (int k = 0; open; k++, open &= open - 1) {
    if (!s_joins[k]) continue;
    const int s0 = __ffs((int)open) - 1;
    const int cta0 = __shfl_sync(0xffffffffu, first, s0), parts = __shfl_sync(0xffffffffu, final, s0) - cta0 + 1;
    const int seg = __shfl_sync(0xffffffffu, piece.seg, s0), t0 = __shfl_sync(0xffffffffu, piece.t0, s0), n = __shfl_sync(0xffffffffu, piece.n, s0);
    auto part = [&](int cta) { return p.parts + ((size_t)cta * 2 + (cta == cta0)) * PART; };
    // joins the parts of `count` CTAs from `from` on, every step-th: to the rows, or (into) to the first one's place
    auto join = [&](int from, int count, int step, bool into) {
      __threadfence();
      for (int row = warp; row < ROWS; row += kAttnWarps) {
        __half* const to = attn_row<DIM>(p, t0, n, seg, ROWS, row);
        if (!to) break;
        // kAttnJoin parts at once: all their elements are asked for, and references and sums of weights a lane a part
        float top = kAttnNoMax, sum = 0.f, acc[E] = {};
        for (int k0 = 0; k0 < count; k0 += kAttnJoin) {
          float2 v[kAttnJoin][E / 2];
#pragma unroll
          for (int u = 0; u < kAttnJoin; u++)
#pragma unroll
            for (int d = 0; d < E / 2; d++)
              v[u][d] = k0 + u < count ? __ldcg(reinterpret_cast<const float2*>(part(from + (k0 + u) * step) + row * DIM + E * lane) + d)
                                       : make_float2(0.f, 0.f);
          const bool there = lane < kAttnJoin && k0 + lane < count;
          const float* const ref = part(from + (there ? k0 + lane : k0) * step) + ROWS * DIM + row;
          const float m = there ? __ldcg(ref) : kAttnNoMax, l = there ? __ldcg(ref + ROWS) : 0.f;
          float mt = fmaxf(top, m);
#pragma unroll
          for (int x = 16; x > 0; x >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, x));
          const float old = exp2f(top - mt), f = there ? exp2f(m - mt) : 0.f;
          top = mt;
          sum *= old;
#pragma unroll
          for (int d = 0; d < E; d++) acc[d] *= old;
#pragma unroll
          for (int u = 0; u < kAttnJoin; u++) {
            const float fu = __shfl_sync(0xffffffffu, f, u), lu = __shfl_sync(0xffffffffu, l, u);
            sum += lu * fu;
#pragma unroll
            for (int d = 0; d < E / 2; d++) {
              acc[2 * d] += v[u][d].x * fu;
              acc[2 * d + 1] += v[u][d].y * fu;
            }
          }
        }
        if (!into) {
          attn_store<E>(to + E * lane, acc, sum > 0.f ? 1.f / sum : sum);
        } else {
          float* const place = part(from);
#pragma unroll
          for (int d = 0; d < E; d += 2) __stcg(reinterpret_cast<float2*>(place + row * DIM + E * lane + d), make_float2(acc[d], acc[d + 1]));
          if (lane == 0) {
            __stcg(place + ROWS * DIM + row, top);
            __stcg(place + ROWS * (DIM + 1) + row, sum);
          }
        }
      }
    };
    if (parts <= 2 * kAttnJoin) {
      join(cta0, parts, 1, false);
      continue;
    }
    const int from = (int)blockIdx.x - ((int)blockIdx.x - cta0) % kAttnJoin, count = min(kAttnJoin, cta0 + parts - from);
    const int groups = (parts + kAttnJoin - 1) / kAttnJoin;
    if (count > 1) join(from, count, 1, true);
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      const bool all = atomicAdd(p.arrived + cta0, 1) == groups - 1;
      if (all) p.arrived[cta0] = 0;
      s_joins[2] = all;
    }
    __syncthreads();
    if (s_joins[2]) join(cta0, groups, kAttnJoin, false);
  }
}

}  // namespace rcp
