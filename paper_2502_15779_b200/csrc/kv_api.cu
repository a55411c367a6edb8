// C ABI of the operators beside the linear layers: the paged 8-bit cache, the attention over it, low-rank adapters.
#include "../../include/rcp.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <mutex>

#include "api.cuh"
#include "kv_append.cuh"
#include "kv_attention.cuh"
#include "kv_attention_umma.cuh"
#include "lora.cuh"

using namespace rcp::api;

namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// elements between rows of `width`: rows that do not overlap and start on 16 bytes
bool stride_ok(int64_t stride, int64_t width, int rows) {
  return stride % 8 == 0 && stride <= (int64_t(1) << 40) && (stride >= width || (rows == 1 && stride >= 0));
}

// The arguments that rcp_kv_append and rcp_kv_attention share.
int check_cache(int tokens, int heads, int kv_heads, int dim, const int32_t* starts, const int32_t* lengths, const int32_t* table, int seqs,
                int width, int max_new, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, int pages, int page,
                rcp::KvSeqs* s) {
  if (!starts || !lengths || !table || !k_cache || !v_cache || !k_scale || !v_scale) return RCP_ERR_NULL;
  if (tokens < 0 || heads < 1 || kv_heads < 1 || heads % kv_heads || heads > RCP_KV_MAX_HEADS || (dim != 64 && dim != 128)) return RCP_ERR_SHAPE;
  if (seqs < 1 || width < 1 || max_new < 0 || pages < 1 || (page != 32 && page != 64 && page != 128)) return RCP_ERR_SHAPE;
  if (seqs > RCP_KV_MAX_SEQS || tokens > RCP_KV_MAX_TOKENS || (int64_t)width * page > RCP_KV_MAX_LENGTH) return RCP_ERR_LIMIT;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned4(starts) || !aligned4(lengths) || !aligned4(table) || !aligned4(k_scale) ||
      !aligned4(v_scale))
    return RCP_ERR_ALIGN;
  const int lg = page == 32 ? 5 : page == 64 ? 6 : 7;
  *s = rcp::KvSeqs{starts, lengths, table, seqs, width, page, lg, pages, tokens, max_new == 0 ? std::max(tokens, 1) : std::min(max_new, std::max(tokens, 1))};
  return RCP_OK;
}

// launch_overlapped with clusters of `size` CTAs
template <typename... KArgs, typename... Args>
cudaError_t launch_clustered(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, int size, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)size, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);
}

template <int DIM, int NT>
int attn_split(const rcp::AttnParams& p, cudaStream_t st) {
  using L = rcp::AttnLayout<DIM, NT>;
  static_assert(L::bytes <= 232448, "227 KB of shared memory");
  static std::mutex mu;
  static bool done[kMaxDevices] = {};
  RCP_CUDA(set_max_smem(rcp::kv_attention_split_kernel<DIM, NT>, L::bytes, mu, done));
  RCP_CUDA(launch_overlapped(rcp::kv_attention_split_kernel<DIM, NT>, dim3(std::min(sm_count(), rcp::kAttnMaxCtas)), dim3(rcp::kAttnWarps * 32),
                             L::bytes, st, p));
  return RCP_OK;
}

// Rows of a sequence (new tokens x query heads of a key head) up to which the split kernel takes it. Its time goes by sequences x key heads x row
// tiles of 24 x keys, over all SMs; the prompt kernel's by keys, as long as its CTAs (256 rows of a key head) run at once: no split along the keys.
// Where the table has room for long sequences the two meet at some 8000 rows x key heads x sequences: split against prompt kernel, us, 8 key heads of
// 128, 8000 keys: one sequence x 800 rows 132 : 143, two x 256 80 : 145, x 512 162 : 147, four x 256 136 : 149, x 512 247 : 148, eight x 64 71 : 134,
// x 128 140 : 136; 4000 keys: sixteen x 32 69 : 72, x 64 91 : 74, 64 x 32 190 : 226, x 64 257 : 216. Short sequences: as many as the split kernel can give
// a CTA to each row tile and key head (900 keys: one x 256 15.6 : 25.8, four x 64 15.2 : 19.0, x 256, more than that, 35.7 : 28.0; 300 keys: one x 256
// 11.3 : 15.9, four x 64 11.3 : 11.2, x 256 27.6 : 18.4).
int attn_few_rows(int seqs, int kv_heads, int64_t room) {
  const int64_t segments = (int64_t)seqs * kv_heads;
  if (room <= 1024) return rcp::kAttnMaxRows * (seqs <= 32 ? (int)std::max<int64_t>(1, sm_count() / segments) : 1);
  return (int)std::max<int64_t>(2 * rcp::kAttnMaxRows, 8000 / segments);
}

template <int DIM, bool LIMITED>
int attn_prompt_launch(const rcp::AttnParams& p, cudaStream_t st) {
  using L = rcp::PromptLayout<DIM>;
  static_assert(L::bytes <= 232448, "227 KB of shared memory");
  static std::mutex mu;
  static bool done[kMaxDevices] = {};
  RCP_CUDA(set_max_smem(rcp::kv_attention_prompt_kernel<DIM, LIMITED>, L::bytes, mu, done));
  const int64_t ctas = ((int64_t)p.s.tokens * p.group / rcp::kPromptRows + p.s.seqs) * p.kv_heads;
  if (ctas > INT_MAX) return RCP_ERR_LIMIT;
  RCP_CUDA(launch_overlapped(rcp::kv_attention_prompt_kernel<DIM, LIMITED>, dim3((unsigned)ctas), dim3(rcp::kPromptThreads), L::bytes, st, p));
  return RCP_OK;
}

int attn_prompt(const rcp::AttnParams& p, int dim, bool limited, cudaStream_t st) {
  if (limited) return dim == 64 ? attn_prompt_launch<64, true>(p, st) : attn_prompt_launch<128, true>(p, st);
  return dim == 64 ? attn_prompt_launch<64, false>(p, st) : attn_prompt_launch<128, false>(p, st);
}

// The records of the adapters' tiles stand behind what attention keeps zero in front of its parts (its status and counters; the linear calls' status is the first
// word too), so that one workspace may serve all of them in turn.
constexpr size_t kLoraRecordsAt = rcp::kAttnPartsAt;
static_assert(kLoraRecordsAt % 16 == 0, "records are read 16 bytes at a time");

template <int STEPS>
int lora_many(rcp::LoraParams p, int tiles, cudaStream_t st) {
  using L = rcp::UpLayout<STEPS>;
  static std::mutex mu;
  static bool down_done[kMaxDevices] = {}, up_done[2][kMaxDevices] = {};
  RCP_CUDA(set_max_smem(rcp::lora_down_kernel<STEPS>, (int)rcp::lora_down_smem(16 * STEPS), mu, down_done));
  const bool wide = p.N % 8 == 0 && aligned16(p.base) && aligned16(p.y);
  const auto up = wide ? rcp::lora_up_kernel<STEPS, true> : rcp::lora_up_kernel<STEPS, false>;
  RCP_CUDA(set_max_smem(up, L::bytes, mu, up_done[wide]));
  // A tile's adapters one after another, or among several CTAs where there are few (97 tokens of four adapters, 546 x 3008, rank 56: 34 us, 13 so).
  const int down_splits = std::max(1, std::min(8, 2 * sm_count() / (tiles * p.parts)));
  RCP_CUDA(launch_clustered(rcp::lora_down_kernel<STEPS>, dim3(tiles * p.parts, down_splits), dim3(rcp::kLoraThreads), rcp::lora_down_smem(p.rank), p.parts, st, p));
  // Column tiles of a CTA: few waves of CTAs, and short ones, because tiles in which tokens of two requests meet take twice as long (2011 tokens of
  // six requests, 28672 columns, us a call: 3 to 6 tiles a CTA 93 (5 is the choice), 8 94.5, 13 105; one wave of 25 tiles 135 against 106 a step before).
  const int cols = (p.N + rcp::kUpCols - 1) / rcp::kUpCols, at_once = sm_count() * std::min<int>(3, 232448 / (L::bytes + 2048));
  double least = 0;
  for (int n = 1; n <= std::min(cols, 16); n++) {
    const int64_t ctas = (int64_t)((cols + n - 1) / n) * tiles;
    const double cost = (double)((ctas + at_once - 1) / at_once + 1) * (n + 0.7);   // (a CTA's beginning is most of a tile)
    if (n == 1 || cost < least) { least = cost; p.up_tiles = n; }
  }
  const int ctas = (cols + p.up_tiles - 1) / p.up_tiles;
  const int up_splits = (int)std::max<int64_t>(1, std::min<int64_t>(8, at_once / ((int64_t)ctas * tiles)));
  RCP_CUDA(launch_overlapped(up, dim3(ctas, tiles, up_splits), dim3(rcp::kLoraThreads), L::bytes, st, p));
  return RCP_OK;
}

}  // namespace

extern "C" {

int rcp_kv_append(const void* q_f16, int64_t q_stride, const void* k_f16, int64_t k_stride, const void* v_f16, int64_t v_stride, int tokens,
                  int heads, int kv_heads, int dim, const float* rope, int rope_positions, int rot, int interleaved, const int32_t* starts,
                  const int32_t* lengths, const int32_t* table, int seqs, int width, int max_new, void* k_cache, void* v_cache, float* k_scale,
                  float* v_scale, int pages, int page, void* q_out_f16, void* stream) {
  if (!k_f16 || !v_f16 || (q_f16 && (!q_out_f16 || !rope))) return RCP_ERR_NULL;
  rcp::AppendParams p{};
  const int rc = check_cache(tokens, q_f16 ? heads : kv_heads, kv_heads, dim, starts, lengths, table, seqs, width, max_new, k_cache, v_cache, k_scale,
                             v_scale, pages, page, &p.s);
  if (rc != RCP_OK) return rc;
  const int64_t kv_width = (int64_t)kv_heads * dim;
  if (!stride_ok(k_stride, kv_width, tokens) || !stride_ok(v_stride, kv_width, tokens) ||
      (q_f16 && !stride_ok(q_stride, (int64_t)heads * dim, tokens)))
    return RCP_ERR_SHAPE;
  // every position that the table has room for has a row of cosines
  if (rope && (rot < 16 || rot > dim || rot % 16 || rope_positions < width * page)) return RCP_ERR_SHAPE;
  if (!aligned16(k_f16) || !aligned16(v_f16) || !aligned16(q_f16) || !aligned16(q_out_f16) || !aligned16(rope)) return RCP_ERR_ALIGN;
  if (tokens == 0) return RCP_OK;
  p.q = static_cast<const __half*>(q_f16);
  p.k = static_cast<const __half*>(k_f16);
  p.v = static_cast<const __half*>(v_f16);
  p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
  p.rope = reinterpret_cast<const float2*>(rope);
  p.rot = rope ? rot : 0;
  p.interleaved = interleaved != 0;
  p.heads = heads; p.kv_heads = kv_heads; p.dim = dim;
  p.k_cache = static_cast<uint8_t*>(k_cache);
  p.v_cache = static_cast<uint8_t*>(v_cache);
  p.k_scale = k_scale; p.v_scale = v_scale;
  p.q_out = static_cast<__half*>(q_out_f16);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool one = p.s.max_new == 1;
  const int threads = !one && page * dim > 4096 ? 256 : rcp::kAppendThreads, query_tokens = threads / (dim / 16);
  int64_t ctas;
  if (one) {
    const int per_warp = 512 / dim;
    ctas = p.candidates = (int)(((int64_t)seqs * ((2 * kv_heads + per_warp - 1) / per_warp) + 3) / 4);
  } else {
    // candidates for blocks with new tokens: so many to each sequence, or by search over starts
    const int64_t per = (p.s.max_new + page - 2) / page + 1, direct = per * seqs, found = tokens / page + 2 * (int64_t)seqs;
    p.direct = direct <= found ? (int)per : 0;
    p.candidates = (int)std::min(direct, found);
    ctas = (int64_t)p.candidates * kv_heads * 2;
  }
  if (q_f16) {
    // eight heads a thread, fewer where there would be too few CTAs to share the latency
    const int64_t groups = (tokens + query_tokens - 1) / query_tokens;
    int each = 8;
    while (each > 1 && groups * ((heads + each - 1) / each) < 2 * sm_count()) each /= 2;
    p.query_splits = (heads + each - 1) / each;
    ctas += groups * p.query_splits;
  }
  if (ctas > INT_MAX) return RCP_ERR_LIMIT;
  const dim3 grid((unsigned)ctas), block(threads);
  if (one) RCP_CUDA(launch_overlapped(rcp::kv_append_one_kernel, grid, block, 0, st, p));
  else if (page * dim == 16384) RCP_CUDA(launch_overlapped(rcp::kv_append_kernel<4, 256>, grid, block, 0, st, p));
  else if (page * dim == 8192) RCP_CUDA(launch_overlapped(rcp::kv_append_kernel<2, 256>, grid, block, 0, st, p));
  else if (page * dim == 4096) RCP_CUDA(launch_overlapped(rcp::kv_append_kernel<2, 128>, grid, block, 0, st, p));
  else RCP_CUDA(launch_overlapped(rcp::kv_append_kernel<1, 128>, grid, block, 0, st, p));
  return RCP_OK;
}

size_t rcp_kv_attention_workspace_bytes(void) { return rcp::kAttnWorkspaceBytes; }

int rcp_kv_attention_variant(int variant, int polls, const void* q_f16, int64_t q_stride, int tokens, int heads, int kv_heads, int dim, float sm_scale,
                             const int32_t* starts, const int32_t* lengths, const int32_t* table, int seqs, int width, int max_new, const void* k_cache,
                             const void* v_cache, const float* k_scale, const float* v_scale, int pages, int page, void* out_f16, void* workspace,
                             void* stream) {
  if (variant < RCP_ATTENTION_AUTO || variant > RCP_ATTENTION_PROMPT) return RCP_ERR_VARIANT;
  if (polls < -1 || polls > (int)rcp::kPromptPolls) return RCP_ERR_SHAPE;
  if (!q_f16 || !out_f16) return RCP_ERR_NULL;
  rcp::AttnParams p{};
  const int rc = check_cache(tokens, heads, kv_heads, dim, starts, lengths, table, seqs, width, max_new, k_cache, v_cache, k_scale, v_scale, pages,
                             page, &p.s);
  if (rc != RCP_OK) return rc;
  if (!stride_ok(q_stride, (int64_t)heads * dim, tokens) || !std::isfinite(sm_scale) || sm_scale < 0.f) return RCP_ERR_SHAPE;
  if (!aligned16(q_f16) || !aligned16(out_f16) || !aligned16(workspace)) return RCP_ERR_ALIGN;
  if (!workspace) return RCP_ERR_WORKSPACE;
  if (tokens == 0) return RCP_OK;
  p.q = static_cast<const __half*>(q_f16);
  p.q_stride = q_stride;
  p.heads = heads; p.kv_heads = kv_heads; p.group = heads / kv_heads;
  auto inverse = [](uint32_t d) { return d == 1 ? 0u : (uint32_t)(((uint64_t(1) << 32) + d - 1) / d); };
  p.group_inv = inverse((uint32_t)p.group);
  p.kv_heads_inv = inverse((uint32_t)kv_heads);
  p.scale_log2 = sm_scale * 1.4426950408889634f;
  p.k_cache = static_cast<const uint8_t*>(k_cache);
  p.v_cache = static_cast<const uint8_t*>(v_cache);
  p.k_scale = k_scale; p.v_scale = v_scale;
  p.out = static_cast<__half*>(out_f16);
  p.status = static_cast<int32_t*>(workspace);
  p.polls = (uint32_t)polls;
  p.arrived = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + rcp::kAttnArrivedAt);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + rcp::kAttnPartsAt);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int64_t rows = (int64_t)p.s.max_new * p.group;
  const int64_t room = (int64_t)width * page;
  // (attn_quotient: rows and segments of a sequence below 2^16)
  if (variant == RCP_ATTENTION_SPLIT && (rows > 60000 || (rows + rcp::kAttnMaxRows - 1) / rcp::kAttnMaxRows * kv_heads > 65535)) return RCP_ERR_VARIANT;
  if (variant == RCP_ATTENTION_PROMPT) return attn_prompt(p, dim, polls >= 0, st);
  if (variant == RCP_ATTENTION_AUTO && rows > attn_few_rows(seqs, kv_heads, room)) {
    // (the prompt kernel runs anyway, and has CTAs free for all that is not as short as single tokens)
    const int few = room <= 1024 ? rcp::kAttnMaxRows : 2 * rcp::kAttnMaxRows;
    p.few = seqs > 1 ? few : 0;
    const int rc2 = attn_prompt(p, dim, polls >= 0, st);
    if (rc2 != RCP_OK || seqs == 1) return rc2;
    rows = few;   // and the sequences with few rows
  }
  const int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 3;
  if (dim == 64) return nt == 1 ? attn_split<64, 1>(p, st) : nt == 2 ? attn_split<64, 2>(p, st) : attn_split<64, 3>(p, st);
  return nt == 1 ? attn_split<128, 1>(p, st) : nt == 2 ? attn_split<128, 2>(p, st) : attn_split<128, 3>(p, st);
}

int rcp_kv_attention(const void* q_f16, int64_t q_stride, int tokens, int heads, int kv_heads, int dim, float sm_scale, const int32_t* starts,
                     const int32_t* lengths, const int32_t* table, int seqs, int width, int max_new, const void* k_cache, const void* v_cache,
                     const float* k_scale, const float* v_scale, int pages, int page, void* out_f16, void* workspace, void* stream) {
  return rcp_kv_attention_variant(RCP_ATTENTION_AUTO, -1, q_f16, q_stride, tokens, heads, kv_heads, dim, sm_scale, starts, lengths, table, seqs, width, max_new,
                                  k_cache, v_cache, k_scale, v_scale, pages, page, out_f16, workspace, stream);
}

size_t rcp_lora_workspace_bytes(int M, int rank) {
  if (M < 1 || M > 65535 || rank < 8 || rank > RCP_LORA_MAX_RANK || rank % 8) return 0;
  return kLoraRecordsAt + (size_t)((M + rcp::kLoraTile - 1) / rcp::kLoraTile) * rcp::lora_record_bytes(rank);
}

int rcp_lora_add(const void* x_f16, int64_t x_stride, const void* a_f16, const void* b_f16, const int32_t* adapter, const float* scaling,
                 const void* base_f16, int M, int N, int K, int rank, int adapters, void* y_f16, void* workspace, void* stream) {
  if (!x_f16 || !a_f16 || !b_f16 || !adapter || !scaling || !y_f16) return RCP_ERR_NULL;
  if (!workspace) return RCP_ERR_WORKSPACE;
  if (M < 1 || M > 65535 || N < 1 || K < 64 || K > 65536 || K % 64 || rank < 8 || rank > RCP_LORA_MAX_RANK || rank % 8 || adapters < 1)
    return RCP_ERR_SHAPE;
  if (N > RCP_LORA_MAX_N) return RCP_ERR_LIMIT;   // (column indexes go some thousands beyond a row's end)
  if (!stride_ok(x_stride, K, M)) return RCP_ERR_SHAPE;
  if (!aligned16(x_f16) || !aligned16(a_f16) || !aligned16(b_f16) || !aligned16(workspace) || !aligned4(adapter) || !aligned4(scaling) ||
      ((reinterpret_cast<uintptr_t>(base_f16) | reinterpret_cast<uintptr_t>(y_f16)) & 1u))
    return RCP_ERR_ALIGN;
  rcp::LoraParams p{static_cast<const __half*>(x_f16), x_stride, static_cast<const __half*>(a_f16), static_cast<const __half*>(b_f16), adapter,
                    scaling, static_cast<const __half*>(base_f16), static_cast<__half*>(y_f16), static_cast<uint8_t*>(workspace) + kLoraRecordsAt, M, N, K, rank, adapters,
                    1, 1};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (M <= rcp::kLoraFew) {
    RCP_CUDA(launch_overlapped(rcp::lora_few_kernel, dim3(M * rcp::kLoraCluster), dim3(rcp::kLoraThreads), 0, st, p));
    return RCP_OK;
  }
  // as many CTAs for the parts of K as there is room for
  const int tiles = (M + rcp::kLoraTile - 1) / rcp::kLoraTile;
  p.parts = 8;
  while (p.parts > 1 && (tiles * p.parts > 2 * sm_count() || p.parts > K / 64)) p.parts /= 2;
  switch ((rank - 1) / 16) {
    case 0: return lora_many<1>(p, tiles, st);
    case 1: return lora_many<2>(p, tiles, st);
    case 2: return lora_many<3>(p, tiles, st);
    case 3: return lora_many<4>(p, tiles, st);
    case 4: return lora_many<5>(p, tiles, st);
    case 5: return lora_many<6>(p, tiles, st);
    case 6: return lora_many<7>(p, tiles, st);
    default: return lora_many<8>(p, tiles, st);
  }
}

}  // extern "C"
