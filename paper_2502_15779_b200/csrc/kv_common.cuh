// The paged cache of keys and values (rcp_kv_append, rcp_kv_attention): geometry, which tokens belong to which sequence, and the
// numbers it holds.
//
// Numbers. A block is what one page holds of one key head. Its values are e4m3 codes times a scale of the block that is a power of two, the
// smallest with the block's largest magnitude at most 448 (e4m3's largest) times it. e4m3 is a floating format, so a power of two
// costs no precision against the exact quotient, and a block whose scale grows when a larger token comes in is rescaled by
// shifting exponents: exact, except where a value leaves the format's range of 2^-9 .. 448 at the lower end. With a
// linear 8-bit format every growth would round what is already there once more.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace rcp {

constexpr int kKvExpMin = -40, kKvExpMax = 9;   // exponents of a block's scale
constexpr float kKvCap = 131072.f;              // magnitudes are cut off here: above twice the largest fp16 number, below 448 * 2^kKvExpMax

struct KvSeqs {
  const int32_t* starts;    // [seqs + 1]
  const int32_t* lengths;   // [seqs]
  const int32_t* table;     // [seqs][width]
  int seqs, width, page, lg_page, pages, tokens, max_new;
};

// What a sequence's entries say, cut to what exists: nothing that is read by these numbers can lie outside the tensors, whatever
// the entries are.
struct KvSeq {
  int t0, n;      // its new tokens are rows t0 .. t0 + n - 1
  int first;      // position of the first of them (negative where a length is below the number of new tokens)
  int end;        // positions that exist: 0 .. end - 1 (tokens beyond max_new have none: nothing is stored for them)
};
__device__ __forceinline__ KvSeq kv_seq(const KvSeqs& s, int b) {
  KvSeq r;
  const int a = s.starts[b], e = s.starts[b + 1], len = s.lengths[b];
  r.t0 = min(max(a, 0), s.tokens);
  const int t1 = min(max(e, r.t0), s.tokens);
  // (a length is at most what int holds; below zero it is taken as zero, and no more tokens than that have a position)
  r.n = min(t1 - r.t0, s.max_new);
  r.first = max(len, 0) - (t1 - r.t0);
  r.end = max(min(r.first + r.n, s.width << s.lg_page), 0);
  return r;
}
// Sequence of row t (0 <= t < starts[seqs]): the last one that starts at or in front of it.
__device__ __forceinline__ int kv_find(const int32_t* starts, int seqs, int t) {
  int lo = 0, hi = seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// exponent of the scale of a block whose largest magnitude is `amax` (finite, >= 0): smallest e with amax <= 1.75 * 2^8 * 2^e
__device__ __forceinline__ int kv_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  return min(max((int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), kKvExpMin), kKvExpMax);
}
__device__ __forceinline__ int kv_stored_exponent(float scale) {
  return min(max((int)((__float_as_uint(scale) >> 23) & 255u) - 127, kKvExpMin), kKvExpMax);
}
__device__ __forceinline__ float kv_pow2(int e) { return __int_as_float((e + 127) << 23); }

}  // namespace rcp
