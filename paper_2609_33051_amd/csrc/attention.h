// Argument blocks and device helpers of the attention layer's operators
// (rotary positions, the 4-bit cache, attention).
#pragma once

#include "mixer.h"

namespace skssm {

// A paged cache in 4 bits: records of 16 tokens of one head, 17 D bytes (keys, values, their exponents).
struct Cache {
  uint8_t* data;
  int pages, heads, shift;  // 2^shift records (16 tokens each) a page
};

// The new tokens of a batch and where their sequences lie in the cache.
struct NewTokens {
  Sequences seq;
  const int32_t* lengths;
  const int32_t* table;
  size_t ld_table;
  int columns;
  // Place of sequence b's i-th of n new tokens.  Lengths below -2^30 count as that, so that no place wraps.
  __device__ __forceinline__ int place(int b, int n, int i) const {
    const int length = lengths[b];
    return (length < -(1 << 30) ? -(1 << 30) : length) - n + i;
  }
  // The page of a sequence's record `tile`, or -1 where there is none.
  __device__ __forceinline__ int page(const Cache& c, int b, int tile) const {
    const int j = tile >> c.shift;
    if (j >= columns) return -1;
    const int p = table[(size_t)b * ld_table + j];
    return (unsigned)p < (unsigned)c.pages ? p : -1;
  }
};

template <int D> __device__ __forceinline__ uint8_t* record(const Cache& c, int page, int head, int tile) {
  return c.data + ((((size_t)page * c.heads + head) << c.shift) + (tile & ((1 << c.shift) - 1))) * (17 * D);
}

struct Rotation {
  const float* angles;
  const int32_t* positions;
  int places, rotated, interleaved;
};

struct CacheAppendArgs {
  NewTokens tok;  // lengths NULL: no cache (sketchssm_rotary)
  Cache cache;
  Rotation rot;
  int H, D;       // query heads (0: none), channels
  const void* q;
  size_t ldq, q_head;
  void* y;        // the rotated queries
  size_t ldy, y_head;
  const void* k;
  size_t ldk, k_head;
  const void* v;
  size_t ldv, v_head;
};
int run_append(const CacheAppendArgs& a, int io, void* stream);

struct ReadArgs {
  NewTokens tok;
  Cache cache;
  int D;
  void* k;
  void* v;
};
int run_cache_read(const ReadArgs& a, int io, void* stream);

struct AttentionArgs {
  NewTokens tok;
  Cache cache;
  int H, group;    // query heads, and how many share a key head
  uint32_t magic, bits;
  // n / group of 0 <= n < 2^31, with 2^bits >= group, magic = floor(2^32 (2^bits - group) / group) + 1: the product is n (2^bits / group - 1), a
  // little more, over 2^32.
  __device__ __forceinline__ int by_group(int n) const { return (int)((__umulhi((uint32_t)n, magic) + (uint32_t)n) >> bits); }
  float scale;
  const void* q;
  size_t ldq, q_head;
  void* out;
  size_t ld_out;
  float* scales;
  size_t ld_scales;
  float* work;     // [share][key heads][2]: a tile's sums, maxima and sums of weights
  int* plan;       // at the workspace's start (NULL: no tile can be split)
  int share;       // workgroups of attention_kernel a key head
  int most;        // rounds that a key head can have
  int span;        // pieces of 8 channels a workgroup of join_kernel
};
int run_attention(const AttentionArgs& a, int D, int io, bool fp8, void* stream);
size_t attention_workspace(int batch, int tokens, int H, int G, int D, int columns, int page);

}  // namespace skssm
