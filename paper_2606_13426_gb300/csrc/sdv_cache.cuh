// sdv_cache.cuh - the paged 8-bit key/value cache.
//
// Codes are e4m3.  Keys are [pages, H, block, D], values [pages, H, D, block] (a value row is
// contiguous along the tokens, the axis that the product with the probabilities sums over), and
// each page has one fp32 scale per head for its keys and one for its values.  Token i of sequence
// b is in row i % block of page page_table[b, i / block].
#pragma once

#include <cuda_fp8.h>

#include "sdv_tokens.cuh"

namespace sdv {

struct CacheView {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  const int32_t* table;
  int64_t pages;
  int max_pages;                    // entries of a row of the table
  int H, D, block;
};

// Tokens of a sequence at most: a position less a span, or plus a step, is an int.
constexpr int64_t kMaxTokens = 1 << 30;
constexpr int kChunk = 16;          // tokens: a block is a whole number of chunks

inline int check_cache(const void* k, const void* v, const void* ks, const void* vs, int64_t pages, const void* table,
                       int max_pages, int H, int D, int block) {
  if (!k || !v || !ks || !vs || !table) return SDV_EINVAL;
  if (pages < 1 || pages > 0x7fffffff || max_pages < 1 || H < 1 || H > 65535 || (D != 64 && D != 128)) return SDV_EINVAL;
  if (block < kChunk || block > SDV_MAX_BLOCK || block % kChunk) return SDV_EINVAL;
  if ((int64_t)max_pages * block > kMaxTokens) return SDV_EINVAL;
  if (!aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(ks, 4) || !aligned_to(vs, 4) || !aligned_to(table, 4))
    return SDV_EALIGN;
  return SDV_OK;
}

}  // namespace sdv
