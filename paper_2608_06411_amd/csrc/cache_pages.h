// What the cache's kernels share: places of tokens in the pages, and the
// 4-bit codes.
#pragma once

#include "internal.h"

namespace mapk {

// A sequence's tokens, within what its table can name.
__device__ __forceinline__ int cache_len(const CachePages& c, int b) {
  const long long cap = (long long)c.max_pages << c.shift;
  const int n = max(c.len[b], 0);
  return n < cap ? n : static_cast<int>(cap);
}

// The page of token j (0 <= j < max_pages << shift), or -1 if its entry is no
// page of the pool.
__device__ __forceinline__ int cache_page(const CachePages& c, int b, int j) {
  const int p = c.table[(long long)b * c.max_pages + (j >> c.shift)];
  return static_cast<unsigned>(p) < static_cast<unsigned>(c.n_pages) ? p : -1;
}

// Row number of (page, head, place): times head_dim it is the offset of the
// token's values.  64 bits: a pool may pass 4 GiB.
__device__ __forceinline__ long long cache_row(const CachePages& c, int page, int head, int j) {
  return (((long long)page * c.heads + head) << c.shift) + (j & ((1 << c.shift) - 1));
}

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// Codes 2 SEL and 2 SEL + 1 of eight (a word), times a power of two: two bf16.
// Exact (a level has two significant bits); the scale's exponent 255 gives NaN.
template <int SEL> __device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
__device__ __forceinline__ uint4 fp4_eight(uint32_t codes, float scale) {
  return make_uint4(fp4_pair<0>(codes, scale), fp4_pair<1>(codes, scale), fp4_pair<2>(codes, scale),
                    fp4_pair<3>(codes, scale));
}
// The scale as the conversion reads it (its exponent).
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace mapk
