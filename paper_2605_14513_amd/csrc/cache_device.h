// What the kernels on the paged key/value cache share (gfx950).
#pragma once

#include "heart_internal.h"

namespace heart {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_c;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_c;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_c;

// The sequences of a call: token ranges (cu, or `per` new tokens each) and lengths.
struct CacheSeqs {
  const int *cu, *kv_len, *page_table;
  int T, B, per;        // new tokens, sequences, T / B
  int cap;              // max_pages * page: positions a sequence can have
  int page_shift, max_pages, n_pages;
};

constexpr long long kMostGroups = (1ll << 24) - 1;  // workgroups of 256 threads: a launch has less than 2^32 threads

inline CacheSeqs cache_seqs(const heart_cache &c, int T, const int *cu_q) {
  return CacheSeqs{cu_q, c.kv_len, c.page_table, T, c.B, T / c.B, c.max_pages * c.page, __builtin_ctz((unsigned)c.page),
                   c.max_pages, c.n_pages};
}

// Page of a position (0 <= pos < cap) of sequence b, -1 if the table names none.
__device__ __forceinline__ int cache_page(const CacheSeqs &s, int b, int pos) {
  const int id = s.page_table[(long long)b * s.max_pages + (pos >> s.page_shift)];
  return (unsigned)id < (unsigned)s.n_pages ? id : -1;
}

// What a cache's elements are (heart_cache's type).
enum CacheKind { kBf16 = HEART_CACHE_BF16, kE4m3 = HEART_CACHE_E4M3, kInt8 = HEART_CACHE_INT8 };

// Two codes (the lower or the upper half of w) as bf16 times a power of two: exact.
template <bool kUpper>
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t w, float unit) {
  const bf16x2_c r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, unit, kUpper);
  return __builtin_bit_cast(uint32_t, r);
}
// 2^(exp - 127) as the conversions take it: by the exponent bits alone (0: 2^-127, though as a float it is 0; 255: NaN)
__device__ __forceinline__ float unit_of(uint32_t exp) { return __uint_as_float(exp << 23); }

}  // namespace heart
