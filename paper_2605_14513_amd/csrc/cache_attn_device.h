// What the kernels of heart_cache_attn share: the call, its sequences, which keys a query sees, tiles (gfx950).
#pragma once

#include "cache_device.h"

namespace heart {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(2))) int i32x2_t;

union Frag8 {
  u32x4_t u;
  bf16x8_t v;
};

__device__ __forceinline__ uint32_t cvt_pk_bf16(float lo, float hi) {
  f32x2_t f = {lo, hi};
  bf16x2_t b = __builtin_convertvector(f, bf16x2_t);
  return __builtin_bit_cast(uint32_t, b);
}

constexpr int kSplitSeqs = 256;  // most sequences of a call whose keys are divided: every wavefront looks at all, up to four a lane

// K or V of the cache
struct CacheTensor {
  const uint8_t *p, *exp;
  long long page, head;  // bytes
  uint32_t row;          // bytes between tokens
};
struct AttnCall {
  CacheTensor k, v;
  CacheSeqs s;
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  long long qt, qh, ot, oh;  // elements
  int H, G, causal, window;
  float scale_log2e;
  int4 *items;  // (divided keys) of each tile of a key head: number of its first part, parts, distance of their numbers
  float *part;
  int n_items, rounds, whole, tail;  // tiles of all heads; how their keys are divided (struct Division)
  unsigned long long *flags, mark;  // (divided keys, few rows) of the parts; what a set flag holds in this call
};

// One sequence as a kernel sees it.
struct Seq {
  int first, n, len;  // first new token, new tokens, cached tokens that there is room for
  int pos0;           // position of the first new token (may be negative)
};
__device__ __forceinline__ Seq seq_of(const AttnCall &c, int b) {
  Seq s;
  s.first = c.s.cu ? c.s.cu[b] : b * c.s.per;
  const int end = c.s.cu ? c.s.cu[b + 1] : s.first + c.s.per;
  // (token numbers outside the call's tensors: no tokens)
  s.n = s.first >= 0 && end > s.first && end <= c.s.T ? end - s.first : 0;
  const int kv = min(max(c.s.kv_len[b], 0), 0x7fffffff - 0x1000);
  s.pos0 = kv - s.n;
  s.len = min(kv, c.s.cap);
  return s;
}
// Keys lo .. hi - 1 that the query at position p sees: of those by the length, the ones that there is room for.
__device__ __forceinline__ void seen_by(const AttnCall &c, const Seq &s, int p, int &lo, int &hi) {
  hi = s.pos0 + s.n;
  if (c.causal) {
    uint32_t end = (uint32_t)max(p, 0) + 1u;
    if (c.causal > 1) end = (end - 1u) / (uint32_t)c.causal * (uint32_t)c.causal + (uint32_t)c.causal;  // < 2^32
    hi = p < 0 ? 0 : (int)min(end, (uint32_t)hi);
  }
  lo = c.window ? max(0, hi - c.window) : 0;
  hi = min(hi, s.len);
  lo = min(lo, hi);
}
// Tiles of TILE rows.
template <int TILE>
__device__ __forceinline__ int tiles_of(const AttnCall &c, const Seq &s) {
  return (s.n * c.G + TILE - 1) / TILE;
}
// Stages of STAGE keys that a tile of the sequence walks through at most (what the division of the keys goes by).
template <int TILE, int STAGE>
__device__ __forceinline__ int stages_of(const AttnCall &c, const Seq &s) {
  int st = (s.len + STAGE - 1) / STAGE;
  if (c.window) {
    const long long span = (long long)c.window + TILE / c.G + max(c.causal, 1);
    st = (int)min((long long)st, span / STAGE + 2);
  }
  return max(st, 1);
}
// Tiles are numbered so that a number's sequence can be found from the token ranges: those of sequence b start at
// first G / TILE + b, which leaves room for a short last tile of each.
template <int TILE>
__device__ __forceinline__ int tile_start(const AttnCall &c, int b) {
  const int first = c.s.cu ? c.s.cu[b] : b * c.s.per;
  return (int)((unsigned)max(first, 0) * (unsigned)c.G / TILE) + b;
}
// The last sequence whose tiles start at or before `tile`.
template <int TILE>
__device__ __forceinline__ int seq_of_tile(const AttnCall &c, int tile, int lane) {
  if (!c.s.cu) {
    // (b (per G / TILE + 1) rounded down: one division finds b or its neighbour)
    int b = min((int)((long long)tile * TILE / ((long long)c.s.per * c.G + TILE)), c.s.B - 1);
    while (b > 0 && tile_start<TILE>(c, b) > tile) --b;
    while (b + 1 < c.s.B && tile_start<TILE>(c, b + 1) <= tile) ++b;
    return b;
  }
  int lo = 0, n = c.s.B;  // (starts grow with b: 64 places at a time)
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const bool before = lane * step < n && tile_start<TILE>(c, at) <= tile;
    const int k = max(__popcll(__ballot(before)) - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Row r of a tile's sequence: where its query, output and log-sum-exp are.
struct Row {
  int token, head;
};
__device__ __forceinline__ Row row_of(const AttnCall &c, const Seq &s, int h, int r) {
  const int i = (int)((unsigned)r / (unsigned)c.G);
  return Row{s.first + i, h * c.G + r - i * c.G};
}

// The same for the rows of a tile that starts at row r0, by their number in it: i / G for i up to G + tile by a product with
// 1 / G, which is off by less than one.
struct Rows {
  int first, i0, rest, G;
  float inv;
  __device__ __forceinline__ Rows(const AttnCall &c, const Seq &s, int r0)
      : first(s.first), i0((int)((unsigned)r0 / (unsigned)c.G)), rest(r0 - i0 * c.G), G(c.G), inv(1.f / (float)c.G) {}
  __device__ __forceinline__ int token(int r) const {  // of the sequence's new tokens
    const int x = rest + r;
    int q = (int)((float)x * inv);
    q += (q + 1) * G <= x ? 1 : 0;
    q -= q * G > x ? 1 : 0;
    return i0 + q;
  }
  __device__ __forceinline__ Row row(int h, int r) const {
    const int q = token(r);
    return Row{first + q, h * G + rest + r - (q - i0) * G};
  }
};

// What a workgroup works on.
struct Work {
  int b, h, m;            // sequence, key head, tile
  int part, parts, step;  // (divided keys) part of the tile's stages, their number, distance of their numbers
  int slot;               // number of the part
};

// Tiles of TILE rows of a call at most, of all heads.
inline long long most_items(int tile, int B, int H, int T, int Hq) { return ((long long)T * (Hq / H) / tile + B) * H; }

// Few rows a key head (cache_attn_few.hip).
bool cache_attn_few(int B, int H, int T, int Hq);
size_t cache_attn_few_workspace_bytes(int B, int H, int D, int T, int Hq);
int launch_cache_attn_few(const heart_cache &c, int T, int Hq, AttnCall &a, void *workspace, hipStream_t st);

}  // namespace heart
