// heart_cache_attn where a key head has few rows (single tokens, drafts of a few): bound by reading the cache.
//
// A tile is 16 rows, and a workgroup's four wavefronts divide the keys of its part among them, slice by slice, each
// with a softmax state of its own that is put together at the end.  Every wavefront brings its own slices into its own
// part of LDS, so the loop has no barrier, only waits for the wavefront's own loads:
//   S^T (keys x rows) = K . Q^T,  O^T (d x rows) += V^T . P^T     with v_mfma_f32_16x16x32_bf16 (16x16x16 for slices of 16)
// In the 16x16 accumulator a lane holds one row (lane % 16) and keys 4 (lane / 16) + 0..3; exponentiated they are, as they
// are, the B operand of the second product, whose A operand the transposing LDS reads deliver in the same order of keys.
//
// K and V slices (16 to 64 keys) are double-buffered, 8 KB a slice, by LDS-direct loads; K of
// slice i + 2 is issued as soon as the fragments of K of slice i are in registers, V likewise, so 8 to 16 KB a wavefront, 64
// to 128 KB a CU, are on their way at any time.  Codes stay codes in LDS: K is converted with its row's power of two at the
// fragment read; V as it is, its powers of two go into the weights, which are multiplied by them before they are
// rounded (a power of two rounds nothing).
//
// int8: codes are bf16 as they are, scales (one for 16 rows, which lie in a page) are factors of the logits and of the weights.
//
// Dividing the keys: struct Shares.  The workgroup that finds all parts of a tile there adds them up.  Little is not divided
// (int8, kFewAll).
//
// 64 ragged sequences of up to 8192 tokens, 8 key heads of 128, e4m3 (385 MB) and int8 74 us, 5.2 TB/s; one of 120001 tokens, bf16
// (492 MB) 84 us, 5.8 TB/s, int8 (246 MB) 53, 4.6; 64 of 16384, bf16 (4.3 GB) 6.8 TB/s, of 32768 in e4m3 6.6 (a plain read 7.1).  One of
// 1000 tokens, two heads: 9.9 us, int8 8.9, bound by latency.
#include <type_traits>

#include "cache_attn_device.h"

namespace heart {

constexpr int kFewTile = 16;     // rows of a workgroup
constexpr int kFewWaves = 4;     // its wavefronts, and
constexpr int kFewAll = 16;      // those of a workgroup that has all keys of a tile at once, a slice a wavefront
constexpr int kFewStage = 128;   // keys that shares are measured in
constexpr int kFewMin = 2;       // shortest share, in stages
constexpr int kFewCut = 1;       // fewest stages of a part: a cut closer to an end of its tile goes there
// A call that reads more than this (by the length of its shares, what its tiles cost beside their stages among it) loads past
// the caches (nt): as nothing of it is read twice, and what the memory-side cache (256 MB) could keep for the next call would
// be gone before.  us with and without: 64 sequences of 16384 tokens, 8 heads (4.3 GB) 625 / 710 (6.87 / 6.05 TB/s), of 4096
// (1.1 GB) 161 / 185, 32 of 1024 (128 MB) 30.0 / 31.7, where they are not in that cache, of 512 (64 MB) 23.8 / 24.3, but
// 23.4 / 21.7 where they are (three such caches in turn).
constexpr long long kFewOnce = 80ll << 20;
constexpr int kFewItems = 8192;   // most tiles of a call whose keys are divided
constexpr int kFewPlaces = 512;   // shares at most: places for workgroups, two a CU

template <int D>
constexpr int kFewPart = kFewTile * (D + 2);  // floats of a part: rows of D, references, row sums

// How the keys of all tiles (sequences; of each, heads, tiles) are dealt out.  Every wavefront finds its own from the lengths:
// no plan, no queue, and no workgroup waits for another.
//   parts   where there are places for parts of at most 2, 4 or 8 stages of every tile: one each (one token of 1000 keys, two
//           heads: 11.3 us with shares, 9.9 with parts)
//   shares  else the stages, one tile's after the other's, are one sequence, which is cut into equal shares; lengths are in half
//           stages, and a tile costs COST beside its stages (64 ragged sequences: 81 us with shares; 86 to 95 with parts of
//           different lengths in two or three rounds of workgroups)
// (NB: sequences a lane.  One where that is enough: code that is jumped over has to be fetched all the same.)
template <int COST, int NB_>
struct Shares {
  static constexpr int NB = NB_;
  Seq s[NB];                           // sequences 64 j + lane:
  int tiles[NB], st[NB], before[NB];   // tiles of a head, stages of each, length of what is before
  int n, step, rest, total;
  int part_log;                        // (parts) log2 of a part's stages at most, 0 = shares
  __device__ __forceinline__ int parts_of(int j) const { return (st[j] + (1 << part_log) - 1) >> part_log; }
  __device__ __forceinline__ int cut(int k) const { return k * step + min(k, rest); }
  // the last cut at or before v
  __device__ __forceinline__ int last_cut(int v) const {
    const int longer = rest * (step + 1);
    return v < longer ? (int)((unsigned)v / (unsigned)(step + 1)) : rest + (int)((unsigned)(v - longer) / (unsigned)step);
  }
  // stages of a tile of `len` before a cut d behind the tile's start
  __device__ __forceinline__ static int inside(int d, int len) {
    const int x = (d - COST + 1) >> 1;
    return x >= len ? len : x < kFewCut ? 0 : len - x < kFewCut ? len : x;
  }
  // of a divided tile (one with a cut at least kFewCut from either end) at `tile0`: share of its first part, number of parts
  __device__ __forceinline__ void cut_parts(int tile0, int len, int &first, int &parts) const {
    first = last_cut(tile0 + 2 * kFewCut + COST - 2);
    parts = last_cut(tile0 + 2 * (len - kFewCut) + COST) + 1 - first;
  }
  // false: no work
  __device__ __forceinline__ bool find(const AttnCall &c, int places, int lane) {
    int at = 0;
    bool falls = false;  // (token ranges that fall somewhere overlap: sums could leave 32 bits)
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int b = j * 64 + lane;
      s[j] = Seq{0, 0, 0, 0};
      tiles[j] = 0;
      st[j] = 1;
      before[j] = 0;
      if (j * 64 < c.s.B) {
        if (b < c.s.B) {
          s[j] = seq_of(c, b);
          falls = falls || (c.s.cu && c.s.cu[b + 1] < c.s.cu[b]);
          tiles[j] = tiles_of<kFewTile>(c, s[j]);
          st[j] = stages_of<kFewTile, kFewStage>(c, s[j]);
        }
        const int len = tiles[j] * c.H * (2 * st[j] + COST), end = at + wave_scan_i32(len);
        before[j] = end - len;
        at = __builtin_amdgcn_readlane(end, 63);
      }
    }
    total = at;
    n = 0;
    for (part_log = 1; part_log <= 3; ++part_log) {
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (j * 64 < c.s.B) n += tiles[j] * parts_of(j);
      n = __builtin_amdgcn_readfirstlane(wave_sum_i32(n)) * c.H;
      if (n <= places) return at > 0 && !__any(falls);
      n = 0;
    }
    part_log = 0;
    n = min(places, max(at / (2 * kFewMin + COST), 1));
    step = (int)((unsigned)at / (unsigned)n);
    rest = at - step * n;
    return at > 0 && !__any(falls);
  }
};

template <int D, CacheKind kKind, int WAVES>
struct FewShape {
  static constexpr bool kCodes = kKind != kBf16;
  static constexpr int ROWB = kCodes ? D : 2 * D;        // bytes of a row
  static constexpr int SK = 4096 / ROWB;                 // keys of a slice
  static constexpr int NT = SK / 16;                     // key tiles of 16
  static constexpr int TENSOR_B = SK * ROWB;             // bytes of a slice of K or V
  static constexpr int SLICE_B = 2 * TENSOR_B + (kCodes ? 256 : 0);
  static constexpr int WAVE_B = (WAVES > kFewWaves ? 1 : 2) * SLICE_B;  // double-buffered, but where there is one slice
  static constexpr int NI = 16 * ROWB / 1024;            // LDS-direct loads of 16 rows
};

// (int8) Four codes as bf16, which has room for them: fp32 cut to its upper half.
__device__ __forceinline__ u32x2_t ints_to_bf16(uint32_t w) {
  uint32_t f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __float_as_uint((float)(int8_t)(w >> (8 * i)));
  return u32x2_t{__builtin_amdgcn_perm(f[1], f[0], 0x07060302u), __builtin_amdgcn_perm(f[3], f[2], 0x07060302u)};
}

// SEQS: sequences a lane where the keys are divided, 0 = they are not
template <int D, CacheKind kKind, int SEQS, int WAVES = kFewWaves>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4 > 2 ? WAVES / 4 : 2) void cache_attn_few_kernel(const AttnCall c) {
  using F = FewShape<D, kKind, WAVES>;
  constexpr bool kAll = WAVES > kFewWaves;  // (all keys at once)
  static_assert(!kAll || SEQS == 0, "not divided");
  constexpr bool kCodes = F::kCodes, kInts = kKind == kInt8;
  constexpr bool kSplit = SEQS > 0;
  constexpr int TILE = kFewTile, ROWB = F::ROWB, SK = F::SK, NT = F::NT, NI = F::NI;
  constexpr int NC = ROWB / 16, RPB = 256 / ROWB, RPI = 1024 / ROWB;  // chunks of a row, rows per 256 bytes, rows of a load
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int NLOAD = NT * NI;                       // loads of K (or V) of a slice
  constexpr int PER = 2 * NLOAD + (kCodes ? 1 : 0);    // all of a slice
  constexpr float ninf = -__builtin_inff(), kSlack = 8.f;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ float s_ref[WAVES][TILE], s_sum[WAVES][TILE];
  __shared__ bool s_all;
  const uint32_t smem_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);

  // ---- what to work on -----------------------------------------------------------------------
  // (shares) the share's number and ends; of the tile: its sequence, number in it, start; of the sequence: tiles of a head and
  // of all, stages of a tile
  using Sh = Shares<512 / ROWB, kSplit ? SEQS : 1>;
  [[maybe_unused]] Sh sh;
  int share = 0, cut0 = 0, cut1 = 0, b = 0, number = 0, tile0 = 0, n_head = 1, n_seq = 0, len = 1;
  int first_part = 0, parts = 0;  // (parts, and of a divided tile) number of its first part, their number
  Seq s;
  auto enter = [&](int j, int l) __attribute__((always_inline)) {
    b = j * 64 + l;
    s = Seq{__builtin_amdgcn_readlane(sh.s[j].first, l), __builtin_amdgcn_readlane(sh.s[j].n, l),
            __builtin_amdgcn_readlane(sh.s[j].len, l), __builtin_amdgcn_readlane(sh.s[j].pos0, l)};
    len = __builtin_amdgcn_readlane(sh.st[j], l);
    n_head = __builtin_amdgcn_readlane(sh.tiles[j], l);
    n_seq = n_head * c.H;
    tile0 = __builtin_amdgcn_readlane(sh.before[j], l);
    number = 0;
  };
  if constexpr (kSplit) {
    if (!sh.find(c, (int)gridDim.x, lane)) return;
    share = (int)blockIdx.x;
    if (share >= sh.n) return;
    if (sh.part_log) {
      int at = 0;
#pragma unroll
      for (int j = 0; j < Sh::NB; ++j)
        if (j * 64 < c.s.B) {
          const int of_tile = sh.parts_of(j), all = sh.tiles[j] * c.H * of_tile;
          const int end = at + wave_scan_i32(all);
          const unsigned long long here = __ballot(end - all <= share && share < end);
          if (here) {
            const int l = __ffsll((long long)here) - 1;
            enter(j, l);
            parts = __builtin_amdgcn_readlane(of_tile, l);
            const int r = share - __builtin_amdgcn_readlane(end - all, l);
            number = (int)((unsigned)r / (unsigned)parts);
            first_part = share - (r - number * parts);
          }
          at = __builtin_amdgcn_readlane(end, 63);
        }
    } else {
      cut0 = sh.cut(share);
      cut1 = sh.cut(share + 1);
#pragma unroll
      for (int j = 0; j < Sh::NB; ++j)
        if (j * 64 < c.s.B) {
          const unsigned long long here =
              __ballot(sh.before[j] <= cut0 && cut0 < sh.before[j] + sh.tiles[j] * c.H * (2 * sh.st[j] + 512 / ROWB));
          if (here) {
            enter(j, __ffsll((long long)here) - 1);
            number = (int)((unsigned)(cut0 - tile0) / (unsigned)(2 * len + 512 / ROWB));
            tile0 += number * (2 * len + 512 / ROWB);
          }
        }
    }
  } else {
    const int tile = (int)(blockIdx.x / (unsigned)c.H);
    b = seq_of_tile<kFewTile>(c, tile, lane);
    s = seq_of(c, b);
    number = __builtin_amdgcn_readfirstlane(tile - tile_start<kFewTile>(c, b));
    if (number < 0 || number >= tiles_of<kFewTile>(c, s)) return;
  }
  // ---- LDS layout: 16-byte chunk c of slice row r at chunk position c ^ f(r), so that the rows read together fall into
  // different banks
  auto swizzle = [](int is_v, int r) {
    if (!is_v) return (r / RPB) % NC;
    if constexpr (kCodes) return (r / RPB) % (NC / 2) + (r / 16) % 2 * (NC / 2);
    return 2 * ((r / RPB) % (NC / 2));
  };
  // K fragments: row l16 of a tile; chunk 4 ks + g (bf16: one k-step; codes: two)
  constexpr int KR = kCodes ? KS / 2 : KS;
  uint32_t koff[KR];
#pragma unroll
  for (int i = 0; i < KR; ++i) koff[i] = (uint32_t)(l16 * ROWB + (((4 * i + g) ^ swizzle(0, l16)) * 16));
  // V^T fragments: 16 lanes name a block of 4 keys x 16 d (bf16) or 8 keys x 16 d (codes), lane i receives d = i
  uint32_t voff[DT];
  {
    const int r = kCodes ? (l16 < 8 ? 4 * g + (l16 >> 1) : 16 + 4 * g + ((l16 >> 1) - 4)) : 4 * g + (l16 >> 2);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const int ch = kCodes ? dt : 2 * dt + ((l16 & 3) >> 1);
      voff[dt] = (uint32_t)(r * ROWB + ((ch ^ swizzle(1, r)) * 16) + (l16 & 1) * 8);
    }
  }
  // LDS-direct loads: lane l fills chunk position l % NC of row l / NC of a load's rows
  uint32_t dma_off[2][NI];
#pragma unroll
  for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
    for (int ii = 0; ii < NI; ++ii) {
      const int r = ii * RPI + lane / NC;
      dma_off[is_v][ii] = (uint32_t)r * (is_v ? c.v.row : c.k.row) + (uint32_t)(((lane % NC) ^ swizzle(is_v, r)) * 16);
    }
  // (rows of odd tiles: V codes are swizzled differently there)
  uint32_t dma_off2[kCodes ? NI : 1];
  if constexpr (kCodes) {
#pragma unroll
    for (int ii = 0; ii < NI; ++ii) {
      const int r = ii * RPI + lane / NC;
      dma_off2[ii] = (uint32_t)r * c.v.row + (uint32_t)(((lane % NC) ^ swizzle(1, r + 16)) * 16);
    }
  }

  for (;;) {
  int x0 = 0, x1 = len;  // stages of the tile that belong to the share; a cut near an end of the tile is at that end
  if constexpr (kSplit) {
    if (sh.part_log) {
      x0 = (share - first_part) * len / parts;
      x1 = (share - first_part + 1) * len / parts;
    } else {
      x0 = Sh::inside(cut0 - tile0, len);
      x1 = Sh::inside(cut1 - tile0, len);
      if (x1 == 0) return;
    }
  }
  if (x0 < x1) {
  const int head = __builtin_amdgcn_readfirstlane(kSplit ? (n_head == 1 ? number : (int)((unsigned)number / (unsigned)n_head))
                                                         : (int)(blockIdx.x % (unsigned)c.H));
  const int m = kSplit ? number - head * n_head : number;
  const int rows = s.n * c.G, r0 = m * TILE, n_rows = min(TILE, rows - r0);
  const Rows at0(c, s, r0);  // tokens of the tile's rows
  int first_key, end_key, ignore;
  seen_by(c, s, s.pos0 + at0.token(0), first_key, ignore);
  seen_by(c, s, s.pos0 + at0.token(n_rows - 1), ignore, end_key);
  int stage0 = first_key / kFewStage, n_stage = max((end_key + kFewStage - 1) / kFewStage - stage0, 0);
  const bool partial = kSplit && x1 - x0 < len;
  const int tile_end = __builtin_amdgcn_readfirstlane(end_key);  // keys from here on no row of the tile sees: zeros
  if (partial) {
    // (of the n_stage stages that this tile has: len is that of the sequence's longest)
    const int y0 = n_stage == len ? x0 : (int)((long long)x0 * n_stage / len);
    const int y1 = n_stage == len ? x1 : (int)((long long)x1 * n_stage / len);
    stage0 += y0;
    n_stage = y1 - y0;
    end_key = min(end_key, (stage0 + n_stage) * kFewStage);
  }
  const int key0 = __builtin_amdgcn_readfirstlane(stage0 * kFewStage + wave * SK);  // of this wavefront's slice 0
  end_key = __builtin_amdgcn_readfirstlane(end_key);
  const int n_slice = __builtin_amdgcn_readfirstlane(max((end_key - key0 + WAVES * SK - 1) / (WAVES * SK), 0));

  int lo, hi;  // keys that this lane's row sees of the part
  seen_by(c, s, s.pos0 + at0.token(min(l16, n_rows - 1)), lo, hi);
  if (l16 >= n_rows) lo = 0, hi = end_key;  // (rows past the end see what is there)
  hi = min(hi, end_key);
  // slices from all_lo on and before all_hi need no mask (in vector registers: as scalars they made the loop 7 % slower, 64 ragged
  // sequences in e4m3 73.6 -> 78.8 us)
  const int all_lo = (int)wave_max_u32((uint32_t)lo);
  const int all_hi = (int)wave_min_u32((uint32_t)hi);

  // ---- page ids of slices base .. base + 63, lane l that of slice base + l, by tile
  int ids[NT];
  auto load_ids = [&](int base) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const long long key = key0 + (long long)(base + lane) * (WAVES * SK) + 16 * n;
      ids[n] = key < end_key ? cache_page(c.s, b, (int)key) : -1;
    }
  };
  // (codes) of slices i, i + 1, i + 2: all ones where the tile's page is one
  uint32_t named[3][NT];
  const int in_page = (1 << c.s.page_shift) - 1;
  const uint32_t wave_lds = smem_lds + (uint32_t)(wave * F::WAVE_B);
  unsigned char *const wave_mem = smem + wave * F::WAVE_B;
  // (half stages times 128 keys: bytes of K and V)
  const bool once = !kAll && (!kSplit || (long long)sh.total * (128 * ROWB) > kFewOnce);
  // K (V) of slice i to buffer i & 1
  auto bring = [&](int is_v, int i) __attribute__((always_inline)) {
    const CacheTensor &x = is_v ? c.v : c.k;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int key = key0 + i * (WAVES * SK) + 16 * n, off = key & in_page;
      const int id = i < n_slice ? __builtin_amdgcn_readlane(ids[n], i & 63) : -1;
      const uint64_t addr = (uint64_t)(x.p + max(id, 0) * x.page + head * x.head + off * (long long)x.row);
      const int there = id < 0 ? 0 : min(tile_end - key, 16);
      u32x4_t rs;
      rs.x = __builtin_amdgcn_readfirstlane((uint32_t)addr);
      rs.y = __builtin_amdgcn_readfirstlane((uint32_t)(addr >> 32) & 0xffffu);
      rs.z = __builtin_amdgcn_readfirstlane(there > 0 ? (uint32_t)(there - 1) * x.row + (uint32_t)ROWB : 0u);
      rs.w = 0x00020000u;
#pragma unroll
      for (int ii = 0; ii < NI; ++ii) {
        const uint32_t dst = wave_lds + (uint32_t)((i & 1) * F::SLICE_B + is_v * F::TENSOR_B + (n * NI + ii) * 1024);
        const uint32_t voffset = kCodes && is_v && (n & 1) ? dma_off2[kCodes ? ii : 0] : dma_off[is_v][ii];
        // (the compiler does not see this instruction's LDS write: completion is awaited by count.  M0 is saved and
        // restored, it may hold a value of the compiler's)
        uint32_t m0_saved;
        if (once)
          asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                       "buffer_load_dwordx4 %2, %3, 0 offen nt lds\n\ts_mov_b32 m0, %0"
                       : "=&s"(m0_saved) : "s"(dst), "v"(voffset), "s"(rs) : "memory");
        else
          asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                       "buffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                       : "=&s"(m0_saved) : "s"(dst), "v"(voffset), "s"(rs) : "memory");
      }
    }
  };
  // (codes) exponents of slice i, 4 bytes a lane: K of its tiles, then V; pages that are none: of page 0.  Of int8 the scales, one a tile.
  auto bring_exps = [&](int i, int ahead) __attribute__((always_inline)) {
    if constexpr (kCodes) {
      const int dw = lane % (kInts ? 2 * NT : 8 * NT), n = (kInts ? dw : dw >> 2) % NT;
      int id = -1;
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        const int id_m = i < n_slice ? __builtin_amdgcn_readlane(ids[m], i & 63) : -1;
        named[ahead][m] = id_m < 0 ? 0u : 0xffffffffu;
        id = n == m ? id_m : id;
      }
      id = max(id, 0);
      const int key = key0 + i * (WAVES * SK) + 16 * n;
      const uint8_t *base = dw >= (kInts ? NT : 4 * NT) ? c.v.exp : c.k.exp;
      const uint8_t *addr = kInts ? base + ((long long)id * c.H + head) * 4
                                  : base + ((((long long)id * c.H + head) << c.s.page_shift) + (key & in_page) + 4 * (dw & 3));
      const uint32_t dst = wave_lds + (uint32_t)((i & 1) * F::SLICE_B + 2 * F::TENSOR_B);
      uint32_t m0_saved;
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                   "global_load_lds_dword %2, off\n\ts_mov_b32 m0, %0"
                   : "=&s"(m0_saved) : "s"(dst), "v"(addr) : "memory");
    }
  };

  // ---- state of the rows -----------------------------------------------------------------------
  Frag8 qf[KS];
  f32x4_t o[DT];
  float m_ref = ninf, c0 = 0.f, l_run = 0.f;  // reference exponent, minus that in raw logits, this lane's part of the row sum
  float less = 0.f;  // (int8) minus the reference exponent, where there is one
  {
    const Row at = at0.row(head, min(l16, n_rows - 1));
    const uint16_t *src = c.q + at.token * c.qt + at.head * c.qh;
    // (codes: a lane's 16 bytes are d 16 (4 i + g) .. of k-steps 2 i and 2 i + 1)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[ks].u = *reinterpret_cast<const u32x4_t *>(src + (kCodes ? 16 * (4 * (ks / 2) + g) + 8 * (ks & 1) : 32 * ks + 8 * g));
  }
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const float scale_log2e = c.scale_log2e, inv_scale = 1.f / scale_log2e;

  if (n_slice > 0) {
    load_ids(0);
    bring(0, 0);
    bring_exps(0, 0);
    bring(1, 0);
    if constexpr (!kAll) {
      bring(0, 1);
      bring_exps(1, 1);
      bring(1, 1);
    }
    for (int i = 0; i < (kAll ? 1 : n_slice); ++i) {
      const unsigned char *sk = wave_mem + (i & 1) * F::SLICE_B, *sv = sk + F::TENSOR_B, *se = sk + 2 * F::TENSOR_B;
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NLOAD + (kAll ? 0 : PER)) : "memory");  // K and exponents of slice i are there
      const int key = key0 + i * (WAVES * SK);
      // ---- S^T ------------------------------------------------------------------------------
      Frag8 kf[NT][KS];
      float vu[NT][4];  // (codes) powers of two of V's rows 16 n + 4 g + 0..3, or their scale
      float factor[NT];  // of the logits
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        factor[n] = scale_log2e;
        if constexpr (kInts) {
          const uint32_t *units = reinterpret_cast<const uint32_t *>(se);
          factor[n] *= __uint_as_float(units[n] & named[0][n]);
#pragma unroll
          for (int e = 0; e < 4; ++e) vu[n][e] = __uint_as_float(units[NT + n] & named[0][n]);
#pragma unroll
          for (int j = 0; j < KR; ++j) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(sk + 16 * n * ROWB + koff[j]);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const u32x2_t a = ints_to_bf16(x[2 * p]), b = ints_to_bf16(x[2 * p + 1]);
              kf[n][2 * j + p].u = u32x4_t{a.x, a.y, b.x, b.y};
            }
          }
        } else if constexpr (kCodes) {
          // (a page that is none has exponents of another: 0, so that its zeros stay zeros)
          const float ku = unit_of(min((uint32_t)se[16 * n + l16] & named[0][n], 254u));
          const uint32_t ve = *reinterpret_cast<const uint32_t *>(se + 16 * NT + 16 * n + 4 * g) & named[0][n];
#pragma unroll
          for (int e = 0; e < 4; ++e)  // (2^-127 is a subnormal number)
            vu[n][e] = __uint_as_float(min(max(((ve >> (8 * e)) & 0xffu) << 23, 0x00400000u), 254u << 23));
#pragma unroll
          for (int j = 0; j < KR; ++j) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(sk + 16 * n * ROWB + koff[j]);
#pragma unroll
            for (int p = 0; p < 2; ++p)
              kf[n][2 * j + p].u = u32x4_t{codes_to_bf16<false>(x[2 * p], ku), codes_to_bf16<true>(x[2 * p], ku),
                                           codes_to_bf16<false>(x[2 * p + 1], ku), codes_to_bf16<true>(x[2 * p + 1], ku)};
          }
        } else {
#pragma unroll
          for (int j = 0; j < KS; ++j) kf[n][j].u = *reinterpret_cast<const u32x4_t *>(sk + 16 * n * ROWB + koff[j]);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the fragments are in registers: their buffer is free)
      if constexpr (!kAll) {
        if (((i + 2) & 63) == 0) load_ids(i + 2);
        bring(0, i + 2);
        bring_exps(i + 2, 2);
      }
      f32x4_t x[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        f32x4_t acc = {c0, c0, c0, c0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[n][ks].v, qf[ks].v, acc, 0, 0, 0);
        if constexpr (kInts) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[n][e] = fmaf(acc[e], factor[n], less);
        } else {
          x[n] = acc * scale_log2e;
        }
      }
      if (key < all_lo || key + SK > all_hi) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = key + 16 * n + 4 * g + e;
            if (j < lo || j >= hi) x[n][e] = ninf;
          }
      }
      // ---- the reference moves where a logit exceeds it by more than the slack ------------------
      float m = ninf;
#pragma unroll
      for (int n = 0; n < NT; ++n) m = fmaxf(fmaxf(fmaxf(m, x[n][0]), x[n][1]), fmaxf(x[n][2], x[n][3]));
      const bool first = m_ref == ninf;
      if (__any(m > kSlack || (first && m > ninf))) {
        uint32_t a, b;
        swap_rows16(__float_as_uint(m), a, b);
        m = fmaxf(__uint_as_float(a), __uint_as_float(b));
        swap_halves32(__float_as_uint(m), a, b);
        m = fmaxf(__uint_as_float(a), __uint_as_float(b));
        const bool bump = m > kSlack || (first && m > ninf);
        const float delta = bump ? m : 0.f, m_new = bump ? (first ? 0.f : m_ref) + m : m_ref;
        const float alpha = bump ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.f;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
#pragma unroll
        for (int n = 0; n < NT; ++n) x[n] -= delta;
        m_ref = m_new;
        if constexpr (kInts) less = m_new == ninf ? 0.f : -m_new;
        else c0 = m_new == ninf ? 0.f : -m_new * inv_scale;
      }
      // ---- weights ------------------------------------------------------------------------------
      // (as a sum of two bf16: the weights of few rows can have 16 bits where reading the cache is what takes the time)
      Frag8 pf[(NT + 1) / 2], pl[(NT + 1) / 2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = __builtin_amdgcn_exp2f(x[n][e]);
          l_run += p[e];
          if constexpr (kCodes) p[e] *= vu[n][e];
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const uint32_t w = cvt_pk_bf16(p[e], p[e + 1]);
          pf[n / 2].u[2 * (n & 1) + e / 2] = w;
          pl[n / 2].u[2 * (n & 1) + e / 2] = cvt_pk_bf16(p[e] - bf16lo(w), p[e + 1] - bf16hi(w));
        }
      }
      // ---- O^T ------------------------------------------------------------------------------------
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kAll ? 0 : PER + NLOAD + (kCodes ? 1 : 0)) : "memory");  // V of slice i is there
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
        typedef __attribute__((address_space(3))) i32x2_t lds_i32x2;
        if constexpr (NT > 1) {
#pragma unroll
          for (int kp = 0; kp < NT / 2; ++kp) {
            const unsigned char *at = sv + 32 * kp * ROWB + voff[dt];
            Frag8 a;
            if constexpr (kCodes) {
              const i32x2_t r = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(at));
              if constexpr (kInts) {
                const u32x2_t y0 = ints_to_bf16((uint32_t)r.x), y1 = ints_to_bf16((uint32_t)r.y);
                a.u = u32x4_t{y0.x, y0.y, y1.x, y1.y};
              } else
              a.u = u32x4_t{codes_to_bf16<false>((uint32_t)r.x, 1.f), codes_to_bf16<true>((uint32_t)r.x, 1.f),
                            codes_to_bf16<false>((uint32_t)r.y, 1.f), codes_to_bf16<true>((uint32_t)r.y, 1.f)};
            } else {
              const u32x2_t r = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at)));
              const u32x2_t r2 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 16 * ROWB)));
              a.u = u32x4_t{r.x, r.y, r2.x, r2.y};
            }
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, pl[kp].v, o[dt], 0, 0, 0);
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, pf[kp].v, o[dt], 0, 0, 0);
          }
        } else {
          const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(sv + voff[dt]));
          const u32x2_t b = {pf[0].u[0], pf[0].u[1]}, b2 = {pl[0].u[0], pl[0].u[1]};
          o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, __builtin_bit_cast(s16x4_t, b2), o[dt], 0, 0, 0);
          o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, __builtin_bit_cast(s16x4_t, b), o[dt], 0, 0, 0);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if constexpr (!kAll) bring(1, i + 2);
#pragma unroll
      for (int n = 0; n < NT; ++n) named[0][n] = named[1][n], named[1][n] = named[2][n];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads past the end are still on their way to LDS)
  }

  // ---- the four wavefronts' states put together ---------------------------------------------------
  float *so = reinterpret_cast<float *>(smem);
  static_assert(TILE * D * 4 <= F::WAVE_B, "a wavefront's output fits its part of LDS");
  {
    uint32_t x, y;
    swap_rows16(__float_as_uint(l_run), x, y);
    float l = __uint_as_float(x) + __uint_as_float(y);
    swap_halves32(__float_as_uint(l), x, y);
    l = __uint_as_float(x) + __uint_as_float(y);
    if (g == 0) {
      s_ref[wave][l16] = m_ref;
      s_sum[wave][l16] = l;
    }
  }
  // (16-byte chunk c of row r at c ^ (r % 16))
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    *reinterpret_cast<f32x4_t *>(so + (size_t)wave * (F::WAVE_B / 4) + l16 * D + (((4 * dt + g) ^ l16) * 4)) = o[dt];
  __syncthreads();
  constexpr int CH = D / 8;  // threads of a row, 8 elements each
  auto write_row = [&](int r, int ch, f32x4_t y0, f32x4_t y1, float ref, float l) __attribute__((always_inline)) {
    const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN stays one, in the log-sum-exp too)
    const Row at = at0.row(head, r);
    *reinterpret_cast<u32x4_t *>(c.out + at.token * c.ot + at.head * c.oh + 8 * ch) =
        u32x4_t{cvt_pk_bf16(y0[0] * inv, y0[1] * inv), cvt_pk_bf16(y0[2] * inv, y0[3] * inv),
                cvt_pk_bf16(y1[0] * inv, y1[1] * inv), cvt_pk_bf16(y1[2] * inv, y1[3] * inv)};
    if (c.lse && ch == 0)
      c.lse[(long long)at.head * c.s.T + at.token] = l == 0.f ? ninf : (ref + log2f(l)) * 0.6931471805599453f;
  };
  constexpr int kAgent = 16;  // (sc1: past the L2 of this XCD, where the workgroups of all XCDs meet)
  auto part_rsrc = [&](int slot) __attribute__((always_inline)) -> __amdgpu_buffer_rsrc_t {
    return __builtin_amdgcn_make_buffer_rsrc(c.part + (size_t)slot * kFewPart<D>, 0, (int)(kFewPart<D> * sizeof(float)), 0x00020000);
  };
  for (int i = t; i < n_rows * CH; i += 64 * WAVES) {
    const int r = i / CH, ch = i % CH;
    float ref = ninf;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) ref = fmaxf(ref, s_ref[w][r]);
    const float fin = ref == ninf ? 0.f : ref;
    float l = 0.f;
    f32x4_t y0 = {0.f, 0.f, 0.f, 0.f}, y1 = y0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_ref[w][r] - fin);
      const float *src = so + (size_t)w * (F::WAVE_B / 4) + r * D;
      l = fmaf(s_sum[w][r], f, l);
      y0 += *reinterpret_cast<const f32x4_t *>(src + (((2 * ch) ^ (r & 15)) * 4)) * f;
      y1 += *reinterpret_cast<const f32x4_t *>(src + (((2 * ch + 1) ^ (r & 15)) * 4)) * f;
    }
    if (partial) {
      const __amdgpu_buffer_rsrc_t dst = part_rsrc(2 * share + (x0 == 0));
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, y0), dst, (uint32_t)(r * D + 8 * ch) * 4u, 0, kAgent);
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, y1), dst, (uint32_t)(r * D + 8 * ch + 4) * 4u, 0, kAgent);
      if (ch == 0) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(ref), dst, (uint32_t)(TILE * D + r) * 4u, 0, kAgent);
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(l), dst, (uint32_t)(TILE * D + TILE + r) * 4u, 0, kAgent);
      }
    } else {
      write_row(r, ch, y0, y1, ref, l);
    }
  }
  if constexpr (kSplit) if (partial) {
    // ---- the parts of a divided tile are added up by the workgroup that finds all of them there --------
    if (!sh.part_log) sh.cut_parts(tile0, len, first_part, parts);
    const int k0 = __builtin_amdgcn_readfirstlane(first_part);
    parts = __builtin_amdgcn_readfirstlane(parts);
    // (a share leaves two parts at most: that of the tile it starts in, and of one that starts in it)
    auto slot = [&](int i) { return 2 * (k0 + i) + (i == 0); };
    auto flag = [&](int i) { return c.flags + slot(i); };
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // the part is there for all XCDs
    if (wave == 0) {
      // A part's flag holds the call's mark, which no other call has, so memory of any contents is one without parts.  Each
      // workgroup sets its own and then looks at all: the last of them to be set sees all.  (Two may see all: both write
      // the same bits.)  Whoever does clears them, so that a captured call can be replayed.
      if (lane == 0) (void)__hip_atomic_exchange(flag(share - k0), c.mark, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      bool all = true;
      for (int i = lane; i < parts; i += 64)
        all = all && __hip_atomic_load(flag(i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == c.mark;
      all = __all(all);
      if (all)
        for (int i = lane; i < parts; i += 64) __hip_atomic_store(flag(i), 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (lane == 0) s_all = all;
    }
    __syncthreads();
    if (s_all) {
      // rows' parts are dealt out to groups of D/8 threads (few rows have many parts), whose sums meet in LDS
      constexpr int NG = 256 / CH;
      const __amdgpu_buffer_rsrc_t all_parts =
          __builtin_amdgcn_make_buffer_rsrc(c.part, 0, (int)(2u * gridDim.x * (uint32_t)(kFewPart<D> * sizeof(float))), 0x00020000);
      float(*g_o)[D] = reinterpret_cast<float(*)[D]>(smem);
      float *g_ref = reinterpret_cast<float *>(smem) + NG * D, *g_sum = g_ref + NG;
      const int grp = t / CH, ch = t % CH;
      // groups of a row: as many as there are, MP parts a group at least
      constexpr int MP = 4;
      const int gp = max(min(NG / n_rows, (parts + MP - 1) / MP), 1), r = grp / gp, p0 = grp % gp;
      static_assert(kFewTile <= NG, "a group a row at least");
      const bool mine = r < n_rows;
      float ref = ninf, l = 0.f;
      f32x4_t y0 = {0.f, 0.f, 0.f, 0.f}, y1 = y0;
      if (mine)
        for (int p = p0; p < parts; p += MP * gp) {
          float ms[MP], ls[MP];
          f32x4_t u[MP], v[MP];
#pragma unroll
          for (int i = 0; i < MP; ++i) {
            const uint32_t at = (uint32_t)slot(min(p + i * gp, parts - 1)) * (uint32_t)(kFewPart<D> * sizeof(float));
            ms[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(all_parts, at + (uint32_t)(TILE * D + r) * 4u, 0, kAgent));
            ls[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(all_parts, at + (uint32_t)(TILE * D + TILE + r) * 4u, 0, kAgent));
            u[i] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(all_parts, at + (uint32_t)(r * D + 8 * ch) * 4u, 0, kAgent));
            v[i] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(all_parts, at + (uint32_t)(r * D + 8 * ch + 4) * 4u, 0, kAgent));
          }
          const float old = ref;
#pragma unroll
          for (int i = 0; i < MP; ++i)
            if (p + i * gp < parts) ref = fmaxf(ref, ms[i]);
          const float fin = ref == ninf ? 0.f : ref;
          const float alpha = __builtin_amdgcn_exp2f(old - fin);
          l *= alpha;
          y0 *= alpha;
          y1 *= alpha;
#pragma unroll
          for (int i = 0; i < MP; ++i) {
            if (p + i * gp >= parts) continue;
            const float w = __builtin_amdgcn_exp2f(ms[i] - fin);
            l = fmaf(ls[i], w, l);
            y0 += u[i] * w;
            y1 += v[i] * w;
          }
        }
      if (gp == 1) {
        if (mine) write_row(r, ch, y0, y1, ref, l);
      } else {
        *reinterpret_cast<f32x4_t *>(&g_o[grp][8 * ch]) = y0;
        *reinterpret_cast<f32x4_t *>(&g_o[grp][8 * ch + 4]) = y1;
        if (ch == 0) {
          g_ref[grp] = ref;
          g_sum[grp] = l;
        }
        __syncthreads();
        if (mine && p0 == 0) {
          ref = ninf;
          for (int i = 0; i < gp; ++i) ref = fmaxf(ref, g_ref[grp + i]);
          const float fin = ref == ninf ? 0.f : ref;
          l = 0.f;
          y0 = y1 = f32x4_t{0.f, 0.f, 0.f, 0.f};
          for (int i = 0; i < gp; ++i) {
            const float w = __builtin_amdgcn_exp2f(g_ref[grp + i] - fin);
            l = fmaf(g_sum[grp + i], w, l);
            y0 += *reinterpret_cast<const f32x4_t *>(&g_o[grp + i][8 * ch]) * w;
            y1 += *reinterpret_cast<const f32x4_t *>(&g_o[grp + i][8 * ch + 4]) * w;
          }
          write_row(r, ch, y0, y1, ref, l);
        }
      }
    }
  }
  if constexpr (kSplit) __syncthreads();  // (the LDS is free for the next tile)
  }
  if (!kSplit || sh.part_log) return;
  tile0 += 2 * len + 512 / ROWB;
  if (tile0 >= cut1) return;
  if (++number >= n_seq) {
    // the next sequence that has tiles
    bool found = false;
#pragma unroll
    for (int j = 0; j < Sh::NB; ++j)
      if (j * 64 < c.s.B && !found) {
        const unsigned long long here = __ballot(sh.tiles[j] > 0 && sh.before[j] == tile0);
        if (here) {
          enter(j, __ffsll((long long)here) - 1);
          found = true;
        }
      }
  }
  }
}

// Rows a sequence and key head, on average (all that is known of them here), that this kernel is for: those of one tile.  us, where all
// sequences of a call are alike, of this kernel and of the one for
// tiles of 128 rows (cache_attn.hip): 16 rows: one sequence of 2000 keys, two heads 12.6 / 16.1, of 30000, eight heads 44.6 / 47.7, 16 of
// 4000 48.9 / 51.8, in e4m3 31.4 / 39.4, 64 of 1000 44.8 / 43.3, in e4m3 27.2 / 31.6; 24 rows (two tiles): 18 to 35 % slower
// than that where one sequence is divided, 5 % faster to 9 % slower in batches.
bool cache_attn_few(int B, int H, int T, int Hq) { return (long long)T * (Hq / H) <= (long long)kFewTile * B; }
// The same where tiles have little to read, of int8 (keys: what the page tables have room for, as lengths are not known here; one that has
// room for more than these goes to the other kernel however short its sequences are): tiles at most (512 are one round of places), their
// keys together, and of one.  us of this kernel and of the other, D = 128: 24 rows, 8 heads of 1000 keys 12.6 / 18.8, of
// 4000 17.1 / 20.4, 16 sequences 23.1 / 28.9 and 53.8 / 46.3; 64 rows, 8 heads of 300 keys 12.4 / 15.9, of 4000 20.7 / 20.8, 16 sequences
// 18.0 / 25.3 and 91.9 / 54.8; 64 sequences, 24 rows, 300 keys 25.6 / 21.1; 64 rows, two heads of 16000 keys 35.5 / 28.4; 256 rows, 8 heads
// of 300 keys 8.8 / 17.0, of 1500 20.1 / 22.5; 500 rows, 8 heads of 700 keys 17.4 / 21.1.  Around 640 tiles: 26 sequences of 32 rows, 8 heads (624) of 100 keys
// 9.6 / 17.4, of 500 18.8 / 29.4; 500 rows, 500 keys, 16 heads (512) 16.0 / 22.3, 20 heads (640) 28.5 / 25.3.
constexpr long long kIntTiles = 640, kIntKeys = 5 << 16, kIntLongest = 4096;
bool cache_attn_int8_few(const heart_cache &c, int T, int Hq) {
  if (cache_attn_few(c.B, c.H, T, Hq)) return true;
  const long long tiles = most_items(kFewTile, c.B, c.H, T, Hq), room = (long long)c.max_pages * c.page;
  return (long long)T * (Hq / c.H) <= (long long)kIntRows * c.B && tiles <= kIntTiles && room <= kIntLongest && tiles * room <= kIntKeys;
}
// int8: a workgroup of sixteen wavefronts has a tile, whose keys (by the room of the page tables) are a slice of 4 KB for each at most:
// nothing is divided, so no parts have to meet, and no loop.  One a CU.  us, divided (or four wavefronts) and so: one token of 1000 keys, two
// heads of 64 11.3 / 8.9 (11.0 under any table with room for more than 1024), 16 sequences of 64 keys, 8 heads 8.7 / 6.8, of 1000
// 14.5 / 10.5; 8 rows, 8 heads of 128, 480 keys 11.9 / 8.1; 32 sequences of 200 keys, 8 heads (384 items) 8.7 / 11.1.
constexpr long long kFewAllItems = 256;
static bool few_divides(int B, long long items) { return B <= kSplitSeqs && items <= kFewItems; }

size_t cache_attn_few_workspace_bytes(int B, int H, int D, int T, int Hq) {
  if (!few_divides(B, most_items(kFewTile, B, H, T, Hq))) return 0;
  return 2 * (size_t)kFewPlaces * (sizeof(unsigned long long) + (size_t)(kFewTile * (D + 2)) * sizeof(float));
}

template <int D, CacheKind kKind>
static int launch_few_t(const AttnCall &c, bool split, bool all, long long grid, hipStream_t st) {
  const int dev = current_device();
  if (dev < 0) return fail(HEART_EHIP, "heart_cache_attn: cannot identify the current device");
  auto run_waves = [&](auto seqs, auto waves) -> int {
    constexpr int W = decltype(waves)::value, bytes = W * FewShape<D, kKind, W>::WAVE_B;
    static_assert(bytes >= (256 / (D / 8)) * (D + 2) * 4, "sums of the parts fit the LDS");
    auto kern = cache_attn_few_kernel<D, kKind, decltype(seqs)::value, W>;
    static DeviceFlags attr_set;  // per instantiation: the attribute is per function and device
    if (hipError_t e = set_max_lds_once(attr_set, dev, reinterpret_cast<const void *>(kern), bytes))
      return fail(HEART_EHIP, "hipFuncSetAttribute(max dynamic LDS %d): %s", bytes, hipGetErrorString(e));
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(64 * W), bytes, st, c);
    return check_launch("cache_attn_few_kernel");
  };
  if constexpr (kKind == kInt8)
    if (all) return run_waves(std::integral_constant<int, 0>{}, std::integral_constant<int, kFewAll>{});
  auto run = [&](auto seqs) -> int { return run_waves(seqs, std::integral_constant<int, kFewWaves>{}); };
  if (!split) return run(std::integral_constant<int, 0>{});
  return c.s.B <= 64 ? run(std::integral_constant<int, 1>{}) : run(std::integral_constant<int, kSplitSeqs / 64>{});
}

int launch_cache_attn_few(const heart_cache &hc, int T, int Hq, AttnCall &a, void *workspace, hipStream_t st) {
  const long long items = most_items(kFewTile, hc.B, hc.H, T, Hq);
  if (items > kMostGroups) return fail(HEART_EUNSUPPORTED, "heart_cache_attn: grid too large");
  const long long stages = ((long long)a.s.cap + kFewStage - 1) / kFewStage;
  const bool split = workspace && few_divides(hc.B, items) && stages <= (1ll << 27) / items;  // (sums of lengths fit 32 bits)
  const bool all = hc.type == HEART_CACHE_INT8 && a.s.cap <= kFewAll * (4096 / hc.D) && items <= kFewAllItems;
  long long grid = items;
  if (split && !all) {
    const long long most = items * ((stages + kFewMin - 1) / kFewMin);  // parts at most
    grid = most < kFewPlaces ? most : kFewPlaces;
    a.flags = (unsigned long long *)workspace;
    a.part = (float *)(a.flags + 2 * kFewPlaces);
    a.mark = call_mark();
  }
  auto of_kind = [&](auto d) -> int {
    constexpr int D = decltype(d)::value;
    if (hc.type == HEART_CACHE_INT8) return launch_few_t<D, kInt8>(a, split, all, grid, st);
    return hc.type == HEART_CACHE_E4M3 ? launch_few_t<D, kE4m3>(a, split, false, grid, st) : launch_few_t<D, kBf16>(a, split, false, grid, st);
  };
  return hc.D == 128 ? of_kind(std::integral_constant<int, 128>{}) : of_kind(std::integral_constant<int, 64>{});
}

}  // namespace heart
