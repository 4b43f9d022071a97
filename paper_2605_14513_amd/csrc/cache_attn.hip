// heart_cache_attn: softmax attention of a chunk of new tokens over the paged key/value cache.
//
// Work.  The queries that share a key head (G query heads of each new token of a sequence) are rows of one product: row
// r of sequence b and key head h is token r / G, query head h G + r % G.  A workgroup has a tile of 128 rows
// (some of int8 256), a wavefront 32 of them, and walks through the keys in stages of 64.
//
// Tiles are computed transposed, as in the block-sparse kernel, so that no accumulator moves between lanes:
//   S^T (keys x rows) = K . Q^T,   O^T (d x rows) += V^T . P^T     with v_mfma_f32_32x32x16_bf16
// A lane holds one row (lane % 32) and 16 of 32 keys (8 (r/4) + 4 (lane/32) + r % 4): the softmax state of a row is a scalar
// of two lanes, and the exponentiated accumulator is, as it is, the B operand of the second product.
//
// One pass with a running reference exponent, which moves only when a logit exceeds it by more than 2^8, and a running
// sum.  Weights are rounded to bf16 for the second product (error against 64 bits 0.0018 to 0.0020 in the 2-norm, 0.0016 of it
// the rounding of the output): a sum of two bf16, as few rows have, would be half as many matrix instructions again where
// these set the time.  The row sum adds the weights unrounded.
// The accumulators of S^T start from minus that reference.  K of slice s + 1 and V of slice s (32 keys) are worked
// on in turn: B(s) multiplies K while the VALU exponentiates slice s, C(s) multiplies V while it folds the
// maximum of slice s + 1.
//
// Stages.  K stage i holds slices 2i, 2i + 1; V stage i slices 2i - 1, 2i, so that one barrier per 64 keys retires both. Each
// of the four wavefronts brings 16 rows of a stage (of eight 8), and pages hold a multiple of 16 tokens, so a wavefront needs one
// page for a stage: a buffer descriptor over the rows that are there (rows that no query of the tile sees, from kv_len on
// in any case, and pages that the table does not name, are out of its range and arrive as zeros).  The page ids of 64
// stages lie in one register, a lane each.
//   bf16: LDS-direct loads, double-buffered, two slices ahead.
//   e4m3: the codes are loaded into registers a stage earlier still and written to LDS as the bf16 values that they
//     stand for, once for all wavefronts; converting at each fragment read would be four times the work, more VALU
//     time than the products take.
//   int8: the same, as f16, which a code becomes in one instruction (bf16 would take one and a half), with f16 products: K as the codes
//     are, its scales, of 16 rows each, as factors of the logits; V times its scale (of 11 bits; exact for those that are written
//     here) by a power of two of the part, half an instruction more; Q by its
//     row's power of two.  Weights in f16 have 11 bits, and the largest of a row is 2^7 at least, which keeps small ones from f16's
//     least.  Eight wavefronts share a stage's conversion where tiles of 256 rows fill the chip (wide_tiles).
//
// Bound by the matrix instructions and the power that they draw.  PFLOP/s: 4680 queries of 12 heads over 32760 keys in bf16
// 1.03 to 1.07 (matrix pipes busy 59 % of the cycles), of 40 heads in e4m3 0.99 to 1.04 (53 %: the conversions); a bf16 matrix
// product of 8192^3 1.20; of 40 heads in int8 0.97 to 1.06 (53 %; tiles of 128 rows 0.91 to 0.95; D = 64, always of 128 rows, 0.79, where bf16
// has 0.87).  Boxes differ by a tenth: on one box, in turn, bf16 1.10 to 1.14, e4m3 1.06, int8 1.05.  Calls of few tiles are bound by
// latency: 16 sequences with 8 drafts of 24 heads, window 4096, 21 us.
#include <type_traits>

#include "cache_attn_device.h"

namespace heart {

constexpr int kTile = 128;      // rows of a workgroup
constexpr int kStage = 64;      // keys of a stage
constexpr int kPlaces = 512;    // places for workgroups: two a CU
constexpr int kMinStages = 4;   // fewest stages of a part (8 queries of 32000 keys, 3 key heads: 28 us, 31 with 2 or 3)
constexpr int kPartCost = 8;    // what a part costs beside its stages (launch, first loads, 64 KB written and read), in stages

// floats of one wavefront's part: accumulators, reference exponent and row sum of every lane
template <int D>
constexpr int kPartFloats = 64 * (D / 2) + 128;

// (divided keys) The part of workgroup w: the sequences' parts one after the other; of a sequence, head after head, parts,
// tiles, so that workgroups that read the same keys are neighbours.  Parts have at most L stages, the least L with which
// there are no more parts than places, or than twice the places where that ends sooner (300 tiles of one length: two rounds
// of thirds, not one round of wholes in 300 of 512 places): found from the lengths by every wavefront on its own.
// (NB: sequences a lane.  One where that is enough: code that is jumped over has to be fetched all the same.)
template <int NB>
__device__ __forceinline__ bool find_part(const AttnCall &c, int w_xcd, int w_slot, int lane, Work &k) {
  int wgs[NB], st[NB];  // tiles of all heads, stages of a tile
  int most = 1, tiles = 0;
  float all = 0.f;
  bool falls = false;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int b = j * 64 + lane;
    wgs[j] = 0;
    st[j] = 1;
    if (j * 64 < c.s.B && b < c.s.B) {
      const Seq s = seq_of(c, b);
      falls = falls || (c.s.cu && c.s.cu[b + 1] < c.s.cu[b]);
      wgs[j] = tiles_of<kTile>(c, s) * c.H;
      st[j] = stages_of<kTile, kStage>(c, s);
      most = max(most, wgs[j] ? st[j] : 1);
      tiles += wgs[j];
      all += (float)wgs[j] * (float)st[j];
    }
  }
  // Token ranges that fall somewhere overlap: there can be more tiles than places, and records that nobody writes, though the merge
  // finds their tiles.  No work then, and records of no parts for all tiles that the merge can find (fewer than kPlaces).
  if (__any(falls)) {
    const int i = w_slot * kNumXcd + w_xcd;
    if (i < kPlaces && threadIdx.x == 0) c.items[i] = int4{0, 0, 0, 0};
    return false;
  }
  most = __builtin_amdgcn_readfirstlane((int)wave_max_u32((uint32_t)most));
  tiles = __builtin_amdgcn_readfirstlane(wave_sum_i32(tiles));
  all = wave_sum_f32(all);
  // parts of a tile: st / L rounded up, or, by the rounding of the quotient, one more or less of many
  auto parts_of = [&](int j, float inv) -> int { return (int)fmaf((float)(st[j] - 1), inv, 1.f); };
  auto count = [&](int L) -> int {
    const float inv = __builtin_amdgcn_rcpf((float)L);
    int n = 0;
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (j * 64 < c.s.B) n += wgs[j] * parts_of(j, inv);
    return __builtin_amdgcn_readfirstlane(wave_sum_i32(n));
  };
  // the least L with at most `places` parts, which are between all / L and all / L + tiles
  auto least = [&](int places) -> int {
    const int up = __builtin_amdgcn_readfirstlane((int)(all / (float)places));
    const int room = places - tiles;
    int lo = min(max(up, kMinStages), most);
    int hi = room > 0 ? min(__builtin_amdgcn_readfirstlane((int)(all / (float)room)) + 2, most) : most;
    hi = max(hi, lo);
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (count(mid) <= places) hi = mid;
      else lo = mid + 1;
    }
    return lo;
  };
  int L = least(kPlaces), total = count(L), room = kPlaces;
  if (c.rounds > 1 && L > kPartCost) {
    const int two = least(2 * kPlaces);
    if (2 * two + kPartCost < L) L = two, total = count(L), room = 2 * kPlaces;
  }
  // (one part each: the quotients' rounding let a part too many through)
  if (total > room) L = 0x3fffffff, total = count(L);
  // XCD x has the x-th eighth of the parts
  const int w = w_xcd * total / kNumXcd + w_slot;
  if (w >= (w_xcd + 1) * total / kNumXcd) return false;
  const float inv = __builtin_amdgcn_rcpf((float)L);
  int at = 0;
#pragma unroll
  for (int j = 0; j < NB; ++j)
    if (j * 64 < c.s.B) {
      const int parts = parts_of(j, inv), n = wgs[j] * parts;
      const int end = at + wave_scan_i32(n), start = end - n;
      const unsigned long long here = __ballot(start <= w && w < end);
      if (here) {
        const int l = __ffsll((long long)here) - 1;
        k.b = j * 64 + l;
        k.parts = __builtin_amdgcn_readlane(parts, l);
        k.step = (int)((unsigned)__builtin_amdgcn_readlane(wgs[j], l) / (unsigned)c.H);  // tiles
        const unsigned r = (unsigned)(w - __builtin_amdgcn_readlane(start, l)), q = k.step == 1 ? r : r / (unsigned)k.step;
        k.m = (int)(r - q * (unsigned)k.step);
        k.h = (int)(q / (unsigned)k.parts);
        k.part = (int)q - k.h * k.parts;
      }
      at = __builtin_amdgcn_readlane(end, 63);
    }
  k.slot = w;
  return true;
}

// kWhole: a workgroup per tile.  kParts: find_part.  kTail: the tiles of a last round that would not fill the places are
// divided, c.tail parts each.
enum CacheMode { kWhole, kParts, kPartsWide, kTail };  // (kPartsWide: of more than 64 sequences)
// Tile and key head of item i, of n_items = tiles H.  Where there are eight heads or a multiple, an XCD (workgroups are dealt to
// them in turn) has every eighth head, one after the other, so that its workgroups find each other's keys in its L2 (40 heads
// of 32760 keys in e4m3: 3000 to 3090 us, 3100 to 3130 with all heads at once).
__device__ __forceinline__ void item_at(const AttnCall &c, int i, int n_items, int &tile, int &h) {
  if (c.H % kNumXcd == 0) {
    const int n = (int)((unsigned)n_items / (unsigned)c.H), s = i / kNumXcd;
    h = s / n * kNumXcd + i % kNumXcd;
    tile = s % n;
  } else {
    tile = (int)((unsigned)i / (unsigned)c.H);
    h = i - tile * c.H;
  }
}

// (int8) Codes in a quarter of the bytes of w as f16, exactly: with the sign bit turned, the byte below 0x64 is 1024 + 128 + code.
// Two of them, from byte 2 kUpper on; less 1152 they are the codes, before anything multiplies them: 1152 times a scale has no room
// in f16 for scales of more than 7 significant bits, and what it lost would be added to all elements of a page alike.
template <bool kUpper>
__device__ __forceinline__ f16x2_t codes_up(uint32_t turned) {
  return __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, turned, kUpper ? 0x04030402u : 0x04010400u));
}

template <int D, CacheKind kKind, CacheMode kMode, int WAVES = kTile / 32>
__global__ __launch_bounds__(64 * WAVES, 2) void cache_attn_kernel(const AttnCall c) {
  constexpr int TILE = 32 * WAVES, THREADS = 64 * WAVES, ROWS = kStage / WAVES;  // rows of a tile, rows that a wavefront brings of a stage
  static_assert(WAVES == 4 || (kKind == kInt8 && (kMode == kWhole || kMode == kTail)), "wide tiles: of int8, those of a last round divided");
  constexpr bool kCodes = kKind != kBf16, kInts = kKind == kInt8;
  constexpr int DT = D / 32;             // 32-wide d tiles of the output
  constexpr int KS = D / 16;             // k-steps of the first product
  constexpr int CPR = D / 8;             // 16-byte chunks of a row in LDS
  constexpr int ROWB = D * 2;            // bytes of a row in LDS
  constexpr int RPB = 16 / CPR;          // rows per 256 bytes (one pass over the 64 banks)
  constexpr int TILE_B = kStage * ROWB;  // bytes of a stage of K or V
  constexpr int RPI = 64 / CPR;          // rows that an LDS-direct load covers
  constexpr int IPW = ROWS / RPI;          // such loads per wavefront and stage
  constexpr int LPC = D / 16;            // (codes) lanes that hold a row, 16 codes each
  constexpr int RPC = 64 / LPC;          // rows of one load
  constexpr int CPW = ROWS / RPC;          // loads per wavefront and stage
  constexpr int SO = D + 8;              // LDS row stride of the output staging (elements)
  // weights are at most 2^(kTop + 8), and the largest of a row is 2^kTop at least
  constexpr float kTop = kInts ? 7.f : 0.f, kRescaleSlack = kTop + 8.f;
  constexpr float ninf = -__builtin_inff();
  const float scale_log2e = c.scale_log2e, kInitScale = 1.f / scale_log2e;

  // LDS: [K stage 0][K stage 1][V stage 0][V stage 1], reused for the output at the end
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ __align__(16) float s_unit[kInts ? 2 : 1][4];  // (int8) scales of a K stage's rows, 16 each
  __shared__ uint32_t s_top[WAVES];                             // (int8) V's largest scale
  const uint32_t smem_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;

  const int t = threadIdx.x;
  const int lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int l32 = lane & 31, hf = lane >> 5;

  // ---- what to work on ---------------------------------------------------------------------
  Work wk{0, 0, 0, 0, 1, 1, 0};
  constexpr bool kSplit = kMode != kWhole;
  int rec = 0;  // (divided keys) where to note the tile's parts
  constexpr bool kInParts = kMode == kParts || kMode == kPartsWide;
  if constexpr (kInParts) {
    if (!find_part<kMode == kParts ? 1 : kSplitSeqs / 64>(c, (int)(blockIdx.x % kNumXcd), (int)(blockIdx.x / kNumXcd), lane, wk))
      return;
  } else {
    int i = (int)blockIdx.x, tile;
    if constexpr (kMode == kTail) {
      // (of the divided tiles: part after part, so that workgroups that read the same keys are neighbours)
      const int n_tail = c.n_items - c.whole, j = i - c.whole;
      if (j >= 0) {
        wk.part = j / n_tail;
        rec = j - wk.part * n_tail;
        i = c.whole + rec;
        wk.parts = c.tail;
        wk.step = n_tail;
        wk.slot = j;
      }
    }
    item_at(c, i, c.n_items, tile, wk.h);
    wk.b = seq_of_tile<TILE>(c, tile, lane);
    wk.m = tile - tile_start<TILE>(c, wk.b);
  }
  wk.b = __builtin_amdgcn_readfirstlane(wk.b);
  wk.m = __builtin_amdgcn_readfirstlane(wk.m);
  const Seq s = seq_of(c, wk.b);
  const int tiles = tiles_of<TILE>(c, s);
  if (wk.m < 0 || wk.m >= tiles) return;
  if constexpr (kInParts) rec = (tile_start<TILE>(c, wk.b) + wk.m) * c.H + wk.h;
  else wk.m = tiles - 1 - wk.m;  // (later tiles see more keys: first)
  const int rows = s.n * c.G, r0 = wk.m * TILE;
  int lo, hi, first_key, end_key, ignore;
  seen_by(c, s, s.pos0 + r0 / c.G, first_key, ignore);
  seen_by(c, s, s.pos0 + min(r0 + TILE - 1, rows - 1) / c.G, ignore, end_key);
  const int tile_end = __builtin_amdgcn_readfirstlane(end_key);  // keys from here on no row of the tile sees: zeros
  int stage0 = first_key / kStage, n_stage = max((end_key + kStage - 1) / kStage - stage0, 0);
  int parts = 1;
  if constexpr (kSplit) {
    const int per = max((n_stage + wk.parts - 1) / wk.parts, kMode == kTail ? 2 * kPartCost : 1);
    parts = max((n_stage + per - 1) / per, 1);
    if (wk.part == 0 && t == 0 && (kInParts || wk.parts > 1)) c.items[rec] = int4{wk.slot, parts, wk.step, 0};
    if (wk.part >= parts) return;
    stage0 += wk.part * per;
    n_stage = min(per, n_stage - wk.part * per);
    end_key = min(end_key, (stage0 + n_stage) * kStage);
  }
  stage0 = __builtin_amdgcn_readfirstlane(stage0);
  n_stage = __builtin_amdgcn_readfirstlane(n_stage);
  end_key = __builtin_amdgcn_readfirstlane(end_key);
  const int key0 = stage0 * kStage;
  const int row = r0 + wave * 32 + l32;
  const bool active = r0 + wave * 32 < rows;  // (of the wavefront)

  // keys that this lane's row sees among those of this part; rows past the end see what is there
  seen_by(c, s, s.pos0 + min(row, rows - 1) / c.G, lo, hi);
  if (row >= rows) lo = 0, hi = end_key;
  hi = min(hi, end_key);
  // slices from all_lo on and before all_hi need no mask
  const int all_lo = __builtin_amdgcn_readfirstlane((int)wave_max_u32((uint32_t)lo));
  const int all_hi = __builtin_amdgcn_readfirstlane((int)wave_min_u32((uint32_t)hi));

  // ---- per-lane constants of the LDS layout ---------------------------------------------
  // Chunk c (16 bytes) of stage row r is stored at chunk position c ^ f(r):
  //   K: f(r) = (r / RPB) % CPR            -- the 16 rows that a quarter-wave reads at one chunk fall
  //                                           into 16 distinct 4-bank groups
  //   V: f(r) = 4 * ((r / RPB) % (CPR/4))  -- so do the 4 rows x 4 chunks of a transposing read
  auto swizzle = [](int is_v, int r) { return is_v ? 4 * ((r / RPB) % (CPR / 4)) : (r / RPB) % CPR; };
  // K fragment of k-step ks: row l32 of the slice, chunk 2 ks + hf
  uint32_t koff[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) koff[ks] = (uint32_t)(l32 * ROWB + (((2 * ks + hf) ^ swizzle(0, l32)) * 16));
  // V^T fragment through ds_read_b64_tr_b16: in 16 lanes, lane s names 4 consecutive d of one key (key s / 4, d chunk
  // s % 4) and lane i receives d = i of keys 0..3.  A fragment is keys 16 s2 + 4 hf + 0..3 and 16 s2 + 8 + 4 hf + 0..3 of
  // the slice, the order in which the accumulator of S^T holds them.
  uint32_t voff[DT];
  {
    const int s16 = lane & 15, g16 = (lane >> 4) & 1;
    const int rowv = 4 * hf + (s16 >> 2);
    const int fv4 = swizzle(1, rowv) / 4;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      voff[dt] = (uint32_t)(rowv * ROWB + ((4 * (dt ^ fv4) + 2 * g16 + ((s16 & 3) >> 1)) * 16) + (s16 & 1) * 8);
  }

  // ---- bringing K and V ----------------------------------------------------------------------
  // The wavefront's ROWS rows of stage i (of this part) are keys key0 + 64 i + ROWS wave .. of K, 32 before that of V.
  // Page ids of stages base .. base + 63, lane l that of stage base + l.
  int ids[2];
  float units[2];  // (int8) their scales
  auto load_ids = [&](int base) __attribute__((always_inline)) {
#pragma unroll
    for (int is_v = 0; is_v < 2; ++is_v) {
      const int key = key0 + (base + lane) * kStage - 32 * is_v + ROWS * wave;
      ids[is_v] = -1;
      if (base + lane <= n_stage && key >= 0 && key < tile_end) ids[is_v] = cache_page(c.s, wk.b, key);
      if constexpr (kInts) {
        const float u = reinterpret_cast<const float *>(is_v ? c.v.exp : c.k.exp)[(long long)max(ids[is_v], 0) * c.H + wk.h];
        units[is_v] = ids[is_v] < 0 ? 0.f : u;
      }
    }
  };
  const int in_page = (1 << c.s.page_shift) - 1;
  // rows that are there of the wavefront's ROWS of a stage, the address of the first one's element 0 and exponent
  auto rows_at = [&](int is_v, int i, uint64_t &addr, uint64_t &exp_addr) __attribute__((always_inline)) -> int {
    const CacheTensor &x = is_v ? c.v : c.k;
    const int key = key0 + i * kStage - 32 * is_v + ROWS * wave;
    const int id = __builtin_amdgcn_readlane(ids[is_v], i & 63);
    const int off = key & in_page;
    addr = (uint64_t)(x.p + max(id, 0) * x.page + wk.h * x.head + off * (long long)x.row);
    if constexpr (kKind == kE4m3) exp_addr = (uint64_t)(x.exp + ((((long long)max(id, 0) * c.H + wk.h) << c.s.page_shift) + off));
    return id < 0 ? 0 : min(tile_end - key, ROWS);
  };
  // LDS-direct loads (bf16): one instruction moves 16 bytes per lane to 1 KB of consecutive LDS; lane l lands at chunk
  // position l % CPR of row l / CPR and therefore fetches chunk (l % CPR) ^ f(row).
  uint32_t dma_off[2][kCodes ? 1 : IPW];
  if constexpr (!kCodes) {
#pragma unroll
    for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
      for (int ii = 0; ii < IPW; ++ii) {
        const int r = ii * RPI + lane / CPR;
        dma_off[is_v][ii] = (uint32_t)r * (is_v ? c.v.row : c.k.row) + (uint32_t)(((lane % CPR) ^ swizzle(is_v, wave * ROWS + r)) * 16);
      }
  }
  u32x4_t dma_rs[2];
  auto dma_begin = [&](int is_v, int i) __attribute__((always_inline)) {
    uint64_t addr, unused = 0;
    const int n = rows_at(is_v, i, addr, unused);
    const uint32_t bytes = n > 0 ? (uint32_t)(n - 1) * (is_v ? c.v.row : c.k.row) + (uint32_t)ROWB : 0u;
    dma_rs[is_v].x = __builtin_amdgcn_readfirstlane((uint32_t)addr);
    dma_rs[is_v].y = __builtin_amdgcn_readfirstlane((uint32_t)(addr >> 32) & 0xffffu);
    dma_rs[is_v].z = __builtin_amdgcn_readfirstlane(bytes);
    dma_rs[is_v].w = 0x00020000u;
  };
  auto dma = [&](int is_v, int ii, int buf) __attribute__((always_inline)) {
    const uint32_t dst = smem_lds + (uint32_t)((2 * is_v + buf) * TILE_B + (wave * IPW + ii) * 1024);
    // (the compiler does not see this instruction's LDS write, so it adds no waits of its own: completion is awaited
    // before the barrier that publishes the stage.  M0 is saved and restored: it may hold a value of the compiler's)
    uint32_t m0_saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                 "buffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0_saved) : "s"(dst), "v"(dma_off[is_v][kCodes ? 0 : ii]), "s"(dma_rs[is_v]) : "memory");
  };
  // codes: a stage in registers, written to LDS as 16-bit values
  u32x4_t raw[2][CPW];
  uint32_t raw_exp[2][CPW];
  float raw_unit[2];  // (int8) of the wavefront's rows
  f16x2_t v_mul;      // (int8) V's scale in units of v_unit, of the stage that is stored
  const int crow = lane / LPC, cchunk = lane % LPC;
  auto load_codes = [&](int is_v, int i) __attribute__((always_inline)) {
    const uint32_t stride = is_v ? c.v.row : c.k.row;
    uint64_t addr, exp_addr = 0;
    const int n = rows_at(is_v, i, addr, exp_addr);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        (void *)addr, 0, n > 0 ? (int)((uint32_t)(n - 1) * stride + (uint32_t)D) : 0, 0x00020000);
    const __amdgpu_buffer_rsrc_t es = __builtin_amdgcn_make_buffer_rsrc((void *)exp_addr, 0, max(n, 0), 0x00020000);
#pragma unroll
    for (int ii = 0; ii < CPW; ++ii) {
      const int r = ii * RPC + crow;
      raw[is_v][ii] = __builtin_amdgcn_raw_buffer_load_b128(rs, (uint32_t)r * stride + (uint32_t)cchunk * 16u, 0, 0);
      if constexpr (kKind == kE4m3) raw_exp[is_v][ii] = __builtin_amdgcn_raw_buffer_load_b8(es, (uint32_t)r, 0, 0);
    }
    // (K's without the sign that a NaN may have, for load_factors)
    if constexpr (kInts)
      raw_unit[is_v] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(__float_as_int(units[is_v]), i & 63) & (is_v ? ~0u : 0x7fffffffu));
  };
  // (int8) V in f16 is in units of a power of two, 2^5 of which are above the largest scale of the part: known where the page ids
  // of its first stages are, of long parts after a look at the others
  float v_unit = 1.f, to_v_unit = 1.f;
  auto find_v_unit = [&]() __attribute__((always_inline)) {
    const uint32_t mine = __float_as_uint(units[1]);
    uint32_t top = mine < 0x7f800000u ? mine : 0u;
    if (n_stage > 63) {
      const float *scales = reinterpret_cast<const float *>(c.v.exp);
#pragma unroll 4
      for (int p = ((key0 + 63 * kStage) >> c.s.page_shift) + t; p <= (end_key - 1) >> c.s.page_shift; p += THREADS) {
        const int id = cache_page(c.s, wk.b, p << c.s.page_shift);
        const uint32_t u = __float_as_uint(scales[(long long)max(id, 0) * c.H + wk.h]);
        top = heart_op_umax(top, id >= 0 && u < 0x7f800000u ? u : 0u);
      }
    }
    top = wave_max_u32(top);
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = heart_op_umax(top, s_top[w]);
    const uint32_t up = heart_op_umin(258u - (top >> 23), 253u);  // 2^(4 - exponent of the largest)
    to_v_unit = __uint_as_float(up << 23);
    v_unit = __uint_as_float((254u - up) << 23);
  };
  auto store_codes = [&](int is_v, int ii, int p, int buf) __attribute__((always_inline)) {
    const int r = wave * ROWS + ii * RPC + crow, f = swizzle(is_v, r);
    unsigned char *dst = smem + (2 * is_v + buf) * TILE_B + r * ROWB;
    const u32x4_t x = raw[is_v][ii];
    if constexpr (kInts) {
      // K as the codes are (its scales go into the logits), V times its scale
      if (is_v && ii == 0 && p == 0) {
        const _Float16 u = (_Float16)(raw_unit[1] * to_v_unit);
        v_mul = f16x2_t{u, u};
      }
      const f16x2_t less = {(_Float16)-1152.f, (_Float16)-1152.f};
      u32x4_t y;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t turned = x[2 * p + w] ^ 0x80808080u;
        const f16x2_t a = codes_up<false>(turned) + less, b = codes_up<true>(turned) + less;
        y[2 * w] = __builtin_bit_cast(uint32_t, is_v ? a * v_mul : a);
        y[2 * w + 1] = __builtin_bit_cast(uint32_t, is_v ? b * v_mul : b);
      }
      *reinterpret_cast<u32x4_t *>(dst + (((2 * cchunk + p) ^ f) * 16)) = y;
      // (where two wavefronts have 16 rows, the first's are there if any are)
      if (!is_v && ii == 0 && p == 0 && wave * ROWS % 16 == 0) s_unit[buf][wave * ROWS / 16] = raw_unit[0];
      return;
    }
    const float unit = unit_of(raw_exp[is_v][ii]);
    const u32x4_t y = {codes_to_bf16<false>(x[2 * p], unit), codes_to_bf16<true>(x[2 * p], unit),
                       codes_to_bf16<false>(x[2 * p + 1], unit), codes_to_bf16<true>(x[2 * p + 1], unit)};
    *reinterpret_cast<u32x4_t *>(dst + (((2 * cchunk + p) ^ f) * 16)) = y;
  };
  // step j of KS of bringing stage i to buffer `buf`; (codes) stage i is in registers, stage i + 1 is loaded behind it
  auto bring = [&](int j, int i, int buf) __attribute__((always_inline)) {
    if constexpr (kCodes) {
#pragma unroll
      for (int hh = 0; hh < 4 * CPW; ++hh)
        if (hh * KS / (4 * CPW) == j) store_codes(hh / (2 * CPW), hh / 2 % CPW, hh % 2, buf);
      if (j == KS / 2 - 1) load_codes(0, i + 1);
      if (j == KS - 1) load_codes(1, i + 1);
    } else {
#pragma unroll
      for (int ii = 0; ii < 2 * IPW; ++ii)
        if (ii * KS / (2 * IPW) == j) {
          if (ii % IPW == 0) dma_begin(ii / IPW, i);
          dma(ii / IPW, ii % IPW, buf);
        }
    }
  };
  auto bring_all = [&](int i, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < KS; ++j) bring(j, i, buf);
  };
  // the page ids of the stages to come, where those of the register end: stage `next` is the next one to be addressed
  auto more_ids = [&](int next) __attribute__((always_inline)) {
    if ((next & 63) == 0) load_ids(next);
  };
  auto publish = [&]() __attribute__((always_inline)) {
    if constexpr (!kCodes) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };

  // ---- state of the rows ----------------------------------------------------------------------
  Frag8 qf[KS];       // Q fragments (B operand of S^T = K Q^T)
  f32x16_t o[DT];     // O^T
  float m_ref = ninf; // reference exponent (log2 domain)
  f32x16_t cinit;     // start of the S^T accumulators: minus the reference, in raw logits
  float l_run = 0.f;  // running sum over this lane's keys, relative to m_ref
  {
    const Row at = row_of(c, s, wk.h, min(row, rows - 1));
    const uint16_t *src = c.q + at.token * c.qt + at.head * c.qh + hf * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks].u = *reinterpret_cast<const u32x4_t *>(src + ks * 16);
  }
  // (int8) Q in f16, with its row's power of two outside: exact but for elements below 2^-31 of the row's largest
  float row_unit = scale_log2e;  // logits in log2 units are this times K's scale times the accumulator
  if constexpr (kInts) {
    uint32_t top = 0, sw0, sw1;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int w = 0; w < 4; ++w)
        top = heart_op_umax(top, heart_op_umax(qf[ks].u[w] & 0x7fffu, (qf[ks].u[w] >> 16) & 0x7fffu));
    swap_halves32(top, sw0, sw1);
    const uint32_t up = heart_op_umin(268u - (heart_op_umax(sw0, sw1) >> 7), 253u);  // 2^(14 - exponent of the largest)
    const float mul = __uint_as_float(up << 23);
    row_unit = __uint_as_float((254u - up) << 23) * scale_log2e;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int w = 0; w < 4; ++w) qf[ks].u[w] = cvt_pk_f16(bf16lo(qf[ks].u[w]) * mul, bf16hi(qf[ks].u[w]) * mul);
  }
  auto mfma = [](const Frag8 &a, const Frag8 &b, const f32x16_t &acc) __attribute__((always_inline)) {
    if constexpr (kInts) return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.h, b.h, acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, acc, 0, 0, 0);
  };
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) cinit[r] = 0.f;

  // ---- the stream of MFMAs -----------------------------------------------------------------
  // Every MFMA takes its A operand from a ring of PF registers that LDS reads fill PF positions ahead, across phases
  // and the loop's end; only the barriers restart the ring.  A loop body is 4 slices, so that buffers are constants.
  constexpr int NPV = 2 * DT;
  constexpr int STEP = KS + NPV;
  constexpr int SEQ = 4 * STEP;
  constexpr int G_B0 = STEP, G_B1 = 3 * STEP;  // positions right after the barriers
  constexpr int PF = 4;
  static_assert(16 % KS == 0 && SEQ % PF == 0 && PF <= KS && PF <= NPV, "stream layout");
  auto fetch = [&](int g) __attribute__((always_inline)) -> u32x4_t {
    g %= SEQ;
    const int n = g / STEP + 1, r = g % STEP;
    const int buf = (n >> 1) & 1, row0 = (n & 1) * 32;
    if (r < KS) return *reinterpret_cast<const u32x4_t *>(smem + buf * TILE_B + row0 * ROWB + koff[r]);
    const int m = r - KS;
    const unsigned char *p = smem + (2 + buf) * TILE_B + (row0 + 16 * (m / DT)) * ROWB + voff[m % DT];
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(p));
    const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(p + 8 * ROWB));
    const u32x2_t x = __builtin_bit_cast(u32x2_t, a), y = __builtin_bit_cast(u32x2_t, b);
    return u32x4_t{x.x, x.y, y.x, y.y};
  };
  Frag8 ring[PF];
  auto prefetch_after = [&](int g) __attribute__((always_inline)) {
    const int t2 = g + PF;
    const bool crosses = (g < G_B0 && t2 >= G_B0) || (g < G_B1 && t2 >= G_B1);
    if (!crosses) ring[t2 % PF].u = fetch(t2);
  };
  auto refill = [&](int g0) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < PF; ++j) ring[(g0 + j) % PF].u = fetch(g0 + j);
  };

  f32x16_t sacc[2];  // S^T of the slice being exponentiated and of the next one
  Frag8 pf[2];       // P^T of the current slice
  // Weights of a slice: 8 pairs of 3 micro-ops that are pinned, a few at a time, behind MFMAs (about 24 cycles of a
  // wavefront's VALU work hide behind one); the row sum adds the unrounded weights.
  float xt0 = 0.f, xt1 = 0.f;
  auto exp_uop = [&](const f32x16_t &x, int u) __attribute__((always_inline)) {
    const int r = 2 * (u / 3), st = u % 3;
    if (st == 0) {
      xt0 = __builtin_amdgcn_exp2f(x[r]);
      asm volatile("" : "+v"(xt0));
    } else if (st == 1) {
      xt1 = __builtin_amdgcn_exp2f(x[r + 1]);
      asm volatile("" : "+v"(xt1));
    } else {
      uint32_t pk = kInts ? cvt_pk_f16(xt0, xt1) : cvt_pk_bf16(xt0, xt1);
      l_run += xt0 + xt1;
      asm volatile("" : "+v"(pk), "+v"(l_run));
      pf[r / 8].u[(r % 8) / 2] = pk;
    }
  };
  constexpr int UB = 16 / KS;  // micro-ops of a B slot
  constexpr int UC = 8 / DT;   // micro-ops of a C slot m < DT
  // (int8) what turns accumulators of the slice of position g into logits relative to the reference: factors of its two
  // groups of 16 keys, and the reference.  (Factors are no smaller than a normal number, so that -inf stays -inf; compared as
  // whole numbers, so that a positive NaN stays one.)
  float factor[2], less = 0.f;
  auto load_factors = [&](int g) __attribute__((always_inline)) {
    if constexpr (kInts) {
      const int n = g / STEP + 1;
      const f32x2_t u = *reinterpret_cast<const f32x2_t *>(&s_unit[(n >> 1) & 1][(n & 1) * 2]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        factor[i] = __int_as_float(max(__float_as_int(u[i] * row_unit), 0x00800000));
      }
    }
  };
  auto to_logit = [&](float x, int r) __attribute__((always_inline)) -> float {
    if constexpr (kInts) return fmaf(x, factor[r / 8], less);
    else return x * scale_log2e;
  };
  auto qk_step = [&](int dst, int g0, auto &&extra) __attribute__((always_inline)) {
    f32x16_t acc;
    const f32x16_t &prev = sacc[dst ^ 1];
    load_factors(g0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      acc = mfma(ring[(g0 + ks) % PF], qf[ks], ks == 0 ? cinit : acc);
      prefetch_after(g0 + ks);
#pragma unroll
      for (int u = 0; u < UB; ++u) exp_uop(prev, ks * UB + u);
      extra(ks);
      __builtin_amdgcn_sched_barrier(0);
    }
    sacc[dst] = acc;
  };
  // logits of keys that the row does not see: none (slice `i` of the part)
  auto mask_slice = [&](f32x16_t &x, int i) __attribute__((always_inline)) {
    const int key = key0 + 32 * i;
    if (key < all_lo || key + 32 > all_hi) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = key + 8 * (r >> 2) + 4 * hf + (r & 3);
        if (j < lo || j >= hi) x[r] = ninf;
      }
    }
  };
  auto max_part = [&](const f32x16_t &x, int i, float m) __attribute__((always_inline)) -> float {
    m = fmaxf(fmaxf(m, x[4 * i]), x[4 * i + 1]);
    return fmaxf(fmaxf(m, x[4 * i + 2]), x[4 * i + 3]);
  };
  // After the maximum of a slice (relative to the reference): the reference moves only where some logit exceeds it by
  // more than the slack.  A slice without visible keys has maximum -inf and moves nothing.
  auto finish_max = [&](float m_rel, f32x16_t &x) __attribute__((always_inline)) {
    const bool first = m_ref == ninf;
    if (__any(m_rel > kRescaleSlack || (first && m_rel > ninf))) {
      uint32_t sw0, sw1;
      swap_halves32(__float_as_uint(m_rel), sw0, sw1);
      m_rel = fmaxf(__uint_as_float(sw0), __uint_as_float(sw1));
      const bool bump = m_rel > kRescaleSlack || (first && m_rel > ninf);
      const float base = first ? 0.f : m_ref;
      const float delta = bump ? m_rel - kTop : 0.f;
      const float m_new = bump ? base + (m_rel - kTop) : m_ref;
      const float alpha = bump ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.f;  // 0 the first time
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] -= delta;
      m_ref = m_new;
      if constexpr (kInts) {
        less = m_ref == ninf ? 0.f : -m_ref;
      } else {
        const float c0 = m_ref == ninf ? 0.f : -m_ref * kInitScale;
#pragma unroll
        for (int r = 0; r < 16; ++r) cinit[r] = c0;
      }
    }
  };
  // O^T += V^T P^T of the slice in sacc[cur]; the second half of the slots scales sacc[cur ^ 1] to log2 units and folds
  // its maximum (the mask, where there is one, follows: finish_slice)
  auto pv_step = [&](int cur, int g0) __attribute__((always_inline)) -> float {
    float m_loc = ninf;
    f32x16_t &nx = sacc[cur ^ 1];
    const f32x16_t &cx = sacc[cur];
#pragma unroll
    for (int m = 0; m < NPV; ++m) {
      o[m % DT] = mfma(ring[(g0 + m) % PF], pf[m / DT], o[m % DT]);
      prefetch_after(g0 + m);
      if (m < DT) {
#pragma unroll
        for (int u = 0; u < UC; ++u) exp_uop(cx, 16 + m * UC + u);
      }
      if (m >= DT) {
#pragma unroll
        for (int i = 0; i < 4 / DT; ++i) {
          const int p = (m - DT) * (4 / DT) + i;
#pragma unroll
          for (int e = 0; e < 4; ++e) nx[4 * p + e] = to_logit(nx[4 * p + e], 4 * p + e);
          m_loc = max_part(nx, p, m_loc);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    return m_loc;
  };
  auto no_extra = [](int) {};

  if (n_stage > 0) {
    // ---- prologue: stages 0 and 1 ------------------------------------------------------------
    load_ids(0);
    if constexpr (kCodes) {
      load_codes(0, 0);
      load_codes(1, 0);
    }
    if constexpr (kInts) find_v_unit();
    bring_all(0, 0);
    bring_all(1, 1);
    publish();
    // pairs of slices st, st + 1; stage st + 2 is brought to the buffer that stage st left
    if (active) {
      {
        f32x16_t acc = cinit;  // zeros: no reference yet
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          Frag8 a;
          a.u = fetch(3 * STEP + ks);  // K of slice 0: buffer 0, rows 0
          acc = mfma(a, qf[ks], acc);
        }
        load_factors(3 * STEP);
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = to_logit(acc[r], r);
        sacc[0] = acc;
        mask_slice(sacc[0], 0);
        float m_loc = ninf;
#pragma unroll
        for (int i = 0; i < 4; ++i) m_loc = max_part(sacc[0], i, m_loc);
        finish_max(m_loc, sacc[0]);
      }
      refill(0);
      float m_loc;
      for (int st = 0; st < n_stage; st += 2) {
        qk_step(1, 0, no_extra);
        mask_slice(sacc[1], 2 * st + 1);
        m_loc = pv_step(0, KS);
        finish_max(m_loc, sacc[1]);
        publish();
        more_ids(st + 2 + kCodes);
        refill(G_B0);
        qk_step(0, STEP, [&](int ks) { bring(ks, st + 2, 0); });
        mask_slice(sacc[0], 2 * st + 2);
        m_loc = pv_step(1, STEP + KS);
        finish_max(m_loc, sacc[0]);
        if (st + 1 >= n_stage) break;
        qk_step(1, 2 * STEP, no_extra);
        mask_slice(sacc[1], 2 * st + 3);
        m_loc = pv_step(0, 2 * STEP + KS);
        finish_max(m_loc, sacc[1]);
        publish();
        more_ids(st + 3 + kCodes);
        refill(G_B1);
        qk_step(0, 3 * STEP, [&](int ks) { bring(ks, st + 3, 1); });
        mask_slice(sacc[0], 2 * st + 4);
        m_loc = pv_step(1, 3 * STEP + KS);
        finish_max(m_loc, sacc[0]);
      }
    } else {
      // (no rows: the wavefront only brings its part of the stages)
      for (int st = 0; st < n_stage; ++st) {
        publish();
        more_ids(st + 2 + kCodes);
        if (st & 1) bring_all(st + 2, 1);
        else bring_all(st + 2, 0);
      }
    }
    publish();  // (loads of stages past the end may still be in flight towards LDS)
  }

  if (kSplit && parts > 1) {
    // ---- part of a tile: unnormalised output and its softmax state, as the lanes hold them ----
    if (!active) return;
    float *dst = c.part + ((size_t)wk.slot * WAVES + wave) * kPartFloats<D>;
    dst[64 * 16 * DT + lane] = m_ref;
    dst[64 * 16 * DT + 64 + lane] = l_run;
    f32x4_t *o4 = reinterpret_cast<f32x4_t *>(dst);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        o4[(4 * dt + g) * 64 + lane] = f32x4_t{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]} * v_unit;
    return;
  }

  // ---- epilogue: normalise, stage through LDS, coalesced bf16 store -----------------------
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;  // (a NaN stays one, in the log-sum-exp too)
  if (c.lse && hf == 0 && row < rows) {
    const Row at = row_of(c, s, wk.h, row);
    c.lse[(long long)at.head * c.s.T + at.token] = l_tot == 0.f ? ninf : (m_ref + log2f(l_tot)) * 0.6931471805599453f;
  }
  uint16_t *sO = reinterpret_cast<uint16_t *>(smem);  // [TILE][SO]
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      u32x2_t pk;
      pk.x = cvt_pk_bf16(o[dt][4 * g + 0] * inv * v_unit, o[dt][4 * g + 1] * inv * v_unit);
      pk.y = cvt_pk_bf16(o[dt][4 * g + 2] * inv * v_unit, o[dt][4 * g + 3] * inv * v_unit);
      *reinterpret_cast<u32x2_t *>(sO + (wave * 32 + l32) * SO + dt * 32 + 8 * g + 4 * hf) = pk;
    }
  __syncthreads();
  constexpr int OCH = TILE * CPR / THREADS, STEP_R = THREADS / CPR;
#pragma unroll
  for (int it = 0; it < OCH; ++it) {
    const int r = t / CPR + it * STEP_R;
    if (r0 + r < rows) {
      const Row at = row_of(c, s, wk.h, r0 + r);
      *reinterpret_cast<u32x4_t *>(c.out + at.token * c.ot + at.head * c.oh + (t % CPR) * 8) =
          *reinterpret_cast<const u32x4_t *>(sO + r * SO + (t % CPR) * 8);
    }
  }
}

constexpr int kMergeGroups = 4, kMergeParts = 4;  // groups, parts of a group in flight

// Adds up the parts of the tiles whose keys were divided: a workgroup has 32 rows, a wavefront 32 columns, lanes as above.
// Bound by latency (the parts come from the L2s and the memory-side cache): the parts are dealt to four groups of
// wavefronts, four parts at a time each, and the groups' sums meet in LDS (8 queries of 32000 keys, 3 key heads in 125
// parts each, D = 64: the call takes 28 us, 53 with one group).
template <int D, CacheMode kMode, int WAVES = kTile / 32>
__global__ __launch_bounds__(D * 2 * kMergeGroups) void cache_attn_merge_kernel(const AttnCall c) {
  constexpr float ninf = -__builtin_inff();
  constexpr int DT = D / 32, NP = kMergeParts, TILE = 32 * WAVES;
  __shared__ float meet[kMergeGroups - 1][DT][18][64];
  const int lane = threadIdx.x & 63, l32 = lane & 31, hf = lane >> 5;
  const int dt = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6) % DT);
  const int group = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6) / DT);
  const int wave = (int)(blockIdx.x % WAVES), item = (int)(blockIdx.x / WAVES);
  int tile, h;
  if constexpr (kMode == kTail) item_at(c, c.whole + item, c.n_items, tile, h);
  else tile = item / c.H, h = item % c.H;
  const int b = seq_of_tile<TILE>(c, tile, lane);
  int m = __builtin_amdgcn_readfirstlane(tile - tile_start<TILE>(c, b));
  const Seq s = seq_of(c, b);
  const int tiles = tiles_of<TILE>(c, s);
  if (m < 0 || m >= tiles) return;
  if constexpr (kMode == kTail) m = tiles - 1 - m;
  const int rows = s.n * c.G, row = m * TILE + wave * 32 + l32;
  if (m * TILE + wave * 32 >= rows) return;
  const int4 it = c.items[item];
  if (it.y <= 1) return;
  float ref = ninf, l = 0.f;
  f32x4_t o[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) o[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int s0 = group; s0 < it.y; s0 += kMergeGroups * NP) {
    float ms[NP], ls[NP];
    f32x4_t x[NP][4];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const float *src = c.part + ((size_t)(it.x + min(s0 + kMergeGroups * i, it.y - 1) * it.z) * WAVES + wave) * kPartFloats<D>;
      ms[i] = src[64 * (D / 2) + lane];
      ls[i] = src[64 * (D / 2) + 64 + lane];
      const f32x4_t *o4 = reinterpret_cast<const f32x4_t *>(src) + 4 * 64 * dt + lane;
#pragma unroll
      for (int g = 0; g < 4; ++g) x[i][g] = o4[64 * g];
    }
    const float old = ref;
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (s0 + kMergeGroups * i < it.y) ref = fmaxf(ref, ms[i]);
    // (a part whose logits are all -inf keeps the reference -inf: its weight is 0)
    const float fin = ref == ninf ? 0.f : ref;
    const float alpha = __builtin_amdgcn_exp2f(old - fin);
    l *= alpha;
#pragma unroll
    for (int g = 0; g < 4; ++g) o[g] *= alpha;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (s0 + kMergeGroups * i >= it.y) continue;
      const float w = __builtin_amdgcn_exp2f(ms[i] - fin);
      l = fmaf(ls[i], w, l);
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[g][e] = fmaf(x[i][g][e], w, o[g][e]);
    }
  }
  if (group) {
    float(*to)[64] = meet[group - 1][dt];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) to[4 * g + e][lane] = o[g][e];
    to[16][lane] = ref;
    to[17][lane] = l;
  }
  __syncthreads();
  if (group) return;
#pragma unroll
  for (int j = 0; j < kMergeGroups - 1; ++j) {
    const float(*from)[64] = meet[j][dt];
    const float other = from[16][lane], top = fmaxf(ref, other), fin = top == ninf ? 0.f : top;
    const float a = __builtin_amdgcn_exp2f(ref - fin), b2 = __builtin_amdgcn_exp2f(other - fin);
    ref = top;
    l = fmaf(from[17][lane], b2, l * a);
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[g][e] = fmaf(from[4 * g + e][lane], b2, o[g][e] * a);
  }
  const float l_tot = l + __shfl_xor(l, 32, 64);
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
  if (row >= rows) return;
  const Row at = row_of(c, s, h, row);
  if (c.lse && dt == 0 && hf == 0)
    c.lse[(long long)at.head * c.s.T + at.token] = l_tot == 0.f ? ninf : (ref + log2f(l_tot)) * 0.6931471805599453f;
  uint16_t *dst = c.out + at.token * c.ot + at.head * c.oh + 32 * dt + 4 * hf;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    u32x2_t pk;
    pk.x = cvt_pk_bf16(o[g][0] * inv, o[g][1] * inv);
    pk.y = cvt_pk_bf16(o[g][2] * inv, o[g][3] * inv);
    *reinterpret_cast<u32x2_t *>(dst + 8 * g) = pk;
  }
}

// How the keys of a call of n_items tiles are divided: by that number, that of the sequences and that of the places (of short sequences, by the
// page tables' room, otherwise: launch_cache_attn).
struct Division {
  CacheMode mode;
  int rounds;       // (kParts) of workgroups at most
  int whole, tail;  // (kTail) tiles that are not divided, parts of each other
  long long slots() const { return mode == kParts ? (long long)rounds * kPlaces : mode == kTail ? slots_tail : 0; }
  long long slots_tail;
  float cost = 0.f;  // (the last round's tiles) rounds that all take
};
// Fewer tiles than places: all are divided, but of one sequence only where that gives three parts in two rounds.  Up to
// kTailRounds rounds: the r tiles of the last one, into as many parts (8 at most, two for each place in all) as let it end soonest, a part
// costing 0.03 of a whole tile beside its keys.  us whole -> divided, 4680 queries, 32760 keys: 4 heads of 37 tiles 534 -> 330, 8
// (296 tiles) 763 -> 637, 14 (518) 1375 -> 1010, 16 (592) 1389 -> 1169, 18 1445 -> 1320, 32 2352 -> 2252; 9360 keys, 16 heads, 334 -> 300.
constexpr int kTailRounds = 8, kBrief = 80 * kStage;
static Division divide_last(long long n_items, int places) {
  const int r = (int)(n_items % places);
  const float before = (float)(n_items / places);
  if (n_items < places || n_items > (long long)kTailRounds * places || r == 0) return {kWhole, 1, 0, 1, 0, before + (r ? 1.f : 0.f)};
  int best = 1;
  float least = 1e9f;
  for (int p = 1; p <= 8 && r * p <= 2 * places; ++p) {
    const float cost = (float)((r * p + places - 1) / places) / p + (p > 1 ? 0.03f * p * r / places + 0.02f : 0.f);
    if (cost < least) least = cost, best = p;
  }
  if (best == 1) return {kWhole, 1, 0, 1, 0, before + 1.f};
  return {kTail, 1, (int)n_items - r, best, (long long)r * best, before + least};
}
static Division divide(int B, long long n_items) {
  if (n_items < kPlaces && B <= kSplitSeqs && (B > 1 || 3 * n_items <= 2 * kPlaces))
    return {kParts, 3 * n_items > kPlaces ? 2 : 1, 0, 1, 0};
  return divide_last(n_items, kPlaces);
}

// int8, D = 128: tiles of 256 rows, eight wavefronts, that share what it takes to turn codes into f16 (238 VALU instructions of a
// wavefront and stage, some 40 fewer).  Where long sequences have four tiles each, on average, and the rounds of the chip's 256 places, the last one
// divided if that pays, are full but for a seventh.  us of tiles of 128 and of 256, 4680 queries of 32760 keys: 40 heads (760 tiles)
// 3366 / 2994, 24 (456) 2152 / 1895, 16 (304) 1266 / 1193, 12 (228) 1076 / 974, 8 (152) 772 / 869; six ragged prompts of up to 2048 tokens, 40 on 8
// heads, 12000 keys 755 / 739; 4680 keys, 40 heads, 313 / 316; 64 of up to 256 tokens, 8 heads 135 / 149.
constexpr int kWideTile = 256, kWidePlaces = 256;
static bool may_be_wide(int type, int B, int H, int D, int T, int Hq) {
  return type == HEART_CACHE_INT8 && D == 128 && (long long)T * (Hq / H) >= 4ll * kWideTile * B;
}
static bool wide_tiles(const heart_cache &c, int T, int Hq, bool divided, Division &d) {
  if (!may_be_wide(c.type, c.B, c.H, c.D, T, Hq) || (long long)c.max_pages * c.page <= kBrief) return false;
  const long long tiles = most_items(kWideTile, c.B, c.H, T, Hq);
  Division w = divide_last(tiles, kWidePlaces);
  if (!divided) w = {kWhole, 1, 0, 1, 0, (float)((tiles + kWidePlaces - 1) / kWidePlaces)};
  if (7.f * (float)tiles < 6.f * kWidePlaces * w.cost) return false;
  d = w;
  return true;
}

size_t cache_attn_workspace_bytes(int type, int B, int H, int D, int T, int Hq) {
  const size_t few = cache_attn_few_workspace_bytes(B, H, D, T, Hq);
  if (cache_attn_few(B, H, T, Hq)) return few;
  const Division d = divide(B, most_items(kTile, B, H, T, Hq));
  const size_t part = D == 128 ? kPartFloats<128> : kPartFloats<64>;
  const size_t many = d.mode == kWhole ? 0 : kPlaces * sizeof(int4) + (size_t)d.slots() * 4 * part * sizeof(float);
  // (which kernel it is goes by the page tables' room too, which is not known here)
  if (may_be_wide(type, B, H, D, T, Hq)) {
    const Division w = divide_last(most_items(kWideTile, B, H, T, Hq), kWidePlaces);
    const size_t wide = w.mode == kWhole ? 0 : kPlaces * sizeof(int4) + (size_t)w.slots() * (kWideTile / 32) * part * sizeof(float);
    return wide > many ? wide : many;
  }
  return type == HEART_CACHE_INT8 && (long long)T * (Hq / H) <= (long long)kIntRows * B && few > many ? few : many;
}

template <int D, CacheKind kKind>
static int launch_t(const AttnCall &c, const Division &d, bool wide, hipStream_t st) {
  const int dev = current_device();
  if (dev < 0) return fail(HEART_EHIP, "heart_cache_attn: cannot identify the current device");
  auto run_waves = [&](auto mode, long long grid, auto waves) -> int {
    constexpr int W = decltype(waves)::value;
    constexpr int lds = 4 * kStage * D * 2, staging = 32 * W * (D + 8) * 2, bytes = lds > staging ? lds : staging;
    auto kern = cache_attn_kernel<D, kKind, decltype(mode)::value, W>;
    static DeviceFlags attr_set;  // per instantiation: the attribute is per function and device
    if (hipError_t e = set_max_lds_once(attr_set, dev, reinterpret_cast<const void *>(kern), bytes))
      return fail(HEART_EHIP, "hipFuncSetAttribute(max dynamic LDS %d): %s", bytes, hipGetErrorString(e));
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(64 * W), bytes, st, c);
    return check_launch("cache_attn_kernel");
  };
  auto run = [&](auto mode, long long grid) -> int { return run_waves(mode, grid, std::integral_constant<int, kTile / 32>{}); };
  if constexpr (kKind == kInt8 && D == 128)
    if (wide) {
      constexpr int W = kWideTile / 32;
      const std::integral_constant<int, W> waves{};
      if (d.mode == kWhole) return run_waves(std::integral_constant<CacheMode, kWhole>{}, c.n_items, waves);
      if (int rc = run_waves(std::integral_constant<CacheMode, kTail>{}, c.whole + d.slots(), waves)) return rc;
      hipLaunchKernelGGL((cache_attn_merge_kernel<D, kTail, W>), dim3((unsigned)((c.n_items - c.whole) * W)), dim3(D * 2 * kMergeGroups), 0, st, c);
      return check_launch("cache_attn_merge_kernel");
    }
  if (d.mode == kWhole) return run(std::integral_constant<CacheMode, kWhole>{}, c.n_items);
  if (d.mode == kParts) {
    const int rc = c.s.B <= 64 ? run(std::integral_constant<CacheMode, kParts>{}, d.slots())
                               : run(std::integral_constant<CacheMode, kPartsWide>{}, d.slots());
    if (rc) return rc;
    hipLaunchKernelGGL((cache_attn_merge_kernel<D, kParts>), dim3((unsigned)(c.n_items * 4)), dim3(D * 2 * kMergeGroups), 0, st, c);
  } else {
    if (int rc = run(std::integral_constant<CacheMode, kTail>{}, c.whole + d.slots())) return rc;
    hipLaunchKernelGGL((cache_attn_merge_kernel<D, kTail>), dim3((unsigned)((c.n_items - c.whole) * 4)), dim3(D * 2 * kMergeGroups), 0, st, c);
  }
  return check_launch("cache_attn_merge_kernel");
}

int launch_cache_attn(const heart_cache &c, int T, int Hq, const void *q, const long long qs[2], const int *cu_q, int causal,
                      int window, float scale, void *out, const long long os[2], float *lse, void *workspace,
                      hipStream_t st) {
  const long long eb = c.type == HEART_CACHE_BF16 ? 2 : 1;
  AttnCall a{};
  a.k = CacheTensor{(const uint8_t *)c.k, c.k_exp, c.k_stride[0] * eb, c.k_stride[1] * eb, (uint32_t)(c.k_stride[2] * eb)};
  a.v = CacheTensor{(const uint8_t *)c.v, c.v_exp, c.v_stride[0] * eb, c.v_stride[1] * eb, (uint32_t)(c.v_stride[2] * eb)};
  a.s = cache_seqs(c, T, cu_q);
  a.q = (const uint16_t *)q;
  a.out = (uint16_t *)out;
  a.lse = lse;
  a.qt = qs[0], a.qh = qs[1], a.ot = os[0], a.oh = os[1];
  a.H = c.H, a.G = Hq / c.H, a.causal = causal, a.window = window;
  a.scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf((float)c.D)) * 1.4426950408889634f;
  if (c.type == HEART_CACHE_INT8 ? cache_attn_int8_few(c, T, Hq) : cache_attn_few(c.B, c.H, T, Hq))
    return launch_cache_attn_few(c, T, Hq, a, workspace, st);
  const long long items = most_items(kTile, c.B, c.H, T, Hq);
  if (items > kMostGroups) return fail(HEART_EUNSUPPORTED, "heart_cache_attn: grid too large");
  Division d = divide(c.B, items);
  // (page tables with room for so few tokens, all that is known of lengths here: a second round of parts, and the launch that adds them
  // up, gain nothing: causal attention of 4680 tokens to themselves, 8 heads 87 us whole, 93 divided, 16 heads 124, 129.  As short
  // sequences of a table with more room are divided all the same.  16 sequences of 4000 tokens and 48 queries, eight heads in
  // e4m3: 77 whole, 44 in one round of parts)
  if (a.s.cap <= kBrief) {
    if (d.mode == kTail || (c.B == 1 && 2 * items > kPlaces)) d = {kWhole, 1, 0, 1, 0};
    d.rounds = 1;
  }
  if (!workspace) d = {kWhole, 1, 0, 1, 0};
  const bool wide = wide_tiles(c, T, Hq, workspace != nullptr, d);
  a.n_items = (int)(wide ? most_items(kWideTile, c.B, c.H, T, Hq) : items);
  a.rounds = d.rounds;
  a.whole = d.whole;
  a.tail = d.tail;
  a.items = (int4 *)workspace;
  a.part = workspace ? (float *)(a.items + kPlaces) : nullptr;
  auto of_kind = [&](auto dim) -> int {
    constexpr int D = decltype(dim)::value;
    if (c.type == HEART_CACHE_INT8) return launch_t<D, kInt8>(a, d, wide, st);
    return c.type == HEART_CACHE_E4M3 ? launch_t<D, kE4m3>(a, d, false, st) : launch_t<D, kBf16>(a, d, false, st);
  };
  return c.D == 128 ? of_kind(std::integral_constant<int, 128>{}) : of_kind(std::integral_constant<int, 64>{});
}

}  // namespace heart
