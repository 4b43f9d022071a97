// heart_cache_attn where a key head has few rows (single tokens, drafts of a few): bound by reading the cache.
//
// A tile is 16 or 32 rows, and a workgroup's four wavefronts divide the keys of its part among them, slice by slice, each
// with a softmax state of its own that is put together at the end.  Every wavefront brings its own slices into its own
// part of LDS, so the loop has no barrier, only waits for the wavefront's own loads:
//   S^T (keys x rows) = K . Q^T,  O^T (d x rows) += V^T . P^T     with v_mfma_f32_16x16x32_bf16 (16x16x16 for slices of 16)
// In the 16x16 accumulator a lane holds one row (lane % 16) and keys 4 (lane / 16) + 0..3; exponentiated they are, as they
// are, the B operand of the second product, whose A operand the transposing LDS reads deliver in the same order of keys.
//
// K and V slices (32 keys; 16 of bf16 rows of 256 bytes) are double-buffered, 8 KB a slice, by LDS-direct loads; K of
// slice i + 2 is issued as soon as the fragments of K of slice i are in registers, V likewise, so 8 to 16 KB a wavefront, 64
// to 128 KB a CU, are on their way at any time.  Codes stay codes in LDS: K is converted with its row's power of two at the
// fragment read; V as it is, its powers of two go into the weights, which are multiplied by them before they are
// rounded (a power of two rounds nothing).
//
// Dividing the keys: see part_of_few.  Parts are added up by a second launch.
#include <type_traits>

#include "cache_attn_device.h"

namespace heart {

constexpr int kFewStage = 128;    // keys that parts are measured in: four wavefronts' slices
#ifndef FEW_MIN
#define FEW_MIN 4
#endif
#ifndef FEW_TARGET
#define FEW_TARGET 1024
#endif
constexpr int kFewMin = FEW_MIN;        // fewest stages of a part
constexpr int kFewTarget = FEW_TARGET;  // parts of a call, about
constexpr int kMergeThreads = 512;

template <int D, int NR>
constexpr int kFewPart = 16 * NR * (D + 2);  // floats of a part: rows of D, references, row sums

// The part of workgroup w.  Parts have at most L stages: as many as give kFewTarget parts in all (four to a place for a
// workgroup: parts of different calls' lengths level each other out), but kFewMin at least.  Every wavefront finds that from the
// lengths on its own.  Their order: sequences; of each, heads, parts, tiles.
template <int TILE>
__device__ __forceinline__ bool part_of_few(const AttnCall &c, int w_xcd, int w_slot, int slots, int lane, Work &k) {
  constexpr int NB = kSplitSeqs / 64;
  int wgs[NB], st[NB];
  float all = 0.f;
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int b = j * 64 + lane;
    wgs[j] = 0;
    st[j] = 1;
    if (j * 64 < c.s.B && b < c.s.B) {
      const Seq s = seq_of(c, b);
      wgs[j] = tiles_of<TILE>(c, s) * c.H;
      st[j] = stages_of<TILE, kFewStage>(c, s);
      all += (float)wgs[j] * (float)st[j];
    }
  }
  all = wave_sum_f32(all);
  int L = max(kFewMin, (int)(all / (float)c.target) + 1);
  int at = 0, w = 0, end_x = 0;
  for (int again = 0;; ++again) {
    int n = 0;
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (j * 64 < c.s.B) n += wgs[j] * (int)((unsigned)(st[j] + L - 1) / (unsigned)L);
    const int total = __builtin_amdgcn_readfirstlane(wave_sum_i32(n));
    // (more than there is room for: only of token ranges that overlap, which then are not divided)
    if (total > slots && again == 0) {
      L = 0x40000000;
      continue;
    }
    w = (int)((long long)w_xcd * total / kNumXcd) + w_slot;
    end_x = (int)((long long)(w_xcd + 1) * total / kNumXcd);
    break;
  }
  if (w >= end_x) return false;
#pragma unroll
  for (int j = 0; j < NB; ++j)
    if (j * 64 < c.s.B) {
      const int parts = (int)((unsigned)(st[j] + L - 1) / (unsigned)L), n = wgs[j] * parts;
      const int end = at + wave_scan_i32(n), start = end - n;
      const unsigned long long here = __ballot(start <= w && w < end);
      if (here) {
        const int l = __ffsll((long long)here) - 1;
        k.b = j * 64 + l;
        k.parts = __builtin_amdgcn_readlane(parts, l);
        k.step = __builtin_amdgcn_readlane(wgs[j], l) / c.H;
        const int r = w - __builtin_amdgcn_readlane(start, l);
        k.h = r / (k.parts * k.step);
        k.part = r / k.step % k.parts;
        k.m = r % k.step;
      }
      at = __builtin_amdgcn_readlane(end, 63);
    }
  k.slot = w;
  return true;
}

template <int D, bool kCodes>
struct FewShape {
  static constexpr int ROWB = kCodes ? D : 2 * D;        // bytes of a row
  static constexpr int SK = ROWB == 256 ? 16 : 32;       // keys of a slice
  static constexpr int NT = SK / 16;                     // key tiles of 16
  static constexpr int TENSOR_B = SK * ROWB;             // bytes of a slice of K or V
  static constexpr int SLICE_B = 2 * TENSOR_B + (kCodes ? 256 : 0);
  static constexpr int WAVE_B = 2 * SLICE_B;             // double-buffered
  static constexpr int NI = 16 * ROWB / 1024;            // LDS-direct loads of 16 rows
  static constexpr int per_cu() { return 160 * 1024 / (4 * WAVE_B + 1024) < 4 ? 160 * 1024 / (4 * WAVE_B + 1024) : 4; }
};

template <int D, bool kCodes, int NR, bool kSplit>
__global__ __launch_bounds__(256, 2) void cache_attn_few_kernel(const AttnCall c, int slots) {
  using F = FewShape<D, kCodes>;
  constexpr int TILE = 16 * NR, ROWB = F::ROWB, SK = F::SK, NT = F::NT, NI = F::NI;
  constexpr int NC = ROWB / 16, RPB = 256 / ROWB, RPI = 1024 / ROWB;  // chunks of a row, rows per 256 bytes, rows of a load
  constexpr int KS = D / 32, DT = D / 16;
  constexpr int NLOAD = NT * NI;                       // loads of K (or V) of a slice
  constexpr int PER = 2 * NLOAD + (kCodes ? 1 : 0);    // all of a slice
  constexpr float ninf = -__builtin_inff(), kSlack = 8.f;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ float s_ref[4][TILE], s_sum[4][TILE];
  const uint32_t smem_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)smem;
  const int t = threadIdx.x, lane = t & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);

  // ---- what to work on -----------------------------------------------------------------------
  Work wk{0, 0, 0, 0, 1, 1, 0};
  if constexpr (kSplit) {
    if (!part_of_few<TILE>(c, (int)(blockIdx.x % kNumXcd), (int)(blockIdx.x / kNumXcd), slots, lane, wk)) return;
  } else {
    const int tile = (int)(blockIdx.x / (unsigned)c.H);
    wk.h = (int)(blockIdx.x % (unsigned)c.H);
    wk.b = seq_of_tile<TILE>(c, tile, lane);
    wk.m = tile - tile_start<TILE>(c, wk.b);
  }
  wk.b = __builtin_amdgcn_readfirstlane(wk.b);
  wk.m = __builtin_amdgcn_readfirstlane(wk.m);
  wk.h = __builtin_amdgcn_readfirstlane(wk.h);
  const Seq s = seq_of(c, wk.b);
  if (wk.m < 0 || wk.m >= tiles_of<TILE>(c, s)) return;
  const int rows = s.n * c.G, r0 = wk.m * TILE;
  int first_key, end_key, ignore;
  seen_by(c, s, s.pos0 + r0 / c.G, first_key, ignore);
  seen_by(c, s, s.pos0 + min(r0 + TILE - 1, rows - 1) / c.G, ignore, end_key);
  int stage0 = first_key / kFewStage, n_stage = max((end_key + kFewStage - 1) / kFewStage - stage0, 0);
  int parts = 1;
  if constexpr (kSplit) {
    const int per = max((n_stage + wk.parts - 1) / wk.parts, 1);
    parts = max((n_stage + per - 1) / per, 1);
    if (wk.part == 0 && t == 0)
      c.items[(long long)(tile_start<TILE>(c, wk.b) + wk.m) * c.H + wk.h] = int4{wk.slot, parts, wk.step, 0};
    if (wk.part >= parts) return;
    stage0 += wk.part * per;
    n_stage = min(per, n_stage - wk.part * per);
    end_key = min(end_key, (stage0 + n_stage) * kFewStage);
  }
  const int key0 = __builtin_amdgcn_readfirstlane(stage0 * kFewStage + wave * SK);  // of this wavefront's slice 0
  end_key = __builtin_amdgcn_readfirstlane(end_key);
  const int n_slice = __builtin_amdgcn_readfirstlane(max((end_key - key0 + 4 * SK - 1) / (4 * SK), 0));

  int lo[NR], hi[NR], all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = r0 + 16 * n + l16;
    seen_by(c, s, s.pos0 + min(row, rows - 1) / c.G, lo[n], hi[n]);
    if (row >= rows) lo[n] = 0, hi[n] = end_key;  // (rows past the end see what is there)
    hi[n] = min(hi[n], end_key);
    all_lo = max(all_lo, (int)wave_max_u32((uint32_t)lo[n]));
    all_hi = min(all_hi, (int)wave_min_u32((uint32_t)hi[n]));
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
  // (rows 16 .. 31 of a slice: V codes are swizzled differently there)
  uint32_t dma_off2[kCodes ? NI : 1];
  if constexpr (kCodes) {
#pragma unroll
    for (int ii = 0; ii < NI; ++ii) {
      const int r = ii * RPI + lane / NC;
      dma_off2[ii] = (uint32_t)r * c.v.row + (uint32_t)(((lane % NC) ^ swizzle(1, r + 16)) * 16);
    }
  }

  // ---- page ids of slices base .. base + 63, lane l that of slice base + l, by tile
  int ids[NT];
  auto load_ids = [&](int base) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const long long key = key0 + (long long)(base + lane) * (4 * SK) + 16 * n;
      ids[n] = key < end_key ? cache_page(c.s, wk.b, (int)key) : -1;
    }
  };
  // (codes) of slices i, i + 1, i + 2: all ones where the tile's page is one
  uint32_t named[3][NT];
  const int in_page = (1 << c.s.page_shift) - 1;
  const uint32_t wave_lds = smem_lds + (uint32_t)(wave * F::WAVE_B);
  unsigned char *const wave_mem = smem + wave * F::WAVE_B;
  // K (V) of slice i to buffer i & 1
  auto bring = [&](int is_v, int i) __attribute__((always_inline)) {
    const CacheTensor &x = is_v ? c.v : c.k;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int key = key0 + i * (4 * SK) + 16 * n, off = key & in_page;
      const int id = i < n_slice ? __builtin_amdgcn_readlane(ids[n], i & 63) : -1;
      const uint64_t addr = (uint64_t)(x.p + max(id, 0) * x.page + wk.h * x.head + off * (long long)x.row);
      const int there = id < 0 ? 0 : min(s.len - key, 16);
      u32x4_t rs;
      rs.x = __builtin_amdgcn_readfirstlane((uint32_t)addr);
      rs.y = __builtin_amdgcn_readfirstlane((uint32_t)(addr >> 32) & 0xffffu);
      rs.z = __builtin_amdgcn_readfirstlane(there > 0 ? (uint32_t)(there - 1) * x.row + (uint32_t)ROWB : 0u);
      rs.w = 0x00020000u;
#pragma unroll
      for (int ii = 0; ii < NI; ++ii) {
        const uint32_t dst = wave_lds + (uint32_t)((i & 1) * F::SLICE_B + is_v * F::TENSOR_B + (n * NI + ii) * 1024);
        const uint32_t voffset = kCodes && is_v && n == 1 ? dma_off2[kCodes ? ii : 0] : dma_off[is_v][ii];
        // (the compiler does not see this instruction's LDS write: completion is awaited by count.  M0 is saved and
        // restored, it may hold a value of the compiler's)
        uint32_t m0_saved;
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0_saved) : "s"(dst), "v"(voffset), "s"(rs) : "memory");
      }
    }
  };
  // (codes) exponents of slice i, 4 bytes a lane: K of tiles 0 and 1, V of tiles 0 and 1; pages that are none: of page 0
  auto bring_exps = [&](int i, int ahead) __attribute__((always_inline)) {
    if constexpr (kCodes) {
      const int n = (lane >> 2) & 1;
      const int id0 = i < n_slice ? __builtin_amdgcn_readlane(ids[0], i & 63) : -1;
      const int id1 = i < n_slice ? __builtin_amdgcn_readlane(ids[NT - 1], i & 63) : -1;
      named[ahead][0] = id0 < 0 ? 0u : 0xffffffffu;
      named[ahead][NT - 1] = id1 < 0 ? 0u : 0xffffffffu;
      const int id = max(n ? id1 : id0, 0), key = key0 + i * (4 * SK) + 16 * n;
      const uint8_t *base = lane & 8 ? c.v.exp : c.k.exp;
      const uint8_t *addr = base + ((((long long)id * c.H + wk.h) << c.s.page_shift) + (key & in_page) + 4 * (lane & 3));
      const uint32_t dst = wave_lds + (uint32_t)((i & 1) * F::SLICE_B + 2 * F::TENSOR_B);
      uint32_t m0_saved;
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                   "global_load_lds_dword %2, off\n\ts_mov_b32 m0, %0"
                   : "=&s"(m0_saved) : "s"(dst), "v"(addr) : "memory");
    }
  };

  // ---- state of the rows -----------------------------------------------------------------------
  Frag8 qf[NR][KS];
  f32x4_t o[NR][DT];
  float m_ref[NR], c0[NR], l_run[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const Row at = row_of(c, s, wk.h, min(r0 + 16 * n + l16, rows - 1));
    const uint16_t *src = c.q + at.token * c.qt + at.head * c.qh;
    // (codes: a lane's 16 bytes are d 16 (4 i + g) .. of k-steps 2 i and 2 i + 1)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[n][ks].u = *reinterpret_cast<const u32x4_t *>(src + (kCodes ? 16 * (4 * (ks / 2) + g) + 8 * (ks & 1) : 32 * ks + 8 * g));
    m_ref[n] = ninf;
    c0[n] = 0.f;
    l_run[n] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[n][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const float scale_log2e = c.scale_log2e, inv_scale = 1.f / scale_log2e;

  if (n_slice > 0) {
    load_ids(0);
    bring(0, 0);
    bring_exps(0, 0);
    bring(1, 0);
    bring(0, 1);
    bring_exps(1, 1);
    bring(1, 1);
    for (int i = 0; i < n_slice; ++i) {
      const unsigned char *sk = wave_mem + (i & 1) * F::SLICE_B, *sv = sk + F::TENSOR_B, *se = sk + 2 * F::TENSOR_B;
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NLOAD + PER) : "memory");  // K and exponents of slice i are there
      const int key = key0 + i * (4 * SK);
      // ---- S^T ------------------------------------------------------------------------------
      Frag8 kf[NT][KS];
      float vu[NT][4];  // (codes) powers of two of V's rows 16 n + 4 g + 0..3
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if constexpr (kCodes) {
          // (a page that is none has exponents of another: 0, so that its zeros stay zeros)
          const float ku = unit_of(min((uint32_t)se[16 * n + l16] & named[0][n], 254u));
          const uint32_t ve = *reinterpret_cast<const uint32_t *>(se + 32 + 16 * n + 4 * g) & named[0][n];
#pragma unroll
          for (int e = 0; e < 4; ++e) vu[n][e] = unit_of(min((ve >> (8 * e)) & 0xffu, 254u));
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
      if (((i + 2) & 63) == 0) load_ids(i + 2);
      bring(0, i + 2);
      bring_exps(i + 2, 2);
      f32x4_t x[NR][NT];
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int kt = 0; kt < NT; ++kt) {
          f32x4_t acc = {c0[n], c0[n], c0[n], c0[n]};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kt][ks].v, qf[n][ks].v, acc, 0, 0, 0);
          x[n][kt] = acc * scale_log2e;
        }
      if (key < all_lo || key + SK > all_hi) {
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int kt = 0; kt < NT; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = key + 16 * kt + 4 * g + e;
              if (j < lo[n] || j >= hi[n]) x[n][kt][e] = ninf;
            }
      }
      // ---- the reference moves where a logit exceeds it by more than the slack ------------------
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float m = ninf;
#pragma unroll
        for (int kt = 0; kt < NT; ++kt) m = fmaxf(fmaxf(fmaxf(m, x[n][kt][0]), x[n][kt][1]), fmaxf(x[n][kt][2], x[n][kt][3]));
        const bool first = m_ref[n] == ninf;
        if (__any(m > kSlack || (first && m > ninf))) {
          uint32_t a, b;
          swap_rows16(__float_as_uint(m), a, b);
          m = fmaxf(__uint_as_float(a), __uint_as_float(b));
          swap_halves32(__float_as_uint(m), a, b);
          m = fmaxf(__uint_as_float(a), __uint_as_float(b));
          const bool bump = m > kSlack || (first && m > ninf);
          const float delta = bump ? m : 0.f, m_new = bump ? (first ? 0.f : m_ref[n]) + m : m_ref[n];
          const float alpha = bump ? __builtin_amdgcn_exp2f(m_ref[n] - m_new) : 1.f;
          l_run[n] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) o[n][dt] *= alpha;
#pragma unroll
          for (int kt = 0; kt < NT; ++kt) x[n][kt] -= delta;
          m_ref[n] = m_new;
          c0[n] = m_new == ninf ? 0.f : -m_new * inv_scale;
        }
      }
      // ---- weights ------------------------------------------------------------------------------
      Frag8 pf[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int kt = 0; kt < NT; ++kt) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = __builtin_amdgcn_exp2f(x[n][kt][e]);
            l_run[n] += p[e];
            if constexpr (kCodes) p[e] *= vu[kt][e];
          }
          pf[n].u[2 * kt] = cvt_pk_bf16(p[0], p[1]);
          pf[n].u[2 * kt + 1] = cvt_pk_bf16(p[2], p[3]);
        }
      // ---- O^T ------------------------------------------------------------------------------------
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PER + NLOAD + (kCodes ? 1 : 0)) : "memory");  // V of slice i is there
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
        typedef __attribute__((address_space(3))) i32x2_t lds_i32x2;
        if constexpr (kCodes) {
          const i32x2_t r = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(sv + voff[dt]));
          Frag8 a;
          a.u = u32x4_t{codes_to_bf16<false>((uint32_t)r.x, 1.f), codes_to_bf16<true>((uint32_t)r.x, 1.f),
                        codes_to_bf16<false>((uint32_t)r.y, 1.f), codes_to_bf16<true>((uint32_t)r.y, 1.f)};
#pragma unroll
          for (int n = 0; n < NR; ++n) o[n][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, pf[n].v, o[n][dt], 0, 0, 0);
        } else if constexpr (NT == 2) {
          const u32x2_t r = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(sv + voff[dt])));
          const u32x2_t r2 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(sv + 16 * ROWB + voff[dt])));
          Frag8 a;
          a.u = u32x4_t{r.x, r.y, r2.x, r2.y};
#pragma unroll
          for (int n = 0; n < NR; ++n) o[n][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, pf[n].v, o[n][dt], 0, 0, 0);
        } else {
          const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(sv + voff[dt]));
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const u32x2_t b = {pf[n].u[0], pf[n].u[1]};
            o[n][dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, __builtin_bit_cast(s16x4_t, b), o[n][dt], 0, 0, 0);
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      bring(1, i + 2);
#pragma unroll
      for (int n = 0; n < NT; ++n) named[0][n] = named[1][n], named[1][n] = named[2][n];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads past the end are still on their way to LDS)
  }

  // ---- the four wavefronts' states put together ---------------------------------------------------
  float *so = reinterpret_cast<float *>(smem);
  static_assert(TILE * D * 4 <= F::WAVE_B, "a wavefront's output fits its part of LDS");
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    uint32_t a, b;
    swap_rows16(__float_as_uint(l_run[n]), a, b);
    float l = __uint_as_float(a) + __uint_as_float(b);
    swap_halves32(__float_as_uint(l), a, b);
    l = __uint_as_float(a) + __uint_as_float(b);
    // (16-byte chunk c of row r at c ^ (r % 16))
    if (g == 0) {
      s_ref[wave][16 * n + l16] = m_ref[n];
      s_sum[wave][16 * n + l16] = l;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<f32x4_t *>(so + (size_t)wave * (F::WAVE_B / 4) + (16 * n + l16) * D + (((4 * dt + g) ^ l16) * 4)) = o[n][dt];
  }
  __syncthreads();
  constexpr int CH = D / 8;  // threads of a row
  for (int i = t; i < TILE * CH; i += 256) {
    const int r = i / CH, ch = i % CH;
    if (r0 + r >= rows) continue;
    float ref = ninf;
#pragma unroll
    for (int w = 0; w < 4; ++w) ref = fmaxf(ref, s_ref[w][r]);
    const float fin = ref == ninf ? 0.f : ref;
    float l = 0.f;
    f32x4_t y0 = {0.f, 0.f, 0.f, 0.f}, y1 = y0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_ref[w][r] - fin);
      const float *src = so + (size_t)w * (F::WAVE_B / 4) + r * D;
      l = fmaf(s_sum[w][r], f, l);
      y0 += *reinterpret_cast<const f32x4_t *>(src + (((2 * ch) ^ (r & 15)) * 4)) * f;
      y1 += *reinterpret_cast<const f32x4_t *>(src + (((2 * ch + 1) ^ (r & 15)) * 4)) * f;
    }
    if (kSplit && parts > 1) {
      float *dst = c.part + (size_t)wk.slot * kFewPart<D, NR>;
      *reinterpret_cast<f32x4_t *>(dst + r * D + 8 * ch) = y0;
      *reinterpret_cast<f32x4_t *>(dst + r * D + 8 * ch + 4) = y1;
      if (ch == 0) {
        dst[TILE * D + r] = ref;
        dst[TILE * D + TILE + r] = l;
      }
    } else {
      const float inv = l > 0.f ? 1.f / l : 0.f;
      const Row at = row_of(c, s, wk.h, r0 + r);
      *reinterpret_cast<u32x4_t *>(c.out + at.token * c.ot + at.head * c.oh + 8 * ch) =
          u32x4_t{cvt_pk_bf16(y0[0] * inv, y0[1] * inv), cvt_pk_bf16(y0[2] * inv, y0[3] * inv),
                  cvt_pk_bf16(y1[0] * inv, y1[1] * inv), cvt_pk_bf16(y1[2] * inv, y1[3] * inv)};
      if (c.lse && ch == 0)
        c.lse[(long long)at.head * c.s.T + at.token] = l > 0.f ? (ref + log2f(l)) * 0.6931471805599453f : ninf;
    }
  }
}

// Adds up the parts of a tile of a key head: a workgroup per tile, its rows' parts dealt out to groups of D/8 threads (few
// rows have many parts), whose sums meet in LDS.
template <int D, int NR>
__global__ __launch_bounds__(kMergeThreads) void cache_attn_few_merge_kernel(const AttnCall c) {
  constexpr int TILE = 16 * NR, CH = D / 8, NG = kMergeThreads / CH;
  constexpr float ninf = -__builtin_inff();
  __shared__ float s_o[NG][D], s_ref[NG], s_sum[NG];
  const int t = threadIdx.x, lane = t & 63, item = (int)blockIdx.x;
  const int tile = item / c.H, h = item % c.H;
  const int b = seq_of_tile<TILE>(c, tile, lane), m = __builtin_amdgcn_readfirstlane(tile - tile_start<TILE>(c, b));
  const Seq s = seq_of(c, b);
  if (m < 0 || m >= tiles_of<TILE>(c, s)) return;
  const int4 it = c.items[item];
  if (it.y <= 1) return;
  const int n = min(TILE, s.n * c.G - m * TILE);  // rows
  const int grp = t / CH, ch = t % CH;
  const int gp = n >= NG ? 1 : NG / n;  // groups of a row
  const int at_once = NG / gp;
  for (int base = 0; base < n; base += at_once) {
    const int r = base + grp / gp, p0 = grp % gp;
    const bool mine = grp < at_once * gp && r < n;
    float ref = ninf, l = 0.f;
    f32x4_t y0 = {0.f, 0.f, 0.f, 0.f}, y1 = y0;
    if (mine)
      for (int p = p0; p < it.y; p += 4 * gp) {
        float ms[4], ls[4];
        f32x4_t a[4], d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float *src = c.part + (size_t)(it.x + min(p + i * gp, it.y - 1) * it.z) * kFewPart<D, NR>;
          ms[i] = src[TILE * D + r];
          ls[i] = src[TILE * D + TILE + r];
          a[i] = *reinterpret_cast<const f32x4_t *>(src + r * D + 8 * ch);
          d[i] = *reinterpret_cast<const f32x4_t *>(src + r * D + 8 * ch + 4);
        }
        const float old = ref;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (p + i * gp < it.y) ref = fmaxf(ref, ms[i]);
        const float fin = ref == ninf ? 0.f : ref;
        const float alpha = __builtin_amdgcn_exp2f(old - fin);
        l *= alpha;
        y0 *= alpha;
        y1 *= alpha;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (p + i * gp >= it.y) continue;
          const float w = __builtin_amdgcn_exp2f(ms[i] - fin);
          l = fmaf(ls[i], w, l);
          y0 += a[i] * w;
          y1 += d[i] * w;
        }
      }
    if (base) __syncthreads();
    *reinterpret_cast<f32x4_t *>(&s_o[grp][8 * ch]) = y0;
    *reinterpret_cast<f32x4_t *>(&s_o[grp][8 * ch + 4]) = y1;
    if (ch == 0) {
      s_ref[grp] = ref;
      s_sum[grp] = l;
    }
    __syncthreads();
    if (mine && p0 == 0) {
      ref = ninf;
      for (int i = 0; i < gp; ++i) ref = fmaxf(ref, s_ref[grp + i]);
      const float fin = ref == ninf ? 0.f : ref;
      l = 0.f;
      y0 = y1 = f32x4_t{0.f, 0.f, 0.f, 0.f};
      for (int i = 0; i < gp; ++i) {
        const float w = __builtin_amdgcn_exp2f(s_ref[grp + i] - fin);
        l = fmaf(s_sum[grp + i], w, l);
        y0 += *reinterpret_cast<const f32x4_t *>(&s_o[grp + i][8 * ch]) * w;
        y1 += *reinterpret_cast<const f32x4_t *>(&s_o[grp + i][8 * ch + 4]) * w;
      }
      const float inv = l > 0.f ? 1.f / l : 0.f;
      const Row at = row_of(c, s, h, m * TILE + r);
      *reinterpret_cast<u32x4_t *>(c.out + at.token * c.ot + at.head * c.oh + 8 * ch) =
          u32x4_t{cvt_pk_bf16(y0[0] * inv, y0[1] * inv), cvt_pk_bf16(y0[2] * inv, y0[3] * inv),
                  cvt_pk_bf16(y1[0] * inv, y1[1] * inv), cvt_pk_bf16(y1[2] * inv, y1[3] * inv)};
      if (c.lse && ch == 0)
        c.lse[(long long)at.head * c.s.T + at.token] = l > 0.f ? (ref + log2f(l)) * 0.6931471805599453f : ninf;
    }
  }
}

#ifndef FEW_ROWS
#define FEW_ROWS 64
#endif
// Rows a sequence and key head, on average, that this kernel is for.
bool cache_attn_few(int B, int H, int T, int Hq) { return (long long)T * (Hq / H) <= (long long)FEW_ROWS * B; }
static int row_groups(int B, int H, int T, int Hq) { return (long long)T * (Hq / H) <= 16ll * B ? 1 : 2; }

static long long few_slots(long long items) { return kFewTarget + items + kNumXcd; }

size_t cache_attn_few_workspace_bytes(int B, int H, int D, int T, int Hq) {
  if (B > kSplitSeqs) return 0;
  const int nr = row_groups(B, H, T, Hq);
  const long long items = most_items(16 * nr, B, H, T, Hq);
  if (items >= 4 * kFewTarget) return 0;
  return (size_t)items * sizeof(int4) + (size_t)few_slots(items) * 16 * nr * (D + 2) * sizeof(float);
}

template <int D, bool kCodes, int NR>
static int launch_few_t(const AttnCall &c, bool split, long long items, long long grid, int slots, hipStream_t st) {
  const int dev = current_device();
  if (dev < 0) return fail(HEART_EHIP, "heart_cache_attn: cannot identify the current device");
  constexpr int bytes = 4 * FewShape<D, kCodes>::WAVE_B;
  auto run = [&](auto kern, long long n) -> int {
    static DeviceFlags attr_set;
    if (hipError_t e = set_max_lds_once(attr_set, dev, reinterpret_cast<const void *>(kern), bytes))
      return fail(HEART_EHIP, "hipFuncSetAttribute(max dynamic LDS %d): %s", bytes, hipGetErrorString(e));
    hipLaunchKernelGGL(kern, dim3((unsigned)n), dim3(256), bytes, st, c, slots);
    return check_launch("cache_attn_few_kernel");
  };
  if (!split) return run(cache_attn_few_kernel<D, kCodes, NR, false>, items);
  if (int rc = run(cache_attn_few_kernel<D, kCodes, NR, true>, grid)) return rc;
  hipLaunchKernelGGL((cache_attn_few_merge_kernel<D, NR>), dim3((unsigned)items), dim3(kMergeThreads), 0, st, c);
  return check_launch("cache_attn_few_merge_kernel");
}

int launch_cache_attn_few(const heart_cache &hc, int T, int Hq, AttnCall &a, void *workspace, hipStream_t st) {
  const int nr = row_groups(hc.B, hc.H, T, Hq);
  const long long items = most_items(16 * nr, hc.B, hc.H, T, Hq);
  if (items > 0x7fffffffLL) return fail(HEART_EUNSUPPORTED, "heart_cache_attn: grid too large");
  // parts of a tile at most; with one there is nothing to divide
  const long long most = ((long long)a.s.cap + kFewStage * kFewMin - 1) / (kFewStage * kFewMin);
  const bool split = workspace && most > 1 && cache_attn_few_workspace_bytes(hc.B, hc.H, hc.D, T, Hq) > 0;
  const long long slots = few_slots(items);
  long long grid = 0;
  if (split) {
    a.items = (int4 *)workspace;
    a.part = (float *)(a.items + items);
    a.target = kFewTarget;
    const long long n = items * most < slots ? items * most : slots;
    grid = (n + kNumXcd - 1) / kNumXcd * kNumXcd;
  }
  const bool codes = hc.type == HEART_CACHE_E4M3;
  auto go = [&](auto d, auto n) -> int {
    constexpr int D = decltype(d)::value, NR = decltype(n)::value;
    return codes ? launch_few_t<D, true, NR>(a, split, items, grid, (int)slots, st)
                 : launch_few_t<D, false, NR>(a, split, items, grid, (int)slots, st);
  };
  const std::integral_constant<int, 128> d128;
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  if (hc.D == 128) return nr == 1 ? go(d128, one) : go(d128, two);
  return nr == 1 ? go(d64, one) : go(d64, two);
}

}  // namespace heart
