// heart_cache_write, heart_cache_read: rows of new keys and values into the pages of their sequences, and the cached rows
// of whole sequences back.  Both move each byte once and are bound by memory, or by latency where there are few tokens.
//
// A wavefront has 16 tokens of one head, K and V.  Pages hold a multiple of 16 tokens, so 16 cached rows that start at a
// multiple of 16 lie in one page: reading needs one table entry for a wavefront, in scalar registers.  New tokens start
// anywhere, so in writing each of the first 16 lanes finds the place of one token and the others take it from there; the
// rows themselves are loaded meanwhile.  A row of D elements is held by D/8 neighbouring lanes: the maximum over a row is
// three or four lane exchanges on the VALU.
//
// us: reading 32760 tokens of 12 heads of 128 from e4m3 (303 MB in and out) 60 (5.1 TB/s, a copy of 512 MB 4.7), of 40 heads 189;
// writing 4680 tokens of 40 heads and reading them back 62; the tokens of 64 sequences 4.5.  Stores past the caches make the
// first 53, but the pooling that reads what was read back then takes 36 instead of 23.
#include "cache_device.h"

namespace heart {

constexpr int kRowsWave = 16;  // tokens of a wavefront

// Maximum over the D/8 lanes (8 or 16, aligned) that hold a row.
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = heart_op_umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));   // quad_perm [1,0,3,2]
  v = heart_op_umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));   // quad_perm [2,3,0,1]
  v = heart_op_umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));  // row_half_mirror
  if constexpr (LANES == 16)
    v = heart_op_umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false));  // row_mirror
  return v;
}

struct CacheSide {  // K or V
  const uint16_t *src;
  long long st, sh;      // token, head (bf16 elements)
  uint8_t *dst, *exp;
  long long dp, dh, dt;  // page, head, token (bytes)
};

// One row's 8 elements of a lane as codes under 2^(byte - 127).  The row's largest finite element a = 1.m * 2^(E-127) has to
// fit under 448 = 1.75 * 2^8: byte = E - 8, one more if m > 0.75; at least 1.  The product by the inverse is exact (or
// far below half the smallest code), so the conversion rounds once, to the nearest code, ties to even.
template <int LANES>
__device__ __forceinline__ u32x2_c row_codes(const u32x4_c &x, uint32_t &byte) {
  uint32_t top = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t lo = x[w] & 0x7fffu, hi = (x[w] >> 16) & 0x7fffu;
    top = heart_op_umax(top, lo < 0x7f80u ? lo : 0u);
    top = heart_op_umax(top, hi < 0x7f80u ? hi : 0u);
  }
  top = row_max<LANES>(top);
  const int e = (int)(top >> 7) - 8 + ((top & 0x7fu) > 96u ? 1 : 0);
  byte = top == 0 ? 127u : (uint32_t)(e < 1 ? 1 : e);
  const float inv = __uint_as_float((254u - byte) << 23);
  u32x2_c out;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = x[2 * p + i / 2], bits = i % 2 ? w & 0xffff0000u : w << 16;
      const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
      f[i] = finite ? __uint_as_float(bits) * inv : __uint_as_float(0x7fc00000u);
    }
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], r, true);
    out[p] = (uint32_t)r;
  }
  return out;
}

template <int D, bool kCodes>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheSide k, CacheSide v, CacheSeqs s, int H, int n_waves) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, NI = kRowsWave / RPI;
  const int lane = threadIdx.x & 63;
  const int w = (int)blockIdx.x * 4 + (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w >= n_waves) return;
  const int h = w % H, t0 = w / H * kRowsWave;  // (heads fastest: a token's rows are read together)
  const int sub = lane / LPR, col = lane % LPR;
  u32x4_c xk[NI], xv[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int t = min(t0 + i * RPI + sub, s.T - 1);
    xk[i] = *reinterpret_cast<const u32x4_c *>(k.src + t * k.st + h * k.sh + col * 8);
    xv[i] = *reinterpret_cast<const u32x4_c *>(v.src + t * v.st + h * v.sh + col * 8);
  }
  // place of token t0 + lane: sequence = number of ends that are not behind it
  const int t = t0 + lane;
  int b = 0, first = 0, n = s.per;
  if (s.cu) {
    int before = 0;
    for (int base = 0; base < s.B; base += 64) {
      const int end = base + lane < s.B ? s.cu[base + lane + 1] : 0x7fffffff;
      int mine = 0;
#pragma unroll
      for (int i = 0; i < kRowsWave; ++i) {
        const int ends = __popcll(__ballot(end <= t0 + i));
        mine = lane == i ? ends : mine;
      }
      before += mine;
    }
    b = before;
    if (b < s.B) {
      first = s.cu[b];
      n = s.cu[b + 1] - first;
    }
  } else {
    b = min(t, s.T - 1) / s.per;
    first = b * s.per;
  }
  int page = -1, off = 0;
  // (where ranges fall, the number of ends need not be that of a sequence that has the token)
  if (lane < kRowsWave && t < s.T && b < s.B && t >= first && t - first < n) {
    const long long pos = (long long)s.kv_len[b] - n + (t - first);
    if (pos >= 0 && pos < s.cap) {
      page = cache_page(s, b, (int)pos);
      off = (int)pos & ((1 << s.page_shift) - 1);
    }
  }
  const int page_size = 1 << s.page_shift;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int pg = __shfl(page, i * RPI + sub, 64), o = __shfl(off, i * RPI + sub, 64);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const CacheSide &c = side ? v : k;
      const u32x4_c &x = side ? xv[i] : xk[i];
      uint8_t *dst = c.dst + pg * c.dp + h * c.dh + o * c.dt;
      if constexpr (kCodes) {
        uint32_t byte;
        const u32x2_c y = row_codes<LPR>(x, byte);
        if (pg >= 0) {
          *reinterpret_cast<u32x2_c *>(dst + col * 8) = y;
          if (col == 0) c.exp[((long long)pg * H + h) * page_size + o] = (uint8_t)byte;
        }
      } else {
        if (pg >= 0) *reinterpret_cast<u32x4_c *>(dst + col * 16) = x;
      }
    }
  }
}

struct CacheOut {  // K or V
  const uint8_t *src, *exp;
  long long sp, sh, st;  // page, head, token (bytes)
  uint16_t *dst;
  long long db, dh, dt;  // batch, head, token (bf16 elements)
};

template <int D, bool kCodes>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheOut k, CacheOut v, CacheSeqs s, int H, int N, int tiles) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, NI = kRowsWave / RPI;
  const int lane = threadIdx.x & 63, sub = lane / LPR, col = lane % LPR;
  const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = (int)(blockIdx.x % (unsigned)tiles), bh = (int)(blockIdx.x / (unsigned)tiles);
  const int b = bh / H, h = bh % H;
  const int n0 = (tile * 4 + wave) * kRowsWave;
  const int n1 = min(min(s.kv_len[b], s.cap), N);
  if (n0 >= n1) return;
  const int page = cache_page(s, b, n0), o0 = n0 & ((1 << s.page_shift) - 1);
  u32x4_c x[2][NI];
  uint32_t byte[2][NI];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const CacheOut &c = side ? v : k;
    const uint8_t *src = c.src + (long long)max(page, 0) * c.sp + h * c.sh;
    const uint8_t *exp = kCodes ? c.exp + (((long long)max(page, 0) * H + h) << s.page_shift) : nullptr;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int o = o0 + i * RPI + sub;
      if constexpr (kCodes) {
        const u32x2_c y = *reinterpret_cast<const u32x2_c *>(src + o * c.st + col * 8);
        x[side][i] = u32x4_c{y.x, y.y, 0, 0};
        byte[side][i] = exp[o];
      } else {
        x[side][i] = *reinterpret_cast<const u32x4_c *>(src + o * c.st + col * 16);
      }
    }
  }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const CacheOut &c = side ? v : k;
    uint16_t *dst = c.dst + b * c.db + h * c.dh;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int n = n0 + i * RPI + sub;
      u32x4_c y = x[side][i];
      if constexpr (kCodes) {
        const float unit = unit_of(byte[side][i]);
        y = u32x4_c{codes_to_bf16<false>(y.x, unit), codes_to_bf16<true>(y.x, unit), codes_to_bf16<false>(x[side][i].y, unit),
                    codes_to_bf16<true>(x[side][i].y, unit)};
      }
      if (page < 0) y = u32x4_c{0, 0, 0, 0};
      if (n < n1) *reinterpret_cast<u32x4_c *>(dst + n * c.dt + col * 8) = y;
    }
  }
}

int launch_cache_write(const heart_cache &c, int T, const void *k, const long long ks[2], const void *v,
                       const long long vs[2], const int *cu_q, hipStream_t st) {
  const bool codes = c.type == HEART_CACHE_E4M3;
  const long long eb = codes ? 1 : 2, waves = ((long long)T + kRowsWave - 1) / kRowsWave * c.H;
  if (waves > 4 * kMostGroups) return fail(HEART_EUNSUPPORTED, "heart_cache_write: too many rows (T = %d, H = %d)", T, c.H);
  const CacheSide sk{(const uint16_t *)k, ks[0], ks[1], (uint8_t *)c.k, c.k_exp, c.k_stride[0] * eb, c.k_stride[1] * eb,
                     c.k_stride[2] * eb};
  const CacheSide sv{(const uint16_t *)v, vs[0], vs[1], (uint8_t *)c.v, c.v_exp, c.v_stride[0] * eb, c.v_stride[1] * eb,
                     c.v_stride[2] * eb};
  const CacheSeqs seqs = cache_seqs(c, T, cu_q);
  auto run = [&](auto kern) -> int {
    hipLaunchKernelGGL(kern, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, sk, sv, seqs, c.H, (int)waves);
    return check_launch("cache_write_kernel");
  };
  if (c.D == 128) return codes ? run(cache_write_kernel<128, true>) : run(cache_write_kernel<128, false>);
  return codes ? run(cache_write_kernel<64, true>) : run(cache_write_kernel<64, false>);
}

int launch_cache_read(const heart_cache &c, int N, void *k, const long long ks[3], void *v, const long long vs[3],
                      hipStream_t st) {
  const bool codes = c.type == HEART_CACHE_E4M3;
  const long long eb = codes ? 1 : 2, cap = (long long)c.max_pages * c.page;
  const long long tiles = ((N < cap ? N : cap) + 4 * kRowsWave - 1) / (4 * kRowsWave);
  if ((long long)c.B * c.H > kMostGroups / tiles)
    return fail(HEART_EUNSUPPORTED, "heart_cache_read: too many rows (B = %d, H = %d, N = %d)", c.B, c.H, N);
  const CacheOut ok{(const uint8_t *)c.k, c.k_exp, c.k_stride[0] * eb, c.k_stride[1] * eb, c.k_stride[2] * eb,
                    (uint16_t *)k, ks[0], ks[1], ks[2]};
  const CacheOut ov{(const uint8_t *)c.v, c.v_exp, c.v_stride[0] * eb, c.v_stride[1] * eb, c.v_stride[2] * eb,
                    (uint16_t *)v, vs[0], vs[1], vs[2]};
  const CacheSeqs seqs = cache_seqs(c, 0, nullptr);
  auto run = [&](auto kern) -> int {
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * c.B * c.H)), dim3(256), 0, st, ok, ov, seqs, c.H, N, (int)tiles);
    return check_launch("cache_read_kernel");
  };
  if (c.D == 128) return codes ? run(cache_read_kernel<128, true>) : run(cache_read_kernel<128, false>);
  return codes ? run(cache_read_kernel<64, true>) : run(cache_read_kernel<64, false>);
}

}  // namespace heart
