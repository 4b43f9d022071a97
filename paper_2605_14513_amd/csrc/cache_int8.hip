// heart_cache_write for caches of type HEART_CACHE_INT8: rows of new keys and values as 8-bit whole numbers under a scale for
// each page and head.
//
// A scale is m 2^e with m = 4 .. 7, the least under which the block's largest element is at most 127.  Elements are bf16 (8
// significant bits), so a quotient x / s is a half of an odd number or farther than 2^-12 of its size from one: computed to the last
// bit it is rounded as the exact quotient is, and codes do not depend on how the division is done.
//
// A job is one page of a sequence that new tokens are in, one head, K or V: its rows, up to 64 KB in four wavefronts, stay in registers
// between their maximum and their codes, so each byte is moved once.  Where the page has tokens from before, its scale stays if it is
// large enough; else their codes are divided anew, which is the only case that reads them.  The jobs of a sequence start at the
// number  first / page + 2 b  (n tokens are in n / page + 2 pages at most), which every wavefront inverts on its own.
//
// Bound by memory, by latency where there are few tokens.  4680 tokens of 40 heads of 128 (144 MB in and out) 27 us, 5.3 TB/s (as a
// copy of 512 MB), with one, two or four wavefronts for a page of 64 tokens alike; one token of each of 64 sequences 4.5.
// Where all of their pages' scales grow it is as much in pages of 16 tokens, 3 more of 64, 17 more of 256 (8 heads: 34 MB read, as much written).
#include <type_traits>

#include "cache_device.h"

namespace heart {

struct BlockSide {  // K or V
  const uint16_t *src;
  long long st, sh;      // token, head (bf16 elements)
  uint8_t *dst;
  float *scale;          // [n_pages,H]
  long long dp, dh, dt;  // page, head, token (bytes)
};

__device__ __forceinline__ int job_start(const CacheSeqs &s, int b) {
  const int first = s.cu ? s.cu[b] : b * s.per;
  return (max(first, 0) >> s.page_shift) + 2 * b;
}
// The last sequence whose jobs start at or before `job`.
__device__ __forceinline__ int seq_of_job(const CacheSeqs &s, int job, int lane) {
  int lo = 0, n = s.B;  // (starts grow with b: 64 places at a time)
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const bool before = lane * step < n && at < s.B && job_start(s, at) <= job;
    const int k = max(__popcll(__ballot(before)) - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The least number of 3 significant bits with 127 of it at least `top`, the bits of a bf16 magnitude; NaN for what is not finite.
__device__ __forceinline__ float block_scale(uint32_t top) {
  if (top >= 0x7f80u) return __uint_as_float(0x7fc00000u);
  if (top == 0) return 0.f;
  const float q = __uint_as_float(top << 16) / 127.f;  // (127 m has ten bits: a quotient of three bits is exact)
  return fmaxf(__uint_as_float((__float_as_uint(q) + 0x1fffffu) & ~0x1fffffu), 1.17549435e-38f);
}

// round(x / s) as the low byte of the result: the quotient to the last bit by Markstein's method (the product with the reciprocal, corrected
// by its residual), then the sum with 1.5 * 2^23, which rounds to whole numbers, ties to even.
__device__ __forceinline__ uint32_t code_of(float x, float s, float inv) {
  const float q0 = x * inv;
  const float q = fmaf(fmaf(-q0, s, x), inv, q0);
  return __float_as_uint(q + 12582912.f);
}
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
  return ab | cd << 16;
}

// WAVES wavefronts for a job, a workgroup of 256 threads for 4 / WAVES jobs.
template <int D, int PAGE, int WAVES>
__global__ __launch_bounds__(256) void cache_write_blocks_kernel(BlockSide k, BlockSide v, CacheSeqs s, int H, int n_jobs) {
  constexpr int LPR = D / 8, RPI = 64 / LPR, ROWS = PAGE / WAVES, NI = ROWS / RPI;  // lanes of a row, rows of a load and a wavefront
  static_assert(NI >= 1 && NI * RPI * WAVES == PAGE, "a page is a whole number of loads");
  __shared__ uint32_t s_top[4];
  const int lane = threadIdx.x & 63, sub = lane / LPR, col = lane % LPR;
  const int wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = (int)blockIdx.x * (4 / WAVES) + wave / WAVES;
  if (at >= n_jobs) return;  // (all of a job's wavefronts)
  // heads fastest: a token's rows are read together
  const int rest = (int)((unsigned)at / (unsigned)H), h = at - rest * H, is_v = rest & 1, job = rest >> 1;
  const BlockSide &c = is_v ? v : k;
  const int b = seq_of_job(s, job, lane);
  const int first = s.cu ? s.cu[b] : b * s.per, n = (s.cu ? s.cu[b + 1] : first + s.per) - first;
  // (token numbers outside the call's tensors: no tokens)
  if (first < 0 || n <= 0 || (long long)first + n > s.T) return;
  const long long pos0 = (long long)s.kv_len[b] - n;  // position of the first new token, of which those below 0 are left out
  const long long p_lo = max(pos0, 0ll), p_hi = min(pos0 + n, (long long)s.cap);
  const int m = job - job_start(s, b);
  const long long lo = ((p_lo >> s.page_shift) + m) << s.page_shift;  // position of the page's first token
  if (m < 0 || lo >= p_hi) return;
  const int page = cache_page(s, b, (int)lo);
  const int o0 = (int)max(p_lo - lo, 0ll), o1 = (int)min(p_hi - lo, (long long)PAGE);  // rows of the page that are new
  const uint16_t *src = c.src + (first + (lo - pos0)) * c.st + h * c.sh + col * 8;
  const int r0 = WAVES > 1 ? wave % WAVES * ROWS : 0;
  u32x4_c x[NI];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = r0 + i * RPI + sub;
    x[i] = u32x4_c{0, 0, 0, 0};
    // (past the caches: these rows are read once, the codes that are stored here are read next.  4680 tokens of 40 heads written and
    // 9360 read back 82.7 us, 87.3 without)
    if (r >= o0 && r < o1) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_c *>(src + r * c.st));
  }
  if (page < 0) return;  // (here, so that rows are on their way meanwhile)
  float *scale_at = c.scale + ((long long)page * H + h);
  const float had = o0 > 0 ? *scale_at : 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) top = heart_op_umax(top, heart_op_umax(x[i][w] & 0x7fffu, (x[i][w] >> 16) & 0x7fffu));
  top = wave_max_u32(top);
  if constexpr (WAVES > 1) {
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = heart_op_umax(top, s_top[w]);
  }
  const float need = block_scale(top);
  const bool grows = need > had;
  const float scale = grows ? need : need != need ? need : had;  // (a NaN of the scale stays one while the page has that token)
  const bool some = scale > 0.f && scale < __builtin_inff();
  const float inv = some ? 1.f / scale : 0.f;
  uint8_t *dst = c.dst + page * c.dp + h * c.dh + col * 8;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int r = r0 + i * RPI + sub;
    u32x2_c y;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint32_t q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t w = x[i][2 * p + e / 2];
        q[e] = code_of(__uint_as_float(e % 2 ? w & 0xffff0000u : w << 16), scale, inv);
      }
      y[p] = some ? pack4(q[0], q[1], q[2], q[3]) : 0u;
    }
    if (r >= o0 && r < o1) *reinterpret_cast<u32x2_c *>(dst + r * c.dt) = y;
  }
  if (grows && o0 > 0) {
    // the codes from before, divided anew: whole numbers times one scale over the other
    for (int r = r0 + sub; r < min(r0 + ROWS, o0); r += RPI) {
      u32x2_c y = *reinterpret_cast<const u32x2_c *>(dst + r * c.dt);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint32_t q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = code_of((float)(int8_t)(y[p] >> (8 * e)) * had, scale, inv);
        y[p] = pack4(q[0], q[1], q[2], q[3]);
      }
      *reinterpret_cast<u32x2_c *>(dst + r * c.dt) = y;
    }
  }
  if ((grows || o0 == 0 || scale != scale) && lane == 0 && (WAVES == 1 || wave % WAVES == 0)) *scale_at = scale;
}

int launch_cache_write_blocks(const heart_cache &c, int T, const void *k, const long long ks[2], const void *v,
                              const long long vs[2], const int *cu_q, hipStream_t st) {
  const long long jobs = ((long long)T / c.page + 2ll * c.B) * c.H * 2;
  if (jobs > kMostGroups) return fail(HEART_EUNSUPPORTED, "heart_cache_write: too many rows (T = %d, H = %d)", T, c.H);
  const BlockSide sk{(const uint16_t *)k, ks[0], ks[1], (uint8_t *)c.k, (float *)c.k_exp, c.k_stride[0], c.k_stride[1], c.k_stride[2]};
  const BlockSide sv{(const uint16_t *)v, vs[0], vs[1], (uint8_t *)c.v, (float *)c.v_exp, c.v_stride[0], c.v_stride[1], c.v_stride[2]};
  const CacheSeqs seqs = cache_seqs(c, T, cu_q);
  auto run = [&](auto kern, int waves) -> int {
    const long long groups = (jobs * waves + 3) / 4;
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(256), 0, st, sk, sv, seqs, c.H, (int)jobs);
    return check_launch("cache_write_blocks_kernel");
  };
  auto of_page = [&](auto d) -> int {
    constexpr int D = decltype(d)::value;
    switch (c.page) {
      case 16: return run(cache_write_blocks_kernel<D, 16, 1>, 1);
      case 32: return run(cache_write_blocks_kernel<D, 32, 1>, 1);
      case 64: return run(cache_write_blocks_kernel<D, 64, 4>, 4);
      case 128: return run(cache_write_blocks_kernel<D, 128, 4>, 4);
      default: return run(cache_write_blocks_kernel<D, 256, 4>, 4);
    }
  };
  return c.D == 128 ? of_page(std::integral_constant<int, 128>{}) : of_page(std::integral_constant<int, 64>{});
}

}  // namespace heart
