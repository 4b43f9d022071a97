// heart_cache_plan: pages, token ranges, slots and positions of a step's new tokens, from the requests' lengths.
//
// Five prefix sums over the requests say all: pages that go back, pages asked for, tokens of those whose pages are there, and
// pages and tokens of those that are granted.  A workgroup computes them in three rounds (sums saturate: lengths may be
// anything).  What they place -- pages back on the list, pages from it into the table, a slot and a position for each token -- is
// independent, each item found by a search in the sums.
//
// Bound by latency: chains of loads, each of which takes a microsecond where another XCD wrote what it reads, and launches.  So
// sums that are searched lie in LDS, and there are as few launches as can be (enum PlanMode).  us: three requests 4.5, 256 with drafts
// 6.8, 1500 with 655 K tokens (8 MB out) 13.8.  More than 4096 requests: three launches, the later two of which search in memory: 6000
// with 654 K tokens 29 (4096 with as many, by two launches, 20), 6000 or 20000 with one token each 37 and 71, 20000 of which 200 or
// three get one 92 and 173 (last_before_wave).
#include <algorithm>

#include "heart_internal.h"

namespace heart {

// kAlone   few new tokens: one workgroup, one launch.
// kShared  many of not too many requests: a first launch whose workgroups all compute the sums, and give pages back; what the
//          sums come from stays as it is until the second, which places the rest.
// kLarge   more requests than a workgroup holds: sums, pages back, the rest.
enum PlanMode { kAlone, kShared, kLarge };
constexpr int kPlanThreads = 1024;   // of a workgroup that sums
constexpr int kPlanEach = 4;         // requests of a thread, where there are more than threads
constexpr int kPlanHeld = kPlanThreads * kPlanEach;  // requests that a workgroup holds
constexpr int kPlanSumGroups = 64;   // most workgroups that sum
constexpr int kPlanGroups = 2048;    // most workgroups of 256 threads that place items
// New tokens that one workgroup places alone.  us alone, shared: 8 requests of 800 tokens 5.4, 9.1, of 8000 8.8, 9.0; 256 of 4096
// 8.4, 10.6, of 8192 12.4, 11.0; 1000 of 4000 9.6, 12.2, of 8000 14.1, 12.6.
// And places in the table, all of which may go back, 1024 of them in a microsecond where one workgroup does it: 256 requests that get a
// token each 7.0, 11.1, where 16 of them end, of 282 pages each, 11.7, 12.2; 1024 of which 90 end, of 120 pages, 23.6, 14.5; all
// 2^18 pages at once 282, 15.  As many pages go back as are taken in the long run, a page a request in `page` tokens: so steps of
// many are rare, and the bound is on what the rarest takes.
constexpr int kPlanFew = 6000, kPlanFewPages = 1 << 18;

struct PlanCall {
  int B, M, shift, n_pages, T;
  const int *keep, *add;
  int *kv_len, *table, *list, *n_free, *cu, *positions;
  long long *slots;
  int4 *req;   // (many items) of each request: PlanRequest; behind them one PlanTotals
};
// tokens kept, pages at entry, pages that go back before its own, pages taken before its own
struct PlanRequest {
  int kept, own;
  uint32_t back, taken;
};
struct PlanTotals {
  int free, top;         // pages on the list at entry, and with those that go back
  uint32_t back, taken;  // all pages
};
static_assert(sizeof(PlanRequest) == sizeof(int4) && sizeof(PlanTotals) == sizeof(int4), "records of 16 bytes");

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
// inclusive prefix sum over the wavefront (wave_scan_i32)
__device__ __forceinline__ uint32_t wave_scan_sat(uint32_t v) {
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
  v = add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
  return v;
}

// Prefix sums over the workgroup of two values at a time.
struct PlanSums {
  uint32_t (*wave_sum)[2][kPlanThreads / 64];  // two rounds' worth: one barrier a round
  int round;
  // before[i]: sum over the threads before this one, all[i]: over all
  __device__ __forceinline__ void scan(const uint32_t (&v)[2], uint32_t (&before)[2], uint32_t (&all)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      incl[i] = wave_scan_sat(v[i]);
      if (lane == 63) wave_sum[round & 1][i][wave] = incl[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t s = wave_scan_sat(lane < kPlanThreads / 64 ? wave_sum[round & 1][i][lane] : 0u);
      const uint32_t here = wave ? (uint32_t)__shfl((int)s, wave - 1, 64) : 0u;
      const uint32_t prev = (uint32_t)__shfl_up((int)incl[i], 1, 64);
      before[i] = add_sat(here, lane ? prev : 0u);
      all[i] = (uint32_t)__builtin_amdgcn_readlane((int)s, 63);
    }
    ++round;
  }
};

// The last b in [lo, hi] with first(b) <= x; first(lo) <= x.
template <typename F>
__device__ __forceinline__ int last_before(int lo, int hi, uint32_t x, F &&first) {
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (first(mid) <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
// The same for x0 + lane, of all B, by the whole wavefront: 64 places at a time for x0, then the 64 requests behind that one for
// all lanes, and again 64 where that is not enough.  Few loads follow one another where most requests have items; where hardly any
// have, one for each 64 of the requests up to the last lane's, and, as lanes behind the last item look for requests too, in that
// item's wavefront up to the last request: 20000 of which three get a token take 173 us, where all get one 71.
template <typename F>
__device__ __forceinline__ int last_before_wave(int B, uint32_t x0, int lane, F &&first) {
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const bool before = lane * step < n && at < B && first(at) <= x0;
    const int k = max(__popcll(__ballot(before)) - 1, 0);
    lo += k * step;
    n = min(step, n - k * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const uint32_t x = heart_op_umin(add_sat(x0, (uint32_t)lane), 0xfffffffeu);  // (never what stands for no request)
  int b = lo;
  for (int from = lo + 1;; from += 64) {
    const uint32_t mine = from + lane < B ? first(from + lane) : 0xffffffffu;
    int k = 0;
#pragma unroll
    for (int step = 32; step; step >>= 1)
      if ((uint32_t)__shfl((int)mine, k + step - 1, 64) <= x) k += step;
    if ((uint32_t)__shfl((int)mine, k, 64) <= x) ++k;
    if (b == from - 1) b += k;  // (all that came before were passed)
    if (!__any(b == from + 63)) return b;
  }
}

__device__ __forceinline__ int pages_of(const PlanCall &c, int tokens) { return (int)(((unsigned)tokens + (1u << c.shift) - 1u) >> c.shift); }

// A request as the items need it.
struct PlanPlace {
  int kept;
  uint32_t first;  // of the items
};

// Page i of those that go back, of request b: to the list, the first on top.  (Its place in the table is empty, until it is taken.)
__device__ __forceinline__ void give_back(const PlanCall &c, int n_free, int top, uint32_t i, int b, const PlanPlace &r) {
  int *at = c.table + (long long)b * c.M + pages_of(c, r.kept) + (int)(i - r.first);
  const long long to = (long long)top - 1 - i;
  if (to >= n_free) c.list[to] = *at;
  *at = -1;
}
// (i < the pages taken <= top)
__device__ __forceinline__ int page_taken(const PlanCall &c, int top, uint32_t i) { return c.list[top - 1 - (int)i]; }
// Page i of those that are taken, of request b.
__device__ __forceinline__ void take(const PlanCall &c, int top, uint32_t i, int b, const PlanPlace &r) {
  c.table[(long long)b * c.M + pages_of(c, r.kept) + (int)(i - r.first)] = page_taken(c, top, i);
}
// Token t of request b, whose pages that are taken are those from `taken` on: its position and slot.
__device__ __forceinline__ void find_token(const PlanCall &c, int top, int t, int b, const PlanPlace &r, uint32_t taken, int &pos, long long &slot) {
  pos = r.kept + (t - (int)r.first);
  const int p = pos >> c.shift, had = pages_of(c, r.kept);
  const int id = p < had ? c.table[(long long)b * c.M + p] : page_taken(c, top, taken + (uint32_t)(p - had));
  slot = (unsigned)id < (unsigned)c.n_pages ? ((long long)id << c.shift) + (pos & ((1 << c.shift) - 1)) : -1;
}
__device__ __forceinline__ void put_token(const PlanCall &c, int t, int pos, long long slot) {
  if (c.slots) c.slots[t] = slot;
  if (c.positions) c.positions[t] = pos;
}

// EACH: requests of a thread at a time.
template <PlanMode kMode, int EACH>
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(const PlanCall c) {
  static_assert(kMode != kAlone || EACH == 1, "a thread a request");
  constexpr int CHUNK = kPlanThreads * EACH;
  __shared__ uint32_t wave_sum[2][2][kPlanThreads / 64];
  __shared__ uint32_t s_back[kMode == kLarge ? 1 : CHUNK];  // pages that go back before a request's own, pages taken, tokens
  __shared__ uint32_t s_taken[kMode == kAlone ? CHUNK : 1], s_first[kMode == kAlone ? CHUNK : 1];
  __shared__ int s_kept[kMode == kLarge ? 1 : CHUNK];
  const int t = threadIdx.x;
  const bool writes = kMode == kAlone || blockIdx.x == 0;  // (the others compute the same)
  const long long cap = (long long)c.M << c.shift;
  PlanSums sums{wave_sum, 0};
  const int n_free = min(max(*c.n_free, 0), c.n_pages);

  auto lengths = [&](int b, int &kept, int &own) __attribute__((always_inline)) {
    const int kv = (int)min((long long)max(c.kv_len[b], 0), cap);
    kept = c.keep ? min(max(c.keep[b], 0), kv) : kv;
    own = pages_of(c, kv);
  };
  // (more requests than the workgroup holds: all that goes back first)
  uint32_t back_all = 0;
  if constexpr (kMode == kLarge) {
    uint32_t mine[2] = {0, 0}, unused[2], all[2];
    for (int b = t; b < c.B; b += kPlanThreads) {
      int kept, own;
      lengths(b, kept, own);
      mine[0] = add_sat(mine[0], (uint32_t)(own - pages_of(c, kept)));
    }
    sums.scan(mine, unused, all);
    back_all = all[0];
  }
  uint32_t back0 = 0, need0 = 0, asked0 = 0, taken0 = 0, tokens0 = 0;  // sums over the requests before this chunk
  int top = 0;
  for (int b0 = 0; b0 < c.B; b0 += CHUNK) {
    const int b = b0 + t * EACH;  // (the thread's first)
    int kept[EACH], own[EACH], want[EACH];
    uint32_t need[EACH], v[2] = {0, 0}, before[2], all[2];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      kept[e] = own[e] = want[e] = 0;
      if (b + e < c.B) {
        lengths(b + e, kept[e], own[e]);
        want[e] = max(c.add[b + e], 0);
      }
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int had = pages_of(c, kept[e]);
      if ((long long)kept[e] + want[e] > cap) want[e] = 0;  // (does not fit the table)
      need[e] = (uint32_t)(pages_of(c, kept[e] + want[e]) - had);
      v[0] = add_sat(v[0], (uint32_t)(own[e] - had));
      v[1] = add_sat(v[1], need[e]);
    }
    sums.scan(v, before, all);
    uint32_t back = add_sat(back0, before[0]), asked = add_sat(need0, before[1]);
    back0 = add_sat(back0, all[0]);
    need0 = add_sat(need0, all[1]);
    if constexpr (kMode != kLarge) back_all = all[0];
    top = (int)min((unsigned long long)n_free + back_all, (unsigned long long)c.n_pages);
    // pages are there, or none are needed
    v[0] = v[1] = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      asked = add_sat(asked, need[e]);
      if (need[e] > 0 && asked > (uint32_t)top) want[e] = 0;
      v[0] = add_sat(v[0], (uint32_t)want[e]);
    }
    sums.scan(v, before, all);
    uint32_t tokens = add_sat(asked0, before[0]);
    asked0 = add_sat(asked0, all[0]);
    v[0] = v[1] = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      tokens = add_sat(tokens, (uint32_t)want[e]);
      if (tokens > (uint32_t)c.T) want[e] = 0;
      if (want[e] == 0) need[e] = 0;
      v[0] += need[e];
      v[1] += (uint32_t)want[e];
    }
    sums.scan(v, before, all);
    uint32_t taken = taken0 + before[0], first = tokens0 + before[1];
    taken0 += all[0];
    tokens0 += all[1];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      if (b + e >= c.B) break;
      if constexpr (kMode != kLarge) {
        s_back[b + e] = back;
        s_kept[b + e] = kept[e];
      }
      if constexpr (kMode == kAlone) {
        s_taken[b] = taken;
        s_first[b] = first;
        c.kv_len[b] = kept[e] + want[e];
      } else if (writes) {
        c.req[b + e] = __builtin_bit_cast(int4, PlanRequest{kept[e], own[e], back, taken});
      }
      if (writes) c.cu[b + e] = (int)first;
      back = add_sat(back, (uint32_t)(own[e] - pages_of(c, kept[e])));
      taken += need[e];
      first += (uint32_t)want[e];
    }
  }
  if (writes && t == 0) {
    c.cu[c.B] = (int)tokens0;
    if constexpr (kMode == kAlone) *c.n_free = top - (int)taken0;
    else c.req[c.B] = __builtin_bit_cast(int4, PlanTotals{n_free, top, back_all, taken0});
  }
  if constexpr (kMode != kLarge) {
    __syncthreads();
    const unsigned long long step = (unsigned long long)gridDim.x * kPlanThreads;
    for (unsigned long long i = blockIdx.x * (unsigned long long)kPlanThreads + t; i < back_all; i += step) {
      const int b = last_before(0, c.B - 1, (uint32_t)i, [&](int x) { return s_back[x]; });
      give_back(c, n_free, top, (uint32_t)i, b, PlanPlace{s_kept[b], s_back[b]});
    }
  }
  if constexpr (kMode == kAlone) {
    __threadfence_block();
    __syncthreads();  // the list is whole, and places that are taken are empty
    for (uint32_t i = t; i < taken0; i += kPlanThreads) {
      const int b = last_before(0, c.B - 1, i, [&](int x) { return s_taken[x]; });
      take(c, top, i, b, PlanPlace{s_kept[b], s_taken[b]});
    }
    for (int i = t; i < c.T; i += 2 * kPlanThreads) {
      int pos[2] = {-1, -1};
      long long slot[2] = {-1, -1};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int x = i + e * kPlanThreads;
        if (x < (int)tokens0) {
          const int b = last_before(0, c.B - 1, (uint32_t)x, [&](int y) { return s_first[y]; });
          find_token(c, top, x, b, PlanPlace{s_kept[b], s_first[b]}, s_taken[b], pos[e], slot[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (i + e * kPlanThreads < c.T) put_token(c, i + e * kPlanThreads, pos[e], slot[e]);
    }
  }
}

__device__ __forceinline__ PlanRequest plan_request(const PlanCall &c, int b) { return __builtin_bit_cast(PlanRequest, c.req[b]); }

__global__ __launch_bounds__(256) void cache_plan_back_kernel(const PlanCall c) {
  const PlanTotals all = __builtin_bit_cast(PlanTotals, c.req[c.B]);
  const int lane = threadIdx.x & 63;
  const unsigned long long step = (unsigned long long)gridDim.x * 256;
  for (unsigned long long i = blockIdx.x * 256u + (threadIdx.x & ~63u); i < all.back; i += step) {
    const int b = last_before_wave(c.B, (uint32_t)i, lane, [&](int x) { return plan_request(c, x).back; });
    const PlanRequest r = plan_request(c, b);
    if (i + lane < all.back) give_back(c, all.free, all.top, (uint32_t)i + lane, b, PlanPlace{r.kept, r.back});
  }
}

// Pages taken and lengths (the first `takers` workgroups), and tokens.  kHeld: of at most kPlanHeld requests, whose sums are
// searched in LDS.
template <bool kHeld>
__global__ __launch_bounds__(256) void cache_plan_place_kernel(const PlanCall c, int takers) {
  __shared__ uint32_t s_first[kHeld ? kPlanHeld : 1];
  const PlanTotals all = __builtin_bit_cast(PlanTotals, c.req[c.B]);
  const int lane = threadIdx.x & 63;
  const bool takes = (int)blockIdx.x < takers;
  const uint32_t group = takes ? blockIdx.x : blockIdx.x - takers, step = (takes ? takers : gridDim.x - takers) * 256u;
  const uint32_t mine = group * 256 + (threadIdx.x & ~63u);
  auto sum = [&](int b) { return takes ? plan_request(c, b).taken : (uint32_t)c.cu[b]; };
  if constexpr (kHeld) {
#pragma unroll 4
    for (int b = threadIdx.x; b < c.B; b += 256) s_first[b] = sum(b);
    __syncthreads();
  }
  // the request of item i + lane (i below `n`)
  auto request = [&](uint32_t i, uint32_t n, uint32_t &first) __attribute__((always_inline)) -> int {
    if constexpr (kHeld) {
      const int b = last_before(0, c.B - 1, heart_op_umin(i + lane, n - 1), [&](int x) { return s_first[x]; });
      first = s_first[b];
      return b;
    } else {
      const int b = last_before_wave(c.B, i, lane, sum);
      first = sum(b);
      return b;
    }
  };
  if (takes) {
    for (unsigned long long i = mine; i < all.taken; i += step) {
      uint32_t first;
      const int b = request((uint32_t)i, all.taken, first);
      if (i + lane < all.taken) take(c, all.top, (uint32_t)i + lane, b, PlanPlace{plan_request(c, b).kept, first});
    }
    for (unsigned long long b = mine + lane; b < (unsigned)c.B; b += step)
      c.kv_len[b] = plan_request(c, (int)b).kept + (c.cu[b + 1] - c.cu[b]);
    if (mine + lane == 0) *c.n_free = all.top - (int)all.taken;
    return;
  }
  // (two tokens of a thread at a time: what they load is on its way together)
  const uint32_t tokens = (uint32_t)c.cu[c.B];
  constexpr int N = 2;
  for (unsigned long long i0 = mine; i0 < (unsigned)c.T; i0 += (unsigned long long)N * step) {
    int pos[N];
    long long slot[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const uint32_t i = (uint32_t)i0 + e * step;  // (at most 2^30 and two steps)
      pos[e] = -1;
      slot[e] = -1;
      if (i < tokens) {
        uint32_t first;
        const int b = request(i, tokens, first);
        const PlanRequest r = plan_request(c, b);
        if (i + lane < tokens) find_token(c, all.top, (int)i + lane, b, PlanPlace{r.kept, first}, r.taken, pos[e], slot[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const uint32_t x = (uint32_t)i0 + e * step + lane;
      if (x < (uint32_t)c.T) put_token(c, (int)x, pos[e], slot[e]);
    }
  }
}

static bool plan_alone(int B, int max_pages, int T) {
  return B <= kPlanThreads && T <= kPlanFew && (long long)B * max_pages <= kPlanFewPages;
}

size_t cache_plan_workspace_bytes(int B, int max_pages, int T) {
  return plan_alone(B, max_pages, T) ? 0 : ((size_t)B + 1) * sizeof(int4);
}

int launch_cache_plan(int B, int max_pages, int page, int n_pages, int T, const int *keep, const int *add, int *kv_len,
                      int *page_table, int *free_pages, int *n_free, int *cu_q, long long *slots, int *positions, void *workspace,
                      hipStream_t st) {
  const PlanCall c{B, max_pages, __builtin_ctz((unsigned)page), n_pages, T, keep, add, kv_len, page_table, free_pages, n_free, cu_q,
                   positions, slots, (int4 *)workspace};
  if (plan_alone(B, max_pages, T)) {
    hipLaunchKernelGGL((cache_plan_kernel<kAlone, 1>), dim3(1), dim3(kPlanThreads), 0, st, c);
    return check_launch("cache_plan_kernel");
  }
  // (what the items are at most, as far as it is known here)
  auto groups = [](long long items, int each, int most) { return dim3((unsigned)std::min((items + each - 1) / each, (long long)most)); };
  const long long back = std::min((long long)n_pages, (long long)B * max_pages);
  const dim3 take = groups(std::max((long long)B, std::min(back, (long long)T / page + B)), 256, kPlanSumGroups);
  const dim3 place(take.x + groups((T + 1ll) / 2, 256, kPlanGroups).x);
  if (B <= kPlanHeld) {
    hipLaunchKernelGGL((cache_plan_kernel<kShared, kPlanEach>), groups(back, kPlanThreads, kPlanSumGroups), dim3(kPlanThreads), 0, st, c);
    if (int rc = check_launch("cache_plan_kernel")) return rc;
    hipLaunchKernelGGL(cache_plan_place_kernel<true>, place, dim3(256), 0, st, c, (int)take.x);
    return check_launch("cache_plan_place_kernel");
  }
  hipLaunchKernelGGL((cache_plan_kernel<kLarge, kPlanEach>), dim3(1), dim3(kPlanThreads), 0, st, c);
  if (int rc = check_launch("cache_plan_kernel")) return rc;
  hipLaunchKernelGGL(cache_plan_back_kernel, groups(back, 256, kPlanGroups), dim3(256), 0, st, c);
  if (int rc = check_launch("cache_plan_back_kernel")) return rc;
  hipLaunchKernelGGL(cache_plan_place_kernel<false>, place, dim3(256), 0, st, c, (int)take.x);
  return check_launch("cache_plan_place_kernel");
}

}  // namespace heart
