// heart_cache_plan: pages, token ranges, slots and positions of a step's new tokens, from the requests' lengths.
//
// Four prefix sums over the requests say all: pages that go back, pages asked for, tokens of those whose pages are there, and
// pages and tokens of those that are granted.  One workgroup computes them, a thread a request (sums saturate: lengths may be
// anything).  What they place -- pages back on the list, pages from it into the table, a slot and a position for each token -- is
// independent, each item found by a search in the sums.
//
// Bound by latency: a chain of loads, three rounds of sums, loads from the list, stores.  A call of few tokens is one launch, one
// of many three, as items are then dealt to the chip, and pages have to be back on the list before they are taken from it.
#include "heart_internal.h"

namespace heart {

constexpr int kPlanThreads = 1024;   // of the workgroup that sums: requests at a time
constexpr int kPlanGroups = 512;     // workgroups of 256 threads that place items
constexpr int kPlanFew = 8192;       // new tokens, and
constexpr int kPlanFewPages = 1 << 16;  // places in the table, that one workgroup places alone

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

__device__ __forceinline__ int pages_of(const PlanCall &c, int tokens) { return (int)(((unsigned)tokens + (1u << c.shift) - 1u) >> c.shift); }

// Page i of those that go back: to the list, the first on top; its place in the table is empty, or will be taken.
template <typename R>
__device__ __forceinline__ void give_back(const PlanCall &c, const PlanTotals &all, uint32_t i, R &&req) {
  const int b = last_before(0, c.B - 1, i, [&](int x) { return req(x).back; });
  const PlanRequest r = req(b);
  const int p = pages_of(c, r.kept) + (int)(i - r.back);
  if (p >= r.own) return;  // (sums that saturate)
  int *at = c.table + (long long)b * c.M + p;
  const long long to = (long long)all.top - 1 - i;
  if (to >= all.free) c.list[to] = *at;
  const uint32_t next = b + 1 < c.B ? req(b + 1).taken : all.taken;
  if ((uint32_t)(p - pages_of(c, r.kept)) >= next - r.taken) *at = -1;
}
// (i < all.taken <= all.top)
__device__ __forceinline__ int page_taken(const PlanCall &c, const PlanTotals &all, uint32_t i) { return c.list[all.top - 1 - (int)i]; }
template <typename R>
__device__ __forceinline__ void take(const PlanCall &c, const PlanTotals &all, uint32_t i, R &&req) {
  const int b = last_before(0, c.B - 1, i, [&](int x) { return req(x).taken; });
  const PlanRequest r = req(b);
  c.table[(long long)b * c.M + pages_of(c, r.kept) + (int)(i - r.taken)] = page_taken(c, all, i);
}
// Token t, of one of the requests lo .. hi, or of none (t >= tokens).
template <typename R, typename C>
__device__ __forceinline__ void place(const PlanCall &c, const PlanTotals &all, int t, int tokens, int lo, int hi, R &&req, C &&cu) {
  long long slot = -1;
  int pos = -1;
  if (t < tokens) {
    const int b = last_before(lo, hi, (uint32_t)t, cu);
    const PlanRequest r = req(b);
    pos = r.kept + (t - (int)cu(b));
    const int p = pos >> c.shift, had = pages_of(c, r.kept);
    const int id = p < had ? c.table[(long long)b * c.M + p] : page_taken(c, all, r.taken + (uint32_t)(p - had));
    if ((unsigned)id < (unsigned)c.n_pages) slot = ((long long)id << c.shift) + (pos & ((1 << c.shift) - 1));
  }
  if (c.slots) c.slots[t] = slot;
  if (c.positions) c.positions[t] = pos;
}

// kAlone: of at most kPlanThreads requests, whose items the workgroup places itself.
template <bool kAlone>
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(const PlanCall c) {
  __shared__ uint32_t wave_sum[2][2][kPlanThreads / 64];
  __shared__ PlanRequest s_req[kAlone ? kPlanThreads : 1];
  __shared__ int s_cu[kAlone ? kPlanThreads + 1 : 1];
  const int t = threadIdx.x;
  const long long cap = (long long)c.M << c.shift;
  PlanSums sums{wave_sum, 0};
  const int n_free = min(max(*c.n_free, 0), c.n_pages);

  auto lengths = [&](int b, int &kept, int &own) __attribute__((always_inline)) {
    const int kv = (int)min((long long)max(c.kv_len[b], 0), cap);
    kept = c.keep ? min(max(c.keep[b], 0), kv) : kv;
    own = pages_of(c, kv);
  };
  // (more requests than threads: all that goes back first)
  uint32_t back_all = 0;
  if constexpr (!kAlone) {
    uint32_t mine[2] = {0, 0}, unused[2], all[2];
    for (int b = t; b < c.B; b += kPlanThreads) {
      int kept, own;
      lengths(b, kept, own);
      mine[0] = add_sat(mine[0], (uint32_t)(own - pages_of(c, kept)));
    }
    sums.scan(mine, unused, all);
    back_all = all[0];
  }
  uint32_t back0 = 0, need0 = 0, asked0 = 0, taken0 = 0, tokens0 = 0;  // sums over the requests before this thousand
  int top = 0;
  for (int b0 = 0; b0 < c.B; b0 += kPlanThreads) {
    const int b = b0 + t;
    int kept = 0, own = 0, want = 0;
    if (b < c.B) {
      lengths(b, kept, own);
      want = max(c.add[b], 0);
    }
    const int had = pages_of(c, kept);
    const bool fits = want > 0 && (long long)kept + want <= cap;
    uint32_t v[2] = {(uint32_t)(own - had), fits ? (uint32_t)(pages_of(c, kept + want) - had) : 0u}, before[2], all[2];
    const uint32_t need = v[1];
    sums.scan(v, before, all);
    const uint32_t back = add_sat(back0, before[0]);
    const uint32_t asked = add_sat(add_sat(need0, before[1]), need);  // with its own
    back0 = add_sat(back0, all[0]);
    need0 = add_sat(need0, all[1]);
    if constexpr (kAlone) back_all = all[0];
    top = (int)min((unsigned long long)n_free + back_all, (unsigned long long)c.n_pages);
    // pages are there
    const bool paged = fits && (need == 0 || asked <= (uint32_t)top);
    v[0] = paged ? (uint32_t)want : 0u;
    v[1] = 0;
    sums.scan(v, before, all);
    const bool given = paged && add_sat(add_sat(asked0, before[0]), (uint32_t)want) <= (uint32_t)c.T;
    asked0 = add_sat(asked0, all[0]);
    v[0] = given ? need : 0u;
    v[1] = given ? (uint32_t)want : 0u;
    sums.scan(v, before, all);
    const uint32_t taken = taken0 + before[0], first = tokens0 + before[1];
    taken0 += all[0];
    tokens0 += all[1];
    if (b < c.B) {
      const PlanRequest r{kept, own, back, taken};
      if constexpr (kAlone) {
        s_req[b] = r;
        s_cu[b] = (int)first;
      } else {
        c.req[b] = __builtin_bit_cast(int4, r);
      }
      c.cu[b] = (int)first;
      c.kv_len[b] = kept + (given ? want : 0);
    }
  }
  const PlanTotals all{n_free, top, back_all, taken0};
  if (t == 0) {
    c.cu[c.B] = (int)tokens0;
    *c.n_free = top - (int)taken0;
    if constexpr (kAlone) s_cu[c.B] = (int)tokens0;
    else c.req[c.B] = __builtin_bit_cast(int4, all);
  }
  if constexpr (kAlone) {
    __syncthreads();
    auto req = [&](int b) -> const PlanRequest & { return s_req[b]; };
    for (uint32_t i = t; i < all.back; i += kPlanThreads) give_back(c, all, i, req);
    __threadfence_block();
    __syncthreads();  // the list is whole
    for (uint32_t i = t; i < all.taken; i += kPlanThreads) take(c, all, i, req);
    for (int i = t; i < c.T; i += kPlanThreads)
      place(c, all, i, (int)tokens0, 0, c.B - 1, req, [&](int b) { return (uint32_t)s_cu[b]; });
  }
}

__global__ __launch_bounds__(256) void cache_plan_back_kernel(const PlanCall c) {
  const PlanTotals all = __builtin_bit_cast(PlanTotals, c.req[c.B]);
  auto req = [&](int b) { return __builtin_bit_cast(PlanRequest, c.req[b]); };
  const unsigned long long step = (unsigned long long)gridDim.x * 256;
  for (unsigned long long i = blockIdx.x * 256u + threadIdx.x; i < all.back; i += step) give_back(c, all, (uint32_t)i, req);
}

__global__ __launch_bounds__(256) void cache_plan_place_kernel(const PlanCall c) {
  const PlanTotals all = __builtin_bit_cast(PlanTotals, c.req[c.B]);
  auto req = [&](int b) { return __builtin_bit_cast(PlanRequest, c.req[b]); };
  auto cu = [&](int b) { return (uint32_t)c.cu[b]; };
  const uint32_t step = gridDim.x * 256, mine = blockIdx.x * 256 + threadIdx.x;
  for (unsigned long long i = mine; i < all.taken; i += step) take(c, all, (uint32_t)i, req);
  const int tokens = c.cu[c.B];
  for (long long i = mine; i < c.T; i += step) place(c, all, (int)i, tokens, 0, c.B - 1, req, cu);
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
    hipLaunchKernelGGL(cache_plan_kernel<true>, dim3(1), dim3(kPlanThreads), 0, st, c);
    return check_launch("cache_plan_kernel");
  }
  hipLaunchKernelGGL(cache_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, st, c);
  if (int rc = check_launch("cache_plan_kernel")) return rc;
  hipLaunchKernelGGL(cache_plan_back_kernel, dim3(kPlanGroups), dim3(256), 0, st, c);
  if (int rc = check_launch("cache_plan_back_kernel")) return rc;
  hipLaunchKernelGGL(cache_plan_place_kernel, dim3(kPlanGroups), dim3(256), 0, st, c);
  return check_launch("cache_plan_place_kernel");
}

}  // namespace heart
