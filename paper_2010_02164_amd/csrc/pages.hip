// Block tables and slot maps of a serving step, from the requests' lengths.
//
// Everything that depends on the order of requests is a prefix sum over them:
// where a released request's pages go on the free list, and how many tokens
// and pages the requests before one take (a request is granted while both
// sums, its own share included, stay within what there is, which is a prefix
// of the requests). So one workgroup holds all requests and does one scan of
// three sums; a step is bound by its latency - lengths, scan, free list, table,
// each a trip to memory -, not by its bytes (20 a request, 12 a token). A step
// of few tokens has its slots written by the same workgroup: where each request
// has one new token by the request's thread, else each token finds its request
// by bisection of q_start in LDS; more tokens go to a second, wide kernel. 1024
// requests with a token each: 11 us; 37 with 300 to 2900: 6 and 3.
#include "serve.h"

namespace sb {
namespace {

constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64;
// Tokens that the planning workgroup writes itself (1024 tokens of 256 requests:
// 6.0 us, 7.7 with k_slots; 4096: 9.1 and 7.9).
constexpr int FUSED_TOKENS = 2 * PLAN_THREADS;

struct Sums {
  long long gone, tokens, pages;
};

struct PlanShared {
  Sums wave[PLAN_WAVES];
  unsigned long long granted_tokens, granted_pages;
  int more;   // whether a request was granted more than one token
  int need[PLAN_THREADS], first[PLAN_THREADS], held[PLAN_THREADS];
  int q_start[SB_PLAN_MAX_REQUESTS + 1];
};

// Exclusive prefix of v over the workgroup's threads; total: their sum.
__device__ __forceinline__ Sums scan_block(const Sums &v, PlanShared &sh, Sums &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  Sums x = v;
  x.gone = (long long)wave_scan((unsigned long long)x.gone);
  x.tokens = (long long)wave_scan((unsigned long long)x.tokens);
  x.pages = (long long)wave_scan((unsigned long long)x.pages);
  if (lane == 63) sh.wave[w] = x;
  __syncthreads();
  Sums before = {0, 0, 0};
  total = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < PLAN_WAVES; ++i) {
    const Sums s = sh.wave[i];
    if (i < w) {
      before.gone += s.gone;
      before.tokens += s.tokens;
      before.pages += s.pages;
    }
    total.gone += s.gone;
    total.tokens += s.tokens;
    total.pages += s.pages;
  }
  return {before.gone + x.gone - v.gone, before.tokens + x.tokens - v.tokens, before.pages + x.pages - v.pages};
}

// Slot and position of new token t; start: q_start, in LDS.
__device__ __forceinline__ void put_slot(const sb_plan_args &a, const int *start, int t) {
  const int B = a.n_requests;
  long long slot = -1;
  int pos = -1;
  if (t < start[B]) {
    int lo = 0, hi = B;   // start[lo] <= t < start[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= t) lo = mid;
      else hi = mid;
    }
    pos = a.lens_out[lo] - (start[lo + 1] - t);
    const int c = pos / a.page_size;
    const int page = a.table[(long long)lo * a.table_stride + c];
    if (page >= 0 && page < a.n_pages) slot = (long long)page * a.page_size + (pos - c * a.page_size);
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
}

// PER neighbouring requests a thread.
template <int PER>
__global__ __launch_bounds__(PLAN_THREADS) void k_plan(sb_plan_args a, int fused) {
  __shared__ PlanShared sh;
  const int B = a.n_requests, ps = a.page_size, lane = threadIdx.x & 63, b0 = threadIdx.x * PER;
  const long long room = (long long)a.max_pages * ps;
  int len[PER], want[PER], held[PER], toks[PER], need[PER];
  int page[PER];   // that a request's next token goes to, as far as it has one
  if (threadIdx.x == 0) {
    sh.granted_tokens = sh.granted_pages = 0;
    sh.more = 0;
  }
  const int free0 = min(max(*a.n_free, 0), a.n_pages);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    len[i] = b0 + i < B ? a.lens[b0 + i] : 0;
    want[i] = b0 + i < B ? a.add[b0 + i] : 0;
  }
  Sums mine = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    len[i] = (int)min((long long)max(len[i], 0), room);
    held[i] = (int)(((unsigned)len[i] + (unsigned)ps - 1u) / (unsigned)ps);
    toks[i] = want[i] > 0 && (long long)len[i] + want[i] <= room ? want[i] : 0;
    need[i] = toks[i] ? (int)(((unsigned)len[i] + (unsigned)toks[i] + (unsigned)ps - 1u) / (unsigned)ps) - held[i] : 0;
    page[i] = toks[i] && held[i] * (long long)ps > len[i] ? a.table[(long long)(b0 + i) * a.table_stride + held[i] - 1] : -1;
    mine.gone += want[i] < 0 ? held[i] : 0;
    mine.tokens += toks[i];
    mine.pages += need[i];
  }
  Sums total, at = scan_block(mine, sh, total);
  const int stack = (int)min((long long)free0 + total.gone, (long long)a.n_pages);

  // Released pages onto the free list: the wave copies one request after the
  // other, 64 pages at once.
  if (total.gone > 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int n = want[i] < 0 ? held[i] : 0;
      unsigned long long m = __ballot(n > 0);
      while (m) {
        const int src = __builtin_ctzll(m);
        m &= m - 1;
        const int b = (int)(threadIdx.x - lane + src) * PER + i, count = __shfl(n, src, 64);
        const long long to = free0 + __shfl(at.gone, src, 64);
        for (int c = lane; c < count; c += 64)
          if (to + c < a.n_pages) a.free_list[to + c] = a.table[(long long)b * a.table_stride + c];
      }
      at.gone += n;
    }
  }
  // Grants.
  int first[PER];
  long long start[PER], last_t = 0, last_p = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    start[i] = at.tokens;
    first[i] = (int)min(at.pages, (long long)stack);
    at.tokens += toks[i];
    at.pages += need[i];
    if (at.tokens <= a.token_cap && at.pages <= stack) {
      last_t = at.tokens;   // sums up to the last request that is granted
      last_p = at.pages;
    } else {
      toks[i] = need[i] = 0;
    }
  }
  // (The sums only grow, so the last granted one's are everybody's totals.)
  const unsigned long long granted = __ballot(last_t > 0);
  bool several = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) several |= toks[i] > 1;
  if (granted && lane == 63 - __builtin_clzll(granted)) {
    atomicMax(&sh.granted_tokens, (unsigned long long)last_t);
    atomicMax(&sh.granted_pages, (unsigned long long)last_p);
  }
  if (several) sh.more = 1;
  __syncthreads();   // also: the pushes are there before the pops
  const long long T = (long long)sh.granted_tokens;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = b0 + i;
    if (need[i] == 1) {   // a step of single tokens: one page here and there
      const int fresh = a.free_list[stack - 1 - first[i]];
      a.table[(long long)b * a.table_stride + held[i]] = fresh;
      if (page[i] < 0) page[i] = fresh;
    }
    if (sh.more) {
      // Several pages: a wave copies one request after the other, so neighbours
      // go to different waves (64 requests in one wave: 10 us).
      sh.need[threadIdx.x] = need[i];
      sh.first[threadIdx.x] = first[i];
      sh.held[threadIdx.x] = held[i];
      __syncthreads();
      const int e = lane * PLAN_WAVES + (int)(threadIdx.x >> 6), e_need = sh.need[e], e_first = sh.first[e], e_held = sh.held[e];
      unsigned long long m = __ballot(e_need > 1);
      while (m) {
        const int src = __builtin_ctzll(m);
        m &= m - 1;
        const int bb = (src * PLAN_WAVES + (int)(threadIdx.x >> 6)) * PER + i;
        const int n = __shfl(e_need, src, 64), f = __shfl(e_first, src, 64), h = __shfl(e_held, src, 64);
        for (int c = lane; c < n; c += 64)
          a.table[(long long)bb * a.table_stride + h + c] = a.free_list[stack - 1 - f - c];
      }
      __syncthreads();
    }
    if (b < B) {
      // The tokens asked for before it, all of which are granted if it is, or
      // all that are.
      const int q = (int)min(start[i], T);
      a.q_start[b] = q;
      if (fused) sh.q_start[b] = q;
      if (fused && !sh.more && toks[i]) {
        const bool there = page[i] >= 0 && page[i] < a.n_pages;
        a.slots[q] = there ? (long long)page[i] * ps + (unsigned)len[i] % (unsigned)ps : -1;
        a.positions[q] = len[i];
      }
      a.granted[b] = toks[i];
      a.lens_out[b] = want[i] < 0 ? 0 : len[i] + toks[i];
    }
  }
  if (threadIdx.x == 0) {
    a.q_start[B] = (int)T;
    sh.q_start[B] = (int)T;
    *a.n_free_out = stack - (int)sh.granted_pages;
  }
  if (!fused) return;
  __syncthreads();
  for (int t = threadIdx.x + (sh.more ? 0 : (int)T); t < a.token_cap; t += PLAN_THREADS) put_slot(a, sh.q_start, t);
}

constexpr int SLOT_THREADS = 256;

__global__ __launch_bounds__(SLOT_THREADS) void k_slots(sb_plan_args a) {
  extern __shared__ int start[];
  for (int b = threadIdx.x; b <= a.n_requests; b += SLOT_THREADS) start[b] = a.q_start[b];
  __syncthreads();
  const int t = blockIdx.x * SLOT_THREADS + threadIdx.x;
  if (t < a.token_cap) put_slot(a, start, t);
}

}  // namespace

hipError_t launch_plan(const sb_plan_args &a, hipStream_t s) {
  const int fused = a.token_cap <= FUSED_TOKENS;
  if (a.n_requests <= PLAN_THREADS) hipLaunchKernelGGL(k_plan<1>, dim3(1), dim3(PLAN_THREADS), 0, s, a, fused);
  else if (a.n_requests <= 2 * PLAN_THREADS) hipLaunchKernelGGL(k_plan<2>, dim3(1), dim3(PLAN_THREADS), 0, s, a, fused);
  else hipLaunchKernelGGL(k_plan<SB_PLAN_MAX_REQUESTS / PLAN_THREADS>, dim3(1), dim3(PLAN_THREADS), 0, s, a, fused);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || fused) return e;
  hipLaunchKernelGGL(k_slots, dim3((a.token_cap + SLOT_THREADS - 1) / SLOT_THREADS), dim3(SLOT_THREADS),
                     (a.n_requests + 1) * sizeof(int), s, a);
  return hipGetLastError();
}

}  // namespace sb
