// Block tables and slot maps of a serving step, from the requests' lengths.
//
// Everything that depends on the order of requests is a prefix sum over them:
// where a released request's pages go on the free list, and how many tokens
// and pages the requests before one take (a request is granted while both
// sums, its own share included, stay within what there is, which is a prefix
// of the requests). So one workgroup holds all requests, 8 a thread, and does
// three scans; a step is bound by its latency, not by its bytes (20 a request,
// 12 a token). The tokens' slots are written by a second, wide kernel, each
// token finding its request by bisection of q_start.
#include "serve.h"

namespace sb {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_PER = SB_PLAN_MAX_REQUESTS / PLAN_THREADS;

// Exclusive prefix of v over the workgroup's threads; total: their sum.
__device__ __forceinline__ long long scan_block(long long v, long long *wsum, long long &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();   // the last scan's sums have been read
  if (lane == 63) wsum[w] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < PLAN_THREADS / 64; ++i) {
    const long long s = wsum[i];
    before += i < w ? s : 0;
    all += s;
  }
  total = all;
  return before + x - v;
}

__global__ __launch_bounds__(PLAN_THREADS) void k_plan(sb_plan_args a) {
  __shared__ long long wsum[PLAN_THREADS / 64];
  __shared__ long long granted_sum[2];
  const int B = a.n_requests, ps = a.page_size, lane = threadIdx.x & 63;
  const int per = (B + PLAN_THREADS - 1) / PLAN_THREADS;
  const long long room = (long long)a.max_pages * ps;
  int len[PLAN_PER], want[PLAN_PER], held[PLAN_PER], at[PLAN_PER];
  if (threadIdx.x < 2) granted_sum[threadIdx.x] = 0;

  // Released pages, and their places on the free list.
  long long mine = 0;
#pragma unroll
  for (int i = 0; i < PLAN_PER; ++i) {
    const int b = threadIdx.x * per + i;
    const bool on = i < per && b < B;
    len[i] = on ? (int)min((long long)max(a.lens[b], 0), room) : 0;
    want[i] = on ? a.add[b] : 0;
    held[i] = (int)(((long long)len[i] + ps - 1) / ps);
    at[i] = (int)mine;
    mine += want[i] < 0 ? held[i] : 0;
  }
  const int free0 = min(max(*a.n_free, 0), a.n_pages);
  long long gone;
  long long base = scan_block(mine, wsum, gone);
#pragma unroll
  for (int i = 0; i < PLAN_PER; ++i) {
    if (i >= per) break;
    // The wave copies one released request after the other, 64 pages at once.
    unsigned long long m = __ballot(want[i] < 0 && held[i] > 0);
    while (m) {
      const int src = __builtin_ctzll(m);
      m &= m - 1;
      const int b = (int)(threadIdx.x - lane + src) * per + i;
      const int n = __shfl(held[i], src, 64);
      const long long to = free0 + __shfl(base, src, 64) + __shfl(at[i], src, 64);
      for (int c = lane; c < n; c += 64)
        if (to + c < a.n_pages) a.free_list[to + c] = a.table[(long long)b * a.table_stride + c];
    }
  }
  const int stack = (int)min((long long)free0 + gone, (long long)a.n_pages);

  // Grants: prefix sums of the tokens and pages asked for.
  int toks[PLAN_PER], need[PLAN_PER];
  long long st = 0, sp = 0;
#pragma unroll
  for (int i = 0; i < PLAN_PER; ++i) {
    toks[i] = want[i] > 0 && (long long)len[i] + want[i] <= room ? want[i] : 0;
    need[i] = toks[i] ? (int)(((long long)len[i] + toks[i] + ps - 1) / ps) - held[i] : 0;
    st += toks[i];
    sp += need[i];
  }
  long long all;
  long long bt = scan_block(st, wsum, all);   // its barriers also order the pushes before the pops
  long long bp = scan_block(sp, wsum, all);
  long long last_t = 0, last_p = 0;           // sums up to this thread's last request that is granted
  int first[PLAN_PER];
#pragma unroll
  for (int i = 0; i < PLAN_PER; ++i) {
    first[i] = 0;
    const bool fits = bt + toks[i] <= a.token_cap && bp + need[i] <= stack;
    bt += toks[i];
    bp += need[i];
    if (fits) {
      first[i] = (int)(bp - need[i]);
      last_t = bt;
      last_p = bp;
    } else {
      toks[i] = need[i] = 0;
    }
  }
  // (The sums only grow, so the largest granted one is everybody's total.)
  atomicMax(&granted_sum[0], last_t);
  atomicMax(&granted_sum[1], last_p);
  __syncthreads();
  const long long T = granted_sum[0];
#pragma unroll
  for (int i = 0; i < PLAN_PER; ++i) {
    if (i >= per) break;
    const int b = threadIdx.x * per + i;
    const bool on = b < B;
    if (!on) toks[i] = need[i] = 0;
    unsigned long long m = __ballot(need[i] > 1);
    if (on && need[i] == 1) {   // a step of single tokens: one page here and there
      a.table[(long long)b * a.table_stride + held[i]] = a.free_list[stack - 1 - first[i]];
    }
    while (m) {
      const int src = __builtin_ctzll(m);
      m &= m - 1;
      const int bb = (int)(threadIdx.x - lane + src) * per + i;
      const int n = __shfl(need[i], src, 64), f = __shfl(first[i], src, 64), h = __shfl(held[i], src, 64);
      for (int c = lane; c < n; c += 64)
        a.table[(long long)bb * a.table_stride + h + c] = a.free_list[stack - 1 - f - c];
    }
  }
  // First tokens: the sum before each request, or all of them behind the
  // last granted one.
  long long s0 = 0;
#pragma unroll
  for (int i = 0; i < PLAN_PER; ++i) s0 += toks[i];
  s0 = scan_block(s0, wsum, all);
#pragma unroll
  for (int i = 0; i < PLAN_PER; ++i) {
    const int b = threadIdx.x * per + i;
    if (i < per && b < B) {
      a.q_start[b] = (int)s0;
      s0 += toks[i];
      a.granted[b] = toks[i];
      a.lens_out[b] = want[i] < 0 ? 0 : len[i] + toks[i];
    }
  }
  if (threadIdx.x == 0) {
    a.q_start[B] = (int)T;
    *a.n_free_out = stack - (int)granted_sum[1];
  }
}

constexpr int SLOT_THREADS = 256;

__global__ __launch_bounds__(SLOT_THREADS) void k_slots(sb_plan_args a) {
  const int t = blockIdx.x * SLOT_THREADS + threadIdx.x;
  if (t >= a.token_cap) return;
  const int B = a.n_requests;
  long long slot = -1;
  int pos = -1;
  if (t < a.q_start[B]) {
    int lo = 0, hi = B;   // q_start[lo] <= t < q_start[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.q_start[mid] <= t) lo = mid;
      else hi = mid;
    }
    pos = a.lens_out[lo] - a.granted[lo] + t - a.q_start[lo];
    const int c = pos / a.page_size;
    const int page = a.table[(long long)lo * a.table_stride + c];
    if (page >= 0 && page < a.n_pages) slot = (long long)page * a.page_size + (pos - c * a.page_size);
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
}

}  // namespace

hipError_t launch_plan(const sb_plan_args &a, hipStream_t s) {
  hipLaunchKernelGGL(k_plan, dim3(1), dim3(PLAN_THREADS), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.token_cap == 0) return e;
  hipLaunchKernelGGL(k_slots, dim3((a.token_cap + SLOT_THREADS - 1) / SLOT_THREADS), dim3(SLOT_THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace sb
