// Page tables on the device: pages given back and given out as all sequences go to their next lengths, and where the rows of the next call lie.
//
// Integers only.  Prefix sums over the sequences say for each how many pages lie in front of its own among those given back and asked for, so every page
// and every row is then found on its own: the j-th page given out comes from place there - 1 - j of the stack, where it was before, or, above that,
// is the r-th one given back, looked up in the table that it leaves.  Nothing is read that the same step writes.
//
// Where rows and sequences are few one workgroup does everything, a sequence a thread, with all sums in LDS: latency is all that counts there.  Else one workgroup
// takes the sums, and a second launch moves pages and places rows with as many threads as there are.
#include "common.h"
#include "kernels.h"

namespace covspec {

namespace {

constexpr int PT = 1024;
constexpr int kFewSeq = 1024, kFewRows = 4096;   // one workgroup does everything

// Exclusive prefix sums of two numbers a thread over a workgroup, and their totals.
struct Two { long a, b; };
__device__ __forceinline__ Two exscan2(Two v, Two* waves, Two* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  Two inc = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long x = __shfl_up(inc.a, o, 64), y = __shfl_up(inc.b, o, 64);
    if (lane >= o) { inc.a += x; inc.b += y; }
  }
  __syncthreads();                               // the sums of an earlier call have been read
  if (lane == 63) waves[w] = inc;
  __syncthreads();
  Two before = {0, 0}, all = {0, 0};
#pragma unroll
  for (int k = 0; k < PT / 64; ++k) {
    const Two x = waves[k];
    if (k < w) { before.a += x.a; before.b += x.b; }
    all.a += x.a;
    all.b += x.b;
  }
  *total = all;
  return Two{before.a + inc.a - v.a, before.b + inc.b - v.b};
}

// What the sums leave: for each sequence the first page it gives back and what it held, how many given back and asked for lie in front of its
// own; [S]: the totals.  asked -1: nothing is given to it.
struct Plan {
  int *keep, *held, *given, *asked, *scalars;    // scalars: the stack's height before, pages given back, behind both, behind the step
};
__host__ __device__ inline Plan plan_at(int* ws, int S) { return Plan{ws, ws + S, ws + 2 * S, ws + 3 * S + 1, ws + 4 * S + 1}; }

__device__ __forceinline__ int between(int v, int lo, int hi) { return min(max(v, lo), hi); }

// First index of v[0 .. n] whose value is beyond x, less one.
__device__ __forceinline__ int last_not_beyond(const int* v, int n, int x) {
  int lo = 0, hi = n + 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (v[mid] <= x) lo = mid + 1; else hi = mid;
  }
  return lo - 1;
}

struct Sums { int before, given, there, after; };
// The j-th page that is given out.
__device__ __forceinline__ int page_given(const Pages& p, const Plan& pl, const Sums& u, int j) {
  const int at = u.there - 1 - j;
  if (at < u.before) return p.free_pages[at];
  const int r = u.before + u.given - 1 - at;      // in the order of the sequences
  const int s = last_not_beyond(pl.given, p.S - 1, r);
  return p.pages[(long)s * p.max_pages + pl.keep[s] + (r - pl.given[s])];
}

// Pages of sequence s that move, by `threads` threads.
__device__ __forceinline__ void move_pages(const Pages& p, const Plan& pl, const Sums& u, int s, int thread, int threads) {
  const int held = pl.held[s], keep = pl.keep[s], given = pl.given[s], back = pl.given[s + 1] - given, asked = pl.asked[s];
  int* const row = p.pages + (long)s * p.max_pages;
  for (int i = thread; i < back; i += threads) {
    const int at = u.before + u.given - 1 - (given + i);
    if (at < u.after) p.free_pages[at] = row[keep + i];
  }
  if (asked >= 0)
    for (int i = thread; i < keep - held; i += threads) row[held + i] = page_given(p, pl, u, asked + i);      // keep: what it will hold
}

__device__ __forceinline__ void place_row(const Pages& p, const Plan& pl, const Sums& u, const int* start, const int* length, int total, int t) {
  long slot = -1;
  int pos = -1;
  if (t < total) {
    const int s = last_not_beyond(start, p.S, t);
    pos = length[s] - start[s + 1] + t;
    const int at = pos >> p.page_shift, held = pl.held[s];
    int page = -1;
    if (at >= held) {
      if (pl.asked[s] >= 0) page = page_given(p, pl, u, pl.asked[s] + at - held);
    } else {
      page = p.pages[(long)s * p.max_pages + at];
    }
    if (page >= 0 && page < p.n_pages) slot = ((long)page << p.page_shift) | (pos & ((1 << p.page_shift) - 1));
  }
  if (p.slots) p.slots[t] = slot;
  if (p.positions) p.positions[t] = pos;
}

__global__ __launch_bounds__(PT) void pages_plan_kernel(Pages p, int* __restrict__ ws) {
  __shared__ Two waves[PT / 64];
  __shared__ int most;                           // rows that have room: those up to the first sequence whose rows do not fit
  const Plan pl = plan_at(ws, p.S);
  const int tid = threadIdx.x;
  if (tid == 0) most = 0;
  // pages given back and asked for
  Two carry = {0, 0}, total;
  for (int s0 = 0; s0 < p.S; s0 += PT) {
    const int s = s0 + tid;
    int back = 0, asks = 0;
    if (s < p.S) {
      const int held = between(p.held[s], 0, p.max_pages), need = (int)(((long)max(p.want[s], 0) + (1 << p.page_shift) - 1) >> p.page_shift);
      const int goal = need <= p.max_pages ? need : held, keep = max(goal, between(p.borrowed[s], 0, held));
      back = max(held - keep, 0);
      asks = max(goal - held, 0);
      pl.keep[s] = keep;
      pl.held[s] = held;
    }
    const Two at = exscan2(Two{back, asks}, waves, &total);
    if (s < p.S) {
      pl.given[s] = (int)(carry.a + at.a);
      pl.asked[s] = (int)(carry.b + at.b);
    }
    carry.a += total.a;
    carry.b += total.b;
  }
  Sums u;
  u.before = between(p.n_free[0], 0, p.n_pages);
  u.given = (int)carry.a;
  u.there = min(u.before + u.given, p.n_pages);
  // who is served, and rows
  const int capacity = p.T;
  long rows_before = 0, taken = 0;
  for (int s0 = 0; s0 < p.S; s0 += PT) {
    const int s = s0 + tid;
    int want = 0, rows = 0, held = 0, now = 0, asks = 0;
    bool fits = false, served = false;
    if (s < p.S) {
      want = max(p.want[s], 0);
      rows = between(p.rows[s], 0, want);
      held = pl.held[s];
      const int need = (int)(((long)want + (1 << p.page_shift) - 1) >> p.page_shift);
      fits = need <= p.max_pages;
      asks = fits ? max(need - held, 0) : 0;
      served = asks == 0 || pl.asked[s] + asks <= u.there;
      now = !fits || !served ? held : need;
    }
    const int n = fits && served ? rows : 0;
    const Two at = exscan2(Two{n, served ? asks : 0}, waves, &total);
    if (s < p.S) {
      const long upto = rows_before + at.a + n;
      const bool room = n == 0 || upto <= capacity;
      const bool ok = fits && served;
      if (upto <= capacity) atomicMax(&most, (int)upto);
      p.outcome[s] = ok ? room ? 0 : 2 : 1;
      p.length[s] = ok && room ? want : (int)min((long)want - rows, (long)now << p.page_shift);
      p.start[s + 1] = (int)min(upto, (long)capacity + 1);            // beyond `most`: none, below
      if (asks == 0 || !served) pl.asked[s] = -1;
      p.borrowed[s] = between(p.borrowed[s], 0, now);
      p.held[s] = now;
    }
    rows_before += total.a;
    taken += total.b;
  }
  u.after = u.there - (int)taken;
  __syncthreads();
  const int filled = most;
  for (int s = tid; s < p.S; s += PT)
    if (p.start[s + 1] > filled) p.start[s + 1] = filled;
  if (tid == 0) {
    p.start[0] = 0;
    p.n_free[0] = u.after;
    pl.given[p.S] = u.given;
    pl.scalars[0] = u.before;
    pl.scalars[1] = u.given;
    pl.scalars[2] = u.there;
    pl.scalars[3] = u.after;
  }
}

// Exclusive sums of two numbers a thread, and their totals; fewer than 2^31 in all.  `sums` is used by no other call.
struct Two32 { int a, b; };
__device__ __forceinline__ Two32 exscan2_32(Two32 v, Two32* sums, Two32* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int a = wave_inscan(v.a), b = wave_inscan(v.b);
  if (lane == 63) sums[w] = Two32{a, b};
  __syncthreads();
  const Two32 mine = lane < PT / 64 ? sums[lane] : Two32{0, 0};
  const int ups_a = wave_inscan(mine.a), ups_b = wave_inscan(mine.b);
  *total = Two32{__builtin_amdgcn_readlane(ups_a, PT / 64 - 1), __builtin_amdgcn_readlane(ups_b, PT / 64 - 1)};
  const int at = __builtin_amdgcn_readfirstlane(w);
  return Two32{__builtin_amdgcn_readlane(ups_a - mine.a, at) + a - v.a, __builtin_amdgcn_readlane(ups_b - mine.b, at) + b - v.b};
}

// ALL: pages and rows as well; else the sums go to the workspace, as those of pages_plan_kernel.
template <bool ALL>
__global__ __launch_bounds__(PT) void pages_few_kernel(Pages p, int* __restrict__ ws) {
  __shared__ Two32 sums[2][PT / 64];
  __shared__ int keep_of[kFewSeq], held_of[kFewSeq], given_of[kFewSeq + 1], asked_of[kFewSeq], length_of[kFewSeq], start_of[kFewSeq + 1], filled;
  const int s = threadIdx.x;
  const bool real = s < p.S;
  int want = 0, rows = 0, held = 0, borrowed = 0;
  if (real) {
    want = max(p.want[s], 0);
    rows = between(p.rows[s], 0, want);
    held = between(p.held[s], 0, p.max_pages);
    borrowed = between(p.borrowed[s], 0, held);
  }
  Sums u;
  u.before = between(p.n_free[0], 0, p.n_pages);
  const int need = (int)(((long)want + (1 << p.page_shift) - 1) >> p.page_shift);
  const bool fits = need <= p.max_pages;
  const int goal = fits ? need : held, keep = max(goal, borrowed), back = max(held - keep, 0), asks = max(goal - held, 0);
  Two32 total;
  const Two32 front = exscan2_32(Two32{back, asks}, sums[0], &total);
  u.given = total.a;
  u.there = min(u.before + u.given, p.n_pages);
  const bool served = asks == 0 || front.b + asks <= u.there, ok = fits && served;
  const int now = ok ? need : held, n = ok ? min(rows, p.T + 1) : 0;                   // 2^10 (2^20 + 1) rows at most
  const Two32 ahead = exscan2_32(Two32{n, served ? asks : 0}, sums[1], &total);
  u.after = u.there - total.b;
  const int upto = ahead.a + n;
  const bool room = n == 0 || upto <= p.T;
  if (s == 0) { filled = 0; start_of[0] = 0; given_of[p.S] = u.given; }
  __syncthreads();
  if (real && upto <= p.T) atomicMax(&filled, upto);
  __syncthreads();
  const Plan to = plan_at(ws, p.S);
  if (real) {
    const int start = min(upto, filled), length = ok && room ? want : (int)min((long)want - rows, (long)now << p.page_shift), asked = asks > 0 && served ? front.b : -1;
    if constexpr (ALL) {
      keep_of[s] = keep;
      held_of[s] = held;
      given_of[s] = front.a;
      asked_of[s] = asked;
      length_of[s] = length;
      start_of[s + 1] = start;
    } else {
      to.keep[s] = keep;
      to.held[s] = held;
      to.given[s] = front.a;
      to.asked[s] = asked;
    }
    p.outcome[s] = ok ? room ? 0 : 2 : 1;
    p.length[s] = length;
    p.start[s + 1] = start;
    p.held[s] = now;
    p.borrowed[s] = min(borrowed, now);
  }
  if (s == 0) {
    p.start[0] = 0;
    p.n_free[0] = u.after;
    if constexpr (!ALL) {
      to.given[p.S] = u.given;
      to.scalars[0] = u.before;
      to.scalars[1] = u.given;
      to.scalars[2] = u.there;
      to.scalars[3] = u.after;
    }
  }
  if constexpr (ALL) {
    __syncthreads();
    const Plan pl = {keep_of, held_of, given_of, asked_of, nullptr};
    for (int t = threadIdx.x; t < p.T; t += PT) place_row(p, pl, u, start_of, length_of, filled, t);
    for (int i = threadIdx.x >> 4; i < p.S; i += PT / 16) move_pages(p, pl, u, i, threadIdx.x & 15, 16);
  }
}

constexpr int MT = 256;
__global__ __launch_bounds__(MT) void pages_move_kernel(Pages p, int* __restrict__ ws, int row_groups) {
  const Plan pl = plan_at(ws, p.S);
  const Sums u = {pl.scalars[0], pl.scalars[1], pl.scalars[2], pl.scalars[3]};
  if ((int)blockIdx.x < row_groups) {
    // where the sequences begin is looked up in LDS, where a step of the search takes a fifth of the time
    __shared__ int starts[kFewSeq + 1];
    const int total = p.start[p.S];
    const bool near = p.S <= kFewSeq && (int)(blockIdx.x * MT) < total;
    if (near) {
      for (int s = threadIdx.x; s <= p.S; s += MT) starts[s] = p.start[s];
      __syncthreads();
    }
    const int* const start = near ? starts : p.start;
    const int t = blockIdx.x * MT + threadIdx.x;
    if (t < p.T) place_row(p, pl, u, start, p.length, total, t);
  } else {
    const int s = (blockIdx.x - row_groups) * (MT / 64) + threadIdx.x / 64;
    if (s < p.S) move_pages(p, pl, u, s, threadIdx.x & 63, 64);
  }
}

}  // namespace

size_t pages_workspace_bytes(int S) { return ((size_t)4 * S + 1 + 4) * sizeof(int); }

hipError_t launch_pages(const Pages& p, void* ws, hipStream_t stream) {
  if (p.S <= kFewSeq && p.T <= kFewRows) {
    hipLaunchKernelGGL(pages_few_kernel<true>, dim3(1), dim3(PT), 0, stream, p, (int*)ws);
    return hipGetLastError();
  }
  if (p.S <= kFewSeq && p.T <= 1 << 20)          // sums of 2^10 of these stay below 2^31
    hipLaunchKernelGGL(pages_few_kernel<false>, dim3(1), dim3(PT), 0, stream, p, (int*)ws);
  else
    hipLaunchKernelGGL(pages_plan_kernel, dim3(1), dim3(PT), 0, stream, p, (int*)ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int row_groups = p.slots || p.positions ? (p.T + MT - 1) / MT : 0;
  hipLaunchKernelGGL(pages_move_kernel, dim3(row_groups + (p.S + MT / 64 - 1) / (MT / 64)), dim3(MT), 0, stream, p, (int*)ws, row_groups);
  return hipGetLastError();
}

}  // namespace covspec
