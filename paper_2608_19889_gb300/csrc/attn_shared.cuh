// Which blocks a group of rows has in common, as the kernels of the attention over shared
// prefixes work it out for themselves (each from the same few numbers, in shared memory).
#pragma once

#include <limits.h>

#include "kernels.h"

// Blocks c0 .. c1 - 1 are seen whole by every live row of a group: those that the caller says are shared, up to the
// shortest row's last whole block, from the first one that lies inside every row's window. A group shares nothing
// (c1 = c0 = 0) with fewer than two live rows or fewer than `least` such blocks, and none does if all together spare
// fewer reads of a block than `least_spared`.
struct GroupPlan {
  int* c0;    // [N]
  int* c1;    // [N]
  int* lead;  // [N] its first live row, whose table entries stand for all
  int* live;  // [N] its live rows
  int* said;  // [N] blocks that the caller says are shared
  int* from;  // [N + 1] rows
  int* spared;  // [1]
  static constexpr int INTS = 6;  // per group, and two more
  AXON_DEV GroupPlan(int* at, int N)
      : c0(at), c1(at + N), lead(at + 2 * N), live(at + 3 * N), said(at + 4 * N), from(at + 5 * N), spared(at + 6 * N + 1) {}
};

// Position of row b's query; -1: the row sees nothing.
AXON_DEV int live_pos(const PagedAttnArgs& p, int b) {
  const int pos = p.ctx[b];
  return pos < p.blocks_per_seq * 16ll ? max(pos, -1) : -1;
}
// The group of row b; -1: none.
AXON_DEV int group_of(const GroupPlan& g, int N, int b) {
  int lo = -1, hi = N - 1;  // the last group that does not begin after b
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (g.from[mid] <= b) lo = mid; else hi = mid - 1;
  }
  return lo >= 0 && b < g.from[lo + 1] ? lo : -1;
}
// Called by the THREADS threads of the CTA from thread FIRST on, which meet at barrier 2; `report`: sets the error bits.
// Small calls wait for memory once.
template <int THREADS, int FIRST>
AXON_DEV void plan_groups(const PagedAttnArgs& p, const SharedGroups& s, const GroupPlan& g, bool report) {
  const int tid = static_cast<int>(threadIdx.x) - FIRST;
  auto meet = [] { asm volatile("barrier.cta.sync 2, %0;" ::"n"(THREADS) : "memory"); };
  int pos = tid < p.B ? live_pos(p, tid) : -1;
  bool bad = false;
  for (int i = tid; i < s.N; i += THREADS) {
    const int r0 = s.offsets[i], r1 = s.offsets[i + 1], said = s.prefix[i];
    bad |= r0 < 0 || r1 < r0 || r1 > p.B;
    if (said < 0 && report) set_err(p.err, DEVERR_POS);
    g.said[i] = said > 0 ? said >> 4 : 0;
    g.from[i] = r0;
    if (i == s.N - 1) g.from[s.N] = r1;
    g.c0[i] = 0;
    g.c1[i] = INT_MAX;
    g.lead[i] = INT_MAX;
    g.live[i] = 0;
  }
  if (tid == 0) *g.spared = 0;
  int any = 0;
  asm volatile(
      "{\n .reg .pred a, b;\n setp.ne.s32 a, %1, 0;\n barrier.cta.red.or.pred b, 2, %2, a;\n selp.s32 %0, 1, 0, b;\n}"
      : "=r"(any)
      : "r"(static_cast<int>(bad)), "n"(THREADS)
      : "memory");
  if (any) {
    // inconsistent offsets: nobody shares anything
    if (report && tid == 0) set_err(p.err, DEVERR_SEQ);
    for (int i = tid; i < s.N; i += THREADS) g.c0[i] = g.c1[i] = 0;
    meet();
    return;
  }
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    const int b = b0 + tid;
    if (b0) pos = b < p.B ? live_pos(p, b) : -1;
    const int n = pos >= 0 ? group_of(g, s.N, b) : -1;
    const int lo = p.window > 0 && pos >= p.window ? pos - p.window + 1 : 0;
    const unsigned in = __ballot_sync(0xffffffffu, n >= 0);
    if (!in) continue;
    const int some = __shfl_sync(0xffffffffu, n, __ffs(in) - 1);
    if (__all_sync(0xffffffffu, n < 0 || n == some)) {
      // the usual warp: rows of one group
      const int from = __reduce_max_sync(0xffffffffu, n >= 0 ? lo : 0), to = __reduce_min_sync(0xffffffffu, n >= 0 ? pos : INT_MAX);
      const int first = __reduce_min_sync(0xffffffffu, n >= 0 ? b : INT_MAX);
      if ((tid & 31) == 0) {
        atomicMax(&g.c0[some], from);
        atomicMin(&g.c1[some], to);
        atomicMin(&g.lead[some], first);
        atomicAdd(&g.live[some], __popc(in));
      }
    } else if (n >= 0) {
      atomicMax(&g.c0[n], lo);
      atomicMin(&g.c1[n], pos);
      atomicMin(&g.lead[n], b);
      atomicAdd(&g.live[n], 1);
    }
  }
  meet();
  for (int i = tid; i < s.N; i += THREADS) {
    int c0 = 0, c1 = 0;
    if (g.live[i] > 1 && g.said[i] > 0) {
      c0 = (g.c0[i] + 15) >> 4;
      c1 = min(g.said[i], (g.c1[i] + 1) >> 4);
      if (c1 - c0 < s.least) c0 = c1 = 0;
      if (c1 > c0) atomicAdd(g.spared, static_cast<int>(min(static_cast<long long>(c1 - c0) * (g.live[i] - 1), 1ll << 20)));
    }
    g.c0[i] = c0;
    g.c1[i] = c1;
  }
  meet();
  if (*g.spared < s.least_spared) {
    for (int i = tid; i < s.N; i += THREADS) g.c0[i] = g.c1[i] = 0;
    meet();
  }
}
// What plan_groups reports, where nobody needs the plan.
template <int THREADS>
AXON_DEV void check_groups(const PagedAttnArgs& p, const SharedGroups& s) {
  for (int i = threadIdx.x; i < s.N; i += THREADS) {
    const int r0 = s.offsets[i], r1 = s.offsets[i + 1];
    if (r0 < 0 || r1 < r0 || r1 > p.B) set_err(p.err, DEVERR_SEQ);
    if (s.prefix[i] < 0) set_err(p.err, DEVERR_POS);
  }
}
