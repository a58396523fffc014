// Which blocks a group of rows has in common, as the kernels of the attention over shared
// prefixes work it out for themselves (each from the same few numbers, in shared memory).
#pragma once

#include <limits.h>

#include "kernels.h"

// Blocks c0 .. c1 - 1 are seen whole by every live row of a group: those that the caller says are shared, up to the
// shortest row's last whole block, from the first one that lies inside every row's window. A group shares nothing
// (c1 = c0 = 0) with fewer than two live rows or fewer than `least` such blocks.
struct GroupPlan {
  int* c0;    // [N]
  int* c1;    // [N]
  int* lead;  // [N] its first live row, whose table entries stand for all
  int* last;  // [N] its last live row
};

// Position of row b's query; -1: the row sees nothing.
AXON_DEV int live_pos(const PagedAttnArgs& p, int b) {
  const int pos = p.ctx[b];
  return pos < p.blocks_per_seq * 16ll ? max(pos, -1) : -1;
}
// The group of row b; -1: none.
AXON_DEV int group_of(const SharedGroups& s, int b) {
  int lo = -1, hi = s.N - 1;  // the last group that does not begin after b
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.offsets[mid] <= b) lo = mid; else hi = mid - 1;
  }
  return lo >= 0 && b < s.offsets[lo + 1] ? lo : -1;
}
// Called by all threads of the CTA; `report`: sets the error bits.
template <int THREADS>
AXON_DEV void plan_groups(const PagedAttnArgs& p, const SharedGroups& s, const GroupPlan& g, bool report) {
  const int tid = threadIdx.x;
  bool bad = false;
  for (int i = tid; i < s.N; i += THREADS) {
    const int r0 = s.offsets[i], r1 = s.offsets[i + 1];
    bad |= r0 < 0 || r1 < r0 || r1 > p.B;
    g.c0[i] = 0;
    g.c1[i] = INT_MAX;
    g.lead[i] = INT_MAX;
    g.last[i] = -1;
  }
  if (__syncthreads_or(bad)) {
    // inconsistent offsets: nobody shares anything
    if (report && tid == 0) set_err(p.err, DEVERR_SEQ);
    for (int i = tid; i < s.N; i += THREADS) g.c0[i] = g.c1[i] = 0;
    __syncthreads();
    return;
  }
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    const int b = b0 + tid;
    const int pos = b < p.B ? live_pos(p, b) : -1;
    const int n = pos >= 0 ? group_of(s, b) : -1;
    const int lo = p.window > 0 && pos >= p.window ? pos - p.window + 1 : 0;
    const unsigned in = __ballot_sync(0xffffffffu, n >= 0);
    if (!in) continue;
    const int some = __shfl_sync(0xffffffffu, n, __ffs(in) - 1);
    if (__all_sync(0xffffffffu, n < 0 || n == some)) {
      // the usual warp: rows of one group
      const int from = __reduce_max_sync(0xffffffffu, n >= 0 ? lo : 0), to = __reduce_min_sync(0xffffffffu, n >= 0 ? pos : INT_MAX);
      const int first = __reduce_min_sync(0xffffffffu, n >= 0 ? b : INT_MAX), last = __reduce_max_sync(0xffffffffu, n >= 0 ? b : -1);
      if ((tid & 31) == 0) {
        atomicMax(&g.c0[some], from);
        atomicMin(&g.c1[some], to);
        atomicMin(&g.lead[some], first);
        atomicMax(&g.last[some], last);
      }
    } else if (n >= 0) {
      atomicMax(&g.c0[n], lo);
      atomicMin(&g.c1[n], pos);
      atomicMin(&g.lead[n], b);
      atomicMax(&g.last[n], b);
    }
  }
  __syncthreads();
  for (int i = tid; i < s.N; i += THREADS) {
    const int said = s.prefix[i];
    if (said < 0 && report) set_err(p.err, DEVERR_POS);
    int c0 = 0, c1 = 0;
    if (g.last[i] > g.lead[i] && said > 0) {
      c0 = (g.c0[i] + 15) >> 4;
      c1 = min(said >> 4, (g.c1[i] + 1) >> 4);
      if (c1 - c0 < s.least) c0 = c1 = 0;
    }
    g.c0[i] = c0;
    g.c1[i] = c1;
  }
  __syncthreads();
}
