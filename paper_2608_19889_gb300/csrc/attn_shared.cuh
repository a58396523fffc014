// Which blocks a group of rows has in common, as the kernels of the attention over shared
// prefixes work it out for themselves (each from the same few numbers, in shared memory).
#pragma once

#include <limits.h>

#include "kernels.h"
#include "own_split.h"

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
  int* pages;   // [1] pages of the rows' own parts, of one kv head
  int* cost;    // [1] of the prefix pass
  int* rows;    // [1] rows that see something
  int* own;     // [1] SMs for the rows' own parts
  static constexpr int ints(int N) { return 6 * N + 6; }
  AXON_DEV GroupPlan(int* at, int N)
      : c0(at), c1(at + N), lead(at + 2 * N), live(at + 3 * N), said(at + 4 * N), from(at + 5 * N), spared(at + 6 * N + 1),
        pages(spared + 1), cost(spared + 2), rows(spared + 3), own(spared + 4) {}
};

// Pages of a row: `sink` pages from the front, then those from page `first` on, without the `gap` pages from
// `gap_at` on, which the row's group has in common.
struct RowPages {
  int pos, lo, sink, first, n, gap_at, gap;
};
AXON_DEV RowPages row_pages(const PagedAttnArgs& p, int pos, int2 common = make_int2(INT_MAX, INT_MAX)) {
  RowPages r;
  r.pos = pos;
  r.gap_at = common.x;
  r.gap = common.y - common.x;
  if (pos < 0) {
    r.lo = r.sink = r.first = r.n = r.gap = 0;
    return r;
  }
  r.lo = (p.window > 0 && pos >= p.window) ? pos - p.window + 1 : 0;
  r.first = r.lo >> 4;
  r.sink = min((min(p.sinks, pos + 1) + 15) >> 4, r.first);
  r.n = r.sink + (pos >> 4) + 1 - r.first - r.gap;
  return r;
}

// A group of the prefix pass: its items are `pairs` per kv head, of two tiles of PW rows; the last one may have one tile.
struct Span {
  int rows, pages, pairs;
  unsigned steps, last_cost;  // of an item; the cost of a step of the last pair, the others' is COST_TWO
  unsigned per_head;          // cost of a kv head's items
  AXON_DEV Span(int rows_, int pages_, int PW) : rows(rows_), pages(pages_) {
    pairs = (rows + 2 * PW - 1) / (2 * PW);
    steps = static_cast<unsigned>(pages + 7) >> 3;
    last_cost = rows - (pairs - 1) * 2 * PW > PW ? COST_TWO : pairs > 1 ? COST_LAST : COST_ONE;
    per_head = steps * ((pairs - 1) * COST_TWO + last_cost);
  }
  AXON_DEV unsigned cost(int pair) const { return pair == pairs - 1 ? last_cost : COST_TWO; }
  AXON_DEV unsigned item(int g, int pair) const { return g * per_head + pair * steps * COST_TWO; }
};

// The two passes run beside each other, each on SMs of its own: how many of them the rows' own parts take, so that both end
// together. An even number, or all. Called by a warp. (57 rows of 1500 to 5500 tokens, 48 of them on 4001 in common: 73.5 us,
// 99 with one pass after the other; 64 rows in groups of 4: 53 and 57.5; 64 rows on 32768 tokens: 83 and 91.)
AXON_DEV int own_sms(unsigned pages, unsigned rows, unsigned cost, int d, int sms) {
  if (cost == 0 || sms < 4) return sms;
  const unsigned own = own_work(pages, rows, d);
  unsigned best = 0xffffffffu;
#pragma unroll 1
  for (int S = 2 + 2 * (threadIdx.x & 31); S < sms; S += 64) best = min(best, split_time(own, cost, S, sms) << 10 | (1023 - S));
  return 1023 - static_cast<int>(__reduce_min_sync(0xffffffffu, best) & 1023);
}

// Position of row b's query; -1: the row sees nothing. (From L2, like all that the plan comes from: the rows' own parts start
// before the kernel in front of them has ended, and an SM's L1 may hold what was there before.)
AXON_DEV int live_pos(const PagedAttnArgs& p, int b) {
  const int pos = __ldcg(p.ctx + b);
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
// The blocks that row b has in common with others, from the first and to the last; none: both behind all.
AXON_DEV int2 common_of(const GroupPlan& g, int N, int b) {
  const int n = group_of(g, N, b);
  return n >= 0 && g.c1[n] > g.c0[n] ? make_int2(g.c0[n], g.c1[n]) : make_int2(INT_MAX, INT_MAX);
}
// Called by the THREADS threads of the CTA from thread FIRST on, which meet at barrier 2; `report`: sets the error bits.
// Small calls wait for memory once.
template <int THREADS, int FIRST>
AXON_DEV void plan_groups(const PagedAttnArgs& p, const SharedGroups& s, const GroupPlan& g, bool report) {
  const int tid = static_cast<int>(threadIdx.x) - FIRST;
  auto meet = [] { asm volatile("barrier.cta.sync 2, %0;" ::"n"(THREADS) : "memory"); };
  int pos = tid < p.B ? live_pos(p, tid) : -1;
  bool bad = false;
#pragma unroll 1
  for (int i = tid; i < s.N; i += THREADS) {
    const int r0 = __ldcg(s.offsets + i), r1 = __ldcg(s.offsets + i + 1), said = __ldcg(s.prefix + i);
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
  if (tid == 0) *g.spared = *g.pages = *g.cost = *g.rows = 0;
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
    if (tid == 0) *g.own = s.sms;
    meet();
    return;
  }
#pragma unroll 1
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    const int b = b0 + tid;
    if (b0) pos = b < p.B ? live_pos(p, b) : -1;
    const int n = pos >= 0 ? group_of(g, s.N, b) : -1;
    const int pages = __reduce_add_sync(0xffffffffu, row_pages(p, pos).n);
    const int rows = __popc(__ballot_sync(0xffffffffu, pos >= 0));
    if ((tid & 31) == 0 && rows) {
      atomicAdd(g.pages, pages);
      atomicAdd(g.rows, rows);
    }
    const int lo = p.window > 0 && pos >= p.window ? pos - p.window + 1 : 0;
    const unsigned in = __ballot_sync(0xffffffffu, n >= 0);
    if (!in) continue;
    const int some = __shfl_sync(0xffffffffu, n, __ffs(in) - 1);
    if (__all_sync(0xffffffffu, n < 0 || n == some)) {
      // the usual warp: rows of one group
      const int from = __reduce_max_sync(0xffffffffu, n >= 0 ? lo : 0);
      const int to = __reduce_min_sync(0xffffffffu, n >= 0 ? pos : INT_MAX);
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
#pragma unroll 1
  for (int i = tid; i < s.N; i += THREADS) {
    int c0 = 0, c1 = 0;
    if (g.live[i] > 1 && g.said[i] > 0) {
      c0 = (g.c0[i] + 15) >> 4;
      c1 = min(g.said[i], (g.c1[i] + 1) >> 4);
      if (c1 - c0 < s.least) c0 = c1 = 0;
      if (c1 > c0) {
        atomicAdd(g.spared, static_cast<int>(min(static_cast<long long>(c1 - c0) * (g.live[i] - 1), 1ll << 20)));
        atomicSub(g.pages, (c1 - c0) * g.live[i]);
        atomicAdd(g.cost, static_cast<int>(Span(g.from[i + 1] - g.from[i], c1 - c0, s.tile).per_head * p.G));
      }
    }
    g.c0[i] = c0;
    g.c1[i] = c1;
  }
  meet();
  const bool few = *g.spared < s.least_spared;
  if (few)
    for (int i = tid; i < s.N; i += THREADS) g.c0[i] = g.c1[i] = 0;
  if (tid < 32) {
    const int own = few ? s.sms : own_sms(static_cast<unsigned>(*g.pages) * p.G, *g.rows * p.G, *g.cost, p.d, s.sms);
    if (tid == 0) *g.own = own;
  }
  meet();
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
