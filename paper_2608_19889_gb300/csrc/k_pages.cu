// Blocks of the paged cache: copied, shared between rows, taken, given back and
// moved together, all in stream order on the device.
//
// State (the caller's): a table [R][P] of block numbers (-1: none), the tokens
// ctx[r] that row r holds, and refs[b], the table entries that name block b; a block
// is free when refs is 0. Free blocks are handed out lowest number first, so that
// every result is determined by the state alone.
//
// Tables and counts are latency: chains of dependent loads over a few hundred KB.
// One cluster of eight CTAs ranks the free blocks, each CTA a contiguous
// range of them, with hardware barriers between its phases in place of launches (a launch costs
// the host about 2.2 us, a phase of the cluster about 1); what touches block contents is a second
// launch over the whole GPU. Copies are bound by HBM: every byte is read and written
// once, a warp moving 2 KB with four 16-byte loads per lane in flight. Measured (GPU time in a
// captured row of calls): a fork of four rows 7.4 us, a reservation of 7 rows among 724 blocks 5.6
// and of 448 rows among 93,952 blocks 16.4 (rows are compared with each other, and the blocks
// ranked); 1.57 GB read and written by a compaction in 239 us, 6.6 TB/s, 97 % of the copy bandwidth.
#include <cooperative_groups.h>
#include <math.h>

#include "kernels.h"

namespace cg = cooperative_groups;

namespace {

constexpr int CL = 8;      // CTAs of the cluster
constexpr int MT = 1024;   // their threads
constexpr int CT = 256;    // threads of the other kernels
constexpr int TILE = 2048; // bytes that a warp copies at a time

// Sum over the CTA of v (its MT threads), and the sum over the threads before.
AXON_DEV int cta_scan(int v, int* sm, int& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  __syncthreads();
  if (lane == 31) sm[warp] = inc;
  __syncthreads();
  // every warp sums the warps' totals: one shared read per lane
  int w = sm[lane];
  const int before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
  all = __reduce_add_sync(0xffffffffu, w);
  return before + inc - v;
}

// Shared state of a cluster kernel: a CTA's sums, read by the others.
struct ClusterShared {
  int scan[32];
  int sum[2];
};

// v summed over the CTA into slot `which`, then over the CTAs: those before, and all.
AXON_DEV void cluster_sum(int v, ClusterShared* sh, int which, int& before, int& all) {
  cg::cluster_group cluster = cg::this_cluster();
  int mine;
  cta_scan(v, sh->scan, mine);
  if (threadIdx.x == 0) sh->sum[which] = mine;
  cluster.sync();
  before = all = 0;
  const int me = static_cast<int>(cluster.block_rank());
#pragma unroll
  for (int r = 0; r < CL; ++r) {
    const int x = *cluster.map_shared_rank(&sh->sum[which], r);
    all += x;
    before += r < me ? x : 0;
  }
}

// This CTA's range of the blocks.
struct Range {
  int lo, hi;
};
AXON_DEV Range my_range(int N) {
  const int per = ((N + CL - 1) / CL + 3) & ~3;
  const int lo = min(N, static_cast<int>(blockIdx.x) * per);
  return Range{lo, min(N, lo + per)};
}
// Four consecutive blocks from b: which are free. Counts are read past L1: atomics change them
// during a call.
AXON_DEV unsigned free4(const PagesArgs& a, int b, int hi) {
  unsigned bits = 0;
  if (b + 4 <= hi && (reinterpret_cast<uintptr_t>(a.refs) & 15) == 0) {
    const int4 v = __ldcg(reinterpret_cast<const int4*>(a.refs + b));
    bits = (v.x == 0 ? 1u : 0u) | (v.y == 0 ? 2u : 0u) | (v.z == 0 ? 4u : 0u) | (v.w == 0 ? 8u : 0u);
  } else {
    for (int i = 0; i < 4; ++i)
      if (b + i < hi && __ldcg(a.refs + b + i) == 0) bits |= 1u << i;
  }
  return bits;
}
AXON_DEV int count_free(const PagesArgs& a, Range r, int below) {
  int n = 0;
  for (int b = r.lo + threadIdx.x * 4; b < r.hi; b += MT * 4) {
    unsigned bits = free4(a, b, r.hi);
    if (b + 4 > below) bits &= b < below ? (1u << (below - b)) - 1u : 0u;
    n += __popc(bits);
  }
  return n;
}

// ------------------------------------------------------------------ copies
// Block src[i] to block dst[i] for i < n, all layers, keys and values. Entries with a
// negative number on either side are skipped; with CHECK, numbers out of range are reported.
template <bool CHECK>
AXON_DEV void copy_blocks(const PagesArgs& a, const int* src, const int* dst, int n, int worker, int workers) {
  const int lane = threadIdx.x & 31;
  const unsigned tiles = static_cast<unsigned>(a.block_bytes / TILE);
  const unsigned per = 2u * a.L * tiles;  // tiles of a block
  const unsigned long long total = static_cast<unsigned long long>(per) * n;
  for (unsigned long long t = worker; t < total; t += workers) {
    // 64-bit divisions only where the numbers need them
    const unsigned i = total >> 32 ? static_cast<unsigned>(t / per) : static_cast<unsigned>(t) / per;
    const unsigned rest = static_cast<unsigned>(t - static_cast<unsigned long long>(i) * per);
    const int plane = rest / tiles, tile = rest - plane * tiles;
    const int s = src[i], d = dst[i];
    if (CHECK && (s < 0 || d < 0 || s >= a.N || d >= a.N)) {
      set_err(a.err, DEVERR_BLOCK);
      continue;
    }
    if (s < 0 || d < 0) continue;
    char* const pool = static_cast<char*>(plane >= a.L ? a.v : a.k);
    const long long layer = plane >= a.L ? plane - a.L : plane;
    const char* from = pool + (layer * a.N + s) * a.block_bytes + static_cast<long long>(tile) * TILE + lane * 16;
    char* to = pool + (layer * a.N + d) * a.block_bytes + static_cast<long long>(tile) * TILE + lane * 16;
    uint4 v[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = ld_stream16(from + x * 512);
#pragma unroll
    for (int x = 0; x < 4; ++x) __stcs(reinterpret_cast<uint4*>(to + x * 512), v[x]);
  }
}

__global__ void __launch_bounds__(CT) copy_kernel(PagesArgs a, const int* src, const int* dst, int n) {
  grid_dep_launch();
  grid_dep_wait();
  copy_blocks<true>(a, src, dst, n, (blockIdx.x * CT + threadIdx.x) >> 5, (gridDim.x * CT) >> 5);
}

// ----------------------------------------------------------------- release
// One row per blockIdx.x. window < 0: everything the row holds, and its length; else the
// blocks that no query from position ctx[row] on can see.
__global__ void __launch_bounds__(CT) release_kernel(PagesArgs a, const int* rows, int window, int sinks) {
  grid_dep_launch();
  grid_dep_wait();
  const int r = rows ? rows[blockIdx.x] : blockIdx.x;
  if (r < 0 || r >= a.R) {
    if (threadIdx.x == 0) set_err(a.err, DEVERR_SEQ);
    return;
  }
  int lo = 0, hi = a.P;
  if (window >= 0) {
    const int n = a.ctx[r];
    if (n < 0 || n > a.P * 16) {
      if (threadIdx.x == 0) set_err(a.err, DEVERR_POS);
      return;
    }
    lo = (sinks + 15) >> 4;
    hi = window > 0 && n >= window ? (n - window + 1) >> 4 : 0;
  } else if (threadIdx.x == 0 && blockIdx.y == 0) {
    a.ctx[r] = 0;
  }
  for (int j = lo + blockIdx.y * CT + threadIdx.x; j < hi; j += gridDim.y * CT) {
    // exchanged, so that a row named twice gives its blocks back once
    const int b = atomicExch(a.table + static_cast<long long>(r) * a.P + j, -1);
    if (b < 0) continue;
    if (b >= a.N) {
      set_err(a.err, DEVERR_BLOCK);
    } else if (atomicSub(a.refs + b, 1) <= 0) {
      atomicAdd(a.refs + b, 1);
      set_err(a.err, DEVERR_BLOCK);
    }
  }
}

// ----------------------------------------------------------------- reserve
// Free blocks, ranked, to the wants of a list in order: give(i, k, block) for the k-th block
// of entry i. Every thread of the cluster calls it; need is complete and visible.
template <typename Give>
AXON_DEV void hand_out(const PagesArgs& a, const int* need, int n, int* pre, ClusterShared* sh, Give give) {
  const Range range = my_range(a.N);
  int base, free_all;
  cluster_sum(count_free(a, range, range.hi), sh, 0, base, free_all);
  int wanted = 0;  // pre[i]: blocks wanted before entry i
  for (int i0 = 0; i0 < n; i0 += MT) {
    const int i = i0 + threadIdx.x;
    int all;
    const int x = cta_scan(i < n ? __ldcg(need + i) : 0, sh->scan, all);
    if (i < n) pre[i] = wanted + x;
    wanted += all;
  }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0 && wanted > free_all) set_err(a.err, DEVERR_POOL);
  for (int b0 = range.lo; b0 < range.hi && base < wanted; b0 += MT * 4) {
    const int b = b0 + threadIdx.x * 4;
    unsigned bits = b < range.hi ? free4(a, b, range.hi) : 0;
    int all;
    int rank = base + cta_scan(__popc(bits), sh->scan, all);
    while (bits && rank < wanted) {
      const int x = __ffs(bits) - 1;
      bits &= bits - 1;
      int lo = 0, hi = n;  // last entry with pre <= rank
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (pre[m] <= rank) lo = m; else hi = m;
      }
      give(lo, rank - pre[lo], b + x);
      ++rank;
    }
    base += all;
  }
  // no CTA leaves while another may read its sums
  cg::this_cluster().sync();
}

// need[i]: blocks that row rows[i] lacks for more[i] tokens; first[i]: its first entry
// without one. A warp per row.
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(MT)
    reserve_kernel(PagesArgs a, const int* rows, const int* more, int n, int* need, int* first) {
  extern __shared__ int pre[];
  __shared__ ClusterShared sh;
  grid_dep_launch();
  grid_dep_wait();
  const int lane = threadIdx.x & 31;
  for (int i = (blockIdx.x * MT + threadIdx.x) >> 5; i < n; i += CL * MT / 32) {
    const int r = rows ? rows[i] : i;
    int take = 0, at = 0;
    bool bad = r < 0 || r >= a.R;
    if (rows)
      for (int k = lane; k < i; k += 32) bad |= rows[k] == r;  // named before
    bad = __any_sync(0xffffffffu, bad);
    const int ctx = bad ? 0 : a.ctx[r], m = more[i];
    if (bad) {
      if (lane == 0) set_err(a.err, DEVERR_SEQ);
    } else if (ctx < 0 || m < 0 || ctx > a.P * 16 || m > a.P * 16 - ctx) {
      if (lane == 0) set_err(a.err, DEVERR_POS);
    } else {
      at = (ctx + 15) >> 4;
      const int end = (ctx + m + 15) >> 4;
      const int* t = a.table + static_cast<long long>(r) * a.P;
      int held = at;  // one past the last entry that has a block
      bool hole = false;
      for (int j = at + lane; j < end; j += 32)
        if (t[j] >= 0) held = j + 1;
      held = __reduce_max_sync(0xffffffffu, held);
      for (int j = at + lane; j < held; j += 32) hole |= t[j] < 0;
      if (__any_sync(0xffffffffu, hole)) {
        if (lane == 0) set_err(a.err, DEVERR_SEQ);  // blocks are held from the front
      } else {
        at = held;
        take = max(0, end - at);
      }
    }
    if (lane == 0) {
      need[i] = take;
      first[i] = at;
    }
  }
  // hand_out's first barrier completes the lists
  hand_out(a, need, n, pre, &sh, [&](int i, int k, int block) {
    const int r = rows ? rows[i] : i;
    a.table[static_cast<long long>(r) * a.P + __ldcg(first + i) + k] = block;
    a.refs[block] = 1;
  });
}

// -------------------------------------------------------------------- fork
struct ForkWork {
  int* want;  // [n] 1: the last block is copied
  int* kind;  // [n] 0: refused or src = dst (nothing changes), 1: whole blocks only, 2: with a copy
  int* len;   // [n]
  int* part;  // [n] block that is copied
  int* to;    // [n] and its place, -1: none
  int* snap;  // [n][P] what the row gets
};

// References dropped and taken by atomics, whose order does not matter; the tables are only
// read, so that every row is taken as it was. Then the copies' places. A warp per 128
// entries of a row.
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(MT)
    fork_kernel(PagesArgs a, const int* src, const int* dst, int n, ForkWork w) {
  extern __shared__ int pre[];
  __shared__ ClusterShared sh;
  grid_dep_launch();
  grid_dep_wait();
  const int lane = threadIdx.x & 31;
  const int segs = (a.P + 127) / 128;
  for (long long task = (blockIdx.x * MT + threadIdx.x) >> 5; task < static_cast<long long>(n) * segs; task += CL * MT / 32) {
    const int i = static_cast<int>(task / segs), seg = static_cast<int>(task - static_cast<long long>(i) * segs);
    const int s = src[i], d = dst[i];
    bool bad = s < 0 || s >= a.R || d < 0 || d >= a.R;
    for (int k = lane; k < i; k += 32) bad |= dst[k] == d;
    bad = __any_sync(0xffffffffu, bad);
    const int len = bad ? 0 : a.ctx[s];
    const bool off = !bad && (len < 0 || len > a.P * 16);
    const bool skip = bad || off || s == d;
    const int nb = (len + 15) >> 4;
    const int* from = a.table + static_cast<long long>(skip ? 0 : s) * a.P;
    int last = -1;
    if (!skip && (len & 15)) {
      last = from[nb - 1];
      if (last >= a.N) last = -1;
    }
    if (lane == 0 && seg == 0) {
      if (bad) set_err(a.err, DEVERR_SEQ);
      if (off) set_err(a.err, DEVERR_POS);
      if (!skip && (len & 15) && last < 0) set_err(a.err, DEVERR_BLOCK);
      w.want[i] = last >= 0;
      w.kind[i] = skip ? 0 : last >= 0 ? 2 : 1;
      w.len[i] = len;
      w.part[i] = last < 0 ? -1 : last;
      w.to[i] = -1;
    }
    if (skip) continue;
    const int* old = a.table + static_cast<long long>(d) * a.P;
    for (int j = seg * 128 + lane; j < min(a.P, seg * 128 + 128); j += 32) {
      const int o = old[j];
      if (o >= a.N)
        set_err(a.err, DEVERR_BLOCK);
      else if (o >= 0)
        atomicSub(a.refs + o, 1);
      int b = j < nb ? from[j] : -1;
      if (b >= a.N) {
        set_err(a.err, DEVERR_BLOCK);
        b = -1;
      }
      // the block that is copied is held until then
      if (b >= 0) atomicAdd(a.refs + b, 1);
      if ((len & 15) && j == nb - 1) b = -1;
      w.snap[static_cast<long long>(i) * a.P + j] = b < 0 ? -1 : b;
    }
  }
  cg::this_cluster().sync();
  hand_out(a, w.want, n, pre, &sh, [&](int i, int, int block) {
    w.to[i] = block;
    a.refs[block] = 1;
  });
}

// Rows written, the copied blocks given back by the entries that held them, and copied.
__global__ void __launch_bounds__(CT) fork_write_kernel(PagesArgs a, const int* dst, int n, ForkWork w) {
  grid_dep_launch();
  grid_dep_wait();
  const long long cells = static_cast<long long>(n) * a.P;
  for (long long x = blockIdx.x * CT + threadIdx.x; x < cells; x += static_cast<long long>(gridDim.x) * CT) {
    const int i = static_cast<int>(x / a.P), j = static_cast<int>(x - static_cast<long long>(i) * a.P);
    const int kind = w.kind[i];
    if (!kind) continue;
    const int len = w.len[i];
    int b = w.snap[x];
    if (kind == 2 && j == len >> 4) {
      b = w.to[i];
      atomicSub(a.refs + w.part[i], 1);
    }
    a.table[static_cast<long long>(dst[i]) * a.P + j] = b;
    if (j == 0) a.ctx[dst[i]] = (len & 15) && w.to[i] < 0 ? len & ~15 : len;
  }
  copy_blocks<false>(a, w.part, w.to, n, (blockIdx.x * CT + threadIdx.x) >> 5, (gridDim.x * CT) >> 5);
}

// ----------------------------------------------------------------- compact
// Live blocks from number `live` on go to the free numbers below it, k-th to k-th.
// rank[b]: such a block's k, or -1; from[k], hole[k]; moved[b]: a block's number
// afterwards; info: moves, live.
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(MT)
    compact_kernel(PagesArgs a, int* rank, int* from, int* hole, int* info, int* moved, int* live_out) {
  __shared__ ClusterShared sh;
  grid_dep_launch();
  grid_dep_wait();
  const Range range = my_range(a.N);
  int base, free_all, unused, moves;
  cluster_sum(count_free(a, range, range.hi), &sh, 0, base, free_all);
  const int live = a.N - free_all;
  cluster_sum(count_free(a, range, live), &sh, 1, unused, moves);  // free numbers below `live`
  for (int b0 = range.lo; b0 < range.hi; b0 += MT * 4) {
    const int b = b0 + threadIdx.x * 4;
    const unsigned bits = b < range.hi ? free4(a, b, range.hi) : 0;
    int all;
    int f = base + cta_scan(__popc(bits), sh.scan, all);  // free blocks before
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int at = b + x;
      if (at >= range.hi) break;
      const bool is_free = (bits >> x) & 1;
      int k = -1;
      if (is_free) {
        if (at < live) hole[f] = at;
        ++f;
      } else if (at >= live) {
        k = (at - f) - (live - moves);  // live blocks before, less those below `live`
        from[k] = at;
      }
      rank[at] = k;
      if (moved) moved[at] = is_free ? -1 : at;
    }
    base += all;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    info[0] = moves;
    info[1] = live;
    if (live_out) *live_out = live;
  }
  cg::this_cluster().sync();
}

__global__ void __launch_bounds__(CT) compact_move_kernel(PagesArgs a, const int* rank, const int* from, const int* hole,
                                                          const int* info, int* moved) {
  grid_dep_launch();
  grid_dep_wait();
  const int n = info[0], live = info[1];
  const long long me = blockIdx.x * CT + threadIdx.x, threads = static_cast<long long>(gridDim.x) * CT;
  for (long long k = me; k < n; k += threads) {
    const int s = from[k], d = hole[k];
    a.refs[d] = a.refs[s];
    a.refs[s] = 0;
    if (moved) moved[s] = d;
  }
  const long long cells = static_cast<long long>(a.R) * a.P;
  for (long long x = me; x < cells; x += threads) {
    const int b = a.table[x];
    if (b < 0) continue;
    if (b >= a.N) {
      set_err(a.err, DEVERR_BLOCK);
      continue;
    }
    if (b < live) continue;
    const int k = rank[b];
    if (k >= 0)
      a.table[x] = hole[k];
    else
      set_err(a.err, DEVERR_BLOCK);  // names a block that nothing counts
  }
  copy_blocks<false>(a, from, hole, n, static_cast<int>(me >> 5), static_cast<int>(threads >> 5));
}

template <typename K, typename... Args>
cudaError_t launch_k(const LaunchCtx& lc, K kernel, dim3 grid, int threads, size_t smem, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr[2];
  cfg.numAttrs = chain_attrs(lc, attr);
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// CTAs for `tiles` warp-sized copies and `cells` table entries: at most 64 per SM: eight at a time, so
// that late ones even out the SMs (1.57 GB read and written: 253 us with eight, 247 with 16, 237 with 64).
unsigned move_grid(const LaunchCtx& lc, double tiles, double cells) {
  const double want = fmax(tiles / (CT / 32), cells / CT);
  const double most = lc.num_sms * 64.0;
  return static_cast<unsigned>(fmax(1.0, fmin(most, want)));
}

}  // namespace

size_t pages_work_ints(int N, int R, int P) {
  const size_t fork = static_cast<size_t>(R) * (5 + P);
  const size_t compact = 3 * static_cast<size_t>(N) + 2;
  return fork > compact ? fork : compact;
}

cudaError_t launch_pages_copy(const LaunchCtx& lc, const PagesArgs& a, const int* src, const int* dst, int n) {
  const double tiles = 2.0 * a.L * n * (a.block_bytes / TILE);
  return launch_k(lc, copy_kernel, dim3(move_grid(lc, tiles, 0)), CT, 0, a, src, dst, n);
}

cudaError_t launch_pages_release(const LaunchCtx& lc, const PagesArgs& a, const int* rows, int n, int window, int sinks) {
  const int y = (a.P + 4 * CT - 1) / (4 * CT);  // (the kernel takes what is left in turns)
  return launch_k(lc, release_kernel, dim3(n, y < 64 ? y : 64), CT, 0, a, rows, window, sinks);
}

cudaError_t launch_pages_reserve(const LaunchCtx& lc, const PagesArgs& a, const int* rows, const int* more, int n) {
  return launch_k(lc, reserve_kernel, dim3(CL), MT, static_cast<size_t>(n) * 4, a, rows, more, n, a.work, a.work + n);
}

cudaError_t launch_pages_fork(const LaunchCtx& lc, const PagesArgs& a, const int* src, const int* dst, int n) {
  ForkWork w;
  w.want = a.work;
  w.kind = w.want + n;
  w.len = w.kind + n;
  w.part = w.len + n;
  w.to = w.part + n;
  w.snap = w.to + n;
  cudaError_t e = launch_k(lc, fork_kernel, dim3(CL), MT, static_cast<size_t>(n) * 4, a, src, dst, n, w);
  if (e != cudaSuccess) return e;
  const double tiles = 2.0 * a.L * n * (a.block_bytes / TILE);
  return launch_k(lc, fork_write_kernel, dim3(move_grid(lc, tiles, static_cast<double>(n) * a.P)), CT, 0, a, dst, n, w);
}

cudaError_t launch_pages_compact(const LaunchCtx& lc, const PagesArgs& a, int* moved, int* live) {
  int* info = a.work;
  int* rank = info + 2;
  int* from = rank + a.N;
  int* hole = from + a.N;
  cudaError_t e = launch_k(lc, compact_kernel, dim3(CL), MT, 0, a, rank, from, hole, info, moved, live);
  if (e != cudaSuccess) return e;
  const double tiles = 2.0 * a.L * a.N * (a.block_bytes / TILE);
  return launch_k(lc, compact_move_kernel, dim3(move_grid(lc, tiles, static_cast<double>(a.R) * a.P)), CT, 0, a,
                  static_cast<const int*>(rank), static_cast<const int*>(from), static_cast<const int*>(hole),
                  static_cast<const int*>(info), moved);
}
