// Blocks of the paged cache: copied, shared between rows, taken, given back and
// moved together, all in stream order on the device.
//
// State (the caller's): a table [R][P] of block numbers (-1: none), the tokens
// ctx[r] that row r holds, and refs[b], the table entries that name block b; a block
// is free when refs is 0. Free blocks are handed out lowest number first, so that
// every result is determined by the state alone: each CTA counts the free blocks of
// a 4096-block chunk, and the next kernel ranks them with the sum over the chunks
// before. Tables and counts are latency (a few dependent loads per launch); copies
// are bound by HBM: every byte is read and written once, a warp moving 2 KB with
// four 16-byte loads per lane in flight.
#include "kernels.h"

namespace {

constexpr int CHUNK = 4096;     // blocks per CTA of the counting kernels
constexpr int CT = 256;         // their threads
constexpr int PER = CHUNK / CT; // blocks per thread
constexpr int TILE = 2048;      // bytes that a warp copies at a time

// Sum over the CTA of v, and the sum over the threads before.
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
  int add = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < CT / 32; ++w) {
    add += w < warp ? sm[w] : 0;
    all += sm[w];
  }
  return add + inc - v;
}

// Entries `count` of list `v`: how many come before this CTA's chunk, and in all.
AXON_DEV int sum_before(const int* v, int chunks, int mine, int* sm, int& all) {
  int b = 0, t = 0;
  for (int i = threadIdx.x; i < chunks; i += CT) {
    const int x = v[i];
    t += x;
    b += i < mine ? x : 0;
  }
  int dummy;
  cta_scan(b, sm, dummy);
  cta_scan(t, sm, all);
  return dummy;
}

// The free blocks (refs 0) of this thread's PER consecutive blocks, as bits.
AXON_DEV unsigned free_bits(const PagesArgs& a, int chunk) {
  const int b0 = chunk * CHUNK + threadIdx.x * PER;
  unsigned bits = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (b0 + i < a.N && a.refs[b0 + i] == 0) bits |= 1u << i;
  return bits;
}

__global__ void __launch_bounds__(CT) count_kernel(PagesArgs a, int* counts) {
  __shared__ int sm[CT / 32];
  grid_dep_launch();
  grid_dep_wait();
  int all;
  cta_scan(__popc(free_bits(a, blockIdx.x)), sm, all);
  if (threadIdx.x == 0) counts[blockIdx.x] = all;
}

// ------------------------------------------------------------------ copies
// Block src[i] to block dst[i] for i < n, all layers, keys and values. Entries with a
// negative number on either side are skipped; with CHECK, numbers out of range are reported.
template <bool CHECK>
AXON_DEV void copy_blocks(const PagesArgs& a, const int* src, const int* dst, int n, int worker, int workers) {
  const int lane = threadIdx.x & 31;
  const int tiles = static_cast<int>(a.block_bytes / TILE);
  const long long per = 2ll * a.L * tiles, total = per * n;
  for (long long t = worker; t < total; t += workers) {
    const int i = static_cast<int>(t / per);
    const int rest = static_cast<int>(t - i * per);
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
// need[i]: blocks that row rows[i] lacks for more[i] tokens; first[i]: its first
// entry without one. CTAs past the chunks take the rows, a thread each.
__global__ void __launch_bounds__(CT) reserve_count_kernel(PagesArgs a, const int* rows, const int* more, int n,
                                                           int chunks, int* counts, int* need, int* first) {
  __shared__ int sm[CT / 32];
  grid_dep_launch();
  grid_dep_wait();
  if (static_cast<int>(blockIdx.x) < chunks) {
    int all;
    cta_scan(__popc(free_bits(a, blockIdx.x)), sm, all);
    if (threadIdx.x == 0) counts[blockIdx.x] = all;
    return;
  }
  // a warp per row: named before?, then its entries
  const int i = ((blockIdx.x - chunks) * CT + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (i >= n) return;
  const int r = rows ? rows[i] : i;
  int take = 0, at = 0;
  bool bad = r < 0 || r >= a.R;
  if (rows)
    for (int k = lane; k < i; k += 32) bad |= rows[k] == r;
  bad = __any_sync(0xffffffffu, bad);
  if (bad) {
    if (lane == 0) set_err(a.err, DEVERR_SEQ);
  } else {
    const int ctx = a.ctx[r], m = more[i];
    if (ctx < 0 || m < 0 || ctx > a.P * 16 || m > a.P * 16 - ctx) {
      if (lane == 0) set_err(a.err, DEVERR_POS);
    } else {
      at = (ctx + 15) >> 4;
      const int end = (ctx + m + 15) >> 4;
      const int* t = a.table + static_cast<long long>(r) * a.P;
      int held = at;  // one past the last entry that has a block
      for (int j = at + lane; j < end; j += 32)
        if (t[j] >= 0) held = j + 1;
      held = __reduce_max_sync(0xffffffffu, held);
      int holes = 0;
      for (int j = at + lane; j < held; j += 32) holes |= t[j] < 0;
      if (__any_sync(0xffffffffu, holes)) {
        if (lane == 0) set_err(a.err, DEVERR_SEQ);  // blocks are held from the front
      } else {
        at = held;
        take = max(0, end - at);
      }
    }
  }
  if (lane == 0) {
    need[i] = take;
    first[i] = at;
  }
}

// Free blocks, ranked, to the lists' wants in order. `give(i, k, block)` is called for the
// k-th block of entry i; returns the total wanted and the free blocks in all.
template <typename Give>
AXON_DEV void hand_out(const PagesArgs& a, const int* counts, int chunks, const int* need, int n, int* pre, int* sm,
                       int& wanted, int& free_all, Give give) {
  // pre[i]: blocks wanted before entry i
  wanted = 0;
  for (int i0 = 0; i0 < n; i0 += CT) {
    const int i = i0 + threadIdx.x;
    int all;
    const int x = cta_scan(i < n ? need[i] : 0, sm, all);
    if (i < n) pre[i] = wanted + x;
    wanted += all;
  }
  const int base = sum_before(counts, chunks, blockIdx.x, sm, free_all);
  if (base >= wanted) return;
  unsigned bits = free_bits(a, blockIdx.x);
  int all;
  int rank = base + cta_scan(__popc(bits), sm, all);
  while (bits && rank < wanted) {
    const int x = __ffs(bits) - 1;
    bits &= bits - 1;
    int lo = 0, hi = n;  // last entry with pre <= rank
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] <= rank) lo = mid; else hi = mid;
    }
    give(lo, rank - pre[lo], blockIdx.x * CHUNK + threadIdx.x * PER + x);
    ++rank;
  }
}

__global__ void __launch_bounds__(CT) reserve_kernel(PagesArgs a, const int* rows, int n, int chunks, const int* counts,
                                                     const int* need, const int* first) {
  extern __shared__ int pre[];
  __shared__ int sm[CT / 32];
  grid_dep_launch();
  grid_dep_wait();
  int wanted, free_all;
  hand_out(a, counts, chunks, need, n, pre, sm, wanted, free_all, [&](int i, int k, int block) {
    const int r = rows ? rows[i] : i;
    a.table[static_cast<long long>(r) * a.P + first[i] + k] = block;
    a.refs[block] = 1;
  });
  if (blockIdx.x == 0 && threadIdx.x == 0 && wanted > free_all) set_err(a.err, DEVERR_POOL);
}

// -------------------------------------------------------------------- fork
// Per entry: what the row gets. state 0: refused or src = dst (nothing changes), 1: whole
// blocks only, 2: the last block is copied.
struct ForkWork {
  int* state;  // [n], as the wants of hand_out: 1 where a block is wanted
  int* kind;   // [n]
  int* len;    // [n]
  int* part;   // [n] block that is copied
  int* to;     // [n] and its place, -1: none
  int* snap;   // [n][P]
};

// grid (n, y): entry blockIdx.x. References dropped and taken by atomics, whose order does
// not matter; the tables are only read, so that every row is taken as it was.
__global__ void __launch_bounds__(CT) fork_refs_kernel(PagesArgs a, const int* src, const int* dst, ForkWork w) {
  grid_dep_launch();
  grid_dep_wait();
  const int i = blockIdx.x;
  const int s = src[i], d = dst[i];
  bool bad = s < 0 || s >= a.R || d < 0 || d >= a.R;
  for (int k = threadIdx.x; k < i; k += CT) bad |= dst[k] == d;
  bad = __syncthreads_or(bad);
  const int len = bad ? 0 : a.ctx[s];
  const bool off = !bad && (len < 0 || len > a.P * 16);
  const bool lead = threadIdx.x == 0 && blockIdx.y == 0;
  if (lead) {
    if (bad) set_err(a.err, DEVERR_SEQ);
    if (off) set_err(a.err, DEVERR_POS);
  }
  const bool skip = bad || off || s == d;
  const int nb = (len + 15) >> 4;
  const int* from = a.table + static_cast<long long>(skip ? 0 : s) * a.P;
  int last = -1;
  if (!skip && (len & 15)) {
    last = from[nb - 1];
    if (last >= a.N) last = -1;
  }
  if (lead) {
    w.state[i] = last >= 0;
    w.kind[i] = skip ? 0 : last >= 0 ? 2 : 1;
    w.len[i] = len;
    w.part[i] = last;
    w.to[i] = -1;
    if (!skip && (len & 15) && last < 0) set_err(a.err, DEVERR_BLOCK);
  }
  if (skip) return;
  const int* old = a.table + static_cast<long long>(d) * a.P;
  for (int j = blockIdx.y * CT + threadIdx.x; j < a.P; j += gridDim.y * CT) {
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

__global__ void __launch_bounds__(CT) fork_take_kernel(PagesArgs a, int n, int chunks, const int* counts, ForkWork w) {
  extern __shared__ int pre[];
  __shared__ int sm[CT / 32];
  grid_dep_launch();
  grid_dep_wait();
  int wanted, free_all;
  hand_out(a, counts, chunks, w.state, n, pre, sm, wanted, free_all, [&](int i, int, int block) {
    w.to[i] = block;
    a.refs[block] = 1;
  });
  if (blockIdx.x == 0 && threadIdx.x == 0 && wanted > free_all) set_err(a.err, DEVERR_POOL);
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
// rank[b]: such a block's k, or -1; from[k], hole[k]; moved[b]: a block's number afterwards.
__global__ void __launch_bounds__(CT) compact_rank_kernel(PagesArgs a, int chunks, const int* counts, int* rank, int* from,
                                                          int* hole, int* n_moves, int* moved, int* live_out) {
  __shared__ int sm[CT / 32];
  grid_dep_launch();
  grid_dep_wait();
  int free_all, all;
  const int free_before = sum_before(counts, chunks, blockIdx.x, sm, free_all);
  const int live = a.N - free_all;
  // free numbers below `live`: those of the chunks before it, and of its own chunk
  const int edge = live / CHUNK;
  int below = sum_before(counts, chunks, edge, sm, all);
  if (edge < chunks) {
    const int b0 = edge * CHUNK + threadIdx.x * PER;
    const int keep = max(0, min(PER, live - b0));
    int more;
    cta_scan(__popc(free_bits(a, edge) & ((1u << keep) - 1u)), sm, more);
    below += more;
  }
  const int moves = below;
  const unsigned bits = free_bits(a, blockIdx.x);
  int f = free_before + cta_scan(__popc(bits), sm, all);
  const int b0 = blockIdx.x * CHUNK + threadIdx.x * PER;
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int b = b0 + x;
    if (b >= a.N) break;
    const bool is_free = (bits >> x) & 1;
    if (is_free) {
      if (b < live) hole[f] = b;
      rank[b] = -1;
      ++f;
    } else if (b >= live) {
      // live blocks before b, less those below `live`
      const int k = (b - f) - (live - moves);
      rank[b] = k;
      from[k] = b;
    } else {
      rank[b] = -1;
    }
    if (moved) moved[b] = is_free ? -1 : b;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    n_moves[0] = moves;
    n_moves[1] = live;
    if (live_out) *live_out = live;
  }
}

__global__ void __launch_bounds__(CT) compact_move_kernel(PagesArgs a, const int* rank, const int* from, const int* hole,
                                                          const int* n_moves, int* moved) {
  grid_dep_launch();
  grid_dep_wait();
  const int n = n_moves[0], live = n_moves[1];
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
cudaError_t launch_k(const LaunchCtx& lc, K kernel, dim3 grid, size_t smem, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(CT);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr[2];
  cfg.numAttrs = chain_attrs(lc, attr);
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

int chunk_count(int N) { return (N + CHUNK - 1) / CHUNK; }

// CTAs for `tiles` warp-sized copies and `cells` table entries: at most six per SM.
unsigned move_grid(const LaunchCtx& lc, double tiles, double cells) {
  const double want = fmax(tiles / (CT / 32), cells / CT);
  const double most = lc.num_sms * 6.0;
  return static_cast<unsigned>(fmax(1.0, fmin(most, want)));
}

}  // namespace

size_t pages_work_ints(int N, int R, int P) {
  const size_t chunks = chunk_count(N);
  const size_t fork = static_cast<size_t>(R) * (5 + P);
  const size_t compact = 3 * static_cast<size_t>(N) + 2;
  return chunks + (fork > compact ? fork : compact);
}

cudaError_t launch_pages_copy(const LaunchCtx& lc, const PagesArgs& a, const int* src, const int* dst, int n) {
  const double tiles = 2.0 * a.L * n * (a.block_bytes / TILE);
  return launch_k(lc, copy_kernel, dim3(move_grid(lc, tiles, 0)), 0, a, src, dst, n);
}

cudaError_t launch_pages_release(const LaunchCtx& lc, const PagesArgs& a, const int* rows, int n, int window, int sinks) {
  const unsigned y = static_cast<unsigned>((a.P + 4 * CT - 1) / (4 * CT));
  return launch_k(lc, release_kernel, dim3(n, y), 0, a, rows, window, sinks);
}

cudaError_t launch_pages_reserve(const LaunchCtx& lc, const PagesArgs& a, const int* rows, const int* more, int n) {
  const int chunks = chunk_count(a.N);
  int* counts = a.work;
  int* need = counts + chunks;
  int* first = need + n;
  const int row_ctas = (n + CT / 32 - 1) / (CT / 32);
  cudaError_t e = launch_k(lc, reserve_count_kernel, dim3(chunks + row_ctas), 0, a, rows, more, n, chunks, counts, need, first);
  if (e != cudaSuccess) return e;
  return launch_k(lc, reserve_kernel, dim3(chunks), static_cast<size_t>(n) * 4, a, rows, n, chunks,
                  static_cast<const int*>(counts), static_cast<const int*>(need), static_cast<const int*>(first));
}

cudaError_t launch_pages_fork(const LaunchCtx& lc, const PagesArgs& a, const int* src, const int* dst, int n) {
  const int chunks = chunk_count(a.N);
  int* counts = a.work;
  ForkWork w;
  w.state = counts + chunks;
  w.kind = w.state + n;
  w.len = w.kind + n;
  w.part = w.len + n;
  w.to = w.part + n;
  w.snap = w.to + n;
  const unsigned y = static_cast<unsigned>((a.P + 4 * CT - 1) / (4 * CT));
  cudaError_t e = launch_k(lc, fork_refs_kernel, dim3(n, y), 0, a, src, dst, w);
  if (e == cudaSuccess) e = launch_k(lc, count_kernel, dim3(chunks), 0, a, counts);
  if (e == cudaSuccess)
    e = launch_k(lc, fork_take_kernel, dim3(chunks), static_cast<size_t>(n) * 4, a, n, chunks,
                 static_cast<const int*>(counts), w);
  if (e != cudaSuccess) return e;
  const double tiles = 2.0 * a.L * n * (a.block_bytes / TILE);
  return launch_k(lc, fork_write_kernel, dim3(move_grid(lc, tiles, static_cast<double>(n) * a.P)), 0, a, dst, n, w);
}

cudaError_t launch_pages_compact(const LaunchCtx& lc, const PagesArgs& a, int* moved, int* live) {
  const int chunks = chunk_count(a.N);
  int* counts = a.work;
  int* n_moves = counts + chunks;
  int* rank = n_moves + 2;
  int* from = rank + a.N;
  int* hole = from + a.N;
  cudaError_t e = launch_k(lc, count_kernel, dim3(chunks), 0, a, counts);
  if (e == cudaSuccess)
    e = launch_k(lc, compact_rank_kernel, dim3(chunks), 0, a, chunks, static_cast<const int*>(counts), rank, from, hole,
                 n_moves, moved, live);
  if (e != cudaSuccess) return e;
  const double tiles = 2.0 * a.L * a.N * (a.block_bytes / TILE);
  return launch_k(lc, compact_move_kernel, dim3(move_grid(lc, tiles, static_cast<double>(a.R) * a.P)), 0, a,
                  static_cast<const int*>(rank), static_cast<const int*>(from), static_cast<const int*>(hole),
                  static_cast<const int*>(n_moves), moved);
}
