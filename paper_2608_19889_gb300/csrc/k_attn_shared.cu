// Attention of one new token per row where rows share the first blocks of their context: the
// prefix pass over the blocks in common, once per group, and the join with each row's own part,
// which the one-token kernel (k_attn_paged.cu) takes.
//
//   o = sum over parts of 2^(m_i - m) O_i / sum of 2^(m_i - m) l_i,  m = max m_i
//   (m_i, l_i, O_i): a part's maximum, sum of 2^(s - m_i) and sum of 2^(s - m_i) v
//
// The blocks in common are read once for all rows of a group and hold no masked token, so that the prefix
// pass is a plain product: a tile is 128 (row, query head) pairs of one kv head, PW = 128 / (H/G) rows; an item is
// two tiles of a group and a kv head, which share the keys, 128 per step (eight blocks). Where the rows fill one tile
// only, both pipelines take it, every other step each: else its products would wait for its softmax. The steps of all
// items form one line, which the CTAs (one per SM) split evenly: an item's parts go to the workspace, as many as
// CTAs have a share of it, and the join adds them up in their order, so that results do not depend on timing.
// Warps:
//   0..3, 4..7  softmax of tile 0 and 1, one thread per (row, head);
//   8, 10       TMA producers, of queries and keys, and of values, through a ring of tiles (16 boxes of 2 KB per tile take
//               one warp 1100 cycles to ask for);
//   9, 11       MMA issuers of tile 0 and 1 (S = Q K^T into TMEM, O += P V with P from TMEM).
// The softmax warps first run a step on nothing, while the others work out what is in common: its 1500 instructions
// come from memory the first time, which took 9000 cycles instead of 1600, and most launches take ten or twenty steps.
// P enters the product in two 16-bit terms, as in the other attention kernels.
//
// The bound is the tensor pipe where the rows fill two tiles (three products of 128 x 128 x 128 per tile and step, 1536 cycles, a
// third of them the second terms'), and HBM where they fill one. Measured: 64 rows of 40 / 8 heads of 128 on 32768 tokens,
// 157 tokens each of their own, 83 us in all: the pass 57 on 128 SMs, 0.75 PFLOP/s without the second terms, a step of two tiles
// 2.05 us (3900 cycles); the own parts beside it. 64 rows of 32 / 8 heads in groups of 4 on 512 to 4096 tokens 53 us, the
// pass 32 of them, at 4.7 TB/s. Start, plan and the first step's code take 10 us, the join 4 to 6.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "attn_shared.cuh"
#include "attn_tc.cuh"
#include "kernels.h"

namespace {

constexpr int THREADS = 384;
constexpr int KT = 128;    // keys per step
constexpr float LAG = 4.f; // how far a row's scores may exceed its m (log2)
constexpr int MAX_N = SHARED_MAX_GROUPS;

template <int HD>
struct SCfg {
  static constexpr int CH = HD / 64;                // 64-dim chunks (128-byte swizzled rows)
  static constexpr int CHUNK = 128 * 128;           // bytes of one 128-row chunk
  static constexpr int TILE = CH * CHUNK;           // Q, K or V tile
  static constexpr int STAGES = HD == 128 ? 4 : 8;  // K and V tiles in flight
  static constexpr int BARS = 2 * STAGES + 18;
  static constexpr int PLAN = 4 * (GroupPlan::ints(MAX_N) + MAX_N + 1);
  static constexpr int SMEM = 2 * TILE + STAGES * TILE + 8 * BARS + 16 + PLAN + 1024;
};

// How the line is dealt: `workers` CTAs, the first `extra` of them one more than `share`; a CTA takes the steps that begin
// in its range, which holds one at least.
struct Deal {
  unsigned total, workers, share, extra;
  AXON_DEV unsigned begin(unsigned w) const { return w * share + min(w, extra); }
  AXON_DEV unsigned worker_of(unsigned u) const {
    const unsigned cut = extra * (share + 1);
    return u < cut ? u / (share + 1) : extra + (u - cut) / share;
  }
};
AXON_DEV Deal deal(unsigned total, unsigned ctas, unsigned least_steps) {
  Deal d;
  d.total = total;
  d.workers = min(ctas, max(1u, total / (COST_TWO * least_steps)));
  d.share = total / d.workers;
  d.extra = total - d.share * d.workers;
  return d;
}

// A CTA's share of an item.
struct Part {
  int g, r0, p0, rows;  // kv head, the group's first row, the item's first row in it, rows of the item
  int page0, pages;     // blocks
  int lead;
  bool one;             // one tile, in both pipelines
  int odd;              // one: the pipeline that takes its first step, since a stage of the ring is always the same one's
  int at;               // its first (row, head) in the workspace
  int steps;
  unsigned next;        // where the next part begins
  // steps of pipeline w
  AXON_DEV int count(int w, int PW) const { return one ? (steps + 1 - (w ^ odd)) >> 1 : w * PW < rows ? steps : 0; }
};

// In front of the parts' first (row, head): twice those of the items before it, which all lie inside B * H, and 256 for each
// CTA before, since an item has that many (row, head) pairs at most (twice those of its tile, if it has one) and
// each CTA adds a part at most.
// (Below 2^31: the launcher saw to it.)
AXON_DEV int part_at(int r0, int rows, int g, int p0, int H, int HPG, unsigned worker) {
  return 2 * (r0 * H + (g * rows + p0) * HPG) + 256 * static_cast<int>(worker);
}

// This CTA's number among the `workers` of the prefix pass; not below them: it leaves its SM to the rows' own parts, which take
// `own` SMs. These come in pairs, the even one and the next, since two SMs share a way to the memory: beside one that
// streams own parts a CTA of the prefix pass took 70 us instead of 63. Should too few CTAs be on the other SMs, the last ones
// to come work wherever they are.
AXON_DEV unsigned number_of(const SharedGroups& sg, int own, int workers) {
  const int pairs = sg.sms / 2;
  if (pairs < 2) return blockIdx.x;
  const int at = static_cast<int>(sm_id() % sg.sms) / 2;
  const bool works = (at + 1) * (own / 2) / pairs == at * (own / 2) / pairs;
  // CTAs that came, and their numbers
  const unsigned old = atomicAdd(reinterpret_cast<unsigned*>(sg.next) + 2, works ? 0x10001u : 0x10000u);
  const int given = static_cast<int>(old & 0xffff), to_come = static_cast<int>(gridDim.x - 1 - (old >> 16));
  if (works) return given;
  return workers - given > to_come ? atomicAdd(reinterpret_cast<unsigned*>(sg.next) + 2, 1u) & 0xffff : UINT_MAX;
}

template <int HD, typename T16>
__global__ void __launch_bounds__(THREADS, 1)
    attn_prefix_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const PagedAttnArgs p, const SharedGroups sg, int PW,
                       int pool_rows) {
  using C = SCfg<HD>;
  constexpr int NS = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  const uint32_t sQ = base, sKV = base + 2 * C::TILE, bars = sKV + NS * C::TILE;
  auto kv_full = [&](int s) { return bars + 8 * s; };
  auto kv_empty = [&](int s) { return bars + 8 * (NS + s); };
  const uint32_t more = bars + 8 * (2 * NS);
  auto q_full = [&](int w) { return more + 8 * w; };
  auto q_empty = [&](int w) { return more + 8 * (2 + w); };
  auto s_full = [&](int w) { return more + 8 * (4 + w); };
  auto p_full = [&](int w) { return more + 8 * (6 + w); };
  auto o_full = [&](int w) { return more + 8 * (8 + w); };
  auto o_empty = [&](int w) { return more + 8 * (10 + w); };
  auto turn = [&](int w) { return more + 8 * (12 + w); };
  auto warm = [&](int w) { return more + 8 * (14 + w); };
  auto met = [&](int w) { return more + 8 * (16 + w); };
  const uint32_t tmem_slot = bars + 8 * C::BARS;
  int* const plan = reinterpret_cast<int*>(smem_raw + (tmem_slot + 16 - raw));
  const GroupPlan gp(plan, sg.N);
  unsigned* const before = reinterpret_cast<unsigned*>(plan + GroupPlan::ints(sg.N));  // [N + 1] cost of the groups before
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int HPG = p.H / p.G, PC = 2 * PW;

  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(kv_full(s), 1);
      mbar_init(kv_empty(s), 2);  // both issuers
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(q_full(w), 1);
      mbar_init(q_empty(w), 1);
      mbar_init(s_full(w), 1);
      mbar_init(p_full(w), 128);
      mbar_init(o_full(w), 1);
      mbar_init(o_empty(w), 128);
      mbar_init(turn(w), 1);
      mbar_init(warm(w), 128);
      mbar_init(met(w), 1);
    }
    fence_mbar_init();
    fence_proxy_async();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<const uint32_t*>(smem_raw + (tmem_slot - raw));
  // what the parts' owners need to know is there once `ready` lets them pass
  auto ready = [&]() { asm volatile("barrier.cta.sync 1, 384;" ::: "memory"); };
  auto make_ready = [&]() { asm volatile("barrier.cta.sync 2, 128;\n\tbarrier.cta.arrive 1, 384;" ::: "memory"); };
  Deal d{};
  unsigned u0 = 0, u1 = 0;
  // CTAs that the line is dealt to; the others leave their SMs to the rows' own parts
  auto ctas = [&]() { return static_cast<unsigned>(min(static_cast<int>(gridDim.x), max(1, sg.sms - *gp.own))); };
  __shared__ unsigned s_worker;
  unsigned worker = 0;  // of the line
  auto take_share = [&]() {
    d = deal(before[sg.N], ctas(), sg.least_steps);
    worker = s_worker;
    u1 = worker < d.workers && d.total ? d.begin(worker + 1) : 0;
    u0 = u1 ? d.begin(worker) : 0;
  };
  // The part with the first step that begins at u or after it (u < u1); no steps: none does. The same in all lanes.
  // done: steps of the CTA before it.
  auto part_of = [&](unsigned u, int done) {
    Part t;
    t.odd = done & 1;
    for (;;) {
      int lo = 0, hi = sg.N - 1;  // the last group that begins at u or before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (before[mid] <= u) lo = mid; else hi = mid - 1;
      }
      const Span s(gp.from[lo + 1] - gp.from[lo], gp.c1[lo] - gp.c0[lo], PW);
      const unsigned off = u - before[lo];
      t.g = static_cast<int>(off / s.per_head);
      const unsigned in = off - t.g * s.per_head;
      const int pair = min(static_cast<int>(in / (s.steps * COST_TWO)), s.pairs - 1);
      const unsigned cost = s.cost(pair), begin = before[lo] + s.item(t.g, pair), first = (u - begin + cost - 1) / cost;
      if (first >= s.steps) {  // the rest of a step that the CTA before has
        u = begin + s.steps * cost;
        if (u < u1) continue;
        t.steps = 0;
        t.next = u1;
        return t;
      }
      // steps that begin before u1
      const unsigned last = begin + first * cost < u1 ? min(s.steps, (u1 - begin + cost - 1) / cost) : first;
      t.steps = static_cast<int>(last - first);
      t.next = begin + last * cost;
      t.r0 = gp.from[lo];
      t.p0 = pair * PC;
      t.rows = min(PC, s.rows - t.p0);
      t.one = t.rows <= PW;
      t.page0 = gp.c0[lo] + 8 * static_cast<int>(first);
      t.pages = min(gp.c1[lo] - t.page0, 8 * t.steps);
      t.lead = gp.lead[lo];
      t.at = part_at(t.r0, s.rows, t.g, t.p0, p.H, HPG, worker);
      return t;
    }
  };

  if (warp >= 8) {
    // Before `ready`, since the softmax warps wait for these registers; and once for all that these warps do, since what
    // follows a place where the branches meet may be given registers that only the softmax warps have.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    grid_dep_wait();
    grid_dep_launch();  // the rows' own parts, which wait for nothing of this kernel until their end
    plan_groups<128, 256>(p, sg, gp, blockIdx.x == 0);
    if (warp == 9 && lane == 0) s_worker = number_of(sg, *gp.own, ctas());
    if (warp == 11 && blockIdx.x == gridDim.x - 1) {
      // the plan for the rows' own parts, which find it there as a rule
      for (int b = lane; b < p.B; b += 32) sg.common[b] = common_of(gp, sg.N, b);
      __threadfence();
      __syncwarp();
      if (lane == 0) *static_cast<volatile int*>(sg.next + 3) = *gp.own;
    }
    if (warp == 8) {
      unsigned sum = 0;
      for (int i0 = 0; i0 < sg.N; i0 += 32) {
        const int i = i0 + lane;
        unsigned n = 0;
        if (i < sg.N && gp.c1[i] > gp.c0[i]) n = Span(gp.from[i + 1] - gp.from[i], gp.c1[i] - gp.c0[i], PW).per_head * p.G;
        unsigned inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned t = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += t;
        }
        if (i < sg.N) before[i] = sum + inc - n;
        sum += __shfl_sync(0xffffffffu, inc, 31);
      }
      if (lane == 0) before[sg.N] = sum;
    }
    make_ready();
    take_share();
    if (!(warp & 1)) {
      // ---------------------------------------------------------- producers
      const int kv = warp == 8 ? 0 : 1;
      int iq[2] = {0, 0}, it = kv;  // queries; tiles of the ring, this warp's every other one
      bool ok = true;
      for (unsigned u = u0; u < u1 && ok;) {
        const Part t = part_of(u, it >> 1);
        u = t.next;
        if (!t.steps) break;
        // pool row of this lane's block of step s; past the last block and for table entries
        // out of range (reported) the row lies outside the pool, where a box reads zeros
        auto pool_row = [&](int s) {
          const int i = s * 8 + lane;
          if (lane >= 8 || i >= t.pages) return pool_rows;
          const int blk = __ldcg(p.block_table + static_cast<long long>(t.lead) * p.blocks_per_seq + t.page0 + i);
          if (blk < 0 || blk >= p.num_blocks) {
            set_err(p.err, DEVERR_BLOCK);
            return pool_rows;
          }
          return (blk * p.G + t.g) * 16;
        };
        int next = pool_row(0);
        for (int w = 0; w < 2 && !kv; ++w) {
          if (!t.count(w, PW)) continue;
          ok = __all_sync(0xffffffffu, wait_bar(q_empty(w), (iq[w] & 1) ^ 1, p.err));
          if (!ok) break;
          if (lane == 0) {
            mbar_arrive_expect_tx(q_full(w), HPG * PW * HD * 2);
            for (int c = 0; c < C::CH; ++c)
              tma_load_3d(sQ + w * C::TILE + c * C::CHUNK, &tmQ, q_full(w), c * 64, t.g * HPG,
                          t.r0 + t.p0 + (t.one ? 0 : w * PW));
          }
          ++iq[w];
        }
        for (int s = 0; s < t.steps && ok; ++s, it += 2) {
          const int y = next, st = it % NS;
          next = pool_row(s + 1);
          ok = __all_sync(0xffffffffu, wait_bar(kv_empty(st), ((it / NS) & 1) ^ 1, p.err));
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(kv_full(st), C::TILE);
          __syncwarp();
          if (lane < 8)
            for (int c = 0; c < C::CH; ++c)
              tma_load_2d(sKV + st * C::TILE + c * C::CHUNK + lane * 2048, kv ? &tmV : &tmK, kv_full(st), c * 64, y);
        }
      }
      if (kv && blockIdx.x == 0) {
        // what the join has to know of the rows
        if (lane == 0) sg.plan[0] = make_int4(static_cast<int>(d.total), static_cast<int>(ctas()), sg.least_steps, 0);
        for (int b = lane; b < p.B; b += 32) {
          const int n = live_pos(p, b) >= 0 ? group_of(gp, sg.N, b) : -1;
          sg.plan[1 + b] = n >= 0 && gp.c1[n] > gp.c0[n]
                               ? make_int4(gp.c1[n] - gp.c0[n], static_cast<int>(before[n]), gp.from[n],
                                           gp.from[n + 1] - gp.from[n])
                               : make_int4(0, 0, 0, 0);
        }
      }
      // Nothing may be on its way to the CTA's shared memory when it goes away: neither copies nor the arrivals that the
      // tensor pipe makes for the issuers' last commits, which come after the one that lets the softmax warps finish. (A
      // stage that is given back was filled.)
      for (int w = 0; w < 2; ++w)
        if (iq[w] > 0) wait_bar(q_empty(w), (iq[w] - 1) & 1, p.err);
      for (int i = max(it - NS, kv); i < it; i += 2) wait_bar(kv_empty(i % NS), (i / NS) & 1, p.err);
      if (!ok) {
        for (int w = 0; w < 2; ++w)
          if (iq[w] > 0) wait_bar(q_full(w), (iq[w] - 1) & 1, p.err);
        for (int i = max(it - NS, kv); i < it; i += 2) wait_bar(kv_full(i % NS), (i / NS) & 1, p.err);
      }
    } else {
      // -------------------------------------------------------- MMA issuers
      // A warp per tile, in turns: one tile's products run under the other's softmax.
      const int w = warp == 9 ? 0 : 1;
      const bool leader = elect_one();
      constexpr uint32_t id_s = idesc_f32acc(128, KT, MmaFmt<T16>::v);
      constexpr uint32_t id_o = idesc_f32acc(128, HD, MmaFmt<T16>::v) | (1u << 16);  // B stored N-contiguous
      const uint64_t dQ = smem_desc_sw128(sQ + w * C::TILE), dK = smem_desc_sw128(sKV), dV = v_desc<C::CHUNK>(sKV);
      const uint32_t tS = tmem + w * KT, tO = tmem + 2 * KT + w * HD;
      uint32_t st = 0, ph = 0;  // ring: next stage and its phase
      auto next_stage = [&]() {
        st = st + 1 == NS ? 0 : st + 1;
        ph ^= st == 0;
      };
      auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bar(bar, parity, p.err)) != 0; };
      uint32_t ph_q = 0, ph_p = 0;  // phases of this tile's parts and steps
      uint32_t turns = 0;
      wait_all(warm(w), 0);  // (nothing of the step on nothing is read; its stores are done)
      auto my_turn = [&]() { return wait_all(turn(w), (turns & 1) ^ (w ^ 1)); };
      // scores from the keys in stage st; the turn passes two products before the end
      auto scores = [&](bool last) {
        const uint64_t kd = dK + st * (C::TILE >> 4);
        if (leader) {
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            const int off = ((k >> 2) * C::CHUNK + (k & 3) * 32) >> 4;
            if (k == HD / 16 - 2) mbar_arrive(turn(w ^ 1));
            tc_mma_f16(tS, dQ + off, kd + off, id_s, k != 0);
          }
          tc_commit(s_full(w));
          if (last) tc_commit(q_empty(w));
        }
        ++turns;
      };
      auto pass_turn = [&]() {
        if (leader) mbar_arrive(turn(w ^ 1));
        ++turns;
      };
      auto products = [&](uint32_t sv, int blocks, bool first) {
        const uint64_t vd = dV + sv * (C::TILE >> 4);
        if (!first && blocks == 8) {
          if (leader) {
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              tc_mma_f16_ts(tO, tS + x * 8, vd + x * 128, id_o, 1u);
              tc_mma_f16_ts(tO, tS + KT / 2 + x * 8, vd + x * 128, id_o, 1u);
            }
          }
        } else if (leader) {
          // the first step starts the sums; blocks past the last hold no values
#pragma unroll 1
          for (int x = 0; x < blocks; ++x) {
            tc_mma_f16_ts(tO, tS + x * 8, vd + x * 128, id_o, !first || x != 0 ? 1u : 0u);
            tc_mma_f16_ts(tO, tS + KT / 2 + x * 8, vd + x * 128, id_o, 1u);
          }
        }
      };
      int done = 0;
      bool apart = false;  // the issuers have gone through the ring each on its own
      uint32_t meetings = 0;
      for (unsigned u = u0; u < u1;) {
        const Part t = part_of(u, done);
        u = t.next;
        if (!t.steps) break;
        done += t.steps;
        const int nt_all = __shfl_sync(0xffffffffu, t.steps, 0), pages = __shfl_sync(0xffffffffu, t.pages, 0);
        const int nt = __shfl_sync(0xffffffffu, t.count(w, PW), 0);
        if (__shfl_sync(0xffffffffu, static_cast<int>(t.one), 0)) {
          // Every other step; nobody else uses its stages, so that each is given back for both issuers. A stage has the same
          // issuer in all such parts: an issuer that came to a stage of the other one could take the fill before the last
          // for the one that it waits for, their parities being the same.
          apart = true;
          const uint32_t st0 = st, ph0 = ph;
          auto stage_of = [&](int s, int kv, uint32_t& phase) {
            const uint32_t at = st0 + 2 * s + kv;
            phase = ph0 ^ ((at / NS) & 1);
            return at % NS;
          };
          bool ok = !nt || wait_all(q_full(w), ph_q);
          for (int k = 0; k < nt && ok; ++k) {
            const int s = 2 * k + (w ^ t.odd);
            uint32_t phk, phv;
            const uint32_t sk = stage_of(s, 0, phk), sv = stage_of(s, 1, phv);
            ok = wait_all(kv_full(sk), phk);
            if (!ok) break;
            tc_fence_after();
            if (leader) {
              const uint64_t kd = dK + sk * (C::TILE >> 4);
#pragma unroll
              for (int x = 0; x < HD / 16; ++x) {
                const int off = ((x >> 2) * C::CHUNK + (x & 3) * 32) >> 4;
                tc_mma_f16(tS, dQ + off, kd + off, id_s, x != 0);
              }
              tc_commit(s_full(w));
              if (k + 1 == nt) tc_commit(q_empty(w));
              tc_commit(kv_empty(sk));
              tc_commit(kv_empty(sk));
            }
            ok = wait_all(kv_full(sv), phv) && (k != 0 || wait_all(o_empty(w), ph_q ^ 1)) && wait_all(p_full(w), ph_p);
            if (!ok) break;
            tc_fence_after();
            ph_p ^= 1;
            products(sv, min(8, pages - 8 * s), k == 0);
            if (leader) {
              if (k + 1 == nt) tc_commit(o_full(w));
              tc_commit(kv_empty(sv));
              tc_commit(kv_empty(sv));
            }
          }
          if (!ok) break;
          if (nt) ph_q ^= 1;
          const uint32_t at = st0 + 2 * nt_all;
          ph = ph0 ^ ((at / NS) & 1);
          st = at % NS;
          continue;
        }
        bool ok = true;
        if (apart) {
          // for the same reason both have seen the fills of all stages so far before they go through the ring together
          apart = false;
          if (leader) mbar_arrive(met(w ^ 1));
          ok = wait_all(met(w), meetings & 1);
          ++meetings;
        }
        ok = ok && wait_all(kv_full(st), ph) && (!nt || wait_all(q_full(w), ph_q)) && my_turn();
        if (!ok) break;
        tc_fence_after();
        if (nt)
          scores(nt == 1);
        else
          pass_turn();
        if (leader) tc_commit(kv_empty(st));
        next_stage();
        for (int s = 0; s < nt_all; ++s) {
          const bool keys = s + 1 < nt_all;
          const uint32_t sv = st, phv = ph;
          next_stage();
          ok = wait_all(kv_full(sv), phv) && (!keys || wait_all(kv_full(st), ph)) &&
               (!nt || s != 0 || wait_all(o_empty(w), ph_q ^ 1)) && my_turn() && (!nt || wait_all(p_full(w), ph_p));
          if (!ok) break;
          tc_fence_after();
          if (nt) {
            ph_p ^= 1;
            products(sv, min(8, pages - 8 * s), s == 0);
            // MMAs run in issue order: the next scores may overwrite the probabilities just
            // issued, and s_full implies that O is up to date
            if (keys) {
              scores(s + 2 == nt);
            } else {
              pass_turn();
              if (leader) tc_commit(o_full(w));
            }
          } else {
            pass_turn();
          }
          if (leader) tc_commit(kv_empty(sv));
          if (keys) {
            if (leader) tc_commit(kv_empty(st));
            next_stage();
          }
        }
        if (!ok) break;
        if (nt) ph_q ^= 1;
      }
    }
    __syncwarp();
  } else {
    // --------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    const int w = warp >> 2;
    const int i = threadIdx.x & 127;  // row of the tile
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lanes + w * KT, tO = tmem + lanes + 2 * KT + w * HD;
    const float sl2 = p.scale_log2;
    const uint64_t sl2p = pk2(sl2, sl2);
    int ns_ = 0, no = 0;  // scores and outputs taken
    bool ok = true;
    unsigned u = 0;
    int done = 0;  // steps
    {
      uint32_t zero[32];
#pragma unroll
      for (int c = 0; c < 32; ++c) zero[c] = 0;
      for (int c = 0; c < KT; c += 32) tmem_st32(tS + c, zero);
      tmem_wait_st();
    }
    // the first round: a step on nothing (zeros)
    for (bool dry = true; ok; dry = false) {
      int nt = 0, left = KT, stride = 0;  // steps; keys from a step on, and to the next one
      bool valid = false;
      int at = 0;
      if (!dry) {
        if (u >= u1) break;
        const Part t = part_of(u, done);
        if (!t.steps) break;
        u = t.next;
        done += t.steps;
        nt = t.count(w, PW);
        stride = t.one ? 2 * KT : KT;
        left = 16 * t.pages - (t.one ? (w ^ t.odd) * KT : 0);
        valid = i < HPG * PW && (t.one ? 0 : w * PW * HPG) + i < t.rows * HPG;
        at = t.at + w * (t.one ? t.rows : PW) * HPG + i;
        if (!nt) {
          if (t.one && valid) sg.stats[at] = make_float2(-INFINITY, -1.f);  // one step: nothing for this pipeline
          continue;
        }
      }
      float m = valid ? -INFINITY : 0.f;
      uint64_t l2 = pk2(0.f, 0.f);
      for (int s_ = dry ? -1 : 0; s_ < nt; ++s_, left -= stride) {
        if (!dry) {
          ok = __all_sync(0xffffffffu, wait_bar(s_full(w), ns_ & 1, p.err));
          if (!ok) break;
          ++ns_;
        }
        tc_fence_after();
        float s[KT];
        tmem_ld32(tS, reinterpret_cast<uint32_t*>(s));
        tmem_ld32(tS + 32, reinterpret_cast<uint32_t*>(s) + 32);
        tmem_ld32(tS + 64, reinterpret_cast<uint32_t*>(s) + 64);
        tmem_ld32(tS + 96, reinterpret_cast<uint32_t*>(s) + 96);
        tmem_wait_ld();
        if (left < KT) {
#pragma unroll
          for (int c = 16; c < KT; ++c) s[c] = c < left ? s[c] : -INFINITY;
        }
        float m4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int c = 4; c < 124; c += 8) {
#pragma unroll
          for (int y = 0; y < 4; ++y) m4[y] = max3(m4[y], s[c + y], s[c + 4 + y]);
        }
        const float mx = max3(max3(m4[0], s[124], s[125]), max3(m4[1], s[126], s[127]), max3(m4[2], m4[3], m4[3])) * sl2;
        const bool up = valid && mx > (m == -INFINITY ? m : m + LAG);
        if (__any_sync(0xffffffffu, up)) {
          const float f = up ? (m == -INFINITY ? 0.f : ex2(m - mx)) : 1.f;
          m = up ? mx : m;
          const uint64_t f2 = pk2(f, f);
          l2 = mul2(l2, f2);
          if (s_ > 0) {
#pragma unroll 1
            for (int c = 0; c < HD; c += 32) {
              float o[32];
              tmem_ld32(tO + c, reinterpret_cast<uint32_t*>(o));
              tmem_wait_ld();
#pragma unroll
              for (int x = 0; x < 32; x += 2) upk2(mul2(pk2(o[x], o[x + 1]), f2), o[x], o[x + 1]);
              tmem_st32(tO + c, reinterpret_cast<uint32_t*>(o));
            }
            tmem_wait_st();
          }
        }
        const float nb = m == -INFINITY ? 0.f : -m;
        const uint64_t nbp = pk2(nb, nb);
        uint32_t pr[KT / 2], rest[KT / 2];
        uint64_t sum[4] = {0, 0, 0, 0};  // pairs of 0.f
#pragma unroll
        for (int c = 0; c < KT / 2; ++c) {
          float a, e;
          upk2(fma2(pk2(s[2 * c], s[2 * c + 1]), sl2p, nbp), a, e);
          a = ex2(a);
          e = ex2(e);
          pr[c] = pack_p<T16>(a, e);
          rest[c] = pack_rest<T16>(a, e, pr[c]);
          sum[c & 3] = add2(sum[c & 3], pk2(a, e));
        }
        tmem_st32(tS, pr);
        tmem_st32(tS + 32, pr + 32);
        tmem_st32(tS + 64, rest);
        tmem_st32(tS + 96, rest + 32);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(dry ? warm(w) : p_full(w));
        l2 = add2(l2, add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
      }
      if (dry) {
        ready();
        take_share();
        u = u0;
        continue;
      }
      if (!ok) break;
      ok = __all_sync(0xffffffffu, wait_bar(o_full(w), no & 1, p.err));
      if (!ok) break;
      ++no;
      tc_fence_after();
      float* const dst = sg.part + static_cast<long long>(at) * HD;
#pragma unroll 1
      for (int c = 0; c < HD; c += 32) {
        uint32_t o[32];
        tmem_ld32(tO + c, o);
        tmem_wait_ld();
        if (c + 32 == HD) {
          tc_fence_before();
          mbar_arrive(o_empty(w));
        }
        if (valid) {
#pragma unroll
          for (int x = 0; x < 32; x += 8) st_global32(dst + c + x, o + x);
        }
      }
      if (valid) {
        float la, lb;
        upk2(l2, la, lb);
        sg.stats[at] = make_float2(m, la + lb);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

constexpr int JT = 128;  // threads of the join
constexpr int MAX_SMS = 512, MAX_PARTS = 2 * MAX_SMS;

// One CTA per row and query head: the parts of its item, in order, and the row's own.
template <int HD, typename T16>
__global__ void __launch_bounds__(JT) attn_join_kernel(const PagedAttnArgs p, const SharedGroups sg, int PW) {
  __shared__ float s_f[MAX_PARTS + 1];
  __shared__ float s_red[2][JT / 32];
  __shared__ float4 s_o[JT];
  grid_dep_launch();
  const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  grid_dep_wait();
  const int4 gp = __ldcg(sg.plan + 1 + b), all = __ldcg(sg.plan);
  if (!(b | h | tid)) *reinterpret_cast<int4*>(sg.next) = make_int4(0, 0, 0, 0);
  if (!gp.x) return;
  const Deal d = deal(static_cast<unsigned>(all.x), static_cast<unsigned>(all.y), static_cast<unsigned>(all.z));
  const Span sp(gp.w, gp.x, PW);
  const int HPG = p.H / p.G, g = h / HPG, r0 = gp.z, pair = (b - r0) / (2 * PW), p0 = pair * 2 * PW;
  const unsigned begin = static_cast<unsigned>(gp.y) + sp.item(g, pair);
  const unsigned w0 = d.worker_of(begin);
  const int ctas = static_cast<int>(d.worker_of(begin + (sp.steps - 1) * sp.cost(pair)) - w0) + 1;
  // one tile: two parts of each CTA
  const int rows = min(2 * PW, sp.rows - p0), two = rows <= PW ? 1 : 0, parts = ctas << two;
  const int at = part_at(r0, sp.rows, g, p0, p.H, HPG, w0) + (b - r0 - p0) * HPG + h - g * HPG;
  const long long own = static_cast<long long>(b) * p.H + h;
  auto place = [&](int i) { return at + 256 * (i >> two) + (two & i) * rows * HPG; };

  // factors: the parts', and the row's own last
  float2 st[MAX_PARTS / JT + 1];
  float M = -INFINITY;
#pragma unroll
  for (int k = 0; k < MAX_PARTS / JT + 1; ++k) {
    const int i = tid + k * JT;
    st[k] = make_float2(-INFINITY, 0.f);
    if (i <= parts) st[k] = i < parts ? __ldcg(sg.stats + place(i)) : __ldcg(sg.state_stats + own);
    M = fmaxf(M, st[k].x);
  }
  M = warp_max(M);
  if ((tid & 31) == 0) s_red[0][tid >> 5] = M;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < JT / 32; ++k) M = fmaxf(M, s_red[0][k]);
  const float top = M == -INFINITY ? 0.f : M;
  float L = 0.f;
#pragma unroll
  for (int k = 0; k < MAX_PARTS / JT + 1; ++k) {
    const int i = tid + k * JT;
    if (i > parts) break;
    // a sum below 0: nobody wrote the part. All others count, those of a factor 0 too: a value that is infinite or not a
    // number shows wherever it is visible
    const bool none = st[k].y < 0.f;
    const float f = none ? -1.f : exp2f(st[k].x - top);
    s_f[i] = f;
    L += none ? 0.f : f * st[k].y;
  }
  L = warp_sum(L);
  if ((tid & 31) == 0) s_red[1][tid >> 5] = L;
  __syncthreads();
  L = 0.f;
#pragma unroll
  for (int k = 0; k < JT / 32; ++k) L += s_red[1][k];

  constexpr int X = HD / 4, PG = JT / X;  // 16-byte pieces of a row; threads that share them
  const int x = tid % X, pg = tid / X;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = pg; i0 <= parts; i0 += 8 * PG) {
    float4 o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = i0 + k * PG;
      o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i > parts) continue;
      const float* const from = i < parts ? sg.part + static_cast<long long>(place(i)) * HD : sg.state + own * HD;
      o[k] = __ldcg(reinterpret_cast<const float4*>(from) + x);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = i0 + k * PG;
      const float f = i <= parts ? s_f[i] : -1.f;
      if (!(f < 0.f)) v = make_float4(v.x + f * o[k].x, v.y + f * o[k].y, v.z + f * o[k].z, v.w + f * o[k].w);
    }
  }
  s_o[tid] = v;
  __syncthreads();
  if (pg) return;
#pragma unroll
  for (int k = 1; k < PG; ++k) {
    const float4 e = s_o[k * X + x];
    v = make_float4(v.x + e.x, v.y + e.y, v.z + e.z, v.w + e.w);
  }
  const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
  *reinterpret_cast<uint2*>(static_cast<T16*>(p.o) + b * p.o_row + h * p.o_head + x * 4) =
      make_uint2(pack_out<T16>(v.x * inv, v.y * inv), pack_out<T16>(v.z * inv, v.w * inv));
  if (p.lse && x == 0) p.lse[own] = (M + log2f(L)) * 0.69314718055994531f;
}

template <int HD, typename T16>
cudaError_t prepare_hd() {
  return cudaFuncSetAttribute(attn_prefix_kernel<HD, T16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SCfg<HD>::SMEM);
}

template <int HD, typename T16>
cudaError_t launch_prefix_hd(const LaunchCtx& lc, const PagedAttnArgs& a, const SharedGroups& s, const AttnMaps& maps) {
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(THREADS);
  // no more CTAs than the longest rows that the table allows could keep busy
  const long long items = (static_cast<long long>(a.B) / (2 * attn_tile_positions(a.H, a.G)) + std::min(s.N, a.B / 2)) * a.G;
  const long long steps = items * ((a.blocks_per_seq + 7) / 8) / s.least_steps;
  cfg.gridDim = dim3(static_cast<unsigned>(std::max(1ll, std::min<long long>(lc.num_sms, steps))));
  cfg.dynamicSmemBytes = SCfg<HD>::SMEM;
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr[2];
  cfg.numAttrs = chain_attrs(lc, attr);
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, attn_prefix_kernel<HD, T16>, maps.q, maps.k, maps.v, a, s, attn_tile_positions(a.H, a.G),
                            maps.pool_rows);
}
template <int HD, typename T16>
cudaError_t launch_join_hd(const LaunchCtx& lc, const PagedAttnArgs& a, const SharedGroups& s) {
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(JT);
  cfg.gridDim = dim3(a.B, a.H);
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr[2];
  cfg.numAttrs = chain_attrs(lc, attr);
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, attn_join_kernel<HD, T16>, a, s, attn_tile_positions(a.H, a.G));
}

template <int HD, typename T16>
cudaError_t launch_hd(const LaunchCtx& lc, const PagedAttnArgs& a, const SharedGroups& s, const AttnMaps& maps) {
  if (s.alone) return launch_attn_paged_own(lc, a, s);
  // The prefix pass leaves its SMs with all their memory as shared memory, where 28 KB of L1 hold the loads in flight: a pass of
  // the rows' own parts took 1.6 times as long on them (104 and 170 us). So these two ask for what the own parts' CTAs need.
  LaunchCtx small = lc;
  small.carveout = attn_paged_own_carveout(a, s);
  cudaError_t e = launch_prefix_hd<HD, T16>(lc, a, s, maps);
  if (e == cudaSuccess) e = launch_attn_paged_own(small, a, s);
  return e == cudaSuccess ? launch_join_hd<HD, T16>(small, a, s) : e;
}

constexpr size_t ALIGN = 256;
size_t aligned(size_t n) { return (n + ALIGN - 1) / ALIGN * ALIGN; }

}  // namespace

cudaError_t prepare_attn_shared_kernels() {
  cudaError_t e = prepare_hd<64, bf16>();
  if (e == cudaSuccess) e = prepare_hd<64, f16>();
  if (e == cudaSuccess) e = prepare_hd<128, bf16>();
  if (e == cudaSuccess) e = prepare_hd<128, f16>();
  return e;
}

// Plan, the rows' own states, the prefix pass's parts, from a multiple of 256 bytes on.
size_t shared_attn_bytes(int B, int H, int d, int num_sms) {
  const size_t own = static_cast<size_t>(B) * H, parts = 2 * own + 256 * static_cast<size_t>(num_sms);
  return ALIGN + aligned(16 * (1 + PAGED_ATTN_MAX_B)) + aligned(8 * PAGED_ATTN_MAX_B) + aligned(8 * own) + aligned(8 * parts) +
         4 * static_cast<size_t>(d) * (own + parts);
}
void shared_attn_carve(SharedGroups* s, void* work, int B, int H, int d, int num_sms) {
  const size_t own = static_cast<size_t>(B) * H, parts = 2 * own + 256 * static_cast<size_t>(num_sms);
  char* at = reinterpret_cast<char*>(aligned(reinterpret_cast<uintptr_t>(work)));
  s->plan = reinterpret_cast<int4*>(at);
  at += aligned(16 * (1 + PAGED_ATTN_MAX_B));
  s->common = reinterpret_cast<int2*>(at);
  at += aligned(8 * PAGED_ATTN_MAX_B);
  s->state_stats = reinterpret_cast<float2*>(at);
  at += aligned(8 * own);
  s->stats = reinterpret_cast<float2*>(at);
  at += aligned(8 * parts);
  s->state = reinterpret_cast<float*>(at);
  s->part = s->state + own * d;
}

// AXON_SHARED_MIN_BYTES sets another limit, for measurements and tests of small cases; what is not a whole number, digits
// alone, does not.
static long long least_bytes() {
  const char* const limit = getenv("AXON_SHARED_MIN_BYTES");
  if (!limit || !*limit || limit[strspn(limit, "0123456789")]) return 128ll << 20;
  return std::min(strtoll(limit, nullptr, 10), 1ll << 60);
}

// Blocks read again come from L2, at some 10 TB/s, and the prefix pass and the join take some 13 us: less than 128 MB of
// them is faster read again. GPU time of rows with 16 to 64 tokens of their own, 32 / 8 heads of 128, shared / each for
// itself: 4 rows on 4096 tokens (50 MB spared) 21 / 18 us, 8 groups of 4 on 1024 (100 MB) 31 / 25, 16 rows on 4096 (251 MB)
// 26 / 35, 8 groups of 4 on 4096 (403 MB) 41 / 83.
void shared_attn_rules(SharedGroups* s, const PagedAttnArgs& a, int num_sms) {
  const long long block = 64ll * a.d * a.G;  // bytes of a block's keys and values
  const long long row = paged_attn_most_pages(1, 1, a.blocks_per_seq, a.window, a.sinks);
  s->least = 8;
  const long long bytes = least_bytes();
  s->least_spared = static_cast<int>(std::min((bytes + block - 1) / block, 1ll << 20));
  s->least_steps = 2;
  s->alone = row * (a.B - 1) < s->least_spared;
  s->sms = num_sms;
  s->tile = attn_tile_positions(a.H, a.G);
  s->next = a.ticket + paged_attn_ticket_bytes(num_sms) / 4 - 4;
}

cudaError_t launch_attn_shared(const LaunchCtx& lc, const PagedAttnArgs& a, const SharedGroups& s, const AttnMaps& maps) {
  if (a.H / a.G > 16 || a.B < 1 || a.B > PAGED_ATTN_MAX_B || s.N < 1 || s.N > MAX_N || !a.block_table || lc.num_sms > MAX_SMS ||
      2ll * a.B * a.H + 256ll * lc.num_sms > INT_MAX)
    return cudaErrorInvalidValue;
  if (a.d == 64) return lc.f16 ? launch_hd<64, f16>(lc, a, s, maps) : launch_hd<64, bf16>(lc, a, s, maps);
  if (a.d == 128) return lc.f16 ? launch_hd<128, f16>(lc, a, s, maps) : launch_hd<128, bf16>(lc, a, s, maps);
  return cudaErrorInvalidValue;
}
