// Attention of chunks of new tokens over the paged cache (axon_attn_prefill): causal,
// grouped queries, optional sliding window with sinks, on the 5th-generation tensor
// cores.
//
//   o = sum_t p_t v_t / sum_t p_t,  p_t = 2^(s_t - m),  s_t = scale log2(e) q.k_t
//
// A tile is 128 rows = PW consecutive positions x the H/G query heads of one kv head
// (PW = 128 / (H/G)). An item is two such tiles of consecutive positions, which share the
// keys: 128 per step (eight 16-token blocks), those of the sinks first. One CTA per SM takes items in
// turn; the copies and the first scores of the next item run under the end of the
// one before. Warps:
//   0..3, 4..7  softmax of tile 0 and 1, one thread per row (no shuffles), with 208
//               registers each (setmaxnreg), so that 128 scores stay in registers;
//   8           TMA producer: Q of an item, K and V through a ring of 32 KB (16 KB)
//               stages, lane i fetching the table entry of block i;
//   9, 11       MMA issuers of tile 0 and 1: S = Q K^T into TMEM, O += P V with P read back
//               from TMEM;
//   10          finds the items, two ahead, and publishes them.
// The 512 TMEM columns hold S0, S1 (128 each, later both terms of P, 64 each) and O0, O1.
//
// A probability enters the product in two 16-bit terms, p and what its rounding lost: 2^-17 of
// it is left out (bf16), so the output's own rounding is the only one that counts. Error against 64
// bits over that of a result rounded once, 64 and 128 dims, 16 to 2500 keys: 1.000 in both types;
// with one term 1.07 to 1.35, which is also more than the model's prefill kernel (k_attn_tc.cu,
// second terms for 16 keys of a step) loses, so that a model would have paid for its sinks in
// precision. The price is half as many products again; both in turn on one box, warm caches:
// 8191 positions 361 us against 282, a mixed batch 37.9 against 31.1, 16 tokens 7.8 either way.
//
// m is not the running maximum but a bound that lags: the maximum of a row's first visible step,
// raised (and O rescaled) only when it has become too small. Rounding to 16 bits is
// relative, so the error of a probability does not depend on m; what must hold is that
// none overflows, and the row sum of a step, which is needed anyway, tells: above 2^14 the
// step is taken again with m raised. So the usual step reads its scores once and
// computes no maximum. Steps under a mask, and a row's first, pass over the scores
// before that. The row sum is fp32, of the unrounded probabilities.
//
// Bound: the tensor pipe. A 128 x 128 tile at head_dim 128 takes 1536 tensor cycles (2 x 3 x 128^3
// operations at 8192 per cycle), 3072 for both, and per scheduler 512 cycles of the exponential
// unit and about 600 issue slots; the softmax of one tile runs under the products of the other.
// 8191 positions under a 4096-key window with sinks, 32 query heads, 8 kv heads: 386 to 420 us
// over the boxes, 0.98 to 1.07 PFLOP/s of the formula's operations and 1.47 to 1.60 of the pipe's, 77 to
// 84 % of the burst rate of cuBLAS (1.90); the pipe is active in 81 % of an SM's cycles. Instruction counts and fetches of the issuers matter (measured with one term): waits
// inlined with long loops 372 -> 369 us without them, issuers in uniform registers and in
// turns 369 -> 336, items in an order that evens out 336 -> 317, no local memory 309 -> 297.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "attn_tc.cuh"
#include "kernels.h"

namespace {

constexpr int THREADS = 384;
constexpr int KT = 128;  // keys per step
constexpr float LAG = 4.f;          // how far a maximum that is looked at may exceed m (log2)
constexpr float SUM_MAX = 16384.f;  // largest sum of a row's 128 probabilities

template <int HD>
struct KCfg {
  static constexpr int CH = HD / 64;                // 64-dim chunks (128-byte swizzled rows)
  static constexpr int CHUNK = 128 * 128;           // bytes of one 128-row chunk
  static constexpr int TILE = CH * CHUNK;           // Q, K or V tile
  static constexpr int STAGES = HD == 128 ? 5 : 8;  // K and V tiles in flight
  static constexpr int BARS = 2 * STAGES + 14 + 4;
  static constexpr int SMEM = 2 * TILE + STAGES * TILE + 8 * BARS + 2 * 32 + 16 + 1024;
};

// mbar_wait with a loop of few instructions: the kernel waits in some twenty places, and its
// instruction fetches are on the critical path.
AXON_DEV bool wait_bar(uint32_t bar, uint32_t parity, int* err) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
#pragma unroll 1
  while (!mbar_try_wait(bar, parity)) {
    if (global_ns() - t0 > 2000000000ull) {
      set_err(err, DEVERR_TIMEOUT);
      return false;
    }
  }
  return true;
}
AXON_DEV void st_global32(void* at, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
AXON_DEV void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Shared memory of CTA `rank` of the cluster, at the address that it has here.
AXON_DEV float ld_cluster(uint32_t at, int rank) {
  float v;
  asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %1, %2;\n ld.shared::cluster.f32 %0, [a];\n}"
               : "=f"(v)
               : "r"(at), "r"(rank)
               : "memory");
  return v;
}
AXON_DEV float4 ld_cluster4(uint32_t at, int rank) {
  float4 v;
  asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %4, %5;\n ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n}"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(at), "r"(rank)
               : "memory");
  return v;
}
AXON_DEV bool elect_one() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
  return r != 0;
}
AXON_DEV uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
AXON_DEV float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// A probability is at most the sum of its step, SUM_MAX: none saturates.
static_assert(SUM_MAX < 65504.f, "probabilities have to fit fp16");

// Bits c of 0 .. 15 with lo <= base + c < hi.
AXON_DEV uint32_t bits16(int base, int lo, int hi) {
  const int a = min(max(lo - base, 0), 16), b = min(max(hi - base, 0), 16);
  return b > a ? (1u << b) - (1u << a) : 0u;
}

// A work item: tiles of PC = 2 PW positions of one sequence's chunk and one kv head.
struct Item {
  int b, g, p0, row0, S, past;  // b < 0: none
};

// Item `item` of the launch: sequences whose chunks fill both tiles before the others (single
// tokens of a mixed batch, whose items are shorter), else in order; a sequence's position
// pairs from the end (those with the most keys first), the kv heads of a pair together.
// Offsets and lengths that do not fit are reported and give no items.
AXON_DEV Item find_item(const ChunkArgs& p, int PC, long long item) {
  Item r;
  r.b = -1;
  r.g = static_cast<int>(item % p.G);
  const long long pair = item / p.G;
  const int lane = threadIdx.x & 31;
  long long before = 0;
  for (int b0 = 0, rest = 0; rest < 2; b0 += 32) {
    if (b0 >= p.B) {  // once more, for the others
      b0 = -32;
      ++rest;
      continue;
    }
    int r0 = 0, len = 0, ps = 0;
    if (b0 + lane < p.B) {
      r0 = p.cu ? p.cu[b0 + lane] : (b0 + lane) * p.max_chunk;
      const int r1 = p.cu ? p.cu[b0 + lane + 1] : r0 + p.max_chunk;
      ps = p.cu ? p.past[b0 + lane] : 0;
      len = r1 - r0;
      const bool off = r0 < 0 || r1 < r0 || r1 > p.T || len > p.max_chunk;
      const bool far = ps < 0 || ps > p.blocks_per_seq * 16 - len;
      if (off || far) {
        if (off || len) set_err(p.err, off ? DEVERR_SEQ : DEVERR_POS);
        len = 0;
      }
      if ((b0 + lane == 0 && r0 != 0) || (b0 + lane == p.B - 1 && r1 != p.T)) set_err(p.err, DEVERR_SEQ);
    }
    const int mine = (2 * len > PC) == (rest == 0) ? (len + PC - 1) / PC : 0;
    int end = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, end, o);
      if (lane >= o) end += t;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, pair < before + end);
    if (hit) {
      const int src = __ffs(hit) - 1;
      r.b = b0 + src;
      r.row0 = __shfl_sync(0xffffffffu, r0, src);
      r.S = __shfl_sync(0xffffffffu, len, src);
      r.past = __shfl_sync(0xffffffffu, ps, src);
      r.p0 = static_cast<int>(before + __shfl_sync(0xffffffffu, end, src) - 1 - pair) * PC;
      return r;
    }
    before += __shfl_sync(0xffffffffu, end, 31);
  }
  return r;
}

// Into how many parts an item of `steps` key steps is split by a cluster of `parts` CTAs. With
// one-term probabilities a step took 1.3 us and joining the parts 6 us (8B width): 16 rows after 1000 cached tokens, 8
// steps, unsplit / 2 / 4 parts 15.9 / 16.5 / 13.4 us; after 500, 12.4 / 15.7; after 2000 (8
// parts) 26.0 / 15.5; 120 rows after 2000 31.1 / 20.2 (4 parts).
__host__ __device__ inline int split_of(int steps, int parts) {
  while (parts > 1 && steps < (parts == 2 ? 10 : 2 * parts)) parts >>= 1;
  return parts;
}

// Which blocks an item's tiles see: `ns` blocks of sinks, then those from `jlo` on. This CTA
// takes them from number `base` on, nb(w) of them for tile w; clears(w): among them is the block with
// the last token, and slots after it.
struct Span {
  int nw, jlo, ns, pend, base, parts;  // parts: how many CTAs have a share
  int nb0, nb1;
  bool clears0, clears1;
  AXON_DEV int nb(int w) const { return w ? nb1 : nb0; }
  AXON_DEV bool clears(int w) const { return w ? clears1 : clears0; }
  AXON_DEV int steps(int w) const { return (nb(w) + 7) >> 3; }
};
AXON_DEV Span span_of(const ChunkArgs& p, const Item& it, int PW, int part, int parts) {
  Span s;
  s.nw = it.p0 + PW < it.S ? 2 : 1;
  const int first = it.past + it.p0;
  s.jlo = p.window > 0 && first >= p.window ? (first - p.window + 1) >> 4 : 0;
  s.ns = min((p.sinks + 15) >> 4, s.jlo);
  s.pend = it.past + min(it.p0 + s.nw * PW, it.S);
  const int pend0 = it.past + min(it.p0 + PW, it.S);
  const int n0 = s.ns + ((pend0 + 15) >> 4) - s.jlo, n1 = s.ns + ((s.pend + 15) >> 4) - s.jlo;
  const int all = s.nw == 2 ? n1 : n0, steps = (all + 7) >> 3;
  s.parts = split_of(steps, parts);
  s.base = part < s.parts ? 8 * (steps * part / s.parts) : all;
  const int end = part < s.parts ? min(all, 8 * (steps * (part + 1) / s.parts)) : all;
  const bool last = (s.pend & 15) && end == all && end > s.base;
  s.clears0 = last && n0 == all;
  s.clears1 = last && n1 == all;
  s.nb0 = max(0, min(n0, end) - s.base);
  s.nb1 = max(0, min(n1, end) - s.base);
  return s;
}

// SPLIT: a cluster of CTAs shares one item, each with a part of its keys, and joins their
// states through distributed shared memory.
template <int HD, typename T16, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
    attn_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                      const __grid_constant__ CUtensorMap tmV, const ChunkArgs p, int PW, int pool_rows, int parts) {
  using C = KCfg<HD>;
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
  auto item_full = [&](int k) { return more + 8 * (12 + k); };
  auto item_empty = [&](int k) { return more + 8 * (14 + k); };
  auto turn = [&](int w) { return more + 8 * (16 + w); };
  const uint32_t items = bars + 8 * C::BARS;  // two Items of 32 bytes
  const uint32_t tmem_slot = items + 64;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int HPG = p.H / p.G;
  const int part = SPLIT ? static_cast<int>(blockIdx.x) % parts : 0;

  grid_dep_launch();
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
      mbar_init(item_full(w), 1);
      mbar_init(item_empty(w), 11);  // the producer, the issuers and the softmax warps
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
  grid_dep_wait();

  // The k-th item of this CTA, as warp 10 published it; called by whole warps. b < 0: no more
  // (or a wait ran out).
  auto take_item = [&](int k) {
    Item it;
    it.b = -1;
    if (SPLIT) {
      if (k > 0) return it;  // the cluster's one item, found before the roles part
    } else if (!__all_sync(0xffffffffu, wait_bar(item_full(k & 1), (k >> 1) & 1, p.err))) {
      return it;
    }
    const int* d = reinterpret_cast<const int*>(smem_raw + (items - raw) + 32 * (k & 1));
    it.b = d[0];
    it.g = d[1];
    it.p0 = d[2];
    it.row0 = d[3];
    it.S = d[4];
    it.past = d[5];
    __syncwarp();
    if (!SPLIT && lane == 0) mbar_arrive(item_empty(k & 1));
    return it;
  };
  auto put_item = [&](int k, const Item& it) {
    int* d = reinterpret_cast<int*>(smem_raw + (items - raw) + 32 * (k & 1));
    d[0] = it.b;
    d[1] = it.g;
    d[2] = it.p0;
    d[3] = it.row0;
    d[4] = it.S;
    d[5] = it.past;
  };
  if (SPLIT) {
    // every thread knows it, without a wait that could run out: they meet at barriers
    if (warp == 10) {
      const Item it = find_item(p, 2 * PW, blockIdx.x / parts);
      if (lane == 0) put_item(0, it);
    }
    __syncthreads();
  }

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 10) {
      // -------------------------------------------------------------- items
      for (int k = 0; !SPLIT; ++k) {
        // there and back over the CTAs, since items get shorter along a sequence
        const unsigned at = k & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
        const Item it = find_item(p, 2 * PW, at + static_cast<long long>(k) * gridDim.x);
        if (!__all_sync(0xffffffffu, wait_bar(item_empty(k & 1), ((k >> 1) & 1) ^ 1, p.err))) break;
        if (lane == 0) {
          put_item(k, it);
          mbar_arrive(item_full(k & 1));
        }
        __syncwarp();
        if (it.b < 0) break;
      }
    } else if (warp == 8) {
      // ----------------------------------------------------------- producer
      int iq[2] = {0, 0}, it = 0;
      bool ok = true;
      for (int k = 0; ok; ++k) {
        const Item item = take_item(k);
        if (item.b < 0) break;
        const Span sp = span_of(p, item, PW, part, SPLIT ? parts : 1);
        for (int w = 0; w < sp.nw; ++w) {
          if (!sp.nb(w)) continue;
          ok = __all_sync(0xffffffffu, wait_bar(q_empty(w), (iq[w] & 1) ^ 1, p.err));
          if (!ok) break;
          if (lane == 0) {
            mbar_arrive_expect_tx(q_full(w), HPG * PW * HD * 2);
            for (int c = 0; c < C::CH; ++c)
              tma_load_3d(sQ + w * C::TILE + c * C::CHUNK, &tmQ, q_full(w), c * 64, item.g * HPG,
                          item.row0 + item.p0 + w * PW);
          }
          ++iq[w];
        }
        const int nb = sp.nb(sp.nw - 1), nt = (nb + 7) >> 3;
        // pool row of this lane's block of step t; past the last block and for table entries
        // out of range (reported) the row lies outside the pool, where a box reads zeros
        auto pool_row = [&](int t) {
          const int i = t * 8 + lane;
          if (lane >= 8 || t >= nt || i >= nb) return pool_rows;
          const int x = i + sp.base;
          const int j = x < sp.ns ? x : x - sp.ns + sp.jlo;
          const int blk = p.block_table ? p.block_table[static_cast<long long>(item.b) * p.blocks_per_seq + j]
                                        : item.b * p.blocks_per_seq + j;
          if (blk < 0 || blk >= p.num_blocks) {
            set_err(p.err, DEVERR_BLOCK);
            return pool_rows;
          }
          return p.pool_row0 + (blk * p.G + item.g) * 16;
        };
        int next = pool_row(0);
        for (int t = 0; t < nt && ok; ++t) {
          const int y = next;
          next = pool_row(t + 1);
          for (int kv = 0; kv < 2; ++kv, ++it) {
            const int s = it % NS;
            ok = __all_sync(0xffffffffu, wait_bar(kv_empty(s), ((it / NS) & 1) ^ 1, p.err));
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(kv_full(s), C::TILE);
            __syncwarp();
            if (lane < 8)
              for (int c = 0; c < C::CH; ++c)
                tma_load_2d(sKV + s * C::TILE + c * C::CHUNK + lane * 2048, kv ? &tmV : &tmK, kv_full(s), c * 64, y);
          }
        }
      }
      // every copy lands before the CTA's shared memory goes away
      for (int w = 0; w < 2; ++w)
        if (iq[w] > 0) wait_bar(q_full(w), (iq[w] - 1) & 1, p.err);
      for (int i = it > NS ? it - NS : 0; i < it; ++i) wait_bar(kv_full(i % NS), (i / NS) & 1, p.err);
    } else if (warp != 10) {
      // -------------------------------------------------------- MMA issuers
      // A warp per tile. What an issuer itself executes is on the critical path (a product takes 64
      // cycles), so its values are the same in all lanes by construction, which lets the
      // descriptors live in uniform registers; one elected lane issues.
      const int w = warp == 9 ? 0 : 1;
      const bool lead = elect_one();
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
      uint32_t ph_q = 0, ph_p = 0;  // phases of this tile's items and steps
      uint32_t turns = 0;
      // The issuers alternate: one tile's products run under the other's softmax. (Left to
      // themselves they fall into step, both waiting for their softmax at the same time.)
      auto my_turn = [&]() { return wait_all(turn(w), (turns & 1) ^ (w ^ 1)); };
      // scores from the keys in stage st; the turn passes two products before the end, which is
      // what the other needs to start
      auto scores = [&](bool last) {
        const uint64_t kd = dK + st * (C::TILE >> 4);
        if (lead) {
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
        if (lead) mbar_arrive(turn(w ^ 1));
        ++turns;
      };
      auto same = [&](int v) { return __shfl_sync(0xffffffffu, v, 0); };
      Item item = take_item(0);
      for (int k = 0; same(item.b) >= 0; ++k) {
        const Span sp = span_of(p, item, PW, part, SPLIT ? parts : 1);
        const int nb = same(w < sp.nw ? sp.nb(w) : 0), nt = (nb + 7) >> 3;  // of this tile
        const int nt_all = same(sp.steps(sp.nw - 1));
        if (!nt_all) break;  // a CTA of a cluster without a share
        bool ok = wait_all(kv_full(st), ph) && (!nt || wait_all(q_full(w), ph_q)) && my_turn();
        if (!ok) break;
        tc_fence_after();
        if (nt)
          scores(nt == 1);
        else
          pass_turn();
        if (lead) tc_commit(kv_empty(st));
        next_stage();
        for (int t = 0; t < nt_all; ++t) {
          const bool mine = t < nt, keys = t + 1 < nt_all;
          const uint32_t sv = st, phv = ph;
          next_stage();
          ok = wait_all(kv_full(sv), phv) && (!keys || wait_all(kv_full(st), ph)) &&
               (!mine || t != 0 || wait_all(o_empty(w), ph_q ^ 1)) && my_turn() && (!mine || wait_all(p_full(w), ph_p));
          if (!ok) break;
          tc_fence_after();
          if (mine) {
            const uint64_t vd = dV + sv * (C::TILE >> 4);
            ph_p ^= 1;
            const int blocks = nb - 8 * t;
            if (t != 0 && blocks >= 8) {
              if (lead) {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                  tc_mma_f16_ts(tO, tS + x * 8, vd + x * 128, id_o, 1u);
                  tc_mma_f16_ts(tO, tS + KT / 2 + x * 8, vd + x * 128, id_o, 1u);
                }
              }
            } else if (lead) {
              // the first step starts the sums; blocks past the last hold no values
#pragma unroll 1
              for (int x = 0; x < min(8, blocks); ++x) {
                tc_mma_f16_ts(tO, tS + x * 8, vd + x * 128, id_o, (t | x) != 0 ? 1u : 0u);
                tc_mma_f16_ts(tO, tS + KT / 2 + x * 8, vd + x * 128, id_o, 1u);
              }
            }
            // MMAs run in issue order: the next scores may overwrite the probabilities just
            // issued, and s_full implies that O is up to date
            if (t + 1 < nt) {
              scores(t + 2 == nt);
            } else {
              pass_turn();
              if (lead) tc_commit(o_full(w));
            }
          } else {
            pass_turn();
          }
          if (lead) tc_commit(kv_empty(sv));
          if (keys) {
            if (lead) tc_commit(kv_empty(st));
            next_stage();
          }
        }
        if (!ok) break;
        if (nt) ph_q ^= 1;
        item = take_item(k + 1);
      }
    }
    __syncwarp();
  } else {
    // --------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int w = warp >> 2;
    const int i = threadIdx.x & 127;  // row of the tile
    const int pl = i / HPG, h = i - pl * HPG;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lanes + w * KT, tO = tmem + lanes + 2 * KT + w * HD;
    const float sl2 = p.scale_log2;
    const uint64_t sl2p = pk2(sl2, sl2);
    const bool wide = ((reinterpret_cast<uintptr_t>(p.o) | static_cast<uintptr_t>(p.o_row * 2) |
                        static_cast<uintptr_t>(p.o_head * 2)) & 31) == 0;  // 32-byte stores: whole sectors
    int ns_ = 0, no = 0, it = 0;  // scores and outputs taken; stages used by the items before
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const Item item = take_item(k);
      if (item.b < 0) break;
      const Span sp = span_of(p, item, PW, part, SPLIT ? parts : 1);
      const int nt_all = sp.steps(sp.nw - 1);
      if (sp.parts == 1 && (w >= sp.nw || !nt_all)) {
        it += 2 * nt_all;
        continue;
      }
      const int ip = item.p0 + w * PW + pl;
      const bool valid = i < HPG * PW && ip < item.S;
      const int pos = valid ? item.past + ip : -1;
      const int lo = (p.window > 0 && pos >= p.window) ? pos - p.window + 1 : 0;
      const int nt = w < sp.nw ? sp.steps(w) : 0;
      float m = valid ? -INFINITY : 0.f;
      uint64_t l2 = pk2(0.f, 0.f);
      for (int t = 0; t < nt; ++t) {
        const int tok0 = (sp.jlo - sp.ns + sp.base + t * 8) * 16;  // token of column 0, of steps past the sinks
        // padding rows reach no output: they alone never ask for it
        bool look = __any_sync(0xffffffffu, valid && (sp.base + t * 8 < sp.ns || tok0 + KT - 1 > pos || tok0 < lo || m == -INFINITY));
        ok = __all_sync(0xffffffffu, wait_bar(s_full(w), ns_ & 1, p.err));
        if (!ok) break;
        ++ns_;
        tc_fence_after();
        uint32_t pr[KT / 2], rest[KT / 2];
        uint64_t sum[4];
#pragma unroll 1
        for (int round = 0; round < 2; ++round) {
          if (look) {
            // Hidden scores to -inf (written back), and m raised to the step's maximum where it is far
            // below: a rolled loop over 64 columns, for the few steps that need it. Columns without a
            // mask are passed over once every row has a bound (a first step takes it from the first keys
            // that each row sees; should later ones exceed it by far, the sum tells).
            float mx = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < KT; c += 64) {
              uint32_t see[4], all = 0xffffu;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int blk = sp.base + t * 8 + c / 16 + x, at = blk < sp.ns ? blk * 16 : tok0 + c + x * 16;
                see[x] = bits16(at, lo, pos + 1) | bits16(at, 0, min(p.sinks, pos + 1));
                all &= see[x];
              }
              const bool mask = !round && __any_sync(0xffffffffu, valid && all != 0xffffu);
              if (!mask && !round && !__any_sync(0xffffffffu, fmaxf(m, mx) == -INFINITY)) continue;
              float s[64];
              tmem_ld32(tS + c, reinterpret_cast<uint32_t*>(s));
              tmem_ld32(tS + c + 32, reinterpret_cast<uint32_t*>(s) + 32);
              tmem_wait_ld();
              if (mask) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                  for (int u = 0; u < 16; ++u) s[x * 16 + u] = (see[x] >> u) & 1 ? s[x * 16 + u] : -INFINITY;
                tmem_st32(tS + c, reinterpret_cast<uint32_t*>(s));
                tmem_st32(tS + c + 32, reinterpret_cast<uint32_t*>(s) + 32);
              }
              float m4[4] = {mx, s[0], s[1], s[2]};
#pragma unroll
              for (int u = 3; u < 59; u += 8) {
#pragma unroll
                for (int y = 0; y < 4; ++y) m4[y] = max3(m4[y], s[u + y], s[u + 4 + y]);
              }
              mx = max3(max3(m4[0], s[59], s[60]), max3(m4[1], s[61], s[62]), max3(m4[2], m4[3], s[63]));
            }
            tmem_wait_st();
            const float mt = mx * sl2;
            const bool up = valid && mt > (m == -INFINITY ? m : m + LAG);
            if (__any_sync(0xffffffffu, up)) {
              const float f = up ? (m == -INFINITY ? 0.f : ex2(m - mt)) : 1.f;
              m = up ? mt : m;
              const uint64_t f2 = pk2(f, f);
              l2 = mul2(l2, f2);
              if (t > 0) {
#pragma unroll 1
                for (int c = 0; c < HD; c += 32) {
                  float o[32];
                  tmem_ld32(tO + c, reinterpret_cast<uint32_t*>(o));
                  tmem_wait_ld();
#pragma unroll
                  for (int u = 0; u < 32; u += 2) upk2(mul2(pk2(o[u], o[u + 1]), f2), o[u], o[u + 1]);
                  tmem_st32(tO + c, reinterpret_cast<uint32_t*>(o));
                }
                tmem_wait_st();
              }
            }
          }
          const float nb = m == -INFINITY ? 0.f : -m;
          const uint64_t nbp = pk2(nb, nb);
          float s[KT];
          tmem_ld32(tS, reinterpret_cast<uint32_t*>(s));
          tmem_ld32(tS + 32, reinterpret_cast<uint32_t*>(s) + 32);
          tmem_wait_ld();
          tmem_ld32(tS + 64, reinterpret_cast<uint32_t*>(s) + 64);
          tmem_ld32(tS + 96, reinterpret_cast<uint32_t*>(s) + 96);
#pragma unroll
          for (int x = 0; x < 4; ++x) sum[x] = 0;  // pairs of 0.f
#pragma unroll
          for (int c = 0; c < KT / 2; ++c) {
            if (c == KT / 4) tmem_wait_ld();
            float a, e;
            upk2(fma2(pk2(s[2 * c], s[2 * c + 1]), sl2p, nbp), a, e);
            a = ex2(a);
            e = ex2(e);
            pr[c] = pack_p<T16>(a, e);
            rest[c] = pack_rest<T16>(a, e, pr[c]);
            sum[c & 3] = add2(sum[c & 3], pk2(a, e));
          }
          sum[0] = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
          float sa, sb;
          upk2(sum[0], sa, sb);
          if (round || !__any_sync(0xffffffffu, valid && !(sa + sb <= SUM_MAX))) break;
          look = true;  // a score far above m: raise it and take the step again
        }
        tmem_st32(tS, pr);
        tmem_st32(tS + 32, pr + 32);
        tmem_st32(tS + 64, rest);
        tmem_st32(tS + 96, rest + 32);
        // the slots past the last token, before the product reads them
        if (sp.clears(w) && t == nt - 1) {
          const int iv = it + 2 * t + 1, sv = iv % NS;
          ok = __all_sync(0xffffffffu, wait_bar(kv_full(sv), (iv / NS) & 1, p.err));
          if (!ok) break;
          const int end = min(8, sp.nb(w) - 8 * t) * 16, first = end - 16 + (sp.pend & 15);
          for (int x = i; x < (end - first) * C::CH * 8; x += 128) {
            const int row = first + x / (C::CH * 8), piece = x % (C::CH * 8);
            *reinterpret_cast<uint4*>(smem_raw + (sKV - raw) + sv * C::TILE + (piece >> 3) * C::CHUNK + row * 128 +
                                      (piece & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(p_full(w));
        l2 = add2(l2, sum[0]);
      }
      it += 2 * nt_all;
      if (SPLIT && sp.parts > 1) {
        // the row's state into the stages that the keys and values no longer need
        if (nt && ok) ok = __all_sync(0xffffffffu, wait_bar(o_full(w), 0, p.err));
        tc_fence_after();
        asm volatile("barrier.cta.sync 1, 256;" ::: "memory");  // both tiles' products are done
        float la, lb;
        upk2(l2, la, lb);
        float* const stats = reinterpret_cast<float*>(smem_raw + (sKV - raw)) + (w * 128 + i) * 2;
        stats[0] = nt && ok ? m : -INFINITY;
        stats[1] = nt && ok ? la + lb : 0.f;
        // 16-byte pieces exchanged within the row, so that a warp's 32 rows fall on all banks
        uint4* const mine = reinterpret_cast<uint4*>(smem_raw + (sKV - raw) + 2048) + (w * 128 + i) * (HD / 4);
#pragma unroll 1
        for (int c = 0; c < HD; c += 32) {
          uint32_t o[32];
          if (nt && ok) {
            tmem_ld32(tO + c, o);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int u = 0; u < 32; ++u) o[u] = 0;
          }
#pragma unroll
          for (int u = 0; u < 8; ++u)
            mine[(c / 4 + u) ^ (i & (HD / 4 - 1))] = make_uint4(o[4 * u], o[4 * u + 1], o[4 * u + 2], o[4 * u + 3]);
        }
        break;
      }
      if (!ok) break;
      ok = __all_sync(0xffffffffu, wait_bar(o_full(w), no & 1, p.err));
      if (!ok) break;
      ++no;
      tc_fence_after();
      float la, lb;
      upk2(l2, la, lb);
      const float l = la + lb;
      const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
      uint4* dst = reinterpret_cast<uint4*>(static_cast<T16*>(p.o) + (static_cast<long long>(item.row0) + ip) * p.o_row +
                                            (item.g * HPG + h) * p.o_head);
#pragma unroll
      for (int c = 0; c < HD; c += 64) {
        uint32_t o[64];
        tmem_ld32(tO + c, o);
        tmem_ld32(tO + c + 32, o + 32);
        tmem_wait_ld();
        if (c + 64 == HD) {
          tc_fence_before();
          mbar_arrive(o_empty(w));
        }
        if (valid) {
#pragma unroll
          for (int u = 0; u < 64; u += 16) {
            uint32_t v[8];
#pragma unroll
            for (int x = 0; x < 8; ++x)
              v[x] = pack2<T16>(__uint_as_float(o[u + 2 * x]) * inv, __uint_as_float(o[u + 2 * x + 1]) * inv);
            if (wide) {
              st_global32(dst + ((c + u) >> 3), v);
            } else {
              dst[(c + u) >> 3] = make_uint4(v[0], v[1], v[2], v[3]);
              dst[((c + u) >> 3) + 1] = make_uint4(v[4], v[5], v[6], v[7]);
            }
          }
        }
      }
    }
  }
  // whether the cluster shares its item is the same for all of its CTAs and threads
  const int* const d = reinterpret_cast<const int*>(smem_raw + (items - raw));
  const int shares = SPLIT && d[0] >= 0 ? span_of(p, Item{d[0], d[1], d[2], d[3], d[4], d[5]}, PW, part, parts).parts : 1;
  if (SPLIT && shares > 1) {
    // each of its CTAs joins a share of the 256 rows
    __syncwarp();
    cluster_sync();
    if (warp < 8 && part < shares) {
      const int rows = 256 / shares;       // 32 .. 128: a row per 256 / rows threads
      const int per = 256 / rows, R = part * rows + threadIdx.x / per;
      const int w = R >> 7, i = R & 127, pl = i / HPG, h = i - pl * HPG, ip = d[2] + w * PW + pl;
      if (i < HPG * PW && ip < d[4]) {
        float M = -INFINITY, L = 0.f, f[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          f[x] = -INFINITY;
          if (x < shares) f[x] = ld_cluster(sKV + (w * 128 + i) * 8, x);
          M = fmaxf(M, f[x]);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          f[x] = M == -INFINITY ? 0.f : ex2(f[x] - M);
          if (x < shares) L += f[x] * ld_cluster(sKV + (w * 128 + i) * 8 + 4, x);
        }
        const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
        T16* const dst = static_cast<T16*>(p.o) + (static_cast<long long>(d[3]) + ip) * p.o_row + (d[1] * HPG + h) * p.o_head;
        for (int c = threadIdx.x % per; c < HD / 4; c += per) {
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          const uint32_t at = sKV + 2048 + ((w * 128 + i) * (HD / 4) + (c ^ (i & (HD / 4 - 1)))) * 16;
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            if (x < shares) {
              const float4 e = ld_cluster4(at, x);
              v = make_float4(v.x + f[x] * e.x, v.y + f[x] * e.y, v.z + f[x] * e.z, v.w + f[x] * e.w);
            }
          }
          *reinterpret_cast<uint2*>(dst + c * 4) = make_uint2(pack2<T16>(v.x * inv, v.y * inv), pack2<T16>(v.z * inv, v.w * inv));
        }
      }
    }
    __syncwarp();
    cluster_sync();  // nobody's shared memory goes away while another reads it
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int HD, typename T16>
cudaError_t prepare_hd() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  const cudaError_t e = cudaFuncSetAttribute(attn_chunk_kernel<HD, T16, false>, attr, KCfg<HD>::SMEM);
  return e == cudaSuccess ? cudaFuncSetAttribute(attn_chunk_kernel<HD, T16, true>, attr, KCfg<HD>::SMEM) : e;
}

// Clusters of 2, 4 and 8 CTAs that run at the same time (a GPC's SMs are no multiple of
// eight), by device.
std::atomic<int> g_clusters[64][4];

template <int HD, typename T16>
cudaError_t count_clusters() {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  for (int i = 1; i < 4 && e == cudaSuccess; ++i) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {1u << i, 1, 1};
    cfg.gridDim = dim3(1u << i);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = KCfg<HD>::SMEM;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, attn_chunk_kernel<HD, T16, true>, &cfg);
    g_clusters[dev & 63][i].store(n, std::memory_order_relaxed);
  }
  return e;
}

// CTAs that share an item: the most whose clusters all run at once, for the longest row that
// the table allows (a shorter one is split less, on the device).
int parts_for(const ChunkArgs& a, long long items, int PC) {
  long long keys = a.blocks_per_seq * 16ll;
  if (a.window > 0) keys = std::min(keys, 0ll + a.window + PC + a.sinks);
  const int steps = static_cast<int>(std::min((keys + KT - 1) / KT, 1ll << 20));
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 1;
  for (int i = 3; i > 0; --i)
    if (items <= g_clusters[dev & 63][i].load(std::memory_order_relaxed) && split_of(steps, 1 << i) == 1 << i) return 1 << i;
  return 1;
}

template <int HD, typename T16>
cudaError_t launch_hd(const LaunchCtx& lc, const ChunkArgs& a, const AttnMaps& maps) {
  const int PW = attn_tile_positions(a.H, a.G), PC = 2 * PW;
  const long long items = (static_cast<long long>(a.T) / PC + a.B) * a.G;  // at most
  const int parts = parts_for(a, items, PC);
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = KCfg<HD>::SMEM;
  cfg.stream = lc.stream;
  cudaLaunchAttribute chain[2], attr[3];
  cfg.numAttrs = chain_attrs(lc, chain);
  for (unsigned i = 0; i < cfg.numAttrs; ++i) attr[i] = chain[i];
  cfg.attrs = attr;
  if (parts > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim = {static_cast<unsigned>(parts), 1, 1};
    ++cfg.numAttrs;
    cfg.gridDim = dim3(static_cast<unsigned>(items) * parts);
    return cudaLaunchKernelEx(&cfg, attn_chunk_kernel<HD, T16, true>, maps.q, maps.k, maps.v, a, PW, maps.pool_rows, parts);
  }
  cfg.gridDim = dim3(static_cast<unsigned>(items < lc.num_sms ? items : lc.num_sms));
  return cudaLaunchKernelEx(&cfg, attn_chunk_kernel<HD, T16, false>, maps.q, maps.k, maps.v, a, PW, maps.pool_rows, 1);
}

}  // namespace

cudaError_t prepare_attn_chunk_kernels() {
  cudaError_t e = prepare_hd<64, bf16>();
  if (e == cudaSuccess) e = prepare_hd<64, f16>();
  if (e == cudaSuccess) e = prepare_hd<128, bf16>();
  if (e == cudaSuccess) e = prepare_hd<128, f16>();
  if (e == cudaSuccess) e = count_clusters<128, f16>();  // (all of them hold a whole SM per CTA)
  return e;
}

bool make_attn_maps_strided(AttnMaps* maps, const void* q, long long rows, long long q_row, long long q_head,
                            const void* kpool, const void* vpool, long long pool_rows, int H, int G, int d, bool f16) {
  if (pool_rows > 0x7fffff00ll) return false;  // box rows are 32-bit coordinates
  maps->pool_rows = static_cast<int>(pool_rows);
  return make_tma_3d_16(&maps->q, q, d, H, rows, H / G, attn_tile_positions(H, G), f16, q_head, q_row) &&
         make_tma_2d_16(&maps->k, kpool, pool_rows, d, 16, f16) && make_tma_2d_16(&maps->v, vpool, pool_rows, d, 16, f16);
}

cudaError_t launch_attn_chunk(const LaunchCtx& lc, const ChunkArgs& a, const AttnMaps& maps) {
  if (a.H / a.G > 16 || a.B < 1 || a.T < 1) return cudaErrorInvalidValue;
  if (a.d == 64) return lc.f16 ? launch_hd<64, f16>(lc, a, maps) : launch_hd<64, bf16>(lc, a, maps);
  if (a.d == 128) return lc.f16 ? launch_hd<128, f16>(lc, a, maps) : launch_hd<128, bf16>(lc, a, maps);
  return cudaErrorInvalidValue;
}
