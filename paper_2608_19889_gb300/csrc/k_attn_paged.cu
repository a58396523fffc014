// Attention of one new token per sequence over the paged cache: causal, grouped
// queries, optional sliding window whose first tokens (sinks) stay visible.
//
//   o = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - m),  m = max_t scale q.k_t
//   t visible  <=>  t <= pos and (window = 0 or t > pos - window or t < sinks)
//
// Every visible key and value is read once: the bound is HBM (2 * d * 2 bytes per
// key and kv head against 4 * d * H/G operations). Measured at 8B width (32 query heads,
// 8 kv heads of 128; copy bandwidth 6.80 TB/s): 131072 keys of one row 537 MB in 86.5 us,
// 6.2 TB/s, 524288 keys 6.9 TB/s, 64 rows of 512 to 4096 tokens under a window of 2048 with
// sinks 450 MB in 75.3 us, 6.0 TB/s; the slope over lengths is 7.0 TB/s and what is fixed is
// 6 to 9 us: launch, lengths, table, first keys, and the join at the end.
//
// Work is cut evenly whatever the lengths: the visible 16-token pages of all
// (sequence, kv head) items form one line of units, which the workers (groups of
// 1, 2 or 4 warps, the warps of a group taking pages in turn) split into equal
// ranges. An item inside one range is finished there; the partial states (m, sum,
// O) of an item cut between workers go to the workspace, and the last of them to
// take a ticket joins them in order, so that results do not depend on timing. More than
// 16 parts are joined in two levels, by many workers: one CTA reading a few hundred parts, eight
// in flight, took longer than the pass over the keys (2 kv heads of 64, 32768 keys: 47.6 us
// with one level, 12.2 with two).
//
// A page's products run on mma.sync with the keys as the 16-row operand and the
// H/G heads (padded to 8 or 16) as the 8-wide one, S^T = K Q^T and O^T = V^T P^T:
// 8 heads fill the tile, where heads as rows would leave half of it empty. Keys
// and values go from global memory straight into the operand registers: the sum
// over dims and the order of output dims are free, so lane (r, c) takes 16-byte
// pieces of key rows r and r + 8, and of value rows 2c, 2c+1, 2c+8, 2c+9, whose
// 16-bit halves are then paired by byte permutes. P turns from accumulator to operand layout
// by movmatrix. P has two 16-bit terms (the products are far from bounding), so
// that the output's only rounding that counts is its own.
#include <math.h>

#include "attn_shared.cuh"
#include "kernels.h"

namespace {

constexpr int DW = 4;  // warps per CTA; three CTAs per SM (168 registers), a page of 8 KB in flight per warp

template <int HD, int NT>
struct DCfg {
  static constexpr int HEADS = 8 * NT;
  static constexpr int PITCH = HD + 4;                       // floats per head row of a warp's state
  static constexpr int STATE = HEADS * PITCH + 2 * HEADS;    // O, m, sum
  static constexpr int PART = HEADS * (HD + 2);              // floats of a partial state in the workspace
};

AXON_DEV uint32_t movm(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
AXON_DEV void group_sync(int group, int warps) {
  if (warps == 1)
    __syncwarp();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(warps * 32) : "memory");
}
// Two probabilities in [0, 1] as one 16-bit pair, and what the rounding lost.
template <typename T> AXON_DEV uint32_t pack_prob(float a, float b, float& ra, float& rb);
template <> AXON_DEV uint32_t pack_prob<bf16>(float a, float b, float& ra, float& rb) {
  const uint32_t p = pack_bf2(a, b);
  ra = a - bf_lo(p);
  rb = b - bf_hi(p);
  return p;
}
template <> AXON_DEV uint32_t pack_prob<f16>(float a, float b, float& ra, float& rb) {
  __half2 h = __floats2half2_rn(a, b);
  const float2 f = __half22float2(h);
  ra = a - f.x;
  rb = b - f.y;
  return *reinterpret_cast<uint32_t*>(&h);
}

// What a kernel may read that starts before the one in front of it has ended, from L2: an SM's L1 may hold what was there before.
template <bool SH, typename T> AXON_DEV T read(const T* at) { return SH ? __ldcg(at) : *at; }
// 16 bytes of a key or value. SH: the newest ones were written by the kernel before the prefix pass, which has waited for it
// before it lets this one start, but this one has waited for nothing; so a load that the non-coherent path may not serve. (As
// fast: 73.5 us and 73.9 for 57 rows with long own parts, 52.5 and 52.7 for groups of four; by .cg 75.8 and 52.7.)
template <bool SH> AXON_DEV uint4 read16(const void* at) { return SH ? ld_relaxed16(at) : ld_stream16(at); }
// Position of row b's query; -1: the row sees nothing.
template <bool SH> AXON_DEV int row_pos(const PagedAttnArgs& p, int b) {
  const int pos = read<SH>(p.ctx + b);
  if (pos < p.blocks_per_seq * 16ll) return max(pos, -1);
  set_err(p.err, DEVERR_POS);
  return -1;
}

// The share of CTA `cta` of `ctas`.
// LO: q has a second 16-bit term, and o one too where o_lo is given. SH: without the pages that a row's group has in
// common; a row that has some leaves its state for the join.
template <int HD, typename T16, int NT, bool LO, bool SH>
AXON_DEV void paged_items(const PagedAttnArgs& p, const SharedGroups& sg, float* const state, const unsigned* const before,
                          const int* const rpos, const int2* const shared, int* const s_last, unsigned ctas, unsigned cta) {
  using C = DCfg<HD, NT>;
  constexpr int KI = HD / 32;  // 16-byte pieces per key row and lane
  constexpr int VI = HD / 64;  // 16-byte pieces per value row and lane
  constexpr int MT = HD / 16;  // 16-dim tiles of O^T
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3;
  const int HPG = p.H / p.G;
  auto common = [&](int b) { return SH && !sg.alone ? shared[b] : make_int2(INT_MAX, INT_MAX); };
  const unsigned total = before[p.B] * p.G;  // below 2^31: the launcher saw to it

  // ---- rows that see nothing
  for (int b = cta; b < p.B; b += ctas) {
    if (before[b + 1] != before[b]) continue;
    if (SH && row_pages(p, rpos[b], common(b)).gap > 0) {
      // everything that the row sees is in common
      for (int i = tid; i < p.H * (HD / 4); i += DW * 32) {
        const long long at = static_cast<long long>(b) * p.H + i / (HD / 4);
        reinterpret_cast<float4*>(sg.state)[static_cast<long long>(b) * p.H * (HD / 4) + i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i % (HD / 4) == 0) sg.state_stats[at] = make_float2(-INFINITY, 0.f);
      }
      continue;
    }
    for (int i = tid; i < p.H * (HD / 8); i += DW * 32) {
      const int h = i / (HD / 8), x = i % (HD / 8);
      const long long at = b * p.o_row + h * p.o_head + x * 8;
      *reinterpret_cast<uint4*>(static_cast<T16*>(p.o) + at) = make_uint4(0, 0, 0, 0);
      if (LO && p.o_lo) *reinterpret_cast<uint4*>(static_cast<T16*>(p.o_lo) + at) = make_uint4(0, 0, 0, 0);
      if (p.lse && x == 0) p.lse[static_cast<long long>(b) * p.H + h] = -INFINITY;
    }
  }
  if (total == 0) return;

  // ---- workers: more warps share an item the longer the items are
  const unsigned avg = total / (p.B * p.G);
  int gs = avg >= 16 ? 4 : avg >= 4 ? 2 : 1;
  // more items than warps, as on the SMs that the prefix pass leaves: each takes whole ones, and has nobody to join
  // with (64 rows in groups of 4: 51.5 us when it was tried, 57 without this)
  if (SH && !sg.alone) {
    if (p.B * p.G >= ctas * DW)
      gs = 1;
    else if (p.B * p.G >= ctas * (DW / 2))
      gs = min(gs, 2);
  }
  const int group = warp / gs, wg = warp - group * gs;
  const unsigned all_groups = ctas * (DW / gs);
  // two pages per warp at least: less work per worker costs more joins than it saves (16 rows of
  // 256 keys, 8B width: 12.8 us with one page, 10.3 with two)
  const unsigned nw = min(all_groups, max(1u, total / (2 * gs)));
  const unsigned wid = cta + ctas * group;
  if (wid >= nw) return;
  // the first `extra` workers take a page more than the others
  const unsigned share = total / nw, extra = total - share * nw;
  const unsigned u0 = wid * share + min(wid, extra), u1 = u0 + share + (wid < extra ? 1 : 0);
  auto worker_of = [&](unsigned u) {
    const unsigned cut = extra * (share + 1);
    return u < cut ? u / (share + 1) : extra + (u - cut) / share;
  };

  int b = 0;
  {
    int hi = p.B;  // last row with before * G <= u0
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (before[mid] * p.G <= u0) b = mid; else hi = mid;
    }
  }
  const long long page_elems = 16ll * HD, block_elems = p.G * page_elems;
  const T16* const kpool = static_cast<const T16*>(p.k);
  const T16* const vpool = static_cast<const T16*>(p.v);
  float* const mine = state + warp * C::STATE;
  const float sl2 = p.scale_log2;

  for (unsigned u = u0; u < u1;) {
    while (before[b + 1] * p.G <= u) ++b;
    const RowPages rp = row_pages(p, rpos[b], common(b));
    const unsigned row0 = before[b] * p.G;
    const int g = static_cast<int>((u - row0) / rp.n);
    const unsigned item0 = row0 + static_cast<unsigned>(g) * rp.n;
    const int off = static_cast<int>(u - item0);
    const int cnt = static_cast<int>(min(static_cast<unsigned>(rp.n - off), u1 - u));

    // ---- this warp's pages: off + wg, off + wg + gs, ...
    const int pages = cnt > wg ? (cnt - wg + gs - 1) / gs : 0;
    auto logical = [&](int k) {  // page of the row that is this warp's k-th
      const int i = off + wg + k * gs;
      const int j = i < rp.sink ? i : i - rp.sink + rp.first;
      return SH && j >= rp.gap_at ? j + rp.gap : j;
    };
    auto entries = [&](int k0) {  // pool blocks of this warp's pages k0 .. k0 + 31, one per lane
      const int k = k0 + lane;
      if (k >= pages) return -1;
      const int j = logical(k);
      const int blk = p.block_table ? read<SH>(p.block_table + static_cast<long long>(b) * p.blocks_per_seq + j)
                                    : b * p.blocks_per_seq + j;
      if (blk >= 0 && blk < p.num_blocks) return blk;
      set_err(p.err, DEVERR_BLOCK);
      return -1;
    };
    int ent = entries(0);

    // ---- queries of the item's heads as the 8-wide operand
    uint32_t q[NT][KI][4];
    uint32_t ql[NT][KI][4];  // LO
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0), w = v;
        if (n * 8 + r < HPG) {
          const long long at = b * p.q_row + (g * HPG + n * 8 + r) * p.q_head + (4 * i + c) * 8;
          v = read<SH>(reinterpret_cast<const uint4*>(static_cast<const T16*>(p.q) + at));
          if (LO) w = ld16(static_cast<const T16*>(p.q_lo) + at);
        }
        q[n][i][0] = v.x; q[n][i][1] = v.y; q[n][i][2] = v.z; q[n][i][3] = v.w;
        ql[n][i][0] = w.x; ql[n][i][1] = w.y; ql[n][i][2] = w.z; ql[n][i][3] = w.w;
      }

    float m[NT][2], l[NT][2], o[NT][MT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
#pragma unroll
      for (int j = 0; j < MT; ++j) o[n][j][0] = o[n][j][1] = o[n][j][2] = o[n][j][3] = 0.f;
    }

    uint4 kv[2][KI], vv[4][VI];
    auto seen = [&](int t) { return t <= rp.pos && (t >= rp.lo || t < p.sinks); };
    // every token of the page is visible: the usual page, loaded without predicates
    auto whole_page = [&](int blk, int t0) {
      return blk >= 0 && t0 + 15 <= rp.pos && (t0 >= rp.lo || t0 + 15 < p.sinks);
    };
    const long long kofs = g * page_elems + r * HD + c * 8, vofs = g * page_elems + 2 * c * HD + r * 8;
    auto load_k = [&](int blk, int t0, bool all) {
      const T16* at = kpool + blk * block_elems + kofs;
      if (all) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < KI; ++i) kv[x][i] = read16<SH>(at + x * 8 * HD + i * 32);
      } else {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < KI; ++i)
            kv[x][i] = (blk >= 0 && seen(t0 + r + 8 * x)) ? read16<SH>(at + x * 8 * HD + i * 32) : make_uint4(0, 0, 0, 0);
      }
    };
    // rows of tokens that are not visible are left out, not multiplied by zero:
    // what a page holds there may be anything
    auto load_v = [&](int blk, int t0, bool all) {
      const T16* at = vpool + blk * block_elems + vofs;
      if (all) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int i = 0; i < VI; ++i) vv[x][i] = read16<SH>(at + ((x & 1) + 8 * (x >> 1)) * HD + i * 64);
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int t = (x & 1) + 8 * (x >> 1);
#pragma unroll
          for (int i = 0; i < VI; ++i)
            vv[x][i] = (blk >= 0 && seen(t0 + 2 * c + t)) ? read16<SH>(at + t * HD + i * 64) : make_uint4(0, 0, 0, 0);
        }
      }
    };
    if (pages > 0) {
      int blk = __shfl_sync(0xffffffffu, ent, 0), t0 = logical(0) * 16;
      bool all = whole_page(blk, t0);
      load_k(blk, t0, all);
      load_v(blk, t0, all);
      for (int k = 0; k < pages; ++k) {
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float e[4] = {0.f, 0.f, 0.f, 0.f}, f[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < KI; ++i) {
            const uint32_t a0[4] = {kv[0][i].x, kv[1][i].x, kv[0][i].y, kv[1][i].y};
            const uint32_t a1[4] = {kv[0][i].z, kv[1][i].z, kv[0][i].w, kv[1][i].w};
            mma16816<T16>(e, a0, &q[n][i][0]);
            mma16816<T16>(f, a1, &q[n][i][2]);
            if (LO) {
              mma16816<T16>(e, a0, &ql[n][i][0]);
              mma16816<T16>(f, a1, &ql[n][i][2]);
            }
          }
#pragma unroll
          for (int x = 0; x < 4; ++x) s[n][x] = e[x] + f[x];
        }
        const bool ok0 = all || (blk >= 0 && seen(t0 + r)), ok1 = all || (blk >= 0 && seen(t0 + r + 8));
        if (((k + 1) & 31) == 0) ent = entries(k + 1);
        const int nblk = __shfl_sync(0xffffffffu, ent, (k + 1) & 31), nt0 = logical(k + 1) * 16;
        const bool more = k + 1 < pages;
        const bool nall = whole_page(nblk, nt0);
        if (more) load_k(nblk, nt0, nall);

        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float mx[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            s[n][x] = ok0 ? s[n][x] * sl2 : -INFINITY;
            s[n][2 + x] = ok1 ? s[n][2 + x] * sl2 : -INFINITY;
            mx[x] = fmaxf(s[n][x], s[n][2 + x]);
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], w));
            mx[x] = fmaxf(mx[x], m[n][x]);
          }
          if (__any_sync(0xffffffffu, mx[0] > m[n][0] || mx[1] > m[n][1])) {
            const float f0 = mx[0] > m[n][0] ? ex2(m[n][0] - mx[0]) : 1.f;
            const float f1 = mx[1] > m[n][1] ? ex2(m[n][1] - mx[1]) : 1.f;
            m[n][0] = mx[0];
            m[n][1] = mx[1];
            l[n][0] *= f0;
            l[n][1] *= f1;
#pragma unroll
            for (int j = 0; j < MT; ++j) {
              o[n][j][0] *= f0;
              o[n][j][1] *= f1;
              o[n][j][2] *= f0;
              o[n][j][3] *= f1;
            }
          }
          const float b0 = m[n][0] == -INFINITY ? 0.f : m[n][0], b1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
          const float p0 = ex2(s[n][0] - b0), p1 = ex2(s[n][1] - b1);
          const float p2 = ex2(s[n][2] - b0), p3 = ex2(s[n][3] - b1);
          l[n][0] += p0 + p2;
          l[n][1] += p1 + p3;
          float r0, r1, r2, r3, z;
          ph[n][0] = movm(pack_prob<T16>(p0, p1, r0, r1));
          ph[n][1] = movm(pack_prob<T16>(p2, p3, r2, r3));
          pl[n][0] = movm(pack_prob<T16>(r0, r1, z, z));
          pl[n][1] = movm(pack_prob<T16>(r2, r3, z, z));
        }
#pragma unroll
        for (int i = 0; i < VI; ++i) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            auto word = [&](const uint4& v) { return x == 0 ? v.x : x == 1 ? v.y : x == 2 ? v.z : v.w; };
            const uint32_t w0 = word(vv[0][i]), w1 = word(vv[1][i]), w2 = word(vv[2][i]), w3 = word(vv[3][i]);
            const uint32_t a[4] = {__byte_perm(w0, w1, 0x5410), __byte_perm(w0, w1, 0x7632),
                                   __byte_perm(w2, w3, 0x5410), __byte_perm(w2, w3, 0x7632)};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma16816<T16>(o[n][4 * i + x], a, ph[n]);
              mma16816<T16>(o[n][4 * i + x], a, pl[n]);
            }
          }
        }
        if (more) load_v(nblk, nt0, nall);
        all = nall;
        blk = nblk;
        t0 = nt0;
      }
    }

    // ---- the group's states, joined
    float* const sO = mine;
    float* const sM = mine + C::HEADS * C::PITCH;
    float* const sL = sM + C::HEADS;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l[n][x] += __shfl_xor_sync(0xffffffffu, l[n][x], w);
        if (r == 0) {
          sM[n * 8 + 2 * c + x] = m[n][x];
          sL[n * 8 + 2 * c + x] = l[n][x];
        }
#pragma unroll
        for (int i = 0; i < VI; ++i)
#pragma unroll
          for (int w = 0; w < 2; ++w)
            *reinterpret_cast<float4*>(sO + (n * 8 + 2 * c + x) * C::PITCH + (r + 8 * i) * 8 + w * 4) =
                make_float4(o[n][4 * i + 2 * w][x], o[n][4 * i + 2 * w][2 + x], o[n][4 * i + 2 * w + 1][x],
                            o[n][4 * i + 2 * w + 1][2 + x]);
      }
    }
    group_sync(group, gs);
    const bool whole = off == 0 && cnt == rp.n;
    const float* const gstate = state + group * gs * C::STATE;
    const int gl = wg * 32 + lane;
    constexpr int PX = HD / 4;  // 4-dim pieces of a head
    auto finish = [&](int h, int x, float4 v, float M, float L) {
      if (SH && rp.gap > 0) {
        const long long at = static_cast<long long>(b) * p.H + g * HPG + h;
        *reinterpret_cast<float4*>(sg.state + at * HD + x * 4) = v;
        if (x == 0) sg.state_stats[at] = make_float2(M, L);
        return;
      }
      const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
      const long long at = b * p.o_row + (g * HPG + h) * p.o_head + x * 4;
      v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      const uint2 w = make_uint2(pack_out<T16>(v.x, v.y), pack_out<T16>(v.z, v.w));
      *reinterpret_cast<uint2*>(static_cast<T16*>(p.o) + at) = w;
      if (LO && p.o_lo) {
        const T16* hv = reinterpret_cast<const T16*>(&w);
        *reinterpret_cast<uint2*>(static_cast<T16*>(p.o_lo) + at) =
            make_uint2(pack2<T16>(v.x - to_f(hv[0]), v.y - to_f(hv[1])), pack2<T16>(v.z - to_f(hv[2]), v.w - to_f(hv[3])));
      }
      if (p.lse && x == 0)
        p.lse[static_cast<long long>(b) * p.H + g * HPG + h] = (M + log2f(L)) * 0.69314718055994531f;
    };
    // parts of the item: workers first .. last hold one each, in this slot of the workspace
    const unsigned first = worker_of(item0), last = worker_of(item0 + rp.n - 1);
    auto slot = [&](unsigned w) { return 2ll * w + (w > first ? 0 : 1); };
    auto put = [&](float* at, int h, int x, float4 v, float M, float L) {
      *reinterpret_cast<float4*>(at + h * HD + x * 4) = v;
      if (x == 0) {
        at[C::HEADS * HD + h] = M;
        at[C::HEADS * HD + C::HEADS + h] = L;
      }
    };
    for (int i = gl; i < HPG * PX; i += gs * 32) {
      const int h = i / PX, x = i % PX;
      float M = -INFINITY, L = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < gs; ++w) M = fmaxf(M, gstate[w * C::STATE + C::HEADS * C::PITCH + h]);
      const float base = M == -INFINITY ? 0.f : M;
      for (int w = 0; w < gs; ++w) {
        const float* st = gstate + w * C::STATE;
        const float f = ex2(st[C::HEADS * C::PITCH + h] - base);
        L += f * st[C::HEADS * C::PITCH + C::HEADS + h];
        const float4 e = *reinterpret_cast<const float4*>(st + h * C::PITCH + x * 4);
        v = make_float4(v.x + f * e.x, v.y + f * e.y, v.z + f * e.z, v.w + f * e.w);
      }
      if (whole)
        finish(h, x, v, M, L);
      else
        put(p.part + slot(wid) * C::PART, h, x, v, M, L);
    }
    group_sync(group, gs);
    if (!whole) {
      // `count` parts from worker w0 on, `step` apart, joined in order: into a slot of the second
      // level, or into the output
      const long long joined = 2ll * gridDim.x * DW;  // second level's slots
      auto join = [&](unsigned w0, int count, int step, bool out) {
        const long long from = step > 1 ? joined : 0;
        for (int i = gl; i < HPG * PX; i += gs * 32) {
          const int h = i / PX, x = i % PX;
          float M = -INFINITY, L = 0.f;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int j0 = 0; j0 < count; j0 += 8) {
            float pm[8], ps[8];
            float4 pv[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              pm[y] = -INFINITY;
              ps[y] = 0.f;
              pv[y] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (j0 + y < count) {
                const float* at = p.part + (from + slot(w0 + (j0 + y) * step)) * C::PART;
                pm[y] = __ldcg(at + C::HEADS * HD + h);
                ps[y] = __ldcg(at + C::HEADS * HD + C::HEADS + h);
                pv[y] = __ldcg(reinterpret_cast<const float4*>(at + h * HD + x * 4));
              }
            }
            float nm = M;
#pragma unroll
            for (int y = 0; y < 8; ++y) nm = fmaxf(nm, pm[y]);
            const float base = nm == -INFINITY ? 0.f : nm;
            const float f = ex2(M - base);
            M = nm;
            L *= f;
            v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              const float e = ex2(pm[y] - base);
              L += e * ps[y];
              v = make_float4(v.x + e * pv[y].x, v.y + e * pv[y].y, v.z + e * pv[y].z, v.w + e * pv[y].w);
            }
          }
          if (out) {
            finish(h, x, v, M, L);
          } else {
            put(p.part + (joined + slot(w0)) * C::PART, h, x, v, M, L);
          }
        }
      };
      // whether this is the last of `count` arrivals at a ticket (which is zero again then)
      auto last_of = [&](int* ticket, int count) {
        group_sync(group, gs);
        if (gl == 0) {
          const bool is_last = atom_add_acq_rel_gpu(ticket, 1) == count - 1;
          if (is_last) *ticket = 0;
          s_last[group] = is_last;
        }
        group_sync(group, gs);
        return s_last[group] != 0;
      };
      const int parts = static_cast<int>(last - first + 1);
      int radix = 16;
      while (radix * radix < parts) radix += 16;
      bool joiner = true;
      int step = 1, count = parts;
      if (parts > radix) {
        // two levels: the last of each `radix` neighbours joins them, the last of these joins the results
        const int j = static_cast<int>(wid - first) / radix * radix, n = min(radix, parts - j);
        joiner = last_of(p.ticket + gridDim.x * DW + slot(first + j), n);
        if (joiner) join(first + j, n, 1, false);
        step = radix;
        count = (parts + radix - 1) / radix;
      }
      if (joiner && last_of(p.ticket + first, count)) join(first, count, step, true);
      group_sync(group, gs);
    }
    u += cnt;
  }
}

template <int HD, typename T16, int NT, bool LO, bool SH>
AXON_DEV void paged_decode(const PagedAttnArgs& p, const SharedGroups& sg) {
  using C = DCfg<HD, NT>;
  extern __shared__ __align__(16) float sm[];
  float* const state = sm;                                        // [DW][STATE]
  unsigned* const before = reinterpret_cast<unsigned*>(sm + DW * C::STATE);  // [B + 1] pages of the rows before
  int* const rpos = reinterpret_cast<int*>(before + p.B + 1);                // [B] the rows' positions
  __shared__ int s_scan[DW], s_last[DW], s_cta;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  grid_dep_launch();
  // (SH: the prefix pass before this kernel lets it start once its inputs are there)
  if (!SH || sg.alone) grid_dep_wait();
  // CTAs that the work is cut for, and this one's number among them. SH: whoever comes takes the next number, until none is
  // left, so that all is done wherever and whenever the CTAs run.
  unsigned ctas = gridDim.x, cta = blockIdx.x;
  // SH: [B] the pages that the row has in common with others, from the first and to the last; then the plan they come from
  int2* const shared = reinterpret_cast<int2*>(before + 2 * p.B + 2);
  if (SH && !sg.alone) {
    // those that come when the prefix pass ends find that nothing is left
    volatile int* const next = sg.next;
    if (tid == 0) {
      const int all = next[1], own = next[3];
      s_cta = atomicAdd(sg.next, 1);
      s_last[0] = all > 0 && s_cta >= all;
      s_last[1] = own;
      __threadfence();
    }
    __syncthreads();
    if (s_last[0]) return;
    // the plan, read where the prefix pass has written it (1 us), else worked out (2.7 us)
    const GroupPlan gp(reinterpret_cast<int*>(shared + p.B), sg.N);
    int own = s_last[1];
    if (own > 0) {
      for (int b = tid; b < p.B; b += DW * 32) shared[b] = __ldcg(sg.common + b);
    } else {
      plan_groups<DW * 32, 0>(p, sg, gp, false);
      own = *gp.own;
      for (int b = tid; b < p.B; b += DW * 32) shared[b] = common_of(gp, sg.N, b);
    }
    ctas = min(gridDim.x, (NT == 1 ? 3 : 2) * own);
    if (tid == 0) next[1] = static_cast<int>(ctas);
    cta = s_cta;
    if (cta >= ctas) return;
    __syncthreads();
  }
  auto common = [&](int b) { return SH && !sg.alone ? shared[b] : make_int2(INT_MAX, INT_MAX); };

  // ---- pages before each row
  if (p.B <= 32) {
    if (warp == 0) {
      const int pos = lane < p.B ? row_pos<SH>(p, lane) : -1;
      const int n = row_pages(p, pos, SH && pos >= 0 ? common(lane) : make_int2(INT_MAX, INT_MAX)).n;
      int inc = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      if (lane < p.B) {
        before[lane] = inc - n;
        rpos[lane] = pos;
      }
      if (lane == 31) before[p.B] = inc;
    }
  } else {
    int base = 0;
    for (int b0 = 0; b0 < p.B; b0 += DW * 32) {
      const int b = b0 + tid;
      const int pos = b < p.B ? row_pos<SH>(p, b) : -1;
      const int n = row_pages(p, pos, SH && pos >= 0 ? common(b) : make_int2(INT_MAX, INT_MAX)).n;
      int inc = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      if (lane == 31) s_scan[warp] = inc;
      __syncthreads();
      int add = 0, all = 0;
#pragma unroll
      for (int w = 0; w < DW; ++w) {
        add += w < warp ? s_scan[w] : 0;
        all += s_scan[w];
      }
      if (b < p.B) {
        before[b] = base + add + inc - n;
        rpos[b] = pos;
      }
      base += all;
      __syncthreads();
    }
    if (tid == 0) before[p.B] = base;
  }
  __syncthreads();

  for (;;) {
    paged_items<HD, T16, NT, LO, SH>(p, sg, state, before, rpos, shared, s_last, ctas, cta);
    if (!SH) return;
    if (sg.alone) {
      if (blockIdx.x == gridDim.x - 1) check_groups<DW * 32>(p, sg);
      return;
    }
    __syncthreads();
    if (tid == 0) s_cta = atomicAdd(sg.next, 1);
    __syncthreads();
    cta = s_cta;
    if (cta >= ctas) return;
  }
}

template <int HD, typename T16, int NT, bool LO>
__global__ void __launch_bounds__(DW * 32, NT == 1 ? 3 : 2) attn_paged_decode_kernel(const PagedAttnArgs p) {
  paged_decode<HD, T16, NT, LO, false>(p, SharedGroups{});
}
// The rows' own parts beside the prefix pass. The same bound: 267 MB of 57 rows of 1 to 4096 tokens in 54 us on 144 SMs, 4.9 TB/s: a
// warp takes 1.5 us for a page, which is HBM's rate, and 8 us for an item's ends.
template <int HD, typename T16, int NT>
__global__ void __launch_bounds__(DW * 32, NT == 1 ? 3 : 2) attn_paged_own_kernel(const PagedAttnArgs p, const SharedGroups sg) {
  paged_decode<HD, T16, NT, false, true>(p, sg);
  grid_dep_wait();  // this kernel's end means the prefix pass's too, for the join
}

template <int HD, int NT>
constexpr size_t smem_bytes(int B) {
  return static_cast<size_t>(DW) * DCfg<HD, NT>::STATE * 4 + (2 * static_cast<size_t>(B) + 1) * 4;
}

// What the rows' own parts need beyond it: a pair of words for the alignment, the rows' common pages, the plan.
size_t shared_smem(int B, int N) { return 4 * (2 + 2 * static_cast<size_t>(B) + GroupPlan::ints(N)); }

template <int HD, typename T16>
cudaError_t prepare_hd() {
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  const int one = static_cast<int>(smem_bytes<HD, 1>(PAGED_ATTN_MAX_B));
  const int two = static_cast<int>(smem_bytes<HD, 2>(PAGED_ATTN_MAX_B));
  cudaError_t e = cudaFuncSetAttribute(attn_paged_decode_kernel<HD, T16, 1, false>, attr, one);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_paged_decode_kernel<HD, T16, 1, true>, attr, one);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_paged_decode_kernel<HD, T16, 2, false>, attr, two);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_paged_decode_kernel<HD, T16, 2, true>, attr, two);
  const int plan = static_cast<int>(shared_smem(PAGED_ATTN_MAX_B, SHARED_MAX_GROUPS));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_paged_own_kernel<HD, T16, 1>, attr, one + plan);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attn_paged_own_kernel<HD, T16, 2>, attr, two + plan);
  return e;
}

template <int HD, typename T16, int NT, bool LO>
cudaError_t launch_nt(const LaunchCtx& lc, const PagedAttnArgs& a, const SharedGroups* sg = nullptr) {
  const size_t smem = smem_bytes<HD, NT>(a.B) + (sg ? shared_smem(a.B, sg->N) : 0);
  // no more CTAs than pages that can be visible, at a page per warp
  const long long pages = paged_attn_most_pages(a.B, a.G, a.blocks_per_seq, a.window, a.sinks);
  const long long most = static_cast<long long>(lc.num_sms) * (NT == 1 ? 3 : 2);
  if (pages > 0x7fffffff) return cudaErrorInvalidValue;
  const long long grid = min(most, (pages + DW - 1) / DW);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(DW * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr[2];
  cfg.numAttrs = chain_attrs(lc, attr);
  cfg.attrs = attr;
  if (sg) return cudaLaunchKernelEx(&cfg, attn_paged_own_kernel<HD, T16, NT>, a, *sg);
  return cudaLaunchKernelEx(&cfg, attn_paged_decode_kernel<HD, T16, NT, LO>, a);
}

template <int HD, typename T16>
cudaError_t launch_own_hd(const LaunchCtx& lc, const PagedAttnArgs& a, const SharedGroups& sg) {
  return a.H / a.G <= 8 ? launch_nt<HD, T16, 1, false>(lc, a, &sg) : launch_nt<HD, T16, 2, false>(lc, a, &sg);
}

template <int HD, typename T16>
cudaError_t launch_hd(const LaunchCtx& lc, const PagedAttnArgs& a) {
  if (a.q_lo) return a.H / a.G <= 8 ? launch_nt<HD, T16, 1, true>(lc, a) : launch_nt<HD, T16, 2, true>(lc, a);
  return a.H / a.G <= 8 ? launch_nt<HD, T16, 1, false>(lc, a) : launch_nt<HD, T16, 2, false>(lc, a);
}

}  // namespace

size_t paged_attn_part_bytes(int H, int G, int d, int num_sms) {
  const bool two = H / G > 8;
  const size_t workers = static_cast<size_t>(num_sms) * (two ? 2 : 3) * DW;
  return 2 * 2 * workers * (two ? 16 : 8) * (d + 2) * 4;
}
// A ticket per cut item, which goes by its first worker (no other cut item begins there), and one per
// worker's slot. They stand in front of the states and their number goes by the SMs alone,
// so that no call's states lie where another shape or batch has its tickets.
// Four counters stand behind them, for the CTAs where rows share prefixes.
size_t paged_attn_ticket_bytes(int num_sms) { return 4 * 3 * static_cast<size_t>(num_sms) * 3 * DW + 16; }

cudaError_t prepare_attn_paged_kernels() {
  cudaError_t e = prepare_hd<64, bf16>();
  if (e == cudaSuccess) e = prepare_hd<64, f16>();
  if (e == cudaSuccess) e = prepare_hd<128, bf16>();
  if (e == cudaSuccess) e = prepare_hd<128, f16>();
  return e;
}

cudaError_t launch_attn_paged_decode(const LaunchCtx& lc, const PagedAttnArgs& a) {
  if (a.H / a.G > 16 || a.B < 1 || a.B > PAGED_ATTN_MAX_B || (a.o_lo && !a.q_lo))
    return cudaErrorInvalidValue;
  if (a.d == 64) return lc.f16 ? launch_hd<64, f16>(lc, a) : launch_hd<64, bf16>(lc, a);
  if (a.d == 128) return lc.f16 ? launch_hd<128, f16>(lc, a) : launch_hd<128, bf16>(lc, a);
  return cudaErrorInvalidValue;
}

int attn_paged_own_carveout(const PagedAttnArgs& a, const SharedGroups& s) {
  const bool two = a.H / a.G > 8;
  const size_t own = a.d == 64 ? two ? smem_bytes<64, 2>(a.B) : smem_bytes<64, 1>(a.B)
                               : two ? smem_bytes<128, 2>(a.B) : smem_bytes<128, 1>(a.B);
  const size_t cta = own + shared_smem(a.B, s.N) + 2048;  // static, and what an SM keeps for a CTA
  return static_cast<int>(min(size_t{100}, ((two ? 2 : 3) * cta * 100 + (228 << 10) - 1) / (228 << 10)));
}

cudaError_t launch_attn_paged_own(const LaunchCtx& lc, const PagedAttnArgs& a, const SharedGroups& s) {
  if (a.H / a.G > 16 || a.B < 1 || a.B > PAGED_ATTN_MAX_B || a.q_lo || s.N > SHARED_MAX_GROUPS) return cudaErrorInvalidValue;
  if (a.d == 64) return lc.f16 ? launch_own_hd<64, f16>(lc, a, s) : launch_own_hd<64, bf16>(lc, a, s);
  if (a.d == 128) return lc.f16 ? launch_own_hd<128, f16>(lc, a, s) : launch_own_hd<128, bf16>(lc, a, s);
  return cudaErrorInvalidValue;
}
