// A token per row from its logits: temperature, top-k, top-p, min-p and a given random number.
//
//   w_i = exp((l_i - max) / temperature), in the order of the logits (equal ones by number):
//   the first k; of these the fewest whose sum reaches top_p of the k's; of these w_i >= min_p.
//   The token is the first, by number, at which the running sum of the kept weights passes u times their sum.
//
// Which token that is hangs on which side of a border a sum of up to 10^5 weights falls. fp32 sums (2^-24
// a step) would give another token than the formula's every few hundred draws, and atomics another from
// run to run. So weights are 64-bit integers, 2^44 w rounded, from w exact to about 2^-41 of its value (the
// exponent as a pair of fp32 numbers; powers of two from a table of 2^(-j/512) and three terms of a series):
// sums of integers are exact and have no order. A weight is off by half a unit and by 2^-41 of itself; n of them by n 2^-45 of
// the largest, 2^-26 for the longest vocabulary if all erred alike (finer units would take sums past 64 bits). The token
// is the one that 64-bit arithmetic gives unless u or top_p falls that near to a border, or min_p to a weight. Weights
// below half a unit are 0.
//
// A cluster of CTAs takes a row, each CTA a slice of it, which it keeps in shared memory, so that
// logits are read from HBM once whatever follows. Cuts (top-k, top-p) are found on histograms of counts
// or weights: 1024 bins that are even in the exponent, 32 per octave, joined over the cluster through distributed
// shared memory; a weight goes into a bin 16 bits at a time, so that no atomic has to return its carry
// (64-bit atomics on shared memory are loops). Where few logits are left, one CTA settles all of it among them; the
// crossing bin's logits go into lists, and the cut is found among these by their float bits, 10 at a time, by one CTA
// where they are 1024 at most. After a cut by weights each CTA knows its own sum, and only the one that the draw falls
// into adds up its weights again, warp by warp.
//
// The bound is the instructions, 62 a logit for the weights' histogram and 48 for their sum, and the cluster's
// barriers, 0.7 us each and as much again for the slowest CTA; the floor, reading the logits once, is far off.
// Measured: 1 row of 151936 logits with top-k and top-p 12.2 us, by temperature alone 10.1, the largest alone 4.4;
// 33 rows of 152064 16-bit logits that ask for different things 38.5 us; 64 rows of 128256 fp32 logits by top-p, two CTAs
// per SM and 1.7 times what runs at once, 76 us (a CTA: 1.5 us to load, 2 for the maximum, 7 for the histogram, 4 for the
// crossing, 3 for the lists, 4.5 for the cut); 512 rows of 32000 by temperature 58.5 us.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>

#include "kernels.h"

namespace cg = cooperative_groups;

namespace {

constexpr int ST = 512;        // threads
constexpr int SW = ST / 32;    // warps
constexpr int NB = 1024;       // bins
constexpr int MAX_CL = 16;     // CTAs of a cluster
constexpr int STEPS = 512;     // steps of an octave
constexpr int K_END = 45 * STEPS;  // weights from here on are 0
constexpr int BIN_SHIFT = 4;   // 32 bins per octave
constexpr int MAX_SLICE = 46 * 1024;  // logits of a CTA: 184 KB
static_assert(SAMPLE_MAX_VOCAB / MAX_CL <= MAX_SLICE, "the largest vocabulary has to fit a cluster");
static_assert(MAX_SLICE / ST <= 128, "sums of a thread's weights have to fit 32 bits");

typedef unsigned long long u64;

// 2^(-j/512) as a pair of fp32 numbers, by the series of exp in 64 bits.
struct PowerTable {
  float hi[STEPS], lo[STEPS];
  constexpr PowerTable() : hi(), lo() {
    for (int j = 0; j < STEPS; ++j) {
      const double y = -j * (0.693147180559945309417232 / STEPS);
      double term = 1.0, sum = 0.0;
      for (int n = 1; n < 30; ++n) {
        sum += term;
        term *= y / n;
      }
      hi[j] = static_cast<float>(sum);
      lo[j] = static_cast<float>(sum - static_cast<double>(hi[j]));
    }
  }
};
__device__ constexpr PowerTable g_powers{};

// A row's scale. With s = l - base the exponent (base 2) of a logit is s (ch + cl); its step j is s ch in 512ths, rounded,
// and k = top - j >= 1 counts the steps below the largest logit's.
struct Scale {
  float base, ch, cl;
  int top;
};

constexpr float MAGIC = 12582912.f;  // 1.5 * 2^23: adding it rounds |x| <= 2^22 to an integer, in the low bits
constexpr int MAGIC_BITS = 0x4b400000;

// Steps of logit l below the top; not below K_END (unsigned) where its weight is 0, -infinity and numbers that are none among
// them: s ch * 512 + MAGIC is then a float of another size or sign, whose bits lie far from MAGIC's.
AXON_DEV unsigned steps_of(const Scale& c, float l) {
  const float n = (l - c.base) * -c.ch;
  return static_cast<unsigned>(c.top + MAGIC_BITS - __float_as_int(fmaf(n, -static_cast<float>(STEPS), MAGIC)));
}

// Weights of two logits, in units of 2^-22 (hi) and 2^-44 (lo, signed), rounded; k: their steps. 2^(s (ch + cl) - top / 512) =
// 2^-(k/512) (1 - y + y^2/2 - y^3/6), y = (j/512 - s (ch + cl)) ln 2 < 6.8e-4, every sum and product that counts as a
// pair of fp32 numbers: exact to about 2^-41.
struct Weights {
  unsigned k[2];
  int hi[2], lo[2];
};
AXON_DEV Weights weights(const Scale& c, float l0, float l1, const float2* powers) {
  constexpr float LN2 = 0.693147182464599609375f, LN2_LO = -1.90465429995776804525e-9f;
  const uint64_t one = pk2(-1.f, -1.f);
  const uint64_t s = add2(pk2(l0, l1), pk2(-c.base, -c.base));
  const uint64_t n = mul2(s, pk2(-c.ch, -c.ch));
  uint64_t e = fma2(s, pk2(c.ch, c.ch), n);  // what the product lost
  e = fma2(s, pk2(c.cl, c.cl), e);
  constexpr float S = static_cast<float>(STEPS);
  const uint64_t t = fma2(n, pk2(-S, -S), pk2(MAGIC, MAGIC));
  const uint64_t g = fma2(add2(t, pk2(-MAGIC, -MAGIC)), pk2(1.f / S, 1.f / S), n);  // exact
  Weights w;
  float t0, t1;
  upk2(t, t0, t1);
  w.k[0] = static_cast<unsigned>(c.top + MAGIC_BITS - __float_as_int(t0));
  w.k[1] = static_cast<unsigned>(c.top + MAGIC_BITS - __float_as_int(t1));
  const float2 p0 = powers[w.k[0] & (STEPS - 1)], p1 = powers[w.k[1] & (STEPS - 1)];
  const uint64_t th = pk2(p0.x, p1.x), tl = pk2(p0.y, p1.y);
  const uint64_t yh = mul2(g, pk2(LN2, LN2)), ny = mul2(g, pk2(-LN2, -LN2));
  uint64_t yl = fma2(g, pk2(-LN2, -LN2), yh);  // y = yh - yl
  yl = fma2(g, pk2(-LN2_LO, -LN2_LO), yl);
  yl = fma2(e, pk2(LN2, LN2), yl);
  const uint64_t y = fma2(yl, one, yh);
  const uint64_t r = fma2(mul2(y, y), fma2(y, pk2(-1.f / 6.f, -1.f / 6.f), pk2(0.5f, 0.5f)), yl);
  // (th + tl) (1 - yh + r) = vh + vl
  const uint64_t q = mul2(th, yh), vh = fma2(q, one, th);
  const uint64_t lost = fma2(q, one, fma2(vh, one, th));
  const uint64_t vl = add2(fma2(th, r, fma2(th, ny, q)), add2(lost, fma2(tl, ny, tl)));
  // times 2^22 of the octave, in two integers
  const uint64_t sc = pk2(__uint_as_float((149u - w.k[0] / STEPS) << 23), __uint_as_float((149u - w.k[1] / STEPS) << 23));
  const uint64_t a = mul2(vh, sc), whole = add2(fma2(vl, sc, a), pk2(MAGIC, MAGIC));
  const uint64_t rest = fma2(vl, sc, fma2(add2(whole, pk2(-MAGIC, -MAGIC)), one, a));
  float h0, h1, r0, r1;
  upk2(whole, h0, h1);
  upk2(fma2(rest, pk2(4194304.f, 4194304.f), pk2(MAGIC, MAGIC)), r0, r1);
  w.hi[0] = __float_as_int(h0) - MAGIC_BITS;
  w.hi[1] = __float_as_int(h1) - MAGIC_BITS;
  w.lo[0] = __float_as_int(r0) - MAGIC_BITS;
  w.lo[1] = __float_as_int(r1) - MAGIC_BITS;
  return w;
}
AXON_DEV u64 joined(int hi, int lo) {
  return (static_cast<u64>(static_cast<unsigned>(hi)) << 22) + static_cast<u64>(static_cast<long long>(lo));
}
AXON_DEV u64 weight(const Scale& c, float l, const float2* powers) {
  const Weights w = weights(c, l, l, powers);
  return w.k[0] < K_END ? joined(w.hi[0], w.lo[0]) : 0;
}

// v in [0, 1) in units of 2^-64, rounded down; 0 for what is not above 0. (Integer code on purpose, here and for
// the scale: an SM does two 64-bit floating-point operations per cycle, and a division by all threads took 4 us.)
AXON_DEV u64 fraction64(float v) {
  if (!(v > 0.f)) return 0;
  const unsigned b = __float_as_uint(v);
  const u64 digits = (b & 0x7fffffu) | 0x800000u;  // v = digits * 2^(exponent - 150); below 2^-126 next to nothing
  const int up = static_cast<int>(b >> 23) - 86;
  return up >= 0 ? digits << up : up > -24 ? digits >> -up : 0;
}

// Logits as integers of the same order: the bits of the float, without those that logits of TL never differ in.
template <typename TL> struct Key { static constexpr int DROP = 0; };
template <> struct Key<bf16> { static constexpr int DROP = 16; };
template <> struct Key<f16> { static constexpr int DROP = 13; };
template <typename TL> AXON_DEV unsigned sample_key(float v) {
  const unsigned b = __float_as_uint(v + 0.f);  // -0 is 0
  return (b & 0x80000000u ? ~b : b | 0x80000000u) >> Key<TL>::DROP;
}
template <typename TL> AXON_DEV float sample_value(unsigned k) {
  constexpr int D = Key<TL>::DROP;
  k <<= D;
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k & ~((1u << D) - 1));
}

constexpr int FEW = 256;    // logits among which one CTA settles everything
constexpr int LIST = 512;   // a CTA's part of a list
constexpr int SOME = 1024;  // logits of a bin among which the cut is found without more bins
struct Shared {
  unsigned hist[2][2][NB];  // amounts, used in turn: as they come, bits 0 .. 15 and 16 .. 31; then 64 bits in two words
  unsigned high[NB];        // bits from 32 on, as they come
  u64 octave[2][NB / 32];   // this CTA's sums of 32 bins, with the histogram of the same turn
  float many[2][NB / 32];   // weights: about how many logits they are
  float2 powers[STEPS];
  uint2 mine[LIST];         // this CTA's list: key, number
  uint2 all[SOME];          // all CTAs' lists, in the first one
  uint2 near[32];           // of these, those about the cut
  unsigned mine_n, near_n;
  unsigned estimate;        // of the logits up to the crossing bin
  u64 below;                // this CTA's amounts below it
  u64 goal;                 // what the running sum had to reach
  bool any;                 // whether it did
  u64 cta[2];               // what the cluster exchanges, in turn
  u64 warp[SW];
  u64 found[3];             // the crossing bin: number, what is needed of it, all of it
  unsigned ends[2];
};

// v < 2^63 summed over the warp, 21 bits at a time; the sum is below 2^63.
AXON_DEV u64 warp_sum64(u64 v) {
  constexpr unsigned M = (1u << 21) - 1;
  const unsigned a = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v) & M);
  const unsigned b = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v >> 21) & M);
  const unsigned c = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v >> 42));
  return a + (static_cast<u64>(b) << 21) + (static_cast<u64>(c) << 42);
}
AXON_DEV u64 warp_scan64(u64 v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  return v;
}

template <typename TL>
struct Row {
  AXON_DEV static unsigned key_of(float v) { return sample_key<TL>(v); }
  AXON_DEV static float of_key(unsigned k) { return sample_value<TL>(k); }
  const SampleArgs& p;
  Shared& sh;
  const float* val;  // this CTA's slice
  int n, first;      // its length and the number of its first token
  int rank, CL;
  int turn = 0;      // exchanges so far
  int pass = 0;      // histograms so far
  int end;           // n rounded up to 128; there it holds NaN, which is never kept
  int seg;           // elements per warp, a multiple of 128
  Scale c;
  float m;           // the largest logit
  float share = 1.f;       // top-p, below 1: asked for
  u64 least = 0;     // min-p: the smallest weight that may stay
  u64 target = 0;    // what the last crossing's running sum had to reach
  u64 own = 0;       // known: this CTA's weights that are kept (first those up to the crossing bin)
  bool known = false;
  // what is kept: logits above vcut, and equal ones up to number icut
  float vcut = -INFINITY;
  int icut = 0x7fffffff;

  AXON_DEV bool kept(float l, int i) const {
    return l >= vcut && (icut == 0x7fffffff || l > vcut || first + i <= icut);  // icut: the same for all
  }
  AXON_DEV void cut_at(float v, int number) {
    vcut = v;
    icut = number;
  }

  // v (the same in all threads of a CTA): summed over the CTAs before this one, and over all.
  AXON_DEV void exchange(u64 v, u64& before, u64& all) {
    cg::cluster_group cluster = cg::this_cluster();
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) sh.cta[turn & 1] = v;
    cluster.sync();
    const u64 x = lane < CL ? *cluster.map_shared_rank(&sh.cta[turn & 1], lane) : 0;
    all = warp_sum64(x);
    before = warp_sum64(lane < rank ? x : 0);
    ++turn;
  }

  // Adds to bin b of the current histogram. Weights go there 16 bits at a time: no sum of a CTA's at most 2^16 logits
  // carries into the next word, and nothing has to come back from an atomic (64-bit ones on shared memory are loops).
  template <bool MASS>
  AXON_DEV void add(int b, u64 amount) {
    unsigned* h = &sh.hist[pass & 1][0][b];
    const unsigned low = static_cast<unsigned>(amount);
    if (MASS) {
      atomicAdd(h, low & 0xffffu);
      atomicAdd(h + NB, low >> 16);
      if (amount >> 32) atomicAdd(&sh.high[b], static_cast<unsigned>(amount >> 32));
    } else {
      atomicAdd(h, low);
    }
  }
  // This thread's bins of the current histogram, 2t and 2t + 1; weights as 64-bit numbers, in place of the words.
  template <bool MASS>
  AXON_DEV void own_bins(u64 (&a)[2]) {
    uint2* const l = reinterpret_cast<uint2*>(&sh.hist[pass & 1][0][0]) + threadIdx.x;
    a[0] = l->x;
    a[1] = l->y;
    if (MASS) {
      uint2* const m = reinterpret_cast<uint2*>(&sh.hist[pass & 1][1][0]) + threadIdx.x;
      uint2* const h = reinterpret_cast<uint2*>(&sh.high[0]) + threadIdx.x;
      a[0] += (static_cast<u64>(m->x) << 16) + (static_cast<u64>(h->x) << 32);
      a[1] += (static_cast<u64>(m->y) << 16) + (static_cast<u64>(h->y) << 32);
      *l = make_uint2(static_cast<unsigned>(a[0]), static_cast<unsigned>(a[1]));
      *m = make_uint2(static_cast<unsigned>(a[0] >> 32), static_cast<unsigned>(a[1] >> 32));
      *h = make_uint2(0, 0);
    }
  }
  AXON_DEV void clear(int which) {
    for (int i = threadIdx.x; i < 2 * NB; i += ST) (&sh.hist[which][0][0])[i] = 0;
  }

  // The smallest whole number that is at least part * sum, and at least 1; part < 1.
  AXON_DEV static u64 share_of(float part, u64 sum) {
    const u64 f = fraction64(part);
    return max(u64{1}, __umul64hi(f, sum) + (f * sum != 0));
  }
  // floor(u * sum) for u clamped to [0, 1)
  AXON_DEV static u64 draw(float u, u64 sum) {
    return u > 0.f ? __umul64hi(fraction64(fminf(u, 0.999999940395355224609375f)), sum) : 0;
  }

  // The first of this CTA's bins at which the running sum reaches `goal` goes to sh.found; a: this thread's bins 2t and 2t + 1.
  AXON_DEV void scan_bins(const u64 (&a)[2], u64 goal) {
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const u64 inc = warp_scan64(a[0] + a[1]);
    if (lane == 31) sh.warp[warp] = inc;
    __syncthreads();
    u64 sum = warp_sum64(lane < warp ? sh.warp[lane] : 0) + inc - a[0] - a[1];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (sum < goal && sum + a[i] >= goal) {
        sh.found[0] = 2 * t + i;
        sh.found[1] = goal - sum;
        sh.found[2] = a[i];
      }
      sum += a[i];
    }
    __syncthreads();
  }
  // About how many logits have that much weight in bin b: at least that many, and 2 % more at most, since a bin's weights
  // are that close to each other.
  AXON_DEV static float logits_of(u64 amount, int b) {
    return static_cast<float>(amount) * exp2f(b * (static_cast<float>(1 << BIN_SHIFT) / STEPS) - 44.f);
  }
  // The same for the sums of all CTAs' bins: first the 32 bins that it is among, by each CTA's sums of so many, then these,
  // by one warp. (All bins of all CTAs read by each took 10000 cycles with 8 CTAs, this 4000.) Clears the other
  // histogram, which everybody has read. With part_of >= 0 also how many logits there are up to the bin, and this CTA's
  // amounts below it.
  template <bool MASS>
  AXON_DEV bool crossing(float part_of, u64 goal) {
    cg::cluster_group cluster = cg::this_cluster();
    const int which = pass & 1, t = threadIdx.x, lane = t & 31;
    __syncthreads();
    {
      u64 a[2];
      own_bins<MASS>(a);
      u64 sum = a[0] + a[1];
      float n = MASS && part_of >= 0.f ? logits_of(a[0], 2 * t) + logits_of(a[1], 2 * t + 1) : 0.f;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (MASS) n += __shfl_xor_sync(0xffffffffu, n, o);
      }
      if ((t & 15) == 0) {
        sh.octave[which][t >> 4] = sum;
        if (MASS) sh.many[which][t >> 4] = n;
      }
    }
    cluster.sync();
    ++pass;
    if (t < 32) {
      u64 sum = 0, mine = 0;
      float n = 0.f;
#pragma unroll 4
      for (int r = 0; r < CL; ++r) {
        const u64 x = *cluster.map_shared_rank(&sh.octave[which][lane], r);
        sum += x;
        mine = r == rank ? x : mine;
        if (MASS) n += *cluster.map_shared_rank(&sh.many[which][lane], r);
      }
      u64 inc = warp_scan64(sum);
      const u64 all = __shfl_sync(0xffffffffu, inc, 31);
      target = part_of >= 0.f ? share_of(part_of, all) : goal;
      const unsigned at = __ballot_sync(0xffffffffu, inc >= target);
      if (at) {
        const int o = __ffs(at) - 1;
        const u64 before = __shfl_sync(0xffffffffu, inc - sum, o);
        u64 below = lane < o ? mine : 0;
        n = lane < o ? n : 0.f;
        sum = 0;
#pragma unroll 4
        for (int r = 0; r < CL; ++r) {
          const unsigned* h = cluster.map_shared_rank(&sh.hist[which][0][0], r);
          const u64 x = h[o * 32 + lane] + (MASS ? static_cast<u64>(h[NB + o * 32 + lane]) << 32 : 0);
          sum += x;
          mine = r == rank ? x : mine;
        }
        inc = warp_scan64(sum);
        const int f = __ffs(__ballot_sync(0xffffffffu, before + inc >= target)) - 1;
        if (MASS && part_of >= 0.f) {
          if (lane <= f && o * 32 + lane < NB - 1) n += logits_of(sum, o * 32 + lane);
          below = warp_sum64(below + (lane < f ? mine : 0));
          const unsigned logits = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(fminf(n, 1e6f)));
          if (lane == 0) {
            sh.estimate = logits;
            sh.below = below;
          }
        }
        if (lane == f) {
          sh.found[0] = o * 32 + f;
          sh.found[1] = target - before - (inc - sum);
          sh.found[2] = sum;
        }
      }
      if (lane == 0) {
        sh.goal = target;
        sh.any = at != 0;
      }
    }
    clear(which ^ 1);
    __syncthreads();
    target = sh.goal;
    if (MASS && part_of >= 0.f) own = sh.below;
    return sh.any;
  }

  AXON_DEV static int bin_of(unsigned k) { return min(static_cast<int>(k) >> BIN_SHIFT, NB - 1); }

  // The smallest key for which in(logit) holds, if it holds from some logit to the largest; called by a whole warp. `near`
  // is tried first (the full search took 2000 cycles).
  template <typename F>
  AXON_DEV unsigned lowest_key(float near, F in) const {
    unsigned lo = 0, hi = key_of(m);
    const int lane = threadIdx.x & 31;
    const unsigned k0 = key_of(near), at0 = k0 - 16 + lane;
    if (fabsf(near) < INFINITY && k0 > 16 && k0 < hi) {
      const unsigned hits = __ballot_sync(0xffffffffu, at0 >= hi || in(of_key(at0)));
      if (hits && !(hits & 1)) return min(hi, k0 - 16 + __ffs(hits) - 1);
    }
    while (lo < hi) {
      const unsigned step = (hi - lo) / 32 + 1, at = min(hi, lo + lane * step);  // (hi - lo) < 2^32 - 32
      const unsigned hits = __ballot_sync(0xffffffffu, in(of_key(at)));
      const int f = hits ? __ffs(hits) - 1 : 32;
      const unsigned top = f < 32 ? min(hi, lo + f * step) : hi;
      lo = f > 0 ? min(hi, lo + (f - 1) * step) + 1 : lo;
      hi = top;
    }
    return lo;
  }
  // ... whose bin is at most b.
  AXON_DEV unsigned lowest_in(int b) const {
    const int steps = b == NB - 1 ? K_END : (b + 1) << BIN_SHIFT;
    const float near = c.base + (static_cast<float>(c.top - steps) + 0.5f) / (c.ch * STEPS);
    return lowest_key(near, [&](float l) {
      const unsigned k = steps_of(c, l);
      return k < K_END && bin_of(k) <= b;
    });
  }

  // f(in, l, i, k, hi, lo) for the logits val[i], i0 <= i < i1 (multiples of 128; the slice is padded), by this warp, with
  // their steps and weights; in: kept, and of a weight. Where no lane keeps one of four, they are passed over.
  template <typename F>
  AXON_DEV void each(int i0, int i1, F f) {
    const bool some = vcut > -INFINITY;
    for (int i = i0 + (threadIdx.x & 31) * 4; i < i1; i += 128) {
      const float4 v = *reinterpret_cast<const float4*>(val + i);
      const float l[4] = {v.x, v.y, v.z, v.w};
      if (some && !__any_sync(0xffffffffu, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) >= vcut)) continue;
#pragma unroll
      for (int x = 0; x < 4; x += 2) {
        const Weights w = weights(c, l[x], l[x + 1], sh.powers);
#pragma unroll
        for (int y = 0; y < 2; ++y)
          f(w.k[y] < K_END && kept(l[x + y], i + x + y), l[x + y], i + x + y, w.k[y], w.hi[y], w.lo[y]);
      }
    }
  }
  // f(in, l, i), without weights; in: kept.
  template <typename F>
  AXON_DEV void each_plain(int i0, int i1, F f) {
    for (int i = i0 + (threadIdx.x & 31) * 4; i < i1; i += 128) {
      const float4 v = *reinterpret_cast<const float4*>(val + i);
      const float l[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int x = 0; x < 4; ++x) f(kept(l[x], i + x), l[x], i + x);
    }
  }
  // The amount of elements i0 .. i1 - 1 in every lane of the warp that calls it: how many equal v, or the sum of weights.
  template <bool TIES>
  AXON_DEV u64 amount(int i0, int i1, float v) {
    if (TIES) {
      unsigned n = 0;
      each_plain(i0, i1, [&](bool in, float l, int) { n += in && l == v; });
      return __reduce_add_sync(0xffffffffu, n);
    }
    int hi = 0, lo = 0;  // at most MAX_SLICE / ST elements per thread
    each(i0, i1, [&](bool in, float, int, unsigned, int h, int l) {
      hi += in ? h : 0;
      lo += in ? l : 0;
    });
    return warp_sum64(joined(hi, lo));
  }

  // The first token, by number, at which the running sum of the amounts passes t(sum of all): its number, and
  // its amount, in one thread of the cluster; -1 in the others.
  template <bool TIES, typename T>
  AXON_DEV int locate(float v, T t, u64& its, u64& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    u64 x = 0, here = own, before;  // x: the warps' amounts
    auto count = [&]() {
      const u64 mine = amount<TIES>(warp * seg, min(end, warp * seg + seg), v);
      __syncthreads();
      if (lane == 0) sh.warp[warp] = mine;
      __syncthreads();
      x = lane < SW ? sh.warp[lane] : 0;
    };
    const bool later = !TIES && known;  // most CTAs never have to
    if (!later) {
      count();
      here = warp_sum64(x);
    }
    exchange(here, before, all);
    const u64 target = t(all);
    if (target < before || target - before >= here) return -1;  // another CTA's
    if (later) count();
    u64 rest = target - before;
    u64 inc = warp_scan64(x);
    int at = __ffs(__ballot_sync(0xffffffffu, inc > rest)) - 1;  // the warp's part that it falls into
    rest -= __shfl_sync(0xffffffffu, inc - x, at);
    // which all warps share
    const int i0 = at * seg, i1 = min(end, i0 + seg), sub = (seg / 128 + SW - 1) / SW * 128;
    const u64 part = amount<TIES>(i0 + warp * sub, min(i1, i0 + warp * sub + sub), v);
    __syncthreads();
    if (lane == 0) sh.warp[warp] = part;
    __syncthreads();
    x = lane < SW ? sh.warp[lane] : 0;
    inc = warp_scan64(x);
    at = __ffs(__ballot_sync(0xffffffffu, inc > rest)) - 1;
    if (at != warp) return -1;
    rest -= __shfl_sync(0xffffffffu, inc - x, at);
    for (int i = i0 + warp * sub + 4 * lane; i < i1; i += 128) {
      const float4 f = *reinterpret_cast<const float4*>(val + i);
      const float l[4] = {f.x, f.y, f.z, f.w};
      u64 a[4];
#pragma unroll
      for (int y = 0; y < 4; ++y)
        a[y] = !kept(l[y], i + y) ? 0 : TIES ? static_cast<u64>(l[y] == v) : weight(c, l[y], sh.powers);
      const u64 mine4 = a[0] + a[1] + a[2] + a[3], sum = warp_scan64(mine4);
      const unsigned hit = __ballot_sync(0xffffffffu, sum > rest);
      if (hit) {
        if (lane != __ffs(hit) - 1) return -1;
        rest -= sum - mine4;
        int y = 0;
        for (; y < 3 && a[y] <= rest; ++y) rest -= a[y];
        its = y == 0 ? a[0] : y == 1 ? a[1] : y == 2 ? a[2] : a[3];
        return first + i + y;
      }
      rest -= __shfl_sync(0xffffffffu, sum, 31);
    }
    return -1;
  }

  // The logits that are kept and of keys lo .. hi, all CTAs': how many; and, if they are at most `most` and no CTA has more
  // than its list holds, in the first one's sh.all.
  AXON_DEV int gather(unsigned lo, unsigned hi, int most) {
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) sh.mine_n = 0;
    __syncthreads();
    const float from = fmaxf(of_key(lo), vcut), to = of_key(hi);
    const int i1 = min(end, warp * seg + seg);
    for (int i = warp * seg + 4 * lane; i < i1; i += 128) {
      const float4 v = *reinterpret_cast<const float4*>(val + i);
      const float l[4] = {v.x, v.y, v.z, v.w};
      bool any = false;
#pragma unroll
      for (int x = 0; x < 4; ++x) any |= l[x] >= from && l[x] <= to;
      if (!any) continue;
      for (int x = 0; x < 4; ++x) {
        const float f = x == 0 ? v.x : x == 1 ? v.y : x == 2 ? v.z : v.w;
        if (f >= from && f <= to && kept(f, i + x)) {
          const unsigned at = atomicAdd(&sh.mine_n, 1u);
          if (at < LIST) sh.mine[at] = make_uint2(key_of(f), first + i + x);
        }
      }
    }
    cluster.sync();
    const unsigned here = lane < CL ? *cluster.map_shared_rank(&sh.mine_n, lane) : 0;
    const int nc = __any_sync(0xffffffffu, here > LIST) ? 0x7fffffff : static_cast<int>(__reduce_add_sync(0xffffffffu, here));
    if (nc <= most && rank == 0) {
      for (int r = warp; r < CL; r += SW) {
        const unsigned count = __shfl_sync(0xffffffffu, here, r);
        const unsigned before = __reduce_add_sync(0xffffffffu, lane < r ? here : 0);
        const uint2* from = cluster.map_shared_rank(&sh.mine[0], r);
        for (unsigned i = lane; i < count; i += 32) sh.all[before + i] = from[i];
      }
    }
    __syncthreads();
    return nc;
  }

  // All that matters is among the nc logits in the first CTA's sh.all: the first k of them
  // stay (k > 0) and then the share, or those that the running sum of all weights needs to reach the target (k = 0); min-p;
  // the draw.
  AXON_DEV void settle(int nc, u64 k, float u, int* token, float* prob) {
    // two threads per logit; the weights are where the histograms were
    const int tid = threadIdx.x, i = tid >> 1;
    u64* const w = reinterpret_cast<u64*>(&sh.hist[0][0][0]);
    const uint2 me = i < nc ? sh.all[i] : make_uint2(0, 0);
    const u64 mine = i < nc ? weight(c, of_key(me.x), sh.powers) : 0;
    if (i < nc && !(tid & 1)) w[i] = mine;
    __syncthreads();
    unsigned ahead = 0;
    u64 sum = 0;
    for (int j = tid & 1; j < nc; j += 2) {
      const uint2 x = sh.all[j];
      const bool in = x.x > me.x || (x.x == me.x && x.y < me.y);
      ahead += in;
      sum += in ? w[j] : 0;
    }
    ahead += __shfl_xor_sync(0xffffffffu, ahead, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    bool stays = i < nc && (k == 0 || ahead < k);
    u64 goal = target;
    if (k > 0 && share < 1.f) goal = share_of(fmaxf(share, 0.f), cta_sum(stays && !(tid & 1) ? mine : 0));
    if (k == 0 || share < 1.f) stays = stays && sum < goal;
    stays = stays && (ahead == 0 || mine >= least);
    __syncthreads();
    if (i < nc && !(tid & 1) && !stays) w[i] = 0;
    const u64 total = cta_sum(stays && !(tid & 1) ? mine : 0), t = draw(u, total);
    sum = 0;
    for (int j = tid & 1; j < nc; j += 2) sum += sh.all[j].y < me.y ? w[j] : 0;
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    if (stays && !(tid & 1) && sum <= t && t - sum < mine) {
      *token = static_cast<int>(me.y);
      if (prob) *prob = static_cast<float>(static_cast<double>(mine) / static_cast<double>(total));
    }
  }
  // The cut among the nc logits in the first CTA's sh.all: key and, in the low word, the last number of it that stays. By bins
  // of this CTA alone, until one key is left.
  template <bool MASS>
  AXON_DEV u64 cut_list(int nc, u64 need) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned lo = 0xffffffffu, hi = 0;
    for (int i = tid; i < nc; i += ST) {
      lo = min(lo, sh.all[i].x);
      hi = max(hi, sh.all[i].x);
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) sh.warp[warp] = (static_cast<u64>(hi) << 32) | lo;
    for (int w = 0; w < 2; ++w) clear(w);
    __syncthreads();
    const u64 x = sh.warp[lane & (SW - 1)];
    lo = __reduce_min_sync(0xffffffffu, static_cast<unsigned>(x));
    hi = __reduce_max_sync(0xffffffffu, static_cast<unsigned>(x >> 32));
    u64 amount = ~u64{0};
    for (;;) {
      const int shift = max(0, 32 - __clz(hi - lo) - 10);
      __syncthreads();
      for (int i = tid; i < nc; i += ST) {
        const unsigned key = sh.all[i].x;
        if (key >= lo && key <= hi) add<MASS>((hi - key) >> shift, MASS ? weight(c, of_key(key), sh.powers) : 1);
      }
      __syncthreads();
      const int which = pass & 1;
      u64 a[2];
      own_bins<MASS>(a);
      scan_bins(a, need);
      hi -= static_cast<unsigned>(sh.found[0]) << shift;
      lo = max(lo, hi - min(hi, (1u << shift) - 1));
      need = sh.found[1];
      amount = sh.found[2];
      clear(which);
      __syncthreads();
      if (lo == hi) break;
      // a warp's worth of logits left, as a rule after the first bins: in order
      if (tid == 0) sh.near_n = 0;
      __syncthreads();
      for (int i = tid; i < nc; i += ST) {
        const uint2 x = sh.all[i];
        if (x.x < lo || x.x > hi) continue;
        const unsigned at = atomicAdd(&sh.near_n, 1u);
        if (at < 32) sh.near[at] = x;
      }
      __syncthreads();
      const int left = static_cast<int>(sh.near_n);
      if (left > 32) continue;
      if (warp == 0) {
        const uint2 me = lane < left ? sh.near[lane] : make_uint2(0, 0);
        const u64 w = lane < left ? MASS ? weight(c, of_key(me.x), sh.powers) : 1 : 0;
        u64 ahead = 0;
        bool last = true;  // of equal ones
        for (int j = 0; j < left; ++j) {
          const uint2 x = sh.near[j];
          const u64 wj = __shfl_sync(0xffffffffu, w, j);
          if (x.x > me.x || (x.x == me.x && x.y < me.y)) ahead += wj;
          last = last && !(x.x == me.x && x.y > me.y);
        }
        if (lane < left && ahead < need && ahead + w >= need)
          sh.found[0] = (static_cast<u64>(me.x) << 32) | (last ? 0x7fffffffu : me.y);
      }
      __syncthreads();
      return sh.found[0];
    }
    const u64 one = MASS ? weight(c, of_key(lo), sh.powers) : 1;
    if (amount == one) return (static_cast<u64>(lo) << 32) | 0x7fffffffu;
    const u64 which = (need + one - 1) / one;  // of the equal ones, by number
    for (int i = tid; i < nc; i += ST) {
      if (sh.all[i].x != lo) continue;
      unsigned n = 1;
      for (int j = 0; j < nc; ++j) n += sh.all[j].x == lo && sh.all[j].y < sh.all[i].y;
      if (n == which) sh.found[0] = (static_cast<u64>(lo) << 32) | sh.all[i].y;
    }
    __syncthreads();
    return sh.found[0];
  }
  // own: with those of this CTA's list (the crossing bin's) that are kept
  AXON_DEV void add_listed() {
    u64 sum = 0;
    for (int i = threadIdx.x; i < static_cast<int>(sh.mine_n); i += ST) {
      const float l = of_key(sh.mine[i].x);
      if (kept(l, static_cast<int>(sh.mine[i].y) - first)) sum += weight(c, l, sh.powers);
    }
    own += cta_sum(sum);
    known = true;
  }
  // v summed over the CTA
  AXON_DEV u64 cta_sum(u64 v) {
    const int lane = threadIdx.x & 31;
    v = warp_sum64(v);
    __syncthreads();
    if (lane == 0) sh.warp[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum64(lane < SW ? sh.warp[lane] : 0);
  }

  // Cuts what is kept to its first k, or (MASS, k = 0) to the fewest whose weights reach the share. true: the token is written.
  template <bool MASS>
  AXON_DEV bool cut(u64 k, float u, int* token, float* prob) {
    const int tid = threadIdx.x, i0 = (tid >> 5) * seg, i1 = min(end, i0 + seg);
    __syncthreads();  // the histogram is cleared
    if (MASS)
      each(i0, i1, [&](bool in, float, int, unsigned s, int hi, int lo) {
        if (in) add<true>(bin_of(s), joined(hi, lo));
      });
    else
      each_plain(i0, i1, [&](bool in, float l, int) {
        const unsigned s = steps_of(c, l);
        if (in && s < K_END) add<false>(bin_of(s), 1);
      });
    if (!crossing<MASS>(MASS ? fmaxf(share, 0.f) : -1.f, k)) return false;
    const int b = static_cast<int>(sh.found[0]);
    u64 need = sh.found[1], amount = sh.found[2];
    // keys of the bin
    if (tid < 64) {
      const unsigned key = tid < 32 ? lowest_in(b) : b > 0 ? lowest_in(b - 1) - 1 : key_of(m);
      if ((tid & 31) == 0) sh.ends[tid >> 5] = key;
    }
    __syncthreads();
    unsigned lo = sh.ends[0], hi = sh.ends[1];
    // Few in these bins? (How many is known of a count, and nearly of weights.)
    if (MASS ? sh.estimate <= FEW : k - need + amount <= FEW) {
      const int nc = gather(lo, key_of(m), FEW);
      if (nc <= FEW) {
        if (rank == 0) settle(nc, k, u, token, prob);
        return true;
      }
      cg::this_cluster().sync();  // the counts are read before the next list begins
    }
    // The logits of the bin in lists, where they have room.
    const float about = MASS ? logits_of(amount, b) : static_cast<float>(amount);
    bool listed = false;
    if (about <= CL * (LIST * 3 / 4) || b == NB - 1) {
      const int nc = gather(lo, hi, SOME);
      if (nc <= SOME) {
        u64 before, all;
        const u64 at = rank == 0 ? cut_list<MASS>(nc, need) : 0;
        exchange(at, before, all);
        const float v = of_key(static_cast<unsigned>(all >> 32));
        cut_at(v, min(static_cast<int>(all & 0x7fffffffu), v == vcut ? icut : 0x7fffffff));
        if (MASS) add_listed();
        return false;
      }
      listed = nc < 0x7fffffff;
    }
    // (the next pass's histogram was cleared with the crossing; the others may still read the last one)
    while (lo < hi && (MASS || need < amount)) {
      const unsigned width = hi - lo;  // less one
      const int shift = max(0, 32 - __clz(width) - 10);
      auto count = [&](unsigned key) {
        if (key >= lo && key <= hi) add<MASS>((hi - key) >> shift, MASS ? weight(c, of_key(key), sh.powers) : 1);
      };
      if (listed) {
        for (int i = tid; i < static_cast<int>(sh.mine_n); i += ST) count(sh.mine[i].x);
      } else {
        each_plain(i0, i1, [&](bool in, float l, int) {
          if (in) count(key_of(l));
        });
      }
      crossing<MASS>(-1.f, need);
      hi -= static_cast<unsigned>(sh.found[0]) << shift;
      lo = max(lo, hi - min(hi, (1u << shift) - 1));
      need = sh.found[1];
      amount = sh.found[2];
    }
    const float v = of_key(lo);
    // one logit, or (not MASS) some that all stay; of equal ones the first some stay
    if (MASS) {
      const u64 w = weight(c, v, sh.powers);
      need = (need + w - 1) / w;
      amount /= w;
    }
    if (need == amount) {
      cut_at(v, v == vcut ? icut : 0x7fffffff);
      if (MASS && listed) add_listed();
      return false;
    }
    u64 its, all, before;
    const int at = locate<true>(v, [&](u64) { return need - 1; }, its, all);
    __syncthreads();
    if (tid == 0) sh.found[0] = 0;
    __syncthreads();
    if (at >= 0) sh.found[0] = at + 1;
    __syncthreads();
    exchange(sh.found[0], before, all);
    cut_at(v, static_cast<int>(all) - 1);
    if (MASS && listed) add_listed();
    return false;
  }
};

template <typename TL> AXON_DEV void unpack16(const uint4& w, float* f);
template <> AXON_DEV void unpack16<float>(const uint4& w, float* f) {
  f[0] = __uint_as_float(w.x); f[1] = __uint_as_float(w.y); f[2] = __uint_as_float(w.z); f[3] = __uint_as_float(w.w);
}
template <> AXON_DEV void unpack16<bf16>(const uint4& w, float* f) {
  f[0] = bf_lo(w.x); f[1] = bf_hi(w.x); f[2] = bf_lo(w.y); f[3] = bf_hi(w.y);
  f[4] = bf_lo(w.z); f[5] = bf_hi(w.z); f[6] = bf_lo(w.w); f[7] = bf_hi(w.w);
}
template <> AXON_DEV void unpack16<f16>(const uint4& w, float* f) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
    f[2 * i] = h.x;
    f[2 * i + 1] = h.y;
  }
}

template <typename TL>
__global__ void __launch_bounds__(ST) sample_kernel(const SampleArgs p, int CL, int slice) {
  extern __shared__ __align__(16) float val[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / CL, rank = blockIdx.x % CL;
  cg::cluster_group cluster = cg::this_cluster();
  for (int i = tid; i < STEPS; i += ST) sh.powers[i] = make_float2(g_powers.hi[i], g_powers.lo[i]);
  for (int i = tid; i < 5 * NB; i += ST) (&sh.hist[0][0][0])[i] = 0;  // (high follows)
  grid_dep_launch();
  grid_dep_wait();

  // ---- the slice, and the largest logit (maxima pass over what is not a number)
  const int first = min(rank * slice, p.V), n = min(slice, p.V - first);
  const TL* const x = static_cast<const TL*>(p.logits) + b * p.row_stride + first;
  float best = -INFINITY;
  constexpr int PER = 16 / sizeof(TL);
  int done = 0;
  if ((reinterpret_cast<uintptr_t>(x) & 15) == 0) {
    done = n / PER * PER;
    constexpr int UN = 4;
    for (int i0 = tid * PER; i0 < done; i0 += UN * ST * PER) {
      uint4 w[UN];
#pragma unroll
      for (int k = 0; k < UN; ++k)
        if (i0 + k * ST * PER < done) w[k] = ld_stream16(x + i0 + k * ST * PER);
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const int i = i0 + k * ST * PER;
        if (i >= done) continue;
        float f[PER];
        unpack16<TL>(w[k], f);
#pragma unroll
        for (int e = 0; e < PER; ++e) best = fmaxf(best, f[e]);
#pragma unroll
        for (int e = 0; e < PER; e += 4)
          *reinterpret_cast<float4*>(val + i + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      }
    }
  }
  for (int i = done + tid; i < n; i += ST) {
    val[i] = to_f(x[i]);
    best = fmaxf(best, val[i]);
  }
  const int end = (n + 127) & ~127;
  for (int i = n + tid; i < end; i += ST) val[i] = __int_as_float(0x7fffffff);
  Row<TL> row{p, sh, val, n, first, rank, CL};
  row.end = end;
  row.seg = ((slice + SW - 1) / SW + 127) / 128 * 128;
  best = warp_max(best);
  if (lane == 0) sh.warp[warp] = __float_as_uint(best);
  __syncthreads();
  best = warp_max(lane < SW ? __uint_as_float(static_cast<unsigned>(sh.warp[lane])) : -INFINITY);
  if (tid == 0) sh.cta[1] = __float_as_uint(best);
  cluster.sync();
  float m = warp_max(lane < CL ? __uint_as_float(static_cast<unsigned>(*cluster.map_shared_rank(&sh.cta[1], lane))) : -INFINITY);
  u64 all = 0;

  const float temp = p.temperature ? p.temperature[b] : 1.f;
  const float low = p.min_p ? p.min_p[b] : 0.f;
  const bool nothing = m == -INFINITY, greedy = nothing || !(temp > 0.f);
  if (greedy || low > 1.f) {
    // the first of the largest alone
    int at = 0x7fffffff;
    for (int i = tid; i < n; i += ST)
      if (val[i] == m) at = min(at, first + i);
    at = __reduce_min_sync(0xffffffffu, at);
    __syncthreads();
    if (lane == 0) sh.warp[warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < SW; ++w) at = min(at, static_cast<int>(sh.warp[w]));
      sh.cta[0] = at;
    }
    cluster.sync();
    if (rank == 0 && warp == 0) {
      at = __reduce_min_sync(0xffffffffu, lane < CL ? static_cast<int>(*cluster.map_shared_rank(&sh.cta[0], lane)) : 0x7fffffff);
      if (lane == 0) {
        p.tokens[b] = nothing ? -1 : at;
        if (p.prob) p.prob[b] = nothing ? 0.f : 1.f;
      }
    }
    cluster.sync();  // nobody's shared memory goes away while another reads it
    return;
  }
  if (m == INFINITY) {  // infinite logits share everything
    for (int i = tid; i < n; i += ST) val[i] = val[i] == INFINITY ? 0.f : -INFINITY;
    m = 0.f;
  }
  // log2(e) / temperature as a pair: the quotient, and the quotient of what it left
  constexpr float LOG2E = 1.44269502162933349609375f, LOG2E_LO = 1.92596299112661746887e-8f;
  row.c.ch = fminf(LOG2E / temp, 3e38f);
  row.c.cl = 0.f;
  if (temp > 1e-30f && temp < 1e30f) row.c.cl = (fmaf(-row.c.ch, temp, LOG2E) + LOG2E_LO) / temp;
  row.m = m;
  // Far from 0 the logits that count lie within a factor of two of the largest: their distance from it is exact.
  row.c.base = fabsf(m) * row.c.ch < 128.f ? 0.f : m;
  row.c.top = 0;
  row.c.top = 1 - static_cast<int>(steps_of(row.c, m));
  __syncthreads();

  const int k = p.top_k ? p.top_k[b] : 0;
  const float share = p.top_p ? p.top_p[b] : 1.f, random = p.u[b];
  if (share < 1.f) row.share = share;
  if (low > 0.f) {
    const u64 most = weight(row.c, m, sh.powers);
    row.least = low < 1.f ? Row<TL>::share_of(low, most) : most;
  }
  int* const token = p.tokens + b;
  float* const prob = p.prob ? p.prob + b : nullptr;
  if ((k > 0 && k < p.V && row.template cut<false>(k, random, token, prob)) ||
      (row.share < 1.f && row.template cut<true>(0, random, token, prob))) {
    cluster.sync();
    return;
  }
  if (row.least) {
    if (warp == 0) {
      const unsigned key = row.lowest_key(
          NAN, [&](float l) { return l > -INFINITY && weight(row.c, l, sh.powers) >= row.least; });
      if (lane == 0) sh.ends[0] = key;
    }
    __syncthreads();
    const float v = Row<TL>::of_key(sh.ends[0]);
    if (v > row.vcut) {
      row.cut_at(v, 0x7fffffff);
      row.known = false;
    }
  }
  u64 its = 0;
  const int at = row.template locate<false>(0.f, [&](u64 sum) { return Row<TL>::draw(random, sum); }, its, all);
  if (at >= 0) {
    *token = at;
    if (prob) *prob = static_cast<float>(static_cast<double>(its) / static_cast<double>(all));
  }
  cluster.sync();
}

// CTAs per row: as many as run at once (two per SM), and slices of no more than 24K logits, two of which an SM holds with all else
// where they are below 19K. 64 rows of 128256 by top-p: 76 us with 16K, 82 with 32K, 139 with 8K (clusters of 16, a
// barrier of which waits for the slowest of as many); 512 rows of 32000 by temperature 58 with 16K, 71 with 32K, 77 with 8K.
int cluster_for(const LaunchCtx& lc, int B, int V) {
  int CL = 1;
  while (CL < MAX_CL && (V > CL * 24 * 1024 || (2ll * B * CL <= 2 * lc.num_sms && V / CL > 2 * ST))) CL *= 2;
  return CL;
}

template <typename TL>
cudaError_t launch_type(const LaunchCtx& lc, const SampleArgs& a) {
  const int CL = cluster_for(lc, a.B, a.V);
  const int slice = ((a.V + CL - 1) / CL + 127) & ~127;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.B) * CL);
  cfg.blockDim = dim3(ST);
  cfg.dynamicSmemBytes = static_cast<size_t>(slice) * 4;
  cfg.stream = lc.stream;
  cudaLaunchAttribute chain[2], attr[3];
  cfg.numAttrs = chain_attrs(lc, chain);
  for (unsigned i = 0; i < cfg.numAttrs; ++i) attr[i] = chain[i];
  attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
  attr[cfg.numAttrs].val.clusterDim = {static_cast<unsigned>(CL), 1, 1};
  ++cfg.numAttrs;
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, sample_kernel<TL>, a, CL, slice);
}

template <typename TL>
cudaError_t prepare_type() {
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<TL>, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SLICE * 4);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(sample_kernel<TL>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  return e;
}

}  // namespace

cudaError_t prepare_sample_kernels() {
  cudaError_t e = prepare_type<float>();
  if (e == cudaSuccess) e = prepare_type<bf16>();
  if (e == cudaSuccess) e = prepare_type<f16>();
  return e;
}

cudaError_t launch_sample(const LaunchCtx& lc, const SampleArgs& a, int precision) {
  if (a.V < 1 || a.V > SAMPLE_MAX_VOCAB || a.B < 1) return cudaErrorInvalidValue;
  if (precision == 1) return launch_type<float>(lc, a);
  return precision == 2 ? launch_type<f16>(lc, a) : launch_type<bf16>(lc, a);
}
