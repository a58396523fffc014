// A token per row from its logits: temperature, top-k, top-p, min-p and a given random number.
//
//   w_i = exp((l_i - max) / temperature), in the order of the logits (equal ones by number):
//   the first k; of these the fewest whose sum reaches top_p of the k's; of these w_i >= min_p.
//   The token is the first, by number, at which the running sum of the kept weights passes u times their sum.
//
// Which token that is hangs on which side of a border a sum of up to 10^5 weights falls. fp32 sums (2^-24
// a step) would give another token than the formula's every few hundred draws, and atomics another from
// run to run. So weights are 64-bit integers, 2^44 w rounded, exact to about 2^-41 of their value (the
// exponent as a pair of fp32 numbers; powers of two from a table of 2^(-j/256) and three terms of a series):
// sums of integers are exact and have no order, and the token is the one that 64-bit arithmetic
// gives unless u falls within some 2^-40 of a border.
//
// A cluster of CTAs takes a row, each CTA a slice of it, which it keeps in shared memory, so that
// logits are read from HBM once whatever follows. Cuts (top-k, top-p) are found on histograms of counts
// or weights: 1024 bins that are even in the exponent, then the crossing bin's interval of float
// bits in 1024 parts, until a part holds one number or one logit; each CTA adds up the bins of all
// the others through distributed shared memory. A weight goes into a bin as two 32-bit atomics with
// the carry between them (64-bit atomics on shared memory are loops).
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
constexpr float X_END = 45.5f; // exponents from here on have weight 0
constexpr int MAX_SLICE = SAMPLE_MAX_VOCAB / MAX_CL;

typedef unsigned long long u64;

// 2^(-j/256) * 2^44 for j = -128 .. 128, by the series of exp in 64 bits.
struct PowerTable {
  u64 v[257];
  constexpr PowerTable() : v() {
    for (int j = -128; j <= 128; ++j) {
      const double y = -j * (0.693147180559945309417232 / 256.0);
      double term = 1.0, sum = 0.0;
      for (int n = 1; n < 30; ++n) {
        sum += term;
        term *= y / n;
      }
      v[j + 128] = static_cast<u64>(sum * 17592186044416.0 + 0.5);
    }
  }
};
__device__ constexpr PowerTable g_powers{};

// A row's scale: exponent (base 2) of logit l is (m - l) (ch + cl).
struct Scale {
  float m, ch, cl;
};

AXON_DEV float exponent(const Scale& c, float l) { return (c.m - l) * c.ch; }

AXON_DEV u64 weight(const Scale& c, float l, const u64* powers) {
  const float s = c.m - l, p = s * c.ch;
  if (!(p < X_END)) return 0;  // also -infinity
  // what m - l and the product lost
  const float back = s - c.m, lost = (c.m - (s - back)) + (-l - back);
  float e = fmaf(s, c.ch, -p);
  e = fmaf(s, c.cl, e);
  e = fmaf(lost, c.ch, e);
  const float n = rintf(p), f = p - n, j = rintf(f * 256.f);
  const float g = fmaf(j, -1.f / 256.f, f);  // exact; the exponent is n + j / 256 + g + e
  // 2^-(g + e) = 1 - y + y^2 / 2 - y^3 / 6 + y^4 / 24, y = (g + e) ln 2 < 1.4e-3
  constexpr float LN2 = 0.693147182464599609375f, LN2_LO = -1.90465429995776804525e-9f;
  const float yh = g * LN2;
  float yl = fmaf(g, LN2, -yh);
  yl = fmaf(g, LN2_LO, yl);
  yl = fmaf(e, LN2, yl);
  const float y = yh + yl;
  const float q = y * y * fmaf(y, fmaf(y, 1.f / 24.f, -1.f / 6.f), 0.5f);
  constexpr float Q40 = 1099511627776.f;
  const int r = __float2int_rn(yh * -Q40) + __float2int_rn((q - yl) * Q40);  // 2^-40 steps
  const u64 w0 = powers[static_cast<int>(j) + 128];
  const long long more = (static_cast<long long>(r) * static_cast<long long>(w0 >> 14)) >> 26;
  const u64 w = w0 + static_cast<u64>(more);
  return ((2 * w >> static_cast<int>(n)) + 1) >> 1;
}

// Floats as integers of the same order.
AXON_DEV unsigned key_of(float v) {
  const unsigned b = __float_as_uint(v);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
AXON_DEV float of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

struct Shared {
  unsigned hist[2][3][NB];  // low and high words of the amounts, counts; used in turn
  u64 powers[257];
  u64 cta[2];               // what the cluster exchanges, in turn
  u64 warp[SW];
  u64 found[3];             // the crossing bin: number, what is needed of it, its count
  unsigned ends[2];
};

AXON_DEV u64 warp_sum64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
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

struct Row {
  const SampleArgs& p;
  Shared& sh;
  const float* val;  // this CTA's slice
  int n, first;      // its length and the number of its first token
  int rank, CL;
  int turn = 0;      // exchanges so far
  int pass = 0;      // histograms so far
  int seg;           // elements per warp, a multiple of 32
  Scale c;
  // what is kept: logits above vcut, and equal ones up to number icut
  float vcut = -INFINITY;
  int icut = 0x7fffffff;

  AXON_DEV bool kept(float l, int i) const { return l > vcut || (l == vcut && first + i <= icut); }

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

  // Adds to bin b of the current histogram.
  AXON_DEV void add(int b, u64 amount, bool mass, bool count) {
    unsigned* h = &sh.hist[pass & 1][0][b];
    if (mass) {
      const unsigned lo = static_cast<unsigned>(amount), hi = static_cast<unsigned>(amount >> 32);
      const unsigned up = hi + (atomicAdd(h, lo) > ~lo);
      if (up) atomicAdd(h + NB, up);
      if (count) atomicAdd(h + 2 * NB, 1u);
    } else {
      atomicAdd(h, 1u);
    }
  }
  AXON_DEV void clear(int which) {
    for (int i = threadIdx.x; i < 3 * NB; i += ST) (&sh.hist[which][0][0])[i] = 0;
  }

  // The bins of all CTAs; the first at which the running sum reaches the target goes to sh.found.
  // share: the target is this part of the sum, else `target`. Returns whether there is one.
  AXON_DEV bool crossing(bool mass, bool count, float share, u64 target) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const int which = pass & 1, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    ++pass;
    // this thread's bins: 2t, 2t + 1
    u64 a[2] = {0, 0};
    unsigned m[2] = {0, 0};
    for (int r = 0; r < CL; ++r) {
      const unsigned* h = cluster.map_shared_rank(&sh.hist[which][0][0], r);
      const uint2 lo = reinterpret_cast<const uint2*>(h)[t];
      a[0] += lo.x;
      a[1] += lo.y;
      if (mass) {
        const uint2 hi = reinterpret_cast<const uint2*>(h + NB)[t];
        a[0] += static_cast<u64>(hi.x) << 32;
        a[1] += static_cast<u64>(hi.y) << 32;
        if (count) {
          const uint2 k = reinterpret_cast<const uint2*>(h + 2 * NB)[t];
          m[0] += k.x;
          m[1] += k.y;
        }
      }
    }
    const u64 inc = warp_scan64(a[0] + a[1]);
    if (lane == 31) sh.warp[warp] = inc;
    clear(which ^ 1);  // everybody has read it before the barrier above
    __syncthreads();
    const u64 x = lane < SW ? sh.warp[lane] : 0;
    const u64 all = warp_sum64(x);
    u64 sum = warp_sum64(lane < warp ? x : 0) + inc - a[0] - a[1];
    if (share >= 0.f) {
      const u64 part = static_cast<u64>(static_cast<double>(share) * 18446744073709551616.0);  // share < 1
      target = __umul64hi(part, all) + (part * all != 0);
      if (target == 0) target = 1;
    }
    const bool any = all >= target;
    if (any) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (sum < target && sum + a[i] >= target) {
          sh.found[0] = 2 * t + i;
          sh.found[1] = target - sum;
          sh.found[2] = mass ? m[i] : a[i];
        }
        sum += a[i];
      }
    }
    __syncthreads();
    return any;
  }

  AXON_DEV int bin_of(float x) const { return min(static_cast<int>(x * (NB / X_END)), NB - 1); }

  // The smallest key whose bin is at most b; called by a whole warp.
  AXON_DEV unsigned lowest_key(int b) const {
    unsigned lo = 0, hi = key_of(c.m);  // hi: bin 0
    const int lane = threadIdx.x & 31;
    while (lo < hi) {
      const unsigned step = (hi - lo) / 32 + 1, at = min(hi, lo + lane * step);  // (hi - lo) < 2^32 - 32
      const float x = exponent(c, of_key(at));
      const bool in = x < X_END && bin_of(x) <= b;  // monotone: false, then true
      const unsigned hits = __ballot_sync(0xffffffffu, in);
      const int f = hits ? __ffs(hits) - 1 : 32;
      const unsigned top = f < 32 ? min(hi, lo + f * step) : hi;
      lo = f > 0 ? min(hi, lo + (f - 1) * step) + 1 : lo;
      hi = top;
    }
    return lo;
  }

  // Sum of `amount(l, i)` over this warp's part of the slice; in every lane.
  template <typename F>
  AXON_DEV u64 warp_amount(int i0, int i1, F amount) {
    u64 s = 0;
    for (int i = i0 + (threadIdx.x & 31); i < i1; i += 32) s += amount(val[i], i);
    return warp_sum64(s);
  }

  // The first token, by number, at which the running sum of the amounts passes t(sum of all): its number, and
  // its amount, in the threads of one warp of the cluster; -1 in the others.
  template <typename F, typename T>
  AXON_DEV int locate(F amount, T t, u64& its, u64& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const u64 mine = warp_amount(warp * seg, min(n, warp * seg + seg), amount);
    if (lane == 0) sh.warp[warp] = mine;
    __syncthreads();
    u64 x = lane < SW ? sh.warp[lane] : 0, before;
    const u64 here = warp_sum64(x);
    exchange(here, before, all);
    const u64 target = t(all);
    if (target < before || target - before >= here) return -1;  // another CTA's
    u64 rest = target - before;
    u64 inc = warp_scan64(x);
    int at = __ffs(__ballot_sync(0xffffffffu, inc > rest)) - 1;  // the warp's part that it falls into
    rest -= __shfl_sync(0xffffffffu, inc - x, at);
    // which all warps share
    const int i0 = at * seg, i1 = min(n, i0 + seg), sub = (seg / 32 + SW - 1) / SW * 32;
    const u64 part = warp_amount(i0 + warp * sub, min(i1, i0 + warp * sub + sub), amount);
    __syncthreads();
    if (lane == 0) sh.warp[warp] = part;
    __syncthreads();
    x = lane < SW ? sh.warp[lane] : 0;
    inc = warp_scan64(x);
    at = __ffs(__ballot_sync(0xffffffffu, inc > rest)) - 1;
    if (at != warp) return -1;
    rest -= __shfl_sync(0xffffffffu, inc - x, at);
    for (int i = i0 + warp * sub; i < i1; i += 32) {
      const u64 a = i + lane < i1 ? amount(val[i + lane], i + lane) : 0;
      const u64 sum = warp_scan64(a);
      const unsigned hit = __ballot_sync(0xffffffffu, sum > rest);
      if (hit) {
        const int f = __ffs(hit) - 1;
        its = __shfl_sync(0xffffffffu, a, f);
        return first + i + f;
      }
      rest -= __shfl_sync(0xffffffffu, sum, 31);
    }
    return -1;
  }

  // Cuts what is kept to its first k (share < 0), or to the fewest whose weights reach this share.
  AXON_DEV void cut(float share, u64 k) {
    const bool mass = share >= 0.f;
    const int i0 = (threadIdx.x >> 5) * seg + (threadIdx.x & 31), i1 = min(n, ((threadIdx.x >> 5) + 1) * seg);
    __syncthreads();  // the histogram is cleared
    for (int i = i0; i < i1; i += 32) {
      const float l = val[i], x = exponent(c, l);
      if (x < X_END && kept(l, i)) add(bin_of(x), mass ? weight(c, l, sh.powers) : 1, mass, false);
    }
    if (!crossing(mass, false, share, k)) return;
    const int b = static_cast<int>(sh.found[0]);
    u64 need = sh.found[1], count = mass ? 0 : sh.found[2];
    // keys of the bin
    if (threadIdx.x < 32) {
      const unsigned lo = lowest_key(b), hi = b > 0 ? lowest_key(b - 1) - 1 : key_of(c.m);
      if (threadIdx.x == 0) {
        sh.ends[0] = lo;
        sh.ends[1] = hi;
      }
    }
    __syncthreads();
    unsigned lo = sh.ends[0], hi = sh.ends[1];
    while (lo < hi && !(mass ? count == 1 : need == count)) {
      const unsigned width = hi - lo;  // less one
      const int shift = max(0, 32 - __clz(width) - 10);
      for (int i = i0; i < i1; i += 32) {
        const float l = val[i];
        const unsigned key = key_of(l);
        if (key >= lo && key <= hi && kept(l, i))
          add((hi - key) >> shift, mass ? weight(c, l, sh.powers) : 1, mass, true);
      }
      crossing(mass, true, -1.f, need);
      hi -= static_cast<unsigned>(sh.found[0]) << shift;
      lo = max(lo, hi - min(hi, (1u << shift) - 1));
      need = sh.found[1];
      count = sh.found[2];
    }
    const float v = of_key(lo);
    if (mass ? count == 1 : need == count) {
      if (v != vcut) icut = 0x7fffffff;
      vcut = v;
      return;
    }
    // one logit, of which the first some are kept
    if (mass) {
      const u64 w = weight(c, v, sh.powers);
      need = (need + w - 1) / w;
    }
    u64 its, all, before;
    const float was = vcut;
    const int was_i = icut;
    const int at = locate([&](float l, int i) -> u64 { return l == v && (l > was || first + i <= was_i); },
                          [&](u64) { return need - 1; }, its, all);
    __syncthreads();
    if (threadIdx.x == 0) sh.found[0] = 0;
    __syncthreads();
    if (at >= 0 && (threadIdx.x & 31) == 0) sh.found[0] = at + 1;
    __syncthreads();
    exchange(sh.found[0], before, all);
    vcut = v;
    icut = static_cast<int>(all) - 1;
  }
};

template <typename TL>
AXON_DEV float logit(const TL* x) {
  const float v = to_f(*x);
  return v == v ? v + 0.f : -INFINITY;  // -0 becomes 0
}
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
  for (int i = tid; i < 257; i += ST) sh.powers[i] = g_powers.v[i];
  for (int i = tid; i < 6 * NB; i += ST) (&sh.hist[0][0][0])[i] = 0;
  grid_dep_launch();
  grid_dep_wait();

  // ---- the slice, and the largest logit with the lowest number
  const int first = min(rank * slice, p.V), n = min(slice, p.V - first);
  const TL* const x = static_cast<const TL*>(p.logits) + b * p.row_stride + first;
  float best = -INFINITY;
  int at = 0;
  auto take = [&](float v, int i) {
    if (v > best) {
      best = v;
      at = i;
    }
  };
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
        for (int e = 0; e < PER; ++e) {
          f[e] = f[e] == f[e] ? f[e] + 0.f : -INFINITY;
          take(f[e], i + e);
        }
#pragma unroll
        for (int e = 0; e < PER; e += 4) *reinterpret_cast<float4*>(val + i + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      }
    }
  }
  for (int i = done + tid; i < n; i += ST) {
    const float v = logit(x + i);
    take(v, i);
    val[i] = v;
  }
  u64 key = best > -INFINITY ? argmax_key(best, first + at) : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
  if (lane == 0) sh.warp[warp] = key;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < SW; ++w) key = max(key, sh.warp[w]);
    sh.cta[1] = key;
  }
  cluster.sync();
  key = lane < CL ? *cluster.map_shared_rank(&sh.cta[1], lane) : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
  const int top = static_cast<int>(0xffffffffu - static_cast<unsigned>(key));

  const float temp = p.temperature ? p.temperature[b] : 1.f;
  if (key == 0 || !(temp > 0.f)) {
    // nothing to choose from, or the largest
    if (rank == 0 && tid == 0) {
      p.tokens[b] = key ? top : -1;
      if (p.prob) p.prob[b] = key ? 1.f : 0.f;
    }
    cluster.sync();  // nobody's shared memory goes away while another reads it
    return;
  }
  float m = of_key(static_cast<unsigned>(key >> 32));
  if (m == INFINITY) {  // infinite logits share everything
    for (int i = tid; i < n; i += ST) val[i] = val[i] == INFINITY ? 0.f : -INFINITY;
    m = 0.f;
  }
  const double scale = 1.4426950408889634074 / static_cast<double>(temp);
  Row row{p, sh, val, n, first, rank, CL};
  row.seg = ((slice + SW - 1) / SW + 31) / 32 * 32;
  row.c.m = m;
  row.c.ch = static_cast<float>(fmin(scale, 3e38));
  row.c.cl = static_cast<float>(fmin(scale, 3e38) - row.c.ch);
  __syncthreads();

  const int k = p.top_k ? p.top_k[b] : 0;
  if (k > 0 && k < p.V) row.cut(-1.f, k);
  const float share = p.top_p ? p.top_p[b] : 1.f;
  if (share < 1.f) row.cut(fmaxf(share, 0.f), 0);
  const float low = p.min_p ? p.min_p[b] : 0.f;
  if (low > 0.f) {
    // w >= min_p is l >= m + temperature ln(min_p), rounded up to a float
    const float v = __double2float_ru(static_cast<double>(m) + static_cast<double>(temp) * log(static_cast<double>(low)));
    if (v > row.vcut) {
      row.vcut = v;
      row.icut = 0x7fffffff;
    }
    if (v > m) {  // the first is kept in any case
      row.vcut = m;
      row.icut = top;
    }
  }
  const float random = p.u[b];
  u64 its = 0, all = 0;
  const int token = row.locate(
      [&](float l, int i) -> u64 { return row.kept(l, i) ? weight(row.c, l, sh.powers) : 0; },
      [&](u64 sum) {
        if (!(random > 0.f)) return u64{0};
        const float under = fminf(random, 0.999999940395355224609375f);
        return __umul64hi(static_cast<u64>(static_cast<double>(under) * 18446744073709551616.0), sum);
      },
      its, all);
  if (token >= 0 && lane == 0) {
    p.tokens[b] = token;
    if (p.prob) p.prob[b] = static_cast<float>(static_cast<double>(its) / static_cast<double>(all));
  }
  cluster.sync();
}

// CTAs per row.
int cluster_for(const LaunchCtx& lc, int B, int V) {
  int CL = 1;
  while (CL < MAX_CL && ((V + CL - 1) / CL > MAX_SLICE || (static_cast<long long>(B) * CL < 2 * lc.num_sms && V / CL > 2 * ST))) CL *= 2;
  return CL;
}

template <typename TL>
cudaError_t launch_type(const LaunchCtx& lc, const SampleArgs& a) {
  const int CL = cluster_for(lc, a.B, a.V);
  const int slice = ((a.V + CL - 1) / CL + 7) & ~7;
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
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<TL>, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SLICE * 4 + 32);
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
