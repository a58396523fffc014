// New tokens on their way into a paged cache: rotary positions applied to the queries and
// keys of each token, keys and values written to the token's slot.
//
//   (x, y) -> (x cos a - y sin a, y cos a + x sin a),  a = position * f_j
//
// for the pairs of the first `rotary` dims of a head: dims (j, j + rotary / 2), or (2j, 2j + 1) in the
// interleaved layout. Cosines and sines come from a table that is made once, in 64 bits
// (an angle of position 10^5 in 32 bits is off by 4e-3), and rounded to fp32; products are fp32,
// with one rounding to the cache's type (2^-9 of the value in bf16, against 2^-23 from the table).
//
// A unit is 16 dims of a head, 8 pairs: two 16-byte pieces in, two out (twice that in fp32), and
// 64 bytes of the table, which serve the same unit of HL heads of the token. Bound: HBM, (H + 2G) d
// elements read and written per token; small calls are a launch and three dependent
// loads (length, block, data): 2.0 us for one token of 14 / 2 heads of 64.
#include <algorithm>

#include "kernels.h"

namespace {

constexpr int AT = 256;  // threads

struct Pos {
  long long slot;  // row of [blocks][G][16] where kv head 0 of the token goes; negative: nowhere
  int pos;         // negative: the row is skipped
};

// Offsets or lengths that do not fit. A chunk takes part as a whole or not at all.
AXON_DEV int bad_chunk(const AppendArgs& p, int r0, int r1, int past) {
  if (r0 < 0 || r1 < r0 || r1 > p.T) return DEVERR_SEQ;
  return r1 > r0 && (past < 0 || past > p.most - (r1 - r0)) ? DEVERR_POS : 0;
}

AXON_DEV Pos place_of(const AppendArgs& p, int t) {
  int b = t, pos;
  if (p.cu) {
    int lo = 0, hi = p.B - 1;  // the last chunk that does not begin after t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.cu[mid] <= t) lo = mid; else hi = mid - 1;
    }
    b = lo;
    const int r0 = p.cu[b], r1 = p.cu[b + 1], past = p.past[b];
    if (t < r0 || t >= r1 || bad_chunk(p, r0, r1, past)) return Pos{-1, -1};
    pos = past + t - r0;
  } else {
    pos = p.past[b];
    if (pos < 0) return Pos{-1, -1};
    if (pos >= p.most) {
      set_err(p.err, DEVERR_POS);
      return Pos{-1, -1};
    }
  }
  const long long at = static_cast<long long>(b) * p.blocks_per_seq + (pos >> 4);
  const long long blk = p.block_table ? p.block_table[at] : at;
  if (blk < 0 || blk >= p.num_blocks) {
    set_err(p.err, DEVERR_BLOCK);
    return Pos{-1, pos};
  }
  return Pos{blk * p.G * 16 + (pos & 15), pos};
}

template <typename T>
struct Unit {
  static constexpr int W = sizeof(T) / 2;  // 16-byte words per piece of 8 elements
  uint4 a[W], b[W];
};
template <typename T>
AXON_DEV void load_unit(Unit<T>& u, const T* x, int a, int b) {
#pragma unroll
  for (int i = 0; i < Unit<T>::W; ++i) {
    u.a[i] = ld16(reinterpret_cast<const uint4*>(x + a) + i);
    u.b[i] = ld16(reinterpret_cast<const uint4*>(x + b) + i);
  }
}
template <typename T>
AXON_DEV void store_unit(T* x, int a, int b, const Unit<T>& u) {
#pragma unroll
  for (int i = 0; i < Unit<T>::W; ++i) {
    reinterpret_cast<uint4*>(x + a)[i] = u.a[i];
    reinterpret_cast<uint4*>(x + b)[i] = u.b[i];
  }
}
AXON_DEV uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
template <typename T> AXON_DEV void unpack(const uint4* w, float* f);
template <> AXON_DEV void unpack<bf16>(const uint4* w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf_lo(word(w[0], i));
    f[2 * i + 1] = bf_hi(word(w[0], i));
  }
}
template <> AXON_DEV void unpack<f16>(const uint4* w, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = word(w[0], i);
    const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&v));
    f[2 * i] = h.x;
    f[2 * i + 1] = h.y;
  }
}
template <> AXON_DEV void unpack<float>(const uint4* w, float* f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(word(w[i >> 2], i & 3));
}
template <typename T> AXON_DEV void repack(const float* f, uint4* w) {
  w[0] = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
}
template <> AXON_DEV void repack<float>(const float* f, uint4* w) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]),
                      __float_as_uint(f[4 * i + 3]));
}

AXON_DEV void rotate(float& x, float& y, float c, float s) {
  const float turned = x * c - y * s;
  y = y * c + x * s;
  x = turned;
}

// tokens: per CTA. Heads are numbered queries, keys, values.
template <typename T, int HL>
__global__ void __launch_bounds__(AT) append_kernel(const AppendArgs p, int tokens) {
  __shared__ Pos s_pos[AT];
  const int tid = threadIdx.x;
  grid_dep_launch();
  grid_dep_wait();
  const int U = p.d >> 4, heads = p.H + 2 * p.G, parts = (heads + HL - 1) / HL, per = parts * U;
  const int t0 = blockIdx.x * tokens, n = min(tokens, p.T - t0);
  if (p.cu && blockIdx.x == 0 && blockIdx.y == 0) {
    for (int b = tid; b < p.B; b += AT) {
      const int r0 = p.cu[b], r1 = p.cu[b + 1];
      int e = bad_chunk(p, r0, r1, p.past[b]);
      if ((b == 0 && r0 != 0) || (b == p.B - 1 && r1 != p.T)) e |= DEVERR_SEQ;
      if (e) set_err(p.err, e);
    }
  }
  for (int t = tid; t < n; t += AT) s_pos[t] = place_of(p, t0 + t);
  __syncthreads();
  const int turning = p.rotary >> 4;  // units with rotated pairs
  for (int i = blockIdx.y * AT + tid; i < n * per; i += gridDim.y * AT) {
    const int tl = i / per, x = i - tl * per, hp = x / U, u = x - hp * U;
    const Pos at = s_pos[tl];
    if (at.pos < 0) continue;
    const long long t = t0 + tl;
    const bool turn = u < turning, half = turn && !p.interleaved;
    // first dims of the unit's two pieces
    const int a = half ? u * 8 : u * 16, b = half ? u * 8 + p.rotary / 2 : u * 16 + 8;
    Unit<T> v[HL];
#pragma unroll
    for (int j = 0; j < HL; ++j) {
      const int h = hp + j * parts;
      if (h >= heads || (h >= p.H && at.slot < 0)) continue;
      const int which = h < p.H ? 0 : h < p.H + p.G ? 1 : 2, hh = h - (which == 0 ? 0 : which == 1 ? p.H : p.H + p.G);
      load_unit(v[j], static_cast<const T*>(p.x[which]) + t * p.x_row[which] + hh * p.x_head[which], a, b);
    }
    float cs[16];
    if (turn) {
      const float4* r = reinterpret_cast<const float4*>(p.rope + (static_cast<long long>(at.pos) * p.rotary + u * 16));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 e = __ldg(r + k);
        cs[4 * k] = e.x; cs[4 * k + 1] = e.y; cs[4 * k + 2] = e.z; cs[4 * k + 3] = e.w;
      }
    }
#pragma unroll
    for (int j = 0; j < HL; ++j) {
      const int h = hp + j * parts;
      if (h >= heads || (h >= p.H && at.slot < 0)) continue;
      if (turn && h < p.H + p.G) {
        float e[16];
        unpack<T>(v[j].a, e);
        unpack<T>(v[j].b, e + 8);
        if (half) {
#pragma unroll
          for (int k = 0; k < 8; ++k) rotate(e[k], e[k + 8], cs[2 * k], cs[2 * k + 1]);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) rotate(e[2 * k], e[2 * k + 1], cs[2 * k], cs[2 * k + 1]);
        }
        repack<T>(e, v[j].a);
        repack<T>(e + 8, v[j].b);
      }
      T* to;
      if (h < p.H) {
        to = static_cast<T*>(p.o) + t * p.o_row + h * p.o_head;
      } else {
        const int g = h - p.H, kg = g < p.G ? g : g - p.G;
        to = static_cast<T*>(g < p.G ? p.k : p.v) + (at.slot + kg * 16ll) * p.d;
      }
      store_unit(to, a, b, v[j]);
    }
  }
}

// units: that a CTA takes, about
template <typename T, int HL>
cudaError_t launch_hl(const LaunchCtx& lc, const AppendArgs& a, int units) {
  const int per = (a.H + 2 * a.G + HL - 1) / HL * (a.d >> 4);
  const int tokens = std::min(AT, std::max(1, units / per));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((a.T + tokens - 1) / tokens, tokens > 1 ? 1 : std::min((per + AT - 1) / AT, 65535));
  cfg.blockDim = dim3(AT);
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr[2];
  cfg.numAttrs = chain_attrs(lc, attr);
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, append_kernel<T, HL>, a, tokens);
}

// Three heads per thread share its cosines and sines and keep six loads in flight, but leave SMs idle
// where there are few tokens; with many, CTAs of two units per thread halve the fixed part (lookups,
// barrier). 32 / 8 heads of 128, GPU time of one head and a unit per thread / three heads, one unit /
// three heads, two units: 128 tokens 3.3 / 3.2 / 4.4 us, 384 4.3 / 4.3 / 5.5, 1024 7.6 / 6.0 / 7.0,
// 8191 55 / 37 / 35 (5.9 TB/s, 87 % of the copy bandwidth); 1572 tokens of 16 / 16 heads 14.0 / 10.4 / 9.3.
template <typename T>
cudaError_t launch_type(const LaunchCtx& lc, const AppendArgs& a) {
  const long long units = static_cast<long long>(a.T) * (a.H + 2 * a.G) * (a.d >> 4);
  if (units <= 6ll * AT * lc.num_sms) return launch_hl<T, 1>(lc, a, AT);
  return launch_hl<T, 3>(lc, a, units / 3 < 4ll * AT * lc.num_sms ? AT : 2 * AT);
}

struct Freqs {
  double f[64];
};
// One thread per (position, pair): the angle in 64 bits.
__global__ void __launch_bounds__(AT) rope_table_kernel(float2* out, int positions, int pairs, const Freqs freqs) {
  grid_dep_launch();
  grid_dep_wait();
  const long long i = static_cast<long long>(blockIdx.x) * AT + threadIdx.x;
  if (i >= static_cast<long long>(positions) * pairs) return;
  const long long pos = i / pairs;
  double s, c;
  sincos(static_cast<double>(pos) * freqs.f[i - pos * pairs], &s, &c);
  out[i] = make_float2(static_cast<float>(c), static_cast<float>(s));
}

}  // namespace

cudaError_t launch_append(const LaunchCtx& lc, const AppendArgs& a, int elem_bytes) {
  if (elem_bytes == 4) return launch_type<float>(lc, a);
  return lc.f16 ? launch_type<f16>(lc, a) : launch_type<bf16>(lc, a);
}

cudaError_t launch_rope_table(const LaunchCtx& lc, float* out, int positions, int pairs, const double* freqs) {
  if (pairs < 1 || pairs > 64 || positions < 1) return cudaErrorInvalidValue;
  Freqs f = {};
  for (int j = 0; j < pairs; ++j) f.f[j] = freqs[j];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((static_cast<long long>(positions) * pairs + AT - 1) / AT));
  cfg.blockDim = dim3(AT);
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr[2];
  cfg.numAttrs = chain_attrs(lc, attr);
  cfg.attrs = attr;
  return cudaLaunchKernelEx(&cfg, rope_table_kernel, reinterpret_cast<float2*>(out), positions, pairs, f);
}
