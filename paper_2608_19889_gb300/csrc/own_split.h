// How the SMs are divided between the prefix pass of an attention over shared prefixes and the rows' own parts beside it.
//
// The prefix pass's CTAs and those of the own parts that come before its plan is there work this out each for themselves, in
// different kernels, and cut their work by the result: they have to agree to the last bit. So all of it is whole numbers
// (in fp32 a product that one kernel fuses with a sum and the other does not turned the number in some one case of a
// million, with several million own pages).
#pragma once

#ifdef __CUDACC__
#define OWN_SPLIT_FN __host__ __device__ __forceinline__
#else
#define OWN_SPLIT_FN inline
#endif

// What a step of the prefix pass costs, in 0.4 us: 2.05 us with two tiles (the tensor pipe's 1.6), 1.5 with one whose 64 KB come
// from HBM, 1.25 with one whose keys the group's other items read too.
constexpr unsigned COST_TWO = 5, COST_ONE = 4, COST_LAST = 3;

// What the rows' own parts take on an SM, in 1/16 of it: a page of 128 dims (twelve warps share the SM, and each has 1.5 us
// for a page; half of it with 64 dims), and a row's kv head (15 us of a warp: table, first keys, the warps' and parts' states
// joined); and what they take to begin, once the CTAs of the prefix pass that have nothing to do are gone.
constexpr unsigned OWN_PAGE = 5, OWN_ROW = 50, OWN_BEGIN = 4 * 16;

// All own parts, in 1/16 of 0.4 us of one SM. Bounds keep it below 2^32: pages to 2^28, 512 GB of a cache of 16-bit
// elements, and rows (times kv heads) to 2^25.
OWN_SPLIT_FN unsigned own_work(unsigned pages, unsigned rows, int d) {
  const unsigned p = pages < 1u << 28 ? pages : 1u << 28, r = rows < 1u << 25 ? rows : 1u << 25;
  return (d == 64 ? p * OWN_PAGE / 2 : p * OWN_PAGE) + r * OWN_ROW;
}

// How long both passes take, in 1/16 of 0.4 us, with S of the SMs (0 < S < sms) for own parts of that much work and the others
// for a prefix pass of that cost; below 2^22.
OWN_SPLIT_FN unsigned split_time(unsigned own, unsigned cost, int S, int sms) {
  const unsigned line = (cost < 1u << 28 ? cost : (1u << 28) - 1) * 16;
  const unsigned a = OWN_BEGIN + own / static_cast<unsigned>(S), b = line / static_cast<unsigned>(sms - S);
  const unsigned t = a > b ? a : b, least = 2 * COST_TWO * 16;
  return t < least ? least : t < (1u << 22) - 1 ? t : (1u << 22) - 1;
}
