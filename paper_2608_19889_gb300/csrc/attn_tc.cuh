// What the tcgen05 attention kernels share: copies of query boxes, products with P in
// TMEM, TMEM loads and stores, packed fp32 arithmetic, and probabilities in 16 bits.
#pragma once

#include "kernels.h"

AXON_DEV void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

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
AXON_DEV bool elect_one() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
  return r != 0;
}
AXON_DEV float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// D[tmem] (+)= A[tmem] * B[smem desc] (A: 128 lanes, two 16-bit values per column).
AXON_DEV void tc_mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(
          d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

AXON_DEV void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
      "%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
AXON_DEV void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
      "%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
AXON_DEV void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
AXON_DEV void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two probabilities as a pair of 16-bit values (fp16: the caller's are below 65504, no saturation needed).
template <typename T> AXON_DEV uint32_t pack_p(float lo, float hi);
template <> AXON_DEV uint32_t pack_p<bf16>(float lo, float hi) { return pack_bf2(lo, hi); }
template <> AXON_DEV uint32_t pack_p<f16>(float lo, float hi) {
  __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}
// What the two 16-bit roundings in p lost of a and e.
template <typename T> AXON_DEV uint32_t pack_rest(float a, float e, uint32_t p);
template <> AXON_DEV uint32_t pack_rest<bf16>(float a, float e, uint32_t p) {
  return pack_bf2(a - bf_lo(p), e - bf_hi(p));
}
template <> AXON_DEV uint32_t pack_rest<f16>(float a, float e, uint32_t p) {
  const float2 r = __half22float2(*reinterpret_cast<__half2*>(&p));
  return pack_p<f16>(a - r.x, e - r.y);
}
// lo += the low, hi += the high 16-bit value of p.
template <typename T> AXON_DEV void add_p(float& lo, float& hi, uint32_t p);
template <> AXON_DEV void add_p<bf16>(float& lo, float& hi, uint32_t p) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n add.f32.bf16 %0, l, %0;\n add.f32.bf16 %1, h, %1;\n}"
      : "+f"(lo), "+f"(hi)
      : "r"(p));
}
template <> AXON_DEV void add_p<f16>(float& lo, float& hi, uint32_t p) {
  asm("{\n .reg .f16 l, h;\n mov.b32 {l, h}, %2;\n add.f32.f16 %0, l, %0;\n add.f32.f16 %1, h, %1;\n}"
      : "+f"(lo), "+f"(hi)
      : "r"(p));
}

// The V tile as the B operand of P V: N = dims (contiguous in memory), K =
// tokens at 128-byte pitch; 8-token groups 1024 bytes apart, the second 64
// dims one chunk further (CHUNK bytes).
template <int CHUNK>
AXON_DEV uint64_t v_desc(uint32_t addr) {
  uint64_t d = smem_desc_sw128(addr);
  d &= ~(static_cast<uint64_t>(0x3FFFu) << 16);
  d |= static_cast<uint64_t>(CHUNK >> 4) << 16;
  return d;
}
