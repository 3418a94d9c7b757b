// Device helpers the attention kernels share: products with an operand in TMEM or in
// the MN-major layout, TMEM traffic, reads of a cluster peer's shared memory, masks.
#pragma once

#include "common.cuh"

namespace oos {

// D[tmem] (+)= A[tmem] * B[smem]: A (M = 128 rows, one per lane) as packed
// bf16 pairs, K index 2c and 2c + 1 in column c (low half first)
OOS_DEV void tc_mma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Shared-memory descriptor of an MN-major operand in the 128-byte-swizzled
// layout: 64 consecutive MN elements (bf16) per 128-byte row, one row per K
// index, 8-row / 1024-byte swizzle atoms.  `lbo` is the byte distance between
// consecutive 64-element MN blocks, the stride between 8-row K groups is 1024.
OOS_DEV uint64_t smem_desc_sw128_mn(uint32_t saddr, uint32_t lbo) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((lbo >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
OOS_DEV void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 2^x by the hardware approximation (relative error ~2^-22; -inf gives +0)
OOS_DEV float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 16-byte chunk c of row r of a 128-byte-swizzled tile (rows 128 bytes apart,
// 8-row / 1024-byte swizzle atoms, tile base 1024-aligned)
OOS_DEV uint32_t sw128(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }
// 32 lanes x 32 bit, 16 consecutive columns per thread, TMEM <- raw words
OOS_DEV void tmem_st16u(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
OOS_DEV void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 lanes x 32 bit, 32 consecutive columns per thread, without waiting: the
// caller issues several, then tmem_wait_ld_regs over every register loaded
OOS_DEV void tmem_ld32_nowait(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
// wait for the thread's outstanding TMEM loads; the empty statements after it
// make every later use of v[0..n) depend on the wait
template <int N>
OOS_DEV void tmem_wait_ld_regs(float (&v)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}
// 64 columns of one lane row starting at taddr
OOS_DEV void tmem_ld64(uint32_t taddr, float (&v)[64]) {
  tmem_ld32_nowait(taddr, v);
  tmem_ld32_nowait(taddr + 32, v + 32);
  tmem_wait_ld_regs(v);
}
OOS_DEV float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}
OOS_DEV float2 ld_cluster2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
// 128-bit masks as (lo: bits 0..63, hi: bits 64..127)
OOS_DEV void shr128(unsigned long long lo, unsigned long long hi, int s, unsigned long long& rlo,
                    unsigned long long& rhi) {
  if (s >= 128) { rlo = 0; rhi = 0; }
  else if (s >= 64) { rlo = s == 64 ? hi : hi >> (s - 64); rhi = 0; }
  else if (s == 0) { rlo = lo; rhi = hi; }
  else { rlo = (lo >> s) | (hi << (64 - s)); rhi = hi >> s; }
}
OOS_DEV void shl128(unsigned long long lo, unsigned long long hi, int s, unsigned long long& rlo,
                    unsigned long long& rhi) {
  if (s >= 128) { rlo = 0; rhi = 0; }
  else if (s >= 64) { rhi = s == 64 ? lo : lo << (s - 64); rlo = 0; }
  else if (s == 0) { rlo = lo; rhi = hi; }
  else { rhi = (hi << s) | (lo >> (64 - s)); rlo = lo << s; }
}

// a CTA's own copies or MMAs draining after an abort: bounded by the default limit
OOS_DEV void drain_wait(uint64_t* bar, uint32_t parity) {
  const unsigned long long t0 = globaltimer();
  while (!mbar_test(smem_addr(bar), parity) && globaltimer() - t0 < kWaitLimitNs) {
  }
}

}  // namespace oos
