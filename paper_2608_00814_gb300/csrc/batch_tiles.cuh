// What the tensor-core kernels of many rows share (batch_tiles.cu, batch_tiles8.cu).
#pragma once

#include "attn.cuh"
#include "batch_attn.cuh"

namespace oos {

constexpr int kTlRows = 128, kTlKeys = 128, kTlD = 128;
constexpr int kTlDBlock = kTlKeys * 128;            // 64 of d by 128 keys, 128-byte swizzle
constexpr int kTlTile = 2 * kTlDBlock;              // 32 KB
constexpr int kTlMaxSplits = kMaxPrefixParts;
constexpr int kTlStaged = 2 * kTlRows * ((kPartLd + kTlMaxSplits + 2) * 4 + 8);   // bytes of staged rows and their weights
// TMEM columns: S, P of either stream, O of either
constexpr int kTlTmS = 0, kTlTmP = kTlKeys, kTlTmO = 2 * kTlKeys, kTlTmCols = 512;

// one column of the thread's lane row
OOS_DEV uint32_t tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
  asm volatile("" : "+r"(r));
  return r;
}
OOS_DEV void tmem_st32(uint32_t taddr, const float (&v)[32]) {
  tmem_st16u(taddr, reinterpret_cast<const uint32_t*>(v));
  tmem_st16u(taddr + 16, reinterpret_cast<const uint32_t*>(v) + 16);
}

// A wait of at most kWaitLimitNs; false: it ran out here or elsewhere in the block.  The
// thread sleeps on the barrier: polls read shared memory, whose bandwidth the products'
// operands need whole.
OOS_DEV bool tl_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int32_t* status) {
  const uint32_t addr = smem_addr(bar);
  if (mbar_test(addr, parity)) return true;
  const unsigned long long t0 = globaltimer();
  while (true) {
    if (mbar_test_sleep(addr, parity, 20000u)) return true;
    if (*abort) return false;
    if (globaltimer() - t0 > kWaitLimitNs) {
      *abort = 1;
      *status = OOS_ETIMEOUT;
      return false;
    }
  }
}

// two fp32 at once
OOS_DEV float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%1, %2};\n\tmov.b64 y, {%3, %4};\n\tmov.b64 z, {%5, %6};\n\t"
      "fma.rn.f32x2 %0, x, y, z;\n\t}"
      : "=l"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
OOS_DEV float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%1, %2};\n\tmov.b64 y, {%3, %4};\n\tadd.rn.f32x2 %0, x, y;\n\t}"
      : "=l"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
// s plus the two bf16 of w, in fp32
OOS_DEV void add_bf16x2(float2& s, uint32_t w) {
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tadd.rn.f32.bf16 %0, x, %0;\n\tadd.rn.f32.bf16 %1, y, %1;\n\t}"
      : "+f"(s.x), "+f"(s.y)
      : "r"(w));
}
OOS_DEV float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// A block's staged rows (O, m, l; both streams' apart) into out, with the prefix's parts: the
// eight softmax warps from soft0 on, behind a barrier.  U: parts of a row on their way at once.
template <typename TQ, int U>
OOS_DEV void join_rows(const BatchAttnArgs& a, const TileRows& t, int dual, int g, float* stage, int soft0) {
  const int rows = t.rows, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  const int halves = dual ? 1 : 2, parts = halves + a.p_splits;   // <= 18
  const long long part_rows = (long long)a.batch.n_tokens * a.group, part_step = (long long)a.pages.nkv * part_rows * kPartLd;
  const float* pre = a.part_o + ((long long)g * part_rows + (long long)t.q0 * a.group + t.r0) * kPartLd;
  float* s_w = stage + 2 * kTlRows * kPartLd;   // [part][row]: weight over the sum of all
  long long* s_out = reinterpret_cast<long long*>(s_w + (kTlMaxSplits + 2) * 2 * kTlRows);   // [row]: where it goes
  {
    const int r = threadIdx.x - 32 * soft0;   // a thread per row
    if (r < rows) {
      float2 ml[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        ml[k] = k < halves ? *reinterpret_cast<const float2*>(stage + (k * kTlRows + r) * kPartLd + kTlD) : make_float2(-INFINITY, 0.f);
      float top = max_nan(ml[0].x, ml[1].x);
#pragma unroll 4
      for (int k = 0; k < a.p_splits; ++k) top = max_nan(top, pre[k * part_step + r * kPartLd + kTlD]);
      auto weight = [&](float m) { return m == -INFINITY ? 0.f : exp2f(m - top); };
      float den = weight(ml[0].x) * ml[0].y + weight(ml[1].x) * ml[1].y;
#pragma unroll 4
      for (int k = 0; k < a.p_splits; ++k) {
        const float2 q = *reinterpret_cast<const float2*>(pre + k * part_step + r * kPartLd + kTlD);
        const float w = weight(q.x);
        s_w[(halves + k) * 2 * kTlRows + r] = w;
        den += w * q.y;
      }
      const float f = den == 0.f ? 0.f : 1.f / den;   // a row without keys: zeros
      s_w[r] = weight(ml[0].x) * f;
      if (!dual) s_w[2 * kTlRows + r] = weight(ml[1].x) * f;
      for (int k = 0; k < a.p_splits; ++k) s_w[(halves + k) * 2 * kTlRows + r] *= f;
      const int row = t.r0 + r;
      s_out[r] = (long long)(t.q0 + row / a.group) * a.out_stride + (g * a.group + row % a.group) * kTlD;
    }
  }
  asm volatile("bar.sync 1, 256;" ::: "memory");
  // 16 lanes a row, eight columns each; R pairs of rows of a warp at once
  constexpr int R = 4;
  const int col = (lane & 15) * 8;
  const bool vec = (((uintptr_t)a.out | (uintptr_t)(a.out_stride * 2)) & 15) == 0;
#pragma unroll 1
  for (int r0 = 2 * (warp - soft0) + (lane >> 4); r0 - (lane >> 4) < rows; r0 += 16 * R) {
    float o[R][8];
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) o[k][e] = 0.f;
#pragma unroll 1
    for (int i0 = 0; i0 < parts; i0 += U) {
      float4 v[U][R][2];
      float f[U][R];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u;
        if (i >= parts) continue;
        const float* src = i < halves ? stage + i * kTlRows * kPartLd : pre + (i - halves) * part_step;
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const int r = min(r0 + 16 * k, rows - 1);
          v[u][k][0] = *reinterpret_cast<const float4*>(src + r * kPartLd + col);
          v[u][k][1] = *reinterpret_cast<const float4*>(src + r * kPartLd + col + 4);
          f[u][k] = s_w[i * 2 * kTlRows + r];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u >= parts) continue;
#pragma unroll
        for (int k = 0; k < R; ++k) {
          const float x[8] = {v[u][k][0].x, v[u][k][0].y, v[u][k][0].z, v[u][k][0].w, v[u][k][1].x, v[u][k][1].y, v[u][k][1].z, v[u][k][1].w};
#pragma unroll
          for (int e = 0; e < 8; ++e) o[k][e] = f[u][k] != 0.f ? fmaf(f[u][k], x[e], o[k][e]) : o[k][e];   // no weight counts for nothing
        }
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (r0 + 16 * k >= rows) continue;
      TQ* out = (TQ*)a.out + s_out[r0 + 16 * k] + col;
      if (vec) {
        store_vec<TQ, 8>(out, o[k]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = from_f32<TQ>(o[k][e]);
      }
    }
  }
}

// The same into the parts of the block's key range.  The whole block, behind a barrier.
template <bool SEQ>
OOS_DEV void store_part(const BatchAttnArgs& a, const TileRows& t, int dual, int split, int part0, int g, float* stage, int soft0) {
  const int rows = t.rows, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (!dual && warp >= soft0) {   // both streams' sums of the same rows
    for (int r = warp - soft0; r < rows; r += 8) {
      float* ra = stage + r * kPartLd;
      const float* rb = ra + kTlRows * kPartLd;
      const float2 ma = *reinterpret_cast<const float2*>(ra + kTlD), mb = *reinterpret_cast<const float2*>(rb + kTlD);
      const float top = max_nan(ma.x, mb.x);
      const float wa = ma.x == -INFINITY ? 0.f : exp2f(ma.x - top), wb = mb.x == -INFINITY ? 0.f : exp2f(mb.x - top);
      float4 va = *reinterpret_cast<const float4*>(ra + 4 * lane);
      const float4 vb = *reinterpret_cast<const float4*>(rb + 4 * lane);
      va = make_float4(va.x * wa + vb.x * wb, va.y * wa + vb.y * wb, va.z * wa + vb.z * wb, va.w * wa + vb.w * wb);
      __syncwarp();
      *reinterpret_cast<float4*>(ra + 4 * lane) = va;
      if (lane == 0) *reinterpret_cast<float2*>(ra + kTlD) = make_float2(top, ma.y * wa + mb.y * wb);
    }
  }
  fence_async_smem();
  __syncthreads();
  if (threadIdx.x == 0) {
    if (SEQ) pdl_wait();   // a kernel that waits for this one counts on the one before, too
    float* dst = a.part_o + (((long long)(part0 + split) * a.pages.nkv + g) * a.batch.n_tokens * a.group +
                             (long long)t.q0 * a.group + t.r0) * kPartLd;
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_addr(stage)),
                 "r"(rows * kPartLd * 4)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
}

}  // namespace oos
