// Attention of a batch step over the shared prefix, 16-bit types with heads of 128:
// the rows of all sequences against the prefix's keys, so that each key tile is read
// once per 256 rows.  Leaves every row's unnormalised O, maximum and sum for the join
// with the sequence's own keys (batch_pages.cu).
//
// tcgen05, rows (token, head of one kv head's group) packed without regard to the
// sequences.  A block has two streams of work, each with its weights P and its O in
// TMEM and four softmax warps of its own, a thread per row:
//   two row tiles   (more than 128 rows left): both streams take every key tile
//   one row tile    the streams take the even and the odd key tiles
// so that one stream's softmax runs under the other's products.  A unit of work is a
// (key tile, stream) pair, taken in turn.
//
// The streams share one score buffer, held only from a product's issue until the threads
// have its row in registers, so that the next unit's scores run under this one's
// exponentials and wait for no P.V; one thread issues the scores, one the P.V products,
// and the tensor cores take them turn by turn.  (A buffer for each stream with P over it
// makes a stream's scores, weights and P.V follow each other: 159 us against 145 for 1024
// rows of 8 heads over 32768 keys.  One thread for both kinds, a unit's scores before the
// P.V of the one before: 197.)
//
// P, 16-bit pairs in TMEM, is the A operand of P.V and is handed over in halves of 64
// keys; the sum l is of the unrounded weights.  The running maximum moves only when a
// tile exceeds it by 2^8 (the threads rescale their O rows in TMEM then).
// Keys past the prefix's end arrive as zeros (the tensor map ends there), so masking
// their scores is enough.
//
// A block stages its rows over the K/V ring and stores them with one bulk copy, a part
// per key range; the next kernel adds the parts up.  (Ranges joined inside a cluster,
// through distributed shared memory, took 10 us for 256 rows of 11 ranges.)
#include <math.h>
#include <string.h>

#include <algorithm>

#include "attn.cuh"
#include "batch_attn.cuh"

namespace oos {

constexpr int kPxRows = 128, kPxKeys = 128, kPxD = 128;
constexpr int kPxDBlock = kPxKeys * 128;            // 64 of d by 128 keys, 128-byte swizzle
constexpr int kPxTile = 2 * kPxDBlock;              // 32 KB
constexpr int kPxKStages = 3, kPxVStages = 2;
constexpr int kPxOffK = 0;
constexpr int kPxOffV = kPxOffK + kPxKStages * kPxTile;
constexpr int kPxOffQ = kPxOffV + kPxVStages * kPxTile;   // two row tiles
constexpr int kPxOffExp = kPxOffQ + 2 * kPxTile;          // row exponents of converted queries
constexpr int kPxOffBar = kPxOffExp + 2 * kPxRows * 4;
constexpr int kPxSmem = kPxOffBar + 256 + 1024;           // + alignment slack
constexpr int kPxThreads = 384;
constexpr int kPxSoft0 = 4;                               // softmax warps 4..7 and 8..11
constexpr int kPxRegsIo = 56, kPxRegsSoft = 224, kPxRegsLaunch = 168;
constexpr int kPxMaxSplits = 16;
static_assert(128 * kPxRegsIo + (kPxThreads - 128) * kPxRegsSoft <= kPxThreads * kPxRegsLaunch, "register split");
static_assert(2 * kPxRows * kPartLd * 4 <= kPxOffQ, "staged rows over the ring");
static_assert(kPxSmem <= 227 * 1024, "shared memory per block");
// TMEM columns: S, P of either stream, O of either
constexpr int kPxTmS = 0, kPxTmP = kPxKeys, kPxTmO = 2 * kPxKeys, kPxTmCols = 512;

struct PrefixArgs {
  CUtensorMap kmap, vmap;   // [prefix_len][nkv][d] as (d, kv head, slot)
  BatchAttnArgs a;
};

// A wait of at most kWaitLimitNs; false: it ran out here or elsewhere in the block.  The
// thread sleeps on the barrier: polls read shared memory, whose bandwidth the products'
// operands need whole.
OOS_DEV bool px_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int32_t* status) {
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
OOS_DEV float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

template <typename TQ, bool F16>
__global__ void __launch_bounds__(kPxThreads, 1) k_attn_prefix(const __grid_constant__ PrefixArgs p) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr bool CONVERT = F16 && std::is_same<TQ, __nv_bfloat16>::value;
  // binary16 weights carry 2^4, so that fewer of the small ones fall below its range
  constexpr float kBias = F16 ? 4.f : 0.f;
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + kPxOffBar);
  uint64_t* kfull = bar;           // [3] transaction bytes
  uint64_t* kempty = bar + 3;      // [3] its score products done
  uint64_t* vfull = bar + 6;       // [2] transaction bytes
  uint64_t* vempty = bar + 8;      // [2] its P.V products done
  uint64_t* sfull = bar + 10;      // [2] scores of a stream done
  uint64_t* pfull = bar + 12;      // [stream][key half] four softmax warps: P written
  uint64_t* pvdone = bar + 16;     // [2] P.V of a stream done
  uint64_t* sfree = bar + 18;      // [2] four softmax warps: scores in registers
  uint64_t* qready = bar + 20;     // eight warps: queries in shared memory
  uint64_t* odone = bar + 21;      // both issuers: all products done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + 22);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const BatchAttnArgs& a = p.a;
  int32_t* status = a.status;
  const int S = a.p_splits, split = blockIdx.x % S, pair = blockIdx.x / S, g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row0 = pair * 2 * kPxRows;
  const int rows = min(2 * kPxRows, a.batch.n_tokens * a.group - row0);
  const int dual = rows > kPxRows ? 1 : 0;
  const int n_all = (a.prefix_len + kPxKeys - 1) / kPxKeys;
  const int t0 = (int)((long long)n_all * split / S);
  const int n_tiles = (int)((long long)n_all * (split + 1) / S) - t0;
  const int units = n_tiles << dual;                  // unit u: tile u >> dual, stream u & 1
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int i = 0; i < 3; ++i) {
      mbar_init(&kfull[i], 1);
      mbar_init(&kempty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&vfull[i], 1);
      mbar_init(&vempty[i], 1);
      mbar_init(&sfull[i], 1);
      mbar_init(&pfull[2 * i], 4);
      mbar_init(&pfull[2 * i + 1], 4);
      mbar_init(&pvdone[i], 1);
      mbar_init(&sfree[i], 4);
    }
    mbar_init(qready, 8);
    mbar_init(odone, 2);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 2) tmem_alloc(tmem_slot, kPxTmCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  float* stage = reinterpret_cast<float*>(sm);

  if (warp < kPxSoft0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPxRegsIo));
    if ((warp == 0 || warp == 3) && lane == 0) {
      // ---------------------------------------------------------- loaders: K and V tiles
      const bool v = warp == 3;
      const CUtensorMap* map = v ? &p.vmap : &p.kmap;
      uint64_t* full = v ? vfull : kfull;
      uint64_t* empty = v ? vempty : kempty;
      const int stages = v ? kPxVStages : kPxKStages;
      tma_prefetch_desc(map);
      const uint64_t pol = policy_evict_last();   // the other row tiles read it too
      int n = 0;
      for (; n < n_tiles; ++n) {
        const int st = n % stages;
        if (n >= stages && !px_wait(&empty[st], (uint32_t)(n / stages - 1) & 1u, abort_flag, status)) break;
        unsigned char* dst = sm + (v ? kPxOffV : kPxOffK) + st * kPxTile;
        mbar_arrive_expect_tx(&full[st], kPxTile);
        tma_load_3d(dst, map, &full[st], 0, g, (t0 + n) * kPxKeys, pol);
        tma_load_3d(dst + kPxDBlock, map, &full[st], 64, g, (t0 + n) * kPxKeys, pol);
      }
      // every copy issued has landed before the block goes on
      for (int i = n > stages ? n - stages : 0; i < n; ++i) drain_wait(&full[i % stages], (uint32_t)(i / stages) & 1u);
    } else if (warp == 1 && lane == 0) {
      // ---------------------------------------------------------- scores
      constexpr uint32_t idesc = F16 ? idesc_f16_f32(kPxRows, kPxKeys) : idesc_bf16_f32(kPxRows, kPxKeys);
      const uint64_t kdesc = smem_desc_sw128(smem_addr(sm + kPxOffK)), qdesc = smem_desc_sw128(smem_addr(sm + kPxOffQ));
      bool ok = px_wait(qready, 0, abort_flag, status);
      for (int u = 0; u < units && ok; ++u) {
        const int i = u >> dual, st = i % kPxKStages, x = u & 1;
        if (!dual || x == 0) ok = px_wait(&kfull[st], (uint32_t)(i / kPxKStages) & 1u, abort_flag, status);
        if (u > 0) ok = ok && px_wait(&sfree[x ^ 1], (uint32_t)((u - 1) >> 1) & 1u, abort_flag, status);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kPxD / 16; ++k) {
          const uint64_t o = (uint64_t)(((k >> 2) * kPxDBlock) >> 4) + 2 * (k & 3);
          tc_mma_bf16(tmem + kPxTmS, qdesc + o + (uint64_t)(((dual ? x : 0) * kPxTile) >> 4),
                      kdesc + o + (uint64_t)((st * kPxTile) >> 4), idesc, k > 0 ? 1u : 0u);
        }
        tc_commit(&sfull[x]);
        if (!dual || x == 1) tc_commit(&kempty[st]);
      }
      tc_commit(odone);
    } else if (warp == 2 && lane == 0) {
      // ---------------------------------------------------------- P.V
      constexpr uint32_t idesc = (F16 ? idesc_f16_f32(kPxRows, kPxD) : idesc_bf16_f32(kPxRows, kPxD)) | (1u << 16);
      const uint64_t vdesc = smem_desc_sw128_mn(smem_addr(sm + kPxOffV), kPxDBlock);
      bool ok = true;
      for (int u = 0; u < units && ok; ++u) {
        const int i = u >> dual, st = i % kPxVStages, x = u & 1, use = u >> 1;   // use: of this stream
        if (!dual || x == 0) ok = px_wait(&vfull[st], (uint32_t)(i / kPxVStages) & 1u, abort_flag, status);
        for (int h = 0; h < 2 && ok; ++h) {   // the first half's product runs under the second's exponentials
          ok = px_wait(&pfull[2 * x + h], (uint32_t)use & 1u, abort_flag, status);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const int k = 4 * h + kk;
            tc_mma_bf16_ts(tmem + kPxTmO + x * kPxD, tmem + kPxTmP + x * (kPxKeys / 2) + 8 * k,
                           vdesc + (uint64_t)((st * kPxTile + k * 16 * 128) >> 4), idesc, (k > 0 || use > 0) ? 1u : 0u);
          }
        }
        if (!ok) break;
        tc_commit(&pvdone[x]);
        if (!dual || x == 1) tc_commit(&vempty[st]);
      }
      tc_commit(odone);
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPxRegsSoft));
    // ------------------------------------------------------------ softmax: stream x, a thread per row
    const int x = (warp - kPxSoft0) >> 2, q4 = warp & 3;
    const int lrow = q4 * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    float* s_exp = reinterpret_cast<float*>(sm + kPxOffExp);
    // queries of the stream's row tile (one row tile: the first stream's warps), two rows
    // of 16 lanes at a time, into the swizzled layout
    if (x == 0 || dual) {
      unsigned char* qs = sm + kPxOffQ + x * kPxTile;
      const int c = lane & 15;
      uint4 w[16];   // all rows' loads in flight: four at a time took 8 us
      const uint16_t* q0 = (const uint16_t*)a.q + g * a.group * kPxD + c * 8;
      const bool vec = (((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 15) == 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = x * kPxRows + q4 * 32 + 2 * i + (lane >> 4), row = row0 + r;
        const uint16_t* q = q0 + (long long)(row / a.group) * a.q_stride + (row % a.group) * kPxD;
        w[i] = make_uint4(0, 0, 0, 0);
        if (r < rows) {
          if (vec) {
            w[i] = *reinterpret_cast<const uint4*>(q);
          } else {
            w[i] = make_uint4((uint32_t)q[0] | (uint32_t)q[1] << 16, (uint32_t)q[2] | (uint32_t)q[3] << 16,
                              (uint32_t)q[4] | (uint32_t)q[5] << 16, (uint32_t)q[6] | (uint32_t)q[7] << 16);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = q4 * 32 + 2 * i + (lane >> 4);
        if constexpr (CONVERT) {
          float mx = fmaxf(fmaxf(fabsf(bf16_lo(w[i].x)), fabsf(bf16_hi(w[i].x))), fmaxf(fabsf(bf16_lo(w[i].y)), fabsf(bf16_hi(w[i].y))));
          mx = fmaxf(mx, fmaxf(fmaxf(fabsf(bf16_lo(w[i].z)), fabsf(bf16_hi(w[i].z))), fmaxf(fabsf(bf16_lo(w[i].w)), fabsf(bf16_hi(w[i].w)))));
#pragma unroll
          for (int s = 1; s < 16; s *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
          const int e2 = row_exponent(mx);
          const float f = exp2i(-e2);
          w[i] = make_uint4(scaled_half2(w[i].x, f), scaled_half2(w[i].y, f), scaled_half2(w[i].z, f), scaled_half2(w[i].w, f));
          if (c == 0) s_exp[x * kPxRows + r] = exp2i(e2);
        }
        *reinterpret_cast<uint4*>(qs + (c >> 3) * kPxDBlock + sw128(r, c & 7)) = w[i];
      }
      fence_async_smem();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(qready);
    float sc = a.scale_log2;
    if constexpr (CONVERT) {
      // one row tile: the second stream's rows are the first's, written by its warps
      asm volatile("bar.sync 1, 256;" ::: "memory");
      sc *= s_exp[(dual ? x : 0) * kPxRows + lrow];
    }
    const int mine = dual ? n_tiles : (n_tiles + 1 - x) >> 1;   // tiles of this stream
    const uint32_t ts = tmem + lane_off + kPxTmS, tp = tmem + lane_off + kPxTmP + x * (kPxKeys / 2);
    const uint32_t to = tmem + lane_off + kPxTmO + x * kPxD;
    float m = -INFINITY, l = 0.f;
    for (int j = 0; j < mine; ++j) {
      if (!__all_sync(0xffffffffu, px_wait(&sfull[x], (uint32_t)j & 1u, abort_flag, status))) break;
      tc_fence_after();
      const int key0 = (t0 + (dual ? j : 2 * j + x)) * kPxKeys;
      float sv[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32_nowait(ts + 32 * c, sv + 32 * c);
      tmem_wait_ld_regs(sv);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sfree[x]);
      const int n_ok = a.prefix_len - key0;
      if (n_ok < kPxKeys) {
#pragma unroll
        for (int i = 0; i < 128; ++i)
          if (i >= n_ok) sv[i] = -INFINITY;
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < 128; i += 2) mx[(i >> 1) & 3] = max3_nan(mx[(i >> 1) & 3], sv[i], sv[i + 1]);
      const float tmax = max_nan(max_nan(mx[0], mx[1]), max_nan(mx[2], mx[3])) * sc - kBias;
      const bool move = !(tmax <= m + 8.f);   // a NaN moves it, and stays
      // the tile before has left this P and is in O
      if (j > 0) {
        if (!__all_sync(0xffffffffu, px_wait(&pvdone[x], (uint32_t)(j - 1) & 1u, abort_flag, status))) break;
        tc_fence_after();
      }
      if (__any_sync(0xffffffffu, move)) {
        const float f = !move ? 1.f : m == -INFINITY ? 0.f : exp2f(m - tmax);
        if (j > 0) {
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            float ov[32];
            tmem_ld32_nowait(to + 32 * c, ov);
            tmem_wait_ld_regs(ov);
#pragma unroll
            for (int i = 0; i < 32; ++i) ov[i] *= f;
            tmem_st16u(to + 32 * c, reinterpret_cast<const uint32_t*>(ov));
            tmem_st16u(to + 32 * c + 16, reinterpret_cast<const uint32_t*>(ov + 16));
          }
        }
        l *= f;
        if (move) m = tmax;
      }
      // weights 2^(s sc - m); without a finite score yet every score is -inf, and gives 0
      const float neg = m == -INFINITY ? 0.f : -m;
      const float2 sc2 = make_float2(sc, sc), neg2 = make_float2(neg, neg);
      float2 ps[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 2 * h; c < 2 * h + 2; ++c) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            float2 e = fma2(make_float2(sv[32 * c + i], sv[32 * c + i + 1]), sc2, neg2);
            e = make_float2(ex2_approx(e.x), ex2_approx(e.y));
            ps[(i >> 1) & 1] = add2(ps[(i >> 1) & 1], e);
            if constexpr (F16) {
              const __half2 v = __floats2half2_rn(e.x, e.y);
              pk[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
            } else {
              const __nv_bfloat162 v = __floats2bfloat162_rn(e.x, e.y);
              pk[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
            }
          }
          tmem_st16u(tp + 16 * c, pk);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pfull[2 * x + h]);
      }
      l += (ps[0].x + ps[0].y) + (ps[1].x + ps[1].y);
    }
    // the ring and TMEM are free once all products are done (the issuer always says so)
    drain_wait(odone, 0);
    tc_fence_after();
    const bool have = mine > 0 && !*abort_flag;
    float* row = stage + (size_t)(x * kPxRows + lrow) * kPartLd;
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
      float ov[32];
      tmem_ld32_nowait(to + 32 * c, ov);
      tmem_wait_ld_regs(ov);
#pragma unroll
      for (int i = 0; i < 32; i += 4)
        *reinterpret_cast<float4*>(row + 32 * c + i) =
            have ? make_float4(ov[i], ov[i + 1], ov[i + 2], ov[i + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    *reinterpret_cast<float2*>(row + kPxD) = make_float2(have ? m : -INFINITY, have ? l : 0.f);
  }
  tc_fence_before();
  __syncthreads();   // rows staged
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, kPxTmCols);
  }
  if (!dual && warp >= kPxSoft0) {   // both streams' sums of the same rows
    for (int r = warp - kPxSoft0; r < rows; r += 8) {
      float* ra = stage + r * kPartLd;
      const float* rb = ra + kPxRows * kPartLd;
      const float2 ma = *reinterpret_cast<const float2*>(ra + kPxD), mb = *reinterpret_cast<const float2*>(rb + kPxD);
      const float top = max_nan(ma.x, mb.x);
      const float wa = ma.x == -INFINITY ? 0.f : exp2f(ma.x - top), wb = mb.x == -INFINITY ? 0.f : exp2f(mb.x - top);
      float4 va = *reinterpret_cast<const float4*>(ra + 4 * lane);
      const float4 vb = *reinterpret_cast<const float4*>(rb + 4 * lane);
      va = make_float4(va.x * wa + vb.x * wb, va.y * wa + vb.y * wb, va.z * wa + vb.z * wb, va.w * wa + vb.w * wb);
      __syncwarp();
      *reinterpret_cast<float4*>(ra + 4 * lane) = va;
      if (lane == 0) *reinterpret_cast<float2*>(ra + kPxD) = make_float2(top, ma.y * wa + mb.y * wb);
    }
  }
  fence_async_smem();
  __syncthreads();
  if (threadIdx.x == 0) {
    float* dst = a.part_o + (((long long)split * a.pages.nkv + g) * a.batch.n_tokens * a.group + row0) * kPartLd;
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_addr(stage)),
                 "r"(rows * kPartLd * 4)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
}

// ---- host
template <typename TQ, bool F16>
static cudaError_t launch_prefix(const PrefixArgs& p, dim3 grid, cudaStream_t st) {
  // the register split must not ask for more than the block is launched with
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = kernel_ready(ready, (const void*)k_attn_prefix<TQ, F16>, kPxSmem, kPxRegsLaunch);
  return e == cudaSuccess ? launch(false, k_attn_prefix<TQ, F16>, grid, dim3(kPxThreads), kPxSmem, st, p) : e;
}

// The count of key ranges with the shortest schedule, in us: waves of one block per SM,
// each of a block's tiles (about 0.7 per row tile) and its beginning and end (5), and
// the parts, written and read once at about 8 bytes per ps.
PrefixPlan plan_prefix_tc(long long rows, int nkv, int prefix_len, int n_sms) {
  PrefixPlan p;
  p.pairs = (int)((rows + 2 * kPxRows - 1) / (2 * kPxRows));
  p.splits = 1;
  const long long items = (long long)p.pairs * nkv;
  const int tiles = (prefix_len + kPxKeys - 1) / kPxKeys;
  const double tile = rows > kPxRows ? 1.4 : 0.7, part = 2.0 * rows * nkv * kPartLd * 4 / 8e6;
  double best = 0;
  for (int s = 1; s <= kPxMaxSplits && s <= tiles; ++s) {
    const double cost = (double)((items * s + n_sms - 1) / n_sms) * (tile * ((tiles + s - 1) / s) + 5.0) + part * s;
    if (s > 1 && cost >= best) continue;
    best = cost;
    p.splits = s;
  }
  return p;
}

cudaError_t launch_prefix_tc(const BatchAttnArgs& a, const PrefixPlan& plan, int dtype, int kv_dtype, cudaStream_t st) {
  PrefixArgs p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  const uint64_t dims[3] = {(uint64_t)kPxD, (uint64_t)a.pages.nkv, (uint64_t)a.prefix_len};
  const uint64_t strides[2] = {(uint64_t)kPxD * 2, (uint64_t)a.pages.nkv * kPxD * 2};
  const uint32_t box[3] = {64, 1, (uint32_t)kPxKeys};
  const bool f16 = kv_dtype == OOS_DTYPE_F16;
  if (!encode_bf16_map(&p.kmap, a.pk, 3, dims, strides, box, f16) || !encode_bf16_map(&p.vmap, a.pv, 3, dims, strides, box, f16))
    return cudaErrorInvalidValue;
  const dim3 grid((unsigned)(plan.pairs * plan.splits), a.pages.nkv);
  if (!f16) return launch_prefix<__nv_bfloat16, false>(p, grid, st);
  if (dtype == OOS_DTYPE_BF16) return launch_prefix<__nv_bfloat16, true>(p, grid, st);
  return launch_prefix<__half, true>(p, grid, st);
}

}  // namespace oos
