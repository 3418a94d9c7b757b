// Attention of a batch step over the sequences' own pages, 16-bit types with heads of
// 128, where a sequence has few rows (a decoding token's group), and the join with the
// prefix's parts.
//
// A block owns a tile of 8 or 16 rows (token, head of one kv head's group) of one
// sequence and a range of its keys; the blocks of the other ranges of the same rows are
// its cluster.  Pages are gathered by 16-byte asynchronous copies, a key row of 256 bytes
// by 16 lanes, whatever the page size: keys that are not there arrive as zeros.  The
// keys are dealt to the block's four warps in chunks of 16, each warp with a ring of its
// own, no block barrier before the end; several blocks per SM cover each other's waits.
// Products run on mma.sync m16n8k16, operands by ldmatrix from rows whose 16-byte chunks
// are swizzled by the key.
//
// Long sequences are bound by HBM (16 of 2000 keys on average, 8 kv heads: 48 us with the
// prefix's kernel beside it, the bytes take 26), short ones by what a block does once --
// lookups that follow each other, query fragments, the join -- at the 12 warps per SM that
// the registers leave (256 of 150 keys, 2048 blocks: 40 us for 23 us of bytes; 47 before
// the join took own and prefix's parts apart and lookups lost their divisions).  Fewer
// warps a block and more blocks (2 x 6, 3 x 4 per SM) took 45 and 41 us where 4 x 3 took
// 34; blocks that stay and take chunk after chunk, their parts joined by a kernel of its
// own, 40.
//
// Every row keeps its maximum, moved only when a chunk exceeds it by 2^8, and its sum in
// fp32.  Weights enter P.V as binary16 (2^-11, small ones see kHalfBias), or as two bf16 halves
// (2^-16 together, where one bf16 would round to 2^-8), whose second product costs nothing
// beside the reads.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "attn.cuh"
#include "batch_attn.cuh"

namespace oos {

constexpr int kPgWarps = 4;
__host__ __device__ constexpr int narrow_stages(int nt) { return nt == 1 ? 2 : 3; }
__host__ __device__ constexpr int pg_blocks(int nt) { return nt == 1 ? 3 : 2; }   // per SM
constexpr int kPgD = 128;
constexpr int kPgRow = 2 * kPgD;                 // bytes of a key row
constexpr int kPgChunkBytes = 2 * 16 * kPgRow;   // 16 keys, K and V
constexpr int pg_smem(int stages) { return stages * kPgWarps * kPgChunkBytes; }
static_assert(kPgWarps * 8 * kPartLd * 4 <= pg_smem(2) && kPgWarps * 16 * kPartLd * 4 <= pg_smem(3), "staged rows over the rings");

OOS_DEV void lds128(uint32_t addr, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
}
OOS_DEV uint32_t lds16(uint32_t addr) {
  uint16_t w;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(addr) : "memory");
  return w;
}
// an 8 x 8 block of 16-bit values, a row per four lanes, turned over its diagonal
OOS_DEV uint32_t movmatrix_trans(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
OOS_DEV void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
OOS_DEV void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
template <bool F16>
OOS_DEV void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// whether a value of the V of the 16 keys at buf is infinite or NaN
template <bool F16>
OOS_DEV bool chunk_not_finite(uint32_t buf) {
  constexpr uint32_t kExp = F16 ? 0x7c007c00u : 0x7f807f80u;
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t w[4];
    lds128(buf + 16 * kPgRow + (i * 32 + (threadIdx.x & 31)) * 16, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= __vcmpeq2(w[e] & kExp, kExp);
  }
  return __any_sync(0xffffffffu, bad != 0);
}

// Keys by rows: S^T = K Q^T and O^T = V^T P^T, the keys (and then d) on the product's 16
// rows and NT * 8 query rows on its columns, so that a decoding token's group of up to 8
// heads costs one product of 8 columns where rows of 16 would cost two.
template <typename TQ, bool F16, int NT>
__global__ void __launch_bounds__(kPgWarps * 32, pg_blocks(NT)) k_attn_pages(const __grid_constant__ BatchAttnArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int ROWS = 8 * NT, STAGES = narrow_stages(NT);
  constexpr float kBias = F16 ? kHalfBias : 0.f;
  constexpr bool CONVERT = F16 && std::is_same<TQ, __nv_bfloat16>::value;
  __shared__ TreeScratch s_tree;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = blockIdx.y, S = a.s_splits, split = blockIdx.x % S;
  // behind the prefix's kernel, which has waited for what the caller wrote before it
  // triggers, only the join waits
  if (a.p_splits == 0) pdl_wait();
  pdl_trigger();
  TileRows t;
  if (!sequence_tile(a, blockIdx.x / S, ROWS, &t)) {          // the whole cluster
    if (blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();       // the grid must not end before the one it follows
    return;
  }
  const unsigned long long (*anc)[2] = nullptr;
  if (a.parent) anc = tree_sets(a, t.q0, t.n, &s_tree);
  const int last = (t.r0 + t.rows - 1) / a.group;
  const int n_keys = anc ? t.len : max(0, min(t.len, t.first + last + 1));
  const int units = (n_keys + 63) / 64;
  const int k0 = (int)((long long)units * split / S) * 64;
  const int k1 = min(n_keys, (int)((long long)units * (split + 1) / S) * 64);
  const int n_chunks = max(0, k1 - k0 + 63) / 64;             // of 64 keys, 16 per warp

  // ---- the first page lookups and the queries' loads go out together
  int key = k0 + warp * 16 + (lane & 15);   // of this warp's 16 in the chunk that is looked up next
  int col = key / a.pages.page_size, in_page = key - col * a.pages.page_size;
  const int* table = a.batch.table + (size_t)t.seq * a.batch.max_pages;
  const int cols = 64 / a.pages.page_size, rest = 64 - cols * a.pages.page_size;   // of a chunk
  auto next_slot = [&]() {   // its place in the pages, -1: none
    long long at = -1;
    if (key < k1) {   // no further than the table
      const int page = __ldg(table + col);
      if (page >= 0 && page < a.pages.n_pages) at = (long long)page * a.pages.page_size + in_page;
      else *a.status = OOS_EBATCH;
    }
    key += 64;
    col += cols;
    in_page += rest;
    if (in_page >= a.pages.page_size) {
      in_page -= a.pages.page_size;
      ++col;
    }
    return at;
  };
  long long slot[STAGES];
#pragma unroll
  for (int c = 0; c < STAGES; ++c) slot[c] = next_slot();
  // B fragments of the query rows, all of d: column lane / 4 of each 8 rows
  uint32_t qf[8][NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 8 * n + (lane >> 2), row = t.r0 + r;
    const bool on = r < t.rows;
    const uint16_t* q = (const uint16_t*)a.q + (long long)(t.q0 + (on ? row / a.group : 0)) * a.q_stride +
                        (g * a.group + row % a.group) * kPgD + (lane & 3) * 2;
    const bool pairs = (((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 3) == 0;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint16_t* p = q + kk * 16 + e * 8;
        uint32_t x = 0;
        if (on) x = pairs ? *reinterpret_cast<const uint32_t*>(p) : (uint32_t)p[0] | (uint32_t)p[1] << 16;
        qf[kk][n][e] = x;
      }
  }

  // ---- copies: this warp's keys of chunk c into its own ring
  const uint32_t ring = smem_addr(smem) + warp * (STAGES * kPgChunkBytes);
  const long long key_bytes = (long long)a.pages.nkv * kPgRow;
  const uint8_t* kg = a.pages.k + (long long)g * kPgRow + (lane & 15) * 16;
  const uint8_t* vg = a.pages.v + (long long)g * kPgRow + (lane & 15) * 16;
  auto copy = [&](int c, long long at_lane) {
    if (c < n_chunks) {
      const uint32_t dst = ring + (c % STAGES) * kPgChunkBytes;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = 2 * i + (lane >> 4);
        const long long at = __shfl_sync(0xffffffffu, at_lane, key);
        const uint32_t o = key * kPgRow + (((lane & 15) ^ (key & 7)) << 4);
        const bool ok = at >= 0;
        const long long off = ok ? at * key_bytes : 0;
        cp_async16(dst + o, kg + off, ok);
        cp_async16(dst + 16 * kPgRow + o, vg + off, ok);
      }
    }
    cp_async_commit();
  };
  uint32_t valid[STAGES];   // keys that are there, of the chunks on their way
#pragma unroll
  for (int c = 0; c < STAGES - 1; ++c) {
    copy(c, slot[c]);
    valid[c] = __ballot_sync(0xffffffffu, slot[c] >= 0) & 0xffffu;
  }
  long long next = slot[STAGES - 1];   // looked up a chunk ahead

  // a column's two rows of this thread: 8 n + 2 (lane & 3) + e
  float sc[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float p2 = 1.f;
    if constexpr (CONVERT) {
      float mx = 0.f;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
#pragma unroll
        for (int e = 0; e < 2; ++e) mx = fmaxf(mx, fmaxf(fabsf(bf16_lo(qf[kk][n][e])), fabsf(bf16_hi(qf[kk][n][e]))));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const int e2 = row_exponent(mx);
      p2 = exp2i(e2);
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
#pragma unroll
        for (int e = 0; e < 2; ++e) qf[kk][n][e] = scaled_half2(qf[kk][n][e], exp2i(-e2));
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) sc[n][e] = a.scale_log2 * __shfl_sync(0xffffffffu, p2, ((lane & 3) * 2 + e) * 4);
  }
  int token[NT][2];
  unsigned long long an[NT][2][2] = {};
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * n + (lane & 3) * 2 + e;
      token[n][e] = (t.r0 + r) / a.group;
      if (anc && r < t.rows) {
        an[n][e][0] = anc[token[n][e]][0];
        an[n][e][1] = anc[token[n][e]][1];
      }
    }
  const int tok_lo = t.r0 / a.group, tok_hi = last;

  float o[8][NT][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      m[n][e] = -INFINITY;
      l[n][e] = 0.f;
    }
  }
  // ldmatrix rows of this lane: K as it lies, V transposed on the way
  const uint32_t a_key = (lane & 7) + ((lane >> 3) & 1) * 8, a_chunk = lane >> 4;
  const uint32_t v_key = (lane & 7) + (lane >> 4) * 8, v_chunk = (lane >> 3) & 1;

#pragma unroll 1
  for (int c = 0; c < n_chunks; ++c) {
    cp_async_wait<STAGES - 2>();
    __syncwarp();
    const uint32_t there = valid[0];
#pragma unroll
    for (int i = 0; i + 2 < STAGES; ++i) valid[i] = valid[i + 1];
    copy(c + STAGES - 1, next);
    valid[STAGES - 2] = __ballot_sync(0xffffffffu, next >= 0) & 0xffffu;
    next = next_slot();
    const int key0 = k0 + c * 64 + warp * 16;
    // nothing there, or no row that sees the first key (warp-uniform)
    if (there == 0 || (!anc && key0 > t.first + tok_hi)) continue;
    const uint32_t buf = ring + (c % STAGES) * kPgChunkBytes;
    float s[NT][4], s2[NT][4];   // even and odd steps of d apart: half as long a chain of products
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = s2[n][e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      uint32_t k4[4];
      ldsm4(buf + a_key * kPgRow + (((2 * kk + a_chunk) ^ (a_key & 7)) << 4), k4);
#pragma unroll
      for (int n = 0; n < NT; ++n) mma16816<F16>(kk & 1 ? s2[n] : s[n], k4, qf[kk][n][0], qf[kk][n][1]);
    }
    // keys of the chunk that each of this thread's rows sees
    const int seen = t.first - key0;   // those before it are committed
    const bool full = there == 0xffffu && (anc ? seen : seen + tok_lo + 1) >= 16;
    uint32_t bits[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        bits[n][e] = 0xffffu;
        if (!full) {
          const int lead = max(0, min(16, anc ? seen : seen + token[n][e] + 1));
          uint32_t b = (1u << lead) - 1;
          if (anc) {
            unsigned long long lo, hi;
            if (seen >= 0) shl128(an[n][e][0], an[n][e][1], min(seen, 128), lo, hi);
            else shr128(an[n][e][0], an[n][e][1], min(-seen, 128), lo, hi);
            b |= (uint32_t)lo;
          }
          bits[n][e] = b & there;
        }
      }
    // A key that some of the rows do not see must not reach them through 0 times a v
    // that is not finite: such a chunk (the last ones of a sequence only) is summed apart.
    // One token's rows see all keys that are there, unless a tree hides its siblings.
    const bool apart = !full && (anc || tok_lo != tok_hi) && chunk_not_finite<F16>(buf);
    bool move = false;
    float mn[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        s[n][e] += s2[n][e];
        s[n][2 + e] += s2[n][2 + e];
        if (!full) {
          if (!((bits[n][e] >> (lane >> 2)) & 1)) s[n][e] = -INFINITY;
          if (!((bits[n][e] >> (8 + (lane >> 2))) & 1)) s[n][2 + e] = -INFINITY;
        }
        float mx = max_nan(s[n][e], s[n][2 + e]);
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 16)) * sc[n][e] - kBias;
        mn[n][e] = !(mx <= m[n][e] + 8.f) ? mx : m[n][e];   // a NaN moves it, and stays
        move = move || mn[n][e] != m[n][e];
      }
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float f = m[n][e] == mn[n][e] ? 1.f : m[n][e] == -INFINITY ? 0.f : exp2f(m[n][e] - mn[n][e]);
          l[n][e] *= f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[i][n][e] *= f;
            o[i][n][2 + e] *= f;
          }
          m[n][e] = mn[n][e];
        }
    }
    // weights, and as B fragments: an 8 x 8 block of (key, row) turned to (row, key)
    uint32_t pf[NT][2], pl[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      // without a finite score yet every score is -inf, and gives 0
      const float neg[2] = {m[n][0] == -INFINITY ? 0.f : -m[n][0], m[n][1] == -INFINITY ? 0.f : -m[n][1]};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = ex2_approx(fmaf(s[n][2 * h], sc[n][0], neg[0])), p1 = ex2_approx(fmaf(s[n][2 * h + 1], sc[n][1], neg[1]));
        s[n][2 * h] = p0;
        s[n][2 * h + 1] = p1;
        if constexpr (F16) {   // the sum is of the weights as they are multiplied
          const __half2 v = __floats2half2_rn(p0, p1);
          pf[n][h] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&v));
          s[n][2 * h] = __low2float(v);
          s[n][2 * h + 1] = __high2float(v);
        } else {
          // the upper half cut off, and a lower one that is positive where the weight is: an
          // infinite v stays infinite under both (of a NaN weight the lower one is NaN)
          const float h0 = __uint_as_float(__float_as_uint(p0) & 0xffff0000u);
          const float h1 = __uint_as_float(__float_as_uint(p1) & 0xffff0000u);
          const __nv_bfloat162 v = __floats2bfloat162_rn(h0, h1);
          const __nv_bfloat162 r = __floats2bfloat162_rn(fmaxf(p0 - h0, p0 * 0x1p-60f), fmaxf(p1 - h1, p1 * 0x1p-60f));
          pf[n][h] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&v));
          pl[n][h] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&r));
        }
        l[n][0] += s[n][2 * h];
        l[n][1] += s[n][2 * h + 1];
      }
    }
    if (apart) {
#pragma unroll 1
      for (int key = 0; key < 16; ++key)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float mine = key & 8 ? s[n][2 + e] : s[n][e];
            const float p = __shfl_sync(0xffffffffu, mine, (key & 7) * 4 + (lane & 3));
            if (!((bits[n][e] >> key) & 1)) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t w = lds16(buf + (16 + key) * kPgRow + ((((2 * i + h)) ^ (key & 7)) << 4) + (lane >> 2) * 2);
                o[i][n][2 * h + e] += p * (F16 ? __half2float(__ushort_as_half((unsigned short)w)) : bf16_lo(w));
              }
          }
      continue;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t v4[4];
      ldsm4_trans(buf + (16 + v_key) * kPgRow + (((2 * i + v_chunk) ^ (v_key & 7)) << 4), v4);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma16816<F16>(o[i][n], v4, pf[n][0], pf[n][1]);
        if constexpr (!F16) mma16816<F16>(o[i][n], v4, pl[n][0], pl[n][1]);
      }
    }
  }
  cp_async_wait<0>();
  __syncthreads();
  // ---- join: O rows with (m, l), staged over the rings, of every warp and every block of
  // the cluster, and the prefix's parts; at most 32
  float* stage = reinterpret_cast<float*>(smem);   // [warp][row][kPartLd]
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int x = 4; x < 32; x *= 2) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
      float* row = stage + (warp * ROWS + 8 * n + (lane & 3) * 2 + e) * kPartLd;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) row[16 * i + 8 * h + (lane >> 2)] = o[i][n][2 * h + e];
      if (lane < 4) *reinterpret_cast<float2*>(row + kPgD) = make_float2(m[n][e], l[n][e]);
    }
  const int pre_parts = a.own_part ? 0 : a.p_splits;
  if (!a.own_part) pdl_wait();   // the prefix's parts
  __syncthreads();
  if (S > 1) {
    cluster_arrive_release();
    cluster_wait_acquire();
  }
  const int own = kPgWarps * S;
  const long long part_rows = (long long)a.batch.n_tokens * a.group, part_step = (long long)a.pages.nkv * part_rows * kPartLd;
  const float* pre = a.part_o + ((long long)g * part_rows + (long long)t.q0 * a.group + t.r0) * kPartLd;
#pragma unroll 1
  for (int r = t.rows * split / S + warp; r < t.rows * (split + 1) / S; r += kPgWarps) {
    // a lane per part; the prefix's columns are on their way before the weights are known
    constexpr int U = 16;
    static_assert(U >= kMaxPrefixParts, "all of them");
    const float* mine = stage + (lane % kPgWarps * ROWS + r) * kPartLd + kPgD;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < own) ml = S > 1 ? ld_cluster2(dsmem_addr(mine, lane / kPgWarps)) : *reinterpret_cast<const float2*>(mine);
    else if (lane < own + pre_parts) ml = *reinterpret_cast<const float2*>(pre + (lane - own) * part_step + r * kPartLd + kPgD);
    float4 v[U];
    if (pre_parts > 0) {
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (i < pre_parts) v[i] = *reinterpret_cast<const float4*>(pre + i * part_step + r * kPartLd + 4 * lane);
    }
    const bool on = ml.x != -INFINITY;   // a NaN is, and reaches the sum
    const float top = warp_max(ml.x);
    const float w = on ? exp2f(ml.x - top) : 0.f;
    const float den = warp_sum(on ? w * ml.y : 0.f);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](int i, const float4& x) {
      const float wi = __shfl_sync(0xffffffffu, w, i);
      if (wi == 0.f) return;   // a part without weight counts for nothing, whatever it holds
      acc.x += wi * x.x;
      acc.y += wi * x.y;
      acc.z += wi * x.z;
      acc.w += wi * x.w;
    };
#pragma unroll 1
    for (int s = 0; s < S; ++s) {
      float4 x[kPgWarps];
#pragma unroll
      for (int i = 0; i < kPgWarps; ++i) {
        const float* p = stage + (i * ROWS + r) * kPartLd + 4 * lane;
        x[i] = S > 1 ? ld_cluster4(dsmem_addr(p, s)) : *reinterpret_cast<const float4*>(p);
      }
#pragma unroll
      for (int i = 0; i < kPgWarps; ++i) add(s * kPgWarps + i, x[i]);
    }
    if (pre_parts > 0) {
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (i < pre_parts) add(own + i, v[i]);
    }
    if (a.own_part) {
      float* to = a.part_o + a.p_splits * part_step + ((long long)g * part_rows + (long long)t.q0 * a.group + t.r0 + r) * kPartLd;
      *reinterpret_cast<float4*>(to + 4 * lane) = acc;
      // the maximum over the parts passes a NaN by, the sum does not: stored with a maximum of
      // -inf it would read as a part without keys
      if (lane == 0) *reinterpret_cast<float2*>(to + kPgD) = make_float2(den == den ? top : den, den);
    } else {
      store_row<TQ>(a, g, t.q0, t.r0 + r, weighted_mean(acc, den));
    }
  }
  if (S > 1) {   // a peer may still read this block's rows
    cluster_arrive_release();
    cluster_wait_acquire();
  }
  if (a.own_part && blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();   // a kernel that waits for this one counts on the prefix's
}

PagesPlan plan_pages_tc(long long rows, int n_seqs, int nkv, long long most_keys, int n_sms) {
  PagesPlan p;
  p.tile_rows = rows <= 8ll * n_seqs ? 8 : 16;
  p.tiles = (int)(n_seqs + rows / p.tile_rows);
  // blocks for every SM twice, each with 128 keys at least; a cluster holds 4 ranges
  // (their parts and the prefix's fit the join's 32 lanes)
  const long long want = 4ll * n_sms / std::max(1ll, (long long)p.tiles * nkv);
  p.splits = (int)std::max(1ll, std::min({want, most_keys / 128, 4ll}));
  const long long live = std::max((long long)n_seqs, (rows + p.tile_rows - 1) / p.tile_rows) * nkv * p.splits;
  const int per_sm = pg_blocks(p.tile_rows / 8);
  p.sms = (int)std::min<long long>(n_sms, (live + per_sm - 1) / per_sm);
  p.part = false;
  return p;
}

static cudaError_t launch_pages(std::atomic<uint64_t>& ready, const void* kernel, int smem, const BatchAttnArgs& a,
                                const PagesPlan& p, cudaStream_t st) {
  const cudaError_t e = kernel_ready(ready, kernel, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)(p.tiles * p.splits), a.pages.nkv);
  lc.blockDim = dim3(kPgWarps * 32);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (p.splits > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = p.splits;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // starts while the prefix's kernel drains
  attr[n++].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = attr;
  lc.numAttrs = n;
  void* args[1] = {const_cast<BatchAttnArgs*>(&a)};
  return cudaLaunchKernelExC(&lc, kernel, args);
}

template <typename TQ, bool F16>
static cudaError_t launch_pages_of(const BatchAttnArgs& a, const PagesPlan& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready[2] = {};
  if (p.tile_rows == 8) return launch_pages(ready[0], (const void*)k_attn_pages<TQ, F16, 1>, pg_smem(narrow_stages(1)), a, p, st);
  return launch_pages(ready[1], (const void*)k_attn_pages<TQ, F16, 2>, pg_smem(narrow_stages(2)), a, p, st);
}

cudaError_t launch_pages_tc(const BatchAttnArgs& a, const PagesPlan& p, int dtype, int kv_dtype, cudaStream_t st) {
  if (kv_dtype == OOS_DTYPE_BF16) return launch_pages_of<__nv_bfloat16, false>(a, p, st);
  if (dtype == OOS_DTYPE_BF16) return launch_pages_of<__nv_bfloat16, true>(a, p, st);
  return launch_pages_of<__half, true>(a, p, st);
}

}  // namespace oos
