// Attention of a batch step over the sequences' own 8-bit pages, 16-bit queries with heads of
// 128, where a sequence has few rows (a decoding token's group), and the join with the
// prefix's parts.
//
// A block owns a tile of 8 or 16 rows (token, head of one kv head's group) of one sequence
// and a range of its keys, dealt to its four warps 32 at a time: two blocks of 16 positions,
// each with one scale.  Every warp has a ring of its own, filled by 16-byte asynchronous
// copies (a key row is 128 bytes: 8 lanes), and no block barrier before the end.  Places and
// scales of 16 such pairs are looked up at once, a lane each.
//
// S^T = K Q^T (keys on the product's 16 rows) takes the codes of K as they are, on
// mma.sync m16n8k32 of e4m3: a row of q, scaled by a power of two so that its largest element
// lies in [2^7, 2^8), is the sum of two (bf16) or three (binary16) e4m3 parts, each the
// rounded rest of the one before times 2^5.  That holds 8 (11) bits exactly, down to elements
// of 2^-8 (2^-6) of the largest, and smaller ones to 2^-22 of it.  The parts' products cost what one of
// 16-bit K would, whose conversion would cost more than both.  Sums of e4m3 products are
// full fp32 (truncated) on this chip.
//
// O^T = V^T P^T takes V as bf16: a transposed load of pairs of codes brings the same two of
// d for neighbouring keys, and the bytes of either d, moved apart, are bf16 numbers of
// 2^-120 the value.  The missing 2^120 and V's scale are powers of two in the weights, which
// are two bf16 halves (2^-16).  The bits of a NaN code would read as 480, so V's rows are also
// multiplied by zero as e4m3 (a product of 32 of d a step, half of what Q K^T takes); where
// that says so, the columns are set to NaN in the rows that see the key.  A NaN that a row does
// not see is multiplied as 480 by 0.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "attn.cuh"
#include "batch_attn.cuh"
#include "codes8.cuh"

namespace oos {

constexpr int kP8Warps = 4, kP8D = 128;
constexpr int kP8Keys = 2 * kScaleBlock;               // of a warp at a time
constexpr int kP8Half = kScaleBlock * kP8D;            // bytes of K (or V) of a block of positions
constexpr int kP8Stage = 4 * kP8Half;                  // both blocks, K and V
constexpr int p8_stages(int nt) { return nt == 1 ? 2 : 3; }
constexpr int p8_blocks(int nt) { return nt == 1 ? 3 : 2; }   // per SM
constexpr int p8_smem(int nt) { return p8_stages(nt) * kP8Warps * kP8Stage; }
static_assert(kP8Warps * 16 * kPartLd * 4 <= p8_smem(1), "staged rows over the rings");
constexpr int kP8Unit = kP8Warps * kP8Keys;            // keys of a block's round
constexpr int kP8MaxParts = 32;                        // of a row, the prefix's among them

OOS_DEV void ldm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
OOS_DEV void ldm4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
OOS_DEV uint32_t turned8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
OOS_DEV void mma_e4m3(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
OOS_DEV void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <typename TQ, int NT>
__global__ void __launch_bounds__(kP8Warps * 32, p8_blocks(NT)) k_attn_pages8(const __grid_constant__ BatchAttnArgs a) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr int ROWS = 8 * NT, STAGES = p8_stages(NT);
  constexpr int PARTS = std::is_same<TQ, __nv_bfloat16>::value ? 2 : 3;
  __shared__ TreeScratch s_tree;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = blockIdx.y, S = a.s_splits, split = blockIdx.x % S;
  // behind the prefix's kernel, which has waited for what the caller wrote before it
  // triggers, only the join waits
  if (a.p_splits == 0) pdl_wait();
  pdl_trigger();
  TileRows t;
  if (!sequence_tile(a, blockIdx.x / S, ROWS, &t)) {
    if (blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();       // the grid must not end before the one it follows
    return;
  }
  const unsigned long long (*anc)[2] = nullptr;
  if (a.parent) anc = tree_sets(a, t.q0, t.n, &s_tree);
  const int last = (t.r0 + t.rows - 1) / a.group;
  const int n_keys = anc ? t.len : max(0, min(t.len, t.first + last + 1));
  // as many ranges as have two rounds each; the others are empty
  const int units = (n_keys + kP8Unit - 1) / kP8Unit, ranges = max(1, min(S, units / 2));
  const int k0 = split < ranges ? (int)((long long)units * split / ranges) * kP8Unit : n_keys;
  const int k1 = split < ranges ? min(n_keys, (int)((long long)units * (split + 1) / ranges) * kP8Unit) : n_keys;
  const int n_rounds = max(0, k1 - k0 + kP8Unit - 1) / kP8Unit;

  // ---- places and scales of 16 rounds: lane 2 r + h has block h of round r
  const int* table = a.batch.table + (size_t)t.seq * a.batch.max_pages;
  const int per_page = a.pages.page_size / kScaleBlock;
  auto look_up = [&](int round, long long& block, int& sk, int& sv) {   // block of the pool, -1: none
    const int key = k0 + (round + (lane >> 1)) * kP8Unit + warp * kP8Keys + (lane & 1) * kScaleBlock;
    block = -1;
    sk = sv = 127;
    if (round + (lane >> 1) < n_rounds && key < k1) {   // no further than the table
      const int b = key / kScaleBlock, col = b / per_page, page = __ldg(table + col);
      if (page >= 0 && page < a.pages.n_pages) {
        block = (long long)page * per_page + (b - col * per_page);
        sk = __ldg(a.k_scale + block * a.pages.nkv + g);
        sv = __ldg(a.v_scale + block * a.pages.nkv + g);
      } else {
        *a.status = OOS_EBATCH;
      }
    }
  };
  long long block = -1, block2 = -1;   // of this batch of 16 rounds and the next
  int sk = 127, sv = 127, sk2 = 127, sv2 = 127;
  look_up(0, block, sk, sv);

  // ---- copies: this warp's two blocks of a round into its own ring
  const uint32_t ring = smem_addr(smem) + warp * (STAGES * kP8Stage);
  const long long key_bytes = (long long)a.pages.nkv * kP8D;
  const uint8_t* kg = a.pages.k + (long long)g * kP8D + (lane & 7) * 16;
  const uint8_t* vg = a.pages.v + (long long)g * kP8D + (lane & 7) * 16;
  auto copy = [&](int round, int place, long long from) {   // from: a lane's block of the batch
    if (round < n_rounds) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const long long at = __shfl_sync(0xffffffffu, from, 2 * (round & 15) + h);
        const int n = k1 - (k0 + round * kP8Unit + warp * kP8Keys + h * kScaleBlock);   // keys from its first on
        const uint32_t dst = ring + place * kP8Stage + h * 2 * kP8Half;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 4 * i + (lane >> 3);
          const bool ok = at >= 0 && key < n;
          const long long off = ok ? (at * kScaleBlock + key) * key_bytes : 0;
          const uint32_t o = key * kP8D + (((lane & 7) ^ (key & 7)) << 4);
          cp_async16(dst + o, kg + off, ok);
          cp_async16(dst + kP8Half + o, vg + off, ok);
        }
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int c = 0; c < STAGES - 1; ++c) copy(c, c, block);

  // ---- the queries' e4m3 parts as B fragments: row lane / 4 of each 8, d = 32 kk + 16 e + 4 (lane % 4) ..
  uint32_t qf[PARTS][NT][4][2];
  float sc[NT][2];   // a column's two rows of this thread: 8 n + 2 (lane & 3) + e
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 8 * n + (lane >> 2), row = t.r0 + r;
    const bool on = r < t.rows;
    const TQ* q = (const TQ*)a.q + (long long)(t.q0 + (on ? row / a.group : 0)) * a.q_stride +
                  (g * a.group + row % a.group) * kP8D + (lane & 3) * 4;
    const bool wide = (((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 7) == 0;
    float x[4][2][4], mx = 0.f;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        Vec<TQ, 4> v = {};
        if (on && wide) v = *reinterpret_cast<const Vec<TQ, 4>*>(q + 32 * kk + 16 * e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (on && !wide) v.v[i] = q[32 * kk + 16 * e + i];
          x[kk][e][i] = on ? finite_or_nan(to_f32(v.v[i])) : 0.f;
          mx = fmaxf(mx, fabsf(x[kk][e][i]));
        }
      }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const int e2 = row_exponent(mx);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float (&y)[4] = x[kk][e];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = y[i] * exp2i(-e2) * 128.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const uint16_t w0 = f32x2_e4m3(y[0], y[1]), w1 = f32x2_e4m3(y[2], y[3]);
          qf[p][n][kk][e] = (uint32_t)w0 | (uint32_t)w1 << 16;
          const float2 z0 = e4m3x2_f32(w0), z1 = e4m3x2_f32(w1);
          y[0] = (y[0] - z0.x) * 32.f;
          y[1] = (y[1] - z0.y) * 32.f;
          y[2] = (y[2] - z1.x) * 32.f;
          y[3] = (y[3] - z1.y) * 32.f;
        }
      }
#pragma unroll
    for (int e = 0; e < 2; ++e) sc[n][e] = a.scale_log2 * __shfl_sync(0xffffffffu, exp2i(e2), ((lane & 3) * 2 + e) * 4);
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
  // ldmatrix rows of this lane: 8 keys of a 16-byte column, the 16 keys of one column and of the next
  const uint32_t l_key = lane & 15, l_col = lane >> 4;

#pragma unroll 1
  for (int c = 0; c < n_rounds; ++c) {
    cp_async_wait<STAGES - 2>();
    __syncwarp();
    if ((c & 15) == 8) look_up((c & ~15) + 16, block2, sk2, sv2);
    {
      const int ahead = c + STAGES - 1;
      copy(ahead, ahead % STAGES, (ahead ^ c) & 16 ? block2 : block);
    }
    const int key0 = k0 + c * kP8Unit + warp * kP8Keys;
    const uint32_t buf = ring + (c % STAGES) * kP8Stage;
    int there[2], ek[2], ev[2];   // keys of either block that are there, from its first on; its exponents
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int from = 2 * (c & 15) + h;
      there[h] = __shfl_sync(0xffffffffu, block, from) >= 0 ? max(0, min(kScaleBlock, k1 - key0 - h * kScaleBlock)) : 0;
      ek[h] = scale_exp(__shfl_sync(0xffffffffu, sk, from));
      ev[h] = scale_exp(__shfl_sync(0xffffffffu, sv, from));
    }
    if ((c & 15) == 15) {
      block = block2;
      sk = sk2;
      sv = sv2;
    }
    // nothing there, or no row that sees the first key (warp-uniform)
    if (there[0] + there[1] == 0 || (!anc && key0 > t.first + tok_hi)) continue;
    float s[2][NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float acc[PARTS][NT][4];
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[p][n][e] = 0.f;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        uint32_t k4[4];
        ldm4(buf + h * 2 * kP8Half + l_key * kP8D + (((2 * kk + l_col) ^ (l_key & 7)) << 4), k4);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int p = 0; p < PARTS; ++p) mma_e4m3(acc[p][n], k4, qf[p][n][kk][0], qf[p][n][kk][1]);
      }
      const float pk = pow2f(ek[h] - 7);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = acc[PARTS - 1][n][e];
#pragma unroll
          for (int p = PARTS - 2; p >= 0; --p) v = fmaf(v, 0x1p-5f, acc[p][n][e]);
          s[h][n][e] = v * (sc[n][e & 1] * pk);
        }
    }
    // keys that each of this thread's rows sees
    const int seen = t.first - key0;   // those before it are committed
    const bool full = there[0] + there[1] == kP8Keys && (anc ? seen : seen + tok_lo + 1) >= kP8Keys;
    uint32_t bits[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) bits[n][e] = ~0u;
    if (!full) {
      const uint32_t here = ((1u << there[0]) - 1) | ((1u << there[1]) - 1) << 16;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int lead = max(0, min(kP8Keys, anc ? seen : seen + token[n][e] + 1));
          uint32_t b = lead == 32 ? ~0u : (1u << lead) - 1;
          if (anc) {
            unsigned long long lo, hi;
            if (seen >= 0) shl128(an[n][e][0], an[n][e][1], min(seen, 128), lo, hi);
            else shr128(an[n][e][0], an[n][e][1], min(-seen, 128), lo, hi);
            b |= (uint32_t)lo;
          }
          bits[n][e] = b & here;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!((bits[n][e] >> (16 * h + (lane >> 2))) & 1)) s[h][n][e] = -INFINITY;
            if (!((bits[n][e] >> (16 * h + 8 + (lane >> 2))) & 1)) s[h][n][2 + e] = -INFINITY;
          }
        }
    }
    bool move = false;
    float mn[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float mx = max_nan(max_nan(s[0][n][e], s[0][n][2 + e]), max_nan(s[1][n][e], s[1][n][2 + e]));
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
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
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (there[h] == 0) continue;
      // the weights' factor 2^(120 + ev), as far as it fits beside their 2^8; the rest goes to V
      const int ew = min(ev[h], -1);
      const float pv = pow2f(120 + ew);
      uint32_t pf[NT][2], pl[NT][2];   // two bf16 halves, as B fragments: 8 x 8 of (key, row) turned to (row, key)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // without a finite score yet every score is -inf, and gives 0
        const float neg[2] = {m[n][0] == -INFINITY ? 0.f : -m[n][0], m[n][1] == -INFINITY ? 0.f : -m[n][1]};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float p0 = ex2_approx(s[h][n][2 * u] + neg[0]), p1 = ex2_approx(s[h][n][2 * u + 1] + neg[1]);
          l[n][0] += p0;
          l[n][1] += p1;
          p0 *= pv;
          p1 *= pv;
          const uint32_t hi = __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);   // cut off
          const __nv_bfloat162 lo = __floats2bfloat162_rn(p0 - bf16_lo(hi), p1 - bf16_hi(hi));
          pf[n][u] = turned8x8(hi);
          pl[n][u] = turned8x8(*reinterpret_cast<const uint32_t*>(&lo));
        }
      }
      const uint32_t vbuf = buf + (2 * h + 1) * kP8Half;
      const bool large = ev[h] > ew;   // warp-uniform, as all of a block's is
      const uint32_t fv = (uint32_t)(ev[h] - ew + 127) << 7, fv2 = fv | fv << 16;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[4];   // keys 0-7 and 8-15 of 16 columns, and of the next 16
        ldm4_trans(vbuf + l_key * kP8D + (((2 * i + l_col) ^ (l_key & 7)) << 4), w);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t v[4] = {even_codes(w[2 * j]), odd_codes(w[2 * j]), even_codes(w[2 * j + 1]), odd_codes(w[2 * j + 1])};
          if (large) {
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = mul_bf16x2(v[x], fv2);
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_bf16(o[2 * i + j][n], v[0], v[1], v[2], v[3], pf[n][0], pf[n][1]);
            mma_bf16(o[2 * i + j][n], v[0], v[1], v[2], v[3], pl[n][0], pl[n][1]);
          }
        }
      }
      // a NaN in V: rows of zero times it
      float nan[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        uint32_t v4[4];
        ldm4(vbuf + l_key * kP8D + (((2 * kk + l_col) ^ (l_key & 7)) << 4), v4);
        mma_e4m3(nan, v4, 0u, 0u);
      }
      if (__any_sync(0xffffffffu, nan[0] != 0.f || nan[2] != 0.f)) {   // a column for all
#pragma unroll 1
        for (int key = 0; key < kScaleBlock; ++key)
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              // column d = 16 i + 2 (lane / 4) + u
              const uint32_t code = smem[vbuf - smem_addr(smem) + key * kP8D + ((i ^ (key & 7)) << 4) + 2 * (lane >> 2) + u];
              if ((code & 0x7f) != 0x7f) continue;
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if ((bits[n][e] >> (16 * h + key)) & 1) o[i][n][2 * u + e] = __int_as_float(0x7fffffff);
            }
      }
    }
  }
  cp_async_wait<0>();
  __syncthreads();
  // ---- join: O rows with (m, l), staged over the rings, of every warp, and the prefix's parts
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
        *reinterpret_cast<float2*>(row + 16 * i + 2 * (lane >> 2)) = make_float2(o[i][n][e], o[i][n][2 + e]);
      if (lane < 4) *reinterpret_cast<float2*>(row + kP8D) = make_float2(m[n][e], l[n][e]);
    }
  const int pre_parts = a.own_part ? 0 : a.p_splits;
  if (!a.own_part) pdl_wait();   // the prefix's parts
  __syncthreads();
  const long long part_rows = (long long)a.batch.n_tokens * a.group, part_step = (long long)a.pages.nkv * part_rows * kPartLd;
  const float* pre = a.part_o + ((long long)g * part_rows + (long long)t.q0 * a.group + t.r0) * kPartLd;
#pragma unroll 1
  for (int r = warp; r < t.rows; r += kP8Warps) {
    // a lane per part; the prefix's columns are on their way before the weights are known
    constexpr int U = 16;
    static_assert(U >= kMaxPrefixParts, "all of them");
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < kP8Warps) ml = *reinterpret_cast<const float2*>(stage + (lane * ROWS + r) * kPartLd + kP8D);
    else if (lane < kP8Warps + pre_parts) ml = *reinterpret_cast<const float2*>(pre + (lane - kP8Warps) * part_step + r * kPartLd + kP8D);
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
#pragma unroll
    for (int i = 0; i < kP8Warps; ++i) add(i, *reinterpret_cast<const float4*>(stage + (i * ROWS + r) * kPartLd + 4 * lane));
    if (pre_parts > 0) {
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (i < pre_parts) add(kP8Warps + i, v[i]);
    }
    if (a.own_part) {
      float* to = a.part_o + (a.p_splits + split) * part_step + ((long long)g * part_rows + (long long)t.q0 * a.group + t.r0 + r) * kPartLd;
      *reinterpret_cast<float4*>(to + 4 * lane) = acc;
      // the maximum over the parts passes a NaN by, the sum does not: stored with a maximum of
      // -inf it would read as a part without keys
      if (lane == 0) *reinterpret_cast<float2*>(to + kP8D) = make_float2(den == den ? top : den, den);
    } else {
      store_row<TQ>(a, g, t.q0, t.r0 + r, weighted_mean(acc, den));
    }
  }
  if (a.own_part && blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();   // a kernel that waits for this one counts on the prefix's
}

PagesPlan plan_pages8_tc(long long rows, int n_seqs, int nkv, long long most_keys, int n_sms) {
  PagesPlan p;
  p.tile_rows = rows <= 8ll * n_seqs ? 8 : 16;
  p.tiles = (int)(n_seqs + rows / p.tile_rows);
  const long long live = std::max((long long)n_seqs, (rows + p.tile_rows - 1) / p.tile_rows) * nkv;
  // ranges enough for eight blocks an SM, each with two rounds at least
  const long long want = 8ll * n_sms / live;
  p.splits = (int)std::max(1ll, std::min({want, most_keys / (2 * kP8Unit), (long long)kP8MaxParts - kMaxPrefixParts}));
  p.sms = (int)std::min<long long>(n_sms, (live * p.splits + p8_blocks(p.tile_rows / 8) - 1) / p8_blocks(p.tile_rows / 8));
  p.part = p.splits > 1;
  return p;
}

template <typename TQ, int NT>
static cudaError_t launch_pages8_of(const BatchAttnArgs& a, const PagesPlan& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = kernel_ready(ready, (const void*)k_attn_pages8<TQ, NT>, p8_smem(NT));
  if (e != cudaSuccess) return e;
  return launch(true, k_attn_pages8<TQ, NT>, dim3((unsigned)(p.tiles * p.splits), a.pages.nkv), dim3(kP8Warps * 32), p8_smem(NT), st, a);
}

cudaError_t launch_pages8_tc(const BatchAttnArgs& a, const PagesPlan& p, int dtype, cudaStream_t st) {
  if (dtype == OOS_DTYPE_BF16)
    return p.tile_rows == 8 ? launch_pages8_of<__nv_bfloat16, 1>(a, p, st) : launch_pages8_of<__nv_bfloat16, 2>(a, p, st);
  return p.tile_rows == 8 ? launch_pages8_of<__half, 1>(a, p, st) : launch_pages8_of<__half, 2>(a, p, st);
}

}  // namespace oos
