// Attention of a batch step over the sequences' own 8-bit pages, 16-bit queries with heads of
// 128, where a sequence has few rows (a decoding token's group), and the join with the
// prefix's parts.
//
// A block owns a tile of 8 or 16 rows (token, head of one kv head's group) of one sequence
// and a range of its keys, dealt to its four warps 32 at a time: two blocks of 16 positions,
// each with one scale.  Every warp has a ring of its own, filled by TMA, a block of positions
// a copy (what lies behind the sequence's end comes along and is masked), and no block
// barrier before the end.  Places and scales of 16 such pairs are looked up at once by the
// lane that issues the copy.
//
// Where sequences are cut into ranges, how many each gets follows from all lengths, which
// are on the device: every warp adds them up and finds its block's place, so that ranges
// are about as long everywhere.
//
// Both products are mma.sync m16n8k16 of binary16 with keys or d on the 16 rows, and take
// the codes through the conversion of two at a time, which is exact: two operations of half
// rate for four codes (moving bits takes eleven issue slots; products of e4m3 itself are as
// fast, but leave the sum of each to four additions).
//
// S^T = K Q^T.  A word of codes is four neighbours of d, so a step's 16 of d are taken in the
// order 4 (lane % 4) + 0, 1 and + 2, 3 on both sides.  bf16 rows of q are scaled by a power of
// two that brings their largest element to [1, 2): exact down to 2^-14 of that, smaller ones
// to 2^-25 of it.
//
// O^T = V^T P^T.  A transposed load of pairs of codes brings the same two of d for
// neighbouring keys; a byte permutation puts either d's together.  V's scale 2^e is in the
// weights, 2^(s + e - M + 7) with M a maximum of s + e, rounded to binary16: to 2^-11, below
// 2^-21 of the row's largest weight times scale to 2^-32 of that.  The sum of the weights is of
// 2^(s - m), with a maximum of its own, so that scales far apart cost it nothing.  Maxima move
// when a score passes them by 2^8, which one comparison a score finds; only then lanes meet.
//
// A NaN in V reaches every row that sees its key.  Where some rows do not, in the units
// behind a row's own position, such codes are taken out and their columns set.
//
// 64 requests of up to 4000 keys and 2048 shared ones, 32 heads over 8: 58 us, 4.0 TB/s, and
// the longest requests' blocks end last; 6 requests of up to 64000, 64 heads: 70 us, 5.5 TB/s.
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
constexpr int p8_smem(int nt) { return p8_stages(nt) * kP8Warps * kP8Stage + 1024; }   // + alignment slack
static_assert(kP8Warps * 16 * kPartLd * 4 <= p8_smem(1) - 1024, "staged rows over the rings");
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
OOS_DEV void mma_half(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
OOS_DEV uint32_t half2_of(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

struct Pages8Args {
  CUtensorMap kmap, vmap;   // codes [n_pages][page_size][nkv][128], as pairs
  BatchAttnArgs a;
  int extra;                // blocks beside one for each tile of rows, to share among long sequences
};

// The tile and range of keys of block i: every sequence's keys are cut into as many ranges
// (at most `most_ranges`) of equal numbers of rounds as `extra` blocks more allow.  The whole warp;
// false: no such block.
OOS_DEV bool balanced_tile(const Pages8Args& p, int i, int tile_rows, int most_ranges, TileRows* t, int* split, int* ranges) {
  const BatchAttnArgs& a = p.a;
  const BatchView& b = a.batch;
  const int lane = threadIdx.x & 31;
  const long long most = min((long long)b.max_pages * a.pages.page_size, (long long)kMaxKeys);
  struct Seq {
    int q0, n, len, tiles, units;
  };
  auto look = [&](int seq, bool report) {
    Seq s = {0, 0, 0, 0, 0};
    if (seq >= b.n_seqs) return s;
    const int q0 = b.q_start[seq], q1 = b.q_start[seq + 1], given = b.seq_len[seq], len = max(0, given);
    const bool in_order = q0 >= 0 && q1 <= b.n_tokens && q0 <= q1, ok = in_order && (!a.parent || q1 - q0 <= kMaxTreeRows);
    if (report && (!ok || given < q1 - q0 || len > most)) *a.status = in_order && !ok ? OOS_ETREE : OOS_EBATCH;
    if (!ok) return s;
    s.q0 = q0;
    s.n = q1 - q0;
    s.len = (int)min((long long)len, most);
    s.tiles = (s.n * a.group + tile_rows - 1) / tile_rows;   // n_tokens * nq stays below 2^26
    s.units = (s.len + kP8Unit - 1) / kP8Unit;
    return s;
  };
  const bool report = i == 0 && blockIdx.y == 0 && threadIdx.x < 32;
  long long total = 0;
  for (int s0 = 0; s0 < b.n_seqs; s0 += 32) {
    const Seq s = look(s0 + lane, report);
    total += (long long)s.tiles * s.units;
  }
#pragma unroll
  for (int x = 16; x; x /= 2) total += __shfl_xor_sync(0xffffffffu, total, x);
  const int target = (int)max(2ll, min((total + p.extra - 1) / p.extra, (long long)kMaxKeys));   // rounds of a range
  int base = 0;
  for (int s0 = 0; s0 < b.n_seqs; s0 += 32) {
    const Seq s = look(s0 + lane, false);
    const int r = max(1, min(most_ranges, (s.units + target - 1) / target));
    int upto = s.tiles * r;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) {
      const int v = __shfl_up_sync(0xffffffffu, upto, x);
      if (lane >= x) upto += v;
    }
    const uint32_t above = __ballot_sync(0xffffffffu, base + upto > i);
    if (above == 0) {
      base += __shfl_sync(0xffffffffu, upto, 31);
      continue;
    }
    const int src = __ffs(above) - 1;
    t->seq = s0 + src;
    t->q0 = __shfl_sync(0xffffffffu, s.q0, src);
    t->n = __shfl_sync(0xffffffffu, s.n, src);
    t->len = __shfl_sync(0xffffffffu, s.len, src);
    t->first = t->len - t->n;
    *ranges = __shfl_sync(0xffffffffu, r, src);
    const int at = i - base - __shfl_sync(0xffffffffu, upto - s.tiles * r, src);
    *split = at % *ranges;
    t->r0 = at / *ranges * tile_rows;
    t->rows = min(tile_rows, t->n * a.group - t->r0);
    return true;
  }
  return false;
}

template <typename TQ, int NT>
__global__ void __launch_bounds__(kP8Warps * 32, p8_blocks(NT)) k_attn_pages8(const __grid_constant__ Pages8Args p) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int ROWS = 8 * NT, STAGES = p8_stages(NT);
  __shared__ TreeScratch s_tree;
  __shared__ uint64_t s_full[kP8Warps][STAGES];
  const BatchAttnArgs& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = blockIdx.y, S = a.s_splits;
  uint64_t* full = s_full[warp];
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) mbar_init(full + i, 2);   // a lane for each block of positions
    mbar_fence_init();
    tma_prefetch_desc(&p.kmap);
    tma_prefetch_desc(&p.vmap);
  }
  __syncwarp();
  // behind the prefix's kernel, which has waited for what the caller wrote before it
  // triggers, only the join waits
  if (a.p_splits == 0) pdl_wait();
  pdl_trigger();
  TileRows t;
  int split = 0, ranges = 1;
  if (!(S > 1 ? balanced_tile(p, blockIdx.x, ROWS, S, &t, &split, &ranges) : sequence_tile(a, blockIdx.x, ROWS, &t))) {
    if (blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();       // the grid must not end before the one it follows
    return;
  }
  const unsigned long long (*anc)[2] = nullptr;
  if (a.parent) anc = tree_sets(a, t.q0, t.n, &s_tree);
  const int last = (t.r0 + t.rows - 1) / a.group;
  const int n_keys = anc ? t.len : max(0, min(t.len, t.first + last + 1));
  const int units = (n_keys + kP8Unit - 1) / kP8Unit;
  const int k0 = (int)((long long)units * split / ranges) * kP8Unit;
  const int k1 = min(n_keys, (int)((long long)units * (split + 1) / ranges) * kP8Unit);
  const int n_rounds = max(0, k1 - k0 + kP8Unit - 1) / kP8Unit;

  // ---- places and scales of 16 rounds: lane 2 r + h has block h of round r
  const int* table = a.batch.table + (size_t)t.seq * a.batch.max_pages;
  const int per_page = a.pages.page_size / kScaleBlock;
  struct Place {
    int page, slot;   // of the first position; page -1: none
    int scales;       // K's byte and V's, and above them 1
  };
  auto look_up = [&](int round) {
    Place at = {-1, 0, 127 | 127 << 8};
    const int key = k0 + (round + (lane >> 1)) * kP8Unit + warp * kP8Keys + (lane & 1) * kScaleBlock;
    if (round + (lane >> 1) < n_rounds && key < k1) {   // no further than the table
      const int b = key / kScaleBlock, col = b / per_page, page = __ldg(table + col);
      if (page >= 0 && page < a.pages.n_pages) {
        const int in_page = b - col * per_page;
        const long long block = ((long long)page * per_page + in_page) * a.pages.nkv + g;
        at = {page, in_page * kScaleBlock, 1 << 16 | __ldg(a.k_scale + block) | __ldg(a.v_scale + block) << 8};
      } else {
        *a.status = OOS_EBATCH;
      }
    }
    return at;
  };
  Place place = look_up(0), place2 = {-1, 0, 0};   // of this batch of 16 rounds and the next

  // ---- copies: this warp's two blocks of a round into its own ring
  unsigned char* ring = smem + warp * (STAGES * kP8Stage);
  const uint64_t policy = t.n * a.group <= ROWS ? policy_evict_first() : policy_evict_last();   // read once, or by other tiles too
  auto copy = [&](int round, int stage, const Place& at) {
    if (round < n_rounds && (lane >> 1) == (round & 15)) {
      if (at.page >= 0) {
        unsigned char* dst = ring + stage * kP8Stage + (lane & 1) * 2 * kP8Half;
        mbar_arrive_expect_tx(full + stage, 2 * kP8Half);
        tma_load_4d(dst, &p.kmap, full + stage, 0, g, at.slot, at.page, policy);
        tma_load_4d(dst + kP8Half, &p.vmap, full + stage, 0, g, at.slot, at.page, policy);
      } else {
        mbar_arrive(full + stage);
      }
    }
  };
  auto landed = [&](int stage, uint32_t parity) {   // a wait of at most kWaitLimitNs
    const uint32_t addr = smem_addr(full + stage);
    if (mbar_test_sleep(addr, parity, 20000u)) return true;
    const unsigned long long t0 = globaltimer();
    while (!mbar_test_sleep(addr, parity, 20000u)) {
      if (globaltimer() - t0 > kWaitLimitNs) {
        *a.status = OOS_ETIMEOUT;
        return false;
      }
    }
    return true;
  };
#pragma unroll
  for (int c = 0; c < STAGES - 1; ++c) copy(c, c, place);

  // ---- the queries as B fragments: row lane / 4 of each 8, d = 16 k + 4 (lane % 4) ..
  uint32_t qf[NT][8][2];
  float sc[NT][2];   // a column's two rows of this thread: 8 n + 2 (lane & 3) + e
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 8 * n + (lane >> 2), row = t.r0 + r;
    const bool on = r < t.rows;
    const TQ* q = (const TQ*)a.q + (long long)(t.q0 + (on ? row / a.group : 0)) * a.q_stride +
                  (g * a.group + row % a.group) * kP8D + (lane & 3) * 4;
    const bool wide = (((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 7) == 0;
    float x[8][4], mx = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      Vec<TQ, 4> v = {};
      if (on && wide) v = *reinterpret_cast<const Vec<TQ, 4>*>(q + 16 * k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (on && !wide) v.v[i] = q[16 * k + i];
        x[k][i] = on ? finite_or_nan(to_f32(v.v[i])) : 0.f;
        mx = fmaxf(mx, fabsf(x[k][i]));
      }
    }
    int e2 = 0;
    if constexpr (std::is_same<TQ, __nv_bfloat16>::value) {
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      e2 = row_exponent(mx);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      qf[n][k][0] = half2_of(x[k][0] * exp2i(-e2), x[k][1] * exp2i(-e2));
      qf[n][k][1] = half2_of(x[k][2] * exp2i(-e2), x[k][3] * exp2i(-e2));
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

  // O of rows 8 n + 2 (lane & 3) + e is in 2^(mo - 7), l in 2^m
  float o[8][NT][4], m[NT][2], mo[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      m[n][e] = mo[n][e] = -INFINITY;
      l[n][e] = 0.f;
    }
  }
  // ldmatrix rows of this lane: 8 keys of a 16-byte column, the 16 keys of one column and of the next
  const uint32_t l_key = lane & 15, l_col = lane >> 4;

  int at = 0;   // of the ring
  uint32_t parity = 0;
#pragma unroll 1
  for (int c = 0; c < n_rounds; ++c) {
    if (!__all_sync(0xffffffffu, landed(at, parity))) {
      for (int i = 1; i < STAGES; ++i) {   // the copies on their way end before the block does
        if (++at == STAGES) at = 0, parity ^= 1;
        if (c + i < n_rounds) landed(at, parity);
      }
      break;
    }
    if ((c & 15) == 8) place2 = look_up((c & ~15) + 16);
    {
      const int ahead = c + STAGES - 1;
      copy(ahead, at == 0 ? STAGES - 1 : at - 1, (ahead ^ c) & 16 ? place2 : place);
    }
    const int key0 = k0 + c * kP8Unit + warp * kP8Keys;
    const uint32_t buf = smem_addr(ring) + at * kP8Stage;
    if (++at == STAGES) at = 0, parity ^= 1;
    int there[2], ek[2], ev[2];   // keys of either block that are there, from its first on; its exponents
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int w = __shfl_sync(0xffffffffu, place.scales, 2 * (c & 15) + h);
      there[h] = w >> 16 ? max(0, min(kScaleBlock, k1 - key0 - h * kScaleBlock)) : 0;
      ek[h] = scale_exp(w & 255);
      ev[h] = scale_exp(w >> 8 & 255);
    }
    if ((c & 15) == 15) place = place2;
    __syncwarp();
    // nothing there, or no row that sees the first key (warp-uniform)
    if (there[0] + there[1] == 0 || (!anc && key0 > t.first + tok_hi)) continue;
    float s[2][NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[h][n][e] = 0.f;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        uint32_t k4[4];   // keys 0-7 and 8-15 of 16 of d, and of the next 16
        ldm4(buf + h * 2 * kP8Half + l_key * kP8D + (((2 * kk + l_col) ^ (l_key & 7)) << 4), k4);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t a0 = e4m3x2_half2((uint16_t)k4[2 * j]), a2 = e4m3x2_half2((uint16_t)(k4[2 * j] >> 16));
          const uint32_t a1 = e4m3x2_half2((uint16_t)k4[2 * j + 1]), a3 = e4m3x2_half2((uint16_t)(k4[2 * j + 1] >> 16));
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_half(s[h][n], a0, a1, a2, a3, qf[n][2 * kk + j][0], qf[n][2 * kk + j][1]);
        }
      }
      const float pk = pow2f(ek[h]);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[h][n][e] *= sc[n][e & 1] * pk;
    }
    // keys that each of this thread's rows sees
    const int seen = t.first - key0;   // those before it are committed
    const bool whole = there[0] + there[1] == kP8Keys && (anc ? seen : seen + tok_lo + 1) >= kP8Keys;
    uint32_t bits[NT][2];
    if (!whole) {
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
    const float fv[2] = {(float)ev[0], (float)ev[1]};
    bool move = false;   // a NaN is above any maximum
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          move = move || !(max_nan(s[h][n][e], s[h][n][2 + e]) <= fminf(m[n][e] + 8.f, mo[n][e] + 8.f - fv[h]));
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float top[2] = {max_nan(s[0][n][e], s[0][n][2 + e]), max_nan(s[1][n][e], s[1][n][2 + e])};
          float mx = max_nan(top[0], top[1]), mv = max_nan(top[0] + fv[0], top[1] + fv[1]);
#pragma unroll
          for (int x = 4; x < 32; x *= 2) {
            mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, x));
            mv = max_nan(mv, __shfl_xor_sync(0xffffffffu, mv, x));
          }
          auto moved = [](float& was, float to) {   // and the factor of what stands in 2^was
            if (to <= was + 8.f) return 1.f;
            const float f = was == -INFINITY ? 0.f : exp2f(was - to);
            was = to;
            return f;
          };
          l[n][e] *= moved(m[n][e], mx);
          const float f = moved(mo[n][e], mv);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[i][n][e] *= f;
            o[i][n][2 + e] *= f;
          }
        }
    }
    // without a finite score yet every score is -inf, and gives 0
    uint32_t pf[2][NT][2];   // as B fragments: 8 x 8 of (key, row) turned to (row, key)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float by[2] = {m[n][0] == -INFINITY ? 0.f : -m[n][0], m[n][1] == -INFINITY ? 0.f : -m[n][1]};
      const float byo[2] = {mo[n][0] == -INFINITY ? 0.f : kHalfBias - mo[n][0], mo[n][1] == -INFINITY ? 0.f : kHalfBias - mo[n][1]};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float s0 = s[h][n][2 * u], s1 = s[h][n][2 * u + 1];
          l[n][0] += ex2_approx(s0 + by[0]);
          l[n][1] += ex2_approx(s1 + by[1]);
          pf[h][n][u] = turned8x8(half2_of(ex2_approx(s0 + (byo[0] + fv[h])), ex2_approx(s1 + (byo[1] + fv[h]))));
        }
    }
    auto add_block = [&](int h, const uint32_t (&pf)[NT][2], auto some_masked) {
      const uint32_t vbuf = buf + (2 * h + 1) * kP8Half;
      uint32_t nan = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[4];   // keys 0-7 and 8-15 of 16 columns, and of the next 16
        ldm4_trans(vbuf + l_key * kP8D + (((2 * i + l_col) ^ (l_key & 7)) << 4), w);
        if (some_masked) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t is = ((w[x] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            nan |= is;
            w[x] &= ~((is >> 7) * 0xffu);
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t lo = __byte_perm(w[2 * j], 0, 0x3120), hi = __byte_perm(w[2 * j + 1], 0, 0x3120);   // even of d, odd of d
          const uint32_t a0 = e4m3x2_half2((uint16_t)lo), a1 = e4m3x2_half2((uint16_t)(lo >> 16));
          const uint32_t a2 = e4m3x2_half2((uint16_t)hi), a3 = e4m3x2_half2((uint16_t)(hi >> 16));
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_half(o[2 * i + j][n], a0, a1, a2, a3, pf[n][0], pf[n][1]);
        }
      }
      if (some_masked && __any_sync(0xffffffffu, nan != 0)) {   // the columns' rows that see the key
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
    };
    if (whole) {
      add_block(0, pf[0], std::false_type());
      add_block(1, pf[1], std::false_type());
    } else {
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        uint32_t now[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int u = 0; u < 2; ++u) now[n][u] = h ? pf[1][n][u] : pf[0][n][u];
        if ((h ? there[1] : there[0]) > 0) add_block(h, now, std::true_type());
      }
    }
  }
  __syncthreads();
  // ---- join: O rows with (m, l), staged over the rings, of every warp, and the prefix's parts
  constexpr float kUnbias = 0x1p-7f;
  static_assert(kHalfBias == 7.f, "the weights' power");
  float* stage = reinterpret_cast<float*>(smem);   // [warp][row][kPartLd]
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int x = 4; x < 32; x *= 2) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
      float* row = stage + (warp * ROWS + 8 * n + (lane & 3) * 2 + e) * kPartLd;
      const float f = mo[n][e] == -INFINITY ? 1.f : exp2f(mo[n][e] - m[n][e]);   // O in 2^m, too
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<float2*>(row + 16 * i + 2 * (lane >> 2)) = make_float2(o[i][n][e] * kUnbias * f, o[i][n][2 + e] * kUnbias * f);
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
      // parts that the sequence has no ranges for
      if (split == ranges - 1 && lane < S - ranges) *reinterpret_cast<float2*>(to + (1 + lane) * part_step + kP8D) = make_float2(-INFINITY, 0.f);
    } else {
      store_row<TQ>(a, g, t.q0, t.r0 + r, weighted_mean(acc, den));
    }
  }
  if (a.own_part && blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();   // a kernel that waits for this one counts on the prefix's
}

PagesPlan plan_pages8_tc(long long rows, int n_seqs, int nkv, bool prefix, long long most_keys, int n_sms) {
  PagesPlan p = {};
  const int per_sm = p8_blocks(rows <= 8ll * n_seqs ? 1 : 2);
  p.tile_rows = rows <= 8ll * n_seqs ? 8 : 16;
  p.tiles = (int)(n_seqs + rows / p.tile_rows);
  const long long live = std::max((long long)n_seqs, (rows + p.tile_rows - 1) / p.tile_rows) * nkv;
  // Ranges, each with two rounds at least, for as many blocks as the chip holds: a block's
  // beginning and end cost as much as a few rounds (6 requests of up to 64000 keys, 8 kv heads:
  // 70 us, for twice as many 76, three times 87).
  const long long most = (long long)per_sm * n_sms, ranges = std::min<long long>(kP8MaxParts - (prefix ? kMaxPrefixParts : 0), most_keys / (2 * kP8Unit));
  p.extra = (int)((most - live) / nkv);
  p.splits = p.extra > 0 ? (int)std::max(1ll, ranges) : 1;
  p.sms = (int)std::min<long long>(n_sms, ((p.splits > 1 ? most : live) + per_sm - 1) / per_sm);
  p.part = p.splits > 1;
  return p;
}

template <typename TQ, int NT>
static cudaError_t launch_pages8_of(const Pages8Args& a, const PagesPlan& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = kernel_ready(ready, (const void*)k_attn_pages8<TQ, NT>, p8_smem(NT));
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)(p.tiles + (p.splits > 1 ? p.extra : 0)), a.a.pages.nkv);
  return launch(true, k_attn_pages8<TQ, NT>, grid, dim3(kP8Warps * 32), p8_smem(NT), st, a);
}

cudaError_t launch_pages8_tc(const BatchAttnArgs& a, const PagesPlan& p, int dtype, cudaStream_t st) {
  Pages8Args args;
  memset(&args, 0, sizeof(args));
  args.a = a;
  args.extra = p.extra;
  // two codes an element of the copy
  const uint64_t row = (uint64_t)a.pages.nkv * kP8D;
  const uint64_t dims[4] = {kP8D / 2, (uint64_t)a.pages.nkv, (uint64_t)a.pages.page_size, (uint64_t)a.pages.n_pages};
  const uint64_t strides[3] = {kP8D, row, row * a.pages.page_size};
  const uint32_t box[4] = {kP8D / 2, 1, (uint32_t)kScaleBlock, 1};
  if (!encode_bf16_map(&args.kmap, a.pages.k, 4, dims, strides, box, false) ||
      !encode_bf16_map(&args.vmap, a.pages.v, 4, dims, strides, box, false))
    return cudaErrorInvalidValue;
  if (dtype == OOS_DTYPE_BF16)
    return p.tile_rows == 8 ? launch_pages8_of<__nv_bfloat16, 1>(args, p, st) : launch_pages8_of<__nv_bfloat16, 2>(args, p, st);
  return p.tile_rows == 8 ? launch_pages8_of<__half, 1>(args, p, st) : launch_pages8_of<__half, 2>(args, p, st);
}

}  // namespace oos
