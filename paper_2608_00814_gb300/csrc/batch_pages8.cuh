// Rows of a sequence against 32 of its own keys in 8-bit pages, a warp's work (batch_pages8.cu,
// batch_stream8.cu): 16-bit queries with heads of 128, 8 or 16 rows (token, head of one kv head's
// group).
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
#pragma once

#include <math.h>

#include <type_traits>

#include "attn.cuh"
#include "batch_attn.cuh"
#include "pages8.cuh"

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

struct P8Maps {
  CUtensorMap k, v;   // codes [n_pages][page_size][nkv][128], as pairs
};

// Where 16 positions with one scale lie
struct P8Place {
  int page, slot;   // of the first position; page -1: none
  int scales;       // K's byte and V's, and above them 1
};
// of the sequence whose row of the page table is given; block: its positions 16 block ..
OOS_DEV P8Place p8_place(const BatchAttnArgs& a, int g, int seq, int block) {
  const int per_page = a.pages.page_size / kScaleBlock;
  const int col = block / per_page, page = __ldg(a.batch.table + (size_t)seq * a.batch.max_pages + col);
  if (page < 0 || page >= a.pages.n_pages) {
    *a.status = OOS_EBATCH;
    return {-1, 0, 127 | 127 << 8};
  }
  const int in_page = block - col * per_page;
  const long long at = ((long long)page * per_page + in_page) * a.pages.nkv + g;
  return {page, in_page * kScaleBlock, 1 << 16 | __ldg(a.k_scale + at) | __ldg(a.v_scale + at) << 8};
}

// A warp's ring of STAGES times 32 keys' K and V
template <int STAGES>
struct P8Ring {
  unsigned char* data;
  uint64_t* full;      // [STAGES]
  uint64_t policy;
  int at = 0;          // the stage that is read next
  uint32_t parity = 0;

  OOS_DEV void init() {
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int i = 0; i < STAGES; ++i) mbar_init(full + i, 2);   // a lane for each block of positions
      mbar_fence_init();
    }
    __syncwarp();
  }
  // one lane for each of the two blocks, h
  OOS_DEV void copy(const P8Maps& map, int g, int stage, int h, const P8Place& from) {
    if (from.page >= 0) {
      unsigned char* dst = data + stage * kP8Stage + h * 2 * kP8Half;
      mbar_arrive_expect_tx(full + stage, 2 * kP8Half);
      tma_load_4d(dst, &map.k, full + stage, 0, g, from.slot, from.page, policy);
      tma_load_4d(dst + kP8Half, &map.v, full + stage, 0, g, from.slot, from.page, policy);
    } else {
      mbar_arrive(full + stage);
    }
  }
  OOS_DEV int behind() const { return at == 0 ? STAGES - 1 : at - 1; }   // the stage read last
  OOS_DEV void next() {
    if (++at == STAGES) {
      at = 0;
      parity ^= 1;
    }
  }
  OOS_DEV bool landed(int32_t* status) const {   // a wait of at most kWaitLimitNs
    const uint32_t addr = smem_addr(full + at);
    if (mbar_test_sleep(addr, parity, 20000u)) return true;
    const unsigned long long t0 = globaltimer();
    while (!mbar_test_sleep(addr, parity, 20000u)) {
      if (globaltimer() - t0 > kWaitLimitNs) {
        *status = OOS_ETIMEOUT;
        return false;
      }
    }
    return true;
  }
  // the whole warp; `more` copies on their way behind this one end before it gives up
  OOS_DEV bool wait(int32_t* status, int more) {
    if (__all_sync(0xffffffffu, landed(status))) return true;
    for (int i = 0; i < more; ++i) {
      next();
      landed(status);
    }
    return false;
  }
};

// Rows of a tile in a warp: thread's rows 8 n + 2 (lane % 4) + e, columns 16 i + 2 (lane / 4) + 0, 1
template <typename TQ, int NT>
struct P8Rows {
  uint32_t qf[NT][8][2];
  float sc[NT][2];
  int token[NT][2];                     // from the sequence's first
  unsigned long long an[NT][2][2];      // ancestors, with a tree
  int tok_lo, tok_hi;
  // O is in 2^(mo - 7), l in 2^m; o: column 0 of rows e = 0, 1, and column 1
  float o[8][NT][4], m[NT][2], mo[NT][2], l[NT][2];

  OOS_DEV void clear() {
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
  }

  // ancestors(token): where they are, two words; nullptr: no tree
  template <typename F>
  OOS_DEV void load(const BatchAttnArgs& a, int g, const TileRows& t, F ancestors) {
    const int lane = threadIdx.x & 31;
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

#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * n + (lane & 3) * 2 + e;
        token[n][e] = (t.r0 + r) / a.group;
        an[n][e][0] = an[n][e][1] = 0;
        if (a.parent && r < t.rows) ancestors(token[n][e], an[n][e]);
      }
    tok_lo = t.r0 / a.group;
    tok_hi = (t.r0 + t.rows - 1) / a.group;
  }

  // 32 keys from key0 on, of n_keys; scales: P8Place's of both blocks; data: the stage
  OOS_DEV void unit(const BatchAttnArgs& a, const TileRows& t, const unsigned char* data, int key0, int n_keys, const int (&scales)[2]) {
    const int lane = threadIdx.x & 31;
    const bool anc = a.parent != nullptr;
    const uint32_t buf = smem_addr(data);
    // ldmatrix rows of this lane: 8 keys of a 16-byte column, the 16 keys of one column and of the next
    const uint32_t l_key = lane & 15, l_col = lane >> 4;
    int there[2], ek[2], ev[2];   // keys of either block that are there, from its first on; its exponents
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      there[h] = scales[h] >> 16 ? max(0, min(kScaleBlock, n_keys - key0 - h * kScaleBlock)) : 0;
      ek[h] = scale_exp(scales[h] & 255);
      ev[h] = scale_exp(scales[h] >> 8 & 255);
    }
    // nothing there, or no row that sees the first key (warp-uniform)
    if (there[0] + there[1] == 0 || (!anc && key0 > t.first + tok_hi)) return;
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
        for (int e = 0; e < 4; ++e) s[h][n][e] *= fminf(sc[n][e & 1] * pk, kMostFactor);
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
              const uint32_t code = data[vbuf - buf + key * kP8D + ((i ^ (key & 7)) << 4) + 2 * (lane >> 2) + u];
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

  OOS_DEV void add_lanes() {   // l's shares of the 8 lanes that hold a row
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int x = 4; x < 32; x *= 2) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
  }
  // O, m and l of the thread's row (n, e) to `row`, O in 2^m too
  OOS_DEV void store(int n, int e, float* row) const {
    static_assert(kHalfBias == 7.f, "the weights' power");
    const int lane = threadIdx.x & 31;
    const float f = mo[n][e] == -INFINITY ? 1.f : exp2f(mo[n][e] - m[n][e]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      *reinterpret_cast<float2*>(row + 16 * i + 2 * (lane >> 2)) = make_float2(o[i][n][e] * 0x1p-7f * f, o[i][n][2 + e] * 0x1p-7f * f);
    if (lane < 4) *reinterpret_cast<float2*>(row + kP8D) = make_float2(m[n][e], l[n][e]);
  }
};

bool p8_maps(const BatchAttnArgs& a, P8Maps* maps);

}  // namespace oos
