// Attention of a batch step on tensor cores over the sequences' own 8-bit pages, 16-bit
// queries with heads of 128, for what has many rows: the kernel of batch_tiles.cu (its
// streams, its score buffer, its softmax) with other operands.
//
// Scores: tcgen05 kind::f8f6f4, K's codes as they are, copied page by page into the swizzled
// layout.  A row of q, scaled by a power of two so that its largest element lies in [2^7, 2^8), is a
// sum of two (bf16) or three (binary16) e4m3 parts whose products add up in one accumulator:
// what is left of an element is below half of e4m3's smallest step, 2^-10, 2^-17 of the largest.  These
// products run at twice the rate of 16-bit ones, and K needs no conversion.  Its scales go
// to the scores, a factor for each 16 columns of the thread's row.
//
// P.V: kind::f16.  Four warps convert V, each two blocks of 16 positions of a tile, from a
// ring of copies of the codes.
//   bf16 queries: weights and V are bf16.  Bytes are moved apart into numbers of 2^-120 of the
//     value, a product with 2^(120 + scale) does the rest, exactly.  It leaves the codes of four
//     neighbours in the order 0, 2, 1, 3; O's columns are put right when they are staged.  A NaN
//     code's bits would come out as 480 and are set to NaN by the thread that finds them.
//   binary16 queries: weights and V are binary16, 2^-11 instead of 2^-8.  The codes go through
//     the conversion of two at a time, and the scale 2^e is a factor of the weight,
//     2^(score + e - m + 7) with m a maximum of score + e: what a row adds up is rounded to
//     2^-11, below 2^-21 of its largest term (448 2^e times the weight) to 2^-32 of that.  The sum of the weights is
//     taken of unrounded ones without the scales, which has all of them down to 2^-37 of the
//     largest while every e is 48 at most, either way.  From the first tile with another e on it
//     has exponentials of its own, with a maximum of the scores alone.
//
// 13 prompts of up to 300 tokens, 40 heads over 8, 1000 shared and up to 1800 own keys in
// binary16: 200 us (tiles of 16 rows, before this kernel: 783); 16 trees of up to 64 nodes, 32
// heads, 2048 shared and up to 464 own keys in bf16: 60 (128).  The shared keys are the other
// kernel's.  Without them the prompts take 119 us (16-bit pages 138): neither the conversion (9
// us), nor K's copies (7), nor the exponentials (12) bound it, but what a block of few key tiles
// does one after the other.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "batch_tiles.cuh"
#include "pages8.cuh"

namespace oos {

constexpr int kT8Codes = kTlKeys * kTlD;   // bytes of a tile of codes
constexpr int kT8VStages = 2;
constexpr int kT8Threads = 512;            // K; scores; P.V; -; V x 4; softmax x 8
constexpr int kT8Soft0 = 8, kT8V0 = 4;
constexpr int kT8Ordered = 64;             // sequences whose tiles are dealt by length
constexpr int kT8NearExp = 48;             // V's exponents whose weights in binary16 give the sum, too
constexpr int kT8RegsIo = 64, kT8RegsSoft = 192, kT8RegsLaunch = 128;
static_assert(256 * kT8RegsIo + 256 * kT8RegsSoft <= kT8Threads * kT8RegsLaunch, "register split");
// PARTS: of a query
template <int PARTS>
struct T8 {
  static constexpr int kKStages = PARTS == 2 ? 3 : 2, kRaw = PARTS == 2 ? 3 : 2;
  static constexpr int kOffV = kKStages * kT8Codes, kOffRaw = kOffV + kT8VStages * kTlTile, kOffQ = kOffRaw + kRaw * kT8Codes;
  static constexpr int kOffExp = kOffQ + 2 * PARTS * kT8Codes;   // row exponents of the queries
  static constexpr int kOffBar = kOffExp + 2 * kTlRows * 4, kSmem = kOffBar + 384 + 1024;   // + alignment slack
  static_assert(kTlStaged <= kOffExp, "staged rows and their weights over the rings and queries");
  static_assert(kSmem <= 227 * 1024, "shared memory per block");
};

OOS_DEV uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// bytes 0 and 2 (1 and 3) of a word of codes as bf16 of 2^-120 the value
OOS_DEV uint32_t even_codes(uint32_t w) { return ((w << 8) & 0x80008000u) | ((w << 4) & 0x07f007f0u); }
OOS_DEV uint32_t odd_codes(uint32_t w) { return (w & 0x80008000u) | ((w >> 4) & 0x07f007f0u); }

// Instruction descriptor of tcgen05.mma.kind::f8f6f4 with e4m3 A and B (format 0 in both
// fields), fp32 D, both K-major
constexpr uint32_t idesc_e4m3_f32(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
OOS_DEV void tc_mma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Tile i of the sequences' tiles, the longest sequences' first: blocks of many key tiles that
// begin last would leave most SMs idle behind them.  n_seqs <= kT8Ordered, two a lane; each
// adds up the tiles of those before it.  In the sequences' order, heads slowest, the prompts
// above take 233 us and the trees 64.  The whole warp; false: no such tile.
OOS_DEV bool longest_first(const BatchAttnArgs& a, int i, TileRows* t) {
  const BatchView& b = a.batch;
  const int lane = threadIdx.x & 31;
  const long long most = min((long long)b.max_pages * a.pages.page_size, (long long)kMaxKeys);
  int q0[2], n[2], len[2], tiles[2], start[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int seq = lane + 32 * u;
    q0[u] = n[u] = len[u] = tiles[u] = start[u] = 0;
    if (seq >= b.n_seqs) continue;
    const int from = b.q_start[seq], to = b.q_start[seq + 1], given = b.seq_len[seq], held = max(0, given);
    const bool in_order = from >= 0 && to <= b.n_tokens && from <= to, ok = in_order && (!a.parent || to - from <= kMaxTreeRows);
    if (blockIdx.x == 0 && threadIdx.x < 32 && (!ok || given < to - from || held > most))
      *a.status = in_order && !ok ? OOS_ETREE : OOS_EBATCH;
    if (!ok) continue;
    q0[u] = from;
    n[u] = to - from;
    len[u] = (int)min((long long)held, most);
    tiles[u] = (n[u] * a.group + 2 * kTlRows - 1) / (2 * kTlRows);   // n_tokens * nq stays below 2^26
  }
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    if (32 * v >= b.n_seqs) break;
#pragma unroll 4
    for (int x = 0; x < 32; ++x) {
      const int other = __shfl_sync(0xffffffffu, len[v], x), its = __shfl_sync(0xffffffffu, tiles[v], x);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (other > len[u] || (other == len[u] && x + 32 * v < lane + 32 * u)) start[u] += its;
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint32_t who = __ballot_sync(0xffffffffu, i >= start[u] && i < start[u] + tiles[u]);
    if (who == 0) continue;
    const int src = __ffs(who) - 1;
    t->seq = src + 32 * u;
    t->q0 = __shfl_sync(0xffffffffu, q0[u], src);
    t->n = __shfl_sync(0xffffffffu, n[u], src);
    t->len = __shfl_sync(0xffffffffu, len[u], src);
    t->first = t->len - t->n;
    t->r0 = (i - __shfl_sync(0xffffffffu, start[u], src)) * 2 * kTlRows;
    t->rows = min(2 * kTlRows, t->n * a.group - t->r0);
    return true;
  }
  return false;
}

template <typename TQ>
__global__ void __launch_bounds__(kT8Threads, 1) k_attn_tiles8(const __grid_constant__ BatchAttnArgs a) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr bool F16 = !std::is_same<TQ, __nv_bfloat16>::value;   // weights and V, as the queries
  constexpr int PARTS = F16 ? 3 : 2;
  using L = T8<PARTS>;
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + L::kOffBar);
  uint64_t* kfull = bar;           // [3] codes copied
  uint64_t* kempty = bar + 3;      // [3] its score products done
  uint64_t* vfull = bar + 6;       // [2] four V warps: converted
  uint64_t* vempty = bar + 8;      // [2] its P.V products done
  uint64_t* sfull = bar + 10;      // [2] scores of a stream done
  uint64_t* pfull = bar + 12;      // [stream][key half] four softmax warps: P written
  uint64_t* pvdone = bar + 16;     // [2] P.V of a stream done
  uint64_t* sfree = bar + 18;      // [2] four softmax warps: scores in registers
  uint64_t* qready = bar + 20;     // eight warps: queries in shared memory
  uint64_t* odone = bar + 21;      // both issuers: all products done
  uint64_t* sets_read = bar + 22;  // eight warps: ancestors in registers
  // of a V stage, by the V warps: the power of K's scale and 2^-7, V's exponent if the weights take
  // it and the keys that are there, of each 16, and a byte of each warp: a v is NaN (1), an
  // exponent of the weights is not near 0 (2)
  float* s_kpow = reinterpret_cast<float*>(bar + 23);                // [2][8]
  float* s_vexp = s_kpow + 16;                                       // [2][8]
  uint16_t* s_valid = reinterpret_cast<uint16_t*>(s_vexp + 16);      // [2][8]
  uint8_t* s_wild = reinterpret_cast<uint8_t*>(s_valid + 16);        // [2][4]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(s_wild + 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* s_apart = abort_flag + 1;                       // [2] the stream's tile whose P.V is done, + 1
  static_assert(23 * 8 + 32 * 4 + 16 * 2 + 8 + 4 * 4 <= 384, "barrier block");
  int32_t* status = a.status;
  const int S = a.s_splits, nkv = a.pages.nkv, g = blockIdx.x % nkv, at = blockIdx.x / nkv, split = at % S, pair = at / S;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // behind the prefix's kernel, which has waited for what the caller wrote before it
  // triggers, only the end waits for the prefix's parts
  if (a.p_splits == 0) pdl_wait();
  pdl_trigger();
  TileRows t = {};
  if (!(a.batch.n_seqs <= kT8Ordered ? longest_first(a, pair, &t) : sequence_tile(a, pair, 2 * kTlRows, &t))) {
    if (blockIdx.x == 0) pdl_wait();   // the grid must not end before the one it follows
    return;
  }
  const int rows = t.rows;
  const int dual = rows > kTlRows ? 1 : 0;
  // keys of the sequence that some row sees
  const int n_own = a.parent ? t.len : max(0, min(t.len, t.first + (t.r0 + rows - 1) / a.group + 1));
  const int n_all = (n_own + kTlKeys - 1) / kTlKeys;
  const int t0 = (int)((long long)n_all * split / S);
  const int n_tiles = (int)((long long)n_all * (split + 1) / S) - t0;
  const bool joined = S == 1 && !a.own_part;   // its rows go into out
  const int units = n_tiles << dual;                  // unit u: tile u >> dual, stream u & 1
  if (threadIdx.x == 0) {
    for (int i = 0; i < 3; ++i) {
      mbar_init(&kfull[i], 1);
      mbar_init(&kempty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&vfull[i], 4);
      mbar_init(&vempty[i], 1);
      mbar_init(&sfull[i], 1);
      mbar_init(&pfull[2 * i], 4);
      mbar_init(&pfull[2 * i + 1], 4);
      mbar_init(&pvdone[i], 1);
      mbar_init(&sfree[i], 4);
    }
    mbar_init(qready, 8);
    mbar_init(sets_read, 8);
    mbar_init(odone, 2);
    *abort_flag = 0;
    s_apart[0] = s_apart[1] = 0;
    mbar_fence_init();
  }
  if (warp == 2) tmem_alloc(tmem_slot, kTlTmCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  float* stage = reinterpret_cast<float*>(sm);
  const long long key_bytes = (long long)a.pages.nkv * kTlD;
  const int* table = a.batch.table + (size_t)t.seq * a.batch.max_pages;
  const int per_page = a.pages.page_size / kScaleBlock;
  auto block_of = [&](int b) {   // of the pool, of the sequence's block b; -1: none
    const int col = b / per_page, page = __ldg(table + col);   // no further than the table
    if (page >= 0 && page < a.pages.n_pages) return (long long)page * per_page + (b - col * per_page);
    *status = OOS_EBATCH;
    return -1ll;
  };

  if (warp < kT8V0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kT8RegsIo));
    if (warp == 0) {
      // ---------------------------------------------------------- K: 8 lanes a key
      int n = 0, copied = -1;   // copied: a tile on its way
      auto announce = [&]() {
        if (copied < 0) return;
        cp_async_wait<0>();
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&kfull[copied % L::kKStages]);
        copied = -1;
      };
      const uint8_t* src = a.pages.k + (long long)g * kTlD + (lane & 7) * 16;
      for (; n < n_tiles; ++n) {
        const int st = n % L::kKStages, key0 = (t0 + n) * kTlKeys;
        long long at = -1;   // block lane % 8 of the tile
        if (key0 + (lane & 7) * kScaleBlock < n_own) at = block_of(key0 / kScaleBlock + (lane & 7));
        announce();
        // the queries come first
        if (n == 1 && !__all_sync(0xffffffffu, tl_wait(qready, 0, abort_flag, status))) break;
        if (n >= L::kKStages &&
            !__all_sync(0xffffffffu, tl_wait(&kempty[st], (uint32_t)(n / L::kKStages - 1) & 1u, abort_flag, status)))
          break;
        const uint32_t to = smem_addr(sm) + st * kT8Codes;
#pragma unroll 4
        for (int i = 0; i < 32; ++i) {
          const int key = 4 * i + (lane >> 3);
          const long long block = __shfl_sync(0xffffffffu, at, i >> 2);
          const bool ok = block >= 0 && key0 + key < n_own;
          cp_async16(to + sw128(key, lane & 7), src + (ok ? (block * kScaleBlock + (key & 15)) * key_bytes : 0), ok);
        }
        cp_async_commit();
        copied = n;
      }
      announce();
      cp_async_wait<0>();
      // every announced copy is read before the block goes on, or its products were not issued
    } else if (warp == 1 && lane == 0) {
      // ---------------------------------------------------------- scores
      constexpr uint32_t idesc = idesc_e4m3_f32(kTlRows, kTlKeys);
      const uint64_t kdesc = smem_desc_sw128(smem_addr(sm)), qdesc = smem_desc_sw128(smem_addr(sm + L::kOffQ));
      bool ok = tl_wait(qready, 0, abort_flag, status);
      for (int u = 0; u < units && ok; ++u) {
        const int i = u >> dual, st = i % L::kKStages, x = u & 1;
        if (!dual || x == 0) ok = tl_wait(&kfull[st], (uint32_t)(i / L::kKStages) & 1u, abort_flag, status);
        if (u > 0) ok = ok && tl_wait(&sfree[x ^ 1], (uint32_t)((u - 1) >> 1) & 1u, abort_flag, status);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < PARTS * (kTlD / 32); ++k) {   // 32 of d, 32 bytes of a row
          const uint64_t q = (uint64_t)((((dual ? x : 0) * PARTS + k / 4) * kT8Codes) >> 4);
          tc_mma_e4m3(tmem + kTlTmS, qdesc + q + 2 * (k & 3), kdesc + (uint64_t)((st * kT8Codes) >> 4) + 2 * (k & 3), idesc,
                      k > 0 ? 1u : 0u);
        }
        tc_commit(&sfull[x]);
        if (!dual || x == 1) tc_commit(&kempty[st]);
      }
      tc_commit(odone);
    } else if (warp == 2 && lane == 0) {
      // ---------------------------------------------------------- P.V
      constexpr uint32_t idesc = (F16 ? idesc_f16_f32(kTlRows, kTlD) : idesc_bf16_f32(kTlRows, kTlD)) | (1u << 16);
      const uint64_t vdesc = smem_desc_sw128_mn(smem_addr(sm + L::kOffV), kTlDBlock);
      bool ok = true;
      for (int u = 0; u < units && ok; ++u) {
        const int i = u >> dual, st = i % kT8VStages, x = u & 1, use = u >> 1;   // use: of this stream
        if (!dual || x == 0) ok = tl_wait(&vfull[st], (uint32_t)(i / kT8VStages) & 1u, abort_flag, status);
        for (int h = 0; h < 2 && ok; ++h) {   // the first half's product runs under the second's exponentials
          ok = tl_wait(&pfull[2 * x + h], (uint32_t)use & 1u, abort_flag, status);
          if (!ok) break;
          tc_fence_after();
          if (s_apart[x] == use + 1) continue;   // in O already
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const int k = 4 * h + kk;
            tc_mma_bf16_ts(tmem + kTlTmO + x * kTlD, tmem + kTlTmP + x * (kTlKeys / 2) + 8 * k,
                           vdesc + (uint64_t)((st * kTlTile + k * 16 * 128) >> 4), idesc, (k > 0 || use > 0) ? 1u : 0u);
          }
        }
        if (!ok) break;
        tc_commit(&pvdone[x]);
        if (!dual || x == 1) tc_commit(&vempty[st]);
      }
      tc_commit(odone);
    }
    __syncwarp();
  } else if (warp < kT8Soft0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kT8RegsIo));
    // ---------------------------------------------------------- V: blocks v and v + 4 of a tile
    const int v = warp - kT8V0;
    const uint8_t* src = a.pages.v + (long long)g * kTlD + (lane & 7) * 16;
    unsigned char* raw = sm + L::kOffRaw;
    // places and scales of 16 tiles: lane 2 j + h has block v + 4 h of tile j
    auto look_up = [&](int tile, long long& at, int& sk, int& sv) {
      const int b = (t0 + tile + (lane >> 1)) * (kTlKeys / kScaleBlock) + v + 4 * (lane & 1);
      at = -1;
      sk = sv = 127;
      if (tile + (lane >> 1) < n_tiles && (long long)b * kScaleBlock < n_own) {
        at = block_of(b);
        if (at >= 0) {
          sk = __ldg(a.k_scale + at * a.pages.nkv + g);
          sv = __ldg(a.v_scale + at * a.pages.nkv + g);
        }
      }
    };
    long long at = -1, at2 = -1;   // of this batch of 16 tiles and the next
    int sk = 127, sv = 127, sk2 = 127, sv2 = 127;
    look_up(0, at, sk, sv);
    auto copy = [&](int n, long long from) {   // a lane copies what it converts
      if (n < n_tiles) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const long long block = __shfl_sync(0xffffffffu, from, 2 * (n & 15) + h);
          const int left = n_own - (t0 + n) * kTlKeys - (v + 4 * h) * kScaleBlock;   // keys from its first on
          const uint32_t to = smem_addr(raw) + n % L::kRaw * kT8Codes + (v + 4 * h) * (kScaleBlock * kTlD) + lane * 16;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = 4 * i + (lane >> 3);
            const bool ok = block >= 0 && key < left;
            cp_async16(to + i * 512, src + (ok ? (block * kScaleBlock + key) * key_bytes : 0), ok);
          }
        }
      }
      cp_async_commit();
    };
    for (int c = 0; c < L::kRaw - 1; ++c) copy(c, at);
    for (int n = 0; n < n_tiles; ++n) {
      const int st = n % kT8VStages;
      cp_async_wait<L::kRaw - 2>();
      if ((n & 15) == 8) look_up((n & ~15) + 16, at2, sk2, sv2);
      copy(n + L::kRaw - 1, ((n + L::kRaw - 1) ^ n) & 16 ? at2 : at);
      // the second V stage holds the tree's sets until they are read
      if (a.parent && n == 1 && !__all_sync(0xffffffffu, tl_wait(sets_read, 0, abort_flag, status))) break;
      if (n >= kT8VStages &&
          !__all_sync(0xffffffffu, tl_wait(&vempty[st], (uint32_t)(n / kT8VStages - 1) & 1u, abort_flag, status)))
        break;
      bool nan = false, far = false;
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        const int from = 2 * (n & 15) + h, b = v + 4 * h;
        const bool there = __shfl_sync(0xffffffffu, at, from) >= 0;
        const int ek = scale_exp(__shfl_sync(0xffffffffu, sk, from)), ev = scale_exp(__shfl_sync(0xffffffffu, sv, from));
        const int left = n_own - (t0 + n) * kTlKeys - b * kScaleBlock;
        if (lane == 0) {
          s_kpow[8 * st + b] = pow2f(ek - 7);
          if (F16) s_vexp[8 * st + b] = (float)ev;
          s_valid[8 * st + b] = (uint16_t)(there && left > 0 ? (1u << min(left, kScaleBlock)) - 1 : 0u);
        }
        const int e1 = min(ev, 7);
        const uint32_t f1 = (uint32_t)(120 + e1 + 127) << 7, f2 = (uint32_t)(ev - e1 + 127) << 7;   // bf16's
        far = far || abs(ev) > kT8NearExp;
        const unsigned char* in = raw + n % L::kRaw * kT8Codes + b * (kScaleBlock * kTlD) + lane * 16;
        const int c = lane & 7;
        unsigned char* out = sm + L::kOffV + st * kTlTile + (c >> 2) * kTlDBlock;
#pragma unroll 2
        for (int i = 0; i < 4; ++i) {
          const int key = b * kScaleBlock + 4 * i + (lane >> 3);
          const uint4 w4 = *reinterpret_cast<const uint4*>(in + i * 512);
          const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
          uint32_t x[8], top = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[2 * j] = F16 ? e4m3x2_half2((uint16_t)w[j]) : mul_bf16x2(even_codes(w[j]), f1 | f1 << 16);
            x[2 * j + 1] = F16 ? e4m3x2_half2((uint16_t)(w[j] >> 16)) : mul_bf16x2(odd_codes(w[j]), f1 | f1 << 16);
            top |= (w[j] & 0x7f7f7f7fu) + 0x01010101u;
          }
          if (!F16 && ev > 7) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = mul_bf16x2(x[j], f2 | f2 << 16);
          }
          if (top & 0x80808080u) {
            nan = true;
#pragma unroll
            for (int j = 0; j < (F16 ? 0 : 4); ++j) {
              const uint32_t is = ((w[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
              if (is & 0x80u) x[2 * j] |= 0x7fffu;
              if (is & 0x800000u) x[2 * j] |= 0x7fff0000u;
              if (is & 0x8000u) x[2 * j + 1] |= 0x7fffu;
              if (is & 0x80000000u) x[2 * j + 1] |= 0x7fff0000u;
            }
          }
          const uint4 lo = make_uint4(x[0], x[1], x[2], x[3]), hi = make_uint4(x[4], x[5], x[6], x[7]);
          // half the lanes the other half first: no two of a row on the same banks
          const int c0 = 2 * (c & 3), first = c >> 2;
          *reinterpret_cast<uint4*>(out + sw128(key, c0 + first)) = first ? hi : lo;
          *reinterpret_cast<uint4*>(out + sw128(key, c0 + 1 - first)) = first ? lo : hi;
        }
      }
      nan = __any_sync(0xffffffffu, nan);
      if (lane == 0) s_wild[4 * st + v] = (nan ? 1 : 0) | (F16 && far ? 2 : 0);
      if ((n & 15) == 15) {
        at = at2;
        sk = sk2;
        sv = sv2;
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&vfull[st]);
    }
    cp_async_wait<0>();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kT8RegsSoft));
    // ------------------------------------------------------------ softmax: stream x, a thread per row
    const int x = (warp - kT8Soft0) >> 2, q4 = warp & 3;
    const int lrow = q4 * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    float* s_exp = reinterpret_cast<float*>(sm + L::kOffExp);
    // queries of the stream's row tile (one row tile: the first stream's warps), two rows
    // of 16 lanes at a time
    const int c = lane & 15;
    uint4 w[16];   // all rows' loads in flight
    if (x == 0 || dual) {
      const int r = x * kTlRows + lrow, row = t.r0 + r;
      const long long mine = (long long)(t.q0 + row / a.group) * a.q_stride + (g * a.group + row % a.group) * kTlD;
      const uint16_t* q0 = (const uint16_t*)a.q + c * 8;
      const bool wide = (((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 15) == 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int from = 2 * i + (lane >> 4);
        const uint16_t* q = q0 + __shfl_sync(0xffffffffu, mine, from);
        w[i] = make_uint4(0, 0, 0, 0);
        if (x * kTlRows + q4 * 32 + from < rows) {
          if (wide) w[i] = *reinterpret_cast<const uint4*>(q);
          else w[i] = make_uint4((uint32_t)q[0] | (uint32_t)q[1] << 16, (uint32_t)q[2] | (uint32_t)q[3] << 16,
                                 (uint32_t)q[4] | (uint32_t)q[5] << 16, (uint32_t)q[6] | (uint32_t)q[7] << 16);
        }
      }
    }
    // ancestors of the thread's row, while the queries are on their way
    unsigned long long anc0 = 0, anc1 = 0;
    if (a.parent) {
      const unsigned long long (*sets)[2] =
          tree_sets(a, t.q0, t.n, reinterpret_cast<TreeScratch*>(sm + L::kOffV + kTlTile), threadIdx.x - 32 * kT8Soft0,
                    32 * 8, [] { asm volatile("bar.sync 1, 256;" ::: "memory"); });
      const int r = (dual ? x * kTlRows : 0) + lrow;
      if (r < rows) {
        anc0 = sets[(t.r0 + r) / a.group][0];
        anc1 = sets[(t.r0 + r) / a.group][1];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(sets_read);   // the V warps' stores follow
    }
    if (x == 0 || dual) {
      unsigned char* qs = sm + L::kOffQ + x * PARTS * kT8Codes;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = q4 * 32 + 2 * i + (lane >> 4);
        float y[8], mx = 0.f;
        const uint32_t ww[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float2 z;
          if constexpr (PARTS == 2) z = make_float2(bf16_lo(ww[e]), bf16_hi(ww[e]));
          else z = __half22float2(*reinterpret_cast<const __half2*>(&ww[e]));
          y[2 * e] = finite_or_nan(z.x);
          y[2 * e + 1] = finite_or_nan(z.y);
          mx = fmaxf(mx, fmaxf(fabsf(y[2 * e]), fabsf(y[2 * e + 1])));
        }
#pragma unroll
        for (int s = 1; s < 16; s *= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
        const int e2 = row_exponent(mx);
        if (c == 0) s_exp[x * kTlRows + r] = exp2i(e2);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = y[e] * exp2i(-e2) * 128.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          uint16_t z[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[e] = f32x2_e4m3(y[2 * e], y[2 * e + 1]);
            const float2 f = e4m3x2_f32(z[e]);
            y[2 * e] -= f.x;
            y[2 * e + 1] -= f.y;
          }
          *reinterpret_cast<uint2*>(qs + p * kT8Codes + sw128(r, c >> 1) + (c & 1) * 8) =
              make_uint2((uint32_t)z[0] | (uint32_t)z[1] << 16, (uint32_t)z[2] | (uint32_t)z[3] << 16);
        }
      }
      fence_async_smem();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(qready);
    // one row tile: the second stream's rows are the first's, written by its warps
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const float sc = a.scale_log2 * s_exp[(dual ? x * kTlRows : 0) + lrow];
    const int mine = dual ? n_tiles : (n_tiles + 1 - x) >> 1;   // tiles of this stream
    // the thread's token and the stream's first, counted from the sequence's first row
    const int tok = (t.r0 + (dual ? x * kTlRows : 0) + lrow) / a.group, tok_lo = (t.r0 + (dual ? x * kTlRows : 0)) / a.group;
    const uint32_t ts = tmem + lane_off + kTlTmS, tp = tmem + lane_off + kTlTmP + x * (kTlKeys / 2);
    const uint32_t to = tmem + lane_off + kTlTmO + x * kTlD;
    float m = -INFINITY, l = 0.f;
    bool far = false;       // the sum of the weights is in 2^(ml - 7)
    float ml = 0.f;
    for (int j = 0; j < mine; ++j) {
      if (!__all_sync(0xffffffffu, tl_wait(&sfull[x], (uint32_t)j & 1u, abort_flag, status))) break;
      tc_fence_after();
      const int tile = dual ? j : 2 * j + x, i = t0 + tile;   // the block's, and of all keys
      float sv[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32_nowait(ts + 32 * c, sv + 32 * c);
      tmem_wait_ld_regs(sv);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sfree[x]);
      bool apart = false;
      uint32_t see[4];   // keys of the tile that the row sees
      {
        const int vst = tile % kT8VStages, seen = t.first - i * kTlKeys;   // keys committed before the step
        // V is there, and with it the words on the keys
        if (!__all_sync(0xffffffffu, tl_wait(&vfull[vst], (uint32_t)(tile / kT8VStages) & 1u, abort_flag, status))) break;
        uint32_t there = ~0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          see[k] = reinterpret_cast<const uint32_t*>(s_valid)[4 * vst + k];
          there &= see[k];
        }
        const bool full = there == ~0u && (a.parent ? seen : seen + tok_lo + 1) >= kTlKeys;   // of the whole stream
        if (!full) {
          const int lead = max(0, min(kTlKeys, a.parent ? seen : seen + tok + 1));
          unsigned long long lo = lead >= 64 ? ~0ull : (1ull << lead) - 1, hi = lead <= 64 ? 0ull : ~0ull >> (128 - lead);
          if (a.parent) {
            unsigned long long x0, x1;
            if (seen >= 0) shl128(anc0, anc1, min(seen, 128), x0, x1);
            else shr128(anc0, anc1, min(-seen, 128), x0, x1);
            lo |= x0;
            hi |= x1;
          }
          see[0] &= (uint32_t)lo;
          see[1] &= (uint32_t)(lo >> 32);
          see[2] &= (uint32_t)hi;
          see[3] &= (uint32_t)(hi >> 32);
#pragma unroll
          for (int k = 0; k < 128; ++k)
            if (!((see[k >> 5] >> (k & 31)) & 1)) sv[k] = -INFINITY;
          apart = (long long)(i + 1) * kTlKeys > t.first && (reinterpret_cast<const uint32_t*>(s_wild)[vst] & 0x01010101u) != 0;
        }
        if (F16 && !far && (reinterpret_cast<const uint32_t*>(s_wild)[vst] & 0x02020202u) != 0) {
          far = true;
          ml = m;
        }
      }
      // a score's factor; not 0: -inf times it stays
      auto scb = [&](int k) { return fminf(fmaxf(sc * s_kpow[8 * (tile % kT8VStages) + k], 0x1p-126f), kMostFactor); };
      // V's exponent, if the weights take it; read where it is used, for want of registers
      auto v_exp = [&](int k) { return F16 ? s_vexp[8 * (tile % kT8VStages) + k] : 0.f; };
      float tmax = -INFINITY;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float mx[2] = {max_nan(sv[16 * k], sv[16 * k + 1]), max_nan(sv[16 * k + 2], sv[16 * k + 3])};
#pragma unroll
        for (int i = 4; i < 16; i += 2) mx[(i >> 1) & 1] = max3_nan(mx[(i >> 1) & 1], sv[16 * k + i], sv[16 * k + i + 1]);
        tmax = max_nan(tmax, fmaf(max_nan(mx[0], mx[1]), scb(k), v_exp(k)));
      }
      const bool move = !(tmax <= m + 8.f);   // a NaN moves it, and stays
      // the tile before has left this P and is in O
      if (j > 0) {
        if (!__all_sync(0xffffffffu, tl_wait(&pvdone[x], (uint32_t)(j - 1) & 1u, abort_flag, status))) break;
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
        if (!F16 || !far) l *= f;
        if (move) m = tmax;
      }
      if (F16 && far) {
        float smax = -INFINITY;
#pragma unroll
        for (int k = 0; k < 128; ++k) smax = max_nan(smax, sv[k] * scb(k >> 4));
        if (!(smax <= ml + 8.f)) {
          l *= ml == -INFINITY ? 0.f : exp2f(ml - smax);
          ml = smax;
        }
        const float by = ml == -INFINITY ? 0.f : kHalfBias - ml;
#pragma unroll
        for (int k = 0; k < 128; ++k) l += ex2_approx(fmaf(sv[k], scb(k >> 4), by));
      }
      // weights 2^(s sc - m); without a finite score yet every score is -inf, and gives 0
      const float neg = m == -INFINITY ? 0.f : (F16 ? kHalfBias : 0.f) - m;
      float2 ps[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, sum = make_float2(0.f, 0.f);
      float l_new = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 2 * h; c < 2 * h + 2; ++c) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float f = scb(2 * c + (i >> 4)), by = neg + v_exp(2 * c + (i >> 4));
            float2 e = fma2(make_float2(sv[32 * c + i], sv[32 * c + i + 1]), make_float2(f, f), make_float2(by, by));
            e = make_float2(ex2_approx(e.x), ex2_approx(e.y));
            if constexpr (F16) {
              const __half2 v = __floats2half2_rn(e.x, e.y);
              pk[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
              sum = (i & 15) == 0 ? e : add2(sum, e);
              if ((i & 15) == 14) l_new = fmaf(sum.x + sum.y, exp2i(-(int)v_exp(2 * c + (i >> 4))), l_new);
            } else {
              const __nv_bfloat162 v = __floats2bfloat162_rn(e.x, e.y);
              pk[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
              add_bf16x2(ps[(i >> 1) & 1], pk[i / 2]);
            }
          }
          tmem_st16u(tp + 16 * c, pk);
        }
        tmem_wait_st();
        if (apart) continue;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pfull[2 * x + h]);
      }
      if (apart) {
        // P.V of the row by its thread, the keys that it sees alone
        const unsigned char* vt = sm + L::kOffV + tile % kT8VStages * kTlTile;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float ov[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) ov[k] = 0.f;
          if (j > 0) {
            tmem_ld32_nowait(to + 32 * c, ov);
            tmem_wait_ld_regs(ov);
          }
#pragma unroll 1
          for (int k = 0; k < kTlKeys; ++k) {
            const uint32_t pw = tmem_ld1(tp + (k >> 1)), half = k & 1 ? pw >> 16 : pw & 0xffffu;
            const float pk = F16 ? __half2float(__ushort_as_half((unsigned short)half)) : bf16_lo(half);
            const uint32_t word = k < 64 ? (k < 32 ? see[0] : see[1]) : (k < 96 ? see[2] : see[3]);
            const bool on = (word >> (k & 31)) & 1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint4 w = *reinterpret_cast<const uint4*>(vt + (c >> 1) * kTlDBlock + sw128(k, (c & 1) * 4 + e));
              const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int f = 0; f < 4; ++f) {
                const float v0 = F16 ? __low2float(*reinterpret_cast<const __half2*>(&ww[f])) : bf16_lo(ww[f]);
                const float v1 = F16 ? __high2float(*reinterpret_cast<const __half2*>(&ww[f])) : bf16_hi(ww[f]);
                ov[8 * e + 2 * f] = on ? fmaf(pk, v0, ov[8 * e + 2 * f]) : ov[8 * e + 2 * f];
                ov[8 * e + 2 * f + 1] = on ? fmaf(pk, v1, ov[8 * e + 2 * f + 1]) : ov[8 * e + 2 * f + 1];
              }
            }
          }
          tmem_st32(to + 32 * c, ov);
          tmem_wait_st();
        }
        s_apart[x] = j + 1;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&pfull[2 * x]);
          mbar_arrive(&pfull[2 * x + 1]);
        }
      }
      if (!F16) l_new = (ps[0].x + ps[0].y) + (ps[1].x + ps[1].y);
      if (!F16 || !far) l += l_new;
    }
    // the ring and TMEM are free once all products are done (the issuer always says so)
    drain_wait(odone, 0);
    tc_fence_after();
    const bool have = mine > 0 && !*abort_flag;
    float unit = 1.f;   // of O, in the sum's
    if (F16 && far) {
      unit = ml == -INFINITY ? 1.f : exp2f(m - ml);
      m = ml;
    }
    float* row = stage + (size_t)(x * kTlRows + lrow) * kPartLd;
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
      float ov[32];
      tmem_ld32_nowait(to + 32 * c, ov);
      tmem_wait_ld_regs(ov);
#pragma unroll
      for (int i = 0; i < 32; i += 4)
        *reinterpret_cast<float4*>(row + 32 * c + i) =
            !have ? make_float4(0.f, 0.f, 0.f, 0.f)
            : F16 ? make_float4(ov[i] * unit, ov[i + 1] * unit, ov[i + 2] * unit, ov[i + 3] * unit)
                  : make_float4(ov[i], ov[i + 2], ov[i + 1], ov[i + 3]);   // V's order
    }
    *reinterpret_cast<float2*>(row + kTlD) = make_float2(have ? (F16 ? m - kHalfBias : m) : -INFINITY, have ? l : 0.f);
    // here the warps have the registers for two parts at once (64 trees over 2048 keys 213 us,
    // one at a time behind all warps' barrier 227)
    if (joined) {
      asm volatile("bar.sync 1, 256;" ::: "memory");
      join_rows<TQ, 2>(a, t, dual, g, stage, kT8Soft0);
    }
  }
  tc_fence_before();
  __syncthreads();   // rows staged
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, kTlTmCols);
  }
  if (!joined) store_part<true>(a, t, dual, split, a.p_splits, g, stage, kT8Soft0);
}

// ---- host
template <typename TQ, int PARTS>
static cudaError_t launch_tiles8(const BatchAttnArgs& a, dim3 grid, cudaStream_t st) {
  // the register split must not ask for more than the block is launched with
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = kernel_ready(ready, (const void*)k_attn_tiles8<TQ>, T8<PARTS>::kSmem, kT8RegsLaunch);
  return e == cudaSuccess ? launch(true, k_attn_tiles8<TQ>, grid, dim3(kT8Threads), T8<PARTS>::kSmem, st, a) : e;
}

cudaError_t launch_sequence8_tc(const BatchAttnArgs& a, const SequencePlan& plan, int dtype, cudaStream_t st) {
  const dim3 grid((unsigned)(plan.tiles * plan.splits * a.pages.nkv));   // rows are many: below 2^31
  return dtype == OOS_DTYPE_BF16 ? launch_tiles8<__nv_bfloat16, 2>(a, grid, st) : launch_tiles8<__half, 3>(a, grid, st);
}

}  // namespace oos
