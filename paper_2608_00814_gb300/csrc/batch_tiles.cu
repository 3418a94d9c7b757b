// Attention of a batch step on tensor cores, 16-bit types with heads of 128, for what
// has many rows:
//   mixed      the rows of all sequences against the prefix's keys, so that each key tile
//              is read once per 256 rows; a part per key range for the kernel of the
//              sequences' own keys (this one, or batch_pages.cu)
//   sequence   the rows of one sequence against its own pages, and against the prefix
//              before them where its rows fill most of a tile: then nothing is left
//              to join
//
// tcgen05, rows (token, head of one kv head's group).  A block has two streams of work, each with its weights P and its O in
// TMEM and four softmax warps of its own, a thread per row:
//   two row tiles   (more than 128 rows left): both streams take every key tile
//   one row tile    the streams take the even and the odd key tiles
// so that one stream's softmax runs under the other's products.  A unit of work is a
// (key tile, stream) pair, taken in turn.
//
// The streams share one score buffer, held only from a product's issue until the threads
// have its row in registers, so that the next unit's scores run under this one's
// exponentials and wait for no P.V; one thread issues the scores, one the P.V products,
// and the tensor cores take them turn by turn.  (1024 rows of 8 heads over 32768 keys, each
// against the kernel of its day: a buffer for each stream with P over it makes a stream's
// scores, weights and P.V follow each other, 159 us against 145; one thread for both kinds,
// a unit's scores before the P.V of the one before, 197.)
//
// P, 16-bit pairs in TMEM, is the A operand of P.V and is handed over in halves of 64
// keys.  A weight is rounded to the type of V, as the product's operands have one type: by
// up to 2^-8 for bf16, as much as out itself is rounded by.  (A second bf16 half would need
// another 128 columns of TMEM, all of which are taken, and half as much product again.)
// The sum l is of the rounded weights, so that what a row's keys share comes out as it is: a
// twentieth of the time (1024 rows of 8 heads over 32768 keys 126 us; 117 with the sum of the
// weights before they are rounded, which is off by up to 2^-8 from those multiplied).
// The running maximum moves only when a tile exceeds it by 2^8 (the threads rescale their O
// rows in TMEM then).
// Keys past the prefix's end arrive as zeros (the tensor map ends there), and so do those
// without a page, so masking their scores is enough.  Pages are gathered by 16-byte
// asynchronous copies into the layout TMA writes, whatever their size; the copying warp
// waits for them and fences before it tells the products.  A tile in which some rows
// see a key and some do not is searched for a v that is not finite, which 0 times it
// would carry to the wrong rows; its P.V is then summed by the threads of the rows.
//
// A block stages its rows over the K/V ring and stores them with one bulk copy, a part
// per key range; the next kernel adds the parts up.  (Ranges joined inside a cluster,
// through distributed shared memory, took 10 us for 256 rows of 11 ranges.)
#include <math.h>
#include <string.h>

#include <algorithm>

#include "batch_tiles.cuh"

namespace oos {

constexpr int kTlKStages = 3, kTlVStages = 2;
constexpr int kTlOffK = 0;
constexpr int kTlOffV = kTlOffK + kTlKStages * kTlTile;
constexpr int kTlOffQ = kTlOffV + kTlVStages * kTlTile;   // two row tiles
constexpr int kTlOffExp = kTlOffQ + 2 * kTlTile;          // row exponents of converted queries
constexpr int kTlOffBar = kTlOffExp + 2 * kTlRows * 4;
constexpr int kTlSmem = kTlOffBar + 320 + 1024;           // + alignment slack
constexpr int kTlThreads = 384;
constexpr int kTlSoft0 = 4;                               // softmax warps 4..7 and 8..11
constexpr int kTlRegsIo = 88, kTlRegsSoft = 208, kTlRegsLaunch = 168;
static_assert(128 * kTlRegsIo + (kTlThreads - 128) * kTlRegsSoft <= kTlThreads * kTlRegsLaunch, "register split");
static_assert(kTlStaged <= kTlOffQ, "staged rows and their weights over the ring");
static_assert(kTlSmem <= 227 * 1024, "shared memory per block");

struct TileArgs {
  CUtensorMap kmap, vmap;   // prefix [prefix_len][nkv][d] as (d, kv head, slot)
  BatchAttnArgs a;
  int pre_tiles;            // key tiles of the prefix that the block takes
  int part0;                // first part of the workspace that the blocks write
};

// SEQ: the rows of one sequence, its own keys behind the prefix's
template <typename TQ, bool F16, bool SEQ>
__global__ void __launch_bounds__(kTlThreads, 1) k_attn_tiles(const __grid_constant__ TileArgs p) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr bool CONVERT = F16 && std::is_same<TQ, __nv_bfloat16>::value;
  constexpr float kBias = F16 ? kHalfBias : 0.f;
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + kTlOffBar);
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
  uint64_t* sets_read = bar + 22;  // eight warps: ancestors in registers
  uint32_t* s_valid = reinterpret_cast<uint32_t*>(bar + 23);   // [V stage][4]: keys that are there
  uint32_t* s_wild = s_valid + 8;                               // [V stage]: a v is not finite
  uint32_t* tmem_slot = s_wild + 2;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* s_apart = abort_flag + 1;                       // [2] the stream's tile whose P.V is done, + 1
  static_assert(23 * 8 + 10 * 4 + 4 * 4 <= 320, "barrier block");
  const BatchAttnArgs& a = p.a;
  int32_t* status = a.status;
  const int S = SEQ ? a.s_splits : a.p_splits, split = blockIdx.x % S, pair = blockIdx.x / S, g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // behind the prefix's kernel, which has waited for what the caller wrote before it
  // triggers, only the end waits for the prefix's parts
  if (SEQ && a.p_splits == 0) pdl_wait();
  if (SEQ) pdl_trigger();
  TileRows t = {};
  if constexpr (SEQ) {
    if (!sequence_tile(a, pair, 2 * kTlRows, &t)) {
      if (blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();   // the grid must not end before the one it follows
      return;
    }
  } else {
    t.r0 = pair * 2 * kTlRows;
    t.rows = min(2 * kTlRows, a.batch.n_tokens * a.group - t.r0);
  }
  const int rows = t.rows;
  const int dual = rows > kTlRows ? 1 : 0;
  int n_own = 0;   // keys of the sequence that some row sees
  if constexpr (SEQ)
    n_own = a.parent ? t.len : max(0, min(t.len, t.first + (t.r0 + rows - 1) / a.group + 1));
  const int n_pre = p.pre_tiles, n_all = n_pre + (n_own + kTlKeys - 1) / kTlKeys;
  const int t0 = (int)((long long)n_all * split / S);
  const int n_tiles = (int)((long long)n_all * (split + 1) / S) - t0;
  const bool joined = SEQ && S == 1 && !a.own_part;   // its rows go into out
  const int units = n_tiles << dual;                  // unit u: tile u >> dual, stream u & 1
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
  if (!SEQ) {   // the kernel before ran under the set-up
    pdl_wait();
    pdl_trigger();
  }
  const uint32_t tmem = *tmem_slot;
  float* stage = reinterpret_cast<float*>(sm);

  if (warp < kTlSoft0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTlRegsIo));
    if (warp == 0 || warp == 3) {
      // ---------------------------------------------------------- loaders: K and V tiles
      const bool v = warp == 3;
      const CUtensorMap* map = v ? &p.vmap : &p.kmap;
      uint64_t* full = v ? vfull : kfull;
      uint64_t* empty = v ? vempty : kempty;
      const int stages = v ? kTlVStages : kTlKStages;
      if (lane == 0 && n_pre > 0) tma_prefetch_desc(map);
      const uint64_t pol = policy_evict_last();   // the other row tiles read it too
      int n = 0, copied = -1;   // copied: a tile of pages on its way
      auto announce = [&]() {
        if (copied < 0) return;
        cp_async_wait<0>();
        fence_async_smem();
        __syncwarp();
        // keys of this step, which some rows may not see: is a v not finite?
        if (v && (t0 + copied - n_pre + 1) * kTlKeys > t.first) {
          constexpr uint32_t kExp = F16 ? 0x7c00u : 0x7f80u;
          uint32_t top = 0;
#pragma unroll 8
          for (int k = 0; k < kTlTile / 512; ++k) {
            const uint4 w = *reinterpret_cast<const uint4*>(sm + kTlOffV + copied % stages * kTlTile + (k * 32 + lane) * 16);
            top = __vmaxu2(top, __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu)));
          }
          const bool wild = __any_sync(0xffffffffu, (top & 0xffffu) >= kExp || (top >> 16) >= kExp);
          if (lane == 0) s_wild[copied % stages] = wild;
        }
        if (lane == 0) mbar_arrive(&full[copied % stages]);
        copied = -1;
      };
      for (; n < n_tiles; ++n) {
        const int st = n % stages, i = t0 + n;
        unsigned char* dst = sm + (v ? kTlOffV : kTlOffK) + st * kTlTile;
        const bool pages = SEQ && i >= n_pre;
        long long slot[4];   // of keys lane + 32 j
        if (pages) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int key = (i - n_pre) * kTlKeys + 32 * j + lane;
            slot[j] = -1;
            if (key < n_own) {
              slot[j] = page_slot(a.batch, a.pages.page_size, a.pages.n_pages, t.seq, key);
              if (slot[j] < 0) *status = OOS_EBATCH;
            }
          }
        }
        announce();
        // the queries of a sequence come first: behind five tiles of keys they took 5 us
        if (SEQ && n == 1 && !__all_sync(0xffffffffu, tl_wait(qready, 0, abort_flag, status))) break;
        // the second V stage holds the tree's sets until they are read
        if (SEQ && a.parent && v && n == 1 && !__all_sync(0xffffffffu, tl_wait(sets_read, 0, abort_flag, status))) break;
        if (n >= stages &&
            !__all_sync(0xffffffffu, tl_wait(&empty[st], (uint32_t)(n / stages - 1) & 1u, abort_flag, status)))
          break;
        if (!pages) {
          if (lane == 0) {
            mbar_arrive_expect_tx(&full[st], kTlTile);
            tma_load_3d(dst, map, &full[st], 0, g, i * kTlKeys, pol);
            tma_load_3d(dst + kTlDBlock, map, &full[st], 64, g, i * kTlKeys, pol);
          }
          continue;
        }
        const uint8_t* src = (v ? a.pages.v : a.pages.k) + (long long)g * (2 * kTlD) + (lane & 15) * 16;
        const long long key_bytes = (long long)a.pages.nkv * (2 * kTlD);
        const uint32_t to = smem_addr(dst) + ((lane & 15) >> 3) * kTlDBlock;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (v) {
            const uint32_t there = __ballot_sync(0xffffffffu, slot[j] >= 0);
            if (lane == 0) s_valid[4 * st + j] = there;
          }
#pragma unroll 4
          for (int k = 0; k < 16; ++k) {   // two keys at a time, 16 lanes each
            const int key = 2 * k + (lane >> 4);
            const long long at = __shfl_sync(0xffffffffu, slot[j], key);
            cp_async16(to + sw128(32 * j + key, lane & 7), src + (at >= 0 ? at * key_bytes : 0), at >= 0);
          }
        }
        cp_async_commit();
        copied = n;
      }
      announce();
      // every copy issued has landed before the block goes on
      if (lane == 0)
        for (int i = n > stages ? n - stages : 0; i < n; ++i) drain_wait(&full[i % stages], (uint32_t)(i / stages) & 1u);
    } else if (warp == 1 && lane == 0) {
      // ---------------------------------------------------------- scores
      constexpr uint32_t idesc = F16 ? idesc_f16_f32(kTlRows, kTlKeys) : idesc_bf16_f32(kTlRows, kTlKeys);
      const uint64_t kdesc = smem_desc_sw128(smem_addr(sm + kTlOffK)), qdesc = smem_desc_sw128(smem_addr(sm + kTlOffQ));
      bool ok = tl_wait(qready, 0, abort_flag, status);
      for (int u = 0; u < units && ok; ++u) {
        const int i = u >> dual, st = i % kTlKStages, x = u & 1;
        if (!dual || x == 0) ok = tl_wait(&kfull[st], (uint32_t)(i / kTlKStages) & 1u, abort_flag, status);
        if (u > 0) ok = ok && tl_wait(&sfree[x ^ 1], (uint32_t)((u - 1) >> 1) & 1u, abort_flag, status);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kTlD / 16; ++k) {
          const uint64_t o = (uint64_t)(((k >> 2) * kTlDBlock) >> 4) + 2 * (k & 3);
          tc_mma_bf16(tmem + kTlTmS, qdesc + o + (uint64_t)(((dual ? x : 0) * kTlTile) >> 4),
                      kdesc + o + (uint64_t)((st * kTlTile) >> 4), idesc, k > 0 ? 1u : 0u);
        }
        tc_commit(&sfull[x]);
        if (!dual || x == 1) tc_commit(&kempty[st]);
      }
      tc_commit(odone);
    } else if (warp == 2 && lane == 0) {
      // ---------------------------------------------------------- P.V
      constexpr uint32_t idesc = (F16 ? idesc_f16_f32(kTlRows, kTlD) : idesc_bf16_f32(kTlRows, kTlD)) | (1u << 16);
      const uint64_t vdesc = smem_desc_sw128_mn(smem_addr(sm + kTlOffV), kTlDBlock);
      bool ok = true;
      for (int u = 0; u < units && ok; ++u) {
        const int i = u >> dual, st = i % kTlVStages, x = u & 1, use = u >> 1;   // use: of this stream
        if (!dual || x == 0) ok = tl_wait(&vfull[st], (uint32_t)(i / kTlVStages) & 1u, abort_flag, status);
        for (int h = 0; h < 2 && ok; ++h) {   // the first half's product runs under the second's exponentials
          ok = tl_wait(&pfull[2 * x + h], (uint32_t)use & 1u, abort_flag, status);
          if (!ok) break;
          tc_fence_after();
          if (SEQ && s_apart[x] == use + 1) continue;   // in O already
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
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTlRegsSoft));
    // ------------------------------------------------------------ softmax: stream x, a thread per row
    const int x = (warp - kTlSoft0) >> 2, q4 = warp & 3;
    const int lrow = q4 * 32 + lane;
    const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
    float* s_exp = reinterpret_cast<float*>(sm + kTlOffExp);
    // queries of the stream's row tile (one row tile: the first stream's warps), two rows
    // of 16 lanes at a time, into the swizzled layout
    const int c = lane & 15;
    uint4 w[16];   // all rows' loads in flight
    if (x == 0 || dual) {
      // one division a thread, its own row's; at two per load the addresses took 3 us
      const int r = x * kTlRows + lrow, row = t.r0 + r;
      const long long mine = (long long)(t.q0 + row / a.group) * a.q_stride + (g * a.group + row % a.group) * kTlD;
      const uint16_t* q0 = (const uint16_t*)a.q + c * 8;
      if ((((uintptr_t)a.q | (uintptr_t)(a.q_stride * 2)) & 15) == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int from = 2 * i + (lane >> 4);
          const uint16_t* q = q0 + __shfl_sync(0xffffffffu, mine, from);
          w[i] = make_uint4(0, 0, 0, 0);
          if (x * kTlRows + q4 * 32 + from < rows) w[i] = *reinterpret_cast<const uint4*>(q);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int from = 2 * i + (lane >> 4);
          const uint16_t* q = q0 + __shfl_sync(0xffffffffu, mine, from);
          w[i] = make_uint4(0, 0, 0, 0);
          if (x * kTlRows + q4 * 32 + from < rows)
            w[i] = make_uint4((uint32_t)q[0] | (uint32_t)q[1] << 16, (uint32_t)q[2] | (uint32_t)q[3] << 16,
                              (uint32_t)q[4] | (uint32_t)q[5] << 16, (uint32_t)q[6] | (uint32_t)q[7] << 16);
        }
      }
    }
    // ancestors of the thread's row, while the queries are on their way
    unsigned long long anc0 = 0, anc1 = 0;
    if (SEQ && a.parent) {
      const unsigned long long (*sets)[2] =
          tree_sets(a, t.q0, t.n, reinterpret_cast<TreeScratch*>(sm + kTlOffV + kTlTile), threadIdx.x - 32 * kTlSoft0,
                    32 * 8, [] { asm volatile("bar.sync 1, 256;" ::: "memory"); });
      const int r = (dual ? x * kTlRows : 0) + lrow;
      if (r < rows) {
        anc0 = sets[(t.r0 + r) / a.group][0];
        anc1 = sets[(t.r0 + r) / a.group][1];
      }
      fence_async_smem();   // the loader's copies follow
      __syncwarp();
      if (lane == 0) mbar_arrive(sets_read);
    }
    if (x == 0 || dual) {
      unsigned char* qs = sm + kTlOffQ + x * kTlTile;
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
          if (c == 0) s_exp[x * kTlRows + r] = exp2i(e2);
        }
        *reinterpret_cast<uint4*>(qs + (c >> 3) * kTlDBlock + sw128(r, c & 7)) = w[i];
      }
      fence_async_smem();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(qready);
    float sc = a.scale_log2;
    if constexpr (CONVERT) {
      // one row tile: the second stream's rows are the first's, written by its warps
      asm volatile("bar.sync 1, 256;" ::: "memory");
      sc *= s_exp[(dual ? x : 0) * kTlRows + lrow];
    }
    const int mine = dual ? n_tiles : (n_tiles + 1 - x) >> 1;   // tiles of this stream
    // the thread's token and the stream's first, counted from the sequence's first row
    const int tok = (t.r0 + (dual ? x * kTlRows : 0) + lrow) / a.group, tok_lo = (t.r0 + (dual ? x * kTlRows : 0)) / a.group;
    const uint32_t ts = tmem + lane_off + kTlTmS, tp = tmem + lane_off + kTlTmP + x * (kTlKeys / 2);
    const uint32_t to = tmem + lane_off + kTlTmO + x * kTlD;
    float m = -INFINITY, l = 0.f;
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
      uint32_t see[4] = {~0u, ~0u, ~0u, ~0u};   // keys of the tile that the row sees
      if (!SEQ || i < n_pre) {
        const int n_ok = a.prefix_len - i * kTlKeys;
        if (n_ok < kTlKeys) {
#pragma unroll
          for (int k = 0; k < 128; ++k)
            if (k >= n_ok) sv[k] = -INFINITY;
        }
      } else {
        const int vst = tile % kTlVStages, seen = t.first - (i - n_pre) * kTlKeys;   // keys committed before the step
        // V has landed, and with it the word on which keys are there
        if (!__all_sync(0xffffffffu, tl_wait(&vfull[vst], (uint32_t)(tile / kTlVStages) & 1u, abort_flag, status))) break;
        uint32_t there = ~0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          see[k] = s_valid[4 * vst + k];
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
          apart = (i - n_pre + 1) * kTlKeys > t.first && s_wild[vst] != 0;
        }
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < 128; i += 2) mx[(i >> 1) & 3] = max3_nan(mx[(i >> 1) & 3], sv[i], sv[i + 1]);
      const float tmax = max_nan(max_nan(mx[0], mx[1]), max_nan(mx[2], mx[3])) * sc - kBias;
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
            if constexpr (F16) {
              const __half2 v = __floats2half2_rn(e.x, e.y);
              pk[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
              ps[(i >> 1) & 1] = add2(ps[(i >> 1) & 1], __half22float2(v));
            } else {
              const __nv_bfloat162 v = __floats2bfloat162_rn(e.x, e.y);
              pk[i / 2] = *reinterpret_cast<const uint32_t*>(&v);
              add_bf16x2(ps[(i >> 1) & 1], pk[i / 2]);
            }
          }
          tmem_st16u(tp + 16 * c, pk);
        }
        tmem_wait_st();
        if (SEQ && apart) continue;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pfull[2 * x + h]);
      }
      if (SEQ && apart) {
        // P.V of the row by its thread, the keys that it sees alone
        const unsigned char* vt = sm + kTlOffV + tile % kTlVStages * kTlTile;
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
      l += (ps[0].x + ps[0].y) + (ps[1].x + ps[1].y);
    }
    // the ring and TMEM are free once all products are done (the issuer always says so)
    drain_wait(odone, 0);
    tc_fence_after();
    const bool have = mine > 0 && !*abort_flag;
    float* row = stage + (size_t)(x * kTlRows + lrow) * kPartLd;
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
    *reinterpret_cast<float2*>(row + kTlD) = make_float2(have ? m : -INFINITY, have ? l : 0.f);
  }
  tc_fence_before();
  __syncthreads();   // rows staged
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, kTlTmCols);
  }
  if (!joined) {
    store_part<SEQ>(a, t, dual, split, p.part0, g, stage, kTlSoft0);
  } else if constexpr (SEQ) {
    if (warp >= kTlSoft0) join_rows<TQ, 1>(a, t, dual, g, stage, kTlSoft0);
  }
}

// ---- host
template <typename TQ, bool F16, bool SEQ>
static cudaError_t launch_tiles(const TileArgs& p, dim3 grid, cudaStream_t st) {
  // the register split must not ask for more than the block is launched with
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = kernel_ready(ready, (const void*)k_attn_tiles<TQ, F16, SEQ>, kTlSmem, kTlRegsLaunch);
  return e == cudaSuccess ? launch(true, k_attn_tiles<TQ, F16, SEQ>, grid, dim3(kTlThreads), kTlSmem, st, p) : e;
}

// us: a row tile's work on a key tile, and a block's beginning and end (with pages: the
// lookups, the masks and the output besides).  A tile's is 0.90 with two row tiles over a
// long prefix; cut by that number, the cases timed are the same but for 128 trees of 15
// nodes on average over 2000 keys, 216 us instead of 150.
constexpr double kTlTileUs = 0.83, kTlBlockUs = 8.0, kTlSeqBlockUs = 12.0;
static double waves(long long blocks, int n_sms) { return (double)((blocks + n_sms - 1) / n_sms); }   // one block per SM

// The count of key ranges with the shortest schedule: waves, each of a block's tiles and
// its beginning and end, and the parts, written and read once at about 8 bytes per ps, or
// 3 where the pages' kernel of few rows reads them (64 sequences of one token, 32 heads
// over 8192 keys: 11 ranges 50 us with the pages', 16 by 8 bytes per ps 53).  Where that
// kernel's blocks, own_sms full of them, then fit beside these, and these are not estimated
// a quarter longer for it, fewer: the two run at once (8 sequences: 8 ranges 20 us, 10 or
// 16 26).
PrefixPlan plan_prefix_tc(long long rows, int nkv, int prefix_len, int own_sms, int n_sms) {
  PrefixPlan p;
  p.pairs = (int)((rows + 2 * kTlRows - 1) / (2 * kTlRows));
  p.splits = 1;
  const int tiles = (prefix_len + kTlKeys - 1) / kTlKeys;
  const double tile = (rows > kTlRows ? 2 : 1) * kTlTileUs, part = 2.0 * rows * nkv * kPartLd * 4 / (own_sms > 0 ? 3e6 : 8e6);
  auto us = [&](int s) {
    return waves((long long)p.pairs * nkv * s, n_sms) * (tile * ((tiles + s - 1) / s) + kTlBlockUs) + part * s;
  };
  for (int s = 2; s <= kTlMaxSplits && s <= tiles; ++s)
    if (us(s) < us(p.splits)) p.splits = s;
  const int beside = (int)std::min<long long>(kTlMaxSplits, (n_sms - own_sms) / ((long long)p.pairs * nkv));
  if (own_sms > 0 && beside >= 1 && beside < p.splits && us(beside) <= 1.25 * us(p.splits)) p.splits = beside;
  p.us = us(p.splits);
  return p;
}

// Sequences of many rows.  They take the prefix along where that is estimated shorter than
// a kernel for it and its parts.  The lengths are on the device: two tiles of own keys are
// assumed (4 prompts of up to 200 tokens, 1000 prefix and up to 6000 own keys: 116 us, with
// one tile 189; one tree, 2048 and up to 8000 keys: 41, with six tiles 38), and for ranges of
// own keys alone no more than eight (one tree over up to 8000 keys: 42 us, with four 52, with
// sixteen 37).  The table may be wider than its sequences need: with eight times the columns
// 16 trees over 2048 + up to 400 keys take 57 us (58 otherwise) and 13 prompts the same 275.
SequencePlan plan_sequence_tc(long long rows, int n_seqs, int nkv, int prefix_len, long long most_keys, int n_sms) {
  SequencePlan p = {};
  p.tiles = (int)(n_seqs + rows / (2 * kTlRows));   // numbers; tiles that have rows, about:
  const long long live = (long long)n_seqs * ((rows + 2ll * kTlRows * n_seqs - 1) / (2ll * kTlRows * n_seqs));
  const int pre = (prefix_len + kTlKeys - 1) / kTlKeys;
  const double tile = (rows > (long long)kTlRows * n_seqs ? 2 : 1) * kTlTileUs;
  const long long own = (most_keys + kTlKeys - 1) / kTlKeys;   // at most
  // the shortest schedule of `tiles` key tiles, and the splits it takes
  auto schedule = [&](double tiles, long long most, double extra, int* splits) {
    double best = 0;
    for (int s = 1; s <= kTlMaxSplits && s <= std::max(1ll, most / 2); ++s) {
      const double us = waves(live * nkv * s, n_sms) * (tile * tiles / s + kTlSeqBlockUs + extra) +
                        (s > 1 ? 4.0 + s * 2.0 * rows * nkv * kPartLd * 4 / 8e6 : 0.0);
      if (s > 1 && us >= best) continue;
      best = us;
      *splits = s;
    }
    return best;
  };
  int split_with = 1, split_own = 1;
  const double with_prefix = schedule(pre + 2.0, pre + own, 0.0, &split_with);
  p.takes_prefix = false;
  if (pre > 0) {
    const PrefixPlan apart = plan_prefix_tc(rows, nkv, prefix_len, 0, n_sms);
    p.takes_prefix = with_prefix <= apart.us + schedule(2.0, own, 2.0 * apart.splits, &split_own);
  }
  if (!p.takes_prefix) schedule((double)std::min(own, 8ll), own, 0.0, &split_own);
  p.splits = p.takes_prefix ? split_with : split_own;
  return p;
}

static bool encode_prefix(const BatchAttnArgs& a, bool f16, TileArgs* p) {
  const uint64_t dims[3] = {(uint64_t)kTlD, (uint64_t)a.pages.nkv, (uint64_t)a.prefix_len};
  const uint64_t strides[2] = {(uint64_t)kTlD * 2, (uint64_t)a.pages.nkv * kTlD * 2};
  const uint32_t box[3] = {64, 1, (uint32_t)kTlKeys};
  p->pre_tiles = (a.prefix_len + kTlKeys - 1) / kTlKeys;
  return encode_bf16_map(&p->kmap, a.pk, 3, dims, strides, box, f16) && encode_bf16_map(&p->vmap, a.pv, 3, dims, strides, box, f16);
}

cudaError_t launch_prefix_tc(const BatchAttnArgs& a, const PrefixPlan& plan, int dtype, int kv_dtype, cudaStream_t st) {
  TileArgs p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  const bool f16 = kv_dtype == OOS_DTYPE_F16;
  if (!encode_prefix(a, f16, &p)) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)(plan.pairs * plan.splits), a.pages.nkv);
  if (!f16) return launch_tiles<__nv_bfloat16, false, false>(p, grid, st);
  if (dtype == OOS_DTYPE_BF16) return launch_tiles<__nv_bfloat16, true, false>(p, grid, st);
  return launch_tiles<__half, true, false>(p, grid, st);
}

cudaError_t launch_sequence_tc(const BatchAttnArgs& a, const SequencePlan& plan, int dtype, int kv_dtype, cudaStream_t st) {
  TileArgs p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  p.part0 = a.p_splits;
  const bool f16 = kv_dtype == OOS_DTYPE_F16;
  if (a.prefix_len > 0 && plan.takes_prefix && !encode_prefix(a, f16, &p)) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)(plan.tiles * plan.splits), a.pages.nkv);
  if (!f16) return launch_tiles<__nv_bfloat16, false, true>(p, grid, st);
  if (dtype == OOS_DTYPE_BF16) return launch_tiles<__nv_bfloat16, true, true>(p, grid, st);
  return launch_tiles<__half, true, true>(p, grid, st);
}

}  // namespace oos
