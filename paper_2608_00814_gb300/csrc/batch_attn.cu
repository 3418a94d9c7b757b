// Attention of a batch step over a shared prefix and each sequence's pages.
//
// Row (token i, q head h) of sequence b sees the prefix's keys and, of its own
// sequence, the positions up to its own (or, with a tree, the committed ones and
// its ancestors).  The keys fall into parts -- ranges of the prefix, ranges of the
// sequence's positions -- and each part leaves an unnormalised row
//   O = sum 2^(s - m) v,  m = max s,  l = sum 2^(s - m),  s = scale log2(e) q.k
// in the workspace; a last kernel joins a row's parts.  In the prefix's parts the
// rows of all sequences stand in one tile, so that its keys are read once for
// all; in the sequence's parts a tile holds rows of one sequence.
//
// k_attn_rows: CUDA cores, fp32 products, for every type and head size.  The 16-bit
// types with heads of 128 take the tensor-core kernels of batch_tiles.cu and
// batch_pages.cu.
#include <math.h>

#include <algorithm>

#include "batch_attn.cuh"

namespace oos {

constexpr int kRowKeys = 32;       // keys per tile
constexpr int kRowThreads = 128;
constexpr int kMaxParts = 32;      // parts of a row (a lane each in the join)

// RT rows x 32 keys per step, 128 threads: thread (r, c) of 16 x 8 (of 4 x 32 with 4 rows)
// has RT / 16 rows (one) and keys c, c + 8, c + 16, c + 24 (c) of S, and four columns in
// 32 (in 128) of O.  The threads of a row share its statistics by shuffles.
//
// Bound by latency: lookups, loads, products, statistics and products of a tile follow each
// other (40 sequences of up to 3 rows, 6 heads of 128, 900 + up to 300 keys, 16-row tiles:
// 82 us, issue slots 39 % used, shared memory 40 %).  So a tile's places are looked up under
// the tile before, the keys are dealt to as many blocks as help, and sequences of few rows
// have tiles of 4 or 8, more of whose blocks fit on an SM (the same: 61 us).
template <typename TQ, typename TK, int RT, int VEC>
__global__ void __launch_bounds__(kRowThreads, RT == 64 ? 3 : RT == 16 ? 4 : 6) k_attn_rows(const BatchAttnArgs a) {
  extern __shared__ __align__(16) float sm[];
  constexpr int GROUPS = RT < 16 ? RT : 16, RPT = RT / GROUPS, TPR = kRowThreads / GROUPS;   // TPR: threads of a row
  constexpr int KPT = kRowKeys / TPR, CPT = kMaxHeadDim / (4 * TPR);                         // keys, column quads of a thread
  const int d = a.pages.d, ld = ((d + 3) & ~3) + 4, tid = threadIdx.x;
  float* s_q = sm;                          // [RT][ld]
  float* s_k = s_q + RT * ld;               // [32][ld]
  float* s_v = s_k + kRowKeys * ld;
  float* s_p = s_v + kRowKeys * ld;         // [RT][36]
  constexpr int ldp = kRowKeys + 4;
  __shared__ TreeScratch s_tree;
  __shared__ long long s_at[2][kRowKeys];   // slot of each key in its buffer, -1: none; of two tiles in turn

  // behind the prefix's launch, which has waited for what the caller wrote before it
  // triggers, only the end waits
  if (!a.own_part) pdl_wait();
  pdl_trigger();
  const int g = blockIdx.y;
  const bool prefix = (int)blockIdx.x < a.p_tiles * a.p_splits;
  const int local = prefix ? blockIdx.x : blockIdx.x - a.p_tiles * a.p_splits;
  const int tile = prefix ? local / a.p_splits : local / a.s_splits;
  const int split = prefix ? local % a.p_splits : local % a.s_splits;
  const int splits = prefix ? a.p_splits : a.s_splits;
  TileRows t;
  if (prefix) {
    t.seq = -1;
    t.q0 = 0;
    t.r0 = tile * RT;
    t.rows = min(RT, a.batch.n_tokens * a.group - t.r0);
    t.first = t.len = a.prefix_len;
  } else if (!sequence_tile(a, tile, RT, &t)) {
    if (a.own_part && blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();   // the join counts on the prefix's launch, too
    return;
  }
  const unsigned long long (*anc)[2] = nullptr;
  if (!prefix && a.parent) anc = tree_sets(a, t.q0, t.n, &s_tree);
  // the keys any row of the tile sees, dealt to the splits in whole tiles
  const int last = (t.r0 + t.rows - 1) / a.group;   // its last token, counted from q0
  const int n_keys = prefix || anc ? t.len : max(0, min(t.len, t.first + last + 1));
  const int n_tiles = (n_keys + kRowKeys - 1) / kRowKeys;
  const int k0 = (int)((long long)n_tiles * split / splits) * kRowKeys;
  const int k1 = min(n_keys, (int)((long long)n_tiles * (split + 1) / splits) * kRowKeys);

  for (int i = tid; i < RT * (ld - 4); i += kRowThreads) {
    const int r = i / (ld - 4), c = i % (ld - 4);
    float v = 0.f;
    if (r < t.rows && c < d) {
      const int row = t.r0 + r;
      v = to_f32(((const TQ*)a.q)[(long long)(t.q0 + row / a.group) * a.q_stride + (g * a.group + row % a.group) * d + c]);
    }
    s_q[r * ld + c] = v;
  }
  const int tr = tid / TPR, tc = tid % TPR;
  float o[RPT][CPT][4], m[RPT], l[RPT];
#pragma unroll
  for (int r = 0; r < RPT; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < CPT; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[r][c][e] = 0.f;
  }
  const long long heads_d = (long long)a.pages.nkv * d;
  auto look_up = [&](int key0) {   // the places of a tile's keys, while the tile before is worked on
    if (tid >= kRowKeys) return;
    const int key = key0 + tid;
    long long at = -1;
    if (key < k1) {
      at = prefix ? key : page_slot(a.batch, a.pages.page_size, a.pages.n_pages, t.seq, key);
      if (at < 0) *a.status = OOS_EBATCH;
    }
    s_at[(key0 - k0) / kRowKeys & 1][tid] = at;
  };
  look_up(k0);
  for (int key0 = k0; key0 < k1; key0 += kRowKeys) {
    __syncthreads();   // the tile before is read, this one's places are known
    const long long* at_of = s_at[(key0 - k0) / kRowKeys & 1];
    const TK* kb = (const TK*)(prefix ? a.pk : a.pages.k);
    const TK* vb = (const TK*)(prefix ? a.pv : a.pages.v);
    const int chunks = (ld - 4) / VEC;
    for (int i = tid; i < kRowKeys * chunks; i += kRowThreads) {
      const int key = i / chunks, c = (i % chunks) * VEC;
      float kv[VEC], vv[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) kv[e] = vv[e] = 0.f;   // keys that are not there must not reach a sum
      if (at_of[key] >= 0 && c < d) {
        const long long off = at_of[key] * heads_d + (long long)g * d + c;
        load_vec<TK, VEC>(kb + off, kv);
        load_vec<TK, VEC>(vb + off, vv);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        s_k[key * ld + c + e] = kv[e];
        s_v[key * ld + c + e] = vv[e];
      }
    }
    look_up(key0 + kRowKeys);
    __syncthreads();
    float s[RPT][KPT];
    bool see[RPT][KPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r)
#pragma unroll
      for (int j = 0; j < KPT; ++j) s[r][j] = 0.f;
    for (int c = 0; c < ld - 4; c += 4) {
      float4 kk[KPT];
#pragma unroll
      for (int j = 0; j < KPT; ++j) kk[j] = *reinterpret_cast<const float4*>(s_k + (tc + TPR * j) * ld + c);
#pragma unroll
      for (int r = 0; r < RPT; ++r) {
        const float4 qq = *reinterpret_cast<const float4*>(s_q + (tr * RPT + r) * ld + c);
#pragma unroll
        for (int j = 0; j < KPT; ++j)
          s[r][j] += qq.x * kk[j].x + qq.y * kk[j].y + qq.z * kk[j].z + qq.w * kk[j].w;
      }
    }
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
      const int token = (t.r0 + tr * RPT + r) / a.group;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < KPT; ++j) {
        const int key = key0 + tc + TPR * j, own = key - t.first;
        bool ok = at_of[tc + TPR * j] >= 0;
        if (!prefix && own >= 0)
          ok = ok && (anc ? token < t.n && own < kMaxTreeRows && ((anc[token][own >> 6] >> (own & 63)) & 1) : own <= token);
        see[r][j] = ok;
        s[r][j] = ok ? s[r][j] * a.scale_log2 : -INFINITY;
        mx = max_nan(mx, s[r][j]);
      }
#pragma unroll
      for (int x = 1; x < TPR; x *= 2) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, x));
      const float mn = max_nan(m[r], mx);
      const bool live = mn != -INFINITY;
      const float f = m[r] == -INFINITY ? 0.f : exp2f(m[r] - mn);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < KPT; ++j) {
        const float p = live ? exp2f(s[r][j] - mn) : 0.f;
        sum += p;
        s_p[(tr * RPT + r) * ldp + tc + TPR * j] = see[r][j] ? p : -1.f;   // negative: not seen
      }
#pragma unroll
      for (int x = 1; x < TPR; x *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      l[r] = l[r] * f + sum;
      m[r] = mn;
#pragma unroll
      for (int c = 0; c < CPT; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[r][c][e] *= f;
    }
    __syncwarp();   // a row's weights are written and read by the same lanes
#pragma unroll 8
    for (int key = 0; key < kRowKeys; ++key) {
      float p[RPT];
#pragma unroll
      for (int r = 0; r < RPT; ++r) p[r] = s_p[(tr * RPT + r) * ldp + key];
#pragma unroll
      for (int c = 0; c < CPT; ++c) {
        const int col = tc * 4 + 4 * TPR * c;
        if (col >= d) continue;
        const float4 v = *reinterpret_cast<const float4*>(s_v + key * ld + col);
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
          if (p[r] < 0.f) continue;   // whatever its v is
          o[r][c][0] += p[r] * v.x;
          o[r][c][1] += p[r] * v.y;
          o[r][c][2] += p[r] * v.z;
          o[r][c][3] += p[r] * v.w;
        }
      }
    }
    __syncwarp();
  }
  const int part = prefix ? split : a.p_splits + split;
  const long long n_rows = (long long)a.batch.n_tokens * a.nq;
#pragma unroll
  for (int r = 0; r < RPT; ++r) {
    const int lr = tr * RPT + r;
    if (lr >= t.rows) continue;
    const int row = t.r0 + lr;
    const long long at = part * n_rows + (long long)(t.q0 + row / a.group) * a.nq + g * a.group + row % a.group;
    if (tc == 0) a.part_ml[at] = make_float2(m[r], l[r]);
#pragma unroll
    for (int c = 0; c < CPT; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int col = tc * 4 + 4 * TPR * c + e;
        if (col < d) a.part_o[at * d + col] = o[r][c][e];
      }
  }
  if (a.own_part && blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();
}

// A warp per row adds its parts up: weights 2^(m - max m), the sum divided by the
// weighted l.  Parts are taken in order, so the result does not depend on timing.
template <typename T>
__global__ void __launch_bounds__(128) k_attn_join(const BatchAttnArgs a) {
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, d = a.pages.d;
  const long long n_rows = (long long)a.batch.n_tokens * a.nq;
  pdl_wait();
  pdl_trigger();
  if (row >= n_rows) return;
  const long long token = row / a.nq;
  if (token >= a.batch.q_start[a.batch.n_seqs] || token < a.batch.q_start[0]) return;   // padding
  const int parts = a.p_splits + a.s_splits;
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < parts) ml = a.part_ml[lane * n_rows + row];
  constexpr int U = 8;   // parts on their way at once
  float v[U][4];
  auto fetch = [&](int p0) {
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (p0 + i < parts && lane + 32 * c < d) v[i][c] = a.part_o[((p0 + i) * n_rows + row) * d + lane + 32 * c];
  };
  fetch(0);
  const float M = warp_max(ml.x);
  const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
  const float den = warp_sum(ml.x == -INFINITY ? 0.f : w * ml.y);
  T* out = (T*)a.out + token * a.out_stride + (row - token * a.nq) * d;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < parts; p0 += U) {
    if (p0 > 0) fetch(p0);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float wp = __shfl_sync(0xffffffffu, w, (p0 + i) & 31);
      if (p0 + i >= parts || wp == 0.f) continue;   // a part without keys leaves its row unwritten
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] += wp * v[i][c];
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (lane + 32 * c < d) out[lane + 32 * c] = from_f32<T>(den == 0.f ? 0.f : acc[c] / den);
}

// The same for the parts of the tensor-core kernels: rows by kv head, heads of 128
template <typename T>
__global__ void __launch_bounds__(256) k_attn_join_parts(const __grid_constant__ BatchAttnArgs a) {
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;   // of [kv head][token * group + head]
  pdl_wait();
  pdl_trigger();
  const int rows = a.batch.n_tokens * a.group;
  if (row >= rows * a.pages.nkv) return;
  const int g = row / rows, r = row - g * rows, token = r / a.group;
  if (token >= a.batch.q_start[a.batch.n_seqs] || token < a.batch.q_start[0]) return;   // padding
  const long long step = (long long)a.pages.nkv * rows * kPartLd;
  const float* p = a.part_o + (long long)row * kPartLd;
  const int parts = a.p_splits + a.s_splits;   // <= 32, a lane each
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < parts) ml = *reinterpret_cast<const float2*>(p + lane * step + 128);
  constexpr int U = 8;   // parts on their way at once
  float4 v[U];
  auto fetch = [&](int p0) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (p0 + i < parts) v[i] = *reinterpret_cast<const float4*>(p + (p0 + i) * step + 4 * lane);
  };
  fetch(0);
  const bool on = ml.x != -INFINITY;   // a NaN is, and reaches the sum
  const float top = warp_max(ml.x);
  const float w = on ? exp2f(ml.x - top) : 0.f;
  const float den = warp_sum(on ? w * ml.y : 0.f);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int p0 = 0; p0 < parts; p0 += U) {
    if (p0 > 0) fetch(p0);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float wi = __shfl_sync(0xffffffffu, w, (p0 + i) & 31);
      if (p0 + i >= parts || wi == 0.f) continue;   // a part without weight counts for nothing, whatever it holds
      acc.x += wi * v[i].x;
      acc.y += wi * v[i].y;
      acc.z += wi * v[i].z;
      acc.w += wi * v[i].w;
    }
  }
  store_row<T>(a, g, 0, r, weighted_mean(acc, den));
}

// ---- host: how a call is cut up
struct BatchAttnPlan {
  bool tc;             // tensor cores: 16-bit types with heads of 128
  bool few;            // .. with few rows per sequence
  PrefixPlan prefix;
  PagesPlan pages;
  SequencePlan sequence;
  int p_rt, rt, p_tiles, p_splits, s_tiles, s_splits;   // CUDA cores: rows of a tile over the prefix, over own keys
  size_t ml_off, bytes;
};

int device_sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return n;
}

cudaError_t kernel_ready(std::atomic<uint64_t>& ready, const void* kernel, int smem, int regs) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (ready.load(std::memory_order_acquire) & bit) return cudaSuccess;
  if (regs) e = check_launch_regs(kernel, regs);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_release);
  return e;
}

static bool plan_batch_attn(int nq, int prefix_len, const oos_paged_cache& c, const oos_batch& b, BatchAttnPlan* p) {
  const int sms = device_sms();
  if (sms <= 0) return false;
  const int G = nq / c.n_kv_heads;
  const long long rows = (long long)b.n_tokens * G;
  const long long most_keys = std::min<long long>((long long)b.max_pages * c.page_size, kMaxKeys);
  p->tc = c.dtype != OOS_DTYPE_F32 && c.head_dim == 128;
  if (p->tc) {
    // Tiles of 16 rows that read their sequence's pages again (from L2), or tiles of up to
    // 256 that are mostly empty.  Trees of 4 rows a node, 8 kv heads, 2048 prefix keys: 24
    // rows on average 67 us against 102 (64 sequences), 30 against 39 (16); 48 rows 42
    // against 40 (16 sequences; over 8192 keys 95 against 106), 16 against 25 (2), but 100
    // against 94 (64); 96 rows 28 against 27 (4).
    p->few = rows <= 32ll * b.n_seqs || (rows <= 64ll * b.n_seqs && rows / 16 * c.n_kv_heads <= 4ll * sms);
    p->sequence = {false, 0, 1};
    if (p->few) p->pages = plan_pages_tc(rows, b.n_seqs, c.n_kv_heads, most_keys, sms);
    else p->sequence = plan_sequence_tc(rows, b.n_seqs, c.n_kv_heads, prefix_len, most_keys, sms);
    p->prefix = prefix_len > 0 && !p->sequence.takes_prefix ? plan_prefix_tc(rows, c.n_kv_heads, prefix_len, p->few ? p->pages.sms : 0, sms)
                                                            : PrefixPlan{0, 0, 0.0};
    // Blocks of few rows that join with the prefix's parts hold their place until those
    // are there.  Where the prefix's last wave leaves SMs free for long -- as much as the
    // chip does in 9 us -- they leave a part of their own and go on, for one more kernel.
    // 256 sequences, 32768 prefix keys (20 us): 137 us against 148; 64 trees of 6 nodes, 2048
    // keys: 67 against 73; 200 sequences of 64 heads, 16000 keys (9.6): 127 against 135; but
    // 64 of 40 heads, 3000 keys (7.4): 56 against 55, 40 over 30000 keys (6.3): 54 against 49.
    if (p->few && p->prefix.splits > 0) {
      const long long blocks = (long long)p->prefix.pairs * c.n_kv_heads * p->prefix.splits, waves = (blocks + sms - 1) / sms;
      const long long left = waves * sms - blocks;   // SMs, in the last wave
      p->pages.part = p->pages.sms > left && p->prefix.us * (double)left / (double)(waves * sms) > 9.0;
    }
    const int parts = p->prefix.splits + (p->few ? (int)p->pages.part : p->sequence.splits > 1 ? p->sequence.splits : 0);
    p->ml_off = 0;
    p->bytes = ((size_t)parts * b.n_tokens * nq * kPartLd * 4 + 255) / 256 * 256;
    return true;
  }
  // One request of 1 token, 9 heads, 2000 keys: 22.8 us with 4 rows, 22.6 with 16; 30 of up to
  // 2 tokens, 9 heads: 42 and 63; 50 of 1 token, 8 heads on one: 46 with 8 rows, 47 with 16.
  p->rt = rows <= 4ll * b.n_seqs ? 4 : rows <= 8ll * b.n_seqs ? 8 : rows <= 16ll * b.n_seqs ? 16 : 64;
  // The prefix's tiles hold rows of all sequences: 16 where there are many, in a launch of
  // their own, which few rows do not pay for (10 rows over a few keys 11 us a call against
  // 13.8; 8 rows over 1500: 21 against 28).
  p->p_rt = rows > 8ll * p->rt ? std::max(p->rt, 16) : p->rt;
  p->p_tiles = prefix_len > 0 ? (int)((rows + p->p_rt - 1) / p->p_rt) : 0;
  p->s_tiles = (int)(b.n_seqs + rows / p->rt);
  // Enough blocks for four per SM, or twelve small ones (84 sequences of 3 rows over 580 keys
  // on average: 64 us; with 8: 78, with 4 of 16 rows 152), each with a tile of keys at least
  // (a tile is a chain of some 4 us: one request of 1 token over 130 keys 10.8 us, with two
  // tiles a block 17.9).
  auto splits = [&](long long tiles, int rt, long long keys) {
    const long long want = (rt < 16 ? 12ll : 4ll) * sms / std::max(1ll, tiles * c.n_kv_heads);
    return (int)std::max(1ll, std::min({want, keys / kRowKeys, (long long)kMaxParts / 2}));
  };
  p->p_splits = prefix_len > 0 ? splits(p->p_tiles, p->p_rt, prefix_len) : 0;
  // tiles that have rows, about
  const long long live = std::max((long long)b.n_seqs, (rows + p->rt - 1) / p->rt);
  p->s_splits = splits(live, p->rt, most_keys);
  const size_t n = (size_t)(p->p_splits + p->s_splits) * b.n_tokens * nq;
  p->ml_off = (n * c.head_dim * 4 + 255) / 256 * 256;
  p->bytes = p->ml_off + (n * 8 + 255) / 256 * 256;
  return true;
}

template <typename TQ, typename TK, int RT, int VEC>
static cudaError_t launch_rows_of(const BatchAttnArgs& a, cudaStream_t st) {
  const int ld = ((a.pages.d + 3) & ~3) + 4;
  auto smem_of = [](int ld_) { return ((RT + 2 * kRowKeys) * ld_ + RT * (kRowKeys + 4)) * 4; };
  const size_t smem = smem_of(ld);
  static std::atomic<uint64_t> ready{0};
  cudaError_t e = kernel_ready(ready, (const void*)k_attn_rows<TQ, TK, RT, VEC>, smem_of(kMaxHeadDim + 4));
  if (e != cudaSuccess) return e;
  const int blocks = a.p_tiles * a.p_splits + a.s_tiles * a.s_splits;
  return launch(true, k_attn_rows<TQ, TK, RT, VEC>, dim3(blocks, a.pages.nkv), dim3(kRowThreads), smem, st, a);
}

template <typename TQ, typename TK>
static cudaError_t launch_rows(const BatchAttnArgs& a, int rt, bool vec, cudaStream_t st) {
  if (rt == 4) return vec ? launch_rows_of<TQ, TK, 4, 4>(a, st) : launch_rows_of<TQ, TK, 4, 1>(a, st);
  if (rt == 8) return vec ? launch_rows_of<TQ, TK, 8, 4>(a, st) : launch_rows_of<TQ, TK, 8, 1>(a, st);
  if (rt == 16) return vec ? launch_rows_of<TQ, TK, 16, 4>(a, st) : launch_rows_of<TQ, TK, 16, 1>(a, st);
  return vec ? launch_rows_of<TQ, TK, 64, 4>(a, st) : launch_rows_of<TQ, TK, 64, 1>(a, st);
}

template <typename TQ, typename TK>
static cudaError_t launch_batch_rows(BatchAttnArgs& a, const BatchAttnPlan& p, cudaStream_t st) {
  a.p_tiles = p.p_tiles;
  a.p_splits = p.p_splits;
  a.s_tiles = p.s_tiles;
  a.s_splits = p.s_splits;
  // rows of whole aligned 4-element groups, else one element at a time
  const uintptr_t any = (uintptr_t)a.pages.k | (uintptr_t)a.pages.v | (uintptr_t)a.pk | (uintptr_t)a.pv;
  const bool vec = a.pages.d % 4 == 0 && any % (4 * sizeof(TK)) == 0;
  cudaError_t e = cudaSuccess;
  if (p.p_tiles > 0 && p.p_rt != p.rt) {   // the prefix's blocks in a launch of their own
    a.s_tiles = 0;
    e = launch_rows<TQ, TK>(a, p.p_rt, vec, st);
    a.s_tiles = p.s_tiles;
    a.p_tiles = 0;
    a.own_part = true;
  }
  if (e == cudaSuccess) e = launch_rows<TQ, TK>(a, p.rt, vec, st);
  if (e != cudaSuccess) return e;
  const long long rows = (long long)a.batch.n_tokens * a.nq;
  return launch(true, k_attn_join<TQ>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, a);
}

static bool attn_shape_ok(int nq, int prefix_len, const oos_paged_cache* c, const oos_batch* b) {
  if (!c || !b || nq < 1 || prefix_len < 0 || prefix_len > kMaxKeys || c->n_kv_heads < 1 || c->page_size < 1 || c->n_pages < 1) return false;
  if (nq % c->n_kv_heads || c->n_kv_heads > 65535 || b->n_seqs < 1 || b->n_tokens < 0 || b->max_pages < 1) return false;
  return (long long)b->n_tokens * nq + b->n_seqs < (1ll << 31) / kMaxParts && nq <= (1 << 20);
}

}  // namespace oos

using namespace oos;

extern "C" {

size_t oos_shared_prefix_attention_workspace_bytes(int32_t n_q_heads, int32_t prefix_len, const oos_paged_cache* cache,
                                                   const oos_batch* batch) {
  if (!attn_shape_ok(n_q_heads, prefix_len, cache, batch)) return 0;
  if (!dtype_ok(cache->dtype) || !head_dim_ok(cache->head_dim)) return 0;
  BatchAttnPlan p;
  return plan_batch_attn(n_q_heads, prefix_len, *cache, *batch, &p) ? std::max<size_t>(p.bytes, 256) : 0;
}

int oos_shared_prefix_attention(int32_t dtype, int32_t n_q_heads, const void* q, int64_t q_stride,
                                const void* prefix_k, const void* prefix_v, int32_t prefix_len,
                                const oos_paged_cache* cache, const oos_batch* batch, const int32_t* tree_parent,
                                float scale, void* out, int64_t out_stride, void* workspace, size_t ws_bytes,
                                int32_t* out_status, void* stream) {
  if (!attn_shape_ok(n_q_heads, prefix_len, cache, batch) || !pages_ok(cache) || !batch_ok(batch) || !out_status)
    return OOS_EINVAL;
  if (!(scale > 0.f) || !(scale < INFINITY)) return OOS_EINVAL;
  if (!dtype_ok(dtype) || !dtype_ok(cache->dtype) || !head_dim_ok(cache->head_dim)) return OOS_EUNSUPPORTED;
  if (dtype != cache->dtype && !(dtype == OOS_DTYPE_BF16 && cache->dtype == OOS_DTYPE_F16)) return OOS_EUNSUPPORTED;
  if (prefix_len > 0 && (!prefix_k || !prefix_v)) return OOS_EINVAL;
  if (cache->dtype != OOS_DTYPE_F32) {
    const uintptr_t any = (uintptr_t)cache->k | (uintptr_t)cache->v |
                          (prefix_len > 0 ? (uintptr_t)prefix_k | (uintptr_t)prefix_v : 0);
    if (any & 15) return OOS_EINVAL;
  }
  if (batch->n_tokens == 0) return OOS_OK;
  const long long w = (long long)n_q_heads * cache->head_dim;
  if (!q || !out || q_stride < w || out_stride < w) return OOS_EINVAL;
  BatchAttnPlan p;
  if (!plan_batch_attn(n_q_heads, prefix_len, *cache, *batch, &p)) return OOS_ECUDA;
  if (!workspace || ((uintptr_t)workspace & 255) || ws_bytes < p.bytes) return OOS_EWORKSPACE;
  BatchAttnArgs a = {};
  a.pages = view_of(*cache);
  a.batch = view_of(*batch);
  a.q = q;
  a.q_stride = q_stride;
  a.pk = prefix_len > 0 ? (const uint8_t*)prefix_k : nullptr;
  a.pv = prefix_len > 0 ? (const uint8_t*)prefix_v : nullptr;
  a.prefix_len = prefix_len;
  a.parent = tree_parent;
  a.nq = n_q_heads;
  a.group = n_q_heads / cache->n_kv_heads;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.out = out;
  a.out_stride = out_stride;
  a.part_o = (float*)workspace;
  a.part_ml = (float2*)((uint8_t*)workspace + p.ml_off);
  a.status = out_status;
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (p.tc) {
    a.p_splits = p.prefix.splits;
    a.s_splits = p.few ? p.pages.splits : p.sequence.splits;
    a.own_part = p.few && p.pages.part;
    e = a.p_splits > 0 ? launch_prefix_tc(a, p.prefix, dtype, cache->dtype, st) : cudaSuccess;
    if (e == cudaSuccess)
      e = p.few ? launch_pages_tc(a, p.pages, dtype, cache->dtype, st)
                : launch_sequence_tc(a, p.sequence, dtype, cache->dtype, st);
    if (p.few) a.s_splits = p.pages.part;   // for the join
    if (e == cudaSuccess && (p.few ? p.pages.part : a.s_splits > 1)) {
      const dim3 grid((unsigned)(((long long)batch->n_tokens * n_q_heads + 7) / 8));
      e = dtype == OOS_DTYPE_BF16 ? launch(true, k_attn_join_parts<__nv_bfloat16>, grid, dim3(256), 0, st, a)
                                  : launch(true, k_attn_join_parts<__half>, grid, dim3(256), 0, st, a);
    }
  } else if (dtype == OOS_DTYPE_F32) {
    e = launch_batch_rows<float, float>(a, p, st);
  } else if (cache->dtype == OOS_DTYPE_BF16) {
    e = launch_batch_rows<__nv_bfloat16, __nv_bfloat16>(a, p, st);
  } else if (dtype == OOS_DTYPE_BF16) {
    e = launch_batch_rows<__nv_bfloat16, __half>(a, p, st);
  } else {
    e = launch_batch_rows<__half, __half>(a, p, st);
  }
  return e == cudaSuccess ? OOS_OK : OOS_ECUDA;
}

}  // extern "C"
