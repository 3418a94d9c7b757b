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
// k_attn_rows (batch_rows.cuh): CUDA cores, fp32 products, for every type and head size.
// The 16-bit types with heads of 128 take the tensor-core kernels of batch_tiles.cu and
// batch_pages.cu, over 8-bit pages batch_tiles8.cu, batch_pages8.cu and batch_stream8.cu.
#include <math.h>

#include <algorithm>

#include "batch_attn.cuh"
#include "batch_rows.cuh"
#include "pages8.cuh"

namespace oos {

constexpr int kMaxParts = 32;      // parts of a row (a lane each in the join)

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
  bool stream;         // 8-bit pages, few rows: equal shares of all keys
  StreamPlan shares;
  size_t shares_off;
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

// own8: pages of 8 bits; c.dtype: the type of the prefix, and of other pages
static bool plan_batch_attn(int nq, int prefix_len, const oos_paged_cache& c, const oos_batch& b, bool own8, BatchAttnPlan* p) {
  const int sms = device_sms();
  *p = {};
  if (sms <= 0) return false;
  const int G = nq / c.n_kv_heads;
  const long long rows = (long long)b.n_tokens * G;
  const long long most_keys = std::min<long long>((long long)b.max_pages * c.page_size, kMaxKeys);
  p->tc = c.dtype != OOS_DTYPE_F32 && c.head_dim == 128;
  if (p->tc && own8) {
    // Tiles of 16 rows that each read their sequence's pages, or tiles of up to 256.  Trees of
    // 4 rows a node, 8 kv heads, 2048 prefix keys: 48 rows on average over up to 400 keys 38 us
    // against 41 (16 sequences) and 93 against 102 (64), 60 rows 44 against 41 and 111 against 118,
    // 72 rows 47 against 44 and 138 against 126.  Where all tiles of 16 fit the chip about twice,
    // more: 72 rows 21 against 33 (4 sequences; up to 4000 keys 37 against 85), 116 rows 17 against
    // 29 (1; up to 4000 keys 30 both), 101 rows 28 against 34 (4); but 96 rows 40 against 36 (8).
    // And over short tables where they fit it once: 232 rows 19 against 33 (1), 154 rows 21
    // against 36 (2), but 164 rows 36 against 39 (4), and 304 rows over up to 4000 keys 52
    // against 41 (1).
    const long long tiles16 = rows / 16 * c.n_kv_heads;
    p->few = rows <= 64ll * b.n_seqs || (rows <= 128ll * b.n_seqs && tiles16 <= 2ll * sms) || (most_keys <= 1024 && tiles16 <= sms);
    p->sequence = {false, 0, 1};
    if (p->few) p->pages = plan_pages8_tc(rows, b.n_seqs, c.n_kv_heads, sms);
    else p->sequence = plan_sequence_tc(rows, b.n_seqs, c.n_kv_heads, 0, most_keys, sms);   // the prefix apart
    p->prefix = prefix_len > 0 ? plan_prefix_tc(rows, c.n_kv_heads, prefix_len, p->few ? p->pages.sms : 0, sms) : PrefixPlan{0, 0, 0.0};
    // Blocks of many rows that join with several parts of the prefix wait for them and read
    // them one after the other; they leave a part too.  Trees of 4 rows a node, 8 kv heads, up to
    // 464 own keys: 8 sequences, 2048 prefix keys in 3 parts 50 us against 61, 4 sequences 36
    // against 56, 16 over 8000 keys 124 against 136; with one part 16 sequences take
    // 66 against 60, 13 prompts of 40 heads 227 against 202.
    p->sequence.part = !p->few && p->prefix.splits > 1;
    const int own = !p->few && (p->sequence.part || p->sequence.splits > 1) ? p->sequence.splits : 0;
    const int parts = p->prefix.splits + own;
    p->ml_off = 0;
    p->bytes = ((size_t)parts * b.n_tokens * nq * kPartLd * 4 + 255) / 256 * 256;
    // Equal shares of all keys, or a block for each tile that joins its rows itself.  One token
    // of 4 rows, 8 kv heads, 2048 prefix keys: 1 sequence of up to 800 keys 15.6 us against 12.5,
    // 16 of them 19.6 against 16.2, 20 of up to 4000 27 against 43; 64 of up to 100 23.0 against
    // 22.6, of up to 300 22.0 against 24.9; 250 of up to 300 45 against 51.
    p->stream = p->few && b.n_seqs <= kStreamSeqs && (most_keys > 1024 || (most_keys > 256 && (long long)b.n_seqs * c.n_kv_heads >= 3ll * sms));
    if (p->stream) {
      p->shares = plan_stream8(rows, b.n_seqs, b.n_tokens, c.n_kv_heads, p->prefix, sms);
      p->shares_off = p->bytes;
      p->bytes += p->shares.bytes;
    }
    return true;
  }
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

// TK: elements of the prefix, and of pages that are not of 8 bits
template <typename TQ, typename TK>
static cudaError_t launch_batch_rows(BatchAttnArgs& a, const BatchAttnPlan& p, int dtype, cudaStream_t st) {
  const bool own8 = a.k_scale != nullptr;
  a.p_tiles = p.p_tiles;
  a.p_splits = p.p_splits;
  a.s_tiles = p.s_tiles;
  a.s_splits = p.s_splits;
  // rows of whole aligned 4-element groups, else one element at a time
  const uintptr_t any = (own8 ? 0 : (uintptr_t)a.pages.k | (uintptr_t)a.pages.v) | (uintptr_t)a.pk | (uintptr_t)a.pv;
  const bool vec = a.pages.d % 4 == 0 && any % (4 * sizeof(TK)) == 0;
  cudaError_t e = cudaSuccess;
  if (p.p_tiles > 0 && (own8 || p.p_rt != p.rt)) {   // the prefix's blocks in a launch of their own
    a.s_tiles = 0;
    e = launch_rows<TQ, TK>(a, p.p_rt, vec, st);
    a.s_tiles = p.s_tiles;
    a.p_tiles = 0;
    a.own_part = true;
  }
  if (e == cudaSuccess) e = own8 ? launch_rows8(a, dtype, p.rt, st) : launch_rows<TQ, TK>(a, p.rt, vec, st);
  if (e != cudaSuccess) return e;
  const long long rows = (long long)a.batch.n_tokens * a.nq;
  return launch(true, k_attn_join<TQ>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, a);
}

static bool attn_shape_ok(int nq, int prefix_len, const oos_paged_cache& c, const oos_batch* b) {
  if (!b || nq < 1 || prefix_len < 0 || prefix_len > kMaxKeys || c.n_kv_heads < 1 || c.page_size < 1 || c.n_pages < 1) return false;
  if (nq % c.n_kv_heads || c.n_kv_heads > 65535 || b->n_seqs < 1 || b->n_tokens < 0 || b->max_pages < 1) return false;
  return (long long)b->n_tokens * nq + b->n_seqs < (1ll << 31) / kMaxParts && nq <= (1 << 20);
}

// the shape and codes of 8-bit pages, beside a prefix of dtype
static oos_paged_cache pages_of(const oos_paged_cache8& c, int dtype) {
  return {dtype, c.n_kv_heads, c.head_dim, c.page_size, c.n_pages, c.k, c.v};
}

static bool attn_dtypes_ok(int dtype, int kv_dtype) {   // of queries, of 16-bit or fp32 keys
  return dtype == kv_dtype || (dtype == OOS_DTYPE_BF16 && kv_dtype == OOS_DTYPE_F16);
}

// c: the pages, of 8 bits where scales are given; c.dtype: the prefix's type then
static int attend(int dtype, int n_q_heads, const void* q, int64_t q_stride, const void* prefix_k, const void* prefix_v,
                  int prefix_len, const oos_paged_cache& c, const uint8_t* k_scale, const uint8_t* v_scale,
                  const oos_batch* batch, const int32_t* tree_parent, float scale, void* out, int64_t out_stride,
                  void* workspace, size_t ws_bytes, int32_t* out_status, void* stream) {
  const bool own8 = k_scale != nullptr;
  if (prefix_len > 0 && (!prefix_k || !prefix_v)) return OOS_EINVAL;
  const uintptr_t prefix = prefix_len > 0 ? (uintptr_t)prefix_k | (uintptr_t)prefix_v : 0, pages = (uintptr_t)c.k | (uintptr_t)c.v;
  if (own8 ? dtype != OOS_DTYPE_F32 && ((prefix | (c.head_dim == 128 ? pages : 0)) & 15)
           : c.dtype != OOS_DTYPE_F32 && ((prefix | pages) & 15))
    return OOS_EINVAL;
  if (batch->n_tokens == 0) return OOS_OK;
  const long long w = (long long)n_q_heads * c.head_dim;
  if (!q || !out || q_stride < w || out_stride < w) return OOS_EINVAL;
  BatchAttnPlan p;
  if (!plan_batch_attn(n_q_heads, prefix_len, c, *batch, own8, &p)) return OOS_ECUDA;
  if (!workspace || ((uintptr_t)workspace & 255) || ws_bytes < p.bytes) return OOS_EWORKSPACE;
  BatchAttnArgs a = {};
  a.pages = view_of(c);
  a.batch = view_of(*batch);
  a.q = q;
  a.q_stride = q_stride;
  a.pk = prefix_len > 0 ? (const uint8_t*)prefix_k : nullptr;
  a.pv = prefix_len > 0 ? (const uint8_t*)prefix_v : nullptr;
  a.prefix_len = prefix_len;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.parent = tree_parent;
  a.nq = n_q_heads;
  a.group = n_q_heads / c.n_kv_heads;
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
    a.s_splits = p.few ? p.pages.splits : p.sequence.splits;   // 0 of few rows over 8-bit pages
    a.own_part = p.few ? p.pages.part : p.sequence.part;
    e = a.p_splits > 0 ? launch_prefix_tc(a, p.prefix, dtype, c.dtype, st) : cudaSuccess;
    if (e == cudaSuccess && p.stream) e = launch_stream8(a, p.shares, (uint8_t*)workspace + p.shares_off, dtype, st);
    else if (e == cudaSuccess)
      e = !p.few ? (own8 ? launch_sequence8_tc(a, p.sequence, dtype, st) : launch_sequence_tc(a, p.sequence, dtype, c.dtype, st))
                 : own8 ? launch_pages8_tc(a, p.pages, dtype, st)
                        : launch_pages_tc(a, p.pages, dtype, c.dtype, st);
    if (p.few) a.s_splits = p.pages.part;   // for the join
    if (e == cudaSuccess && (p.few ? p.pages.part : p.sequence.part || a.s_splits > 1)) {
      const dim3 grid((unsigned)(((long long)batch->n_tokens * n_q_heads + 7) / 8));
      e = dtype == OOS_DTYPE_BF16 ? launch(true, k_attn_join_parts<__nv_bfloat16>, grid, dim3(256), 0, st, a)
                                  : launch(true, k_attn_join_parts<__half>, grid, dim3(256), 0, st, a);
    }
  } else if (dtype == OOS_DTYPE_F32) {
    e = launch_batch_rows<float, float>(a, p, dtype, st);
  } else if (c.dtype == OOS_DTYPE_BF16) {
    e = launch_batch_rows<__nv_bfloat16, __nv_bfloat16>(a, p, dtype, st);
  } else if (dtype == OOS_DTYPE_BF16) {
    e = launch_batch_rows<__nv_bfloat16, __half>(a, p, dtype, st);
  } else {
    e = launch_batch_rows<__half, __half>(a, p, dtype, st);
  }
  return e == cudaSuccess ? OOS_OK : OOS_ECUDA;
}

}  // namespace oos

using namespace oos;

extern "C" {

size_t oos_shared_prefix_attention_workspace_bytes(int32_t n_q_heads, int32_t prefix_len, const oos_paged_cache* cache,
                                                   const oos_batch* batch) {
  if (!cache || !attn_shape_ok(n_q_heads, prefix_len, *cache, batch)) return 0;
  if (!dtype_ok(cache->dtype) || !head_dim_ok(cache->head_dim)) return 0;
  BatchAttnPlan p;
  return plan_batch_attn(n_q_heads, prefix_len, *cache, *batch, false, &p) ? std::max<size_t>(p.bytes, 256) : 0;
}

int oos_shared_prefix_attention(int32_t dtype, int32_t n_q_heads, const void* q, int64_t q_stride,
                                const void* prefix_k, const void* prefix_v, int32_t prefix_len,
                                const oos_paged_cache* cache, const oos_batch* batch, const int32_t* tree_parent,
                                float scale, void* out, int64_t out_stride, void* workspace, size_t ws_bytes,
                                int32_t* out_status, void* stream) {
  if (!cache || !attn_shape_ok(n_q_heads, prefix_len, *cache, batch) || !pages_ok(cache) || !batch_ok(batch) || !out_status)
    return OOS_EINVAL;
  if (!(scale > 0.f) || !(scale < INFINITY)) return OOS_EINVAL;
  if (!dtype_ok(dtype) || !dtype_ok(cache->dtype) || !head_dim_ok(cache->head_dim)) return OOS_EUNSUPPORTED;
  if (!attn_dtypes_ok(dtype, cache->dtype)) return OOS_EUNSUPPORTED;
  return attend(dtype, n_q_heads, q, q_stride, prefix_k, prefix_v, prefix_len, *cache, nullptr, nullptr, batch,
                tree_parent, scale, out, out_stride, workspace, ws_bytes, out_status, stream);
}

size_t oos_shared_prefix_attention8_workspace_bytes(int32_t dtype, int32_t n_q_heads, int32_t prefix_len,
                                                    const oos_paged_cache8* cache, const oos_batch* batch) {
  if (!cache || !attn_shape_ok(n_q_heads, prefix_len, pages_of(*cache, dtype), batch)) return 0;
  if (!dtype_ok(dtype) || !head_dim_ok(cache->head_dim) || cache->page_size % kScaleBlock) return 0;
  BatchAttnPlan p;
  return plan_batch_attn(n_q_heads, prefix_len, pages_of(*cache, dtype), *batch, true, &p) ? std::max<size_t>(p.bytes, 256) : 0;
}

int oos_shared_prefix_attention8(int32_t dtype, int32_t n_q_heads, const void* q, int64_t q_stride,
                                 int32_t prefix_dtype, const void* prefix_k, const void* prefix_v, int32_t prefix_len,
                                 const oos_paged_cache8* cache, const oos_batch* batch, const int32_t* tree_parent,
                                 float scale, void* out, int64_t out_stride, void* workspace, size_t ws_bytes,
                                 int32_t* out_status, void* stream) {
  if (!cache || !attn_shape_ok(n_q_heads, prefix_len, pages_of(*cache, dtype), batch) || !pages8_ok(cache) ||
      !batch_ok(batch) || !out_status)
    return OOS_EINVAL;
  if (!(scale > 0.f) || !(scale < INFINITY)) return OOS_EINVAL;
  if (prefix_len == 0) prefix_dtype = dtype;
  if (!dtype_ok(dtype) || !dtype_ok(prefix_dtype) || !head_dim_ok(cache->head_dim)) return OOS_EUNSUPPORTED;
  if (!attn_dtypes_ok(dtype, prefix_dtype)) return OOS_EUNSUPPORTED;
  return attend(dtype, n_q_heads, q, q_stride, prefix_k, prefix_v, prefix_len, pages_of(*cache, prefix_dtype),
                cache->k_scale, cache->v_scale, batch, tree_parent, scale, out, out_stride, workspace, ws_bytes,
                out_status, stream);
}

}  // extern "C"
