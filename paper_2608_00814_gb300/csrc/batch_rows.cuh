// Attention of a batch step on CUDA cores, fp32 products, for every type and head size:
// a part per range of keys (batch_attn.cu; over 8-bit pages batch_rows8.cu).
#pragma once

#include <type_traits>

#include "batch_attn.cuh"
#include "pages8.cuh"

namespace oos {

constexpr int kRowKeys = 32;       // keys per tile
constexpr int kRowThreads = 128;

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
  constexpr bool SCALED = std::is_same<TK, E4M3>::value;   // 8-bit pages; the prefix in a launch of its own
  __shared__ TreeScratch s_tree;
  __shared__ long long s_at[2][kRowKeys];   // slot of each key in its buffer, -1: none; of two tiles in turn
  // 8-bit pages: powers of two of each key's K and V.  K's goes to its score, behind the
  // call's scale: a product of codes is far from fp32's limits, which scaled ones may pass.
  __shared__ float s_pow[2][2][SCALED ? kRowKeys : 1];

  // behind the prefix's launch, which has waited for what the caller wrote before it
  // triggers, only the end waits
  if (!a.own_part) pdl_wait();
  pdl_trigger();
  const int g = blockIdx.y;
  const bool prefix = !SCALED && (int)blockIdx.x < a.p_tiles * a.p_splits;
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
      if constexpr (SCALED) {
        const long long block = max(at, 0ll) / kScaleBlock * a.pages.nkv + g;
        s_pow[(key0 - k0) / kRowKeys & 1][0][tid] = pow2f(scale_exp(a.k_scale[block]));
        s_pow[(key0 - k0) / kRowKeys & 1][1][tid] = pow2f(scale_exp(a.v_scale[block]));
      }
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
        if constexpr (SCALED) {
          const float fv = s_pow[(key0 - k0) / kRowKeys & 1][1][key];
#pragma unroll
          for (int e = 0; e < VEC; ++e) vv[e] *= fv;
        }
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
        if constexpr (SCALED) s[r][j] = ok ? s[r][j] * s_pow[(key0 - k0) / kRowKeys & 1][0][tc + TPR * j] : -INFINITY;
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

}  // namespace oos
