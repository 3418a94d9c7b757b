// Attention of a batch step: what its kernels share (batch_attn.cu, batch_rows.cuh,
// batch_tiles.cu, batch_pages.cu, and over 8-bit pages batch_tiles8.cu, batch_pages8.cu,
// batch_stream8.cu).
#pragma once

#include "batch.cuh"

namespace oos {

constexpr int kMaxTreeRows = 128;  // rows of a sequence with a tree
constexpr int kMaxPrefixParts = 16;   // of a row, of the tensor-core kernels
constexpr int kPartLd = 128 + 4;   // a row of a part: O, m, l, padded to 16 bytes
// Binary16 weights are 2^(score - maximum + 7): below 2^15 before a maximum moves (which takes
// scores 2^8 above it), and normal numbers, rounded to 2^-11, down to 2^-21 of the largest;
// below that to 2^-32 of the largest.
constexpr float kHalfBias = 7.f;
constexpr int kMaxKeys = 0x7ffff000;   // of a prefix or a sequence: tiles of keys past the last still count in 32 bits

struct BatchAttnArgs {
  PagesView pages;
  BatchView batch;
  const void* q;
  long long q_stride;
  const uint8_t* pk;
  const uint8_t* pv;
  int prefix_len;
  const uint8_t* k_scale;   // of 8-bit pages
  const uint8_t* v_scale;
  const int32_t* parent;
  int nq, group;
  float scale_log2;
  void* out;
  long long out_stride;
  // parts in the workspace: of all rows and keys, part_o [part][token][head][d] and
  // part_ml [part][token][head]; on tensor cores of the prefix only, in part_o
  // [part][kv head][row][kPartLd], row = token * group + head in group: O, m, l
  float* part_o;
  float2* part_ml;
  int p_tiles, p_splits, s_tiles, s_splits;
  bool own_part;   // own keys in a launch behind the prefix's leave their parts for the join
  int32_t* status;
};

OOS_DEV float max_nan(float a, float b) {   // a NaN wins, so that it reaches the output
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Rows of a tile and the keys they may see
struct TileRows {
  int seq;            // -1: the prefix's keys
  int q0;             // first token of the rows counted
  int r0;             // first row of the tile: token q0 + r / group, head r % group
  int rows;           // rows of the tile
  int n;              // rows of the sequence in this step
  int first;          // its positions before them
  int len;            // its positions
};

// Tile `i` of the sequences' tiles of `tile_rows` rows.  Sequence b's tiles start at
// b + floor(q_start[b] group / tile_rows): a count known without a scan, at the price
// of some numbers that no tile has.  The whole warp; false: no such tile.
OOS_DEV bool sequence_tile(const BatchAttnArgs& a, int i, int tile_rows, TileRows* t) {
  const BatchView& b = a.batch;
  auto start = [&](int s) { return s + (long long)b.q_start[s] * a.group / tile_rows; };
  const int seq = warp_count_le(b.n_seqs - 1, start, i);
  const int q0 = b.q_start[seq], q1 = b.q_start[seq + 1], given = b.seq_len[seq], len = max(0, given);
  const long long most = min((long long)b.max_pages * a.pages.page_size, (long long)kMaxKeys);
  const bool in_order = q0 >= 0 && q1 <= b.n_tokens && q0 <= q1;
  const bool ok = in_order && (!a.parent || q1 - q0 <= kMaxTreeRows);
  if (!ok || given < q1 - q0 || len > most) {
    if (threadIdx.x == 0) *a.status = in_order && !ok ? OOS_ETREE : OOS_EBATCH;
  }
  if (!ok || i < start(seq)) return false;
  t->seq = seq;
  t->q0 = q0;
  // counts of rows stay below 2^26 (n_tokens * nq is), those of a table out of order do not
  const long long r0 = (i - start(seq)) * tile_rows, all = (long long)(q1 - q0) * a.group;
  if (r0 >= all) return false;
  t->r0 = (int)r0;
  t->rows = (int)min((long long)tile_rows, all - r0);
  t->n = q1 - q0;
  t->first = len - t->n;
  t->len = (int)min((long long)len, most);
  return true;
}

// Ancestor sets of the sequence's rows, [row] -> 128 bits, itself included, by pointer
// doubling in shared memory: n <= kMaxTreeRows rows, threads tid of n_threads that meet
// at sync().
struct TreeScratch {
  unsigned long long anc[2][kMaxTreeRows][2];
  int up[2][kMaxTreeRows];
};
template <typename SYNC>
OOS_DEV const unsigned long long (*tree_sets(const BatchAttnArgs& a, int q0, int n, TreeScratch* t, int tid, int n_threads,
                                             SYNC sync))[2] {
  for (int i = tid; i < n; i += n_threads) {
    int p = a.parent[q0 + i];
    if (p < -1 || p >= i) {
      *a.status = OOS_ETREE;
      p = -1;
    }
    t->up[0][i] = p;
    t->anc[0][i][0] = i < 64 ? 1ull << i : 0ull;
    t->anc[0][i][1] = i < 64 ? 0ull : 1ull << (i - 64);
  }
  sync();
  int cur = 0;
  for (int step = 1; step < n; step *= 2, cur ^= 1) {
    for (int i = tid; i < n; i += n_threads) {
      const int p = t->up[cur][i];
      t->anc[cur ^ 1][i][0] = t->anc[cur][i][0] | (p >= 0 ? t->anc[cur][p][0] : 0ull);
      t->anc[cur ^ 1][i][1] = t->anc[cur][i][1] | (p >= 0 ? t->anc[cur][p][1] : 0ull);
      t->up[cur ^ 1][i] = p >= 0 ? t->up[cur][p] : -1;
    }
    sync();
  }
  return t->anc[cur];
}
OOS_DEV const unsigned long long (*tree_sets(const BatchAttnArgs& a, int q0, int n, TreeScratch* t))[2] {   // the block
  return tree_sets(a, q0, n, t, threadIdx.x, blockDim.x, [] { __syncthreads(); });
}

OOS_DEV void cp_async16(uint32_t dst, const void* src, bool ok) {   // zeros where not ok
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
OOS_DEV void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
OOS_DEV void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Row `row` of the sequence that starts at token q0, kv head g: the lane's four columns
template <typename TQ>
OOS_DEV void store_row(const BatchAttnArgs& a, int g, int q0, int row, float4 o) {
  const float v[4] = {o.x, o.y, o.z, o.w};
  TQ* out = (TQ*)a.out + (long long)(q0 + row / a.group) * a.out_stride + (g * a.group + row % a.group) * 128 +
            4 * (threadIdx.x & 31);
  if (((uintptr_t)out & 7) == 0) {
    store_vec<TQ, 4>(out, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = from_f32<TQ>(v[e]);
  }
}

// a row's sum over the sum of its weights; a row without keys: zeros
OOS_DEV float4 weighted_mean(float4 o, float den) {
  const float f = den == 0.f ? 0.f : 1.f / den;
  return make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
}

// bf16 queries of a binary16 cache: a power of two per row brings the largest element
// to [1, 2), where binary16 holds bf16's 8 bits exactly (elements below 2^-14 of it
// to 2^-25 of it, far below what their scores are rounded by); the power goes into
// the row's scale.  Zero, infinite or NaN rows stay as they are.
OOS_DEV int row_exponent(float mx) {
  if (!(mx > 0.f) || mx == INFINITY) return 0;
  return max(-126, min(126, (int)(__float_as_uint(mx) >> 23) - 127));
}
OOS_DEV float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
OOS_DEV float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
OOS_DEV float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
OOS_DEV uint32_t scaled_half2(uint32_t w, float f) {
  const __half2 v = __floats2half2_rn(bf16_lo(w) * f, bf16_hi(w) * f);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// the prefix kernel's blocks: what a call is cut into
struct PrefixPlan {
  int splits;   // key ranges, a part each
  int pairs;    // pairs of 128-row tiles
  double us;    // estimated
};
// own_sms: that the blocks of launch_pages_tc would fill, 0 where that kernel does not follow
PrefixPlan plan_prefix_tc(long long rows, int nkv, int prefix_len, int own_sms, int n_sms);
struct PagesPlan {
  int tile_rows;   // of a block: 8 or 16
  int tiles, splits;
  int sms;         // that its blocks fill at once, about
  bool part;       // leaves a part for a join
};
struct SequencePlan {
  bool takes_prefix;   // in the same kernel
  int tiles, splits;
  bool part;           // leaves a part for a join, with one split too
};
SequencePlan plan_sequence_tc(long long rows, int n_seqs, int nkv, int prefix_len, long long most_keys, int n_sms);
PagesPlan plan_pages_tc(long long rows, int n_seqs, int nkv, long long most_keys, int n_sms);
// own keys in 8-bit pages on CUDA cores, tiles of rt rows: parts p_splits ..
cudaError_t launch_rows8(const BatchAttnArgs& a, int dtype, int rt, cudaStream_t st);
// the prefix's parts of every row
cudaError_t launch_prefix_tc(const BatchAttnArgs& a, const PrefixPlan& p, int dtype, int kv_dtype, cudaStream_t st);
// the sequences' own keys, joined with the prefix's p_splits parts into out; with several
// splits of launch_sequence_tc, or own_part, left as parts p_splits .. for k_attn_join_parts
cudaError_t launch_sequence_tc(const BatchAttnArgs& a, const SequencePlan& p, int dtype, int kv_dtype, cudaStream_t st);
cudaError_t launch_pages_tc(const BatchAttnArgs& a, const PagesPlan& p, int dtype, int kv_dtype, cudaStream_t st);
// the same over 8-bit pages, queries of dtype: a block for each tile, which joins its rows itself
PagesPlan plan_pages8_tc(long long rows, int n_seqs, int nkv, int n_sms);
cudaError_t launch_pages8_tc(const BatchAttnArgs& a, const PagesPlan& p, int dtype, cudaStream_t st);
// the same, an equal share of all keys for every warp, and the join; n_seqs <= kStreamSeqs
constexpr int kStreamSeqs = 256;
struct StreamPlan {
  int tile_rows, blocks, places;
  int late;                   // units that the prefix's blocks keep a block behind them from
  int early;                  // blocks that they do not
  size_t tokens_off, bytes;   // of its workspace
};
StreamPlan plan_stream8(long long rows, int n_seqs, int n_tokens, int nkv, const PrefixPlan& prefix, int n_sms);
cudaError_t launch_stream8(const BatchAttnArgs& a, const StreamPlan& p, void* workspace, int dtype, cudaStream_t st);
cudaError_t launch_sequence8_tc(const BatchAttnArgs& a, const SequencePlan& p, int dtype, cudaStream_t st);   // a plan without the prefix

}  // namespace oos
