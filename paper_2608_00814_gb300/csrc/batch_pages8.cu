// Attention of a batch step over the sequences' own 8-bit pages, 16-bit queries with heads of
// 128, where a sequence has few rows (a decoding token's group), and the join with the
// prefix's parts.
//
// A block owns a tile of 8 or 16 rows (token, head of one kv head's group) of one sequence,
// whose keys are dealt to its four warps 32 at a time: two blocks of 16 positions,
// each with one scale.  Every warp has a ring of its own, filled by TMA, a block of positions
// a copy (what lies behind the sequence's end comes along and is masked), and no block
// barrier before the end.  Places and scales of 16 such pairs are looked up at once by the
// lane that issues the copy.
//
// For short sequences and more of them than batch_stream8.cu's table holds; that file's warps
// go from sequence to sequence, and leave the join to a kernel of its own.  One token of one
// request over 1024 shared and 18 own keys: 7.3 us with the prefix's kernel, all latency (9 us
// each when they run apart); 64 of up to 100 own keys, 32 heads, 2048 shared: 22.6.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "batch_pages8.cuh"

namespace oos {

struct Pages8Args {
  P8Maps maps;
  BatchAttnArgs a;
};

template <typename TQ, int NT>
__global__ void __launch_bounds__(kP8Warps * 32, p8_blocks(NT)) k_attn_pages8(const __grid_constant__ Pages8Args p) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int ROWS = 8 * NT, STAGES = p8_stages(NT);
  __shared__ TreeScratch s_tree;
  __shared__ uint64_t s_full[kP8Warps][STAGES];
  const BatchAttnArgs& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = blockIdx.y;
  // behind the prefix's kernel, which has waited for what the caller wrote before it
  // triggers, only the join waits
  if (a.p_splits == 0) pdl_wait();
  pdl_trigger();
  TileRows t;
  if (!sequence_tile(a, blockIdx.x, ROWS, &t)) {
    if (blockIdx.x == 0 && blockIdx.y == 0) pdl_wait();       // the grid must not end before the one it follows
    return;
  }
  const unsigned long long (*anc)[2] = nullptr;
  if (a.parent) anc = tree_sets(a, t.q0, t.n, &s_tree);
  const int n_keys = anc ? t.len : max(0, min(t.len, t.first + (t.r0 + t.rows - 1) / a.group + 1));
  const int n_rounds = (n_keys + kP8Unit - 1) / kP8Unit;
  P8Ring<STAGES> ring = {smem + warp * (STAGES * kP8Stage), s_full[warp],
                         t.n * a.group <= ROWS ? policy_evict_first() : policy_evict_last()};   // read once, or by other tiles too
  ring.init();

  // ---- places and scales of 16 rounds: lane 2 r + h has block h of round r
  auto look_up = [&](int round) {
    const int key = (round + (lane >> 1)) * kP8Unit + warp * kP8Keys + (lane & 1) * kScaleBlock;
    if (round + (lane >> 1) < n_rounds && key < n_keys) return p8_place(a, g, t.seq, key / kScaleBlock);
    return P8Place{-1, 0, 127 | 127 << 8};
  };
  P8Place place = look_up(0), place2 = {-1, 0, 0};   // of this batch of 16 rounds and the next
  auto copy = [&](int round, int stage, const P8Place& from) {
    if (round < n_rounds && (lane >> 1) == (round & 15)) ring.copy(p.maps, g, stage, lane & 1, from);
  };
#pragma unroll
  for (int c = 0; c < STAGES - 1; ++c) copy(c, c, place);
  P8Rows<TQ, NT> rows;
  rows.load(a, g, t, [&](int token, unsigned long long (&to)[2]) {
    to[0] = anc[token][0];
    to[1] = anc[token][1];
  });
  rows.clear();
#pragma unroll 1
  for (int c = 0; c < n_rounds; ++c) {
    if (!ring.wait(a.status, min(STAGES - 1, n_rounds - c) - 1)) break;
    if ((c & 15) == 8) place2 = look_up((c & ~15) + 16);
    const int ahead = c + STAGES - 1;
    copy(ahead, ring.behind(), (ahead ^ c) & 16 ? place2 : place);
    const unsigned char* data = ring.data + ring.at * kP8Stage;
    ring.next();
    int scales[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) scales[h] = __shfl_sync(0xffffffffu, place.scales, 2 * (c & 15) + h);
    if ((c & 15) == 15) place = place2;
    rows.unit(a, t, data, c * kP8Unit + warp * kP8Keys, n_keys, scales);
    __syncwarp();
  }
  __syncthreads();
  // ---- join: O rows with (m, l), staged over the rings, of every warp, and the prefix's parts
  float* stage = reinterpret_cast<float*>(smem);   // [warp][row][kPartLd]
  rows.add_lanes();
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) rows.store(n, e, stage + (warp * ROWS + 8 * n + (lane & 3) * 2 + e) * kPartLd);
  const int pre_parts = a.p_splits;
  pdl_wait();   // the prefix's parts
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
    store_row<TQ>(a, g, t.q0, t.r0 + r, weighted_mean(acc, den));
  }
}

PagesPlan plan_pages8_tc(long long rows, int n_seqs, int nkv, int n_sms) {
  PagesPlan p = {};
  const int per_sm = p8_blocks(rows <= 8ll * n_seqs ? 1 : 2);
  p.tile_rows = rows <= 8ll * n_seqs ? 8 : 16;
  p.tiles = (int)(n_seqs + rows / p.tile_rows);
  const long long live = std::max((long long)n_seqs, (rows + p.tile_rows - 1) / p.tile_rows) * nkv;
  p.sms = (int)std::min<long long>(n_sms, (live + per_sm - 1) / per_sm);
  return p;
}

bool p8_maps(const BatchAttnArgs& a, P8Maps* maps) {
  // two codes an element of the copy
  const uint64_t row = (uint64_t)a.pages.nkv * kP8D;
  const uint64_t dims[4] = {kP8D / 2, (uint64_t)a.pages.nkv, (uint64_t)a.pages.page_size, (uint64_t)a.pages.n_pages};
  const uint64_t strides[3] = {kP8D, row, row * a.pages.page_size};
  const uint32_t box[4] = {kP8D / 2, 1, (uint32_t)kScaleBlock, 1};
  return encode_bf16_map(&maps->k, a.pages.k, 4, dims, strides, box, false) &&
         encode_bf16_map(&maps->v, a.pages.v, 4, dims, strides, box, false);
}

template <typename TQ, int NT>
static cudaError_t launch_pages8_of(const Pages8Args& a, const PagesPlan& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = kernel_ready(ready, (const void*)k_attn_pages8<TQ, NT>, p8_smem(NT));
  if (e != cudaSuccess) return e;
  return launch(true, k_attn_pages8<TQ, NT>, dim3((unsigned)p.tiles, a.a.pages.nkv), dim3(kP8Warps * 32), p8_smem(NT), st, a);
}

cudaError_t launch_pages8_tc(const BatchAttnArgs& a, const PagesPlan& p, int dtype, cudaStream_t st) {
  Pages8Args args;
  memset(&args, 0, sizeof(args));
  args.a = a;
  if (!p8_maps(a, &args.maps)) return cudaErrorInvalidValue;
  if (dtype == OOS_DTYPE_BF16)
    return p.tile_rows == 8 ? launch_pages8_of<__nv_bfloat16, 1>(args, p, st) : launch_pages8_of<__nv_bfloat16, 2>(args, p, st);
  return p.tile_rows == 8 ? launch_pages8_of<__half, 1>(args, p, st) : launch_pages8_of<__half, 2>(args, p, st);
}

}  // namespace oos
