// Attention of a batch step over 8-bit pages where sequences have few rows and may be long:
// every warp takes an equal share of all keys.
//
// The keys of all tiles of rows stand behind one another in units of 32, sequence by
// sequence; warp w takes units w piece .. (w + 1) piece - 1, whatever sequences they belong to.
// The lengths are on the device: each block adds them up into a table in shared memory, in
// which a warp finds the sequence of a unit.  A warp's copies run ahead over the end of a
// sequence, so that the next one's keys are on their way while the last one's rows are
// stored, and no warp waits for another.  Rows of tile i that warp w has seen keys of stand at
// place w + i of the workspace, which no other pair has, as w and i both only grow along the
// units.  k_join8 adds a row's places up, and the prefix's parts.
//
// As many blocks as the chip holds at once are launched; short steps leave some idle.
//
// Bound by HBM while the copies run: 6 requests of up to 64000 keys, 64 heads over 8, take 65 us
// under a profiler, 6.0 TB/s with a beginning of 5 us (lengths, places, first copies), and 68 with
// the join (16-bit pages 233); 64 of up to 4000, 2048 shared, 32 heads 50 (104), where the
// prefix's kernel holds 64 SMs for 12 us and the join takes 4.  The issue slots are 37 % used, by some
// 550 instructions for 8 KB.  Three stages for two blocks an SM: 66 and 54 us.  Other orders of
// the blocks' work were slower: ranges by length for a block each 70 and 58 us, two or
// three times as many 76 and 63 to 87 and 70; copies with other cache policies 72 and 57.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "batch_pages8.cuh"

namespace oos {

constexpr int kS8MaxSeqs = kStreamSeqs;   // of the table in shared memory
constexpr int kS8LeastPiece = 4;     // units of a warp (8: 64 requests of up to 400 keys 28 us, 24 with 4)
constexpr int kS8MaxPlaces = 256;    // of a tile, about: longer pieces otherwise
constexpr int kS8JoinThreads = 128;
// Units that a warp takes in a microsecond, by which the shares of blocks that start when the
// prefix's are done are smaller (64 requests as above: 0 59 us, 0.25 to 0.45 55, 0.65 56; 200 of
// up to 1500 keys 83, 84 to 86, 93; in tiles of 16 rows 64 trees of up to 4 nodes 0 78, 0.15 77,
// 0.3 and 0.45 74, 200 of them over up to 1500 keys 116, 111, 105, 104)
constexpr double kS8UnitsPerUs = 0.3;

// Shares of `piece` units for the first `early` warps, of `late` less for the others
struct S8Shares {
  int piece, early, less;
  OOS_DEV static S8Shares of(long long total, int n_warps, int early, int late, int longest) {
    const int least = max(kS8LeastPiece, (longest + kS8MaxPlaces - 1) / kS8MaxPlaces);
    S8Shares s;
    s.early = early;
    // late warps that would have less than the least have that
    const long long piece = (total + (long long)(n_warps - early) * late + n_warps - 1) / n_warps;
    s.piece = (int)max((long long)least, piece);
    s.less = min(late, s.piece - least);
    return s;
  }
  OOS_DEV long long from(int w) const { return (long long)w * piece - (long long)max(0, w - early) * less; }
  OOS_DEV int warp_of(long long u) const {
    const long long e = (long long)early * piece;
    return u < e ? (int)(u / piece) : early + (int)((u - e) / (piece - less));
  }
};
// what the join needs of a token's sequence
struct S8Token {
  int q0;            // its first token; -1: a sequence that is left out
  int tile0;         // its first tile
  int units;         // of each of its tiles
  long long unit0;   // where its units start
  S8Shares shares;
};
struct Stream8Args {
  P8Maps maps;
  BatchAttnArgs a;
  float* places;     // [kv head][place][row of a tile][kPartLd]
  S8Token* tokens;   // [n_tokens]
  int n_places;
  int early, late;   // warps whose blocks start at once, units that the others have less
};

// Number of the n entries of `from` that are <= x; from[0] is
template <typename T>
OOS_DEV int count_le(const T* from, int n, T x) {
  int lo = 1, hi = n;   // the count lies in [lo, hi]
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (from[mid - 1] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

template <typename TQ, int NT>
__global__ void __launch_bounds__(kP8Warps * 32, p8_blocks(NT)) k_attn_stream8(const __grid_constant__ Stream8Args p) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int ROWS = 8 * NT, STAGES = p8_stages(NT);
  __shared__ uint64_t s_full[kP8Warps][STAGES];
  __shared__ long long s_unit[kS8MaxSeqs + 1];   // first unit of a sequence
  __shared__ int s_tile[kS8MaxSeqs + 1];         // first tile
  __shared__ int s_units[kS8MaxSeqs];            // units of each of its tiles
  __shared__ int s_q0[kS8MaxSeqs], s_n[kS8MaxSeqs], s_len[kS8MaxSeqs];   // its first token, tokens, positions
  __shared__ long long s_sum[kP8Warps];
  __shared__ int s_sum_tiles[kP8Warps], s_longest[kP8Warps];
  const BatchAttnArgs& a = p.a;
  const BatchView& b = a.batch;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int nkv = a.pages.nkv, g = blockIdx.x % nkv, n_warps = (int)gridDim.x / nkv * kP8Warps, w = (int)blockIdx.x / nkv * kP8Warps + warp;
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&p.maps.k);
    tma_prefetch_desc(&p.maps.v);
  }
  // behind the prefix's kernel, which has waited for what the caller wrote before it
  // triggers, only the join waits
  if (a.p_splits == 0) pdl_wait();
  pdl_trigger();

  // ---- the table: thread i has sequences PER i ..
  constexpr int PER = kS8MaxSeqs / (kP8Warps * 32);
  const long long most = min((long long)b.max_pages * a.pages.page_size, (long long)kMaxKeys);
  const bool report = blockIdx.x == 0;
  {
    int tiles[PER], units[PER], sum_tiles = 0, longest = 0;
    long long sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int seq = threadIdx.x * PER + i;
      tiles[i] = units[i] = 0;
      s_q0[seq] = s_n[seq] = s_len[seq] = 0;
      if (seq >= b.n_seqs) continue;
      const int q0 = b.q_start[seq], q1 = b.q_start[seq + 1], given = b.seq_len[seq], len = max(0, given);
      const bool in_order = q0 >= 0 && q1 <= b.n_tokens && q0 <= q1, ok = in_order && (!a.parent || q1 - q0 <= kMaxTreeRows);
      if (report && (!ok || given < q1 - q0 || len > most)) *a.status = in_order && !ok ? OOS_ETREE : OOS_EBATCH;
      if (ok && q1 > q0) {
        s_q0[seq] = q0;
        s_n[seq] = q1 - q0;
        s_len[seq] = (int)min((long long)len, most);
        tiles[i] = ((q1 - q0) * a.group + ROWS - 1) / ROWS;   // n_tokens * nq stays below 2^26
        units[i] = (int)((min((long long)len, most) + kP8Keys - 1) / kP8Keys);
      }
      sum += (long long)tiles[i] * units[i];
      sum_tiles += tiles[i];
      longest = max(longest, units[i]);
    }
    long long upto = sum;
    int upto_tiles = sum_tiles;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) {
      const long long v = __shfl_up_sync(0xffffffffu, upto, x);
      const int vt = __shfl_up_sync(0xffffffffu, upto_tiles, x);
      if (lane >= x) {
        upto += v;
        upto_tiles += vt;
      }
      longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, x));
    }
    if (lane == 31) {
      s_sum[warp] = upto;
      s_sum_tiles[warp] = upto_tiles;
      s_longest[warp] = longest;
    }
    __syncthreads();
    upto -= sum;
    upto_tiles -= sum_tiles;
#pragma unroll
    for (int i = 0; i < kP8Warps; ++i)
      if (i < warp) {
        upto += s_sum[i];
        upto_tiles += s_sum_tiles[i];
      }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int seq = threadIdx.x * PER + i;
      s_unit[seq] = upto;
      s_tile[seq] = upto_tiles;
      s_units[seq] = units[i];
      upto += (long long)tiles[i] * units[i];
      upto_tiles += tiles[i];
    }
    if (threadIdx.x == kP8Warps * 32 - 1) {
      s_unit[kS8MaxSeqs] = upto;
      s_tile[kS8MaxSeqs] = upto_tiles;
    }
  }
  __syncthreads();
  const long long total = s_unit[kS8MaxSeqs];
  S8Shares shares;
  {
    int longest = 0;
#pragma unroll
    for (int i = 0; i < kP8Warps; ++i) longest = max(longest, s_longest[i]);
    shares = S8Shares::of(total, n_warps, min(n_warps, p.early), p.late, longest);
  }
  // what the join needs, by all warps of the first kv head
  if (g == 0) {
    for (int seq = w; seq < b.n_seqs; seq += n_warps) {
      const int q0 = b.q_start[seq], q1 = b.q_start[seq + 1];
      if (s_tile[seq + 1] == s_tile[seq] && !(q0 >= 0 && q1 <= b.n_tokens)) continue;
      const S8Token v = {s_tile[seq + 1] > s_tile[seq] ? q0 : -1, s_tile[seq], s_units[seq], s_unit[seq], shares};
      for (int i = q0 + lane; i < q1; i += 32) p.tokens[i] = v;
    }
  }

  // ---- this warp's units
  const long long u0 = shares.from(w);
  const int n = (int)max(0ll, min(shares.from(w + 1), total) - u0);
  P8Ring<STAGES> ring = {smem + warp * (STAGES * kP8Stage), s_full[warp], policy_evict_first()};
  ring.init();
  // places and scales of 16 units: lane 2 r + h has block h of unit r
  auto look_up = [&](int from) {
    P8Place at = {-1, 0, 127 | 127 << 8};
    const int c = from + (lane >> 1);
    if (c < n) {
      const int seq = count_le(s_unit, b.n_seqs, u0 + c) - 1;
      const int block = (int)(s_n[seq] * a.group <= ROWS ? u0 + c - s_unit[seq] : (u0 + c - s_unit[seq]) % s_units[seq]) * 2 + (lane & 1);
      if ((long long)block * kScaleBlock < s_len[seq]) at = p8_place(a, g, seq, block);
    }
    return at;
  };
  P8Place place = look_up(0), place2 = {-1, 0, 0};   // of this batch of 16 units and the next
  auto copy = [&](int c, int stage, const P8Place& from) {
    if (c < n && (lane >> 1) == (c & 15)) ring.copy(p.maps, g, stage, lane & 1, from);
  };
#pragma unroll
  for (int c = 0; c < STAGES - 1; ++c) copy(c, c, place);

  P8Rows<TQ, NT> rows;
  TileRows t = {};
  int tile = 0, local = 0, units = 0;   // the tile, the unit of its keys that is next, and how many there are
  auto begin = [&](long long u) {
    const int seq = count_le(s_unit, b.n_seqs, u) - 1;
    units = s_units[seq];
    const int k = s_n[seq] * a.group <= ROWS ? 0 : (int)((u - s_unit[seq]) / units);   // of the sequence's tiles
    local = (int)(u - s_unit[seq] - (long long)k * units);
    tile = s_tile[seq] + k;
    t.seq = seq;
    t.q0 = s_q0[seq];
    t.n = s_n[seq];
    t.len = s_len[seq];
    t.first = t.len - t.n;
    t.r0 = k * ROWS;
    t.rows = min(ROWS, t.n * a.group - t.r0);
    // a row's ancestors, up from itself
    rows.load(a, g, t, [&](int token, unsigned long long (&to)[2]) {
      int i = token;
      while (i >= 0) {
        if (i < 64) to[0] |= 1ull << i;
        else to[1] |= 1ull << (i - 64);
        const int up = __ldg(a.parent + t.q0 + i);
        if (up < -1 || up >= i) {
          *a.status = OOS_ETREE;
          break;
        }
        i = up;
      }
    });
    rows.clear();
  };
  auto finish = [&]() {
    rows.add_lanes();
    if ((unsigned)(w + tile) >= (unsigned)p.n_places) return;   // only where offsets out of order give rows twice
    float* to = p.places + ((long long)g * p.n_places + w + tile) * (ROWS * kPartLd);
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * x + (lane & 3) * 2 + e;
        if (r < t.rows) rows.store(x, e, to + r * kPartLd);
      }
  };
#pragma unroll 1
  for (int c = 0; c < n; ++c) {
    if (local == units) {
      if (c > 0) finish();
      begin(u0 + c);
    }
    if (!ring.wait(a.status, min(STAGES - 1, n - c) - 1)) break;
    if ((c & 15) == 8) place2 = look_up((c & ~15) + 16);
    const int ahead = c + STAGES - 1;
    copy(ahead, ring.behind(), (ahead ^ c) & 16 ? place2 : place);
    const unsigned char* data = ring.data + ring.at * kP8Stage;
    ring.next();
    int scales[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) scales[h] = __shfl_sync(0xffffffffu, place.scales, 2 * (c & 15) + h);
    if ((c & 15) == 15) place = place2;
    rows.unit(a, t, data, local * kP8Keys, t.len, scales);
    ++local;
    __syncwarp();
  }
  if (n > 0) finish();
  if (blockIdx.x == 0) pdl_wait();   // a kernel that waits for this one counts on the prefix's
}

// JW warps per row (token, head) take every JW-th place, a lane four columns, and the prefix's
// parts after them.  In a fixed order, whatever the timing.
template <typename T, int ROWS, int JW>
__global__ void __launch_bounds__(kS8JoinThreads) k_join8(const __grid_constant__ Stream8Args p) {
  __shared__ float4 s_o[kS8JoinThreads / 32][32];
  __shared__ float2 s_ml[kS8JoinThreads / 32];
  const BatchAttnArgs& a = p.a;
  const int warp = threadIdx.x >> 5, share = warp % JW, lane = threadIdx.x & 31;
  // no early trigger: blocks of a next call's kernel that find room beside these are dealt
  // unevenly over the SMs and stay so (6 requests of up to 64000 keys, call after call: 93 us, 68 without)
  pdl_wait();
  const int at = blockIdx.x * (kS8JoinThreads / 32 / JW) + warp / JW, rows = a.batch.n_tokens * a.group;
  const int g = at / rows, r = at - g * rows, token = r / a.group;
  const bool in = g < a.pages.nkv;
  S8Token s = {};
  if (in) s = p.tokens[token];   // before it is known that the token has one
  // padding, and tokens of no sequence
  bool on = in && token < a.batch.q_start[a.batch.n_seqs] && token >= a.batch.q_start[0] && s.q0 >= 0 && s.q0 <= token &&
            s.shares.piece >= 1 && s.shares.less < s.shares.piece;
  const float *own = nullptr, *pre = a.part_o + (long long)at * kPartLd;
  int places = 0;
  if (on) {
    const int row = r - s.q0 * a.group, k = row / ROWS, tile = s.tile0 + k;
    const long long u = s.unit0 + (long long)k * s.units;
    const int w0 = s.shares.warp_of(u);
    places = s.units > 0 ? s.shares.warp_of(u + s.units - 1) - w0 + 1 : 0;
    on = tile >= 0 && w0 >= 0 && places >= 0 && (long long)w0 + tile + places <= p.n_places;
    own = p.places + (((long long)g * p.n_places + w0 + tile) * ROWS + row % ROWS) * kPartLd;
  }
  const long long pre_step = (long long)a.pages.nkv * rows * kPartLd;
  const int parts = on ? places + a.p_splits : 0;
  auto part = [&](int i) { return i < places ? own + (long long)i * (ROWS * kPartLd) : pre + (i - places) * pre_step; };
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float top = -INFINITY, den = 0.f;
  constexpr int U = 8;   // parts on their way at once
#pragma unroll 1
  for (int i0 = share; i0 < parts; i0 += U * JW) {
    float4 v[U];
    float2 ml[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      ml[i] = make_float2(-INFINITY, 0.f);
      if (i0 + i * JW >= parts) continue;
      const float* from = part(i0 + i * JW);
      ml[i] = *reinterpret_cast<const float2*>(from + kP8D);
      v[i] = *reinterpret_cast<const float4*>(from + 4 * lane);
    }
    float now = top;
#pragma unroll
    for (int i = 0; i < U; ++i) now = max_nan(now, ml[i].x);
    if (now == -INFINITY) continue;
    const float f = top == -INFINITY ? 0.f : exp2f(top - now);
    acc = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
    den *= f;
    top = now;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const float x = ml[i].x == -INFINITY ? 0.f : exp2f(ml[i].x - now);
      if (x == 0.f) continue;   // a part without weight counts for nothing, whatever it holds
      den += x * ml[i].y;
      acc = make_float4(acc.x + x * v[i].x, acc.y + x * v[i].y, acc.z + x * v[i].z, acc.w + x * v[i].w);
    }
  }
  if constexpr (JW > 1) {
    s_o[warp][lane] = acc;
    if (lane == 0) s_ml[warp] = make_float2(top, den);
    __syncthreads();
    if (share > 0) return;
#pragma unroll
    for (int i = 1; i < JW; ++i) top = max_nan(top, s_ml[warp + i].x);
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    den = 0.f;
#pragma unroll
    for (int i = 0; i < JW; ++i) {
      const float2 ml = s_ml[warp + i];
      const float x = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top);
      if (x == 0.f) continue;
      const float4 v = s_o[warp + i][lane];
      den += x * ml.y;
      acc = make_float4(acc.x + x * v.x, acc.y + x * v.y, acc.z + x * v.z, acc.w + x * v.w);
    }
  }
  if (on) store_row<T>(a, g, 0, r, weighted_mean(acc, den));
}

// ---- host
StreamPlan plan_stream8(long long rows, int n_seqs, int n_tokens, int nkv, const PrefixPlan& prefix, int n_sms) {
  StreamPlan p = {};
  p.tile_rows = rows <= 8ll * n_seqs ? 8 : 16;
  const int slots = p8_blocks(p.tile_rows / 8) * n_sms;
  p.blocks = std::max(1, slots / nkv);
  // the prefix's blocks have an SM each to themselves at first
  const int held = prefix.splits > 0 ? (int)std::min<long long>(n_sms, (long long)prefix.pairs * nkv * prefix.splits) : 0;
  p.early = (n_sms - held) * p8_blocks(p.tile_rows / 8) / nkv;
  p.late = held ? (int)(prefix.us * kS8UnitsPerUs) : 0;
  p.places = p.blocks * kP8Warps + n_seqs + (int)(rows / p.tile_rows);
  p.tokens_off = ((size_t)p.places * nkv * p.tile_rows * kPartLd * 4 + 255) / 256 * 256;
  p.bytes = p.tokens_off + (size_t)n_tokens * sizeof(S8Token);
  return p;
}

template <typename TQ, int NT>
static cudaError_t launch_stream8_of(const Stream8Args& p, const StreamPlan& plan, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};
  cudaError_t e = kernel_ready(ready, (const void*)k_attn_stream8<TQ, NT>, p8_smem(NT));
  if (e == cudaSuccess) e = launch(true, k_attn_stream8<TQ, NT>, dim3((unsigned)(plan.blocks * p.a.pages.nkv)), dim3(kP8Warps * 32), p8_smem(NT), st, p);
  if (e != cudaSuccess) return e;
  // few rows have many places each
  const int rows = p.a.batch.n_tokens * p.a.nq;
  if (rows <= 1024) return launch(true, k_join8<TQ, 8 * NT, 4>, dim3((unsigned)rows), dim3(kS8JoinThreads), 0, st, p);
  return launch(true, k_join8<TQ, 8 * NT, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(kS8JoinThreads), 0, st, p);
}

cudaError_t launch_stream8(const BatchAttnArgs& a, const StreamPlan& plan, void* workspace, int dtype, cudaStream_t st) {
  Stream8Args p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  p.places = (float*)workspace;
  p.tokens = (S8Token*)((uint8_t*)workspace + plan.tokens_off);
  p.n_places = plan.places;
  p.early = plan.early * kP8Warps;
  p.late = plan.late;
  if (!p8_maps(a, &p.maps)) return cudaErrorInvalidValue;
  if (dtype == OOS_DTYPE_BF16)
    return plan.tile_rows == 8 ? launch_stream8_of<__nv_bfloat16, 1>(p, plan, st) : launch_stream8_of<__nv_bfloat16, 2>(p, plan, st);
  return plan.tile_rows == 8 ? launch_stream8_of<__half, 1>(p, plan, st) : launch_stream8_of<__half, 2>(p, plan, st);
}

}  // namespace oos
