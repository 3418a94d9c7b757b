// What becomes of pages between two steps, all layers in one launch: the accepted nodes'
// move to their committed places, and copies of whole pages.
//
// Both only move bytes, scattered in pieces of a position (a page): what they cost beside
// the bytes is the chain of lookups before the first load -- offsets, nodes, page table --
// which every block walks itself.
#include <string.h>

#include <algorithm>

#include "internal.h"
#include "pages8.cuh"

namespace oos {

constexpr int kMaxMoved = 128;    // accepted nodes of a sequence
constexpr int kLayersAtOnce = 64;   // of a launch: their addresses are its arguments
constexpr int kMostLayers = 1024;

struct LayerPtrs {
  uint8_t* data[kLayersAtOnce][2];    // K, V
  uint8_t* scale[kLayersAtOnce][2];   // of 8-bit pages
};
struct CompactArgs {
  LayerPtrs l;
  BatchView batch;
  int page_size, n_pages, nkv, d, row_bytes;   // of a position
  const int32_t* accepted;
  const int32_t* accepted_len;
  int32_t* out_len;    // of the first layers' launch, else null
  int32_t* status;
};
struct CopyArgs {
  LayerPtrs l;
  long long page_bytes;
  int scale_bytes, n_pages, n, chunks;   // chunks of a page
  const int32_t* src;
  const int32_t* dst;
  int32_t* status;
};

// The places (in positions from the first page's start) of a sequence's moves: from[j] to
// to[j], j < the count returned, -1 for a sequence that is left as it is.  The block, of at
// least kMaxMoved threads.
OOS_DEV int look_up_moves(const CompactArgs& a, int seq, long long* from, long long* to) {
  const BatchView& b = a.batch;
  const int q0 = b.q_start[seq], q1 = b.q_start[seq + 1], len = b.seq_len[seq], moved = a.accepted_len[seq];
  const int n = q1 - q0, j = threadIdx.x;
  const long long first = (long long)len - n;
  bool ok = q0 >= 0 && q1 <= b.n_tokens && q0 <= q1 && n <= kMaxMoved && first >= 0 && moved >= 0 && moved <= n;
  if (ok && j < moved) {
    const int node = a.accepted[q0 + j];
    ok = node >= (j ? a.accepted[q0 + j - 1] + 1 : 0) && node < n;
    if (ok) {
      from[j] = page_slot(b, a.page_size, a.n_pages, seq, (int)(first + node));
      to[j] = page_slot(b, a.page_size, a.n_pages, seq, (int)(first + j));
      ok = from[j] >= 0 && to[j] >= 0;
    }
  }
  ok = __syncthreads_and(ok);
  if (threadIdx.x == 0) {
    if (!ok) *a.status = OOS_EBATCH;
    if (a.out_len && blockIdx.y == 0) a.out_len[seq] = ok ? (int)first + moved : len;
  }
  return ok ? moved : -1;
}

// A thread holds columns of U and takes the moves in order, eight at once.  As nodes ascend,
// node j is at j or behind it, and no later move reads what an earlier one wrote.
template <typename U>
__global__ void __launch_bounds__(kMaxMoved) k_compact(const __grid_constant__ CompactArgs a) {
  __shared__ long long from[kMaxMoved], to[kMaxMoved];
  pdl_wait();
  pdl_trigger();
  const int moved = look_up_moves(a, blockIdx.x, from, to);
  uint8_t* base = a.l.data[blockIdx.y >> 1][blockIdx.y & 1];
  for (int c = threadIdx.x * (int)sizeof(U); c < a.row_bytes; c += kMaxMoved * (int)sizeof(U)) {
#pragma unroll 1
    for (int j0 = 0; j0 < moved; j0 += 8) {
      U v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j0 + j < moved && from[j0 + j] != to[j0 + j]) v[j] = *reinterpret_cast<const U*>(base + from[j0 + j] * a.row_bytes + c);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j0 + j < moved && from[j0 + j] != to[j0 + j]) *reinterpret_cast<U*>(base + to[j0 + j] * a.row_bytes + c) = v[j];
    }
  }
}

// 8-bit pages: a warp takes heads of K and V, a lane four columns, and the blocks of positions that are
// moved into one after the other.  A block's sources lie in it or behind it, so they are as
// they were when it is its turn.  W: the lane's columns lie side by side, and move as a word.
template <bool W>
__global__ void __launch_bounds__(kMaxMoved) k_compact8(const __grid_constant__ CompactArgs a) {
  __shared__ long long from[kMaxMoved], to[kMaxMoved];
  pdl_wait();
  pdl_trigger();
  const int moved = look_up_moves(a, blockIdx.x, from, to);
  const int lane = threadIdx.x & 31, warps = kMaxMoved / 32;
  auto load = [&](const uint8_t* row) {
    if constexpr (W) return 4 * lane < a.d ? *reinterpret_cast<const uint32_t*>(row + 4 * lane) : 0u;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 32 * i < a.d) w |= (uint32_t)row[lane + 32 * i] << (8 * i);
    return w;
  };
  auto store = [&](uint8_t* row, uint32_t w) {
    if constexpr (W) {
      if (4 * lane < a.d) *reinterpret_cast<uint32_t*>(row + 4 * lane) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane + 32 * i < a.d) row[lane + 32 * i] = (uint8_t)(w >> (8 * i));
    }
  };
#pragma unroll 1
  for (int p = blockIdx.z * warps + (threadIdx.x >> 5); p < 2 * a.nkv; p += warps * gridDim.z) {
    const int h = p >> 1;
    uint8_t* head = a.l.data[blockIdx.y][p & 1] + (long long)h * a.d;
    uint8_t* scale = a.l.scale[blockIdx.y][p & 1];
    int j1;
#pragma unroll 1
    for (int j0 = 0; j0 < moved; j0 = j1) {
      const long long block = to[j0] / kScaleBlock;
      const int r0 = (int)(to[j0] % kScaleBlock);   // the block's rows r0 .. are moved into, one for each j
      j1 = min(moved, j0 + kScaleBlock - r0);
      // a lane per row of the block: where it comes from, and its exponent there
      const bool mine = lane >= r0 && lane < r0 + (j1 - j0);
      const long long src = mine ? from[j0 + lane - r0] : block * kScaleBlock + (lane & 15);
      const int e_src = scale_exp(scale[src / kScaleBlock * a.nkv + h]);
      const int own = scale_exp(scale[block * a.nkv + h]);
      // the first rows that move are on their way while their scales are looked up
      constexpr int U = 8;
      uint32_t v[U];
      auto fetch = [&](int i0) {
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (j0 + i0 + i < j1) v[i] = load(head + from[j0 + i0 + i] * a.row_bytes);
      };
      fetch(0);
      const int e = __reduce_max_sync(0xffffffffu, e_src);   // >= own: rows that stay, and lanes without one, bring it
      uint8_t* rows = head + block * kScaleBlock * a.row_bytes;
#pragma unroll 1
      for (int i0 = 0; j0 + i0 < j1; i0 += U) {
        if (i0 > 0) fetch(i0);
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int j = j0 + i0 + i;
          if (j >= j1) break;
          const int es = __shfl_sync(0xffffffffu, e_src, r0 + i0 + i);
          if (es < e) v[i] = rescale_codes4(v[i], es - e);
          if (es < e || from[j] != to[j]) store(rows + (long long)(r0 + i0 + i) * a.row_bytes, v[i]);
        }
      }
      if (e > own) {   // the rows that stay, once those that move have been read
#pragma unroll 4
        for (int r = 0; r < kScaleBlock; ++r) {
          if (r >= r0 && r < r0 + (j1 - j0)) continue;
          uint8_t* row = rows + (long long)r * a.row_bytes;
          store(row, rescale_codes4(load(row), own - e));
        }
      }
      if (lane == 0 && e > own) scale[block * a.nkv + h] = (uint8_t)(e + 127);
      __syncwarp();
    }
  }
}

constexpr int kCopyThreads = 256, kCopyLoads = 4;

template <typename U>
__global__ void __launch_bounds__(kCopyThreads) k_pages_copy(const __grid_constant__ CopyArgs a) {
  constexpr long long kChunk = (long long)kCopyThreads * kCopyLoads * sizeof(U);
  pdl_wait();
  pdl_trigger();
  const int layer = blockIdx.y >> 1, side = blockIdx.y & 1;
  uint8_t* base = a.l.data[layer][side];
  const long long units = (long long)a.n * a.chunks;
#pragma unroll 1
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int pair = (int)(u / a.chunks), chunk = (int)(u - (long long)pair * a.chunks);
    const int src = a.src[pair], dst = a.dst[pair];
    if (src < 0 || src >= a.n_pages || dst < 0 || dst >= a.n_pages) {
      if (threadIdx.x == 0) *a.status = OOS_EBATCH;
      continue;
    }
    const uint8_t* from = base + src * a.page_bytes;
    uint8_t* to = base + dst * a.page_bytes;
    const long long o = chunk * kChunk + threadIdx.x * (long long)sizeof(U);
    U v[kCopyLoads];
#pragma unroll
    for (int i = 0; i < kCopyLoads; ++i)
      if (o + i * kCopyThreads * (long long)sizeof(U) < a.page_bytes) v[i] = *reinterpret_cast<const U*>(from + o + i * kCopyThreads * (long long)sizeof(U));
#pragma unroll
    for (int i = 0; i < kCopyLoads; ++i)
      if (o + i * kCopyThreads * (long long)sizeof(U) < a.page_bytes) *reinterpret_cast<U*>(to + o + i * kCopyThreads * (long long)sizeof(U)) = v[i];
    if (chunk == 0 && a.scale_bytes > 0) {
      uint8_t* scale = a.l.scale[layer][side];
      for (int i = threadIdx.x; i < a.scale_bytes; i += kCopyThreads)
        scale[(long long)dst * a.scale_bytes + i] = scale[(long long)src * a.scale_bytes + i];
    }
  }
}

// ---- host
// what the layers of either kind of page have in common; false: they are not all of one shape
struct Layers {
  int n, page_size, n_pages, nkv, d, es;   // es: bytes of an element
  bool scaled;
  uintptr_t addresses;   // of all, or'ed together
};
static bool layers_of(const oos_paged_cache* c, int n, Layers* l) {
  *l = {n, c[0].page_size, c[0].n_pages, c[0].n_kv_heads, c[0].head_dim, dtype_ok(c[0].dtype) ? dtype_size(c[0].dtype) : 0, false, 0};
  for (int i = 0; i < n; ++i) {
    if (!pages_ok(c + i) || c[i].dtype != c[0].dtype || c[i].page_size != l->page_size || c[i].n_pages != l->n_pages ||
        c[i].n_kv_heads != l->nkv || c[i].head_dim != l->d)
      return false;
    l->addresses |= (uintptr_t)c[i].k | (uintptr_t)c[i].v;
  }
  return true;
}
static bool layers_of(const oos_paged_cache8* c, int n, Layers* l) {
  *l = {n, c[0].page_size, c[0].n_pages, c[0].n_kv_heads, c[0].head_dim, 1, true, 0};
  for (int i = 0; i < n; ++i) {
    if (!pages8_ok(c + i) || c[i].page_size != l->page_size || c[i].n_pages != l->n_pages || c[i].n_kv_heads != l->nkv ||
        c[i].head_dim != l->d)
      return false;
    l->addresses |= (uintptr_t)c[i].k | (uintptr_t)c[i].v;
  }
  return true;
}
static void fill(const oos_paged_cache* c, int n, LayerPtrs* p) {
  for (int i = 0; i < n; ++i) {
    p->data[i][0] = (uint8_t*)c[i].k;
    p->data[i][1] = (uint8_t*)c[i].v;
  }
}
static void fill(const oos_paged_cache8* c, int n, LayerPtrs* p) {
  for (int i = 0; i < n; ++i) {
    p->data[i][0] = (uint8_t*)c[i].k;
    p->data[i][1] = (uint8_t*)c[i].v;
    p->scale[i][0] = c[i].k_scale;
    p->scale[i][1] = c[i].v_scale;
  }
}

// The first block writes the new lengths while the others still read the call's arrays: n values
// at p on any of them.
static bool overlaps_batch(const oos_batch& b, const int32_t* accepted, const int32_t* accepted_len, const int32_t* status,
                           const int32_t* p) {
  const long long n = b.n_seqs;
  auto on = [&](const int32_t* q, long long m) { return (uintptr_t)p < (uintptr_t)q + 4 * m && (uintptr_t)q < (uintptr_t)p + 4 * n; };
  return on(b.q_start, n + 1) || on(b.seq_len, n) || on(b.block_table, n * b.max_pages) || on(accepted, b.n_tokens) ||
         on(accepted_len, n) || on(status, 1);
}

template <typename C>
static int compact(const C* layers, int n_layers, const oos_batch* batch, const int32_t* accepted,
                   const int32_t* accepted_len, int32_t* out_seq_len, int32_t* out_status, void* stream) {
  if (!layers || n_layers < 1 || n_layers > kMostLayers || !batch || !batch_ok(batch) || (batch->n_tokens > 0 && !accepted) || !accepted_len ||
      !out_seq_len || !out_status)
    return OOS_EINVAL;
  Layers l;
  if (!layers_of(layers, n_layers, &l)) return OOS_EINVAL;
  if (!l.es || !head_dim_ok(l.d)) return OOS_EUNSUPPORTED;
  const long long row = (long long)l.nkv * l.d * l.es;
  if (row > (1 << 24) || overlaps_batch(*batch, accepted, accepted_len, out_status, out_seq_len)) return OOS_EINVAL;
  CompactArgs a;
  memset(&a, 0, sizeof(a));
  a.batch = view_of(*batch);
  a.page_size = l.page_size;
  a.n_pages = l.n_pages;
  a.nkv = l.nkv;
  a.d = l.d;
  a.row_bytes = (int)row;
  a.accepted = accepted;
  a.accepted_len = accepted_len;
  a.status = out_status;
  const uintptr_t any = l.addresses | (uintptr_t)row;
  cudaStream_t st = (cudaStream_t)stream;
  for (int i = 0; i < n_layers; i += kLayersAtOnce) {
    const int n = std::min(kLayersAtOnce, n_layers - i);
    fill(layers + i, n, &a.l);
    a.out_len = i ? nullptr : out_seq_len;
    dim3 grid(batch->n_seqs, 2 * n);
    cudaError_t e;
    if (l.scaled) {
      // A head's side a warp: two cost as much as what they save of lookups (32 paths of up to 9,
      // 36 layers, 8 kv heads 14.3 us and 14.7; one path in one layer 3.2 and 4.6).
      grid = dim3(batch->n_seqs, n, std::min((2 * l.nkv + kMaxMoved / 32 - 1) / (kMaxMoved / 32), 64));
      const bool words = l.d % 4 == 0 && l.addresses % 4 == 0;
      e = words ? launch(true, k_compact8<true>, grid, dim3(kMaxMoved), 0, st, a)
                : launch(true, k_compact8<false>, grid, dim3(kMaxMoved), 0, st, a);
    } else {
      e = any % 16 == 0  ? launch(true, k_compact<uint4>, grid, dim3(kMaxMoved), 0, st, a)
          : any % 4 == 0 ? launch(true, k_compact<uint32_t>, grid, dim3(kMaxMoved), 0, st, a)
                         : launch(true, k_compact<uint16_t>, grid, dim3(kMaxMoved), 0, st, a);
    }
    if (e != cudaSuccess) return OOS_ECUDA;
  }
  return OOS_OK;
}

template <typename U>
static cudaError_t launch_copy(CopyArgs& a, int n_layers, cudaStream_t st) {
  constexpr long long kChunk = (long long)kCopyThreads * kCopyLoads * sizeof(U);
  const long long chunks = (a.page_bytes + kChunk - 1) / kChunk;
  if (chunks > 0x7fffffffll) return cudaErrorInvalidValue;
  a.chunks = (int)chunks;
  const long long blocks = std::min(chunks * a.n, 1ll << 20);
  return launch(true, k_pages_copy<U>, dim3((unsigned)blocks, 2 * n_layers), dim3(kCopyThreads), 0, st, a);
}

template <typename C>
static int pages_copy(const C* layers, int n_layers, const int32_t* src, const int32_t* dst, int n, int32_t* out_status,
                      void* stream) {
  if (!layers || n_layers < 1 || n_layers > kMostLayers || n < 0 || n > (1 << 20) || !out_status) return OOS_EINVAL;
  Layers l;
  if (!layers_of(layers, n_layers, &l)) return OOS_EINVAL;
  if (!l.es || !head_dim_ok(l.d)) return OOS_EUNSUPPORTED;
  const long long row = (long long)l.nkv * l.d * l.es;
  if (row > (1 << 24)) return OOS_EINVAL;
  if (n == 0) return OOS_OK;
  if (!src || !dst) return OOS_EINVAL;
  CopyArgs a;
  memset(&a, 0, sizeof(a));
  a.page_bytes = row * l.page_size;
  a.scale_bytes = 0;
  if (l.scaled) {
    const long long s = (long long)(l.page_size / kScaleBlock) * l.nkv;
    if (s > 0x7fffffffll) return OOS_EINVAL;
    a.scale_bytes = (int)s;
  }
  a.n_pages = l.n_pages;
  a.n = n;
  a.src = src;
  a.dst = dst;
  a.status = out_status;
  const uintptr_t any = l.addresses | (uintptr_t)(a.page_bytes & 15);
  cudaStream_t st = (cudaStream_t)stream;
  for (int i = 0; i < n_layers; i += kLayersAtOnce) {
    const int m = std::min(kLayersAtOnce, n_layers - i);
    fill(layers + i, m, &a.l);
    const cudaError_t e = any % 16 == 0  ? launch_copy<uint4>(a, m, st)
                          : any % 4 == 0 ? launch_copy<uint32_t>(a, m, st)
                          : any % 2 == 0 ? launch_copy<uint16_t>(a, m, st)
                                         : launch_copy<uint8_t>(a, m, st);
    if (e != cudaSuccess) return OOS_ECUDA;
  }
  return OOS_OK;
}

}  // namespace oos

using namespace oos;

extern "C" {

int oos_paged_compact(const oos_paged_cache* layers, int32_t n_layers, const oos_batch* batch, const int32_t* accepted,
                      const int32_t* accepted_len, int32_t* out_seq_len, int32_t* out_status, void* stream) {
  return compact(layers, n_layers, batch, accepted, accepted_len, out_seq_len, out_status, stream);
}
int oos_paged_compact8(const oos_paged_cache8* layers, int32_t n_layers, const oos_batch* batch,
                       const int32_t* accepted, const int32_t* accepted_len, int32_t* out_seq_len,
                       int32_t* out_status, void* stream) {
  return compact(layers, n_layers, batch, accepted, accepted_len, out_seq_len, out_status, stream);
}
int oos_pages_copy(const oos_paged_cache* layers, int32_t n_layers, const int32_t* src, const int32_t* dst, int32_t n,
                   int32_t* out_status, void* stream) {
  return pages_copy(layers, n_layers, src, dst, n, out_status, stream);
}
int oos_pages_copy8(const oos_paged_cache8* layers, int32_t n_layers, const int32_t* src, const int32_t* dst,
                    int32_t n, int32_t* out_status, void* stream) {
  return pages_copy(layers, n_layers, src, dst, n, out_status, stream);
}

}  // extern "C"
