// Views of the batch operators' arguments (heads.cu, batch_attn.cu): pages, the
// step's ragged rows, and the host's checks of both.
#pragma once

#include <atomic>

#include "common.cuh"
#include "internal.h"

namespace oos {

constexpr int kMaxHeadDim = 128;

// Rotation rates as fractions of a turn per position, in units of 2^-64: the
// product with a position, modulo 2^64, is the angle's fraction of a turn exactly,
// so that far positions need no wide floating point.
struct RopeTurns {
  unsigned long long f[kMaxHeadDim / 2];
};

// cos and sin of pos * rate, the rate in units of 2^-64 turns
OOS_DEV void turn(unsigned long long rate, int pos, float& c, float& s) {
  const unsigned long long t = (unsigned long long)(long long)pos * rate;
  const unsigned long long quarter = (t + (1ull << 61)) >> 62;
  const float x = (float)(long long)(t - (quarter << 62)) * 0x1p-63f;   // in half turns, |x| <= 1/4
  float sn, cs;
  sincospif(x, &sn, &cs);
  const float a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
  c = (quarter + 1) & 2 ? -a : a;
  s = quarter & 2 ? -b : b;
}

struct PagesView {
  uint8_t* k;
  uint8_t* v;
  int page_size, n_pages, nkv, d;
};
struct BatchView {
  int n_seqs, n_tokens, max_pages;
  const int32_t* q_start;
  const int32_t* seq_len;
  const int32_t* table;
};

bool rope_ok(const oos_rope_config* r);
bool pages_ok(const oos_paged_cache* c);
bool batch_ok(const oos_batch* b);
const RopeTurns& rope_turns(const oos_rope_config& r, int d);
int device_sms();   // of the current device, 0 without one
// Once per kernel and device: its shared memory (and, of a kernel that splits its
// registers, that it was compiled for as many as the split takes).  ready: a bit per device
cudaError_t kernel_ready(std::atomic<uint64_t>& ready, const void* kernel, int smem, int regs = 0);
inline int dtype_size(int dtype) { return dtype == OOS_DTYPE_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype >= OOS_DTYPE_F32 && dtype <= OOS_DTYPE_F16; }
inline bool head_dim_ok(int d) { return d >= 2 && d <= kMaxHeadDim && d % 2 == 0; }
inline PagesView view_of(const oos_paged_cache& c) {
  return {(uint8_t*)c.k, (uint8_t*)c.v, c.page_size, c.n_pages, c.n_kv_heads, c.head_dim};
}
inline BatchView view_of(const oos_batch& b) {
  return {b.n_seqs, b.n_tokens, b.max_pages, b.q_start, b.seq_len, b.block_table};
}

// Entries a[1 .. n] that are <= x (a not decreasing): the whole warp, 31 probes and
// a vote per round.  Whatever a holds, the result lies in [0, n].
template <typename F>
OOS_DEV int warp_count_le(int n, F value, long long x) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;   // a[lo] <= x (or lo is 0) and a[hi + 1] > x (or hi is n)
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + (lane + 1) * step;
    const bool le = at <= hi && value(at) <= x;
    const int k = __popc(__ballot_sync(0xffffffffu, le));
    hi = min(hi, lo + (k + 1) * step - 1);
    lo = min(hi, lo + k * step);
  }
  return lo;
}

// Entry of the page table and place in the pages of position s of sequence b, in
// positions from the first page's start; -1: no such page.
OOS_DEV long long page_slot(const BatchView& b, int page_size, int n_pages, int seq, int s) {
  const int col = s / page_size;
  if (s < 0 || col >= b.max_pages) return -1;
  const int page = __ldg(b.table + (size_t)seq * b.max_pages + col);
  if (page < 0 || page >= n_pages) return -1;
  return (long long)page * page_size + (s - col * page_size);
}

OOS_DEV float to_f32(__half v) { return __half2float(v); }
template <typename T>
OOS_DEV T from_f32(float v);
template <>
OOS_DEV float from_f32<float>(float v) { return v; }
template <>
OOS_DEV __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
OOS_DEV __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N elements as one access (N * sizeof(T) is 16, 8 or the element)
template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};
template <typename T, int N>
OOS_DEV void load_vec(const T* p, float (&v)[N]) {
  const Vec<T, N> r = *reinterpret_cast<const Vec<T, N>*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = to_f32(r.v[i]);
}
template <typename T, int N>
OOS_DEV void store_vec(T* p, const float (&v)[N]) {
  Vec<T, N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = from_f32<T>(v[i]);
  *reinterpret_cast<Vec<T, N>*>(p) = r;
}

}  // namespace oos
