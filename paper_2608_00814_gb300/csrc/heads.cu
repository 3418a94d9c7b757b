// Per-head operators of a batch step: RMSNorm of q and k heads with the position
// rotation in the same pass, and the append of K (normed and turned on the way)
// and V to pages.
//
// One head x of d values becomes y = x * rsqrt(mean(x^2) + eps) * gain, and the
// pair (y_m, y_{m+d/2}) turns by a_m = position * rate_m.  Both are one pass over
// memory: a few lanes hold a head, each of them chunks of VEC values of the first
// half and the same chunks of the second, so that every pair is in one lane, the
// norm is a few shuffles and nothing goes through shared memory.  Bound by HBM.
//
// Angles: rate_m / 2 pi is kept as a 64-bit fraction of a turn; times the position
// modulo 2^64 it is the angle's fraction of a turn by integer products alone, off by what
// the rate is off as a double: 2^-55 of a turn per position, 2^-24 at 2^31.  The nearest
// quarter turn comes off exactly, so the fp32 sine and cosine see at most an
// eighth of a turn.  A warp forms each of a token's angles once, dealt over its lanes,
// hands them round by shuffles and keeps them over its heads.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "batch.cuh"

namespace oos {

constexpr int kHeadWarps = 4;      // tokens per block, a warp each
constexpr int kMaxSlices = 1024;   // warps a token's heads are dealt to

struct HeadArgs {
  int n, d, d2;                   // tokens, head size and half of it
  int heads[2];                   // q and k heads (append: 0 and the K heads)
  const void* in[2];
  long long in_stride[2];         // elements
  const void* gain[2];
  void* out[2];
  long long out_stride[2];
  const int32_t* positions;       // nullptr: no rotation
  float eps;
  // append
  const void* v;
  long long v_stride;
  PagesView pages;
  BatchView batch;
  int32_t* status;
};

// T: elements of the inputs and gains, O: of the outputs.  VEC: values per access.
// LANES: lanes per head, NC: chunks of half a head per lane.  APPEND: in[1] goes to
// the pages' K, v to their V.
template <typename T, typename O, int VEC, int LANES, int NC, bool APPEND>
__global__ void __launch_bounds__(kHeadWarps * 32, 4) k_heads(const HeadArgs a, const __grid_constant__ RopeTurns rope) {
  pdl_wait();      // the kernel before may be another call's
  pdl_trigger();   // the next one's launch runs under this one: 2048 tokens 11.8 us a call, 13.2 launched without
  const int lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * kHeadWarps + (threadIdx.x >> 5);
  const int slice = blockIdx.y, slices = gridDim.y;
  if (t >= a.n) return;
  constexpr int GROUPS = 32 / LANES;   // heads of the warp at once
  // Heads in flight per lane, and so registers, against warps: 4 without V (15001 tokens
  // of 40 binary16 heads: 49 us, 92 % of the copy's rate; 2: 60), 2 with it (12600 tokens
  // of 8 heads: 25.5 us, 4: 32).
  constexpr int U = NC * VEC > 8 ? 1 : APPEND ? 2 : 4;
  const int sub = lane % LANES, group = lane / LANES;
  const int pos = a.positions ? a.positions[t] : 0;
  // heads [h0, h1) of this warp, counted over q's and k's
  const int total = a.heads[0] + a.heads[1];
  const int h0 = (int)((unsigned)(total * slice) / slices), h1 = (int)((unsigned)(total * (slice + 1)) / slices);
  auto first = [&](int side) { return max(0, h0 - (side ? a.heads[0] : 0)); };
  auto past = [&](int side) { return min(a.heads[side], h1 - (side ? a.heads[0] : 0)); };
  Vec<T, VEC> x[U][NC][2];
  auto load = [&](int side, int h) {
    const T* in = (const T*)a.in[side] + t * a.in_stride[side];
    const int hi = past(side);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int hh = h + u * GROUPS + group, m = (c * LANES + sub) * VEC;
        const T* p = in + (long long)hh * a.d + m;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          x[u][c][half] = Vec<T, VEC>();
          if (hh < hi && m < a.d2) x[u][c][half] = *reinterpret_cast<const Vec<T, VEC>*>(p + half * a.d2);
        }
      }
  };
  // the first heads' loads go out before everything that waits: an appended row's lookups
  // follow each other through four of them
  const int side0 = APPEND || h0 >= a.heads[0] ? 1 : 0;
  load(side0, first(side0));
  Vec<T, VEC> v[4];
  const T* vin = nullptr;
  int v_chunks = 0;
  if (APPEND) {
    vin = (const T*)a.v + t * a.v_stride + (long long)first(1) * a.d;
    v_chunks = max(0, past(1) - first(1)) * a.d / VEC;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (lane + 32 * u < v_chunks) v[u] = *reinterpret_cast<const Vec<T, VEC>*>(vin + (lane + 32 * u) * VEC);
  }
  // where an appended row goes (the whole warp; a row without a place is left out)
  long long slot = 0;
  if (APPEND) {
    const BatchView& b = a.batch;
    const int seq = warp_count_le(b.n_seqs, [&](int i) { return (long long)b.q_start[i]; }, t);
    if (seq >= b.n_seqs) return;                       // behind the last sequence
    const int q0 = b.q_start[seq], q1 = b.q_start[seq + 1];
    const long long at = (long long)b.seq_len[seq] - (q1 - t);   // a length may be any 32 bits
    slot = t < q0 || t >= q1 || at < 0 ? -1 : page_slot(b, a.pages.page_size, a.pages.n_pages, seq, (int)at);
    if (slot < 0) {
      if (lane == 0) *a.status = OOS_EBATCH;
      return;
    }
  }
  // a lane's pairs, counted over its chunks: (c * LANES + sub) * VEC + i, p = c * VEC + i
  float cs[NC * VEC], sn[NC * VEC];
  if (a.positions) {
    constexpr int MINE = (NC * VEC + GROUPS - 1) / GROUPS;   // group g forms pairs p = g, g + GROUPS, ..
    float mc[MINE], ms[MINE];
#pragma unroll
    for (int k = 0; k < MINE; ++k) {
      const int p = k * GROUPS + group, m = (p / VEC * LANES + sub) * VEC + p % VEC;
      mc[k] = 1.f;
      ms[k] = 0.f;
      if (p < NC * VEC && m < a.d2) turn(rope.f[m], pos, mc[k], ms[k]);
    }
#pragma unroll
    for (int p = 0; p < NC * VEC; ++p) {
      cs[p] = __shfl_sync(0xffffffffu, mc[p / GROUPS], p % GROUPS * LANES + sub);
      sn[p] = __shfl_sync(0xffffffffu, ms[p / GROUPS], p % GROUPS * LANES + sub);
    }
  }
  bool loaded = true;
#pragma unroll 1
  for (int side = side0; side < 2; ++side) {
    const int lo = first(side), hi = past(side);
    if (lo >= hi) continue;
    O* out = APPEND ? (O*)a.pages.k + slot * a.pages.nkv * a.d : (O*)a.out[side] + t * a.out_stride[side];
    const T* gain = (const T*)a.gain[side];
    Vec<T, VEC> g[NC][2];
    if (gain) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int m = (c * LANES + sub) * VEC;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < VEC; ++i)   // element by element: a gain may start anywhere
            if (m < a.d2) g[c][half].v[i] = gain[half * a.d2 + m + i];
      }
    }
#pragma unroll 1
    for (int h = lo; h < hi; h += U * GROUPS) {
      if (!loaded) load(side, h);
      loaded = false;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u * GROUPS >= hi) break;   // warp-uniform
        float r = 1.f;
        if (gain) {
          float ss = 0.f;
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const float lo_ = to_f32(x[u][c][0].v[i]), hi_ = to_f32(x[u][c][1].v[i]);
              ss += lo_ * lo_ + hi_ * hi_;
            }
#pragma unroll
          for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          r = rsqrtf(ss / (float)a.d + a.eps);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int hh = h + u * GROUPS + group, m = (c * LANES + sub) * VEC;
          float y[2][VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            float lo_ = to_f32(x[u][c][0].v[i]), hi_ = to_f32(x[u][c][1].v[i]);
            if (gain) {
              lo_ = lo_ * r * to_f32(g[c][0].v[i]);
              hi_ = hi_ * r * to_f32(g[c][1].v[i]);
            }
            const int p = c * VEC + i;
            y[0][i] = a.positions ? lo_ * cs[p] - hi_ * sn[p] : lo_;
            y[1][i] = a.positions ? hi_ * cs[p] + lo_ * sn[p] : hi_;
          }
          if (hh < hi && m < a.d2) {
            store_vec<O, VEC>(out + (long long)hh * a.d + m, y[0]);
            store_vec<O, VEC>(out + (long long)hh * a.d + a.d2 + m, y[1]);
          }
        }
      }
    }
  }
  if (APPEND) {   // the same heads of V, four accesses in flight
    O* vout = (O*)a.pages.v + slot * a.pages.nkv * a.d + (long long)first(1) * a.d;
#pragma unroll 1
    for (int i0 = lane; i0 < v_chunks; i0 += 4 * 32) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i0 + 32 * u >= v_chunks) continue;
        if (i0 != lane) v[u] = *reinterpret_cast<const Vec<T, VEC>*>(vin + (i0 + 32 * u) * VEC);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i0 + 32 * u >= v_chunks) continue;
        float y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = to_f32(v[u].v[i]);
        store_vec<O, VEC>(vout + (i0 + 32 * u) * VEC, y);
      }
    }
  }
}

bool rope_ok(const oos_rope_config* r) {
  if (!(r->theta > 0.f) || !(r->theta < INFINITY) || !(r->factor == r->factor)) return false;
  return r->factor <= 1.f || (r->low_freq_factor > 0.f && r->high_freq_factor > r->low_freq_factor && r->orig_max_pos >= 1);
}

// A layer's calls come with one configuration: its table of powers is kept per thread.
const RopeTurns& rope_turns(const oos_rope_config& r, int d) {
  static thread_local struct {
    oos_rope_config r;
    int d = 0;
    RopeTurns turns;
  } last;
  if (last.d == d && memcmp(&last.r, &r, sizeof(r)) == 0) return last.turns;
  for (int m = 0; m < kMaxHeadDim / 2; ++m) {
    last.turns.f[m] = 0;
    if (m >= d / 2) continue;
    const double f = rope_rate(r.theta, m, d, r.factor, r.low_freq_factor, r.high_freq_factor, r.orig_max_pos);
    const double t = f / (2.0 * M_PI);
    last.turns.f[m] = (unsigned long long)ldexp(t - floor(t), 64);   // t - floor(t) <= 1 - 2^-53
  }
  last.r = r;
  last.d = d;
  return last.turns;
}

bool pages_ok(const oos_paged_cache* c) {
  return c->n_kv_heads >= 1 && c->page_size >= 1 && c->n_pages >= 1 && c->k && c->v;
}
bool batch_ok(const oos_batch* b) {
  return b->n_seqs >= 1 && b->n_seqs <= (1 << 30) && b->n_tokens >= 0 && b->max_pages >= 1 && b->q_start && b->seq_len && b->block_table;
}

// Rows of the widest access: 16 bytes of T (and the same count of O) where half a
// head divides into them and every row starts on such a boundary, else one element.
static bool wide(const HeadArgs& a, int es, int vec, int out_es) {
  if (a.d2 % vec) return false;
  auto rows = [&](const void* p, long long stride, int es_) {
    return ((uintptr_t)p % (vec * es_)) == 0 && (stride * es_) % (vec * es_) == 0;
  };
  bool ok = true;
  for (int s = 0; s < 2; ++s) {
    if (a.heads[s] && a.in[s]) ok = ok && rows(a.in[s], a.in_stride[s], es);
    if (a.heads[s] && a.out[s]) ok = ok && rows(a.out[s], a.out_stride[s], out_es);
  }
  if (a.v) ok = ok && rows(a.v, a.v_stride, es) && rows(a.pages.k, 0, out_es) && rows(a.pages.v, 0, out_es);
  return ok;
}

template <typename T, typename O, int VEC, int LANES, int NC, bool APPEND>
static cudaError_t launch_heads_of(HeadArgs& a, const RopeTurns& rope, cudaStream_t st) {
  const int sms = device_sms();
  if (sms <= 0) return cudaErrorInvalidDevice;
  // A token's heads go to as many warps as it takes to give every SM 16, so that a
  // few tokens are spread out while many share the angles over all their heads (2048
  // tokens of 40 heads, in a graph: 10.7 us, 11.4 with 32 warps, 13.9 with 48).
  const int total = a.heads[0] + a.heads[1], most = (total * LANES + 31) / 32;
  const int fit = 0x7fffffff / total;   // the kernel deals the heads by total * slices in 32 bits
  const int slices = (int)std::max(1ll, std::min<long long>(std::min({most, kMaxSlices, fit}), 16ll * sms / a.n));
  const dim3 grid((unsigned)((a.n + (long long)kHeadWarps - 1) / kHeadWarps), slices);
  return launch(true, k_heads<T, O, VEC, LANES, NC, APPEND>, grid, dim3(kHeadWarps * 32), 0, st, a, rope);
}

template <typename T, typename O, bool APPEND>
static cudaError_t launch_heads(HeadArgs& a, const RopeTurns& rope, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);   // half a head is at most 8 chunks of 8 or 16 of 4
  if (wide(a, sizeof(T), V, sizeof(O))) {
    const int chunks = a.d2 / V;
    if (chunks <= 4) return launch_heads_of<T, O, V, 4, 1, APPEND>(a, rope, st);
    if (chunks <= 8) return launch_heads_of<T, O, V, 8, 1, APPEND>(a, rope, st);
    return launch_heads_of<T, O, V, 16, 1, APPEND>(a, rope, st);
  }
  if (a.d2 > 32) return launch_heads_of<T, O, 1, 32, 2, APPEND>(a, rope, st);
  return launch_heads_of<T, O, 1, 32, 1, APPEND>(a, rope, st);
}

template <typename T>
static cudaError_t launch_append(int out_dtype, HeadArgs& a, const RopeTurns& rope, cudaStream_t st) {
  if (out_dtype == OOS_DTYPE_F32) return launch_heads<T, float, true>(a, rope, st);
  if (out_dtype == OOS_DTYPE_BF16) return launch_heads<T, __nv_bfloat16, true>(a, rope, st);
  return launch_heads<T, __half, true>(a, rope, st);
}

}  // namespace oos

using namespace oos;

extern "C" {

int oos_qk_norm_rope(int32_t dtype, int32_t n, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* q,
                     int64_t q_stride, const void* k, int64_t k_stride, const void* q_norm, const void* k_norm,
                     float eps, const oos_rope_config* rope, const int32_t* positions, void* q_out,
                     int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
  if (n < 0 || n_q_heads < 0 || n_kv_heads < 0 || n_q_heads + (long long)n_kv_heads < 1 ||
      n_q_heads + (long long)n_kv_heads > (1 << 20) || !(eps >= 0.f))
    return OOS_EINVAL;
  if (!dtype_ok(dtype) || !head_dim_ok(head_dim)) return OOS_EUNSUPPORTED;
  if (rope && !rope_ok(rope)) return OOS_EINVAL;
  if (n == 0) return OOS_OK;
  const long long qw = (long long)n_q_heads * head_dim, kw = (long long)n_kv_heads * head_dim;
  if (n_q_heads && (!q || !q_out || q_stride < qw || q_out_stride < qw)) return OOS_EINVAL;
  if (n_kv_heads && (!k || !k_out || k_stride < kw || k_out_stride < kw)) return OOS_EINVAL;
  if (rope && !positions) return OOS_EINVAL;
  HeadArgs a = {};
  a.n = n;
  a.d = head_dim;
  a.d2 = head_dim / 2;
  a.heads[0] = n_q_heads;
  a.heads[1] = n_kv_heads;
  a.in[0] = q;
  a.in[1] = k;
  a.in_stride[0] = q_stride;
  a.in_stride[1] = k_stride;
  a.gain[0] = q_norm;
  a.gain[1] = k_norm;
  a.out[0] = q_out;
  a.out[1] = k_out;
  a.out_stride[0] = q_out_stride;
  a.out_stride[1] = k_out_stride;
  a.positions = rope ? positions : nullptr;
  a.eps = eps;
  static const RopeTurns none = {};
  const RopeTurns& turns = rope ? rope_turns(*rope, head_dim) : none;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = dtype == OOS_DTYPE_F32    ? launch_heads<float, float, false>(a, turns, st)
                        : dtype == OOS_DTYPE_BF16 ? launch_heads<__nv_bfloat16, __nv_bfloat16, false>(a, turns, st)
                                                  : launch_heads<__half, __half, false>(a, turns, st);
  return e == cudaSuccess ? OOS_OK : OOS_ECUDA;
}

int oos_paged_append(const oos_paged_cache* cache, const oos_batch* batch, int32_t dtype, const void* k,
                     int64_t k_stride, const void* v, int64_t v_stride, const void* k_norm, float eps,
                     const oos_rope_config* rope, const int32_t* positions, int32_t* out_status, void* stream) {
  if (!cache || !batch || !pages_ok(cache) || !batch_ok(batch) || !out_status || !(eps >= 0.f)) return OOS_EINVAL;
  if (!dtype_ok(dtype) || !dtype_ok(cache->dtype) || !head_dim_ok(cache->head_dim)) return OOS_EUNSUPPORTED;
  if (rope && !rope_ok(rope)) return OOS_EINVAL;
  if (batch->n_tokens == 0) return OOS_OK;
  const long long w = (long long)cache->n_kv_heads * cache->head_dim;
  if (!k || !v || k_stride < w || v_stride < w || w > (1 << 24)) return OOS_EINVAL;
  if (rope && !positions) return OOS_EINVAL;
  HeadArgs a = {};
  a.n = batch->n_tokens;
  a.d = cache->head_dim;
  a.d2 = cache->head_dim / 2;
  a.heads[1] = cache->n_kv_heads;
  a.in[1] = k;
  a.in_stride[1] = k_stride;
  a.gain[1] = k_norm;
  a.v = v;
  a.v_stride = v_stride;
  a.positions = rope ? positions : nullptr;
  a.eps = eps;
  a.pages = view_of(*cache);
  a.batch = view_of(*batch);
  a.status = out_status;
  static const RopeTurns none = {};
  const RopeTurns& turns = rope ? rope_turns(*rope, cache->head_dim) : none;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = dtype == OOS_DTYPE_F32    ? launch_append<float>(cache->dtype, a, turns, st)
                        : dtype == OOS_DTYPE_BF16 ? launch_append<__nv_bfloat16>(cache->dtype, a, turns, st)
                                                  : launch_append<__half>(cache->dtype, a, turns, st);
  return e == cudaSuccess ? OOS_OK : OOS_ECUDA;
}

}  // extern "C"
