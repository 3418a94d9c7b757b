// Append of a step's K (normed and turned on the way) and V to 8-bit pages.
//
// A scale belongs to 16 positions of a head, so a warp takes one such block of K or V: its
// rows (up to 16) are loaded, K's are normed and turned as in heads.cu, all stay in
// registers as fp32 while their largest magnitude is found, and are rounded once to the
// scale it needs.  A block of threads holds heads of K (or of V) at the same positions, whose
// angles it forms once, in shared memory.
//
// Where the block held positions before, its scale may only grow, as the codes there would
// gain nothing by a smaller one; when it does, they are read, divided by a power of two and
// rounded again.
//
// Bytes: the rows read once and half (a quarter) as many written.  12600 rows of 8 heads in 24
// sequences: 26 us with rotation alone, 2.7 TB/s (28 normed, fp32 28): not bound by bytes but by
// some 1100 instructions a warp, sixteen warps an SM, as a block's rows stay in registers.  Two
// warps a head in half the registers took 30 to 40 us, three blocks an SM (spilled) 29, four
// heads a block (their angles formed twice as often) 28.  One token of 64 sequences: 4.7 us.
#include <math.h>

#include <algorithm>

#include "internal.h"
#include "pages8.cuh"

namespace oos {

constexpr int kApMaxHeads = 8;   // of a block, a warp each

struct Append8Args {
  Pages8View pages;
  BatchView batch;
  const void* in[2];   // K, V
  long long stride[2];
  const void* gain;
  const int32_t* positions;   // nullptr: no rotation
  float eps;
  int32_t* status;
};

// A code's steps are 2^20 of fp32's, and where a value lies next to the border of two codes
// fp32's own error chooses between them.  For the larger element of a turned pair that is not
// normed it is at most 6.5 half steps of fp32 (2^-24) of the pair's length -- cosine and sine
// 2.5 each, their products and the sum 1.5 -- and so 9.2 steps of its own, as the length is at
// most 2^1/2 of it.  Within ten steps of a border of normal codes such a pair, one in 50000,
// is computed in 64 bits, by a few instructions a pair (no difference in the times above; 0.5
// us where one of 64 tokens' has to be): the bits below a code's tell it, whatever the scale.
// Elsewhere the error chooses.  To find every such value both ends of what it may be would have
// to be rounded, and a third of the normed warps compute one again (35 us, 52 normed); either
// code is as near as the other to 2^-20 of the pair's length.
constexpr uint32_t kBorderSteps = 10;
OOS_DEV uint32_t from_border(float larger) {   // at most 2 kBorderSteps << 12: within that of one
  return (__float_as_uint(larger) - (0x80000u - kBorderSteps)) << 12;
}
// a value of 64 bits so that rounding it again to few bits gives what rounding once does
OOS_DEV float round_to_odd(double v) {
  const float f = __double2float_rz(v);
  return (double)f == v || isnan(v) ? f : __uint_as_float(__float_as_uint(f) | 1u);
}
static __device__ __noinline__ double2 turn64(unsigned long long rate, int pos) {   // cos, sin
  double s, c;
  sincospi((double)(long long)((unsigned long long)(long long)pos * rate) * 0x1p-63, &s, &c);
  return make_double2(c, s);
}

// T: elements of the rows.  A row's half is dealt in chunks of VEC to LANES lanes, NC each;
// 32 / LANES rows at once.  SEARCH: K is turned and not normed.
template <typename T, int VEC, int LANES, int NC, bool SEARCH>
__global__ void __launch_bounds__(kApMaxHeads * 32, 2) k_append8(const Append8Args a, const __grid_constant__ RopeTurns rope) {
  constexpr int ROWS = 32 / LANES, PASSES = kScaleBlock / ROWS;
  // of element m = (c LANES + sub) VEC + i of a half: at (c VEC + i) LANES + sub, so that a
  // row's lanes read neighbours
  __shared__ float2 s_turn[kScaleBlock][NC * LANES * VEC];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, heads = blockDim.x / 32;
  const int d = a.pages.p.d, d2 = d / 2, nkv = a.pages.p.nkv;
  const int side = blockIdx.y & 1, h = (blockIdx.y >> 1) * heads + warp;   // 0: K, 1: V
  pdl_wait();
  pdl_trigger();
  // Sequence b's blocks of positions are numbered from 2 b + floor(q_start[b] / 16): a count
  // known without a scan, at the price of numbers that have none.
  const BatchView& b = a.batch;
  auto start = [&](int s) { return 2ll * s + b.q_start[s] / kScaleBlock; };
  const int seq = warp_count_le(b.n_seqs - 1, start, blockIdx.x);
  const int q0 = b.q_start[seq], q1 = b.q_start[seq + 1], len = b.seq_len[seq];
  const bool in_order = q0 >= 0 && q1 <= b.n_tokens && q0 <= q1;
  const long long before = (long long)len - (q1 - q0);
  if ((!in_order || before < 0) && threadIdx.x == 0) *a.status = OOS_EBATCH;
  if (!in_order || (long long)blockIdx.x < start(seq)) return;
  const long long p0 = (max(before, 0ll) / kScaleBlock + (blockIdx.x - start(seq))) * kScaleBlock;
  if (p0 >= len || q0 == q1) return;
  const long long slot = page_slot(b, a.pages.p.page_size, a.pages.p.n_pages, seq, (int)p0);
  if (slot < 0) {   // the whole block of threads
    if (threadIdx.x == 0) *a.status = OOS_EBATCH;
    return;
  }
  const int lo = (int)max(0ll, before - p0), hi = (int)min((long long)kScaleBlock, len - p0);   // its rows of this step
  const long long t0 = q0 + (p0 - before);   // token of the block's first position
  const int sub = lane % LANES, group = lane / LANES;
  float y[PASSES][NC][2][VEC];
  {
    const T* in = (const T*)a.in[side];
    Vec<T, VEC> x[PASSES][NC][2];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = p * ROWS + group;
      const T* row = in + (t0 + r) * a.stride[side] + (long long)h * d;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int m = (c * LANES + sub) * VEC;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          x[p][c][half] = Vec<T, VEC>();
          if (h < nkv && r >= lo && r < hi && m < d2) x[p][c][half] = *reinterpret_cast<const Vec<T, VEC>*>(row + half * d2 + m);
        }
      }
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < VEC; ++i) y[p][c][half][i] = to_f32(x[p][c][half].v[i]);
  }
  uint8_t* scale = (side ? a.pages.v_scale : a.pages.k_scale) + slot / kScaleBlock * nkv + h;
  const bool begun = lo == 0 && before <= p0;
  int old = kScaleLow;
  if (!begun && h < nkv) old = scale_exp(*scale);
  if (a.positions && side == 0) {
    for (int i = threadIdx.x; i < (hi - lo) * d2; i += blockDim.x) {
      const int r = lo + i / d2, m = i % d2;
      float c, s;
      turn(rope.f[m], a.positions[t0 + r], c, s);
      const int chunk = m / VEC;
      s_turn[r][(chunk / LANES * VEC + m % VEC) * LANES + chunk % LANES] = make_float2(c, s);
    }
    __syncthreads();
  }
  if (h >= nkv) return;
  uint32_t near = 0;   // passes with pairs next to a border
  if (side == 0) {
    const T* gain = SEARCH ? nullptr : (const T*)a.gain;
    float g[NC][2][VEC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {   // element by element: a gain may start anywhere
          const int m = (c * LANES + sub) * VEC;
          g[c][half][i] = gain && m < d2 ? to_f32(gain[half * d2 + m + i]) : 1.f;
        }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = p * ROWS + group;
      if (p * ROWS + ROWS <= lo || p * ROWS >= hi) continue;   // warp-uniform
      float f = 1.f;
      if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < VEC; ++i) ss += y[p][c][0][i] * y[p][c][0][i] + y[p][c][1][i] * y[p][c][1][i];
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        f = rsqrtf(ss / (float)d + a.eps);
      }
      uint32_t least = ~0u;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const int m = (c * LANES + sub) * VEC + i;
          float lo_ = y[p][c][0][i], hi_ = y[p][c][1][i];
          if (gain) {
            lo_ = lo_ * f * g[c][0][i];
            hi_ = hi_ * f * g[c][1][i];
          }
          if ((SEARCH || a.positions) && m < d2 && r >= lo && r < hi) {
            const float2 cs = s_turn[r][(c * VEC + i) * LANES + sub];
            const float turned = lo_ * cs.x - hi_ * cs.y;
            hi_ = hi_ * cs.x + lo_ * cs.y;
            lo_ = turned;
            if (SEARCH) least = min(least, from_border(fmaxf(fabsf(lo_), fabsf(hi_))));
          }
          y[p][c][0][i] = lo_;
          y[p][c][1][i] = hi_;
        }
      if (SEARCH) near |= (least <= 2 * kBorderSteps << 12 ? 1u : 0u) << p;
    }
  }
  float amax = 0.f;   // of what is finite in the block's rows; the others' are zeros
#pragma unroll
  for (int p = 0; p < PASSES; ++p)
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < VEC; ++i) amax = fmaxf(amax, fabsf(y[p][c][half][i]));   // passes a NaN by
  amax = warp_max(amax);
  if (amax == INFINITY) {   // once more, with what is infinite as NaN
    amax = 0.f;
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            y[p][c][half][i] = finite_or_nan(y[p][c][half][i]);
            amax = fmaxf(amax, fabsf(y[p][c][half][i]));
          }
    amax = warp_max(amax);
  }
  const int e = max(old, needed_exp(amax));
  uint8_t* codes = (side ? a.pages.p.v : a.pages.p.k) + slot * nkv * d + (long long)h * d;
  if (!begun && e > old) {   // the positions from before, and what lies behind the step's
    for (int r = 0; r < kScaleBlock; ++r) {
      if (r >= lo && r < hi) continue;
      uint8_t* row = codes + (long long)r * nkv * d;
      if constexpr (VEC >= 4) {
        if (4 * lane < d) {
          uint32_t* w = reinterpret_cast<uint32_t*>(row + 4 * lane);
          *w = rescale_codes4(*w, old - e);
        }
      } else {
        for (int c = lane; c < d; c += 32) row[c] = (uint8_t)rescale_codes4(row[c], old - e);
      }
    }
  }
  const float inv = pow2f(-e);
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int r = p * ROWS + group;
    if (r < lo || r >= hi) continue;
    uint8_t* row = codes + (long long)r * nkv * d;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int m = (c * LANES + sub) * VEC;
        if (m >= d2) continue;
        float v[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = y[p][c][half][i] * inv;
        if constexpr (VEC == 1) {
          row[half * d2 + m] = (uint8_t)f32x2_e4m3(v[0], 0.f);
        } else {
          Vec<uint16_t, VEC / 2> w;
#pragma unroll
          for (int i = 0; i < VEC / 2; ++i) w.v[i] = f32x2_e4m3(v[2 * i], v[2 * i + 1]);
          *reinterpret_cast<Vec<uint16_t, VEC / 2>*>(row + half * d2 + m) = w;
        }
      }
  }
  if constexpr (SEARCH) {
    // a lane's pairs of a row, a lane each, over the codes that are written
    uint32_t who = __ballot_sync(0xffffffffu, near != 0);
    if (who) __syncwarp();
#pragma unroll 1
    for (; who; who &= who - 1) {
      const int from = __ffs(who) - 1, m = (lane / VEC * LANES + from % LANES) * VEC + lane % VEC;
#pragma unroll 1
      for (uint32_t passes = __shfl_sync(0xffffffffu, near, from); passes; passes &= passes - 1) {
        const int r = (__ffs(passes) - 1) * ROWS + from / LANES;
        if (lane >= NC * VEC || m >= d2) continue;
        const T* row = (const T*)a.in[0] + (t0 + r) * a.stride[0] + (long long)h * d + m;
        uint8_t* to = codes + (long long)r * nkv * d + m;
        const double u = to_f32(row[0]), w = to_f32(row[d2]);
        const double2 cs = turn64(rope.f[m], a.positions[t0 + r]);
        // what fp32 passed stays NaN
        if ((to[0] & 0x7f) != 0x7f) to[0] = (uint8_t)f32x2_e4m3(round_to_odd((u * cs.x - w * cs.y) * (double)inv), 0.f);
        if ((to[d2] & 0x7f) != 0x7f) to[d2] = (uint8_t)f32x2_e4m3(round_to_odd((w * cs.x + u * cs.y) * (double)inv), 0.f);
      }
    }
  }
  if (lane == 0 && (begun || e > old)) *scale = (uint8_t)(e + 127);
}

template <typename T, int VEC, int LANES, int NC>
static cudaError_t launch_append8_of(const Append8Args& a, const RopeTurns& rope, cudaStream_t st) {
  const int heads = std::min(a.pages.p.nkv, kApMaxHeads);
  const long long blocks = 2ll * a.batch.n_seqs + a.batch.n_tokens / kScaleBlock;
  const dim3 grid((unsigned)blocks, 2u * (unsigned)((a.pages.p.nkv + heads - 1) / heads));
  return a.positions && !a.gain ? launch(true, k_append8<T, VEC, LANES, NC, true>, grid, dim3(32 * heads), 0, st, a, rope)
                                : launch(true, k_append8<T, VEC, LANES, NC, false>, grid, dim3(32 * heads), 0, st, a, rope);
}

template <typename T>
static cudaError_t launch_append8(const Append8Args& a, const RopeTurns& rope, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  const int d2 = a.pages.p.d / 2;
  bool wide = d2 % V == 0 && ((uintptr_t)a.pages.p.k | (uintptr_t)a.pages.p.v) % V == 0;
  for (int s = 0; s < 2; ++s) wide = wide && (uintptr_t)a.in[s] % 16 == 0 && a.stride[s] * sizeof(T) % 16 == 0;
  if (wide) {
    const int chunks = d2 / V;
    if (chunks <= 4) return launch_append8_of<T, V, 4, 1>(a, rope, st);
    if constexpr (V == 4)
      if (chunks > 8) return launch_append8_of<T, V, 16, 1>(a, rope, st);
    return launch_append8_of<T, V, 8, 1>(a, rope, st);   // d <= 128
  }
  if (d2 > 32) return launch_append8_of<T, 1, 32, 2>(a, rope, st);
  return launch_append8_of<T, 1, 32, 1>(a, rope, st);
}

}  // namespace oos

using namespace oos;

extern "C" int oos_paged_append8(const oos_paged_cache8* cache, const oos_batch* batch, int32_t dtype, const void* k,
                                 int64_t k_stride, const void* v, int64_t v_stride, const void* k_norm, float eps,
                                 const oos_rope_config* rope, const int32_t* positions, int32_t* out_status,
                                 void* stream) {
  if (!cache || !batch || !pages8_ok(cache) || !batch_ok(batch) || !out_status || !(eps >= 0.f)) return OOS_EINVAL;
  if (!dtype_ok(dtype) || !head_dim_ok(cache->head_dim)) return OOS_EUNSUPPORTED;
  if (rope && !rope_ok(rope)) return OOS_EINVAL;
  if (batch->n_tokens == 0) return OOS_OK;
  const long long w = (long long)cache->n_kv_heads * cache->head_dim;
  if (!k || !v || k_stride < w || v_stride < w || w > (1 << 24)) return OOS_EINVAL;
  if (cache->n_kv_heads > 65535 || 2ll * batch->n_seqs + batch->n_tokens / kScaleBlock > 0x7fffffffll) return OOS_EINVAL;
  if (rope && !positions) return OOS_EINVAL;
  Append8Args a = {};
  a.pages = view_of(*cache);
  a.batch = view_of(*batch);
  a.in[0] = k;
  a.in[1] = v;
  a.stride[0] = k_stride;
  a.stride[1] = v_stride;
  a.gain = k_norm;
  a.positions = rope ? positions : nullptr;
  a.eps = eps;
  a.status = out_status;
  static const RopeTurns none = {};
  const RopeTurns& turns = rope ? rope_turns(*rope, cache->head_dim) : none;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = dtype == OOS_DTYPE_F32    ? launch_append8<float>(a, turns, st)
                        : dtype == OOS_DTYPE_BF16 ? launch_append8<__nv_bfloat16>(a, turns, st)
                                                  : launch_append8<__half>(a, turns, st);
  return e == cudaSuccess ? OOS_OK : OOS_ECUDA;
}
