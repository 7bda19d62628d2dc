// Append of new tokens to the paged 8-bit cache, with the position rotation on the way.
//
// Token i of a sequence that holds L tokens goes to position p = L + i.  Its queries and keys are
// rotated by row p of the cosine and sine tables, every product and sum rounded to fp32 once:
//   a' = a cos - b sin,   b' = b cos + a sin
// on the pairs (j, j + rot/2), or (2j, 2j + 1) when interleaved; values past `rot` stay.  Queries
// leave as bf16.  Keys and values are stored as rn_e4m3(x / 2^e), e the least exponent with
// amax <= 448 * 2^e over the finite values of the tokens in the block so far; values that are not
// finite, or 2^108 and more, are stored as NaN.  When a token raises e of a block that holds
// earlier tokens, their codes are multiplied by 2^(e_old - e_new) and rounded again: exact but for
// codes that fall below 2^-6.  A block's first token starts its scale anew, so what a page held
// for an earlier owner does not matter; rows past the new tokens are not touched.
//
// Bound by memory: K, V and q are read once, codes and rotated queries written once.  One warp
// takes one head of K, V or q over the (at most 16) new tokens of one block, so that a block's
// scale and codes have one writer; with one token a sequence, D / 8 lanes take it.
#include "kvpop_paged.cuh"
#include "kvpop_mma.cuh"

namespace kvpop {
namespace {

using namespace paged;

constexpr int AP_WARPS = 8;

struct AppendArgs {
  Pool pool;
  Batch b;
  const void *q, *k, *v;
  long long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs;
  const float *cosT, *sinT;
  bf16* q_out;
  int32_t* err;
  int tasks, HQ, rot, max_pos, interleaved;
};

__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], c = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = c.x; x[5] = c.y; x[6] = c.z; x[7] = c.w;
}

// Values 8 c .. 8 c + 7 of a row, rotated by position pos.
template <typename T>
__device__ __forceinline__ void load_rotated(const AppendArgs& a, const T* row, int c, int pos, float (&x)[8]) {
  load8(row + 8 * c, x);
  if (8 * c >= a.rot) return;
  const int half = a.rot >> 1;
  const long long at = (long long)pos * half;
  if (a.interleaved) {
    const float4 co = *reinterpret_cast<const float4*>(a.cosT + at + 4 * c);
    const float4 si = *reinterpret_cast<const float4*>(a.sinT + at + 4 * c);
    const float cs[4] = {co.x, co.y, co.z, co.w}, sn[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = x[2 * i], w = x[2 * i + 1];
      x[2 * i] = __fsub_rn(__fmul_rn(u, cs[i]), __fmul_rn(w, sn[i]));
      x[2 * i + 1] = __fadd_rn(__fmul_rn(w, cs[i]), __fmul_rn(u, sn[i]));
    }
  } else {
    const bool low = 8 * c < half;
    const int j = low ? 8 * c : 8 * c - half;
    float y[8], cs[8], sn[8];
    load8(row + (low ? 8 * c + half : j), y);
    load8(a.cosT + at + j, cs);
    load8(a.sinT + at + j, sn);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = __fmul_rn(x[i], cs[i]), w = __fmul_rn(y[i], sn[i]);
      x[i] = low ? __fsub_rn(u, w) : __fadd_rn(u, w);
    }
  }
}

// Least e with amax <= 448 * 2^e, at least E_MIN; amax finite.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  return max((int)(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), E_MIN);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Codes of 8 values under the scale 2^e (inv = 2^-e); all finite ones are at most 448 * 2^e.
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float inv) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      y[k] = fabsf(x[2 * i + k]) < VALUE_LIMIT ? x[2 * i + k] * inv : __uint_as_float(0x7fffffffu);
    h[i] = e4m3x2(y[0], y[1]);
  }
  return make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
}
// Codes multiplied by f (a power of two) and rounded again; NaN stays NaN.
__device__ __forceinline__ uint32_t rescale2(uint32_t two, float f) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  const float2 v = __half22float2(*reinterpret_cast<__half2*>(&h));
  return e4m3x2(v.x * f, v.y * f);
}
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  return rescale2(w & 0xffffu, f) | rescale2(w >> 16, f) << 16;
}

// ONE: one token a sequence.  D / 8 lanes per row; a warp takes one (block, head) of up to 16 rows,
// or, with ONE, 32 / (D / 8) of them with one row each.
template <typename T, int D, bool ONE>
__global__ void __launch_bounds__(32 * AP_WARPS) paged_append_kernel(AppendArgs a) {
  constexpr int LPR = D / 8, RPI = 32 / LPR, IT = ONE ? 1 : BLK / RPI;
  const int lane = threadIdx.x & 31, c = lane % LPR, sub = lane / LPR;
  const int slots = 2 * a.pool.H + a.HQ;
  const int warp = blockIdx.x * AP_WARPS + (threadIdx.x >> 5);
  int task = ONE ? warp * RPI + sub : warp;
  const bool live = task < a.tasks;                 // (a whole row's lanes agree; all stay for the shuffles)
  if (!live) task = a.tasks - 1;
  const int unit = task / slots, slot = task % slots;

  // the unit's sequence and block: with token offsets, sequence s owns the units from
  // starts[s] / 16 + 2 s on, which leaves room for each block that n tokens can touch
  int s = unit, blk = 0;
  if (!ONE) {
    int lo = 0, hi = a.b.n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((long long)(a.b.starts[mid] >> 4) + 2 * mid <= unit) lo = mid; else hi = mid - 1;
    }
    s = lo;
    blk = unit - ((a.b.starts[s] >> 4) + 2 * s);
  }
  const SeqTokens t = seq_tokens(a.b, s, a.err);
  const int cap = (int)min((long long)a.b.max_pages << a.pool.page_shift, (long long)INT32_MAX);
  int end = 0, p0 = 0;                              // positions of this block's new tokens: [p0, end)
  if (live && t.len >= 0 && t.n > 0 && blk >= 0) {
    const long long all = (long long)t.len + t.n, first = (long long)(t.len / BLK + blk) * BLK;
    if (first >= cap) {
      if (first < all) report(a.err, ERR_PAGE);
    } else if (first < all) {
      p0 = (int)max(first, (long long)t.len);
      end = (int)min(min(all, first + BLK), (long long)cap);
      if (min(all, first + BLK) > cap) report(a.err, ERR_PAGE);
      if (a.rot > 0 && end > a.max_pos) {
        report(a.err, ERR_ROTATION);
        end = a.max_pos;
      }
    }
  }
  const bool some = p0 < end;
  if (!ONE && !some) return;                        // warp-uniform

  if (slot >= 2 * a.pool.H) {                       // ------------------------------ queries
    const int h = slot - 2 * a.pool.H;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int pos = ONE ? p0 : p0 + it * RPI + sub;
      if (pos < end) {
        const long long tok = t.first + (pos - t.len);
        float x[8];
        load_rotated(a, static_cast<const T*>(a.q) + tok * a.q_ts + h * a.q_hs, c, pos, x);
        uint4 o;
        o.x = pack_bf16(x[0], x[1]);
        o.y = pack_bf16(x[2], x[3]);
        o.z = pack_bf16(x[4], x[5]);
        o.w = pack_bf16(x[6], x[7]);
        *reinterpret_cast<uint4*>(a.q_out + (tok * a.HQ + h) * D + 8 * c) = o;
      }
    }
    if (!ONE) return;
  }
  // ------------------------------------------------------------------ keys and values
  const bool kv = slot < 2 * a.pool.H && some;      // (ONE: lanes of queries stay for the shuffles)
  const bool is_v = slot >= a.pool.H;
  const int h = is_v ? slot - a.pool.H : slot;
  const int id = kv ? page_of(a.b, a.pool, s, p0, a.err) : -1;   // a block lies in one page
  const T* src = static_cast<const T*>(is_v ? a.v : a.k) + h * (is_v ? a.v_hs : a.k_hs);
  const long long ts = is_v ? a.v_ts : a.k_ts;
  const long long at = ((long long)max(id, 0) * a.pool.H + h) * a.pool.page;
  const int row0 = p0 & (a.pool.page - 1), head = row0 & (BLK - 1);   // rows of the block before p0
  float* scale = (is_v ? a.pool.vs : a.pool.ks) + (at + row0) / BLK;
  // one lane reads the block's scale and writes it
  const int lead = ONE ? lane - c : 0;
  float was = lane == lead && id >= 0 && head > 0 ? *scale : 0.f;
  float x[IT][8], amax = 0.f;
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int pos = ONE ? p0 : p0 + it * RPI + sub;
    if (id >= 0 && pos < end) {
      const T* row = src + (t.first + (pos - t.len)) * ts;
      if (is_v) load8(row + 8 * c, x[it]);
      else load_rotated(a, row, c, pos, x[it]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = fabsf(x[it][i]);
        amax = fmaxf(amax, y < VALUE_LIMIT ? y : 0.f);
      }
    }
  }
#pragma unroll
  for (int o = ONE ? LPR / 2 : 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  was = __shfl_sync(0xffffffffu, was, lead);
  if (id < 0) return;
  unsigned char* rows = (is_v ? a.pool.v : a.pool.k) + (at + (row0 - head)) * D;
  float sc = pow2(scale_exponent(amax));
  if (head > 0) {
    if (sc > was) {                                 // earlier codes move to the larger scale
      const float f = was / sc;
      for (int r = ONE ? 0 : sub; r < head; r += ONE ? 1 : RPI) {
        uint2* w = reinterpret_cast<uint2*>(rows + r * D + 8 * c);
        uint2 u = *w;
        u.x = rescale4(u.x, f);
        u.y = rescale4(u.y, f);
        *w = u;
      }
    } else {
      sc = was;
    }
  }
  const float inv = 1.f / sc;                       // exact: sc is a power of two
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int pos = ONE ? p0 : p0 + it * RPI + sub;
    if (pos < end) *reinterpret_cast<uint2*>(rows + (head + (pos - p0)) * D + 8 * c) = codes8(x[it], inv);
  }
  if (lane == lead) *scale = sc;
}

template <typename T, int D>
cudaError_t launch(AppendArgs& a, cudaStream_t stream) {
  const bool one = a.b.starts == nullptr;
  const long long tasks = (2 * a.pool.H + a.HQ) * (one ? (long long)a.b.n_seq : a.b.n_tokens / BLK + 2ll * a.b.n_seq);
  if (tasks > INT32_MAX - 32 * AP_WARPS) return cudaErrorInvalidValue;   // (refused before)
  a.tasks = (int)tasks;
  const int per_block = AP_WARPS * (one ? 32 / (D / 8) : 1), grid = (a.tasks + per_block - 1) / per_block;
  if (one) paged_append_kernel<T, D, true><<<(unsigned)grid, 32 * AP_WARPS, 0, stream>>>(a);
  else paged_append_kernel<T, D, false><<<(unsigned)grid, 32 * AP_WARPS, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_append(const Pool& pool, const Batch& b, const void* q, long long q_ts, long long q_hs,
                                int HQ, const void* k, long long k_ts, long long k_hs, const void* v,
                                long long v_ts, long long v_hs, int dtype, const float* cos_, const float* sin_,
                                int rot, int max_pos, int interleaved, void* q_out, int32_t* err,
                                cudaStream_t stream) {
  AppendArgs a{};
  a.pool = pool;
  a.b = b;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_ts = q_ts; a.q_hs = q_hs;
  a.k_ts = k_ts; a.k_hs = k_hs;
  a.v_ts = v_ts; a.v_hs = v_hs;
  a.cosT = cos_;
  a.sinT = sin_;
  a.rot = rot;
  a.max_pos = max_pos;
  a.interleaved = interleaved;
  a.q_out = static_cast<bf16*>(q_out);
  a.HQ = q ? HQ : 0;
  a.err = err;
  if (dtype == KVPOP_BF16) return pool.d == 128 ? launch<bf16, 128>(a, stream) : launch<bf16, 64>(a, stream);
  return pool.d == 128 ? launch<float, 128>(a, stream) : launch<float, 64>(a, stream);
}

}  // namespace kvpop
