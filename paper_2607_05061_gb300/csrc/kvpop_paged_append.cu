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
// takes one head of K or V, or two of q, over the (at most 16) new tokens of one block, so that a
// block's scale and codes have one writer; with one token a sequence, D / 8 lanes take a head.  16384
// tokens of 5 prompts with 32 query and 8 KV heads (bf16) take 88 us, 413 MB at 4.7 TB/s: the warps
// wait for their loads (less since they send their rows to L2 ahead: 98 before), and the issue slots
// are half taken by rotations and conversions.  One or four query heads a warp were slower.  64
// sequences' single tokens take 2.7 us, a launch and three loads in a row.
#include "kvpop_paged.cuh"
#include "kvpop_mma.cuh"
#include "kvpop_ptx.cuh"

namespace kvpop {
namespace {

using namespace paged;

constexpr int AP_WARPS = 4, AP_QH = 2;

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

// Loads that no store of this kernel can change.  (As volatile assembly they stay behind
// griddepcontrol.wait, and in the order in which they are written.)
__device__ __forceinline__ uint4 ld16(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ float4 ld16f(const float* p) {
  const uint4 v = ld16(p);
  return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}
// 8 values as they lie in memory
template <typename T>
struct Raw;
template <>
struct Raw<bf16> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = ld16(p); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = ld16f(p);
    b = ld16f(p + 4);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};

// What a lane's 8 values of a row are: their place, their pairs' (the same where it holds both),
// and where its cosines and sines lie in a row of the tables.
struct Lane {
  int own, other, angle;
  bool turned, low;
};
__device__ __forceinline__ Lane lane_of(const AppendArgs& a, int c, bool rotate) {
  const int half = a.rot >> 1;
  Lane n;
  n.own = 8 * c;
  n.turned = rotate && 8 * c < a.rot;
  n.low = 8 * c < half;
  n.other = !n.turned || a.interleaved ? 8 * c : n.low ? 8 * c + half : 8 * c - half;
  n.angle = a.interleaved ? 4 * c : n.low ? 8 * c : 8 * c - half;
  return n;
}
// Cosines and sines of 8 pairs (of 4 when interleaved); the sines of the pairs' first values are
// negated, so that u cos + w sin is the rotation of either.
struct Turn {
  float cs[8] = {}, sn[8] = {};
};
__device__ __forceinline__ Turn turn_of(const AppendArgs& a, const Lane& n, const float* cosR, const float* sinR) {
  Turn t;
  if (!n.turned) return t;
  Raw<float> cs, sn;
  if (a.interleaved) {
    cs.a = cs.b = ld16f(cosR);
    sn.a = sn.b = ld16f(sinR);
  } else {
    cs.load(cosR);
    sn.load(sinR);
  }
  cs.get(t.cs);
  sn.get(t.sn);
  if (n.low && !a.interleaved)
#pragma unroll
    for (int i = 0; i < 8; ++i) t.sn[i] = -t.sn[i];
  return t;
}
template <typename T>
__device__ __forceinline__ void rotated(const AppendArgs& a, const Lane& n, const Turn& t, const Raw<T>& own,
                                        const Raw<T>& other, float (&x)[8]) {
  own.get(x);
  if (!n.turned) return;
  if (a.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = x[2 * i], w = x[2 * i + 1];
      x[2 * i] = __fsub_rn(__fmul_rn(u, t.cs[i]), __fmul_rn(w, t.sn[i]));
      x[2 * i + 1] = __fadd_rn(__fmul_rn(w, t.cs[i]), __fmul_rn(u, t.sn[i]));
    }
  } else {
    float y[8];
    other.get(y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __fadd_rn(__fmul_rn(x[i], t.cs[i]), __fmul_rn(y[i], t.sn[i]));
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
// Codes of 8 values under the scale 2^e (inv = 2^-e); all finite ones are at most 448 * 2^e, unless
// `special`: then those that no scale holds become NaN (a NaN does by itself).
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float inv, bool special) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
  if (special)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(fabsf(x[i]) < VALUE_LIMIT)) y[i] = __uint_as_float(0x7fffffffu);
  return make_uint2(e4m3x2(y[0], y[1]) | e4m3x2(y[2], y[3]) << 16, e4m3x2(y[4], y[5]) | e4m3x2(y[6], y[7]) << 16);
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

// Sends every RPI-th of a lane's `rows` rows to L2, for up to NH heads: the loads that follow, a few
// rows at a time, then wait for L2 only.
template <typename T, int IT, int RPI, int NH>
__device__ __forceinline__ void ahead(const T* p, long long ts, long long hs, int heads, int rows, int c) {
  constexpr int PER = 128 / (8 * (int)sizeof(T));   // lanes that share a line
  if (c % PER) return;
#pragma unroll
  for (int it = 0; it < IT; ++it)
#pragma unroll
    for (int e = 0; e < NH; ++e)
      if (it * RPI < rows && e < heads) prefetch_l2_line(p + it * RPI * ts + e * hs);
}

// ONE: one token a sequence.  D / 8 lanes per row; a warp takes one (block, head) of up to 16 rows,
// or, with ONE, 32 / (D / 8) of them with one row each.
template <typename T, int D, bool ONE>
__global__ void __launch_bounds__(32 * AP_WARPS, 8) paged_append_kernel(AppendArgs a) {
  constexpr int LPR = D / 8, RPI = 32 / LPR, IT = ONE ? 1 : BLK / RPI, QH = ONE ? 1 : AP_QH;
  const int lane = threadIdx.x & 31, c = lane % LPR, sub = lane / LPR;
  constexpr bool KEEP = !ONE && D == 64;            // rotated rows stay in shared memory: 8 values a lane and turn
  __shared__ float4 keepS[KEEP ? AP_WARPS : 1][KEEP ? 2 * IT : 1][32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // a slot: a head of K or of V, or QH heads of q, which share their positions' cosines and sines
  const int slots = 2 * a.pool.H + (a.HQ + QH - 1) / QH;
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
    const int h0 = (slot - 2 * a.pool.H) * QH;
    const Lane n = lane_of(a, c, true);
    int pos = ONE ? p0 : p0 + sub;
    const long long tok = t.first + (pos - t.len);
    const T* from = static_cast<const T*>(a.q) + tok * a.q_ts + h0 * a.q_hs;
    const float *cosR = a.cosT + (long long)pos * (a.rot >> 1) + n.angle, *sinR = a.sinT + (cosR - a.cosT);
    bf16* to = a.q_out + (tok * a.HQ + h0) * D + n.own;
    if (!ONE) ahead<T, IT, RPI, QH>(from + n.own, a.q_ts, a.q_hs, min(a.HQ - h0, QH), end - pos, c);
#pragma unroll 1
    for (int it = 0; it < IT; ++it) {
      if (pos < end) {
        const Turn turn = turn_of(a, n, cosR, sinR);
        Raw<T> own[QH], other[QH];
#pragma unroll
        for (int e = 0; e < QH; ++e) {
          const T* row = from + (h0 + e < a.HQ ? e * a.q_hs : 0);
          own[e].load(row + n.own);
          other[e].load(row + n.other);
        }
#pragma unroll
        for (int e = 0; e < QH; ++e) {
          float x[8];
          rotated(a, n, turn, own[e], other[e], x);
          const uint4 o = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
          if (h0 + e < a.HQ) *reinterpret_cast<uint4*>(to + e * D) = o;
        }
      }
      pos += RPI;
      from += RPI * a.q_ts;
      cosR += RPI * (a.rot >> 1);
      sinR += RPI * (a.rot >> 1);
      to += (long long)RPI * a.HQ * D;
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
  const Lane n = lane_of(a, c, !is_v);
  // The rows are used twice, for the largest value and for the codes.  At d = 64 they stay in 4 KB of
  // shared memory a warp (4 prompts of 4000 tokens, 8 and 32 heads 42 us, 44 read again); at d = 128
  // they are read again, from L2: 8 KB a warp cost a quarter of the warps, whose loads are what the
  // first pass waits for (16384 tokens 98 us, 88 read again; half of the rows kept 88), and registers
  // more of them (170).
  const int pos0 = ONE ? p0 : p0 + sub;
  const T* const from = src + (t.first + (pos0 - t.len)) * ts;
  const long long angle0 = (long long)pos0 * (a.rot >> 1) + n.angle;
  if (!ONE && id >= 0) ahead<T, IT, RPI, 1>(from + n.own, ts, 0, 1, end - pos0, c);
  auto read = [&](int it, float (&x)[8]) {
    const T* row = from + it * RPI * ts;
    const long long at = angle0 + it * RPI * (a.rot >> 1);
    Raw<T> own, other;
    own.load(row + n.own);
    other.load(row + n.other);
    rotated(a, n, turn_of(a, n, a.cosT + at, a.sinT + at), own, other, x);
  };
  auto value = [&](int it, float (&x)[8], bool again) {
    if (!KEEP || !again) {
      read(it, x);
    } else {
      const float4 u = keepS[threadIdx.x >> 5][2 * it][lane], w = keepS[threadIdx.x >> 5][2 * it + 1][lane];
      x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
      x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    }
  };
  auto largest = [&](float limit) {
    float m = 0.f;
    if (id >= 0)
#pragma unroll 2
      for (int it = 0; it < IT; ++it)
        if (pos0 + it * RPI < end) {
          float x[8];
          value(it, x, limit > 0.f);
          if (KEEP && limit == 0.f) {
            keepS[threadIdx.x >> 5][2 * it][lane] = make_float4(x[0], x[1], x[2], x[3]);
            keepS[threadIdx.x >> 5][2 * it + 1][lane] = make_float4(x[4], x[5], x[6], x[7]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) m = fmaxf(m, limit > 0.f && !(fabsf(x[i]) < limit) ? 0.f : fabsf(x[i]));
        }
#pragma unroll
    for (int o = ONE ? LPR / 2 : 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
  };
  float amax = largest(0.f);                        // (a NaN is no maximum)
  const bool special = !(amax < VALUE_LIMIT);       // values that no scale holds: not counted
  if (__any_sync(0xffffffffu, special)) amax = largest(VALUE_LIMIT);
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
  unsigned char* to = rows + (head + (pos0 - p0)) * D + n.own;
#pragma unroll 2
  for (int it = 0; it < IT; ++it)
    if (pos0 + it * RPI < end) {
      float x[8];
      value(it, x, true);
      *reinterpret_cast<uint2*>(to + it * RPI * D) = codes8(x, inv, special);
    }
  if (lane == lead) *scale = sc;
}

template <typename T, int D>
cudaError_t launch(AppendArgs& a, cudaStream_t stream) {
  const bool one = a.b.starts == nullptr;
  const long long tasks = (2 * a.pool.H + (one ? a.HQ : (a.HQ + AP_QH - 1) / AP_QH)) * (one ? (long long)a.b.n_seq : a.b.n_tokens / BLK + 2ll * a.b.n_seq);
  if (tasks > INT32_MAX - 32 * AP_WARPS) return cudaErrorInvalidValue;   // (refused before)
  a.tasks = (int)tasks;
  const int per_block = AP_WARPS * (one ? 32 / (D / 8) : 1), grid = (a.tasks + per_block - 1) / per_block;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(32 * AP_WARPS);
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return one ? cudaLaunchKernelEx(&cfg, paged_append_kernel<T, D, true>, a)
             : cudaLaunchKernelEx(&cfg, paged_append_kernel<T, D, false>, a);
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
