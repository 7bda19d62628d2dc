// Grouped-query attention over the paged 8-bit cache: a stream of the cache through mma.sync.
//
// For query row r = (new token i, query head g) of one (sequence, KV head) and the positions
// t <= L + i it sees, with K_t = code 2^ek, V_t = code 2^ev and the scales of t's block:
//   x_t = (q . K_t) / sqrt(d),   y = sum_t softmax(x)_t V_t,   lse = log sum_t exp(x_t).
//
// Bound by the cache's bytes (2 d + 1/2 per position and KV head).  A warp takes one block of 16
// positions at a time, S^T = K Q^T and O^T += V^T P^T as m16n8k16 with the positions (then the
// values) as the 16-row operand and NT groups of 8 query rows as the 8-column one, so that each
// byte is read and converted once for all query heads.  Lanes load whole rows straight into
// registers: the order of the contraction index is free, so a lane takes 16 neighbouring bytes of
// a row, which become its operand words by e4m3 -> f16 conversion alone; for V the bytes of two
// positions are interleaved first.  f16 holds every e4m3 value, and q, scaled by a power of two
// per row, to 2^-39 of the row's largest value, so the products are exact.
//
// The scales cost next to nothing: ek multiplies the logits, and ev joins the exponent,
//   p_t = 2^(x_t log2 e + ev - M + 7),  O = sum p_t code_t,  l = sum p_t 2^-ev,  y = O / l,
// where M, the running base of a row, moves when a term exceeds it by 2^8.  p_t lies in [0, 2^15]:
// rounded to f16 it has 11 bits, enough for a bf16 result (SPLIT false); for an fp32 result it is
// the sum of two f16 values, 22 bits, and the second product is taken too (SPLIT).
//
// The blocks of all (sequence, KV head, row group) units form one list that is cut evenly over a
// grid of resident CTAs; a CTA's 8 warps take its blocks in turn and join their rows in warp
// order.  A unit that lies in several CTAs' parts is joined, in the order of the parts, by the CTA
// that arrives last (no CTA waits).
#include <algorithm>

#include "kvpop_mma.cuh"
#include "kvpop_paged.cuh"

namespace kvpop {
namespace {

using namespace paged;

constexpr int AT_WARPS = 8, AT_THREADS = 32 * AT_WARPS;
constexpr int AT_CTAS = 2;             // resident per SM
constexpr int AT_MAX_ROWS = 32;        // query rows of a unit at most
constexpr float AT_OFF = 7.f, AT_STEP = 8.f;

struct AttendArgs {
  Pool pool;
  Batch b;
  const bf16* q;
  long long q_ts, q_hs;
  void* out;
  float* lse;
  float* part;                         // [grid][2][rows][D + 2]
  int* count;                          // [grid], zero between calls
  int32_t* err;
  float c;                             // log2(e) / sqrt(d)
  int G, out_f32;
  int skip_long;                       // the tcgen05 kernel takes sequences with long_rows
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
      " {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// four e4m3 bytes -> two words of two f16
__device__ __forceinline__ void cvt4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ uint32_t movm(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint4 ldg16(const unsigned char* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ldg8(const unsigned char* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Units of a sequence: H x row groups, each of `tiles` blocks (one at least, so that a row that
// sees nothing is written too).
struct SeqUnits {
  int first, n, len, ctx, groups, tiles;
  __device__ long long work(int H) const { return (long long)H * groups * tiles; }
};
template <int ROWS>
__device__ __forceinline__ SeqUnits seq_units(const AttendArgs& a, int s) {
  const SeqTokens t = seq_tokens(a.b, s, a.err);
  SeqUnits u;
  u.first = t.first;
  u.len = t.len;
  u.n = t.n;
  u.groups = (int)(((long long)t.n * a.G + ROWS - 1) / ROWS);
  if (a.skip_long && long_rows(t, a.G)) u.groups = 0;
  u.ctx = u.groups > 0 ? context(a.b, a.pool, t, a.err) : 0;
  u.tiles = max((u.ctx + BLK - 1) / BLK, 1);
  return u;
}

// Four values of a finished row, and its normaliser.  A row that saw nothing: zeros and -inf.
template <int D>
__device__ __forceinline__ void write_out(const AttendArgs& a, int first, int h, int r, int cc, float4 y, float m,
                                          float l) {
  const int i = r / a.G;
  const long long row = (long long)(first + i) * a.pool.H * a.G + h * a.G + (r - i * a.G);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  y.x *= inv; y.y *= inv; y.z *= inv; y.w *= inv;
  if (a.out_f32)
    reinterpret_cast<float4*>(a.out)[row * (D / 4) + cc] = y;
  else
    reinterpret_cast<uint2*>(a.out)[row * (D / 4) + cc] = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
  if (cc == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (m - AT_OFF + log2f(l)) * 0.69314718055994530942f;
}

template <int D, int NT, bool SPLIT>
__global__ void __launch_bounds__(AT_THREADS, NT == 1 ? AT_CTAS : 1) paged_attend_kernel(AttendArgs a) {
  constexpr int ROWS = 8 * NT, KW = D / 16, VW = D / 32;   // words a lane holds of a K / V row
  constexpr int RS = 8 * (D + 4);                          // a warp's 8 rows in shared memory
  __shared__ float accS[AT_WARPS * RS];
  __shared__ float mS[AT_WARPS][ROWS], lS[AT_WARPS][ROWS];
  __shared__ long long scanS[AT_THREADS / 32 + 1];
  __shared__ int lastS;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const int H = a.pool.H, G = a.G;

  // ---- this CTA's part of the list: [w0, w1), and the sequence that w0 lies in
  const int per = (a.b.n_seq + AT_THREADS - 1) / AT_THREADS, sA = min(tid * per, a.b.n_seq);
  const int sB = min(sA + per, a.b.n_seq);
  long long mine = 0;
  for (int s = sA; s < sB; ++s) mine += seq_units<ROWS>(a, s).work(H);
  long long pre = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, pre, o);
    if (lane >= o) pre += y;
  }
  if (lane == 31) scanS[warp] = pre;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < AT_WARPS; ++w) {
    if (w < warp) pre += scanS[w];
    total += scanS[w];
  }
  __syncthreads();
  // parts of at least one block a warp
  const long long grid = max(min((long long)gridDim.x, total / AT_WARPS), 1ll);
  auto part_start = [&](long long c) { return c * total / grid; };
  auto part_of = [&](long long w) {                        // the part that block w lies in
    long long c = w * grid / total;
    while (c + 1 < grid && part_start(c + 1) <= w) ++c;
    while (part_start(c) > w) --c;
    return c;
  };
  if (blockIdx.x >= grid || total == 0) return;
  const long long w0 = part_start(blockIdx.x), w1 = part_start(blockIdx.x + 1);
  if (w0 >= w1) return;
  __shared__ int s0S;
  __shared__ long long b0S;
  if (pre - mine <= w0 && w0 < pre) {
    long long base = pre - mine;
    int s = sA;
    for (; s < sB; ++s) {
      const long long k = seq_units<ROWS>(a, s).work(H);
      if (w0 < base + k) break;
      base += k;
    }
    s0S = s;
    b0S = base;
  }
  __syncthreads();
  int s = s0S;
  long long base = b0S;                                    // list position of sequence s
  SeqUnits u = seq_units<ROWS>(a, s);

  for (long long w = w0; w < w1;) {
    while (w >= base + u.work(H)) {                        // (sequences without tokens have no blocks)
      base += u.work(H);
      u = seq_units<ROWS>(a, ++s);
    }
    const int unit = (int)((w - base) / u.tiles), h = unit % H, grp = unit / H;
    const long long ustart = base + (long long)unit * u.tiles;
    const int ta = (int)(w - ustart), tb = (int)min((long long)u.tiles, w1 - ustart);
    w = ustart + tb;
    const int row0 = grp * ROWS, rows = min(ROWS, u.n * G - row0);

    // ---- query rows, each scaled by a power of two, and what that makes of the logits
    uint32_t qf[NT][KW][2];
    float rc[NT][2];
    int lim[NT][2];                                        // last position a row sees
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = row0 + 8 * j + g;
      const bool ok = 8 * j + g < rows;
      const bf16* qp = a.q + (long long)(u.first + (ok ? r / G : 0)) * a.q_ts + (long long)(h * G + (ok ? r % G : 0)) * a.q_hs;
      uint32_t raw[KW][2];
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < KW; k += 4)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint4 v = ok ? *reinterpret_cast<const uint4*>(qp + 16 * k + 16 * t4 + 8 * e) : make_uint4(0, 0, 0, 0);
          raw[k + 2 * e][0] = v.x; raw[k + 2 * e][1] = v.y;
          raw[k + 2 * e + 1][0] = v.z; raw[k + 2 * e + 1][1] = v.w;
          top = max(top, max(max(v.x & 0x7fffu, v.x >> 16 & 0x7fffu), max(v.y & 0x7fffu, v.y >> 16 & 0x7fffu)));
          top = max(top, max(max(v.z & 0x7fffu, v.z >> 16 & 0x7fffu), max(v.w & 0x7fffu, v.w >> 16 & 0x7fffu)));
        }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // 2^up brings the largest value into [2^14, 2^15)
      const int up = max(min(14 - ((int)(top >> 7) - 127), 110), -113);
      const float f = __uint_as_float((uint32_t)(up + 127) << 23);
#pragma unroll
      for (int k = 0; k < KW; ++k)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          qf[j][k][e] = pack_f16(__uint_as_float(raw[k][e] << 16) * f, __uint_as_float(raw[k][e] & 0xffff0000u) * f);
      const float down = a.c * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        rc[j][e] = __shfl_sync(0xffffffffu, down, (2 * t4 + e) * 4);
        const int rr = min(row0 + 8 * j + 2 * t4 + e, row0 + rows - 1);
        lim[j][e] = min(u.len + rr / G, u.ctx - 1);
      }
    }
    const int lim_lo = min(u.len + row0 / G, u.ctx - 1);   // the unit's rows see at least 0 .. lim_lo
    const int lim_hi = min(u.len + (row0 + rows - 1) / G, u.ctx - 1);   // and at most 0 .. lim_hi

    float o[NT][KW][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      m[j][0] = m[j][1] = -INFINITY;
      l[j][0] = l[j][1] = 0.f;
#pragma unroll
      for (int k = 0; k < KW; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][k][e] = 0.f;
    }

    // ---- the stream
    auto page = [&](int t) { return t * BLK <= lim_hi ? page_of(a.b, a.pool, s, t * BLK, a.err) : -1; };
    auto block_at = [&](int id, int t) {                   // row of the pools, in blocks
      return ((long long)max(id, 0) * H + h) * (a.pool.page / BLK) + (t & (a.pool.page / BLK - 1));
    };
    uint32_t kr[2][KW], vr[4][VW];
    float ks, vs;
    auto load_k = [&](long long blk) {
      const unsigned char* p = a.pool.k + (blk * BLK + g) * D + 16 * t4;
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int k = 0; k < KW; k += 4) {
          const uint4 v = ldg16(p + e * 8 * D + 16 * k);
          kr[e][k] = v.x; kr[e][k + 1] = v.y; kr[e][k + 2] = v.z; kr[e][k + 3] = v.w;
        }
      ks = a.pool.ks[blk];
    };
    auto load_v = [&](long long blk) {
      const unsigned char* p = a.pool.v + (blk * BLK + 2 * t4) * D + 4 * VW * g;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned char* pe = p + ((e & 1) + 8 * (e >> 1)) * D;
        if constexpr (VW == 4) {
          const uint4 v = ldg16(pe);
          vr[e][0] = v.x; vr[e][1] = v.y; vr[e][2] = v.z; vr[e][3] = v.w;
        } else {
          const uint2 v = ldg8(pe);
          vr[e][0] = v.x; vr[e][1] = v.y;
        }
      }
      vs = a.pool.vs[blk];
    };
    int t = ta + warp;
    int id = t < tb ? page(t) : -1, id_next = t + AT_WARPS < tb ? page(t + AT_WARPS) : -1;
    if (t < tb && id >= 0) {
      load_k(block_at(id, t));
      load_v(block_at(id, t));
    }
    for (; t < tb; t += AT_WARPS) {
      const int tn = t + AT_WARPS;
      const bool next = tn < tb && id_next >= 0;
      const long long bn = block_at(id_next, tn);
      if (id >= 0) {                                       // (warp-uniform; otherwise no row sees the block)
        float sc[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j) sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
#pragma unroll
        for (int k = 0; k < KW; ++k) {
          uint32_t a0, a1, a2, a3;
          cvt4(kr[0][k], a0, a2);
          cvt4(kr[1][k], a1, a3);
#pragma unroll
          for (int j = 0; j < NT; ++j) mma_f16(sc[j], a0, a1, a2, a3, qf[j][k][0], qf[j][k][1]);
        }
        const float ksc = ks;
        if (next) load_k(bn);
        const int ebits = (int)(__float_as_uint(vs) >> 23);
        const float ev = (float)(ebits - 127), vinv = __uint_as_float((uint32_t)(254 - ebits) << 23);
        const bool edge = t * BLK + BLK - 1 > lim_lo;      // some row does not see the whole block
        // exponents from the row's base, in one rounding: as long as there is none (-inf) every
        // logit is too large
        float y[NT][4];
        auto exponents = [&](float off, bool based) {
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              y[j][e] = fmaf(sc[j][e], rc[j][e & 1] * ksc, based ? ev + (off - m[j][e & 1]) : ev);
              if (edge && t * BLK + g + 8 * (e >> 1) > lim[j][e & 1]) y[j][e] = -INFINITY;
            }
        };
        exponents(AT_OFF, true);
        bool up = false;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) up |= y[j][e] > AT_OFF + AT_STEP;
        if (__any_sync(0xffffffffu, up)) {
          exponents(0.f, false);
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float mx = fmaxf(y[j][e], y[j][e + 2]);
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
              mx = fmaxf(mx, m[j][e]);
              const float al = m[j][e] == -INFINITY ? 0.f : ex2(m[j][e] - mx);
              m[j][e] = mx;
              l[j][e] *= al;
#pragma unroll
              for (int k = 0; k < KW; ++k) {
                o[j][k][e] *= al;
                o[j][k][e + 2] *= al;
              }
            }
          exponents(AT_OFF, true);
        }
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
          for (int e = 0; e < 4; ++e) y[j][e] = ex2(y[j][e]);
#pragma unroll
          for (int e = 0; e < 2; ++e) l[j][e] = fmaf(y[j][e] + y[j][e + 2], vinv, l[j][e]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t hi = pack_f16(y[j][2 * e], y[j][2 * e + 1]);
            ph[j][e] = movm(hi);
            if (SPLIT) {
              const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              pl[j][e] = movm(pack_f16(y[j][2 * e] - b.x, y[j][2 * e + 1] - b.y));
            }
          }
        }
        uint32_t bad = 0;                                  // NaN among the values of an edge block
        if (edge) {
          // Values that some row does not see: past lim_hi nothing is known of them, and a NaN
          // must not reach the rows before it, where its weight is 0.
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool gone = t * BLK + 2 * t4 + (e & 1) + 8 * (e >> 1) > lim_hi;
#pragma unroll
            for (int k = 0; k < VW; ++k) {
              if (gone) vr[e][k] = 0;
#pragma unroll
              for (int y = 0; y < 4; ++y)
                if ((vr[e][k] >> (8 * y) & 0x7fu) == 0x7fu) bad |= 1u << e;
            }
          }
        }
        uint32_t nan_at[4][VW];                            // 0xff in the bytes that are NaN
        if (edge && __any_sync(0xffffffffu, bad != 0)) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int k = 0; k < VW; ++k) {
              uint32_t mask = 0;
#pragma unroll
              for (int y = 0; y < 4; ++y)
                if ((vr[e][k] >> (8 * y) & 0x7fu) == 0x7fu) mask |= 0xffu << (8 * y);
              nan_at[e][k] = mask;
              vr[e][k] &= ~mask;
            }
          // rows that do see such a value get it: NaN in that column
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int pos = t * BLK + 2 * y + (e & 1) + 8 * (e >> 1);
#pragma unroll
              for (int k = 0; k < VW; ++k) {
                const uint32_t mask = __shfl_sync(0xffffffffu, nan_at[e][k], (lane & ~3) + y);
#pragma unroll
                for (int z = 0; z < 4; ++z)
                  if (mask >> (8 * z) & 1u)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                      for (int x = 0; x < 2; ++x)
                        if (pos <= lim[j][x]) o[j][2 * k + (z >> 1)][2 * (z & 1) + x] = __uint_as_float(0x7fffffffu);
              }
            }
        }
#pragma unroll
        for (int k = 0; k < VW; ++k)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            // bytes 2 e, 2 e + 1 of word k of the four positions: values 2 (2 k + e) and the next
            uint32_t a0, a1, a2, a3;
            cvt4(__byte_perm(vr[0][k], vr[1][k], e ? 0x7362 : 0x5140), a0, a1);
            cvt4(__byte_perm(vr[2][k], vr[3][k], e ? 0x7362 : 0x5140), a2, a3);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              mma_f16(o[j][2 * k + e], a0, a1, a2, a3, ph[j][0], ph[j][1]);
              if (SPLIT) mma_f16(o[j][2 * k + e], a0, a1, a2, a3, pl[j][0], pl[j][1]);
            }
          }
        if (next) load_v(bn);
      } else if (next) {
        load_k(bn);
        load_v(bn);
      }
      id = id_next;
      id_next = tn + AT_WARPS < tb ? page(tn + AT_WARPS) : -1;
    }

    // ---- the warps' rows join, 8 at a time
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[j][e] += __shfl_xor_sync(0xffffffffu, l[j][e], x);
        if (g == 0) {
          mS[warp][8 * j + 2 * t4 + e] = m[j][e];
          lS[warp][8 * j + 2 * t4 + e] = l[j][e];
        }
      }
    const bool whole = ta == 0 && tb == u.tiles;
    const long long c0 = whole ? 0 : part_of(ustart), c1 = whole ? 0 : part_of(ustart + u.tiles - 1);
    float* mypart = a.part + ((long long)blockIdx.x * 2 + (blockIdx.x == c0 ? 1 : 0)) * ROWS * (D + 2);
#pragma unroll 1
    for (int j = 0; j < NT; ++j) {
      __syncthreads();
#pragma unroll
      for (int jj = 0; jj < NT; ++jj)
        if (jj == j) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int col = 8 * j + 2 * t4 + e;
            float mt = mS[0][col];
#pragma unroll
            for (int x = 1; x < AT_WARPS; ++x) mt = fmaxf(mt, mS[x][col]);
            const float f = m[jj][e] == -INFINITY ? 0.f : ex2(m[jj][e] - mt);
            float* p = accS + warp * RS + (2 * t4 + e) * (D + 4) + 2 * KW * g;
#pragma unroll
            for (int k = 0; k < KW; ++k)
              *reinterpret_cast<float2*>(p + 2 * k) = make_float2(o[jj][k][e] * f, o[jj][k][e + 2] * f);
          }
        }
      __syncthreads();
      for (int i = tid; i < 8 * (D / 4); i += AT_THREADS) {
        const int r = i / (D / 4), cc = i % (D / 4), col = 8 * j + r;
        if (col >= rows) continue;
        float mt = mS[0][col], lt = 0.f;
#pragma unroll
        for (int x = 1; x < AT_WARPS; ++x) mt = fmaxf(mt, mS[x][col]);
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < AT_WARPS; ++x) {
          const float4 z = *reinterpret_cast<const float4*>(accS + x * RS + r * (D + 4) + 4 * cc);
          y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
          lt += lS[x][col] * (mS[x][col] == -INFINITY ? 0.f : ex2(mS[x][col] - mt));
        }
        if (whole) {
          write_out<D>(a, u.first, h, row0 + col, cc, y, mt, lt);
        } else {
          float* p = mypart + (long long)col * (D + 2);
          __stcg(reinterpret_cast<float2*>(p + 4 * cc), make_float2(y.x, y.y));
          __stcg(reinterpret_cast<float2*>(p + 4 * cc + 2), make_float2(y.z, y.w));
          if (cc == 0) __stcg(reinterpret_cast<float2*>(p + D), make_float2(mt, lt));
        }
      }
    }
    if (!whole) {
      __threadfence();
      __syncthreads();
      if (tid == 0) lastS = atomicAdd(a.count + c0, 1) == (int)(c1 - c0);
      __syncthreads();
      if (lastS) {
        __threadfence();
        for (int i = tid; i < rows * (D / 4); i += AT_THREADS) {
          const int col = i / (D / 4), cc = i % (D / 4);
          float mt = -INFINITY, lt = 0.f;
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
          for (long long c = c0; c <= c1; ++c) {
            const float* p = a.part + ((c * 2 + (c == c0 ? 1 : 0)) * ROWS + col) * (D + 2);
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(p + D));
            const float2 ya = __ldcg(reinterpret_cast<const float2*>(p + 4 * cc));
            const float2 yb = __ldcg(reinterpret_cast<const float2*>(p + 4 * cc + 2));
            const float mn = fmaxf(mt, ml.x);
            // (a NaN in a part without a base stays one)
            const float fo = mt == -INFINITY ? 0.f : ex2(mt - mn);
            const float fn = ml.x == -INFINITY ? 0.f : ex2(ml.x - mn);
            y.x = y.x * fo + ya.x * fn;
            y.y = y.y * fo + ya.y * fn;
            y.z = y.z * fo + yb.x * fn;
            y.w = y.w * fo + yb.y * fn;
            lt = lt * fo + ml.y * fn;
            mt = mn;
          }
          write_out<D>(a, u.first, h, row0 + col, cc, y, mt, lt);
        }
        if (tid == 0) a.count[c0] = 0;
      }
    }
    __syncthreads();                                       // shared memory is free for the next unit
  }
}

template <int D, int NT>
cudaError_t launch(const AttendArgs& a, int grid, cudaStream_t stream) {
  if (a.out_f32) paged_attend_kernel<D, NT, true><<<grid, AT_THREADS, 0, stream>>>(a);
  else paged_attend_kernel<D, NT, false><<<grid, AT_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}
template <int D>
cudaError_t launch_d(const AttendArgs& a, int sms, long long rows, cudaStream_t stream) {
  if (rows <= 8) return launch<D, 1>(a, AT_CTAS * sms, stream);
  if (rows <= 16) return launch<D, 2>(a, sms, stream);
  return launch<D, 4>(a, sms, stream);
}

size_t counter_bytes(int sms) { return ((size_t)AT_CTAS * sms * 4 + 255) / 256 * 256; }

}  // namespace

size_t paged_attend_workspace(int sms) {
  return counter_bytes(sms) + (size_t)AT_CTAS * sms * 2 * AT_MAX_ROWS * (128 + 2) * 4;
}

cudaError_t launch_paged_attend(const Pool& pool, const Batch& b, const void* q, long long q_ts, long long q_hs,
                                int HQ, void* out, int out_f32, float* lse, void* workspace, int sms,
                                int32_t* err, cudaStream_t stream) {
  AttendArgs a{};
  a.pool = pool;
  a.b = b;
  a.q = static_cast<const bf16*>(q);
  a.q_ts = q_ts;
  a.q_hs = q_hs;
  a.out = out;
  a.out_f32 = out_f32;
  a.lse = lse;
  a.count = static_cast<int*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + counter_bytes(sms));
  a.err = err;
  a.c = (float)(1.4426950408889634 / sqrt((double)pool.d));
  a.G = HQ / pool.H;
  long long rows = (long long)a.G * (b.starts ? b.max_new : 1);
  if (rows > LONG_ROWS && b.starts && paged_prompt_fits(pool, b, HQ)) {
    a.skip_long = 1;
    rows = LONG_ROWS;
    const cudaError_t e = launch_paged_prompt(pool, b, q, q_ts, q_hs, HQ, out, out_f32, lse, err, stream);
    if (e != cudaSuccess) return e;
  }
  return pool.d == 128 ? launch_d<128>(a, sms, rows, stream) : launch_d<64>(a, sms, rows, stream);
}

}  // namespace kvpop
