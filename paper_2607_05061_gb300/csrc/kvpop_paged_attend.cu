// Grouped-query attention over the paged 8-bit cache: a stream of the cache through mma.sync.
//
// For query row r = (new token i, query head g) of one (sequence, KV head) and the positions
// t <= L + i it sees, with K_t = code 2^ek, V_t = code 2^ev and the scales of t's block:
//   x_t = (q . K_t) / sqrt(d),   y = sum_t softmax(x)_t V_t,   lse = log sum_t exp(x_t).
//
// Bound by the cache's bytes (2 d + 1/2 per position and KV head).  A warp takes one block of 16
// positions at a time, S^T = K Q^T and O^T += V^T P^T as m16n8k16 with the positions (then the
// values) as the 16-row operand and NT groups of 8 query rows as the 8-column one, so that each
// byte is read and converted once for all query heads.  Each warp has its own ring of blocks in
// shared memory, which its lanes fill by 16-byte cp.async (swizzled so that the reads below touch
// every bank once) and read alone: no warp waits for another, and the ring runs on across the ends
// of units while the warps join their rows.  (TMA was slower here: a copy takes about 140 clocks
// of its engine whatever its size, and a page of 16 positions makes 2 KB pieces; 64 sequences of
// 8192 tokens 226 us with 8 KB boxes, 277 with 2 KB ones.)  The order of the contraction index is
// free, so a lane takes neighbouring bytes of a row, which become its operand words by
// e4m3 -> f16 conversion alone; for V the bytes of two positions are interleaved first.  f16 holds
// every e4m3 value, and q, scaled by a power of two per row, to 2^-39 of the row's largest value,
// so the products are exact.
//
// The scales cost little: ek multiplies the logits, and ev the weights,
//   w_t = 2^(x_t log2 e - M + 2),  p_t = w_t 2^(ev + 5),  O = sum p_t code_t,  l = sum w_t,  y = O / (32 l),
// where M, the running base of a row, moves when x_t log2 e + ev exceeds it by 8.  p_t lies in [0, 2^15]:
// rounded to f16 it has 11 bits, enough for a bf16 result (SPLIT false); for an fp32 result it is
// the sum of two f16 values, 22 bits, and the second product is taken too (SPLIT).  The tensor
// cores cut their fp32 sums off instead of rounding them, which adds up along a row (2.1e-6 of the
// result over 512 blocks): with SPLIT a block's product is formed from zero and added by a rounded
// fp32 sum (5e-7).
//
// The blocks of all (sequence, KV head, row group) units form one list that is cut evenly over the
// SMs; a CTA's warps take its blocks in turn and join their rows in warp order.  A unit that lies in
// several CTAs' parts is joined, in the order of the parts, by the CTA that arrives last, at its end (no
// CTA waits); many parts join in groups first.
//
// 64 sequences of 8192 positions, 32 query and 8 KV heads: 167 us, 0.94 of the copy rate; one of
// 131072 52 us (40 by the copy rate: 7 until the stream runs, 5 for the join of 38 parts a head).
// One CTA of 12 warps an SM took the same for the former and 93 instead of 66 for 40 ragged ones: it
// streams nothing while its rows join.
#include <algorithm>
#include <type_traits>

#include "kvpop_mma.cuh"
#include "kvpop_paged.cuh"
#include "kvpop_ptx.cuh"

namespace kvpop {
namespace {

using namespace paged;

// What the two ends of a unit cost, in blocks (us at 0, 16, 32, 64: 40 ragged sequences of up to
// 20000 tokens 82, 71, 66, 67; 128 of 200 to 1500 70, 53, 51, 53; 64 of 8192 170, 169, 170, 172).
constexpr int AT_ENDS = 32;
// Blocks of a unit that one CTA takes whole: always, and where there is work for all CTAs.  us with
// units of up to 0, 24, 48, 96 blocks never cut: 64 sequences of 512 (33 blocks) 25.8, 26.0, 23.1, 23.1;
// 8 of 700 11.2, 11.2, 13.2, 13.2; one of 332 8.8, 8.5, 8.5, 8.5; 128 of 200 to 1500 52.1, 52.0, 52.6, 55.7.
constexpr int AT_TINY = 24, AT_SHORT = 48;
constexpr int AT_CTAS = 2;             // resident per SM: one streams while the other joins its rows
constexpr int AT_MAX_ROWS = 32;        // query rows of a unit at most
constexpr int AT_JOIN = 8;             // parts that are loaded at once
// Parts of a unit that one CTA joins; more join in groups first, and then the groups.  us without
// groups, in groups of 8, of 16: one sequence of 131072 and 8 KV heads (38 parts) 55.4, 52.7, 53.9; 4 of
// 20000 and 2 heads (38) 24.6, 19.9, 21.8; one of 100000 and 1 head (304) 80, 25.3, 23.5.
constexpr int AT_FEW = 16;
__device__ __forceinline__ int group_of(int parts) { return parts > 128 ? 16 : 8; }

// The rings: a block's 16 rows of K, then of V.  The 16-byte chunk c of row r lies at chunk
// c ^ (r mod 8) of its 128 bytes (d = 128), or c ^ (r / 2 mod 4) of its 64 (d = 64).
template <int D, int W>
struct Ring {
  static constexpr int BLOCK = 2 * BLK * D, ST = W == 8 ? 5 : (W == 6 ? 3 : 5) * (128 / D);
  static constexpr int OFF_ACC = W * ST * BLOCK;                       // a warp's 8 rows: 8 (d + 4) floats
  static constexpr int OFF_Q = OFF_ACC + W * 8 * (D + 4) * 4;          // 4 groups of query operands
  static constexpr int BYTES = OFF_Q + 4 * (D / 16) * 256;
  static __device__ __forceinline__ int chunk_at(int r, int c) {
    return r * D + ((c ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4);
  }
  // a lane's i-th 16 bytes of K: bytes D/4 t + 16 i .. of row r
  static __device__ __forceinline__ int k_at(int r, int t, int i) { return chunk_at(r, D == 128 ? 2 * t + i : t); }
  // a lane's bytes of V: bytes D/8 g .. of row r
  static __device__ __forceinline__ int v_at(int r, int g) {
    return D == 128 ? chunk_at(r, g) : chunk_at(r, g >> 1) + 8 * (g & 1);
  }
};

struct AttendArgs {
  Pool pool;
  Batch b;
  const bf16* q;
  long long q_ts, q_hs;
  void* out;
  float* lse;
  float* part;                         // [grid][2][rows][D + 4]
  int* count;                          // [2][grid] of units and of groups, zero between calls
  int32_t* err;
  float c;                             // log2(e) / sqrt(d)
  float inv_g;                         // 1 / G
  int G, out_f32;
  int one;                             // row groups of a single token
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
// the same from zero
__device__ __forceinline__ void mma_f16_0(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                          uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
      " {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Units of a sequence: H x row groups, each of `blocks` blocks (one at least, so that a row that
// sees nothing is written too).  In the list a unit takes span() places: what its beginning and end
// cost a CTA, in blocks, comes on top, and the places behind its blocks are empty.
struct SeqUnits {
  int first, n, len, ctx, groups, blocks;
  __device__ int span() const { return blocks + AT_ENDS; }
  __device__ long long work(int H) const { return (long long)H * groups * span(); }
};
template <int ROWS>
__device__ __forceinline__ SeqUnits seq_units(const AttendArgs& a, int s) {
  const SeqTokens t = seq_tokens(a.b, s, a.err);
  SeqUnits u;
  u.first = t.first;
  u.len = t.len;
  u.n = t.n;
  u.groups = t.n > 1 ? (int)(((long long)t.n * a.G + ROWS - 1) / ROWS) : t.n * a.one;
  if (a.skip_long && long_rows(t, a.G)) u.groups = 0;
  u.ctx = u.groups > 0 ? context(a.b, a.pool, t, a.err) : 0;
  u.blocks = max((u.ctx + BLK - 1) / BLK, 1);
  return u;
}
__device__ __forceinline__ long long div_pos(long long a, long long b) {   // a, b >= 0
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
// A unit of the list.
struct Unit {
  SeqUnits u;
  long long base, start;               // list positions of its sequence and of itself
  int s, h, row0, rows;                // sequence, KV head, rows of the sequence
  int tok0, rem0;                      // row0 = tok0 G + rem0
  int lim_hi;                          // its rows see at most 0 .. lim_hi
  __device__ __forceinline__ long long end() const { return start + u.span(); }
};
// A unit that lies in several CTAs' parts, the first of them p0.
struct Cut {
  Unit x;
  long long p0;
  int parts, first, n, last;           // of all parts, those that join with this CTA's first
};
// The unit that list position w lies in, from an earlier one (or from a sequence and its base).
template <int ROWS>
__device__ __forceinline__ void seek(const AttendArgs& a, Unit& x, long long w) {
  while (w >= x.base + x.u.work(a.pool.H)) {               // (sequences without tokens have no blocks)
    x.base += x.u.work(a.pool.H);
    x.u = seq_units<ROWS>(a, ++x.s);
  }
  const int unit = (int)div_pos(w - x.base, x.u.span());
  x.h = unit / x.u.groups;
  const int grp = unit - x.h * x.u.groups;
  x.start = x.base + (long long)unit * x.u.span();
  x.row0 = grp * ROWS;
  x.rows = min(ROWS, x.u.n * a.G - x.row0);
  x.tok0 = x.row0 / a.G;
  x.rem0 = x.row0 - x.tok0 * a.G;
  x.lim_hi = last_seen(x.u.len, (x.row0 + x.rows - 1) / a.G, x.u.ctx);
}
// Token and head of the unit's row i, without an integer division (i < 32, G up to 2^20: the
// quotient is at most 32, and its distance from the next whole number at least 1 / (2 G)).
__device__ __forceinline__ void token_of(const AttendArgs& a, const Unit& x, int i, int& tok, int& head) {
  const int r = x.rem0 + i, q = a.G >= 64 ? (r >= a.G) : (int)(((float)r + 0.5f) * a.inv_g);
  tok = x.tok0 + q;
  head = r - q * a.G;
}

// Four values of a finished row, and its normaliser.  A row that saw nothing: zeros and -inf.
template <int D>
__device__ __forceinline__ void write_out(const AttendArgs& a, const Unit& x, int i, int cc, float4 y, float m,
                                          float l) {
  int tok, head;
  token_of(a, x, i, tok, head);
  const long long row = ((long long)(x.u.first + tok) * a.pool.H + x.h) * a.G + head;
  const float inv = l == 0.f ? 0.f : (1.f / P_SCALE) / l;
  y.x *= inv; y.y *= inv; y.z *= inv; y.w *= inv;
  if (a.out_f32)
    reinterpret_cast<float4*>(a.out)[row * (D / 4) + cc] = y;
  else
    reinterpret_cast<uint2*>(a.out)[row * (D / 4) + cc] = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
  if (cc == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (m - W_OFF + log2f(l)) * 0.69314718055994530942f;
}

template <int D, int NT, int W, bool SPLIT>
__global__ void __launch_bounds__(32 * W, AT_CTAS) paged_attend_kernel(AttendArgs a) {
  using R = Ring<D, W>;
  constexpr int ROWS = 8 * NT, KW = D / 16, VW = D / 32;   // words a lane holds of a K / V row
  constexpr int RS = 8 * (D + 4);                          // a warp's 8 rows in shared memory
  constexpr bool QS = NT >= 2;                             // query operands in shared memory: no registers left
  extern __shared__ __align__(128) unsigned char sma[];
  float* accS = reinterpret_cast<float*>(sma + R::OFF_ACC);
  uint2* qS = reinterpret_cast<uint2*>(sma + R::OFF_Q);
  __shared__ float mS[W][ROWS], lS[W][ROWS];
  __shared__ float scaleS[W][R::ST][2];
  __shared__ long long scanS[W], foundS[2];
  __shared__ int foundsS[2], lastS;
  __shared__ Cut cutS[2];
  __shared__ Unit unitS[2], aheadS[W];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const int H = a.pool.H;
  // Behind the kernel of the long sequences, which lets this one start when all that came before is
  // done, nothing is to be waited for but that this one does not end first: its last CTA sees to that,
  // the others leave their places to those that have not begun.
  if (!a.skip_long) asm volatile("griddepcontrol.wait;" ::: "memory");
  auto leave = [&] {
    if (a.skip_long && blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
  };
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // ---- the list, and this CTA's part [w0, w1) of it
  const int per = (a.b.n_seq + 32 * W - 1) / (32 * W), sA = min(tid * per, a.b.n_seq), sB = min(sA + per, a.b.n_seq);
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
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w < warp) pre += scanS[w];
    total += scanS[w];
  }
  if (total == 0) {
    leave();
    return;
  }
  const long long share = max(div_pos(total + gridDim.x - 1, gridDim.x), (long long)W);   // a block a warp at least
  long long w0 = share * blockIdx.x, w1 = min(w0 + share, total);
  if (w0 >= total) {
    leave();
    return;
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {                            // the sequences of its first and its last block
    const long long w = e ? w1 - 1 : w0;
    if (pre - mine <= w && w < pre) {
      long long base = pre - mine;
      int s = sA;
      for (; s + 1 < sB; ++s) {
        const long long k = seq_units<ROWS>(a, s).work(H);
        if (w < base + k) break;
        base += k;
      }
      foundsS[e] = s;
      foundS[e] = base;
    }
  }
  __syncthreads();
  Unit x;
  x.s = foundsS[1];
  x.base = foundS[1];
  x.u = seq_units<ROWS>(a, x.s);
  seek<ROWS>(a, x, w1 - 1);
  // a short unit is not cut: it belongs to the part that it begins in
  auto uncut = [&] { return x.u.blocks <= AT_TINY || (x.u.blocks <= AT_SHORT && x.u.span() <= share); };
  if (uncut()) w1 = x.end();
  if (x.start > w0) {
    if (foundsS[0] != x.s) {
      x.s = foundsS[0];
      x.base = foundS[0];
      x.u = seq_units<ROWS>(a, x.s);
    }
    seek<ROWS>(a, x, w0);
  }
  if (x.start < w0 && (uncut() || w0 >= x.start + x.u.blocks)) w0 = x.end();
  if (w0 >= w1) {
    leave();
    return;
  }
  seek<ROWS>(a, x, w0);
  if (tid < W) aheadS[tid] = x;
  if (tid == 0) unitS[0] = x;

  // ---- the warp's ring: every W-th block of the part
  const uint32_t ring = smem_u32(sma) + warp * (R::ST * R::BLOCK);
  // a lane copies the 16 bytes at 512 i + 16 lane of a block's K and of its V
  constexpr int RPI = 512 / D;
  const int r0 = lane / (D / 16), c0 = lane % (D / 16), put0 = R::chunk_at(r0, c0), put1 = R::chunk_at(r0 + RPI, c0);
  bool more = true;                                        // the next block to ask for: its slot,
  int slot = 0, nt = (int)(w0 - x.start) + warp, stop = (int)min((long long)x.u.blocks, w1 - x.start);   // place, its unit's end,
  int nh = x.h, seen = x.lim_hi, id = -1;                  // head, last position that is seen, and page
  const int32_t* row = a.b.table + (long long)x.s * a.b.table_stride;
  __syncthreads();
  auto look = [&] {
    while (more && nt >= stop) {
      Unit y = aheadS[warp];
      if (!(more = y.end() < w1)) break;
      seek<ROWS>(a, y, y.end());
      __syncwarp();
      if (lane == 0) aheadS[warp] = y;
      __syncwarp();
      nt -= stop;
      stop = (int)min((long long)y.u.blocks, w1 - y.start);
      nh = y.h;
      seen = y.lim_hi;
      row = a.b.table + (long long)y.s * a.b.table_stride;
    }
    if (more && nt * BLK <= seen) id = row[nt * BLK >> a.pool.page_shift];
  };
  auto ask = [&] {
    if (more) {
      const int pos = nt * BLK;
      float* sc = &scaleS[warp][slot][0];
      if (pos <= seen && (unsigned)id < (unsigned)a.pool.n_pages) {
        const long long rows0 = ((long long)id * H + nh) * a.pool.page + (pos & (a.pool.page - 1));
        const unsigned char *kp = a.pool.k + rows0 * D + 16 * lane, *vp = a.pool.v + rows0 * D + 16 * lane;
        const uint32_t dst = ring + slot * R::BLOCK;
#pragma unroll
        for (int i = 0; i < BLK / RPI; ++i) {
          const uint32_t at = dst + (i & 1 ? put1 : put0) + 512 * (i & ~1);
          cp_async16(at, kp + 512 * i, 16);
          cp_async16(at + BLK * D, vp + 512 * i, 16);
        }
        if (lane < 2) cp_async4(smem_u32(sc + lane), (lane ? a.pool.vs : a.pool.ks) + rows0 / BLK);
      } else if (lane == 0) {                              // no row sees the block, or a bad page
        if (pos <= seen) report(a.err, ERR_PAGE);
        sc[1] = -1.f;
      }
      nt += W;
      slot = slot + 1 == R::ST ? 0 : slot + 1;
      look();
    }
    cp_commit();
  };
  look();
#pragma unroll 1
  for (int i = 0; i < R::ST; ++i) ask();

  int cuts = 0, came[2] = {0, 0};                          // units in several parts; parts that came before this one
  int next = warp, done = 0, stage = 0, turn = 0;          // the warp's next block of the CTA's; blocks so far
  for (long long w = w0; w < w1; turn ^= 1) {              // (never begins behind a unit's blocks)
    x = unitS[turn];
    seek<ROWS>(a, x, w);
    if (tid == 0) unitS[turn ^ 1] = x;                     // (read again behind the next barrier)
    const int ta = (int)(w - x.start), tb = (int)min((long long)x.u.blocks, w1 - x.start);
    const int lim_lo = last_seen(x.u.len, x.tok0, x.u.ctx), lim_hi = x.lim_hi;   // all rows see 0 .. lim_lo
    w = x.end();

    // ---- query rows, each scaled by a power of two, and what that makes of the logits
    uint32_t qf[NT][KW][2];
    float rc[NT][2];
    int lim[NT][2];                                        // last position a row sees
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const bool ok = 8 * j + g < x.rows;
      int tok, head;
      token_of(a, x, ok ? 8 * j + g : 0, tok, head);
      const bf16* qp = a.q + (long long)(x.u.first + tok) * a.q_ts + (long long)(x.h * a.G + head) * a.q_hs + 4 * KW * t4;
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < KW; k += 2) {
        const uint4 v = ok ? *reinterpret_cast<const uint4*>(qp + 4 * k) : make_uint4(0, 0, 0, 0);
        qf[j][k][0] = v.x; qf[j][k][1] = v.y;
        qf[j][k + 1][0] = v.z; qf[j][k + 1][1] = v.w;
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
        for (int e = 0; e < 2; ++e) {
          const uint32_t v = qf[j][k][e];
          qf[j][k][e] = pack_f16(__uint_as_float(v << 16) * f, __uint_as_float(v & 0xffff0000u) * f);
        }
      if (QS && warp == j)
#pragma unroll
        for (int k = 0; k < KW; ++k) qS[(j * KW + k) * 32 + lane] = make_uint2(qf[j][k][0], qf[j][k][1]);
      const float down = a.c * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        rc[j][e] = __shfl_sync(0xffffffffu, down, (2 * t4 + e) * 4);
        token_of(a, x, min(8 * j + 2 * t4 + e, x.rows - 1), tok, head);
        lim[j][e] = last_seen(x.u.len, tok, x.u.ctx);
      }
    }
    if (QS) __syncthreads();

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
    const int done0 = done;
    done += tb - ta;
    auto block = [&](auto at_edge) {
      constexpr bool edge = decltype(at_edge)::value;      // some row does not see the whole block
      const int t = ta + next - done0;                     // the block's place in the unit
      cp_wait<R::ST - 1>();
      __syncwarp();
      const float ks = scaleS[warp][stage][0], vs = scaleS[warp][stage][1];
      const unsigned char* kp = sma + (warp * R::ST + stage) * R::BLOCK;
      if (vs >= 0.f) {                                     // (warp-uniform)
        float sc[NT][4], sd[NT][4];                        // (two sums, even and odd words)
#pragma unroll
        for (int k = 0; k < KW; k += 4) {
          const uint4 ka = *reinterpret_cast<const uint4*>(kp + R::k_at(g, t4, k >> 2));
          const uint4 kb = *reinterpret_cast<const uint4*>(kp + R::k_at(g + 8, t4, k >> 2));
          const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t a0, a1, a2, a3;
            cvt4(wa[i], a0, a2);
            cvt4(wb[i], a1, a3);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              const uint2 b = QS ? qS[(j * KW + k + i) * 32 + lane] : make_uint2(qf[j][k + i][0], qf[j][k + i][1]);
              if (k + i < 2) mma_f16_0(i & 1 ? sd[j] : sc[j], a0, a1, a2, a3, b.x, b.y);
              else mma_f16(i & 1 ? sd[j] : sc[j], a0, a1, a2, a3, b.x, b.y);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[j][e] += sd[j][e];
        uint32_t vr[4][VW];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const unsigned char* q = kp + BLK * D + R::v_at(2 * t4 + (e & 1) + 8 * (e >> 1), g);
          if constexpr (VW == 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(q);
            vr[e][0] = v.x; vr[e][1] = v.y; vr[e][2] = v.z; vr[e][3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(q);
            vr[e][0] = v.x; vr[e][1] = v.y;
          }
        }
        uint32_t va[VW][2][4];                             // the values as operands
        auto values = [&] {
#pragma unroll
          for (int k = 0; k < VW; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // bytes 2 e, 2 e + 1 of word k of the four positions: values 2 (2 k + e) and the next
              cvt4(__byte_perm(vr[0][k], vr[1][k], e ? 0x7362 : 0x5140), va[k][e][0], va[k][e][1]);
              cvt4(__byte_perm(vr[2][k], vr[3][k], e ? 0x7362 : 0x5140), va[k][e][2], va[k][e][3]);
            }
        };
        constexpr bool EARLY = W == 6 && !edge;            // while the logits are on their way, where registers allow
        if (EARLY) values();
        const float ev = (float)((int)(__float_as_uint(vs) >> 23) - 127);
        // exponents from the row's base, in one rounding: as long as there is none (-inf) every
        // logit is too large
        float y[NT][4];
        auto exponents = [&](bool based) {
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              y[j][e] = fmaf(sc[j][e], rc[j][e & 1] * ks, based ? W_OFF - m[j][e & 1] : 0.f);
              if (edge && t * BLK + g + 8 * (e >> 1) > lim[j][e & 1]) y[j][e] = -INFINITY;
            }
        };
        exponents(true);
        bool up = false;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) up |= y[j][e] > W_OFF + BASE_STEP - ev;
        if (__any_sync(0xffffffffu, up)) {
          exponents(false);
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float mx = fmaxf(y[j][e], y[j][e + 2]);
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
              mx = fmaxf(mx + ev, m[j][e]);
              const float2 f = down2(m[j][e] - mx);
              const float al = f.x * f.y;
              m[j][e] = mx;
              l[j][e] = l[j][e] * f.x * f.y;
#pragma unroll
              for (int k = 0; k < KW; ++k) {
                o[j][k][e] *= al;
                o[j][k][e + 2] *= al;
              }
            }
          exponents(true);
        }
        const float pf = vs * P_SCALE;
        const uint64_t pf2 = f2_pack(pf, pf);
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
          for (int e = 0; e < 4; ++e) y[j][e] = ex2(y[j][e]);
#pragma unroll
          for (int e = 0; e < 2; ++e) l[j][e] += y[j][e] + y[j][e + 2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float p0, p1;
            f2_unpack(f2_mul(f2_pack(y[j][2 * e], y[j][2 * e + 1]), pf2), p0, p1);
            const uint32_t hi = pack_f16(p0, p1);
            ph[j][e] = movm(hi);
            if (SPLIT) {
              const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              pl[j][e] = movm(pack_f16(p0 - b.x, p1 - b.y));
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
#pragma unroll 1
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
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
        if (!EARLY) values();
#pragma unroll
        for (int k = 0; k < VW; ++k)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t a0 = va[k][e][0], a1 = va[k][e][1], a2 = va[k][e][2], a3 = va[k][e][3];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              if (SPLIT) {
                float z[4];
                mma_f16_0(z, a0, a1, a2, a3, pl[j][0], pl[j][1]);
                mma_f16(z, a0, a1, a2, a3, ph[j][0], ph[j][1]);
                float (&y)[4] = o[j][2 * k + e];
                f2_unpack(f2_add(f2_pack(y[0], y[1]), f2_pack(z[0], z[1])), y[0], y[1]);
                f2_unpack(f2_add(f2_pack(y[2], y[3]), f2_pack(z[2], z[3])), y[2], y[3]);
              } else {
                mma_f16(o[j][2 * k + e], a0, a1, a2, a3, ph[j][0], ph[j][1]);
              }
            }
          }
      }
      __syncwarp();                                        // every lane has read the block
      ask();
      stage = stage + 1 == R::ST ? 0 : stage + 1;
      next += W;
    };
    const int whole = min(done, done0 + (lim_lo + 1) / BLK - ta);   // blocks before this every row sees whole
#pragma unroll 1
    while (next < whole) block(std::false_type{});
#pragma unroll 1
    while (next < done) block(std::true_type{});

    // ---- the warps' rows join, 8 at a time
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int z = 4; z < 32; z <<= 1) l[j][e] += __shfl_xor_sync(0xffffffffu, l[j][e], z);
        if (g == 0) {
          mS[warp][8 * j + 2 * t4 + e] = m[j][e];
          lS[warp][8 * j + 2 * t4 + e] = l[j][e];
        }
      }
#pragma unroll 1
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int jj = 0; jj < NT; ++jj)
        if (jj == j) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float* p = accS + warp * RS + (2 * t4 + e) * (D + 4) + 2 * KW * g;
#pragma unroll
            for (int k = 0; k < KW; ++k)
              *reinterpret_cast<float2*>(p + 2 * k) = make_float2(o[jj][k][e], o[jj][k][e + 2]);
          }
        }
      __syncthreads();
      const Unit& y = unitS[turn ^ 1];
      const bool whole = ta == 0 && tb == y.u.blocks;
      const long long p0 = whole ? 0 : div_pos(y.start, share);   // the part that the unit begins in
      float* mypart = a.part + ((long long)blockIdx.x * 2 + (blockIdx.x == p0 ? 1 : 0)) * ROWS * (D + 4);
      for (int i = tid; i < 8 * (D / 4); i += 32 * W) {
        const int r = i / (D / 4), cc = i % (D / 4), col = 8 * j + r;
        if (col >= y.rows) continue;
        float mw[W], mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int z = 0; z < W; ++z) mt = fmaxf(mt, mw[z] = mS[z][col]);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int z = 0; z < W; ++z) {
          const float4 b = *reinterpret_cast<const float4*>(accS + z * RS + r * (D + 4) + 4 * cc);
          const float2 f2 = down2(mw[z] - mt);
          const float f = f2.x * f2.y;                     // (a NaN among the sums stays one)
          v.x = fmaf(b.x, f, v.x);
          v.y = fmaf(b.y, f, v.y);
          v.z = fmaf(b.z, f, v.z);
          v.w = fmaf(b.w, f, v.w);
          lt = fmaf(lS[z][col] * f2.x, f2.y, lt);
        }
        if (whole) {
          write_out<D>(a, y, col, cc, v, mt, lt);
        } else {
          float* p = mypart + (long long)col * (D + 4);
          __stcg(reinterpret_cast<float4*>(p + 4 * cc), v);
          if (cc == 0) __stcg(reinterpret_cast<float2*>(p + D), make_float2(mt, lt));
        }
      }
      __syncthreads();                                     // shared memory is free for the next rows
    }
    if (ta != 0 || tb != unitS[turn ^ 1].u.blocks) {       // (the part's first unit, or its last)
      if (tid == 0) {
        Cut& y = cutS[cuts];
        y.x = unitS[turn ^ 1];
        y.p0 = div_pos(y.x.start, share);
        y.parts = (int)(div_pos(y.x.start + y.x.u.blocks - 1, share) - y.p0) + 1;
        // many parts join in groups; a group's counter is that of its last part, which is no other unit's
        const bool grouped = y.parts > AT_FEW;
        const int group = group_of(y.parts);
        y.first = grouped ? (int)(blockIdx.x - y.p0) / group * group : 0;
        y.n = grouped ? min(group, y.parts - y.first) : y.parts;
        __threadfence();
        came[0] = came[1];                                 // (not waited for: the value is used at the end)
        came[1] = atomicAdd(grouped ? a.count + gridDim.x + y.p0 + y.first + y.n - 1 : a.count + y.p0, 1);
      }
      ++cuts;
    }
  }
  // ---- units in several parts: the CTA that came last joins them, in their order
  if (cuts > 0) {
    if (tid == 0) {
      cutS[cuts - 1].last = came[1] == cutS[cuts - 1].n - 1;
      if (cuts > 1) cutS[0].last = came[0] == cutS[0].n - 1;
    }
    __syncthreads();
#pragma unroll 1
    for (int e = 0; e < cuts; ++e) {
      const Cut& y = cutS[e];
      if (!y.last) continue;
      // the parts begin, begin + stride, ...: all of the unit, those of a group, or the groups' sums,
      // which lie in the places of their first parts
      int begin = y.first, stride = 1, n = y.n;
      bool all = n == y.parts, again;
      if (tid == 0) (all ? a.count + y.p0 : a.count + gridDim.x + y.p0 + begin + n - 1)[0] = 0;
#pragma unroll 1
      do {
        __threadfence();
        again = false;
        const int at_ml = stride == 1 ? D : D + 2;
        for (int i = tid; i < y.x.rows * (D / 4); i += 32 * W) {
          const int col = i / (D / 4), cc = i % (D / 4);
          auto place = [&](int k) { return a.part + (((y.p0 + k) * 2 + (k == 0)) * ROWS + col) * (D + 4); };
          float mt = -INFINITY, lt = 0.f;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int c0 = 0; c0 < n; c0 += AT_JOIN) {        // (a batch's loads are on their way together)
            float2 ml[AT_JOIN];
            float4 b[AT_JOIN];
#pragma unroll
            for (int c = 0; c < AT_JOIN; ++c) {            // (past the last part: the last again)
              const float* p = place(begin + min(c0 + c, n - 1) * stride);
              ml[c] = __ldcg(reinterpret_cast<const float2*>(p + at_ml));
              b[c] = __ldcg(reinterpret_cast<const float4*>(p + 4 * cc));
            }
            float mn = mt;
#pragma unroll
            for (int c = 0; c < AT_JOIN; ++c) mn = fmaxf(mn, ml[c].x);
            const float2 f2 = down2(mt - mn);
            const float fo = f2.x * f2.y;
            v.x *= fo; v.y *= fo; v.z *= fo; v.w *= fo;
            lt = lt * f2.x * f2.y;
#pragma unroll
            for (int c = 0; c < AT_JOIN; ++c)
              if (c0 + c < n) {                            // (a NaN in a part without a base stays one)
                const float2 g2 = down2(ml[c].x - mn);
                const float fn = g2.x * g2.y;
                v.x = fmaf(b[c].x, fn, v.x);
                v.y = fmaf(b[c].y, fn, v.y);
                v.z = fmaf(b[c].z, fn, v.z);
                v.w = fmaf(b[c].w, fn, v.w);
                lt = fmaf(ml[c].y * g2.x, g2.y, lt);
              }
            mt = mn;
          }
          if (all) {
            write_out<D>(a, y.x, col, cc, v, mt, lt);
          } else {
            float* p = place(begin);
            __stcg(reinterpret_cast<float4*>(p + 4 * cc), v);
            if (cc == 0) __stcg(reinterpret_cast<float2*>(p + D + 2), make_float2(mt, lt));
          }
        }
        if (!all) {
          const int groups = (y.parts - 1) / group_of(y.parts) + 1;
          __syncthreads();
          if (tid == 0) {
            __threadfence();
            lastS = atomicAdd(a.count + y.p0, 1) == groups - 1;
            if (lastS) a.count[y.p0] = 0;
          }
          __syncthreads();
          again = lastS;
          all = true;
          begin = 0;
          stride = group_of(y.parts);
          n = groups;
        }
      } while (again);
    }
  }
  leave();
}

template <int D, int NT, int W, bool SPLIT>
cudaError_t launch(const AttendArgs& a, int grid, cudaStream_t stream) {
  using R = Ring<D, W>;
  auto k = paged_attend_kernel<D, NT, W, SPLIT>;
  static std::atomic<unsigned long long> raised{0};
  const cudaError_t e = raise_smem_limit_once(raised, k, R::BYTES);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(32 * W);
  cfg.dynamicSmemBytes = R::BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a);
}
template <int D>
cudaError_t launch_d(AttendArgs& a, int sms, cudaStream_t stream) {
  const int grid = AT_CTAS * sms;
  // Groups of 8 rows a warp takes at once, and its registers (2 CTAs of 6 warps of 168, of 4 of 255, or,
  // for one group at d = 64, of 8 of 128: 64 sequences of 8192 102 us, 108 with 6), by the rows that a
  // sequence has on average.  One group streams at the rate of HBM and reads a cache once for each; more
  // read it less often, and compute longer.  16 sequences of 10000 positions and 4 heads, us for 8 / 16 /
  // 24 / 32 / 48 / 64 rows: fp32 results, groups of 1 38, 59, 77, 101, 141, 183; of 2 46, 50, 79, 79, 108,
  // 139; of 3 67, 71, 75, 120, 122, 167.  bf16: 1 37, 58, 71, 97, 131, 163; 2 42, 45, 66, 67, 89, 114; 3 49,
  // 52, 56, 87, 88, 119; 4 56, 59, 63, 67, 104, 106.  Lengths of 8 to 24 rows, 900 to 9000 positions: fp32
  // 68, 63, 78; bf16 62, 54, 58, 66.  (fp32 results of 4 groups, and of 2 with 6 warps, were slower throughout.)
  const long long rows = !a.b.starts || a.skip_long ? a.G : ((long long)a.b.n_tokens * a.G + a.b.n_seq - 1) / a.b.n_seq;
  const int nt = rows <= 8 ? 1 : a.out_f32 ? (rows > 20 && rows <= 24 ? 3 : 2)
                 : rows <= 18 ? 2 : rows <= 24 || (rows > 32 && rows <= 48) ? 3 : 4;
  a.one = (a.G + 8 * nt - 1) / (8 * nt);
  if (a.out_f32)
    return nt == 1 ? launch<D, 1, D == 64 ? 8 : 6, true>(a, grid, stream) : nt == 2 ? launch<D, 2, 4, true>(a, grid, stream)
                                                            : launch<D, 3, 4, true>(a, grid, stream);
  return nt == 1 ? launch<D, 1, D == 64 ? 8 : 6, false>(a, grid, stream) : nt == 2 ? launch<D, 2, 6, false>(a, grid, stream)
         : nt == 3 ? launch<D, 3, 4, false>(a, grid, stream) : launch<D, 4, 4, false>(a, grid, stream);
}

size_t counter_bytes(int sms) { return ((size_t)AT_CTAS * sms * 8 + 255) / 256 * 256; }

}  // namespace

static size_t part_bytes(int sms) { return (size_t)AT_CTAS * sms * 2 * AT_MAX_ROWS * (128 + 4) * 4; }
// [counters here][there] [partial results here][there]
size_t paged_attend_workspace(int sms) {
  return counter_bytes(sms) + paged_prompt_counters(sms) + part_bytes(sms) + paged_prompt_parts(sms);
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
  char* const counters = static_cast<char*>(workspace) + counter_bytes(sms);
  char* const parts = counters + paged_prompt_counters(sms);
  a.part = reinterpret_cast<float*>(parts);
  a.err = err;
  a.c = (float)(1.4426950408889634 / sqrt((double)pool.d));
  a.G = HQ / pool.H;
  a.inv_g = 1.f / (float)a.G;
  if (b.starts && (long long)a.G * b.max_new > LONG_ROWS && paged_prompt_fits(pool, b, HQ)) {
    a.skip_long = 1;
    const cudaError_t e = launch_paged_prompt(pool, b, q, q_ts, q_hs, HQ, out, out_f32, lse, counters,
                                              parts + part_bytes(sms), sms, err, stream);
    if (e != cudaSuccess) return e;
  }
  return pool.d == 128 ? launch_d<128>(a, sms, stream) : launch_d<64>(a, sms, stream);
}

}  // namespace kvpop
