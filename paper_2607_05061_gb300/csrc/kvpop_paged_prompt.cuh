// Attention of many new tokens a sequence over the paged 8-bit cache, on tcgen05.
//
// The mathematics is that of kvpop_paged_attend.cu: f16 products that are exact for the logits,
// the value scales in the weights' operand, p = 2^(x log2 e - M + 2) 2^(ev + 5) as one f16 (bf16
// results) or the sum of two (fp32 results, SPLIT).  A CTA owns 256 consecutive rows (token, query head) of
// one (sequence, KV head), as two halves of 128 rows, and streams the positions they see in blocks
// of 64, the same bytes for both halves.  Roles:
//  * 3 converter warps: bulk copies bring the bytes of keys and values into shared memory, two tiles
//    ahead for each warp, which writes them as f16 into a ring of 7 or 10 128B-swizzled tiles (a
//    block's keys, then its values), with the scales beside them.
//  * 1 MMA warp: S = Q K^T (M 128, N 64, K d) per half, and O += P V (N d, K 64) with P in tensor
//    memory and the values read MN-major from their rows.
//  * 2 x 4 softmax warps, a thread per row: logits into registers, the row's maximum,
//    probabilities over the logits.
// Tensor memory: O (2 x 128 columns) and two buffers of logits (4 x 64), P in the place of its
// logits.  The logits of block j + 2 follow the product with block j into its buffer in the order
// the MMAs are issued, and those of block j + 1 are there when a row is done with block j, so a
// block costs a softmax warp one wait and one signal.  O adds up cut off: after a chain of blocks the
// softmax warps move it to running sums in L2, where it is added rounded, and the next product starts
// from zero.
//
// What bounds it, for a block of 64 positions (d = 128, about 1950 clocks; the two products' share of
// the tensor rate is 1024): the products, which the MMA warp issues for 1630 clocks, 1070 of them for
// S, whose 128 query rows come from shared memory for every 64 keys (66 clocks a step of 16, 32 by
// the tensor rate), and the softmax's 1270 clocks a warp, which wait for each other across the
// halves.  A tile costs 7 to 9 us besides: queries, first products, output.
// A prompt of 8192 tokens with 32 query and 8 KV heads takes 503 us (bf16 results; 773 with fp32
// ones), 57% of the bf16 rate; at d = 64 331 (520).  Measured before, in order: blocks of 128 in one
// buffer, where a half's rows and its products took turns, 672; blocks of 64 with P in a place of its
// own, two waits and two signals a block, 622; P over its logits 575; queries and results read and
// written by rows, the converters' first tiles beside them 549; blocks that all rows see whole apart,
// without the masks' selects, 497 (503 since the weights are apart from the products' operand).  Not kept: softmax warps that ask for the next logits before the
// exponentials (642 then) or signal behind the next block's loads (504); register splits between the
// roles (631); two threads a row (1799); a CTA that takes tile after tile (770: spills).
#pragma once

#include <type_traits>

#include "kvpop_mma.cuh"
#include "kvpop_paged.cuh"
#include "kvpop_ptx.cuh"
#include "kvpop_tc05.cuh"

namespace kvpop {
namespace {

using namespace paged;
using namespace tc05;

constexpr int PP_HALF = 128, PP_ROWS = 2 * PP_HALF, PP_KEYS = 64;
constexpr int PP_MMA_WARP = 8, PP_CONV_WARP = 9, PP_CONV = 3;    // warps 0-7: softmax, 8: MMA, 9-11: converters
constexpr int PP_THREADS = 32 * (PP_CONV_WARP + PP_CONV);
constexpr int PP_RING = 10, PP_SCALES = 16;              // tiles at most; blocks whose scales are held
constexpr int PP_TMEM = 512;                             // O_h: 128 h (d = 64: and Q_h, 128 h + 64); S_h,b: 256 + 128 h + 64 b
constexpr int PP_PARTS = 8, PP_LEAST = 8;                // parts of a tile at most; blocks of a part at least
constexpr int PP_MORE_PARTS = 32;                        // parts of a tile at most, where another kernel joins them
// barriers
constexpr int PB_FULL = 0;                               // [ring] converters -> MMA
constexpr int PB_EMPTY = PB_FULL + PP_RING;              // [ring] MMA -> converters
constexpr int PB_S = PB_EMPTY + PP_RING;                 // [2][2] MMA -> softmax: logits of even, odd blocks there
constexpr int PB_P = PB_S + 4;                           // [2][2] softmax -> MMA: their probabilities there
// A wait by parity does not tell the phase it is for from the one two before.  At block j the product
// with block j - 2 is done (the logits of j follow it) and that with j is not begun, so that j - 1 can be
// waited for; at the end nothing says that the last but one is done: the end has a barrier of its own.
constexpr int PB_O = PB_P + 4;                           // [2] MMA -> softmax: a product done
constexpr int PB_END = PB_O + 2;                         // MMA -> softmax: all products done
constexpr int PB_RAW = PB_END + 1;                       // [converters][2] bytes there
constexpr int PB_SLOT = PB_RAW + 2 * PP_CONV;            // MMA -> softmax: the place for running sums claimed
constexpr int PB_N = PB_SLOT + 1;
// Blocks whose products add up in tensor memory before a row's sums move on.  The tensor cores cut off
// what they add, by 0.7 of 2^-23 of the sum so far each time (values of one sign, 16384 positions in one
// sum: 8.8e-5 of an fp32 result; in chains of 32, 16, 8 blocks 4e-6, 2.1e-6, 1.2e-6, and a prompt of 8192
// takes 674, 707, 770 us, 629 in one sum).  256 blocks leave a bf16 result 3e-5, a 60th of its rounding;
// where no tile has more, the kernel is without the moves (a prompt of 8192 503 us, 510 with them).
constexpr int PP_CHAIN = 8, PP_CHAIN_BF16 = 256;
constexpr int PP_NANW = (PP_ROWS + 2 * PP_KEYS) / 32;    // words of the map of NaN values

struct PromptArgs {
  Pool pool;
  Batch b;
  const bf16* q;
  long long q_ts, q_hs;
  void* out;
  float* lse;
  int32_t* err;
  float* part;                                           // [slots][d / 8][256][8] sums of parts
  float2* part_ml;                                       // [slots][256] their bases and normalisers
  int* count;                                            // [slots] parts there, zero between calls
  float* sum;                                            // [SMs][d / 4][256][4] running sums of CTAs
  int* claim;                                            // [SMs] places of `sum` in use, zero between calls
  float c;                                               // log2(e) / sqrt(d)
  int G, out_f32, sms;
  Parts to;                                              // PARTS: what takes the place of sequences, and of results
};

// 32 bytes, 32-byte aligned
__device__ __forceinline__ void st32(void* p, const float* v) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]),
               "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

template <int D>
struct PL {
  static constexpr int QB = PP_HALF * D * 2, KB = PP_KEYS * D * 2;
  // Queries in tensor memory where there is room (d = 64): from shared memory their 128 rows bound the
  // products with 64 keys (the 8 of a block 527 clocks, 399 with them there; 8192 tokens 349 us, 329).
  static constexpr bool Q_TMEM = D == 64;
  static constexpr int RING = D == 128 ? 7 : PP_RING, RAW = PP_KEYS * D;   // tiles of f16; bytes of a tile of codes
  static constexpr int OFF_RING = 2 * QB, OFF_RAW = OFF_RING + RING * KB, OFF_BAR = OFF_RAW + 2 * PP_CONV * RAW;
  static constexpr int OFF_TMEM = OFF_BAR + 8 * PB_N, OFF_NAN = (OFF_TMEM + 4 + 15) / 16 * 16;
  // [16 blocks] of 4 groups: key scales, value exponents (-inf: not to be seen), value scales times 32, 0 or -inf
  static constexpr int OFF_SCALE = OFF_NAN + 4 * PP_NANW, SCALES = 16;
  static constexpr int OFF_KEEP = OFF_SCALE + PP_SCALES * SCALES * 4;   // what only the end needs
  static constexpr int OFF_BASE = OFF_KEEP + 48;         // [rows] bases of the running sums
  static constexpr int BYTES = OFF_BASE + PP_ROWS * 4;
  static_assert(PP_PARTS * PP_ROWS * 4 <= OFF_BAR, "");  // factors of the parts, where queries and ring were
};

// f16 A and B, fp32 D, M x N, optional MN-major B
__device__ __forceinline__ uint32_t idesc_f16(int M, int N, int b_mn_major) {
  return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
// 16 e4m3 bytes -> 16 f16
__device__ __forceinline__ void cvt16(const uint4& w, uint4& a, uint4& b) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(o[2 * i]), "=r"(o[2 * i + 1])
        : "r"(u[i]));
  a = make_uint4(o[0], o[1], o[2], o[3]);
  b = make_uint4(o[4], o[5], o[6], o[7]);
}
__device__ __forceinline__ bool has_nan(uint32_t w) {   // an e4m3 NaN (0x7f, 0xff) among four bytes
  const uint32_t x = (w & 0x7f7f7f7fu) + 0x01010101u;   // no byte carries: 0x7f + 1 = 0x80
  return (x & 0x80808080u) != 0;
}
__device__ __forceinline__ uint32_t drop_nan(uint32_t w) {
  const uint32_t x = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return w & ~((x >> 7) * 255u);
}

// Blocks of a part at most, by all lanes of a warp.  A tile costs what ENDS blocks do besides its
// own (5 to 7 us; a block takes 0.7 us at d = 64, 1.0 at 128), and its parts, if it is cut, JOIN
// blocks each: one SM reads them all.  Where every part has an SM of its own, the longest is what
// the call takes; else they fill the SMs in turn, and half of the longest is left at the end.
// JOINED: they are.  Else another kernel reads them, over all SMs.
template <bool JOINED>
__device__ __forceinline__ int share_of(int tiles, int most, float all, int sms, int parts, int lane) {
  constexpr float ENDS = 7.f, JOIN = JOINED ? 3.f : 0.125f;
  const int c = min(lane + 1, parts), b = (most - 1) / c + 1;
  const float n = c == 1 ? (float)tiles : fmaxf(__fdividef(all, (float)b) + 0.5f * (float)tiles, (float)tiles);
  const float one = ENDS + (c > 1 ? JOIN * (float)c : 0.f), each = __frcp_rn((float)sms);
  float cost = n <= (float)sms ? one + (float)b : (all + n * one) * each + 0.5f * ((float)b + one);
  if (c > 1 && b < PP_LEAST) cost = 3e38f;
  const unsigned key = __reduce_min_sync(0xffffffffu, (__float_as_uint(cost) & ~31u) | (unsigned)(c - 1));
  return __shfl_sync(0xffffffffu, b, key & 31u);
}

// A place for running sums, of the first thread that asks; -1: none was free.  There is one for every
// CTA that can run at once, and the SM's own is the one that its last CTA gave back.
__device__ __noinline__ int claim_place(int* claim, int sms) {
  unsigned at;
  asm volatile("mov.u32 %0, %%smid;" : "=r"(at));
  for (int i = 0; i < 64 * sms; ++i, ++at)
    if (atomicCAS(claim + at % (unsigned)sms, 0, 1) == 0) return (int)(at % (unsigned)sms);
  return -1;
}
// A row's sums in tensor memory (by all lanes) join the running ones: O 2^up is added to them, in L2; or
// (set) they become O + 2^-up of them, or O.
template <int D>
__device__ __noinline__ void move_sums(uint32_t tO, float* to, float up, bool set, bool none) {
  const float f = set ? ex2(-up) : ex2(up);
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    float o[32];
    tmem_ld32(tO + c * 32, o);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i, to += 4 * PP_ROWS) {
      float* v = o + 4 * i;
      if (!set) {
        asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(to), "f"(v[0] * f), "f"(v[1] * f),
                     "f"(v[2] * f), "f"(v[3] * f)
                     : "memory");
      } else {
        const float4 b = none ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcg(reinterpret_cast<const float4*>(to));
        __stcg(reinterpret_cast<float4*>(to), make_float4(fmaf(b.x, f, v[0]), fmaf(b.y, f, v[1]), fmaf(b.z, f, v[2]),
                                                          fmaf(b.w, f, v[3])));
      }
    }
  }
}

// The sums in tensor memory become O + f times the running ones.
template <int D>
__device__ __noinline__ void fetch_sums(uint32_t tO, const float* from, float f) {
  __threadfence();
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c, tO += 32) {
    float4 b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i, from += 4 * PP_ROWS) b[i] = __ldcg(reinterpret_cast<const float4*>(from));
    float o[32];
    tmem_ld32(tO, o);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      o[4 * i] = fmaf(b[i].x, f, o[4 * i]);
      o[4 * i + 1] = fmaf(b[i].y, f, o[4 * i + 1]);
      o[4 * i + 2] = fmaf(b[i].z, f, o[4 * i + 2]);
      o[4 * i + 3] = fmaf(b[i].w, f, o[4 * i + 3]);
    }
    tmem_st32(tO, o);
    tmem_wait_st();
  }
}

// CHAINED: the sums move on after each chain of blocks.  PARTS: the tiles are those of a.to.entries, and
// rows leave as sums.
template <int D, bool SPLIT, bool CHAINED, bool PARTS>
__global__ void __launch_bounds__(PP_THREADS, 1) paged_prompt_kernel(PromptArgs a) {
  using L = PL<D>;
  constexpr int RING = L::RING, CHAIN = SPLIT ? PP_CHAIN : PP_CHAIN_BF16;
  extern __shared__ __align__(1024) unsigned char smp[];
  const uint32_t sb = smem_u32(smp);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = a.pool.H, G = a.G;
  // What came before is done; the sequences with few rows may come into the SMs that are done with this.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8u * (uint32_t)i; };
  uint32_t* nanS = reinterpret_cast<uint32_t*>(smp + L::OFF_NAN);

  // ---- the tile: sequence s owns the places from starts[s] G / 256 + s on, which leaves one for
  // each of its tiles.  Later tokens see more, and go first.
  const unsigned order = gridDim.x - 1 - blockIdx.x;
  int place = (int)(order / (unsigned)H), h = (int)(order % (unsigned)H), part = blockIdx.y;
  auto first_place = [&](int s) { return (long long)a.b.starts[s] * G / PP_ROWS + s; };
  int s = -1, tiles = 0, most = 0;                       // tiles of all sequences, blocks of the longest
  float all_blocks = 0.f;
  int all_tiles = 0;
  if constexpr (PARTS) {
    // all tiles' first parts, then their second ones, ...; the plan has made the list
    all_tiles = a.to.tiles[TILES_ALL];
    if (all_tiles == 0) return;
    part = (int)(blockIdx.x / (unsigned)all_tiles);
    const int tile = all_tiles - 1 - (int)(blockIdx.x % (unsigned)all_tiles);
    place = tile / H;
    h = tile - place * H;
    for (int i0 = 0; i0 < a.b.n_seq && s < 0; i0 += 32) {
      const int i = i0 + lane;
      const Entry e = a.to.entries[i < a.b.n_seq ? i : 0];
      const int k = i < a.b.n_seq && e.place >= 0 ? (int)(((long long)e.n * G + PP_ROWS - 1) / PP_ROWS) : 0;
      const unsigned who = __ballot_sync(0xffffffffu, k > 0 && e.place <= place && place < e.place + k);
      if (who) s = i0 + __ffs(who) - 1;
    }
  } else
  for (int i0 = 0; i0 < a.b.n_seq; i0 += 32) {           // (each warp for itself)
    const int i = i0 + lane;
    const bool in = i < a.b.n_seq;
    const bool has = in && first_place(i) <= place && (i + 1 == a.b.n_seq || place < first_place(i + 1));
    const unsigned who = __ballot_sync(0xffffffffu, has);
    if (who) s = i0 + __ffs(who) - 1;
    if (gridDim.y > 1) {
      if (in) {
        const SeqTokens t = seq_tokens(a.b, i, a.err);
        if (long_rows(t, G)) {
          const long long end = min((long long)t.len + t.n, (long long)a.b.max_pages << a.pool.page_shift);
          const int k = (int)(((long long)t.n * G + PP_ROWS - 1) / PP_ROWS) * H, b = (int)(end / PP_KEYS) + 1;
          tiles += k;
          most = max(most, b);
          all_blocks += (float)k * (float)((min((long long)t.len, end) / PP_KEYS + 1 + b) >> 1);
        }
      }
    } else if (who) {
      break;
    }
  }
  if (s < 0) return;                                     // (offsets that do not ascend)
  int share = PARTS ? a.to.tiles[TILES_SHARE] : INT32_MAX;         // blocks of a part at most
  if (!PARTS && gridDim.y > 1) {
    tiles = __reduce_add_sync(0xffffffffu, tiles);
    most = __reduce_max_sync(0xffffffffu, most);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all_blocks += __shfl_xor_sync(0xffffffffu, all_blocks, o);
    share = max(share_of<true>(tiles, most, all_blocks, a.sms, (int)gridDim.y, lane), 1);
  }
  Entry e{};
  SeqTokens t;
  if constexpr (PARTS) {
    e = a.to.entries[s];
    t = SeqTokens{e.first, e.n, e.len};
  } else {
    t = seq_tokens(a.b, s, a.err);
  }
  const long long row0l = (place - (PARTS ? e.place : first_place(s))) * PP_ROWS, all_rows = (long long)t.n * G;
  if ((!PARTS && !long_rows(t, G)) || row0l < 0 || row0l >= all_rows) return;
  const int row0 = (int)row0l, rows = (int)min((long long)PP_ROWS, all_rows - row0l);
  const int ctx = PARTS ? e.ctx : context(a.b, a.pool, t, a.err);
  const int begin = PARTS ? e.begin / PP_KEYS : 0;       // first block
  const int32_t* const trow = a.b.table + (long long)(PARTS ? e.row : s) * a.b.table_stride;
  const int lim_lo = last_seen(t.len, row0 / G, ctx);    // every row sees 0 .. lim_lo
  const int lim_hi = last_seen(t.len, (row0 + rows - 1) / G, ctx);   // none sees past lim_hi
  const int blocks = PARTS ? max(lim_hi / PP_KEYS + 1 - begin, 1) : lim_hi / PP_KEYS + 1;
  const int cut = min((blocks - 1) / share + 1, PARTS ? max(min(a.to.room / all_tiles, PP_MORE_PARTS), 1) : (int)gridDim.y);
  if (part >= cut) return;
  const int blk0 = (int)((long long)blocks * part / cut), nblk = (int)((long long)blocks * (part + 1) / cut) - blk0;
  const int key0 = (begin + blk0) * PP_KEYS;             // first position of the part
  const int nan0 = (lim_lo + 1) / PP_KEYS * PP_KEYS;     // first position of the NaN map

  if (tid == 0) {
    for (int i = 0; i < RING; ++i) {
      mbar_init(bar(PB_FULL + i), 1);
      mbar_init(bar(PB_EMPTY + i), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(PB_S + i), 1);
      mbar_init(bar(PB_P + i), 4);
    }
    for (int i = 0; i < 2 * PP_CONV; ++i) mbar_init(bar(PB_RAW + i), 1);
    mbar_init(bar(PB_O + 0), 1);
    mbar_init(bar(PB_O + 1), 1);
    mbar_init(bar(PB_END), 1);
    mbar_init(bar(PB_SLOT), 1);
    mbar_fence_init();
  }
  if (tid < PP_NANW) nanS[tid] = 0;
  // The end reads these from here: in registers they would be spilled around the roles' loops.
  volatile int* keep = reinterpret_cast<volatile int*>(smp + L::OFF_KEEP);
  if (tid == 0) {
    keep[0] = t.first;
    keep[1] = row0;
    keep[2] = rows;
    keep[3] = cut;
    keep[4] = place;
    keep[5] = h;
    keep[6] = nan0;
    keep[7] = -1;
    if (PARTS) {
      keep[8] = s;
      if (part == 0) a.to.tiles[TILES_PARTS + place * H + h] = cut;
    }
  }
  if (warp == PP_MMA_WARP) tmem_alloc(sb + L::OFF_TMEM, PP_TMEM);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smp + L::OFF_TMEM);

  // ---- query rows as f16, each scaled by a power of two.  A warp reads whole rows, 16 bytes a
  // lane; rc and lim are those of the row that the thread owns in the softmax.
  float rc = 0.f;
  int lim = -1;
  if (warp < PP_MMA_WARP) {
    constexpr int LPR = D / 8, RPI = 32 / LPR, IT = 32 / RPI;   // lanes of a row, rows at a time
    const int r = row0 + min(tid, rows - 1), tok = r / G;
    const long long off = (t.first + tok) * a.q_ts + (long long)(h * G + (r - tok * G)) * a.q_hs;
    const int c = lane % LPR, sub = lane / LPR;
    if (tid < rows) lim = last_seen(t.len, tok, ctx);
    uint4 v[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const long long o = __shfl_sync(0xffffffffu, off, i * RPI + sub);
      v[i] = *reinterpret_cast<const uint4*>(a.q + o + 8 * c);
    }
    int mine = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      uint32_t top = __vmaxu2(__vmaxu2(u[0] & 0x7fff7fffu, u[1] & 0x7fff7fffu),
                              __vmaxu2(u[2] & 0x7fff7fffu, u[3] & 0x7fff7fffu));
      top = max(top >> 16, top & 0xffffu);
#pragma unroll
      for (int k = 1; k < LPR; k <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, k));
      const int up = max(min(14 - ((int)(top >> 7) - 127), 110), -113);   // the largest to [2^14, 2^15)
      const int its = __shfl_sync(0xffffffffu, up, lane % RPI * LPR);
      if (lane / RPI == i) mine = its;
      const float f = __uint_as_float((uint32_t)(up + 127) << 23);
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        o[k] = pack_h2(__uint_as_float(u[k] << 16) * f, __uint_as_float(u[k] & 0xffff0000u) * f);
      const int row = warp * 32 + i * RPI + sub;         // (rows that are none: the last one again)
      *reinterpret_cast<uint4*>(smp + (row >> 7) * L::QB + tile_off(row & 127, c, PP_HALF)) =
          make_uint4(o[0], o[1], o[2], o[3]);
    }
    rc = a.c * __uint_as_float((uint32_t)(127 - mine) << 23);
    if (L::Q_TMEM) {                                     // a thread moves its row on
      __syncwarp();
      float q[32];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 u = *reinterpret_cast<const uint4*>(smp + (tid >> 7) * L::QB + tile_off(tid & 127, i, PP_HALF));
        q[4 * i] = __uint_as_float(u.x);
        q[4 * i + 1] = __uint_as_float(u.y);
        q[4 * i + 2] = __uint_as_float(u.z);
        q[4 * i + 3] = __uint_as_float(u.w);
      }
      tmem_st32(tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * 128 + 64, q);
      tmem_wait_st();
      fence_before();
    } else {
      fence_async_smem();
    }
    // (only the products wait for them: the converters are on their way)
    asm volatile("bar.arrive 1, %0;" ::"n"(32 * PP_MMA_WARP + 32) : "memory");
  }
  // page of a position, -1 where the rows do not see it
  auto page16 = [&](int pos) {
    if constexpr (PARTS) {
      const int id = pos <= lim_hi ? trow[pos >> a.pool.page_shift] : -1;
      return (unsigned)id < (unsigned)a.pool.n_pages ? id : -1;
    } else {
      return pos <= lim_hi ? page_of(a.b, a.pool, s, pos, a.err) : -1;
    }
  };
  auto wait = [&](int b, int parity) {                   // the whole warp; false: gave up
    if (__all_sync(0xffffffffu, mbar_try_wait(bar(b), parity))) return true;
    return (bool)__all_sync(0xffffffffu, mbar_wait(bar(b), parity, a.err, ERR_WAIT));
  };
  float m = -INFINITY, l = 0.f;
  bool ok = true;

  if (warp >= PP_CONV_WARP) {
    // ---------------------------------------------------------------- converters
    // Tile i (keys of block i / 2, or its values) is warp i mod 3's.  Its bytes are asked for two of
    // the warp's tiles ahead, as bulk copies, which the fence of a tile does not wait for.
    constexpr int LPR = D / 16, RPI = 32 / LPR, IT = PP_KEYS / RPI, PER = PP_KEYS / BLK;   // lanes of a row, rows at a time
    // (d = 128: 8 neighbouring lanes hold half of two neighbouring rows, so that their stores, even
    // chunks and then odd ones, touch every bank)
    const int c = D == 128 ? (lane & 3) + (lane >> 1 & 4) : lane % LPR;
    const int sub = D == 128 ? (lane >> 2 & 1) + 2 * (lane >> 4) : lane / LPR, tiles = 2 * nblk;
    const int cw = warp - PP_CONV_WARP, per_copy = min(a.pool.page, PP_KEYS);
    auto group_pos = [&](int i) { return key0 + (i >> 1) * PP_KEYS + (lane & (PER - 1)) * BLK; };
    auto look = [&](int i) { return trow[min(group_pos(i), lim_hi) >> a.pool.page_shift]; };   // page of group lane mod 4
    auto is_page = [&](int id) { return (unsigned)id < (unsigned)a.pool.n_pages; };
    auto head_of = [&](int id) { return ((long long)(is_page(id) ? id : 0) * H + h) * a.pool.page; };
    // the warp's n-th tile into its buffer n mod 2: whole groups, as far as they are in one page
    auto fetch = [&](int n, int id) {
      const int i = cw + n * PP_CONV, pos = group_pos(i);
      const bool go = lane < PER && (lane * BLK & (per_copy - 1)) == 0 && pos <= lim_hi && is_page(id);
      const uint32_t to = bar(PB_RAW + 2 * cw + (n & 1));
      const int copies = __popc(__ballot_sync(0xffffffffu, go));
      if (lane == 0) mbar_arrive_expect_tx(to, copies * per_copy * D);
      __syncwarp();
      if (go)
        bulk_g2s(sb + L::OFF_RAW + (2 * cw + (n & 1)) * L::RAW + lane * BLK * D,
                 (i & 1 ? a.pool.v : a.pool.k) + (head_of(id) + (pos & (a.pool.page - 1))) * D, per_copy * D, to);
    };
    // lanes 0-3: the scales of the groups' keys, 4-7: of their values
    auto scale_of = [&](int i, int id) {
      return (lane & PER ? a.pool.vs : a.pool.ks)[(head_of(id) + (group_pos(i) & (a.pool.page - 1))) / BLK];
    };
    const int mine = (tiles - cw + PP_CONV - 1) / PP_CONV;   // tiles of the warp
    int id = look(cw), id1 = look(cw + PP_CONV), id2 = look(cw + 2 * PP_CONV), asked = min(mine, 2), had = 0;
    float scale = scale_of(cw, id);
    if (mine > 0) fetch(0, id);
    if (mine > 1) fetch(1, id1);
#pragma unroll 1
    for (int n = 0; n < mine; ++n) {
      const int i = cw + n * PP_CONV, st = i % RING, pos0 = key0 + (i >> 1) * PP_KEYS;
      if (!wait(PB_RAW + 2 * cw + (n & 1), n >> 1 & 1)) break;
      had = n + 1;
      uint4 w[IT];
      const unsigned char* raw = smp + L::OFF_RAW + (2 * cw + (n & 1)) * L::RAW + sub * D + 16 * c;
#pragma unroll
      for (int x = 0; x < IT; ++x) w[x] = *reinterpret_cast<const uint4*>(raw + x * RPI * D);
      __syncwarp();                                      // every lane has its bytes
      if (n + 2 < mine) {
        fetch(n + 2, id2);
        asked = n + 3;
      }
      if (i >= RING && !wait(PB_EMPTY + st, (i / RING - 1) & 1)) break;
      const bool seen = group_pos(i) <= lim_hi, in = seen && is_page(id);
      if (seen && !in) report(a.err, ERR_PAGE);
      if (!in) scale = 0.f;                              // (nothing to see)
      if (!__all_sync(0xffffffffu, in && pos0 + PP_KEYS - 1 <= lim_hi)) {
#pragma unroll
        for (int x = 0; x < IT; ++x) {
          const bool ok_ = __shfl_sync(0xffffffffu, (int)in, x * RPI / BLK) && pos0 + x * RPI + sub <= lim_hi;
          if (!ok_) w[x] = make_uint4(0, 0, 0, 0);
        }
      }
      if (!(i & 1) && lane < 2 * PER) {                  // both scales with the keys, which the logits wait for
        float* to = reinterpret_cast<float*>(smp + L::OFF_SCALE) + (i >> 1) % PP_SCALES * L::SCALES + lane;
        const uint32_t e = __float_as_uint(scale) >> 23;
        to[0] = lane < PER ? scale : scale > 0.f ? (float)((int)e - 127) : -INFINITY;
        if (lane >= PER) {
          to[PER] = scale * P_SCALE;
          to[2 * PER] = scale > 0.f ? 0.f : -INFINITY;
        }
      }
      if ((i & 1) && pos0 + PP_KEYS - 1 > lim_lo) {
        // Values that some row does not see: a NaN must not reach the rows before it, where its
        // weight is 0.  Its column is set at the end, for the rows that see it.
#pragma unroll
        for (int x = 0; x < IT; ++x)
          if (has_nan(w[x].x) || has_nan(w[x].y) || has_nan(w[x].z) || has_nan(w[x].w)) {
            const int at = pos0 + x * RPI + sub - nan0;
            atomicOr(nanS + (at >> 5), 1u << (at & 31));
            w[x] = make_uint4(drop_nan(w[x].x), drop_nan(w[x].y), drop_nan(w[x].z), drop_nan(w[x].w));
          }
      }
      unsigned char* tile = smp + L::OFF_RING + st * L::KB;
#pragma unroll
      for (int x = 0; x < IT; ++x) {
        uint4 p, q;
        cvt16(w[x], p, q);
        const int row = x * RPI + sub;
        *reinterpret_cast<uint4*>(tile + tile_off(row, 2 * c, PP_KEYS)) = p;
        *reinterpret_cast<uint4*>(tile + tile_off(row, 2 * c + 1, PP_KEYS)) = q;
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(PB_FULL + st));
      // (here: the fence above waits for every load that is on its way)
      id = id1;
      id1 = id2;
      id2 = look(i + 3 * PP_CONV);
      scale = scale_of(i + PP_CONV, id);
    }
    for (; had < asked; ++had) wait(PB_RAW + 2 * cw + (had & 1), had >> 1 & 1);   // (gave up: no copy is left behind)
  } else if (warp == PP_MMA_WARP) {
    // ---------------------------------------------------------------- MMA issue
    const uint32_t idS = idesc_f16(128, PP_KEYS, 0), idO = idesc_f16(128, D, 1);
    const bool lead = elect_one();
    if (CHAINED && nblk > CHAIN) {                       // (while the queries come)
      if (lane == 0) {
        keep[7] = claim_place(a.claim, a.sms);
        mbar_arrive(bar(PB_SLOT));
      }
      __syncwarp();
    }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * PP_MMA_WARP + 32) : "memory");
    fence_after();
    const uint64_t qd0 = kmajor_desc(sb, PP_HALF, 0), kd0 = kmajor_desc(sb + L::OFF_RING, PP_KEYS, 0);
    const uint64_t vd0 = mnmajor_desc(sb + L::OFF_RING, PP_KEYS, 0);
    auto issue_s = [&](int hf, int j) {                  // logits of half hf against block j
      const int st = 2 * j % RING;
      if (hf == 0) {
        if (!(ok = ok && wait(PB_FULL + st, (2 * j / RING) & 1))) return;
        fence_after();
      }
      if (lead) {
        const uint64_t kd = desc_at(kd0, st * L::KB), qd = desc_at(qd0, hf * L::QB);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint32_t to = tmem + 256 + hf * 128 + (j & 1) * 64;
          const uint64_t kk = kmajor_step(kd, PP_KEYS, ks);
          if (L::Q_TMEM) mma_bf16_ts(to, tmem + hf * 128 + 64 + 8 * ks, kk, idS, ks > 0);
          else mma_bf16(to, kmajor_step(qd, PP_HALF, ks), kk, idS, ks > 0);
        }
        commit(bar(PB_S + 2 * hf + (j & 1)));
        if (hf == 1) commit(bar(PB_EMPTY + st));
      }
      __syncwarp();
    };
    for (int j = 0; j < min(nblk, 2) && ok; ++j) {
      issue_s(0, j);
      if (ok) issue_s(1, j);
    }
    for (int j = 0; j < nblk && ok; ++j) {
      const int st = (2 * j + 1) % RING;
      const uint64_t vd = desc_at(vd0, st * L::KB);
      if (!(ok = wait(PB_FULL + st, ((2 * j + 1) / RING) & 1))) break;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        if (!(ok = ok && wait(PB_P + 2 * hf + (j & 1), j >> 1 & 1))) break;
        fence_after();
        if (lead) {
          const uint32_t tP = tmem + 256 + hf * 128 + (j & 1) * 64, dO = tmem + hf * 128;
#pragma unroll
          for (int k = 0; k < PP_KEYS / 16; ++k) {
            const uint64_t vk = desc_at(vd, k * 16 * 128);
            mma_bf16_ts(dO, tP + 8 * k, vk, idO, (CHAINED ? j & (CHAIN - 1) : j) > 0 || k > 0);
            if (SPLIT) mma_bf16_ts(dO, tP + 32 + 8 * k, vk, idO, 1);
          }
          commit(bar(PB_O + hf));
          if (hf == 1) commit(bar(PB_EMPTY + st));
        }
        __syncwarp();
        if (j + 2 < nblk) issue_s(hf, j + 2);
      }
    }
    if (lead && ok) commit(bar(PB_END));
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- softmax rows
    const int hf = warp >> 2;
    const uint32_t trow = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tO = tmem + trow + hf * 128;
    // The tensor cores cut their sums off, which adds up along a row: the sums of CHAIN blocks join the
    // running ones, rounded, while the product with the next block waits for its probabilities.
    float* const baseS = reinterpret_cast<float*>(smp + L::OFF_BASE) + tid;
    auto move_on = [&](int j) {
      if (!wait(PB_O + hf, (j - 1) & 1) || !wait(PB_SLOT, 0)) return false;
      fence_after();
      const int place = keep[7];
      if (place < 0) {
        report(a.err, ERR_WAIT);
        return false;
      }
      float up = m - *baseS;                             // (no base before, no sums; no base at all: both are 0)
      const bool none = j == CHAIN, set = __any_sync(0xffffffffu, none || !(up <= 40.f));
      if (none || m == -INFINITY) up = 0.f;
      move_sums<D>(tO, a.sum + ((long long)place * (D / 4) * PP_ROWS + tid) * 4, up, set, none);
      if (set) *baseS = m;
      return true;
    };
    auto block = [&](int j, auto at_edge) {
      constexpr bool edge = decltype(at_edge)::value;
      if (!wait(PB_S + 2 * hf + (j & 1), j >> 1 & 1)) return false;
      fence_after();
      const uint32_t tS = tmem + trow + 256 + hf * 128 + (j & 1) * 64;
      float v[64];
      tmem_ld32(tS, *reinterpret_cast<float(*)[32]>(v));
      tmem_ld32(tS + 32, *reinterpret_cast<float(*)[32]>(v + 32));
      const float4* sc = reinterpret_cast<const float4*>(smp + L::OFF_SCALE + j % PP_SCALES * L::SCALES * 4);
      const float4 ks4 = sc[0], ev4 = sc[1], pf4 = sc[2], see4 = sc[3];
      const float ks[4] = {ks4.x, ks4.y, ks4.z, ks4.w}, ev[4] = {ev4.x, ev4.y, ev4.z, ev4.w};
      const float pf[4] = {pf4.x, pf4.y, pf4.z, pf4.w}, seen[4] = {see4.x, see4.y, see4.z, see4.w};
      tmem_wait_ld();
      const int see = lim - key0 - j * PP_KEYS;                 // last column the row sees
      if (edge) {
#pragma unroll
        for (int i = 0; i < 64; ++i)
          if (i > see) v[i] = -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* x = v + 16 * e;
        const float m0 = fmax3(x[0], x[1], x[2]), m1 = fmax3(x[3], x[4], x[5]), m2 = fmax3(x[6], x[7], x[8]);
        const float m3 = fmax3(x[9], x[10], x[11]), m4 = fmax3(x[12], x[13], x[14]);
        const float bm = fmaxf(fmax3(m0, m1, m2), fmax3(m3, m4, x[15]));
        top = fmaxf(top, fmaf(bm, rc * ks[e], ev[e]));
      }
      const bool move = top > m + BASE_STEP;
      if (__any_sync(0xffffffffu, move)) {
        const float mn = move ? top : m;
        const float2 f = down2(m - mn);
        if (j > 0) {
          if (!wait(PB_O + hf, (j - 1) & 1)) return false;   // the product before has to be in O
          fence_after();
          const float g = move ? f.x * f.y : 1.f;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            float o[32];
            tmem_ld32(tO + c * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= g;
            tmem_st32(tO + c * 32, o);
          }
          tmem_wait_st();
        }
        if (move) l = l * f.x * f.y;
        m = mn;
      }
      const float base = m == -INFINITY ? 0.f : W_OFF - m;
      float lb = 0.f;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float hi[16], lo_[16];
#pragma unroll
        for (int e = 2 * c; e < 2 * c + 2; ++e) {
          const float cc = rc * ks[e], add = seen[e] + base;
          const uint64_t c2 = f2_pack(cc, cc), a2 = f2_pack(add, add), pf2 = f2_pack(pf[e], pf[e]);
          uint64_t s0 = 0ull, s1 = 0ull;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int at = 16 * e + 2 * i, k = 8 * (e & 1) + i;
            float x0, x1;
            f2_unpack(f2_fma(f2_pack(v[at], v[at + 1]), c2, a2), x0, x1);
            if (edge) {                                  // (here: -inf times a factor that is 0 is no -inf)
              if (at > see) x0 = -INFINITY;
              if (at + 1 > see) x1 = -INFINITY;
            }
            x0 = ex2(x0);
            x1 = ex2(x1);
            const uint64_t w2 = f2_pack(x0, x1);
            if (i & 1) s1 = f2_add(s1, w2); else s0 = f2_add(s0, w2);
            f2_unpack(f2_mul(w2, pf2), x0, x1);
            const uint32_t w = pack_h2(x0, x1);
            hi[k] = __uint_as_float(w);
            if (SPLIT) {
              const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&w));
              lo_[k] = __uint_as_float(pack_h2(x0 - b.x, x1 - b.y));
            }
          }
          float x0, x1;
          f2_unpack(f2_add(s0, s1), x0, x1);
          lb += x0 + x1;
        }
        tmem_st16(tS + 16 * c, hi);
        if (SPLIT) tmem_st16(tS + 32 + 16 * c, lo_);
      }
      l += lb;
      tmem_wait_st();
      if (CHAINED && (j & (CHAIN - 1)) == 0 && j > 0 && !move_on(j)) return false;
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(PB_P + 2 * hf + (j & 1)));
      return true;
    };
    // the blocks that every row sees whole, and the others
    const int whole = min(max((lim_lo + 1 - key0) / PP_KEYS, 0), nblk);
    int j = 0;
#pragma unroll 1
    for (; j < whole && ok; ++j) ok = block(j, std::false_type{});
#pragma unroll 1
    for (; j < nblk && ok; ++j) ok = block(j, std::true_type{});
    if (ok) ok = wait(PB_END, 0);
  }
  fence_before();
  __syncthreads();                                       // every product is done; shared memory is free
  fence_after();

  const int first = keep[0], row0_ = keep[1], rows_ = keep[2], cut_ = keep[3], h_ = keep[5], nan0_ = keep[6];
  const long long HQ = (long long)H * G, pair = (long long)keep[4] * H + h_, slot = PARTS ? blockIdx.x : pair * gridDim.y + blockIdx.y;
  auto row_of = [&](int r) {                             // of the outputs
    const int tok = r / G;
    return (first + tok) * HQ + h_ * G + (r - tok * G);
  };
  const bool wide = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
  auto write = [&](long long row, int c, const float* v) {   // 8 values of a row of the output
    if (a.out_f32) {
      float* to = reinterpret_cast<float*>(a.out) + row * D + 8 * c;
      if (wide) {
        st32(to, v);
      } else {
        reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
      }
    } else {
      reinterpret_cast<uint4*>(a.out)[row * (D / 8) + c] =
          make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
  };
  if (warp < PP_MMA_WARP && ok) {                        // a thread writes its row, 32 bytes at a time
    const uint32_t tO = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * 128;
    uint32_t any = 0;
    for (int i = 0; i < PP_NANW; ++i) any |= nanS[i];
    const float inv = PARTS || cut_ > 1 ? 1.f : l == 0.f ? 0.f : (1.f / P_SCALE) / l;   // (a part's rows stay as they are)
    const long long row = row_of(row0_ + min(tid, rows_ - 1)) + (PARTS && keep[8] < a.to.n_groups ? a.to.rows : 0);
    if (CHAINED && keep[7] >= 0)
      fetch_sums<D>(tO, a.sum + ((long long)keep[7] * (D / 4) * PP_ROWS + tid) * 4,
                    ex2(fminf(reinterpret_cast<float*>(smp + L::OFF_BASE)[tid] - m, 0.f)));
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      float o[32];
      tmem_ld32(tO + c * 32, o);
      tmem_wait_ld();
      if (l == 0.f)
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = 0.f;
      if (any) {                                         // NaN values that this row sees
        for (int w = 0; w < PP_NANW; ++w)
          for (uint32_t bits = nanS[w]; bits; bits &= bits - 1) {
            const int pos = nan0_ + 32 * w + __ffs(bits) - 1, id = page16(pos);
            if (pos > lim || id < 0) continue;
            const unsigned char* p = a.pool.v + (((long long)id * H + h_) * a.pool.page + (pos & (a.pool.page - 1))) * D + 32 * c;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if ((p[i] & 0x7f) == 0x7f) o[i] = __uint_as_float(0x7fffffffu);
          }
      }
      if (tid < rows_) {
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] *= inv;
        if (cut_ > 1) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            st32(a.part + (PARTS ? (slot * PP_ROWS + tid) * D + 32 * c + 8 * i : ((slot * (D / 8) + 4 * c + i) * PP_ROWS + tid) * 8),
                 o + 8 * i);
        } else if (a.out_f32) {
#pragma unroll
          for (int i = 0; i < 4; ++i) write(row, 4 * c + i, o + 8 * i);
        } else {
          uint32_t* to = reinterpret_cast<uint32_t*>(a.out) + (row * D + 32 * c) / 2;
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i] = pack_bf16(o[2 * i], o[2 * i + 1]);
          if (wide) {
            st32(to, reinterpret_cast<const float*>(w));
            st32(to + 8, reinterpret_cast<const float*>(w + 8));
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              reinterpret_cast<uint4*>(to)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
          }
        }
      }
    }
    if (cut_ > 1) {
      __stcg(a.part_ml + slot * PP_ROWS + tid, make_float2(m, l));
    } else if (PARTS) {
      if (tid < rows_) a.to.ml[row] = make_float2(m, l);
    } else if (lim >= 0 && a.lse) {
      a.lse[row] = l == 0.f ? -INFINITY : (m - W_OFF + log2f(l)) * 0.69314718055994530942f;
    }
  }
  fence_before();
  if (!PARTS && cut_ > 1) __threadfence();
  __syncthreads();
  if (warp == PP_MMA_WARP) tmem_dealloc(tmem, PP_TMEM);
  if (CHAINED && tid == 0 && keep[7] >= 0) atomicExch(a.claim + keep[7], 0);   // (its sums are read)
  if (!PARTS && cut_ > 1) {
    // the part that comes last joins them, in their order (a part whose waits ran out comes too)
    int* const count = a.count + pair;
    volatile int* last = reinterpret_cast<volatile int*>(smp + L::OFF_TMEM);
    __syncthreads();
    if (tid == 0) *last = atomicAdd(count, 1) == cut_ - 1;
    __syncthreads();
    if (*last) {
      __threadfence();
      // a row's factors of the parts, and its normaliser
      const long long slot0 = pair * gridDim.y;
      float* const fS = reinterpret_cast<float*>(smp);   // [parts][rows]
      for (int rw = tid; rw < rows_; rw += PP_THREADS) {
        float2 ml[PP_PARTS];
#pragma unroll
        for (int c = 0; c < PP_PARTS; ++c)
          if (c < cut_) ml[c] = __ldcg(a.part_ml + (slot0 + c) * PP_ROWS + rw);
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int c = 0; c < PP_PARTS; ++c)
          if (c < cut_) mt = fmaxf(mt, ml[c].x);
#pragma unroll
        for (int c = 0; c < PP_PARTS; ++c)
          if (c < cut_) {
            const float2 f = down2(ml[c].x - mt);          // (times a NaN: a NaN)
            lt = fmaf(ml[c].y * f.x, f.y, lt);
            fS[c * PP_ROWS + rw] = f.x * f.y;
          }
        const float inv = lt == 0.f ? 0.f : (1.f / P_SCALE) / lt;
        for (int c = 0; c < cut_; ++c) fS[c * PP_ROWS + rw] *= inv;
        if (a.lse)
          a.lse[row_of(row0_ + rw)] =
              lt == 0.f ? -INFINITY : (mt - W_OFF + log2f(lt)) * 0.69314718055994530942f;
      }
      __syncthreads();
      constexpr int ITEMS = PP_ROWS * (D / 8);           // of 8 values, two a thread at once
      for (int i = tid; i < ITEMS; i += 2 * PP_THREADS) {
        float v[2][8] = {};
        for (int c0 = 0; c0 < cut_; c0 += 4) {
          float4 b[2][4][2];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (c0 + c >= cut_) break;
              const int at = min(i + u * PP_THREADS, ITEMS - 1), part = c0 + c;
              const float4* p = reinterpret_cast<const float4*>(
                  a.part + (((slot0 + part) * (D / 8) + at / PP_ROWS) * PP_ROWS + min(at % PP_ROWS, rows_ - 1)) * 8);
              b[u][c][0] = __ldcg(p);
              b[u][c][1] = __ldcg(p + 1);
            }
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (c0 + c < cut_) {
                const int rw = min(min(i + u * PP_THREADS, ITEMS - 1) % PP_ROWS, rows_ - 1);
                const float f = fS[(c0 + c) * PP_ROWS + rw];
                const float4 x = b[u][c][0], y = b[u][c][1];
                float (&z)[8] = v[u];
                z[0] = fmaf(x.x, f, z[0]); z[1] = fmaf(x.y, f, z[1]); z[2] = fmaf(x.z, f, z[2]); z[3] = fmaf(x.w, f, z[3]);
                z[4] = fmaf(y.x, f, z[4]); z[5] = fmaf(y.y, f, z[5]); z[6] = fmaf(y.z, f, z[6]); z[7] = fmaf(y.w, f, z[7]);
              }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int at = i + u * PP_THREADS;
          if (at < ITEMS && at % PP_ROWS < rows_) write(row_of(row0_ + at % PP_ROWS), at / PP_ROWS, v[u]);
        }
      }
      if (tid == 0) *count = 0;
    }
  }
}

template <int D, bool SPLIT, bool CHAINED, bool PARTS>
cudaError_t launch_prompt(const PromptArgs& a, dim3 grid, cudaStream_t stream) {
  auto k = paged_prompt_kernel<D, SPLIT, CHAINED, PARTS>;
  const size_t smem = PL<D>::BYTES;
  static std::atomic<unsigned long long> raised{0};
  const cudaError_t e = raise_smem_limit_once(raised, k, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(PP_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a);
}

// Places for parts of tiles: 3 an SM (60 MB at d = 128).
long long slots_of(int sms) { return 3ll * sms; }

}  // namespace
}  // namespace kvpop
