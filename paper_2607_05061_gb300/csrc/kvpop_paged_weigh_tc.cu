// Attention weights of the paged 8-bit cache's positions for many query rows, on tcgen05.
//
// The mathematics is that of kvpop_paged_weigh.cu.  Positions are the rows of the products: a tile is
// 256 positions of one (sequence, KV head), as bf16 (which holds every e4m3 value) in tensor memory,
// and its query rows (token, query head) come as blocks of 128 columns, unchanged.  A thread owns one
// position:
//   x = S ks c - lse log2 e,   sum += 2^x,
// one fma, one exponential and one addition a value; there is no maximum to keep, since a weight is
// no more than 1.  A position's sum is added to its weight at the end of the tile.
//
// All (tile, block) pairs form one list, tile after tile, that is cut evenly over the SMs; a tile that
// lies in several CTAs' parts is added up, in their order, by the CTA that arrives last, at its end.
// Roles:
//  * 8 softmax warps;
//  * 4 warps that bring the positions of the tiles to come into the other half of the operand's tensor
//    memory: their pages two tiles before, their bytes one;
//  * 1 MMA warp: S = K Q^T (M 128, N 128, K d) per half of the tile, one buffer a half;
//  * 3 producer warps: query rows by 16-byte cp.async into 128B-swizzled slots, with lse and the last
//    position that each row sees beside them.  Where all of a sequence's rows fit the slots they stay
//    there for all tiles of the head.
// A wait by parity misses a phase when the one after it is complete too, so a barrier's next phase needs an
// arrival of everyone who waits for this one.  Operands (AFULL) are given back (AEMPTY) by the MMA warp, when
// their products are done, and by each softmax warp, as it begins the tile: the position warps are two tiles
// ahead of the last of them at most.  Query slots (FULL) are given back (EMPTY) by both, so that the producers
// are ST blocks ahead at most.  Logits (SFULL) are given back (PFULL) by their half's warps: the MMA warp is
// one block ahead.
// Tensor memory: S 2 x 128 columns, operands 2 x (2 x d / 2).
//
// A block of 256 positions by 128 rows takes the tensor cores 1024 clocks at d = 128 and the exponential
// unit as many; in a long prompt it takes about 2300, most of them the chain of a half: logits into
// registers, product (680 with its issue), logits there again (300), while a softmax warp works 1500
// clocks on its 128 columns beside the other half's.  Leaving out exponentials, normalisers' loads, or
// the copies of rows changed 4 to 15% of it; unrolled code counts (the masked columns in a loop: 3%).
// 6001 tokens, 8 KV and 32 query heads 145 us, 0.53 of the bf16 rate; the last 37 to 64 tokens of three
// prompts of 9001 to 17011 30.6 us, where a tile of two blocks waits for its ends.
// Measured before: 64-column products of four buffers (177, half of the tensor rate), 16 softmax warps
// (175), registers moved between the roles (spills).
#include <type_traits>

#include "kvpop_mma.cuh"
#include "kvpop_paged.cuh"
#include "kvpop_ptx.cuh"
#include "kvpop_tc05.cuh"

namespace kvpop {
namespace {

using namespace paged;
using namespace tc05;

constexpr int WT_HALF = 128, WT_KEYS = 256, WT_BN = 128;
constexpr int WT_SOFT = 8, WT_MMA_WARP = WT_SOFT, WT_COPY_WARP = WT_SOFT + 1, WT_COPY = 3;
constexpr int WT_KEY_WARP = WT_COPY_WARP + WT_COPY, WT_KEY = 4;
constexpr int WT_THREADS = 32 * (WT_KEY_WARP + WT_KEY);
constexpr int WT_OLD = 8;                                // tiles whose scales and weights so far are held
// Tiles of up to that many blocks are not cut.  us with 8, 16, 32 (d = 128, 4 heads a KV head): 3 sequences of 9000
// with 600 new tokens (19 blocks) 141, 149, 142; 6 of 3000 with 500 (16) 95, 102, 102; one of 2000 with 700 (22)
// 30, 39, 42; 2 of 16000 with 1000 (32) 138, 140, 159; d = 64 alike.  (Rows that stay in the slots are whole tiles.)
constexpr int WT_WHOLE = 8;
// What a tile's ends cost beside its blocks, in blocks (a prompt of 6001 tokens: 0 177 us, 2 150, 3 145, 4 147, 6 149).
constexpr int WT_ENDS = 3;
constexpr float kLog2E = 1.4426950408889634f;

struct WeighTcArgs {
  Pool pool;
  Batch b;
  const bf16* q;
  long long q_ts, q_hs;
  const float* lse;
  float* mass;
  long long positions;
  float* part;                                           // [CTAs][2][256] sums of cut tiles
  int* count;                                            // [CTAs] parts there, zero between calls
  int32_t* err;
  float c;                                               // log2(e) / sqrt(d)
  int G, least;                                          // sequences with more than `least` rows
};

template <int D>
struct WL {
  static constexpr int ST = D == 128 ? 4 : 8, SLOT = WT_BN * D * 2;
  static constexpr int OFF_NL = ST * SLOT;               // [slot][128] -lse log2 e
  static constexpr int OFF_LIM = OFF_NL + ST * WT_BN * 4;   // [slot][128] last position seen, -1: none
  static constexpr int OFF_FLAG = OFF_LIM + ST * WT_BN * 4; // [slot] a byte for each 32 rows: whether one sees none
  static constexpr int OFF_RAW = (OFF_FLAG + ST * 4 + 15) / 16 * 16;   // [2] bytes of tiles to come, a thread's pieces apart
  // a thread's page of a tile to come, and scale and weight so far of tiles there and to come: in registers
  // they were spilled, and a load that is spilled is waited for
  static constexpr int OFF_ID = OFF_RAW + 2 * WT_KEYS * D, OFF_SC = OFF_ID + 2 * WT_KEYS * 4, OFF_OLD = OFF_SC + WT_OLD * WT_KEYS * 4;
  static constexpr int OFF_BAR = OFF_OLD + WT_OLD * WT_KEYS * 4;
  static constexpr int FULL = 0, EMPTY = ST, SFULL = 2 * ST, PFULL = SFULL + 2, AFULL = PFULL + 2, AEMPTY = AFULL + 2,
                       END = AEMPTY + 2, N_BAR = END + 1;
  static constexpr int OFF_TMEM = OFF_BAR + 8 * N_BAR, BYTES = OFF_TMEM + 16;
  static_assert(ST <= WT_WHOLE, "");
};

// A sequence's tiles, of one head.
struct WSeqT {
  int first, n, len, ctx, tiles, blocks;                 // blocks of all its rows; 0 tiles: not this kernel's
  __device__ __forceinline__ int skipped(int G, int kt) const {   // blocks whose rows all lie before the tile
    const long long t0 = (long long)kt * WT_KEYS;
    return t0 <= len ? 0 : (int)((t0 - len) * G / WT_BN);
  }
  __device__ __forceinline__ int here(int G, int kt) const { return blocks - skipped(G, kt); }
  // places of the tiles before kt: their blocks, and what a tile's ends cost, in blocks
  __device__ __forceinline__ long long before(int G, int kt) const {
    const int full = min(kt, min(tiles, len / WT_KEYS + 1));
    long long w = (long long)full * blocks;
    if (kt > full) {                                     // sum of blocks - (2 G k - up), k from full to kt - 1
      const long long up = ((long long)len * G + WT_BN - 1) / WT_BN, k = kt - full;
      w += k * (blocks + up) - (long long)G * ((long long)kt * (kt - 1) - (long long)full * (full - 1));
    }
    return w + (long long)WT_ENDS * kt;
  }
};
__device__ __forceinline__ WSeqT wseq_t(const WeighTcArgs& a, int s) {
  const SeqTokens t = seq_tokens(a.b, s, a.err);
  WSeqT x;
  x.first = t.first;
  x.n = t.n;
  x.len = t.len;
  x.ctx = x.tiles = x.blocks = 0;
  if (t.len >= 0 && (long long)t.n * a.G > a.least) {
    x.ctx = context(a.b, a.pool, t, a.err);
    x.tiles = (x.ctx + WT_KEYS - 1) / WT_KEYS;
    x.blocks = (int)(((long long)t.n * a.G + WT_BN - 1) / WT_BN);
  }
  return x;
}
// A tile of the list: blocks [b0, b1) of it are this CTA's.
struct Tile {
  WSeqT x;
  int s, h, kt, b0, b1;
  long long at, end;                                     // places of b0, and of the CTA's end, in the list
  __device__ __forceinline__ bool valid() const { return at < end; }
  __device__ __forceinline__ void cut() { b1 = (int)min((long long)x.blocks, b0 + (end - at)); }
  __device__ __forceinline__ bool same_head(const Tile& o) const { return s == o.s && h == o.h; }
};
__device__ __forceinline__ void advance(const WeighTcArgs& a, Tile& t) {
  t.at += t.x.blocks - t.b0 + WT_ENDS;
  if (t.at >= t.end) return;
  if (++t.kt == t.x.tiles) {
    t.kt = 0;
    if (++t.h == a.pool.H) {
      t.h = 0;
      do t.x = wseq_t(a, ++t.s);                         // (there is one: the list goes on)
      while (t.x.tiles == 0);
    }
  }
  t.b0 = t.x.skipped(a.G, t.kt);
  t.cut();
}
// The tile that place w of the list lies in (by a whole warp); w: below the total.  b0 may lie behind its
// blocks.
__device__ Tile find(const WeighTcArgs& a, long long w, int lane) {
  Tile t;
  long long base = 0;
  t.s = -1;
  for (int s0 = 0; s0 < a.b.n_seq && t.s < 0; s0 += 32) {
    long long mine = 0;
    if (s0 + lane < a.b.n_seq) {
      const WSeqT x = wseq_t(a, s0 + lane);
      mine = x.before(a.G, x.tiles) * a.pool.H;
    }
    long long pre = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, pre, o);
      if (lane >= o) pre += y;
    }
    const unsigned has = __ballot_sync(0xffffffffu, w < base + pre);
    const int who = has ? __ffs(has) - 1 : 31;
    if (has) t.s = s0 + who;
    base += __shfl_sync(0xffffffffu, has ? pre - mine : pre, who);
  }
  t.s = max(t.s, 0);
  t.x = wseq_t(a, t.s);
  const long long each = max(t.x.before(a.G, t.x.tiles), 1ll), rem = w - base;
  t.h = (int)(rem / each);
  const long long in = rem - each * t.h;
  int lo = 0, hi = max(t.x.tiles - 1, 0);                // the last tile that begins at or before it
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.x.before(a.G, mid) <= in) lo = mid; else hi = mid - 1;
  }
  t.kt = lo;
  t.b0 = t.x.skipped(a.G, lo) + (int)(in - t.x.before(a.G, lo));
  t.at = w;
  return t;
}

template <int D>
__global__ void __launch_bounds__(WT_THREADS, 1) paged_weigh_tc_kernel(WeighTcArgs a) {
  using L = WL<D>;
  constexpr int ST = L::ST, RAW = D / 16;                // 16-byte pieces of a row
  extern __shared__ __align__(1024) unsigned char smt[];
  __shared__ Tile edgeS[2], aheadS[WT_KEY];
  __shared__ long long edgeW[2], shareS;
  __shared__ int lastS;
  const uint32_t sb = smem_u32(smt);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, H = a.pool.H, G = a.G;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8u * (uint32_t)i; };

  // ---- the CTA's part of the list.  A tile of few blocks is not cut: it belongs to the part that it begins in.
  if (warp < 2) {
    long long total = 0;
    for (int s = lane; s < a.b.n_seq; s += 32) {
      const WSeqT x = wseq_t(a, s);
      total += x.before(G, x.tiles) * H;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    const long long share = (total + gridDim.x - 1) / gridDim.x;
    long long w = min(share * (blockIdx.x + warp), total);
    Tile t{};
    if (w < total) {
      t = find(a, w, lane);
      const int skip = t.x.skipped(G, t.kt);
      if (t.b0 >= t.x.blocks || (t.b0 > skip && t.x.blocks - skip <= WT_WHOLE)) {
        w += t.x.blocks - t.b0 + WT_ENDS;
        t = w < total ? find(a, w, lane) : Tile{};
      }
    }
    if (lane == 0) {
      edgeS[warp] = t;
      edgeW[warp] = w;
      shareS = share;
    }
  }
  if (tid == 64) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(bar(L::FULL + i), 4 * 32 + 4);
      mbar_init(bar(L::EMPTY + i), 1 + WT_SOFT);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(L::SFULL + i), 1);
      mbar_init(bar(L::PFULL + i), WT_SOFT / 2);
      mbar_init(bar(L::AFULL + i), WT_KEY);
      mbar_init(bar(L::AEMPTY + i), 1 + WT_SOFT);
    }
    mbar_init(bar(L::END), 1);
    mbar_fence_init();
  }
  if (warp == WT_MMA_WARP) tmem_alloc(sb + L::OFF_TMEM, 512);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smt + L::OFF_TMEM);
  Tile t = edgeS[0];
  t.at = edgeW[0];
  t.end = edgeW[1];
  const long long share = shareS;
  if (t.valid()) t.cut();
  auto wait = [&](int b, uint32_t parity) {              // the whole warp; false: gave up
    if (__all_sync(0xffffffffu, mbar_try_wait(bar(b), parity))) return true;
    return (bool)__all_sync(0xffffffffu, mbar_wait(bar(b), parity, a.err, ERR_WAIT));
  };
  // All of a head's rows fit the slots: its blocks from the first tile's on are loaded once.  `pos` counts
  // the loads so far, the same in every role.
  auto stays = [&](const Tile& x) { return x.x.blocks <= ST; };
  uint32_t pos = 0;
  bool ok = true;

  if (warp >= WT_KEY_WARP) {
    // ---------------------------------------------------------------- positions
    // Tiles by their number j: the pages of j + 2, the bytes of j + 1, and tile j into the operand.  A
    // thread: rows `lane` of the warp's 32 in either half, whose pages, scales and weights so far it asks
    // for; their bytes the warp copies as whole lines.
    const int kw = warp - WT_KEY_WARP;
    const uint32_t tl = tmem + ((uint32_t)(kw * 32) << 16);
    if (lane == 0) aheadS[kw] = t;
    __syncwarp();
    int pos_of[2] = {-1, -1}, head_of = 0;               // of the tile whose pages are on their way
    const float* old_of = nullptr;                       // weight so far of position 0 of its head
    int old_len = 0;
    auto mine = [&](int off, int n, int hh) { return reinterpret_cast<float*>(smt + off) + n * WT_KEYS + hh * WT_HALF + kw * 32 + lane; };
    auto look = [&](int j) {
      pos_of[0] = pos_of[1] = -1;
      Tile ahead = aheadS[kw];
      if (!ahead.valid()) return;
      head_of = ahead.h;
      old_of = a.mass + ((long long)ahead.s * H + ahead.h) * a.positions;
      old_len = ahead.x.len;
      const int32_t* const row = a.b.table + (long long)ahead.s * a.b.table_stride;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int at = ahead.kt * WT_KEYS + hh * WT_HALF + kw * 32 + lane;
        if (at < ahead.x.ctx) {
          pos_of[hh] = at;
          cp_async4(smem_u32(mine(L::OFF_ID, j & 1, hh)), row + (at >> a.pool.page_shift));
        }
      }
      advance(a, ahead);
      __syncwarp();
      if (lane == 0) aheadS[kw] = ahead;
      __syncwarp();
    };
    // chunk c of row r lies at chunk c ^ r of the row's 128 (64) bytes
    auto chunk_of = [&](int row, int c) { return row * D + ((c ^ (row & (RAW - 1))) << 4); };
    auto fetch = [&](int j) {                            // (the pages are there)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        int id = -1;
        if (pos_of[hh] >= 0) {
          id = __float_as_int(*mine(L::OFF_ID, j & 1, hh));
          if ((unsigned)id >= (unsigned)a.pool.n_pages) {
            report(a.err, ERR_PAGE);
            id = -1;
          }
        }
        const long long at = id < 0 ? -1 : ((long long)id * H + head_of) * a.pool.page + (pos_of[hh] & (a.pool.page - 1));
        const uint32_t dst = sb + L::OFF_RAW + (j & 1) * (WT_KEYS * D) + (hh * WT_HALF + kw * 32) * D;
#pragma unroll
        for (int i = 0; i < RAW; ++i) {
          const int row = i * (32 / RAW) + lane / RAW, c = lane % RAW;
          const long long o = __shfl_sync(0xffffffffu, at, row);
          cp_async16(dst + chunk_of(row, c), a.pool.k + (o < 0 ? 0 : o) * D + 16 * c, o < 0 ? 0 : 16);
        }
        if (id >= 0) cp_async4(smem_u32(mine(L::OFF_SC, j % WT_OLD, hh)), a.pool.ks + at / BLK);
        else *mine(L::OFF_SC, j % WT_OLD, hh) = 0.f;
        if (pos_of[hh] >= 0 && pos_of[hh] < old_len) cp_async4(smem_u32(mine(L::OFF_OLD, j % WT_OLD, hh)), old_of + pos_of[hh]);
        else *mine(L::OFF_OLD, j % WT_OLD, hh) = 0.f;
      }
    };
    auto store = [&](int buf) {
      __syncwarp();
#pragma unroll 1
      for (int hh = 0; hh < 2; ++hh) {
        const unsigned char* const raw = smt + L::OFF_RAW + buf * (WT_KEYS * D) + (hh * WT_HALF + kw * 32) * D;
#pragma unroll 1
        for (int c = 0; c < RAW; c += 2) {
          float w[16];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(raw + chunk_of(lane, c + i));
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t lo, hi;
              cvt4(u[k], lo, hi);
              const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo));
              const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              w[8 * i + 2 * k] = __uint_as_float(pack_bf16(x.x, x.y));
              w[8 * i + 2 * k + 1] = __uint_as_float(pack_bf16(y.x, y.y));
            }
          }
          tmem_st16(tl + 256 + buf * D + hh * (D / 2) + 8 * c, w);
        }
      }
      tmem_wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(L::AFULL + buf));
    };
    look(0);
    cp_commit();
    cp_wait<0>();
    fetch(0);
    look(1);
    cp_commit();
    for (int j = 0; t.valid() && ok; ++j) {
      cp_wait<0>();
      fetch(j + 1);                                      // (the bytes before them are in the operand)
      look(j + 2);
      cp_commit();
      if (j >= 2 && !(ok = wait(L::AEMPTY + (j & 1), (j / 2 - 1) & 1))) break;
      fence_after();
      store(j & 1);
      advance(a, t);
    }
    cp_wait<0>();
  } else if (warp >= WT_COPY_WARP) {
    // ---------------------------------------------------------------- query rows
    // The warps take groups of 32 rows in turn.  A group's addresses and normalisers are asked for one
    // group ahead.
    const int cw = warp - WT_COPY_WARP;
    struct Group {
      long long off;
      float l;
      int lim;
    };
    int b = t.b0;                                        // the load of number `pos`: block b of tile t
    auto end = [&] { return stays(t) ? t.x.blocks : t.b1; };
    auto next_load = [&] {
      ++pos;
      if (++b < end()) return;
      const Tile was = t;
      do advance(a, t);
      while (t.valid() && stays(t) && t.same_head(was));
      b = t.b0;
    };
    auto group = [&](int k) {
      Group x;
      const long long r = (long long)b * WT_BN + 32 * k + lane;
      const bool in = t.valid() && r < (long long)t.x.n * G;
      const int tok = in ? (int)((uint32_t)r / (uint32_t)G) : 0, g = in ? (int)r - tok * G : 0;
      x.off = in ? (t.x.first + tok) * a.q_ts + (long long)(t.h * G + g) * a.q_hs : -1;
      x.l = in ? a.lse[((long long)(t.x.first + tok) * H + t.h) * G + g] : -INFINITY;
      x.lim = last_seen(t.x.len, tok, t.x.ctx);
      return x;
    };
    int k = cw;
    bool more = t.valid();
    Group x = group(k);
    while (more && ok) {
      const uint32_t p = pos;
      const int st = p % ST, kk = k;
      const Group y = x;
      if ((k += WT_COPY) >= 4) {                         // the group after this one
        k -= 4;
        next_load();
      }
      more = t.valid();
      x = group(k);
      if (p >= (uint32_t)ST && !(ok = wait(L::EMPTY + st, (p / ST - 1) & 1))) break;
      const uint32_t dst = sb + st * L::SLOT;
      constexpr int LPR = D / 8, RPI = 32 / LPR;         // lanes of a row, rows at a time
      const int c = lane % LPR, sub = lane / LPR;
#pragma unroll
      for (int i = 0; i < LPR; ++i) {
        const int rr = i * RPI + sub;
        const long long o = __shfl_sync(0xffffffffu, y.off, rr);
        cp_async16(dst + tile_off(kk * 32 + rr, c, WT_BN), a.q + (o < 0 ? 0 : o) + 8 * c, o < 0 ? 0 : 16);
      }
      cp_async_arrive_noinc(bar(L::FULL + st));
      const bool gone = y.l == -INFINITY;
      reinterpret_cast<float*>(smt + L::OFF_NL)[st * WT_BN + kk * 32 + lane] = gone ? 0.f : -y.l * kLog2E;
      reinterpret_cast<int*>(smt + L::OFF_LIM)[st * WT_BN + kk * 32 + lane] = gone ? -1 : y.lim;
      const bool none = __any_sync(0xffffffffu, gone);
      __syncwarp();
      if (lane == 0) {
        (smt + L::OFF_FLAG)[st * 4 + kk] = none;
        mbar_arrive(bar(L::FULL + st));
      }
    }
    cp_wait<0>();
  } else if (warp == WT_MMA_WARP) {
    // ---------------------------------------------------------------- MMA issue
    const uint32_t idS = idesc_bf16(128, WT_BN, 0);
    const bool lead = elect_one();
    const uint64_t bd0 = kmajor_desc(sb, WT_BN, 0);
    uint32_t step = 0;
    int first = t.b0;                                    // block that lies in the head's first slot
    for (uint32_t i = 0; t.valid() && ok; ++i) {
      if (!(ok = wait(L::AFULL + (i & 1), i >> 1 & 1))) break;
      fence_after();
      const uint32_t tA = tmem + 256 + (i & 1) * D;
      const bool stay = stays(t);
      for (int b = t.b0; b < t.b1 && ok; ++b, ++step) {
        const uint32_t p = stay ? pos + (b - first) : pos;
        const int st = p % ST;
        if (!(ok = wait(L::FULL + st, p / ST & 1))) break;
        fence_async_smem();
        const uint64_t bd = desc_at(bd0, st * L::SLOT);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          if (step > 0 && !(ok = ok && wait(L::PFULL + hh, (step - 1) & 1))) break;
          fence_after();
          if (lead) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              mma_bf16_ts(tmem + hh * 128, tA + hh * (D / 2) + ks * 8, kmajor_step(bd, WT_BN, ks), idS, ks > 0);
            commit(bar(L::SFULL + hh));
            if (hh == 1 && !stay) commit(bar(L::EMPTY + st));
          }
          __syncwarp();
        }
        if (!stay) ++pos;
      }
      if (lead) commit(bar(L::AEMPTY + (i & 1)));
      __syncwarp();
      const Tile was = t;
      advance(a, t);
      if (!t.valid() || !t.same_head(was)) {
        if (stay && ok) {                                // the head's slots are free
          const int k = was.x.blocks - first;
          if (lead)
            for (int j = 0; j < k; ++j) commit(bar(L::EMPTY + (pos + j) % ST));
          __syncwarp();
          pos += k;
        }
        first = t.b0;
      }
    }
    if (lead) commit(bar(L::END));                       // every product is done before the CTA ends
    __syncwarp();
    wait(L::END, 0);
  } else {
    // ---------------------------------------------------------------- softmax
    // a thread: one position, in half hh of the tile, and all columns.  While one half's warps work on
    // their logits the tensor core forms the other's.
    const int hh = warp >> 2, r = tid;
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const float* const nlS = reinterpret_cast<const float*>(smt + L::OFF_NL);
    const int* const limS = reinterpret_cast<const int*>(smt + L::OFF_LIM);
    const int* const flagS = reinterpret_cast<const int*>(smt + L::OFF_FLAG);
    uint32_t step = 0;
    int first = t.b0;
    for (uint32_t i = 0; t.valid() && ok; ++i) {
      if (!(ok = wait(L::AFULL + (i & 1), i >> 1 & 1))) break;
      const float* const of = reinterpret_cast<const float*>(smt) + (i % WT_OLD) * WT_KEYS + r;
      const float scale = of[L::OFF_SC / 4];             // 0: no position, or a bad page
      const float before = of[L::OFF_OLD / 4];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(L::AEMPTY + (i & 1)));
      const uint64_t cc = f2_pack(a.c * scale, a.c * scale);
      const int t0 = t.kt * WT_KEYS, tp = t0 + r, t1 = min(t0 + WT_KEYS, t.x.ctx) - 1;
      // blocks from here on have rows that see the whole tile: tokens from t1 - len on
      const int all_see = t1 <= t.x.len ? 0 : (int)(((long long)(t1 - t.x.len) * G + WT_BN - 1) / WT_BN);
      float* const to = a.mass + ((long long)t.s * H + t.h) * a.positions + tp;
      const bool whole = t.b0 == t.x.skipped(G, t.kt) && t.b1 == t.x.blocks;
      const bool stay = stays(t);
      float sum = 0.f;
      for (int b = t.b0; b < t.b1; ++b, ++step) {
        const uint32_t p = stay ? pos + (b - first) : pos;
        const int st = p % ST;
        if (!(ok = wait(L::FULL + st, p / ST & 1) && wait(L::SFULL + hh, step & 1))) break;
        fence_after();
        const bool edge = b < all_see || flagS[st] != 0;
        uint64_t s0 = 0ull, s1 = 0ull;
        const uint32_t tS = tl + hh * 128;
        const float4* const nl = reinterpret_cast<const float4*>(nlS + st * WT_BN);
        const int4* const lim = reinterpret_cast<const int4*>(limS + st * WT_BN);
        auto there = [&] {                               // the logits are in registers
          tmem_wait_ld();
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(L::PFULL + hh));
        };
        auto columns = [&](const float (&w)[32], int u, auto at_edge) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float4 n4 = nl[8 * u + k];
            float x0, x1, x2, x3;
            f2_unpack(f2_fma(f2_pack(w[4 * k], w[4 * k + 1]), cc, f2_pack(n4.x, n4.y)), x0, x1);
            f2_unpack(f2_fma(f2_pack(w[4 * k + 2], w[4 * k + 3]), cc, f2_pack(n4.z, n4.w)), x2, x3);
            if constexpr (decltype(at_edge)::value) {
              const int4 l4 = lim[8 * u + k];
              x0 = tp <= l4.x ? x0 : -INFINITY;
              x1 = tp <= l4.y ? x1 : -INFINITY;
              x2 = tp <= l4.z ? x2 : -INFINITY;
              x3 = tp <= l4.w ? x3 : -INFINITY;
            }
            s0 = f2_add(s0, f2_pack(ex2(x0), ex2(x1)));
            s1 = f2_add(s1, f2_pack(ex2(x2), ex2(x3)));
          }
        };
        if (!edge) {
#pragma unroll 1
          for (int u = 0; u < 4; u += 2) {
            float v[2][32];
            tmem_ld32(tS + 32 * u, v[0]);
            tmem_ld32(tS + 32 * u + 32, v[1]);
            if (u == 0) tmem_wait_ld(); else there();
            columns(v[0], u, std::false_type{});
            columns(v[1], u + 1, std::false_type{});
          }
        } else {                                         // (few blocks, little code)
#pragma unroll 1
          for (int u = 0; u < 4; ++u) {
            float v[32];
            tmem_ld32(tS + 32 * u, v);
            if (u < 3) tmem_wait_ld(); else there();
            columns(v, u, std::true_type{});
          }
        }
        float y0, y1;
        f2_unpack(f2_add(s0, s1), y0, y1);
        sum += y0 + y1;
        if (!stay) {
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(L::EMPTY + st));
          ++pos;
        }
      }
      if (!ok) break;
      if (scale == 0.f) sum = 0.f;
      if (whole) {
        if (tp < t.x.ctx) *to = before + sum;
      } else {                                           // (the part's first tile, or its last)
        const bool begins = t.b0 == t.x.skipped(G, t.kt);
        __stcg(a.part + ((long long)blockIdx.x * 2 + begins) * WT_KEYS + r, sum);
      }
      const Tile was = t;
      advance(a, t);
      if (!t.valid() || !t.same_head(was)) {
        if (stay) {
          const int k = was.x.blocks - first;
          __syncwarp();
          if (lane == 0)
            for (int j = 0; j < k; ++j) mbar_arrive(bar(L::EMPTY + (pos + j) % ST));
          pos += k;
        }
        first = t.b0;
      }
    }
  }
  fence_before();
  __syncthreads();
  if (warp == WT_MMA_WARP) tmem_dealloc(tmem, 512);

  // ---- tiles in several parts: the CTA that comes last adds them up
#pragma unroll 1
  for (int e = 0; e < 2; ++e) {
    Tile c = edgeS[e];                                   // the first tile, and the one that the part ends in
    const long long w = edgeW[e];
    if (edgeW[0] >= edgeW[1] || (e == 1 && c.x.tiles == 0)) break;
    const int skip = c.x.skipped(G, c.kt), here = c.x.blocks - skip;
    const long long start = w - (c.b0 - skip);
    // a part of the first tile, if that began earlier; the beginning of the one that the part ends in
    if (c.b0 == skip || (e == 1 && start < edgeW[0])) continue;
    const long long p0 = start / share;
    const int parts = (int)((start + here - 1) / share - p0) + 1;
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      lastS = atomicAdd(a.count + p0, 1) == parts - 1;
      if (lastS) a.count[p0] = 0;
    }
    __syncthreads();
    if (lastS && tid < WT_KEYS) {
      __threadfence();
      const int tp = c.kt * WT_KEYS + tid;
      if (tp < c.x.ctx) {
        float sum = 0.f;
        for (int p = 0; p < parts; ++p) sum += __ldcg(a.part + ((p0 + p) * 2 + (p == 0)) * WT_KEYS + tid);
        float* const to = a.mass + ((long long)c.s * H + c.h) * a.positions + tp;
        *to = (tp < c.x.len ? *to : 0.f) + sum;
      }
    }
    __syncthreads();
  }
}

template <int D>
cudaError_t launch(const WeighTcArgs& a, int grid, cudaStream_t stream) {
  auto k = paged_weigh_tc_kernel<D>;
  static std::atomic<unsigned long long> raised{0};
  const cudaError_t e = raise_smem_limit_once(raised, k, WL<D>::BYTES);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(WT_THREADS);
  cfg.dynamicSmemBytes = WL<D>::BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a);
}

}  // namespace

size_t paged_weigh_workspace(int sms) { return (size_t)sms * 2 * WT_KEYS * 4; }

cudaError_t launch_paged_weigh_tc(const Pool& pool, const Batch& b, const void* q, long long q_ts, long long q_hs,
                                  int HQ, const float* lse, float* mass, long long positions, int least, int* count,
                                  float* part, int sms, int32_t* err, cudaStream_t stream) {
  WeighTcArgs a{};
  a.pool = pool;
  a.b = b;
  a.q = static_cast<const bf16*>(q);
  a.q_ts = q_ts;
  a.q_hs = q_hs;
  a.lse = lse;
  a.mass = mass;
  a.positions = positions;
  a.part = part;
  a.count = count;
  a.err = err;
  a.c = (float)(1.4426950408889634 / sqrt((double)pool.d));
  a.G = HQ / pool.H;
  a.least = least;
  return pool.d == 128 ? launch<128>(a, sms, stream) : launch<64>(a, sms, stream);
}

}  // namespace kvpop
