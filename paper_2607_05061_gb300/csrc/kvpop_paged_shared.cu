// Attention over the paged 8-bit cache for sequences that share prefixes.
//
// The sequences of a group have the same first positions.  With S the shared ones and O_s a
// sequence's own, a row's softmax over both is joined from two:
//   m = max(m_S, m_O),  l = l_S 2^(m_S - m) + l_O 2^(m_O - m),  y = (A_S 2^(m_S - m) + A_O 2^(m_O - m)) / l,
// A being the sums of weights times values relative to m.  S is read once for the rows of all the
// group's tokens, as a sequence with that many tokens whose positions all of them see.
//
// Four kernels in a row: the plan writes the list of parts (each group's, each sequence's own); the
// attention's two kernels take them as they take sequences, those with many rows on tcgen05, whose
// positions are cut over all SMs, and beside them the stream for few rows; the join reads each row's
// sums.  The number of shared positions is a multiple of 64 (blocks of the tcgen05 kernel): what is
// left of a prefix counts as the sequences' own.
//
// 64 sequences over 32768 shared positions with 100 to 2000 of their own (8 KV and 32 query heads, fp32
// results): 100 us, 565 for the same table without groups.  3 of them are the plan, 9 the join; between them
// the shared part on tcgen05 (the second product twice) runs beside the own ones, each on SMs of its own.
// Sharing pays from some 65000 positions saved on (members times prefix, 8 KV heads, d = 128: re-reading
// below that comes from L2): 16 members over 4096 positions 27 us either way, over 16384 48 and 71, 4 over
// 16384 26 and 25, 64 over 1024 34 and 34, over 16384 50 and 253.
#include "kvpop_paged_attend.cuh"
#include "kvpop_paged_prompt.cuh"

namespace kvpop {
namespace {

constexpr int PLAN_THREADS = 256;
constexpr int FEW_ROWS = 8;            // that the kernel for few rows takes at once
constexpr int ANY_LEN = 0x7fffff00;    // as a length: its tokens see all positions there are

struct PlanArgs {
  Pool pool;
  Batch b;
  const int32_t *groups, *prefix;
  int32_t* err;
  Entry* entries;
  int n_groups, G, tiles;              // tiles of the tcgen05 kernel that there is room for, of one head (0: not launched)
  int own_tiles;                       // whether it takes sequences' own parts
  int* tiles_out;                      // Parts::tiles
  int room, sms;                       // CTAs that parts may take
  int one;                             // groups of rows of one token, for the other kernel
  float block_us;                      // of the tcgen05 kernel
};

__global__ void __launch_bounds__(PLAN_THREADS) shared_plan_kernel(PlanArgs a) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = a.b.n_seq, ng = a.n_groups;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int s = tid; s < n; s += PLAN_THREADS) {
    const SeqTokens t = seq_tokens(a.b, s, a.err);
    Entry e;
    e.first = t.first;
    e.n = t.n;
    e.len = t.len;
    e.ctx = t.n > 0 ? context(a.b, a.pool, t, a.err) : 0;
    e.begin = 0;
    e.row = s;
    e.group = e.place = -1;
    a.entries[ng + s] = e;
  }
  __syncthreads();
  for (int g = warp; g < ng; g += PLAN_THREADS / 32) {
    int from = a.groups[g], to = a.groups[g + 1], before = 0;   // (places of two groups would have neither's sums)
    for (int i = lane; i < g; i += 32) before = max(before, a.groups[i]);
    before = __reduce_max_sync(0xffffffffu, before);
    if (from < before || to < from || to > n) {
      if (lane == 0) report(a.err, ERR_BATCH);
      from = to = 0;
    }
    int least = a.prefix[g], members = 0, lead = INT32_MAX, first = INT32_MAX, end = 0;
    for (int s = from + lane; s < to; s += 32) {
      const Entry& e = a.entries[ng + s];
      if (e.n <= 0) continue;
      first = min(first, e.first);
      end = max(end, e.first + e.n);
      if (e.len < 0) continue;
      ++members;
      lead = min(lead, s);
      least = min(least, min(e.len, e.ctx));
    }
    members = __reduce_add_sync(0xffffffffu, members);
    lead = __reduce_min_sync(0xffffffffu, lead);
    least = __reduce_min_sync(0xffffffffu, least);
    first = __reduce_min_sync(0xffffffffu, first);
    end = __reduce_max_sync(0xffffffffu, end);
    const int shared = members < 2 ? 0 : max(least, 0) / SHARED_STEP * SHARED_STEP;
    if (lane == 0) {
      Entry e;
      e.first = shared > 0 ? first : 0;
      e.n = shared > 0 ? end - first : 0;
      e.len = ANY_LEN;
      e.ctx = shared;
      e.begin = 0;
      e.row = shared > 0 ? lead : 0;
      e.group = e.place = -1;
      a.entries[g] = e;
    }
    if (shared > 0)
      for (int s = from + lane; s < to; s += 32) {
        Entry& e = a.entries[ng + s];
        if (e.n > 0 && e.len >= 0) {
          e.begin = shared;
          e.group = g;
        }
      }
  }
  if (a.tiles == 0) return;
  __syncthreads();
  if (warp == 0) {                     // tiles of those with many rows
    int place = 0, most = 0;           // blocks of the longest
    float all_blocks = 0.f;
    for (int i0 = 0; i0 < ng + n; i0 += 32) {
      const int i = i0 + lane;
      int k = 0;
      if (i < ng + n && (i < ng || a.own_tiles)) {
        const Entry& e = a.entries[i];
        const long long rows = (long long)e.n * a.G;
        if (e.len >= 0 && rows > LONG_ROWS) k = (int)min((rows + PP_ROWS - 1) / PP_ROWS, (long long)(1 << 24));
      }
      int pre = k;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, pre, o);
        if (lane >= o) pre = min(pre + y, 1 << 28);
      }
      if (k > 0) {
        if (place + pre <= a.tiles) {
          Entry& e = a.entries[i];
          e.place = place + pre - k;
          const int b = max((e.ctx + PP_KEYS - 1) / PP_KEYS - e.begin / PP_KEYS, 1);
          most = max(most, b);
          // a group's tokens see all positions, a sequence's half of its new ones on average
          const int lo = i < ng ? b : min(max((e.len - e.begin) / PP_KEYS + 1, 1), b);
          all_blocks += (float)(k * a.pool.H) * 0.5f * (float)(lo + b);
        } else {
          report(a.err, ERR_BATCH);    // (offsets that do not ascend: the other kernel takes it)
          pre = 0;
        }
      }
      place += __reduce_max_sync(0xffffffffu, place + pre <= a.tiles ? pre : 0);
    }
    // all of them cut alike, so that their parts have a CTA each
    most = __reduce_max_sync(0xffffffffu, most);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all_blocks += __shfl_xor_sync(0xffffffffu, all_blocks, o);
    const int all = place * a.pool.H;
    int share = INT32_MAX, few = AT_CTAS * a.sms;
    const int most_parts = all > 0 ? min(a.room / all, PP_MORE_PARTS) : 0;
    if (most_parts > 1) share = max(share_of<false>(all, most, all_blocks, a.sms, most_parts, lane), 1);
    // Both kernels fill the SMs, one after the other, unless this leaves some of them to the other: then
    // they run side by side.  us of a place of its list and CTA, and of both kernels' ends, set on 64 sequences over
    // 32768 positions with 100 to 2000 own ones (one after the other 116 us, side by side 100), three ragged
    // groups (58, 49) and drafted tokens over two prefixes (28, 26); with 0.1 or 0.2 us a place, ends of 6 or 12,
    // within 12% of that.  Over 24 to 128 sequences of 100 to 4000 own positions over 4096 to 65536 shared ones, both
    // types and head sizes, 1 to 8 KV heads, 1 and 4 groups (86 measured): what this chooses takes 0.70 to 1.03
    // of one after the other, but once 1.11 (64 of 100 over 4096, fp32: 36.9, 33.2).
    constexpr float PLACE_US = 0.14f, FEW_US = 10.f, ENDS_US = 9.f;
    float work = 0.f;
    for (int i = lane; i < ng + n; i += 32) {
      const Entry& e = a.entries[i];
      if (e.place >= 0) continue;
      const float units = e.n > 1 ? ceilf((float)e.n * (float)a.G / (float)FEW_ROWS) : (float)(e.n * a.one);
      work += units * (float)(max((e.ctx + BLK - 1) / BLK - e.begin / BLK, 1) + AT_ENDS);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) work += __shfl_xor_sync(0xffffffffu, work, o);
    work *= (float)a.pool.H * PLACE_US / (float)AT_CTAS;
    if (all > 0 && all < a.sms) {
      const int c = lane + 1, used = all * c, b = (most - 1) / c + 1;
      const bool can = c <= most_parts && used <= a.sms - 8 && (c == 1 || b >= PP_LEAST);
      const float cost = can ? fmaxf(ENDS_US + (float)b * a.block_us, FEW_US + work / (float)(a.sms - used)) : 3e38f;
      const unsigned key = __reduce_min_sync(0xffffffffu, (__float_as_uint(cost) & ~31u) | (unsigned)lane);
      const int at = key & 31u;
      const float best = __shfl_sync(0xffffffffu, cost, at);
      const float alone = ENDS_US + (float)min(share, most) * a.block_us + FEW_US + work / (float)a.sms;
      if (best < alone && best < 3e38f) {
        share = max(__shfl_sync(0xffffffffu, b, at), 1);
        few = AT_CTAS * (a.sms - all * (at + 1));
      }
    }
    if (lane == 0) {
      a.tiles_out[TILES_ALL] = all;
      a.tiles_out[TILES_SHARE] = share;
      a.tiles_out[TILES_FEW] = few;
    }
  }
}

struct JoinArgs {
  Batch b;
  Parts from;
  const float* part;                   // sums of the tcgen05 kernel's cut tiles
  const float2* part_ml;
  void* out;
  float* lse;
  int H, G, out_f32;
};
constexpr int JOIN_WARPS = 4;

// A warp joins one row: a lane has one or two parts' bases, then four (d = 128) values of all parts.
template <int D>
__global__ void __launch_bounds__(32 * JOIN_WARPS) shared_join_kernel(JoinArgs a) {
  constexpr int CH = D / 4, AT_ONCE = 32 / CH, BATCH = 10;   // lanes of a row, parts at once, and on their way
  const int lane = threadIdx.x & 31, cc = lane % CH, sub = lane / CH, HQ = a.H * a.G;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long row = (long long)blockIdx.x * JOIN_WARPS + (threadIdx.x >> 5);
  const int tok = (int)(row / HQ), hq = (int)(row - (long long)tok * HQ), h = hq / a.G, g = hq - h * a.G;
  if (tok >= a.b.n_tokens) return;
  int s = tok;
  if (a.b.starts) {
    if (tok < a.b.starts[0] || tok >= a.b.starts[a.b.n_seq]) return;   // nobody's
    int lo = 0, hi = a.b.n_seq - 1;              // the last sequence that starts at or before the token
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.b.starts[mid] <= tok) lo = mid; else hi = mid - 1;
    }
    s = lo;
  }
  const int all = a.part ? a.from.tiles[TILES_ALL] : 0;  // a tile's parts lie that far apart
  // a row's sums: one row of `sums`, or a tile's parts
  struct Source {
    const float* p;
    const float2* ml;
    int n;
  };
  auto source = [&](const Entry& e, bool group) {
    Source x;
    const int r = (tok - e.first) * a.G + g;
    const int pair = e.place >= 0 ? (e.place + r / PP_ROWS) * a.H + h : 0;
    x.n = e.place >= 0 ? a.from.tiles[TILES_PARTS + pair] : 1;
    const long long at = row + (group ? a.from.rows : 0), slot0 = all - 1 - pair;
    x.p = x.n > 1 ? a.part + (slot0 * PP_ROWS + r % PP_ROWS) * D + 4 * cc : a.from.sums + at * D + 4 * cc;
    x.ml = x.n > 1 ? a.part_ml + slot0 * PP_ROWS + r % PP_ROWS : a.from.ml + at;
    return x;
  };
  const Entry own = a.from.entries[a.from.n_groups + s];
  const Source o = source(own, false);
  Source sh{};
  if (own.group >= 0) sh = source(a.from.entries[own.group], true);
  const int n = o.n + sh.n;                      // (at most 64 parts)
  float2 ml[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = lane + 32 * i;
    ml[i] = make_float2(-INFINITY, 0.f);
    if (c < n) ml[i] = __ldcg(c < o.n ? o.ml + (long long)c * all * PP_ROWS : sh.ml + (long long)(c - o.n) * all * PP_ROWS);
  }
  float4 v[BATCH];
  const long long step = (long long)all * D * PP_ROWS;
  auto fetch = [&](int c0) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int c = c0 + i * AT_ONCE + sub;
      const float* p = c < o.n ? o.p + c * step : sh.p + (c - o.n) * step;
      if (c < n) v[i] = __ldcg(reinterpret_cast<const float4*>(p));
    }
  };
  fetch(0);
  float top = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
  float f[2], l = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 f2 = down2(ml[i].x - top);
    f[i] = f2.x * f2.y;
    l = fmaf(ml[i].y * f2.x, f2.y, l);           // (a NaN stays one; no part: 0)
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int c0 = 0;;) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int c = c0 + i * AT_ONCE + sub;
      const float f0 = __shfl_sync(0xffffffffu, f[0], c & 31), f1 = __shfl_sync(0xffffffffu, f[1], c & 31);
      if (c < n) {
        const float fc = c < 32 ? f0 : f1;
        y.x = fmaf(v[i].x, fc, y.x);
        y.y = fmaf(v[i].y, fc, y.y);
        y.z = fmaf(v[i].z, fc, y.z);
        y.w = fmaf(v[i].w, fc, y.w);
      }
    }
    c0 += BATCH * AT_ONCE;
    if (c0 >= n) break;
    fetch(c0);
  }
  if (AT_ONCE == 2) {
    y.x += __shfl_xor_sync(0xffffffffu, y.x, 16);
    y.y += __shfl_xor_sync(0xffffffffu, y.y, 16);
    y.z += __shfl_xor_sync(0xffffffffu, y.z, 16);
    y.w += __shfl_xor_sync(0xffffffffu, y.w, 16);
  }
  const float inv = l == 0.f ? 0.f : (1.f / P_SCALE) / l;
  y.x *= inv; y.y *= inv; y.z *= inv; y.w *= inv;
  if (sub == 0) {
    if (a.out_f32)
      reinterpret_cast<float4*>(a.out)[row * CH + cc] = y;
    else
      reinterpret_cast<uint2*>(a.out)[row * CH + cc] = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
  }
  if (lane == 0 && a.lse) a.lse[row] = l == 0.f ? -INFINITY : (top - W_OFF + log2f(l)) * 0.69314718055994530942f;
}

template <typename A>
cudaError_t launch_after(void (*k)(A), long long grid, int threads, const A& a, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a);
}

// Tiles of the tcgen05 kernel at most, of one head: groups' parts, and sequences' own.
long long group_tiles(const Batch& b, int n_groups, int G) {
  const long long rows = (long long)b.n_tokens * G;
  return rows > LONG_ROWS ? rows / PP_ROWS + std::min<long long>(n_groups, rows / (LONG_ROWS + 1)) : 0;
}
long long own_tiles(const Batch& b, int G) {
  const long long rows = (long long)b.n_tokens * G;
  return b.starts && (long long)b.max_new * G > LONG_ROWS ? rows / PP_ROWS + std::min<long long>(b.n_seq, rows / (LONG_ROWS + 1)) : 0;
}

struct Layout {
  size_t tiles, ml, sums, bytes;
};
Layout layout(const Batch& b, int n_groups, int HQ, int H, int d) {
  const long long rows = (long long)b.n_tokens * HQ, tiles = (group_tiles(b, n_groups, HQ / H) + own_tiles(b, HQ / H)) * H;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Layout l;
  l.tiles = up((size_t)((long long)n_groups + b.n_seq) * sizeof(Entry));
  l.ml = l.tiles + up((size_t)(tiles + TILES_PARTS) * 4);
  l.sums = l.ml + up((size_t)rows * 2 * sizeof(float2));
  l.bytes = l.sums + (size_t)rows * 2 * d * 4;
  return l;
}

// The kernel for few rows, FEW_ROWS at once.  us so / 16 at once, over 4096 shared positions and 4 KV heads:
// 32 sequences with 1000 own positions, 16 query heads, d = 128 fp32 36.3 / 37.4, bf16 32.3 / 37.9, d = 64 31.2 /
// 31.3, 27.5 / 30.9; 3 with 3000 21.3 / 27.0, 20.7 / 25.7, 18.8 / 21.0, 18.7 / 21.4; 7 of 2 tokens and 4 heads
// 22.1 / 29.1, 21.8 / 26.6, 20.2 / 22.0, 19.8 / 22.2; 5 of 3 tokens over 8192 28.7 / 32.8, 27.0 / 29.2, 26.1 /
// 24.5, 25.4 / 23.5.
template <int D>
cudaError_t launch_few(const AttendArgs& a, int sms, bool precise, cudaStream_t stream) {
  const int grid = AT_CTAS * sms;
  constexpr int W = D == 64 ? 8 : 6;
  return precise ? launch_attend<D, 1, W, true, true>(a, grid, stream) : launch_attend<D, 1, W, false, true>(a, grid, stream);
}

}  // namespace

bool paged_shared_fits(const Pool& pool, const Batch& b, int n_groups, int HQ) {
  const int G = HQ / pool.H;
  return ((long long)b.n_tokens * G / PP_ROWS + b.n_seq + ((long long)b.n_tokens * G / PP_ROWS + n_groups)) * pool.H <= INT32_MAX &&
         (long long)n_groups + b.n_seq <= INT32_MAX / 2 &&
         ((long long)b.n_tokens * HQ + JOIN_WARPS) / JOIN_WARPS <= INT32_MAX;
}
size_t paged_shared_scratch(const Pool& pool, const Batch& b, int n_groups, int HQ) {
  return layout(b, n_groups, HQ, pool.H, pool.d).bytes;
}

cudaError_t launch_paged_shared(const Pool& pool, const Batch& b, const int32_t* groups, const int32_t* prefix,
                                int n_groups, const void* q, long long q_ts, long long q_hs, int HQ, void* out,
                                int out_f32, float* lse, void* workspace, void* scratch, int sms, int32_t* err,
                                cudaStream_t stream) {
  const int H = pool.H, G = HQ / H;
  const Layout lay = layout(b, n_groups, HQ, H, pool.d);
  char* const base = static_cast<char*>(scratch);
  const long long own = own_tiles(b, G), tiles = group_tiles(b, n_groups, G) + own;
  PlanArgs plan{};
  plan.pool = pool;
  plan.b = b;
  plan.groups = groups;
  plan.prefix = prefix;
  plan.err = err;
  plan.entries = reinterpret_cast<Entry*>(base);
  plan.n_groups = n_groups;
  plan.G = G;
  plan.tiles = (int)tiles;
  plan.own_tiles = own > 0;
  plan.tiles_out = reinterpret_cast<int*>(base + lay.tiles);
  // a CTA for every tile there may be, and a part on every SM beside them; parts have a place for their sums
  const long long grid_tc = tiles * H + sms;
  plan.room = (int)std::min<long long>(grid_tc, slots_of(sms));
  plan.sms = sms;
  plan.one = (G + FEW_ROWS - 1) / FEW_ROWS;
  plan.block_us = pool.d == 128 ? (out_f32 ? 1.5f : 0.95f) : out_f32 ? 1.f : 0.7f;
  cudaError_t e = launch_after(shared_plan_kernel, 1, PLAN_THREADS, plan, stream);
  if (e != cudaSuccess) return e;
  Parts to{};
  to.entries = plan.entries;
  to.n_groups = n_groups;
  to.rows = (long long)b.n_tokens * HQ;
  to.tiles = plan.tiles_out;
  to.ml = reinterpret_cast<float2*>(base + lay.ml);
  to.sums = reinterpret_cast<float*>(base + lay.sums);
  Batch list = b;                      // of parts
  list.n_seq = n_groups + b.n_seq;
  to.room = plan.room;
  char* const counters = static_cast<char*>(workspace) + counter_bytes(sms);
  char* const parts = counters + paged_prompt_counters(sms);

  const float c = (float)(1.4426950408889634 / sqrt((double)pool.d));
  JoinArgs join{};
  if (tiles > 0) {
    PromptArgs a{};
    a.pool = pool;
    a.b = list;
    a.q = static_cast<const bf16*>(q);
    a.q_ts = q_ts;
    a.q_hs = q_hs;
    a.out = to.sums;
    a.out_f32 = 1;
    a.err = err;
    a.c = c;
    a.G = G;
    a.sms = sms;
    a.count = reinterpret_cast<int*>(counters);
    a.part = reinterpret_cast<float*>(parts + part_bytes(sms));
    a.part_ml = reinterpret_cast<float2*>(a.part + slots_of(sms) * PP_ROWS * pool.d);
    a.sum = a.part + slots_of(sms) * PP_ROWS * (pool.d + 2);
    a.claim = a.count + slots_of(sms);
    a.to = to;
    const dim3 grid((unsigned)grid_tc);
    const bool chained = ((long long)b.max_pages << pool.page_shift) > PP_CHAIN_BF16 * PP_KEYS;
    if (pool.d == 128)
      e = out_f32 ? launch_prompt<128, true, true, true>(a, grid, stream)
          : chained ? launch_prompt<128, false, true, true>(a, grid, stream) : launch_prompt<128, false, false, true>(a, grid, stream);
    else
      e = out_f32 ? launch_prompt<64, true, true, true>(a, grid, stream)
          : chained ? launch_prompt<64, false, true, true>(a, grid, stream) : launch_prompt<64, false, false, true>(a, grid, stream);
    if (e != cudaSuccess) return e;
    join.part = a.part;
    join.part_ml = a.part_ml;
  }
  AttendArgs a{};
  a.pool = pool;
  a.b = list;
  a.q = static_cast<const bf16*>(q);
  a.q_ts = q_ts;
  a.q_hs = q_hs;
  a.count = static_cast<int*>(workspace);
  a.part = reinterpret_cast<float*>(parts);
  a.err = err;
  a.c = c;
  a.G = G;
  a.inv_g = 1.f / (float)G;
  a.skip_long = tiles > 0;
  a.one = plan.one;
  a.to = to;
  e = pool.d == 128 ? launch_few<128>(a, sms, out_f32 != 0, stream) : launch_few<64>(a, sms, out_f32 != 0, stream);
  if (e != cudaSuccess) return e;
  join.b = b;
  join.from = to;
  join.out = out;
  join.lse = lse;
  join.H = H;
  join.G = G;
  join.out_f32 = out_f32;
  const long long grid = (to.rows + JOIN_WARPS - 1) / JOIN_WARPS;
  return pool.d == 128 ? launch_after(shared_join_kernel<128>, grid, 32 * JOIN_WARPS, join, stream)
                       : launch_after(shared_join_kernel<64>, grid, 32 * JOIN_WARPS, join, stream);
}

}  // namespace kvpop
