// Attention weights of the paged 8-bit cache's positions, added up over query rows.
//
// For a sequence with L tokens held and new tokens i at places L + i, and one KV head with its G
// query heads, every position t < L + n gets
//   mass_t = (t < L ? mass_t : 0) + sum over rows (i, g) with t <= L + i of exp(q.K_t / sqrt(d) - lse),
// lse being the rows' normalisers as the attention returned them.  A row whose lse is -inf saw
// nothing and adds nothing.
//
// The keys are the wide side: a warp takes blocks of 16 positions, S^T = K Q^T as m16n8k16 in f16,
// where e4m3 values and scaled bf16 queries are exact (as in the attention), and each product is
// turned into its weight by one fma and one exponential.  A position's sum stays with its warp, so
// there are no atomics and no order that changes.  Bound by the keys' bytes for single tokens
// (d + 1/4 + 8 a position and head): 64 sequences of 8192 positions and 8 heads 96 us, 0.89 of the copy
// rate.  More than 32 rows go to the tcgen05 kernel.
#include "kvpop_paged.cuh"
#include "kvpop_mma.cuh"
#include "kvpop_ptx.cuh"

namespace kvpop {
namespace {

using namespace paged;

constexpr int WG_WARPS = 8, WG_CTAS = 2;
// Rows of a sequence above which it goes to the tcgen05 kernel, whose time hardly depends on them.  us here for
// up to 8, 32, 64 rows / there: 16 sequences of 10000 positions and 4 heads, d = 128 18, 36, 64 / 49; d = 64 15,
// 25, 45 / 40; 64 of 2000 and 8 heads 31, 57, 107 / 75; d = 64 23, 38, 72 / 60; 2 of 3000 and 2 heads 5.7, 9.4,
// 16 / 12.
constexpr int WG_ROWS = 32;

struct WeighArgs {
  Pool pool;
  Batch b;
  const bf16* q;
  long long q_ts, q_hs;
  const float* lse;                    // [n_tokens][H * G]
  float* mass;                         // [n_seq][H][positions]
  long long positions;
  int32_t* err;
  float c;                             // log2(e) / sqrt(d)
  int G;
  int most;                            // sequences with more rows are the tcgen05 kernel's
};

// A warp's ring of blocks: 16 rows of keys, their weights so far and their scale.  The 16-byte chunk c
// of row r lies at chunk c ^ (r mod 8) of its 128 bytes (d = 128), or c ^ (r / 2 mod 4) of its 64.
template <int D>
struct WRing {
  static constexpr int ST = D == 128 ? 5 : 10, KEYS = BLK * D, BLOCK = KEYS + 128, BYTES = WG_WARPS * ST * BLOCK;
  static __device__ __forceinline__ int chunk_at(int r, int c) {
    return r * D + ((c ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4);
  }
  static __device__ __forceinline__ int k_at(int r, int t, int i) { return chunk_at(r, D == 128 ? 2 * t + i : t); }
};

// What a sequence is in the list: H x blocks, each of `passes` places.
struct WSeq {
  SeqTokens t;
  int ctx, blocks, passes;
  __device__ long long work(int H) const { return (long long)H * blocks * passes; }
};
template <int ROWS>
__device__ __forceinline__ WSeq wseq(const WeighArgs& a, int s) {
  WSeq w;
  w.t = seq_tokens(a.b, s, a.err);
  if ((long long)w.t.n * a.G > a.most) w.t.n = 0;
  w.ctx = w.t.n > 0 ? context(a.b, a.pool, w.t, a.err) : 0;
  w.blocks = (w.ctx + BLK - 1) / BLK;
  w.passes = (int)(((long long)w.t.n * a.G + ROWS - 1) / ROWS);
  return w;
}

template <int D, int NT>
__global__ void __launch_bounds__(32 * WG_WARPS, WG_CTAS) paged_weigh_kernel(WeighArgs a) {
  using R = WRing<D>;
  constexpr int ROWS = 8 * NT, KW = D / 16;
  extern __shared__ __align__(128) unsigned char smw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3, H = a.pool.H;
  // Behind the tcgen05 kernel, which lets this one start when all that came before is done, nothing is to be
  // waited for but that this one does not end first: its last CTA sees to that.
  const bool beside = a.most < INT32_MAX;
  if (!beside) asm volatile("griddepcontrol.wait;" ::: "memory");
  auto leave = [&] {
    if (beside && blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
  };
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // ---- the list of all blocks, and the warp's part of it: the blocks that begin in [w0, w1)
  long long total = 0;
  for (int s = lane; s < a.b.n_seq; s += 32) total += wseq<ROWS>(a, s).work(H);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (total == 0) return leave();
  const long long parts = (long long)gridDim.x * WG_WARPS, part = (long long)blockIdx.x * WG_WARPS + warp;
  const long long w0 = total / parts * part + total % parts * part / parts;
  const long long w1 = total / parts * (part + 1) + total % parts * (part + 1) / parts;
  if (w0 >= w1) return leave();
  int s = -1;
  long long base = 0;
  for (int s0 = 0; s0 < a.b.n_seq && s < 0; s0 += 32) {
    const long long mine = s0 + lane < a.b.n_seq ? wseq<ROWS>(a, s0 + lane).work(H) : 0;
    long long pre = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, pre, o);
      if (lane >= o) pre += y;
    }
    const unsigned has = __ballot_sync(0xffffffffu, w0 < base + pre);
    if (has) {
      const int who = __ffs(has) - 1;
      s = s0 + who;
      base += __shfl_sync(0xffffffffu, pre - mine, who);
    } else {
      base += __shfl_sync(0xffffffffu, pre, 31);
    }
  }
  const uint32_t ring = smem_u32(smw) + warp * (R::ST * R::BLOCK);
  unsigned char* const ringp = smw + warp * (R::ST * R::BLOCK);
  constexpr int RPI = 512 / D;
  const int r0 = lane / (D / 16), c0 = lane % (D / 16), put0 = R::chunk_at(r0, c0), put1 = R::chunk_at(r0 + RPI, c0);

  WSeq x = wseq<ROWS>(a, s);
  for (long long w = w0; w < w1;) {
    while (w >= base + x.work(H)) {
      base += x.work(H);
      if (++s >= a.b.n_seq) return leave();
      x = wseq<ROWS>(a, s);
    }
    // blocks [k0, k1) of KV head h
    const long long blk = (w - base + x.passes - 1) / x.passes;
    const int h = (int)(blk / x.blocks), k0 = (int)(blk - (long long)h * x.blocks);
    if (h >= H) {                                      // (the last block began before the part)
      w = base + x.work(H);
      continue;
    }
    const long long unit = base + (long long)h * x.blocks * x.passes;
    const int k1 = (int)min((w1 - unit + x.passes - 1) / x.passes, (long long)x.blocks);
    w = unit + (long long)(k1 == x.blocks ? x.blocks : k1) * x.passes;
    if (k0 >= k1) {
      w = max(w, w1);
      continue;
    }
    float* const mass = a.mass + ((long long)s * H + h) * a.positions;
    const int32_t* const row = a.b.table + (long long)s * a.b.table_stride;
#pragma unroll 1
    for (int pass = 0; pass < x.passes; ++pass) {
      const int row0 = pass * ROWS, rows = (int)min((long long)ROWS, (long long)x.t.n * a.G - row0);
      // the last block that some row of the pass sees; the first pass sets all blocks
      const int seen = last_seen(x.t.len, (row0 + rows - 1) / a.G, x.ctx);
      const int end = pass == 0 ? k1 : min(k1, seen / BLK + 1);
      int asked = k0;
      auto ask = [&] {
        if (asked < end) {
          const int pos = asked * BLK, id = pos < x.ctx ? row[pos >> a.pool.page_shift] : -1;
          const uint32_t dst = ring + (asked - k0) % R::ST * R::BLOCK;
          float* const tail = reinterpret_cast<float*>(ringp + (asked - k0) % R::ST * R::BLOCK + R::KEYS);
          if ((unsigned)id < (unsigned)a.pool.n_pages) {
            const long long at = ((long long)id * H + h) * a.pool.page + (pos & (a.pool.page - 1));
            const unsigned char* kp = a.pool.k + at * D + 16 * lane;
#pragma unroll
            for (int i = 0; i < BLK / RPI; ++i) cp_async16(dst + (i & 1 ? put1 : put0) + 512 * (i & ~1), kp + 512 * i, 16);
            if (lane == 16) cp_async4(dst + R::KEYS + 64, a.pool.ks + at / BLK);
          } else if (lane == 16) {
            report(a.err, ERR_PAGE);
            tail[16] = -1.f;
          }
          if (lane < 16 && pos + lane < x.ctx) cp_async4(dst + R::KEYS + 4 * lane, mass + pos + lane);
          ++asked;
        }
        cp_commit();
      };
      __syncwarp();
#pragma unroll 1
      for (int i = 0; i < R::ST; ++i) ask();
      // ---- query rows, each scaled by a power of two, and what that makes of the logits
      uint32_t qf[NT][KW][2];
      float rc[NT][2], nl[NT][2];
      int lim[NT][2];                                  // last position a row sees
      bool all = rows == ROWS;                         // rows that are none, or saw nothing, are always masked
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const bool ok = 8 * j + g < rows;
        const int r = row0 + (ok ? 8 * j + g : 0), tok = r / a.G;
        const bf16* qp = a.q + (long long)(x.t.first + tok) * a.q_ts + (long long)(h * a.G + (r - tok * a.G)) * a.q_hs + 4 * KW * t4;
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
        const float down = a.c * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          rc[j][e] = __shfl_sync(0xffffffffu, down, (2 * t4 + e) * 4);
          const int i = 8 * j + 2 * t4 + e, rr = row0 + min(i, rows - 1), tk = rr / a.G;
          const float l = a.lse[((long long)(x.t.first + tk) * H + h) * a.G + (rr - tk * a.G)];
          lim[j][e] = i < rows && l != -INFINITY ? last_seen(x.t.len, tk, x.ctx) : -1;
          nl[j][e] = -l * 1.4426950408889634f;
          all &= l != -INFINITY;
        }
      }
      // all rows see 0 .. lim_lo
      const int lim_lo = __all_sync(0xffffffffu, all) ? last_seen(x.t.len, row0 / a.G, x.ctx) : -1;
#pragma unroll 1
      for (int k = k0; k < end; ++k) {
        cp_wait<R::ST - 1>();
        __syncwarp();
        const unsigned char* kp = ringp + (k - k0) % R::ST * R::BLOCK;
        const float* tail = reinterpret_cast<const float*>(kp + R::KEYS);
        const float ks = tail[16];
        float sum[2] = {0.f, 0.f};
        if (ks >= 0.f) {
          float sc[NT][4], sd[NT][4];
#pragma unroll
          for (int kk = 0; kk < KW; kk += 4) {
            const uint4 ka = *reinterpret_cast<const uint4*>(kp + R::k_at(g, t4, kk >> 2));
            const uint4 kb = *reinterpret_cast<const uint4*>(kp + R::k_at(g + 8, t4, kk >> 2));
            const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a0, a1, a2, a3;
              cvt4(wa[i], a0, a2);
              cvt4(wb[i], a1, a3);
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                float (&z)[4] = i & 1 ? sd[j] : sc[j];
                if (kk + i < 2) mma_f16_0(z, a0, a1, a2, a3, qf[j][kk + i][0], qf[j][kk + i][1]);
                else mma_f16(z, a0, a1, a2, a3, qf[j][kk + i][0], qf[j][kk + i][1]);
              }
            }
          }
          const bool edge = k * BLK + BLK - 1 > lim_lo;
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float y = ex2(fmaf(sc[j][e] + sd[j][e], rc[j][e & 1] * ks, nl[j][e & 1]));
              if (edge && k * BLK + g + 8 * (e >> 1) > lim[j][e & 1]) y = 0.f;
              sum[e >> 1] += y;
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
          sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
        }
        // lanes of the first quarter write rows 0-7, of the second 8-15
        const int r = g + 8 * t4, pos = k * BLK + r;
        if (t4 < 2 && pos < x.ctx && (ks >= 0.f || pass == 0)) {
          const float before = pass == 0 && pos >= x.t.len ? 0.f : tail[r];
          mass[pos] = before + (t4 ? sum[1] : sum[0]);
        }
        __syncwarp();
        ask();
      }
      cp_wait<0>();
      __syncwarp();
    }
  }
  leave();
}

template <int D, int NT>
cudaError_t launch(const WeighArgs& a, int grid, cudaStream_t stream) {
  auto k = paged_weigh_kernel<D, NT>;
  static std::atomic<unsigned long long> raised{0};
  const cudaError_t e = raise_smem_limit_once(raised, k, WRing<D>::BYTES);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(32 * WG_WARPS);
  cfg.dynamicSmemBytes = WRing<D>::BYTES;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a);
}

}  // namespace

cudaError_t launch_paged_weigh(const Pool& pool, const Batch& b, const void* q, long long q_ts, long long q_hs,
                               int HQ, const float* lse, float* mass, long long positions, void* workspace, int sms,
                               int32_t* err, cudaStream_t stream) {
  const int G = HQ / pool.H;
  const long long most_rows = b.starts ? (long long)b.max_new * G : G;
  WeighArgs a{};
  a.most = INT32_MAX;
  if (most_rows > WG_ROWS) {
    a.most = WG_ROWS;
    // [counters][sums of parts], where the attention has its own
    char* const w = static_cast<char*>(workspace);
    const cudaError_t e = launch_paged_weigh_tc(pool, b, q, q_ts, q_hs, HQ, lse, mass, positions, WG_ROWS,
                                                reinterpret_cast<int*>(w),
                                                reinterpret_cast<float*>(w + paged_attend_parts(sms)), sms, err, stream);
    if (e != cudaSuccess || !b.starts) return e;         // (without offsets all sequences have G rows)
  }
  a.pool = pool;
  a.b = b;
  a.q = static_cast<const bf16*>(q);
  a.q_ts = q_ts;
  a.q_hs = q_hs;
  a.lse = lse;
  a.mass = mass;
  a.positions = positions;
  a.err = err;
  a.c = (float)(1.4426950408889634 / sqrt((double)pool.d));
  a.G = G;
  const int grid = WG_CTAS * sms;
  // groups of 8 rows at once, by the most that a sequence here has
  const int nt = most_rows <= 8 ? 1 : most_rows <= 16 ? 2 : 4;
  if (pool.d == 128)
    return nt == 1 ? launch<128, 1>(a, grid, stream) : nt == 2 ? launch<128, 2>(a, grid, stream) : launch<128, 4>(a, grid, stream);
  return nt == 1 ? launch<64, 1>(a, grid, stream) : nt == 2 ? launch<64, 2>(a, grid, stream) : launch<64, 4>(a, grid, stream);
}

}  // namespace kvpop
