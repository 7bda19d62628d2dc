// Eviction from the paged 8-bit cache by accumulated attention weight.
//
// For one (sequence, KV head) with L positions of weight m_t, kept are all if L <= keep, else the
// first `sinks`, the last `window`, and of those between the keep - sinks - window of largest m
// (NaN as -inf, -0 as 0, the lower position first among equals), in the order of their positions.
// Slot j of the new pages gets the j-th of them: its code times its block's scale, under the scale
// of its new block, the least 2^e with amax <= 448 2^e over the block's finite values:
//   code' = rn_e4m3(code 2^(e_old - e)),
// which is exact but for codes that fall below 2^-6.
//
// Two kernels.  The first finds the threshold of a row by three passes over the digits (11, 11 and
// 10 bits) of order-preserving keys, from shared memory where they fit, then writes the kept
// positions in order: a warp counts what it keeps of its stretch, and numbers it behind the others.
// A cluster of CTAs takes a row where there are few.  The second moves 16 slots of K and V a warp:
// rows come as whole 128 or 64 bytes.  Bound by memory: the weights once, each kept row read and
// written once.  64 sequences of 4160 to 4224 tokens and 8 heads (d = 128) to 4096: 183 us, 14 of them the
// selection; 1.1 GB, 0.89 of the copy rate for both, 0.91 for the move.  That is with a table as wide as its rows:
// the lengths are not known here, and a CTA's shared memory goes by the positions that the table has room for.
// The same rows in tables of 8192, 16384, 49152 and 131072 positions 217, 187, 211, 210 us.
#include <cooperative_groups.h>

#include "kvpop_paged.cuh"
#include "kvpop_mma.cuh"
#include "kvpop_ptx.cuh"

namespace cg = cooperative_groups;

namespace kvpop {
namespace {

using namespace paged;

constexpr int EV_WARPS = 16, EV_THREADS = 32 * EV_WARPS, EV_BINS = 2048;
constexpr int EV_CACHED = 48 * 1024;   // keys that a CTA holds at most (192 KB)
constexpr int MV_WARPS = 4;             // 64 sequences: 182.9 us (184.4 with 8, 190 with 16)

struct EvictArgs {
  Pool pool;
  Batch b;
  PagedEvict e;
  int32_t* err;
  int cached;                          // keys that a CTA has room for
};

// Tokens that a sequence holds, as far as its row of the table reaches; -1: idle.
__device__ __forceinline__ int held_of(const EvictArgs& a, int s) {
  const int len = a.b.lens[s];
  const long long cap = min((long long)a.b.max_pages << a.pool.page_shift, (long long)(INT32_MAX - 1024));
  if (len > cap) report(a.err, ERR_PAGE);
  return len < 0 ? -1 : (int)min((long long)len, cap);
}
// Larger weights have larger keys.
__device__ __forceinline__ uint32_t key_of(float m) {
  const uint32_t u = __float_as_uint(canon_score(m));
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// (four CTAs an SM, as long as their keys fit: with 40 registers 512 rows of 4200 took two waves)
__global__ void __launch_bounds__(EV_THREADS, 4) evict_select_kernel(EvictArgs a) {
  extern __shared__ uint32_t keyS[];
  __shared__ __align__(16) uint32_t histS[EV_BINS], sumS[EV_BINS];   // the CTA's counts, and its share of the cluster's
  __shared__ uint32_t warpS[2][EV_WARPS], foundS[2], sumsS[2];
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long row = blockIdx.x / C;
  const int s = (int)(row / a.pool.H), L = held_of(a, s), keep = a.e.keep;
  int32_t* const kept = a.e.kept + row * keep;
  if (a.e.new_lens && row % a.pool.H == 0 && rank == 0 && tid == 0) a.e.new_lens[s] = min(L, keep);
  const int at = rank * EV_THREADS + tid, step = C * EV_THREADS;
  if (L <= keep) {
    for (int i = at; i < keep; i += step) kept[i] = i < L ? i : -1;
    return;
  }
  const int lo = a.e.sinks, hi = L - a.e.window, want = keep - a.e.sinks - a.e.window;
  for (int i = at; i < lo; i += step) kept[i] = i;
  for (int i = at; i < a.e.window; i += step) kept[lo + want + i] = hi + i;
  if (want == 0) return;

  const int per = (hi - lo + C - 1) / C, first = lo + rank * per, n = max(min(per, hi - first), 0);
  const float* const m = a.e.mass + row * a.e.positions + first;
  const bool cached = per <= a.cached;
  auto key = [&](int i) { return cached ? keyS[i] : key_of(m[i]); };
  if (cached)
    for (int i = tid; i < n; i += EV_THREADS) keyS[i] = key_of(m[i]);
  for (int i = tid; i < EV_BINS; i += EV_THREADS) histS[i] = sumS[i] = 0;
  if (C > 1) cluster.sync(); else __syncthreads();

  // ---- the want-th largest key, digit by digit
  uint32_t prefix = 0, left = (uint32_t)want;          // of the keys that begin with prefix, left are wanted
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    const int shift = p == 0 ? 21 : p == 1 ? 10 : 0, bins = p == 2 ? 1024 : 2048;
    for (int i = tid; i < n; i += EV_THREADS) {
      const uint32_t k = key(i);
      if (p == 0 || k >> (shift + (p == 2 ? 10 : 11)) == prefix) atomicAdd(histS + (k >> shift & (bins - 1)), 1u);
    }
    __syncthreads();
    // the bins from the highest down, 4 (or 2) a thread
    constexpr int PER = EV_BINS / EV_THREADS;
    const int mine = p == 2 ? PER / 2 : PER, low = bins - mine * (tid + 1);   // bins low .. low + mine - 1
    uint32_t c[PER], sum = 0;
    if (C > 1) {
      // The cluster's counts of a pass come together in one of its CTAs: few bins are not empty.  (Read from
      // all CTAs by all, they took 7 us a pass.)
      uint32_t* const all = cluster.map_shared_rank(sumS, p);
      for (int i = tid; i < bins; i += EV_THREADS) {
        const uint32_t x = histS[i];
        if (x) atomicAdd(all + i, x);
        histS[i] = 0;
      }
      cluster.sync();
      const uint2 lo2 = *reinterpret_cast<const uint2*>(all + low);
      c[0] = lo2.x;
      c[1] = lo2.y;
      c[2] = c[3] = 0;
      if (mine == PER) {
        const uint2 hi2 = *reinterpret_cast<const uint2*>(all + low + 2);
        c[2] = hi2.x;
        c[3] = hi2.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        c[i] = i < mine ? histS[low + i] : 0;
        if (i < mine) histS[low + i] = 0;
      }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += c[i];
    uint32_t pre = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, pre, o);
      if (lane >= o) pre += y;
    }
    if (lane == 31) warpS[0][warp] = pre;
    __syncthreads();
    for (int w = 0; w < warp; ++w) pre += warpS[0][w];
    uint32_t above = pre - sum;
    if (above < left && left <= pre) {
#pragma unroll
      for (int i = PER - 1; i >= 0; --i) {
        if (above < left && left <= above + c[i]) {
          foundS[0] = (uint32_t)(low + i);
          foundS[1] = above;
        }
        above += c[i];
      }
    }
    __syncthreads();
    prefix = prefix << (p == 2 ? 10 : 11) | foundS[0];
    left -= foundS[1];
  }

  // ---- the kept ones in order: all above the threshold, and the first `left` that equal it
  const int stretch = ((n + EV_WARPS - 1) / EV_WARPS + 31) / 32 * 32, i0 = warp * stretch, i1 = min(i0 + stretch, n);
  uint32_t above = 0, equal = 0;
  for (int i = i0; i < i1; i += 32) {
    const uint32_t k = i + lane < i1 ? key(i + lane) : 0;
    above += __popc(__ballot_sync(0xffffffffu, i + lane < i1 && k > prefix));
    equal += __popc(__ballot_sync(0xffffffffu, i + lane < i1 && k == prefix));
  }
  if (lane == 0) {
    warpS[0][warp] = above;
    warpS[1][warp] = equal;
  }
  __syncthreads();
  uint32_t gt = 0, eq = 0, all_gt = 0, all_eq = 0;
  for (int w = 0; w < EV_WARPS; ++w) {
    if (w < warp) {
      gt += warpS[0][w];
      eq += warpS[1][w];
    }
    all_gt += warpS[0][w];
    all_eq += warpS[1][w];
  }
  if (C > 1) {
    if (tid == 0) {
      sumsS[0] = all_gt;
      sumsS[1] = all_eq;
    }
    cluster.sync();
    for (int r = 0; r < rank; ++r) {
      const uint32_t* other = cluster.map_shared_rank(sumsS, r);
      gt += other[0];
      eq += other[1];
    }
  }
  for (int i = i0; i < i1; i += 32) {
    const bool in = i + lane < i1;
    const uint32_t k = in ? key(i + lane) : 0, below = (1u << lane) - 1u;
    const uint32_t G = __ballot_sync(0xffffffffu, in && k > prefix), E = __ballot_sync(0xffffffffu, in && k == prefix);
    const uint32_t g = gt + __popc(G & below), e = eq + __popc(E & below);
    if (in && (k > prefix || (k == prefix && e < left))) kept[lo + (int)(g + min(e, left))] = first + i + lane;
    gt += __popc(G);
    eq += __popc(E);
  }
  if (C > 1) cluster.sync();                           // (no CTA leaves while its sums are read)
}

// Largest magnitude code of 16 bytes that is no NaN.  (Four bytes at a time their maxima took the move 69% of
// the ALUs; as f16, registers and so warps.)
__device__ __forceinline__ uint32_t top_code(uint4 w) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = u[i] & 0x7f7f7f7fu;
    t = __vmaxu2(t, x & 0x00ff00ffu);
    t = __vmaxu2(t, __byte_perm(x, 0, 0x4341));
  }
  t = max(t & 0xffffu, t >> 16);
  if (t == 0x7fu) {                                    // a NaN among them
    t = 0;
    for (int i = 0; i < 16; ++i) {
      const uint32_t x = u[i >> 2] >> 8 * (i & 3) & 0x7fu;
      if (x != 0x7fu) t = max(t, x);
    }
  }
  return t;
}
__device__ __forceinline__ float code_value(uint32_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
  return __half2float(__ushort_as_half((unsigned short)h));
}
// Four codes times f, a power of two below 2^16, rounded again (f16 holds what does not round to 0).
__device__ __forceinline__ uint32_t scaled4(uint32_t w, __half2 f) {
  uint32_t lo, hi;
  cvt4(w, lo, hi);
  const __half2 a = __hmul2(*reinterpret_cast<__half2*>(&lo), f), b = __hmul2(*reinterpret_cast<__half2*>(&hi), f);
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f16x2 l, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 h, %2;\n\t"
      "mov.b32 %0, {l, h};\n\t}"
      : "=r"(r)
      : "r"(*reinterpret_cast<const uint32_t*>(&a)), "r"(*reinterpret_cast<const uint32_t*>(&b)));
  return r;
}

template <int D>
__global__ void __launch_bounds__(32 * MV_WARPS) evict_move_kernel(EvictArgs a, int blocks, long long units) {
  constexpr int LPR = D / 16, RPI = 32 / LPR, IT = BLK / RPI;
  const int lane = threadIdx.x & 31, c = lane % LPR, sub = lane / LPR;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long unit = (long long)blockIdx.x * MV_WARPS + (threadIdx.x >> 5);
  if (unit >= units) return;
  const long long row = unit / blocks;
  const int slot0 = (int)(unit - row * blocks) * BLK, s = (int)(row / a.pool.H), h = (int)(row - (long long)s * a.pool.H);
  const int n = min(min(held_of(a, s), a.e.keep) - slot0, BLK);
  if (n <= 0) return;
  const int id_to = a.e.to[s * a.e.to_stride + (slot0 >> a.pool.page_shift)];
  if ((unsigned)id_to >= (unsigned)a.pool.n_pages) {
    if (lane == 0) report(a.err, ERR_PAGE);
    return;
  }
  // lanes 0-15: the rows' places and key scales, 16-31: the value scales
  const int r = lane & 15;
  long long at = -1;
  float scale = 0.f;
  if (r < n) {
    const int pos = a.e.kept[row * a.e.keep + slot0 + r], id = page_of(a.b, a.pool, s, pos, a.err);
    if (id >= 0) {
      at = ((long long)id * a.pool.H + h) * a.pool.page + (pos & (a.pool.page - 1));
      scale = (lane < 16 ? a.pool.ks : a.pool.vs)[at / BLK];
    }
    if (lane < 16 && a.e.new_mass)
      a.e.new_mass[row * a.e.new_positions + slot0 + r] = a.e.mass[row * a.e.positions + pos];
  }
  uint4 w[2][IT];
  long long from[IT];
#pragma unroll
  for (int i = 0; i < IT; ++i) from[i] = __shfl_sync(0xffffffffu, at, i * RPI + sub);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv)
#pragma unroll
    for (int i = 0; i < IT; ++i)
      w[kv][i] = from[i] >= 0 ? __ldcs(reinterpret_cast<const uint4*>((kv ? a.pool.v : a.pool.k) + from[i] * D + 16 * c))
                              : make_uint4(0, 0, 0, 0);
  const long long dst = ((long long)id_to * a.pool.H + h) * a.pool.page + (slot0 & (a.pool.page - 1));
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    float f[IT], top = 0.f;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      f[i] = __shfl_sync(0xffffffffu, scale, 16 * kv + i * RPI + sub);
      top = fmaxf(top, code_value(top_code(w[kv][i])) * f[i]);
    }
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));   // (not negative)
    const int e = scale_exponent(top);
    const float inv = pow2(-e);
    bool far = false, same = true;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      // (codes that are not 0 are at least 2^-9 and become 448 at most: above 2^18 there are zeros and NaN alone,
      // and times inf, which 2^100 / 2^-96 would be, a zero is none)
      f[i] = fminf(f[i] * inv, 1048576.f);
      far |= f[i] > 32768.f;
      same &= f[i] == 1.f || from[i] < 0;
    }
    if (__any_sync(0xffffffffu, !same)) {
      if (!__any_sync(0xffffffffu, far)) {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          const __half2 f2 = __float2half2_rn(f[i]);
          uint4& u = w[kv][i];
          u = make_uint4(scaled4(u.x, f2), scaled4(u.y, f2), scaled4(u.z, f2), scaled4(u.w, f2));
        }
      } else {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          uint4& u = w[kv][i];
          u = make_uint4(rescale4(u.x, f[i]), rescale4(u.y, f[i]), rescale4(u.z, f[i]), rescale4(u.w, f[i]));
        }
      }
    }
    unsigned char* const to = (kv ? a.pool.v : a.pool.k) + dst * D + 16 * c;
#pragma unroll
    for (int i = 0; i < IT; ++i)
      if (from[i] >= 0) __stcs(reinterpret_cast<uint4*>(to + (i * RPI + sub) * D), w[kv][i]);   // (used once, both: 3% of the time)
    if (lane == 0) (kv ? a.pool.vs : a.pool.ks)[dst / BLK] = pow2(e);
  }
}

// The launch's last attribute (after `n` others), and its stream.
void after_the_last(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* at, int n, cudaStream_t stream) {
  at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[n].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = n + 1;
  cfg.stream = stream;
}

}  // namespace

cudaError_t launch_paged_evict(const Pool& pool, const Batch& b, const PagedEvict& e, int sms, int32_t* err,
                               cudaStream_t stream) {
  EvictArgs a{};
  a.pool = pool;
  a.b = b;
  a.e = e;
  a.err = err;
  const long long rows = (long long)b.n_seq * pool.H, cap = (long long)b.max_pages << pool.page_shift;
  // CTAs of a row: more than one where the rows alone do not fill the SMs and may be long (20 rows of up to
  // 60000 positions: 53 us in all with all CTAs' counts read by each, 29 with the counts brought together)
  const int C = cap > 32768 && rows * 8 <= 4 * sms ? 8 : cap > 8192 && rows * 4 <= 4 * sms ? 4 : 1;
  a.cached = (int)std::min<long long>((cap + C - 1) / C, EV_CACHED);
  const size_t smem = (size_t)a.cached * 4;
  static std::atomic<unsigned long long> raised{0};
  cudaError_t err_ = raise_smem_limit_once(raised, evict_select_kernel, (size_t)EV_CACHED * 4);
  if (err_ != cudaSuccess) return err_;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  cfg.gridDim = dim3((unsigned)(rows * C));
  cfg.blockDim = dim3(EV_THREADS);
  cfg.dynamicSmemBytes = smem;
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  after_the_last(cfg, at, 1, stream);
  err_ = cudaLaunchKernelEx(&cfg, evict_select_kernel, a);
  if (err_ != cudaSuccess) return err_;
  const int blocks = (int)((std::min<long long>(e.keep, cap) + BLK - 1) / BLK);
  const long long units = rows * blocks;
  cfg.gridDim = dim3((unsigned)((units + MV_WARPS - 1) / MV_WARPS));
  cfg.blockDim = dim3(32 * MV_WARPS);
  cfg.dynamicSmemBytes = 0;
  after_the_last(cfg, at, 0, stream);
  return pool.d == 128 ? cudaLaunchKernelEx(&cfg, evict_move_kernel<128>, a, blocks, units)
                       : cudaLaunchKernelEx(&cfg, evict_move_kernel<64>, a, blocks, units);
}

}  // namespace kvpop
