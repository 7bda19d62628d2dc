// Attention of many new tokens a sequence over the paged 8-bit cache, on tcgen05.
//
// The mathematics is that of kvpop_paged_attend.cu: f16 products that are exact for the logits,
// the value scales in the exponent, p = 2^(x log2 e + ev - M + 7) as one f16 (bf16 results) or
// the sum of two (fp32 results, SPLIT).  A CTA owns 256 consecutive rows (token, query head) of
// one (sequence, KV head), as two halves of 128 rows, and streams the positions they see in blocks
// of 128, the same bytes for both halves.  Roles:
//  * 4 converter warps bring the bytes of a block's keys, then of its values, into registers while
//    the ones before are used, and write them as f16 into a ring of 5 128B-swizzled tiles.
//  * 1 MMA warp: S = Q K^T (M 128, N 128, K d) per half, and O += P V (N d, K 128) with P in
//    tensor memory and the values read MN-major from their rows.
//  * 2 x 4 softmax warps, a thread per row: the row's maximum, then its probabilities, written
//    over the logits 32 columns at a time and handed over in two parts, so that the product with
//    the first half of the block runs while the second is formed.
// Tensor memory: O (2 x d columns) and S (2 x 128) leave no second S buffer at d = 128, so the two
// halves alternate: one's logits and products run beside the other's exponentials.
#include "kvpop_mma.cuh"
#include "kvpop_paged.cuh"
#include "kvpop_ptx.cuh"
#include "kvpop_tc05.cuh"

namespace kvpop {
namespace {

using namespace paged;
using namespace tc05;

constexpr int PP_HALF = 128, PP_ROWS = 2 * PP_HALF, PP_KEYS = 128;
constexpr int PP_MMA_WARP = 8, PP_CONV_WARP = 12, PP_CONV = 4;   // warps 0-7: softmax, 8: MMA, 12-15: converters
constexpr int PP_THREADS = 32 * (PP_CONV_WARP + PP_CONV);
// Registers of a thread: at launch, and of the softmax, MMA and converter warpgroups.
constexpr int PP_REGS = 128, PP_REGS_ROW = 200, PP_REGS_MMA = 56, PP_REGS_CONV = 56;
static_assert(PP_THREADS * PP_REGS <= 65536 && 2 * PP_REGS_ROW + PP_REGS_MMA + PP_REGS_CONV <= 4 * PP_REGS, "");
constexpr int PP_RING = 5;
constexpr int PP_TMEM = 512;                             // O_h: 128 h; S_h: 256 + 128 h
constexpr float PP_OFF = 7.f, PP_STEP = 8.f;
// barriers
constexpr int PB_FULL = 0;                               // [ring] converters -> MMA
constexpr int PB_EMPTY = PB_FULL + PP_RING;              // [ring] MMA -> converters
constexpr int PB_S = PB_EMPTY + PP_RING;                 // [2] MMA -> softmax
constexpr int PB_P = PB_S + 2;                           // [2][2] softmax -> MMA, two parts
constexpr int PB_O = PB_P + 4;                           // [2] MMA -> softmax
constexpr int PB_N = PB_O + 2;
constexpr int PP_NANW = (PP_ROWS + 2 * PP_KEYS) / 32;    // words of the map of NaN values

struct PromptArgs {
  Pool pool;
  Batch b;
  const bf16* q;
  long long q_ts, q_hs;
  void* out;
  float* lse;
  int32_t* err;
  float c;                                               // log2(e) / sqrt(d)
  int G, out_f32;
};

template <int D>
struct PL {
  static constexpr int QB = PP_HALF * D * 2, KB = PP_KEYS * D * 2;
  static constexpr int OFF_RING = 2 * QB, OFF_BAR = OFF_RING + PP_RING * KB;
  static constexpr int OFF_TMEM = OFF_BAR + 8 * PB_N, OFF_NAN = (OFF_TMEM + 4 + 15) / 16 * 16;
  static constexpr int OFF_SCALE = OFF_NAN + 4 * PP_NANW;  // [8 warps][2][24] key scales, value exponents, 2^-those
  static constexpr int BYTES = OFF_SCALE + 8 * 2 * 24 * 4;
  static constexpr int OUT_WARP = 32 * D * 4;            // a warp's finished rows, in the ring
  static_assert(8 * OUT_WARP <= OFF_BAR, "");
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

// Registers of a thread from here on, for a whole warpgroup.
template <int N, bool MORE>
__device__ __forceinline__ void set_registers() {
  if (MORE) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// (volatile: read where it is used, not kept in registers that a row of logits needs)
__device__ __forceinline__ float2 lds2(uint32_t p) {
  float2 v;
  asm volatile("ld.volatile.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(p));
  return v;
}

template <int D, bool SPLIT>
__global__ void __launch_bounds__(PP_THREADS, 1) paged_prompt_kernel(PromptArgs a) {
  using L = PL<D>;
  extern __shared__ __align__(1024) unsigned char smp[];
  const uint32_t sb = smem_u32(smp);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = a.pool.H, G = a.G;
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8u * (uint32_t)i; };
  uint32_t* nanS = reinterpret_cast<uint32_t*>(smp + L::OFF_NAN);

  // ---- the tile: sequence s owns the places from starts[s] G / 256 + s on, which leaves one for
  // each of its tiles.  Later tokens see more, and go first.
  const unsigned order = gridDim.x - 1 - blockIdx.x;
  const int place = (int)(order / (unsigned)H), h = (int)(order % (unsigned)H);
  auto first_place = [&](int s) { return (long long)a.b.starts[s] * G / PP_ROWS + s; };
  int lo = 0, hi = a.b.n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first_place(mid) <= place) lo = mid; else hi = mid - 1;
  }
  const int s = lo;
  const SeqTokens t = seq_tokens(a.b, s, a.err);
  const long long row0l = (place - first_place(s)) * PP_ROWS, all_rows = (long long)t.n * G;
  if (!long_rows(t, G) || row0l < 0 || row0l >= all_rows) return;
  const int row0 = (int)row0l, rows = (int)min((long long)PP_ROWS, all_rows - row0l);
  const int ctx = context(a.b, a.pool, t, a.err);
  const int lim_lo = min(t.len + row0 / G, ctx - 1);     // every row sees 0 .. lim_lo
  const int lim_hi = min(t.len + (row0 + rows - 1) / G, ctx - 1);   // none sees past lim_hi
  const int nblk = lim_hi / PP_KEYS + 1;
  const int nan0 = (lim_lo + 1) / PP_KEYS * PP_KEYS;     // first position of the NaN map

  if (tid == 0) {
    for (int i = 0; i < PP_RING; ++i) {
      mbar_init(bar(PB_FULL + i), PP_CONV);
      mbar_init(bar(PB_EMPTY + i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(PB_S + i), 1);
      mbar_init(bar(PB_O + i), 1);
      mbar_init(bar(PB_P + 2 * i), 4);
      mbar_init(bar(PB_P + 2 * i + 1), 4);
    }
    mbar_fence_init();
  }
  if (tid < PP_NANW) nanS[tid] = 0;
  if (warp == PP_MMA_WARP) tmem_alloc(sb + L::OFF_TMEM, PP_TMEM);

  // ---- query rows as f16, each scaled by a power of two (a softmax thread has its row)
  float rc = 0.f;
  int lim = -1;
  if (warp < PP_MMA_WARP) {
    const int r = row0 + tid;
    const bool ok = tid < rows;
    const int tok = ok ? r / G : 0;
    if (ok) lim = min(t.len + tok, ctx - 1);
    const uint4* qp = reinterpret_cast<const uint4*>(a.q + (long long)(t.first + tok) * a.q_ts +
                                                     (long long)(h * G + (ok ? r - tok * G : 0)) * a.q_hs);
    uint4 v[D / 8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      v[i] = ok ? qp[i] : make_uint4(0, 0, 0, 0);
      const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) top = max(top, max(u[k] & 0x7fffu, u[k] >> 16 & 0x7fffu));
    }
    const int up = max(min(14 - ((int)(top >> 7) - 127), 110), -113);   // the largest to [2^14, 2^15)
    const float f = __uint_as_float((uint32_t)(up + 127) << 23);
    rc = a.c * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        o[k] = pack_h2(__uint_as_float(u[k] << 16) * f, __uint_as_float(u[k] & 0xffff0000u) * f);
      *reinterpret_cast<uint4*>(smp + (tid >> 7) * L::QB + tile_off(tid & 127, i, PP_HALF)) =
          make_uint4(o[0], o[1], o[2], o[3]);
    }
    fence_async_smem();
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smp + L::OFF_TMEM);
  // page of a block of 16 positions, -1 where the rows see none of it
  auto page16 = [&](int pos) { return pos <= lim_hi ? page_of(a.b, a.pool, s, pos, a.err) : -1; };
  auto uniform = [](bool x) { return __all_sync(0xffffffffu, x); };
  float m = -INFINITY, l = 0.f;
  bool ok = true;

  if (warp >= PP_CONV_WARP) {
    // ---------------------------------------------------------------- converters
    set_registers<PP_REGS_CONV, false>();
    constexpr int LPR = D / 16, RPI = 32 / LPR, IT = 32 / RPI;   // lanes of a row, rows at a time
    const int cw = warp - PP_CONV_WARP, c = lane % LPR, sub = lane / LPR;
    uint4 w[IT];
    int id[2];
    auto lookup = [&](int j) {
#pragma unroll
      for (int e = 0; e < 2; ++e) id[e] = j < nblk ? page16(j * PP_KEYS + cw * 32 + 16 * e) : -1;
    };
    auto load = [&](int j, const unsigned char* pages) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int row = i * RPI + sub, pos = j * PP_KEYS + cw * 32 + row, pg = id[(i * RPI) >> 4];
        w[i] = make_uint4(0, 0, 0, 0);
        if (pg >= 0 && pos <= lim_hi)
          w[i] = __ldg(reinterpret_cast<const uint4*>(
              pages + (((long long)pg * H + h) * a.pool.page + (pos & (a.pool.page - 1))) * D + 16 * c));
      }
    };
    lookup(0);
    load(0, a.pool.k);
    for (int i = 0; i < 2 * nblk && ok; ++i) {
      const int j = i >> 1, st = i % PP_RING;
      if (i >= PP_RING && !(ok = uniform(mbar_wait(bar(PB_EMPTY + st), (i / PP_RING - 1) & 1, a.err, ERR_WAIT)))) break;
      if ((i & 1) && (j + 1) * PP_KEYS - 1 > lim_lo) {
        // Values that some row does not see: a NaN must not reach the rows before it, where its
        // weight is 0.  Its column is set at the end, for the rows that see it.
#pragma unroll
        for (int x = 0; x < IT; ++x) {
          const bool bad = has_nan(w[x].x) || has_nan(w[x].y) || has_nan(w[x].z) || has_nan(w[x].w);
          if (bad) {
            const int pos = j * PP_KEYS + cw * 32 + x * RPI + sub;
            if (pos >= nan0) {
              atomicOr(nanS + ((pos - nan0) >> 5), 1u << ((pos - nan0) & 31));
              w[x] = make_uint4(drop_nan(w[x].x), drop_nan(w[x].y), drop_nan(w[x].z), drop_nan(w[x].w));
            }
          }
        }
      }
      unsigned char* tile = smp + L::OFF_RING + st * L::KB;
#pragma unroll
      for (int x = 0; x < IT; ++x) {
        uint4 p, q;
        cvt16(w[x], p, q);
        const int row = cw * 32 + x * RPI + sub;
        // (d = 128: lanes of the upper 64 values store their second chunk first, so that the 8
        // lanes of a row touch all banks)
        const int first = D == 128 ? c >> 2 : 0;
        *reinterpret_cast<uint4*>(tile + tile_off(row, 2 * c + first, PP_KEYS)) = first ? q : p;
        *reinterpret_cast<uint4*>(tile + tile_off(row, 2 * c + 1 - first, PP_KEYS)) = first ? p : q;
      }
      fence_async_smem();                                // (it would wait for loads before it)
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(PB_FULL + st));
      if (i & 1) {
        load(j + 1, a.pool.k);                           // (pages looked up below, one item ago)
      } else {
        load(j, a.pool.v);
        lookup(j + 1);
      }
    }
  } else if (warp >= PP_MMA_WARP) {
    set_registers<PP_REGS_MMA, false>();
    if (warp == PP_MMA_WARP) {
    // ---------------------------------------------------------------- MMA issue
    const uint32_t idS = idesc_f16(128, PP_KEYS, 0), idO = idesc_f16(128, D, 1);
    const bool lead = elect_one();
    const uint64_t qd0 = kmajor_desc(sb, PP_HALF, 0), kd0 = kmajor_desc(sb + L::OFF_RING, PP_KEYS, 0);
    const uint64_t vd0 = mnmajor_desc(sb + L::OFF_RING, PP_KEYS, 0);
    auto wait = [&](int b, int parity) {
      ok = ok && mbar_wait(bar(b), parity, a.err, ERR_WAIT);
      ok = uniform(ok);
      if (ok) fence_after();
    };
    auto issue_s = [&](int hf, int j) {                  // logits of half hf against block j
      const int st = 2 * j % PP_RING;
      if (hf == 0) wait(PB_FULL + st, (2 * j / PP_RING) & 1);
      if (ok && lead) {
        const uint64_t kd = desc_at(kd0, st * L::KB), qd = desc_at(qd0, hf * L::QB);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          mma_bf16(tmem + 256 + hf * 128, kmajor_step(qd, PP_HALF, ks), kmajor_step(kd, PP_KEYS, ks), idS, ks > 0);
        commit(bar(PB_S + hf));
        if (hf == 1) commit(bar(PB_EMPTY + st));
      }
      __syncwarp();
    };
    issue_s(0, 0);
    issue_s(1, 0);
    for (int j = 0; j < nblk && ok; ++j) {
      const int st = (2 * j + 1) % PP_RING;
      const uint64_t vd = desc_at(vd0, st * L::KB);
#pragma unroll 1
      for (int hf = 0; hf < 2 && ok; ++hf) {
        if (hf == 0) wait(PB_FULL + st, ((2 * j + 1) / PP_RING) & 1);
        const uint32_t tP = tmem + 256 + hf * 128, dO = tmem + hf * 128;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          wait(PB_P + 2 * hf + part, j & 1);
          if (ok && lead) {
#pragma unroll
            for (int k = 4 * part; k < 4 * part + 4; ++k) {
              const uint32_t ta = tP + 32 * (k >> 1) + 8 * (k & 1);
              const uint64_t vk = desc_at(vd, k * 16 * 128);
              mma_bf16_ts(dO, ta, vk, idO, j > 0 || k > 0);
              if (SPLIT) mma_bf16_ts(dO, ta + 16, vk, idO, 1);
            }
          }
          __syncwarp();
        }
        if (ok && lead) {
          commit(bar(PB_O + hf));
          if (hf == 1) commit(bar(PB_EMPTY + st));
        }
        __syncwarp();
        if (j + 1 < nblk) issue_s(hf, j + 1);
      }
    }
    }
  } else {
    // ---------------------------------------------------------------- softmax rows
    set_registers<PP_REGS_ROW, true>();
    const int hf = warp >> 2;
    const uint32_t trow = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tO = tmem + trow + hf * 128, tS = tmem + trow + 256 + hf * 128;
    // lanes 0-7: key scales of a block's 8 groups of 16 positions; 8-15: value exponents, -inf where
    // there is nothing to see; 16-23: 2^-those, 0
    auto scale_of = [&](int j) {
      float x = 0.f;
      if (lane < 24) {
        const int pos = j * PP_KEYS + (lane & 7) * 16, id = j < nblk ? page16(pos) : -1;
        const long long at = (((long long)max(id, 0) * H + h) * a.pool.page + (pos & (a.pool.page - 1))) / BLK;
        if (lane < 8) {
          x = id >= 0 ? a.pool.ks[at] : 0.f;
        } else {
          const uint32_t e = __float_as_uint(a.pool.vs[at]) >> 23;
          if (lane < 16) x = id >= 0 ? (float)((int)e - 127) : -INFINITY;
          else x = id >= 0 ? __uint_as_float((254u - e) << 23) : 0.f;
        }
      }
      return x;
    };
    const uint32_t scaleS = sb + L::OFF_SCALE + warp * 192;
    float scale = scale_of(0);
    for (int j = 0; j < nblk; ++j) {
      const uint32_t sc = scaleS + (j & 1) * 96;
      if (lane < 24) asm volatile("st.shared.f32 [%0], %1;" ::"r"(sc + 4 * lane), "f"(scale) : "memory");
      scale = scale_of(j + 1);
      if (!(ok = uniform(mbar_wait(bar(PB_S + hf), j & 1, a.err, ERR_WAIT)))) break;
      fence_after();
      const bool edge = (j + 1) * PP_KEYS - 1 > lim_lo;
      const int see = lim - j * PP_KEYS;                 // last column the row sees
      float v[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(tS + 32 * c, *reinterpret_cast<float(*)[32]>(v + 32 * c));
      tmem_wait_ld();
      if (edge) {
#pragma unroll
        for (int i = 0; i < 128; ++i)
          if (i > see) v[i] = -INFINITY;
      }
      float top = -INFINITY;
      float2 ks2, ev2, vi2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float* x = v + 16 * e;
        if (!(e & 1)) {
          ks2 = lds2(sc + 4 * e);
          ev2 = lds2(sc + 4 * (8 + e));
        }
        const float m0 = fmax3(x[0], x[1], x[2]), m1 = fmax3(x[3], x[4], x[5]), m2 = fmax3(x[6], x[7], x[8]);
        const float m3 = fmax3(x[9], x[10], x[11]), m4 = fmax3(x[12], x[13], x[14]);
        const float bm = fmaxf(fmax3(m0, m1, m2), fmax3(m3, m4, x[15]));
        top = fmaxf(top, fmaf(bm, rc * (e & 1 ? ks2.y : ks2.x), e & 1 ? ev2.y : ev2.x));
      }
      const bool move = top > m + PP_STEP;
      const float mn = move ? top : m;
      const float al = m == -INFINITY ? 0.f : ex2(m - mn);
      if (j > 0 && __any_sync(0xffffffffu, move)) {
        // PV_{j-1} has to be in O before O changes
        if (!(ok = uniform(mbar_wait(bar(PB_O + hf), (j - 1) & 1, a.err, ERR_WAIT)))) break;
        fence_after();
        const float f = move ? al : 1.f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          float o[32];
          tmem_ld32(tO + c * 32, o);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] *= f;
          tmem_st32(tO + c * 32, o);
        }
        tmem_wait_st();
      }
      if (move) l *= al;
      m = mn;
      const float base = m == -INFINITY ? 0.f : PP_OFF - m;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float hi[16], lo_[16];
        ks2 = lds2(sc + 8 * c);
        ev2 = lds2(sc + 32 + 8 * c);
        vi2 = lds2(sc + 64 + 8 * c);
#pragma unroll
        for (int e = 2 * c; e < 2 * c + 2; ++e) {
          const float cc = rc * (e & 1 ? ks2.y : ks2.x), add = (e & 1 ? ev2.y : ev2.x) + base;
          const uint64_t c2 = f2_pack(cc, cc), a2 = f2_pack(add, add);
          uint64_t s0 = 0ull, s1 = 0ull;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int at = 16 * e + 2 * i, k = 8 * (e & 1) + i;
            float x0, x1;
            f2_unpack(f2_fma(f2_pack(v[at], v[at + 1]), c2, a2), x0, x1);
            if (edge) {                                  // (-inf times a factor that is 0 is no -inf)
              if (at > see) x0 = -INFINITY;
              if (at + 1 > see) x1 = -INFINITY;
            }
            x0 = ex2(x0);
            x1 = ex2(x1);
            const uint32_t w = pack_h2(x0, x1);
            hi[k] = __uint_as_float(w);
            if (SPLIT) {
              const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&w));
              lo_[k] = __uint_as_float(pack_h2(x0 - b.x, x1 - b.y));
            }
            if (i & 1) s1 = f2_add(s1, f2_pack(x0, x1)); else s0 = f2_add(s0, f2_pack(x0, x1));
          }
          float x0, x1;
          f2_unpack(f2_add(s0, s1), x0, x1);
          l = fmaf(x0 + x1, e & 1 ? vi2.y : vi2.x, l);
        }
        tmem_st16(tS + 32 * c, hi);
        if (SPLIT) tmem_st16(tS + 32 * c + 16, lo_);
        if (c & 1) {
          tmem_wait_st();
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(PB_P + 2 * hf + (c >> 1)));
        }
      }
    }
    if (ok) ok = uniform(mbar_wait(bar(PB_O + hf), (nblk - 1) & 1, a.err, ERR_WAIT));
  }
  fence_before();
  __syncthreads();                                       // every product is done; shared memory is free
  fence_after();

  if (warp < PP_MMA_WARP && ok) {
    const uint32_t tO = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * 128;
    uint32_t any = 0;
    for (int i = 0; i < PP_NANW; ++i) any |= nanS[i];
    unsigned char* stage = smp + warp * L::OUT_WARP;
    const float inv = l == 0.f ? 0.f : 1.f / l;
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
            const int pos = nan0 + 32 * w + __ffs(bits) - 1, id = page16(pos);
            if (pos > lim || id < 0) continue;
            const unsigned char* p = a.pool.v + (((long long)id * H + h) * a.pool.page + (pos & (a.pool.page - 1))) * D + 32 * c;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if ((p[i] & 0x7f) == 0x7f) o[i] = __uint_as_float(0x7fffffffu);
          }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<float4*>(stage + lane * (4 * D) + (((c * 8 + i) ^ (lane & 7)) << 4)) =
            make_float4(o[4 * i] * inv, o[4 * i + 1] * inv, o[4 * i + 2] * inv, o[4 * i + 3] * inv);
    }
    const long long HQ = (long long)H * G;
    if (lim >= 0 && a.lse) {
      const int r = row0 + tid, tok = r / G;
      a.lse[(t.first + tok) * HQ + h * G + (r - tok * G)] =
          l == 0.f ? -INFINITY : (m - PP_OFF + log2f(l)) * 0.69314718055994530942f;
    }
    __syncwarp();
    constexpr int LPR = D / 4, RPI = 32 / LPR;           // whole rows leave, D / 4 lanes each
    for (int i = 0; i < 32; i += RPI) {
      const int rw = i + lane / LPR, cc = lane % LPR, r = row0 + warp * 32 + rw;
      if (warp * 32 + rw >= rows) break;
      const float4 v = *reinterpret_cast<const float4*>(stage + rw * (4 * D) + ((cc ^ (rw & 7)) << 4));
      const int tok = r / G;
      const long long row = (t.first + tok) * HQ + h * G + (r - tok * G);
      if (a.out_f32)
        reinterpret_cast<float4*>(a.out)[row * (D / 4) + cc] = v;
      else
        reinterpret_cast<uint2*>(a.out)[row * (D / 4) + cc] = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    }
  }
  fence_before();
  __syncthreads();
  if (warp == PP_MMA_WARP) tmem_dealloc(tmem, PP_TMEM);
}

template <int D, bool SPLIT>
cudaError_t launch(const PromptArgs& a, long long places, cudaStream_t stream) {
  auto k = paged_prompt_kernel<D, SPLIT>;
  const size_t smem = PL<D>::BYTES;
  static std::atomic<unsigned long long> raised{0};
  const cudaError_t e = raise_smem_limit_once(raised, k, smem);
  if (e != cudaSuccess) return e;
  k<<<(unsigned)(places * a.pool.H), PP_THREADS, smem, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

bool paged_prompt_fits(const Pool& pool, const Batch& b, int HQ) {
  return ((long long)b.n_tokens * (HQ / pool.H) / PP_ROWS + b.n_seq) * pool.H <= INT32_MAX;
}

cudaError_t launch_paged_prompt(const Pool& pool, const Batch& b, const void* q, long long q_ts, long long q_hs,
                                int HQ, void* out, int out_f32, float* lse, int32_t* err, cudaStream_t stream) {
  PromptArgs a{};
  a.pool = pool;
  a.b = b;
  a.q = static_cast<const bf16*>(q);
  a.q_ts = q_ts;
  a.q_hs = q_hs;
  a.out = out;
  a.out_f32 = out_f32;
  a.lse = lse;
  a.err = err;
  a.c = (float)(1.4426950408889634 / sqrt((double)pool.d));
  a.G = HQ / pool.H;
  const long long places = (long long)b.n_tokens * a.G / PP_ROWS + b.n_seq;
  if (pool.d == 128) return out_f32 ? launch<128, true>(a, places, stream) : launch<128, false>(a, places, stream);
  return out_f32 ? launch<64, true>(a, places, stream) : launch<64, false>(a, places, stream);
}

}  // namespace kvpop
