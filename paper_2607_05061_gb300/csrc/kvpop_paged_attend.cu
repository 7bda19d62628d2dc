// Attention over the paged 8-bit cache: launches of the kernel for few rows, beside the one for many.
#include "kvpop_paged_attend.cuh"

namespace kvpop {
namespace {

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
    return nt == 1 ? launch_attend<D, 1, D == 64 ? 8 : 6, true, false>(a, grid, stream) : nt == 2 ? launch_attend<D, 2, 4, true, false>(a, grid, stream)
                                                            : launch_attend<D, 3, 4, true, false>(a, grid, stream);
  return nt == 1 ? launch_attend<D, 1, D == 64 ? 8 : 6, false, false>(a, grid, stream) : nt == 2 ? launch_attend<D, 2, 6, false, false>(a, grid, stream)
         : nt == 3 ? launch_attend<D, 3, 4, false, false>(a, grid, stream) : launch_attend<D, 4, 4, false, false>(a, grid, stream);
}

}  // namespace

// [counters here][there] [partial results here][there]
size_t paged_attend_parts(int sms) { return counter_bytes(sms) + paged_prompt_counters(sms); }
// The weights' counters and sums lie in the same places.
static_assert(AT_CTAS * 8 >= (int)sizeof(int), "a counter an SM");
size_t paged_attend_workspace(int sms) {
  return paged_attend_parts(sms) + std::max(part_bytes(sms) + paged_prompt_parts(sms), paged_weigh_workspace(sms));
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
