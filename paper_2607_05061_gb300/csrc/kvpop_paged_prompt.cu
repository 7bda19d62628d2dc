// Attention of many new tokens a sequence over the paged 8-bit cache: launches of the tcgen05 kernel.
#include "kvpop_paged_prompt.cuh"

namespace kvpop {

using namespace paged;

bool paged_prompt_fits(const Pool& pool, const Batch& b, int HQ) {
  return ((long long)b.n_tokens * (HQ / pool.H) / PP_ROWS + b.n_seq) * pool.H <= INT32_MAX;
}
// [parts there][claims]; [sums of parts][their bases and normalisers][running sums]
size_t paged_prompt_counters(int sms) { return ((size_t)(slots_of(sms) + sms) * 4 + 255) / 256 * 256; }
size_t paged_prompt_parts(int sms) { return (size_t)slots_of(sms) * PP_ROWS * (128 + 2) * 4 + (size_t)sms * PP_ROWS * 128 * 4; }

cudaError_t launch_paged_prompt(const Pool& pool, const Batch& b, const void* q, long long q_ts, long long q_hs,
                                int HQ, void* out, int out_f32, float* lse, void* counters, void* parts, int sms,
                                int32_t* err, cudaStream_t stream) {
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
  a.sms = sms;
  a.count = static_cast<int*>(counters);
  a.part = static_cast<float*>(parts);
  a.part_ml = reinterpret_cast<float2*>(a.part + slots_of(sms) * PP_ROWS * pool.d);
  a.sum = a.part + slots_of(sms) * PP_ROWS * (pool.d + 2);
  a.claim = a.count + slots_of(sms);
  // Tiles are cut where there may be too few of them for the SMs; the most there can be counts, as
  // the lengths are not known here.
  const long long most = ((long long)b.n_tokens * a.G / PP_ROWS + b.n_seq) * pool.H, cuts = slots_of(sms) / most;
  const dim3 grid((unsigned)most, (unsigned)(cuts < 1 ? 1 : cuts < PP_PARTS ? cuts : PP_PARTS));
  // what the table has room for bounds the blocks of a tile
  const bool chained = ((long long)b.max_pages << pool.page_shift) > PP_CHAIN_BF16 * PP_KEYS;
  if (pool.d == 128)
    return out_f32 ? launch_prompt<128, true, true, false>(a, grid, stream)
           : chained ? launch_prompt<128, false, true, false>(a, grid, stream) : launch_prompt<128, false, false, false>(a, grid, stream);
  return out_f32 ? launch_prompt<64, true, true, false>(a, grid, stream)
         : chained ? launch_prompt<64, false, true, false>(a, grid, stream) : launch_prompt<64, false, false, false>(a, grid, stream);
}

}  // namespace kvpop
