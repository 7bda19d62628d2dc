// Paged 8-bit key/value cache: what its kernels share.
//
// A page holds `page` consecutive positions of one sequence for every KV head, keys and values
// apart: [n_pages][H][page][d] e4m3 bytes.  A block is 16 consecutive positions; each (block, KV
// head) has one scale for its keys and one for its values, [n_pages][H][page / 16] fp32, always a
// power of two 2^e with e in [-96, 100].  e4m3 has the same relative precision at every scale, so
// a power of two costs nothing against amax / 448, and products by scales are exact.
#pragma once

#include <cuda_fp16.h>

#include <atomic>

#include "kvpop_internal.cuh"
#include "kvpop_mma.cuh"

namespace kvpop {
namespace paged {

constexpr int BLK = 16;                // positions that share a scale
constexpr int E_MIN = -96;             // smallest scale exponent
constexpr float VALUE_LIMIT = 3.2451855e32f;   // 2^108: from here on a value is stored as NaN
enum : int {
  ERR_PAGE = 41,                       // a page number outside the pool, or a position past the table
  ERR_BATCH = 42,                      // token offsets that are not ascending, or more than max_new tokens
  ERR_ROTATION = 43,                   // a position past the rotation table
  ERR_WAIT = 44,                       // a wait for a copy, a product or a row ran out
};

struct Batch {                         // kvpop_paged_batch
  const int32_t* table;                // [n_seq] rows of max_pages page numbers, table_stride apart
  const int32_t* lens;                 // [n_seq] tokens held before the new ones, -1: idle
  const int32_t* starts;               // [n_seq + 1] first new token of each sequence, or null: one each
  long long table_stride;
  int max_pages, n_seq, n_tokens, max_new;
};

struct Pool {                          // kvpop_paged_pool
  unsigned char *k, *v;
  float *ks, *vs;
  int n_pages, H, d, page, page_shift;
};

__device__ __forceinline__ void report(int32_t* err, int code) {
  if (err) atomicCAS(err, 0, code);
}

// New tokens of a sequence: first, first + n are rows of the batch's token tensors whatever
// `starts` holds.
struct SeqTokens {
  int first, n, len;
};
__device__ __forceinline__ SeqTokens seq_tokens(const Batch& b, int s, int32_t* err) {
  SeqTokens t;
  t.len = b.lens[s];
  if (b.starts == nullptr) {
    t.first = s;
    t.n = 1;
  } else {
    const int a = b.starts[s], e = b.starts[s + 1];
    t.first = min(max(a, 0), b.n_tokens);
    t.n = max(min(e, b.n_tokens) - t.first, 0);
    if (a < 0 || e < a || e > b.n_tokens) report(err, ERR_BATCH);
  }
  return t;
}

// Page of a sequence's position `pos` (pos / page below max_pages); -1, recorded, if it is none.
__device__ __forceinline__ int page_of(const Batch& b, const Pool& p, int s, int pos, int32_t* err) {
  const int id = b.table[(long long)s * b.table_stride + (pos >> p.page_shift)];
  if ((unsigned)id < (unsigned)p.n_pages) return id;
  report(err, ERR_PAGE);
  return -1;
}

// Positions a sequence's tokens see at most, as far as its row of the table reaches.
__device__ __forceinline__ int context(const Batch& b, const Pool& p, const SeqTokens& t, int32_t* err) {
  const long long all = t.len < 0 ? 0 : (long long)t.len + t.n;
  const long long cap = min((long long)b.max_pages << p.page_shift, (long long)(INT32_MAX - 1024));
  if (all > cap) report(err, ERR_PAGE);
  return (int)min(all, cap);
}

// Last position that token `tok` of a sequence sees, -1 if none, for any length (len + tok may pass an int).
__device__ __forceinline__ int last_seen(int len, int tok, int ctx) {
  return (int)min((unsigned)len + 1u + (unsigned)tok, (unsigned)ctx) - 1;
}

// Whether a sequence's rows go to the tcgen05 kernel, where one is launched.  us by the rows (4 query
// heads), the kernel for few rows / tcgen05: 16 sequences of 10000 positions and 4 KV heads, d = 128, fp32
// results 32: 79 / 203, 64: 139 / 202, 80: 166 / 203, 96: 197 / 203; bf16 48: 88 / 135, 64: 106 / 136,
// 80: 142 / 137; 64 of 4000 and 8 heads fp32 48: 328 / 447, 64: 430 / 445, 80: 533 / 449; bf16 48: 248 / 295,
// 64: 298 / 292, 80: 428 / 294; d = 64 fp32 64: 324 / 296, bf16 48: 173 / 202, 64: 203 / 201.  4 of 2000 lie
// within 40 us either way.
constexpr int LONG_ROWS = 64;
__device__ __forceinline__ bool long_rows(const SeqTokens& t, int G) {
  return t.len >= 0 && (long long)t.n * G > LONG_ROWS;
}

// The attention kernels keep two things of a row's positions, with x_t the logit (times log2 e), 2^ev_t
// the scale of the position's values and M a base no less than the largest x + ev so far but for 2^8:
//   w_t = 2^(x_t - M + 2), whose sum is l, and p_t = w_t 2^(ev_t + 5) <= 2^15, the operand of O = sum p_t code_t;
//   y = O / (32 l),  lse = (M - 2 + log2 l) log 2.
// The scale is multiplied into p and stays out of w: the weight of a position counts whatever its values
// are (zeros have the smallest scale, 2^-96).  With 2^E the scale of the values that M came from, l lies
// between 2^(2 - E) and 2^(10 - E) for each position: with E between -96 and 100 it is a float for 2^21
// positions, and no weight above 2^-28 of the row's largest falls below 2^-126.
constexpr float W_OFF = 2.f, P_SCALE = 32.f, BASE_STEP = 8.f;
// Bases of sums to be joined may lie further apart (up to 196) than one factor reaches, while the weights
// they stand for are alike: 2^d as two factors.  No base (-inf) gives 0, two of them a factor for zeros.
__device__ __forceinline__ float2 down2(float d) {
  return make_float2(ex2(fmaxf(d, -90.f)), ex2(fminf(d + 90.f, 0.f)));
}

// raise_smem_limit once per device (`done`: one bit each, of one kernel): it takes longer on the
// host than a launch.
template <typename K>
inline cudaError_t raise_smem_limit_once(std::atomic<unsigned long long>& done, K* func, size_t need) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = raise_smem_limit(func, need);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

}  // namespace paged

cudaError_t launch_paged_append(const paged::Pool& pool, const paged::Batch& b, const void* q, long long q_ts,
                                long long q_hs, int HQ, const void* k, long long k_ts, long long k_hs,
                                const void* v, long long v_ts, long long v_hs, int dtype, const float* cos_,
                                const float* sin_, int rot, int max_pos, int interleaved, void* q_out,
                                int32_t* err, cudaStream_t stream);

// Bytes of the attention's workspace on a device with that many SMs.  The counters at its start have
// to be zero before the first call and are zero after every call.
size_t paged_attend_workspace(int sms);
cudaError_t launch_paged_attend(const paged::Pool& pool, const paged::Batch& b, const void* q, long long q_ts,
                                long long q_hs, int HQ, void* out, int out_f32, float* lse, void* workspace,
                                int sms, int32_t* err, cudaStream_t stream);

// The same for sequences with long_rows, where paged_prompt_fits.  Its share of the workspace:
// counters (zero between calls) and partial results.
bool paged_prompt_fits(const paged::Pool& pool, const paged::Batch& b, int HQ);
size_t paged_prompt_counters(int sms);
size_t paged_prompt_parts(int sms);
cudaError_t launch_paged_prompt(const paged::Pool& pool, const paged::Batch& b, const void* q, long long q_ts,
                                long long q_hs, int HQ, void* out, int out_f32, float* lse, void* counters,
                                void* parts, int sms, int32_t* err, cudaStream_t stream);

}  // namespace kvpop
