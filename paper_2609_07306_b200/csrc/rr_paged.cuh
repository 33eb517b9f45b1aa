// What the operators of the paged key/value cache share: checks of the cache's description, page lookup,
// the sequence of a token.
#pragma once
#include "rr_common.cuh"

constexpr int RR_PAGED_MAX_DH = 256;

inline int rr_paged_check(const rr_paged_kv* kv) {
  if (!kv || !kv->k || !kv->v || !kv->page_table) return RR_ERR_INVALID_ARG;
  if (kv->num_pages < 1 || kv->page_tokens < 1 || kv->kv_heads < 1 || kv->batch < 1 || kv->pages_per_seq < 1) return RR_ERR_INVALID_ARG;
  if (kv->page_stride < 0 || kv->head_stride < 0 || kv->token_stride < 0 || kv->table_stride < 0) return RR_ERR_INVALID_ARG;
  if (kv->dtype != RR_BF16 && kv->dtype != RR_F32) return RR_ERR_UNSUPPORTED;
  if (kv->dh < 1 || kv->dh > RR_PAGED_MAX_DH) return RR_ERR_UNSUPPORTED;
  const size_t e = kv->dtype == RR_BF16 ? 2 : 4;
  if ((((uintptr_t)kv->k | (uintptr_t)kv->v) & (e - 1)) || ((uintptr_t)kv->page_table & 3) || ((uintptr_t)kv->status & 3)) return RR_ERR_INVALID_ARG;
  return RR_OK;
}

// Whether two runs of bytes have none in common (an empty one, or one that is not given, has none).
inline bool rr_apart(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return !a || !b || na <= 0 || nb <= 0 || (x < y ? y - x >= (uint64_t)na : x - y >= (uint64_t)nb);
}

template <typename T> __device__ __forceinline__ float rr_to_f32(T x);
template <> __device__ __forceinline__ float rr_to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float rr_to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T rr_from_f32(float x);
template <> __device__ __forceinline__ float rr_from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 rr_from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// The sequence of new token t, the last b with cu[b] <= t; -1 for padding behind the last one.  Called by a
// converged warp: each round reads 32 evenly spaced entries, so that 1024 sequences take two dependent loads.
__device__ __forceinline__ int rr_sequence_of_warp(const int32_t* __restrict__ cu, int batch, int t) {
  const int lane = threadIdx.x & 31;
  if (t >= __ldg(cu + batch)) return -1;
  int lo = 0, n = batch;                               // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const bool le = lane * step < n && __ldg(cu + at) <= t;
    const unsigned votes = __ballot_sync(0xFFFFFFFFu, le);
    const int last = votes ? 31 - __clz(votes) : 0;    // ascending: the votes are a prefix
    n = min(step, n - last * step);
    lo += last * step;
  }
  return lo;
}
// The same for one thread.
__device__ __forceinline__ int rr_sequence_of(const int32_t* __restrict__ cu, int batch, int t) {
  if (t >= __ldg(cu + batch)) return -1;
  int lo = 0, hi = batch;
  while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (__ldg(cu + mid) <= t) lo = mid; else hi = mid; }
  return lo;
}
