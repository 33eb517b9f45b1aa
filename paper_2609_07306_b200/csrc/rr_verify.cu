// Verification of drafted tokens.
//
// Sampled:  draft x behind row t is accepted if p_t(x) > u_t q_t(x);  with a of n accepted, the token more is the first j with
//   sum_{i <= j} w_i > u sum_i w_i,   w = max(p_a - q_a, 0) for a < n, p_n for a = n;
//   the accepted tokens and the one more are then distributed as the target's own.
// Greedy:   draft x is accepted if it is the row's lowest best.
//
// Sampled, a step reads two numbers a draft and one row (two, if a draft was rejected) a sequence; greedy, all rows.  Bound by memory for
// batches, by latency for one sequence.
// Sampled: a cluster takes a sequence, each CTA a run of blocks of the vocabulary; which drafts are accepted every CTA
// finds for itself (a few dependent loads, instead of a barrier).  A warp reads a block of 256 entries at a time, eight per lane from each row, the next block's loads
// in front of this one's arithmetic, and leaves its lanes' sums; the CTAs exchange their totals, the one that has the threshold finds block and
// entry, so the row is read once but for that block.  Products, differences and sums are 64-bit: the first two are exact for probabilities of up
// to 24 bits, and a sum over the vocabulary is off by some 1e-14, so that a random number falls between two results about never.  For 64 sequences
// against 131071 tokens (49 MB) two conversions, two selections and two 64-bit sums an entry are, by their number, some 2 us; the rest is the rows, an uneven end (one row or two for
// the same CTAs) and the search behind them.
// (Rings of blocks in shared memory, filled by bulk copies: 27 us; fewer warps fit, and each has its chain of 64-bit sums.)
// Greedy: a cluster takes a row, whoever's it is (sequences with many drafts would hold up the others), 16 bytes at a time where rows
// allow it; only maxima are taken (a packed maximum of two bf16 costs one instruction), a thread keeps its first best vector, and the entry inside it is looked
// up at the end.  The rows' best tokens go to `out`, where a second kernel, a warp per sequence, compares them with the drafts.
// Measured: those 64 sequences 15.9 us, 20.1 from memory, in bf16 15.0 and 17.2, without the draft's probabilities 13.8 and 16.5; one sequence against 32768 tokens 6.4 us; greedy, 415 rows of 131072 in bf16 (109 MB) 22 us
// from memory, 36 us where rows do not lie on 16 bytes.  The sampled kernel has 64 registers, for four CTAs an SM, and spills 56 bytes (bf16: 16).
#include <cooperative_groups.h>
#include <utility>
#include "rr_paged.cuh"

namespace cg = cooperative_groups;

namespace {

// The kernels may be launched before the one in front of them has ended (rr_launch_pdl), so nothing is read by way of the read-only path.  Behind
// its wait every CTA reads the same few numbers in the beginning: through L1 (all from L2: 2 us more).

constexpr int NT = 256, NW = NT / 32, BLOCK = 256, MAX_CL = 8;
constexpr int SUMS = 64;                                // blocks' sums that a CTA keeps

struct Span { int first, n; };                          // a sequence's first row, its drafts (-1: it has no rows)

template <bool L2 = false> __device__ __forceinline__ int load(const int32_t* p) { return L2 ? __ldcg(p) : *p; }
template <bool L2 = false>
__device__ __forceinline__ Span span_of(const rr_verify_args& a, int b) {
  const int first = a.cu ? max(load<L2>(a.cu + b), 0) : b, end = a.cu ? min(load<L2>(a.cu + b + 1), a.rows) : b + 1;
  return Span{first, max(end - first, 0) - 1};
}

// Probabilities are positive and finite (bits 1 to those of the largest number), or 0.
__device__ __forceinline__ float weight(float x) { return __float_as_uint(x) - 1u < 0x7F7FFFFFu ? x : 0.f; }
template <typename T>
__device__ __forceinline__ double probability(const void* rows, int64_t stride, int row, int x) {
  return weight(rr_to_f32(((const T*)rows)[row * stride + x]));
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
  return x;
}
__device__ __forceinline__ void write_lengths(const rr_verify_args& a, int b, const Span& s, int accepted, int len) {
  if (a.room && s.n >= 0 && (long long)len + s.n + 1 > a.room[b]) accepted = -1;       // (its rows are not in the cache)
  a.accepted[b] = accepted;
  if (a.new_lens) a.new_lens[b] = len + (s.n < 0 ? 0 : accepted + 1);
}
// A sequence's results but the token behind the accepted drafts.
__device__ __forceinline__ void write_accepted(const rr_verify_args& a, int b, const Span& s, int accepted) {
  const int lane = threadIdx.x & 31;
  for (int i = lane; i <= s.n; i += 32)
    if (i != accepted) a.out[s.first + i] = i < accepted ? a.tokens[s.first + i + 1] : -1;
  if (lane == 0) write_lengths(a, b, s, accepted, a.new_lens || a.room ? a.lens[b] : 0);
}

// A drafted token is in the vocabulary.
__device__ __forceinline__ bool in_vocab(const rr_verify_args& a, int x) {
  const bool ok = x >= 0 && x < a.vocab;
  if (!ok && a.status) atomicOr(a.status, RR_STATUS_BAD_INDEX);
  return ok;
}

// ---- sampled ----------------------------------------------------------------------------------------------------
// max(p - q, 0) of an entry, 0 if it is left out.
__device__ __forceinline__ double weight_of(float p, float q, bool out) {
  const float x = weight(p), y = weight(q);
  return x > y && !out ? (double)x - (double)y : 0.0;
}
// The lane's eight of a block, without the entry `but`.
template <typename T>
__device__ __noinline__ double one_by_one(const T* prow, const T* qrow, int vocab, int first, int but) {
  double s = 0.0;
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    const int j = first + (int)(threadIdx.x & 31) + 32 * i;
    if (j < vocab) s += weight_of(rr_to_f32(prow[j]), qrow ? rr_to_f32(qrow[j]) : 0.f, j == but);
  }
  return s;
}

// A block of a row of the target's and of one of the draft's (0 where there is none): entries first + lane + 32 i.
template <typename T> struct Block {
  T p[8], q[8];
  __device__ __forceinline__ void load(const T* prow, const T* qrow, int vocab, int first) {
    const int j0 = first + (threadIdx.x & 31);
    if (first + BLOCK <= vocab) {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = prow[j0 + 32 * i];
      if (qrow) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = qrow[j0 + 32 * i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = j0 + 32 * i < vocab;
        p[i] = in ? prow[j0 + 32 * i] : rr_from_f32<T>(0.f);
        q[i] = in && qrow ? qrow[j0 + 32 * i] : rr_from_f32<T>(0.f);
      }
    }
  }
  // The sum of the lane's eight weights, in 64 bits throughout.  With z = max(x, y) the weight is z - y: 0 where x - y is below 0 or x is NaN.
  // An infinite number makes a sum that is none, and the eight are looked at one by one, as are those of the block with `but`.  (One conversion an entry instead of
  // two, of the difference rounded to FP32, with its rest added in FP32: sums of eight off by up to 7e-15, and slower, 17.1 against 15.9 us for 64 sequences of 131071.)
  __device__ __forceinline__ double sum(const T* prow, const T* qrow, int vocab, int first, int but) const {
    double s[2] = {0.0, 0.0};
    if (qrow) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = fmaxf(rr_to_f32(q[i]), 0.f), z = fmaxf(rr_to_f32(p[i]), y);
        s[i & 1] += (double)z - (double)y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i & 1] += (double)fmaxf(rr_to_f32(p[i]), 0.f);
    }
    const double all = s[0] + s[1];
    return !isfinite(all) || (but >= first && but < first + BLOCK) ? one_by_one(prow, qrow, vocab, first, but) : all;
  }
};

struct Found { double lanes[SUMS][33]; double sums[SUMS]; double total; };

// Of a warp's 32 weights the first whose running sum, from `run` on, is over `limit`, else the last one that is not 0 (at = 32: none is).
struct Hit { int at; bool over; double before, end; };  // the sums before it and behind all
__device__ __noinline__ Hit find(double w, double run, double limit) {
  const int lane = threadIdx.x & 31;
  double upto = w;
#pragma unroll 1
  for (int d = 1; d < 32; d *= 2) { const double y = __shfl_up_sync(0xFFFFFFFFu, upto, d); if (lane >= d) upto += y; }
  upto += run;
  const unsigned over = __ballot_sync(0xFFFFFFFFu, w > 0.0 && upto > limit), some = __ballot_sync(0xFFFFFFFFu, w > 0.0);
  Hit h;
  h.at = over ? __ffs(over) - 1 : some ? 31 - __clz(some) : 32;
  h.over = over != 0;
  h.before = __shfl_sync(0xFFFFFFFFu, upto - w, h.at & 31);
  h.end = __shfl_sync(0xFFFFFFFFu, upto, 31);
  return h;
}

template <typename T>
__global__ void __launch_bounds__(NT, 4)
verify_sampled_kernel(const __grid_constant__ rr_verify_args a) {
  __shared__ Found f;
  cg::cluster_group cl = cg::this_cluster();
  const int ctas = cl.num_blocks(), cta = cl.block_rank(), b = blockIdx.x / ctas;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  rr_pdl_wait();
  rr_pdl_trigger();
  const Span s = span_of(a, b);
  if (s.n < 0) {                                        // (uniform in the cluster)
    if (cta == 0 && warp == 0) write_accepted(a, b, s, 0);
    return;
  }
  // which drafts are accepted: every warp for itself
  const double u = fmax((double)a.uniform[s.first + s.n], 0.0);
  int accepted = 0;
  for (int i0 = 0; i0 < s.n; i0 += 32) {
    const int i = i0 + lane, t = s.first + i;
    bool ok = true;
    if (i < s.n) {
      const int x = a.tokens[t + 1];
      const double r = a.uniform[t];
      ok = in_vocab(a, x);
      if (ok) {
        const double p = probability<T>(a.target, a.target_stride, t, x), q = a.draft ? probability<T>(a.draft, a.draft_stride, t, x) : 1.0;
        ok = p > r * q;
      }
    }
    const unsigned rejected = __ballot_sync(0xFFFFFFFFu, !ok);
    if (rejected) { accepted = i0 + __ffs(rejected) - 1; break; }
    accepted = min(i0 + 32, s.n);
  }
  if (cta == 0 && warp == NW - 1) write_accepted(a, b, s, accepted);
  const int row = s.first + accepted;
  const T* const p = (const T*)a.target + row * a.target_stride;
  const T* q = nullptr;
  int but = -1;
  if (accepted < s.n) {
    if (a.draft) q = (const T*)a.draft + row * a.draft_stride;
    else but = a.tokens[row + 1];
  }
  // blocks of this CTA; a kept sum stands for `per` of them
  const int blocks = (a.vocab + BLOCK - 1) / BLOCK, share = (blocks + ctas - 1) / ctas, from = min(cta * share, blocks), mine = min(share, blocks - from);
  const int per = (share + SUMS - 1) / SUMS, sums = (mine + per - 1) / per;
  int token = -1;
  bool here = false, none = false;
  for (int pass = 0; pass < 2; ++pass) {
    Block<T> now, next;
    int k = warp, i = warp * per;                       // kept sum and block
    double sum = 0.0;
    if (k < sums) now.load(p, q, a.vocab, (from + i) * BLOCK);
    while (k < sums) {
      const int at = (from + i) * BLOCK;
      const bool last = i + 1 >= min((k + 1) * per, mine);
      const int k_next = last ? k + NW : k, i_next = last ? k_next * per : i + 1;
      if (k_next < sums) next.load(p, q, a.vocab, (from + i_next) * BLOCK);
      sum += now.sum(p, q, a.vocab, at, but);
      if (last) {
        f.lanes[k][lane] = sum;
        sum = 0.0;
      }
      now = next;
      k = k_next;
      i = i_next;
    }
    __syncthreads();
    {                                                   // four threads add up a kept sum's lanes
      const int k = threadIdx.x / 4, part = threadIdx.x & 3;
      double x = 0.0;
      if (k < sums)
        for (int i = 0; i < 8; ++i) x += f.lanes[k][8 * part + i];
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
      if (part == 0) f.sums[k] = x;
    }
    __syncthreads();
    if (warp == 0) {
      const double x = warp_sum(f.sums[lane] + f.sums[lane + 32]);
      if (lane == 0) f.total = x;
    }
    cl.sync();
    // every warp finds the CTA that has the threshold
    const double theirs = lane < ctas ? *cl.map_shared_rank(&f.total, lane) : 0.0;
    const double limit = u * warp_sum(theirs);
    auto read = cl.barrier_arrive();                    // (each CTA waits for the others to have read its total before it ends or writes another one)
    Hit h = find(theirs, 0.0, limit);
    if (h.at == 32) {                                   // no weight: the rejected row has no more than the draft's anywhere
      none = !q && but < 0;
      cl.barrier_wait(std::move(read));
      if (none) break;
      q = nullptr;
      but = -1;
      continue;
    }
    here = h.at == cta;
    if (!here || warp != 0) {
      cl.barrier_wait(std::move(read));
      break;
    }
    // the kept sum (two lie side by side in a lane), then the block, then the entry
    static_assert(SUMS == 64, "two per lane");
    h = find(f.sums[2 * lane] + f.sums[2 * lane + 1], h.before, limit);
    k = 2 * h.at;
    double run = h.before;
    const double first = f.sums[k], second = f.sums[k + 1];
    if (!(first > 0.0 && (run + first > limit || !(second > 0.0)))) ++k, run += first;
    h.over = false;
#pragma unroll 1
    for (int i = k * per; i < min((k + 1) * per, mine) && !h.over; ++i) {
      const int at = (from + i) * BLOCK;
      now.load(p, q, a.vocab, at);
#pragma unroll
      for (int e = 0; e < 8; ++e) f.lanes[e][lane] = weight_of(rr_to_f32(now.p[e]), q ? rr_to_f32(now.q[e]) : 0.f, at + lane + 32 * e == but);
      __syncwarp();
      double x = 0.0;                                   // four lanes add up 32 entries, then these
#pragma unroll
      for (int e = 0; e < 8; ++e) x += f.lanes[lane / 4][8 * (lane & 3) + e];
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
      h = find((lane & 3) ? 0.0 : x, run, limit);
      run = h.end;
      if (h.at < 32) {
        const int e = h.at / 4;
        token = at + 32 * e + find(f.lanes[e][lane], h.before, limit).at;
      }
      __syncwarp();
    }
    cl.barrier_wait(std::move(read));
    break;
  }
  // the CTA that has the token, or the first one where all weights are 0
  if (threadIdx.x == 0 && (here || (none && cta == 0))) a.out[row] = token;
}

// ---- greedy -----------------------------------------------------------------------------------------------------
// Larger keys are larger scores, equal keys equal scores; 0: NaN.
__device__ __forceinline__ uint32_t score_key(float x) { return x == x ? rr_order_key(x) : 0u; }

template <typename T, int VEC> struct Vec;
template <> struct Vec<float, 4> {
  float4 v;
  __device__ __forceinline__ float best() const { return fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)); }
};
template <> struct Vec<__nv_bfloat16, 8> {
  __nv_bfloat162 v[4];
  __device__ __forceinline__ float best() const {       // (a maximum with one NaN is the other number)
    const __nv_bfloat162 m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
};
template <typename T> struct Vec<T, 1> {
  T v;
  __device__ __forceinline__ float best() const { return rr_to_f32(v); }
};

struct Best { uint32_t key; int at; };

// The largest key of the warp, the lowest place of several.
__device__ __forceinline__ Best warp_best(Best x) {
  const uint32_t key = __reduce_max_sync(0xFFFFFFFFu, x.key);
  return Best{key, __reduce_min_sync(0xFFFFFFFFu, x.key == key ? x.at : INT32_MAX)};
}

// The best token of each row, -1 where all scores are NaN.
template <typename T, int VEC>
__global__ void __launch_bounds__(NT)
best_kernel(const __grid_constant__ rr_verify_args a) {
  __shared__ Best s_warp[NW], s_cta;
  cg::cluster_group cl = cg::this_cluster();
  const int ctas = cl.num_blocks(), cta = cl.block_rank(), t = blockIdx.x / ctas;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  rr_pdl_wait();
  rr_pdl_trigger();
  if (a.cu && t >= a.cu[a.batch]) return;       // padding (uniform in the cluster)
  using V = Vec<T, VEC>;
  const int vecs = a.vocab / VEC, share = (vecs + ctas - 1) / ctas, from = min(cta * share, vecs), to = min(from + share, vecs);
  const T* const row = (const T*)a.target + t * a.target_stride;
  Best x{0u, INT32_MAX};
#pragma unroll 8
  for (int v = from + threadIdx.x; v < to; v += NT) {
    V e;
    if constexpr (VEC == 1) e.v = row[v];
    else { const uint4 raw = ((const uint4*)row)[v]; e = *(const V*)&raw; }
    const uint32_t key = score_key(e.best());
    if (key > x.key) x = Best{key, v};
  }
  if (cta == ctas - 1 && threadIdx.x == 0)              // the entries behind the last vector
    for (int j = vecs * VEC; j < a.vocab; ++j)
      if (const uint32_t key = score_key(rr_to_f32(row[j])); key > x.key) x = Best{key, vecs};
  x = warp_best(x);
  if (lane == 0) s_warp[warp] = x;
  __syncthreads();
  if (warp == 0) {
    x = warp_best(lane < NW ? s_warp[lane] : Best{0u, INT32_MAX});
    // the first entry of the vector that is as good
    const int j = x.key ? x.at * VEC + lane : 0;
    const unsigned same = __ballot_sync(0xFFFFFFFFu, x.key && lane < VEC && j < a.vocab && score_key(rr_to_f32(row[j])) == x.key);
    if (lane == 0) s_cta = Best{x.key, x.key ? x.at * VEC + __ffs(same) - 1 : INT32_MAX};
  }
  cl.sync();
  if (cta == 0 && warp == 0) {
    x = warp_best(lane < ctas ? *cl.map_shared_rank(&s_cta, lane) : Best{0u, INT32_MAX});
    if (lane == 0) a.out[t] = x.key ? x.at : -1;
  }
  cl.sync();                                            // no CTA leaves before its best has been read
}

// The drafts against the rows' best tokens, which are in `out`: up to the first that differs they are the accepted tokens and the one more.  Launched along with
// best_kernel, which starts it when all before itself has ended, so only `out` has to be waited for.  What is read in front of the wait comes by way of L2, where the ended
// kernels have left it; that L1 holds nothing older is certain behind the wait only.
__global__ void __launch_bounds__(128)
compare_kernel(const __grid_constant__ rr_verify_args a) {
  const int lane = threadIdx.x & 31, b = blockIdx.x * 4 + (threadIdx.x >> 5);
  const bool mine = b < a.batch;
  const Span s = mine ? span_of<true>(a, b) : Span{0, -1};
  int x = lane < s.n ? load<true>(a.tokens + s.first + lane + 1) : 0;
  const int len = mine && (a.new_lens || a.room) ? load<true>(a.lens + b) : 0;
  rr_pdl_wait();
  rr_pdl_trigger();
  if (!mine) return;
  int accepted = max(s.n, 0);
  for (int i0 = 0; i0 < s.n; i0 += 32) {
    const int i = i0 + lane;
    bool ok = true;
    if (i < s.n) {
      if (i0 > 0) x = a.tokens[s.first + i + 1];
      ok = in_vocab(a, x) && x == __ldcg(a.out + s.first + i);
    }
    const unsigned rejected = __ballot_sync(0xFFFFFFFFu, !ok);
    if (rejected) { accepted = i0 + __ffs(rejected) - 1; break; }
  }
  for (int i = accepted + 1 + lane; i <= s.n; i += 32) a.out[s.first + i] = -1;
  if (lane == 0) write_lengths(a, b, s, accepted, len);
}

// CTAs that share each of `n` things (sequences, rows) of `work` entries: at most eight, no less than `least` entries for one, and no more than per_sm in all for an
// SM (415 rows of 131072: one CTA a row 21.8 us, two 17.4, four 23.3, of which the last ones wait for places; 6 rows: 9.2, 6.7, 5.5).  Four CTAs of the sampled kernel
// run on an SM; of the greedy kernel's vector builds six (34 registers), while per_sm is eight, as for the others: between 112 and 148, 223 and 296, 445 and 592 rows
// some CTAs wait (440 rows 22.7 us, 500 30.7).
int cluster_of(int n, int work, int least, int per_sm) {
  int c = MAX_CL;
  while (c > 1 && (work < c * least || (int64_t)n * c > per_sm * rr_sm_count())) c /= 2;
  return c;
}

cudaError_t launch(void (*kernel)(rr_verify_args), const rr_verify_args& a, int n, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)(n * cluster)); cfg.blockDim = dim3(NT);
  cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 2;
  rr_count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

int done(cudaError_t e) { return e == cudaSuccess ? RR_OK : rr_cuda_fail(e, "rr_verify_drafts"); }

}  // namespace

extern "C" int rr_verify_drafts(const rr_verify_args* a, void* stream) {
  if (!a || !a->out || !a->accepted || !a->tokens || (!a->target && a->rows > 0)) return RR_ERR_INVALID_ARG;
  if (a->rows < 0 || a->batch < 1 || a->vocab < 1 || (!a->cu && a->rows != a->batch)) return RR_ERR_INVALID_ARG;
  if (a->target_stride < 0 || a->draft_stride < 0 || ((a->new_lens || a->room) && !a->lens) || (a->draft && !a->uniform)) return RR_ERR_INVALID_ARG;
  if (a->dtype != RR_BF16 && a->dtype != RR_F32) return RR_ERR_UNSUPPORTED;
  if (a->vocab > (1 << 30) || a->batch > (1 << 27)) return RR_ERR_TOO_LARGE;
  const uintptr_t e = a->dtype == RR_BF16 ? 1 : 3;
  if ((((uintptr_t)a->target | (uintptr_t)a->draft) & e) ||
      (((uintptr_t)a->tokens | (uintptr_t)a->cu | (uintptr_t)a->uniform | (uintptr_t)a->lens | (uintptr_t)a->out | (uintptr_t)a->accepted |
        (uintptr_t)a->new_lens | (uintptr_t)a->status | (uintptr_t)a->room) & 3)) return RR_ERR_INVALID_ARG;
  // Results are written while inputs are read.  (A sequence's length is read by the thread that writes its results: these may take its place.)
  const bool bf16 = a->dtype == RR_BF16;
  const int64_t rows = 4 * (int64_t)a->rows, row = 4 * (int64_t)a->batch, entry = bf16 ? 2 : 4;
  const struct { const void* p; int64_t n; } results[] = {{a->out, rows}, {a->accepted, row}, {a->new_lens, row}},
    inputs[] = {{a->tokens, rows}, {a->cu, row + 4}, {a->uniform, rows}, {a->lens, row}, {a->room, row}, {a->status, 4},
                {a->target, a->rows > 0 ? entry * ((a->rows - 1) * a->target_stride + a->vocab) : 0},
                {a->draft, a->rows > 0 ? entry * ((a->rows - 1) * a->draft_stride + a->vocab) : 0}};
  for (int i = 0; i < 3; ++i) {
    for (const auto& in : inputs)
      if (!(in.p == a->lens && results[i].p == a->lens && i > 0) && !rr_apart(results[i].p, results[i].n, in.p, in.n)) return RR_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (!rr_apart(results[i].p, results[i].n, results[j].p, results[j].n)) return RR_ERR_INVALID_ARG;
  }
  cudaStream_t st = (cudaStream_t)stream;
  if (a->uniform) {
    const int cluster = cluster_of(a->batch, a->vocab, NW * BLOCK, 4);
    return done(launch(bf16 ? verify_sampled_kernel<__nv_bfloat16> : verify_sampled_kernel<float>, *a, a->batch, cluster, st));
  }
  const int ctas = (a->batch + 3) / 4;
  if (a->rows == 0) {                                   // (nothing to be launched along with)
    rr_count_launch();
    compare_kernel<<<ctas, 128, 0, st>>>(*a);
    return done(cudaPeekAtLastError());
  }
  const bool vec = ((uintptr_t)a->target & 15) == 0 && (a->target_stride * (bf16 ? 2 : 4)) % 16 == 0;
  auto* const kernel = bf16 ? (vec ? best_kernel<__nv_bfloat16, 8> : best_kernel<__nv_bfloat16, 1>) : (vec ? best_kernel<float, 4> : best_kernel<float, 1>);
  if (const cudaError_t e = launch(kernel, *a, a->rows, cluster_of(a->rows, a->vocab, NT * 32, 8), st); e != cudaSuccess) return done(e);
  rr_count_launch();
  return done(rr_launch_pdl(compare_kernel, ctas, 128, 0, st, *a));
}
