// Verification of drafted tokens.
//
// Sampled:  draft x behind row t is accepted if p_t(x) > u_t q_t(x);  with a of n accepted, the token more is the first j with
//   sum_{i <= j} w_i > u sum_i w_i,   w = max(p_a - q_a, 0) for a < n, p_n for a = n;
//   the accepted tokens and the one more are then distributed as the target's own.
// Greedy:   draft x is accepted if it is the row's lowest best.
//
// Sampled, a step reads two numbers a draft and one row (two, if a draft was rejected) a sequence; greedy, all rows.  Bound by memory for
// batches, by latency for one sequence.  A cluster takes a sequence, each CTA a run of blocks of the vocabulary; which drafts are accepted every CTA
// finds for itself (a few dependent loads, instead of a barrier).  Sampled: a warp adds up a block of 256 entries at a time, eight per lane in
// flight from each row, and leaves the block's sum; the CTAs exchange their sums, the one that has the threshold finds block and entry, so the row is
// read once but for that block.  Products, differences and sums are 64-bit: the first two are exact for probabilities of up to 24 bits,
// and a sum over the vocabulary is off by some 1e-14, so that a random number falls between two results about never.
// Greedy: 16 bytes at a time where rows allow it; only maxima are taken (a packed maximum of two bf16 costs one instruction), a thread keeps its first best
// vector, and the entry inside it is looked up at the end.
#include <cooperative_groups.h>
#include "rr_paged.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int NT = 512, NW = NT / 32, BLOCK = 256, MAX_CL = 8;
constexpr int MAX_SUMS = 1024;                          // blocks' sums that a CTA keeps
constexpr int ROWS = 16;                                // greedy: rows looked at between two exchanges

struct Span { int first, n; };                          // a sequence's first row, its drafts (-1: it has no rows)

__device__ __forceinline__ Span span_of(const rr_verify_args& a, int b) {
  const int first = a.cu ? max(__ldg(a.cu + b), 0) : b, end = a.cu ? min(__ldg(a.cu + b + 1), a.rows) : b + 1;
  return Span{first, max(end - first, 0) - 1};
}

// Probabilities are finite and positive, or 0.
template <typename T>
__device__ __forceinline__ float weight(T x) {
  const float f = rr_to_f32(x);
  return f > 0.f && f <= 3.402823466e38f ? f : 0.f;
}
template <typename T>
__device__ __forceinline__ float probability(const void* rows, int64_t stride, int row, int x) {
  return weight(__ldg((const T*)rows + row * stride + x));
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
  return x;
}
__device__ __forceinline__ double warp_prefix(double x) {               // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) { const double y = __shfl_up_sync(0xFFFFFFFFu, x, d); if (lane >= d) x += y; }
  return x;
}

// Accepted drafts and lengths, but for the token more.
__device__ __forceinline__ void write_accepted(const rr_verify_args& a, int b, const Span& s, int accepted, int more) {
  const int lane = threadIdx.x & 31;
  for (int i = lane; i <= s.n; i += 32)
    a.out[s.first + i] = i < accepted ? a.tokens[s.first + i + 1] : i == accepted ? more : -1;
  if (lane == 0) {
    a.accepted[b] = accepted;
    if (a.new_lens) a.new_lens[b] = a.lens[b] + (s.n < 0 ? 0 : accepted + 1);
  }
}

// A drafted token is in the vocabulary.
__device__ __forceinline__ bool in_vocab(const rr_verify_args& a, int x) {
  const bool ok = x >= 0 && x < a.vocab;
  if (!ok && a.status) atomicOr(a.status, RR_STATUS_BAD_INDEX);
  return ok;
}

// ---- sampled ----------------------------------------------------------------------------------------------------
// The weights of a row: p - q where there is q, without the entry `but` (-1: none).
template <typename T> struct Weights {
  const T* p;
  const T* q;
  int but, vocab;
  __device__ __forceinline__ double at(int j) const {
    if (j >= vocab || j == but) return 0.0;
    const double w = (double)weight(__ldg(p + j)) - (q ? (double)weight(__ldg(q + j)) : 0.0);
    return w > 0.0 ? w : 0.0;
  }
  // Entries first + lane + 32 i of a block: the loads in front of the arithmetic.
  __device__ __forceinline__ void block(int first, double (&w)[8]) const {
    T x[8], y[8];
    const int j0 = first + (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = j0 + 32 * i;
      const bool in = j < vocab;
      x[i] = in ? __ldg(p + j) : rr_from_f32<T>(0.f);
      y[i] = in && q ? __ldg(q + j) : rr_from_f32<T>(0.f);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double d = (double)weight(x[i]) - (double)weight(y[i]);
      w[i] = d > 0.0 && j0 + 32 * i != but ? d : 0.0;
    }
  }
};

struct Found { double sums[MAX_SUMS]; double total; double warp[NW]; };

// The first entry of a warp's 32 whose running sum, from `run` on, is over `limit`, else the last one with a weight; 32 if none has.
__device__ __forceinline__ int first_over(double w, double run, double limit) {
  const double upto = run + warp_prefix(w);             // (by all lanes)
  const unsigned over = __ballot_sync(0xFFFFFFFFu, w > 0.0 && upto > limit);
  if (over) return __ffs(over) - 1;
  const unsigned some = __ballot_sync(0xFFFFFFFFu, w > 0.0);
  return some ? 31 - __clz(some) : 32;
}

template <typename T>
__global__ void __launch_bounds__(NT)
verify_sampled_kernel(const __grid_constant__ rr_verify_args a) {
  __shared__ Found f;
  cg::cluster_group cl = cg::this_cluster();
  const int ctas = cl.num_blocks(), cta = cl.block_rank(), b = blockIdx.x / ctas;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Span s = span_of(a, b);
  if (s.n < 0) {                                        // (uniform in the cluster)
    if (cta == 0 && warp == 0) write_accepted(a, b, s, 0, -1);
    return;
  }
  // which drafts are accepted: every warp for itself
  int accepted = 0;
  for (int i0 = 0; i0 < s.n; i0 += 32) {
    const int i = i0 + lane, t = s.first + i;
    bool ok = true;
    if (i < s.n) {
      const int x = __ldg(a.tokens + t + 1);
      ok = in_vocab(a, x);
      if (ok) {
        const double p = probability<T>(a.target, a.target_stride, t, x), q = a.draft ? probability<T>(a.draft, a.draft_stride, t, x) : 1.0;
        ok = p > (double)__ldg(a.uniform + t) * q;
      }
    }
    const unsigned rejected = __ballot_sync(0xFFFFFFFFu, !ok);
    if (rejected) { accepted = i0 + __ffs(rejected) - 1; break; }
    accepted = min(i0 + 32, s.n);
  }
  const int row = s.first + accepted;
  Weights<T> w{(const T*)a.target + row * a.target_stride, nullptr, -1, a.vocab};
  if (accepted < s.n) {
    if (a.draft) w.q = (const T*)a.draft + row * a.draft_stride;
    else w.but = __ldg(a.tokens + row + 1);
  }
  const double u = fmax((double)__ldg(a.uniform + s.first + s.n), 0.0);
  // blocks of this CTA; a kept sum stands for `per` of them
  const int blocks = (a.vocab + BLOCK - 1) / BLOCK, share = (blocks + ctas - 1) / ctas, from = min(cta * share, blocks), mine = min(share, blocks - from);
  const int per = (share + MAX_SUMS - 1) / MAX_SUMS, sums = (mine + per - 1) / per;
  int token = -1;
  bool here = false, none = false;
  for (int pass = 0; pass < 2; ++pass) {
    for (int k = warp; k < sums; k += NW) {
      double sum = 0.0;
      for (int i = k * per; i < min((k + 1) * per, mine); ++i) {
        double x[8];
        w.block((from + i) * BLOCK, x);
        sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      }
      sum = warp_sum(sum);
      if (lane == 0) f.sums[k] = sum;
    }
    __syncthreads();
    if (warp == 0) {
      double sum = 0.0;
      for (int k = lane; k < sums; k += 32) sum += f.sums[k];
      sum = warp_sum(sum);
      if (lane == 0) f.total = sum;
    }
    cl.sync();
    // every warp finds the CTA that has the threshold
    const double theirs = lane < ctas ? *cl.map_shared_rank(&f.total, lane) : 0.0;
    const double run = warp_prefix(theirs), total = __shfl_sync(0xFFFFFFFFu, run, 31), limit = u * total;
    const int who = first_over(theirs, 0.0, limit);
    cl.sync();                                          // the sums have been read (nothing of another CTA's is read from here on)
    if (who == 32) {                                    // no weight: the rejected row has no more than the draft's anywhere
      none = !w.q && w.but < 0;
      if (none) break;
      w.q = nullptr;
      w.but = -1;
      continue;
    }
    here = who == cta;
    if (!here || warp != 0) break;
    // the kept sum, then the block, then the entry
    double before = __shfl_sync(0xFFFFFFFFu, run - theirs, who), before_k = before;
    int k = 0;
    for (int k0 = 0; k0 < sums; k0 += 32) {
      const double x = k0 + lane < sums ? f.sums[k0 + lane] : 0.0, upto = warp_prefix(x);
      const int l = first_over(x, before, limit);
      if (l < 32) k = k0 + l, before_k = before + __shfl_sync(0xFFFFFFFFu, upto - x, l);
      if (__any_sync(0xFFFFFFFFu, x > 0.0 && before + upto > limit)) break;
      before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    before = before_k;
    bool over = false;
    for (int i = k * per; i < min((k + 1) * per, mine) && !over; ++i) {
      double x[8];
      w.block((from + i) * BLOCK, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double upto = warp_prefix(x[e]);
        const int l = first_over(x[e], before, limit);
        if (!over && l < 32) token = (from + i) * BLOCK + 32 * e + l;
        over = over || __any_sync(0xFFFFFFFFu, x[e] > 0.0 && before + upto > limit);
        before += __shfl_sync(0xFFFFFFFFu, upto, 31);
      }
    }
    break;
  }
  // a CTA that has the token, or the first one where all weights are 0
  if (warp == 0 && (here || (none && cta == 0))) write_accepted(a, b, s, accepted, token);
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

template <typename T, int VEC>
__global__ void __launch_bounds__(NT)
verify_greedy_kernel(const __grid_constant__ rr_verify_args a) {
  __shared__ Best s_warp[ROWS][NW], s_cta[ROWS];
  __shared__ int s_best[ROWS];
  static_assert(ROWS == NW, "a warp per row");
  cg::cluster_group cl = cg::this_cluster();
  const int ctas = cl.num_blocks(), cta = cl.block_rank(), b = blockIdx.x / ctas;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Span s = span_of(a, b);
  if (s.n < 0) {
    if (cta == 0 && warp == 0) write_accepted(a, b, s, 0, -1);
    return;
  }
  using V = Vec<T, VEC>;
  const int vecs = a.vocab / VEC, share = (vecs + ctas - 1) / ctas, from = min(cta * share, vecs), to = min(from + share, vecs);
  const bool tail = cta == ctas - 1 && threadIdx.x == 0;                // the entries behind the last vector
  int accepted = 0, more = -1;
  for (int i0 = 0;; i0 += ROWS) {
    const int rows = min(ROWS, s.n + 1 - i0);
    for (int r = 0; r < rows; ++r) {
      const T* const row = (const T*)a.target + (s.first + i0 + r) * a.target_stride;
      Best x{0u, INT32_MAX};
#pragma unroll 4
      for (int v = from + threadIdx.x; v < to; v += NT) {
        V e;
        if constexpr (VEC == 1) e.v = __ldg(row + v);
        else { const uint4 raw = __ldg((const uint4*)row + v); e = *(const V*)&raw; }
        const uint32_t key = score_key(e.best());
        if (key > x.key) x = Best{key, v};
      }
      if (tail)
        for (int j = vecs * VEC; j < a.vocab; ++j)
          if (const uint32_t key = score_key(rr_to_f32(__ldg(row + j))); key > x.key) x = Best{key, vecs};
      x = warp_best(x);
      if (lane == 0) s_warp[r][warp] = x;
    }
    __syncthreads();
    if (warp < rows) {
      const Best x = warp_best(lane < NW ? s_warp[warp][lane] : Best{0u, INT32_MAX});
      // the first entry of the vector that is as good
      const T* const row = (const T*)a.target + (s.first + i0 + warp) * a.target_stride;
      const int j = x.key ? x.at * VEC + lane : 0;
      const unsigned same = __ballot_sync(0xFFFFFFFFu, x.key && lane < VEC && j < a.vocab && score_key(rr_to_f32(__ldg(row + j))) == x.key);
      if (lane == 0) s_cta[warp] = Best{x.key, x.key ? x.at * VEC + __ffs(same) - 1 : INT32_MAX};
    }
    cl.sync();
    if (warp < rows) {
      const Best x = warp_best(lane < ctas ? *cl.map_shared_rank(&s_cta[warp], lane) : Best{0u, INT32_MAX});
      if (lane == 0) s_best[warp] = x.key ? x.at : -1;
    }
    cl.sync();
    const int i = i0 + lane;
    bool ok = true;
    if (lane < rows && i < s.n) {
      const int x = __ldg(a.tokens + s.first + i + 1);
      ok = in_vocab(a, x) && x == s_best[lane];
    } else if (lane == rows - 1) {
      ok = false;                                       // the row behind the last draft
    }
    const unsigned stop = __ballot_sync(0xFFFFFFFFu, !ok);
    if (stop) {
      accepted = i0 + __ffs(stop) - 1;
      more = s_best[__ffs(stop) - 1];
      break;
    }
    __syncthreads();                                    // (before the next rows' results)
  }
  if (cta == 0 && warp == 0) write_accepted(a, b, s, accepted, more);
}

// CTAs per sequence: eight share one, fewer where a CTA would get less than a block of the vocabulary for each of its warps.
int cluster_of(int vocab) {
  int n = MAX_CL;
  while (n > 1 && vocab < n * NW * BLOCK) n /= 2;
  return n;
}

int launch(void (*kernel)(rr_verify_args), const rr_verify_args& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  const int n = cluster_of(a.vocab);
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = n; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(a.batch * n)); cfg.blockDim = dim3(NT);
  cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = 1;
  rr_count_launch();
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
  return e == cudaSuccess ? RR_OK : rr_cuda_fail(e, "rr_verify_drafts");
}

}  // namespace

extern "C" int rr_verify_drafts(const rr_verify_args* a, void* stream) {
  if (!a || !a->out || !a->accepted || !a->tokens || (!a->target && a->rows > 0)) return RR_ERR_INVALID_ARG;
  if (a->rows < 0 || a->batch < 1 || a->vocab < 1 || (!a->cu && a->rows != a->batch)) return RR_ERR_INVALID_ARG;
  if (a->target_stride < 0 || a->draft_stride < 0 || (a->new_lens && !a->lens) || (a->draft && !a->uniform)) return RR_ERR_INVALID_ARG;
  if (a->dtype != RR_BF16 && a->dtype != RR_F32) return RR_ERR_UNSUPPORTED;
  if (a->vocab > (1 << 30) || a->batch > (1 << 27)) return RR_ERR_TOO_LARGE;
  const uintptr_t e = a->dtype == RR_BF16 ? 1 : 3;
  if ((((uintptr_t)a->target | (uintptr_t)a->draft) & e) ||
      (((uintptr_t)a->tokens | (uintptr_t)a->cu | (uintptr_t)a->uniform | (uintptr_t)a->lens | (uintptr_t)a->out | (uintptr_t)a->accepted |
        (uintptr_t)a->new_lens | (uintptr_t)a->status) & 3)) return RR_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  const bool bf16 = a->dtype == RR_BF16;
  if (a->uniform) return launch(bf16 ? verify_sampled_kernel<__nv_bfloat16> : verify_sampled_kernel<float>, *a, st);
  const bool vec = ((uintptr_t)a->target & 15) == 0 && (a->target_stride * (bf16 ? 2 : 4)) % 16 == 0;
  if (bf16) return launch(vec ? verify_greedy_kernel<__nv_bfloat16, 8> : verify_greedy_kernel<__nv_bfloat16, 1>, *a, st);
  return launch(vec ? verify_greedy_kernel<float, 4> : verify_greedy_kernel<float, 1>, *a, st);
}
