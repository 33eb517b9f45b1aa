// New keys and values into a paged cache, keys and queries rotated by their positions on the way.
//
// Token t of sequence b at position p = lens[b] + (t - cu[b]):
//   K[page(b, p)][h][p % ps] = R(p) k[t, h],   V[...] = v[t, h],   q_out[t, h] = R(p) q[t, h]
// R(p) turns pair j of a head's first `rot` entries by p * inv_freq[j].  In turns that is p * (inv_freq[j] / 2 pi), formed in 64 bits: both
// roundings are below 2^-53 of it, 2^-22 of a turn at the last position, 2^-32 up to position 2^21.  Its fractional part is exact there; the
// sine and cosine of what is left (at most half a turn) are FP32's.  All heads of a token share its angles.
// With positions of several axes (time, height, width of a patch of an image or a video) pair j turns by positions[axis_of[j]][t] * inv_freq[j]; where
// the token goes in the cache is still counted in tokens.  That build has one load in front of another more (the pair's axis, then its position).
//
// The work is one read and one write of every entry: bound by memory for prompts, by latency for a decoding
// step.  A CTA takes a token; its threads take 16 bytes each (the two halves of eight or four pairs) and rotate in FP32 with one
// rounding.  Shapes and strides that do not split into 16-byte pieces go entry by entry.  Measured: 17000 tokens of 32 query and 8 key heads of
// 128, bf16 (418 MB): 67 us, 6.2 TB/s, 95 % of a copy's rate, with positions of three axes 70 us, entry by entry 214 us; one token for each of 64 sequences: 3.5 us, with axes
// 3.9 us.  (Loads in front of the angles, two pieces a thread: 130 us; the pieces' places have to be worked out twice then.)
#include "rr_paged.cuh"

namespace {

constexpr int MOST_NT = 256;                           // threads of a CTA: this, or half of them

struct AppendParams {
  rr_paged_kv kv;
  rr_append_args a;
  rr_axes_args x;                                      // read by the build with axes only
};

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Piece { T x[VEC]; };

// All of a sequence's new tokens have room: a page may otherwise be another sequence's, too.
__device__ __forceinline__ bool has_room(const rr_append_args& a, int b, int n) { return !a.room || (long long)a.lens[b] + n <= a.room[b]; }

template <typename T, int VEC, bool AXES>
__global__ void __launch_bounds__(MOST_NT)
kv_append_kernel(const __grid_constant__ AppendParams P) {
  __shared__ float s_cos[RR_PAGED_MAX_DH / 2], s_sin[RR_PAGED_MAX_DH / 2];
  __shared__ int s_pos;
  __shared__ long long s_at;                           // element offset of the token's place in the cache; -1: left out
  const rr_paged_kv& kv = P.kv;
  const rr_append_args& a = P.a;
  const int tid = threadIdx.x, NT = blockDim.x, t = blockIdx.x;
  if (blockIdx.x == gridDim.x - 1 && a.new_lens)
    for (int b = tid; b < kv.batch; b += NT) {
      const int n = max(a.cu ? a.cu[b + 1] - a.cu[b] : 1, 0);
      a.new_lens[b] = a.lens[b] + (has_room(a, b, n) ? n : 0);
    }
  if (t >= a.tokens) return;
  if (tid < 32) {
    const int b = a.cu ? rr_sequence_of_warp(a.cu, kv.batch, t) : t;
    if (tid == 0) {
      int pos = -1;
      long long at = -1;
      if (b >= 0) {
        const long long p = (long long)a.lens[b] + (a.cu ? t - a.cu[b] : 0);
        const long long col = p / kv.page_tokens;
        const bool room = has_room(a, b, a.cu ? a.cu[b + 1] - a.cu[b] : 1);
        bool ok = p >= 0 && col < kv.pages_per_seq;
        int page = -1;
        if (ok) page = kv.page_table[b * kv.table_stride + col];
        ok = ok && page >= 0 && page < kv.num_pages && room;
        if (ok) at = page * kv.page_stride + (p - col * kv.page_tokens) * kv.token_stride;
        else if (kv.status) atomicOr(kv.status, room ? RR_STATUS_BAD_INDEX : RR_STATUS_NO_PAGES);
        pos = p < 0 ? 0 : (int)min(p, 0x7FFFFFFFLL);
      }
      s_pos = pos;
      s_at = at;
    }
  }
  __syncthreads();
  const int pos = s_pos;
  const long long at = s_at;
  if (pos < 0) return;                                 // padding
  const int half = a.rot / 2, dh = kv.dh;
  for (int j = tid; j < half; j += NT) {
    int at_j = pos;
    if constexpr (AXES) {
      const int axis = P.x.axis_of ? P.x.axis_of[j] : 0;
      at_j = 0;                                        // (a pair of no axis is not turned)
      if (axis >= 0 && axis < P.x.axes) at_j = P.x.positions[axis * P.x.axis_stride + t * P.x.token_stride];
      else if (kv.status) atomicOr(kv.status, RR_STATUS_BAD_INDEX);
    }
    const double turns = (double)at_j * ((double)a.inv_freq[j] * 0.15915494309189533577);  // 1 / (2 pi)
    sincospif(2.0f * (float)(turns - rint(turns)), &s_sin[j], &s_cos[j]);
  }
  __syncthreads();
  // Pieces of a head: of the rotated part, then of the rest.  Halves: a rotated piece is VEC pairs (two
  // loads); neighbours: VEC / 2 pairs in one load (VEC == 1: a pair as two loads, like halves).
  const bool two = !a.interleaved || VEC == 1;
  const int turned = two ? half / VEC : a.rot / VEC;
  const int per_head = turned + (dh - a.rot) / VEC, flat = dh / VEC;
  const int nq = a.q ? a.q_heads * per_head : 0, nk = at >= 0 ? kv.kv_heads * per_head : 0, nv = at >= 0 ? kv.kv_heads * flat : 0;
  using V = Piece<T, VEC>;
  for (int u = tid; u < nq + nk + nv; u += NT) {
    const T* src;
    T* dst;
    int i;
    if (u < nq) {
      const int h = u / per_head;
      i = u - h * per_head;
      src = (const T*)a.q + t * a.q_token_stride + h * a.q_head_stride;
      dst = (T*)a.q_out + t * a.out_token_stride + h * a.out_head_stride;
    } else if (u < nq + nk) {
      const int w = u - nq, h = w / per_head;
      i = w - h * per_head;
      src = (const T*)a.k + t * a.k_token_stride + h * a.k_head_stride;
      dst = (T*)kv.k + at + h * kv.head_stride;
    } else {
      const int w = u - nq - nk, h = w / flat, e = (w - h * flat) * VEC;
      src = (const T*)a.v + t * a.v_token_stride + h * a.v_head_stride;
      dst = (T*)kv.v + at + h * kv.head_stride;
      *(V*)(dst + e) = *(const V*)(src + e);
      continue;
    }
    if (i >= turned) {
      const int e = a.rot + (i - turned) * VEC;
      *(V*)(dst + e) = *(const V*)(src + e);
    } else if (two) {
      const int j = i * VEC, e0 = a.interleaved ? 2 * j : j, e1 = a.interleaved ? e0 + 1 : j + half;
      V x = *(const V*)(src + e0), y = *(const V*)(src + e1);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float c = s_cos[j + e], s = s_sin[j + e], p = rr_to_f32(x.x[e]), q = rr_to_f32(y.x[e]);
        x.x[e] = rr_from_f32<T>(p * c - q * s);
        y.x[e] = rr_from_f32<T>(q * c + p * s);
      }
      *(V*)(dst + e0) = x;
      *(V*)(dst + e1) = y;
    } else {
      V x = *(const V*)(src + i * VEC);
#pragma unroll
      for (int e = 0; e + 1 < VEC; e += 2) {
        const int j = (i * VEC + e) / 2;
        const float c = s_cos[j], s = s_sin[j], p = rr_to_f32(x.x[e]), q = rr_to_f32(x.x[e + 1]);
        x.x[e] = rr_from_f32<T>(p * c - q * s);
        x.x[e + 1] = rr_from_f32<T>(q * c + p * s);
      }
      *(V*)(dst + i * VEC) = x;
    }
  }
}

// Whether every piece of `vec` entries starts on its own size.
bool pieces(const rr_paged_kv& kv, const rr_append_args& a, int vec, size_t bytes) {
  uint64_t s = (uint64_t)kv.page_stride | kv.head_stride | kv.token_stride | a.k_token_stride | a.k_head_stride | a.v_token_stride |
               a.v_head_stride | (uint64_t)kv.dh | (uint64_t)(a.interleaved ? a.rot : a.rot / 2);
  uint64_t p = (uintptr_t)kv.k | (uintptr_t)kv.v | (uintptr_t)a.k | (uintptr_t)a.v;
  if (a.q) {
    s |= (uint64_t)a.q_token_stride | a.q_head_stride | a.out_token_stride | a.out_head_stride;
    p |= (uintptr_t)a.q | (uintptr_t)a.q_out;
  }
  return s % vec == 0 && (p & (bytes - 1)) == 0;
}

template <bool AXES>
int append(const rr_paged_kv* kv, const rr_append_args* a, const rr_axes_args* x, void* stream, const char* who) {
  const int rc = rr_paged_check(kv);
  if (rc != RR_OK) return rc;
  if (!a || !a->k || !a->v || !a->lens) return RR_ERR_INVALID_ARG;
  if (a->tokens < 0 || (!a->cu && a->tokens != kv->batch)) return RR_ERR_INVALID_ARG;
  if (a->q && (!a->q_out || a->q_heads < 1)) return RR_ERR_INVALID_ARG;
  if (a->rot < 0 || a->rot > kv->dh || (a->rot & 1) || (a->rot > 0 && !a->inv_freq)) return RR_ERR_INVALID_ARG;
  if (a->interleaved != 0 && a->interleaved != 1) return RR_ERR_INVALID_ARG;
  const int64_t row = 4 * (int64_t)kv->batch;
  // (lengths are written while others are read)
  if (a->new_lens == a->lens || !rr_apart(a->new_lens, row, a->lens, row) || !rr_apart(a->new_lens, row, a->cu, row + 4) || !rr_apart(a->new_lens, row, a->room, row))
    return RR_ERR_INVALID_ARG;
  if (a->k_token_stride < 0 || a->k_head_stride < 0 || a->v_token_stride < 0 || a->v_head_stride < 0 || a->q_token_stride < 0 ||
      a->q_head_stride < 0 || a->out_token_stride < 0 || a->out_head_stride < 0) return RR_ERR_INVALID_ARG;
  const uintptr_t e = kv->dtype == RR_BF16 ? 1 : 3;
  if ((((uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)a->q | (uintptr_t)(a->q ? a->q_out : nullptr)) & e) ||
      (((uintptr_t)a->lens | (uintptr_t)a->cu | (uintptr_t)a->new_lens | (uintptr_t)a->inv_freq | (uintptr_t)a->room) & 3)) return RR_ERR_INVALID_ARG;
  if constexpr (AXES) {
    if (!x || !x->positions || a->rot == 0 || x->axes < 1 || x->axis_stride < 0 || x->token_stride < 0) return RR_ERR_INVALID_ARG;
    if (((uintptr_t)x->positions | (uintptr_t)x->axis_of) & 3) return RR_ERR_INVALID_ARG;
  }
  if (a->tokens == 0 && !a->new_lens) return RR_OK;
  const AppendParams P{*kv, *a, x ? *x : rr_axes_args{}};
  const int grid = a->tokens > 0 ? a->tokens : 1;
  // Few tokens: a token's own time counts, which more threads make shorter (64 tokens: 0.7 us less than with half of them).  Many: what all warps of a CTA do alike
  // -- barriers, the sequence, the angles' loop -- costs issue slots, which half of them halve (17000 tokens, 418 MB: 79 us with 256 threads, 69 with 128; 4737 tokens 22.6 us with 128, 4736 24.3 with 256).
  const int NT = grid > 32 * rr_sm_count() ? MOST_NT / 2 : MOST_NT;
  cudaStream_t st = (cudaStream_t)stream;
  if (kv->dtype == RR_BF16) {
    if (pieces(*kv, *a, 8, 16)) kv_append_kernel<__nv_bfloat16, 8, AXES><<<grid, NT, 0, st>>>(P);
    else kv_append_kernel<__nv_bfloat16, 1, AXES><<<grid, NT, 0, st>>>(P);
  } else {
    if (pieces(*kv, *a, 4, 16)) kv_append_kernel<float, 4, AXES><<<grid, NT, 0, st>>>(P);
    else kv_append_kernel<float, 1, AXES><<<grid, NT, 0, st>>>(P);
  }
  rr_count_launch();
  const cudaError_t err = cudaPeekAtLastError();
  return err == cudaSuccess ? RR_OK : rr_cuda_fail(err, who);
}

}  // namespace

extern "C" int rr_kv_append(const rr_paged_kv* kv, const rr_append_args* a, void* stream) {
  return append<false>(kv, a, nullptr, stream, "rr_kv_append");
}

extern "C" int rr_kv_append_axes(const rr_paged_kv* kv, const rr_append_args* a, const rr_axes_args* x, void* stream) {
  return append<true>(kv, a, x, stream, "rr_kv_append_axes");
}
