// Rows of attention over a paged cache that have to be looked at again: see the marks in rr_attend_paged.cuh.
#pragma once
#include "rr_attend_paged.cuh"

namespace rrattn {

constexpr unsigned FULL = 0xFFFFFFFFu;

template <typename T> __device__ __forceinline__ float4 load4(const T* p, bool vec, int n);
template <> __device__ __forceinline__ float4 load4<float>(const float* p, bool vec, int n) {
  if (vec) return *(const float4*)p;
  return make_float4(p[0], n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, n > 3 ? p[3] : 0.f);
}
template <> __device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16* p, bool vec, int n) {
  if (vec) {
    const uint2 t = *(const uint2*)p;
    return make_float4(__uint_as_float(t.x << 16), __uint_as_float(t.x & 0xFFFF0000u), __uint_as_float(t.y << 16), __uint_as_float(t.y & 0xFFFF0000u));
  }
  return make_float4(__bfloat162float(p[0]), n > 1 ? __bfloat162float(p[1]) : 0.f, n > 2 ? __bfloat162float(p[2]) : 0.f, n > 3 ? __bfloat162float(p[3]) : 0.f);
}

// A marked row's outputs are what they should be unless one of the tokens that it may not see but was multiplied with holds an infinity or NaN
// among its values; a row that sees one of its own stays as it is.  Only these tokens are looked at: of the prefix those behind the row's
// limit, of its own or a range row's list those that share a tile with the last one seen by some row of the item.  Where one is found the row is computed
// from the definition: a token that it does not see is not read.  (Up to 32 rows on the tensor cores multiply the other quarters' tokens with weight 0, too.
// A NaN among these is the row's own if the row sees it, as it does unless it is found; an infinity is an infinity in its quarter's partial
// and NaN in the others': `force`.)  `parts` warps take 32 tokens in turn, 8 of them in flight; one alone writes the row's
// output, of several each leaves its part for the join.  Bound by these loads' latency, and by the cache's traffic where many
// rows are computed again.  Measured, a prompt of 8192 tokens, 32 heads on 8 of 128, 1.24 ms: with a NaN that all rows see 6.1 ms (looked at),
// that only the last token sees 13.4 ms (193 tokens' rows computed again).
struct Part { float *o, *m, *l; };                     // [256], [1], [1], in shared memory

// The query token, head and limit of row `row` of a ranges call.
__device__ __forceinline__ RowAt range_row(const Params& P, long long row) {
  const int mg = P.m * P.group;
  const long long rr = quot(row, mg), per = quot(rr, P.n_q);
  const int idx = (int)(row - rr * mg), i = (int)(rr - per * P.n_q), b = (int)per / P.route_heads, len = seq_end(P, b);
  RowAt a;
  a.t = i * P.m + idx / P.group;
  a.h = (int)per % P.route_heads * P.group + idx % P.group;
  a.limit = P.causal ? max(len - P.n_q * P.m + a.t + 1, 0) : len;
  return a;
}

// Calls body(at) with the lanes' places of 32 tokens at a time (-1: none) for the list's tokens in [from, to), every parts-th time.
template <class F>
__device__ __forceinline__ void each_tokens(const Params& P, const Seg& s, int from, int to, int part, int parts, F&& body) {
  const int lane = threadIdx.x & 31, spans = s.slots ? P.slots : 1;
  int turn = 0;
  for (int j = 0; j < spans; ++j) {
    int lo = s.tok0, hi = s.tok1;
    if (s.slots) slot_span(s, j, lo, hi);
    lo = max(lo, from);
    hi = min(hi, to);
    for (int t = lo; t < hi; t += 32) {
      if (turn == part) body(t + lane < hi ? token_at(P, s, t + lane) : -1LL);
      turn = turn + 1 == parts ? 0 : turn + 1;
    }
  }
}

// The row's output, a lane its columns 4 lane .. and 128 + 4 lane ...  No weight at all: zeros for a row without tokens, NaN for one whose tokens are all at -inf.
template <typename T>
__device__ __forceinline__ void write_row(const Params& P, long long out, float m, float l, const float4 (&o)[2]) {
  const int e0 = (threadIdx.x & 31) * 4;
  const float inv = l == 0.f ? (m == NINF ? 0.f : __int_as_float(0x7fc00000)) : 1.f / l;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const float y[4] = {o[v].x, o[v].y, o[v].z, o[v].w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (e0 + 128 * v + j < P.dh) ((T*)P.out)[out + e0 + 128 * v + j] = rr_from_f32<T>(y[j] * inv);
  }
}

template <typename T, int NV>                          // NV groups of 128 columns
__device__ __noinline__ bool look_again(const Params& P, long long row, bool force, int part, int parts, Part y) {
  constexpr int N = 8 / NV;                            // tokens' loads in flight
  const int lane = threadIdx.x & 31, e0 = lane * 4;
  Seg s;
  s.prefix = 0; s.prefix_pages = nullptr; s.slots = nullptr; s.tok0 = 0;
  long long q, out;
  int limit, behind;                                   // behind: unseen tokens from there on were not multiplied
  if (P.slots) {
    const long long rr = quot(row, P.m * P.group), per = quot(rr, P.n_q);
    const RowAt a = range_row(P, row);
    s.b = (int)per / P.route_heads;
    s.kvh = (int)per % P.route_heads / (P.route_heads / P.kv_heads);
    s.slots = P.ranges + rr * P.slots * 2;
    s.tok1 = seq_len(P, s.b);
    q = s.b * P.qb + a.h * P.qh + a.t * P.qt;
    out = s.b * P.ob + a.h * P.oh + a.t * P.ot;
    limit = a.limit;
    behind = s.tok1;
  } else {
    const int t = (int)quot(row, P.heads), h = (int)(row - (long long)t * P.heads);
    const Plan plan = plan_of(P);
    s.b = P.cu ? rr_sequence_of(P.cu, P.batch, t) : t;
    s.kvh = h / P.group;
    s.tok1 = seq_len(P, s.b);
    s.prefix = P.prefix;
    s.prefix_pages = P.prefix_pages ? P.prefix_pages : P.table + plan.source * P.table_stride;
    const int n = seq_count(P, s.b), len = seq_end(P, s.b);
    q = t * P.qt + h * P.qh;
    out = t * P.ot + h * P.oh;
    limit = P.causal ? max(len - n + (t - seq_first(P, s.b)) + 1, 0) : len;
    behind = (int)min((long long)s.tok1, (long long)limit + ROWS / P.group + 1 + TILE);
    if (prefix_tiles(plan) > 0) behind = max(behind, plan.prefix);
  }
  s.pages = P.table + s.b * P.table_stride;
  auto values = [&](const void* from, long long at, int i0, float4 (&x)[N][NV]) {
    auto load = [&](bool vec) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const long long o = __shfl_sync(FULL, at, i0 + i);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int e = e0 + 128 * v;
          x[i][v] = o >= 0 && e < P.dh ? load4<T>((const T*)from + o + e, vec, P.dh - e) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
    };
    if (P.vk) load(true); else load(false);            // (one branch for all loads: they are under way together)
  };
  if (!force) {
    const int tok1 = s.tok1;
    bool found = false;
    s.tok1 = max(tok1, behind);                        // (a sequence shorter than the prefix has been multiplied with all of it)
    each_tokens(P, s, limit, behind, 0, 1, [&](long long at) {
#pragma unroll 1
      for (int i0 = 0; i0 < 32; i0 += N) {
        float4 x[N][NV];
        values(P.v, at, i0, x);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int v = 0; v < NV; ++v) found = found || !(isfinite(x[i][v].x) && isfinite(x[i][v].y) && isfinite(x[i][v].z) && isfinite(x[i][v].w));
      }
    });
    s.tok1 = tok1;
    if (!__any_sync(FULL, found)) return false;
  }
  float4 qv[NV], o[2];
  float m = NINF, l = 0.f;
  bool seen = false;
  o[0] = o[1] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int e = e0 + 128 * v;
    qv[v] = e < P.dh ? load4<T>((const T*)P.q + q + e, P.vq, P.dh - e) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  each_tokens(P, s, 0, limit, part, parts, [&](long long at) {
    const unsigned sees = __ballot_sync(FULL, at >= 0);
    seen = seen || sees != 0;
#pragma unroll 1
    for (int i0 = 0; i0 < 32; i0 += N) {
      if (!(sees >> i0 & ((1u << N) - 1))) continue;
      float4 k[N][NV], w[N][NV];
      values(P.k, at, i0, k);
      values(P.v, at, i0, w);
      float z[N], top = NINF;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        z[i] = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) z[i] = fmaf(qv[v].w, k[i][v].w, fmaf(qv[v].z, k[i][v].z, fmaf(qv[v].y, k[i][v].y, fmaf(qv[v].x, k[i][v].x, z[i]))));
#pragma unroll
        for (int off = 16; off; off >>= 1) z[i] += __shfl_xor_sync(FULL, z[i], off);
        z[i] = sees >> (i0 + i) & 1 ? z[i] * P.scale_log2 : NINF;
        top = fmaxf(top, z[i]);
      }
      const float now = fmaxf(m, top), ref = now == NINF ? 0.f : now, f = exp2f(m - ref);
      m = now;
      l *= f;
#pragma unroll
      for (int v = 0; v < NV; ++v) { o[v].x *= f; o[v].y *= f; o[v].z *= f; o[v].w *= f; }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (!(sees >> (i0 + i) & 1)) continue;
        const float p = exp2f(z[i] - ref);
        l += p;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          o[v].x = fmaf(p, w[i][v].x, o[v].x); o[v].y = fmaf(p, w[i][v].y, o[v].y);
          o[v].z = fmaf(p, w[i][v].z, o[v].z); o[v].w = fmaf(p, w[i][v].w, o[v].w);
        }
      }
    }
  });
  if (seen && m == NINF) m = LOWEST;
  if (parts == 1) {
    write_row<T>(P, out, m, l, o);
  } else {
    if (lane == 0) { *y.m = m; *y.l = l; }
    *(float4*)(y.o + e0) = o[0];
    *(float4*)(y.o + e0 + 128) = o[1];
  }
  return true;
}
template <typename T>
__device__ __forceinline__ bool look_again(const Params& P, long long row, bool force, int part, int parts, const Part& y) {
  return P.dh <= 128 ? look_again<T, 1>(P, row, force, part, parts, y) : look_again<T, 2>(P, row, force, part, parts, y);
}

}  // namespace rrattn
