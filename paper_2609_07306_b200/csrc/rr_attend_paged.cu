// rr_attend_shared and rr_attend_paged_ranges: checks, workspace, the plan and join kernels, and the kernel that
// processes segments on the ordinary pipes (fp32, and bf16 widths other than 64 and 128).
#include <algorithm>
#include <cmath>
#include <type_traits>
#include "rr_attend_paged_again.cuh"

using namespace rrattn;

namespace {

// ---- plan --------------------------------------------------------------------------------------------------
// cum[b] = tiles of all items before sequence b's: the prefix's, then the sequences' own, in their order.  The prefix's pages stand in the row of
// the first sequence that has all of the prefix (a row tells nothing of places behind its own sequence's length), or of the longest one.
constexpr int PLAN_NT = 1024;
__global__ void __launch_bounds__(PLAN_NT) plan_kernel(const __grid_constant__ Params P) {
  __shared__ long long s_warp[PLAN_NT / 32];
  __shared__ int3 s_plan[PLAN_NT / 32];
  rr_pdl_wait();
  rr_pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // the sequences apart: if their row tiles are at most an eighth more than those of all rows together
  int tiles = 0, len = -1, at = 0;                      // row tiles; tokens of the prefix, and the lowest b that has as many
  for (int b = tid; b < P.batch; b += PLAN_NT) {
    const int n = seq_len(P, b);
    if (n > 0) tiles += own_row_tiles(P, b);
    if (min(n, P.prefix) > len) { len = min(n, P.prefix); at = b; }
  }
  auto reduce = [&]() {
    tiles = __reduce_add_sync(FULL, tiles);
    const int most = __reduce_max_sync(FULL, len);
    at = __reduce_min_sync(FULL, len == most ? at : 0x7FFFFFFF);
    len = most;
  };
  reduce();
  if (lane == 0) s_plan[warp] = make_int3(tiles, len, at);
  __syncthreads();
  const int3 all = s_plan[lane];
  tiles = all.x; len = all.y; at = all.z;
  reduce();
  const long long packed = prefix_row_tiles(P);
  const Plan plan{P.always_apart || tiles <= packed + packed / 8, at, len, 0};
  const bool apart = plan.apart;
  const long long prefix_all = P.kv_heads * packed * prefix_tiles(plan);
  long long run = P.few_prefix ? 0 : prefix_all, run_few = P.few_prefix ? prefix_all : 0;
  auto scan = [&](long long mine, long long& run) -> long long {     // what is before this thread's, the block's sum added to run
    long long incl = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) { const long long x = __shfl_up_sync(FULL, incl, off); if (lane >= off) incl += x; }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    long long before = run, all = 0;
#pragma unroll
    for (int w = 0; w < PLAN_NT / 32; ++w) { if (w < warp) before += s_warp[w]; all += s_warp[w]; }
    run += all;
    __syncthreads();
    return before + incl - mine;
  };
  for (int b0 = 0; b0 < P.batch; b0 += PLAN_NT) {
    const int b = b0 + tid;
    const bool few = b < P.batch && few_rows_of(P, b);
    if (b < P.batch) check_len(P, b);
    const long long mine = b < P.batch ? (long long)P.kv_heads * own_row_tiles(P, b) * own_tiles(P, b, apart) : 0;
    const long long at = scan(few ? 0 : mine, run);
    if (b < P.batch) P.main.cum[b] = at;
    if (P.few.ctas > 0) {
      const long long at_few = scan(few ? mine : 0, run_few);
      if (b < P.batch) P.few.cum[b] = at_few;
    }
  }
  if (tid == 0) {
    P.main.cum[P.batch] = run;
    if (P.few.ctas > 0) P.few.cum[P.batch] = run_few;
    *P.plan = plan;
  }
}

// ---- join --------------------------------------------------------------------------------------------------
// Where row `row`'s partials are: up to two lists, the n0 first ones of list 0, and n in all.  ONE: each segment leaves one.
template <bool ONE>
struct Partials {
  long long home0, home1, more0, more1, out;           // first partials of the lists, and their further ones
  int c0, c1, cnt0, cnt1, st0, st1, r0, r1, n0, n;
  bool mine, few0, few1, whole, marked;                // whole: one segment with all of the row's tiles has written the output itself

  // partial row of the k-th partial
  __device__ __forceinline__ long long place(const Params& P, int k) const {
    const bool w = k >= n0;
    if (w) k -= n0;
    const int s = w ? st1 : st0, c = ONE ? k : k / s, j = ONE ? 0 : k - c * s, cta = (w ? c1 : c0) + c, r = w ? r1 : r0;
    const Sched& sc = (w ? few1 : few0) ? P.few : P.main;
    if (c == 0) return j == 0 ? (w ? home1 : home0) : (w ? more1 : more0) + (long long)(j - 1) * (w || P.slots ? P.own.step : P.step);
    return sc.slots_at + (long long)cta * sc.cta_rows + r + (j == 0 ? 0 : sc.more_at + (long long)(j - 1) * P.step);
  }
};

template <bool MARKS, bool ONE>
__device__ __forceinline__ Partials<ONE> partials_at(const Params& P, long long row) {
  Partials<ONE> x;
  x.home0 = x.home1 = x.more0 = x.more1 = x.out = 0;
  x.c0 = x.c1 = x.cnt0 = x.cnt1 = x.r0 = x.r1 = 0;
  x.st0 = x.st1 = 1;
  x.few1 = x.whole = x.marked = false;
  x.few0 = P.slots ? P.few.ctas > 0 : P.few_prefix;
  if (P.slots == 0) {
    const int H = P.heads;
    x.mine = row < (long long)P.tokens * H;
    const int t = (int)quot(x.mine ? row : 0, H), h = (int)((x.mine ? row : 0) - (long long)t * H), kvh = h / P.group, g = h - kvh * P.group;
    const int b = P.cu ? rr_sequence_of_warp(P.cu, P.batch, t) : t;
    x.mine = x.mine && b >= 0;                         // (padding: left as it was)
    if (x.mine) {
      const Sched& sp = P.few_prefix ? P.few : P.main;
      const long long all = __ldg(P.main.cum + P.batch), all_p = P.few_prefix ? __ldg(P.few.cum + P.batch) : all, per = (long long)P.tokens * P.group;
      x.out = t * P.ot + h * P.oh;
      const Plan plan = plan_of(P);
      const bool apart = plan.apart;
      const long long np = prefix_tiles(plan), qtp = prefix_row_tiles(P);
      if (np > 0) {
        const long long idx = (long long)t * P.group + g, first = (kvh * qtp + idx / ROWS) * np;
        x.home0 = kvh * per + idx;
        x.r0 = (int)(idx % ROWS);
        if (!ONE) x.more0 = prefix_more_of(P, kvh, x.r0);
        x.c0 = cta_of(sp, first, all_p);
        x.cnt0 = cta_of(sp, first + np - 1, all_p) - x.c0 + 1;
        x.st0 = ONE || P.few_prefix ? 1 : partials_of(P.streams, min((long long)ROWS, per - idx / ROWS * ROWS));
      }
      const int no = own_tiles(P, b, apart);
      if (no > 0) {
        const int t0 = seq_first(P, b), n = seq_count(P, b), qt = own_row_tiles(P, b);
        const long long idx = (long long)(t - t0) * P.group + g;
        x.few1 = few_rows_of(P, b);
        const Sched& sc = x.few1 ? P.few : P.main;
        const long long W = x.few1 ? __ldg(P.few.cum + P.batch) : all, first = __ldg(sc.cum + b) + (kvh * (long long)qt + idx / ROWS) * no;
        x.r1 = (int)(idx % ROWS);
        x.c1 = cta_of(sc, first, W);
        x.cnt1 = cta_of(sc, first + no - 1, W) - x.c1 + 1;
        const long long rows = min((long long)ROWS, (long long)n * P.group - idx / ROWS * ROWS);
        x.st1 = ONE || x.few1 ? 1 : partials_of(P.streams, rows);
        const long long item = (long long)b * P.kv_heads + kvh, at = kvh * per + (long long)t * P.group + g;
        x.home1 = home_of(P, x.st1 > 1, item, at, x.r1);
        if (x.home1 < 0) x.home1 = sc.slots_at + (long long)x.c1 * sc.cta_rows + sc.slot_rows + x.r1;
        if (!ONE && x.st1 > 1) x.more1 = more_of(P, item, at, x.r1);
        x.whole = np == 0 && x.cnt1 == 1 && x.st1 == 1 && !P.in_place;
        if (MARKS) x.marked = x.whole && plan.marked && !x.few1 && leaves_marks(P, rows) && P.marks[at];
      }
    }
  } else {
    const int mg = P.m * P.group;
    x.mine = row < P.range_rows * mg;
    const long long rr = quot(x.mine ? row : 0, mg), per = quot(rr, P.n_q);
    const int idx = (int)((x.mine ? row : 0) - rr * mg), i = (int)(rr - per * P.n_q), r = (int)per % P.route_heads, b = (int)per / P.route_heads;
    x.st0 = ONE ? 1 : partials_of(P.streams, min(ROWS, mg - idx / ROWS * ROWS));
    x.cnt0 = 1;
    x.r0 = idx % ROWS;
    if (P.units) {
      const long long W = range_units(P), first = (rr * ((mg + ROWS - 1) / ROWS) + idx / ROWS) * P.units;
      const Sched& sc = x.few0 ? P.few : P.main;
      x.c0 = cta_of(sc, first, W);
      x.cnt0 = cta_of(sc, first + P.units - 1, W) - x.c0 + 1;
    }
    const Sched& sc = x.few0 ? P.few : P.main;
    x.home0 = home_of(P, x.st0 > 1, rr, row, x.r0);
    if (x.home0 < 0) x.home0 = sc.slots_at + (long long)x.c0 * sc.cta_rows + sc.slot_rows + x.r0;
    if (!ONE && x.st0 > 1) x.more0 = more_of(P, rr, row, x.r0);
    x.whole = x.cnt0 == 1 && x.st0 == 1 && !P.in_place;
    if (MARKS) x.marked = x.mine && x.whole && !x.few0 && leaves_marks(P, min(ROWS, mg - idx / ROWS * ROWS)) && P.marks[row];
    x.out = b * P.ob + (r * P.group + idx % P.group) * P.oh + (i * P.m + idx / P.group) * P.ot;
  }
  x.n0 = x.whole ? 0 : x.cnt0 * x.st0;
  x.n = x.whole ? 0 : x.n0 + x.cnt1 * x.st1;
  return x;
}

// The largest reference of every parts-th partial from `part` on; whether one of them is marked; the lane's first one.
struct First { long long at; float2 ml; };
template <bool ONE>
__device__ __forceinline__ float largest(const Params& P, const Partials<ONE>& p, int part, int parts, bool& marked, First& f) {
  float M = NINF;
  int k = (threadIdx.x & 31) * parts + part;
  f.at = -1;
  f.ml = make_float2(NINF, 0.f);
  if (k < p.n) {
    f.at = p.place(P, k);
    f.ml = P.part_ml[f.at];
    M = f.ml.x;
    marked = marked || has_mark(f.ml.y);
  }
  for (k += 32 * parts; k < p.n; k += 32 * parts) {
    const float2 ml = P.part_ml[p.place(P, k)];
    M = fmaxf(M, ml.x);
    marked = marked || has_mark(ml.y);
  }
#pragma unroll
  for (int off = 16; off; off >>= 1) M = fmaxf(M, __shfl_xor_sync(FULL, M, off));
  return M;
}
__device__ __forceinline__ void add(float4& y, float w, const float4& x) { y.x = fmaf(w, x.x, y.x); y.y = fmaf(w, x.y, y.y); y.z = fmaf(w, x.z, y.z); y.w = fmaf(w, x.w, y.w); }
// Their sum l and output o against the reference M.
template <bool ONE>
__device__ __forceinline__ void joined(const Params& P, const Partials<ONE>& p, int part, int parts, const First& f, float M, float& l, float4 (&o)[2]) {
  const int lane = threadIdx.x & 31, e0 = lane * 4, n = p.n;
  const bool vec = P.dh % 4 == 0;
  l = 0.f;
  o[0] = o[1] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = part; k0 < n; k0 += 32 * parts) {
    const int k = k0 + lane * parts;
    float w = 0.f;
    long long at = f.at;
    float2 ml = f.ml;
    if (k0 != part && k < n) { at = p.place(P, k); ml = P.part_ml[at]; }
    if (k < n) {
      if (ml.x == NINF || (ml.x == LOWEST && ml.y == 0.f)) at = -1;      // nothing in it (and no output written)
      else { w = exp2f(ml.x - M); l = fmaf(w, fabsf(ml.y), l); }
    }
    const int lim = min(32, (n - k0 + parts - 1) / parts);
    for (int u0 = 0; u0 < lim; u0 += 8) {
      float4 x[8][2];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const long long au = __shfl_sync(FULL, at, (u0 + u) & 31);
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int e = e0 + 128 * v;
          x[u][v] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (u0 + u >= lim || au < 0 || e >= P.dh) continue;
          const float* const src = P.part_o + au * P.dh + e;
          if (vec) x[u][v] = *(const float4*)src;
          else x[u][v] = make_float4(src[0], e + 1 < P.dh ? src[1] : 0.f, e + 2 < P.dh ? src[2] : 0.f, e + 3 < P.dh ? src[3] : 0.f);
        }
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float wu = __shfl_sync(FULL, w, (u0 + u) & 31);
        add(o[0], wu, x[u][0]);
        add(o[1], wu, x[u][1]);
      }
    }
  }
#pragma unroll
  for (int off = 16; off; off >>= 1) l += __shfl_xor_sync(FULL, l, off);
}

// A marked row: true if it has been computed again.
template <typename T>
__device__ __noinline__ bool join_again(const Params& P, long long row, int part, int parts, Part y) {
  const Partials<false> p = partials_at<false, false>(P, row);
  bool force = false;                                  // (see look_again)
  if (p.st0 == 8 || p.st1 == 8)
    for (int k = 0; k < p.n; ++k) {
      const long long at = p.place(P, k);
      if (!has_mark(P.part_ml[at].y)) continue;
      for (int e = threadIdx.x & 31; e < P.dh; e += 32) force = force || isinf(P.part_o[at * P.dh + e]);
    }
  return look_again<T>(P, row, __any_sync(FULL, force), part, parts, y);
}
// By one warp, to the end.
template <typename T>
__device__ __noinline__ void join_marked(const Params& P, long long row) {
  if (join_again<T>(P, row, 0, 1, Part{nullptr, nullptr, nullptr})) return;
  const Partials<false> p = partials_at<false, false>(P, row);
  if (p.whole) return;                                 // what is there may stay
  bool marked = false;
  First f;
  const float M = largest(P, p, 0, 1, marked, f);
  float l;
  float4 o[2];
  joined(P, p, 0, 1, f, M, l, o);
  write_row<T>(P, p.out, M, l, o);
}

// WPR warps join the partials of one row: o = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i.  Each warp takes every WPR-th partial, eight of
// them in flight, a lane four columns (and four more 128 further on); the warps' parts are added in their order.  One warp where rows
// are many, eight where they are few (and their partials many: up to a hundred and fifty for a row of one short call).
// MARKS: a row with a marked partial, or of a marked item, is looked at again, and computed again by the same warps if it has to be.  (Calls whose
// kernels leave no marks, nor more than one partial a segment, do without: four sequences of one token behind 2048, 20.0 us, with it 20.7.)
template <typename T, int WPR, bool MARKS>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Params P) {
  __shared__ __align__(16) float s_o[WPR > 1 ? 8 : 1][RR_PAGED_MAX_DH], s_l[8], s_m[8];
  rr_pdl_wait();
  rr_pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % WPR, e0 = lane * 4;
  const long long row = (long long)blockIdx.x * (8 / WPR) + warp / WPR;
  const Partials<!MARKS> p = partials_at<MARKS, !MARKS>(P, row);
  const bool mine = p.mine && (!p.whole || p.marked);
  if (WPR == 1 && !mine) return;
  bool again = p.marked;
  First f;
  float M = largest(P, p, part, WPR, again, f), l;
  if (MARKS && WPR == 1 && __any_sync(FULL, again)) { join_marked<T>(P, row); return; }
  float4 o[2];
  joined(P, p, part, WPR, f, M, l, o);
  if (WPR > 1) {
    if (lane == 0) { s_l[warp] = l; s_m[warp] = M; }
    *(float4*)&s_o[warp][e0] = o[0];
    *(float4*)&s_o[warp][e0 + 128] = o[1];
    if (MARKS) again = __syncthreads_or(again); else __syncthreads();
    if (MARKS && again) {                              // (all warps of the row are here, and agree)
      if (!join_again<T>(P, row, part, WPR, Part{s_o[warp], &s_m[warp], &s_l[warp]}) && p.whole) return;   // (what is there may stay)
      __syncthreads();
    }
    if (part != 0 || !mine) return;
    float top = NINF;
#pragma unroll
    for (int w = 0; w < WPR; ++w) top = fmaxf(top, s_m[warp + w]);
    l = 0.f;
    o[0] = o[1] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WPR; ++w) {
      if (s_m[warp + w] == NINF) continue;
      const float f = exp2f(s_m[warp + w] - top);
      l = fmaf(f, s_l[warp + w], l);
      add(o[0], f, *(const float4*)&s_o[warp + w][e0]);
      add(o[1], f, *(const float4*)&s_o[warp + w][e0 + 128]);
    }
    M = top;
  }
  write_row<T>(P, p.out, M, l, o);
}

// Marked rows of a ranges call whose items are all whole: nothing to join.  (The tensor cores' kernel looks at its own.)
template <typename T>
__global__ void __launch_bounds__(256) marked_kernel(const __grid_constant__ Params P) {
  rr_pdl_wait();
  rr_pdl_trigger();
  const int mg = P.m * P.group;
  const long long rows = P.range_rows * mg;
  for (long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 16; __any_sync(FULL, at < rows); at += (long long)gridDim.x * 256 * 16) {
    const uint4 x = at < rows ? *(const uint4*)(P.marks + at) : make_uint4(0, 0, 0, 0);      // (behind the last row: anything)
    unsigned some = __ballot_sync(FULL, x.x | x.y | x.z | x.w);
    while (some) {
      const int from = __ffs(some) - 1;
      some &= some - 1;
      const long long row0 = __shfl_sync(FULL, at, from);
      for (long long row = row0; row < min(row0 + 16, rows); ++row) {
        const int idx = (int)(row - quot(row, mg) * mg);
        if (leaves_marks(P, min(ROWS, mg - idx / ROWS * ROWS)) && P.marks[row]) look_again<T>(P, row, false, 0, 1, Part{nullptr, nullptr, nullptr});
      }
    }
  }
}

// ---- segments on the ordinary pipes --------------------------------------------------------------------------
// A CTA takes BM = 16 * MR rows at a time through the segment's tokens, BT at a time: thread (ty, tx) of 16 x 16 has the
// logits of rows ty + 16 i and tokens tx + 16 j, and of the output the same rows and 4-column groups tx + 16 j.  Queries, and keys
// and values in turn, stand in shared memory as FP32 rows of dh + 4 entries (16-byte reads of 8 neighbouring rows meet 32
// different banks).  Bound by FP32 multiply-adds where rows are many, by the cache's traffic where they are few (MR = 1).
// Measured: 11 sequences behind 4001 tokens, 1 to 3 queries of 8 heads of 64, fp32: 46 us (the latency of two tiles per CTA, and the join).
constexpr int BT = 64, SNT = 256;

__host__ __device__ constexpr int padded(int dh) { return (dh + 3) / 4 * 4 + 4; }
struct SmemPlan { int q, kv, p, ids, slots, total; };
__host__ __device__ inline SmemPlan smem_plan(int dh, int n_slots, bool only_few) {
  SmemPlan s;
  const int row = padded(dh) * 4;
  s.q = 0;                                             // (few rows: the warps' parts of 4 rows from here on)
  if (only_few) {
    s.kv = s.p = s.ids = 0;
    s.slots = 4 * 4 * ((dh <= 64 ? 64 : dh <= 128 ? 128 : 256) * 4 + 8);
    s.total = s.slots + (2 * n_slots + 1) * 4;
    return s;
  }
  s.kv = s.q + 64 * row;
  s.p = s.kv + BT * row;
  s.ids = s.p + 64 * (BT + 4) * 4;
  s.slots = s.ids + BT * 16;
  s.total = s.slots + (2 * n_slots + 1) * 4;
  return s;
}

struct Ctx {
  float *q, *kv, *p;
  int* id;
  long long* at;
  int *first, *base;                                   // ranges: number of a slot's first token, and its start minus that
  int n_tok;
};

template <typename T, int NV, int MR>
__device__ void rows_block(const Params& P, const Seg& s, const Ctx& c, int r0) {
  constexpr int BM = 16 * MR;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, dh = P.dh, ld = padded(dh), groups = (dh + 3) / 4;
  for (int u = tid; u < BM * groups; u += SNT) {
    const int r = u / groups, e = (u - r * groups) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r0 + r < s.rows) {
      const int idx = s.row0 + r0 + r, dt = idx / P.group;
      const RowAt a{s.t_base + dt, s.h0 + idx - dt * P.group, 0};
      x = load4<T>((const T*)P.q + q_at(P, s, a) + e, P.vq, dh - e);
    }
    *(float4*)(c.q + r * ld + e) = x;
  }
  int limit[MR];
  bool mixed = false;                                  // a token of the list was masked for one of this thread's rows
#pragma unroll
  for (int i = 0; i < MR; ++i) limit[i] = r0 + ty + 16 * i < s.rows ? row_at(P, s, r0 + ty + 16 * i).limit : 0;
  float m[MR], l[MR];
  float4 o[MR][NV];
#pragma unroll
  for (int i = 0; i < MR; ++i) {
    m[i] = NINF; l[i] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) o[i][v] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  uint32_t seen = 0;
  const int num_end = s.tile1 * TILE;
  for (int num0 = s.tile0 * TILE; num0 < num_end; num0 += BT) {
    __syncthreads();                                   // the tile before is done
    if (tid < BT) {
      const int num = num0 + tid;
      int id = NO_TOKEN;
      if (s.slots) {
        if (num < c.n_tok) {
          int lo = 0, hi = P.slots;
          while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (c.first[mid] <= num) lo = mid; else hi = mid; }
          id = c.base[lo] + num;
        }
      } else if (num < s.tok1 - s.tok0) {
        id = s.tok0 + num;
      }
      long long at = -1;
      if (id != NO_TOKEN) { at = token_at(P, s, id); if (at < 0) id = NO_TOKEN; }
      c.id[tid] = id;
      c.at[tid] = at;
    }
    __syncthreads();
    for (int u = tid; u < BT * groups; u += SNT) {
      const int r = u / groups, e = (u - r * groups) * 4;
      const long long at = c.at[r];
      *(float4*)(c.kv + r * ld + e) = at < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : load4<T>((const T*)P.k + at + e, P.vk, dh - e);
    }
    __syncthreads();
    float x[MR][4];
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
#pragma unroll 4
    for (int e = 0; e < groups * 4; e += 4) {
      float4 a[MR], b[4];
#pragma unroll
      for (int i = 0; i < MR; ++i) a[i] = *(const float4*)(c.q + (ty + 16 * i) * ld + e);
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = *(const float4*)(c.kv + (tx + 16 * j) * ld + e);
#pragma unroll
      for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[i][j] = fmaf(a[i].w, b[j].w, fmaf(a[i].z, b[j].z, fmaf(a[i].y, b[j].y, fmaf(a[i].x, b[j].x, x[i][j]))));
    }
    __syncthreads();                                   // the keys are read: the values take their place
    for (int u = tid; u < BT * groups; u += SNT) {
      const int r = u / groups, e = (u - r * groups) * 4;
      const long long at = c.at[r];
      *(float4*)(c.kv + r * ld + e) = at < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : load4<T>((const T*)P.v + at + e, P.vk, dh - e);
    }
#pragma unroll
    for (int i = 0; i < MR; ++i) {
      float top = NINF;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int id = c.id[tx + 16 * j];
        const bool sees = id < limit[i];
        if (sees) seen |= 1u << i;
        else if (id != NO_TOKEN) mixed = true;
        x[i][j] = sees ? x[i][j] * P.scale_log2 : NINF;
        top = fmaxf(top, x[i][j]);
      }
#pragma unroll
      for (int off = 8; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, off));
      const float m_new = fmaxf(m[i], top), ref = m_new == NINF ? 0.f : m_new, f = exp2f(m[i] - ref);
      m[i] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float w = exp2f(x[i][j] - ref);
        sum += w;
        c.p[(ty + 16 * i) * (BT + 4) + tx + 16 * j] = w;
      }
      l[i] = fmaf(l[i], f, sum);
#pragma unroll
      for (int v = 0; v < NV; ++v) { o[i][v].x *= f; o[i][v].y *= f; o[i][v].z *= f; o[i][v].w *= f; }
    }
    __syncthreads();
#pragma unroll 2
    for (int j = 0; j < BT; j += 4) {
      float4 p[MR];
#pragma unroll
      for (int i = 0; i < MR; ++i) p[i] = *(const float4*)(c.p + (ty + 16 * i) * (BT + 4) + j);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (tx + 16 * v) * 4;
        if (e >= groups * 4) continue;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float4 y = *(const float4*)(c.kv + (j + u) * ld + e);
#pragma unroll
          for (int i = 0; i < MR; ++i) {
            const float w = u == 0 ? p[i].x : u == 1 ? p[i].y : u == 2 ? p[i].z : p[i].w;
            o[i][v].x = fmaf(w, y.x, o[i][v].x); o[i][v].y = fmaf(w, y.y, o[i][v].y);
            o[i][v].z = fmaf(w, y.z, o[i][v].z); o[i][v].w = fmaf(w, y.w, o[i][v].w);
          }
        }
      }
    }
  }
  // sums over the row's sixteen threads, partial rows out
#pragma unroll
  for (int i = 0; i < MR; ++i) {
    float sum = l[i];
    int any = seen >> i & 1, masked = mixed, odd = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) odd |= !(isfinite(o[i][v].x) && isfinite(o[i][v].y) && isfinite(o[i][v].z) && isfinite(o[i][v].w));
#pragma unroll
    for (int off = 8; off; off >>= 1) {
      sum += __shfl_xor_sync(FULL, sum, off);
      any |= __shfl_xor_sync(FULL, any, off);
      masked |= __shfl_xor_sync(FULL, masked, off);
      odd |= __shfl_xor_sync(FULL, odd, off);
    }
    const int r = ty + 16 * i;
    if (r0 + r >= s.rows) continue;
    if (any && m[i] == NINF) m[i] = LOWEST;
    const RowAt a = row_at(P, s, r0 + r);
    const long long at = s.part + r0 + r;
    if (tx == 0) {
      if (s.whole) mark_row(P, s.mark + r0 + r, odd && masked);
      else P.part_ml[at] = make_float2(m[i], with_mark(sum, odd && masked));
    }
    const float inv = sum == 0.f ? (m[i] == NINF ? 0.f : __int_as_float(0x7fc00000)) : 1.f / sum;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const float y[4] = {o[i][v].x, o[i][v].y, o[i][v].z, o[i][v].w};
      const int e = (tx + 16 * v) * 4;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (e + u < dh) {
          if (s.whole) ((T*)P.out)[out_at(P, s, a) + e + u] = rr_from_f32<T>(y[u] * inv);
          else P.part_o[at * dh + e + u] = y[u];
        }
    }
  }
}

// Up to FEW rows: nothing to share but the loads, so no tiles.  A warp takes 8 loads of keys and 8 of values at a time, of 32 lanes
// x 4 entries (16 tokens of up to 64 entries, 8 tokens of more), all in flight at once behind the next ones' page look-up, for R rows: the
// dot products' halves are exchanged until a token's logit is left in LPT / 8 lanes, and its weight goes back to the
// token's lanes for the values.  A token that a row does not see is not multiplied, so no row is marked.  The warps' parts
// are joined at the end.  Bound by the cache's traffic (one query per row: through L2) and by latency.
template <typename T, int LPT, int W, int R, int WARPS>      // LPT lanes x W groups of 4 entries per token
__device__ void few_rows(const Params& P, const Seg& s, const Ctx& c, int r0, float* s_part) {
  constexpr int N = 8, TP = 32 / LPT, BLOCK = N * TP, ROW = LPT * W * 4, DUP = LPT / N;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane % LPT, grp = lane / LPT, dh = P.dh;
  float4 q[R][W], acc[R][W];
  int limit[R];
  float m[R], l[R];
  bool seen[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool live = r0 + r < s.rows;
    const RowAt a = live ? row_at(P, s, r0 + r) : RowAt{0, 0, 0};
    limit[r] = a.limit; m[r] = NINF; l[r] = 0.f; seen[r] = false;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int e = (sub + LPT * w) * 4;
      q[r][w] = live && e < dh ? load4<T>((const T*)P.q + q_at(P, s, a) + e, P.vq, dh - e) : make_float4(0.f, 0.f, 0.f, 0.f);
      acc[r][w] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  const int end = min(s.tile1 * TILE, c.n_tok);
  auto seek = [&](int num0, int& id, long long& at) {
    const int num = num0 + lane;
    id = NO_TOKEN;
    at = -1;
    if (lane >= BLOCK || num >= end) return;
    if (s.slots) {
      int lo = 0, hi = P.slots;
      while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (c.first[mid] <= num) lo = mid; else hi = mid; }
      id = c.base[lo] + num;
    } else {
      id = s.tok0 + num;
    }
    at = token_at(P, s, id);
    if (at < 0) id = NO_TOKEN;
  };
  int id, next_id;
  long long at, next_at;
  seek(s.tile0 * TILE + warp * BLOCK, next_id, next_at);
  for (int num0 = s.tile0 * TILE + warp * BLOCK; num0 < end; num0 += WARPS * BLOCK) {
    id = next_id; at = next_at;
    float4 x[N], y[N];
    auto load = [&](const void* from, int w, float4 (&z)[N]) {
      const int e = (sub + LPT * w) * 4;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const long long o = __shfl_sync(FULL, at, i * TP + grp);
        z[i] = o >= 0 && e < dh ? load4<T>((const T*)from + o + e, P.vk, dh - e) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    };
    if (W == 1) { load(P.k, 0, x); load(P.v, 0, y); }
    seek(num0 + WARPS * BLOCK, next_id, next_at);
    const int my_id = __shfl_sync(FULL, id, sub / DUP * TP + grp);     // lane's token: load sub / DUP of its group
    float wt[R];
    unsigned sees[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float d[N];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        if (W > 1) load(P.k, w, x);
#pragma unroll
        for (int i = 0; i < N; ++i)
          d[i] = fmaf(q[r][w].w, x[i].w, fmaf(q[r][w].z, x[i].z, fmaf(q[r][w].y, x[i].y, fmaf(q[r][w].x, x[i].x, w ? d[i] : 0.f))));
      }
#pragma unroll
      for (int n = N / 2, off = LPT / 2; n >= 1; n >>= 1, off >>= 1) {
        const bool up = sub & off;
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const float keep = up ? d[i + n] : d[i], give = up ? d[i] : d[i + n];
          d[i] = keep + __shfl_xor_sync(FULL, give, off);
        }
      }
      float z = d[0];
#pragma unroll
      for (int off = DUP / 2; off; off >>= 1) z += __shfl_xor_sync(FULL, z, off);
      const bool see = my_id < limit[r];
      sees[r] = __ballot_sync(FULL, see);
      z = see ? z * P.scale_log2 : NINF;
      float top = z;
#pragma unroll
      for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, off));
      const float m_new = fmaxf(m[r], top), ref = m_new == NINF ? 0.f : m_new, f = exp2f(m[r] - ref);
      seen[r] = seen[r] || sees[r] != 0;
      m[r] = m_new;
      wt[r] = exp2f(z - ref);
      l[r] = fmaf(l[r], f, sub % DUP ? 0.f : wt[r]);
#pragma unroll
      for (int w = 0; w < W; ++w) { acc[r][w].x *= f; acc[r][w].y *= f; acc[r][w].z *= f; acc[r][w].w *= f; }
    }
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (W > 1) load(P.v, w, y);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int from = grp * LPT + i * DUP;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float u = __shfl_sync(FULL, wt[r], from);
          if (sees[r] >> from & 1) {
            acc[r][w].x = fmaf(u, y[i].x, acc[r][w].x); acc[r][w].y = fmaf(u, y[i].y, acc[r][w].y);
            acc[r][w].z = fmaf(u, y[i].z, acc[r][w].z); acc[r][w].w = fmaf(u, y[i].w, acc[r][w].w);
          }
        }
      }
    }
  }
  // the warp's parts: outputs over the groups of lanes, sums over the lanes; then the warps'
  __syncthreads();                                     // (what was in this memory has been read)
  float2* const s_ml = (float2*)(s_part + WARPS * R * ROW);
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int off = 16; off; off >>= 1) l[r] += __shfl_xor_sync(FULL, l[r], off);
    if (seen[r] && m[r] == NINF) m[r] = LOWEST;
    if (lane == 0) s_ml[warp * R + r] = make_float2(m[r], l[r]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (TP == 2) {
        acc[r][w].x += __shfl_xor_sync(FULL, acc[r][w].x, 16); acc[r][w].y += __shfl_xor_sync(FULL, acc[r][w].y, 16);
        acc[r][w].z += __shfl_xor_sync(FULL, acc[r][w].z, 16); acc[r][w].w += __shfl_xor_sync(FULL, acc[r][w].w, 16);
      }
      if (grp == 0) *(float4*)(s_part + (warp * R + r) * ROW + (sub + LPT * w) * 4) = acc[r][w];
    }
  }
  __syncthreads();
  const int live = min(R, s.rows - r0);
  for (int u = threadIdx.x; u < live * dh; u += WARPS * 32) {
    const int r = u / dh, e = u - r * dh;
    float M = NINF, L = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) M = fmaxf(M, s_ml[w * R + r].x);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float2 ml = s_ml[w * R + r];
      if (ml.x == NINF) continue;
      const float f = exp2f(ml.x - M);
      L = fmaf(f, ml.y, L);
      o = fmaf(f, s_part[(w * R + r) * ROW + e], o);
    }
    const long long at = s.part + r0 + r;
    if (s.whole) {
      const float inv = L == 0.f ? (M == NINF ? 0.f : __int_as_float(0x7fc00000)) : 1.f / L;
      ((T*)P.out)[out_at(P, s, row_at(P, s, r0 + r)) + e] = rr_from_f32<T>(o * inv);
    } else {
      P.part_o[at * dh + e] = o;
      if (e == 0) P.part_ml[at] = make_float2(M, with_mark(L, false));
    }
  }
  __syncthreads();
}

// ONLY_FEW: a call whose items all have up to FEW rows needs no tiles in shared memory; CTAs of four warps, four to an SM, have more
// segments' latencies side by side (2048 rows of 396 tokens, fp32, dh 64: 98 us with eight warps and two to an SM, 75 us).
constexpr int FEW_NT = 128;
template <typename T, int NV, bool ONLY_FEW>
__global__ void __launch_bounds__(ONLY_FEW ? FEW_NT : SNT, ONLY_FEW ? 4 : 2) attend_simt_kernel(const __grid_constant__ Params P) {
  extern __shared__ __align__(16) uint8_t smem[];
  rr_pdl_wait();
  rr_pdl_trigger();
  const SmemPlan L = smem_plan(P.dh, P.slots, ONLY_FEW);
  Ctx c;
  c.q = (float*)(smem + L.q); c.kv = (float*)(smem + L.kv); c.p = (float*)(smem + L.p);
  c.at = (long long*)(smem + L.ids); c.id = (int*)(c.at + BT);
  c.first = (int*)(smem + L.slots); c.base = c.first + P.slots + 1;
  c.n_tok = 0;
  const int lane = threadIdx.x & 31;
  long long u, u1;
  const bool turns = P.slots && !P.units;              // whole items in turn
  const long long W = P.slots ? range_units(P) : __ldg(P.main.cum + P.batch);
  if (turns) { u = blockIdx.x; u1 = W; }
  else { u = share(P.main, blockIdx.x, W); u1 = share(P.main, blockIdx.x + 1, W); }
  while (u < u1) {
    Seg s;
    if (P.slots) {
      const int took = range_segment(P, P.main, blockIdx.x, u, u1, s);
      u += turns ? gridDim.x : took;
      __syncthreads();                                 // the table before is no longer read
      if (threadIdx.x < 32) {
        if (lane == 0) check_len(P, s.b);
        int run = 0;
        for (int j0 = 0; j0 < P.slots; j0 += 32) {
          const int j = j0 + lane;
          int lo = 0, hi = 0;
          if (j < P.slots) slot_span(s, j, lo, hi);
          int incl = hi - lo;
#pragma unroll
          for (int off = 1; off < 32; off <<= 1) { const int x = __shfl_up_sync(FULL, incl, off); if (lane >= off) incl += x; }
          if (j < P.slots) { c.first[j] = run + incl - (hi - lo); c.base[j] = lo - c.first[j]; }
          run += __shfl_sync(FULL, incl, 31);
        }
        if (lane == 0) c.first[P.slots] = run;
      }
      __syncthreads();
      c.n_tok = c.first[P.slots];
      unit_tiles(P, (c.n_tok + TILE - 1) / TILE, s);
    } else {
      u += segment_at(P, P.main, blockIdx.x, u, u1, s);
      c.n_tok = s.tok1 - s.tok0;
    }
    constexpr int LPT = NV == 1 ? 16 : 32, W = NV > 2 ? 2 : 1, R = W == 1 ? 4 : 1, WARPS = (ONLY_FEW ? FEW_NT : SNT) / 32;
    if (ONLY_FEW || s.rows <= FEW) {
      if (s.rows == 1) few_rows<T, LPT, W, 1, WARPS>(P, s, c, 0, c.q);
      else for (int r0 = 0; r0 < s.rows; r0 += R) few_rows<T, LPT, W, R, WARPS>(P, s, c, r0, c.q);
    } else if constexpr (!ONLY_FEW) {
      if (s.rows <= 16) rows_block<T, NV, 1>(P, s, c, 0);
      else for (int r0 = 0; r0 < s.rows; r0 += 64) rows_block<T, NV, 4>(P, s, c, r0);
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------------------
template <typename T>
cudaError_t launch_simt(const Params& P, int grid, cudaStream_t st) {
  const bool few = P.slots && P.m * P.group <= FEW;
  const SmemPlan L = smem_plan(P.dh, P.slots, few);
  auto go = [&](auto kernel, unsigned long long& done) {
    cudaError_t e = rr_once_per_device(done, [&] {
      return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_plan(RR_PAGED_MAX_DH, RR_MAX_RANGE_SLOTS, false).total);
    });
    if (e != cudaSuccess) return e;
    return rr_launch_pdl(kernel, grid, few ? FEW_NT : SNT, (size_t)L.total, st, P);
  };
  static unsigned long long done[8];
  switch ((P.dh + 63) / 64 + (few ? 4 : 0)) {
    case 1: return go(attend_simt_kernel<T, 1, false>, done[0]);
    case 2: return go(attend_simt_kernel<T, 2, false>, done[1]);
    case 3: return go(attend_simt_kernel<T, 3, false>, done[2]);
    case 4: return go(attend_simt_kernel<T, 4, false>, done[3]);
    case 5: return go(attend_simt_kernel<T, 1, true>, done[4]);
    case 6: return go(attend_simt_kernel<T, 2, true>, done[5]);
    case 7: return go(attend_simt_kernel<T, 3, true>, done[6]);
    default: return go(attend_simt_kernel<T, 4, true>, done[7]);
  }
}

size_t up(size_t x) { return (x + 255) / 256 * 256; }
// Rows that a whole item may write without partials and mark.
size_t mark_rows(const Params& P) {
  if (P.in_place) return 0;
  if (P.slots) return P.few.ctas == 0 && leaves_marks(P, (long long)P.m * P.group) ? (size_t)P.range_rows * P.m * P.group : 0;
  return leaves_marks(P, (long long)P.tokens * P.group) ? (size_t)P.tokens * P.heads : 0;
}
// Offsets in the workspace: the plan, part_ml, part_o, marks.
size_t lay_out(Params& P, uint8_t* ws) {
  size_t at = 0;
  if (!P.slots) {
    P.main.cum = (long long*)(ws + at); at += up((size_t)(P.batch + 1) * 8);
    P.few.cum = (long long*)(ws + at); at += up((size_t)(P.batch + 1) * 8);
    P.plan = (Plan*)(ws + at); at += up(sizeof(Plan));
  }
  const size_t rows = (size_t)P.part_rows;
  P.part_ml = (float2*)(ws + at); at += up(rows * sizeof(float2));
  P.part_o = (float*)(ws + at); at += up(rows * P.dh * sizeof(float));
  P.marks = ws + at; at += up(mark_rows(P));
  return at;
}

void groups_of_four(Params& P, int dtype) {
  const uintptr_t b = dtype == RR_BF16 ? 7 : 15;
  P.vq = P.dh % 4 == 0 && ((uintptr_t)P.q & b) == 0 && (P.qb | P.qh | P.qt) % 4 == 0;
  P.vk = P.dh % 4 == 0 && (((uintptr_t)P.k | (uintptr_t)P.v) & b) == 0 && (P.page_stride | P.head_stride | P.token_stride) % 4 == 0;
}

int fill(const rr_paged_kv* kv, Params& P) {
  const int rc = rr_paged_check(kv);
  if (rc != RR_OK) return rc;
  P = Params{};
  P.k = kv->k; P.v = kv->v; P.table = kv->page_table; P.status = kv->status;
  P.page_stride = kv->page_stride; P.head_stride = kv->head_stride; P.token_stride = kv->token_stride; P.table_stride = kv->table_stride;
  P.num_pages = kv->num_pages; P.page_tokens = kv->page_tokens; P.kv_heads = kv->kv_heads; P.dh = kv->dh;
  P.batch = kv->batch; P.pages_per_seq = kv->pages_per_seq;
  P.page_shift = -1;
  for (int i = 0; i < 31; ++i) if (P.page_tokens == 1 << i) P.page_shift = i;
  // (the stride of a dimension of one entry says nothing)
  if (P.num_pages == 1) P.page_stride = 256;
  if (P.kv_heads == 1) P.head_stride = 256;
  if (P.page_tokens == 1) P.token_stride = 256;
  if ((long long)kv->pages_per_seq * kv->page_tokens > 0x7FFFFFFFLL - ROWS) return RR_ERR_TOO_LARGE;
  return RR_OK;
}

bool misaligned(const void* q, const void* out, int dtype) {
  return (((uintptr_t)q | (uintptr_t)out) & (dtype == RR_BF16 ? 1 : 3)) != 0;
}

// The partial rows of a call of `all` rows: items of several partials a row (`items` of up to `last` rows each), rows of an item at most; all_homes: every
// row is joined; prefix_homes: and has a partial of the prefix; main_shares: the main kernel's CTAs cut items.
// Few rows are quartered by the tensor cores' kernel where eight partials a row are no great workspace.
void lay_out_partials(Params& P, long long all, long long items, int last, int most, bool all_homes, bool prefix_homes, bool main_shares) {
  const int split = P.tc ? std::min(last, TILE) : 0, quart = P.tc && (!P.slots || last <= 32) ? std::min(last, 32) : 0;
  for (P.streams = P.tc ? 8 : 1;; P.streams = 2) {
    const int more = P.streams == 8 ? std::max(split, 7 * quart) : split;              // further partials of an item
    long long at = 0, further = 0;
    auto take = [&](long long n) { const long long a = at; at += n; return a; };
    auto take_more = [&](long long n) { further += n; return take(n); };
    P.all_homes = all_homes; P.more_rows = more; P.step = quart;
    if (prefix_homes) { take(all); take_more((long long)P.kv_heads * more); }
    P.own.home = take(all_homes ? all : std::min(items * split, all));
    P.own.home_per_item = !all_homes && items * split <= all ? split : 0;
    const long long by_row = (P.streams - 1) * all;
    P.own.more = take_more(std::min(items * more, by_row));
    P.own.more_per_item = items * more <= by_row ? more : 0;
    P.own.step = (int)(items * more <= by_row ? quart : all);
    auto places = [&](Sched& sc, int rows, int m) {
      sc.slot_rows = rows;
      sc.more_at = all_homes ? rows : 2 * rows;
      sc.cta_rows = sc.more_at + m;
      sc.slots_at = take((long long)sc.ctas * sc.cta_rows);
      further += (long long)sc.ctas * m;
    };
    if (main_shares) places(P.main, most, more);
    if (P.few.ctas > 0 && (!P.slots || P.units)) places(P.few, std::min(most, FEW_ROWS), 0);
    P.part_rows = at;
    if (P.streams != 8 || further * P.dh * 4 <= 192LL << 20) return;
  }
}

int fill_shared(const rr_paged_kv* kv, const rr_shared_args* a, Params& P) {
  const int rc = fill(kv, P);
  if (rc != RR_OK) return rc;
  if (!a || !a->q || !a->out || !a->lens) return RR_ERR_INVALID_ARG;
  if (a->tokens < 0 || (!a->cu && a->tokens != kv->batch) || a->heads < 1 || a->heads % kv->kv_heads != 0) return RR_ERR_INVALID_ARG;
  if (a->prefix_tokens < 0 || (a->causal != 0 && a->causal != 1) || !std::isfinite(a->scale)) return RR_ERR_INVALID_ARG;
  if (!a->prefix_pages && a->prefix_tokens > (long long)kv->pages_per_seq * kv->page_tokens) return RR_ERR_INVALID_ARG;
  if (a->prefix_tokens > 0x7FFFFFFF - ROWS) return RR_ERR_TOO_LARGE;
  if (a->q_token_stride < 0 || a->q_head_stride < 0 || a->out_token_stride < 0 || a->out_head_stride < 0) return RR_ERR_INVALID_ARG;
  if (misaligned(a->q, a->out, kv->dtype) || (((uintptr_t)a->lens | (uintptr_t)a->cu | (uintptr_t)a->prefix_pages) & 3)) return RR_ERR_INVALID_ARG;
  if ((long long)a->tokens * a->heads > (1LL << 30)) return RR_ERR_TOO_LARGE;
  P.q = a->q; P.out = a->out; P.lens = a->lens; P.cu = a->cu; P.prefix_pages = a->prefix_pages;
  P.qt = a->q_token_stride; P.qh = a->q_head_stride; P.ot = a->out_token_stride; P.oh = a->out_head_stride;
  P.in_place = a->q == a->out;
  if (P.in_place && ((a->tokens > 1 && P.qt != P.ot) || (a->heads > 1 && P.qh != P.oh))) return RR_ERR_INVALID_ARG;
  P.tokens = a->tokens; P.heads = a->heads; P.group = a->heads / kv->kv_heads; P.causal = a->causal; P.prefix = a->prefix_tokens;
  P.scale_log2 = a->scale * 1.4426950408889634f;
  P.tc = rr_attend_tc_supported(P, kv->dtype);
  groups_of_four(P, kv->dtype);
  P.main.ctas = rr_sm_count() * (P.tc ? 1 : 2);
  if (P.tc && P.group <= FEW_ROWS) {
    // (three CTAs fit an SM; two rounds of them even out segments of unlike lengths: 64 sequences of 1 to 2000 tokens 172 -> 156 us, three: 163)
    P.few.ctas = rr_sm_count() * 6;
    P.few_prefix = (long long)P.tokens * P.group <= FEW_ROWS;
  }
  const long long rows = (long long)P.tokens * P.group, packed = ceil_div(rows, ROWS);
  // up to four rows in all, or one token of each sequence and no prefix to share: the few kernel has everything
  P.few_waits = P.few.ctas > 0 && (P.few_prefix || (!P.cu && P.prefix == 0));
  // (the sequences' row tiles are at most one less per sequence more than those of all rows together)
  P.always_apart = P.prefix == 0 || P.batch - 1 <= packed / 8;
  const int most = (int)std::min<long long>(ROWS, rows);
  lay_out_partials(P, (long long)P.tokens * P.heads, P.few_waits ? 0 : (long long)P.batch * P.kv_heads, std::min(most, TILE), most,
                   P.in_place || !P.always_apart, !P.always_apart, !P.few_waits);
  return RR_OK;
}

int fill_ranges(const rr_paged_kv* kv, const rr_ranges_args* a, Params& P) {
  const int rc = fill(kv, P);
  if (rc != RR_OK) return rc;
  if (!a || !a->q || !a->out || !a->lens || !a->ranges) return RR_ERR_INVALID_ARG;
  if (a->heads < 1 || a->route_heads < 1 || a->n_q < 1 || a->m < 1 || a->slots < 1) return RR_ERR_INVALID_ARG;
  if (a->route_heads % kv->kv_heads != 0 || a->heads % a->route_heads != 0) return RR_ERR_INVALID_ARG;
  if ((a->causal != 0 && a->causal != 1) || !std::isfinite(a->scale)) return RR_ERR_INVALID_ARG;
  if (a->q_batch_stride < 0 || a->q_head_stride < 0 || a->q_token_stride < 0 || a->out_batch_stride < 0 || a->out_head_stride < 0 || a->out_token_stride < 0)
    return RR_ERR_INVALID_ARG;
  if (misaligned(a->q, a->out, kv->dtype) || (((uintptr_t)a->lens | (uintptr_t)a->ranges) & 3)) return RR_ERR_INVALID_ARG;
  if (a->slots > RR_MAX_RANGE_SLOTS || (long long)a->slots * kv->pages_per_seq * kv->page_tokens > 0x7FFFFFFFLL - ROWS) return RR_ERR_TOO_LARGE;
  if ((long long)a->n_q * a->m > 0x7FFFFFFFLL - ROWS || (long long)a->m * (a->heads / a->route_heads) > 0x7FFFFFFFLL - ROWS) return RR_ERR_TOO_LARGE;
  const double all = (double)kv->batch * a->heads * a->n_q * a->m;
  if (all > (double)(1LL << 30)) return RR_ERR_TOO_LARGE;
  P.q = a->q; P.out = a->out; P.lens = a->lens; P.ranges = a->ranges;
  P.qb = a->q_batch_stride; P.qh = a->q_head_stride; P.qt = a->q_token_stride;
  P.ob = a->out_batch_stride; P.oh = a->out_head_stride; P.ot = a->out_token_stride;
  P.in_place = a->q == a->out;
  if (P.in_place && ((kv->batch > 1 && P.qb != P.ob) || (a->heads > 1 && P.qh != P.oh) || (all > (double)kv->batch * a->heads && P.qt != P.ot)))
    return RR_ERR_INVALID_ARG;
  P.heads = a->heads; P.route_heads = a->route_heads; P.group = a->heads / a->route_heads; P.causal = a->causal;
  P.n_q = a->n_q; P.m = a->m; P.slots = a->slots;
  P.scale_log2 = a->scale * 1.4426950408889634f;
  P.range_rows = (long long)kv->batch * a->route_heads * a->n_q;
  P.tc = rr_attend_tc_supported(P, kv->dtype);
  groups_of_four(P, kv->dtype);
  const int mg = P.m * P.group, last = mg - (mg - 1) / ROWS * ROWS;              // rows of an item's last row tile
  const long long items = P.range_rows * ceil_div(mg, ROWS);
  P.few_waits = P.tc && mg <= FEW_ROWS;
  if (P.few_waits) P.tc = 0;
  P.main.ctas = rr_sm_count() * (P.tc ? 1 : mg <= FEW ? 4 : 2);
  // (three CTAs fit an SM; more of them lose: 2048 rows of 396 tokens 52 us, with nine 61)
  if (P.few_waits) P.few.ctas = rr_sm_count() * 3;
  P.units = items < 8LL * (P.few_waits ? P.few : P.main).ctas ? UNITS : 0;
  lay_out_partials(P, P.range_rows * mg, P.tc && last <= TILE ? P.range_rows : 0, last <= TILE ? last : 0, std::min(ROWS, mg), P.in_place, false, P.units && !P.few_waits);
  return RR_OK;
}

int run(Params& P, int dtype, void* workspace, size_t bytes, cudaStream_t st, const char* what) {
  const size_t need = lay_out(P, (uint8_t*)workspace);
  if (need && !workspace) return RR_ERR_INVALID_ARG;
  if ((uintptr_t)workspace & 255) return RR_ERR_INVALID_ARG;
  if (bytes < need) return RR_ERR_TOO_SMALL;
  cudaError_t e = cudaSuccess;
  int launches = 0;
  if (!P.slots) { e = rr_launch_pdl(plan_kernel, 1, PLAN_NT, 0, st, P); ++launches; }
  const bool few = P.few.ctas > 0, only_few = P.few_waits;
  if (e == cudaSuccess && !only_few) {
    long long grid = P.main.ctas;
    if (P.slots && !P.units) grid = std::min<long long>(grid, P.range_rows * ceil_div((long long)P.m * P.group, ROWS));
    if (P.tc) e = rr_launch_attend_tc(P, (int)grid, st);
    else e = dtype == RR_BF16 ? launch_simt<__nv_bfloat16>(P, (int)grid, st) : launch_simt<float>(P, (int)grid, st);
    ++launches;
  }
  if (e == cudaSuccess && few) {
    e = rr_launch_attend_few(P, P.slots ? P.m * P.group : P.few_prefix ? P.tokens * P.group : P.cu ? FEW_ROWS : P.group, st);
    ++launches;
  }
  if (e == cudaSuccess && P.part_rows > 0) {
    const long long rows = P.slots ? P.range_rows * P.m * P.group : (long long)P.tokens * P.heads;
    const bool few = rows < 8 * rr_sm_count();
    const int grid = (int)(few ? rows : ceil_div(rows, 8));
    const bool marks = !only_few && (P.tc || (P.slots ? (long long)P.m : P.tokens) * P.group > FEW);
    auto join = [&](auto type, auto look) {
      using T = decltype(type);
      constexpr bool M = decltype(look)::value;
      return rr_launch_pdl(few ? join_kernel<T, 8, M> : join_kernel<T, 1, M>, grid, 256, 0, st, P);
    };
    auto typed = [&](auto look) { return dtype == RR_BF16 ? join(__nv_bfloat16(), look) : join(0.f, look); };
    e = marks ? typed(std::true_type()) : typed(std::false_type());
    ++launches;
  }
  if (e == cudaSuccess && P.slots && P.part_rows == 0 && !P.tc && mark_rows(P) > 0) {
    const int grid = (int)std::min<long long>(ceil_div(mark_rows(P), 16 * 256), 2 * rr_sm_count());
    e = dtype == RR_BF16 ? rr_launch_pdl(marked_kernel<__nv_bfloat16>, grid, 256, 0, st, P) : rr_launch_pdl(marked_kernel<float>, grid, 256, 0, st, P);
    ++launches;
  }
  rr_count_launch(launches);
  if (e == cudaSuccess) e = cudaPeekAtLastError();
  return e == cudaSuccess ? RR_OK : rr_cuda_fail(e, what);
}

}  // namespace

extern "C" {

int rr_attend_shared_workspace(const rr_paged_kv* kv, const rr_shared_args* a, size_t* bytes) {
  if (!bytes) return RR_ERR_INVALID_ARG;
  Params P;
  const int rc = fill_shared(kv, a, P);
  if (rc == RR_OK) *bytes = lay_out(P, nullptr);
  return rc;
}

int rr_attend_shared(const rr_paged_kv* kv, const rr_shared_args* a, void* workspace, size_t bytes, void* stream) {
  Params P;
  const int rc = fill_shared(kv, a, P);
  if (rc != RR_OK) return rc;
  if (a->tokens == 0) return RR_OK;
  return run(P, kv->dtype, workspace, bytes, (cudaStream_t)stream, "rr_attend_shared");
}

int rr_attend_paged_ranges_workspace(const rr_paged_kv* kv, const rr_ranges_args* a, size_t* bytes) {
  if (!bytes) return RR_ERR_INVALID_ARG;
  Params P;
  const int rc = fill_ranges(kv, a, P);
  if (rc == RR_OK) *bytes = lay_out(P, nullptr);
  return rc;
}

int rr_attend_paged_ranges(const rr_paged_kv* kv, const rr_ranges_args* a, void* workspace, size_t bytes, void* stream) {
  Params P;
  const int rc = fill_ranges(kv, a, P);
  if (rc != RR_OK) return rc;
  return run(P, kv->dtype, workspace, bytes, (cudaStream_t)stream, "rr_attend_paged_ranges");
}

}  // extern "C"
