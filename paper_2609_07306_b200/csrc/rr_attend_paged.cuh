// Attention over a paged key/value cache: how the work of rr_attend_shared and rr_attend_paged_ranges is cut
// into segments, where a segment's partial results go, and how they are joined.  Three kernels process segments: the tensor cores'
// (rr_attend_paged_tc.cu), one for up to four rows of the same types (rr_attend_paged_few.cu) and the one for every other type and width
// (rr_attend_paged.cu).
//
// An ITEM is up to ROWS query rows that attend to one list of tokens of one key head:
//   shared, prefix   the queries of all sequences and of the G = heads / kv_heads query heads of a key head (row t * G + g),
//                    over the prefix's tokens
//   shared, own      the same rows of one sequence, over its tokens behind the prefix
//   shared, apart    where the sequences' own rows fill their tiles about as well as all rows together (prompts), there is nothing to share but
//                    L2's copy of the prefix: the rows of one sequence over all of its tokens, and a row has one partial less
//   ranges           the m * G queries of a range row, over the tokens of its slots
// A list is walked in tiles of TILE tokens.  A SEGMENT is a run of tiles of an item; it leaves per row a
// partial result: reference maximum m (of logit * log2 e), sum l of 2^(x - m), and the unnormalised output.  The partials
// of a row are joined in a fixed order by join_kernel.
//
// shared: the tiles of all items in one row, N CTAs take equal shares of it (an item may be cut anywhere, a
// CTA's share may span many items), so neither a long prefix of few rows nor one long sequence among short ones leaves SMs idle.
// plan_kernel counts the tiles on the device, where the lengths are, for the few-row kernel's items and the others apart.  A CTA has at most one segment
// that does not begin its item and one that begins an item without ending it; their partial rows have places of the CTA's own.  Items whose rows are joined
// although no CTA cuts them (behind a prefix, or of several partials) have homes by their rows.
// ranges: items are alike.  Where there are fewer than eight per CTA each counts as UNITS units that the CTAs share equally, as the tiles above (a
// segment has the tiles of its units by the item's own number of tiles); where there are more, CTAs take whole items in turn, so that
// neighbouring rows, whose routes overlap, are read at the same time.
#pragma once
#include "rr_paged.cuh"

namespace rrattn {

constexpr int TILE = 128, ROWS = 256, UNITS = 64, FEW_ROWS = 4;
constexpr int NO_TOKEN = 0x7FFFFFFF;                   // id of a place without a token: above every limit
constexpr float NINF = -__builtin_huge_valf();
constexpr float LOWEST = -3.402823466e38f;             // m of a row that saw tokens, all of them at -inf

// Who shares the items: CTAs, the tiles before each sequence's items, and the CTAs' own places among the partial rows: for the segment that does not begin
// its item, behind it for one that begins an item without a home, and behind both for the first one's further partials.
struct Sched {
  int ctas, slot_rows, more_at, cta_rows;              // rows of a segment's place; where a CTA's further partials begin; rows of a CTA's places
  long long* cum;                                      // shared: [batch + 1] tiles before sequence b's items; [batch] = all tiles
  long long slots_at;
};

// Homes of rows among the partial rows: of all rows (Params::all_homes), else of those of items whose segments leave several partials; further
// partials are in `more`, `step` apart.  An item of several partials is a sequence's (or range row's) last row tile with a key head, at most
// 128 rows: homes go by that (per_item rows each), or by the row's index (per_item == 0).  Of the prefix's items all rows have homes, by the
// row's index from 0 on, and behind these the last row tile of each key head has its further partials, Params::more_rows rows.
struct Homes {
  long long home, more;
  int home_per_item, more_per_item, step;
};

// What plan_kernel finds out from the lengths besides the tiles before each sequence's items.
struct Plan {
  int apart;                                           // the sequences attend by themselves, to the prefix too
  int source;                                          // whose row of the table has the prefix's pages
  int prefix;                                          // tokens of the prefix that any sequence has
  int marked;                                          // a row without partials has been marked since
};

struct Params {
  // cache
  const void *k, *v;
  const int32_t* table;
  uint32_t* status;
  long long page_stride, head_stride, token_stride, table_stride;
  int num_pages, page_tokens, page_shift, kv_heads, dh, batch, pages_per_seq;   // page_shift: log2 of page_tokens, -1 if it is no power of two
  // queries
  const void* q;
  void* out;
  long long qb, qh, qt, ob, oh, ot;                    // strides: batch (ranges), head, token
  const int32_t *lens, *cu, *prefix_pages, *ranges;
  int tokens, heads, group, causal;                    // group: query heads of an item
  int prefix;                                          // shared
  int n_q, m, slots, route_heads;                      // ranges (slots > 0)
  float scale_log2;                                    // scale * log2 e
  // schedule
  Sched main, few;                                     // few: items of up to FEW_ROWS rows in a kernel of their own (ctas == 0: no such kernel)
  int tc, units, streams;                              // units: of a ranges item (0: whole items in turn); streams: most partials of a segment's row
  bool few_prefix;                                     // the few kernel has the prefix's items, too: all queries make up to FEW_ROWS rows
  int few_waits;                                       // the few kernel has everything, its inputs are its predecessor's (else it only ends after that)
  int always_apart;                                    // whatever the lengths are
  long long range_rows;                                // batch * route_heads * n_q
  // workspace
  Plan* plan;                                          // shared
  float* part_o;                                       // [part_rows][dh]
  float2* part_ml;                                     // [part_rows]
  long long part_rows;
  Homes own;
  int all_homes, more_rows, step;                      // further partials of a CTA's segment or a prefix item: rows, `step` apart
  uint8_t* marks;                                      // of rows that are written without partials: [tokens * heads] or [range_rows * m * group]
  int vq, vk;                                          // queries / cache rows split into aligned groups of four
  int in_place;                                        // the output is the queries' memory: only the join writes it, a row at a time
};

struct Seg {
  int rows, row0;                                      // rows row0 .. row0 + rows - 1 of the item's group, row = (t - t_base) * group + g
  int t_base, t_seq0, n_seq;                           // first token; own / ranges: first token and number of the sequence's queries
  int b;                                               // sequence, -1: prefix (rows of all sequences)
  int kvh, h0;                                         // key head, first query head
  int tok0, tok1;                                      // dense: the list's tokens
  const int32_t* pages;                                // page list of the tokens, from token `prefix` on
  const int32_t* prefix_pages;
  int prefix;
  bool whole;                                          // all tiles of the rows' only item, nothing to join: the segment writes the output
  const int32_t* slots;                                // ranges: the row's slots, else null
  int tile0, tile1;                                    // the segment's tiles of the list (ranges: once counted)
  int unit0, unit1;                                    // ranges: the segment's units of the item's `units` (of 1 if whole)
  long long part, more;                                // partial row of row 0; of its further partials, `step` apart
  int step;
  long long mark;                                      // row 0's place among the marks
};

// a / b for a >= 0, b > 0; mostly both fit 32 bits, whose division takes a fifth of the time
__host__ __device__ inline long long quot(long long a, long long b) {
  return ((unsigned long long)(a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
__host__ __device__ inline long long ceil_div(long long a, long long b) { return quot(a + b - 1, b); }

// Tokens that sequence b has by its length, and of these those that have places: its table's, and the prefix's, which may have pages of its own.
__device__ __forceinline__ int seq_end(const Params& P, int b) { return max(__ldg(P.lens + b), 0); }
__device__ __forceinline__ int seq_len(const Params& P, int b) {
  const long long cap = max((long long)P.pages_per_seq * P.page_tokens, (long long)P.prefix);
  const int n = seq_end(P, b);
  return n > cap ? (int)cap : n;
}
__device__ __forceinline__ int seq_first(const Params& P, int b) { return P.cu ? __ldg(P.cu + b) : b; }
__device__ __forceinline__ int seq_count(const Params& P, int b) {
  if (!P.cu) return 1;
  const int a = __ldg(P.cu + b), e = min(__ldg(P.cu + b + 1), P.tokens);
  return a < 0 ? 0 : max(e - a, 0);
}
__device__ __forceinline__ Plan plan_of(const Params& P) {
  const int4 x = __ldg((const int4*)P.plan);
  return Plan{x.x, x.y, x.z, x.w};
}
__device__ __forceinline__ long long prefix_tiles(const Plan& plan) { return plan.apart ? 0 : (plan.prefix + TILE - 1) / TILE; }
__device__ __forceinline__ long long prefix_row_tiles(const Params& P) { return ceil_div((long long)P.tokens * P.group, ROWS); }
__device__ __forceinline__ int own_tiles(const Params& P, int b, bool apart) { return (max(seq_len(P, b) - (apart ? 0 : P.prefix), 0) + TILE - 1) / TILE; }
__device__ __forceinline__ int own_row_tiles(const Params& P, int b) { return (int)ceil_div((long long)seq_count(P, b) * P.group, ROWS); }

__device__ __forceinline__ bool few_rows_of(const Params& P, int b) { return P.few.ctas > 0 && (long long)seq_count(P, b) * P.group <= FEW_ROWS; }

// With N = min(ctas, W) CTAs at work, CTA c's share of W tiles is [c W / N, (c + 1) W / N), at least one tile: an item that
// is cut is in consecutive CTAs.  cta_of: the CTA that has tile u.
__device__ __forceinline__ long long share(const Sched& sc, int c, long long W) {
  const long long N = min((long long)sc.ctas, W);
  return c >= N ? W : quot(c * W, N);
}
__device__ __forceinline__ int cta_of(const Sched& sc, long long u, long long W) {
  const long long N = min((long long)sc.ctas, W);
  return (int)(ceil_div((u + 1) * N, W) - 1);
}

// Partials that a segment of `rows` rows leaves per row.
__host__ __device__ inline int partials_of(int streams, long long rows) { return streams == 1 || rows > TILE ? 1 : streams > 2 && rows <= 32 ? 8 : 2; }

// The home of row `at` of all, row r of its row tile, item `item` of several partials: its first partial (-1: none) and its further ones.
__device__ __forceinline__ long long home_of(const Params& P, bool several, long long item, long long at, int r) {
  return P.all_homes || several ? P.own.home + (P.own.home_per_item ? item * P.own.home_per_item + r : at) : -1;
}
__device__ __forceinline__ long long more_of(const Params& P, long long item, long long at, int r) { return P.own.more + (P.own.more_per_item ? item * P.own.more_per_item + r : at); }
__device__ __forceinline__ long long prefix_more_of(const Params& P, int kvh, int r) { return (long long)P.tokens * P.heads + (long long)kvh * P.more_rows + r; }
// Where a segment's partials go (s.mark: the index of its row 0).
__device__ __forceinline__ void place_segment(const Params& P, const Sched& sc, int c, bool begins, long long item, Seg& s) {
  const long long cta = sc.slots_at + (long long)c * sc.cta_rows;
  if (!begins) {
    s.part = cta; s.more = cta + sc.more_at; s.step = P.step;
  } else if (s.b < 0) {
    s.part = s.mark; s.more = prefix_more_of(P, s.kvh, 0); s.step = P.step;
  } else {
    const bool several = &sc == &P.main && partials_of(P.streams, s.rows) > 1;
    s.part = home_of(P, several, item, s.mark, 0);
    if (s.part < 0) s.part = cta + sc.slot_rows;
    s.more = more_of(P, item, s.mark, 0); s.step = P.own.step;
  }
}

// The segment at tile u of CTA c's share, which ends at u1; returns how many tiles of the share it takes.
__device__ __forceinline__ int segment_at(const Params& P, const Sched& sc, int c, long long u, long long u1, Seg& s) {
  const Plan plan = plan_of(P);
  const bool apart = plan.apart;
  const long long np = prefix_tiles(plan), qtp = prefix_row_tiles(P), before = (&sc == &P.few) == P.few_prefix ? P.kv_heads * qtp * np : 0;
  long long first;                                     // first tile of the item
  int tiles;
  const long long row_all = (long long)P.tokens * P.group;
  s.slots = nullptr;
  s.prefix_pages = P.prefix_pages ? P.prefix_pages : P.table + plan.source * P.table_stride;
  s.prefix = P.prefix;
  if (u < before) {
    const long long item = quot(u, np);
    first = item * np;
    tiles = (int)np;
    s.kvh = (int)quot(item, qtp);
    s.row0 = (int)(item - s.kvh * qtp) * ROWS;
    s.rows = (int)min((long long)ROWS, row_all - s.row0);
    s.b = -1;
    s.t_base = 0; s.t_seq0 = 0; s.n_seq = 0;
    s.tok0 = 0; s.tok1 = plan.prefix;
    s.pages = s.prefix_pages;
  } else {
    int lo = 0, hi = P.batch;                          // last b with cum[b] <= u
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (__ldg(sc.cum + mid) <= u) lo = mid; else hi = mid; }
    const int b = lo, qt = own_row_tiles(P, b);
    tiles = own_tiles(P, b, apart);
    const long long base = __ldg(sc.cum + b), item = quot(u - base, tiles);
    first = base + item * tiles;
    s.kvh = (int)quot(item, qt);
    s.row0 = (int)(item - (long long)s.kvh * qt) * ROWS;
    s.n_seq = seq_count(P, b);
    s.rows = (int)min((long long)ROWS, (long long)s.n_seq * P.group - s.row0);
    s.b = b;
    s.t_base = s.t_seq0 = seq_first(P, b);
    s.tok0 = apart ? 0 : P.prefix; s.tok1 = seq_len(P, b);
    s.pages = P.table + b * P.table_stride;
  }
  s.mark = s.kvh * row_all + (long long)s.t_base * P.group + s.row0;
  s.h0 = s.kvh * P.group;
  s.tile0 = (int)(u - first);
  s.tile1 = (int)min((long long)tiles, u1 - first);
  const int took = s.tile1 - s.tile0;
  s.whole = took == tiles && u >= before && np == 0 && !P.in_place;
  if (P.causal && s.b >= 0) {                          // no row sees the tiles from the last row's limit on
    const long long limit = (long long)seq_end(P, s.b) - s.n_seq + (s.row0 + s.rows - 1) / P.group + 1;
    s.tile1 = max(s.tile0, limit <= s.tok0 ? 0 : (int)min((long long)s.tile1, (limit - s.tok0 + TILE - 1) / TILE));
  }
  place_segment(P, sc, c, s.tile0 == 0, (long long)s.b * P.kv_heads + s.kvh, s);
  return took;
}

// The segment at unit u (item u, if they are taken whole) of CTA c's share of a ranges call; its tiles are counted by who reads the
// slots.  Returns how many units it takes.
__device__ __forceinline__ int range_segment(const Params& P, const Sched& sc, int c, long long u, long long u1, Seg& s) {
  const int mg = P.m * P.group, qt = (mg + ROWS - 1) / ROWS, n = P.units ? P.units : 1;
  const long long item = quot(u, n), row = quot(item, qt);
  s.unit0 = (int)(u - item * n);
  s.unit1 = (int)min((long long)n, u1 - item * n);
  s.whole = s.unit1 - s.unit0 == n && !P.in_place;
  s.row0 = (int)(item - row * qt) * ROWS;
  s.rows = min(ROWS, mg - s.row0);
  const int per = (int)quot(row, P.n_q), i = (int)(row - (long long)per * P.n_q), r = per % P.route_heads;
  s.b = per / P.route_heads;
  s.t_seq0 = 0; s.n_seq = P.n_q * P.m;
  s.t_base = i * P.m;
  s.kvh = r / (P.route_heads / P.kv_heads);
  s.h0 = r * P.group;
  s.tok0 = 0; s.tok1 = seq_len(P, s.b);
  s.pages = P.table + s.b * P.table_stride;
  s.slots = P.ranges + row * P.slots * 2;
  s.prefix = 0;
  s.tile0 = s.tile1 = 0;
  s.mark = row * mg + s.row0;
  place_segment(P, sc, c, s.unit0 == 0, row, s);
  return s.unit1 - s.unit0;
}
__device__ __forceinline__ void unit_tiles(const Params& P, int tiles, Seg& s) {
  const int n = P.units ? P.units : 1;
  s.tile0 = (int)((long long)tiles * s.unit0 / n);
  s.tile1 = (int)((long long)tiles * s.unit1 / n);
}
// The units or tiles of all items: a ranges call's are known to the host.
__host__ __device__ __forceinline__ long long range_units(const Params& P) { return P.range_rows * ((P.m * P.group + ROWS - 1) / ROWS) * (P.units ? P.units : 1); }
// A length that the table has no places for is reported; what is behind the table is left out.
__device__ __forceinline__ void check_len(const Params& P, int b) {
  if (P.status && seq_end(P, b) > seq_len(P, b)) atomicOr(P.status, RR_STATUS_BAD_INDEX);
}
// Tokens of one slot: [lo, hi) clipped to the sequence.
__device__ __forceinline__ void slot_span(const Seg& s, int j, int& lo, int& hi) {
  lo = __ldg(s.slots + 2 * j);
  hi = min(__ldg(s.slots + 2 * j + 1), s.tok1);
  if (lo < 0 || hi < lo) lo = hi = 0;
}

struct RowAt { int t, h, limit; };                     // query token, head, tokens below `limit` are seen
__device__ __forceinline__ RowAt row_at(const Params& P, const Seg& s, int r) {
  const int idx = s.row0 + r, dt = idx / P.group;
  RowAt a;
  a.t = s.t_base + dt;
  a.h = s.h0 + idx - dt * P.group;
  int b = s.b, first = s.t_seq0, n = s.n_seq;
  if (b < 0) {
    b = P.cu ? rr_sequence_of(P.cu, P.batch, a.t) : a.t;
    if (b < 0) { a.limit = 0; return a; }
    first = seq_first(P, b);
    n = seq_count(P, b);
  }
  const int len = seq_end(P, b);
  a.limit = P.causal ? max(len - n + (a.t - first) + 1, 0) : len;
  return a;
}
__device__ __forceinline__ long long q_at(const Params& P, const Seg& s, const RowAt& a) { return (s.slots ? s.b * P.qb : 0) + a.h * P.qh + a.t * P.qt; }
__device__ __forceinline__ long long out_at(const Params& P, const Seg& s, const RowAt& a) { return (s.slots ? s.b * P.ob : 0) + a.h * P.oh + a.t * P.ot; }

// Element offset of token `tok` of the segment's list, -1 if its page id is bad.
__device__ __forceinline__ long long token_at(const Params& P, const Seg& s, int tok) {
  const int col = tok / P.page_tokens, page = __ldg((tok < s.prefix ? s.prefix_pages : s.pages) + col);
  if (page < 0 || page >= P.num_pages) { if (P.status) atomicOr(P.status, RR_STATUS_BAD_INDEX); return -1; }
  return page * P.page_stride + s.kvh * P.head_stride + (tok - col * P.page_tokens) * P.token_stride;
}

// ---- marks -------------------------------------------------------------------------------------------------
// A tile is multiplied whole, so a value that a row may not see enters the row's sums with weight 0: nothing, unless it is an
// infinity or NaN.  A row with such a result that had masked tokens of its list is marked, by the sign of its partial's sum or, where it has
// none, by a byte, and looked at again when everything else is done (look_again in rr_attend_paged_again.cuh): the kernels' pipelines do not wait for it.
__device__ __forceinline__ float with_mark(float l, bool mark) { return __uint_as_float((__float_as_uint(l) & 0x7FFFFFFFu) | (mark ? 0x80000000u : 0u)); }
__device__ __forceinline__ void mark_row(const Params& P, long long at, bool mark) {
  P.marks[at] = mark;
  if (mark && P.slots == 0) atomicOr(&P.plan->marked, 1);
}
__device__ __forceinline__ bool has_mark(float l) { return __float_as_uint(l) >> 31; }
// Whether a whole item of `rows` rows leaves marks: those of up to FEW rows multiply no masked token.
constexpr int FEW = 8;
__host__ __device__ inline bool leaves_marks(const Params& P, long long rows) { return rows > (P.tc ? TILE : FEW); }

}  // namespace rrattn

// Up to four rows of each item: `rows` of the call's items.
cudaError_t rr_launch_attend_few(const rrattn::Params& p, int rows, cudaStream_t st);
// bf16, dh 64 or 128, a positive scale, rows on 16-byte boundaries.  (The few kernel needs the same.)
bool rr_attend_tc_supported(const rrattn::Params& p, int dtype);
cudaError_t rr_launch_attend_tc(const rrattn::Params& p, int grid, cudaStream_t st);
