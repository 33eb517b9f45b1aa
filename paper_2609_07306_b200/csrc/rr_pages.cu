// Who owns which page of the paged cache: forks, room for new tokens, compaction.
//
//   refs[p] = entries of the page table (and of the caller) that hold page p;  0: free
//   fork      row b <- row parents[b], all at once;  refs by the difference of the rows
//   reserve   row b: columns [0, c1), c1 = ceil((lens + new) / page); pages to be written are the row's own (refs 1)
//   compact   L pages in use; the i-th of those >= L goes to the i-th free one below L
//
// The bookkeeping is a few integers per row and one pass over refs: bound by latency, not by bytes.  It runs in one cluster of eight
// CTAs, whose hardware barrier separates the steps (a barrier costs less than a launch, and no wait on memory is needed).  What is cheap to know
// about the rows every CTA finds out for itself, a thread per row, instead of a barrier; work on the table's entries is shared by all warps, 128 or 256
// entries of a row at a time.  Free pages are found by all threads together, up to 32 pages per thread, in rounds of 131072
// pages; counts are exchanged through distributed shared memory, and the threads of a CTA look up which entries its free pages' ranks belong to.
// Which page goes where follows from ranks, never from the order of atomics, which only add to counters.  Copies of pages are a second
// kernel over all SMs, which reads on the device how many there are; it is launched along with the first and waits for it, for all layers at once.
// Measured: room for 64 rows in a pool of 25148 pages 8.1 us a call, copies' kernel (with nothing to do) included; half of 512 rows given up and given new prompts, 66837
// pages, 16 us; a step of 256 beams 36 us, 23 of them copies (156 MB); compaction of 8979 pages 6 us and 174 us of copies (1.14 GB, 6.5 TB/s).
#include <cooperative_groups.h>
#include <utility>
#include "rr_paged.cuh"
#include "rr_sm100.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int CL = 8, NT = 512, NW = NT / 32;
constexpr int ROUND = CL * NT * 32;                     // pages of a round: 32 per thread
constexpr int COLS = 256;                               // entries of a row that a warp releases
constexpr int ROWS_ON_CHIP = 2048;                      // rows whose state fits shared memory
constexpr int GIVEN = 4096;                             // pages that a CTA hands out at a time
constexpr int64_t LONG_TABLE = 1 << 16;                 // entries of a table from which a fork takes all SMs
constexpr int MAX_LAYERS = 64;                          // of one launch of the copy

struct Move { int32_t src, dst, tokens; };

// The workspace.  `list`: new rows (fork), entries to be replaced or free pages in rank order (reserve), sources, destinations and new ids (compact).
struct Work {
  int32_t* moves;                                       // [0] how many, [1] pages in use (compact)
  int32_t* replaced;                                    // [batch] entries to be replaced behind the one that the row goes on writing; fork: pages that the row takes
  int32_t* was;                                         // [batch] fork: pages that it held
  int32_t* list;
  int32_t* ranked;                                      // [num_pages]
  Move* move;
  char* rows;                                           // a CTA's state of the rows where it does not fit shared memory
};

struct PoolParams {
  rr_page_pool p;
  Work w;
  const int32_t* arg;                                   // parents or new_tokens
  const int32_t* lens;
  int32_t* new_lens;
  int32_t* remap;
  int32_t new_each, slots;                              // slots of the table of pages that rows go on writing
  int32_t words;                                        // of 32 pages that a warp looks at in a round: 32, fewer in a small pool, whose pages all warps share
};

// A row of a call of reserve: tokens up to column c0 and `part` of it, room up to column c1, pages up to column `held` (of those that stay).
struct Row {
  int c0, part, c1, held;
  int was;                                              // pages before the call
  int want;                                             // the page that the row goes on writing, -1: none
  int replaced;                                         // twice the entries to be replaced, + 1 if that one is among them
  int first;                                            // how many hold it; then the rank of the row's first new page
};
struct Slot { int page, n, first; };                    // how many rows go on writing a page, the first of them

size_t up4(size_t n) { return (n + 3) & ~(size_t)3; }
int slots_of(int batch) {
  int n = 64;
  while (n < 2 * batch) n *= 2;
  return n;
}
int words_of(const rr_page_pool& p) {
  const int n = (p.num_pages + ROUND / 32 - 1) / (ROUND / 32);
  return n < 32 ? n : 32;
}
size_t row_state(const rr_page_pool& p) { return sizeof(Row) * up4(p.batch) + sizeof(Slot) * slots_of(p.batch); }
size_t list_ints(const rr_page_pool& p) {
  const size_t rows = (size_t)p.batch * p.pages_per_seq, pages = 2 * (size_t)p.num_pages;
  return up4(rows > pages ? rows : pages);
}
size_t move_bytes(const rr_page_pool& p) {
  const size_t most = (size_t)(p.batch > p.num_pages / 2 ? p.batch : p.num_pages / 2) + 1;
  return 4 * up4(3 * most);
}
size_t workspace_bytes(const rr_page_pool& p) {
  return 64 + 4 * (2 * up4(p.batch) + list_ints(p) + up4(p.num_pages)) + move_bytes(p) + (p.batch > ROWS_ON_CHIP ? CL * row_state(p) : 0);
}
Work work_of(const rr_page_pool& p, void* ws) {
  Work w;
  w.moves = (int32_t*)ws;
  w.replaced = w.moves + 16;
  w.was = w.replaced + up4(p.batch);
  w.list = w.was + up4(p.batch);
  w.ranked = w.list + list_ints(p);
  w.move = (Move*)(w.ranked + up4(p.num_pages));
  w.rows = (char*)w.move + move_bytes(p);
  return w;
}

__device__ __forceinline__ void report(const rr_page_pool& p, uint32_t bit) { if (p.status) atomicOr(p.status, bit); }
__device__ __forceinline__ bool in_pool(const rr_page_pool& p, int id) { return id >= 0 && id < p.num_pages; }
__device__ __forceinline__ int held_of(const rr_page_pool& p, int b) { return min(max(__ldcg(p.held + b), 0), p.pages_per_seq); }
// One holder less; 1 if the page is free now.
__device__ __forceinline__ int release(const rr_page_pool& p, int id) { return atomicSub(p.refs + id, 1) == 1; }
__device__ __forceinline__ int warp_sum(int x) { return __reduce_add_sync(0xFFFFFFFFu, x); }
__device__ __forceinline__ int warp_prefix(int x) {     // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) { const int y = __shfl_up_sync(0xFFFFFFFFu, x, d); if (lane >= d) x += y; }
  return x;
}
__device__ __forceinline__ void add_free(const rr_page_pool& p, int freed) {
  freed = warp_sum(freed);
  if ((threadIdx.x & 31) == 0 && freed) atomicAdd(p.free_pages, freed);
}

struct Shared { int warp[NW]; int cta[2][CL]; };

// Exclusive prefix of the warps' counts over the cluster, and their sum; all that was written before is visible behind it.  Each CTA leaves its count with
// all others before the barrier, so that none reads another one's memory behind it (and may end before the others do).  Rounds alternate between
// two places: a CTA that is a round ahead overwrites nothing that another one still reads.
__device__ __forceinline__ int2 cluster_prefix(cg::cluster_group& cl, Shared& s, int count, int& round) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) s.warp[warp] = count;
  __syncthreads();
  const int x = lane < NW ? s.warp[lane] : 0;
  int* const places = s.cta[round & 1];
  ++round;
  if (warp == 0) {
    const int cta = warp_sum(x);
    if (lane < CL) *cl.map_shared_rank(places + cl.block_rank(), lane) = cta;
  }
  auto all_here = cl.barrier_arrive();
  const int before = warp_sum(lane < warp ? x : 0);
  cl.barrier_wait(std::move(all_here));
  const int theirs = lane < CL ? places[lane] : 0;
  return make_int2(before + warp_sum(lane < (int)cl.block_rank() ? theirs : 0), warp_sum(theirs));
}

// Code is kept short, with loops left as loops where nothing waits for them: a kernel of this kind runs every instruction about once, and what it
// spent most of its time on was fetching 70 KB of them.

// The first page of this warp in a round that begins at page `at`.
__device__ __forceinline__ long long first_page(cg::cluster_group& cl, int words, long long at) {
  return at + ((long long)cl.block_rank() * NW + (threadIdx.x >> 5)) * 32 * words;
}

// Bit l of lane k (< words): page first + 32 k + l is free.
__device__ __noinline__ uint32_t free_bits(const int32_t* refs, int num_pages, int words, long long first) {
  const int lane = threadIdx.x & 31;
  if (first >= num_pages) return 0;
  const int n = (int)min((long long)num_pages - first, 32LL * words) - lane;
  uint32_t bits = 0;
#pragma unroll 1
  for (int k0 = 0; k0 < words; k0 += 8) {
    int v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 32 * (k0 + k) < n ? __ldcg(refs + first + lane + 32 * (k0 + k)) : 1;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t word = __ballot_sync(0xFFFFFFFFu, v[k] == 0);
      if (lane == k0 + k) bits = word;
    }
  }
  return bits;
}

// ---- fork -------------------------------------------------------------------------------------------------------
// A row is compared with its parent's: beams differ from one another in their last pages only, and equal entries cost two loads.  New entries
// are staged, as a parent's row may be rewritten in the same call.
// Long tables take two ordinary launches over all SMs instead of one cluster (where one group of four in each descends from its first: 512 rows of 2048 entries 9.5 us
// instead of 66, 512 of 256 7.1 instead of 15; 64 of 256 6.0 in the cluster, 8.4 by two launches).
constexpr int FORK_NT = 1024;                           // (a warp per row for 256 rows)
constexpr int LONG_NT = 512;
constexpr int RUN = 128;                                // entries of a row that a warp compares
struct Heir { int parent, held, takes; };               // pages that the row held and takes (-1: it stays)

__device__ __forceinline__ Heir heir_of(const PoolParams& P, int b, bool tell) {
  const rr_page_pool& p = P.p;
  Heir h{__ldcg(P.arg + b), held_of(p, b), -1};
  if (h.parent < -1 || h.parent >= p.batch) {
    if (tell) report(p, RR_STATUS_BAD_INDEX);
    h.parent = b;
  }
  const int given = h.parent < 0 ? 0 : __ldcg(P.lens + h.parent);
  const int len = (int)min((long long)max(given, 0), (long long)p.page_tokens * p.pages_per_seq);
  if (h.parent != b) h.takes = h.parent < 0 ? 0 : (int)min((unsigned)held_of(p, h.parent), ((unsigned)len + p.page_tokens - 1) / p.page_tokens);
  if (tell) {
    if (len != given) report(p, RR_STATUS_BAD_INDEX);
    P.new_lens[b] = len;
  }
  return h;
}

// A run of a row's new entries: staged, with the holders of pages that change; how many pages came free.
__device__ __forceinline__ int stage_run(const PoolParams& P, int b, int c0, const Heir& h) {
  const rr_page_pool& p = P.p;
  const int32_t* const mine = p.page_table + b * p.table_stride;
  const int32_t* const theirs = p.page_table + h.parent * p.table_stride;
  int32_t* const stage = P.w.list + (size_t)b * p.pages_per_seq;
  const int end = min(max(h.held, h.takes), c0 + RUN);
  int freed = 0;
#pragma unroll 2
  for (int c = c0 + (threadIdx.x & 31); c < end; c += 32) {
    const int was = c < h.held ? __ldcg(mine + c) : -1;
    int is = c < h.takes ? __ldcg(theirs + c) : -1;
    if (c < h.takes && !in_pool(p, is)) {               // left out: the column stays, without a page
      is = -1;
      report(p, RR_STATUS_BAD_INDEX);
    }
    stage[c] = is;
    if (was == is) continue;
    if (is >= 0) freed -= atomicAdd(p.refs + is, 1) == 0;               // (one row may let go of a page before another takes it)
    if (in_pool(p, was)) freed += release(p, was);
    else if (c < h.held) report(p, RR_STATUS_BAD_INDEX);
  }
  return freed;
}
__device__ __forceinline__ void write_run(const PoolParams& P, int b, int c0, int held, int takes) {
  int32_t* const mine = P.p.page_table + b * P.p.table_stride;
  const int32_t* const stage = P.w.list + (size_t)b * P.p.pages_per_seq;
#pragma unroll 2
  for (int c = c0 + (threadIdx.x & 31); c < min(max(held, takes), c0 + RUN); c += 32) mine[c] = __ldcg(stage + c);
  if (c0 == 0 && (threadIdx.x & 31) == 0) P.p.held[b] = takes;
}

__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(FORK_NT, 1)
fork_kernel(const __grid_constant__ PoolParams P) {
  extern __shared__ __align__(16) char on_chip[];
  cg::cluster_group cl = cg::this_cluster();
  const rr_page_pool& p = P.p;
  const int rank = cl.block_rank(), warp = (threadIdx.x >> 5) * CL + rank;
  Heir* const heirs = p.batch > ROWS_ON_CHIP ? (Heir*)(P.w.rows + rank * (sizeof(Heir) * ((p.batch + 3) & ~3))) : (Heir*)on_chip;
  rr_pdl_wait();
  rr_pdl_trigger();
  for (int b = threadIdx.x; b < p.batch; b += FORK_NT) heirs[b] = heir_of(P, b, rank == 0);     // in every CTA
  __syncthreads();
  const int parts = (p.pages_per_seq + RUN - 1) / RUN, units = p.batch * parts, each = (units + CL * (FORK_NT / 32) - 1) / (CL * (FORK_NT / 32));
  int freed = 0;
  for (int u = warp * each; u < min((warp + 1) * each, units); ++u)
    if (const Heir h = heirs[u / parts]; h.takes >= 0) freed += stage_run(P, u / parts, u % parts * RUN, h);
  cl.sync();
  for (int u = warp * each; u < min((warp + 1) * each, units); ++u)
    if (const Heir h = heirs[u / parts]; h.takes >= 0) write_run(P, u / parts, u % parts * RUN, h.held, h.takes);
  add_free(p, freed);
}

__global__ void __launch_bounds__(LONG_NT)
fork_stage_kernel(const __grid_constant__ PoolParams P) {
  const rr_page_pool& p = P.p;
  const int lane = threadIdx.x & 31, parts = (p.pages_per_seq + RUN - 1) / RUN, units = p.batch * parts;
  rr_pdl_wait();
  rr_pdl_trigger();
  int freed = 0;
  for (int u = blockIdx.x * (LONG_NT / 32) + (threadIdx.x >> 5); u < units; u += gridDim.x * (LONG_NT / 32)) {
    const int b = u / parts, part = u - b * parts;
    const Heir h = heir_of(P, b, part == 0 && lane == 0);
    if (part == 0 && lane == 0) P.w.replaced[b] = h.takes, P.w.was[b] = h.held;
    if (h.takes >= 0) freed += stage_run(P, b, part * RUN, h);
  }
  add_free(p, freed);
}
__global__ void __launch_bounds__(LONG_NT)
fork_write_kernel(const __grid_constant__ PoolParams P) {
  const int parts = (P.p.pages_per_seq + RUN - 1) / RUN, units = P.p.batch * parts;
  rr_pdl_wait();
  rr_pdl_trigger();
  for (int u = blockIdx.x * (LONG_NT / 32) + (threadIdx.x >> 5); u < units; u += gridDim.x * (LONG_NT / 32)) {
    const int b = u / parts, takes = __ldcg(P.w.replaced + b);
    if (takes >= 0) write_run(P, b, (u - b * parts) * RUN, __ldcg(P.w.was + b), takes);
  }
}

// ---- reserve ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ Row row_of(const PoolParams& P, int b, bool tell) {
  const rr_page_pool& p = P.p;
  const long long cap = (long long)p.page_tokens * p.pages_per_seq;
  int len = __ldcg(P.lens + b), more = P.arg ? __ldcg(P.arg + b) : P.new_each;
  const int held = held_of(p, b);
  const bool bad = len < 0 || more < 0 || (long long)len + more > cap;
  if (bad) {
    if (tell) report(p, RR_STATUS_BAD_INDEX);
    len = (int)min((long long)max(len, 0), cap);
    more = (int)min((long long)max(more, 0), cap - len);
  }
  Row r;
  const unsigned page = p.page_tokens, upto = (unsigned)len + (unsigned)more;
  r.c0 = (int)((unsigned)len / page);
  r.part = (int)((unsigned)len - (unsigned)r.c0 * page);
  r.c1 = (int)(upto / page);
  r.c1 += (unsigned)r.c1 * page != upto;
  r.was = held;
  r.held = min(held, r.c1);
  r.want = more > 0 && r.part > 0 && r.c0 < r.held ? 0 : -1;
  r.replaced = r.first = 0;
  return r;
}

// A row's entries to be replaced behind the one that it goes on writing.
__device__ __forceinline__ int32_t* replaced_of(const PoolParams& P, int b) { return P.w.list + (size_t)b * P.p.pages_per_seq; }

// The rows' new pages in the order of their ranks: for entries to be replaced, then for missing ones.
struct Hand {
  const PoolParams& P;
  const Row* rows;
  int b = 0, freed = 0;                                 // the row of the last page, pages come free
  __device__ __forceinline__ void give(int page, int rank) {
    const rr_page_pool& p = P.p;
    if (rank < rows[b].first || (b + 1 < p.batch && rank >= rows[b + 1].first)) {
      int lo = 0, n = p.batch;                          // the last row that begins at this rank or before it
      while (n > 1) {
        const int half = n / 2;
        if (rows[lo + half].first <= rank) lo += half, n -= half;
        else n = half;
      }
      b = lo;
    }
    const Row& r = rows[b];
    const int m = rank - r.first, n = r.replaced >> 1;
    int32_t* const row = p.page_table + b * p.table_stride;
    int c = r.held + m - n;
    if (m == 0 && (r.replaced & 1)) {                   // the page that the row goes on writing
      c = r.c0;
      freed += release(p, r.want);
      P.w.move[atomicAdd(P.w.moves, 1)] = Move{r.want, page, r.part};
    } else if (m < n) {
      c = __ldcg(replaced_of(P, b) + m - (r.replaced & 1));
      const int old = __ldcg(row + c);
      if (in_pool(p, old)) freed += release(p, old);
    }
    row[c] = page;
    p.refs[page] = 1;
    --freed;
  }
};

__device__ __forceinline__ Slot* slot_of(Slot* slots, int mask, int page, bool add) {
  unsigned h = (unsigned)page * 2654435761u >> 7;
  while (true) {                                        // (half of the slots at most are taken)
    Slot* const t = slots + (h & mask);
    const int k = add ? atomicCAS(&t->page, -1, page) : *(volatile int*)&t->page;
    if (k == page || (add && k == -1)) return t;
    ++h;
  }
}

// Up to which place a row may be written after a call that has given nothing: to the first entry that would have been replaced, be it by a page of its own or, of a page
// that all who hold it go on writing, by those of the others; else to the end of its pages, if some are missing.  refs and table do not change any more.
__device__ __noinline__ int room_of(const PoolParams& P, const Row& r, int b) {
  const rr_page_pool& p = P.p;
  const int replaced = r.replaced >> 1, copied = r.replaced & 1;
  int col = r.held;
  if (r.want >= 0 && __ldcg(p.refs + r.want) > 1) col = r.c0;
  else if (replaced > copied) col = __ldcg(replaced_of(P, b));
  else if (r.held == r.c1) return INT32_MAX;
  return (int)min((long long)col * p.page_tokens, (long long)INT32_MAX);
}

constexpr int LOOK = 4;                                 // entries of a row that a lane loads together
constexpr int NEAR = 4;                                 // entries behind a row's tokens that its thread looks at itself

__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(NT, 1)
reserve_kernel(const __grid_constant__ PoolParams P) {
  extern __shared__ __align__(16) char on_chip[];
  __shared__ Shared s;
  __shared__ int s_scan[NW];
  cg::cluster_group cl = cg::this_cluster();
  const rr_page_pool& p = P.p;
  const int lane = threadIdx.x & 31, my_warp = threadIdx.x >> 5, rank = cl.block_rank(), warp = my_warp * CL + rank;
  int32_t* const given = (int32_t*)on_chip;             // [GIVEN] the CTA's free pages by their rank
  char* const state = p.batch > ROWS_ON_CHIP ? P.w.rows + rank * (sizeof(Row) * ((p.batch + 3) & ~3) + sizeof(Slot) * P.slots) : on_chip + GIVEN * 4;
  Row* const rows = (Row*)state;
  Slot* const slots = (Slot*)(state + sizeof(Row) * ((p.batch + 3) & ~3));
  auto started = cl.barrier_arrive();
  rr_pdl_wait();
  rr_pdl_trigger();
  int round = 0, freed = 0;
  if (warp == 0 && lane == 0) *P.w.moves = 0;
  // 1. the rows, in every CTA, and what the table holds where they will be written; pages behind a row's room are released
  int ids[NEAR];                                        // of the thread's first row
  bool longest = false, shorter = false;
  for (int i = threadIdx.x; i < P.slots; i += NT) slots[i] = Slot{-1, 0, INT32_MAX};
  for (int b = threadIdx.x; b < p.batch; b += NT) {
    Row r = row_of(P, b, rank == 0);
    const int32_t* const row = p.page_table + b * p.table_stride;
    const int c = r.c0 + (r.part > 0);
    if (r.want == 0) r.want = __ldcg(row + r.c0);
    if (b == threadIdx.x) {
#pragma unroll
      for (int i = 0; i < NEAR; ++i) ids[i] = c + i < r.held ? __ldcg(row + c + i) : -1;
    }
    if (r.want != -1 && !in_pool(p, r.want)) {
      r.want = -1;
      if (rank == 0) report(p, RR_STATUS_BAD_INDEX);
    }
    longest |= r.held - c > NEAR;
    shorter |= r.was > r.c1;
    rows[b] = r;
  }
  longest = __syncthreads_or(longest);
  cl.barrier_wait(std::move(started));                  // all CTAs run: their memory may be written from here on
  if (__syncthreads_or(shorter)) {                      // (the same in all CTAs)
    const int parts = (p.pages_per_seq + COLS - 1) / COLS;
    const int each = (p.batch * parts + CL * NW - 1) / (CL * NW);       // (neighbours by one warp: rows that end tend to alternate with such that stay)
    for (int u = warp * each; u < min((warp + 1) * each, p.batch * parts); ++u) {
      const int b = u / parts, c0 = (u - b * parts) * COLS, end = min(rows[b].was, c0 + COLS);
      int32_t* const row = p.page_table + b * p.table_stride;
#pragma unroll 4
      for (int c = max(rows[b].c1, c0) + lane; c < end; c += 32) {
        const int id = __ldcg(row + c);
        row[c] = -1;
        if (in_pool(p, id)) freed += release(p, id);
        else report(p, RR_STATUS_BAD_INDEX);
      }
    }
    cl.sync();
  }
  // 2. nothing changes now.  The free pages of this thread; the rows' entries to be replaced: a page that others hold too and that not all who hold it
  // go on writing with this row as the first of them, and pages behind it that others hold
  int near_refs[NEAR], holders_first = 0;
  if (threadIdx.x < p.batch) {
#pragma unroll
    for (int i = 0; i < NEAR; ++i) near_refs[i] = in_pool(p, ids[i]) ? __ldcg(p.refs + ids[i]) : 2;
    if (const int want = rows[threadIdx.x].want; want >= 0) holders_first = __ldcg(p.refs + want);
  }
  uint32_t bits = free_bits(p.refs, p.num_pages, P.words, first_page(cl, P.words, 0));
  for (int b = threadIdx.x; b < p.batch; b += NT) {
    const int want = rows[b].want;
    if (want < 0) continue;
    const int holders = b == threadIdx.x ? holders_first : __ldcg(p.refs + want);
    rows[b].first = holders;
    if (holders > 1) {
      Slot* const t = slot_of(slots, P.slots - 1, want, true);
      atomicAdd(&t->n, 1);
      atomicMin(&t->first, b);
    }
  }
  __syncthreads();
  if (longest) {                                        // (a warp per row, each row once in the cluster)
    const int each = (p.batch + CL * NW - 1) / (CL * NW);
    for (int b = warp * each; b < min((warp + 1) * each, p.batch); ++b) {
      const Row r = rows[b];
      const int32_t* const row = p.page_table + b * p.table_stride;
      int n = 0;
      for (int at = r.c0 + (r.part > 0); at < r.held; at += 32 * LOOK) {
        int id[LOOK], n_refs[LOOK];
#pragma unroll
        for (int i = 0; i < LOOK; ++i) { const int c = at + 32 * i + lane; id[i] = c < r.held ? __ldcg(row + c) : -1; }
#pragma unroll
        for (int i = 0; i < LOOK; ++i) n_refs[i] = in_pool(p, id[i]) ? __ldcg(p.refs + id[i]) : 2;
#pragma unroll
        for (int i = 0; i < LOOK; ++i) {
          const int c = at + 32 * i + lane;
          const unsigned fresh = __ballot_sync(0xFFFFFFFFu, c < r.held && n_refs[i] > 1);
          if (c < r.held && !in_pool(p, id[i])) report(p, RR_STATUS_BAD_INDEX);
          if (fresh >> lane & 1) replaced_of(P, b)[n + __popc(fresh & ((1u << lane) - 1))] = c;
          n += __popc(fresh);
        }
      }
      if (lane == 0) P.w.replaced[b] = n;
    }
    cl.sync();
  }
  int total = 0;
  for (int at = 0; at < p.batch; at += NT) {
    const int b = at + threadIdx.x;
    int need = 0, replaced = 0, copied = 0;
    if (b < p.batch) {
      const Row r = rows[b];
      int32_t* const list = replaced_of(P, b);
      const bool mine = b % CL == rank;                 // whoever writes what all CTAs find out
      if (r.want >= 0 && r.first > 1) {
        const Slot* const t = slot_of(slots, P.slots - 1, r.want, false);
        copied = *(volatile int*)&t->n != r.first || *(volatile int*)&t->first != b;
      }
      if (longest) {
        replaced = __ldcg(P.w.replaced + b);
      } else {
        const int c = r.c0 + (r.part > 0);
        if (at > 0) {
#pragma unroll
          for (int i = 0; i < NEAR; ++i) ids[i] = c + i < r.held ? __ldcg(p.page_table + b * p.table_stride + c + i) : -1;
#pragma unroll
          for (int i = 0; i < NEAR; ++i) near_refs[i] = in_pool(p, ids[i]) ? __ldcg(p.refs + ids[i]) : 2;
        }
#pragma unroll
        for (int i = 0; i < NEAR; ++i) {
          if (c + i >= r.held || near_refs[i] <= 1) continue;
          if (mine && !in_pool(p, ids[i])) report(p, RR_STATUS_BAD_INDEX);
          if (mine) list[replaced] = c + i;
          ++replaced;
        }
      }
      replaced += copied;
      need = replaced + r.c1 - r.held;
    }
    const int x = warp_prefix(need);
    if (lane == 31) s_scan[my_warp] = x;
    __syncthreads();
    const int before = warp_sum(lane < my_warp ? s_scan[lane] : 0), all = warp_sum(lane < NW ? s_scan[lane] : 0);
    __syncthreads();
    if (b < p.batch) {
      rows[b].replaced = 2 * replaced + copied;
      rows[b].first = total + before + x - need;
    }
    total += all;
  }
  // 3. free pages get their ranks, and each goes to the entry of its rank.  Free pages lie together, often all in one warp, so they are shared by the CTA's
  // threads; many, or those of a pool of several rounds (where a page may come free while the last rounds are still looked at), by the cluster's.
  int freed_now = 0;
  bool enough = true;
  if (total > 0) {
    const bool near = p.num_pages <= ROUND && total <= GIVEN;
    int found = 0, from = 0;
    for (long long at = 0; at < p.num_pages && found < total; at += ROUND) {
      const long long first = first_page(cl, P.words, at);
      if (at > 0) bits = free_bits(p.refs, p.num_pages, P.words, first);
      const int2 n = cluster_prefix(cl, s, warp_sum(__popc(bits)), round);
      if (near) {
        if (my_warp == 0) s_scan[0] = n.x;
        if (my_warp == NW - 1) s_scan[1] = n.x + warp_sum(__popc(bits));
        __syncthreads();
        from = s_scan[0];
      }
      int32_t* const out = near ? given - from : P.w.ranked;
      if (found + n.x < total) {
        int r = found + n.x + warp_prefix(__popc(bits)) - __popc(bits);
        for (uint32_t w = bits; w && r < total; w &= w - 1) out[r++] = (int32_t)first + 32 * lane + __ffs(w) - 1;
      }
      found += n.y;
    }
    enough = found >= total;
    if (near) __syncthreads();
    else cl.sync();
    if (enough) {
      const volatile int32_t* const list = near ? given - from : P.w.ranked;
      const int end = near ? min(s_scan[1], total) : total;
      Hand hand{P, rows};
#pragma unroll 1
      for (int r = near ? from + (int)threadIdx.x : warp * 32 + lane; r < end; r += near ? NT : CL * NT) hand.give(list[r], r);
      freed_now = hand.freed;
    }
  }
  if (!enough && warp == 0 && lane == 0) report(p, RR_STATUS_NO_PAGES);
  for (int b = threadIdx.x; b < p.batch; b += NT) {
    if (b % CL != rank) continue;
    const int held = enough ? rows[b].c1 : rows[b].held;
    if (rows[b].was != held) p.held[b] = held;
    if (p.room) p.room[b] = enough ? INT32_MAX : room_of(P, rows[b], b);
  }
  add_free(p, freed + freed_now);
}

// ---- compact ----------------------------------------------------------------------------------------------------
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(NT, 1)
compact_kernel(const __grid_constant__ PoolParams P) {
  __shared__ Shared s;
  cg::cluster_group cl = cg::this_cluster();
  const rr_page_pool& p = P.p;
  const int lane = threadIdx.x & 31;
  rr_pdl_wait();
  rr_pdl_trigger();
  const bool one_round = p.num_pages <= ROUND;
  cl.sync();                                            // all CTAs run: their memory may be written from here on
  int round = 0, free_all = 0;
  uint32_t bits = 0;
  int2 n = make_int2(0, 0);
  for (long long at = 0; at < p.num_pages; at += ROUND) {
    bits = free_bits(p.refs, p.num_pages, P.words, first_page(cl, P.words, at));
    n = cluster_prefix(cl, s, warp_sum(__popc(bits)), round);
    free_all += n.y;
  }
  const int live = p.num_pages - free_all;
  // Free pages below `live` by their rank, pages in use from there on by their rank among all in use: the last as many of them as there are free ones below.
  int32_t* const dst = P.w.list;
  int32_t* const src = P.w.list + p.num_pages;
  int before = 0, low = 0;
  for (long long at = 0; at < p.num_pages; at += ROUND) {
    const long long first = first_page(cl, P.words, at);
    if (!one_round) {
      bits = free_bits(p.refs, p.num_pages, P.words, first);
      n = cluster_prefix(cl, s, warp_sum(__popc(bits)), round);
    }
    const int upto = before + n.x + warp_prefix(__popc(bits)) - __popc(bits);
#pragma unroll 1
    for (int k = 0; k < P.words && first + 32 * k < p.num_pages; ++k) {
      const uint32_t word = __shfl_sync(0xFFFFFFFFu, bits, k);
      const int page = (int)first + 32 * k + lane, rank = __shfl_sync(0xFFFFFFFFu, upto, k) + __popc(word & ((1u << lane) - 1));
      const bool is_free = word >> lane & 1;
      if (page >= p.num_pages) continue;
      if (is_free && page < live) dst[rank] = page, ++low;
      if (!is_free && page >= live) src[page - rank] = page;
      else P.remap[page] = page;
    }
    before += n.y;
  }
  const int moves = cluster_prefix(cl, s, warp_sum(low), round).y;
  for (int i = cl.block_rank() * NT + threadIdx.x; i < moves; i += CL * NT) {
    const int from = __ldcg(src + live - moves + i), to = __ldcg(dst + i);
    P.remap[from] = to;
    p.refs[to] = __ldcg(p.refs + from);
    p.refs[from] = 0;
    P.w.move[i] = Move{from, to, p.page_tokens};
  }
  if (cl.block_rank() == 0 && threadIdx.x == 0) {
    P.w.moves[0] = moves;
    P.w.moves[1] = live;
    *p.free_pages = free_all;
  }
}

// ---- copies -----------------------------------------------------------------------------------------------------
// A page of one layer's keys or values: the outer of heads and tokens, the inner one, the entries of a head.
struct Layer {
  char* base[2];                                        // keys, values
  int64_t page, outer, mid;                             // bytes
  int32_t heads, row;                                   // bytes of a head's entries
  int8_t unit, token_major, joined;                     // unit: bytes that addresses and strides split into; joined: the inner of heads and tokens lies side by side
};

struct CopyParams {
  Work w;
  int32_t page_tokens, layers;
  rr_page_pool p;
  const int32_t* remap;                                 // of a compaction (with a row of CTAs more for the table), else NULL
  Layer layer[MAX_LAYERS];
};

// The table of a compacted pool, by the CTAs of one row of the grid: 88 with two layers, 3 with 64 (a million entries 111 us, 814).
__device__ __forceinline__ void renumber(const CopyParams& P, int moves) {
  const int live = __ldcg(P.w.moves + 1);
  for (int b = blockIdx.x; b < P.p.batch && moves > 0; b += gridDim.x) {
    int32_t* const row = P.p.page_table + b * P.p.table_stride;
    const int held = held_of(P.p, b);
#pragma unroll 4
    for (int c = threadIdx.x; c < held; c += blockDim.x) {
      const int id = __ldcg(row + c);
      if (!in_pool(P.p, id)) report(P.p, RR_STATUS_BAD_INDEX);
      else if (id >= live) row[c] = __ldcg(P.remap + id);
    }
  }
}

// Where all runs lie on 16 bytes: one thread of a CTA moves pieces of up to 16 KB through a ring in shared memory with bulk copies, two loads ahead of the
// stores, three CTAs per SM.  A piece costs it some hundred instructions, whatever its length; with registers and 16-byte loads the addresses alone took
// longer than the memory (1.1 GB of 64 KB pages: 240 us, now 174 us, 6.5 TB/s).  Pieces of 8 KB, four CTAs: 181 us, and runs of 8 KB or less as here.
constexpr int COPY_NT = 128, PIECE = 16384, STAGES = 4, AHEAD = 2, COPY_CTAS = 3;
constexpr size_t COPY_SMEM = STAGES * PIECE;

__device__ __forceinline__ void bulk_load(void* smem, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(sm100::smem_u32(smem)), "l"(src), "r"(bytes),
               "r"(sm100::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, const void* smem, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;" ::"l"(dst), "r"(sm100::smem_u32(smem)), "r"(bytes) : "memory");
}

__global__ void __launch_bounds__(COPY_NT)
copy_bulk_kernel(const __grid_constant__ CopyParams P) {
  extern __shared__ __align__(128) char ring[];
  __shared__ uint64_t full[STAGES];
  __shared__ char* s_dst[STAGES];
  __shared__ uint32_t s_bytes[STAGES];
  __shared__ uint32_t s_abort;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) sm100::mbar_init(full + i, 1);
    sm100::mbar_fence_init();
    s_abort = 0;
  }
  rr_pdl_wait();
  rr_pdl_trigger();
  const int moves = __ldcg(P.w.moves);
  if ((int)blockIdx.y == 2 * P.layers) {
    renumber(P, moves);
    return;
  }
  if (threadIdx.x != 0) return;
  const Layer& L = P.layer[blockIdx.y >> 1];
  char* const base = L.base[blockIdx.y & 1];
  const int outers = L.token_major ? P.page_tokens : L.heads;
  const int64_t inner = (int64_t)(L.token_major ? L.heads : P.page_tokens) * L.row;      // bytes of a whole run
  const unsigned most = (unsigned)outers * (unsigned)((inner + PIECE - 1) / PIECE);
  const unsigned step_m = gridDim.x / most, step_i = gridDim.x % most;
  unsigned m = blockIdx.x / most, i = blockIdx.x % most;               // move, piece of it
  int loaded = 0, stored = 0;
  auto store = [&] {
    const int st = stored % STAGES;
    if (!sm100::mbar_wait(full + st, stored / STAGES & 1, &s_abort)) return false;
    bulk_store(s_dst[st], ring + st * PIECE, s_bytes[st]);
    ++stored;
    return true;
  };
  auto move_at = [&](unsigned m) {
    const Move* const p = P.w.move + min(m, (unsigned)moves - 1);
    return Move{__ldcg(&p->src), __ldcg(&p->dst), __ldcg(&p->tokens)};
  };
  bool ok = true;
  Move next = moves > 0 ? move_at(m) : Move{};
  while (ok && m < (unsigned)moves) {
    const Move mv = next;
    const unsigned piece = i;
    m += step_m, i += step_i;
    if (i >= most) i -= most, ++m;
    next = move_at(m);
    // the runs of this move: one where everything that is copied lies side by side
    const int64_t length = L.token_major ? inner : (int64_t)mv.tokens * L.row;
    const bool whole = length == L.outer;
    const int runs = whole ? 1 : L.token_major ? mv.tokens : L.heads;
    const int64_t bytes = whole ? length * (L.token_major ? mv.tokens : L.heads) : length;
    const unsigned pieces = (unsigned)((bytes + PIECE - 1) / PIECE), run = pieces == 1 ? piece : whole ? piece >= pieces : piece / pieces;
    if (run >= (unsigned)runs) continue;
    const int64_t at = (int64_t)(piece - run * pieces) * PIECE, off = run * L.outer + at;
    const uint32_t n = (uint32_t)min(bytes - at, (int64_t)PIECE);
    const int st = loaded % STAGES;
    // the store that read this stage last: AHEAD loads are not stored yet, so it is the (STAGES - AHEAD)-th last one
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(STAGES - AHEAD - 1) : "memory");
    s_dst[st] = base + mv.dst * L.page + off;
    s_bytes[st] = n;
    sm100::mbar_expect_tx(full + st, n);
    bulk_load(ring + st * PIECE, base + mv.src * L.page + off, n, full + st);
    ++loaded;
    if (loaded - stored > AHEAD) ok = store();
  }
  while (ok && stored < loaded) ok = store();
  if (!ok) {
    report(P.p, RR_STATUS_TIMEOUT);
    for (int i = stored + 1; i < loaded; ++i) {         // its own copies in flight, again with a limit
      s_abort = 0;
      sm100::mbar_wait(full + i % STAGES, i / STAGES & 1, &s_abort);
    }
  }
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// Everything else: units of 16 bytes (or of an entry, where strides or addresses do not split), eight in flight per thread, two divisions each: 2.3 GB in units of
// 16 bytes 697 us, of four 1590, of two 3130 (365 by bulk copies).
constexpr int UNITS_NT = 256, COPY_UNITS = 8 * UNITS_NT;

template <typename U>
__device__ __forceinline__ void copy_units(const Layer& L, const char* src, char* dst, unsigned first, unsigned units, unsigned inner) {
  U v[COPY_UNITS / UNITS_NT];
  int64_t at[COPY_UNITS / UNITS_NT];
  const unsigned row = L.row / sizeof(U);
#pragma unroll
  for (int i = 0; i < COPY_UNITS / UNITS_NT; ++i) {
    const unsigned u = first + i * UNITS_NT + threadIdx.x;
    at[i] = -1;
    if (u < units) {
      const unsigned o = u / inner, r = u - o * inner, m = r / row;
      at[i] = o * L.outer + m * L.mid + (int64_t)(r - m * row) * sizeof(U);
      v[i] = *(const U*)(src + at[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < COPY_UNITS / UNITS_NT; ++i)
    if (at[i] >= 0) *(U*)(dst + at[i]) = v[i];
}

__global__ void __launch_bounds__(UNITS_NT)
copy_units_kernel(const __grid_constant__ CopyParams P) {
  rr_pdl_wait();
  rr_pdl_trigger();
  const int moves = __ldcg(P.w.moves);
  if ((int)blockIdx.y == 2 * P.layers) {
    renumber(P, moves);
    return;
  }
  const Layer& L = P.layer[blockIdx.y >> 1];
  char* const base = L.base[blockIdx.y & 1];
  const unsigned row = L.row / L.unit, chunks = ((unsigned)L.heads * P.page_tokens * row + COPY_UNITS - 1) / COPY_UNITS;
  for (long long item = blockIdx.x; item < (long long)moves * chunks; item += gridDim.x) {
    const int m = (int)(item / chunks);
    const Move mv{__ldcg(&P.w.move[m].src), __ldcg(&P.w.move[m].dst), __ldcg(&P.w.move[m].tokens)};
    const unsigned first = (unsigned)(item - (long long)m * chunks) * COPY_UNITS;
    const unsigned units = (unsigned)L.heads * mv.tokens * row, inner = (unsigned)(L.token_major ? L.heads : mv.tokens) * row;
    if (first >= units) continue;
    const char* const src = base + mv.src * L.page;
    char* const dst = base + mv.dst * L.page;
    if (L.unit == 16) copy_units<uint4>(L, src, dst, first, units, inner);
    else if (L.unit == 4) copy_units<uint32_t>(L, src, dst, first, units, inner);
    else copy_units<uint16_t>(L, src, dst, first, units, inner);
  }
}

// ---- host -------------------------------------------------------------------------------------------------------
int check_pool(const rr_page_pool* p) {
  if (!p || !p->page_table || !p->refs || !p->held || !p->free_pages) return RR_ERR_INVALID_ARG;
  if (p->num_pages < 1 || p->page_tokens < 1 || p->batch < 1 || p->pages_per_seq < 1) return RR_ERR_INVALID_ARG;
  if (p->table_stride < (p->batch > 1 ? p->pages_per_seq : 0)) return RR_ERR_INVALID_ARG;
  if (((uintptr_t)p->page_table | (uintptr_t)p->refs | (uintptr_t)p->held | (uintptr_t)p->free_pages | (uintptr_t)p->status | (uintptr_t)p->room) & 3) return RR_ERR_INVALID_ARG;
  if (p->num_pages > RR_PAGES_MAX_PAGES || p->batch > RR_PAGES_MAX_BATCH || (int64_t)p->batch * p->pages_per_seq > (1 << 30)) return RR_ERR_TOO_LARGE;
  return RR_OK;
}
int check_workspace(const rr_page_pool* p, const void* ws, size_t bytes) {
  if (!ws || ((uintptr_t)ws & 15)) return RR_ERR_INVALID_ARG;
  return bytes < workspace_bytes(*p) ? RR_ERR_TOO_SMALL : RR_OK;
}
int check_caches(const rr_page_pool* p, const rr_paged_kv* c, int n) {
  if (!c || n < 1) return RR_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const int rc = rr_paged_check(c + i);
    if (rc != RR_OK) return rc;
    if (c[i].num_pages != p->num_pages || c[i].page_tokens != p->page_tokens) return RR_ERR_INVALID_ARG;
    if ((int64_t)c[i].kv_heads * c[i].page_tokens * c[i].dh > (1 << 30)) return RR_ERR_TOO_LARGE;
  }
  return RR_OK;
}

Layer layer_of(const rr_paged_kv& c) {
  Layer L{};
  const int64_t e = c.dtype == RR_BF16 ? 2 : 4, row = c.dh * e;
  L.base[0] = (char*)c.k;
  L.base[1] = (char*)c.v;
  L.page = c.page_stride * e;
  // (a stride of something that there is one of says nothing)
  int64_t head = c.head_stride * e, token = c.token_stride * e;
  if (c.kv_heads == 1) head = token * c.page_tokens;
  if (c.page_tokens == 1) token = row;
  L.token_major = token > head;
  L.outer = L.token_major ? token : head;
  L.mid = L.token_major ? head : token;
  L.joined = L.mid == row;
  const uint64_t all = (uint64_t)L.page | L.outer | L.mid | row | (uintptr_t)c.k | (uintptr_t)c.v;
  L.unit = all % 16 == 0 ? 16 : (int8_t)e;
  L.heads = c.kv_heads;
  L.row = (int32_t)row;
  return L;
}

// The copies that the bookkeeping kernel has listed, in all caches; of a compaction also the table.
int launch_copies(const PoolParams& P, const rr_paged_kv* caches, int n, bool compact, cudaStream_t st, const char* who) {
  static unsigned long long done = 0;
  cudaError_t e = rr_once_per_device(done, [] { return cudaFuncSetAttribute(copy_bulk_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)COPY_SMEM); });
  if (e != cudaSuccess) return rr_cuda_fail(e, who);
  for (int at = 0; at < n; at += MAX_LAYERS) {
    CopyParams C;
    C.w = P.w;
    C.page_tokens = P.p.page_tokens;
    C.layers = n - at < MAX_LAYERS ? n - at : MAX_LAYERS;
    C.p = P.p;
    C.remap = compact && at == 0 ? P.remap : nullptr;
    bool bulk = true;
    for (int i = 0; i < C.layers; ++i) {
      C.layer[i] = layer_of(caches[at + i]);
      bulk = bulk && C.layer[i].unit == 16 && C.layer[i].joined;
    }
    const int rows = 2 * C.layers + (C.remap != nullptr), ctas = rr_sm_count() * (bulk ? COPY_CTAS : 4);
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(ctas / rows > 0 ? ctas / rows : 1, rows);
    cfg.blockDim = dim3(bulk ? COPY_NT : UNITS_NT);
    cfg.dynamicSmemBytes = bulk ? COPY_SMEM : 0;
    cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = 1;
    rr_count_launch();
    if ((e = cudaLaunchKernelEx(&cfg, bulk ? copy_bulk_kernel : copy_units_kernel, C)) != cudaSuccess) return rr_cuda_fail(e, who);
  }
  return RR_OK;
}

int launch_pool(void (*kernel)(PoolParams), const PoolParams& P, int ctas, int threads, size_t smem, cudaStream_t st, const char* who) {
  rr_count_launch();
  const cudaError_t e = rr_launch_pdl(kernel, ctas, threads, smem, st, P);
  return e == cudaSuccess ? RR_OK : rr_cuda_fail(e, who);
}

}  // namespace

extern "C" int rr_pages_workspace(const rr_page_pool* pool, size_t* bytes) {
  const int rc = check_pool(pool);
  if (rc != RR_OK) return rc;
  if (!bytes) return RR_ERR_INVALID_ARG;
  *bytes = workspace_bytes(*pool);
  return RR_OK;
}

extern "C" int rr_pages_fork(const rr_page_pool* pool, const int32_t* parents, const int32_t* lens, int32_t* new_lens, void* workspace, size_t bytes,
                             void* stream) {
  int rc = check_pool(pool);
  if (rc != RR_OK) return rc;
  if (!parents || !lens || !new_lens) return RR_ERR_INVALID_ARG;
  // new_lens is written while parents, lens and the pool's state are read
  const int64_t row = 4 * (int64_t)pool->batch, table = 4 * ((pool->batch - 1) * pool->table_stride + pool->pages_per_seq);
  const bool apart = rr_apart(new_lens, row, parents, row) && rr_apart(new_lens, row, lens, row) && rr_apart(new_lens, row, pool->held, row) &&
                     rr_apart(new_lens, row, pool->room, row) && rr_apart(new_lens, row, pool->refs, 4 * (int64_t)pool->num_pages) &&
                     rr_apart(new_lens, row, pool->free_pages, 4) && rr_apart(new_lens, row, pool->status, 4) && rr_apart(new_lens, row, pool->page_table, table);
  if (!apart) return RR_ERR_INVALID_ARG;
  if (((uintptr_t)parents | (uintptr_t)lens | (uintptr_t)new_lens) & 3) return RR_ERR_INVALID_ARG;
  if ((rc = check_workspace(pool, workspace, bytes)) != RR_OK) return rc;
  PoolParams P{*pool, work_of(*pool, workspace), parents, lens, new_lens, nullptr, 0, 0, 0};
  cudaStream_t st = (cudaStream_t)stream;
  if ((int64_t)pool->batch * pool->pages_per_seq <= LONG_TABLE)
    return launch_pool(fork_kernel, P, CL, FORK_NT, pool->batch > ROWS_ON_CHIP ? 0 : sizeof(Heir) * pool->batch, st, "rr_pages_fork");
  const int64_t units = (int64_t)pool->batch * ((pool->pages_per_seq + RUN - 1) / RUN), ctas = (units + LONG_NT / 32 - 1) / (LONG_NT / 32), most = 4 * rr_sm_count();
  if ((rc = launch_pool(fork_stage_kernel, P, (int)(ctas < most ? ctas : most), LONG_NT, 0, st, "rr_pages_fork")) != RR_OK) return rc;
  return launch_pool(fork_write_kernel, P, (int)(ctas < most ? ctas : most), LONG_NT, 0, st, "rr_pages_fork");
}

extern "C" int rr_pages_reserve(const rr_page_pool* pool, const int32_t* lens, const int32_t* new_tokens, int32_t new_each, const rr_paged_kv* caches,
                                int32_t n, void* workspace, size_t bytes, void* stream) {
  int rc = check_pool(pool);
  if (rc != RR_OK) return rc;
  if (!lens || (((uintptr_t)lens | (uintptr_t)new_tokens) & 3) || (!new_tokens && new_each < 0)) return RR_ERR_INVALID_ARG;
  if ((rc = check_caches(pool, caches, n)) != RR_OK) return rc;
  if ((rc = check_workspace(pool, workspace, bytes)) != RR_OK) return rc;
  PoolParams P{*pool, work_of(*pool, workspace), new_tokens, lens, nullptr, nullptr, new_each, slots_of(pool->batch), words_of(*pool)};
  static unsigned long long done = 0;
  constexpr size_t given = GIVEN * 4, most = given + sizeof(Row) * ROWS_ON_CHIP + sizeof(Slot) * 2 * ROWS_ON_CHIP;
  const cudaError_t e = rr_once_per_device(done, [] { return cudaFuncSetAttribute(reserve_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most); });
  if (e != cudaSuccess) return rr_cuda_fail(e, "rr_pages_reserve");
  rc = launch_pool(reserve_kernel, P, CL, NT, given + (pool->batch > ROWS_ON_CHIP ? 0 : row_state(*pool)), (cudaStream_t)stream, "rr_pages_reserve");
  return rc != RR_OK ? rc : launch_copies(P, caches, n, false, (cudaStream_t)stream, "rr_pages_reserve");
}

extern "C" int rr_pages_compact(const rr_page_pool* pool, const rr_paged_kv* caches, int32_t n, int32_t* new_ids, void* workspace, size_t bytes,
                                void* stream) {
  int rc = check_pool(pool);
  if (rc != RR_OK) return rc;
  if ((uintptr_t)new_ids & 3) return RR_ERR_INVALID_ARG;
  if ((rc = check_caches(pool, caches, n)) != RR_OK) return rc;
  if ((rc = check_workspace(pool, workspace, bytes)) != RR_OK) return rc;
  PoolParams P{*pool, work_of(*pool, workspace), nullptr, nullptr, nullptr, new_ids, 0, 0, words_of(*pool)};
  if (!P.remap) P.remap = P.w.ranked;
  rc = launch_pool(compact_kernel, P, CL, NT, 0, (cudaStream_t)stream, "rr_pages_compact");
  return rc != RR_OK ? rc : launch_copies(P, caches, n, true, (cudaStream_t)stream, "rr_pages_compact");
}
