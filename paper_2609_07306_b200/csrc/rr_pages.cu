// Who owns which page of the paged cache: forks, room for new tokens, compaction.
//
//   refs[p] = entries of the page table (and of the caller) that hold page p;  0: free
//   fork      row b <- row parents[b], all at once;  refs by the difference of the rows
//   reserve   row b: columns [0, c1), c1 = ceil((lens + new) / page); pages to be written are the row's own (refs 1)
//   compact   L pages in use; the i-th of those >= L goes to the i-th free one below L
//
// The bookkeeping is a few integers per row and one pass over refs: bound by latency, not by bytes.  It runs in one cluster of eight
// CTAs, whose hardware barrier separates the steps (a barrier costs less than a launch, and no wait on memory is needed), a warp per row.  Free
// pages are found by all threads together, 32 pages per thread (eight loads of four refs in flight), in rounds of 262144 pages; counts are
// exchanged through distributed shared memory.  Which page goes where follows from ranks, never from the order of atomics, which only add to
// counters.  Copies of pages are a second kernel over all SMs, which reads on the device how many there are; it is launched along with the first
// and waits for it, for all layers at once.
#include <cooperative_groups.h>
#include "rr_paged.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int CL = 8, NT = 1024, NW = NT / 32;
constexpr int WARP_PAGES = 1024, CTA_PAGES = NW * WARP_PAGES, ROUND = CL * CTA_PAGES;
constexpr int MAX_LAYERS = 64;                          // of one launch of the copy
constexpr int COPY_NT = 256, COPY_UNITS = 8 * COPY_NT;  // units of one step of a copying CTA

struct Move { int32_t src, dst, tokens; };

// The workspace.  `list`: free pages in rank order (reserve); `stage`: new rows (fork); src, dst and remap of a compaction.
struct Work {
  int32_t* moves;                                       // [1] how many
  int32_t* want;                                        // [batch] the page that a row will go on writing, -1: none
  int32_t* need;                                        // [batch] new pages of the row; of a fork, the pages that it takes, -1: it stays
  int32_t* rank;                                        // [batch] rank of the row's first new page
  int32_t* list;
  Move* move;
};

struct PoolParams {
  rr_page_pool p;
  Work w;
  const int32_t* arg;                                   // parents or new_tokens
  const int32_t* lens;
  int32_t* new_lens;
  int32_t* remap;
  int32_t new_each;
};

size_t list_ints(const rr_page_pool& p) {
  const size_t rows = (size_t)p.batch * p.pages_per_seq, pages = 3 * (size_t)p.num_pages;
  return ((rows > pages ? rows : pages) + 3) & ~(size_t)3;
}
size_t most_moves(const rr_page_pool& p) { return (size_t)(p.batch > p.num_pages / 2 ? p.batch : p.num_pages / 2) + 1; }
size_t workspace_bytes(const rr_page_pool& p) {
  const size_t rows = ((size_t)p.batch + 3) & ~(size_t)3;
  return 64 + 4 * (3 * rows + list_ints(p)) + sizeof(Move) * most_moves(p);
}
Work work_of(const rr_page_pool& p, void* ws) {
  const size_t rows = ((size_t)p.batch + 3) & ~(size_t)3;
  Work w;
  w.moves = (int32_t*)ws;
  w.want = w.moves + 16;
  w.need = w.want + rows;
  w.rank = w.need + rows;
  w.list = w.rank + rows;
  w.move = (Move*)(w.list + list_ints(p));
  return w;
}

__device__ __forceinline__ void report(const rr_page_pool& p, uint32_t bit) { if (p.status) atomicOr(p.status, bit); }
__device__ __forceinline__ bool in_pool(const rr_page_pool& p, int id) { return id >= 0 && id < p.num_pages; }
__device__ __forceinline__ int held_of(const rr_page_pool& p, int b) { return min(max(__ldcg(p.held + b), 0), p.pages_per_seq); }
// One holder less; 1 if the page is free now.
__device__ __forceinline__ int release(const rr_page_pool& p, int id) { return atomicSub(p.refs + id, 1) == 1; }
__device__ __forceinline__ int warp_sum(int x) { return __reduce_add_sync(0xFFFFFFFFu, x); }

struct Shared { int warp[NW]; int cta[2]; };

// Exclusive prefix of the warps' counts over the cluster, and their sum.  Rounds alternate between the two places, so that a CTA that is a round ahead
// overwrites nothing that another one still reads.
__device__ __forceinline__ int2 cluster_prefix(cg::cluster_group& cl, Shared& s, int count, int& round) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) s.warp[warp] = count;
  __syncthreads();
  int x = s.warp[lane];
#pragma unroll
  for (int d = 1; d < 32; d *= 2) { const int y = __shfl_up_sync(0xFFFFFFFFu, x, d); if (lane >= d) x += y; }
  const int before = __shfl_sync(0xFFFFFFFFu, x, warp) - count, cta = __shfl_sync(0xFFFFFFFFu, x, 31);
  int* const place = &s.cta[round & 1];
  ++round;
  if (threadIdx.x == 0) *place = cta;
  cl.sync();
  const int theirs = lane < CL ? *cl.map_shared_rank(place, lane) : 0;
  return make_int2(before + warp_sum(lane < (int)cl.block_rank() ? theirs : 0), warp_sum(theirs));
}

// Bit 4 i + e: page first + 128 i + 4 lane + e is free.
__device__ __forceinline__ uint32_t free_bits(const rr_page_pool& p, long long first) {
  const int lane = threadIdx.x & 31;
  const bool vec = ((uintptr_t)p.refs & 15) == 0;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long long g = first + i * 128 + lane * 4;
    if (vec && g + 4 <= p.num_pages) {
      const int4 v = __ldcg((const int4*)(p.refs + g));
      bits |= (uint32_t)((v.x == 0) | (v.y == 0) << 1 | (v.z == 0) << 2 | (v.w == 0) << 3) << (4 * i);
    } else {
      for (int e = 0; e < 4; ++e)
        if (g + e < p.num_pages && __ldcg(p.refs + g + e) == 0) bits |= 1u << (4 * i + e);
    }
  }
  return bits;
}

// f(page, rank, is free) for the pages of this thread in a round, rank = free pages before it, `before` of them before this warp's.
template <class F>
__device__ __forceinline__ void each_page(uint32_t bits, int before, long long first, F&& f) {
  const int lane = threadIdx.x & 31;
  uint32_t lo = 0, hi = 0;                              // a byte per i: free pages of the lanes up to this one (at most 128)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo |= (uint32_t)__popc(bits >> (4 * i) & 15) << (8 * i);
    hi |= (uint32_t)__popc(bits >> (16 + 4 * i) & 15) << (8 * i);
  }
  const uint32_t own_lo = lo, own_hi = hi;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const uint32_t a = __shfl_up_sync(0xFFFFFFFFu, lo, d), b = __shfl_up_sync(0xFFFFFFFFu, hi, d);
    if (lane >= d) lo += a, hi += b;
  }
  const uint32_t all_lo = __shfl_sync(0xFFFFFFFFu, lo, 31), all_hi = __shfl_sync(0xFFFFFFFFu, hi, 31);
  lo -= own_lo, hi -= own_hi;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t mine = i < 4 ? lo : hi, all = i < 4 ? all_lo : all_hi;
    int rank = before + (int)(mine >> (8 * (i & 3)) & 255);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool is_free = bits >> (4 * i + e) & 1;
      f(first + i * 128 + lane * 4 + e, rank, is_free);
      rank += is_free;
    }
    before += (int)(all >> (8 * (i & 3)) & 255);
  }
}

// The `need` lowest free pages into w.list (visible after the next barrier); how many were found, at least `need` if there are as many.
__device__ __forceinline__ int find_free(cg::cluster_group& cl, const PoolParams& P, Shared& s, int need, int& round) {
  int found = 0;
  for (long long at = 0; at < P.p.num_pages && found < need; at += ROUND) {
    const long long first = at + (long long)cl.block_rank() * CTA_PAGES + (threadIdx.x >> 5) * WARP_PAGES;
    const uint32_t bits = free_bits(P.p, first);
    const int2 n = cluster_prefix(cl, s, warp_sum(__popc(bits)), round);
    if (found + n.x < need)
      each_page(bits, found + n.x, first, [&](long long page, int rank, bool is_free) { if (is_free && rank < need) P.w.list[rank] = (int32_t)page; });
    found += n.y;
  }
  return found;
}

// ---- fork -------------------------------------------------------------------------------------------------------
// A row is compared with its parent's: beams differ from one another in their last pages only, and equal entries cost two loads.  New entries
// are staged, as a parent's row may be rewritten in the same call.
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(NT, 1)
fork_kernel(const __grid_constant__ PoolParams P) {
  cg::cluster_group cl = cg::this_cluster();
  const rr_page_pool& p = P.p;
  const int lane = threadIdx.x & 31, warp = cl.block_rank() * NW + (threadIdx.x >> 5);
  rr_pdl_wait();
  rr_pdl_trigger();
  int freed = 0;
  for (int b = warp; b < p.batch; b += CL * NW) {
    int parent = P.arg[b];
    if (parent < -1 || parent >= p.batch) {
      if (lane == 0) report(p, RR_STATUS_BAD_INDEX);
      parent = b;
    }
    const int len = parent < 0 ? 0 : P.lens[parent];
    if (lane == 0) {
      if (len < 0) report(p, RR_STATUS_BAD_INDEX);
      P.new_lens[b] = max(len, 0);
    }
    if (parent == b) {
      if (lane == 0) P.w.need[b] = -1;
      continue;
    }
    const int held = held_of(p, b);
    int takes = 0;                                      // pages with tokens of the parent
    if (parent >= 0) takes = (int)min((long long)held_of(p, parent), ((long long)max(len, 0) + p.page_tokens - 1) / p.page_tokens);
    if (lane == 0) P.w.need[b] = takes;
    const int32_t* const mine = p.page_table + b * p.table_stride;
    const int32_t* const theirs = p.page_table + parent * p.table_stride;
    int32_t* const stage = P.w.list + (size_t)b * p.pages_per_seq;
    for (int c = lane; c < max(held, takes); c += 32) {
      const int was = c < held ? mine[c] : -1, is = c < takes ? theirs[c] : -1;
      stage[c] = is;
      if (was == is) continue;
      if (in_pool(p, is)) freed -= atomicAdd(p.refs + is, 1) == 0;      // (one row may let go of a page before another takes it)
      else if (c < takes) report(p, RR_STATUS_BAD_INDEX);
      if (in_pool(p, was)) freed += release(p, was);
      else if (c < held) report(p, RR_STATUS_BAD_INDEX);
    }
  }
  freed = warp_sum(freed);
  if (lane == 0 && freed) atomicAdd(p.free_pages, freed);
  cl.sync();
  for (int b = warp; b < p.batch; b += CL * NW) {
    const int takes = P.w.need[b];
    if (takes < 0) continue;
    const int held = held_of(p, b);
    int32_t* const mine = p.page_table + b * p.table_stride;
    const int32_t* const stage = P.w.list + (size_t)b * p.pages_per_seq;
    for (int c = lane; c < max(held, takes); c += 32)
      if (const int is = stage[c]; mine[c] != is) mine[c] = is;
    __syncwarp();                                       // every lane has read held
    if (lane == 0) p.held[b] = takes;
  }
}

// ---- reserve ----------------------------------------------------------------------------------------------------
struct Room { int c0, part, c1, held; bool writes; };

// Columns of row b: tokens up to column c0 and `part` of it, room up to column c1.
__device__ __forceinline__ Room room_of(const PoolParams& P, int b, bool tell) {
  const rr_page_pool& p = P.p;
  const long long cap = (long long)p.page_tokens * p.pages_per_seq;
  long long len = P.lens[b], more = P.arg ? P.arg[b] : P.new_each;
  const bool bad = len < 0 || more < 0 || len + more > cap;
  if (bad && tell) report(p, RR_STATUS_BAD_INDEX);
  len = min(max(len, 0LL), cap);
  more = min(max(more, 0LL), cap - len);
  Room r;
  r.c0 = (int)(len / p.page_tokens);
  r.part = (int)(len - (long long)r.c0 * p.page_tokens);
  r.c1 = (int)((len + more + p.page_tokens - 1) / p.page_tokens);
  r.held = held_of(p, b);
  r.writes = more > 0;
  return r;
}

// An entry that gets a new page, until it has it: the page that it held, or that it held none of the pool.
__device__ __forceinline__ int marked(int id) { return -2 - id; }
constexpr int MARKED_NONE = INT32_MIN;

// Whether row b copies the page `want` that it goes on writing: others hold it too, and not all who hold it write it with b as the first of them.
__device__ __forceinline__ bool copies(const PoolParams& P, int b, int want) {
  const int lane = threadIdx.x & 31, holders = __ldcg(P.p.refs + want);
  if (holders <= 1) return false;
  int n = 0, before = 0;
  for (int o = lane; o < P.p.batch; o += 32)
    if (__ldcg(P.w.want + o) == want) ++n, before += o < b;
  return warp_sum(before) > 0 || warp_sum(n) != holders;
}

__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(NT, 1)
reserve_kernel(const __grid_constant__ PoolParams P) {
  __shared__ Shared s;
  __shared__ int s_warp[NW];
  cg::cluster_group cl = cg::this_cluster();
  const rr_page_pool& p = P.p;
  const int lane = threadIdx.x & 31, my_warp = threadIdx.x >> 5, warp = cl.block_rank() * NW + my_warp;
  rr_pdl_wait();
  rr_pdl_trigger();
  int freed = 0, round = 0;
  if (warp == 0 && lane == 0) *P.w.moves = 0;
  // 1. pages behind the room are released; which page each row goes on writing
  for (int b = warp; b < p.batch; b += CL * NW) {
    const Room r = room_of(P, b, lane == 0);
    int32_t* const row = p.page_table + b * p.table_stride;
    for (int c = r.c1 + lane; c < r.held; c += 32) {
      const int id = row[c];
      if (in_pool(p, id)) freed += release(p, id);
      else report(p, RR_STATUS_BAD_INDEX);
      row[c] = -1;
    }
    __syncwarp();                                       // every lane has read held
    if (lane == 0) {
      int want = -1;
      if (r.writes && r.part > 0 && r.c0 < min(r.held, r.c1)) {
        want = row[r.c0];
        if (!in_pool(p, want)) want = -1, report(p, RR_STATUS_BAD_INDEX);
      }
      P.w.want[b] = want;
      if (r.c1 < r.held) p.held[b] = r.c1;
    }
    __syncwarp();
  }
  cl.sync();
  // 2. how many pages each row needs: a copy of the page that it goes on writing, its own ones for pages behind that others hold too, missing ones.
  // Counted now, while nothing changes; what is to be replaced is marked in the table.
  for (int b = warp; b < p.batch; b += CL * NW) {
    const Room r = room_of(P, b, false);
    const int want = __ldcg(P.w.want + b);
    int32_t* const row = p.page_table + b * p.table_stride;
    int need = max(r.c1 - r.held, 0);
    if (want >= 0) {
      const bool copied = copies(P, b, want);
      need += copied;
      if (lane == 0 && copied) row[r.c0] = marked(want);
    }
    for (int c0 = r.c0 + (r.part > 0); c0 < r.held; c0 += 32) {
      const int c = c0 + lane, id = c < r.held ? row[c] : 0;
      const bool bad = c < r.held && !in_pool(p, id);
      const bool fresh = bad || (c < r.held && __ldcg(p.refs + id) > 1);
      if (bad) report(p, RR_STATUS_BAD_INDEX);
      if (fresh) row[c] = bad ? MARKED_NONE : marked(id);
      need += __popc(__ballot_sync(0xFFFFFFFFu, fresh));
    }
    if (lane == 0) P.w.need[b] = need;
  }
  cl.sync();
  // 3. each row's first rank: every CTA adds up all rows and keeps those of its own warps
  int total = 0;
  for (int at = 0; at < p.batch; at += NT) {
    const int b = at + threadIdx.x, need = b < p.batch ? __ldcg(P.w.need + b) : 0;
    int x = need;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) { const int y = __shfl_up_sync(0xFFFFFFFFu, x, d); if (lane >= d) x += y; }
    if (lane == 31) s_warp[my_warp] = x;
    __syncthreads();
    int before = warp_sum(lane < my_warp ? s_warp[lane] : 0);
    const int all = warp_sum(s_warp[lane]);
    __syncthreads();
    if (b < p.batch && b % (CL * NW) / NW == (int)cl.block_rank()) P.w.rank[b] = total + before + x - need;
    total += all;
  }
  const int found = total > 0 ? find_free(cl, P, s, total, round) : 0;
  cl.sync();
  // 4. the pages are handed out
  const bool enough = found >= total;
  if (!enough && warp == 0 && lane == 0) report(p, RR_STATUS_NO_PAGES);
  for (int b = warp; b < p.batch; b += CL * NW) {
    const Room r = room_of(P, b, false);
    const int want = __ldcg(P.w.want + b);
    int32_t* const row = p.page_table + b * p.table_stride;
    const int32_t* next = P.w.list + P.w.rank[b];
    if (want >= 0 && row[r.c0] == marked(want)) {
      __syncwarp();
      if (lane == 0) {
        row[r.c0] = enough ? __ldcg(next) : want;
        if (enough) {
          p.refs[__ldcg(next)] = 1;
          freed += release(p, want) - 1;
          P.w.move[atomicAdd(P.w.moves, 1)] = Move{want, __ldcg(next), r.part};
        }
      }
      ++next;
    }
    for (int c0 = r.c0 + (r.part > 0); c0 < r.held; c0 += 32) {
      const int c = c0 + lane, e = c < r.held ? row[c] : 0;
      const unsigned fresh = __ballot_sync(0xFFFFFFFFu, e < 0);
      if (e < 0) {
        const int id = enough ? __ldcg(next + __popc(fresh & ((1u << lane) - 1))) : -1;
        row[c] = enough ? id : e == MARKED_NONE ? -1 : -2 - e;
        if (enough) {
          p.refs[id] = 1;
          freed += (e == MARKED_NONE ? 0 : release(p, -2 - e)) - 1;
        }
      }
      next += __popc(fresh);
    }
    if (enough && r.c1 > r.held) {
      for (int c = r.held + lane; c < r.c1; c += 32) {
        const int id = __ldcg(next + c - r.held);
        row[c] = id;
        p.refs[id] = 1;
        --freed;
      }
      __syncwarp();
      if (lane == 0) p.held[b] = r.c1;
    }
  }
  freed = warp_sum(freed);
  if (lane == 0 && freed) atomicAdd(p.free_pages, freed);
  cl.sync();                                            // no CTA leaves while another one may read its counts
}

// ---- compact ----------------------------------------------------------------------------------------------------
__global__ void __cluster_dims__(CL, 1, 1) __launch_bounds__(NT, 1)
compact_kernel(const __grid_constant__ PoolParams P) {
  __shared__ Shared s;
  cg::cluster_group cl = cg::this_cluster();
  const rr_page_pool& p = P.p;
  const int my_warp = threadIdx.x >> 5;
  rr_pdl_wait();
  rr_pdl_trigger();
  int round = 0, free_all = 0;
  uint32_t bits = 0;
  for (long long at = 0; at < p.num_pages; at += ROUND) {
    bits = free_bits(p, at + (long long)cl.block_rank() * CTA_PAGES + my_warp * WARP_PAGES);
    free_all += cluster_prefix(cl, s, warp_sum(__popc(bits)), round).y;
  }
  const int live = p.num_pages - free_all;
  // Free pages below `live` by their rank, pages in use from there on by their rank among all in use: the last as many of them as there are free ones below.
  int32_t* const dst = P.w.list;
  int32_t* const src = P.w.list + p.num_pages;
  int before = 0, moves = 0;
  for (long long at = 0; at < p.num_pages; at += ROUND) {
    const long long first = at + (long long)cl.block_rank() * CTA_PAGES + my_warp * WARP_PAGES;
    if (p.num_pages > ROUND) bits = free_bits(p, first);
    int low = 0;
    const int2 n = cluster_prefix(cl, s, warp_sum(__popc(bits)), round);
    each_page(bits, before + n.x, first, [&](long long page, int rank, bool is_free) {
      if (page >= p.num_pages) return;
      if (is_free && page < live) dst[rank] = (int32_t)page, ++low;
      if (!is_free && page >= live) src[page - rank] = (int32_t)page;
      else P.remap[page] = (int32_t)page;
    });
    moves += cluster_prefix(cl, s, warp_sum(low), round).y;
    before += n.y;
  }
  cl.sync();
  for (int i = cl.block_rank() * NT + threadIdx.x; i < moves; i += CL * NT) {
    const int from = __ldcg(src + live - moves + i), to = __ldcg(dst + i);
    P.remap[from] = to;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
    P.w.move[i] = Move{from, to, p.page_tokens};
  }
  if (cl.block_rank() == 0 && threadIdx.x == 0) {
    P.w.moves[0] = moves;
    P.w.moves[1] = live;
    *p.free_pages = free_all;
  }
  cl.sync();
}

// ---- copies -----------------------------------------------------------------------------------------------------
// A page of one layer's keys or values as units of 16 bytes (or of an entry, where strides or addresses do not split): the outer of heads and tokens,
// the inner one, the units of a head's entries.  What lies side by side is merged.
struct Layer {
  char* base[2];                                        // keys, values
  int64_t page, outer, mid;                             // bytes
  int32_t heads, row;                                   // units of a head's entries
  int8_t unit, token_major, joined;                     // joined: the inner of heads and tokens lies side by side
};

struct CopyParams {
  Work w;
  int32_t page_tokens, layers;
  // compaction: the table, too
  int32_t remapped;
  rr_page_pool p;
  const int32_t* remap;
  Layer layer[MAX_LAYERS];
};

// Eight units in flight per thread.  Sources and destinations are different pages.
template <typename U>
__device__ __forceinline__ void copy_units(const Layer& L, const char* src, char* dst, unsigned first, unsigned units, unsigned inner) {
  U v[COPY_UNITS / COPY_NT];
  int64_t at[COPY_UNITS / COPY_NT];
#pragma unroll
  for (int i = 0; i < COPY_UNITS / COPY_NT; ++i) {
    const unsigned u = first + i * COPY_NT + threadIdx.x;
    at[i] = -1;
    if (u < units) {
      const unsigned o = u / inner, r = u - o * inner;
      at[i] = o * L.outer;
      if (L.joined) at[i] += (int64_t)r * sizeof(U);
      else { const unsigned m = r / L.row; at[i] += m * L.mid + (int64_t)(r - m * L.row) * sizeof(U); }
      v[i] = *(const U*)(src + at[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < COPY_UNITS / COPY_NT; ++i)
    if (at[i] >= 0) *(U*)(dst + at[i]) = v[i];
}

__global__ void __launch_bounds__(COPY_NT)
copy_kernel(const __grid_constant__ CopyParams P) {
  rr_pdl_wait();
  rr_pdl_trigger();
  const int moves = __ldcg(P.w.moves);
  if ((int)blockIdx.y == 2 * P.layers) {                // the table of a compacted pool
    const int live = __ldcg(P.w.moves + 1);
    for (int b = blockIdx.x; b < P.p.batch && moves > 0; b += gridDim.x) {
      int32_t* const row = P.p.page_table + b * P.p.table_stride;
      const int held = held_of(P.p, b);
      for (int c = threadIdx.x; c < held; c += COPY_NT) {
        const int id = row[c];
        if (!in_pool(P.p, id)) report(P.p, RR_STATUS_BAD_INDEX);
        else if (id >= live) row[c] = __ldcg(P.remap + id);
      }
    }
    return;
  }
  const Layer& L = P.layer[blockIdx.y >> 1];
  char* const base = L.base[blockIdx.y & 1];
  const unsigned chunks = ((unsigned)L.heads * P.page_tokens * L.row + COPY_UNITS - 1) / COPY_UNITS;
  for (long long item = blockIdx.x; item < (long long)moves * chunks; item += gridDim.x) {
    const int m = (int)(item / chunks);
    const Move mv{__ldcg(&P.w.move[m].src), __ldcg(&P.w.move[m].dst), __ldcg(&P.w.move[m].tokens)};
    const unsigned first = (unsigned)(item - (long long)m * chunks) * COPY_UNITS;
    const unsigned units = (unsigned)L.heads * mv.tokens * L.row, inner = (unsigned)(L.token_major ? L.heads : mv.tokens) * L.row;
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
  if (((uintptr_t)p->page_table | (uintptr_t)p->refs | (uintptr_t)p->held | (uintptr_t)p->free_pages | (uintptr_t)p->status) & 3) return RR_ERR_INVALID_ARG;
  if (p->num_pages > RR_PAGES_MAX_PAGES || (int64_t)p->batch * p->pages_per_seq > (1 << 30)) return RR_ERR_TOO_LARGE;
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
  L.row = (int32_t)(row / L.unit);
  return L;
}

// The copies that the bookkeeping kernel has listed, in all caches; of a compaction also the table.
int launch_copies(const PoolParams& P, const rr_paged_kv* caches, int n, bool compact, cudaStream_t st, const char* who) {
  for (int at = 0; at < n; at += MAX_LAYERS) {
    CopyParams C;
    C.w = P.w;
    C.page_tokens = P.p.page_tokens;
    C.layers = n - at < MAX_LAYERS ? n - at : MAX_LAYERS;
    C.remapped = compact && at == 0;
    C.p = P.p;
    C.remap = P.remap;
    for (int i = 0; i < C.layers; ++i) C.layer[i] = layer_of(caches[at + i]);
    const int rows = 2 * C.layers + C.remapped, ctas = rr_sm_count() * 4;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((ctas + rows - 1) / rows, rows);
    cfg.blockDim = dim3(COPY_NT);
    cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = 1;
    rr_count_launch();
    if (const cudaError_t e = cudaLaunchKernelEx(&cfg, copy_kernel, C); e != cudaSuccess) return rr_cuda_fail(e, who);
  }
  return RR_OK;
}

int launch_pool(void (*kernel)(PoolParams), const PoolParams& P, cudaStream_t st, const char* who) {
  rr_count_launch();
  const cudaError_t e = rr_launch_pdl(kernel, CL, NT, 0, st, P);
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
  if (!parents || !lens || !new_lens || lens == new_lens || parents == new_lens) return RR_ERR_INVALID_ARG;
  if (((uintptr_t)parents | (uintptr_t)lens | (uintptr_t)new_lens) & 3) return RR_ERR_INVALID_ARG;
  if ((rc = check_workspace(pool, workspace, bytes)) != RR_OK) return rc;
  PoolParams P{*pool, work_of(*pool, workspace), parents, lens, new_lens, nullptr, 0};
  return launch_pool(fork_kernel, P, (cudaStream_t)stream, "rr_pages_fork");
}

extern "C" int rr_pages_reserve(const rr_page_pool* pool, const int32_t* lens, const int32_t* new_tokens, int32_t new_each, const rr_paged_kv* caches,
                                int32_t n, void* workspace, size_t bytes, void* stream) {
  int rc = check_pool(pool);
  if (rc != RR_OK) return rc;
  if (!lens || (((uintptr_t)lens | (uintptr_t)new_tokens) & 3) || (!new_tokens && new_each < 0)) return RR_ERR_INVALID_ARG;
  if ((rc = check_caches(pool, caches, n)) != RR_OK) return rc;
  if ((rc = check_workspace(pool, workspace, bytes)) != RR_OK) return rc;
  PoolParams P{*pool, work_of(*pool, workspace), new_tokens, lens, nullptr, nullptr, new_each};
  rc = launch_pool(reserve_kernel, P, (cudaStream_t)stream, "rr_pages_reserve");
  return rc != RR_OK ? rc : launch_copies(P, caches, n, false, (cudaStream_t)stream, "rr_pages_reserve");
}

extern "C" int rr_pages_compact(const rr_page_pool* pool, const rr_paged_kv* caches, int32_t n, int32_t* new_ids, void* workspace, size_t bytes,
                                void* stream) {
  int rc = check_pool(pool);
  if (rc != RR_OK) return rc;
  if ((uintptr_t)new_ids & 3) return RR_ERR_INVALID_ARG;
  if ((rc = check_caches(pool, caches, n)) != RR_OK) return rc;
  if ((rc = check_workspace(pool, workspace, bytes)) != RR_OK) return rc;
  PoolParams P{*pool, work_of(*pool, workspace), nullptr, nullptr, nullptr, new_ids, 0};
  if (!P.remap) P.remap = P.w.list + 2 * (size_t)pool->num_pages;
  rc = launch_pool(compact_kernel, P, (cudaStream_t)stream, "rr_pages_compact");
  return rc != RR_OK ? rc : launch_copies(P, caches, n, true, (cudaStream_t)stream, "rr_pages_compact");
}
