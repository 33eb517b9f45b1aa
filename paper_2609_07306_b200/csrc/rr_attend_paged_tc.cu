// Segments of attention over a paged cache on the 5th-generation tensor cores: bf16, dh 64 or 128 (see rr_attend_paged.cuh
// for items, segments and how their partial results are joined).
//
// One CTA per SM walks its segments.  Per tile of 128 tokens and 128 query rows:  S = Q K^T (TMEM, FP32), softmax against a
// running reference, P (bf16, written over S in TMEM) and O += P V (TMEM, FP32).  P has the values' 16 bits because the product takes operands of one
// type; a high and a low part would take a third product and half the TMEM stores again.  The sum is of the unrounded weights.  Error against 64
// bits 0.0022 to 0.0023 relative, 0.0017 for a bf16 output of FP32 weights.  Two streams of four warps:
//   a segment of more than 128 rows is paired: stream 0 has rows 0..127, stream 1 the others, each tile of keys and values is
//   read once for both;
//   one of up to 128 rows is split: both streams have the same rows, stream 0 the even tiles and stream 1 the odd ones, and
//   each leaves a partial result of its own;
//   one of up to 32 rows (a decoding step) is quartered besides: each of a stream's four warps has a copy of the rows in its 32 lanes and 16
//   of every 64 tokens, whose weights alone are not zero there, so that the exponentials are spread over the SM.
// The tensor pipe takes 2 x 520 cycles for a 128 x 128 x 128 tile's two products, the 16384 exponentials take 1024 on the special-function
// unit.  Measured: 545 to 600 us for 475 GFLOP of a routed prompt (up to 870 TFLOP/s, tensor pipe 42 %), 650 for 481 GFLOP of prompts behind a prefix; what
// bounds them is a stream's chain of logits, maximum, exponentials and weights, about 2000 cycles per 64 tokens of two tiles.
//
// Warps 0-3, 4-7: the streams, a thread per row.  8, 11: issue the products, one stream's each.  9: finds the segments.  10: the rows' limits.
// 12-15: copies of token and query rows, 32 rows each.  Where those 32 tokens are runs of 32, 16 or 8 in a page, TMA brings
// a run per copy (and half of 64 entries); else 16 bytes per thread, through whatever pages they lie in, and zeros
// for a place without a token.  Segments go round in a ring, so that the next one's look-ups and queries are there before it begins.
// (16 bytes per thread for every tile cost the copying warps 2000 cycles of a tile, and the streams issue slots; TMA's tile::gather4,
// four token rows per copy, about 100 cycles of issue per copy, 8 us per tile.)
// A stream has 64 columns of S per half tile: one half's logits are there or under way while the other's weights are made (whole tiles of S: 636
// us instead of 595).  A half's logits are issued behind the product with the weights before, which reads the same columns; the tensor
// pipe keeps that order.
//
// The reference of the softmax follows the row's maximum only when that has grown by more than 8 (a factor of
// 256): weights up to 2^8 lose nothing in bf16 and FP32, and the output is rescaled in TMEM a few times per
// segment instead of at every tile.
//
// Every wait is bounded; one that runs out sets RR_STATUS_TIMEOUT, and the CTA waits for its copies and
// products in flight, frees its TMEM and returns.
#include <algorithm>
#include "rr_attend_paged_again.cuh"
#include "rr_sm100.cuh"

using namespace rrattn;
using namespace sm100;

namespace {

constexpr int NT = 512, IDS = 16, FILLS = 16, MAX_RING = 4;
constexpr float GROWTH = 8.f;
constexpr int BY_FMA = 2;                              // of every 8 pairs of exponentials, by multiply-adds (0: 567 us, 1: 551, 2: 544 of a routed prompt)

template <int D> struct Shape {
  static constexpr int HALVES = D / 64, STAGES = D == 128 ? 4 : 8;
  static constexpr int HALF_BYTES = TILE * 128, TILE_BYTES = HALVES * HALF_BYTES;
};

// A wait tells phases apart by their parity only.  In a split segment each issuing warp waits for the tiles of its own stream, so the one
// before on the same place may be the other's, and may not be there yet: `full` goes by the count of fills (fill f in f % FILLS), not by place.
// When a warp waits for fill f, fill f - 16 is long there: f - 16 and f - 16 + STAGES share a place, and the second was asked for, so the first
// had arrived and been released, before the last fill that this warp waited for, or before the queries of this segment (at most 4 before f).
// (The other barriers are waited for in every phase, or, the queries' and the ids', behind one that was told later.)
struct Ctl {
  uint64_t full[FILLS], empty[8], s_full[2][2], p_full[2][2], o_done[2][2], q_full[2], q_empty[2], ids_full[IDS], seg_full[MAX_RING], seg_empty[MAX_RING],
      rows_full[MAX_RING], drain;
  uint32_t tmem_base, abort_flag, marked;              // marked: a row of a call without a join
  Seg seg[MAX_RING];
  int limit[MAX_RING][ROWS];
  int ids[IDS][TILE];
  int4 info[IDS][4];                                   // per copying warp: largest, first, last id; whether they ascend
};

struct Smem {
  template <int D> __host__ __device__ static constexpr int ctl() { return (2 + Shape<D>::STAGES) * Shape<D>::TILE_BYTES; }
  template <int D> __host__ __device__ static constexpr int slots() { return ctl<D>() + (int)((sizeof(Ctl) + 15) / 16 * 16); }
  template <int D> static int total(int n_slots, int ring) { return 1024 + slots<D>() + (n_slots > 0 ? ring * (2 * n_slots + 1) * 4 : 0); }
};

// 16 bytes from global to shared memory, zeros if n == 0.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
// `rows` tokens from place y of a page on, 64 entries from x on; a converged warp calls, one lane issues.
__device__ __forceinline__ void tma_rows_warp(uint32_t dst, const CUtensorMap* map, int x, int y, int head, int page, uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(head), "r"(page), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void expect_tx_warp(uint64_t* bar, uint32_t bytes) {
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}"
               ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// The values as second operand: its rows are the product's summed dimension (tokens), 128 bytes apart, the 64 columns of a half contiguous
// (MN-major, 128-byte swizzle): groups of 8 rows 1024 bytes apart, halves HALF_BYTES apart.
__device__ __forceinline__ uint64_t desc_mn_sw128(uint32_t addr, uint32_t half_bytes) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(half_bytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__host__ __device__ constexpr uint32_t idesc_b_mn(int M, int N) { return umma_idesc_bf16(M, N) | 1u << 16; }

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// No use of these registers is moved above this point.
__device__ __forceinline__ void tie(uint32_t (&r)[32]) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t y; asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo)); return y;
}

// Where a token is: its page (-1: zeros) and place there; box: which of the maps' boxes bring the warp's rows (1, 2, 3: 32, 16, 8 tokens), 0: none
struct Where { int page, place, box; };

// 16 rows x 32 columns: register 4 j + 0, 1 of lane 4 g + q has columns 8 j + 2 q, + 1 of row g, registers 4 j + 2, 3 those of row g + 8.
__device__ __forceinline__ void tmem_ld_16x256_x4(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tie16(uint32_t (&r)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}
// Word j of lane q of every four lanes goes to word q of lane j.
__device__ __forceinline__ void quad_transpose(uint32_t (&w)[4]) {
  const int q = threadIdx.x & 3;
#pragma unroll
  for (int step = 1; step <= 2; step <<= 1) {
    const bool up = q & step;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j & step) continue;
      const uint32_t got = __shfl_xor_sync(FULL, up ? w[j] : w[j | step], step);
      if (up) w[j] = got; else w[j | step] = got;
    }
  }
}

// Pairs of FP32 numbers: one instruction for both.
__device__ __forceinline__ uint64_t two(float lo, float hi) { uint64_t y; asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(lo), "f"(hi)); return y; }
__device__ __forceinline__ void split(uint64_t x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t y; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c)); return y; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t y; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b)); return y; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t y; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b)); return y; }
__device__ __forceinline__ float max3(float a, float b, float c) { float y; asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c)); return y; }
__device__ __forceinline__ float max_nan(float a, float b) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b)); return y; }

// 2^x of a pair by multiply-adds, beside the special-function unit (16 results a cycle and SM), which the exponentials of a tile
// alone would keep busy as long as the tensor pipe.  x = n + r, |r| <= 1/2 (Cody and Waite's reduction; n by adding 1.5 * 2^23), and
// 2^r by the polynomial of degree 4 with constant term 1 whose largest relative error there is smallest (2.9e-6, by linear
// programming over 4001 points; the weights are rounded to bf16, 2^-9).  n <= -127 gives 0, NaN stays NaN.
__device__ __forceinline__ uint64_t exp2_fma(uint64_t x) {
  float x0, x1;
  split(x, x0, x1);
  x = two(max_nan(x0, -127.f), max_nan(x1, -127.f));
  const uint64_t shift = two(12582912.f, 12582912.f), t = add2(x, shift), n = add2(t, two(-12582912.f, -12582912.f));
  const uint64_t r = fma2(n, two(-1.f, -1.f), x);
  uint64_t p = fma2(two(0.009582852944731712f, 0.009582852944731712f), r, two(0.055906426161527634f, 0.055906426161527634f));
  p = fma2(p, r, two(0.24024099111557007f, 0.24024099111557007f));
  p = fma2(p, r, two(0.6931241750717163f, 0.6931241750717163f));
  p = fma2(p, r, two(1.f, 1.f));
  float t0, t1;
  split(t, t0, t1);
  return mul2(p, two(__uint_as_float(__float_as_uint(t0) * 0x800000u + 0x3F800000u), __uint_as_float(__float_as_uint(t1) * 0x800000u + 0x3F800000u)));
}

// Keys and values as [pages][heads][page tokens][entries] with boxes of 32, 16 and 8 tokens.
struct Maps { CUtensorMap k[3], v[3]; };

// Whole items in turn: no join comes behind, so each of the streams' warps looks at the rows that it has marked itself.
__device__ __noinline__ void look_at_own(const Params& P) {
  const int lane = threadIdx.x & 31, mg = P.m * P.group, qt = (mg + ROWS - 1) / ROWS;
  for (long long u = blockIdx.x; u < range_units(P); u += gridDim.x) {
    const long long row = quot(u, qt), row0 = (u - row * qt) * ROWS + (threadIdx.x & ~31u);
    unsigned marked = __ballot_sync(FULL, row0 + lane < mg && P.marks[row * mg + row0 + lane]);
    for (; marked; marked &= marked - 1) look_again<__nv_bfloat16, 1>(P, row * mg + row0 + __ffs(marked) - 1, false, 0, 1, Part{nullptr, nullptr, nullptr});
  }
}

// OWN: no join comes behind.  (A build of its own: the call's stack costs every launch of the kernel a hundredth.)
template <int D, bool OWN>
__global__ void __launch_bounds__(NT, 1)
attend_tc_kernel(const __grid_constant__ Params P, const __grid_constant__ Maps maps, const int ring) {
  using S = Shape<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t q_addr = smem_u32(smem), kv_addr = q_addr + 2 * S::TILE_BYTES;
  Ctl* const c = (Ctl*)(smem + Smem::ctl<D>());
  int* const slot_table = (int*)(smem + Smem::slots<D>());
  volatile uint32_t* const abort_flag = &c->abort_flag;
  const int warp = __shfl_sync(FULL, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < FILLS; ++i) mbar_init(&c->full[i], 4);
    for (int i = 0; i < S::STAGES; ++i) mbar_init(&c->empty[i], 2);
    for (int i = 0; i < 2; ++i) {
      for (int h = 0; h < 2; ++h) { mbar_init(&c->s_full[i][h], 2); mbar_init(&c->p_full[i][h], 128); mbar_init(&c->o_done[i][h], 1); }
      mbar_init(&c->q_full[i], 4); mbar_init(&c->q_empty[i], 2);
    }
    for (int i = 0; i < IDS; ++i) mbar_init(&c->ids_full[i], 4);
    for (int i = 0; i < MAX_RING; ++i) { mbar_init(&c->seg_full[i], 1); mbar_init(&c->seg_empty[i], 15); mbar_init(&c->rows_full[i], 1); }
    mbar_init(&c->drain, 2);
    c->abort_flag = c->marked = 0;
    mbar_fence_init();
    for (int i = 0; i < 3; ++i) { tma_prefetch_desc(&maps.k[i]); tma_prefetch_desc(&maps.v[i]); }
  }
  if (warp == 8) tmem_alloc(&c->tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(FULL, c->tmem_base, 0);
  rr_pdl_wait();
  rr_pdl_trigger();
  // The segment ring as its readers see it: n counts segments.
  auto seg_wait = [&](int n) -> bool { return __all_sync(FULL, mbar_wait_spin(&c->seg_full[n % ring], n / ring & 1, abort_flag)); };
  auto seg_done = [&](int n) { __syncwarp(); if (lane == 0) mbar_arrive(&c->seg_empty[n % ring]); };

  // of the launch's 512 x 128 registers: 256 threads x 184 for the streams, 256 x 72 for the others
  if (warp < 8) {
    regs_up<184>();
    // ===== a stream: thread = row =====
    const int st = warp >> 2, quarter = warp & 3;
    const int r_in = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_tm = tmem + lanes + st * 128, o_tm = tmem + lanes + 256 + st * 128;
    uint32_t s_cnt = 0, o_cnt = 0;
    int tiles = 0;
    bool ok = true;
    for (int n = 0; ok && seg_wait(n); ++n) {
      const Seg& s = c->seg[n % ring];
      if (s.rows == 0) break;
      const bool paired = s.rows > TILE;
      const bool quart = P.streams > 2 && s.rows <= 32;
      const int nt = s.tile1 - s.tile0, r = paired ? st * TILE + r_in : quart ? lane : r_in;
      const int steps = paired ? nt : (nt - st + 1) / 2;
      const bool live = r < s.rows, warp_live = r - lane < s.rows;
      ok = __all_sync(FULL, mbar_wait_spin(&c->rows_full[n % ring], n / ring & 1, abort_flag));
      if (!ok) break;
      const int limit = live ? c->limit[n % ring][r] : 0;
      float ref = NINF, sum = 0.f;
      bool seen = false, mixed = false;
      for (int k = 0; ok && k < 2 * steps; ++k) {      // half a tile, 64 tokens, at a time
        const int h = k & 1, cnt = tiles + (paired ? k >> 1 : (k & ~1) + st);
        // (the issuing warp has waited for the tile's ids before it issued the first half's logits)
        ok = __all_sync(FULL, mbar_wait(&c->s_full[st][h], s_cnt & 1, abort_flag));
        if (!ok) break;
        s_cnt += h;
        tc_fence_after();
        const int* const ids = c->ids[cnt % IDS] + 64 * h;
        // The reference goes up with the largest logit, and what is there is scaled down (ref = -inf: the first finite maximum).
        auto follow = [&](float top) -> bool {
          const float m = live && top != NINF ? top * P.scale_log2 : NINF;
          if (!__any_sync(FULL, m > ref + GROWTH)) return true;
          const float now = m > ref + GROWTH ? m : ref, f = now == ref ? 1.f : ex2(ref - now);
          ref = now;
          sum *= f;
          if (k == 0) return true;
          // the product with the half before may be under way (the one before that is not: this half's logits stand behind it)
          if (!__all_sync(FULL, mbar_wait(&c->o_done[st][h ^ 1], (o_cnt + ((k - 1) >> 1)) & 1, abort_flag))) return false;
          tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < D / 32; ++i) {
            uint32_t o[32];
            tmem_ld32(o_tm + i * 32, o);
            tmem_ld_wait();
            tie(o);
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tmem_st_32x32(o_tm + i * 32, o);
          }
          return true;
        };
        if (quart) {
          // 16 of the 64 columns; the others weigh nothing for this copy of the rows
          uint32_t x[16], p[16];
          const int top_id = max(c->info[cnt % IDS][2 * h].x, c->info[cnt % IDS][2 * h + 1].x);
          tmem_ld16(s_tm + h * 64 + quarter * 16, x);
          if (!__any_sync(FULL, live && top_id >= limit)) {
            seen = true;
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int id = ids[quarter * 16 + j];
              const bool sees = id < limit;
              seen = seen || sees;
              if (!sees) x[j] = 0xFF800000u;
            }
          }
          float top = __uint_as_float(x[0]);
#pragma unroll
          for (int j = 1; j < 15; j += 2) top = max3(top, __uint_as_float(x[j]), __uint_as_float(x[j + 1]));
          ok = follow(fmaxf(top, __uint_as_float(x[15])));
          if (!ok) break;
          const float sub = ref == NINF ? 0.f : ref;
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float e0 = ex2(fmaf(__uint_as_float(x[2 * j]), P.scale_log2, -sub)), e1 = ex2(fmaf(__uint_as_float(x[2 * j + 1]), P.scale_log2, -sub));
            part += e0 + e1;
            p[j] = pack(e0, e1);
            p[8 + j] = 0;
          }
          sum += part;
#pragma unroll
          for (int w = 0; w < 4; ++w) if (w == quarter) tmem_st8(s_tm + h * 64 + w * 8, p); else tmem_st8(s_tm + h * 64 + w * 8, p + 8);
          tmem_st_wait();
        } else if (warp_live) {
          uint32_t x[2][32];
#pragma unroll
          for (int i = 0; i < 2; ++i) tmem_ld32(s_tm + h * 64 + i * 32, x[i]);
          const int4 i0 = c->info[cnt % IDS][2 * h], i1 = c->info[cnt % IDS][2 * h + 1];
          const bool masked = __any_sync(FULL, live && max(i0.x, i1.x) >= limit);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 2; ++i) tie(x[i]);
          if (!masked) {
            seen = true;
          } else {                                     // which columns the row sees, a bit each
            uint32_t see[2] = {0, 0};
            if (i0.w && i1.w && i0.z <= i1.y) {
              int n = 0;                               // ids ascend (every list in order, no bad page inside): the first n columns
#pragma unroll
              for (int step = 32; step; step >>= 1) if (ids[n + step - 1] < limit) n += step;
              n += ids[n] < limit;
              mixed = mixed || (n < 64 && ids[min(n, 63)] != NO_TOKEN);
              see[0] = n >= 32 ? FULL : (1u << n) - 1;
              see[1] = n >= 64 ? FULL : n <= 32 ? 0u : (1u << (n - 32)) - 1;
            } else {
#pragma unroll
              for (int i = 0; i < 2; ++i)
#pragma unroll 4
                for (int j = 0; j < 32; ++j) {
                  const int id = ids[i * 32 + j];
                  if (id < limit) see[i] |= 1u << j;
                  else mixed = mixed || id != NO_TOKEN;
                }
            }
            seen = seen || (see[0] | see[1]) != 0;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 32; ++j) if (!(see[i] >> j & 1)) x[i][j] = 0xFF800000u;
          }
          float t[4];                                  // (four chains)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t* const y = &x[i >> 1][(i & 1) * 16];
            t[i] = __uint_as_float(y[0]);
#pragma unroll
            for (int j = 1; j < 15; j += 2) t[i] = max3(t[i], __uint_as_float(y[j]), __uint_as_float(y[j + 1]));
            t[i] = fmaxf(t[i], __uint_as_float(y[15]));
          }
          ok = follow(fmaxf(max3(t[0], t[1], t[2]), t[3]));
          if (!ok) break;
          const float sub = ref == NINF ? 0.f : ref;
          const uint64_t scale2 = two(P.scale_log2, P.scale_log2), sub2 = two(-sub, -sub);
          uint64_t a[2] = {0, 0};
          uint32_t p[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const uint32_t* const y = &x[j / 16][2 * (j % 16)];
            const uint64_t v = fma2(two(__uint_as_float(y[0]), __uint_as_float(y[1])), scale2, sub2);
            uint64_t e;
            if (j % 8 < BY_FMA) {
              e = exp2_fma(v);
            } else {
              float v0, v1;
              split(v, v0, v1);
              e = two(ex2(v0), ex2(v1));
            }
            a[j & 1] = add2(a[j & 1], e);
            float e0, e1;
            split(e, e0, e1);
            p[j] = pack(e0, e1);
          }
          float s0, s1;
          split(add2(a[0], a[1]), s0, s1);
          sum += s0 + s1;
          tmem_st_32x32(s_tm + h * 64, p);
          tmem_st_wait();
        }
        tc_fence_before();
        mbar_arrive(&c->p_full[st][h]);
      }
      if (!ok) break;
      tiles += nt;
      if (steps > 0) {
        o_cnt += steps;
        ok = __all_sync(FULL, mbar_wait(&c->o_done[st][1], (o_cnt - 1) & 1, abort_flag));
        if (!ok) break;
        tc_fence_after();
      }
      const bool direct = paired && s.whole;
      if (warp_live) {
        if (seen && ref == NINF) ref = LOWEST;
        const int part = paired ? 0 : quart ? st * 4 + quarter : st;
        const long long at = (part == 0 ? s.part : s.more + (long long)(part - 1) * s.step) + r;
        const float inv = sum == 0.f ? (ref == NINF ? 0.f : __int_as_float(0x7fc00000)) : 1.f / sum;
        const RowAt a{s.t_base + (s.row0 + r) / P.group, s.h0 + (s.row0 + r) % P.group, 0};
        __nv_bfloat16* const out = (__nv_bfloat16*)P.out + out_at(P, s, a);
        // only then can a value have come in that its row may not see, or that belongs to another quarter
        mixed = mixed || quart;
        const bool look = __any_sync(FULL, mixed);
        unsigned odd_rows = 0;
        if (direct || steps > 0) {
          // TMEM in blocks of 16 rows x 8 columns: lane 4 g + q has columns 2 q, 2 q + 1 of rows g and g + 8, so that after an exchange
          // inside each four lanes these write 64 bytes of a row together (a thread per row would touch 32 lines per store)
          const int g = lane >> 2, q = lane & 3;
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            const float inv0 = __shfl_sync(FULL, inv, half * 16 + g), inv1 = __shfl_sync(FULL, inv, half * 16 + g + 8);
            const unsigned long long out0 = __shfl_sync(FULL, (unsigned long long)out, half * 16 + g), out1 = __shfl_sync(FULL, (unsigned long long)out, half * 16 + g + 8);
            const bool live0 = r - lane + half * 16 + g < s.rows, live1 = r - lane + half * 16 + g + 8 < s.rows;
            float* const part0 = P.part_o + (at - lane + half * 16 + g) * D;
            if (r - lane + half * 16 >= s.rows) continue;
            uint32_t odd0 = 0, odd1 = 0, all[D / 32][16];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
              if (steps > 0) {
                tmem_ld_16x256_x4(o_tm + ((uint32_t)(half * 16) << 16) + i * 32, all[i]);
              } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) all[i][j] = 0;
              }
            }
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
              uint32_t (&o)[16] = all[i];
              tie16(o);
              if (look) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  odd0 = max(odd0, max(o[4 * j] & 0x7FFFFFFFu, o[4 * j + 1] & 0x7FFFFFFFu));
                  odd1 = max(odd1, max(o[4 * j + 2] & 0x7FFFFFFFu, o[4 * j + 3] & 0x7FFFFFFFu));
                }
              }
              if (direct) {
                uint32_t w0[4], w1[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  w0[j] = pack(__uint_as_float(o[4 * j]) * inv0, __uint_as_float(o[4 * j + 1]) * inv0);
                  w1[j] = pack(__uint_as_float(o[4 * j + 2]) * inv1, __uint_as_float(o[4 * j + 3]) * inv1);
                }
                quad_transpose(w0);                    // lane q: the 8 columns of block q
                quad_transpose(w1);
                if (live0) *reinterpret_cast<uint4*>((__nv_bfloat16*)out0 + i * 32 + q * 8) = make_uint4(w0[0], w0[1], w0[2], w0[3]);
                if (live1) *reinterpret_cast<uint4*>((__nv_bfloat16*)out1 + i * 32 + q * 8) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
              } else {
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                  // even lanes take block j, odd lanes block j + 1: columns 2 (q & 2) .. + 3 of it
#pragma unroll
                  for (int up = 0; up < 2; ++up) {
                    uint32_t m0 = o[4 * j + 2 * up], m1 = o[4 * j + 2 * up + 1], n0 = o[4 * j + 4 + 2 * up], n1 = o[4 * j + 5 + 2 * up];
                    const uint32_t g0 = __shfl_xor_sync(FULL, q & 1 ? m0 : n0, 1), g1 = __shfl_xor_sync(FULL, q & 1 ? m1 : n1, 1);
                    const uint4 y = q & 1 ? make_uint4(g0, g1, n0, n1) : make_uint4(m0, m1, g0, g1);
                    if (up ? live1 : live0)
                      *reinterpret_cast<uint4*>(part0 + up * 8 * D + i * 32 + (j + (q & 1)) * 8 + (q & 2) * 2) = y;
                  }
                }
              }
            }
            if (look) {
              const unsigned b0 = __ballot_sync(FULL, odd0 >= 0x7F800000u), b1 = __ballot_sync(FULL, odd1 >= 0x7F800000u);
              const unsigned mine = lane >> 3 & 1 ? b1 : b0;                 // lanes 8 .. 15 of a half: the rows g + 8
              if (lane >> 4 == half && (mine >> (4 * (lane & 7)) & 15u)) odd_rows = 1;
            }
          }
        }
        if (live) {
          const bool mark = odd_rows && mixed;
          if (direct) {
            mark_row(P, s.mark + r, mark);
            if (OWN && mark) c->marked = 1;
          } else {
            P.part_ml[at] = make_float2(ref, with_mark(sum, mark));
          }
        }
      }
      tc_fence_before();
      seg_done(n);
    }
  } else {
    regs_down<72>();
    if (warp == 9) {
      // ===== the segments =====
      long long u, u1;
      const bool turns = P.slots && !P.units;          // whole items in turn
      const long long W = P.slots ? range_units(P) : __ldg(P.main.cum + P.batch);
      if (turns) { u = blockIdx.x; u1 = W; }
      else { u = share(P.main, blockIdx.x, W); u1 = share(P.main, blockIdx.x + 1, W); }
      for (int n = 0;; ++n) {
        Seg s;
        const bool end = u >= u1;
        if (end) { s.rows = 0; }
        else if (P.slots) { const int took = range_segment(P, P.main, blockIdx.x, u, u1, s); u += turns ? gridDim.x : took; }
        else u += segment_at(P, P.main, blockIdx.x, u, u1, s);
        if (!__all_sync(FULL, mbar_wait_spin(&c->seg_empty[n % ring], (n / ring & 1) ^ 1, abort_flag))) break;
        if (!end && P.slots) {                           // number the row's tokens
          if (lane == 0) check_len(P, s.b);
          int* const first = slot_table + (n % ring) * (2 * P.slots + 1);
          int* const base = first + P.slots + 1;
          int run = 0;
          for (int j0 = 0; j0 < P.slots; j0 += 32) {
            const int j = j0 + lane;
            int lo = 0, hi = 0;
            if (j < P.slots) slot_span(s, j, lo, hi);
            int incl = hi - lo;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) { const int x = __shfl_up_sync(FULL, incl, off); if (lane >= off) incl += x; }
            if (j < P.slots) { first[j] = run + incl - (hi - lo); base[j] = lo - first[j]; }
            run += __shfl_sync(FULL, incl, 31);
          }
          if (lane == 0) first[P.slots] = run;
          unit_tiles(P, (run + TILE - 1) / TILE, s);
        }
        if (lane == 0) c->seg[n % ring] = s;
        __syncwarp();
        if (lane == 0) mbar_arrive(&c->seg_full[n % ring]);
        if (end) break;
      }
    } else if (warp == 10) {
      // ===== the rows' limits =====
      for (int n = 0; seg_wait(n); ++n) {
        const Seg& s = c->seg[n % ring];
        if (s.rows == 0) break;
        if (s.b >= 0) {                                // one sequence: the limit goes up by one from token to token
          const int len = seq_end(P, s.b), past = len - s.n_seq + (s.t_base - s.t_seq0) + 1;
          for (int r = lane; r < s.rows; r += 32) c->limit[n % ring][r] = P.causal ? max(past + (s.row0 + r) / P.group, 0) : len;
        } else {
          for (int r = lane; r < s.rows; r += 32) c->limit[n % ring][r] = row_at(P, s, r).limit;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&c->rows_full[n % ring]);
        seg_done(n);
      }
    } else if (warp >= 12) {
      // ===== copies: keys two tiles ahead of the values, and behind a segment's first keys its queries, into Q places 0 and 1
      // in turn (a paired segment takes two).  Warp w has rows 32 w .. 32 w + 31 =====
      const int w = warp - 12;
      const uint32_t dst0 = (w * 32 + (lane >> 3)) * 128;              // row lane / 8 of this warp's, 16-byte piece lane % 8
      int tiles = 0, place = 0;                        // of all segments so far
      uint32_t fills = 0;
      // Up to two groups of copies are in flight unannounced: with a third one committed the oldest has landed (wait_group 2), the
      // warp's part of it is made visible to the tensor pipe and its barrier told.
      uint64_t *older = nullptr, *newer = nullptr;
      auto tell = [&](uint64_t* bar) { if (lane == 0 && bar) mbar_arrive(bar); };
      auto commit = [&](uint64_t* bar) {
        cp_async_commit();
        if (older) {
          cp_async_wait<2>();
          fence_proxy_async_smem();
          __syncwarp();
          tell(older);
        }
        older = newer;
        newer = bar;
      };
      auto flush = [&]() {
        cp_async_wait<0>();
        fence_proxy_async_smem();
        __syncwarp();
        tell(older);
        tell(newer);
        older = newer = nullptr;
      };
      auto free_slot = [&](uint64_t* bar, uint32_t parity) -> bool {
        if (__all_sync(FULL, mbar_try_wait(bar, parity))) return true;
        flush();                                       // nothing that has arrived waits for the next fill
        return __all_sync(FULL, mbar_wait_spin(bar, parity, abort_flag));
      };
      // 32 rows of D entries; `at`: the lane's row as an element offset, -1 for zeros
      auto rows32 = [&](const void* from, long long at, uint32_t dst) {
        const uint8_t* const src0 = (const uint8_t*)from + (lane & 7) * 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = i * 4 + (lane >> 3);
          const long long o = __shfl_sync(FULL, at, r);
          const uint8_t* const src = src0 + max(o, 0LL) * 2;
          const uint32_t to = dst + dst0 + i * 512 + (((lane & 7) ^ (r & 7)) << 4);
#pragma unroll
          for (int h = 0; h < S::HALVES; ++h) cp_async16(to + h * S::HALF_BYTES, src + h * 128, o >= 0 ? 16u : 0u);
        }
      };
      bool ok = true;
      for (int n = 0; ok && seg_wait(n); ++n) {
        const Seg& s = c->seg[n % ring];
        if (s.rows == 0) break;
        const int* const first = slot_table + (n % ring) * (2 * P.slots + 1);
        const int* const base = first + P.slots + 1;
        const int n_tok = P.slots ? first[P.slots] : s.tok1 - s.tok0, tile0 = s.tile0, tile1 = s.tile1;
        // this lane's token of a tile: `seek` asks for its page, `find` has its id for the streams and its place in the cache
        int tok = NO_TOKEN, page = -1, col = 0, cur = 0;
        auto seek = [&](int tile) {
          const int num = tile * TILE + w * 32 + lane;
          tok = NO_TOKEN;
          if (tile >= tile1 || num >= n_tok) return;
          if (P.slots) {                               // the slot of the list's num-th token, from the tile before's on
            if (first[min(cur + 4, P.slots)] <= num) {
              int lo = cur + 4, hi = P.slots;
              while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (first[mid] <= num) lo = mid; else hi = mid; }
              cur = lo;
            } else {
              while (first[cur + 1] <= num) ++cur;
            }
            tok = base[cur] + num;
          } else {
            tok = s.tok0 + num;
          }
          col = P.page_shift >= 0 ? tok >> P.page_shift : tok / P.page_tokens;
          page = __ldg((tok < s.prefix ? s.prefix_pages : s.pages) + col);
        };
        auto find = [&](int tile) -> Where {
          Where at{-1, 0, 0};
          if (tile >= tile1) return at;
          const int cnt = tiles + tile - tile0;
          if (tok != NO_TOKEN) {
            if (page >= 0 && page < P.num_pages) {
              at.page = page;
              at.place = tok - col * P.page_tokens;
            } else {
              tok = NO_TOKEN;
              if (P.status) atomicOr(P.status, RR_STATUS_BAD_INDEX);
            }
          }
          // the longest runs (32, 16, 8 tokens of a page) that the warp's places, in groups of as many, hold; whether ids ascend
          const int page_up = __shfl_up_sync(FULL, at.page, 1), place_up = __shfl_up_sync(FULL, at.place, 1), tok_up = __shfl_up_sync(FULL, tok, 1);
          const unsigned breaks = __ballot_sync(FULL, page_up != at.page || place_up + 1 != at.place);
          const bool all = __all_sync(FULL, at.page >= 0), ascend = __all_sync(FULL, lane == 0 || tok_up <= tok);
          const int last = __shfl_sync(FULL, tok, 31), top = ascend ? last : __reduce_max_sync(FULL, tok);
          if (all) at.box = !(breaks & ~1u) ? 1 : !(breaks & ~0x00010001u) ? 2 : !(breaks & ~0x01010101u) ? 3 : 0;
          c->ids[cnt % IDS][w * 32 + lane] = tok;
          if (lane == 0) c->info[cnt % IDS][w] = make_int4(top, tok, last, ascend);
          __syncwarp();
          if (lane == 0) mbar_arrive(&c->ids_full[cnt % IDS]);
          return at;
        };
        auto load = [&](const void* cache, const CUtensorMap* map, const Where& at) -> bool {
          const uint32_t st = fills % S::STAGES;
          uint64_t* const full = &c->full[fills % FILLS];
          if (!free_slot(&c->empty[st], (fills / S::STAGES & 1) ^ 1)) return false;
          if (at.box) {
            const int run = 64 >> at.box;
            expect_tx_warp(full, 32 * D * 2);
#pragma unroll 1
            for (int r = 0; r < 32; r += run) {
              const int pg = __shfl_sync(FULL, at.page, r), pl = __shfl_sync(FULL, at.place, r);
#pragma unroll
              for (int h = 0; h < S::HALVES; ++h)
                tma_rows_warp(kv_addr + st * S::TILE_BYTES + h * S::HALF_BYTES + (w * 32 + r) * 128, map + at.box - 1, h * 64, pl, s.kvh, pg, full);
            }
          } else {
            rows32(cache, at.page < 0 ? -1 : at.page * P.page_stride + s.kvh * P.head_stride + at.place * P.token_stride, kv_addr + st * S::TILE_BYTES);
            commit(full);
          }
          ++fills;
          return true;
        };
        if (tile0 < tile1) {                           // K(0) queries K(1) V(0) K(2) V(1) ... K(n-1) V(n-2) V(n-1)
          Where at[3];
          seek(tile0);
          at[0] = find(tile0);
          seek(tile0 + 1);
          ok = load(P.k, maps.k, at[0]);
          const int rows = s.rows;
          for (int h = 0; ok && h < (rows > TILE ? 2 : 1); ++h, ++place) {
            const int q = place & 1, r = h * TILE + (P.streams > 2 && rows <= 32 ? 0 : w * 32) + lane;   // (quartered: four copies)
            ok = free_slot(&c->q_empty[q], (place >> 1 & 1) ^ 1);
            if (!ok) break;
            long long o = -1;
            if (r < rows) {
              const int idx = s.row0 + r, dt = idx / P.group;
              o = q_at(P, s, RowAt{s.t_base + dt, s.h0 + idx - dt * P.group, 0});
            }
            if (r - lane < rows) rows32(P.q, o, q_addr + q * S::TILE_BYTES);
            commit(&c->q_full[q]);
          }
          at[1] = find(tile0 + 1);
          seek(tile0 + 2);
          if (ok && tile0 + 1 < tile1) ok = load(P.k, maps.k, at[1]);
          if (ok) flush();                             // the queries
          for (int t = tile0; ok && t < tile1; ++t) {
            ok = load(P.v, maps.v, at[0]);
            if (!ok) break;
            at[2] = find(t + 2);
            seek(t + 3);
            if (t + 2 < tile1) ok = load(P.k, maps.k, at[2]);
            at[0] = at[1];
            at[1] = at[2];
          }
          if (!ok) break;
          tiles += tile1 - tile0;
        } else {
          // The last groups of the segment before may be unannounced.  With no copies of its own here this warp would go on to wait for
          // a segment that is published only when that one is done, which waits for them.
          flush();
        }
        if (ok) seg_done(n);
      }
      flush();                                         // (do not leave with copies in flight)
      for (uint32_t f = fills > S::STAGES ? fills - S::STAGES : 0; f < fills; ++f)
        for (uint32_t it = 0; it < kSpinLimit && !mbar_try_wait(&c->full[f % FILLS], f / FILLS & 1); ++it) __nanosleep(64);
      __syncwarp();
    } else {
      // ===== products: warp 8 those of stream 0, warp 11 those of stream 1, so that one's waits
      // stand beside the other's products =====
      constexpr uint32_t idesc_s = umma_idesc_bf16(TILE, 64), idesc_o = idesc_b_mn(TILE, D);
      const int st = warp == 8 ? 0 : 1;
      const uint32_t s_tm = tmem + st * 128, o_tm = tmem + 256 + st * 128;
      int place = 0;
      uint32_t tiles = 0, p_cnt = 0;
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(FULL, mbar_wait_spin(bar, parity & 1, abort_flag)); };
      for (int n = 0; ok && seg_wait(n); ++n) {
        const int rows = __shfl_sync(FULL, c->seg[n % ring].rows, 0);
        const int nt = __shfl_sync(FULL, c->seg[n % ring].tile1 - c->seg[n % ring].tile0, 0);
        if (rows == 0) break;
        const bool paired = rows > TILE;
        const int steps = paired ? nt : (nt - st + 1) / 2;
        if (nt == 0) { seg_done(n); continue; }
        const int at = (place + (paired ? st : 0)) & 1;
        ok = wait(&c->q_full[at], (place + (paired ? st : 0)) >> 1);
        const uint64_t qd = umma_desc_k_sw128(q_addr + at * S::TILE_BYTES);
        // Half a tile (64 tokens) has its own columns of S: while one half's weights are made, the other half's logits are there
        // or under way.  Logits of a tile's half stand behind the product with the weights of the same half of the tile before, which
        // reads the same columns; the tensor pipe keeps that order.
        for (int k = 0; ok && k <= steps; ++k) {
          const int tv = paired ? k - 1 : 2 * (k - 1) + st, tk = paired ? k : 2 * k + st;
          const uint32_t fv = 2 * tiles + (tv == nt - 1 ? 2 * nt - 1 : 2 * tv + 2), fk = 2 * tiles + (tk == 0 ? 0 : 2 * tk - 1);
          const uint32_t sv = fv % S::STAGES, sk = fk % S::STAGES;
          if (k > 0) ok = wait(&c->full[fv % FILLS], fv / FILLS);
          for (int h = 0; ok && h < 2; ++h) {
            if (k > 0) {
              ok = wait(&c->p_full[st][h], p_cnt);
              if (!ok) break;
              tc_fence_after();
              const uint64_t vd = desc_mn_sw128(kv_addr + sv * S::TILE_BYTES + h * 64 * 128, S::HALF_BYTES);
#pragma unroll
              for (int j = 0; j < 4; ++j)
                umma_bf16_ts_warp(o_tm, s_tm + h * 64 + j * 8, vd + (uint64_t)(j * 128), idesc_o, (k > 1 || h > 0 || j > 0) ? 1u : 0u);
              umma_commit_warp(&c->o_done[st][h]);
            }
            if (k < steps) {
              if (h == 0) {
                const int cnt = (int)tiles + tk;
                ok = wait(&c->full[fk % FILLS], fk / FILLS) && wait(&c->ids_full[cnt % IDS], cnt / IDS);
                if (!ok) break;
                tc_fence_after();
              }
              const uint64_t kd = umma_desc_k_sw128(kv_addr + sk * S::TILE_BYTES + h * 64 * 128);
#pragma unroll
              for (int j = 0; j < D / 16; ++j) {
                const uint64_t o = (uint64_t)((j >> 2) * (S::HALF_BYTES >> 4) + (j & 3) * 2);
                umma_bf16_warp(s_tm + h * 64, qd + o, kd + o, idesc_s, j > 0 ? 1u : 0u);
              }
              if (lane == 0) mbar_arrive(&c->s_full[st][h]);   // (passes on the ids' arrival)
              umma_commit_warp(&c->s_full[st][h]);
            }
          }
          if (!ok) break;
          if (k > 0) {
            ++p_cnt;
            umma_commit_warp(&c->empty[sv]);
            if (!paired) umma_commit_warp(&c->empty[sv]);
          }
          if (k < steps) {
            umma_commit_warp(&c->empty[sk]);
            if (!paired) umma_commit_warp(&c->empty[sk]);
          }
          if (k == max(steps - 1, 0)) {                // the queries' place: both streams of a split segment have to be done with it
            umma_commit_warp(&c->q_empty[at]);
            if (paired) umma_commit_warp(&c->q_empty[at]);
          }
        }
        if (!ok) break;
        tiles += nt;
        place += paired ? 2 : 1;
        seg_done(n);
      }
      // TMEM is not freed while a product can still write to it
      umma_commit_warp(&c->drain);
      for (uint32_t it = 0; it < kSpinLimit && !mbar_try_wait(&c->drain, 0); ++it) __nanosleep(64);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
    if (lane == 0 && c->abort_flag && P.status) atomicOr(P.status, RR_STATUS_TIMEOUT);
  }
  if (OWN && c->marked && threadIdx.x < ROWS) look_at_own(P);
}

template <int D>
cudaError_t launch(const Params& p, int grid, cudaStream_t st) {
  Maps maps;
  for (int i = 0; i < 3; ++i) {
    const int box = std::min(32 >> i, p.page_tokens);
    cudaError_t m = rr_encode_tmap_bf16_pages(&maps.k[i], p.k, p.dh, p.page_tokens, p.kv_heads, p.num_pages, p.token_stride, p.head_stride, p.page_stride, box);
    if (m == cudaSuccess) m = rr_encode_tmap_bf16_pages(&maps.v[i], p.v, p.dh, p.page_tokens, p.kv_heads, p.num_pages, p.token_stride, p.head_stride, p.page_stride, box);
    if (m != cudaSuccess) return m;
  }
  const int ring = p.slots > 256 ? 2 : MAX_RING;
  static unsigned long long done = 0;
  const cudaError_t e = rr_once_per_device(done, [] {
    const int most = std::max(Smem::total<D>(256, MAX_RING), Smem::total<D>(RR_MAX_RANGE_SLOTS, 2));
    const cudaError_t a = cudaFuncSetAttribute(attend_tc_kernel<D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return a == cudaSuccess ? cudaFuncSetAttribute(attend_tc_kernel<D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) : a;
  });
  if (e != cudaSuccess) return e;
  return rr_launch_pdl(p.slots && p.part_rows == 0 ? attend_tc_kernel<D, true> : attend_tc_kernel<D, false>, grid, NT, (size_t)Smem::total<D>(p.slots, ring), st, p, maps, ring);
}

}  // namespace

bool rr_attend_tc_supported(const Params& p, int dtype) {
  if (dtype != RR_BF16 || (p.dh != 64 && p.dh != 128) || !(p.scale_log2 > 1e-30f)) return false;   // (the largest product has the largest logit)
  if (((uintptr_t)p.k | (uintptr_t)p.v | (uintptr_t)p.q | (uintptr_t)p.out) & 15) return false;
  if (p.page_stride < 8 || p.head_stride < 8 || p.token_stride < 8 || std::max({p.page_stride, p.head_stride, p.token_stride}) >= 1LL << 38) return false;
  return (p.page_stride | p.head_stride | p.token_stride | p.qb | p.qh | p.qt | p.ob | p.oh | p.ot) % 8 == 0;
}

cudaError_t rr_launch_attend_tc(const Params& p, int grid, cudaStream_t st) { return p.dh == 64 ? launch<64>(p, grid, st) : launch<128>(p, grid, st); }
