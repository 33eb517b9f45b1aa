// Segments of up to four query rows over a paged cache: bf16, dh 64 or 128 (see rr_attend_paged.cuh for segments and how their partial
// results are joined).
//
// With so few rows the cache's traffic is all: 16 multiply-adds per byte at most.  The tensor cores' kernel holds two tiles of
// keys and values in shared memory, and a load's latency goes by before a tile's place is free again.  Here every warp has
// two blocks of its own, each 8 loads of keys and 8 of values of 32 lanes x 16 bytes (16 tokens of 128 entries, 32 of 64), which it asks for
// with cp.async as soon as it has read what was there: 12 warps and 192 KB on an SM, and no barrier but the warp's.  The
// dot products' halves are exchanged until a token's logit is left in LPT / 8 lanes; its weight goes back to the token's lanes for the
// values.  A token that a row does not see is not multiplied.  The four warps' parts of a segment are joined at its end.
// Measured: 512 rows of 4096 tokens each, dh 128 (1.07 GB): 166 us; with the loads in registers 184; the tensor cores' kernel 216.
#include <algorithm>
#include <type_traits>
#include "rr_attend_paged.cuh"

using namespace rrattn;

namespace {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int WARPS = 4, NT = WARPS * 32, N = 8, BLOCKS = 2;
constexpr float GROWTH = 8.f;                          // the reference follows a row's maximum when that has grown by more (a factor of 256)
constexpr int BLOCK_BYTES = 2 * N * 512, RING_BYTES = WARPS * BLOCKS * BLOCK_BYTES;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t n) {      // zeros if n == 0
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

__device__ __forceinline__ uint64_t two(float lo, float hi) { uint64_t y; asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(lo), "f"(hi)); return y; }
__device__ __forceinline__ void split(uint64_t x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t y; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c)); return y; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t y; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b)); return y; }
__device__ __forceinline__ uint64_t widen(uint32_t x) { return two(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u)); }

template <int D, int R>
__global__ void __launch_bounds__(NT, 3) attend_few_kernel(const __grid_constant__ Params P) {
  constexpr int LPT = D / 8, TP = 32 / LPT, BLOCK = N * TP, DUP = LPT / N;     // lanes per token, tokens per load and per block
  extern __shared__ __align__(16) uint8_t s_mem[];
  __shared__ __align__(16) float s_o[WARPS][R][D];
  __shared__ float2 s_ml[WARPS][R];
  // Behind the tensor cores' kernel of the same call this one needs nothing of it but that the plan is there (it is: that kernel
  // lets its successor start behind its own wait): CTAs start as that kernel's leave, and wait for its end before their own.
  if (P.few_waits) { rr_pdl_wait(); rr_pdl_trigger(); }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane % LPT, grp = lane / LPT;
  const uint4* const ring = reinterpret_cast<const uint4*>(s_mem) + warp * (BLOCKS * BLOCK_BYTES / 16) + lane;
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
  int* const first = reinterpret_cast<int*>(s_mem + RING_BYTES);
  int* const base = first + P.slots + 1;
  const bool turns = P.slots && !P.units;
  const long long W = P.slots ? range_units(P) : __ldg(P.few.cum + P.batch);
  long long u, u1;
  if (turns) { u = blockIdx.x; u1 = W; }
  else { u = share(P.few, blockIdx.x, W); u1 = share(P.few, blockIdx.x + 1, W); }
  while (u < u1) {
    Seg s;
    int n_tok;
    if (P.slots) {
      const int took = range_segment(P, P.few, blockIdx.x, u, u1, s);
      u += turns ? gridDim.x : took;
      if (warp == 0) {                                 // number the row's tokens
        if (lane == 0) check_len(P, s.b);
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
      }
      __syncthreads();
      n_tok = first[P.slots];
      unit_tiles(P, (n_tok + TILE - 1) / TILE, s);
    } else {
      u += segment_at(P, P.few, blockIdx.x, u, u1, s);
      n_tok = s.tok1 - s.tok0;
    }
    uint64_t q[R][4], acc[R][4];
    int limit[R];
    float m[R], l[R];
    unsigned seen = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const RowAt a = r < s.rows ? row_at(P, s, r) : RowAt{0, 0, 0};
      limit[r] = a.limit; m[r] = NINF; l[r] = 0.f;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < s.rows) v = __ldg(reinterpret_cast<const uint4*>((const __nv_bfloat16*)P.q + q_at(P, s, a) + sub * 8));
      q[r][0] = widen(v.x); q[r][1] = widen(v.y); q[r][2] = widen(v.z); q[r][3] = widen(v.w);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[r][j] = 0;
    }
    const int end = min(s.tile1 * TILE, n_tok);
    int cur = 0;
    // the lane's token of the block at num0, and its place in the cache in units of 16 bytes (-1: none)
    auto seek = [&](int num0, int& id, long long& at) {
      const int num = num0 + lane;
      id = NO_TOKEN;
      at = -1;
      if (lane >= BLOCK || num >= end) return;
      if (P.slots) {
        int lo = cur, hi = P.slots;
        if (first[min(cur + 4, P.slots)] > num) {
          while (first[lo + 1] <= num) ++lo;
        } else {
          lo = cur + 4;
          while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (first[mid] <= num) lo = mid; else hi = mid; }
        }
        cur = lo;
        id = base[lo] + num;
      } else {
        id = s.tok0 + num;
      }
      at = token_at(P, s, id);
      if (at < 0) id = NO_TOKEN;
    };
    // Block k of the warp: in place k % BLOCKS; `ids` of the blocks in flight, `next_*` of the one to be asked for.
    const int step = WARPS * BLOCK, num_first = s.tile0 * TILE + warp * BLOCK;
    int ids[BLOCKS], next_id;
    long long next_at;
    auto ask = [&](int place) {
      const uint32_t dst = ring_addr + place * BLOCK_BYTES;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const long long o = __shfl_sync(FULL, next_at, i * TP + grp), from = max(o, 0LL) + sub * 8;
        cp_async16(dst + i * 512, (const __nv_bfloat16*)P.k + from, o >= 0 ? 16u : 0u);
        cp_async16(dst + (N + i) * 512, (const __nv_bfloat16*)P.v + from, o >= 0 ? 16u : 0u);
      }
    };
    seek(num_first, next_id, next_at);
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) {
      ids[k] = next_id;
      if (num_first + k * step < end) ask(k);
      asm volatile("cp.async.commit_group;" ::: "memory");
      seek(num_first + (k + 1) * step, next_id, next_at);
    }
    int place = 0;
    for (int num0 = num_first; num0 < end; num0 += step) {
      const int id = ids[0];
      asm volatile("cp.async.wait_group %0;" ::"n"(BLOCKS - 1) : "memory");
      __syncwarp();
      const uint4* const x = ring + place * (BLOCK_BYTES / 16);
      const uint4* const y = x + N * 32;
      const int my_id = __shfl_sync(FULL, id, sub / DUP * TP + grp);       // lane's token: load sub / DUP of its group
      float wt[R];
      unsigned sees[R];
      float d[R][N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint4 kk = x[i * 32];
        const uint64_t k0 = widen(kk.x), k1 = widen(kk.y), k2 = widen(kk.z), k3 = widen(kk.w);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float lo, hi;
          split(fma2(q[r][3], k3, fma2(q[r][2], k2, fma2(q[r][1], k1, mul2(q[r][0], k0)))), lo, hi);
          d[r][i] = lo + hi;
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int n = N / 2, off = LPT / 2; n >= 1; n >>= 1, off >>= 1) {
          const bool up = sub & off;
#pragma unroll
          for (int i = 0; i < n; ++i) {
            const float keep = up ? d[r][i + n] : d[r][i], give = up ? d[r][i] : d[r][i + n];
            d[r][i] = keep + __shfl_xor_sync(FULL, give, off);
          }
        }
        float z = d[r][0];
#pragma unroll
        for (int off = DUP / 2; off; off >>= 1) z += __shfl_xor_sync(FULL, z, off);
        const bool see = my_id < limit[r];
        sees[r] = __ballot_sync(FULL, see);
        if (sees[r]) seen |= 1u << r;
        z = see ? z * P.scale_log2 : NINF;
        if (__any_sync(FULL, z > m[r] + GROWTH)) {     // (m = -inf: the first finite logit)
          float top = z;
#pragma unroll
          for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, off));
          const float now = fmaxf(m[r], top), f = exp2f(m[r] - now);
          m[r] = now;
          l[r] *= f;
          const uint64_t f2 = two(f, f);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[r][j] = mul2(acc[r][j], f2);
        }
        wt[r] = exp2f(z - (m[r] == NINF ? 0.f : m[r]));
        if (sub % DUP == 0) l[r] += wt[r];
      }
      unsigned common = FULL;
#pragma unroll
      for (int r = 0; r < R; ++r) common &= sees[r];
      auto weigh = [&](auto all) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int from = grp * LPT + i * DUP;
          const uint4 vv = y[i * 32];
          const uint64_t v0 = widen(vv.x), v1 = widen(vv.y), v2 = widen(vv.z), v3 = widen(vv.w);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float w = __shfl_sync(FULL, wt[r], from);
            if (decltype(all)::value || (sees[r] >> from & 1)) {
              const uint64_t w2 = two(w, w);
              acc[r][0] = fma2(w2, v0, acc[r][0]); acc[r][1] = fma2(w2, v1, acc[r][1]);
              acc[r][2] = fma2(w2, v2, acc[r][2]); acc[r][3] = fma2(w2, v3, acc[r][3]);
            }
          }
        }
      };
      if (common == FULL) weigh(std::true_type()); else weigh(std::false_type());
      __syncwarp();                                    // the place has been read
#pragma unroll
      for (int k = 0; k + 1 < BLOCKS; ++k) ids[k] = ids[k + 1];
      ids[BLOCKS - 1] = next_id;
      if (num0 + BLOCKS * step < end) {
        ask(place);
        seek(num0 + (BLOCKS + 1) * step, next_id, next_at);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      place = place + 1 == BLOCKS ? 0 : place + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // the warp's parts: outputs over the groups of lanes, sums over the lanes; then the warps'
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int off = 16; off; off >>= 1) l[r] += __shfl_xor_sync(FULL, l[r], off);
      if ((seen >> r & 1) && m[r] == NINF) m[r] = LOWEST;
      if (lane == 0) s_ml[warp][r] = make_float2(m[r], l[r]);
      float o[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) split(acc[r][j], o[2 * j], o[2 * j + 1]);
#pragma unroll
      for (int off = LPT; off < 32; off <<= 1)
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += __shfl_xor_sync(FULL, o[j], off);
      if (grp == 0) {
        *(float4*)&s_o[warp][r][sub * 8] = make_float4(o[0], o[1], o[2], o[3]);
        *(float4*)&s_o[warp][r][sub * 8 + 4] = make_float4(o[4], o[5], o[6], o[7]);
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < s.rows * D; e += NT) {
      const int r = e / D, c = e % D;
      float M = NINF, L = 0.f, o = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) M = fmaxf(M, s_ml[w][r].x);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float2 ml = s_ml[w][r];
        if (ml.x == NINF) continue;
        const float f = exp2f(ml.x - M);
        L = fmaf(f, ml.y, L);
        o = fmaf(f, s_o[w][r][c], o);
      }
      if (s.whole) {
        const float inv = L == 0.f ? (M == NINF ? 0.f : __int_as_float(0x7fc00000)) : 1.f / L;
        const int idx = s.row0 + r, dt = idx / P.group;
        ((__nv_bfloat16*)P.out)[out_at(P, s, RowAt{s.t_base + dt, s.h0 + idx - dt * P.group, 0}) + c] = __float2bfloat16_rn(o * inv);
      } else {
        P.part_o[(s.part + r) * D + c] = o;
        if (c == 0) P.part_ml[s.part + r] = make_float2(M, with_mark(L, false));
      }
    }
    __syncthreads();                                   // (the parts and the table are free)
  }
  if (!P.few_waits) { rr_pdl_wait(); rr_pdl_trigger(); }
}

template <int D>
cudaError_t launch(const Params& p, int rows, cudaStream_t st) {
  long long grid = p.few.ctas;
  if (p.slots && !p.units) grid = std::min(grid, p.range_rows);
  const size_t smem = RING_BYTES + (p.slots ? (2 * p.slots + 1) * sizeof(int) : 0);
  static unsigned long long done = 0;
  const cudaError_t e = rr_once_per_device(done, [] {
    const int most = RING_BYTES + (2 * RR_MAX_RANGE_SLOTS + 1) * (int)sizeof(int);
    cudaError_t a = cudaFuncSetAttribute(attend_few_kernel<D, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (a == cudaSuccess) a = cudaFuncSetAttribute(attend_few_kernel<D, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (a == cudaSuccess) a = cudaFuncSetAttribute(attend_few_kernel<D, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return a;
  });
  if (e != cudaSuccess) return e;
  if (rows == 1) return rr_launch_pdl(attend_few_kernel<D, 1>, (int)grid, NT, smem, st, p);
  if (rows == 2) return rr_launch_pdl(attend_few_kernel<D, 2>, (int)grid, NT, smem, st, p);
  return rr_launch_pdl(attend_few_kernel<D, 4>, (int)grid, NT, smem, st, p);
}

}  // namespace

// rows: the most that a segment of the call has (1 to 4).
cudaError_t rr_launch_attend_few(const Params& p, int rows, cudaStream_t st) { return p.dh == 64 ? launch<64>(p, rows, st) : launch<128>(p, rows, st); }
