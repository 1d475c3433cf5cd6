// Split-KV decode for bf16 contexts, head_dim 128, 64-token pages, over two kinds of pages, with or without attention weights: memory-bound.
//
// The first part of an item (item = sequence x KV head) lies in 8-bit pages with a scale each (Q8) or in bf16 pages, its history
// in bf16 pages.  The unit of work is 16 KB of keys and values: one 8-bit page or half a bf16 page (32 tokens), so that units are alike
// in bytes.  As in decode_split.cu the units of all items form one list that is dealt evenly to one CTA per SM, across item
// boundaries, and a second launch merges the items that span CTAs.  Inside a CTA
//   a producer warp : looks up the pages of 32 units at a time, a lane each, and keeps a ring of NSTAGE units full by TMA, two tensor
//                   copies a unit, 128-byte swizzle; a page's scales follow by small copies of their own.
//   a helper warp : rotates the next item's queries and lays them out as mma operands, and merges the last item's parts.
//   NCW warps     : consumers; the unit at ring position n belongs to warp n % NCW (NSTAGE % NCW == 0: see decode_split.cu).
// Tokens are the 16 rows of the mma tiles and the group's query heads their 8 columns, for S = K q^T and for O^T = V^T P^T: no
// row of a tile is idle, half the instructions of tiles that have the heads as rows.  S reaches P's operand layout by movmatrix.
//   8-bit unit: e4m3 becomes f16 exactly, so the operands are f16.  Keys come by 16-byte loads, a lane the bytes 32t .. 32t + 31 of its
//     row: a permutation of the head dimension that the query operand follows.  Values come by the byte form of ldmatrix.trans, four
//     tokens of an element to a register: a permutation of the tokens that the key rows follow.  The rotated query heads
//     are divided by a power of two each, so that their largest element lies in [1, 2), and rounded to f16: exact down to 2^-17; what is below is off by
//     2^-25 at most, half of f16's spacing there.  127 such elements move a score by 2^-18 of the largest |q| times the largest |k|, half of what an fp32
//     sum of 128 products of that size may round off.  A page's scale is applied to its scores and to its P V in fp32.
//   bf16 unit: ldmatrix fragments, bf16 operands.
// P is rounded to f16 or bf16 (11 or 8 significant bits; the sum is of the unrounded values) after a shift of the running maximum by 2^15:
// f16 then holds probabilities down to 2^-29 of the largest without loss.  Scores, sums and O are fp32.
// With weights, the scores of the bf16 rows go to the workspace (4 bytes a row and head), and the second launch turns them into
// probabilities with the item's final maximum and sum.  No atomics: every row belongs to one item.
// Measured: 64 sequences of 8 groups, 4096 8-bit and 1024 bf16 rows each, 124-134 us back to back for 807 MB (6.5 TB/s, the rate of a copy, to 6.0 by how
// the inputs change from pass to pass; 136-151 on its own); 16 ragged ones 36 us
// for 192 MB; one sequence of 720 + 700 rows 8 us.  With weights, 64 sequences of 720 + 2048 bf16 rows, 129 us for 739 MB, ten of them the second launch.
// The tensor pipe is busy for 13-16 %, the issue slots for 22 %: the warps wait for pages.
#include <cuda.h>

#include <type_traits>

#include "common.cuh"

namespace {

constexpr int D = 128;
constexpr int PT = 64;                      // tokens per page
constexpr int HT = 32;                      // tokens of a bf16 unit
constexpr int NCW = 6;                      // consumer warps
constexpr int NSTAGE = 12;
static_assert(NSTAGE % NCW == 0, "a stage must always be consumed by the same warp");
constexpr int THREADS = (NCW + 2) * 32;
constexpr int STAGE_BYTES = 16384;
constexpr int V_OFF = 8192;
constexpr int BOX = HT * 128;               // bf16 unit: [2 halves of the head dimension][32 tokens][64 elements]
constexpr int SM_BAR = NSTAGE * STAGE_BYTES;
constexpr int SM_INFO = SM_BAR + 2 * NSTAGE * 8;          // per stage: key scale, value scale, pool row of the unit's first token
constexpr int SM_MERGE = SM_INFO + NSTAGE * 16;           // NCW x 8 x (2 + 128) floats
constexpr int MROW = 130;
constexpr int SM_Q = SM_MERGE + NCW * 8 * MROW * 4;       // two items' queries as mma operands: bf16, f16, 2^e of the heads, and the items' sizes
constexpr int QBYTES = 2 * 2048 + 64;
constexpr int SM_QBAR = SM_Q + 2 * QBYTES;                // q_full[2], q_empty[2], parts_full, parts_empty
constexpr int SM_MISC = SM_QBAR + 64;                     // abort flag, the CTA's range, scan sums
constexpr int SM_TOTAL = SM_MISC + 128;
constexpr int SM_ALLOC = SM_TOTAL + 1024;
static_assert(SM_ALLOC <= 232448 && SM_MERGE % 16 == 0 && SM_Q % 16 == 0 && QBYTES % 16 == 0, "shared memory");
constexpr uint32_t WAIT_PROBES = 1u << 21;  // ~2.8 s
constexpr uint32_t WHERE_TAG = RC_WHERE_MIXED;
constexpr float SHIFT = 15.f;               // P = 2^(score - running maximum + SHIFT)

struct Share { int T, n_cta, lo, hi, item, start, per_item; };

struct MixParams {
  const __nv_bfloat16* q; const int32_t* q_pos;
  const __nv_bfloat16* k_new; const __nv_bfloat16* v_new;
  const float* k_scale; const float* v_scale; int64_t n_pages8;
  __nv_bfloat16* k_pages; __nv_bfloat16* v_pages; int64_t n_pages;
  const int32_t* res_pt; int max_res_pages; const int32_t* res_len;
  const int32_t* hist_pt; int max_hist_pages; const int32_t* hist_len;
  int n_items, G, Hq, s, per_item;
  bool appended;                            // the last history row is new, whoever wrote it
  void* out; float* part_o; float* part_ml; int2* part_cta;
  float2* item_ml;                          // [item][s] of items that lie in one CTA's range
  float* score;                             // [pool row][s], log2 domain
  const float* weight_in; float* weight_out;
  const float* cos_tab; const float* sin_tab; int max_pos;
  float scale_log2;
  int32_t* status;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  rc_mbar_wait<WAIT_PROBES, WHERE_TAG>(bar, parity, abort_flag, status);
}
// Pages are read once: they are the first to leave L2, so that the scores of the weights are still there when they are read.
__device__ __forceinline__ uint64_t read_once() {
  uint64_t policy;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, uint64_t policy) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4}], [%2], %5;"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "l"(policy) : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, uint64_t policy) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
// the barrier gets one (pre-counted) arrival when all earlier cp.async of this thread have landed
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_tmap(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Two 16 x 16 byte matrices, transposed: register 2m + x of lane (g, t) has rows 4t .. 4t + 3 of column g + 8x of matrix m.
__device__ __forceinline__ void ldsm_b8_t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movm_t(uint32_t a) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// Units of item `it`.  An item without a readable row still counts one, so that its (zero) output is written by somebody.
struct Item { int n_res, n_hist, total, res_len, hist_len; };
template <bool Q8>
__device__ __forceinline__ Item item_units(const MixParams& p, int it) {
  Item u;
  u.res_len = (int)min((int64_t)max(p.res_len[it], 0), (int64_t)p.max_res_pages * PT);
  u.hist_len = (int)min((int64_t)max(p.hist_len[it], 0), (int64_t)p.max_hist_pages * PT);
  u.n_res = Q8 ? (u.res_len + PT - 1) / PT : (u.res_len + HT - 1) / HT;
  u.n_hist = (u.hist_len + HT - 1) / HT;
  u.total = max(u.n_res + u.n_hist, 1);
  return u;
}
// x * j / k for j <= k <= the number of CTAs.  (In 32 bits where they do: a 64-bit division is some hundred instructions, and every warp makes a few
// an item.)
__device__ __forceinline__ int part_of(int x, int j, int k) {
  return x < (1 << 22) ? (int)((uint32_t)x * (uint32_t)j / (uint32_t)k) : (int)((int64_t)x * j / k);
}
// CTA of n whose share of the T units holds unit x
__device__ __forceinline__ int cta_of_unit(int x, int T, int n) {
  return T < (1 << 22) ? (int)((((uint32_t)x + 1u) * (uint32_t)n - 1u) / (uint32_t)T) : (int)((((int64_t)x + 1) * n - 1) / T);
}
// The units [p0, p1) of item `it` (which starts at unit `start` of the list) that are CTA cta's.
__device__ __forceinline__ void own_units(const Share& sh, const Item& u, int cta, int start, int& p0, int& p1) {
  if (sh.per_item > 0) {
    const int k = min(sh.per_item, u.total), j = min(cta % sh.per_item, k);
    p0 = part_of(u.total, j, k); p1 = part_of(u.total, min(j + 1, k), k);
  } else {
    p0 = max(sh.lo - start, 0); p1 = min(sh.hi - start, u.total);
  }
}
// The first and the last CTA that have any of it.
__device__ __forceinline__ int2 span_of(const Share& sh, const Item& u, int cta, int start) {
  if (sh.per_item > 0) {
    const int first = cta - cta % sh.per_item;
    return make_int2(first, first + min(sh.per_item, u.total) - 1);
  }
  return make_int2(cta_of_unit(start, sh.T, sh.n_cta), cta_of_unit(start + u.total - 1, sh.T, sh.n_cta));
}
// Pool row of the first token of unit lp of an item, of the 8-bit pool (8-bit unit) or of the bf16 pool; -1: no such page.
template <bool Q8>
__device__ __forceinline__ int unit_row(const MixParams& p, const Item& u, int it, int lp) {
  const bool res = lp < u.n_res;
  const int x = res ? lp : lp - u.n_res;
  const bool q8 = Q8 && res;
  const int at = q8 ? x : x >> 1;
  const int pg = (res ? p.res_pt + (int64_t)it * p.max_res_pages : p.hist_pt + (int64_t)it * p.max_hist_pages)[at];
  if (pg < 0 || pg >= (q8 ? p.n_pages8 : p.n_pages)) return -1;
  return pg * PT + (q8 ? 0 : (x & 1) * HT);
}
template <bool Q8>
__device__ __forceinline__ int unit_tokens(const Item& u, int lp) {
  if (lp < u.n_res) return Q8 ? min(PT, u.res_len - lp * PT) : min(HT, u.res_len - lp * HT);
  return min(HT, u.hist_len - (lp - u.n_res) * HT);
}

// CTA cta's share of the list (as in decode_split.cu), by a block of THREADS threads; false: it has none.
template <bool Q8>
__device__ __forceinline__ bool share_of(const MixParams& p, int cta, int n_ctas, volatile int* sums, volatile int* range, Share& sh) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  sh.T = 0; sh.n_cta = n_ctas; sh.lo = 0; sh.hi = 1; sh.start = 0; sh.item = 0; sh.per_item = p.per_item;
  if (p.per_item == 0) {
    const int per = (p.n_items + THREADS - 1) / THREADS;
    const int i0 = min(p.n_items, (int)threadIdx.x * per), i1 = min(p.n_items, i0 + per);
    int sum = 0, most = 0;
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
      const int n = item_units<Q8>(p, i).total;
      sum += n;
      most = max(most, n);
    }
    int incl = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += v;
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) { sums[2 * warp] = incl; sums[2 * warp + 1] = most; }
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) before += sums[2 * w];
      sh.T += sums[2 * w];
      most = max(most, sums[2 * w + 1]);
    }
    sh.n_cta = min(n_ctas, sh.T);
    const int k = n_ctas / p.n_items;
    if (k >= 2 && most / k <= sh.T / sh.n_cta + 6) {
      sh.per_item = k;
    } else {
      if (cta >= sh.n_cta) return false;
      sh.lo = part_of(sh.T, cta, sh.n_cta); sh.hi = part_of(sh.T, cta + 1, sh.n_cta);
      before += incl - sum;
      if (sh.lo >= before && sh.lo < before + sum) {
        int i = i0, acc = before;
        for (;; ++i) {
          const int m = item_units<Q8>(p, i).total;
          if (sh.lo < acc + m) break;
          acc += m;
        }
        range[0] = i; range[1] = acc;
      }
      __syncthreads();
      sh.item = range[0]; sh.start = range[1];
    }
  }
  if (sh.per_item > 0) sh.item = min(cta / sh.per_item, p.n_items);
  return sh.item < p.n_items;
}

template <typename TO, bool Q8, bool WEIGHTS>
__global__ void __launch_bounds__(THREADS, 1) mixed_split_kernel(const __grid_constant__ CUtensorMap tm_k8, const __grid_constant__ CUtensorMap tm_v8,
                                                                 const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                                                                 const __grid_constant__ MixParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sm = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* sm_gen = smem_raw + (sm - smem_u32(smem_raw));
  const uint32_t bars = sm + SM_BAR;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm_gen + SM_MISC);
  volatile int* range_sm = reinterpret_cast<volatile int*>(sm_gen + SM_MISC + 8);
  volatile int* sums_sm = reinterpret_cast<volatile int*>(sm_gen + SM_MISC + 32);
  auto full = [&](int i) { return bars + 8u * (uint32_t)i; };
  auto empty = [&](int i) { return bars + 8u * (uint32_t)(NSTAGE + i); };
  const uint32_t qbars = sm + SM_QBAR, parts_full = qbars + 32, parts_empty = qbars + 40;
  auto q_full = [&](int i) { return qbars + 8u * (uint32_t)i; };
  auto q_empty = [&](int i) { return qbars + 16u + 8u * (uint32_t)i; };
  float* mrg = reinterpret_cast<float*>(sm_gen + SM_MERGE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < NSTAGE; ++i) { mbar_init(full(i), Q8 ? 2 : 1); mbar_init(empty(i), 1); }   // (Q8: the loads, and the scales)
    for (int i = 0; i < 2; ++i) { mbar_init(q_full(i), 1); mbar_init(q_empty(i), NCW); }
    mbar_init(parts_full, NCW); mbar_init(parts_empty, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == NCW && lane == 0) {
    prefetch_tmap(&tm_k); prefetch_tmap(&tm_v);
    if (Q8) { prefetch_tmap(&tm_k8); prefetch_tmap(&tm_v8); }
  }
  __syncthreads();
  rc_grid_wait();
  rc_grid_launch_next();

  Share sh;
  if (!share_of<Q8>(p, blockIdx.x, gridDim.x, sums_sm, range_sm, sh)) return;

  // One head of an item from the consumer warps' parts: the result, or the CTA's part of it (slot).
  auto merge_head = [&](int it, int slot, bool whole, int h) {
    const int s = p.s, b = it / p.G, g = it % p.G;
    float mw[NCW], M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NCW; ++w) { mw[w] = mrg[(w * 8 + h) * MROW]; M = fmaxf(M, mw[w]); }
    float L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NCW; ++w) {
      const float f = mw[w] == -INFINITY ? 0.f : ex2(mw[w] - M);
      L += mrg[(w * 8 + h) * MROW + 1] * f;
      const float* ow = mrg + (w * 8 + h) * MROW + 2 + lane * 4;
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] += ow[c] * f;
    }
    if (whole) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      TO* orow = reinterpret_cast<TO*>(p.out) + ((int64_t)b * p.Hq + g * s + h) * D + lane * 4;
      if constexpr (sizeof(TO) == 4) *reinterpret_cast<float4*>(orow) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
      else *reinterpret_cast<uint2*>(orow) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
      if (WEIGHTS && lane == 0) p.item_ml[(int64_t)it * s + h] = make_float2(M, L);
    } else {
      const int row = slot * s + h;
      *reinterpret_cast<float4*>(p.part_o + (int64_t)row * D + lane * 4) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      if (lane == 0) *reinterpret_cast<float2*>(p.part_ml + row * 2) = make_float2(M, L);
    }
  };

  if (warp == NCW) {
    // ===================== producer =====================
    uint32_t n = 0;
    const uint64_t policy = read_once();
    for (int it = sh.item, start = sh.start; start < sh.hi; ++it) {
      const Item u = item_units<Q8>(p, it);
      int p0, p1;
      own_units(sh, u, blockIdx.x, start, p0, p1);
      start += u.total;
      const int real = min(p1, u.n_res + u.n_hist);          // (an item of no rows has a unit of its own, without a page)
      for (int c0 = p0; c0 < p1; c0 += 32) {
        const int lp = c0 + lane;
        int row = -1;
        if (lp < real) {
          row = unit_row<Q8>(p, u, it, lp);
          if (row < 0) rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
        }
        const int cnt = min(32, p1 - c0);
        for (int l = 0; l < cnt; ++l, ++n) {
          const int st = n % NSTAGE;
          const int r = __shfl_sync(0xffffffffu, row, l);
          if (lane == 0) {
            const uint32_t dst = sm + st * STAGE_BYTES, info = sm + SM_INFO + st * 16;
            mbar_wait(empty(st), ((n / NSTAGE) & 1u) ^ 1u, abort_flag, p.status);
            *reinterpret_cast<volatile int*>(sm_gen + SM_INFO + st * 16 + 8) = r;
            if (r >= 0) {
              mbar_expect_tx(full(st), STAGE_BYTES);
              if (Q8 && c0 + l < u.n_res) {
                tma_2d(dst, &tm_k8, full(st), 0, r, policy);
                tma_2d(dst + V_OFF, &tm_v8, full(st), 0, r, policy);
                cp_async4(info, p.k_scale + r / PT);          // (nobody waits for them here: a first unit's copies would wait with them)
                cp_async4(info + 4, p.v_scale + r / PT);
                cp_async_arrive(full(st));
              } else {
                tma_3d(dst, &tm_k, full(st), 0, r, 0, policy);
                tma_3d(dst + V_OFF, &tm_v, full(st), 0, r, 0, policy);
                if (Q8) mbar_arrive(full(st));
              }
            } else {
              mbar_arrive(full(st));                          // nothing to load: the consumer skips the unit
              if (Q8) mbar_arrive(full(st));
            }
          }
          __syncwarp();
        }
      }
    }
  } else if (warp == NCW + 1) {
    // ===================== helper: queries of the next item, merge of the last =====================
    // (Looking up an item's position, rotating its queries and merging its parts in the consumers kept them from their units for some five
    // microseconds an item, longer than the ring lasts.)
    const int s = p.s;
    struct Ahead { int it, start; };                          // next item to prepare
    Ahead a = {sh.item, sh.start};
    struct Done { int it, slot, whole; };                     // an item that was prepared: where its result goes
    int n_prep = 0, n_fin = 0;
    // the queries of the CTA's next item with units, as operands; false: there is none
    auto prepare = [&](Done& d) -> bool {
      for (; a.start < sh.hi;) {
        const int it = a.it++, b = it / p.G, g = it % p.G, start = a.start;
        const int pos_q = p.q_pos[b];
        const __nv_bfloat16* qg = p.q + ((int64_t)b * p.Hq + g * s) * D;
        uint32_t wl[8], wh[8];
#pragma unroll
        for (int h = 0; h < 8; ++h) {
          wl[h] = wh[h] = 0;
          if (h < s) {
            wl[h] = *reinterpret_cast<const uint32_t*>(qg + h * D + 2 * lane);
            wh[h] = *reinterpret_cast<const uint32_t*>(qg + h * D + 64 + 2 * lane);
          }
        }
        const Item u = item_units<Q8>(p, it);
        int p0, p1;
        own_units(sh, u, blockIdx.x, start, p0, p1);
        a.start += u.total;
        if (p0 >= p1) continue;
        const bool pos_ok = pos_q >= 0 && pos_q < p.max_pos;
        if (p0 == 0 && lane == 0) {
          p.part_cta[it] = span_of(sh, u, blockIdx.x, start);
          if (p.hist_len[it] < 1 || p.hist_len[it] != u.hist_len || max(p.res_len[it], 0) != u.res_len) rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
          if (!pos_ok) rc_set_status(p.status, RECACHE_DEV_BAD_POS);
        }
        const int64_t tab = (int64_t)(pos_ok ? pos_q : 0) * 64;
        const float2 c = *reinterpret_cast<const float2*>(p.cos_tab + tab + 2 * lane);
        const float2 sn = *reinterpret_cast<const float2*>(p.sin_tab + tab + 2 * lane);
        mbar_wait(q_empty(n_prep & 1), ((n_prep >> 1) & 1u) ^ 1u, abort_flag, p.status);
        uint8_t* to = sm_gen + SM_Q + (n_prep & 1) * QBYTES;
        // operand register r of lane (head, t) lies at uint4 [r / 4][lane], component r % 4; word w of a head holds elements 2w, 2w + 1
        auto put = [&](int at, int h, int t, int r, uint32_t v) {
          *reinterpret_cast<uint32_t*>(to + at + ((r >> 2) * 32 + h * 4 + t) * 16 + (r & 3) * 4) = v;
        };
#pragma unroll
        for (int h = 0; h < 8; ++h) {
          const float l0 = __uint_as_float(wl[h] << 16), l1 = __uint_as_float(wl[h] & 0xffff0000u);
          const float h0 = __uint_as_float(wh[h] << 16), h1 = __uint_as_float(wh[h] & 0xffff0000u);
          const uint32_t lo = pack_bf16(__fmaf_rn(l0, c.x, -__fmul_rn(h0, sn.x)), __fmaf_rn(l1, c.y, -__fmul_rn(h1, sn.y)));
          const uint32_t hi = pack_bf16(__fmaf_rn(h0, c.x, __fmul_rn(l0, sn.x)), __fmaf_rn(h1, c.y, __fmul_rn(l1, sn.y)));
          // bf16, head dimension in order: elements 16kk + 8x + 2t, + 1 in register 2kk + x
          put(0, h, lane & 3, lane >> 2, lo);
          put(0, h, lane & 3, 8 + (lane >> 2), hi);
          if constexpr (Q8) {
            // f16, divided by 2^e: elements 32t + 4kk + 2x, + 1 in register 2kk + x
            const uint32_t top = __reduce_max_sync(0xffffffffu, max(max(lo & 0x7fffu, (lo >> 16) & 0x7fffu), max(hi & 0x7fffu, (hi >> 16) & 0x7fffu)));
            int e = (int)(top >> 7);                          // biased exponent of the head's largest element
            if (e == 0 || e == 255) e = 127;
            // 2^(127 - e) in two factors: it is no normal number where the head's largest element is (nearly) the greatest or least there is
            const int half = (127 - e) / 2;
            const float d0 = __uint_as_float((uint32_t)(127 + half) << 23), d1 = __uint_as_float((uint32_t)(254 - e - half) << 23);
            put(2048, h, lane >> 4, lane & 15, pack_f16(__uint_as_float(lo << 16) * d0 * d1, __uint_as_float(lo & 0xffff0000u) * d0 * d1));
            put(2048, h, 2 + (lane >> 4), lane & 15, pack_f16(__uint_as_float(hi << 16) * d0 * d1, __uint_as_float(hi & 0xffff0000u) * d0 * d1));
            if (lane == 0) *reinterpret_cast<float*>(to + 4096 + 4 * h) = __uint_as_float((uint32_t)e << 23);
          }
        }
        if (lane == 0) {
          *reinterpret_cast<int4*>(to + 4128) = make_int4(p0, p1, it, u.n_res);
          *reinterpret_cast<int4*>(to + 4144) = make_int4(u.res_len, u.hist_len, (pos_ok && p.hist_len[it] == u.hist_len ? 1 : 0) | (p0 == 0 && p1 == u.total ? 2 : 0), pos_ok ? pos_q : 0);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full(n_prep & 1));
        ++n_prep;
        d.it = it; d.whole = p0 == 0 && p1 == u.total; d.slot = 2 * (int)blockIdx.x + (p0 == 0 ? 1 : 0);
        return true;
      }
      mbar_wait(q_empty(n_prep & 1), ((n_prep >> 1) & 1u) ^ 1u, abort_flag, p.status);
      if (lane == 0) {                                        // an item of no units: there are no more
        *reinterpret_cast<int4*>(sm_gen + SM_Q + (n_prep & 1) * QBYTES + 4128) = make_int4(0, -1, 0, 0);
        mbar_arrive(q_full(n_prep & 1));
      }
      return false;
    };
    auto finish = [&](const Done& d) {
      mbar_wait(parts_full, n_fin & 1u, abort_flag, p.status);
      ++n_fin;
      for (int h = 0; h < s; ++h) merge_head(d.it, d.slot, d.whole, h);
      __syncwarp();
      if (lane == 0) mbar_arrive(parts_empty);
    };
    Done cur, next;
    bool have = prepare(cur);
    while (have) {
      const bool more = prepare(next);
      if (more) finish(cur);                                  // (the last one the consumers merge, a warp to a head: nothing comes after it)
      cur = next;
      have = more;
    }
  } else {
    // ===================== consumers =====================
    const int gq = lane >> 2, tq = lane & 3;                  // fragment row and column pair
    const int s = p.s;
    uint32_t n_base = 0;
    int n_item = 0, last_it = -1, last_slot = 0;
    bool last_whole = false;
    for (;;) {
      mbar_wait(q_full(n_item & 1), (n_item >> 1) & 1u, abort_flag, p.status);
      const uint8_t* q_item = sm_gen + SM_Q + (n_item & 1) * QBYTES;
      const int4 meta = *reinterpret_cast<const int4*>(q_item + 4128), meta2 = *reinterpret_cast<const int4*>(q_item + 4144);
      const int p0 = meta.x, p1 = meta.y, it = meta.z;
      if (p1 < 0 || *abort_flag) break;                        // (abort: a wait ran out)
      last_it = it; last_slot = 2 * (int)blockIdx.x + (p0 == 0 ? 1 : 0); last_whole = (meta2.z & 2) != 0;
      const Item u = {meta.w, 0, 0, meta2.x, meta2.y};
      const bool may_append = p.k_new && (meta2.z & 1);
      const int64_t tab = (int64_t)meta2.w * 64;
      uint32_t qb[8][2];                                      // bf16, head dimension in order
      uint32_t qf[8][2];                                      // f16, elements 32t + 4kk .. + 3 of the head, divided by 2^e
      float up[2] = {1.f, 1.f};                               // 2^e of heads 2t and 2t + 1
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 v = *reinterpret_cast<const uint4*>(q_item + (i * 32 + lane) * 16);
        qb[2 * i][0] = v.x; qb[2 * i][1] = v.y; qb[2 * i + 1][0] = v.z; qb[2 * i + 1][1] = v.w;
      }
      if constexpr (Q8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 v = *reinterpret_cast<const uint4*>(q_item + 2048 + (i * 32 + lane) * 16);
          qf[2 * i][0] = v.x; qf[2 * i][1] = v.y; qf[2 * i + 1][0] = v.z; qf[2 * i + 1][1] = v.w;
        }
        const float2 e = *reinterpret_cast<const float2*>(q_item + 4096 + 8 * tq);
        up[0] = e.x; up[1] = e.y;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty(n_item & 1));

      float o[8][4];                                          // element 16j + g (+ 8 in the upper pair) of heads 2t, 2t + 1
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};   // maximum of heads 2t, 2t + 1; this lane's share of their sums

      // One unit's softmax: scores (rows: tokens) to P as the operand of P V, the rescale factors, scores to the workspace.
      auto softmax = [&](auto tiles, auto q8, float (*sc)[4], const float* f, int valid, int row, uint32_t (*pb)[2], float* corr) {
        constexpr int MT = decltype(tiles)::value;
        constexpr bool U8 = decltype(q8)::value;
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {                       // rows g and g + 8
            const int tok = mt * 16 + (U8 ? 4 * (gq >> 1) + (gq & 1) + 2 * x : gq + 8 * x);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float& v = sc[mt][2 * x + h];
              v = tok < valid ? v * f[h] : -INFINITY;
              mx[h] = fmaxf(mx[h], v);
            }
            if constexpr (WEIGHTS && !U8) {
              if (tok < valid) {
                float* to = p.score + (int64_t)(row + tok) * s + 2 * tq;
                if (2 * tq < s) to[0] = sc[mt][2 * x];
                if (2 * tq + 1 < s) to[1] = sc[mt][2 * x + 1];
              }
            }
          }
        }
        float use[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], off));
          const float m_new = fmaxf(m_run[h], mx[h]);
          const float base = m_new == -INFINITY ? 0.f : m_new;
          corr[h] = ex2(m_run[h] - base);
          use[h] = base - SHIFT;
          m_run[h] = m_new;
          l_run[h] *= corr[h];
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float e0 = ex2(sc[mt][2 * x] - use[0]), e1 = ex2(sc[mt][2 * x + 1] - use[1]);
            l_run[0] += e0; l_run[1] += e1;
            pb[mt][x] = movm_t(U8 ? pack_f16(e0, e1) : pack_bf16(e0, e1));
          }
        }
      };

      const int first = (int)(((uint32_t)warp + NCW - n_base % NCW) % NCW);
      for (int lp = p0 + first; lp < p1; lp += NCW) {
        const uint32_t n = n_base + (uint32_t)(lp - p0);
        const int st = n % NSTAGE;
        mbar_wait(full(st), (n / NSTAGE) & 1u, abort_flag, p.status);
        const float4 info = *reinterpret_cast<const float4*>(sm_gen + SM_INFO + st * 16);
        const int row = __float_as_int(info.z);
        const uint32_t kb = sm + st * STAGE_BYTES, vb = kb + V_OFF;
        const int valid = unit_tokens<Q8>(u, lp);
        if (row >= 0) {
          if (Q8 && lp < u.n_res) {
            // ---- 64 tokens of 8 bits ----
            if (valid < PT) {                                 // slots behind the part: clear their values (0 * NaN would poison O)
              for (int e = lane; e < (PT - valid) * 8; e += 32)
                *reinterpret_cast<uint4*>(sm_gen + st * STAGE_BYTES + V_OFF + (valid + (e >> 3)) * 128 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // a later TMA load overwrites these bytes
              __syncwarp();
            }
            float sc[4][4];
            const int ra = 4 * (gq >> 1) + (gq & 1);          // token of tile row g; + 2: of row g + 8
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
              sc[mt][0] = sc[mt][1] = sc[mt][2] = sc[mt][3] = 0.f;
              const int t0 = mt * 16 + ra, t1 = t0 + 2;
              const uint32_t a0 = kb + t0 * 128, a1 = kb + t1 * 128;
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                const uint4 x = lds128(a0 + (((2 * tq + hf) ^ (t0 & 7)) << 4)), y = lds128(a1 + (((2 * tq + hf) ^ (t1 & 7)) << 4));
                const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  mma_f16(sc[mt], rc_e4m3x2_to_f16x2(xw[i]), rc_e4m3x2_to_f16x2(yw[i]), rc_e4m3x2_to_f16x2(xw[i] >> 16), rc_e4m3x2_to_f16x2(yw[i] >> 16),
                          qf[4 * hf + i][0], qf[4 * hf + i][1]);
              }
            }
            const float f[2] = {info.x * (up[0] * p.scale_log2), info.x * (up[1] * p.scale_log2)};
            uint32_t pb[4][2];
            float corr[2];
            softmax(std::integral_constant<int, 4>(), std::true_type(), sc, f, valid, row, pb, corr);
            float acc[8][4];
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
              const int tok = kt * 16 + (lane & 15);
              const uint32_t rowa = vb + tok * 128;
#pragma unroll
              for (int jj = 0; jj < 4; ++jj) {                // two 16-element chunks of the head dimension
                uint32_t r[4];
                ldsm_b8_t(rowa + (((2 * jj + (lane >> 4)) ^ (tok & 7)) << 4), r);
#pragma unroll
                for (int x = 0; x < 2; ++x)
                  mma_f16(acc[2 * jj + x], rc_e4m3x2_to_f16x2(r[2 * x]), rc_e4m3x2_to_f16x2(r[2 * x + 1]), rc_e4m3x2_to_f16x2(r[2 * x] >> 16),
                          rc_e4m3x2_to_f16x2(r[2 * x + 1] >> 16), pb[kt][0], pb[kt][1]);
              }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[j][i] = fmaf(info.y, acc[j][i], o[j][i] * corr[i & 1]);
          } else {
            // ---- 32 tokens of bf16 ----
            const int hn = u.hist_len - 1;                    // the current token's history row
            const bool appends = may_append && hn >= 0 && lp >= u.n_res && hn / HT == lp - u.n_res;
            if (valid < HT) {
              for (int e = lane; e < (HT - valid) * 16; e += 32)
                *reinterpret_cast<uint4*>(sm_gen + st * STAGE_BYTES + V_OFF + ((e >> 3) & 1) * BOX + (valid + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            if (appends) {
              const int r = hn % HT;
              const __nv_bfloat16* ks = p.k_new + (int64_t)it * D;
              const __nv_bfloat16* vs = p.v_new + (int64_t)it * D;
              uint8_t* kg = sm_gen + st * STAGE_BYTES + r * 128;
              const int64_t to = (int64_t)(row + r) * D;
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const int i = lane + 32 * x;
                const float l = __bfloat162float(ks[i]), h = __bfloat162float(ks[i + 64]);
                const float c = p.cos_tab[tab + i], sn = p.sin_tab[tab + i];
                const __nv_bfloat16 kl = __float2bfloat16_rn(__fmaf_rn(l, c, -__fmul_rn(h, sn)));
                const __nv_bfloat16 kh = __float2bfloat16_rn(__fmaf_rn(h, c, __fmul_rn(l, sn)));
                const __nv_bfloat16 vl = vs[i], vh = vs[i + 64];
                uint8_t* e = kg + (((i >> 3) ^ (r & 7)) << 4) + (i & 7) * 2;
                *reinterpret_cast<__nv_bfloat16*>(e) = kl;
                *reinterpret_cast<__nv_bfloat16*>(e + BOX) = kh;
                *reinterpret_cast<__nv_bfloat16*>(e + V_OFF) = vl;
                *reinterpret_cast<__nv_bfloat16*>(e + V_OFF + BOX) = vh;
                p.k_pages[to + i] = kl; p.k_pages[to + i + 64] = kh;
                p.v_pages[to + i] = vl; p.v_pages[to + i + 64] = vh;
              }
            }
            if (valid < HT || appends) {
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
            }
            float sc[2][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              sc[mt][0] = sc[mt][1] = sc[mt][2] = sc[mt][3] = 0.f;
              const int tok = mt * 16 + (lane & 15);
#pragma unroll
              for (int kk = 0; kk < 8; ++kk) {
                const int c = 2 * kk + (lane >> 4);
                uint32_t a[4];
                ldsm_x4(kb + (c >> 3) * BOX + tok * 128 + (((c & 7) ^ (tok & 7)) << 4), a);
                mma_bf16(sc[mt], a[0], a[1], a[2], a[3], qb[kk][0], qb[kk][1]);
              }
            }
            const float f[2] = {p.scale_log2, p.scale_log2};
            uint32_t pb[2][2];
            float corr[2];
            softmax(std::integral_constant<int, 2>(), std::false_type(), sc, f, valid, row, pb, corr);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[j][i] *= corr[i & 1];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
              const int tok = kt * 16 + (lane >> 4) * 8 + (lane & 7);        // matrices: (tokens 0-7, elements 0-7), (0-7, 8-15), (8-15, 0-7), (8-15, 8-15)
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const int c = 2 * j + ((lane >> 3) & 1);
                uint32_t a[4];
                ldsm_x4_t(vb + (c >> 3) * BOX + tok * 128 + (((c & 7) ^ (tok & 7)) << 4), a);
                mma_bf16(o[j], a[0], a[1], a[2], a[3], pb[kt][0], pb[kt][1]);
              }
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }
      n_base += (uint32_t)(p1 - p0);

      // ---- this warp's part goes to the helper ----
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], off);
      mbar_wait(parts_empty, (n_item & 1u) ^ 1u, abort_flag, p.status);
      ++n_item;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int head = 2 * tq + h;
        if (head < s) {
          float* mine = mrg + (warp * 8 + head) * MROW;
          if (gq == 0) { mine[0] = m_run[h]; mine[1] = l_run[h]; }
#pragma unroll
          for (int j = 0; j < 8; ++j) { mine[2 + 16 * j + gq] = o[j][h]; mine[2 + 16 * j + 8 + gq] = o[j][2 + h]; }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(parts_full);
    }
    if (last_it >= 0) {
      mbar_wait(parts_full, (n_item - 1) & 1u, abort_flag, p.status);
      for (int h = warp; h < s; h += NCW) merge_head(last_it, last_slot, last_whole, h);
    }
  }
  if (*abort_flag) rc_timeout_drain();
}

// Maximum and sum (SHIFT included) of the heads of an item, by a warp: lane 4h + x has head h's.  The item lies in one CTA's range, or spans
// CTAs ab.x .. ab.y, whose parts the four lanes of a head take in turn.  (Written for size: the kernel's warps run at different places, and
// with the merge inlined for each head they waited for instructions more than for anything else.)
__device__ __forceinline__ float2 item_max_sum(const MixParams& p, int it, int2 ab, int lane) {
  const int h = lane >> 2;
  if (ab.x == ab.y) return h < p.s ? p.item_ml[(int64_t)it * p.s + h] : make_float2(-INFINITY, 0.f);
  float M = -INFINITY, L = 0.f;
  if (h < p.s) {
    for (int c0 = ab.x + (lane & 3); c0 <= ab.y; c0 += 20) {   // five parts of the lane's at once
      float2 ml[5];
      float top = M;
#pragma unroll
      for (int x = 0; x < 5; ++x) {
        const int c = c0 + 4 * x;
        ml[x] = make_float2(-INFINITY, 0.f);
        if (c <= ab.y) ml[x] = *reinterpret_cast<const float2*>(p.part_ml + ((c == ab.x ? 2 * c + 1 : 2 * c) * p.s + h) * 2);
      }
#pragma unroll
      for (int x = 0; x < 5; ++x) top = fmaxf(top, ml[x].x);
      const float use = top == -INFINITY ? 0.f : top;
      L *= ex2(M - use);
#pragma unroll
      for (int x = 0; x < 5; ++x) L += ml[x].y * ex2(ml[x].x - use);
      M = top;
    }
  }
  __syncwarp();
#pragma unroll
  for (int off = 1; off < 4; off <<= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, M, off), l2 = __shfl_xor_sync(0xffffffffu, L, off);
    const float m_new = fmaxf(M, m2), use = m_new == -INFINITY ? 0.f : m_new;
    const float a = L * ex2(M - use), b = l2 * ex2(m2 - use);
    L = lane & off ? b + a : a + b;                            // (the same order in both lanes)
    M = m_new;
  }
  return make_float2(M, L);
}

// Second launch.  With weights, block WSUB c + j takes units of CTA c's share, each of its warps a run of them, a lane a token; what it needs
// of lengths, tables and prior weights it reads while the attention's last CTAs run.  The last n_merge blocks combine
// the parts of the items that span CTAs, four warps an output row.
// HS: heads that a lane holds scores of, at least s.  (Three blocks a CTA fit its SM at once beside a merge block; with two or four, 64 sequences
// 131-132 us instead of 129.  One unit on its way a warp: with four, the registers ran out and one sequence took 9.9 us instead of 8.6.)
constexpr int MERGE_WARPS = 8, WSUB = 3, ROW_WARPS = 4;
static_assert(32 * MERGE_WARPS == THREADS, "share_of's block");
template <typename TO, bool Q8, bool WEIGHTS, int HS>
__global__ void __launch_bounds__(32 * MERGE_WARPS, 4) mixed_merge_kernel(const __grid_constant__ MixParams p, int n_rows, int n_merge) {
  // What the attention does not write (lengths, tables, prior weights) may be read before it ends: all its blocks have seen the end of
  // the kernels before it by the time this one comes up.
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = p.s;
  const int n_weigh = gridDim.x - n_merge;
  if ((int)blockIdx.x >= n_weigh) {
    __shared__ float4 part_o[MERGE_WARPS][32];
    __shared__ float2 part_ml[MERGE_WARPS];
    const int row = ((int)blockIdx.x - n_weigh) * (MERGE_WARPS / ROW_WARPS) + warp / ROW_WARPS, sub = warp % ROW_WARPS;
    const int head = row % p.Hq, it = row / p.Hq * p.G + head / s, h = head % s;
    int2 ab = make_int2(0, 0);
    if (p.per_item > 0 && row < n_rows) {                     // one sequence: its parts follow from the lengths
      ab.x = it * p.per_item;
      ab.y = ab.x + min(p.per_item, item_units<Q8>(p, it).total) - 1;
    }
    rc_grid_wait();
    rc_grid_launch_next();
    if (p.per_item == 0 && row < n_rows) ab = p.part_cta[it];
    float M = -INFINITY, L = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int PARTS = 5;                                  // (one sequence of eight groups has 18 parts an item: one round)
    if (ab.x < ab.y) {
      for (int c0 = ab.x + sub; c0 <= ab.y; c0 += PARTS * ROW_WARPS) {
        float2 ml[PARTS];
        float4 v[PARTS];
        float top = M;
#pragma unroll
        for (int x = 0; x < PARTS; ++x) {
          const int c = c0 + x * ROW_WARPS, slot = (c == ab.x ? 2 * c + 1 : 2 * c) * s + h;
          ml[x] = make_float2(-INFINITY, 0.f);
          v[x] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (c <= ab.y) {
            ml[x] = *reinterpret_cast<const float2*>(p.part_ml + slot * 2);
            v[x] = *reinterpret_cast<const float4*>(p.part_o + (int64_t)slot * D + lane * 4);
          }
        }
#pragma unroll
        for (int x = 0; x < PARTS; ++x) top = fmaxf(top, ml[x].x);
        const float use = top == -INFINITY ? 0.f : top, corr = ex2(M - use);
        M = top;
        L *= corr;
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] *= corr;
#pragma unroll
        for (int x = 0; x < PARTS; ++x) {
          const float f = ex2(ml[x].x - use);
          L += ml[x].y * f;
          acc[0] += v[x].x * f; acc[1] += v[x].y * f; acc[2] += v[x].z * f; acc[3] += v[x].w * f;
        }
      }
    }
    part_o[warp][lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (lane == 0) part_ml[warp] = make_float2(M, L);
    __syncthreads();
    if (sub != 0 || row >= n_rows || ab.x >= ab.y) return;
#pragma unroll
    for (int x = 1; x < ROW_WARPS; ++x) M = fmaxf(M, part_ml[warp + x].x);
    const float use = M == -INFINITY ? 0.f : M;
    L = 0.f;
    acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
#pragma unroll
    for (int x = 0; x < ROW_WARPS; ++x) {
      const float f = ex2(part_ml[warp + x].x - use);
      const float4 v = part_o[warp + x][lane];
      L += part_ml[warp + x].y * f;
      acc[0] += v.x * f; acc[1] += v.y * f; acc[2] += v.z * f; acc[3] += v.w * f;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    TO* orow = reinterpret_cast<TO*>(p.out) + (int64_t)row * D + lane * 4;
    if constexpr (sizeof(TO) == 4) *reinterpret_cast<float4*>(orow) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    else *reinterpret_cast<uint2*>(orow) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
    return;
  }
  if constexpr (WEIGHTS) {
    const int cta = blockIdx.x / WSUB, mine = blockIdx.x % WSUB * MERGE_WARPS + warp;
    __shared__ int sums[2 * MERGE_WARPS], range[2];
    bool waits = true;                                        // for the attention's scores; once, on every path out of here too
    auto wait_once = [&] {
      if (waits) { rc_grid_wait(); rc_grid_launch_next(); }
      waits = false;
    };
    Share sh;
    if (!share_of<Q8>(p, cta, n_weigh / WSUB, sums, range, sh)) { wait_once(); return; }
    constexpr int STEP = WSUB * MERGE_WARPS;
    // Each warp takes an equal run of the share's units (of few items then), 32 at a time, a lane a unit: which item it belongs to, by the units
    // of the share's items, 32 of them a lane each; then its pool row.  So a share of any number of items is three loads deep.
    int n_share = sh.hi - sh.lo;
    if (sh.per_item > 0) {
      int p0, p1;
      own_units(sh, item_units<Q8>(p, sh.item), cta, 0, p0, p1);
      n_share = p1 - p0;
    }
    const int u_end = part_of(n_share, mine + 1, STEP);
    for (int u0 = part_of(n_share, mine, STEP); u0 < u_end; u0 += 32) {
      const int want = u0 + lane < u_end ? u0 + lane : n_share;           // index in the share
      int row = -1, tokens = 0, slot = -1, item = -1, begin = 0;   // begin: the item's first unit in the list
      int before = 0;                                         // units of the share's items so far
      if (sh.per_item > 0) {
        const Item u = item_units<Q8>(p, sh.item);
        int p0, p1;
        own_units(sh, u, cta, 0, p0, p1);
        before = p1 - p0;
        if (want < before) { item = sh.item; slot = p0 + want; }
      } else {
        for (int i0 = sh.item, start = sh.start; start < sh.hi && i0 < p.n_items; i0 += 32) {
          const bool there = i0 + lane < p.n_items;
          Item u = {0, 0, 0, 0, 0};
          if (there) u = item_units<Q8>(p, i0 + lane);
          int incl = u.total;
#pragma unroll
          for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
          }
          int p0, p1;
          own_units(sh, u, cta, start + incl - u.total, p0, p1);
          const int own = there ? max(p1 - p0, 0) : 0;
          int upto = own;
#pragma unroll
          for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += v;
          }
          for (uint32_t m = __ballot_sync(0xffffffffu, own > 0); m; m &= m - 1) {
            const int l = __ffs(m) - 1;
            const int hi = before + __shfl_sync(0xffffffffu, upto, l), lo = hi - __shfl_sync(0xffffffffu, own, l);
            const int lp = __shfl_sync(0xffffffffu, p0, l) + want - lo;
            const int first = __shfl_sync(0xffffffffu, start + incl - u.total, l);
            if (want >= lo && want < hi) { item = i0 + l; slot = lp; begin = first; }
          }
          before += __shfl_sync(0xffffffffu, upto, 31);
          start += __shfl_sync(0xffffffffu, incl, 31);
        }
      }
      int info = 0;                                           // 1 + the unit's token that is new
      int2 ab = make_int2(0, 0);
      if (item >= 0) {
        const Item u = item_units<Q8>(p, item);
        if (slot < u.n_res + u.n_hist && !(Q8 && slot < u.n_res)) {       // 8-bit rows have no weight
          row = unit_row<Q8>(p, u, item, slot);
          tokens = unit_tokens<Q8>(u, slot);
        }
        ab = span_of(sh, u, cta, begin);
        const int pos = p.q_pos[item / p.G], last_tok = u.hist_len - 1 - (slot - u.n_res) * HT;
        if (p.appended && pos >= 0 && pos < p.max_pos && p.hist_len[item] == u.hist_len && slot >= u.n_res && last_tok < HT) info = last_tok + 1;
      }
      const int cnt = min(32, u_end - u0);
      int at_item = -1;
      float M[HS], inv[HS];
      for (int j = 0; j < cnt; ++j) {                         // a unit, a lane a token
        const int it = __shfl_sync(0xffffffffu, item, j), r = __shfl_sync(0xffffffffu, row, j), n = __shfl_sync(0xffffffffu, tokens, j);
        const int fresh = __shfl_sync(0xffffffffu, info, j) - 1;
        const int2 span = make_int2(__shfl_sync(0xffffffffu, ab.x, j), __shfl_sync(0xffffffffu, ab.y, j));
        if (r < 0) continue;
        float w = 0.f, sc[HS];
        if (p.weight_in && lane < n && lane != fresh) w = p.weight_in[(int64_t)r + lane];   // (a token that was just appended has none yet)
        wait_once();
        if (lane < n) {
          const float* from = p.score + ((int64_t)r + lane) * s;
          if ((s & 3) == 0) {
#pragma unroll
            for (int h = 0; h < HS; h += 4)
              if (h < s) *reinterpret_cast<float4*>(&sc[h]) = *reinterpret_cast<const float4*>(from + h);
          } else {
#pragma unroll
            for (int h = 0; h < HS; ++h)
              if (h < s) sc[h] = from[h];
          }
        }
        if (it != at_item) {
          at_item = it;
          const float2 ml = item_max_sum(p, it, span, lane);
          const float base = (ml.x == -INFINITY ? 0.f : ml.x) - SHIFT, over = ml.y == 0.f ? 0.f : 1.f / ml.y;
#pragma unroll
          for (int h = 0; h < HS; ++h) { M[h] = __shfl_sync(0xffffffffu, base, 4 * h); inv[h] = __shfl_sync(0xffffffffu, over, 4 * h); }
        }
        if (lane < n) {
#pragma unroll
          for (int h = 0; h < HS; ++h)
            if (h < s) w += ex2(sc[h] - M[h]) * inv[h];
          p.weight_out[(int64_t)r + lane] = w;
        }
      }
    }
    wait_once();
  }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult qres;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess
               ? (EncodeTiledFn)ptr : nullptr;
  }();
  return fn;
}
// 8-bit pool as [rows][128 bytes], box = a page
bool map_pages8(CUtensorMap* m, const void* base, uint64_t n_pages) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {D, n_pages * PT}, strides[1] = {D};
  cuuint32_t box[2] = {D, PT}, es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// bf16 pool as [half of the head dimension][rows][64 elements], box = 32 tokens of both halves
bool map_pages(CUtensorMap* m, const void* base, uint64_t n_pages) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {64, n_pages * PT, 2}, strides[2] = {2 * D, 128};
  cuuint32_t box[3] = {64, HT, 2}, es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t align256(int64_t x) { return (x + 255) & ~(int64_t)255; }
int grid_ctas(const recache_ctx* ctx) { return ctx->sm_count > 0 ? ctx->sm_count : 148; }

}  // namespace

int64_t rc_mixed_split_workspace_bytes(const recache_ctx* ctx, int batch, int64_t n_pages) {
  const int64_t s = ctx->desc.n_q_heads / ctx->desc.n_kv_heads, slots = 2 * (int64_t)grid_ctas(ctx), items = (int64_t)batch * ctx->desc.n_kv_heads;
  return align256(slots * s * D * 4) + align256(slots * s * 8) + align256(items * 8) + align256(items * s * 8) +
         n_pages * PT * s * 4;
}

cudaError_t rc_launch_mixed_split(const recache_ctx* ctx, const MixedArgs& a, cudaStream_t st) {
  const int G = ctx->desc.n_kv_heads, Hq = ctx->desc.n_q_heads, s = Hq / G;
  const bool q8 = a.k8 != nullptr, weights = a.weight_out != nullptr;
  // (a map has a row at least; no page id is valid in an empty pool, so none is loaded)
  const uint64_t n_pages = a.n_pages > 0 ? a.n_pages : 1, n_pages8 = a.n_pages8 > 0 ? a.n_pages8 : 1;
  CUtensorMap tk, tv, tk8 = {}, tv8 = {};
  if (!map_pages(&tk, a.k_pages, n_pages) || !map_pages(&tv, a.v_pages, n_pages)) return cudaErrorInvalidValue;
  if (q8 && (!map_pages8(&tk8, a.k8, n_pages8) || !map_pages8(&tv8, a.v8, n_pages8))) return cudaErrorInvalidValue;
  const int ctas = grid_ctas(ctx);
  const int64_t slots = 2 * (int64_t)ctas, items = (int64_t)a.batch * G;
  MixParams p;
  p.q = (const __nv_bfloat16*)a.q; p.q_pos = a.q_pos;
  p.k_new = (const __nv_bfloat16*)a.k_new; p.v_new = (const __nv_bfloat16*)a.v_new;
  p.k_scale = a.k_scale; p.v_scale = a.v_scale; p.n_pages8 = a.n_pages8;
  p.k_pages = (__nv_bfloat16*)a.k_pages; p.v_pages = (__nv_bfloat16*)a.v_pages; p.n_pages = a.n_pages;
  p.res_pt = a.res_pt; p.max_res_pages = a.max_res_pages; p.res_len = a.res_len;
  p.hist_pt = a.hist_pt; p.max_hist_pages = a.max_hist_pages; p.hist_len = a.hist_len;
  p.n_items = (int)items; p.G = G; p.Hq = Hq; p.s = s; p.per_item = 0;
  p.appended = a.k_new != nullptr;
  p.out = a.o;
  uint8_t* ws = (uint8_t*)a.workspace;
  p.part_o = (float*)ws; ws += align256(slots * s * D * 4);
  p.part_ml = (float*)ws; ws += align256(slots * s * 8);
  p.part_cta = (int2*)ws; ws += align256(items * 8);
  p.item_ml = (float2*)ws; ws += align256(items * s * 8);
  p.score = (float*)ws;
  p.weight_in = a.weight_in; p.weight_out = a.weight_out;
  p.cos_tab = ctx->cos_tab; p.sin_tab = ctx->sin_tab; p.max_pos = ctx->desc.max_pos;
  p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
  p.status = ctx->status;
  // no more CTAs than units there can be
  const int64_t most = items * ((q8 ? 1 : 2) * (int64_t)a.max_res_pages + 2 * (int64_t)a.max_hist_pages);
  unsigned grid = (unsigned)(most > ctas ? ctas : (most > 0 ? most : 1));
  // One sequence: as many CTAs to each of its groups, so that nobody has to look at all lengths first.  Its items have the history in common, but not the
  // first part: where routes of one group are much longer than the others', the launch lasts as long as that group's share (8-bit routes of 20 thousand rows and
  // seven of 500: 13.3 us, where eight alike of the same total take 8.8; of 500 to 12 thousand, 11.0 and 9.3).
  if (a.batch == 1 && (unsigned)G <= grid) { p.per_item = (int)grid / G; grid = (unsigned)(p.per_item * G); }
  // Many items a CTA: the append has a launch of its own (decode_split.cu, same rule)
  if (a.k_new && items > 4 * (int64_t)ctas) {
    DecodeArgs d{a.q, a.q_pos, a.batch, a.k_new, a.v_new, a.k_pages, a.v_pages, a.n_pages, nullptr, 0, nullptr, a.hist_pt, a.max_hist_pages, a.hist_len,
                 a.o, a.out_dtype, nullptr, 0};
    const cudaError_t e = rc_launch_decode_append(ctx, d, st);
    if (e != cudaSuccess) return e;
    p.k_new = p.v_new = nullptr;
  }
  auto run = [&](auto type, auto eight, auto weighs) {
    using TO = decltype(type);
    constexpr bool Q8 = decltype(eight)::value, W = decltype(weighs)::value;
    {
      RcLaunchScope scope(ctx, RC_K_MIXED_ATTN, st);
      const cudaError_t e = rc_launch_overlapped(mixed_split_kernel<TO, Q8, W>, grid, THREADS, SM_ALLOC, st, tk8, tv8, tk, tv, p);
      if (e != cudaSuccess) return e;
    }
    RcLaunchScope scope(ctx, RC_K_MIXED_MERGE, st);
    constexpr int ROWS = MERGE_WARPS / ROW_WARPS;
    const int n_rows = a.batch * Hq, n_merge = (n_rows + ROWS - 1) / ROWS;
    return rc_launch_overlapped(s <= 4 ? mixed_merge_kernel<TO, Q8, W, 4> : mixed_merge_kernel<TO, Q8, W, 8>, n_merge + (W ? WSUB * grid : 0),
                                32 * MERGE_WARPS, 0, st, p, n_rows, n_merge);
  };
  auto by_type = [&](auto eight, auto weighs) {
    return a.out_dtype == RECACHE_F32 ? run(float(), eight, weighs) : run(__nv_bfloat16(), eight, weighs);
  };
  if (q8) return weights ? by_type(std::true_type(), std::true_type()) : by_type(std::true_type(), std::false_type());
  return weights ? by_type(std::false_type(), std::true_type()) : by_type(std::false_type(), std::false_type());
}
