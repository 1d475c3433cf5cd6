// Eviction from paged KV by accumulated attention weight.
//
// An item of more than `budget` rows keeps its last n_recent rows and, of the others, the budget - n_recent of
// greatest weight (the earlier row among equals, NaN below every number), in their order, copied to fresh
// pages: nothing that is read is written, so every page can be copied by a block of its own.
//   1. select: a cluster of blocks to an item, a run of rows to each.  The weights are read once, as order-preserving 32-bit
//      keys, into shared memory; the (budget - n_recent)-th greatest is found 8 bits a pass (a histogram of the keys that still
//      agree with the bits found, summed over the cluster through distributed shared memory), and one pass in row order numbers the kept
//      rows: ballots inside a warp, counts of (greater than the threshold, equal to it) before each warp and block.
//   2. copy: a block to a new page, 16-byte pieces through the list of kept rows.
// Memory-bound: 4 bytes a row of the item, 2 * (2 * 256 + 4) a kept row of 128 bf16 elements.
#include "common.cuh"

namespace {

constexpr int SEL_THREADS = 512, SEL_WARPS = SEL_THREADS / 32;
constexpr int MAX_KEYS = 24 * 1024;          // keys that a block keeps in shared memory; rows past them are read again in every pass
constexpr int LIST = 2048;                   // keys that agree in their first 8 bits and are listed for the later passes
constexpr int COPY_THREADS = 256;

// Greater weight, greater key; NaN 0; -0 as +0.
__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

struct Rows {                                 // an item's rows in the pool
  const int32_t* table; int page_tokens, shift; int64_t n_pages;   // shift: page_tokens as a power of two, or -1
  __device__ __forceinline__ int64_t operator()(int r) const {   // -1: no such page
    const int at = shift >= 0 ? r >> shift : r / page_tokens;
    const int pg = table[at];
    return pg < 0 || pg >= n_pages ? -1 : (int64_t)pg * page_tokens + (r - at * page_tokens);
  }
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The int at `p` in block `rank`'s shared memory.
__device__ __forceinline__ int peer_int(const int* p, uint32_t rank) {
  uint32_t at, to;
  int v;
  at = (uint32_t)__cvta_generic_to_shared(p);
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(to) : "memory");
  return v;
}

__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(const float* weight, const int32_t* table, int max_pages, const int32_t* len_in,
                                                                   int64_t n_pages, int page_tokens, int shift, int budget, int n_recent,
                                                                   const int32_t* free_pages, int64_t n_free_pages, int32_t* new_table,
                                                                   int max_new_pages, int32_t* new_len, int32_t* kept, int key_room, int32_t* status) {
  extern __shared__ uint32_t keys[];          // key_room
  __shared__ int hist[2][256];                // (two, so that a pass may clear one while peers still read the other)
  __shared__ int all[256];
  __shared__ int gt_w[SEL_WARPS], eq_w[SEL_WARPS];
  __shared__ int totals[2];
  __shared__ uint32_t list[LIST];
  __shared__ int s_bin, s_left, s_before, s_list;
  const int C = (int)cluster_size(), rank = (int)cluster_rank();
  const int it = blockIdx.x / C, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  rc_grid_wait();
  rc_grid_launch_next();
  const int64_t room = (int64_t)max_pages * page_tokens;
  auto rows_of = [&](int i) { return (int)min(max((int64_t)len_in[i], (int64_t)0), room); };
  const int n = rows_of(it);
  if (threadIdx.x == 0 && rank == 0) {
    if (n != len_in[it]) rc_set_status(status, RECACHE_DEV_BAD_PAGE);
    new_len[it] = min(n, budget);
  }
  const int32_t* tab = table + (int64_t)it * max_pages;
  int32_t* out = kept + (int64_t)it * budget;
  int32_t* new_tab = new_table + (int64_t)it * max_new_pages;
  const int new_pages = (int)(((int64_t)min(n, budget) + page_tokens - 1) / page_tokens);
  if (n <= budget) {                                       // keeps its pages (the whole cluster leaves here)
    for (int i = rank * SEL_THREADS + threadIdx.x; i < new_pages; i += C * SEL_THREADS) new_tab[i] = tab[i];
    for (int i = rank * SEL_THREADS + threadIdx.x; i < n; i += C * SEL_THREADS) out[i] = i;
    return;
  }
  const Rows row{tab, page_tokens, shift, n_pages};
  const int n_cand = n - n_recent, want = budget - n_recent;   // want < n_cand
  // this block's candidates, in whole warps' runs of 32 rows
  const int per = (int)((((int64_t)n_cand + C - 1) / C + 31) / 32 * 32);
  const int r0 = (int)min((int64_t)n_cand, (int64_t)rank * per), r1 = (int)min((int64_t)n_cand, (int64_t)r0 + per);
  bool bad = false;
  auto fresh_key = [&](int r) {
    const int64_t at = row(r);
    bad |= at < 0;
    return at < 0 ? 0u : order_key(weight[at]);
  };
#pragma unroll 8
  for (int i = threadIdx.x; i < min(r1 - r0, key_room); i += SEL_THREADS) keys[i] = fresh_key(r0 + i);
  auto key_of = [&](int r) { return r - r0 < key_room ? keys[r - r0] : fresh_key(r); };
  if (threadIdx.x == 0) { s_before = 0; s_list = 0; }
  if (threadIdx.x < 256) hist[0][threadIdx.x] = 0;
  __syncthreads();
  // ---- fresh pages: those behind the ones of the items before ----
  if (rank == C - 1) {
    int before = 0;
    for (int i = threadIdx.x; i < it; i += SEL_THREADS) before += rows_of(i) > budget;
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0 && before) atomicAdd(&s_before, before);
    __syncthreads();
    const int64_t first = (int64_t)s_before * new_pages;
    for (int i = threadIdx.x; i < new_pages; i += SEL_THREADS) {
      int pg = -1;
      if (first + i >= n_free_pages) rc_set_status(status, RECACHE_DEV_NO_PAGES);
      else {
        pg = free_pages[first + i];
        if (pg < 0 || pg >= n_pages) { rc_set_status(status, RECACHE_DEV_BAD_PAGE); pg = -1; }
      }
      new_tab[i] = pg;
    }
  }
  // ---- the want-th greatest key ----
  uint32_t found = 0, mask = 0;
  int left = want, n_list = 0;
  if (want > 0) {
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      int* h = hist[pass & 1];
      if (pass >= 2 && n_list <= LIST) {
        for (int i = threadIdx.x; i < n_list; i += SEL_THREADS)
          if ((list[i] & mask) == found) atomicAdd(&h[(list[i] >> shift) & 255u], 1);
      } else {
        for (int i0 = warp * 32; i0 < r1 - r0; i0 += SEL_THREADS) {
          const int i = i0 + lane;
          const uint32_t key = i < r1 - r0 ? key_of(r0 + i) : 0u;
          const bool in = i < r1 - r0 && (key & mask) == found;
          if (in) atomicAdd(&h[(key >> shift) & 255u], 1);
          if (pass == 1) {                                     // those that agree in the first 8 bits, for the passes behind
            const uint32_t who = __ballot_sync(0xffffffffu, in);
            int at = 0;
            if (lane == 0 && who) at = atomicAdd(&s_list, __popc(who));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1u));
            if (in && at < LIST) list[at] = key;
          }
        }
      }
      if (C > 1) cluster_sync(); else __syncthreads();
      if (threadIdx.x < 256) {
        int sum = 0;
        if (C > 1) {
#pragma unroll 8
          for (int k = 0; k < C; ++k) sum += peer_int(&h[threadIdx.x], k);
        } else {
          sum = h[threadIdx.x];
        }
        all[threadIdx.x] = sum;
        hist[1 - (pass & 1)][threadIdx.x] = 0;                 // (the peers read it before the barrier of this pass)
      }
      __syncthreads();
      if (warp == 0) {                                         // the bin that holds the left-th greatest, from the top
        int c[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = all[255 - (lane * 8 + i)]; sum += c[i]; }
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, incl, off);
          if (lane >= off) incl += v;
        }
        int at = incl - sum;
        if (at < left && incl >= left) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (at < left && at + c[i] >= left) { s_bin = 255 - (lane * 8 + i); s_left = left - at; }
            at += c[i];
          }
        }
      }
      __syncthreads();
      found |= (uint32_t)s_bin << shift;
      mask |= 255u << shift;
      left = s_left;
      n_list = s_list;
      __syncthreads();
    }
  }
  // ---- numbers of the kept candidates: greater than the threshold, or one of the first `left` equal to it ----
  const int chunks = (r1 - r0 + 31) / 32, per_warp = (chunks + SEL_WARPS - 1) / SEL_WARPS;
  const int c0 = min(chunks, warp * per_warp), c1 = min(chunks, c0 + per_warp);
  auto flags = [&](int c, uint32_t& gt, uint32_t& eq) {
    const int r = r0 + c * 32 + lane;
    const uint32_t key = r < r1 ? key_of(r) : 0u;
    gt = __ballot_sync(0xffffffffu, r < r1 && want > 0 && key > found);
    eq = __ballot_sync(0xffffffffu, r < r1 && want > 0 && key == found);
  };
  int n_gt = 0, n_eq = 0;
  for (int c = c0; c < c1; ++c) {
    uint32_t gt, eq;
    flags(c, gt, eq);
    n_gt += __popc(gt); n_eq += __popc(eq);
  }
  if (lane == 0) { gt_w[warp] = n_gt; eq_w[warp] = n_eq; }
  __syncthreads();
  if (threadIdx.x < 2) {
    int sum = 0;
    for (int w = 0; w < SEL_WARPS; ++w) sum += (threadIdx.x ? eq_w : gt_w)[w];
    totals[threadIdx.x] = sum;
  }
  if (C > 1) cluster_sync(); else __syncthreads();
  n_gt = n_eq = 0;
  for (int k = 0; k < rank; ++k) { n_gt += peer_int(&totals[0], k); n_eq += peer_int(&totals[1], k); }
  for (int w = 0; w < warp; ++w) { n_gt += gt_w[w]; n_eq += eq_w[w]; }
  for (int c = c0; c < c1; ++c) {
    uint32_t gt, eq;
    flags(c, gt, eq);
    const uint32_t below = (1u << lane) - 1u;
    const int e = n_eq + __popc(eq & below), place = n_gt + __popc(gt & below) + min(e, left);
    if ((gt >> lane & 1u) || ((eq >> lane & 1u) && e < left)) out[place] = r0 + c * 32 + lane;
    n_gt += __popc(gt); n_eq += __popc(eq);
  }
  for (int i = rank * SEL_THREADS + threadIdx.x; i < n_recent; i += C * SEL_THREADS) {
    out[want + i] = n_cand + i;
    bad |= row(n_cand + i) < 0;
  }
  if (bad) rc_set_status(status, RECACHE_DEV_BAD_PAGE);
  if (C > 1) cluster_sync();                                   // the peers have read this block's totals
}

// One block a new page of an item that was over the budget.
__global__ void __launch_bounds__(COPY_THREADS) evict_copy_kernel(uint8_t* k_pages, uint8_t* v_pages, float* weight, const int32_t* table,
                                                                  int max_pages, const int32_t* len_in, int64_t n_pages, int page_tokens, int shift, int budget,
                                                                  const int32_t* new_table, int max_new_pages, const int32_t* kept, int new_pages,
                                                                  int row_bytes) {
  rc_grid_wait();
  rc_grid_launch_next();
  const int it = blockIdx.x / new_pages, p = blockIdx.x % new_pages;
  if (min((int64_t)len_in[it], (int64_t)max_pages * page_tokens) <= budget) return;
  const int pg = new_table[(int64_t)it * max_new_pages + p];
  if (pg < 0) return;
  const Rows row{table + (int64_t)it * max_pages, page_tokens, shift, n_pages};
  const int rows = min(page_tokens, budget - p * page_tokens), segs = row_bytes / 16;
  const int32_t* list = kept + (int64_t)it * budget + (int64_t)p * page_tokens;
  const int64_t to = (int64_t)pg * page_tokens;
  for (int r = threadIdx.x; r < rows; r += COPY_THREADS) {
    const int64_t from = row(list[r]);
    if (from >= 0) weight[to + r] = weight[from];
  }
  for (int e0 = threadIdx.x; e0 < rows * segs; e0 += 4 * COPY_THREADS) {
    uint4 kx[4], vx[4];
    int64_t dst[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = e0 + u * COPY_THREADS;
      dst[u] = -1;
      if (e < rows * segs) {
        const int r = e / segs, c = e - r * segs;
        const int64_t from = row(list[r]);
        if (from >= 0) {
          dst[u] = (to + r) * row_bytes + c * 16;
          kx[u] = *reinterpret_cast<const uint4*>(k_pages + from * row_bytes + c * 16);
          vx[u] = *reinterpret_cast<const uint4*>(v_pages + from * row_bytes + c * 16);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (dst[u] >= 0) {
        *reinterpret_cast<uint4*>(k_pages + dst[u]) = kx[u];
        *reinterpret_cast<uint4*>(v_pages + dst[u]) = vx[u];
      }
  }
}

}  // namespace

cudaError_t rc_launch_evict(const recache_ctx* ctx, const EvictArgs& a, cudaStream_t st) {
  const int pt = ctx->desc.page_tokens, new_pages = (int)(((int64_t)a.budget + pt - 1) / pt);
  const int row_bytes = ctx->desc.head_dim * (ctx->desc.dtype == RECACHE_BF16 ? 2 : 4), sms = ctx->sm_count > 0 ? ctx->sm_count : 148;
  int shift = 0;
  while ((1 << shift) < pt) ++shift;
  if ((1 << shift) != pt) shift = -1;
  if ((int64_t)a.n_items * new_pages > 0x7fffffff || a.n_items > 0x7fffffff / 8) return cudaErrorInvalidValue;
  {
    // Blocks to an item: as many as the card has room for beside the other items' (four blocks an SM), as long as each has some
    // 2048 rows of the longest that the table can hold.
    const int64_t room = (int64_t)a.max_pages * pt;
    int C = 1;
    while (C < 8 && (int64_t)a.n_items * C * 2 <= 4 * sms && room / (2 * C) >= 2048) C *= 2;
    const int64_t rows = (room + C - 1) / C + 32;
    const int key_room = (int)(rows < MAX_KEYS ? rows : MAX_KEYS);
    const cudaError_t e0 = cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_KEYS * 4);
    if (e0 != cudaSuccess) return e0;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = C; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.n_items * C)); cfg.blockDim = dim3(SEL_THREADS); cfg.dynamicSmemBytes = (size_t)key_room * 4; cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = 2;
    RcLaunchScope scope(ctx, RC_K_EVICT_SELECT, st);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, evict_select_kernel, (const float*)a.weight, a.table, a.max_pages, a.len, a.n_pages, pt, shift, a.budget,
                                             a.n_recent, a.free_pages, a.n_free_pages, a.new_table, a.max_new_pages, a.new_len, a.kept, key_room,
                                             ctx->status);
    if (e != cudaSuccess) return e;
  }
  RcLaunchScope scope(ctx, RC_K_EVICT_COPY, st);
  return rc_launch_overlapped(evict_copy_kernel, a.n_items * new_pages, COPY_THREADS, 0, st, (uint8_t*)a.k_pages, (uint8_t*)a.v_pages, a.weight, a.table,
                              a.max_pages, a.len, a.n_pages, pt, shift, a.budget, (const int32_t*)a.new_table, a.max_new_pages, (const int32_t*)a.kept, new_pages,
                              row_bytes);
}
