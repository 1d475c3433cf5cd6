// Eviction from paged KV by accumulated attention weight.
//
// An item of more than `budget` rows keeps its last n_recent rows and, of the others, the budget - n_recent of
// greatest weight (the earlier row among equals, NaN below every number), in their order, copied to fresh
// pages: nothing that is read is written, so every page can be copied by a block of its own.
//   1. select: a block to an item.  Radix select of the (budget - n_recent)-th greatest weight over order-preserving
//      32-bit keys, 8 bits a pass (a histogram of the values that still agree with the bits found), then one pass in row order that
//      numbers the kept rows: block scans of (greater than the threshold, equal to it).
//   2. copy: a block to a new page, 16-byte pieces through the list of kept rows.
// Memory-bound: 4 bytes a row of the item, 2 * (2 * 256 + 4) a kept row of 128 bf16 elements.
#include "common.cuh"

namespace {

constexpr int SEL_THREADS = 1024;
constexpr int PER = 4;                       // rows of a thread in a numbering pass
constexpr int COPY_THREADS = 256;

// Greater weight, greater key; NaN 0; -0 as +0.
__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

struct Rows {                                 // an item's rows in the pool
  const int32_t* table; int max_pages, page_tokens; int64_t n_pages;
  __device__ __forceinline__ int64_t operator()(int r) const {   // -1: no such page
    const int pg = table[r / page_tokens];
    return pg < 0 || pg >= n_pages ? -1 : (int64_t)pg * page_tokens + r % page_tokens;
  }
};

__device__ __forceinline__ int64_t warp_incl(int64_t v, int lane) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int64_t n = __shfl_up_sync(0xffffffffu, v, off);
    if (lane >= off) v += n;
  }
  return v;
}

__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(const float* weight, const int32_t* table, int max_pages, const int32_t* len_in,
                                                                   int64_t n_pages, int page_tokens, int budget, int n_recent,
                                                                   const int32_t* free_pages, int64_t n_free_pages, int32_t* new_table,
                                                                   int max_new_pages, int32_t* new_len, int32_t* kept, int32_t* status) {
  __shared__ int hist[256];
  __shared__ int64_t sums[SEL_THREADS / 32];
  __shared__ int s_bin, s_left, s_before;
  const int it = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  rc_grid_wait();
  rc_grid_launch_next();
  const int64_t room = (int64_t)max_pages * page_tokens;
  auto rows_of = [&](int i) { return (int)min(max((int64_t)len_in[i], (int64_t)0), room); };
  const int n = rows_of(it);
  if (threadIdx.x == 0) {
    if (n != len_in[it]) rc_set_status(status, RECACHE_DEV_BAD_PAGE);
    new_len[it] = min(n, budget);
    s_before = 0;
  }
  const int32_t* tab = table + (int64_t)it * max_pages;
  int32_t* out = kept + (int64_t)it * budget;
  int32_t* new_tab = new_table + (int64_t)it * max_new_pages;
  const int new_pages = (int)(((int64_t)min(n, budget) + page_tokens - 1) / page_tokens);
  if (n <= budget) {                                       // keeps its pages
    for (int i = threadIdx.x; i < new_pages; i += SEL_THREADS) new_tab[i] = tab[i];
    for (int i = threadIdx.x; i < n; i += SEL_THREADS) out[i] = i;
    return;
  }
  const Rows row{tab, max_pages, page_tokens, n_pages};
  auto key_of = [&](int r) {
    const int64_t at = row(r);
    return at < 0 ? 0u : order_key(weight[at]);
  };
  __syncthreads();
  // ---- fresh pages: those behind the ones of the items before ----
  {
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
  const int n_cand = n - n_recent, want = budget - n_recent;   // want < n_cand
  // ---- the want-th greatest key ----
  uint32_t found = 0, mask = 0;
  int left = want;
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 256; i += SEL_THREADS) hist[i] = 0;
      __syncthreads();
      for (int r = threadIdx.x; r < n_cand; r += SEL_THREADS) {
        const uint32_t key = key_of(r);
        if ((key & mask) == found) atomicAdd(&hist[(key >> shift) & 255u], 1);
      }
      __syncthreads();
      if (warp == 0) {                                       // the bin that holds the left-th greatest, from the top
        int at = 0, h[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { h[i] = hist[255 - (lane * 8 + i)]; sum += h[i]; }
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, incl, off);
          if (lane >= off) incl += v;
        }
        at = incl - sum;
        if (at < left && incl >= left) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (at < left && at + h[i] >= left) { s_bin = 255 - (lane * 8 + i); s_left = left - at; }
            at += h[i];
          }
        }
      }
      __syncthreads();
      found |= (uint32_t)s_bin << shift;
      mask |= 255u << shift;
      left = s_left;
      __syncthreads();
    }
  }
  // ---- numbers of the kept rows: greater than the threshold, or one of the first `left` equal to it, or recent ----
  int64_t base = 0;                                          // (greater or recent) << 32 | equal, of the passes before
  bool bad = false;
  for (int r0 = 0; r0 < n; r0 += SEL_THREADS * PER) {
    const int r = r0 + threadIdx.x * PER;
    uint32_t gt = 0, eq = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      if (r + u < n) {
        if (row(r + u) < 0) bad = true;
        if (r + u >= n_cand) gt |= 1u << u;
        else if (want > 0) {
          const uint32_t key = key_of(r + u);
          if (key > found) gt |= 1u << u;
          else if (key == found) eq |= 1u << u;
        }
      }
    }
    const int64_t mine = (int64_t)__popc(gt) << 32 | (int64_t)__popc(eq);
    const int64_t incl = warp_incl(mine, lane);
    __syncthreads();
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    if (warp == 0) {
      const int64_t v = sums[lane];
      sums[lane] = warp_incl(v, lane);
    }
    __syncthreads();
    int64_t at = base + incl - mine + (warp ? sums[warp - 1] : 0);
    base += sums[SEL_THREADS / 32 - 1];
    int n_gt = (int)(at >> 32), n_eq = (int)(at & 0xffffffff);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const bool g = gt >> u & 1u, e = eq >> u & 1u;
      const int place = n_gt + min(n_eq, left);
      if (g || (e && n_eq < left)) out[place] = r + u;
      n_gt += g; n_eq += e;
    }
  }
  if (bad) rc_set_status(status, RECACHE_DEV_BAD_PAGE);
}

// One block a new page of an item that was over the budget.
__global__ void __launch_bounds__(COPY_THREADS) evict_copy_kernel(uint8_t* k_pages, uint8_t* v_pages, float* weight, const int32_t* table,
                                                                  int max_pages, const int32_t* len_in, int64_t n_pages, int page_tokens, int budget,
                                                                  const int32_t* new_table, int max_new_pages, const int32_t* kept, int new_pages,
                                                                  int row_bytes) {
  rc_grid_wait();
  rc_grid_launch_next();
  const int it = blockIdx.x / new_pages, p = blockIdx.x % new_pages;
  if (min((int64_t)len_in[it], (int64_t)max_pages * page_tokens) <= budget) return;
  const int pg = new_table[(int64_t)it * max_new_pages + p];
  if (pg < 0) return;
  const Rows row{table + (int64_t)it * max_pages, max_pages, page_tokens, n_pages};
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
  const int row_bytes = ctx->desc.head_dim * (ctx->desc.dtype == RECACHE_BF16 ? 2 : 4);
  if ((int64_t)a.n_items * new_pages > 0x7fffffff) return cudaErrorInvalidValue;
  {
    RcLaunchScope scope(ctx, RC_K_EVICT_SELECT, st);
    const cudaError_t e = rc_launch_overlapped(evict_select_kernel, a.n_items, SEL_THREADS, 0, st, (const float*)a.weight, a.table, a.max_pages, a.len,
                                               a.n_pages, pt, a.budget, a.n_recent, a.free_pages, a.n_free_pages, a.new_table, a.max_new_pages,
                                               a.new_len, a.kept, ctx->status);
    if (e != cudaSuccess) return e;
  }
  RcLaunchScope scope(ctx, RC_K_EVICT_COPY, st);
  return rc_launch_overlapped(evict_copy_kernel, a.n_items * new_pages, COPY_THREADS, 0, st, (uint8_t*)a.k_pages, (uint8_t*)a.v_pages, a.weight, a.table,
                              a.max_pages, a.len, a.n_pages, pt, a.budget, (const int32_t*)a.new_table, a.max_new_pages, (const int32_t*)a.kept, new_pages,
                              row_bytes);
}
