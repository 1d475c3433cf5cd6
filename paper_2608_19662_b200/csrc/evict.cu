// Eviction from paged KV by accumulated attention weight.
//
// An item of more than `budget` rows keeps its last n_recent rows and, of the others, the budget - n_recent of
// greatest weight (the earlier row among equals, NaN below every number), in their order, copied to fresh
// pages: nothing that is read is written, so all rows can be copied at once.
//   1. select: a cluster of blocks to an item, a run of rows to each.  The weights are read once, as order-preserving 32-bit
//      keys, into shared memory.  The (budget - n_recent)-th greatest is found in three passes of 11, 11 and 10 bits: a histogram of the keys
//      that agree with the bits found so far; a block sums a share of the counters, to which its peers add their few non-zero ones through
//      distributed shared memory.  (Eleven bits first: sign, exponent and
//      two bits more spread weights of one size over some forty counters, where a byte puts them into six, whose atomics queue.)  The
//      keys that agree in the first 11 are listed in the second pass, so that the third looks at few.  One pass in row order numbers
//      the kept rows: ballots inside a warp, counts of (greater than the threshold, equal to it) before each warp and block.
//   2. copy: a block to a new page, 16-byte pieces through the list of kept rows.
// (Both in one launch, the blocks of an item copying a run each: a full server's 512 items take as long, since its blocks select and copy in step,
// and one sequence takes 18 us instead of 12.)
// Memory-bound: 4 bytes a row of the item, 2 * (2 * 256 + 4) a kept row of 128 bf16 elements.  Measured: 512 items cut from some 3000 rows to 2048,
// 16 us + 139 (6.3 TB/s); 32 items of 40-90 thousand rows to 16384, 26 + 87; 8 items of 1088 rows to 1024, 7 + 3.5.  These are with tables as wide as the
// longest item: blocks to an item and room for keys go by the table's width, which the host knows.  With tables ten times as wide, 165 us instead of 158 in
// all, 130 instead of 117, 15 instead of 11.
#include "common.cuh"

namespace {

constexpr int MAX_KEYS = 20 * 1024;          // keys that a block keeps in shared memory; rows past them are read again in every pass
constexpr int BINS = 2048, SUMS = 2 * BINS + BINS / 2;
constexpr int RUN = 128;                     // rows that a warp numbers at a time, four a lane
constexpr int LIST = 1024;                   // keys that agree in their first 11 bits and are listed for the last pass
constexpr int COPY_THREADS = 256;

// Greater weight, greater key; NaN 0; -0 as +0.
__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

struct Rows {                                 // an item's rows in the pool
  const int32_t* table; int page_tokens, shift; int64_t n_pages;   // shift: page_tokens as a power of two, or -1
  __device__ __forceinline__ int operator()(int r) const {   // -1: no such page
    const int at = shift >= 0 ? r >> shift : r / page_tokens;
    const int pg = table[at];
    return pg < 0 || pg >= n_pages ? -1 : pg * page_tokens + (r - at * page_tokens);
  }
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// `p` as it lies in block `rank`'s shared memory.
__device__ __forceinline__ uint32_t peer(const int* p, uint32_t rank) {
  uint32_t to;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return to;
}
__device__ __forceinline__ int peer_load(const int* p, uint32_t rank) {
  int v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ int4 peer_load4(const int* p, uint32_t rank) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(peer(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void peer_add(const int* p, uint32_t rank, int v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.s32 [%0], %1;" ::"r"(peer(p, rank)), "r"(v) : "memory");
}

struct EvictParams {
  uint8_t* k_pages; uint8_t* v_pages; float* weight;
  const int32_t* table; int max_pages; const int32_t* len; int64_t n_pages;
  int page_tokens, shift, budget, n_recent;
  const int32_t* free_pages; int64_t n_free_pages;
  int32_t* new_table; int max_new_pages; int32_t* new_len; int32_t* kept;
  int key_room, segs, seg_shift;              // 16-byte pieces of a row, and as a power of two
  bool by_four;                               // four weights of a page from a multiple of four on are 16 aligned bytes
  int32_t* status;
};

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_select_kernel(const __grid_constant__ EvictParams p) {
  constexpr int WARPS = THREADS / 32;
  extern __shared__ __align__(16) uint32_t keys[];   // key_room, in runs of RUN
  __shared__ __align__(16) int hist[BINS];
  // clusters: a pass's sums, over the cluster, of this block's share of the counters; a place for each pass
  int* all = reinterpret_cast<int*>(keys + p.key_room);
  __shared__ uint32_t list[LIST];
  __shared__ int warp_sum[WARPS], gt_w[WARPS], eq_w[WARPS];
  __shared__ int totals[2];
  __shared__ int s_bin, s_left, s_before, s_list;
  const int C = (int)cluster_size(), rank = (int)cluster_rank();
  const int it = blockIdx.x / C, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  rc_grid_wait();
  rc_grid_launch_next();
  const int64_t room = (int64_t)p.max_pages * p.page_tokens;
  auto rows_of = [&](int i) { return (int)min(max((int64_t)p.len[i], (int64_t)0), room); };
  const int n = rows_of(it);
  if (threadIdx.x == 0 && rank == 0) {
    if (n != p.len[it]) rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
    p.new_len[it] = min(n, p.budget);
  }
  const int32_t* tab = p.table + (int64_t)it * p.max_pages;
  int32_t* out = p.kept + (int64_t)it * p.budget;
  int32_t* new_tab = p.new_table + (int64_t)it * p.max_new_pages;
  const int new_pages = (int)(((int64_t)min(n, p.budget) + p.page_tokens - 1) / p.page_tokens);
  if (n <= p.budget) {                                     // keeps its pages (the whole cluster leaves here)
    for (int i = rank * THREADS + threadIdx.x; i < new_pages; i += C * THREADS) new_tab[i] = tab[i];
    for (int i = rank * THREADS + threadIdx.x; i < n; i += C * THREADS) out[i] = i;
    return;
  }
  const Rows row{tab, p.page_tokens, p.shift, p.n_pages};
  const int n_cand = n - p.n_recent, want = p.budget - p.n_recent;   // want < n_cand
  // this block's candidates, in whole runs of RUN rows
  const int per = (int)((((int64_t)n_cand + C - 1) / C + RUN - 1) / RUN * RUN);
  const int r0 = (int)min((int64_t)n_cand, (int64_t)rank * per), r1 = (int)min((int64_t)n_cand, (int64_t)r0 + per), mine = r1 - r0;
  bool bad = false;
  const int n_keys = min(mine, p.key_room);
  if (want > 0 && p.by_four) {
    // four rows of a page to a load, six loads of a thread at a time: all their pages, then all their weights
    for (int i0 = 4 * threadIdx.x; i0 < n_keys; i0 += 6 * 4 * THREADS) {
      int at[6];
      float4 w[6];
#pragma unroll
      for (int u = 0; u < 6; ++u) at[u] = i0 + u * 4 * THREADS < n_keys ? row(r0 + i0 + u * 4 * THREADS) : -1;
#pragma unroll
      for (int u = 0; u < 6; ++u) w[u] = at[u] >= 0 ? *reinterpret_cast<const float4*>(p.weight + at[u]) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int u = 0; u < 6; ++u) {
        if (i0 + u * 4 * THREADS < n_keys) {
          bad |= at[u] < 0;
          *reinterpret_cast<uint4*>(&keys[i0 + u * 4 * THREADS]) =
              at[u] < 0 ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(order_key(w[u].x), order_key(w[u].y), order_key(w[u].z), order_key(w[u].w));
        }
      }
    }
  } else if (want > 0) {
    for (int i = threadIdx.x; i < n_keys; i += THREADS) {
      const int at = row(r0 + i);
      bad |= at < 0;
      keys[i] = at < 0 ? 0u : order_key(p.weight[at]);
    }
  }
  // four keys from row r0 + i on (i a multiple of 4); behind the block's rows anything
  auto keys_at = [&](int i) {
    if (i < p.key_room) return *reinterpret_cast<const uint4*>(&keys[i]);
    uint32_t k[4];
    for (int u = 0; u < 4; ++u) {
      const int at = i + u < mine ? row(r0 + i + u) : -1;
      bad |= at < 0 && i + u < mine;
      k[u] = at < 0 ? 0u : order_key(p.weight[at]);
    }
    return make_uint4(k[0], k[1], k[2], k[3]);
  };
  if (threadIdx.x == 0) { s_before = 0; s_list = 0; }
  for (int i = threadIdx.x; i < BINS; i += THREADS) hist[i] = 0;
  if (C > 1)
    for (int i = threadIdx.x; i < SUMS; i += THREADS) all[i] = 0;
  if (C > 1) cluster_sync(); else __syncthreads();           // (the sums of every peer are clear)
  // ---- fresh pages: those behind the ones of the items before ----
  if (rank == C - 1) {
    int before = 0;
    for (int i = threadIdx.x; i < it; i += THREADS) before += rows_of(i) > p.budget;
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0 && before) atomicAdd(&s_before, before);
    __syncthreads();
    const int64_t first = (int64_t)s_before * new_pages;
    for (int i = threadIdx.x; i < new_pages; i += THREADS) {
      int pg = -1;
      if (first + i >= p.n_free_pages) rc_set_status(p.status, RECACHE_DEV_NO_PAGES);
      else {
        pg = p.free_pages[first + i];
        if (pg < 0 || pg >= p.n_pages) { rc_set_status(p.status, RECACHE_DEV_BAD_PAGE); pg = -1; }
      }
      new_tab[i] = pg;
    }
  }
  // ---- the want-th greatest key ----
  uint32_t found = 0, mask = 0;
  int left = want;
  if (want > 0) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : BINS;
      int* sums = C > 1 ? all + pass * BINS : hist;
      const int n_list = s_list;
      if (pass == 2 && n_list <= LIST) {
        for (int i = threadIdx.x; i < n_list; i += THREADS)
          if ((list[i] & mask) == found) atomicAdd(&hist[list[i] & (bins - 1)], 1);
      } else {
        for (int i0 = warp * RUN; i0 < mine; i0 += WARPS * RUN) {
          const int i = i0 + 4 * lane;
          const uint4 v = keys_at(i);
          const uint32_t k[4] = {v.x, v.y, v.z, v.w};
          uint32_t in = 0;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if ((k[u] & mask) == found && i + u < mine) {
              atomicAdd(&hist[(k[u] >> shift) & (bins - 1)], 1);
              in |= 1u << u;
            }
          }
          if (pass == 1 && __any_sync(0xffffffffu, in != 0)) {   // one place in the list for the warp's, and the lanes' in a row
            int incl = __popc(in);
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
              const int x = __shfl_up_sync(0xffffffffu, incl, off);
              if (lane >= off) incl += x;
            }
            int at = 0;
            if (lane == 31) at = atomicAdd(&s_list, incl);
            at = __shfl_sync(0xffffffffu, at, 31) + incl - __popc(in);
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (in >> u & 1u) {
                if (at < LIST) list[at] = k[u];
                ++at;
              }
          }
        }
      }
      __syncthreads();
      if (C > 1) {                                             // what this block counted, to the block that sums those counters; few are not 0
        for (int i = threadIdx.x; i < bins; i += THREADS) {
          const int v = hist[i];
          if (v) {
            hist[i] = 0;
            peer_add(&sums[i], i / (bins / C), v);
          }
        }
        cluster_sync();
      }
      // a thread to PER bins, from the top: their counts, and the counts above them
      constexpr int PER = BINS / THREADS;
      const int top = bins - PER * (threadIdx.x + 1);
      int c[PER], sum = 0;
#pragma unroll
      for (int i = 0; i < PER; i += 4) {
        int4 v = make_int4(0, 0, 0, 0);
        if (top >= 0) v = C > 1 ? peer_load4(&sums[top + i], (top + i) / (bins / C)) : *reinterpret_cast<const int4*>(&sums[top + i]);
        c[i] = v.x; c[i + 1] = v.y; c[i + 2] = v.z; c[i + 3] = v.w;
        sum += v.x + v.y + v.z + v.w;
      }
      int incl = sum;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
      }
      if (lane == 31) warp_sum[warp] = incl;
      __syncthreads();
      const int before = incl - sum + __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane] : 0);
      if (before < left && before + sum >= left) {             // one thread's
        int at = before;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) {
          if (at < left && at + c[i] >= left) { s_bin = top + i; s_left = left - at; }
          at += c[i];
        }
      }
      if (C == 1) {
#pragma unroll
        for (int i = 0; i < PER; ++i) hist[PER * threadIdx.x + i] = 0;
      }
      __syncthreads();
      found |= (uint32_t)s_bin << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      left = s_left;
      __syncthreads();
    }
  }
  // ---- numbers of the kept candidates: greater than the threshold, or one of the first `left` equal to it ----
  const int runs = (mine + RUN - 1) / RUN, per_warp = (runs + WARPS - 1) / WARPS;
  const int c0 = min(runs, warp * per_warp), c1 = want > 0 ? min(runs, c0 + per_warp) : c0;
  // a lane's four rows of run c: which are greater, which equal
  auto flags = [&](int c, uint32_t& gt, uint32_t& eq) {
    const int i = c * RUN + 4 * lane;
    const uint4 v = keys_at(i);
    const uint32_t k[4] = {v.x, v.y, v.z, v.w};
    gt = eq = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u < mine) {
        gt |= (k[u] > found ? 1u : 0u) << u;
        eq |= (k[u] == found ? 1u : 0u) << u;
      }
    }
  };
  int n_gt = 0, n_eq = 0;
  for (int c = c0; c < c1; ++c) {
    uint32_t gt, eq;
    flags(c, gt, eq);
    n_gt += __popc(gt); n_eq += __popc(eq);
  }
  n_gt = __reduce_add_sync(0xffffffffu, n_gt); n_eq = __reduce_add_sync(0xffffffffu, n_eq);
  if (lane == 0) { gt_w[warp] = n_gt; eq_w[warp] = n_eq; }
  __syncthreads();
  if (warp == 0) {
    const int a = __reduce_add_sync(0xffffffffu, lane < WARPS ? gt_w[lane] : 0), b = __reduce_add_sync(0xffffffffu, lane < WARPS ? eq_w[lane] : 0);
    if (lane == 0) { totals[0] = a; totals[1] = b; }
  }
  if (C > 1) cluster_sync();
  n_gt = (lane < rank ? peer_load(&totals[0], lane) : 0) + (lane < warp ? gt_w[lane] : 0);
  n_eq = (lane < rank ? peer_load(&totals[1], lane) : 0) + (lane < warp ? eq_w[lane] : 0);
  n_gt = __reduce_add_sync(0xffffffffu, n_gt); n_eq = __reduce_add_sync(0xffffffffu, n_eq);
  for (int c = c0; c < c1; ++c) {
    uint32_t gt, eq;
    flags(c, gt, eq);
    const int both = __popc(gt) << 16 | __popc(eq);
    int incl = both;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += v;
    }
    int g = n_gt + ((incl - both) >> 16), e = n_eq + ((incl - both) & 0xffff);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool is_gt = gt >> u & 1u, is_eq = eq >> u & 1u;
      if (is_gt || (is_eq && e < left)) out[g + min(e, left)] = r0 + c * RUN + 4 * lane + u;
      g += is_gt; e += is_eq;
    }
    const int last = __shfl_sync(0xffffffffu, incl, 31);
    n_gt += last >> 16; n_eq += last & 0xffff;
  }
  for (int i = rank * THREADS + threadIdx.x; i < p.n_recent; i += C * THREADS) {
    out[want + i] = n_cand + i;
    bad |= row(n_cand + i) < 0;
  }
  if (bad) rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
  if (C > 1) cluster_sync();                                   // the peers have read this block's totals
}

// One block a new page of an item that was over the budget.  (A thread has two pieces of keys and of values on their way; four cost 2-4 %.)
__global__ void __launch_bounds__(COPY_THREADS) evict_copy_kernel(const __grid_constant__ EvictParams p, int new_pages) {
  constexpr int AHEAD = 2;
  __shared__ int src[COPY_THREADS];
  rc_grid_wait();
  rc_grid_launch_next();
  const int it = blockIdx.x / new_pages, at_page = blockIdx.x % new_pages;
  if (min((int64_t)p.len[it], (int64_t)p.max_pages * p.page_tokens) <= p.budget) return;
  const int pg = p.new_table[(int64_t)it * p.max_new_pages + at_page];
  if (pg < 0) return;
  const Rows row{p.table + (int64_t)it * p.max_pages, p.page_tokens, p.shift, p.n_pages};
  const int first = at_page * p.page_tokens, rows = min(p.page_tokens, p.budget - first);
  const int32_t* old = p.kept + (int64_t)it * p.budget + first;
  for (int b0 = 0; b0 < rows; b0 += COPY_THREADS) {            // (a page of up to 256 tokens at once)
    const int n = min(COPY_THREADS, rows - b0), to0 = pg * p.page_tokens + b0;
    __syncthreads();
    float w = 0.f;
    int from = -1;
    if (threadIdx.x < n) {
      from = row(old[b0 + threadIdx.x]);
      src[threadIdx.x] = from;
      if (from >= 0) w = p.weight[from];
    }
    __syncthreads();
    for (int e0 = threadIdx.x; e0 < n * p.segs; e0 += AHEAD * COPY_THREADS) {
      uint4 kx[AHEAD], vx[AHEAD];
      int to[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int e = e0 + u * COPY_THREADS;
        to[u] = -1;
        if (e < n * p.segs) {
          const int r = p.seg_shift >= 0 ? e >> p.seg_shift : e / p.segs, c = e - r * p.segs, f = src[r];
          if (f >= 0) {
            to[u] = e;
            kx[u] = *reinterpret_cast<const uint4*>(p.k_pages + ((int64_t)f * p.segs + c) * 16);
            vx[u] = *reinterpret_cast<const uint4*>(p.v_pages + ((int64_t)f * p.segs + c) * 16);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (to[u] >= 0) {
          const int64_t at = ((int64_t)to0 * p.segs + to[u]) * 16;
          *reinterpret_cast<uint4*>(p.k_pages + at) = kx[u];
          *reinterpret_cast<uint4*>(p.v_pages + at) = vx[u];
        }
      }
    }
    if (from >= 0) p.weight[to0 + threadIdx.x] = w;
  }
}

}  // namespace

cudaError_t rc_launch_evict(const recache_ctx* ctx, const EvictArgs& a, cudaStream_t st) {
  const int pt = ctx->desc.page_tokens, sms = ctx->sm_count > 0 ? ctx->sm_count : 148;
  auto power_of = [](int x) { int s = 0; while ((1 << s) < x) ++s; return (1 << s) == x ? s : -1; };
  if (a.n_items > 0x7fffffff / 8) return cudaErrorInvalidValue;
  // Blocks to an item: as long as each has some 2048 rows of the longest that the table can hold, and all are there at once.  (With 32 items of
  // 40-90 thousand rows, eight blocks an item 30 us where sixteen, a cluster size that is not portable, took 59.)
  const int64_t room = (int64_t)a.max_pages * pt, new_pages = ((int64_t)a.budget + pt - 1) / pt;
  if (a.n_items * new_pages > 0x7fffffff) return cudaErrorInvalidValue;
  int C = 1;
  while (C < 8 && room / (2 * C) >= 2048 && (int64_t)a.n_items * C * 2 <= 4 * sms) C *= 2;
  const int64_t rows = ((room + C - 1) / C + RUN - 1) / RUN * RUN;
  const int segs = ctx->desc.head_dim * (ctx->desc.dtype == RECACHE_BF16 ? 2 : 4) / 16;
  EvictParams p{(uint8_t*)a.k_pages, (uint8_t*)a.v_pages, a.weight, a.table, a.max_pages, a.len, a.n_pages, pt, power_of(pt), a.budget, a.n_recent,
                a.free_pages, a.n_free_pages, a.new_table, a.max_new_pages, a.new_len, a.kept, (int)(rows < MAX_KEYS ? rows : MAX_KEYS), segs,
                power_of(segs), pt % 4 == 0 && (reinterpret_cast<uintptr_t>(a.weight) & 15) == 0, ctx->status};
  // 512 threads to a block where all blocks are there at once (two an SM), else 256 (four an SM while the tables hold some ten thousand rows, two from
  // twenty thousand on)
  const bool wide = (int64_t)a.n_items * C <= 2 * sms;
  auto select = [&](auto kernel, unsigned threads) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (MAX_KEYS + SUMS) * 4);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = C; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.n_items * C)); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = (size_t)(p.key_room + (C > 1 ? SUMS : 0)) * 4; cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = 2;
    RcLaunchScope scope(ctx, RC_K_EVICT_SELECT, st);
    return cudaLaunchKernelEx(&cfg, kernel, p);
  };
  const cudaError_t e = wide ? select(evict_select_kernel<512>, 512) : select(evict_select_kernel<256>, 256);
  if (e != cudaSuccess) return e;
  RcLaunchScope scope(ctx, RC_K_EVICT_COPY, st);
  return rc_launch_overlapped(evict_copy_kernel, (unsigned)(a.n_items * new_pages), COPY_THREADS, 0, st, p, (int)new_pages);
}
