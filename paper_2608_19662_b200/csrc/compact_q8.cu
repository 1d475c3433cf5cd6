// Compaction into 8-bit pages: the rows that paged compaction would copy, as e4m3 values with one
// power-of-two scale for a page's keys and one for its values.
//     scale = 2^e,   e = the least integer >= -126 with max|finite x| <= 448 2^e          (1 where the maximum is 0)
// A value is divided by the scale and rounded to the nearest e4m3 value (ties to even).  A power of two makes the division exact, so
// that a value is rounded once, and costs e4m3 nothing: its relative precision is the same all over its range.
//
// Two launches where a page has 64 tokens:
//   1. count: a block to a request: kept tokens of every listed resource (a warp each), lengths of the request's routes.
//   2. pack: persistent blocks, two an SM, each an equal run of the pages of all routes.  Eight warps take the pages: all rows on their way to
//      shared memory at once, the next page's while this one's two maxima are found and its values converted and stored.  Two more warps run
//      ahead of them, by up to RING pages, and list the rows: they find the first route by a prefix over the routes' pages and then walk routes,
//      resources and keep mask in order, 1024 tokens at a time, so that the chain of dependent loads is one per resource and not one per
//      page (page by page, every step waiting behind the stream of rows, the launch took 90 us where it takes 54: 64 sequences; with one
//      lister 56).  They also write the page table.  (As launches of their own the plan, by one block, and the index list took 19 + 20 us.)
// Measured: 64 sequences, 368 thousand rows, 58 us with the count for 285 MB; 16 requests 26 us; one request 11 us, a chain of ten loads.
// Other page sizes go through the launches of the paged compaction, without a row copied, and a kernel that reads its index list.
// Memory-bound: 512 bytes read and 256 written for a row's key and value of 128 bf16 elements.
#include "common.cuh"

namespace {

constexpr int TPB = 256;

// Magnitude bits of a finite value, 0 for infinities and NaN (they take no part in the scale).
__device__ __forceinline__ uint32_t mag_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// e4m3 pair of (lo, hi) * inv; infinities become NaN, as NaN does (the type has no infinity).
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi, float inv) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi * inv), "f"(lo * inv));
  uint32_t v = r;
  if ((__float_as_uint(lo) & 0x7fffffffu) == 0x7f800000u) v |= 0x7fu;
  if ((__float_as_uint(hi) & 0x7fffffffu) == 0x7f800000u) v |= 0x7f00u;
  return v;
}
template <typename T> __device__ __forceinline__ void load16(const uint4& u, float* f);
template <> __device__ __forceinline__ void load16<float>(const uint4& u, float* f) {
  f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
}
template <> __device__ __forceinline__ void load16<__nv_bfloat16>(const uint4& u, float* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}

template <typename T> __device__ __forceinline__ void store8(uint8_t* to, const uint4& u, float inv);
// Largest magnitude bits of 16 bytes of T, infinities and NaN with them: the running maximum m, of pairs of halves for bf16.
template <typename T> __device__ __forceinline__ uint32_t top_of(const uint4& u, uint32_t m) {
  if constexpr (sizeof(T) == 2)
    return __vmaxu2(m, __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu)));
  else
    return max(m, max(max(u.x & 0x7fffffffu, u.y & 0x7fffffffu), max(u.z & 0x7fffffffu, u.w & 0x7fffffffu)));
}
// ... as the bits of a float
template <typename T> __device__ __forceinline__ uint32_t top_bits(uint32_t m) {
  return sizeof(T) == 2 ? max(m & 0xffffu, m >> 16) << 16 : m;
}
// 16 bytes of finite T as e4m3 values of x * 2^-e (inv: 2^-e, for bf16 in both halves of a pair of bf16: the product is exact there too)
template <typename T> __device__ __forceinline__ void store8_finite(uint8_t* to, const uint4& u, uint32_t inv) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t x;
      unsigned short r;
      asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(x) : "r"(w[i]), "r"(inv));
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(__uint_as_float(x & 0xffff0000u)), "f"(__uint_as_float(x << 16)));
      h[i] = r;
    }
    *reinterpret_cast<uint2*>(to) = make_uint2(__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410));
  } else {
    store8<T>(to, u, __uint_as_float(inv));
  }
}

// 16 bytes of T as e4m3 values of x * inv
template <typename T> __device__ __forceinline__ void store8(uint8_t* to, const uint4& u, float inv) {
  constexpr int N = 16 / sizeof(T);
  float f[N];
  load16<T>(u, f);
  uint32_t o[N / 4];
#pragma unroll
  for (int i = 0; i < N; i += 4) o[i / 4] = to_e4m3x2(f[i], f[i + 1], inv) | to_e4m3x2(f[i + 2], f[i + 3], inv) << 16;
  if constexpr (N == 8) *reinterpret_cast<uint2*>(to) = make_uint2(o[0], o[1]);
  else *reinterpret_cast<uint32_t*>(to) = o[0];
}
// Exponent of the scale for a largest magnitude of these bits: 2^(x - 127) * 1.f fits 448 * 2^e = 1.75 * 2^(8 + e) from e = x - 127 - 8 on, or one
// later where 1.f > 1.75.
__device__ __forceinline__ int scale_exponent(uint32_t top) {
  return top == 0 ? 0 : max(-126, (int)(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0));
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // 2^e of a normal number

template <typename T>
__global__ void __launch_bounds__(TPB) pack8_kernel(const T* k_cache, const T* v_cache, int64_t pool_tokens, const int32_t* route_cu,
                                                    const int32_t* route_idx, int64_t row_capacity, const int32_t* page_cu, int n_routes, int G,
                                                    int d, int page_tokens, const int32_t* free_pages, int64_t n_free_pages, int64_t n_pool_pages,
                                                    uint8_t* k8, uint8_t* v8, float* k_scale, float* v_scale, int32_t* status) {
  constexpr int N = 16 / sizeof(T);
  __shared__ uint32_t top;
  rc_grid_wait();
  rc_grid_launch_next();
  const int64_t total = 2 * (int64_t)page_cu[n_routes];
  const int segs = d / N;
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int pi = (int)(w >> 1);
    if (pi >= n_free_pages) break;                       // flagged by the plan
    const int pg = free_pages[pi];
    if (pg < 0 || pg >= n_pool_pages) continue;          // flagged by the plan
    const int route = rc_find_segment(page_cu, n_routes, pi);
    const int64_t first = (int64_t)route_cu[route] + (int64_t)(pi - page_cu[route]) * page_tokens;
    // (an index past the list's capacity was never written)
    const int64_t last = min((int64_t)route_cu[route + 1], min(row_capacity, (int64_t)RC_MAX_ROWS));
    const int rows = (int)min((int64_t)page_tokens, last - first);
    if (rows <= 0) continue;
    const T* src = ((w & 1) ? v_cache : k_cache) + (int64_t)(route % G) * pool_tokens * d;
    uint8_t* dst = ((w & 1) ? v8 : k8) + (int64_t)pg * page_tokens * d;
    uint32_t m = 0;
    for (int e = threadIdx.x; e < rows * segs; e += TPB) {
      const int r = e / segs, c = e - r * segs;
      float f[N];
      load16<T>(*reinterpret_cast<const uint4*>(src + (int64_t)route_idx[first + r] * d + c * N), f);
#pragma unroll
      for (int i = 0; i < N; ++i) m = max(m, mag_bits(f[i]));
    }
    __syncthreads();                                     // `top` may still be read from the page before
    if (threadIdx.x == 0) top = 0;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) atomicMax(&top, m);
    __syncthreads();
    const int e2 = scale_exponent(top);
    const float inv = power(-e2);
    if (threadIdx.x == 0) ((w & 1) ? v_scale : k_scale)[pg] = power(e2);
    for (int e = threadIdx.x; e < rows * segs; e += TPB) {
      const int r = e / segs, c = e - r * segs;
      store8<T>(dst + (int64_t)r * d + c * N, *reinterpret_cast<const uint4*>(src + (int64_t)route_idx[first + r] * d + c * N), inv);
    }
  }
}

// ---- pages of 64 tokens ----
constexpr int PT = 64;
constexpr int COUNT_THREADS = 512;
constexpr int WORKERS = 256;                 // threads that pack
constexpr int LISTERS = 2;                   // warps that list rows, for half of the block's pages each
constexpr int MAX_PAGES = 1 << 30;           // pages that are numbered; no pool has a 32nd of them
constexpr int RING = 32;                     // pages whose rows are listed ahead: 1024 mask tokens fill up to 17
constexpr uint32_t WAIT_PROBES = 1u << 21;   // ~2.8 s

__device__ __forceinline__ int pages_of(int rows) { return (int)(((uint32_t)rows + PT - 1) / PT); }
__device__ __forceinline__ int add_pages(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)MAX_PAGES); }

// 16 keep bytes from token t of the pool on, as bits; tokens >= end (<= pool_tokens) are 0.
__device__ __forceinline__ uint32_t keep_bits(const uint8_t* keep, int64_t t, int64_t end, int64_t pool_tokens) {
  uint32_t bits = 0;
  if (t >= end) return 0;
  const uint8_t* p = keep + t;
  if (t >= 4 && t + 20 <= pool_tokens) {                  // five whole words around them are the mask's own
    const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3u);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(p - shift);
    uint32_t lo = w[0];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t hi = w[i + 1];
      const uint32_t m = __vcmpne4(__funnelshift_r(lo, hi, 8 * shift), 0u) & 0x08040201u;
      bits |= ((m | m >> 8 | m >> 16 | m >> 24) & 15u) << (4 * i);
      lo = hi;
    }
    return t + 16 <= end ? bits : bits & ((1u << (int)(end - t)) - 1u);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (t + i < end && p[i] != 0) bits |= 1u << i;
  return bits;
}

// The same for 32 tokens, asked for early: the words around them, and their bits.
__device__ __forceinline__ bool whole_words(int64_t t, int64_t pool_tokens) { return t >= 4 && t + 36 <= pool_tokens; }
__device__ __forceinline__ void keep_words(const uint8_t* keep, int64_t t, int64_t end, int64_t pool_tokens, uint32_t (&w)[9]) {
  if (t >= end || !whole_words(t, pool_tokens)) return;
  const uint32_t* from = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(keep + t) & ~(uintptr_t)3);
#pragma unroll
  for (int i = 0; i < 9; ++i) w[i] = from[i];
}
__device__ __forceinline__ uint32_t keep_bits32(const uint8_t* keep, int64_t t, int64_t end, int64_t pool_tokens, const uint32_t (&w)[9]) {
  if (t >= end) return 0;
  if (!whole_words(t, pool_tokens)) return keep_bits(keep, t, end, pool_tokens) | keep_bits(keep, t + 16, end, pool_tokens) << 16;
  const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(keep + t) & 3u) * 8u;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = __vcmpne4(__funnelshift_r(w[i], w[i + 1], shift), 0u) & 0x08040201u;
    bits |= ((m | m >> 8 | m >> 16 | m >> 24) & 15u) << (4 * i);
  }
  return t + 32 <= end ? bits : bits & ((1u << (int)(end - t)) - 1u);
}

// kept[r] of the request's resources, route_len[b * G + g].
__global__ void __launch_bounds__(COUNT_THREADS) pack8_count_kernel(const uint8_t* keep, const int32_t* res_off, const int32_t* res_slot,
                                                                    const int32_t* res_len, int total_listed, const uint8_t* vis, int G,
                                                                    int64_t pool_tokens, int32_t* kept, int32_t* route_len, int32_t* status) {
  rc_grid_wait();
  rc_grid_launch_next();
  const int b = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int a = res_off[b], e = res_off[b + 1];
  const bool ok = a >= 0 && e >= a && e <= total_listed;
  if (!ok && threadIdx.x == 0) rc_set_status(status, RECACHE_DEV_BAD_SEQLENS);
  if (ok) {
    for (int r = a + warp; r < e; r += COUNT_THREADS / 32) {
      const int64_t s0 = res_slot[r];
      const int n = res_len[r];
      int cnt = 0;
      if (n < 0 || s0 < 0 || s0 + n > pool_tokens) {
        if (lane == 0) rc_set_status(status, RECACHE_DEV_BAD_SLOT);
      } else {
        for (int j = lane * 16; j < n; j += 512) cnt += __popc(keep_bits(keep, s0 + j, s0 + n, pool_tokens));
      }
      cnt = __reduce_add_sync(0xffffffffu, cnt);
      if (lane == 0) kept[r] = cnt;
    }
  }
  __syncthreads();
  for (int g = warp; g < G; g += COUNT_THREADS / 32) {
    int sum = 0;
    if (ok) {
      for (int r = a + lane; r < e; r += 32) sum = rc_add_rows(sum, vis[(int64_t)g * total_listed + r] ? kept[r] : 0);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) sum = rc_add_rows(sum, __shfl_xor_sync(0xffffffffu, sum, off));
    if (lane == 0) route_len[(int64_t)b * G + g] = sum;
  }
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

struct PackParams {
  const void* k_cache; const void* v_cache; int64_t pool_tokens;
  const uint8_t* keep;
  const int32_t* res_off; const int32_t* res_slot; const int32_t* res_len; int total_listed;
  const uint8_t* vis; int G, n_routes;
  const int32_t* kept; const int32_t* route_len;
  int32_t* route_cu; int32_t* route_idx; int64_t row_capacity;
  int32_t* page_table; int max_pages;
  const int32_t* free_pages; int64_t n_free_pages; int64_t n_pool_pages;
  uint8_t* k8; uint8_t* v8; float* k_scale; float* v_scale;
  int32_t* status;
};
struct Page { int rows, page, group, first; };   // listed rows, page id (< 0: not to be packed), KV group, first row's place in the index list

template <typename T, int NV>   // NV: 16-byte pieces of the page's keys that a thread holds
__global__ void __launch_bounds__(WORKERS + 32 * LISTERS, NV <= 4 ? 2 : 1) pack8_pages_kernel(const __grid_constant__ PackParams p) {
  constexpr int N = 16 / sizeof(T), SEGS = NV * WORKERS / PT, D = SEGS * N;
  extern __shared__ __align__(16) uint8_t pieces[];          // two pages' pieces, each thread's its own
  __shared__ int rows_before[WORKERS + 1], pages_before[WORKERS + 1];     // of the run of routes that thread i counted
  __shared__ int sums[2][WORKERS / 32];
  __shared__ Page rings[LISTERS][RING];
  __shared__ int row_rings[LISTERS][RING * PT];              // pool rows of the rings' pages
  __shared__ uint32_t top[3][2][WORKERS / 32];
  __shared__ __align__(8) uint64_t bars[LISTERS][2 * RING];  // full, empty
  __shared__ volatile int abort_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t bar0 = (uint32_t)__cvta_generic_to_shared(bars);
  auto full = [&](int w, int i) { return bar0 + 8u * (uint32_t)(w * 2 * RING + i); };
  auto empty = [&](int w, int i) { return bar0 + 8u * (uint32_t)(w * 2 * RING + RING + i); };
  auto arrive = [](uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); };
  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < LISTERS * RING; ++i) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(full(i / RING, i % RING)) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(empty(i / RING, i % RING)), "r"(WORKERS / 32) : "memory");
    }
  }
  __syncthreads();                                           // no warp touches a barrier or the abort flag before they are set
  rc_grid_wait();
  rc_grid_launch_next();
  // ---- prefixes over the routes: a thread to a run of them ----
  const int per = (p.n_routes + WORKERS - 1) / WORKERS;
  {
    int rows = 0, pages = 0;
    const int i0 = min(p.n_routes, (int)threadIdx.x * per), i1 = threadIdx.x < WORKERS ? min(p.n_routes, i0 + per) : i0;
    for (int r = i0; r < i1; ++r) { const int n = p.route_len[r]; rows = rc_add_rows(rows, n); pages = add_pages(pages, pages_of(n)); }
    int ir = rows, ip = pages;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, ir, off), y = __shfl_up_sync(0xffffffffu, ip, off);
      if (lane >= off) { ir = rc_add_rows(ir, x); ip = add_pages(ip, y); }
    }
    int er = __shfl_up_sync(0xffffffffu, ir, 1), ep = __shfl_up_sync(0xffffffffu, ip, 1);    // of the lanes before (a sum that stopped cannot be taken back)
    if (lane == 0) er = ep = 0;
    if (lane == 31 && warp < WORKERS / 32) { sums[0][warp] = ir; sums[1][warp] = ip; }
    __syncthreads();
    if (threadIdx.x < WORKERS) {
      for (int w = 0; w < warp; ++w) { er = rc_add_rows(er, sums[0][w]); ep = add_pages(ep, sums[1][w]); }
      rows_before[threadIdx.x] = er; pages_before[threadIdx.x] = ep;
      ir = rc_add_rows(er, rows); ip = add_pages(ep, pages);
      if (threadIdx.x == WORKERS - 1) { rows_before[WORKERS] = ir; pages_before[WORKERS] = ip; }
      if (blockIdx.x == 0) {                                 // the prefix itself, once
        int at = er, page = ep;
        for (int r = i0; r < i1; ++r) {
          const int n = p.route_len[r], n_pages = pages_of(n);
          p.route_cu[r] = at;
          at = rc_add_rows(at, n);
          // (pages that have no number, which nobody below comes to)
          for (int x = MAX_PAGES - page; x < min(n_pages, p.max_pages); ++x) p.page_table[(int64_t)r * p.max_pages + x] = -1;
          page = add_pages(page, n_pages);
        }
        if (threadIdx.x == WORKERS - 1) {
          p.route_cu[p.n_routes] = ir;
          if (ir > p.row_capacity || ir == RC_MAX_ROWS) rc_set_status(p.status, RECACHE_DEV_OVERFLOW);
          if (ip > p.n_free_pages || ip == MAX_PAGES) rc_set_status(p.status, RECACHE_DEV_NO_PAGES);
        }
      }
    }
    __syncthreads();
  }
  // this block's pages; the first lister has the first half of them (the larger), the other the rest, and they are packed in turn
  const int total = pages_before[WORKERS];
  const int block_pi = (int)((int64_t)total * blockIdx.x / gridDim.x), n_pages = (int)((int64_t)total * (blockIdx.x + 1) / gridDim.x) - block_pi;

  if (warp >= WORKERS / 32) {
    // ===================== the rows of each page, in order =====================
    const int me = warp - WORKERS / 32;
    const int first_pi = block_pi + (me ? (n_pages + 1) / 2 : 0), end_pi = block_pi + (me ? n_pages : (n_pages + 1) / 2);
    Page* ring = rings[me];
    int* row_ring = row_rings[me];
    const uint32_t below = (1u << lane) - 1u;
    int n_out = 0, ids = -1;                                 // pages listed; a lane's entry of the free list, for 32 of them
    for (int pi = first_pi; pi < end_pi;) {
      // ---- the route that has page pi ----
      int j = 0;                                             // the run that holds it: the last with pages_before <= pi
#pragma unroll
      for (int i = 0; i < WORKERS / 32; ++i) j += pages_before[i * 32 + lane] <= pi;
      j = __reduce_add_sync(0xffffffffu, j) - 1;
      int base_p = pages_before[j], base_r = rows_before[j], route = -1, first_page = 0, first_row = 0, len = 0;
      for (int r0 = j * per; route < 0 && r0 < p.n_routes; r0 += 32) {
        const int n = r0 + lane < min(p.n_routes, (j + 1) * per) ? p.route_len[r0 + lane] : 0;
        int ip = pages_of(n), ir = n;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, ir, off), y = __shfl_up_sync(0xffffffffu, ip, off);
          if (lane >= off) { ir = rc_add_rows(ir, x); ip = add_pages(ip, y); }
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, add_pages(base_p, ip) > pi);
        int er = __shfl_up_sync(0xffffffffu, ir, 1);
        if (lane == 0) er = 0;
        if (hit) {
          const int l = __ffs(hit) - 1;
          route = r0 + l;
          len = __shfl_sync(0xffffffffu, n, l);
          first_page = base_p + __shfl_sync(0xffffffffu, ip, l) - pages_of(len);
          first_row = rc_add_rows(base_r, __shfl_sync(0xffffffffu, er, l));
        }
        base_p = add_pages(base_p, __shfl_sync(0xffffffffu, ip, 31)); base_r = rc_add_rows(base_r, __shfl_sync(0xffffffffu, ir, 31));
      }
      if (route < 0) break;                                  // (not with lengths that add up to the prefix)
      const int b = route / p.G, g = route % p.G;
      const int rank0 = (pi - first_page) * PT, rank1 = (int)min((int64_t)len, (int64_t)(end_pi - first_page) * PT);
      const int out0 = n_out;                                // the ring's page of rank0
      int lo = rank0, n_open = n_out;                        // ranks below lo are listed; pages below n_open may be written
      // the page of ranks lo .. lo + 63, with its first `rows` listed, goes to the packing warps
      auto close = [&](int rows) {
        if ((n_out & 31) == 0) ids = pi + lane < min((int64_t)end_pi, p.n_free_pages) ? p.free_pages[pi + lane] : -1;
        int page = __shfl_sync(0xffffffffu, ids, n_out & 31);
        if (lane == 0) {
          if (page < 0 || page >= p.n_pool_pages) {
            if (pi < p.n_free_pages) rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
            page = -1;
          }
          if (pi - first_page < p.max_pages) p.page_table[(int64_t)route * p.max_pages + pi - first_page] = page;
          else rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
          // (rows past the index list's capacity are left out, as the copying compaction leaves them out)
          const int64_t at = (int64_t)first_row + lo, in_list = max((int64_t)0, min((int64_t)rows, min(p.row_capacity, (int64_t)RC_MAX_ROWS) - at));
          *reinterpret_cast<int4*>(&ring[n_out % RING]) = make_int4((int)in_list, page, g, (int)at);
          arrive(full(me, n_out % RING));
        }
        ++n_out; ++pi;
        lo += PT;
      };
      auto open_to = [&](int n) {
        for (; n_open < n; ++n_open) rc_mbar_wait<WAIT_PROBES, RC_WHERE_PACK8>(empty(me, n_open % RING), ((n_open / RING) & 1) ^ 1, &abort_flag, p.status);
      };
      // ---- resources that the ranks fall into, 32 listed ones at a time ----
      const int a = p.res_off[b], e = p.res_off[b + 1];
      int before = 0;
      for (int i0 = a; i0 < e && lo < rank1; i0 += 32) {
        const int r = i0 + lane;
        const int has = r < e ? p.kept[r] : 0;               // (four loads at once)
        const int v = r < e && p.vis[(int64_t)g * p.total_listed + r] ? has : 0;
        const int64_t slot = r < e ? p.res_slot[r] : 0;
        const int n = r < e ? p.res_len[r] : 0;
        int incl = v;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, incl, off);
          if (lane >= off) incl = rc_add_rows(incl, x);
        }
        int excl = __shfl_up_sync(0xffffffffu, incl, 1);
        excl = rc_add_rows(before, lane == 0 ? 0 : excl);     // rank of the resource's first kept token
        before = rc_add_rows(before, __shfl_sync(0xffffffffu, incl, 31));
        uint32_t in = __ballot_sync(0xffffffffu, v > 0 && rc_add_rows(excl, v) > rank0 && excl < rank1);
        // 1024 mask tokens at a time, 32 a lane; the next ones' words are asked for before these are listed
        int l = __ffs(in) - 1, j0 = 0;
        uint32_t words[9];
        auto token = [&] { return __shfl_sync(0xffffffffu, slot, l) + j0 + lane * 32; };
        auto end = [&] { return __shfl_sync(0xffffffffu, slot, l) + __shfl_sync(0xffffffffu, n, l); };
        if (l >= 0) keep_words(p.keep, token(), end(), p.pool_tokens, words);
        int rank = l >= 0 ? __shfl_sync(0xffffffffu, excl, l) : 0;       // of the next kept token
        while (l >= 0 && lo < rank1) {
          const int64_t t = token();
          const uint32_t bits = keep_bits32(p.keep, t, end(), p.pool_tokens, words);
          int next_rank = rank;
          j0 += 1024;
          if (j0 >= __shfl_sync(0xffffffffu, n, l)) {
            in &= in - 1;
            l = __ffs(in) - 1; j0 = 0;
          }
          if (l >= 0) keep_words(p.keep, token(), end(), p.pool_tokens, words);
          const int cnt = __popc(bits);
          int upto = cnt;
#pragma unroll
          for (int off = 1; off < 32; off <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += x;
          }
          const int at = rank + upto - cnt;
          next_rank = rank + __shfl_sync(0xffffffffu, upto, 31);
          const int upper = min(next_rank, rank1);
          if (upper > lo) {
            open_to(out0 + (upper - rank0 + PT - 1) / PT);
            // a lane to each token of a lane's 32 in turn: kept tokens come in runs, of up to 32 in one lane's word
            const uint32_t some = __ballot_sync(0xffffffffu, bits && at < rank1 && at + cnt > rank0);
#pragma unroll 4
            for (int x = some ? __ffs(some) - 1 : 32; x < 32 - __clz(some); ++x) {
              const uint32_t word = __shfl_sync(0xffffffffu, bits, x);
              const int place = __shfl_sync(0xffffffffu, at, x) + __popc(word & below);
              if ((word >> lane & 1u) && place >= rank0 && place < rank1)
                row_ring[(out0 * PT + place - rank0) % (RING * PT)] = (int)t + (x - lane) * 32 + lane;
            }
            __syncwarp();
            while (lo < rank1 && min(lo + PT, rank1) <= upper) close(min(PT, rank1 - lo));
          }
          rank = l >= 0 && j0 == 0 ? __shfl_sync(0xffffffffu, excl, l) : next_rank;
        }
      }
      while (lo < rank1) {                                   // (only where the mask changed under the call: no rows)
        open_to(n_out + 1);
        close(0);
      }
    }
  } else {
    // ===================== eight warps: pages =====================
    {  // entries of the page table behind a route's pages
      const int64_t n = (int64_t)p.n_routes * p.max_pages;
      for (int64_t i = (int64_t)blockIdx.x * WORKERS + threadIdx.x; i < n; i += (int64_t)gridDim.x * WORKERS) {
        const int r = (int)(i / p.max_pages), at = (int)(i % p.max_pages);
        if (at >= pages_of(p.route_len[r])) p.page_table[i] = -1;
      }
    }
    const int c = threadIdx.x % SEGS, r0 = threadIdx.x / SEGS;
    constexpr int STEP = WORKERS / SEGS;
    // Pieces go to shared memory, to a place of the thread's own: a page is on its way while the one before is packed.
    const uint32_t hold = (uint32_t)__cvta_generic_to_shared(pieces) + threadIdx.x * 16;
    auto place = [&](int n, int i, int v) { return hold + (uint32_t)((((n & 1) * 2 + v) * NV + i) * WORKERS * 16); };
    int rows = 0, page = -1;
    auto fetch = [&](int n, int& rows, int& page) {
      const int w = n & 1, at = n >> 1, st = at % RING;      // (an odd page is the second lister's)
      rc_mbar_wait<WAIT_PROBES, RC_WHERE_PACK8>(full(w, st), (at / RING) & 1, &abort_flag, p.status);
      const int4 cur = *reinterpret_cast<const int4*>(&rings[w][st]);
      const int listed = abort_flag ? 0 : cur.x;             // (abort: a wait ran out, the page's rows are not there)
      const int* row = row_rings[w] + st * PT;
      page = cur.y;
      rows = page < 0 ? 0 : listed;
      const int64_t group = (int64_t)cur.z * p.pool_tokens;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int r = r0 + i * STEP;
        if (r < rows) {
          const int64_t from = (group + row[r]) * D + c * N;
          cp_async16(place(n, i, 0), (const T*)p.k_cache + from);
          cp_async16(place(n, i, 1), (const T*)p.v_cache + from);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (threadIdx.x < listed) p.route_idx[cur.w + threadIdx.x] = row[threadIdx.x];
      __syncwarp();
      if (lane == 0) arrive(empty(w, st));                   // the listed rows have been read
    };
    if (n_pages > 0) fetch(0, rows, page);
    for (int n = 0; n < n_pages; ++n) {
      int next_rows = 0, next_page = -1;
      if (n + 1 < n_pages) {
        fetch(n + 1, next_rows, next_page);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      uint4 kx[NV], vx[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (r0 + i * STEP < rows) { kx[i] = lds16(place(n, i, 0)); vx[i] = lds16(place(n, i, 1)); }
      // the maxima: of all values first, and only where that is no finite number of the finite ones
      uint32_t mk = 0, mv = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (r0 + i * STEP < rows) { mk = top_of<T>(kx[i], mk); mv = top_of<T>(vx[i], mv); }
      auto block_max = [&](int at) {
        mk = __reduce_max_sync(0xffffffffu, mk); mv = __reduce_max_sync(0xffffffffu, mv);
        if (lane == 0) { top[at][0][warp] = mk; top[at][1][warp] = mv; }
        asm volatile("bar.sync 1, %0;" ::"n"(WORKERS) : "memory");
#pragma unroll
        for (int w = 0; w < WORKERS / 32; ++w) { mk = max(mk, top[at][0][w]); mv = max(mv, top[at][1][w]); }
      };
      mk = top_bits<T>(mk); mv = top_bits<T>(mv);
      block_max(n & 1);
      const bool odd = max(mk, mv) >= 0x7f800000u;           // (alike in all threads)
      if (odd) {
        mk = mv = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (r0 + i * STEP < rows) {
            float f[N];
            load16<T>(kx[i], f);
#pragma unroll
            for (int j = 0; j < N; ++j) mk = max(mk, mag_bits(f[j]));
            load16<T>(vx[i], f);
#pragma unroll
            for (int j = 0; j < N; ++j) mv = max(mv, mag_bits(f[j]));
          }
        }
        block_max(2);
        asm volatile("bar.sync 1, %0;" ::"n"(WORKERS) : "memory");          // (the next such page may be the next one)
      }
      const int ek = scale_exponent(mk), ev = scale_exponent(mv);
      if (threadIdx.x == 0 && rows > 0) { p.k_scale[page] = power(ek); p.v_scale[page] = power(ev); }
      const uint32_t ik = __float_as_uint(power(-ek)), iv = __float_as_uint(power(-ev));
      const uint32_t ik2 = sizeof(T) == 2 ? ik | ik >> 16 : ik, iv2 = sizeof(T) == 2 ? iv | iv >> 16 : iv;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int r = r0 + i * STEP;
        if (r < rows) {
          const int64_t to = ((int64_t)page * PT + r) * D + c * N;
          if (!odd) {
            store8_finite<T>(p.k8 + to, kx[i], ik2);
            store8_finite<T>(p.v8 + to, vx[i], iv2);
          } else {
            store8<T>(p.k8 + to, kx[i], __uint_as_float(ik));
            store8<T>(p.v8 + to, vx[i], __uint_as_float(iv));
          }
        }
      }
      rows = next_rows; page = next_page;
    }
  }
}

}  // namespace

static cudaError_t launch_pages(const recache_ctx* ctx, const Pack8Args& a, cudaStream_t st) {
  const int G = ctx->desc.n_kv_heads, sms = ctx->sm_count > 0 ? ctx->sm_count : 148;
  int32_t* kept = (int32_t*)a.c.workspace;
  int32_t* len = a.c.route_len ? a.c.route_len : (int32_t*)((uint8_t*)a.c.workspace + ((int64_t)a.c.total_listed * 4 + 255) / 256 * 256);
  if (a.c.n_requests > 0) {
    RcLaunchScope scope(ctx, RC_K_COMPACT_COUNT, st);
    const cudaError_t e = rc_launch_overlapped(pack8_count_kernel, a.c.n_requests, COUNT_THREADS, 0, st, a.c.keep, a.c.res_off, a.c.res_slot, a.c.res_len,
                                               a.c.total_listed, a.c.vis, G, a.c.pool_tokens, kept, len, ctx->status);
    if (e != cudaSuccess) return e;
  }
  PackParams p{a.c.k_cache, a.c.v_cache, a.c.pool_tokens, a.c.keep, a.c.res_off, a.c.res_slot, a.c.res_len, a.c.total_listed, a.c.vis, G,
               a.c.n_requests * G, kept, len, a.c.route_cu, a.c.route_idx, a.c.row_capacity, a.c.page_table, a.c.max_pages_per_route, a.c.free_pages,
               a.c.n_free_pages, a.c.n_pool_pages, a.k8, a.v8, a.k_scale, a.v_scale, ctx->status};
  const int64_t most = (int64_t)p.n_routes * p.max_pages;
  RcLaunchScope scope(ctx, RC_K_COMPACT_PACK8, st);
  auto launch = [&](auto kernel, int per_sm) {
    const int64_t wave = (int64_t)per_sm * sms;
    const size_t two_pages = 2 * 2 * (size_t)PT * ctx->desc.head_dim * (ctx->desc.dtype == RECACHE_BF16 ? 2 : 4);
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)two_pages);   // (with the rings over 48 KB)
    if (e != cudaSuccess) return e;
    return rc_launch_overlapped(kernel, (unsigned)(most < 1 ? 1 : most < wave ? most : wave), WORKERS + 32 * LISTERS, two_pages, st, p);
  };
  if (ctx->desc.dtype == RECACHE_BF16)
    return ctx->desc.head_dim == 64 ? launch(pack8_pages_kernel<__nv_bfloat16, 2>, 2) : launch(pack8_pages_kernel<__nv_bfloat16, 4>, 2);
  return ctx->desc.head_dim == 64 ? launch(pack8_pages_kernel<float, 4>, 2) : launch(pack8_pages_kernel<float, 8>, 1);
}

cudaError_t rc_launch_pack8(const recache_ctx* ctx, const Pack8Args& a, cudaStream_t st) {
  if (ctx->desc.page_tokens == PT) return launch_pages(ctx, a, st);
  cudaError_t e = rc_launch_compact(ctx, a.c, st);
  if (e != cudaSuccess || a.c.total_listed == 0 || a.c.n_requests == 0) return e;
  const int G = ctx->desc.n_kv_heads, n_routes = a.c.n_requests * G;
  const int32_t* page_cu = rc_compact_page_cu(ctx, a.c);
  const int64_t most = 2 * (int64_t)n_routes * a.c.max_pages_per_route, wave = 8 * (int64_t)(ctx->sm_count > 0 ? ctx->sm_count : 148);
  const unsigned blocks = (unsigned)(most < wave ? most : wave);
  RcLaunchScope scope(ctx, RC_K_COMPACT_PACK8, st);
  auto launch = [&](auto type) {
    using T = decltype(type);
    return rc_launch_overlapped(pack8_kernel<T>, blocks, TPB, 0, st, (const T*)a.c.k_cache, (const T*)a.c.v_cache, a.c.pool_tokens,
                                (const int32_t*)a.c.route_cu, (const int32_t*)a.c.route_idx, a.c.row_capacity, page_cu, n_routes, G, ctx->desc.head_dim,
                                ctx->desc.page_tokens, a.c.free_pages, a.c.n_free_pages, a.c.n_pool_pages, a.k8, a.v8, a.k_scale, a.v_scale,
                                ctx->status);
  };
  return ctx->desc.dtype == RECACHE_BF16 ? launch(__nv_bfloat16()) : launch(float());
}
