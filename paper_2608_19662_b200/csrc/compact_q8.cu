// Compaction into 8-bit pages: the rows that paged compaction would copy, as e4m3 values with one
// power-of-two scale for a page's keys and one for its values.
//
// The count, plan and gather launches of the compaction come first, without a row copied: they leave the
// index list, the page prefix and the page table.  Then a block takes a page's keys or its values: it loads the rows
// through the index list, finds the largest finite magnitude m and stores every value divided by
//     scale = 2^e,   e = the least integer >= -126 with m <= 448 2^e          (1 where m = 0)
// rounded to the nearest e4m3 value (ties to even).  A power of two makes the division exact, so that a value is rounded
// once, and costs e4m3 nothing: its relative precision is the same all over its range.
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

template <typename T>
__global__ void __launch_bounds__(TPB) pack8_kernel(const T* k_cache, const T* v_cache, int64_t pool_tokens, const int32_t* route_cu,
                                                    const int32_t* route_idx, int64_t row_capacity, const int32_t* page_cu, int n_routes, int G,
                                                    int d, int page_tokens, const int32_t* free_pages, int64_t n_free_pages, int64_t n_pool_pages,
                                                    uint8_t* k8, uint8_t* v8, float* k_scale, float* v_scale, int32_t* status) {
  constexpr int N = 16 / sizeof(T);
  __shared__ uint32_t top;
  rc_grid_wait();
  rc_grid_launch_next();
  const int total = 2 * page_cu[n_routes];
  const int segs = d / N;
  for (int w = blockIdx.x; w < total; w += gridDim.x) {
    const int pi = w >> 1;
    if (pi >= n_free_pages) break;                       // flagged by the plan
    const int pg = free_pages[pi];
    if (pg < 0 || pg >= n_pool_pages) continue;          // flagged by the plan
    const int route = rc_find_segment(page_cu, n_routes, pi);
    const int64_t first = (int64_t)route_cu[route] + (int64_t)(pi - page_cu[route]) * page_tokens;
    // (an index past the list's capacity was never written)
    const int64_t last = min((int64_t)route_cu[route + 1], row_capacity);
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
    // top = 2^(x - 127) * 1.f; it fits 448 * 2^e = 1.75 * 2^(8 + e) from e = x - 127 - 8 on, or one later where 1.f > 1.75
    const int x = (int)(top >> 23);
    const int e2 = top == 0 ? 0 : max(-126, x - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0));
    const float scale = __uint_as_float((uint32_t)(e2 + 127) << 23), inv = __uint_as_float((uint32_t)(127 - e2) << 23);
    if (threadIdx.x == 0) ((w & 1) ? v_scale : k_scale)[pg] = scale;
    for (int e = threadIdx.x; e < rows * segs; e += TPB) {
      const int r = e / segs, c = e - r * segs;
      float f[N];
      load16<T>(*reinterpret_cast<const uint4*>(src + (int64_t)route_idx[first + r] * d + c * N), f);
      uint32_t o[N / 4];
#pragma unroll
      for (int i = 0; i < N; i += 4) o[i / 4] = to_e4m3x2(f[i], f[i + 1], inv) | to_e4m3x2(f[i + 2], f[i + 3], inv) << 16;
      uint8_t* to = dst + (int64_t)r * d + c * N;
      if constexpr (N == 8) *reinterpret_cast<uint2*>(to) = make_uint2(o[0], o[1]);
      else *reinterpret_cast<uint32_t*>(to) = o[0];
    }
  }
}

}  // namespace

cudaError_t rc_launch_pack8(const recache_ctx* ctx, const Pack8Args& a, cudaStream_t st) {
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
