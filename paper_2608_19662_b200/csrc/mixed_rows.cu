// Decode over two kinds of pages, fp32 arithmetic, any supported shape: the first part of an item lies in 8-bit pages with a
// scale each, or in pages of the storage type like its history; with weights, every row's softmax probability, summed over
// the group's heads, is added to the row's weight.
//
// A block per item (sequence, KV head), all of the group's query heads at once, so that a row is read once.
// Each of 8 warps takes 32 rows at a time: a lane per row for the scores, then the lanes side by side along the row
// for P V, with a running maximum and sum per head; the warps' parts are merged through shared memory.  The scores go to the
// workspace where weights are wanted, and the same block turns them into probabilities once maximum and sum are known.
// The item's current token is appended by the block before it reads.  Not a throughput path: 64 sequences of 4096
// 8-bit and 1024 bf16 rows took 1499 us here, 124-134 in mixed_split.cu; with 64 elements a row, which come here, 964.
#include "common.cuh"

namespace {

constexpr int WARPS = 8;
constexpr int MAX_S = 8;                    // query heads of a group

struct RowsParams {
  MixedArgs a;
  int Hq, G, s, page_tokens, max_pos;
  const float* cos_tab; const float* sin_tab;
  float scale;
  float* score;                             // [n_pages][page_tokens][s]
  int32_t* status;
};

template <typename T, int N> __device__ __forceinline__ void load_n(const T* p, float* f) {
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = rc_to_float<T>(p[i]);
}
template <int N> __device__ __forceinline__ void load_n8(const uint8_t* p, float* f) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const uint32_t h = rc_e4m3x2_to_f16x2(*reinterpret_cast<const uint16_t*>(p + i));
    float lo, hi;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
    f[i] = lo; f[i + 1] = hi;
  }
}

template <typename T, typename TO, int D>
__global__ void __launch_bounds__(WARPS * 32) mixed_rows_kernel(const __grid_constant__ RowsParams p) {
  constexpr int HALF = D / 2, CPL = D / 32;
  __shared__ float q_s[MAX_S][D];
  __shared__ float part[WARPS][MAX_S][2 + D];
  __shared__ float2 done[MAX_S];            // maximum, 1 / sum
  const MixedArgs& a = p.a;
  const int it = blockIdx.x, b = it / p.G, g = it % p.G, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, s = p.s, pt = p.page_tokens;
  rc_grid_wait();
  rc_grid_launch_next();
  const int pos = a.q_pos[b];
  const bool pos_ok = pos >= 0 && pos < p.max_pos;
  const int64_t tab = (int64_t)(pos_ok ? pos : 0) * HALF;
  const int n_res = min((int64_t)max(a.res_len[it], 0), (int64_t)a.max_res_pages * pt), n_hist = min((int64_t)max(a.hist_len[it], 0), (int64_t)a.max_hist_pages * pt);
  if (threadIdx.x == 0) {
    if (!pos_ok) rc_set_status(p.status, RECACHE_DEV_BAD_POS);
    if (a.hist_len[it] < 1 || n_hist != a.hist_len[it] || n_res != max(a.res_len[it], 0)) rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
  }
  const int32_t* res_pt = a.res_pt + (int64_t)it * a.max_res_pages;
  const int32_t* hist_pt = a.hist_pt + (int64_t)it * a.max_hist_pages;
  const T* kp = (const T*)a.k_pages;
  const T* vp = (const T*)a.v_pages;
  // pool row of row r of a part, -1 where its page is none
  auto row_of = [&](bool res, int r) -> int64_t {
    const int pg = (res ? res_pt : hist_pt)[r / pt];
    return pg < 0 || pg >= (res && a.k8 ? a.n_pages8 : a.n_pages) ? -1 : (int64_t)pg * pt + r % pt;
  };
  // ---- the current token, and the queries: rotated, tensors of the storage type ----
  const int64_t new_row = a.k_new && n_hist > 0 && n_hist == a.hist_len[it] && pos_ok ? row_of(false, n_hist - 1) : -1;
  if (new_row >= 0) {
    T* kd = (T*)a.k_pages + new_row * D;
    T* vd = (T*)a.v_pages + new_row * D;
    const T* ks = (const T*)a.k_new + (int64_t)it * D;
    const T* vs = (const T*)a.v_new + (int64_t)it * D;
    for (int i = threadIdx.x; i < HALF; i += WARPS * 32) {
      const float lo = rc_to_float<T>(ks[i]), hi = rc_to_float<T>(ks[i + HALF]), c = p.cos_tab[tab + i], sn = p.sin_tab[tab + i];
      kd[i] = rc_from_float<T>(__fmaf_rn(lo, c, -__fmul_rn(hi, sn)));
      kd[i + HALF] = rc_from_float<T>(__fmaf_rn(hi, c, __fmul_rn(lo, sn)));
      vd[i] = vs[i]; vd[i + HALF] = vs[i + HALF];
    }
  }
  for (int e = threadIdx.x; e < s * HALF; e += WARPS * 32) {
    const int h = e / HALF, i = e % HALF;
    const T* qr = (const T*)a.q + ((int64_t)b * p.Hq + g * s + h) * D;
    const float lo = rc_to_float<T>(qr[i]), hi = rc_to_float<T>(qr[i + HALF]), c = p.cos_tab[tab + i], sn = p.sin_tab[tab + i];
    q_s[h][i] = rc_to_float<T>(rc_from_float<T>(__fmaf_rn(lo, c, -__fmul_rn(hi, sn))));
    q_s[h][i + HALF] = rc_to_float<T>(rc_from_float<T>(__fmaf_rn(hi, c, __fmul_rn(lo, sn))));
  }
  __syncthreads();

  float m[MAX_S], l[MAX_S], acc[MAX_S][CPL];
#pragma unroll
  for (int h = 0; h < MAX_S; ++h) {
    m[h] = -INFINITY; l[h] = 0.f;
#pragma unroll
    for (int c = 0; c < CPL; ++c) acc[h][c] = 0.f;
  }
  bool bad = false;
  for (int seg = 0; seg < 2; ++seg) {
    const bool res = seg == 0, q8 = res && a.k8;
    const int n = res ? n_res : n_hist;
    for (int k0 = warp * 32; k0 < n; k0 += WARPS * 32) {
      const int r = k0 + lane;
      int64_t mine = -1;
      if (r < n) {
        mine = row_of(res, r);
        bad |= mine < 0;
      }
      float sc[MAX_S];
#pragma unroll
      for (int h = 0; h < MAX_S; ++h) sc[h] = 0.f;
      float v_scale = 1.f;
      if (mine >= 0) {
        constexpr int N = 4;
        for (int i = 0; i < D; i += N) {
          float f[N];
          if (q8) load_n8<N>(a.k8 + mine * D + i, f);
          else load_n<T, N>(kp + mine * D + i, f);
#pragma unroll
          for (int h = 0; h < MAX_S; ++h) {
            if (h < s) {
#pragma unroll
              for (int j = 0; j < N; ++j) sc[h] = fmaf(f[j], q_s[h][i + j], sc[h]);
            }
          }
        }
        const float f = q8 ? a.k_scale[mine / pt] * p.scale : p.scale;
        if (q8) v_scale = a.v_scale[mine / pt];
#pragma unroll
        for (int h = 0; h < MAX_S; ++h) {
          sc[h] *= f;
          if (a.weight_out && !q8 && h < s) p.score[mine * s + h] = sc[h];
        }
      }
      float pr[MAX_S];
#pragma unroll
      for (int h = 0; h < MAX_S; ++h) {
        if (h >= s) break;
        float mx = mine >= 0 ? sc[h] : -INFINITY;
#pragma unroll
        for (int off = 16; off; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        const float m_new = fmaxf(m[h], mx), m_use = m_new == -INFINITY ? 0.f : m_new;
        const float corr = m[h] == -INFINITY ? 0.f : expf(m[h] - m_use);
        pr[h] = mine >= 0 ? expf(sc[h] - m_use) : 0.f;
        l[h] = l[h] * corr + pr[h];                       // a lane's own rows; summed at the end
        m[h] = m_new;
#pragma unroll
        for (int c = 0; c < CPL; ++c) acc[h][c] *= corr;
      }
      const int cnt = min(32, n - k0);
      for (int j = 0; j < cnt; ++j) {
        const int64_t vr = __shfl_sync(0xffffffffu, mine, j);
        const float vs = __shfl_sync(0xffffffffu, v_scale, j);
        if (vr < 0) continue;
        float f[CPL];
        if (q8) load_n8<CPL>(a.v8 + vr * D + lane * CPL, f);
        else load_n<T, CPL>(vp + vr * D + lane * CPL, f);
#pragma unroll
        for (int h = 0; h < MAX_S; ++h) {
          if (h >= s) break;
          const float ph = __shfl_sync(0xffffffffu, pr[h], j) * vs;
#pragma unroll
          for (int c = 0; c < CPL; ++c) acc[h][c] = fmaf(ph, f[c], acc[h][c]);
        }
      }
    }
  }
  if (bad) rc_set_status(p.status, RECACHE_DEV_BAD_PAGE);
#pragma unroll
  for (int h = 0; h < MAX_S; ++h) {
    if (h >= s) break;
#pragma unroll
    for (int off = 16; off; off >>= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], off);
    if (lane == 0) { part[warp][h][0] = m[h]; part[warp][h][1] = l[h]; }
#pragma unroll
    for (int c = 0; c < CPL; ++c) part[warp][h][2 + lane * CPL + c] = acc[h][c];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < s * D; e += WARPS * 32) {
    const int h = e / D, i = e % D;
    float M = -INFINITY, L = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) M = fmaxf(M, part[w][h][0]);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = part[w][h][0] == -INFINITY ? 0.f : expf(part[w][h][0] - M);
      L += part[w][h][1] * f;
      o += part[w][h][2 + i] * f;
    }
    const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
    if (i == 0) done[h] = make_float2(M, inv);
    reinterpret_cast<TO*>(a.o)[((int64_t)b * p.Hq + g * s + h) * D + i] = rc_from_float<TO>(o * inv);
  }
  if (!a.weight_out) return;
  __syncthreads();
  const int first = a.k8 ? n_res : 0;                      // 8-bit rows have no weight
  for (int r = first + threadIdx.x; r < n_res + n_hist; r += WARPS * 32) {
    const int64_t row = r < n_res ? row_of(true, r) : row_of(false, r - n_res);
    if (row < 0) continue;
    float w = a.weight_in && row != new_row ? a.weight_in[row] : 0.f;   // a token that was just appended has none yet
    for (int h = 0; h < s; ++h) w += done[h].x == -INFINITY ? 0.f : expf(p.score[row * s + h] - done[h].x) * done[h].y;
    a.weight_out[row] = w;
  }
}

}  // namespace

int64_t rc_mixed_rows_workspace_bytes(const recache_ctx* ctx, int64_t n_pages) {
  return n_pages * ctx->desc.page_tokens * (ctx->desc.n_q_heads / ctx->desc.n_kv_heads) * 4;
}

cudaError_t rc_launch_mixed_rows(const recache_ctx* ctx, const MixedArgs& a, cudaStream_t st) {
  const recache_desc& d = ctx->desc;
  RowsParams p{a, d.n_q_heads, d.n_kv_heads, d.n_q_heads / d.n_kv_heads, d.page_tokens, d.max_pos, ctx->cos_tab, ctx->sin_tab,
               (float)(1.0 / sqrt((double)d.head_dim)), (float*)a.workspace, ctx->status};
  RcLaunchScope scope(ctx, RC_K_MIXED_ATTN, st);
  auto launch = [&](auto kernel) { return rc_launch_overlapped(kernel, a.batch * d.n_kv_heads, WARPS * 32, 0, st, p); };
  if (d.dtype == RECACHE_F32) return d.head_dim == 64 ? launch(mixed_rows_kernel<float, float, 64>) : launch(mixed_rows_kernel<float, float, 128>);
  if (a.out_dtype == RECACHE_F32)
    return d.head_dim == 64 ? launch(mixed_rows_kernel<__nv_bfloat16, float, 64>) : launch(mixed_rows_kernel<__nv_bfloat16, float, 128>);
  return d.head_dim == 64 ? launch(mixed_rows_kernel<__nv_bfloat16, __nv_bfloat16, 64>) : launch(mixed_rows_kernel<__nv_bfloat16, __nv_bfloat16, 128>);
}
