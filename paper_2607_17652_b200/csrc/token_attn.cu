// fb_token_attn: one query token per request over everything its pages hold, in its simplest form: a CTA per
// (request, KV head), the group's query heads one after the other, a key a warp at a time; with weights a
// second sweep forms the scores again once the sum is known.
#include <cuda_fp8.h>

#include "fb_common.cuh"

namespace fb {

struct TokenParams {
  const int32_t *kv_len, *page_table;
  float* kv_weight;                 // null: not accumulated
  const __nv_bfloat16* q;
  const void *k_pool, *v_pool;
  const float *k_scale, *v_scale;   // 8-bit pages
  __nv_bfloat16* out;
  int32_t* status;
  int32_t group, n_kv_heads, head_dim, max_pages_per_req, num_pages;
  float sm_scale;
};

template <bool F8>
__global__ void __launch_bounds__(128) token_attn_kernel(const TokenParams p) {
  pdl_wait();
  __shared__ float sh_m[4], sh_l[4], sh_o[4][128], top[kTileM], sum[kTileM];   // (a group has at most 128 heads)
  const int r = blockIdx.x, h = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = p.head_dim;
  const int len = p.kv_len[r];
  const long long cap = (long long)p.max_pages_per_req * kPage;
  if (len < 0) return;
  if (len > cap) { if (threadIdx.x == 0) atomicOr(p.status, FB_ST_BAD_STATE); return; }
  const float ks = F8 ? p.k_scale[h] : 1.f, vs = F8 ? p.v_scale[h] : 1.f;
  const int per = d / 32;
  // the row of key j, or -1 where its page is outside the pool
  auto row = [&](int j) -> long long {
    const int page = p.page_table[(size_t)r * p.max_pages_per_req + j / kPage];
    if (page < 0 || page >= p.num_pages) return -1;
    return (((long long)page * p.n_kv_heads + h) * kPage + j % kPage) * d;
  };
  auto value = [&](const void* pool, long long at) {
    if constexpr (F8) return (float)static_cast<const __nv_fp8_e4m3*>(pool)[at];
    else return __bfloat162float(static_cast<const __nv_bfloat16*>(pool)[at]);
  };
  const size_t head0 = ((size_t)r * p.n_kv_heads + h) * p.group;
  auto score = [&](int g, long long at) {
    float s = 0.f;
    for (int e = 0; e < per; ++e)
      s += __bfloat162float(p.q[(head0 + g) * d + lane * per + e]) * value(p.k_pool, at + lane * per + e);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s * ks * p.sm_scale;
  };
  for (int g = 0; g < p.group; ++g) {
    float m = -INFINITY, l = 0.f, acc[4] = {};
    for (int j = warp; j < len; j += 4) {
      const long long at = row(j);
      if (at < 0) { if (lane == 0) atomicOr(p.status, FB_ST_BAD_PAGE); continue; }
      const float s = score(g, at), mn = fmaxf(m, s), f = expf(m - mn), w = expf(s - mn);
      l = l * f + w;
      for (int e = 0; e < per; ++e) acc[e] = acc[e] * f + w * value(p.v_pool, at + lane * per + e);
      m = mn;
    }
    if (lane == 0) { sh_m[warp] = m; sh_l[warp] = l; }
    for (int e = 0; e < per; ++e) sh_o[warp][lane * per + e] = acc[e];
    __syncthreads();
    float M = -INFINITY, L = 0.f, f[4];
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sh_m[w]);
    for (int w = 0; w < 4; ++w) { f[w] = sh_m[w] == -INFINITY ? 0.f : expf(sh_m[w] - M); L += sh_l[w] * f[w]; }
    if ((int)threadIdx.x < d) {
      float o = 0.f;
      for (int w = 0; w < 4; ++w) o += sh_o[w][threadIdx.x] * f[w];
      p.out[(head0 + g) * d + threadIdx.x] = __float2bfloat16_rn(L > 0.f || L != L ? o / L * vs : 0.f);
    }
    if (threadIdx.x == 0) { top[g] = M; sum[g] = L; }
    __syncthreads();
  }
  if (!p.kv_weight) return;
  for (int j = warp; j < len; j += 4) {
    const long long at = row(j);
    if (at < 0) continue;
    float w = 0.f;
    for (int g = 0; g < p.group; ++g) w += expf(score(g, at) - top[g]) / sum[g];
    if (lane == 0) p.kv_weight[((size_t)r * p.n_kv_heads + h) * cap + j] += w;
  }
}

size_t token_workspace_bytes(const fb_ctx*, bool) { return 256; }

int launch_token_attn(fb_ctx* ctx, const fb_cache* kv, const void* q, const void* k_pool, const void* v_pool,
                      const float* k_scale, const float* v_scale, void* out, int accumulate, void*, int32_t* status,
                      cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  TokenParams p;
  p.kv_len = kv->kv_len; p.page_table = kv->page_table; p.kv_weight = accumulate ? kv->kv_weight : nullptr;
  p.q = static_cast<const __nv_bfloat16*>(q); p.k_pool = k_pool; p.v_pool = v_pool;
  p.k_scale = k_scale; p.v_scale = v_scale; p.out = static_cast<__nv_bfloat16*>(out); p.status = status;
  p.group = ctx->group; p.n_kv_heads = c.n_kv_heads; p.head_dim = c.head_dim;
  p.max_pages_per_req = c.max_pages_per_req; p.num_pages = c.num_pages; p.sm_scale = ctx->sm_scale;
  const dim3 grid(c.max_requests, c.n_kv_heads);
  const auto kernel = c.kv_fp8 ? token_attn_kernel<true> : token_attn_kernel<false>;
  return cuda_err(ctx, launch_pdl(kernel, grid, 128, 0, stream, p), "token_attn_kernel launch");
}

}  // namespace fb
