// Data movement either side of the packed forward: fb_embed_gather and fb_append_kv (at the end of
// this file) and
// fb_scatter_window_kv: Eq. 6 as data movement.  The fresh K/V rows of every
// live window position go to the request's pages at their absolute positions
// (all KV heads), optionally with the rotary embedding applied to the keys.
// HBM-bound: 2 x rows x Hkv x d x 2 bytes read and as many written.
//
// Several CTAs per slot, the slot's tokens dealt among them so that a thread has one work item
// (launch_scatter).  For a (token, head) the head_dim elements are contiguous in the source
// (slot-order rows) and in the destination (pool row of that position), so a thread moves 16-byte
// pieces: with the rotary embedding it owns the two pieces that hold elements i and i + d/2 of
// eight pairs, and the rotation angles come from a table in shared memory, built while the
// loads of the item are in flight.
// Small batches are bound by the chain of dependent loads, large ones by bandwidth and by the
// table's arithmetic.  Call in us, former form (256 threads, four CTAs a slot, loads behind the
// table) -> this one: 1 request 4.8 -> 2.5, 8 requests 4.3 -> 3.9, 128 requests 18.6 -> 14.5
// (84 MB: 5.8 TB/s), 64 requests into 8-bit pages 14.3 -> 11.9, 16 long contexts 20.8 -> 8.4.
#include <cuda_fp8.h>

#include <cmath>
#include <cstring>

#include "fb_common.cuh"

namespace fb {

constexpr int kScatterThreads = 128;

struct ScatterParams {
  const int32_t* n_live; const int32_t* slot_req; const int32_t* slot_pos0;
  const int32_t* page_table;
  const uint4 *k_new, *v_new;
  uint4 *k_pool, *v_pool;
  int32_t* status;
  int32_t bl, n_kv_heads, head_dim, max_pages_per_req, num_pages;
  float rope_base;
  const float *k_scale, *v_scale;   // 8-bit pages: [n_kv_heads]
  double inv_freq[64];              // rope_base^(-2k/d), k < d/2 (formed on the host in fp64)
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// stored byte of x under `scale`: the binary32 quotient, rounded to nearest even onto the E4M3
// grid, saturating at +-448
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d, float scale) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(a, scale), __fdiv_rn(b, scale)), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(c, scale), __fdiv_rn(d, scale)), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}
// eight bf16 (one 16-byte piece) -> eight E4M3 bytes
__device__ __forceinline__ uint2 quant8(const uint4 v, float scale) {
  return make_uint2(e4m3x4(bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y), scale),
                    e4m3x4(bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w), scale));
}

// Cosine and sine of the angle pos * inv_freq: formed and reduced to [-pi, pi] in fp64 (positions reach tens
// of thousands of radians), sine and cosine of the remainder in fp32.
__device__ __forceinline__ float2 rope_cos_sin(int pos, double inv_freq) {
  const double ang = (double)pos * inv_freq;
  const double red = fma(-rint(ang * 0.15915494309189535), 6.283185307179586, ang);
  float sf, cf;
  sincosf((float)red, &sf, &cf);
  return make_float2(cf, sf);
}
// Eight pairs of a head turned: elements i0.. (a) and i0 + d/2.. (b) by the angles whose cosine and sine
// stand in cs[0..8).
__device__ __forceinline__ void rotate8(const uint4 a, const uint4 b, const float2* cs, float lo[8], float hi[8]) {
  const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 p = cs[2 * k], q = cs[2 * k + 1];
    const float x0 = bf16_lo(aw[k]), x1 = bf16_hi(aw[k]), y0 = bf16_lo(bw[k]), y1 = bf16_hi(bw[k]);
    lo[2 * k] = x0 * p.x - y0 * p.y; lo[2 * k + 1] = x1 * q.x - y1 * q.y;
    hi[2 * k] = y0 * p.x + x0 * p.y; hi[2 * k + 1] = y1 * q.x + x1 * q.y;
  }
}

// F8: the pools hold E4M3 bytes (8-byte pieces instead of 16-byte ones), each value divided by
// the scale of its KV head before it is rounded.
template <bool F8>
__global__ void __launch_bounds__(kScatterThreads) scatter_window_kv_kernel(const ScatterParams p) {
  pdl_wait();
  const int slot = blockIdx.x;
  const int n_live = *p.n_live, r = p.slot_req[slot], pos0 = p.slot_pos0[slot];      // (together: one latency)
  if (slot >= n_live) return;
  const int vph = p.head_dim / 8;                    // 16-byte pieces per (token, head)
  const int vpt = p.n_kv_heads * vph;                // ... per token
  const bool rope = p.rope_base > 0.f;
  // cos / sin of pos * base^(-2i/d), once per (token, pair) and shared by all KV heads, for
  // 32 tokens of the slot at a time
  constexpr int kTokBatch = 32;
  __shared__ float2 cs[kTokBatch * 64];              // [token of the batch][pair] (cos, sin), d/2 <= 64
  const int half = p.head_dim / 2;
  // work item = (token, head, piece); with the rotary embedding only the lower half of the
  // pieces is enumerated and each item also handles its partner piece + d/16
  const int per_head = rope ? vph / 2 : vph, partner = rope ? vph / 2 : 0;
  // the slot's tokens are dealt to the gridDim.y CTAs of the slot (each builds the table of its
  // own tokens only)
  const int tpc = (p.bl + (int)gridDim.y - 1) / (int)gridDim.y;
  const int tbeg = (int)blockIdx.y * tpc, tend = min(p.bl, tbeg + tpc);
  const int nh = p.n_kv_heads;
  for (int t0 = tbeg; t0 < tend; t0 += kTokBatch) {
    const int nt = min(kTokBatch, tend - t0), total = nt * nh * per_head;
    for (int i = threadIdx.x; i < (total + kScatterThreads - 1) / kScatterThreads * kScatterThreads; i += kScatterThreads) {
      // the loads first: source rows and page id do not depend on the table
      const int tb = i / (nh * per_head), rem = i % (nh * per_head), h = rem / per_head, v = rem % per_head;
      const int pos = pos0 + t0 + tb;
      uint4 ka, kb, va, vb;
      int page = -1;
      if (i < total) {
        const size_t src = (size_t)(slot * p.bl + t0 + tb) * vpt + h * vph + v;
        if (pos / kPage < p.max_pages_per_req) page = p.page_table[(size_t)r * p.max_pages_per_req + pos / kPage];
        ka = p.k_new[src]; va = p.v_new[src];
        if (rope) { kb = p.k_new[src + partner]; vb = p.v_new[src + partner]; }
      }
      if (rope && i < kScatterThreads) {             // (uniform: the first pass of the batch)
        if (t0 != tbeg) __syncthreads();             // the previous batch has been read
        for (int e = threadIdx.x; e < nt * half; e += kScatterThreads) {
          const int t = e / half, k = e % half;
          cs[e] = rope_cos_sin(pos0 + t0 + t, p.inv_freq[k]);
        }
        __syncthreads();
      }
      if (i >= total) continue;
      if (page < 0 || page >= p.num_pages) { atomicOr(p.status, FB_ST_BAD_PAGE); continue; }
      const size_t dst = (((size_t)page * p.n_kv_heads + h) * kPage + pos % kPage) * vph + v;
      [[maybe_unused]] uint2* k8 = reinterpret_cast<uint2*>(p.k_pool);
      [[maybe_unused]] uint2* v8 = reinterpret_cast<uint2*>(p.v_pool);
      [[maybe_unused]] float ksc = 1.f, vsc = 1.f;
      if constexpr (F8) {
        ksc = p.k_scale[h]; vsc = p.v_scale[h];
        v8[dst] = quant8(va, vsc);
        if (rope) v8[dst + partner] = quant8(vb, vsc);
        else k8[dst] = quant8(ka, ksc);
      } else {
        p.v_pool[dst] = va;
        if (rope) p.v_pool[dst + partner] = vb;
        else p.k_pool[dst] = ka;
      }
      if (!rope) continue;
      float lo[8], hi[8];
      rotate8(ka, kb, cs + tb * half + v * 8, lo, hi);
      if constexpr (F8) {
        k8[dst] = make_uint2(e4m3x4(lo[0], lo[1], lo[2], lo[3], ksc), e4m3x4(lo[4], lo[5], lo[6], lo[7], ksc));
        k8[dst + partner] = make_uint2(e4m3x4(hi[0], hi[1], hi[2], hi[3], ksc), e4m3x4(hi[4], hi[5], hi[6], hi[7], ksc));
      } else {
        p.k_pool[dst] = make_uint4(to_bf16x2(lo[0], lo[1]), to_bf16x2(lo[2], lo[3]), to_bf16x2(lo[4], lo[5]), to_bf16x2(lo[6], lo[7]));
        p.k_pool[dst + partner] = make_uint4(to_bf16x2(hi[0], hi[1]), to_bf16x2(hi[2], hi[3]), to_bf16x2(hi[4], hi[5]), to_bf16x2(hi[6], hi[7]));
      }
    }
  }
}

// The frequencies of a base, in fp64; the context keeps those of the last one (64 powers take 2 us of the host's time).
static void fill_inv_freq(fb_ctx* ctx, double (&inv_freq)[64], float rope_base) {
  const int head_dim = ctx->cfg.head_dim;
  if (ctx->rope_base != rope_base) {
    for (int k = 0; k < 64; ++k)
      ctx->inv_freq[k] = (rope_base > 0.f && k < head_dim / 2)
                             ? exp2(-2.0 * (double)k / (double)head_dim * log2((double)rope_base)) : 0.0;
    ctx->rope_base = rope_base;
  }
  memcpy(inv_freq, ctx->inv_freq, sizeof inv_freq);
}
// one (token, head, pair of pieces) item per thread (two with the embedding off)
static int scatter_ctas_per_slot(const fb_config& c) {
  const int n = c.block_len * c.n_kv_heads * (c.head_dim / 16) / kScatterThreads;
  return n < 1 ? 1 : n < c.block_len ? n : c.block_len;
}

int launch_scatter(fb_ctx* ctx, const fb_pack* pk, const int32_t* page_table, const void* k_new,
                   const void* v_new, void* k_pool, void* v_pool, float rope_base, int32_t* status,
                   cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  ScatterParams p;
  p.n_live = pk->n_live; p.slot_req = pk->slot_req; p.slot_pos0 = pk->slot_pos0;
  p.page_table = page_table;
  p.k_new = static_cast<const uint4*>(k_new); p.v_new = static_cast<const uint4*>(v_new);
  p.k_pool = static_cast<uint4*>(k_pool); p.v_pool = static_cast<uint4*>(v_pool);
  p.status = status;
  p.bl = c.block_len; p.n_kv_heads = c.n_kv_heads; p.head_dim = c.head_dim;
  p.max_pages_per_req = c.max_pages_per_req; p.num_pages = c.num_pages;
  p.rope_base = rope_base;
  p.k_scale = p.v_scale = nullptr;
  fill_inv_freq(ctx, p.inv_freq, rope_base);
  const dim3 grid(c.max_requests * c.wmax, scatter_ctas_per_slot(c));
  return cuda_err(ctx, launch_pdl(scatter_window_kv_kernel<false>, grid, kScatterThreads, 0, stream, p),
                  "scatter_window_kv_kernel launch");
}

int launch_scatter_fp8(fb_ctx* ctx, const fb_pack* pk, const int32_t* page_table, const void* k_new,
                       const void* v_new, void* k_pool8, void* v_pool8, const float* k_scale, const float* v_scale,
                       float rope_base, int32_t* status, cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  ScatterParams p;
  p.n_live = pk->n_live; p.slot_req = pk->slot_req; p.slot_pos0 = pk->slot_pos0;
  p.page_table = page_table;
  p.k_new = static_cast<const uint4*>(k_new); p.v_new = static_cast<const uint4*>(v_new);
  p.k_pool = static_cast<uint4*>(k_pool8); p.v_pool = static_cast<uint4*>(v_pool8);
  p.status = status;
  p.bl = c.block_len; p.n_kv_heads = c.n_kv_heads; p.head_dim = c.head_dim;
  p.max_pages_per_req = c.max_pages_per_req; p.num_pages = c.num_pages;
  p.rope_base = rope_base;
  p.k_scale = k_scale; p.v_scale = v_scale;
  fill_inv_freq(ctx, p.inv_freq, rope_base);
  const dim3 grid(c.max_requests * c.wmax, scatter_ctas_per_slot(c));
  return cuda_err(ctx, launch_pdl(scatter_window_kv_kernel<true>, grid, kScatterThreads, 0, stream, p),
                  "scatter_window_kv_kernel (8-bit pages) launch");
}

// fb_embed_gather: x[i, :] = table[qtok[i], :] for live rows; one warp per row, 16-byte pieces.
__global__ void __launch_bounds__(256) embed_gather_kernel(const int32_t* n_live, const int32_t* qtok,
                                                           const uint4* table, int table_rows, int vec_per_row,
                                                           uint4* x, int bl, int32_t* status) {
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (row >= *n_live * bl) return;
  const int tok = qtok[row];
  if (tok < 0 || tok >= table_rows) { if (lane == 0) atomicOr(status, FB_ST_BAD_TOKEN); return; }
  const uint4* src = table + (size_t)tok * vec_per_row;
  uint4* dst = x + (size_t)row * vec_per_row;
  for (int v = lane; v < vec_per_row; v += 32) dst[v] = src[v];
}

int launch_embed(fb_ctx* ctx, const fb_pack* pk, const void* table, int table_rows, int hidden, void* x,
                 int32_t* status, cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  const int rows = c.max_requests * c.wmax * c.block_len;
  embed_gather_kernel<<<(rows + 7) / 8, 256, 0, stream>>>(pk->n_live, pk->qtok, static_cast<const uint4*>(table),
                                                        table_rows, hidden / 8, static_cast<uint4*>(x),
                                                        c.block_len, status);
  return cuda_err(ctx, cudaGetLastError(), "embed_gather_kernel launch");
}

// fb_append_kv: the newest token of every request goes to storage position kv_len - 1 of its pages.  A
// thread has one (head, piece) of K and of V, as in the scatter above, and the angles of the token stand in
// a table that the CTA builds while the loads are in flight.  Bound by latency: kv_len, then the page id, then
// the stores, a few kilobytes a request.
struct AppendParams {
  const int32_t *kv_len, *tok_pos, *page_table;
  int32_t* kv_pos;
  float* kv_weight;
  const uint4 *k_new, *v_new;
  uint4 *k_pool, *v_pool;
  int32_t* status;
  int32_t n_kv_heads, head_dim, max_pages_per_req, num_pages;
  float rope_base;
  const float *k_scale, *v_scale;   // 8-bit pages: [n_kv_heads]
  double inv_freq[64];
};

constexpr int kAppendThreads = 128;

template <bool F8>
__global__ void __launch_bounds__(kAppendThreads) append_kv_kernel(const AppendParams p) {
  pdl_wait();
  __shared__ float2 cs[64];
  const int r = blockIdx.x, nh = p.n_kv_heads, vph = p.head_dim / 8, half = p.head_dim / 2;
  const bool rope = p.rope_base > 0.f;
  const int per_head = rope ? vph / 2 : vph, partner = rope ? vph / 2 : 0;
  const int i = blockIdx.y * kAppendThreads + threadIdx.x, h = i / per_head, v = i % per_head;
  const bool mine = h < nh;
  const int len = p.kv_len[r], pos = p.tok_pos[r];
  uint4 ka, kb, va, vb;
  if (mine) {                                        // (the rows do not depend on the lengths: one latency)
    const size_t src = ((size_t)r * nh + h) * vph + v;
    ka = p.k_new[src]; va = p.v_new[src];
    if (rope) { kb = p.k_new[src + partner]; vb = p.v_new[src + partner]; }
  }
  if (len <= 0) return;
  const long long cap = (long long)p.max_pages_per_req * kPage;
  const int j = len - 1;
  const int page = len <= cap ? p.page_table[(size_t)r * p.max_pages_per_req + j / kPage] : -1;
  if (rope) {
    if ((int)threadIdx.x < half) cs[threadIdx.x] = rope_cos_sin(pos, p.inv_freq[threadIdx.x]);
    __syncthreads();
  }
  if (len > cap || page < 0 || page >= p.num_pages) {
    if (threadIdx.x == 0) atomicOr(p.status, len > cap ? FB_ST_BAD_STATE : FB_ST_BAD_PAGE);
    return;
  }
  if (!mine) return;
  if (v == 0) {
    const size_t at = ((size_t)r * nh + h) * cap + j;
    if (p.kv_pos) p.kv_pos[at] = pos;
    if (p.kv_weight) p.kv_weight[at] = 0.f;
  }
  const size_t dst = (((size_t)page * nh + h) * kPage + j % kPage) * vph + v;
  float lo[8], hi[8];
  if (rope) rotate8(ka, kb, cs + v * 8, lo, hi);
  if constexpr (F8) {
    const float ksc = p.k_scale[h], vsc = p.v_scale[h];
    uint2* k8 = reinterpret_cast<uint2*>(p.k_pool);
    uint2* v8 = reinterpret_cast<uint2*>(p.v_pool);
    v8[dst] = quant8(va, vsc);
    if (rope) {
      v8[dst + partner] = quant8(vb, vsc);
      k8[dst] = make_uint2(e4m3x4(lo[0], lo[1], lo[2], lo[3], ksc), e4m3x4(lo[4], lo[5], lo[6], lo[7], ksc));
      k8[dst + partner] = make_uint2(e4m3x4(hi[0], hi[1], hi[2], hi[3], ksc), e4m3x4(hi[4], hi[5], hi[6], hi[7], ksc));
    } else {
      k8[dst] = quant8(ka, ksc);
    }
  } else {
    p.v_pool[dst] = va;
    if (rope) {
      p.v_pool[dst + partner] = vb;
      p.k_pool[dst] = make_uint4(to_bf16x2(lo[0], lo[1]), to_bf16x2(lo[2], lo[3]), to_bf16x2(lo[4], lo[5]), to_bf16x2(lo[6], lo[7]));
      p.k_pool[dst + partner] = make_uint4(to_bf16x2(hi[0], hi[1]), to_bf16x2(hi[2], hi[3]), to_bf16x2(hi[4], hi[5]), to_bf16x2(hi[6], hi[7]));
    } else {
      p.k_pool[dst] = ka;
    }
  }
}

int launch_append(fb_ctx* ctx, const fb_cache* kv, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                  const float* k_scale, const float* v_scale, float rope_base, int32_t* status, cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  AppendParams p;
  p.kv_len = kv->kv_len; p.tok_pos = kv->tok_pos; p.page_table = kv->page_table;
  p.kv_pos = kv->kv_pos; p.kv_weight = kv->kv_weight;
  p.k_new = static_cast<const uint4*>(k_new); p.v_new = static_cast<const uint4*>(v_new);
  p.k_pool = static_cast<uint4*>(k_pool); p.v_pool = static_cast<uint4*>(v_pool);
  p.status = status;
  p.n_kv_heads = c.n_kv_heads; p.head_dim = c.head_dim;
  p.max_pages_per_req = c.max_pages_per_req; p.num_pages = c.num_pages;
  p.rope_base = rope_base;
  p.k_scale = k_scale; p.v_scale = v_scale;
  fill_inv_freq(ctx, p.inv_freq, rope_base);
  const int items = c.n_kv_heads * (c.head_dim / (rope_base > 0.f ? 16 : 8));
  const dim3 grid(c.max_requests, (items + kAppendThreads - 1) / kAppendThreads);
  const auto kernel = c.kv_fp8 ? append_kv_kernel<true> : append_kv_kernel<false>;
  return cuda_err(ctx, launch_pdl(kernel, grid, kAppendThreads, 0, stream, p), "append_kv_kernel launch");
}

}  // namespace fb
