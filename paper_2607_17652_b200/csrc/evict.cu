// fb_evict_kv: cuts every cache that holds more than keep[r] keys to that many, per KV head: protected keys first (the
// first `sinks` and the last `recent` positions), then by accumulated attention weight, the lower index on ties.
//
// Attention does not see in which order keys are stored (they are stored rotated), so nothing moves but what has to:
// with m = keep[r], the keys that stay at or above m take the places below m that become free, i-th to i-th.  Sources
// and destinations do not overlap, so every row moves at once, and the caller's prefix of m keys is the whole cache.
//
// Kernel 1, a cluster of 1 to 8 CTAs per (request, KV head): the m-th largest rank by radix selection (11, 11 and 10
// bits of a 32-bit key in shared-memory histograms; ranks are held in registers, 8,192 a CTA), then the lists of
// freed places and of keys to move, both in index order by ballots and one scan.  Bound by its chain of
// about ten block-wide steps; reads 8 bytes a stored key.
// Kernel 2: the rows of K and V, the weights and the positions, eight moves a warp with their loads in flight.
// HBM-bound where many move.
#include <cooperative_groups.h>

#include "fb_common.cuh"

namespace fb {

namespace cg = cooperative_groups;

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr int kSelPer = 16;                       // keys of a thread in registers
constexpr int kSelCap = kSelThreads * kSelPer;    // ... of a CTA
constexpr int kBins = 2048;
constexpr int kMoveThreads = 256, kMoveBatch = 8;

struct EvictParams {
  int32_t *kv_len, *kv_pos;
  const int32_t *tok_pos, *keep, *page_table;
  float* kv_weight;
  uint4 *k_pool, *v_pool;
  int32_t* status;
  int2* info;                                     // [requests x KV heads] moves, new length (-1: the request stays as it is)
  int32_t *to, *from;                             // [requests x KV heads][capacity / 2] places freed, keys that take them
  int32_t n_kv_heads, max_pages_per_req, num_pages, recent, sinks;
};

// Rank of a key as an unsigned number: protected keys above all, a NaN below all, -0 as 0.
__device__ __forceinline__ uint32_t rank_of(float w, int pos, int sinks, long long newest_out) {
  if (pos < sinks || pos > newest_out) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// Exclusive scan of kSelPer * kSelWarps packed pairs of 16-bit counts, in index order; returns the total.  All threads.
__device__ __forceinline__ uint32_t scan_counts(uint32_t* cnt, uint32_t* warp_sum) {
  static_assert(kSelPer * kSelWarps == 256, "eight warps, a count a lane");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __syncthreads();
  uint32_t v = 0, incl = 0;
  if (tid < 256) {
    v = incl = cnt[tid];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) warp_sum[warp] = incl;
  }
  __syncthreads();
  uint32_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const uint32_t x = warp_sum[w];
    before += w < warp ? x : 0;
    total += x;
  }
  if (tid < 256) cnt[tid] = before + incl - v;
  __syncthreads();
  return total;
}

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const EvictParams p) {
  cg::cluster_group cluster = cg::this_cluster();
  const int cl = (int)cluster.num_blocks(), me = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t cnt[kSelPer * kSelWarps], warp_sum[kSelWarps];
  __shared__ uint32_t found[2];                   // digit, keys still to be taken from it
  __shared__ uint32_t mine[3];                    // equal keys; freed places; keys to move, of this CTA
  pdl_wait_then_release();
  const int line = blockIdx.x / cl, r = line / p.n_kv_heads;
  const int n = p.kv_len[r], m = p.keep[r], newest = p.tok_pos[r];
  const long long cap = (long long)p.max_pages_per_req * kPage, newest_out = (long long)newest - p.recent;
  // (the same for all CTAs of the cluster up to here and to the barriers below)
  bool bad = false;
  if (n > 0 && n <= cap && m >= 0 && n > m)
    for (int i = tid; i < (n + kPage - 1) / kPage; i += kSelThreads) {
      const int page = p.page_table[(size_t)r * p.max_pages_per_req + i];
      bad |= page < 0 || page >= p.num_pages;
    }
  bad = __syncthreads_or(bad);
  if (n <= 0 || n > cap || m < 0 || n <= m || bad || m == 0) {
    if (tid == 0 && me == 0) {
      if (n > cap) atomicOr(p.status, FB_ST_BAD_STATE);
      if (bad) atomicOr(p.status, FB_ST_BAD_PAGE);
      p.info[line] = make_int2(0, n > 0 && n <= cap && m == 0 && !bad ? 0 : -1);
    }
    return;
  }
  // this CTA's keys: [lo, hi), those of a thread 512 apart; the first kSelCap stay in registers, the others are formed again
  const int span = (n + cl - 1) / cl, lo = min(n, me * span), hi = min(n, lo + span);
  const float* w = p.kv_weight + (size_t)line * cap;
  const int32_t* pos = p.kv_pos + (size_t)line * cap;
  auto rank_at = [&](int i) { return rank_of(w[i], pos[i], p.sinks, newest_out); };
  uint32_t key[kSelPer];
  {
    float wv[kSelPer];
    int pv[kSelPer];
#pragma unroll
    for (int k = 0; k < kSelPer; ++k) {
      const int i = lo + k * kSelThreads + tid;
      wv[k] = i < hi ? w[i] : 0.f;
      pv[k] = i < hi ? pos[i] : 0;
    }
#pragma unroll
    for (int k = 0; k < kSelPer; ++k) key[k] = rank_of(wv[k], pv[k], p.sinks, newest_out);
  }

  // the m-th largest rank, digit by digit
  uint32_t prefix = 0, need = (uint32_t)m;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above = pass == 0 ? 32 : pass == 1 ? 21 : 10;
    const uint32_t mask = pass == 2 ? 1023u : 2047u;
    if (cl > 1) cluster.sync();                   // (the others have read the histogram of the pass before)
    else __syncthreads();
    for (int b = tid; b < kBins; b += kSelThreads) hist[b] = 0;
    __syncthreads();
    auto count = [&](uint32_t x) {
      if (pass == 0 || (x >> above) == prefix) atomicAdd(&hist[(x >> shift) & mask], 1u);
    };
#pragma unroll
    for (int k = 0; k < kSelPer; ++k)
      if (lo + k * kSelThreads + tid < hi) count(key[k]);
    for (int i = lo + kSelCap + tid; i < hi; i += kSelThreads) count(rank_at(i));
    if (cl > 1) cluster.sync();
    else __syncthreads();
    // four bins a thread, the largest digits first
    uint32_t c[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = 0;
    for (int q = 0; q < cl; ++q) {
      const uint32_t* h = cl > 1 ? cluster.map_shared_rank(hist, q) : hist;
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] += h[kBins - 1 - (4 * tid + j)];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += c[j];
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int v = 0; v < kSelWarps; ++v) before += v < warp ? warp_sum[v] : 0;
    before += incl - sum;
    if (before < need && need <= before + sum) {  // (one thread)
      uint32_t left = need - before;
      int j = 0;
      while (left > c[j]) left -= c[j++];
      found[0] = kBins - 1 - (4 * tid + j);
      found[1] = left;
    }
    __syncthreads();
    prefix = pass == 2 ? prefix << 10 | found[0] : prefix << 11 | found[0];
    need = found[1];
  }
  // `prefix` is that rank; of the keys that have it the first `need` in index order stay
  const uint32_t least = prefix;
  if (tid == 0) mine[0] = hist[least & 1023u];
  if (cl > 1) cluster.sync();
  else __syncthreads();
  uint32_t eq_base = 0;
  for (int q = 0; q < me; ++q) eq_base += *cluster.map_shared_rank(&mine[0], q);

  // which of a thread's keys stay, for kSelCap keys at a time in index order; then the places below m that become free and
  // the keys at or above m that stay, numbered in index order
  const uint32_t below = (1u << lane) - 1u;
  auto stays = [&](const uint32_t (&x)[kSelPer], int base, uint32_t& eq_before) {
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < kSelPer; ++k) {
      const bool in = base + k * kSelThreads + tid < hi;
      if (in && x[k] > least) bits |= 1u << k;
      const uint32_t e = __ballot_sync(0xffffffffu, in && x[k] == least);
      if (lane == 0) cnt[k * kSelWarps + warp] = __popc(e);
    }
    const uint32_t total = scan_counts(cnt, warp_sum);
#pragma unroll
    for (int k = 0; k < kSelPer; ++k) {
      const bool e = base + k * kSelThreads + tid < hi && x[k] == least;
      const uint32_t at = eq_before + cnt[k * kSelWarps + warp] + __popc(__ballot_sync(0xffffffffu, e) & below);
      if (e && at < need) bits |= 1u << k;
    }
    __syncthreads();                              // (cnt is read no more)
    eq_before += total;
    return bits;
  };
  auto number = [&](uint32_t bits, int base, uint32_t& free_before, uint32_t& move_before, bool write) {
#pragma unroll
    for (int k = 0; k < kSelPer; ++k) {
      const int i = base + k * kSelThreads + tid;
      const uint32_t f = __ballot_sync(0xffffffffu, i < hi && i < m && !(bits >> k & 1));
      const uint32_t v = __ballot_sync(0xffffffffu, i < hi && i >= m && (bits >> k & 1));
      if (lane == 0) cnt[k * kSelWarps + warp] = __popc(f) | __popc(v) << 16;
    }
    const uint32_t total = scan_counts(cnt, warp_sum);
    if (write) {
      const size_t half = (size_t)(cap / 2);
#pragma unroll
      for (int k = 0; k < kSelPer; ++k) {
        const int i = base + k * kSelThreads + tid;
        const bool f = i < hi && i < m && !(bits >> k & 1), v = i < hi && i >= m && (bits >> k & 1);
        const uint32_t bf = __ballot_sync(0xffffffffu, f), bv = __ballot_sync(0xffffffffu, v), c = cnt[k * kSelWarps + warp];
        if (f) p.to[line * half + free_before + (c & 0xffffu) + __popc(bf & below)] = i;
        if (v) p.from[line * half + move_before + (c >> 16) + __popc(bv & below)] = i;
      }
    }
    __syncthreads();
    free_before += total & 0xffffu;
    move_before += total >> 16;
  };
  auto ranks = [&](int base, uint32_t (&x)[kSelPer]) {
#pragma unroll
    for (int k = 0; k < kSelPer; ++k) {
      const int i = base + k * kSelThreads + tid;
      x[k] = base == lo ? key[k] : i < hi ? rank_at(i) : 0u;
    }
  };
  uint32_t first_free = 0, first_move = 0;        // (of the whole row, before this CTA's)
  uint32_t eq0 = eq_base, bits0 = 0, x[kSelPer];
  if (cl > 1) {
    // the counts of every CTA first, the numbers of those before it, then the lists
    uint32_t f = 0, v = 0, eq = eq_base;
    for (int base = lo; base < hi; base += kSelCap) {
      ranks(base, x);
      const uint32_t bits = stays(x, base, eq);
      if (base == lo) { bits0 = bits; eq0 = eq; }
      number(bits, base, f, v, false);
    }
    if (tid == 0) { mine[1] = f; mine[2] = v; }
    cluster.sync();
    for (int q = 0; q < me; ++q) {
      first_free += *cluster.map_shared_rank(&mine[1], q);
      first_move += *cluster.map_shared_rank(&mine[2], q);
    }
  }
  uint32_t f = first_free, v = first_move;
  for (int base = lo; base < hi; base += kSelCap) {
    uint32_t bits = bits0;
    if (cl == 1 || base > lo) {
      ranks(base, x);
      bits = stays(x, base, eq0);
    }
    number(bits, base, f, v, true);
  }
  if (me == cl - 1 && tid == 0) p.info[line] = make_int2((int)f, m);
  if (cl > 1) cluster.sync();                     // (what the others read stays until they have)
}

// kVec: 16-byte pieces of a stored row.  A warp takes eight moves: their places by its first eight lanes, then the rows, K and
// V side by side, all loads before the first store.
template <int kVec>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams p) {
  pdl_wait();
  const int line = blockIdx.x, r = line / p.n_kv_heads, h = line % p.n_kv_heads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int2 info = p.info[line];
  if (info.y < 0) return;
  if (h == 0 && blockIdx.y == 0 && threadIdx.x == 0) p.kv_len[r] = info.y;
  const size_t cap = (size_t)p.max_pages_per_req * kPage, list = line * (cap / 2), rec = line * cap;
  const int32_t* pages = p.page_table + (size_t)r * p.max_pages_per_req;
  constexpr int kSide = 32 / (2 * kVec);          // moves side by side: K and V of one (256-byte rows) or of two
  const int side = lane / (2 * kVec), in = lane % (2 * kVec);
  uint4* pool = in < kVec ? p.k_pool : p.v_pool;
  const int piece = in % kVec;
  for (int i0 = (blockIdx.y * (kMoveThreads / 32) + warp) * kMoveBatch; i0 < info.x; i0 += gridDim.y * (kMoveThreads / 32) * kMoveBatch) {
    const int n = min(kMoveBatch, info.x - i0);
    long long dst = 0, src = 0;                   // rows
    if (lane < n) {
      const int to = p.to[list + i0 + lane], at = p.from[list + i0 + lane];
      const float w = p.kv_weight[rec + at];
      const int ps = p.kv_pos[rec + at];
      dst = ((long long)pages[to / kPage] * p.n_kv_heads + h) * kPage + to % kPage;
      src = ((long long)pages[at / kPage] * p.n_kv_heads + h) * kPage + at % kPage;
      p.kv_weight[rec + to] = w;
      p.kv_pos[rec + to] = ps;
    }
    uint4 v[kMoveBatch / kSide];
#pragma unroll
    for (int k = 0; k < kMoveBatch / kSide; ++k) {
      const int j = k * kSide + side;
      const long long s = __shfl_sync(0xffffffffu, src, j);
      if (j < n) v[k] = pool[s * kVec + piece];
    }
#pragma unroll
    for (int k = 0; k < kMoveBatch / kSide; ++k) {
      const int j = k * kSide + side;
      const long long d = __shfl_sync(0xffffffffu, dst, j);
      if (j < n) pool[d * kVec + piece] = v[k];
    }
  }
}

struct EvictWs { size_t info, to, from, total; };
static EvictWs evict_ws(const fb_ctx* ctx) {
  const size_t rows = (size_t)ctx->cfg.max_requests * ctx->cfg.n_kv_heads, half = (size_t)ctx->cfg.max_pages_per_req * kPage / 2;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  EvictWs w;
  w.info = 0;
  w.to = w.info + up(rows * sizeof(int2));
  w.from = w.to + up(rows * half * sizeof(int32_t));
  w.total = w.from + up(rows * half * sizeof(int32_t));
  return w;
}
size_t evict_workspace_bytes(const fb_ctx* ctx) { return evict_ws(ctx).total; }

int launch_evict(fb_ctx* ctx, const fb_cache* kv, const int32_t* keep, int recent, int sinks, void* k_pool, void* v_pool,
                 void* ws, int32_t* status, cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  const EvictWs w = evict_ws(ctx);
  char* base = static_cast<char*>(ws);
  EvictParams p;
  p.kv_len = kv->kv_len; p.kv_pos = kv->kv_pos; p.tok_pos = kv->tok_pos; p.keep = keep; p.page_table = kv->page_table;
  p.kv_weight = kv->kv_weight;
  p.k_pool = static_cast<uint4*>(k_pool); p.v_pool = static_cast<uint4*>(v_pool); p.status = status;
  p.info = reinterpret_cast<int2*>(base + w.info);
  p.to = reinterpret_cast<int32_t*>(base + w.to); p.from = reinterpret_cast<int32_t*>(base + w.from);
  p.n_kv_heads = c.n_kv_heads; p.max_pages_per_req = c.max_pages_per_req; p.num_pages = c.num_pages;
  p.recent = recent; p.sinks = sinks;
  const long long rows = (long long)c.max_requests * c.n_kv_heads, cap = (long long)c.max_pages_per_req * kPage;
  int cl = 1;
  while (cl < 8 && (long long)cl * kSelCap < cap) cl *= 2;
  if (rows * cl > 0x7fffffffll) return set_err(ctx, FB_ERR_UNSUPPORTED, "max_requests * n_kv_heads is too large");
  if (int e = cuda_err(ctx, launch_pdl_cluster(evict_select_kernel, dim3((unsigned)(rows * cl)), kSelThreads, 0, stream, cl, p),
                       "evict_select_kernel launch"))
    return e;
  // about eight CTAs an SM, no more than there can be batches
  const long long batches = (cap / 2 + kMoveBatch * (kMoveThreads / 32) - 1) / (kMoveBatch * (kMoveThreads / 32)), want = 1 + 8 * kSms / rows;
  const dim3 grid((unsigned)rows, (unsigned)(want < batches ? want : batches));
  const int row = c.head_dim * (c.kv_fp8 ? 1 : 2);
  return cuda_err(ctx, launch_pdl(row == 256 ? evict_move_kernel<16> : evict_move_kernel<8>, grid, kMoveThreads, 0, stream, p),
                  "evict_move_kernel launch");
}

}  // namespace fb
