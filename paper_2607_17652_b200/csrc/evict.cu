// fb_evict_kv: cuts every cache that holds more than keep[r] keys to that many, per KV head: protected keys first (the
// first `sinks` and the last `recent` positions, and any above tok_pos), then by accumulated attention weight, the lower index on ties.
//
// Attention does not see in which order keys are stored (they are stored rotated), so nothing moves but what has to:
// with m = keep[r], the keys that stay at or above m take the places below m that become free, i-th to i-th.  Sources
// and destinations do not overlap, so every row moves at once, and the caller's prefix of m keys is the whole cache.
//
// Kernel 1, a cluster of 1 to 8 CTAs per (request, KV head): the rank of the last key that stays, by counting.  The range
// of the ranks is cut into 512 bins, the bin that holds the boundary into 512 again, until all keys of a bin stay
// (two or three times as a rule, four at most; 512 bins that follow the range spread the counts over many addresses); then the lists of freed
// places and of keys to move, both in index order by the threads' own counts and one scan.  Bound by its chain of block-wide steps: loops
// are kept short, since every CTA runs the code once, and what goes between the CTAs of a cluster is kept small (one request
// of 28,123 keys: digits of 11 bits and code unrolled over keys in registers 28 us, this form 16).  Reads 8 bytes a stored key.
// Kernel 2: the rows of K and V, the weights and the positions, eight rows a warp under way.
// HBM-bound where many move, by rows of 128 to 256 bytes that lie apart: 64 requests cut from 1,024 to 8,192 keys to 2,000 move
// 0.49 GB in bf16 in 93 us (5.3 TB/s), 0.25 GB in 8 bits in 53 us (4.6 TB/s); neither more rows under way nor more warps change that.
#include <cooperative_groups.h>

#include "fb_common.cuh"

namespace fb {

namespace cg = cooperative_groups;

constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32;
constexpr int kSelCap = 8192;                     // keys of a CTA, in shared memory
constexpr int kBinBits = 9, kBins = 1 << kBinBits, kMaxCluster = 8;
constexpr int kMoveThreads = 256, kMoveWarps = kMoveThreads / 32, kMoveAhead = 8;

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

// Rank of a key as an unsigned number: protected keys above all, a NaN below all, -0 as 0.  `first`: the first position above
// tok_pos - recent, where there is any that 32 bits hold.
struct Guarded { int sinks, first; bool any; };
__device__ __forceinline__ uint32_t rank_of(float w, int pos, const Guarded& g) {
  const uint32_t u = __float_as_uint(w + 0.f);
  uint32_t k = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  if (w != w) k = 0u;
  return pos < g.sinks || (g.any && pos >= g.first) ? 0xffffffffu : k;
}

// Exclusive scan over the threads (of counts, or of pairs of 16-bit counts); `total`: of all.  All threads.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sum, uint32_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  __syncthreads();                                 // (the scan before has been read)
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kSelWarps; ++w) {
    const uint32_t x = warp_sum[w];
    before += w < warp ? x : 0;
    total += x;
  }
  return before + incl - v;
}

__global__ void __launch_bounds__(kSelThreads, 5) evict_select_kernel(const EvictParams p) {
  cg::cluster_group cluster = cg::this_cluster();
  const int cl = (int)cluster.num_blocks(), me = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ __align__(16) uint32_t key[kSelCap];  // ranks
  __shared__ __align__(16) uint32_t hist[2][kBins];
  __shared__ uint32_t warp_sum[kSelWarps];
  __shared__ uint32_t found[3];                    // bin, keys still to be taken from it, keys in it
  __shared__ uint32_t part[3][kSelWarps];
  __shared__ uint32_t peer[3][4][kMaxCluster];     // what the CTAs of the cluster have told this one, by occasion
  pdl_wait_then_release();
  const int line = blockIdx.x / cl, r = line / p.n_kv_heads;
  const int n = p.kv_len[r], m = p.keep[r], newest = p.tok_pos[r];
  const long long cap = (long long)p.max_pages_per_req * kPage;
  const bool over = n > 0 && n <= cap && m >= 0 && n > m;
  // this CTA's keys: [lo, hi), kSelCap at a time
  const int span = over ? ((n + cl - 1) / cl + 3) & ~3 : 0, lo = min(n, me * span), hi = min(n, lo + span);
  const size_t row = (size_t)line * cap;
  const long long first = (long long)newest - p.recent + 1;
  const Guarded guard{p.sinks, (int)min(max(first, -0x80000000ll), 0x7fffffffll), first <= 0x7fffffffll};
  // A chunk's ranks from its weights and positions, four at a time (a row starts on 256 bytes and is whole pages long, so that
  // the last four stay inside it).
  uint32_t low = 0xffffffffu, high = 0, guards = 0; // of the unprotected ranks, and protected keys
  auto load = [&](int base) {
    const int quads = (min(hi - base, kSelCap) + 3) / 4;
    const float4* w4 = reinterpret_cast<const float4*>(p.kv_weight + row + base);
    const int4* p4 = reinterpret_cast<const int4*>(p.kv_pos + row + base);
#pragma unroll 2
    for (int i = tid; i < quads; i += kSelThreads) {
      const float4 w = w4[i];
      const int4 q = p4[i];
      const uint4 x = make_uint4(rank_of(w.x, q.x, guard), rank_of(w.y, q.y, guard), rank_of(w.z, q.z, guard), rank_of(w.w, q.w, guard));
      reinterpret_cast<uint4*>(key)[i] = x;
      const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (base + 4 * i + j < hi) {
          if (xs[j] == 0xffffffffu) ++guards;
          else { low = min(low, xs[j]); high = max(high, xs[j]); }
        }
    }
  };
  bool bad = false;
  if (over) {
    for (int i = tid; i < (n + kPage - 1) / kPage; i += kSelThreads) {
      const int page = p.page_table[(size_t)r * p.max_pages_per_req + i];
      bad |= page < 0 || page >= p.num_pages;
    }
    if (m > 0) load(lo);
  }
  bad = __syncthreads_or(bad);
  // (the CTAs of a cluster leave together here or meet at all barriers below)
  if (!over || bad || m == 0) {
    if (tid == 0 && me == 0) {
      if (n > cap) atomicOr(p.status, FB_ST_BAD_STATE);
      if (bad) atomicOr(p.status, FB_ST_BAD_PAGE);
      p.info[line] = make_int2(0, over && !bad ? 0 : -1);
    }
    return;
  }
  if (cl > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");       // (this CTA is there: its shared memory may be written)
  const bool chunked = hi - lo > kSelCap;          // (longer than the shared memory of the cluster: chunks are read again in every pass)
  // every key of the CTA, with its index; a chunk other than the one in shared memory is loaded first
  int held = lo;
  auto fetch = [&](int base) {
    if (held == base) return;
    __syncthreads();
    load(base);
    held = base;
    __syncthreads();
  };
  if (chunked)
    for (int base = lo + kSelCap; base < hi; base += kSelCap) fetch(base);       // (for low, high and guards)

  // a value of every CTA to every CTA: put down in the others' shared memory, read behind the barrier
  auto tell = [&](int occasion, int which, uint32_t v) {
    if (tid < cl) *cluster.map_shared_rank(&peer[occasion][which][me], tid) = v;
  };
  {
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    guards = __reduce_add_sync(0xffffffffu, guards);
    if (lane == 0) { part[0][warp] = low; part[1][warp] = high; part[2][warp] = guards; }
    for (int i = tid; i < 2 * kBins; i += kSelThreads) hist[0][i] = 0;
    __syncthreads();
    low = __reduce_min_sync(0xffffffffu, part[0][lane % kSelWarps]);
    high = __reduce_max_sync(0xffffffffu, part[1][lane % kSelWarps]);
    guards = __reduce_add_sync(0xffffffffu, lane < kSelWarps ? part[2][lane] : 0u);
    if (cl > 1) {
      asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
      tell(0, 0, low); tell(0, 1, high); tell(0, 2, guards);
      cluster.sync();
      low = __reduce_min_sync(0xffffffffu, peer[0][0][lane % cl]);
      high = __reduce_max_sync(0xffffffffu, peer[0][1][lane % cl]);
      guards = __reduce_add_sync(0xffffffffu, lane < cl ? peer[0][2][lane] : 0u);
    }
  }
  // The boundary: a range of ranks from `least` on, of which all keys stay, or (then it is a single rank) the first `need` in
  // index order; keys above it stay.
  uint32_t least = 0xffffffffu, need = (uint32_t)m, same = guards;
  if (need > guards) {                             // not among the protected keys alone
    need -= guards;
    least = low;
    int bits = 32 - __clz((int)(high - low));      // ranks are low + [0, 2^bits)
#pragma unroll 1
    for (int pass = 0;; ++pass) {
      uint32_t* h = hist[pass & 1];
      const int shift = max(0, bits - kBinBits);
#pragma unroll 1
      for (int base = lo; base < hi; base += kSelCap) {
        fetch(base);
        const int cnt_keys = min(hi - base, kSelCap);
        const uint32_t most = bits == 0 ? 0u : 0xffffffffu >> (32 - bits);
#pragma unroll 4
        for (int i = tid; i < cnt_keys; i += kSelThreads) {
          const uint32_t x = key[i] - least;       // (below the range: wraps around to a large number)
          if (key[i] != 0xffffffffu && x <= most) atomicAdd(&h[x >> shift], 1u);
        }
      }
      if (cl > 1) cluster.sync();
      else __syncthreads();
      // two bins a thread, the largest first
      uint32_t c0 = 0, c1 = 0;
      const int bin = kBins - 2 - 2 * tid;
      if (cl == 1) {
        const uint2 v = *reinterpret_cast<const uint2*>(h + bin);
        c0 = v.y; c1 = v.x;
      } else {
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q)
          if (q < cl) {
            const uint2 v = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(h + bin, q));
            c0 += v.y; c1 += v.x;
          }
      }
      uint32_t incl = c0 + c1;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
      }
      if (lane == 31) warp_sum[warp] = incl;
      for (int i = tid; i < kBins; i += kSelThreads) hist[(pass & 1) ^ 1][i] = 0;       // (of the next pass; read by all in the one before)
      __syncthreads();
      uint32_t before = 0;
#pragma unroll
      for (int v = 0; v < kSelWarps; ++v) before += v < warp ? warp_sum[v] : 0;
      before += incl - (c0 + c1);
      if (before < need && need <= before + c0 + c1) {       // (one thread)
        const bool second = need - before > c0;
        found[0] = bin + (second ? 0 : 1);
        found[1] = need - before - (second ? c0 : 0);
        found[2] = second ? c1 : c0;
      }
      __syncthreads();
      least += found[0] << shift;
      need = found[1];
      same = found[2];
      bits = shift;
      if (need == same || bits == 0) break;
    }
  }
  const bool ties = need != same;                  // (then the range is one rank)
  uint32_t eq_first = 0;
  if (ties && cl > 1) {                            // equal keys of the CTAs before this one
    uint32_t e = 0;
#pragma unroll 1
    for (int base = lo; base < hi; base += kSelCap) {
      fetch(base);
      for (int i = tid; i < min(hi - base, kSelCap); i += kSelThreads) e += key[i] == least;
    }
    e = __reduce_add_sync(0xffffffffu, e);
    __syncthreads();
    if (lane == 0) part[0][warp] = e;
    __syncthreads();
    tell(1, 0, __reduce_add_sync(0xffffffffu, lane < kSelWarps ? part[0][lane] : 0u));
    cluster.sync();
    eq_first = __reduce_add_sync(0xffffffffu, lane < me ? peer[1][0][lane] : 0u);
  }

  // Twice over the CTA's keys: the counts, of which the CTAs behind it are told, then the lists.  A thread has neighbouring keys
  // (an odd number of them, for the banks), so that its own counts and one scan number them in index order; the lists are put
  // together where the ranks have been and leave in whole lines.
  const size_t half = (size_t)(cap / 2);
  uint32_t frees = 0, moves = 0, eq_before = eq_first;       // of the chunks gone through; in the second go with those of the CTAs before
  uint32_t at = 0, total = 0;                                // of this chunk, before this thread (freed places, keys to move in the high half)
  unsigned long long pick = 0;                               // bit k: the thread's k-th key goes into a list
#pragma unroll 1
  for (int go = 0; go < 2; ++go) {
    if (go == 1) {
      const uint32_t f = frees, v = moves;
      frees = moves = 0;
      if (cl > 1) {
        tell(2, 0, f);
        tell(2, 1, v);
        cluster.sync();
        frees = __reduce_add_sync(0xffffffffu, lane < me ? peer[2][0][lane] : 0u);
        moves = __reduce_add_sync(0xffffffffu, lane < me ? peer[2][1][lane] : 0u);
      }
      if (me == cl - 1 && tid == 0) p.info[line] = make_int2((int)(frees + f), m);
      eq_before = eq_first;
    }
#pragma unroll 1
    for (int base = lo; base < hi; base += kSelCap) {
      const int in = min(hi - base, kSelCap), per = ((in + kSelThreads - 1) / kSelThreads) | 1;
      static_assert(kSelCap / kSelThreads < 64, "a bit a key");
      const int begin = min(in, tid * per), mine = min(in, begin + per) - begin;
      if (go == 0 || chunked) {
        fetch(base);
        uint32_t eq = 0, equal = 0;
        if (ties) {
          for (int k = 0; k < mine; ++k) eq += key[begin + k] == least;
          eq = eq_before + block_scan(eq, warp_sum, equal);
          eq_before += equal;
        }
        uint32_t c = 0;
        pick = 0;
#pragma unroll 4
        for (int k = 0; k < mine; ++k) {
          const uint32_t x = key[begin + k];
          const bool stays = ties ? x > least || (x == least && eq++ < need) : x >= least, under = base + begin + k < m;
          c += under ? (stays ? 0u : 1u) : (stays ? 0x10000u : 0u);
          pick |= (unsigned long long)(under != stays) << k;
        }
        at = block_scan(c, warp_sum, total);
      }
      if (go == 1) {
        const uint32_t n_free = total & 0xffffu, n_move = total >> 16;
        __syncthreads();                           // (the ranks are read no more)
        held = -1;
        uint32_t f = at & 0xffffu, v = n_free + (at >> 16);
        while (pick) {
          const int i = base + begin + __ffsll((long long)pick) - 1;
          pick &= pick - 1;
          key[i < m ? f++ : v++] = i;
        }
        __syncthreads();
        for (int i = tid; i < n_free; i += kSelThreads) p.to[line * half + frees + i] = key[i];
        for (int i = tid; i < n_move; i += kSelThreads) p.from[line * half + moves + i] = key[n_free + i];
      }
      frees += total & 0xffffu;
      moves += total >> 16;
    }
  }
  if (cl > 1) cluster.sync();                      // (no CTA leaves while another may read its histogram)
}

// kVec: 16-byte pieces of a stored row.  The warps of a line have equal contiguous shares of its moves, 32 places at a time by
// their lanes and eight rows under way, K and V side by side.
template <int kVec>
__global__ void __launch_bounds__(kMoveThreads, 3) evict_move_kernel(const EvictParams p) {
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
  const int warps = gridDim.y * kMoveWarps, share = max((info.x + warps - 1) / warps, kMoveAhead);
  const long long begin = (long long)(blockIdx.y * kMoveWarps + warp) * share;
  const int end = (int)min((long long)info.x, begin + share);
  for (int i0 = (int)min(begin, (long long)info.x); i0 < end; i0 += 32) {
    const int n = min(32, end - i0);
    uint32_t dst = 0, src = 0;                    // rows (fewer than 2^32 fit on a device)
    if (lane < n) {
      const int to = p.to[list + i0 + lane], at = p.from[list + i0 + lane];
      const int page_to = pages[to / kPage], page_at = pages[at / kPage];
      const float w = p.kv_weight[rec + at];
      const int ps = p.kv_pos[rec + at];
      dst = ((uint32_t)page_to * p.n_kv_heads + h) * kPage + to % kPage;
      src = ((uint32_t)page_at * p.n_kv_heads + h) * kPage + at % kPage;
      p.kv_weight[rec + to] = w;
      p.kv_pos[rec + to] = ps;
    }
    for (int j0 = 0; j0 < n; j0 += kMoveAhead * kSide) {
      uint4 v[kMoveAhead];
#pragma unroll
      for (int k = 0; k < kMoveAhead; ++k) {
        const int j = j0 + k * kSide + side;
        const size_t s = __shfl_sync(0xffffffffu, src, j);
        if (j < n) v[k] = __ldcg(pool + s * kVec + piece);
      }
#pragma unroll
      for (int k = 0; k < kMoveAhead; ++k) {
        const int j = j0 + k * kSide + side;
        const size_t d = __shfl_sync(0xffffffffu, dst, j);
        if (j < n) pool[d * kVec + piece] = v[k];
      }
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
  // CTAs of a row: enough for its keys in shared memory, and more where rows are few (each has less to go through).  Both by the
  // capacity and the rows of the context, since the lengths are only known on the device: 64 caches of 2,112 keys take 17 us in
  // a context for 2,112 keys, 39 in one for 32,768, and one of 28,123 takes 20 alone in its context, 37 as the only one of 64 rows.
  int cl = 1;
  while (cl < 8 && cl * (long long)kSelCap < cap) cl *= 2;
  while (cl < 8 && rows * cl * 2 <= kSms && cl * 512ll < cap) cl *= 2;
  if (rows * cl > 0x7fffffffll) return set_err(ctx, FB_ERR_UNSUPPORTED, "max_requests * n_kv_heads is too large");
  if (int e = cuda_err(ctx, launch_pdl_cluster(evict_select_kernel, dim3((unsigned)(rows * cl)), kSelThreads, 0, stream, cl, p),
                       "evict_select_kernel launch"))
    return e;
  // about sixteen CTAs an SM (three at a time: lines have unlike numbers of moves), no more than there can be batches
  const long long batch = kMoveAhead * kMoveWarps, batches = (cap / 2 + batch - 1) / batch, want = 1 + 16 * kSms / rows;
  const dim3 grid((unsigned)rows, (unsigned)(want < batches ? want : batches));
  const int row = c.head_dim * (c.kv_fp8 ? 1 : 2);
  return cuda_err(ctx, launch_pdl(row == 256 ? evict_move_kernel<16> : evict_move_kernel<8>, grid, kMoveThreads, 0, stream, p),
                  "evict_move_kernel launch");
}

}  // namespace fb
