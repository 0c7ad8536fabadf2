// fb_token_attn: one query token per request over everything its pages hold,
//   out = sum_j w_j V_j,  w = softmax(sm_scale q K^T),  j < kv_len,
// for all query heads of a KV head at once, so that every stored key and value crosses the memory bus once.
//
// HBM-bound: 4 d operations per key and query head against 2 d values read per key and KV head.
//
// Work.  The keys of a (request, KV head) are cut into tiles, and the tiles of the whole batch, one row behind the
// other, are dealt to the CTAs in equal contiguous shares, whatever the lengths: a row that a CTA holds whole is
// finished by it, one that is cut leaves a piece (reference, sum, unnormalised output) per CTA, and
// token_join_kernel adds the pieces in order.  A CTA starts at most one row that it does not finish and finishes at
// most one that it did not start, so two slots a CTA hold all pieces, however large the batch.
//
// A warp has 16 keys of a tile (32 where a row is 128 bytes) and works alone until its share ends:
//   S^T = K Q^T   (m16n8k16: 16 keys, 8 query heads; padded to 8)   and   O^T += V^T P^T  (16 of d, 8 heads)
// both on registers that the loads fill directly.  A contraction may take its index in any order as long as
// both operands agree, and so may the rows of an output: a lane loads 16 contiguous bytes of a key's row, which are
// the A fragments of two k-steps, and of the rows 2t, 2t+1, 2t+8, 2t+9 of V the 16 bytes that its eight (row block, row)
// places need; pairs of V rows are interleaved by byte permutes, P^T is S^T's fragment transposed by movmatrix.  No
// shared memory, no barrier, no address arithmetic but one base per step, and the next step's K and V are in flight
// while this one's products run.  The tensor pipe (legacy mma.sync) is far from its rate: 4 d x 16 products a key
// against 256 bytes from memory.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "fb_common.cuh"

namespace fb {

constexpr int kTokThreads = 128, kTokWarps = kTokThreads / 32;
constexpr int kTokCtasPerSm = 3;         // (2 where a block has 16 heads: twice the accumulators)
constexpr float kTokLog2e = 1.4426950408889634f;
constexpr float kNoRef = -3.0e38f;       // below every score: the reference of a row that has seen no key
constexpr float kRebase = 8.f;           // a score that far (in powers of two) above the reference moves it

struct TokenParams {
  const int32_t *kv_len, *page_table;
  float* kv_weight;
  const __nv_bfloat16* q;
  const char *k_pool, *v_pool;
  const float *k_scale, *v_scale;        // 8-bit pages: [n_kv_heads]
  __nv_bfloat16* out;
  int32_t* status;
  float* part_o;                         // [2 n_ctas][heads of a block][d] unnormalised outputs of the pieces
  float2* part_ml;                       // [2 n_ctas][heads of a block] reference (log2), sum
  float2* row_ml;                        // [rows][heads of a block] the same of rows that were not cut (weights only)
  float* scores;                         // [requests][KV heads][capacity][group] (log2; weights only)
  int32_t requests, group, n_kv_heads, head_blocks, max_pages_per_req, num_pages, n_ctas;
  float sm_scale;
};

// How keys are laid out over lanes and steps, by the bytes of a row.
template <int D, bool F8>
struct TokShape {
  static constexpr int kRow = D * (F8 ? 1 : 2);          // bytes of a stored row: 256 or 128
  static constexpr int kSub = kRow == 256 ? 1 : 2;       // blocks of 16 keys a warp takes at once
  static constexpr int kKeys = 16 * kSub;                // keys of a warp's step
  static constexpr int kTile = kKeys * kTokWarps;        // keys of a CTA's step
  static constexpr int kU = kRow / 64;                   // 16-byte loads of a K row by four lanes
  static constexpr int kV = kRow / 128;                  // 16-byte loads of a V row by eight lanes
  static constexpr int kMb = D / 16;                     // row blocks of O^T
};
static_assert(kPage % TokShape<128, false>::kKeys == 0 && kPage % TokShape<64, false>::kKeys == 0, "a step stays inside a page");

__device__ __forceinline__ uint4 ld16(const char* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool F8>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F8)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// two E4M3 bytes -> two fp16 (exact)
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// ---------------------------------------------------------------- the deal
// Tiles of request r (none where there is no request, nothing stored or the length is no length).
__device__ __forceinline__ int tok_tiles(const TokenParams& p, int r, int tile) {
  const int len = r < p.requests ? __ldcg(p.kv_len + r) : 0;
  return len > 0 && len <= (long long)p.max_pages_per_req * kPage ? (len + tile - 1) / tile : 0;
}
__device__ __forceinline__ long long warp_sum(long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Tiles of all rows, and of those of the requests before `upto`.  By a whole warp.
__device__ __forceinline__ long long tok_total(const TokenParams& p, int tile, int upto, long long& before) {
  long long all = 0, b = 0;
  for (int r0 = 0; r0 < p.requests; r0 += 32) {
    const int r = r0 + (threadIdx.x & 31), n = tok_tiles(p, r, tile);
    all += n;
    b += r < upto ? n : 0;
  }
  const int rows = p.n_kv_heads * p.head_blocks;
  before = warp_sum(b) * rows;
  return warp_sum(all) * rows;
}
__device__ __forceinline__ long long tok_share(long long total, int n_ctas) {
  const long long s = (total + n_ctas - 1) / n_ctas;
  return s < 1 ? 1 : s;
}

// ---------------------------------------------------------------- the stream
template <int D, bool F8, int NB, bool W>
__global__ void __launch_bounds__(kTokThreads, NB == 1 ? 3 : 2) token_attn_kernel(const TokenParams p) {
  using S = TokShape<D, F8>;
  constexpr int HB = 8 * NB, kStride = D + 1;
  constexpr float kShift = F8 ? 7.f : 0.f;     // fp16 weights: 2^7 above 1, so that 2^-31 of the reference is still there
  __shared__ float sh_o[kTokWarps][HB * kStride];
  __shared__ float2 sh_ml[kTokWarps][HB];
  pdl_wait_then_release();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c = lane >> 2, t = lane & 3;
  long long unused;
  const long long total = tok_total(p, S::kTile, 0, unused), share = tok_share(total, p.n_ctas);
  long long at = (long long)blockIdx.x * share;
  int left = (int)min(share, total - at > 0 ? total - at : 0);
  // rows without work: zeros where nothing is stored, a report where the length is no length
  for (int r = blockIdx.x; r < p.requests; r += p.n_ctas) {
    const int len = __ldcg(p.kv_len + r);
    if (len > (long long)p.max_pages_per_req * kPage && tid == 0) atomicOr(p.status, FB_ST_BAD_STATE);
    if (len != 0) continue;
    uint4* o = reinterpret_cast<uint4*>(p.out) + (size_t)r * p.n_kv_heads * p.group * (D / 8);
    for (int i = tid; i < p.n_kv_heads * p.group * (D / 8); i += kTokThreads) o[i] = make_uint4(0, 0, 0, 0);
  }
  if (left <= 0) return;
  // the request that holds tile `at`
  const int rows = p.n_kv_heads * p.head_blocks;
  int r = 0, nt = 0;
  for (int r0 = 0; r0 < p.requests; r0 += 32) {
    const int n = tok_tiles(p, r0 + lane, S::kTile);
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    const long long end = (long long)incl * rows;
    const unsigned here = __ballot_sync(0xffffffffu, at < end);
    if (here) {
      const int l = __ffs(here) - 1;
      nt = __shfl_sync(0xffffffffu, n, l);
      at -= (long long)(__shfl_sync(0xffffffffu, incl, l) - nt) * rows;
      r = r0 + l;
      break;
    }
    at -= (long long)__shfl_sync(0xffffffffu, incl, 31) * rows;
  }
  if (nt == 0) return;                         // (not reached while nobody writes the lengths)
  int row = (int)(at / nt), tile = (int)(at % nt);

  while (true) {
    const int h = row / p.head_blocks, hb = row % p.head_blocks;
    const int len = __ldcg(p.kv_len + r);
    const int seg = min(left, nt - tile), tile_end = tile + seg;
    const int32_t* pages = p.page_table + (size_t)r * p.max_pages_per_req;
    // queries: head c of each block, in the order in which the lanes hold a key's row
    uint32_t qf[NB][16 * S::kRow / 256 * (F8 ? 2 : 1)];
    float fac[NB][2];
    float ref[NB][2], sum[NB][2];
    float o[NB][S::kMb][4];
    {
      const float ks = F8 ? p.k_scale[h] : 1.f;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int g = hb * HB + nb * 8 + c;
        const __nv_bfloat16* q = p.q + (((size_t)r * p.n_kv_heads + h) * p.group + g) * D;
        constexpr int kQ = D / 32;             // 16-byte pieces of q a lane holds
        uint4 v[kQ];
#pragma unroll
        for (int u = 0; u < kQ; ++u) {
          // bf16 rows: piece u of lane t starts at 32 u + 8 t; 8-bit rows: 16 contiguous elements a load, two pieces
          const int d0 = F8 ? (u >> 1) * 64 + t * 16 + (u & 1) * 8 : u * 32 + t * 8;
          v[u] = g < p.group ? *reinterpret_cast<const uint4*>(q + d0) : make_uint4(0, 0, 0, 0);
        }
        float inv = 1.f;
        if constexpr (F8) {
          // fp16 after an exact scaling of the row by a power of two: its largest element comes to [2^15, 2^16)
          float top = 0.f;
#pragma unroll
          for (int u = 0; u < kQ; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t w = word(v[u], i);
              top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w << 16)), fabsf(__uint_as_float(w & 0xffff0000u))));
            }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const int e = top > 0.f ? min(126, 142 - (int)(__float_as_uint(top) >> 23)) : 0;
          const float up = __uint_as_float((uint32_t)(127 + e) << 23);
          inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
          for (int u = 0; u < kQ; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t w = word(v[u], i);
              const __half2 x = __floats2half2_rn(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up);
              qf[nb][u * 4 + i] = *reinterpret_cast<const uint32_t*>(&x);
            }
        } else {
#pragma unroll
          for (int u = 0; u < kQ; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[nb][u * 4 + i] = word(v[u], i);
        }
        // scores in powers of two; a lane's columns of S^T are the heads 2t and 2t + 1
        const float f = inv * ks * p.sm_scale * kTokLog2e;
        fac[nb][0] = __shfl_sync(0xffffffffu, f, 8 * t);
        fac[nb][1] = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll
        for (int j = 0; j < 2; ++j) { ref[nb][j] = kNoRef; sum[nb][j] = 0.f; }
#pragma unroll
        for (int i = 0; i < S::kMb; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[nb][i][k] = 0.f;
      }
    }

    uint4 kr[8], vr[8];
    // keys of this warp's step of a tile that are stored, and the page entry that holds them
    auto step_keys = [&](int tl) { return max(0, min(S::kKeys, len - (tl * S::kTile + warp * S::kKeys))); };
    auto page_at = [&](int tl) { return tl < tile_end && step_keys(tl) > 0 ? pages[(tl * S::kTile + warp * S::kKeys) / kPage] : 0; };
    auto offset = [&](int page, int tl) {
      return (((size_t)page * p.n_kv_heads + h) * kPage + (tl * S::kTile + warp * S::kKeys) % kPage) * S::kRow;
    };
    auto load_k = [&](size_t off, int n) {
      const char* b = p.k_pool + off + c * S::kRow + t * 16;
#pragma unroll
      for (int s = 0; s < 2 * S::kSub; ++s)
#pragma unroll
        for (int u = 0; u < S::kU; ++u)
          kr[s * S::kU + u] = n == S::kKeys || s * 8 + c < n ? ld16(b + s * 8 * S::kRow + u * 64) : make_uint4(0, 0, 0, 0);
    };
    auto load_v = [&](size_t off, int n) {
      const char* b = p.v_pool + off + 2 * t * S::kRow + c * 16;
#pragma unroll
      for (int s = 0; s < 4 * S::kSub; ++s)
#pragma unroll
        for (int u = 0; u < S::kV; ++u) {
          const int key = (s >> 2) * 16 + (s & 1) + ((s >> 1) & 1) * 8;      // (+ 2t: this lane's)
          vr[s * S::kV + u] = n == S::kKeys || key + 2 * t < n ? ld16(b + key * S::kRow + u * 128) : make_uint4(0, 0, 0, 0);
        }
    };
    int n0 = step_keys(tile), pg = page_at(tile), pg_next = page_at(tile + 1);
    bool bad = n0 > 0 && (pg < 0 || pg >= p.num_pages);
    size_t off = offset(pg, tile);
    if (n0 > 0 && !bad) { load_k(off, n0); load_v(off, n0); }

    for (; tile < tile_end; ++tile) {
      const bool more = tile + 1 < tile_end;
      const int n1 = more ? step_keys(tile + 1) : 0;
      const bool bad1 = n1 > 0 && (pg_next < 0 || pg_next >= p.num_pages);
      const size_t off1 = offset(pg_next, tile + 1);
      pg_next = page_at(tile + 2);
      const bool work = n0 > 0 && !bad, work1 = n1 > 0 && !bad1;
      float s[NB][S::kSub][4];
      if (work) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int b = 0; b < S::kSub; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[nb][b][k] = 0.f;
#pragma unroll
        for (int b = 0; b < S::kSub; ++b)
#pragma unroll
          for (int u = 0; u < S::kU; ++u) {
            const uint4 lo = kr[(2 * b) * S::kU + u], hi = kr[(2 * b + 1) * S::kU + u];
            if constexpr (F8) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t wl = word(lo, i), wh = word(hi, i);
                const uint32_t a[4] = {e4m3x2_to_f16x2(wl), e4m3x2_to_f16x2(wh), e4m3x2_to_f16x2(wl >> 16), e4m3x2_to_f16x2(wh >> 16)};
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) mma16816<F8>(s[nb][b], a, qf[nb][(u * 4 + i) * 2], qf[nb][(u * 4 + i) * 2 + 1]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const uint32_t a[4] = {word(lo, 2 * i), word(hi, 2 * i), word(lo, 2 * i + 1), word(hi, 2 * i + 1)};
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) mma16816<F8>(s[nb][b], a, qf[nb][u * 4 + 2 * i], qf[nb][u * 4 + 2 * i + 1]);
              }
            }
          }
      }
      if (work1) load_k(off1, n1);
      if constexpr (W) {
        if (bad) {                               // (the weights kernel reads every stored position)
          const int j0 = tile * S::kTile + warp * S::kKeys;
          float* to = p.scores + (((size_t)r * p.n_kv_heads + h) * p.max_pages_per_req * kPage + j0) * p.group;
          for (int i = lane; i < n0 * HB; i += 32)
            if (hb * HB + i % HB < p.group) to[(size_t)(i / HB) * p.group + hb * HB + i % HB] = -INFINITY;
        }
      }
      if (bad && lane == 0) atomicOr(p.status, FB_ST_BAD_PAGE);
      if (work) {
        bool move = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int b = 0; b < S::kSub; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              // rows c (k < 2) and c + 8 of the block, heads 2t and 2t + 1
              float x = s[nb][b][k] * fac[nb][k & 1];
              if (n0 < S::kKeys && b * 16 + (k >> 1) * 8 + c >= n0) x = -INFINITY;
              s[nb][b][k] = x;
              move |= x > ref[nb][k & 1] + kRebase;
            }
        if constexpr (W) {
          const int j0 = tile * S::kTile + warp * S::kKeys;
          float* to = p.scores + (((size_t)r * p.n_kv_heads + h) * p.max_pages_per_req * kPage + j0) * p.group;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const int g = hb * HB + nb * 8 + 2 * t;
#pragma unroll
            for (int b = 0; b < S::kSub; ++b)
#pragma unroll
              for (int k = 0; k < 4; k += 2) {
                const int j = b * 16 + (k >> 1) * 8 + c;
                if (j >= n0) continue;
                float* w = to + (size_t)j * p.group + g;
                if (g + 1 < p.group) *reinterpret_cast<float2*>(w) = make_float2(s[nb][b][k], s[nb][b][k + 1]);
                else if (g < p.group) *w = s[nb][b][k];
              }
          }
        }
        if (__any_sync(0xffffffffu, move)) {     // rare after the first steps: the reference goes up to the largest score
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float m = ref[nb][j];
#pragma unroll
              for (int b = 0; b < S::kSub; ++b) m = fmaxf(m, fmaxf(s[nb][b][j], s[nb][b][j + 2]));
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
              const float f = ex2(ref[nb][j] - m);
              ref[nb][j] = m;
              sum[nb][j] *= f;
#pragma unroll
              for (int i = 0; i < S::kMb; ++i) { o[nb][i][j] *= f; o[nb][i][j + 2] *= f; }
            }
        }
        uint32_t pt[NB][S::kSub][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int b = 0; b < S::kSub; ++b)
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
              const float p0 = ex2(s[nb][b][k] - ref[nb][0] + kShift), p1 = ex2(s[nb][b][k + 1] - ref[nb][1] + kShift);
              sum[nb][0] += p0;                  // (the sums are of the weights before they are rounded)
              sum[nb][1] += p1;
              uint32_t two;
              if constexpr (F8) { const __half2 x = __floats2half2_rn(p0, p1); two = *reinterpret_cast<const uint32_t*>(&x); }
              else { const __nv_bfloat162 x = __floats2bfloat162_rn(p0, p1); two = *reinterpret_cast<const uint32_t*>(&x); }
              pt[nb][b][k >> 1] = transpose8x8(two);
            }
#pragma unroll
        for (int b = 0; b < S::kSub; ++b)
#pragma unroll
          for (int i = 0; i < S::kMb; ++i) {
            // rows of O^T: d = 8c + i and 64 + 8c + i (256-byte rows), 8c + 2i and the next (128-byte bf16), 16c + 2i and the next (8-bit)
            uint32_t a[4];
            if constexpr (F8) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t w0 = word(vr[b * 4 + 2 * k], i >> 1), w1 = word(vr[b * 4 + 2 * k + 1], i >> 1);
                const uint32_t z = __byte_perm(w0, w1, i & 1 ? 0x7362 : 0x5140);
                a[2 * k] = e4m3x2_to_f16x2(z);
                a[2 * k + 1] = e4m3x2_to_f16x2(z >> 16);
              }
            } else if constexpr (D == 128) {
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                  a[2 * k + u] = __byte_perm(word(vr[(b * 4 + 2 * k) * 2 + u], i >> 1), word(vr[(b * 4 + 2 * k + 1) * 2 + u], i >> 1),
                                             i & 1 ? 0x7632 : 0x5410);
            } else {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t w0 = word(vr[b * 4 + 2 * k], i), w1 = word(vr[b * 4 + 2 * k + 1], i);
                a[2 * k] = __byte_perm(w0, w1, 0x5410);
                a[2 * k + 1] = __byte_perm(w0, w1, 0x7632);
              }
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma16816<F8>(o[nb][i], a, pt[nb][b][0], pt[nb][b][1]);
          }
      }
      if (work1) load_v(off1, n1);
      n0 = n1; bad = bad1; off = off1;
    }

    // the four warps' shares of the segment, added in order
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float l = sum[nb][j];
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
        const int g = nb * 8 + 2 * t + j;
        if (c == 0) sh_ml[warp][g] = make_float2(ref[nb][j], l);
#pragma unroll
        for (int i = 0; i < S::kMb; ++i) {
          const int lo = F8 ? 16 * c + 2 * i : D == 128 ? 8 * c + i : 8 * c + 2 * i;
          const int hi = !F8 && D == 128 ? 64 + lo : lo + 1;
          sh_o[warp][g * kStride + lo] = o[nb][i][j];
          sh_o[warp][g * kStride + hi] = o[nb][i][j + 2];
        }
      }
    __syncthreads();
    const bool begins = tile_end == seg, ends = tile_end == nt, whole = begins && ends;
    const int slot = 2 * (int)blockIdx.x + (begins ? 1 : 0);
    const float vs = F8 ? p.v_scale[h] : 1.f;
    for (int i = tid; i < HB * D; i += kTokThreads) {
      const int g = i / D, d = i % D;
      if (hb * HB + g >= p.group) break;
      float m = sh_ml[0][g].x;
#pragma unroll
      for (int w = 1; w < kTokWarps; ++w) m = fmaxf(m, sh_ml[w][g].x);
      float l = 0.f, x = 0.f;
#pragma unroll
      for (int w = 0; w < kTokWarps; ++w) {
        const float f = ex2(sh_ml[w][g].x - m);
        l += sh_ml[w][g].y * f;
        x += sh_o[w][g * kStride + d] * f;
      }
      if (whole) {
        p.out[(((size_t)r * p.n_kv_heads + h) * p.group + hb * HB + g) * D + d] = __float2bfloat16_rn(l == 0.f ? 0.f : x / l * vs);
        if constexpr (W)
          if (d == 0) p.row_ml[((size_t)r * rows + row) * HB + g] = make_float2(m, l);
      } else {
        p.part_o[((size_t)slot * HB + g) * D + d] = x;
        if (d == 0) p.part_ml[(size_t)slot * HB + g] = make_float2(m, l);
      }
    }
    left -= seg;
    if (left <= 0) break;
    __syncthreads();
    tile = 0;                                    // (the segment ended with its row: the next row starts)
    if (++row == rows) {
      row = 0;
      do { ++r; nt = tok_tiles(p, r, S::kTile); } while (nt == 0 && r < p.requests);
      if (nt == 0) break;
    }
  }
}

// ---------------------------------------------------------------- the join
// The pieces of a row: CTAs c0..c1 of the deal; piece i lies in slot 2 i + 1 where the row starts in that CTA.
struct TokPieces { long long start, share; int c0, n; };
__device__ __forceinline__ TokPieces tok_pieces(long long start, int nt, long long share) {
  TokPieces k;
  k.start = start; k.share = share;
  k.c0 = (int)(start / share);
  k.n = (int)((start + nt - 1) / share) - k.c0 + 1;
  return k;
}
__device__ __forceinline__ int tok_slot(const TokPieces& k, int i) { return 2 * (k.c0 + i) + ((k.c0 + i) * k.share <= k.start ? 1 : 0); }

// blockIdx.y < heads of a block: joins the pieces of one query head of row blockIdx.x, in order, a piece to D / 4 threads.
// Beyond (weights): adds the softmax weights of a slice of the positions of a (request, KV head).
template <int D, bool F8, int NB, bool W>
__global__ void __launch_bounds__(kTokThreads) token_join_kernel(const TokenParams p) {
  using S = TokShape<D, F8>;
  constexpr int HB = 8 * NB;
  __shared__ float fac[2 * kTokCtasPerSm * kSms];
  __shared__ float red[kTokThreads * 4];
  __shared__ float2 top[kTileM];                 // (a group has at most 128 heads)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rows = p.n_kv_heads * p.head_blocks;
  const bool weights = W && (int)blockIdx.y >= HB;
  const int r = blockIdx.x / rows, row = blockIdx.x % rows, h = row / p.head_blocks, hb = row % p.head_blocks;
  if (weights && hb != 0) return;
  if (!weights && hb * HB + (int)blockIdx.y >= p.group) return;
  // (the lengths are older than the stream kernel, which waited itself before it let this one start)
  const int nt = tok_tiles(p, r, S::kTile);
  if (nt == 0) return;
  long long before;
  const long long share = tok_share(tok_total(p, S::kTile, r, before), p.n_ctas);
  const TokPieces k = tok_pieces(before + (long long)row * nt, nt, share);
  if (!weights) {
    if (k.n == 1) return;
    pdl_wait_only();
    const int g = blockIdx.y;
    float m = kNoRef;
    for (int i = tid; i < k.n; i += kTokThreads) {
      const float2 v = p.part_ml[(size_t)tok_slot(k, i) * HB + g];
      fac[2 * i] = v.x; fac[2 * i + 1] = v.y;
      m = fmaxf(m, v.x);
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    if (lane == 0) red[warp] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    constexpr int kLanes = D / 4, kGroups = kTokThreads / kLanes;
    const int grp = tid / kLanes, d4 = tid % kLanes;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll 4
    for (int i = grp; i < k.n; i += kGroups) {
      const float f = ex2(fac[2 * i] - m);
      const float4 v = reinterpret_cast<const float4*>(p.part_o + ((size_t)tok_slot(k, i) * HB + g) * D)[d4];
      acc.x += v.x * f; acc.y += v.y * f; acc.z += v.z * f; acc.w += v.w * f;
      l += fac[2 * i + 1] * f;
    }
    __syncthreads();
    reinterpret_cast<float4*>(red)[tid] = acc;
    __shared__ float suml[kGroups];
    if (d4 == 0) suml[grp] = l;
    __syncthreads();
    if (tid < D) {
      float x = 0.f, s = 0.f;
#pragma unroll
      for (int w = 0; w < kGroups; ++w) { x += red[w * D + tid]; s += suml[w]; }
      const float vs = F8 ? p.v_scale[h] : 1.f;
      p.out[(((size_t)r * p.n_kv_heads + h) * p.group + hb * HB + g) * D + tid] = __float2bfloat16_rn(s == 0.f ? 0.f : x / s * vs);
    }
  } else if constexpr (W) {
    pdl_wait_only();
    constexpr float kShift = F8 ? 7.f : 0.f;
    // reference and sum of every query head, over the pieces of its row
    for (int g = warp; g < p.group; g += kTokWarps) {
      const int b = g / HB, gl = g % HB;
      const TokPieces q = tok_pieces(before + (long long)(row + b) * nt, nt, share);
      float m = kNoRef, l = 0.f;
      if (q.n == 1) {
        const float2 v = p.row_ml[((size_t)r * rows + row + b) * HB + gl];
        m = v.x; l = v.y;
      } else {
        for (int i = lane; i < q.n; i += 32) m = fmaxf(m, p.part_ml[(size_t)tok_slot(q, i) * HB + gl].x);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
        for (int i = lane; i < q.n; i += 32) {
          const float2 v = p.part_ml[(size_t)tok_slot(q, i) * HB + gl];
          l += v.y * ex2(v.x - m);
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
      }
      if (lane == 0) top[g] = make_float2(m - kShift, l == 0.f ? 0.f : 1.f / l);
    }
    __syncthreads();
    const int len = __ldcg(p.kv_len + r), slices = gridDim.y - HB;
    const size_t base = ((size_t)r * p.n_kv_heads + h) * p.max_pages_per_req * kPage;
    for (int j = ((int)blockIdx.y - HB) * kTokThreads + tid; j < len; j += slices * kTokThreads) {
      const float* s = p.scores + (base + j) * p.group;
      float w = 0.f;
      if (p.group % 4 == 0) {
        for (int g = 0; g < p.group; g += 4) {
          const float4 v = *reinterpret_cast<const float4*>(s + g);
          w += ex2(v.x - top[g].x) * top[g].y;
          w += ex2(v.y - top[g + 1].x) * top[g + 1].y;
          w += ex2(v.z - top[g + 2].x) * top[g + 2].y;
          w += ex2(v.w - top[g + 3].x) * top[g + 3].y;
        }
      } else {
        for (int g = 0; g < p.group; ++g) w += ex2(s[g] - top[g].x) * top[g].y;
      }
      p.kv_weight[base + j] += w;
    }
  }
}

// ---------------------------------------------------------------- host
// One CTA block of 16 heads where the group has more than 8, so that K and V are read once by groups of up to 16.
static int tok_heads(const fb_ctx* ctx) { return ctx->group > 8 ? 16 : 8; }
static int tok_ctas(const fb_ctx* ctx) { return (ctx->group > 8 ? 2 : kTokCtasPerSm) * kSms; }

struct TokWs { size_t part_ml, part_o, row_ml, scores, total; };
static TokWs tok_ws(const fb_ctx* ctx, bool weights) {
  const fb_config& c = ctx->cfg;
  const size_t hb = tok_heads(ctx), rows = (size_t)c.max_requests * c.n_kv_heads * ((ctx->group + hb - 1) / hb);
  const size_t slots = 2 * (size_t)tok_ctas(ctx);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  TokWs w;
  w.part_ml = 0;
  w.part_o = w.part_ml + up(slots * hb * sizeof(float2));
  w.row_ml = w.part_o + up(slots * hb * c.head_dim * sizeof(float));
  w.scores = w.row_ml + (weights ? up(rows * hb * sizeof(float2)) : 0);
  w.total = w.scores + (weights ? up((size_t)c.max_requests * c.n_q_heads * c.max_pages_per_req * kPage * sizeof(float)) : 0);
  return w;
}
size_t token_workspace_bytes(const fb_ctx* ctx, bool weights) { return tok_ws(ctx, weights).total; }

template <int D, bool F8, int NB, bool W>
static int launch_token(fb_ctx* ctx, const TokenParams& p, cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  if (int e = cuda_err(ctx, launch_pdl(token_attn_kernel<D, F8, NB, W>, p.n_ctas, kTokThreads, 0, stream, p), "token_attn_kernel launch"))
    return e;
  const long long rows = (long long)c.max_requests * c.n_kv_heads * p.head_blocks, pairs = (long long)c.max_requests * c.n_kv_heads;
  const long long blocks = ((long long)c.max_pages_per_req * kPage + kTokThreads - 1) / kTokThreads;
  const long long want = 1 + 8 * kSms / pairs;
  const int slices = W ? (int)(want < blocks ? want : blocks) : 0;
  return cuda_err(ctx, launch_pdl(token_join_kernel<D, F8, NB, W>, dim3((unsigned)rows, 8 * NB + slices), kTokThreads, 0, stream, p),
                  "token_join_kernel launch");
}
template <int D, bool F8>
static int launch_token(fb_ctx* ctx, const TokenParams& p, bool weights, cudaStream_t stream) {
  if (ctx->group > 8) return weights ? launch_token<D, F8, 2, true>(ctx, p, stream) : launch_token<D, F8, 2, false>(ctx, p, stream);
  return weights ? launch_token<D, F8, 1, true>(ctx, p, stream) : launch_token<D, F8, 1, false>(ctx, p, stream);
}

int launch_token_attn(fb_ctx* ctx, const fb_cache* kv, const void* q, const void* k_pool, const void* v_pool,
                      const float* k_scale, const float* v_scale, void* out, int accumulate, void* ws, int32_t* status,
                      cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  const TokWs w = tok_ws(ctx, accumulate != 0);
  char* base = static_cast<char*>(ws);
  const int hb = tok_heads(ctx);
  if ((long long)c.max_requests * c.n_q_heads > 0x7fffffffll)
    return set_err(ctx, FB_ERR_UNSUPPORTED, "max_requests * n_q_heads must be below 2^31");
  TokenParams p;
  p.kv_len = kv->kv_len; p.page_table = kv->page_table; p.kv_weight = kv->kv_weight;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k_pool = static_cast<const char*>(k_pool); p.v_pool = static_cast<const char*>(v_pool);
  p.k_scale = k_scale; p.v_scale = v_scale; p.out = static_cast<__nv_bfloat16*>(out); p.status = status;
  p.part_ml = reinterpret_cast<float2*>(base + w.part_ml);
  p.part_o = reinterpret_cast<float*>(base + w.part_o);
  p.row_ml = reinterpret_cast<float2*>(base + w.row_ml);
  p.scores = reinterpret_cast<float*>(base + w.scores);
  p.requests = c.max_requests; p.group = ctx->group; p.n_kv_heads = c.n_kv_heads;
  p.head_blocks = (ctx->group + hb - 1) / hb;
  p.max_pages_per_req = c.max_pages_per_req; p.num_pages = c.num_pages; p.n_ctas = tok_ctas(ctx);
  p.sm_scale = ctx->sm_scale;
  if (c.kv_fp8) return launch_token<128, true>(ctx, p, accumulate, stream);
  return c.head_dim == 128 ? launch_token<128, false>(ctx, p, accumulate, stream)
                           : launch_token<64, false>(ctx, p, accumulate, stream);
}

}  // namespace fb
