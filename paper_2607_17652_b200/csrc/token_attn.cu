// fb_token_attn: one query token per request over everything its pages hold,
//   out = sum_j w_j V_j,  w = softmax(sm_scale q K^T),  j < kv_len,
// for all query heads of a KV head at once, so that every stored key and value crosses the memory bus once.
//
// HBM-bound: 4 d operations per key and query head against 2 d values read per key and KV head.
//
// Work.  The keys of a (request, KV head) are cut into tiles, and the tiles of the whole batch, one row behind the
// other, are dealt to the CTAs in equal contiguous shares, whatever the lengths: a row that a CTA holds whole is
// finished by it, one that is cut leaves a piece (reference, sum, unnormalised output) per CTA, and token_join_kernel
// adds the pieces in their order.  A CTA starts at most one row that it does not finish and finishes at most one that it
// did not start, so two slots a CTA hold all pieces, however large the batch.  (Adding them in the CTA that finds all
// pieces of a row there saves the launch, and its fences and polls cost more than the launch boundary: one request of
// 3,001 keys 9.8 -> 13.0 us, 24 requests 20.6 -> 23.6.)
//
// A warp has 16 keys of a tile (32 where a row is 128 bytes) and works alone until its share ends:
//   S^T = K Q^T   (m16n8k16: 16 keys, 8 query heads; padded to 8)   and   O^T += V^T P^T  (16 of d, 8 heads)
// both on registers that the loads fill directly.  A contraction may take its index in any order as long as
// both operands agree, and so may the rows of an output: a lane loads 16 contiguous bytes of a key's row, which are
// the A fragments of two k-steps, and of the rows 2t, 2t+1, 2t+8, 2t+9 of V the 16 bytes that its eight (row block, row)
// places need; pairs of V rows are interleaved by byte permutes, P^T is S^T's fragment transposed by movmatrix.  No
// shared memory, no barrier, no address arithmetic but one base per step, and the next step's K and V are in flight
// while this one's products run.  The tensor pipe (legacy mma.sync) is far from its rate: 16 d multiply-adds a key for a
// block of 8 heads against 4 d bytes from memory (2 d in 8 bits).
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "fb_common.cuh"

namespace fb {

constexpr int kTokThreads = 128, kTokWarps = kTokThreads / 32;
constexpr int kTokCtasPerSm = 3;         // (2 where a block has 16 heads: twice the accumulators)
constexpr float kTokLog2e = 1.4426950408889634f;
constexpr float kNoRef = -3.0e38f;       // below every score: the reference of a row that has seen no key
constexpr float kRebase = 8.f;           // a score that far (in powers of two) above the reference moves it
// fp16 weights start 2^7 above 1 (the reference lies that far below the score that set it), so that 2^-31 is still there
template <bool F8> constexpr float kTokShift = F8 ? 7.f : 0.f;

using bf16 = __nv_bfloat16;

struct TokPieces;
struct TokenParams {
  const int32_t *kv_len, *page_table;
  float* kv_weight;
  const bf16* q;
  const char *k_pool, *v_pool;
  const float *k_scale, *v_scale;        // 8-bit pages: [n_kv_heads]
  bf16* out;
  int32_t* status;
  float* part_o;                         // [2 n_ctas][heads of a block][d] unnormalised outputs of the pieces
  float2* part_ml;                       // [2 n_ctas][heads of a block] reference (log2), sum
  int2* cut;                             // [n_ctas] row that a CTA has begun and not finished, its pieces (0: none) (more than kDealAgain requests)
  TokPieces* row_pieces;                 // [rows] (the same requests, weights only)
  float2* row_ml;                        // [rows][heads of a block] reference and sum of rows that were not cut (weights only)
  float* scores;                         // [requests][KV heads][capacity][group] (log2; weights only)
  int32_t requests, group, n_kv_heads, head_blocks, max_pages_per_req, num_pages, n_ctas, join_ctas;
  float sm_scale;
};

// Caches of at most kFewCapacity keys in at most kFewRows (request, KV head) rows take a cluster each, where no weights are
// asked for.  us, dealt / a cluster each (32 query and 8 KV heads of 128, GPU time): one request of 200 keys 5.4 / 5.1, of 700 6.9 /
// 5.6, of 3,001 8.4 / 7.9, of 8,192 12.9 / 14.1; 4 requests of 500 to 3,000 keys 12.0 / 11.2, of 1,000 to 8,192 18.5 / 20.8; 16
// requests of 500 to 2,000 19.2 / 21.3; with weights one request of 3,001 9.1 / 10.5.  And one launch less for the host.  These in
// contexts whose capacity is the longest length; the capacity is all that the host knows, and room above the lengths costs:
// one request of 200, 700 and 3,001 keys takes 6.4, 6.6 and 8.0 where the capacity is 4,096, 5.4, 6.6 and 8.4 (dealt) where it is 32,768.
constexpr int kFewCapacity = 4096, kFewRows = 32;

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
static_assert(TokShape<128, false>::kKeys * TokShape<128, false>::kRow == 32 * 128 && TokShape<64, false>::kKeys * TokShape<64, false>::kRow == 32 * 128,
              "the keys of a step are a line a lane");
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
// four E4M3 bytes -> two pairs of fp16 (exact)
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(four));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// ---------------------------------------------------------------- the deal
// Tiles of `len` stored keys (none where there is no request, nothing stored or the length is no length).
__device__ __forceinline__ int tok_tiles(const TokenParams& p, int len, int tile) {
  return len > 0 && len <= (long long)p.max_pages_per_req * kPage ? (len - 1) / tile + 1 : 0;
}
__device__ __forceinline__ int tok_len(const TokenParams& p, int r) { return r < p.requests ? __ldcg(p.kv_len + r) : 0; }
__device__ __forceinline__ long long tok_div(long long a, long long b) {        // (both below 2^31 but in absurd contexts)
  return (a | b) >> 31 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}
// Tiles of all rows (`total`) and of those of the requests before `upto`, and the share of a CTA: an equal one, but with few rows
// at least sqrt(tiles of the longest / 32): a share takes its time tile by tile, the join 32 pieces at a time, and this is where
// both together are least.  us, a row in at most 64 / 128 / 256 / 444 pieces (one request, 8 query heads on one KV head, GPU time):
// 8,192 keys (128 tiles) 8.0 / 8.7 / 8.7 / 8.7, 32,768 13.3 / 11.8 / 13.8 / 13.9, 131,072 42.5 / 27.4 / 24.0 / 24.4.
// By a whole warp; `len`: the lane's length of the first 32 requests.
struct TokDeal { long long total, before, share; };
__device__ __forceinline__ TokDeal tok_deal(const TokenParams& p, int tile, int len, int upto) {
  const int lane = threadIdx.x & 31, rows = p.n_kv_heads * p.head_blocks;
  const int n0 = tok_tiles(p, len, tile);
  int longest = n0;
  long long all, before;
  if (p.requests <= 32) {                        // (32 counts below 2^25 each)
    all = __reduce_add_sync(0xffffffffu, n0);
    before = __reduce_add_sync(0xffffffffu, lane < upto ? n0 : 0);
  } else {
    all = n0;
    before = lane < upto ? n0 : 0;
#pragma unroll 8
    for (int r = 32 + lane; r < p.requests; r += 32) {
      const int n = tok_tiles(p, __ldcg(p.kv_len + r), tile);
      all += n;
      before += r < upto ? n : 0;
      longest = max(longest, n);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      all += __shfl_xor_sync(0xffffffffu, all, o);
      before += __shfl_xor_sync(0xffffffffu, before, o);
    }
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  TokDeal d;
  d.total = all * rows;
  d.before = before * rows;
  d.share = max(max(tok_div(d.total + p.n_ctas - 1, p.n_ctas), (long long)__float2int_rn(__fsqrt_rn(longest / 32.f))), 1ll);
  return d;
}
// The pieces of a row: of CTAs c0, c0 + 1, ...  The first lies in the odd slot of its CTA (the row starts in it), the others in the
// even ones.
struct __align__(8) TokPieces {
  int c0, n;
  __device__ __forceinline__ int slot(int i) const { return 2 * (c0 + i) + (i == 0 ? 1 : 0); }
};
__device__ __forceinline__ TokPieces tok_pieces(long long start, int nt, long long share) {
  TokPieces k;
  k.c0 = (int)tok_div(start, share);
  k.n = (int)tok_div(start + nt - 1, share) - k.c0 + 1;
  return k;
}
// Up to as many requests a CTA of the join has a row and finds its pieces from the lengths, while the stream still runs; for more the
// stream leaves what it has cut per CTA: a CTA leaves one row at most, most rows are whole, and a look at all lengths by
// every CTA of the join takes longer than one read more behind the stream.
constexpr int kDealAgain = 32;

// ---------------------------------------------------------------- the stream
// A warp's share of the keys of query heads [hb * 8 NB, ...) of (request r, KV head h): `steps` steps of S::kKeys keys from key
// `first` on, kStep keys apart (0: step_), of the len that are stored.  Steps may lie behind them.  Leaves reference, sum (of this
// lane's keys) and O^T in the lane's places.
template <int D, bool F8, int NB, bool W, int kStep>
__device__ __forceinline__ void tok_stream(const TokenParams& p, int r, int h, int hb, int len, int first, int steps, int step_,
                                           float (&ref)[NB][2], float (&sum)[NB][2], float (&o)[NB][TokShape<D, F8>::kMb][4]) {
  using S = TokShape<D, F8>;
  constexpr int HB = 8 * NB;
  constexpr float kShift = kTokShift<F8>;
  const int lane = threadIdx.x & 31, c = lane >> 2, t = lane & 3, step = kStep ? kStep : step_;
  // `rem` keys are stored from the step's first one on, `entry` is the page table's entry for it.  Its place inside a page is
  // the same in every step (`step` is whole pages).
  int rem = len - first;
  const int in_page = first % kPage;
  const int32_t* entry = p.page_table + (size_t)r * p.max_pages_per_req + first / kPage;
  const size_t page_bytes = (size_t)p.n_kv_heads * kPage * S::kRow;
  const size_t in_head = ((size_t)h * kPage + in_page) * S::kRow;
  // the page of a step that is `ahead` steps on: only read where that step has keys
  auto page_ahead = [&](int ahead) { return steps > ahead && rem > ahead * step ? __ldcg(entry + ahead * (step / kPage)) : 0; };
  int page0 = page_ahead(0), page1 = page_ahead(1);
  uint4 kr[8], vr[8];
  // (n keys of the step are stored; what lies behind them is not read)
  auto load_k = [&](size_t off, int n) {
    const char* b = p.k_pool + off + c * S::kRow + t * 16;
#pragma unroll
    for (int s = 0; s < 2 * S::kSub; ++s)
#pragma unroll
      for (int u = 0; u < S::kU; ++u)
        kr[s * S::kU + u] = n >= S::kKeys || s * 8 + c < n ? ld16(b + s * 8 * S::kRow + u * 64) : make_uint4(0, 0, 0, 0);
  };
  auto load_v = [&](size_t off, int n) {
    const char* b = p.v_pool + off + 2 * t * S::kRow + c * 16;
#pragma unroll
    for (int s = 0; s < 4 * S::kSub; ++s)
#pragma unroll
      for (int u = 0; u < S::kV; ++u) {
        const int key = (s >> 2) * 16 + (s & 1) + ((s >> 1) & 1) * 8;      // (+ 2t: this lane's)
        vr[s * S::kV + u] = n >= S::kKeys || key + 2 * t < n ? ld16(b + key * S::kRow + u * 128) : make_uint4(0, 0, 0, 0);
      }
  };
  auto inside = [&](int page) { return (unsigned)page < (unsigned)p.num_pages; };
  // (the stream starts before the queries are looked at)
  bool work = rem > 0 && inside(page0);
  if (work) { load_k(page0 * page_bytes + in_head, rem); load_v(page0 * page_bytes + in_head, rem); }
  // The step behind it into L2, a line a lane, while the CTAs still start or change rows and DRAM has time: 64 requests of 1,024 to
  // 8,192 keys, 32 heads on 8 of 128 183 -> 180 us, in 8 bits 103 -> 101, 64 on 4 117 -> 113; 128 of 100 to 600 42.0 -> 40.6; 256 of 64 to
  // 256 45.5 -> 46.1.  (A second step 43 for the 128, 50 for the 256; in the kernel of few rows no gain.)
  auto to_l2 = [&](size_t off) {
    asm volatile("prefetch.global.L2 [%0];" :: "l"(p.k_pool + off + lane * 128));
    asm volatile("prefetch.global.L2 [%0];" :: "l"(p.v_pool + off + lane * 128));
  };
  if constexpr (kStep > 0)
    if (steps > 1 && rem > step && inside(page1)) to_l2(page1 * page_bytes + in_head);
  // queries: head c of each block, in the order in which the lanes hold a key's row
  uint32_t qf[NB][16 * S::kRow / 256 * (F8 ? 2 : 1)];
  float fac[NB][2];
  {
    const float ks = F8 ? p.k_scale[h] : 1.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int g = hb * HB + nb * 8 + c;
      const bf16* q = p.q + (((size_t)r * p.n_kv_heads + h) * p.group + g) * D;
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
        // fp16 after an exact scaling of the row by a power of two: its largest element comes to [2^15, 2^16), so that the
        // elements down to 2^-32 of it are exact (fp16 ends at 2^-24, a bf16 has 8 bits) and no other is off by more than 2^-40 of it
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

  [[maybe_unused]] float* score = nullptr;     // of this warp's first key of the step
  if constexpr (W)
    score = p.scores + (((size_t)r * p.n_kv_heads + h) * p.max_pages_per_req * kPage + first) * p.group + hb * HB;

  for (; steps > 0; --steps) {
    const bool work1 = steps > 1 && rem > step && inside(page1);
    const size_t off1 = page1 * page_bytes + in_head;
    const int page2 = page_ahead(2);
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
              uint32_t a[4];
              e4m3x4_to_f16(word(lo, i), a[0], a[2]);
              e4m3x4_to_f16(word(hi, i), a[1], a[3]);
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
    if (work1) load_k(off1, rem - step);
    if (rem > 0 && !work) {                    // a page outside the pool: its keys are left out
      if (lane == 0) atomicOr(p.status, FB_ST_BAD_PAGE);
      if constexpr (W)                         // (the scores of every stored position are read again)
        for (int i = lane; i < min(rem, S::kKeys) * HB; i += 32)
          if (hb * HB + i % HB < p.group) score[(size_t)(i / HB) * p.group + i % HB] = -INFINITY;
    }
    if (work) {
      bool move = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          // rows c and c + 8 of each block of keys, head 2t + j
          float top = kNoRef;
#pragma unroll
          for (int b = 0; b < S::kSub; ++b) {
            s[nb][b][j] *= fac[nb][j];
            s[nb][b][j + 2] *= fac[nb][j];
            if (rem < S::kKeys) {
              if (b * 16 + c >= rem) s[nb][b][j] = -INFINITY;
              if (b * 16 + 8 + c >= rem) s[nb][b][j + 2] = -INFINITY;
            }
            top = fmaxf(top, fmaxf(s[nb][b][j], s[nb][b][j + 2]));
          }
          move |= top > ref[nb][j] + (kRebase + kShift);
        }
      if constexpr (W) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          if (hb * HB + nb * 8 + 2 * t < p.group) {                // (this lane's heads of the block)
            float* w = score + c * p.group + nb * 8 + 2 * t;
#pragma unroll
            for (int b = 0; b < 2 * S::kSub; ++b) {
              if (rem >= S::kKeys || b * 8 + c < rem) {
                const float x = s[nb][b >> 1][2 * (b & 1)], y = s[nb][b >> 1][2 * (b & 1) + 1];
                if (p.group > 1) *reinterpret_cast<float2*>(w) = make_float2(x, y);
                else *w = x;
              }
              w += 8 * p.group;
            }
          }
      }
      if (__any_sync(0xffffffffu, move)) {     // rare after the first steps: the reference goes up to the largest score
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float m = ref[nb][j] + kShift;
#pragma unroll
            for (int b = 0; b < S::kSub; ++b) m = fmaxf(m, fmaxf(s[nb][b][j], s[nb][b][j + 2]));
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
            m -= kShift;
            const float f = ex2(ref[nb][j] - m);
            ref[nb][j] = m;
            sum[nb][j] *= f;
#pragma unroll
            for (int i = 0; i < S::kMb; ++i) { o[nb][i][j] *= f; o[nb][i][j + 2] *= f; }
          }
      }
      // The weights are rounded to the 16 bits that the second product takes, by at most 2^-8 of themselves in bf16 (2^-11 in fp16):
      // outputs are 2.3e-3 from 64 bits in the 2-norm, 1.7e-3 were they rounded once at the end, as in the block attention.  Their
      // remainders as a second operand would double the instructions and the registers of this product.
      uint32_t pt[NB][S::kSub][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < S::kSub; ++b)
#pragma unroll
          for (int k = 0; k < 4; k += 2) {
            const float p0 = ex2(s[nb][b][k] - ref[nb][0]), p1 = ex2(s[nb][b][k + 1] - ref[nb][1]);
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
              e4m3x4_to_f16(__byte_perm(w0, w1, i & 1 ? 0x7362 : 0x5140), a[2 * k], a[2 * k + 1]);
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
    if (work1) load_v(off1, rem - step);
    // And all along with 2 CTAs on an SM, whose loads of one step do not cover the latency of DRAM: 32 heads on 2 of 128, 64 requests
    // of 1,024 to 8,192 keys 68.1 -> 66.8 us, 64 on 2 119 -> 115, 128 on 8, 16 requests of 16,384 to 32,768 270 -> 255; a step further ahead
    // is slower, and so is any with 3 CTAs: 184.5 -> 188.8.
    if constexpr (NB > 1)
      if (steps > 2 && rem > 2 * step && inside(page2)) to_l2(page2 * page_bytes + in_head);
    work = work1;
    page1 = page2;
    rem -= step;
    entry += step / kPage;
    if constexpr (W) score += step * p.group;
  }
}

// A warp's results to shared memory: reference and sum of every head, O as [head][D + 1].
template <int D, bool F8, int NB>
__device__ __forceinline__ void tok_put(const float (&ref)[NB][2], const float (&sum)[NB][2], const float (&o)[NB][TokShape<D, F8>::kMb][4],
                                        float2* ml, float* to) {
  using S = TokShape<D, F8>;
  const int lane = threadIdx.x & 31, c = lane >> 2, t = lane & 3;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float l = sum[nb][j];
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
      const int g = nb * 8 + 2 * t + j;
      if (c == 0) ml[g] = make_float2(ref[nb][j], l);
#pragma unroll
      for (int i = 0; i < S::kMb; ++i) {
        const int lo = F8 ? 16 * c + 2 * i : D == 128 ? 8 * c + i : 8 * c + 2 * i;
        const int hi = !F8 && D == 128 ? 64 + lo : lo + 1;
        to[g * (D + 1) + lo] = o[nb][i][j];
        to[g * (D + 1) + hi] = o[nb][i][j + 2];
      }
    }
}

template <int D, bool F8, int NB, bool W>
__global__ void __launch_bounds__(kTokThreads, NB == 1 ? 3 : 2) token_attn_kernel(const TokenParams p) {
  using S = TokShape<D, F8>;
  constexpr int HB = 8 * NB, kStride = D + 1;
  __shared__ float sh_o[kTokWarps][HB * kStride];
  __shared__ float2 sh_ml[kTokWarps][HB];
  __shared__ int sh_share;
  pdl_wait_then_release();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rows = p.n_kv_heads * p.head_blocks;
  if (tid == 0 && p.requests > kDealAgain) p.cut[blockIdx.x] = make_int2(0, 0);      // (the same thread sets it)
  int len = tok_len(p, lane);
  const TokDeal deal = tok_deal(p, S::kTile, len, 0);
  long long at = (long long)blockIdx.x * deal.share;
  int left = (int)min(deal.share, deal.total - at > 0 ? deal.total - at : 0);
  if (left <= 0) return;
  if (tid == 0) sh_share = (int)min(deal.share, 0x7fffffffll);       // (read behind the barrier at the end of a segment)
  // the request that holds tile `at`, its length and tiles; 128 lengths under way at a time
  int r = 0, nt = 0;
  if (p.requests == 1) {
    len = __shfl_sync(0xffffffffu, len, 0);
    nt = tok_tiles(p, len, S::kTile);
  }
  for (int r0 = 0; r0 < p.requests && nt == 0; r0 += 128) {
    int lens[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) lens[u] = r0 + u == 0 ? len : r0 + 32 * u < p.requests ? tok_len(p, r0 + 32 * u + lane) : 0;
#pragma unroll 1
    for (int u = 0; u < 4 && nt == 0; ++u) {
      const int mine = u == 0 ? lens[0] : u == 1 ? lens[1] : u == 2 ? lens[2] : lens[3], n = tok_tiles(p, mine, S::kTile);
      int incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      const unsigned here = __ballot_sync(0xffffffffu, at < (long long)incl * rows);
      if (here) {
        const int l = __ffs(here) - 1;
        nt = __shfl_sync(0xffffffffu, n, l);
        len = __shfl_sync(0xffffffffu, mine, l);
        at -= (long long)(__shfl_sync(0xffffffffu, incl, l) - nt) * rows;
        r = r0 + 32 * u + l;
      } else {
        at -= (long long)__shfl_sync(0xffffffffu, incl, 31) * rows;
      }
    }
  }
  if (nt == 0) return;                         // (not reached while nobody writes the lengths)
  int row = (int)tok_div(at, nt), tile = (int)(at - (long long)row * nt);

  while (true) {
    const int h = row / p.head_blocks, hb = row % p.head_blocks;
    const int seg = min(left, nt - tile), tile_end = tile + seg;
    float ref[NB][2], sum[NB][2], o[NB][S::kMb][4];
    tok_stream<D, F8, NB, W, S::kTile>(p, r, h, hb, len, tile * S::kTile + warp * S::kKeys, seg, 0, ref, sum, o);
    tile = tile_end;

    tok_put<D, F8, NB>(ref, sum, o, sh_ml[warp], sh_o[warp]);
    __syncthreads();
    const bool begins = tile_end == seg, whole = begins && tile_end == nt;
    const int slot = 2 * (int)blockIdx.x + (begins ? 1 : 0);
    const float vs = F8 ? p.v_scale[h] : 1.f;
    bf16* out = p.out + (((size_t)r * p.n_kv_heads + h) * p.group + hb * HB) * D;
    const int heads = min(HB, p.group - hb * HB);
    if (begins && tid == 0 && p.requests > kDealAgain) {
      const int rest = nt - seg;                 // of the row, to the CTAs behind this one
      const TokPieces k{(int)blockIdx.x, 1 + rest / sh_share + (rest % sh_share ? 1 : 0)};
      if (W) p.row_pieces[(size_t)r * rows + row] = k;
      if (rest) p.cut[blockIdx.x] = make_int2(r * rows + row, k.n);
    }
    // (four heads at once: 64 requests, 64 heads on 4 112.1 -> 110.1 us, 125 short ones, 16 on one 18.5 -> 17.9, the rest within 1 %)
#pragma unroll 4
    for (int i = tid; i < heads * D; i += kTokThreads) {
      const int g = i / D, d = i % D;
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
        out[i] = __float2bfloat16_rn(l == 0.f ? 0.f : x / l * vs);
        if (W && d == 0) p.row_ml[((size_t)r * rows + row) * HB + g] = make_float2(m, l);
      } else {
        p.part_o[(size_t)slot * HB * D + i] = x;
        if (d == 0) p.part_ml[(size_t)slot * HB + g] = make_float2(m, l);
      }
    }
    left -= seg;
    if (left <= 0) break;
    __syncthreads();                             // (sh_o is read no more)
    tile = 0;                                    // (the segment ended with its row: the next row starts)
    if (++row == rows) {
      row = 0;
      do { ++r; len = tok_len(p, r); nt = tok_tiles(p, len, S::kTile); } while (nt == 0 && r < p.requests);
      if (nt == 0) break;
    }
  }
}

// ---------------------------------------------------------------- few rows
// The keys of a row in one cluster, whose warps take them in turn: with few rows and short caches the pieces meet in distributed
// shared memory, and neither a deal nor a second launch is needed.
template <int NB> constexpr int kFewWarps = NB == 1 ? 6 : 4;
template <int D, bool F8, int NB>
__global__ void __launch_bounds__(kFewWarps<NB> * 32, 2) token_few_kernel(const TokenParams p) {
  namespace cg = cooperative_groups;
  using S = TokShape<D, F8>;
  constexpr int HB = 8 * NB, kWarps = kFewWarps<NB>, kThreads = kWarps * 32, kMaxCluster = 16;
  __shared__ float sh_o[kWarps][HB * (D + 1)];
  __shared__ float2 sh_ml[kWarps][HB];
  __shared__ float part_o[HB * D];               // of this CTA
  __shared__ float2 part_ml[HB];
  cg::cluster_group cluster = cg::this_cluster();
  const int cl = (int)cluster.num_blocks(), me = (int)cluster.block_rank();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const int line = blockIdx.x / cl, r = line / p.n_kv_heads, h = line % p.n_kv_heads, heads = p.group;       // (one block of heads)
  const int len = __ldcg(p.kv_len + r);
  bf16* out = p.out + (size_t)line * heads * D;
  // (the CTAs of a cluster leave together here or meet at the barriers below)
  if (len < 0) return;
  if (len > (long long)p.max_pages_per_req * kPage) {
    if (me == 0 && h == 0 && tid == 0) atomicOr(p.status, FB_ST_BAD_STATE);
    return;
  }
  if (len == 0) {
    if (me == 0)
      for (int i = tid; i < heads * (D / 8); i += kThreads) reinterpret_cast<uint4*>(out)[i] = make_uint4(0, 0, 0, 0);
    return;
  }
  float ref[NB][2], sum[NB][2], o[NB][S::kMb][4];
  const int first = (me * kWarps + warp) * S::kKeys, step = cl * kWarps * S::kKeys, steps = len > first ? (len - first + step - 1) / step : 0;
  tok_stream<D, F8, NB, false, 0>(p, r, h, 0, len, first, steps, step, ref, sum, o);
  tok_put<D, F8, NB>(ref, sum, o, sh_ml[warp], sh_o[warp]);
  const float vs = F8 ? p.v_scale[h] : 1.f;
  __syncthreads();
  for (int i = tid; i < heads * D; i += kThreads) {
    const int g = i / D, d = i % D;
    float m = sh_ml[0][g].x;
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sh_ml[w][g].x);
    float l = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2(sh_ml[w][g].x - m);
      l += sh_ml[w][g].y * f;
      x += sh_o[w][g * (D + 1) + d] * f;
    }
    if (cl == 1) { out[i] = __float2bfloat16_rn(l == 0.f ? 0.f : x / l * vs); continue; }
    part_o[i] = x;
    if (d == 0) part_ml[g] = make_float2(m, l);
  }
  if (cl == 1) return;
  cluster.sync();
  // the CTAs' pieces in order; a CTA forms its share of the outputs
  const int share = (heads * D + cl - 1) / cl;
  for (int i = me * share + tid; i < min(heads * D, (me + 1) * share); i += kThreads) {
    float2 ml[kMaxCluster];
    float v[kMaxCluster], m = kNoRef, l = 0.f, x = 0.f;
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q)
      if (q < cl) {
        ml[q] = *cluster.map_shared_rank(&part_ml[i / D], q);
        v[q] = *cluster.map_shared_rank(&part_o[i], q);
        m = fmaxf(m, ml[q].x);
      }
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q)
      if (q < cl) {
        const float f = ex2(ml[q].x - m);
        l += ml[q].y * f;
        x += v[q] * f;
      }
    out[i] = __float2bfloat16_rn(l == 0.f ? 0.f : x / l * vs);
  }
  cluster.sync();                                // (no CTA leaves while another may read its piece)
}

// ---------------------------------------------------------------- the join
// kv_weight[r, h, j] += sum over the group of exp(score - reference) / sum, from the scores that the stream has left, for
// the positions of a slice, a position to a thread.  16 bytes of scores a key for a group of four, written and read,
// against 256 to 512 of K and V: cheaper than forming them again.
constexpr int kWeightAt = 4;                     // positions of a thread at once
__device__ __forceinline__ void add_weights(const TokenParams& p, const float2* top, size_t base, int len, int slice, int slices) {
  constexpr int kStep = kWeightAt * kTokThreads;
  for (long long j0 = (long long)slice * kStep + threadIdx.x; j0 < len; j0 += (long long)slices * kStep) {
    float w[kWeightAt], old[kWeightAt];
#pragma unroll
    for (int u = 0; u < kWeightAt; ++u) {
      w[u] = 0.f;
      old[u] = j0 + u * kTokThreads < len ? __ldcg(p.kv_weight + base + j0 + u * kTokThreads) : 0.f;
    }
    if (p.group % 4 == 0) {
      for (int g = 0; g < p.group; g += 4) {
        float4 v[kWeightAt];
#pragma unroll
        for (int u = 0; u < kWeightAt; ++u)
          v[u] = j0 + u * kTokThreads < len ? __ldcg(reinterpret_cast<const float4*>(p.scores + (base + j0 + u * kTokThreads) * p.group + g))
                                            : make_float4(0.f, 0.f, 0.f, 0.f);
        const float2 a = top[g], b = top[g + 1], x = top[g + 2], y = top[g + 3];
#pragma unroll
        for (int u = 0; u < kWeightAt; ++u) {
          w[u] += ex2(v[u].x - a.x) * a.y; w[u] += ex2(v[u].y - b.x) * b.y;
          w[u] += ex2(v[u].z - x.x) * x.y; w[u] += ex2(v[u].w - y.x) * y.y;
        }
      }
    } else {
      for (int g = 0; g < p.group; ++g)
#pragma unroll
        for (int u = 0; u < kWeightAt; ++u)
          if (j0 + u * kTokThreads < len) w[u] += ex2(__ldcg(p.scores + (base + j0 + u * kTokThreads) * p.group + g) - top[g].x) * top[g].y;
    }
#pragma unroll
    for (int u = 0; u < kWeightAt; ++u)
      if (j0 + u * kTokThreads < len) p.kv_weight[base + j0 + u * kTokThreads] = old[u] + w[u];
  }
}

// blockIdx.y < p.join_ctas: joins the pieces of every join_ctas-th query head of row blockIdx.x, in order, a piece to D / 4
// threads.  Beyond (weights): a slice of the positions of a (request, KV head).
template <int D, bool F8, int NB, bool W>
__global__ void __launch_bounds__(kTokThreads) token_join_kernel(const TokenParams p) {
  using S = TokShape<D, F8>;
  constexpr int HB = 8 * NB, kLanes = D / 4, kGroups = kTokThreads / kLanes, kAhead = 8;
  __shared__ float2 ml[kTokCtasPerSm * kSms];    // (a CTA leaves one piece of a row)
  __shared__ float4 red[kTokThreads];
  __shared__ float sums[kTokWarps], tops[kTokWarps];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rows = p.n_kv_heads * p.head_blocks;
  const bool weights = W && (int)blockIdx.y >= p.join_ctas;
  // (the kernel behind this one waits for this one alone: one CTA at least has to have waited for the stream; the lengths are
  // older than the stream kernel, which waited itself before it let this one start)
  const bool keeper = blockIdx.x == 0 && blockIdx.y == 0, again = p.requests <= kDealAgain;
  // zeros where nothing is stored, a report where the length is no length; the output only behind the wait, before which
  // the stream's predecessors may still read or write it
  auto empty_row = [&](int of, int n) {
    if (n > (long long)p.max_pages_per_req * kPage && tid == 0) atomicOr(p.status, FB_ST_BAD_STATE);
    if (n != 0) return;
    pdl_wait_only();
    uint4* o = reinterpret_cast<uint4*>(p.out) + (size_t)of * p.n_kv_heads * p.group * (D / 8);
    for (int i = tid; i < p.n_kv_heads * p.group * (D / 8); i += kTokThreads) o[i] = make_uint4(0, 0, 0, 0);
  };
  int r = blockIdx.x / rows, row = blockIdx.x % rows, len = 0, nt = 0;
  TokPieces k{0, 1};
  TokDeal deal{};
  if (again || weights) {                        // CTA x has row x
    if (r >= p.requests) return;                 // (the grid is wide enough for the CTAs of the deal too)
    const int first = again ? tok_len(p, lane) : 0;
    len = tok_len(p, r);
    nt = tok_tiles(p, len, S::kTile);
    if (!weights && blockIdx.y == 0 && row == 0) empty_row(r, len);
    const bool idle = nt == 0 || (weights && row % p.head_blocks != 0);
    if (idle && !keeper) return;
    if (again && nt > 0) {
      deal = tok_deal(p, S::kTile, first, r);
      k = tok_pieces(deal.before + (long long)row * nt, nt, deal.share);
    }
    if (keeper || weights || k.n > 1) pdl_wait_only();
    if (idle) return;
  } else {                                       // CTA x has the row that CTA x of the stream has begun and not finished
    if ((int)blockIdx.x >= p.n_ctas) return;
    if (blockIdx.y == 0)
      for (int of = blockIdx.x; of < p.requests; of += p.n_ctas) empty_row(of, tok_len(p, of));
    pdl_wait_only();
    const int2 cut = __ldcg(p.cut + blockIdx.x);
    if (cut.y == 0) return;
    k = TokPieces{(int)blockIdx.x, cut.y};
    r = cut.x / rows;
    row = cut.x % rows;
  }
  const int h = row / p.head_blocks, hb = row % p.head_blocks;
  auto pieces_of = [&](int of) {
    if (again) return tok_pieces(deal.before + (long long)of * nt, nt, deal.share);
    const int2 v = __ldcg(reinterpret_cast<const int2*>(p.row_pieces) + (size_t)r * rows + of);
    return TokPieces{v.x, v.y};
  };
  if (!weights) {
    if (k.n == 1) return;
    const int heads = min(HB, p.group - hb * HB);
    bf16* out = p.out + (((size_t)r * p.n_kv_heads + h) * p.group + hb * HB) * D;
    // Few pieces: a warp a head, without barriers (64 requests of 1,024 to 8,192 keys, 64 heads on 4: 121.7 -> 116.1 us, 32 on 8 185.8 ->
    // 184.0; 128 of 100 to 600 43.2 -> 41.0).
    if (k.n <= kAhead) {
      for (int g = blockIdx.y * kTokWarps + warp; g < heads; g += p.join_ctas * kTokWarps) {
        constexpr int kSide = 32 / kLanes;       // pieces side by side
        const int side = lane / kLanes, d4 = lane % kLanes;
        float4 v[kAhead / kSide];
#pragma unroll
        for (int u = 0; u < kAhead / kSide; ++u) {
          const int i = u * kSide + side;
          v[u] = i < k.n ? __ldcg(reinterpret_cast<const float4*>(p.part_o + ((size_t)k.slot(i) * HB + g) * D) + d4) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        const float2 x = lane < k.n ? __ldcg(p.part_ml + (size_t)k.slot(lane) * HB + g) : make_float2(kNoRef, 0.f);
        const float vs = F8 ? p.v_scale[h] : 1.f;
        float m = x.x;
#pragma unroll
        for (int o = 1; o < kAhead; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        m = __shfl_sync(0xffffffffu, m, 0);
        const float f = lane < k.n ? ex2(x.x - m) : 0.f;
        float l = x.y * f;
#pragma unroll
        for (int o = 1; o < kAhead; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        l = __shfl_sync(0xffffffffu, l, 0);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < kAhead / kSide; ++u) {
          const float w = __shfl_sync(0xffffffffu, f, u * kSide + side);
          acc.x += v[u].x * w; acc.y += v[u].y * w; acc.z += v[u].z * w; acc.w += v[u].w * w;
        }
        if constexpr (kSide == 2) {
          acc.x += __shfl_xor_sync(0xffffffffu, acc.x, 16); acc.y += __shfl_xor_sync(0xffffffffu, acc.y, 16);
          acc.z += __shfl_xor_sync(0xffffffffu, acc.z, 16); acc.w += __shfl_xor_sync(0xffffffffu, acc.w, 16);
        }
        const float s = l == 0.f ? 0.f : 1.f / l;
        const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x * s * vs, acc.y * s * vs), hi = __floats2bfloat162_rn(acc.z * s * vs, acc.w * s * vs);
        if (side == 0)
          reinterpret_cast<uint2*>(out + (size_t)g * D)[d4] = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      }
      return;
    }
    for (int g = blockIdx.y; g < heads; g += p.join_ctas) {
      const int grp = tid / kLanes, d4 = tid % kLanes;
      const float vs = F8 ? p.v_scale[h] : 1.f;
      // the outputs of the first pieces are under way while references and sums are put together
      auto piece = [&](int i) { return __ldcg(reinterpret_cast<const float4*>(p.part_o + ((size_t)k.slot(i) * HB + g) * D) + d4); };
      float4 v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = grp + u * kGroups < k.n ? piece(grp + u * kGroups) : make_float4(0.f, 0.f, 0.f, 0.f);
      float m = kNoRef;
      for (int i = tid; i < k.n; i += kTokThreads) {
        const float2 x = __ldcg(p.part_ml + (size_t)k.slot(i) * HB + g);
        ml[i] = x;
        m = fmaxf(m, x.x);
      }
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
      if (lane == 0) tops[warp] = m;
      __syncthreads();
      m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i0 = grp; i0 < k.n; i0 += kAhead * kGroups) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int i = i0 + u * kGroups, next = i + kAhead * kGroups;
          if (i < k.n) {
            const float f = ex2(ml[i].x - m);
            acc.x += v[u].x * f; acc.y += v[u].y * f; acc.z += v[u].z * f; acc.w += v[u].w * f;
          }
          if (next < k.n) v[u] = piece(next);
        }
      }
      float l = 0.f;
      for (int i = tid; i < k.n; i += kTokThreads) l += ml[i].y * ex2(ml[i].x - m);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
      if (lane == 0) sums[warp] = l;
      red[tid] = acc;
      __syncthreads();
      if (tid < D) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kGroups; ++w) x += reinterpret_cast<const float*>(red)[w * D + tid];
        const float s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        out[(size_t)g * D + tid] = __float2bfloat16_rn(s == 0.f ? 0.f : x / s * vs);
      }
      __syncthreads();
    }
  } else if constexpr (W) {
    __shared__ float2 top[kTileM];               // reference, 1 / sum (a group has at most 128 heads)
    // Heads by warps; where a warp would have four or more, those of few pieces by threads (64 requests of 1,024 to 8,192 keys, 64 heads
    // on 4: 148.4 -> 144.1 us; 8 heads on one 22.1 -> 22.4, 4 on one the same).
    bool by_warps = NB == 1;
    if constexpr (NB > 1) {
      if (tid < p.group) {
        const int b = tid / HB, gl = tid % HB;
        const TokPieces q = pieces_of(row + b);
        by_warps = q.n > kAhead;
        if (!by_warps) {
          float2 v[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i)
            v[i] = i >= q.n ? make_float2(kNoRef, 0.f) : __ldcg(q.n == 1 ? p.row_ml + ((size_t)r * rows + row + b) * HB + gl
                                                                          : p.part_ml + (size_t)q.slot(i) * HB + gl);
          float m = kNoRef, l = 0.f;
#pragma unroll
          for (int i = 0; i < kAhead; ++i) m = fmaxf(m, v[i].x);
#pragma unroll
          for (int i = 0; i < kAhead; ++i) l += v[i].y * ex2(v[i].x - m);
          top[tid] = make_float2(m, l == 0.f ? 0.f : 1.f / l);
        }
      }
      by_warps = __syncthreads_or(by_warps);
    }
    if (by_warps) {
      for (int g = warp; g < p.group; g += kTokWarps) {
        const int b = g / HB, gl = g % HB;
        const TokPieces q = pieces_of(row + b);
        if (NB > 1 && q.n <= kAhead) continue;
        float m = kNoRef, l = 0.f;
        if (q.n == 1) {
          const float2 v = __ldcg(p.row_ml + ((size_t)r * rows + row + b) * HB + gl);
          m = v.x; l = v.y;
        } else {
          for (int i0 = 0; i0 < q.n; i0 += 32) {   // running reference and sum, 32 pieces at a time
            const float2 v = i0 + lane < q.n ? __ldcg(p.part_ml + (size_t)q.slot(i0 + lane) * HB + gl) : make_float2(kNoRef, 0.f);
            float mx = fmaxf(m, v.x);
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
            float add = v.y * ex2(v.x - mx);
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) add += __shfl_xor_sync(0xffffffffu, add, x);
            l = l * ex2(m - mx) + add;
            m = mx;
          }
        }
        if (lane == 0) top[g] = make_float2(m, l == 0.f ? 0.f : 1.f / l);
      }
    }
    __syncthreads();
    add_weights(p, top, ((size_t)r * p.n_kv_heads + h) * p.max_pages_per_req * kPage, len, blockIdx.y - p.join_ctas, gridDim.y - p.join_ctas);
  }
}

// ---------------------------------------------------------------- host
// One CTA block of 16 heads where the group has more than 8, so that K and V are read once by groups of up to 16.
static int tok_heads(const fb_ctx* ctx) { return ctx->group > 8 ? 16 : 8; }
static int tok_ctas(const fb_ctx* ctx) { return (ctx->group > 8 ? 2 : kTokCtasPerSm) * kSms; }

struct TokWs { size_t part_ml, part_o, cut, row_pieces, row_ml, scores, total; };
static TokWs tok_ws(const fb_ctx* ctx, bool weights) {
  const fb_config& c = ctx->cfg;
  const size_t hb = tok_heads(ctx), rows = (size_t)c.max_requests * c.n_kv_heads * ((ctx->group + hb - 1) / hb);
  const size_t slots = 2 * (size_t)tok_ctas(ctx);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  TokWs w;
  w.part_ml = 0;
  w.part_o = w.part_ml + up(slots * hb * sizeof(float2));
  w.cut = w.part_o + up(slots * hb * c.head_dim * sizeof(float));
  w.row_pieces = w.cut + (c.max_requests > kDealAgain ? up(tok_ctas(ctx) * sizeof(int2)) : 0);
  w.row_ml = w.row_pieces + (weights && c.max_requests > kDealAgain ? up(rows * sizeof(TokPieces)) : 0);
  w.scores = w.row_ml + (weights ? up(rows * hb * sizeof(float2)) : 0);
  w.total = w.scores + (weights ? up((size_t)c.max_requests * c.n_q_heads * c.max_pages_per_req * kPage * sizeof(float)) : 0);
  return w;
}
size_t token_workspace_bytes(const fb_ctx* ctx, bool weights) { return tok_ws(ctx, weights).total; }

// CTAs of a cluster that takes a row (0: the rows are dealt): as many as two an SM allow, at most sixteen, and no more than
// the capacity has work for.
static int tok_cluster(const fb_ctx* ctx, int block_heads, int keys) {
  const fb_config& c = ctx->cfg;
  const long long rows = (long long)c.max_requests * c.n_kv_heads, cap = (long long)c.max_pages_per_req * kPage;
  if (ctx->group > block_heads || cap > kFewCapacity || rows > kFewRows) return 0;
  int cl = 16;
  while (cl > 1 && (rows * cl > 2 * kSms || cl / 2 * keys >= cap)) cl /= 2;
  return cl;
}

template <int D, bool F8, int NB, bool W>
static int launch_token(fb_ctx* ctx, const TokenParams& p, cudaStream_t stream) {
  const fb_config& c = ctx->cfg;
  if constexpr (!W) {
    if (const int cl = tok_cluster(ctx, 8 * NB, kFewWarps<NB> * TokShape<D, F8>::kKeys)) {
      const auto kernel = token_few_kernel<D, F8, NB>;
      int dev = 0;
      if (int e = cuda_err(ctx, cudaGetDevice(&dev), "cudaGetDevice")) return e;
      if (cl > 8 && ctx->token_device != dev) {       // (sixteen have to be asked for; the context remembers where it has)
        if (int e = cuda_err(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1), "cluster attr")) return e;
        ctx->token_device = dev;
      }
      return cuda_err(ctx, launch_pdl_cluster(kernel, (unsigned)(c.max_requests * c.n_kv_heads * cl), kFewWarps<NB> * 32, 0, stream, cl, p),
                      "token_few_kernel launch");
    }
  }
  if (int e = cuda_err(ctx, launch_pdl(token_attn_kernel<D, F8, NB, W>, p.n_ctas, kTokThreads, 0, stream, p), "token_attn_kernel launch"))
    return e;
  // (slices by the rows of the context, since what they hold is only known on the device: one request of 28,123 keys with weights takes
  // 24.5 us alone in its context, 33.3 as the only one of 64 rows)
  const long long pairs = (long long)c.max_requests * c.n_kv_heads, step = kWeightAt * kTokThreads;
  const long long blocks = ((long long)c.max_pages_per_req * kPage + step - 1) / step, want = 1 + 12 * kSms / pairs;
  const int slices = W ? (int)(want < blocks ? want : blocks) : 0;
  const long long rows = pairs * p.head_blocks, joins = c.max_requests <= kDealAgain ? rows : p.n_ctas;
  const long long x = W && rows > joins ? rows : joins;
  return cuda_err(ctx, launch_pdl(token_join_kernel<D, F8, NB, W>, dim3((unsigned)x, p.join_ctas + slices), kTokThreads, 0, stream, p),
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
  p.q = static_cast<const bf16*>(q);
  p.k_pool = static_cast<const char*>(k_pool); p.v_pool = static_cast<const char*>(v_pool);
  p.k_scale = k_scale; p.v_scale = v_scale; p.out = static_cast<bf16*>(out); p.status = status;
  p.part_ml = reinterpret_cast<float2*>(base + w.part_ml);
  p.part_o = reinterpret_cast<float*>(base + w.part_o);
  p.cut = reinterpret_cast<int2*>(base + w.cut);
  p.row_pieces = reinterpret_cast<TokPieces*>(base + w.row_pieces);
  p.row_ml = reinterpret_cast<float2*>(base + w.row_ml);
  p.scores = reinterpret_cast<float*>(base + w.scores);
  p.requests = c.max_requests; p.group = ctx->group; p.n_kv_heads = c.n_kv_heads;
  p.head_blocks = (ctx->group + hb - 1) / hb;
  p.max_pages_per_req = c.max_pages_per_req; p.num_pages = c.num_pages; p.n_ctas = tok_ctas(ctx);
  // (a CTA a head where rows that are cut are few, fewer where they may fill the machine)
  const long long rows = (long long)c.max_requests * c.n_kv_heads * p.head_blocks, per_row = 8 * kSms / (rows < p.n_ctas ? rows : p.n_ctas);
  const int heads = ctx->group < hb ? ctx->group : hb;
  p.join_ctas = per_row < 1 ? 1 : per_row < heads ? (int)per_row : heads;
  p.sm_scale = ctx->sm_scale;
  if (c.kv_fp8) return launch_token<128, true>(ctx, p, accumulate, stream);
  return c.head_dim == 128 ? launch_token<128, false>(ctx, p, accumulate, stream)
                           : launch_token<64, false>(ctx, p, accumulate, stream);
}

}  // namespace fb
