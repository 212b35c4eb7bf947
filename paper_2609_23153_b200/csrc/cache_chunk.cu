// sparkattn_cache_fwd for many query rows per key head (prompts, frames, drafts of many tokens): attention over a paged
// cache on the tensor cores, bf16 or E4M3 pages.
//
// The products, 4 d flops per (row, key), bound it, so an item is 256 query rows of one (sequence, key head): two M = 128
// tiles that share every key tile, since fetching a tile and turning codes into operands costs shared-memory
// bandwidth, which the products themselves use to three quarters (Q and K from shared memory: 64 KB per 128 x 128 x 128).
// SPLIT: where no sequence has more than 128 rows, an item is one M tile, and the two halves of the pipeline take its key tiles in
// turns and add up at the end; each would otherwise wait for itself most of the time.
// The line of all items' key tiles (cache_line.cuh) is cut evenly over one CTA per SM.  Roles:
//   warp 0       TMA producer: pages of K and of V, scales, one descriptor per 16 keys
//   warp 1       issues S_g = Q K^T and O_g += P_g V (tcgen05, accumulators in TMEM: S0 | S1 | O0 | O1)
//   warps 4-7    E4M3: V's codes -> fp16 operand tiles (exact), 64-channel heads K's as well.  Both: V rows that no row of the item
//                sees become zeros, since a page holds anything behind its sequence's last token, and 0 times that need not be 0
//   warps 8-11, 12-15   softmax of half 0 / 1, a thread per row: S from TMEM, weights back over the same columns as the second product's
//                operand, running reference (lazy: O is rescaled only when a weight would pass 2^10), output
// While one softmax warpgroup works on its S, the tensor core runs the other one's PV and next S; tcgen05.mma of one thread
// run in the order of issue, so S_g of the next tile may overwrite the columns that PV_g has read its P from.
// E4M3, 128 channels: K's codes are the first product's operand as they are, against the queries in two E4M3 parts
// (split_queries): twice as many products at twice the rate.  P and V are fp16 (the weights 2^5 at the reference), and V's scale is part of the
// exponent: t = logit + log2(v_scale), the row sum adds weight / v_scale.  bf16 pages: bf16 throughout, the weights too, since A and B of a
// product have one type: out is then 2.0-2.3e-3 from the result in 64 bits, where its own rounding is 1.7e-3.  Weights in two bf16 parts,
// the second one in the other half of S's columns, give 1.7e-3, and half as many products again: three frames of 1560 tokens 851 -> 1184 us, four
// prompts 550 -> 774, five drafted tokens of 8 sequences 69 -> 78.  So one part here, two with few rows, where the memory's time hides the second.
// Measured (E4M3, 128 channels; a library product of bf16 matrices reaches 1704 TFLOP/s in a burst, 1439 for seconds): 4680 new tokens,
// three frames, over 32,760, 12 heads, 897 GFLOP in 807-815 us = 1100-1110 TFLOP/s, called for seconds, at 1.6 GHz and less under the power limit, 897: tensor cores and
// special-function unit are busy 52 % of the clocks each, the rest is the chain that a half goes through once a tile, S, maximum, exponentials, P V.
// Pieces of 2048 tokens of four prompts of up to 8000, 32 heads over 8, causal by token: 507 GFLOP in 500-540 us = 940-1010 TFLOP/s; a causal
// tile at the border costs as much as a whole one.  SPLIT: five drafted tokens of 8 sequences of up to 16,383, 64 heads over 8: 145 MB in 63 us;
// 1 us a tile per SM, a chain of copy, conversion, product, softmax and product that only two tiles at a time share.
// Through a window with first tokens (SINK): the same three frames over five frames up to their own and the first, 269 GFLOP in 296 us = 910 TFLOP/s; pieces of
// 2048 tokens of four prompts, window 1500 and 100 tokens, bf16, 145 GFLOP in 195 us: items are 14 tiles long, and what lies between two of them, 8 us, is a
// fifth of the time (the queries' copies and conversion 2-5, the last product and the output 1-3).  Tried on that without gain: queries' loops
// unrolled, masks by groups of sixteen keys (spills), tiles that a warp sees nothing of done at once, halves of an item that leave tiles to each other where
// rows lie in two frames (293 instead of 297, for a hundred lines), whole output rows through quads of lanes (prompts 2 % faster, drafts 2 % slower).
// (A quarter of the exponentials as a polynomial of degree 4 on the FMA pipe, to spare the special-function unit: 870 us
// either way for three frames of 1560 tokens over 32,760 keys, 710 instead of 672 for four prompts.)
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "cache_line.cuh"
#include "tmap.h"

namespace sparkattn {

constexpr int kChunkKeys = 128, kChunkThreads = 512;
constexpr int kChunkOver = 6;                                   // tiles that the beginning and the end of an item take as long as
constexpr int kChunkGroups = kChunkKeys / 16;
constexpr int kSoftRegs = 208, kConvRegs = 48, kCtrlRegs = 48;      // 2 x 128 x 208 + 2 x 128 x 48 = 512 x 128
constexpr int kChunkInfoRing = 8;                                   // tiles whose descriptors are kept: the K ring and what is still worked on

template <int D, bool FP8>
struct ChunkShape {
  static constexpr bool kRawK = FP8 && D == 128;            // K's codes are an operand
  static constexpr bool kConvK = FP8 && !kRawK;
  static constexpr int kOperand = kChunkKeys * D * 2;       // a 128 x D tile of 16-bit operands: slabs of 64 channels
  static constexpr int kCodes = kChunkKeys * D;             // the same as E4M3 codes
  static constexpr int kQ = kOperand;                       // of one M tile (kRawK: high parts, then low parts)
  static constexpr int kK = kRawK ? kCodes : kOperand;
  static constexpr int RK = kRawK ? 3 : 2, RV = 2;          // rings: K operands, V operands (and V codes)
  static constexpr int kOffK = 2 * kQ, kOffV = kOffK + RK * kK, kOffRaw = kOffV + RV * kOperand;      // raw: V codes, then (kConvK) K codes
  static constexpr int kOffMisc = kOffRaw + (FP8 ? RV * kCodes : 0) + (kConvK ? kCodes : 0);
  static constexpr int kFixed = kOffMisc + 256 /* barriers */ + kChunkInfoRing * kChunkGroups * (int)sizeof(GroupInfo) + 128 + 128 * 8 /* SPLIT: row sums */;
};

// What the logits of a row and 16 keys are multiplied by, kept from 0: a row of zeros has 2^-126 here and a page of zeros 2^-48, whose product
// underflows, and a masked logit, -inf, times 0 would be NaN.  Logits that this changes are below 2^-100.  A NaN, of a broken row, stays.
__device__ __forceinline__ float logit_factor(float row, float key) {
  float c = row * key;
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(c) : "f"(1.17549435e-38f));
  return c;
}

template <int D, bool FP8, bool SPLIT, bool SINK>
__global__ void __launch_bounds__(kChunkThreads, 1)
cache_chunk_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                   const __grid_constant__ CacheFwdParams p) {
  using C = ChunkShape<D, FP8>;
  constexpr int R = SPLIT ? 128 : 256;
  using L = Line<R, kChunkKeys, kChunkOver, SINK>;
  constexpr int kSlab = kChunkKeys * 128;                    // bytes of 64 16-bit channels, or of 128 codes
  constexpr int RK = C::RK, RV = C::RV;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sQ = smem;
  unsigned char* sK = smem + C::kOffK;
  unsigned char* sV = smem + C::kOffV;
  unsigned char* sRaw = smem + C::kOffRaw;
  unsigned char* sRawK = sRaw + RV * C::kCodes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffMisc);
  uint64_t* q_full = bars;            // [2] the item's queries are in shared memory (SPLIT: [0], both warpgroups')
  uint64_t* k_full = bars + 2;        // [RK] operand K tile (its copies; kConvK: 128 arrivals)
  uint64_t* k_free = bars + 5;        // [RK] the S products that read it are complete
  uint64_t* v_full = bars + 8;        // [RV] 128 arrivals
  uint64_t* v_free = bars + 10;       // [RV] the PV products that read it are complete
  uint64_t* raw_full = bars + 12;     // [RV] the copies of a V tile (E4M3: as codes)
  uint64_t* raw_free = bars + 14;     // [RV] E4M3, 128 arrivals
  uint64_t* rawk_full = bars + 16;    // kConvK: the copies of a K tile
  uint64_t* rawk_free = bars + 17;
  uint64_t* s_full = bars + 18;       // [2] S_g complete: the product's arrival and its issuer's (who has seen the tile's descriptor)
  uint64_t* p_full = bars + 20;       // [2] 128 arrivals: weights written, S_g read
  uint64_t* pv_done = bars + 22;      // [2] O_g complete up to a tile: the product's arrival and its issuer's (who has seen V's operand)
  uint64_t* sums_full = bars + 24;    // SPLIT, 128 arrivals: warpgroup 1 has left its row sums, and its O is complete
  uint64_t* sums_free = bars + 25;    // SPLIT, 128 arrivals: they have been taken
  GroupInfo* s_info = reinterpret_cast<GroupInfo*>(bars + 32);          // [ring][groups]
  float2* s_sums = reinterpret_cast<float2*>(s_info + kChunkInfoRing * kChunkGroups);      // [128]
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_sums + 128);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_bad = reinterpret_cast<int*>(s_tmem + 2);
  int* s_warp = s_bad + 2;            // [16]
  int* s_prefix = reinterpret_cast<int*>(smem);       // [B + 1], until every warp has found its place in the line
  const Marks<D, R, FP8> marks{reinterpret_cast<uint32_t*>(smem + C::kFixed)};
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  marks.clear_all();
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full + i, SPLIT ? 256 : 128);
      mbar_init(v_full + i, 128); mbar_init(v_free + i, 1);
      mbar_init(raw_full + i, 1); mbar_init(raw_free + i, 128);
      mbar_init(s_full + i, 2); mbar_init(p_full + i, 128); mbar_init(pv_done + i, 2);
    }
    for (int i = 0; i < RK; ++i) { mbar_init(k_full + i, C::kConvK ? 128 : 1); mbar_init(k_free + i, 1); }
    mbar_init(rawk_full, 1); mbar_init(rawk_free, 128);
    mbar_init(sums_full, 128); mbar_init(sums_free, 128);
    mbar_fence_init();
    *s_abort = 0;
  }
  if (warp == 0) {
    tmem_alloc(s_tmem, 512);
    tmem_relinquish();
  }
  pdl_wait();
  tc_fence_before();
  L::lay_out(p, s_prefix, s_warp);                           // (its barriers also stand between the set-up above and the roles)
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  const int total = s_prefix[p.batch.B], share = L::share_of(p, total);
  if (blockIdx.x == 0) check_call<SINK>(p, s_bad);
  const long long begin = (long long)((int)blockIdx.x - 1) * share;
  const bool works = blockIdx.x > 0 && begin < total;
  const int x0 = works ? (int)begin : 0, x1 = works ? (int)min(begin + share, (long long)total) : 0;
  Stretch<R, kChunkKeys, kChunkOver, SINK> g;
  if (works) g.begin(p, s_prefix, x0, x1);
  if (blockIdx.x > 0 && threadIdx.x == 0) note_border(p, (int)blockIdx.x - 1, works, share, g);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // tiles go where the line's beginnings lie
  __syncthreads();
  if (warp < 4) reg_dec<kCtrlRegs>();
  else if (warp < 8) reg_dec<kConvRegs>();
  if (!works) {
    // fall through to the teardown
  } else if (warp == 0) {
    // --------------------------------------------------------------------------------------------------- copies
    // The stretch goes by in batches of four tiles of a segment, of whose groups of 16 keys every lane looks after one.  Pages are
    // asked for two batches ahead and scales one, across segments.
    constexpr int kBatch = 32 / kChunkGroups;
    GroupBatch now, next, after;
    int t_next = g.t0;
    bool live = true;
    auto ask_pages = [&](GroupBatch& b) {
      while (live && t_next >= g.t1) {
        live = g.next(p);
        t_next = g.t0;
      }
      b = {t_next, live ? min(kBatch, g.t1 - t_next) : 0, g.c.h, 0, -1, 1.0f, 1.0f};
      const int key = SINK ? g.c.item.tile_of(b.t + lane / kChunkGroups) * kChunkKeys + lane % kChunkGroups * 16 : b.t * kChunkKeys + lane * 16;
      if constexpr (SINK) b.key = key;
      if (lane / kChunkGroups < b.n && key < g.c.item.hi && (key + 16 > g.c.item.lo || (SINK && key < p.causal.sink)))
        b.page = p.batch.page_table[(int64_t)g.c.b * p.batch.max_pages + (key >> p.batch.page_shift)];
      t_next += b.n;
    };
    int n = 0;                                               // tiles so far
    bool ok = true;
    const int per_box = kChunkGroups / p.boxes;              // groups of a box
    ask_pages(now);
    ask_pages(next);
    ask_scales<FP8>(p, now);
    while (ok && now.n > 0) {
      // a box is copied if somebody sees one of its groups; the lane of its first group copies it
      int page = now.page;
      if (per_box > 1) page = max(page, __shfl_xor_sync(0xffffffffu, page, 1));
      if (per_box > 2) page = max(page, __shfl_xor_sync(0xffffffffu, page, 2));
      if (per_box > 4) page = max(page, __shfl_xor_sync(0xffffffffu, page, 4));
      const bool copies = page >= 0 && lane % per_box == 0;
      const uint32_t going = __ballot_sync(0xffffffffu, copies);
      const int key = SINK ? now.key : now.t * kChunkKeys + lane * 16, row = key & ((1 << p.batch.page_shift) - 1), at_row = (lane % kChunkGroups) * 16;
      const GroupInfo info = info_of<FP8>(now);
      ask_scales<FP8>(p, next);
      ask_pages(after);
      for (int u = 0; ok && u < now.n; ++u, ++n) {
        const bool my_tile = lane / kChunkGroups == u;
        const int boxes = __popc((going >> (u * kChunkGroups)) & ((1u << kChunkGroups) - 1u));
        // K, then V: as codes that are an operand or become one, or (bf16) where the products read them
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const int slot = kv ? n % RV : C::kConvK ? 0 : n % RK, uses = kv ? n / RV : C::kConvK ? n : n / RK;
          uint64_t* freed = kv ? (FP8 ? raw_free : v_free) + slot : C::kConvK ? rawk_free : k_free + slot;
          uint64_t* full = kv ? raw_full + slot : C::kConvK ? rawk_full : k_full + slot;
          if (uses > 0) ok = __all_sync(0xffffffffu, pipe_wait(freed, (uses - 1) & 1, s_abort, 1 + kv));
          if (!ok) break;
          if (my_tile && copies) {
            const CUtensorMap* map = kv ? &tmap_v : &tmap_k;
            if constexpr (FP8) {
              unsigned char* dst = kv ? sRaw + slot * C::kCodes : C::kConvK ? sRawK : sK + slot * C::kK;
              tma_load_4d(dst + at_row * D, map, full, 0, row, now.h, page);
            } else {
#pragma unroll
              for (int sl = 0; sl < D / 64; ++sl)
                tma_load_4d((kv ? sV : sK) + slot * C::kOperand + sl * kSlab + at_row * 128, map, full, sl * 64, row, now.h, page);
            }
          }
          if (kv == 0) {
            if (my_tile) s_info[(n & (kChunkInfoRing - 1)) * kChunkGroups + lane % kChunkGroups] = info;
            __syncwarp();
          }
          if (lane == 0) {
            if (boxes) mbar_expect_tx(full, boxes * p.box_rows * D * (FP8 ? 1 : 2));
            else mbar_arrive(full);
          }
        }
      }
      now = next;
      next = after;
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------------- products
    constexpr uint32_t idesc_s = make_idesc(FP8 ? 0u : 1u, 128, kChunkKeys, false);       // (E4M3 and fp16 are both 0, each in its kind)
    constexpr uint32_t idesc_o = make_idesc(FP8 ? 0u : 1u, 128, D, true);
    const uint32_t k_hi = (uint32_t)(make_smem_desc_sw128(0, 16) >> 32);
    const uint32_t q_lo = (uint32_t)make_smem_desc_sw128(smem_u32(sQ), 16), k_lo = (uint32_t)make_smem_desc_sw128(smem_u32(sK), 16);
    const uint32_t v_hi = (uint32_t)(make_smem_desc_sw128(0, kSlab) >> 32);
    const uint32_t v_lo = (uint32_t)make_smem_desc_sw128(smem_u32(sV), kSlab);
    int n = 0;                                                // tiles in front of the segment
    uint32_t done[2] = {0, 0}, loaded[2] = {0, 0};            // weights taken and queries seen of half 0, 1
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity, int id) { return __all_sync(0xffffffffu, pipe_wait(bar, parity, s_abort, id)) != 0; };
    // S of tile `at` for half w; `last`: nothing else reads the K tile
    auto s_product = [&](int w, int at, bool last) {
      tc_fence_after();
      if (elect_one()) {
        const uint32_t qa = q_lo + (((SPLIT ? 0 : w) * C::kQ) >> 4), ka = k_lo + (((at % RK) * C::kK) >> 4);
        if constexpr (C::kRawK) {
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_ss<true>(tmem + w * 128, make_desc(qa + ((part * kSlab + kk * 32) >> 4), k_hi), make_desc(ka + ((kk * 32) >> 4), k_hi), idesc_s,
                           (part | kk) != 0 ? 1u : 0u);
        } else {
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_ss<false>(tmem + w * 128, make_desc(qa + ((sl * kSlab + kk * 32) >> 4), k_hi), make_desc(ka + ((sl * kSlab + kk * 32) >> 4), k_hi),
                            idesc_s, (sl | kk) != 0 ? 1u : 0u);
        }
        tc_commit(s_full + w);
        mbar_arrive(s_full + w);
        if (last) tc_commit(k_free + at % RK);
      }
      __syncwarp();
    };
    // O of half w plus the weights times tile `at` (first: instead of what O held)
    auto o_product = [&](int w, int at, bool first, bool last) {
      tc_fence_after();
      if (elect_one()) {
        const uint32_t va = v_lo + (((at % RV) * C::kOperand) >> 4);
#pragma unroll
        for (int kk = 0; kk < kChunkKeys / 16; ++kk)
          mma_ts<false>(tmem + 256 + w * 128, tmem + w * 128 + kk * 8, make_desc(va + ((kk * 16 * 128) >> 4), v_hi), idesc_o, first && kk == 0 ? 0u : 1u);
        tc_commit(pv_done + w);
        mbar_arrive(pv_done + w);
        if (last) tc_commit(v_free + at % RV);
      }
      __syncwarp();
    };
    do {
      const int tiles = g.t1 - g.t0;
      if (tiles == 0) continue;
      if constexpr (SPLIT) {
        // half i & 1 takes tile i
        ok = wait(q_full, loaded[0]++ & 1, 4);
        for (int i = 0; ok && i < min(tiles, 2); ++i) {
          ok = wait(k_full + (n + i) % RK, ((n + i) / RK) & 1, 3);
          if (ok) s_product(i, n + i, true);
        }
        for (int i = 0; ok && i < tiles; ++i) {
          const int w = i & 1;
          ok = wait(v_full + (n + i) % RV, ((n + i) / RV) & 1, 5) && wait(p_full + w, done[w]++ & 1, 6);
          if (!ok) break;
          o_product(w, n + i, i < 2, true);
          if (i + 2 < tiles) {
            ok = wait(k_full + (n + i + 2) % RK, ((n + i + 2) / RK) & 1, 7);
            if (ok) s_product(w, n + i + 2, true);
          }
        }
      } else {
        const int halves = g.rows > 128 ? 2 : 1;
        ok = wait(k_full + n % RK, (n / RK) & 1, 3);
        for (int w = 0; ok && w < halves; ++w) {
          ok = wait(q_full + w, loaded[w]++ & 1, 4);
          if (ok) s_product(w, n, w == halves - 1);
        }
        for (int i = 0; ok && i < tiles; ++i) {
          ok = wait(v_full + (n + i) % RV, ((n + i) / RV) & 1, 5);
          for (int w = 0; ok && w < halves; ++w) {
            ok = wait(p_full + w, done[w]++ & 1, 6);
            if (!ok) break;
            o_product(w, n + i, i == 0, w == halves - 1);
            if (i + 1 < tiles) {
              if (w == 0) ok = wait(k_full + (n + i + 1) % RK, ((n + i + 1) / RK) & 1, 7);
              if (ok) s_product(w, n + i + 1, w == halves - 1);
            }
          }
        }
      }
      n += tiles;
    } while (ok && g.next(p));
  } else if (warp >= 4 && warp < 8) {
    // -------------------------------------------------------------------------------------------------- operands
    const int tid = threadIdx.x - 128;
    int n = 0, segment = 0;
    bool ok = true;
    // a tile of codes as fp16 operands
    auto convert = [&](const unsigned char* codes, unsigned char* operand) {
      const uint32_t raw = smem_u32(codes), to = smem_u32(operand);
      constexpr int kCh = D / 16, kRowsAtOnce = 128 / kCh;                // 16-code chunks of a row
      const int c = tid % kCh;
      const bool swap = D == 128 && c >= 4;                               // (the lanes of a row write eight different banks at a time)
#pragma unroll 4
      for (int r0 = 0; r0 < kChunkKeys; r0 += kRowsAtOnce) {
        const int r = r0 + tid / kCh;
        const uint32_t from = D == 128 ? raw + r * 128 + ((c ^ (r & 7)) << 4) : raw + r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from));
        const uint32_t x[4] = {swap ? v.z : v.x, swap ? v.w : v.y, swap ? v.x : v.z, swap ? v.y : v.w};
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) e4m3_to_half(x[i], h[2 * i], h[2 * i + 1]);
        const uint32_t dst = to + (c >> 2) * kSlab + r * 128;
        const int ck = (c & 3) * 2;
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst + (((ck + swap) ^ (r & 7)) << 4)), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst + (((ck + !swap) ^ (r & 7)) << 4)), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
      }
    };
    do {
      // keys that every row of the item sees
      const int all_lo = visible_keys(p.causal, g.c.seq.first_pos() + fast_div(g.row0 + g.rows - 1, p.by_G), g.c.seq.len).x;
      const int all_hi = visible_keys(p.causal, g.c.seq.first_pos() + fast_div(g.row0, p.by_G), g.c.seq.len).y;
      const bool parts = all_lo > g.c.item.lo || all_hi < g.c.item.hi;
      for (int t = g.t0; ok && t < g.t1; ++t, ++n) {
        const int key0 = g.c.item.tile_of(t) * kChunkKeys;
        const GroupInfo* info = s_info + (n & (kChunkInfoRing - 1)) * kChunkGroups;
        if constexpr (C::kConvK) {
          ok = __all_sync(0xffffffffu, pipe_wait(rawk_full, n & 1, s_abort, 8));
          if (ok && n >= RK) ok = __all_sync(0xffffffffu, pipe_wait(k_free + n % RK, (n / RK - 1) & 1, s_abort, 10));
          if (!ok) break;
          convert(sRawK, sK + (n % RK) * C::kK);
          mbar_arrive(rawk_free);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(k_full + n % RK);
        }
        const int slot = n % RV;
        ok = __all_sync(0xffffffffu, pipe_wait(raw_full + slot, (n / RV) & 1, s_abort, 9));
        if (FP8 && ok && n >= RV) ok = __all_sync(0xffffffffu, pipe_wait(v_free + slot, (n / RV - 1) & 1, s_abort, 11));
        if (!ok) break;
        const bool edge = (key0 < all_lo && !(SINK && key0 + kChunkKeys <= p.causal.sink)) || key0 + kChunkKeys > all_hi || __any_sync(0xffffffffu, lane < kChunkGroups && !info[lane % kChunkGroups].usable);
        if (edge) {
          // V's words: zeros for keys that nobody sees; and see Marks.  (E4M3: every thread what it converts next)
          constexpr int kPer = FP8 ? 16 : 8, kLanes = FP8 ? D / 16 : 1, kRowsAtOnce = 128 / kLanes, kChunks = FP8 ? 1 : D / 8;      // 16-byte chunks
          unsigned char* tile = FP8 ? sRaw + slot * C::kCodes : sV + slot * C::kOperand;
#pragma unroll 1
          for (int i = 0; i < kChunkKeys / kRowsAtOnce * kChunks; ++i) {
            const int r = i / kChunks * kRowsAtOnce + tid / kLanes, c = FP8 ? tid % kLanes : i % kChunks;
            uint4* chunk = reinterpret_cast<uint4*>(tile + (FP8 && D == 64 ? r * 64 + ((c ^ ((r >> 1) & 3)) << 4) : (c >> 3) * kSlab + r * 128 + (((c & 7) ^ (r & 7)) << 4)));
            if (!sees<SINK>(p.causal, make_int2(g.c.item.lo, g.c.item.hi), key0 + r) || !info[r / 16].usable) {
              *chunk = make_uint4(0u, 0u, 0u, 0u);
            } else if (parts) {
              const uint4 x = *chunk;
              if (word_not_finite<FP8>(x.x) || word_not_finite<FP8>(x.y) || word_not_finite<FP8>(x.z) || word_not_finite<FP8>(x.w)) {
                uint32_t* word = reinterpret_cast<uint32_t*>(chunk);
#pragma unroll 1
                for (int j = 0; j < 4; ++j)
                  if (word_not_finite<FP8>(word[j]))
                    word[j] = mark_word<D, R, FP8, SINK>(p, marks, segment, g.c.seq, g.row0, g.rows, key0 + r, c * kPer + j * (kPer / 4), word[j]);
              }
            }
          }
          if constexpr (!FP8) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if constexpr (FP8) {
          convert(sRaw + slot * C::kCodes, sV + slot * C::kOperand);
          // in front of both arrivals: the codes' zeros (edge) before the next copy into their place, the operand before the product
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(raw_free + slot);
        }
        mbar_arrive(v_full + slot);
      }
      ++segment;
    } while (ok && g.next(p));
  } else if (warp >= 8) {
    // --------------------------------------------------------------------------------------------------- softmax
    reg_inc<kSoftRegs>();
    const int w = (warp >> 2) - 2, row = threadIdx.x & 127;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + w * 128 + lane_off, tO = tmem + 256 + w * 128 + lane_off;
    int n = 0;                      // tiles in front of the segment
    int mine = 0;                   // tiles of this warpgroup so far
    int segment = 0;                // of the stretch
    [[maybe_unused]] int merges = 0;
    bool ok = true;
    // A row of the segment at hand: where its output goes, the keys it sees, its logits' factor
    struct Row {
      int there, token, head;       // whether there is such a row; row of the call
      int2 seen;
      float c;
    } at;
    const int r = (SPLIT ? 0 : w * 128) + row;               // the item's row
    // whether this warpgroup has work in the segment (the second one sits out items of up to 128 rows)
    auto idle = [&] { return !SPLIT && w == 1 && g.rows <= 128; };
    // The segment's queries as operand rows.  The S products of the segment before have read this place: their S has been read.
    auto take_queries = [&] {
      at.there = r < g.rows;
      const int in = at.there ? fast_div(g.row0 + r, p.by_G) : 0;
      at.head = at.there ? g.c.h * p.G + (g.row0 + r) - in * p.G : 0;
      at.token = g.c.seq.start + in;
      at.seen = at.there ? visible_keys(p.causal, g.c.seq.first_pos() + in, g.c.seq.len) : make_int2(0, 0x7fffffff);      // (rows that are none need no mask)
      if (g.t0 == g.t1) return;
      float back = 1.0f;
      {
        // A warp's 32 rows, D / 8 lanes a row and 16 bytes a lane, copied to where they will be operands and turned into them there.  In
        // short loops: code that runs once an item comes from memory, and a thread's whole row unrolled took longer than what it does (when this
        // was built, five drafted tokens of 8 sequences of up to 16,383, 64 heads over 8: 72 us, unrolled 79; queries and output at one place each
        // then 67, and 64 with the divisions as multiplications).
        constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes;
        const uint64_t src = at.there ? reinterpret_cast<uint64_t>(p.q + (int64_t)at.token * p.q_stride_t + at.head * p.q_stride_h) : 0ull;
        const int c = lane % kLanes, first = (row & ~31) + lane / kLanes;
        unsigned char* tile = sQ + w * C::kQ;                // (SPLIT: the products read half 0's)
        auto place = [&](int to, int chunk) { return tile + (chunk >> 3) * kSlab + to * 128 + (((chunk & 7) ^ (to & 7)) << 4); };
#pragma unroll 1
        for (int k = 0; k < 32; k += kRowsAtOnce) {
          const uint64_t from = __shfl_sync(0xffffffffu, src, k + lane / kLanes);
          if (from) cp_async16(smem_u32(place(first + k, c)), reinterpret_cast<const uint4*>(from) + c);
          else *reinterpret_cast<uint4*>(place(first + k, c)) = make_uint4(0u, 0u, 0u, 0u);
        }
        cp_async_commit();
        cp_async_wait<0>();
        if constexpr (FP8) {
#pragma unroll 1
          for (int k = 0; k < 32; k += kRowsAtOnce) {
            const uint4 x = *reinterpret_cast<const uint4*>(place(first + k, c));
            float top = largest(largest(largest(largest(0.0f, x.x), x.y), x.z), x.w);
#pragma unroll
            for (int i = 1; i < kLanes; i <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
            const QueryScale s = query_scale(top);
            const float its = __shfl_sync(0xffffffffu, s.back, lane % kRowsAtOnce * kLanes);
            if (lane / kRowsAtOnce == k / kRowsAtOnce) back = its;
            if constexpr (C::kRawK) {
              uint32_t high[2], low[2];
              split_queries(x.x, x.y, s.to, high[0], low[0]);
              split_queries(x.z, x.w, s.to, high[1], low[1]);
              unsigned char* to = place(first + k, c >> 1) + (c & 1) * 8;
              *reinterpret_cast<uint2*>(to) = make_uint2(high[0], high[1]);
              *reinterpret_cast<uint2*>(to + kSlab) = make_uint2(low[0], low[1]);
            } else {
              // fp16: the row's largest entry lies in [128, 256); entries below 2^-24 of it are subnormal numbers, off by at most 2^-32 of it
              uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const __half2 h = __floats2half2_rn(__uint_as_float(y[i] << 16) * s.to, __uint_as_float(y[i] & 0xffff0000u) * s.to);
                y[i] = *reinterpret_cast<const uint32_t*>(&h);
              }
              *reinterpret_cast<uint4*>(place(first + k, c)) = make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(q_full + (SPLIT ? 0 : w));
      }
      at.c = back * p.scale_log2;
    };
    bool live = true, begun = false;
    int tiles = 0, took = 0;        // of the segment: tiles, and those that this warpgroup has taken
    float m = -INFINITY, l = 0.0f;
    struct Past {                   // a segment whose output has not been written
      int there, token, head, slot, set;
      bool whole;
    } past{};
    auto finish = [&] {
      if (took > 0) ok = __all_sync(0xffffffffu, pipe_wait(pv_done + w, (mine - 1) & 1, s_abort, 16 + w));
      if (!ok) return;
      float f_own = 1.0f, f_other = 0.0f;                     // SPLIT: factors of the two halves' O
      bool other = false;
      if constexpr (SPLIT) {
        if (w == 1) {
          s_sums[row] = make_float2(m, l);
          tc_fence_before();
          mbar_arrive(sums_full);
          ok = __all_sync(0xffffffffu, pipe_wait(sums_free, merges++ & 1, s_abort, 18));
          return;
        }
        ok = __all_sync(0xffffffffu, pipe_wait(sums_full, merges++ & 1, s_abort, 19));
        if (!ok) return;
        const float2 its = s_sums[row];
        other = tiles > 1;
        const float to = fmaxf(m, its.x);
        f_own = to == -INFINITY ? 1.0f : fast_exp2(m - to);
        f_other = to == -INFINITY ? 1.0f : fast_exp2(its.x - to);
        l = l * f_own + its.y * f_other;
        m = to;
      }
      tc_fence_after();
      const bool marked = tiles > 0 && *reinterpret_cast<volatile uint32_t*>(marks.any(past.set)) != 0u;
      const bool empty = m == -INFINITY && l == l;            // the row sees no key
      const float inv = empty ? 0.0f : 1.0f / l;
#pragma unroll 1
      for (int ch = 0; ch < D / 32; ++ch) {
        uint32_t o[32];
        tmem_ld32(tO + ch * 32, o);
        tc_wait_ld();
        if constexpr (SPLIT) {
          if (other) {
            uint32_t x[32];
            tmem_ld32(tO + 128 + ch * 32, x);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(fmaf(__uint_as_float(x[j]), f_other, __uint_as_float(o[j]) * f_own));
          }
        }
        if (marked && past.there) {
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(marks.add(past.set, r, ch * 32 + j, __uint_as_float(o[j])));
        }
        if (past.there && past.whole) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + (int64_t)past.token * p.out_stride_t + past.head * p.out_stride_h + ch * 32);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const __nv_bfloat162 h = empty ? __floats2bfloat162_rn(0.0f, 0.0f)
                                             : __floats2bfloat162_rn(__uint_as_float(o[8 * j + 2 * k]) * inv, __uint_as_float(o[8 * j + 2 * k + 1]) * inv);
              x[k] = *reinterpret_cast<const uint32_t*>(&h);
            }
            dst[j] = make_uint4(x[0], x[1], x[2], x[3]);
          }
        } else if (past.there && tiles > 0) {
          // (four channels of a warp's rows side by side: with a row's channels together every store had 32 lines, and an item's end took 4.5 us)
          uint4* dst = reinterpret_cast<uint4*>(p.part_o + (((int64_t)past.slot * (D / 4) + ch * 8) * R + r) * 4);
#pragma unroll
          for (int j = 0; j < 8; ++j) dst[j * R] = empty ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        }
      }
      tc_fence_before();
      if (past.there && past.whole) {
        if (p.lse) p.lse[(int64_t)past.token * p.H + past.head] = empty ? -INFINITY : (m - kBase + log2f(l)) * 0.6931471805599453f;
      } else if (past.there) {
        *reinterpret_cast<float2*>(p.part_ml + ((int64_t)past.slot * R + r) * 2) = make_float2(m, empty ? 0.0f : l);
      }
      if (marked) {
        // this row's marks are taken; the flag stays up for the other rows, and for whoever uses the past.set next, where it finds nothing
#pragma unroll 1
        for (int j = 0; j < Marks<D, R, FP8>::kSigns * Marks<D, R, FP8>::kWords; ++j) marks.row(past.set, r)[j] = 0u;
      }
      if constexpr (SPLIT) mbar_arrive(sums_free);
    };
    // (one place for the queries and one for the output, see take_queries)
    while (true) {
      if constexpr (SPLIT) {
        if (begun) finish();                                 // (the two halves share the queries' place)
        if (!ok) break;
      }
      if (begun) {
        n += tiles;
        live = g.next(p);
        ++segment;
      }
      while (live && idle()) {
        n += g.t1 - g.t0;
        live = g.next(p);
        ++segment;
      }
      // The next segment's queries go first: its first product then runs while the output is read.
      if (live) take_queries();
      if constexpr (!SPLIT) {
        if (begun) finish();
        if (!ok) break;
      }
      if (!live) break;
      tiles = g.t1 - g.t0;
      m = -INFINITY;
      l = 0.0f;
      took = 0;
      const float c_row = at.c;
      const int2 seen = at.seen;
#pragma unroll 1
      for (int i = SPLIT ? w : 0; i < tiles; i += SPLIT ? 2 : 1, ++mine, ++took) {
        ok = __all_sync(0xffffffffu, pipe_wait(s_full + w, mine & 1, s_abort, 12 + w));
        if (!ok) break;
        tc_fence_after();
        uint32_t sr[kChunkKeys];
#pragma unroll
        for (int ch = 0; ch < kChunkKeys / 32; ++ch) tmem_ld32(tS + ch * 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[ch * 32]));
        const GroupInfo* info = s_info + ((n + i) & (kChunkInfoRing - 1)) * kChunkGroups;
        const int key0 = g.c.item.tile_of(g.t0 + i) * kChunkKeys, c_lo = seen.x - key0, c_hi = seen.y - key0;
        const int c_sink = SINK ? p.causal.sink - key0 : 0;
        bool masked = (c_lo > 0 && !(SINK && c_sink >= kChunkKeys)) || c_hi < kChunkKeys;
        if (lane < kChunkGroups) masked = masked || !info[lane].usable;
        masked = __any_sync(0xffffffffu, masked);
        tc_wait_ld();
        if (masked) {
          auto below = [](int x) { return x >= 32 ? 0xffffffffu : x <= 0 ? 0u : (1u << x) - 1u; };
#pragma unroll
          for (int ch = 0; ch < kChunkKeys / 32; ++ch) {
            uint32_t keep = ~below(c_lo - ch * 32);
            if constexpr (SINK) keep |= below(c_sink - ch * 32);
            keep &= below(c_hi - ch * 32);
            if (!info[2 * ch].usable) keep &= 0xffff0000u;
            if (!info[2 * ch + 1].usable) keep &= 0x0000ffffu;
            if (keep != 0xffffffffu) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(keep & (1u << j))) sr[ch * 32 + j] = 0xff800000u;
            }
          }
        }
        // largest t = logit + log2(v scale) of the tile
        float top = -INFINITY;
        if constexpr (FP8) {
#pragma unroll
          for (int q = 0; q < kChunkGroups; ++q) {
            float a = fmaxf(__uint_as_float(sr[16 * q]), __uint_as_float(sr[16 * q + 1])), b = fmaxf(__uint_as_float(sr[16 * q + 2]), __uint_as_float(sr[16 * q + 3]));
#pragma unroll
            for (int j = 4; j < 16; j += 4) {
              a = fmax3(a, __uint_as_float(sr[16 * q + j]), __uint_as_float(sr[16 * q + j + 1]));
              b = fmax3(b, __uint_as_float(sr[16 * q + j + 2]), __uint_as_float(sr[16 * q + j + 3]));
            }
            top = fmaxf(top, fmaf(fmaxf(a, b), logit_factor(c_row, info[q].k), info[q].v_log2));
          }
        } else {
          float mx[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) mx[j] = __uint_as_float(sr[j]);
#pragma unroll
          for (int j = 4; j < kChunkKeys; j += 2) mx[(j >> 1) & 3] = fmax3(mx[(j >> 1) & 3], __uint_as_float(sr[j]), __uint_as_float(sr[j + 1]));
          top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c_row;
        }
        const bool moves = top > m + kLazy;                   // (always for the first key that the row sees)
        if (__any_sync(0xffffffffu, moves)) {
          const float to = moves ? top : m;
          const float f = moves ? fast_exp2(m - to) : 1.0f;   // 0 where nothing has been added up yet
          m = to;
          l *= f;
          if (took > 0) {
            // O is complete up to the tile before
            ok = __all_sync(0xffffffffu, pipe_wait(pv_done + w, (mine - 1) & 1, s_abort, 14 + w));
            if (!ok) break;
            tc_fence_after();
            const uint64_t f2 = pack_f32x2(f, f);
#pragma unroll 1
            for (int ch = 0; ch < D / 16; ++ch) {
              uint32_t o[16];
              tmem_ld16(tO + ch * 16, o);
              tc_wait_ld();
#pragma unroll
              for (int j = 0; j < 16; j += 2) {
                const float2 x = unpack_f32x2(fmul2(pack_f32x2(__uint_as_float(o[j]), __uint_as_float(o[j + 1])), f2));
                o[j] = __float_as_uint(x.x);
                o[j + 1] = __float_as_uint(x.y);
              }
              tmem_st16(tO + ch * 16, o);
            }
            tc_wait_st();
          }
        }
        // weights 2^(t - m + kBase), 32 keys at a time
        const float ref = m == -INFINITY ? 0.0f : kBase - m;
#pragma unroll
        for (int ch = 0; ch < kChunkKeys / 32; ++ch) {
          uint32_t pk[16];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float c = c_row, off = ref, inv = 1.0f;
            if constexpr (FP8) {
              const GroupInfo gi = info[2 * ch + q];
              c = logit_factor(c, gi.k);
              off += gi.v_log2;
              inv = gi.v_inv;
            }
            const uint64_t c2 = pack_f32x2(c, c), off2 = pack_f32x2(off, off);
            uint64_t sum = pack_f32x2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
              const int at = ch * 32 + q * 16 + j;
              const uint64_t e2 = ffma2(pack_f32x2(__uint_as_float(sr[at]), __uint_as_float(sr[at + 1])), c2, off2);
              float2 e = unpack_f32x2(e2);
              e.x = fast_exp2(e.x);
              e.y = fast_exp2(e.y);
              sum = fadd2(sum, pack_f32x2(e.x, e.y));
              if constexpr (FP8) {
                const __half2 h = __floats2half2_rn(e.x, e.y);
                pk[q * 8 + j / 2] = *reinterpret_cast<const uint32_t*>(&h);
              } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(e.x, e.y);
                pk[q * 8 + j / 2] = *reinterpret_cast<const uint32_t*>(&h);
              }
            }
            const float2 s2 = unpack_f32x2(sum);
            l = fmaf(s2.x + s2.y, inv, l);
          }
          tmem_st16(tS + ch * 16, pk);
        }
        tc_wait_st();
        tc_fence_before();
        mbar_arrive(p_full + w);
      }
      if (!ok) break;
      past = {at.there, at.token, at.head, 2 * ((int)blockIdx.x - 1) + (g.first ? 0 : 1), segment, g.whole};
      begun = true;
    }
  }
  // -------------------------------------------------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) report_abort(p.status, *s_abort);
  if (warp == 0) {
    if (*s_abort) __nanosleep(200000);      // let copies and products in flight land before the CTA's resources go
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int D, bool FP8, bool SPLIT>
static int launch_chunk(const sparkattn_cache_t& c, CacheFwdParams& p, const void* k_cache, const void* v_cache, cudaStream_t stream) {
  using C = ChunkShape<D, FP8>;
  constexpr int R = SPLIT ? 128 : 256;
  CUtensorMap mk, mv;
  int rc;
  p.box_rows = c.page;
  p.boxes = kChunkKeys / p.box_rows;
  if ((rc = make_page_map(&mk, k_cache, FP8 ? 1 : 2, c, p.box_rows)) != SPARKATTN_OK) return rc;
  if ((rc = make_page_map(&mv, v_cache, FP8 ? 1 : 2, c, p.box_rows)) != SPARKATTN_OK) return rc;
  constexpr int smem = C::kFixed + Marks<D, R, FP8>::kBytes;
  static_assert(smem <= 232448 && (kCacheMaxSequences + 1) * 4 <= 2 * C::kQ, "fits an SM");
  auto kern = p.causal.sink > 0 ? cache_chunk_kernel<D, FP8, SPLIT, true> : cache_chunk_kernel<D, FP8, SPLIT, false>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return SPARKATTN_E_CUDA;
  if ((rc = launch_kernel(kern, dim3(p.workers + 1), kChunkThreads, smem, true, stream, mk, mv, p)) != SPARKATTN_OK) return rc;
  return launch_kernel(combine_rows_kernel<D, R>, dim3(p.workers - 1, kCombineRowsCtas), kCombineRowsThreads, 0, true, stream, p);
}

int launch_cache_chunk(const sparkattn_cache_t& c, int rows, CacheFwdParams& p, const void* k_cache, const void* v_cache, cudaStream_t stream) {
  auto go = [&](auto d, auto e4m3) {
    constexpr int D = decltype(d)::value;
    constexpr bool FP8 = decltype(e4m3)::value;
    return rows == 128 ? launch_chunk<D, FP8, true>(c, p, k_cache, v_cache, stream) : launch_chunk<D, FP8, false>(c, p, k_cache, v_cache, stream);
  };
  using std::integral_constant;
  if (c.dtype == SPARKATTN_FP8_E4M3)
    return c.d == 128 ? go(integral_constant<int, 128>{}, integral_constant<bool, true>{}) : go(integral_constant<int, 64>{}, integral_constant<bool, true>{});
  return c.d == 128 ? go(integral_constant<int, 128>{}, integral_constant<bool, false>{}) : go(integral_constant<int, 64>{}, integral_constant<bool, false>{});
}

}  // namespace sparkattn
