// sparkattn_cache_fwd for many query rows per key head (prompts, frames, drafts of many tokens): attention over a paged
// cache on the tensor cores, bf16 or E4M3 pages.
//
// The products, 4 d flops per (row, key), bound it, so an item is 256 query rows of one (sequence, key head): two M = 128
// tiles that share every key tile, since fetching a tile and turning its codes into operands costs shared-memory
// bandwidth, which the products themselves use to three quarters (Q and K from shared memory: 64 KB per 128 x 128 x 128).
// The line of all items' key tiles (cache_line.cuh) is cut evenly over one CTA per SM.  Roles:
//   warp 0       TMA producer: pages of K and of V, scales, one descriptor per 16 keys
//   warp 1       issues S_g = Q_g K^T and O_g += P_g V (tcgen05, accumulators in TMEM: S0 | S1 | O0 | O1)
//   warps 4-7    E4M3: codes -> fp16 operand tiles (exact).  Both: V rows that no row of the item sees become zeros, since
//                a page holds anything behind its sequence's last token, and 0 times that need not be 0
//   warps 8-11, 12-15   softmax of tile 0 / 1, a thread per row: S from TMEM, weights back over the same columns as the second product's
//                operand, running reference (lazy: O is rescaled only when a weight would pass 2^10), output
// While one softmax warpgroup works on its S, the tensor core runs the other one's PV and next S; tcgen05.mma of one thread
// run in the order of issue, so S_g of the next tile may overwrite the columns that PV_g has read its P from.
// E4M3: Q, P and V are fp16 (the queries scaled by a power of two per row, the weights by 2^5 at the reference), and V's scale
// is part of the exponent: t = logit + log2(v_scale), the row sum adds weight / v_scale.  bf16 pages: bf16 throughout.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "cache_line.cuh"
#include "tmap.h"

namespace sparkattn {

constexpr int kChunkKeys = 128, kChunkThreads = 512;
constexpr int kChunkGroups = kChunkKeys / 16;
constexpr int kSoftRegs = 192, kConvRegs = 72, kCtrlRegs = 56;      // 2 x 128 x 192 + 128 x 72 + 128 x 56 = 512 x 128
constexpr int kInfoRing = 4;

template <int D, bool FP8>
struct ChunkShape {
  static constexpr int kOperand = kChunkKeys * D * 2;       // a 128 x D tile of 16-bit operands: slabs of 64 channels
  static constexpr int kRaw = kChunkKeys * D;               // the same as E4M3 codes
  static constexpr int kOffK = 2 * kOperand, kOffV = 4 * kOperand, kOffRaw = 6 * kOperand;
  static constexpr int kOffMisc = kOffRaw + (FP8 ? 2 * kRaw : 0);
  static constexpr int kMisc = 256 /* barriers */ + kInfoRing * kChunkGroups * (int)sizeof(GroupInfo) + 128;
  static constexpr int kBytes = kOffMisc + kMisc;
};

template <int D, bool FP8>
__global__ void __launch_bounds__(kChunkThreads, 1)
cache_chunk_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                   const __grid_constant__ CacheFwdParams p) {
  using C = ChunkShape<D, FP8>;
  using L = Line<kChunkRows, kChunkKeys>;
  constexpr int kSlab = kChunkKeys * 128;                    // bytes of 64 operand channels
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sQ = smem;
  unsigned char* sK = smem + C::kOffK;
  unsigned char* sV = smem + C::kOffV;
  unsigned char* sRaw = smem + C::kOffRaw;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffMisc);
  uint64_t* q_full = bars;            // [2] 128 arrivals: the item's queries are in shared memory
  uint64_t* k_full = bars + 2;        // [2] operand K tile (E4M3: 128 arrivals; bf16: its copies)
  uint64_t* k_free = bars + 4;        // [2] the S products that read it are complete
  uint64_t* v_full = bars + 6;        // [2] 128 arrivals
  uint64_t* v_free = bars + 8;        // [2] the PV products that read it are complete
  uint64_t* raw_full = bars + 10;     // [2] E4M3: codes of a K (0) or V (1) tile; bf16: [slot] the copies of a V tile
  uint64_t* raw_free = bars + 12;     // [2] E4M3, 128 arrivals
  uint64_t* s_full = bars + 14;       // [2] S_g complete: the product's arrival and its issuer's (who has seen the tile's descriptor)
  uint64_t* p_full = bars + 16;       // [2] 128 arrivals: weights written, S_g read
  uint64_t* pv_done = bars + 18;      // [2]
  GroupInfo* s_info = reinterpret_cast<GroupInfo*>(bars + 32);          // [ring][groups]
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_info + kInfoRing * kChunkGroups);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_bad = reinterpret_cast<int*>(s_tmem + 2);
  int* s_warp = s_bad + 2;            // [16]
  int* s_prefix = reinterpret_cast<int*>(smem);       // [B + 1], until every warp has found its place in the line
  const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full + i, 128);
      mbar_init(k_full + i, FP8 ? 128 : 1); mbar_init(k_free + i, 1);
      mbar_init(v_full + i, 128); mbar_init(v_free + i, 1);
      mbar_init(raw_full + i, 1); mbar_init(raw_free + i, 128);
      mbar_init(s_full + i, 2); mbar_init(p_full + i, 128); mbar_init(pv_done + i, 1);
    }
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
  if (blockIdx.x == 0) check_call(p, s_bad);
  const long long begin = (long long)((int)blockIdx.x - 1) * share;
  const bool works = blockIdx.x > 0 && begin < total;
  const int x0 = works ? (int)begin : 0, x1 = works ? (int)min(begin + share, (long long)total) : 0;
  Stretch<kChunkRows, kChunkKeys> g;
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
    int n = 0;                                               // tiles so far
    bool ok = true;
    do {
      const int32_t* table = p.batch.page_table + (int64_t)g.c.b * p.batch.max_pages;
      constexpr int kBatch = 32 / kChunkGroups;
      int page_n;
      GroupInfo info_n;
      auto look_up = [&](int t) {
        const bool in = t + lane / kChunkGroups < g.t1;
        page_n = look_up_group<FP8>(p, table, g.c.h, in ? t * kChunkKeys + lane * 16 : 0x7fffff00, g.c.item.lo, g.c.item.hi, info_n);
      };
      look_up(g.t0);
      for (int t = g.t0; ok && t < g.t1; t += kBatch) {
        const int page = page_n;
        const GroupInfo info = info_n;
        if (t + kBatch < g.t1) look_up(t + kBatch);
        for (int u = 0; ok && u < kBatch && t + u < g.t1; ++u, ++n) {
          const int slot = n & 1;
          const int per = kChunkGroups / p.boxes;
          const int box = lane % p.boxes, src = u * kChunkGroups + box * per;
          int box_page = -1;
          for (int i = 0; i < per; ++i) box_page = max(box_page, __shfl_sync(0xffffffffu, page, src + i));
          const bool copies = lane < p.boxes && box_page >= 0;
          const int going = __popc(__ballot_sync(0xffffffffu, copies));
          const int key = (t + u) * kChunkKeys + box * p.box_rows, row = key & ((1 << p.batch.page_shift) - 1);
          // K, then V.  E4M3: both have one slot of codes; bf16: they land where the products read them
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            uint64_t* freed = FP8 ? raw_free + kv : (kv ? v_free : k_free) + slot;
            const int uses = FP8 ? n : n >> 1;               // how often the slot has been filled
            if (uses > 0) ok = __all_sync(0xffffffffu, pipe_wait(freed, (uses - 1) & 1, s_abort, 1 + kv));
            if (!ok) break;
            if (kv == 0 && lane / kChunkGroups == u) s_info[(n & (kInfoRing - 1)) * kChunkGroups + lane % kChunkGroups] = info;
            __syncwarp();
            uint64_t* full = FP8 ? raw_full + kv : (kv ? raw_full : k_full) + slot;
            if (lane == 0) {
              if (going) mbar_expect_tx(full, going * p.box_rows * D * (FP8 ? 1 : 2));
              else mbar_arrive(full);
            }
            __syncwarp();
            if (copies) {
              const CUtensorMap* map = kv ? &tmap_v : &tmap_k;
              if constexpr (FP8) {
                tma_load_4d(sRaw + kv * C::kRaw + box * p.box_rows * D, map, full, 0, row, g.c.h, box_page);
              } else {
#pragma unroll
                for (int sl = 0; sl < D / 64; ++sl)
                  tma_load_4d((kv ? sV : sK) + slot * C::kOperand + sl * kSlab + box * p.box_rows * 128, map, full, sl * 64, row, g.c.h, box_page);
              }
            }
          }
        }
      }
    } while (ok && g.next(p));
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------------- products
    constexpr uint32_t idesc_s = make_idesc(FP8 ? 0u : 1u, 128, kChunkKeys, false);
    constexpr uint32_t idesc_o = make_idesc(FP8 ? 0u : 1u, 128, D, true);
    const uint32_t k_hi = (uint32_t)(make_smem_desc_sw128(0, 16) >> 32);
    const uint32_t q_lo = (uint32_t)make_smem_desc_sw128(smem_u32(sQ), 16), k_lo = (uint32_t)make_smem_desc_sw128(smem_u32(sK), 16);
    const uint32_t v_hi = (uint32_t)(make_smem_desc_sw128(0, kSlab) >> 32);
    const uint32_t v_lo = (uint32_t)make_smem_desc_sw128(smem_u32(sV), kSlab);
    int n = 0;
    uint32_t done[2] = {0, 0};                                // tiles of warpgroup 0, 1 so far (the second sits out items of up to 128 rows)
    uint32_t seg[2] = {0, 0};
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity, int id) { return __all_sync(0xffffffffu, pipe_wait(bar, parity, s_abort, id)) != 0; };
    do {
      const int tiles = g.t1 - g.t0, groups = g.rows > 128 ? 2 : 1;
      auto s_product = [&](int w, int at) {                   // S_w of tile `at`
        if (elect_one()) {
          const uint32_t qa = q_lo + ((w * C::kOperand) >> 4), ka = k_lo + (((at & 1) * C::kOperand) >> 4);
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_ss<false>(tmem + w * 128, make_desc(qa + ((sl * kSlab + kk * 32) >> 4), k_hi), make_desc(ka + ((sl * kSlab + kk * 32) >> 4), k_hi),
                            idesc_s, (sl | kk) != 0 ? 1u : 0u);
          tc_commit(s_full + w);
          mbar_arrive(s_full + w);
          if (w == groups - 1) tc_commit(k_free + (at & 1));
        }
        __syncwarp();
      };
      ok = wait(k_full + (n & 1), (n >> 1) & 1, 3);
      for (int w = 0; ok && w < groups; ++w) {
        ok = wait(q_full + w, seg[w] & 1, 4);
        if (!ok) break;
        ++seg[w];
        tc_fence_after();
        s_product(w, n);
      }
      for (int i = 0; ok && i < tiles; ++i, ++n) {
        ok = wait(v_full + (n & 1), (n >> 1) & 1, 5);
        for (int w = 0; ok && w < groups; ++w) {
          ok = wait(p_full + w, done[w] & 1, 6);
          if (!ok) break;
          ++done[w];
          tc_fence_after();
          if (elect_one()) {
            const uint32_t va = v_lo + (((n & 1) * C::kOperand) >> 4);
#pragma unroll
            for (int kk = 0; kk < kChunkKeys / 16; ++kk)
              mma_ts<false>(tmem + 256 + w * 128, tmem + w * 128 + kk * 8, make_desc(va + ((kk * 16 * 128) >> 4), v_hi), idesc_o,
                            (i == 0 && kk == 0) ? 0u : 1u);
            tc_commit(pv_done + w);
            if (w == groups - 1) tc_commit(v_free + (n & 1));
          }
          __syncwarp();
          if (i + 1 < tiles) {
            if (w == 0) ok = wait(k_full + ((n + 1) & 1), ((n + 1) >> 1) & 1, 7);
            if (!ok) break;
            tc_fence_after();
            s_product(w, n + 1);
          }
        }
      }
    } while (ok && g.next(p));
  } else if (warp >= 4 && warp < 8) {
    // -------------------------------------------------------------------------------------------------- operands
    const int tid = threadIdx.x - 128;
    int n = 0;
    bool ok = true;
    do {
      for (int t = g.t0; ok && t < g.t1; ++t, ++n) {
        const int slot = n & 1;
        // rows of the V tile that may be anything
        const int z_lo = g.c.item.lo - t * kChunkKeys, z_hi = g.c.item.hi - t * kChunkKeys;
        if constexpr (FP8) {
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv) {
            ok = __all_sync(0xffffffffu, pipe_wait(raw_full + kv, n & 1, s_abort, 8 + kv));
            if (ok && n >= 2) ok = __all_sync(0xffffffffu, pipe_wait((kv ? v_free : k_free) + slot, ((n >> 1) - 1) & 1, s_abort, 10 + kv));
            if (!ok) break;
            const uint32_t raw = smem_u32(sRaw + kv * C::kRaw), to = smem_u32((kv ? sV : sK) + slot * C::kOperand);
            constexpr int kCh = D / 16, kRowsAtOnce = 128 / kCh;                // 16-code chunks of a row
            const int c = tid % kCh;
#pragma unroll 4
            for (int r0 = 0; r0 < kChunkKeys; r0 += kRowsAtOnce) {
              const int r = r0 + tid / kCh;
              const uint32_t from = D == 128 ? raw + r * 128 + ((c ^ (r & 7)) << 4) : raw + r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
              uint4 v;
              asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from));
              if (kv == 1 && (r < z_lo || r >= z_hi || !s_info[(n & (kInfoRing - 1)) * kChunkGroups + r / 16].usable)) v = make_uint4(0u, 0u, 0u, 0u);
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
              uint32_t h[8];
#pragma unroll
              for (int i = 0; i < 4; ++i) e4m3_to_half(w[i], h[2 * i], h[2 * i + 1]);
              const uint32_t dst = to + (c >> 2) * kSlab + r * 128;
              const int ck = (c & 3) * 2;
              asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst + ((ck ^ (r & 7)) << 4)), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
              asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst + (((ck + 1) ^ (r & 7)) << 4)), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
            }
            mbar_arrive(raw_free + kv);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive((kv ? v_full : k_full) + slot);
          }
        } else {
          ok = __all_sync(0xffffffffu, pipe_wait(raw_full + slot, (n >> 1) & 1, s_abort, 9));
          if (!ok) break;
          const GroupInfo* info = s_info + (n & (kInfoRing - 1)) * kChunkGroups;
          const int r = tid;
          if (r < z_lo || r >= z_hi || !info[r / 16].usable) {
            const uint32_t to = smem_u32(sV + slot * C::kOperand);
#pragma unroll 1
            for (int i = 0; i < D / 8; ++i)
              asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(to + (i >> 3) * kSlab + r * 128 + ((i & 7) << 4)), "r"(0u) : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          mbar_arrive(v_full + slot);
        }
      }
    } while (ok && g.next(p));
  } else if (warp >= 8) {
    // --------------------------------------------------------------------------------------------------- softmax
    reg_inc<kSoftRegs>();
    const int w = (warp >> 2) - 2, row = threadIdx.x & 127;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + w * 128 + lane_off, tO = tmem + 256 + w * 128 + lane_off;
    int n = 0;                      // tiles so far
    int mine = 0;                   // ... of this warpgroup
    bool ok = true;
    do {
      if (w == 1 && g.rows <= 128) {
        n += g.t1 - g.t0;
        continue;
      }
      const int r = w * 128 + row;                           // the item's row
      const bool there = r < g.rows;
      const int token = there ? (g.row0 + r) / p.G : 0, head = there ? g.c.h * p.G + (g.row0 + r) - token * p.G : 0;
      const int2 seen = there ? visible_keys(p.causal, g.c.seq.first_pos() + token, g.c.seq.len) : make_int2(0, 0);
      // the row's queries as an operand row (the last item's S products, which read this place, are complete: their S has been read)
      float back = 1.0f;
      {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(g.c.seq.start + token) * p.q_stride_t + head * p.q_stride_h);
        uint4 v[D / 8];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) v[i] = there ? src[i] : make_uint4(0u, 0u, 0u, 0u);
        if constexpr (FP8) {
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            const uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t a = (x[j] & 0x7fffu) << 16, b = x[j] & 0x7fff0000u;
              if (a < 0x7f800000u) top = max(top, a);
              if (b < 0x7f800000u) top = max(top, b);
            }
          }
          const int e = min(max((int)(top >> 23), 1), 253);
          back = __uint_as_float((uint32_t)e << 23);
          const float to = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const __half2 h = __floats2half2_rn(__uint_as_float(x[j] << 16) * to, __uint_as_float(x[j] & 0xffff0000u) * to);
              x[j] = *reinterpret_cast<const uint32_t*>(&h);
            }
            v[i] = make_uint4(x[0], x[1], x[2], x[3]);
          }
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
          *reinterpret_cast<uint4*>(sQ + w * C::kOperand + (i >> 3) * kSlab + row * 128 + (((i & 7) ^ (row & 7)) << 4)) = v[i];
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(q_full + w);
      }
      const float c_row = back * p.scale_log2;
      float m = -INFINITY, l = 0.0f;
      for (int t = g.t0; t < g.t1; ++t, ++n, ++mine) {
        ok = __all_sync(0xffffffffu, pipe_wait(s_full + w, mine & 1, s_abort, 12 + w));
        if (!ok) break;
        tc_fence_after();
        uint32_t sr[kChunkKeys];
#pragma unroll
        for (int ch = 0; ch < kChunkKeys / 32; ++ch) tmem_ld32(tS + ch * 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[ch * 32]));
        const GroupInfo* info = s_info + (n & (kInfoRing - 1)) * kChunkGroups;
        const int c_lo = seen.x - t * kChunkKeys, c_hi = seen.y - t * kChunkKeys;
        bool masked = c_lo > 0 || c_hi < kChunkKeys;
        if (lane < kChunkGroups) masked = masked || !info[lane].usable;
        masked = __any_sync(0xffffffffu, masked);
        tc_wait_ld();
        if (masked) {
          auto below = [](int x) { return x >= 32 ? 0xffffffffu : x <= 0 ? 0u : (1u << x) - 1u; };
#pragma unroll
          for (int ch = 0; ch < kChunkKeys / 32; ++ch) {
            uint32_t keep = below(c_hi - ch * 32) & ~below(c_lo - ch * 32);
            if (!info[2 * ch].usable) keep &= 0xffff0000u;
            if (!info[2 * ch + 1].usable) keep &= 0x0000ffffu;
            if (keep != 0xffffffffu) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(keep & (1u << i))) sr[ch * 32 + i] = 0xff800000u;
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
            for (int i = 4; i < 16; i += 4) {
              a = fmax3(a, __uint_as_float(sr[16 * q + i]), __uint_as_float(sr[16 * q + i + 1]));
              b = fmax3(b, __uint_as_float(sr[16 * q + i + 2]), __uint_as_float(sr[16 * q + i + 3]));
            }
            top = fmaxf(top, fmaf(fmaxf(a, b), c_row * info[q].k, info[q].v_log2));
          }
        } else {
          float mx[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) mx[i] = __uint_as_float(sr[i]);
#pragma unroll
          for (int i = 4; i < kChunkKeys; i += 2) mx[(i >> 1) & 3] = fmax3(mx[(i >> 1) & 3], __uint_as_float(sr[i]), __uint_as_float(sr[i + 1]));
          top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c_row;
        }
        const bool moves = top > m + kLazy;                   // (always for the first key that the row sees)
        if (__any_sync(0xffffffffu, moves)) {
          const float to = moves ? top : m;
          const float f = moves ? fast_exp2(m - to) : 1.0f;   // 0 where nothing has been added up yet
          m = to;
          l *= f;
          if (t > g.t0) {
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
              for (int i = 0; i < 16; i += 2) {
                const float2 x = unpack_f32x2(fmul2(pack_f32x2(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), f2));
                o[i] = __float_as_uint(x.x);
                o[i + 1] = __float_as_uint(x.y);
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
              c *= gi.k;
              off += gi.v_log2;
              inv = gi.v_inv;
            }
            const uint64_t c2 = pack_f32x2(c, c), off2 = pack_f32x2(off, off);
            uint64_t sum = pack_f32x2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const int at = ch * 32 + q * 16 + i;
              const float2 e = unpack_f32x2(ffma2(pack_f32x2(__uint_as_float(sr[at]), __uint_as_float(sr[at + 1])), c2, off2));
              const float a = fast_exp2(e.x), b = fast_exp2(e.y);
              sum = fadd2(sum, pack_f32x2(a, b));
              if constexpr (FP8) {
                const __half2 h = __floats2half2_rn(a, b);
                pk[q * 8 + i / 2] = *reinterpret_cast<const uint32_t*>(&h);
              } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
                pk[q * 8 + i / 2] = *reinterpret_cast<const uint32_t*>(&h);
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
      // ------------------------------------------------------------------------------------- the segment's end
      ok = __all_sync(0xffffffffu, pipe_wait(pv_done + w, (mine - 1) & 1, s_abort, 16 + w));
      if (!ok) break;
      tc_fence_after();
      const int slot = 2 * ((int)blockIdx.x - 1) + (g.first ? 0 : 1);
      const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
#pragma unroll 1
      for (int ch = 0; ch < D / 32; ++ch) {
        uint32_t o[32];
        tmem_ld32(tO + ch * 32, o);
        tc_wait_ld();
        if (there && g.whole) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + (int64_t)(g.c.seq.start + token) * p.out_stride_t + head * p.out_stride_h + ch * 32);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(o[8 * i + 2 * j]) * inv, __uint_as_float(o[8 * i + 2 * j + 1]) * inv);
              x[j] = *reinterpret_cast<const uint32_t*>(&h);
            }
            dst[i] = make_uint4(x[0], x[1], x[2], x[3]);
          }
        } else if (there) {
          uint4* dst = reinterpret_cast<uint4*>(p.part_o + ((int64_t)slot * kChunkRows + r) * D + ch * 32);
#pragma unroll
          for (int i = 0; i < 8; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
      }
      tc_fence_before();
      if (there && g.whole) {
        if (p.lse) p.lse[(int64_t)(g.c.seq.start + token) * p.H + head] = l == 0.0f ? -INFINITY : (m - kBase + log2f(l)) * 0.6931471805599453f;
      } else if (there) {
        *reinterpret_cast<float2*>(p.part_ml + ((int64_t)slot * kChunkRows + r) * 2) = make_float2(m, l);
      }
    } while (g.next(p));
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

template <int D, bool FP8>
static int launch_chunk(const sparkattn_cache_t& c, const sparkattn_batch_t& b, CacheFwdParams& p, const void* k_cache, const void* v_cache,
                        cudaStream_t stream) {
  using C = ChunkShape<D, FP8>;
  CUtensorMap mk, mv;
  int rc;
  p.box_rows = c.page;
  p.boxes = kChunkKeys / p.box_rows;
  if ((rc = make_page_map(&mk, k_cache, FP8 ? 1 : 2, c, p.box_rows)) != SPARKATTN_OK) return rc;
  if ((rc = make_page_map(&mv, v_cache, FP8 ? 1 : 2, c, p.box_rows)) != SPARKATTN_OK) return rc;
  static_assert(C::kBytes <= 232448 && (kCacheMaxSequences + 1) * 4 <= 2 * C::kOperand, "fits an SM");
  constexpr int smem = C::kBytes;
  auto kern = cache_chunk_kernel<D, FP8>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return SPARKATTN_E_CUDA;
  if ((rc = launch_kernel(kern, dim3(p.workers + 1), kChunkThreads, smem, true, stream, mk, mv, p)) != SPARKATTN_OK) return rc;
  return launch_kernel(combine_kernel<D, kChunkRows>, dim3(p.workers - 1, 16), kCombineThreads, 0, true, stream, p);
}

int launch_cache_chunk(const sparkattn_cache_t& c, const sparkattn_batch_t& b, CacheFwdParams& p, const void* k_cache, const void* v_cache,
                       cudaStream_t stream) {
  if (c.dtype == SPARKATTN_FP8_E4M3)
    return c.d == 128 ? launch_chunk<128, true>(c, b, p, k_cache, v_cache, stream) : launch_chunk<64, true>(c, b, p, k_cache, v_cache, stream);
  return c.d == 128 ? launch_chunk<128, false>(c, b, p, k_cache, v_cache, stream) : launch_chunk<64, false>(c, b, p, k_cache, v_cache, stream);
}

}  // namespace sparkattn
