// sparkattn_cache_fwd for few query rows per key head (decoding, verifying drafted tokens): attention over a paged cache,
// bf16 or E4M3 pages.
//
// A (sequence, key head) with G query heads and n new tokens has G n query rows over the same keys.  The work is reading
// the keys and values once: 2 d bytes (E4M3) a token against 4 d G n flops, far below the tensor cores' rate, so what
// counts is that every SM always has copies in flight, and that long and short sequences come out even.
//   Work split: the tiles of 64 keys of all (sequence, key head, row tile) stand in one line, which is cut into equal
//     stretches, one per CTA, two CTAs per SM.  A CTA's stretch is a sequence of segments (parts of items); an item that
//     lies in one stretch is finished there, one that several stretches share leaves partial results (maximum, sum,
//     unnormalised output) in the workspace, which combine_kernel, launched behind, adds up in a fixed order.
//   Copies: one warp requests the tiles with TMA (boxes of up to 64 rows of a page), as far ahead as the ring is deep, across
//     segment borders.  It also fetches page numbers and scales, 32 groups of 16 keys at a time, one batch ahead.
//   Products: four warps, each with 16 keys of every tile and online-softmax state of its own (merged when a segment
//     ends), so that nothing in the loop waits for another warp.  S^T = K Q^T and O^T = V^T P^T as m16n8k16 products with the
//     rows as the N side: eight rows fill an instruction, where rows on the M side would leave half of it empty.
//     The channel order of the first product and the key order of the second are free, so every lane takes its
//     operands from shared memory 16 bytes at a time: 16 channels of a key, of which four make a fragment.  E4M3 becomes
//     fp16 (exact) on the way, V's bytes of two keys interleaved by a byte permutation; the queries are fp16, scaled by
//     a power of two per row.  P^T is S^T's accumulator transposed by movmatrix.
//   Scales: k's multiplies the logits.  v's goes into the exponent: with t = logit + log2(v_scale), the weights of the second
//     product are 2^(t - m), m a running reference of t, and the row sum adds weight / v_scale.  So neither costs a
//     multiplication per element.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "cache_line.cuh"
#include "tmap.h"

namespace sparkattn {

constexpr int kTileKeys = 64, kGroupKeys = 16, kGroups = kTileKeys / kGroupKeys;
constexpr int kComputeWarps = 4, kDecodeThreads = 32 * (kComputeWarps + 1);

// ---------------------------------------------------------------------------------------------------------- fragments
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return (uint32_t)h.x | (uint32_t)h.y << 16;
}
template <bool FP8>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (FP8)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Shared memory of a tile as TMA leaves it: slabs of at most 128 bytes a row, 16-byte chunks swizzled within 8 rows.
template <int ROW_BYTES>
__device__ __forceinline__ uint32_t chunk_offset(int row, int chunk) {
  if constexpr (ROW_BYTES == 64) return row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);
  else return (chunk >> 3) * (kTileKeys * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}

// CTAs per SM, as registers and the rings allow
constexpr int decode_ctas_per_sm(int D, bool fp8, int R) { return R == 8 ? (fp8 ? 4 : D == 64 ? 3 : 2) : D == 64 ? 3 : 2; }

template <int D, bool FP8, int NT>
struct DecodeShape {
  static constexpr int R = 8 * NT;
  static constexpr int kElt = FP8 ? 1 : 2;
  static constexpr int kRowBytes = D * kElt;
  static constexpr int kTileBytes = kTileKeys * kRowBytes;
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kOPitch = D + 4;
  static constexpr int kPerSM = decode_ctas_per_sm(D, FP8, R);
  static constexpr int kMergeBytes = kComputeWarps * R * (kOPitch + 2) * 4;
  static constexpr int fixed_bytes(int B, int stages) {
    return kMergeBytes + stages * (kGroups * (int)sizeof(GroupInfo) + 16) + 64 + (B + 1) * 4 + 64;
  }
};

template <int D, bool FP8, int NT>
__global__ void __launch_bounds__(kDecodeThreads, DecodeShape<D, FP8, NT>::kPerSM)
cache_decode_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ CacheFwdParams p) {
  using S = DecodeShape<D, FP8, NT>;
  constexpr int R = S::R, kRowBytes = S::kRowBytes;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* after = smem + p.stages * S::kStageBytes;
  float* s_o = reinterpret_cast<float*>(after);                                      // [warps][R][pitch]
  float2* s_ml = reinterpret_cast<float2*>(s_o + kComputeWarps * R * S::kOPitch);    // [warps][R]
  GroupInfo* s_info = reinterpret_cast<GroupInfo*>(s_ml + kComputeWarps * R);        // [stages][groups]
  uint64_t* full = reinterpret_cast<uint64_t*>(s_info + p.stages * kGroups);
  uint64_t* empty = full + p.stages;
  uint64_t* merged = empty + p.stages;                                               // a segment's parts are in shared memory
  uint64_t* taken = merged + 1;                                                      // ... and have been read
  volatile int* s_abort = reinterpret_cast<volatile int*>(taken + 1);
  int* s_bad = const_cast<int*>(s_abort) + 1;
  int* s_warp = s_bad + 2;
  int* s_prefix = s_warp + 8;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
    for (int i = 0; i < p.stages; ++i) { mbar_init(full + i, 2); mbar_init(empty + i, kComputeWarps); }
    mbar_init(merged, kComputeWarps);
    mbar_init(taken, kComputeWarps);
    mbar_fence_init();
    *s_abort = 0;
  }
  pdl_wait();
  Line<R, kTileKeys>::lay_out(p, s_prefix, s_warp);
  const int total = s_prefix[p.batch.B], share = Line<R, kTileKeys>::share_of(p, total);
  if (blockIdx.x == 0) {
    check_call(p, s_bad);
    return;
  }
  const int worker = blockIdx.x - 1;
  const long long begin = (long long)worker * share;
  const bool works = begin < total;
  const int x0 = (int)begin, x1 = (int)min(begin + share, (long long)total);
  Stretch<R, kTileKeys> g;
  if (works) g.begin(p, s_prefix, x0, x1);
  if (threadIdx.x == 0) note_border(p, worker, works, share, g);
  if (!works) return;

  if (warp == kComputeWarps) {
    // ------------------------------------------------------------------------------------------------------ copies
    int stage = 0, use = 0;
    bool ok = true;
    do {
      const int32_t* table = p.batch.page_table + (int64_t)g.c.b * p.batch.max_pages;
      constexpr int kBatch = 32 / kGroups;                   // tiles whose groups the lanes look up together
      // lane l looks after group l of a batch: its page and scales, asked for a batch ahead
      int page_n;
      GroupInfo info_n;
      auto look_up = [&](int t) {
        const bool in = t + lane / kGroups < g.t1;
        page_n = look_up_group<FP8>(p, table, g.c.h, in ? t * kTileKeys + lane * kGroupKeys : 0x7fffff00, g.c.item.lo, g.c.item.hi, info_n);
      };
      look_up(g.t0);
      for (int t = g.t0; ok && t < g.t1; t += kBatch) {
        const int page = page_n;
        const GroupInfo info = info_n;
        if (t + kBatch < g.t1) look_up(t + kBatch);
        for (int u = 0; u < kBatch && t + u < g.t1; ++u) {
          if (use > 0) ok = mbar_wait(empty + stage, (use - 1) & 1, s_abort, p.status, 1);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          // lane i copies box i of K, lane i + boxes box i of V: as many of them as have a page
          const int box = lane & (p.boxes - 1);
          const int src = u * kGroups + box * (kGroups / p.boxes);
          const int at_page = __shfl_sync(0xffffffffu, page, src);
          // (a box may begin before the first visible key and still hold some: any group of it will do)
          int box_page = at_page;
          for (int i = 1; i < kGroups / p.boxes; ++i) box_page = max(box_page, __shfl_sync(0xffffffffu, page, src + i));
          const bool copies = lane < 2 * p.boxes && box_page >= 0;
          const uint32_t going = __ballot_sync(0xffffffffu, copies);
          if (lane == 0) {
            if (going) mbar_expect_tx(full + stage, __popc(going) * p.box_rows * kRowBytes);
            else mbar_arrive(full + stage);
          }
          __syncwarp();
          if (copies) {
            const bool is_v = lane >= p.boxes;
            const int key = (t + u) * kTileKeys + box * p.box_rows;
            unsigned char* dst = smem + stage * S::kStageBytes + (is_v ? S::kTileBytes : 0);
            const CUtensorMap* map = is_v ? &tmap_v : &tmap_k;
            const int row = key & ((1 << p.batch.page_shift) - 1);
            constexpr int kSlab = kRowBytes > 128 ? 128 : kRowBytes;
#pragma unroll
            for (int sl = 0; sl < kRowBytes / kSlab; ++sl)
              tma_load_4d(dst + sl * (kTileKeys * kSlab) + box * p.box_rows * kSlab, map, full + stage, sl * (kSlab / S::kElt), row, g.c.h, box_page);
          }
          // the groups' notes follow, so that the first copies do not wait for the first scales
          if (lane / kGroups == u) s_info[stage * kGroups + lane % kGroups] = info;
          __syncwarp();
          if (lane == 0) mbar_arrive(full + stage);
          if (++stage == p.stages) { stage = 0; ++use; }
        }
      }
    } while (ok && g.next(p));
    // (nobody leaves before the copies have landed: the computing warps wait for every tile)
  } else {
    // ---------------------------------------------------------------------------------------------------- products
    const int g8 = lane >> 2, t4 = lane & 3;
    constexpr int kSteps = D / 16;                     // k-steps of the first product, m-tiles of the second
    constexpr int kChunkCh = 16 / S::kElt;             // channels of a 16-byte chunk
    int stage = 0, use = 0, segments = 0;
    bool ok = true;
    do {
      // the rows' queries as the first product's B operand: lane (g8, t4) has channels of row g8
      uint32_t qf[NT][kSteps][2];
      float c_row[NT][2];                              // of the accumulators' rows 2 t4 and 2 t4 + 1: logit -> log2 units
      int lo[NT][2], hi[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 8 + g8, row = g.row0 + r;
        const bool there = r < g.rows;
        const int token = there ? row / p.G : 0, head = there ? g.c.h * p.G + (row - token * p.G) : 0;
        const __nv_bfloat16* src = p.q + (int64_t)(g.c.seq.start + token) * p.q_stride_t + head * p.q_stride_h;
        uint2 raw[kSteps];
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const int chunk = t4 + 4 * (j / (kChunkCh / 4));
          raw[j] = there ? *reinterpret_cast<const uint2*>(src + chunk * kChunkCh + (j % (kChunkCh / 4)) * 4) : make_uint2(0u, 0u);
        }
        float back = 1.0f;
        if constexpr (FP8) {
          // fp16 queries: the row times the power of two that brings its largest entry to [1, 2)
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            const uint32_t w[2] = {raw[j].x, raw[j].y};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t a = (w[i] & 0x7fffu) << 16, b = w[i] & 0x7fff0000u;
              if (a < 0x7f800000u) top = max(top, a);
              if (b < 0x7f800000u) top = max(top, b);
            }
          }
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const int e = min(max((int)(top >> 23), 1), 253);
          back = __uint_as_float((uint32_t)e << 23);
          const float to = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            const uint32_t w[2] = {raw[j].x, raw[j].y};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const __half2 h = __floats2half2_rn(__uint_as_float(w[i] << 16) * to, __uint_as_float(w[i] & 0xffff0000u) * to);
              qf[nt][j][i] = *reinterpret_cast<const uint32_t*>(&h);
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < kSteps; ++j) { qf[nt][j][0] = raw[j].x; qf[nt][j][1] = raw[j].y; }
        }
        const int2 seen = there ? visible_keys(p.causal, g.c.seq.first_pos() + token, g.c.seq.len) : make_int2(0, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int from = (2 * t4 + i) * 4;
          c_row[nt][i] = __shfl_sync(0xffffffffu, back, from) * p.scale_log2;
          lo[nt][i] = __shfl_sync(0xffffffffu, seen.x, from);
          hi[nt][i] = __shfl_sync(0xffffffffu, seen.y, from);
        }
      }
      // keys that every row sees need no mask
      int all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (nt * 8 + 2 * t4 + i < g.rows) { all_lo = max(all_lo, lo[nt][i]); all_hi = min(all_hi, hi[nt][i]); }
      all_lo = (int)__reduce_max_sync(0xffffffffu, (unsigned)all_lo);
      all_hi = (int)__reduce_min_sync(0xffffffffu, (unsigned)all_hi);

      float o[kSteps][NT][4], m[NT][2], l[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -INFINITY;
        l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) o[i][nt][0] = o[i][nt][1] = o[i][nt][2] = o[i][nt][3] = 0.0f;
      }
      for (int t = g.t0; t < g.t1; ++t) {
        ok = __all_sync(0xffffffffu, mbar_wait(full + stage, use & 1, s_abort, p.status, 2));
        if (!ok) break;
        const GroupInfo info = s_info[stage * kGroups + warp];
        const int key0 = t * kTileKeys + warp * kGroupKeys;
        if (!info.usable) {                            // nothing here for any row
          __syncwarp();
          if (lane == 0) mbar_arrive(empty + stage);
          if (++stage == p.stages) { stage = 0; ++use; }
          continue;
        }
        const uint32_t s_k = smem_u32(smem + stage * S::kStageBytes), s_v = s_k + S::kTileBytes;
        const int row0 = warp * kGroupKeys;
        // S^T: the product's row 2 t + e (of 0..7) is key 4 t + e of the group, row 8 + 2 t + e key 4 t + 2 + e
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.0f;
        {
          const int ka = row0 + 4 * (g8 >> 1) + (g8 & 1), kb = ka + 2;
#pragma unroll
          for (int c = 0; c < kRowBytes / 64; ++c) {
            const uint4 va = lds16(s_k + chunk_offset<kRowBytes>(ka, t4 + 4 * c)), vb = lds16(s_k + chunk_offset<kRowBytes>(kb, t4 + 4 * c));
            const uint32_t wa[4] = {va.x, va.y, va.z, va.w}, wb[4] = {vb.x, vb.y, vb.z, vb.w};
#pragma unroll
            for (int j = 0; j < kChunkCh / 4; ++j) {
              uint32_t a[4];
              if constexpr (FP8) {
                a[0] = e4m3_to_half2(wa[j] & 0xffffu); a[2] = e4m3_to_half2(wa[j] >> 16);
                a[1] = e4m3_to_half2(wb[j] & 0xffffu); a[3] = e4m3_to_half2(wb[j] >> 16);
              } else {
                a[0] = wa[2 * j]; a[2] = wa[2 * j + 1];
                a[1] = wb[2 * j]; a[3] = wb[2 * j + 1];
              }
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_16816<FP8>(s[nt], a, qf[nt][c * (kChunkCh / 4) + j][0], qf[nt][c * (kChunkCh / 4) + j][1]);
            }
          }
        }
        // V of keys 4 t4 .. 4 t4 + 3, channels D/8 g8 ..
        constexpr int kVWords = D / 8 * S::kElt / 4;    // 32-bit words of a lane's channels: 2, 4 or 8
        uint32_t vw[4][kVWords];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = row0 + 4 * t4 + i;
          if constexpr (kVWords == 2) {
            const uint2 w = lds8(s_v + chunk_offset<kRowBytes>(key, g8 >> 1) + (g8 & 1) * 8);
            vw[i][0] = w.x; vw[i][1] = w.y;
          } else {
#pragma unroll
            for (int c = 0; c < kVWords / 4; ++c) {
              const uint4 w = lds16(s_v + chunk_offset<kRowBytes>(key, g8 * (kVWords / 4) + c));
              vw[i][4 * c] = w.x; vw[i][4 * c + 1] = w.y; vw[i][4 * c + 2] = w.z; vw[i][4 * c + 3] = w.w;
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + stage);
        if (++stage == p.stages) { stage = 0; ++use; }
        // t = logit + log2(v scale); keys a row does not see get -inf
        float tt[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) tt[nt][i] = fmaf(s[nt][i], c_row[nt][i & 1] * info.k, info.v_log2);
        if (key0 < all_lo || key0 + kGroupKeys > all_hi) {
          const int ka = key0 + 4 * (g8 >> 1) + (g8 & 1);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = ka + (i & 2);
              if (key < lo[nt][i & 1] || key >= hi[nt][i & 1]) tt[nt][i] = -INFINITY;
            }
          // what no row sees may be anything, and 0 times that need not be 0
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = key0 + 4 * t4 + i;
            if (key < g.c.item.lo || key >= g.c.item.hi) {
#pragma unroll
              for (int w = 0; w < kVWords; ++w) vw[i][w] = 0u;
            }
          }
        }
        bool moves = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) moves = moves || tt[nt][i] > m[nt][i & 1] + kLazy;
        if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float top = fmaxf(tt[nt][i], tt[nt][i + 2]);
#pragma unroll
              for (int k = 4; k < 32; k <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
              const float to = fmaxf(m[nt][i], top);
              f[i] = to == -INFINITY ? 1.0f : fast_exp2(m[nt][i] - to);
              m[nt][i] = to;
              l[nt][i] *= f[i];
            }
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[k][nt][i] *= f[i & 1];
          }
        }
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float ref = m[nt][i & 1];
            w[i] = fast_exp2(tt[nt][i] - (ref == -INFINITY ? 0.0f : ref - kBase));
          }
          l[nt][0] = fmaf(w[0] + w[2], info.v_inv, l[nt][0]);
          l[nt][1] = fmaf(w[1] + w[3], info.v_inv, l[nt][1]);
          if constexpr (FP8) {
            const __half2 a = __floats2half2_rn(w[0], w[1]), b = __floats2half2_rn(w[2], w[3]);
            pf[nt][0] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&a));
            pf[nt][1] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&b));
          } else {
            const __nv_bfloat162 a = __floats2bfloat162_rn(w[0], w[1]), b = __floats2bfloat162_rn(w[2], w[3]);
            pf[nt][0] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&a));
            pf[nt][1] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&b));
          }
        }
        // O^T: m-tile i has channels D/8 g8 + 2i (rows g8) and + 2i + 1 (rows 8 + g8)
        if constexpr (FP8) {
#pragma unroll
          for (int w = 0; w < kVWords; ++w) {
            const uint32_t e01 = __byte_perm(vw[0][w], vw[1][w], 0x5140), f01 = __byte_perm(vw[0][w], vw[1][w], 0x7362);
            const uint32_t e23 = __byte_perm(vw[2][w], vw[3][w], 0x5140), f23 = __byte_perm(vw[2][w], vw[3][w], 0x7362);
            uint32_t a[4] = {e4m3_to_half2(e01 & 0xffffu), e4m3_to_half2(e01 >> 16), e4m3_to_half2(e23 & 0xffffu), e4m3_to_half2(e23 >> 16)};
            uint32_t b[4] = {e4m3_to_half2(f01 & 0xffffu), e4m3_to_half2(f01 >> 16), e4m3_to_half2(f23 & 0xffffu), e4m3_to_half2(f23 >> 16)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma_16816<true>(o[2 * w][nt], a, pf[nt][0], pf[nt][1]);
              mma_16816<true>(o[2 * w + 1][nt], b, pf[nt][0], pf[nt][1]);
            }
          }
        } else {
#pragma unroll
          for (int w = 0; w < kVWords; ++w) {
            uint32_t a[4] = {__byte_perm(vw[0][w], vw[1][w], 0x5410), __byte_perm(vw[0][w], vw[1][w], 0x7632),
                             __byte_perm(vw[2][w], vw[3][w], 0x5410), __byte_perm(vw[2][w], vw[3][w], 0x7632)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_16816<false>(o[w][nt], a, pf[nt][0], pf[nt][1]);
          }
        }
      }
      if (!ok) break;
      // ------------------------------------------------------------------------------------- the warps' parts together
      if (segments > 0) ok = __all_sync(0xffffffffu, mbar_wait(taken, (segments - 1) & 1, s_abort, p.status, 3));
      if (!ok) break;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float sum = l[nt][i];
#pragma unroll
          for (int k = 4; k < 32; k <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
          const int r = nt * 8 + 2 * t4 + i;
          if (g8 == 0) s_ml[warp * R + r] = make_float2(m[nt][i], sum);
          float* dst = s_o + (warp * R + r) * S::kOPitch + g8 * (D / 8);
#pragma unroll
          for (int k = 0; k < kSteps; ++k) *reinterpret_cast<float2*>(dst + 2 * k) = make_float2(o[k][nt][i], o[k][nt][i + 2]);
        }
      __syncwarp();
      if (lane == 0) mbar_arrive(merged);
      ok = __all_sync(0xffffffffu, mbar_wait(merged, segments & 1, s_abort, p.status, 4));
      if (!ok) break;
      const int slot = 2 * worker + (g.first ? 0 : 1);
      constexpr int kPer = D / 8;                            // threads of a row, eight channels each
      for (int task = threadIdx.x; task < g.rows * kPer; task += 32 * kComputeWarps) {
        const int r = task / kPer, ch = (task % kPer) * 8;
        float2 ml[kComputeWarps];
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kComputeWarps; ++w) { ml[w] = s_ml[w * R + r]; top = fmaxf(top, ml[w].x); }
        float sum = 0.0f, acc[8] = {};
#pragma unroll
        for (int w = 0; w < kComputeWarps; ++w) {
          const float f = top == -INFINITY ? 0.0f : fast_exp2(ml[w].x - top);
          sum = fmaf(ml[w].y, f, sum);
          const float* src = s_o + (w * R + r) * S::kOPitch + ch;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = fmaf(src[j], f, acc[j]);
        }
        if (g.whole) {
          const int row = g.row0 + r, token = g.c.seq.start + row / p.G, head = g.c.h * p.G + row % p.G;
          const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(acc[2 * j] * inv, acc[2 * j + 1] * inv);
            w[j] = *reinterpret_cast<const uint32_t*>(&h);
          }
          *reinterpret_cast<uint4*>(p.out + (int64_t)token * p.out_stride_t + head * p.out_stride_h + ch) = make_uint4(w[0], w[1], w[2], w[3]);
          if (p.lse && ch == 0) p.lse[(int64_t)token * p.H + head] = sum == 0.0f ? -INFINITY : (top - kBase + log2f(sum)) * 0.6931471805599453f;
        } else {
          float4* dst = reinterpret_cast<float4*>(p.part_o + ((int64_t)slot * R + r) * D + ch);
          dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
          dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
          if (ch == 0) *reinterpret_cast<float2*>(p.part_ml + ((int64_t)slot * R + r) * 2) = make_float2(top, sum);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(taken);
      ++segments;
    } while (g.next(p));
  }
  if (*s_abort) __nanosleep(200000);      // let copies in flight land before the CTA's memory goes
}

// ------------------------------------------------------------------------------------------------------------ host side
namespace {
constexpr size_t align256(size_t x) { return (x + 255) / 256 * 256; }
// rows of an item, and stretches of the line: up to 16 rows per key head take this file's kernel, more the tensor cores' (cache_chunk.cu)
struct Plan {
  int R, workers;
  size_t borders, ml, o;       // bytes of the workspace's parts behind the header
};
Plan plan_of(const sparkattn_cache_t& c, const sparkattn_batch_t& b, int H) {
  const long long rows = (long long)(H / c.H) * b.max_new;
  Plan p;
  p.R = rows <= 8 ? 8 : rows <= 16 ? 16 : kChunkRows;
  const bool fp8 = c.dtype == SPARKATTN_FP8_E4M3;
  p.workers = current_sm_count() * (p.R == kChunkRows ? 1 : decode_ctas_per_sm(c.d, fp8, p.R));
  p.borders = align256((size_t)p.workers * sizeof(Border));
  p.ml = align256((size_t)2 * p.workers * p.R * 8);
  p.o = (size_t)2 * p.workers * p.R * c.d * 4;
  return p;
}
}  // namespace

size_t cache_fwd_workspace_bytes(const sparkattn_cache_t& c, const sparkattn_batch_t& b, int H) {
  const Plan p = plan_of(c, b, H);
  return kWorkspaceHeaderBytes + p.borders + p.ml + p.o;
}

template <int D, bool FP8, int NT>
static int launch_decode(const sparkattn_cache_t& c, const sparkattn_batch_t& b, CacheFwdParams& p, const void* k_cache, const void* v_cache,
                         cudaStream_t stream) {
  using S = DecodeShape<D, FP8, NT>;
  CUtensorMap mk, mv;
  int rc;
  p.box_rows = c.page < kTileKeys ? c.page : kTileKeys;
  p.boxes = kTileKeys / p.box_rows;
  if ((rc = make_page_map(&mk, k_cache, S::kElt, c, p.box_rows)) != SPARKATTN_OK) return rc;
  if ((rc = make_page_map(&mv, v_cache, S::kElt, c, p.box_rows)) != SPARKATTN_OK) return rc;
  // as deep a ring as the CTAs of an SM leave each other; fewer CTAs where a great many sequences leave no room for two tiles
  for (int per = S::kPerSM; per > 0; --per) {
    p.stages = (227 * 1024 / per - 1024 - S::fixed_bytes(b.B, 12)) / S::kStageBytes;
    if (p.stages >= 2) break;
  }
  if (p.stages > 12) p.stages = 12;
  if (p.stages < 2) return SPARKATTN_E_UNSUPPORTED_SHAPE;
  const int smem = p.stages * S::kStageBytes + S::fixed_bytes(b.B, p.stages);
  auto kern = cache_decode_kernel<D, FP8, NT>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return SPARKATTN_E_CUDA;
  if ((rc = launch_kernel(kern, dim3(p.workers + 1), kDecodeThreads, smem, true, stream, mk, mv, p)) != SPARKATTN_OK) return rc;
  return launch_kernel(combine_kernel<D, S::R>, dim3(p.workers - 1), kCombineThreads, 0, true, stream, p);
}

int launch_cache_fwd(const sparkattn_cache_t& c, const sparkattn_batch_t& b, const sparkattn_rows_t& q, int H, const void* k_cache,
                     const void* v_cache, const float* k_scale, const float* v_scale, int frame_tokens, int window, float softmax_scale,
                     const sparkattn_rows_t& out, float* lse, void* workspace, cudaStream_t stream) {
  CacheFwdParams p{};
  p.batch = make_batch_view(c, b);
  p.causal = {frame_tokens, window};
  p.q = static_cast<const __nv_bfloat16*>(q.data);
  p.out = static_cast<__nv_bfloat16*>(out.data);
  p.q_stride_t = q.stride_t; p.q_stride_h = q.stride_h;
  p.out_stride_t = out.stride_t; p.out_stride_h = out.stride_h;
  p.k_scale = k_scale; p.v_scale = v_scale;
  p.lse = lse;
  p.H = H; p.Hk = c.H; p.G = H / c.H;
  p.scale_log2 = (softmax_scale > 0.0f ? softmax_scale : 1.0f / sqrtf((float)c.d)) * 1.4426950408889634f;
  p.least = 1;
  const Plan plan = plan_of(c, b, H);
  if (plan.workers < 1) return SPARKATTN_E_CUDA;
  p.workers = plan.workers;
  char* base = static_cast<char*>(workspace);
  p.status = reinterpret_cast<int32_t*>(base);
  base += kWorkspaceHeaderBytes;
  p.borders = reinterpret_cast<Border*>(base);
  base += plan.borders;
  p.part_ml = reinterpret_cast<float*>(base);
  base += plan.ml;
  p.part_o = reinterpret_cast<float*>(base);
  if (plan.R == kChunkRows) return launch_cache_chunk(c, b, p, k_cache, v_cache, stream);
  const bool fp8 = c.dtype == SPARKATTN_FP8_E4M3;
  auto go = [&](auto d, auto e4m3) {
    return plan.R == 8 ? launch_decode<decltype(d)::value, decltype(e4m3)::value, 1>(c, b, p, k_cache, v_cache, stream)
                       : launch_decode<decltype(d)::value, decltype(e4m3)::value, 2>(c, b, p, k_cache, v_cache, stream);
  };
  using std::integral_constant;
  if (c.d == 128) return fp8 ? go(integral_constant<int, 128>{}, integral_constant<bool, true>{}) : go(integral_constant<int, 128>{}, integral_constant<bool, false>{});
  return fp8 ? go(integral_constant<int, 64>{}, integral_constant<bool, true>{}) : go(integral_constant<int, 64>{}, integral_constant<bool, false>{});
}

}  // namespace sparkattn
