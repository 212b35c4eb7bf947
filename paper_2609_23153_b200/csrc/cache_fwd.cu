// sparkattn_cache_fwd for few query rows per key head (decoding, verifying drafted tokens): attention over a paged cache,
// bf16 or E4M3 pages.
//
// A (sequence, key head) with G query heads and n new tokens has G n query rows over the same keys.  The work is reading
// the keys and values once: 2 d bytes (E4M3) a token against 4 d G n flops, far below the tensor cores' rate, so what
// counts is that every SM always has copies in flight, and that long and short sequences come out even.
//   Work split: an item is a (sequence, key head); a tile is 128 of its keys (bf16 with 128 channels: 64).  Two CTAs per SM.  Either
//     each item belongs to a thread-block cluster, whose CTAs take equal runs of its tiles and add up maximum, sum and
//     unnormalised output through distributed shared memory; or the tiles of all items stand in one line (cache_line.cuh), which is
//     cut into equal stretches, one per CTA: an item that lies in one stretch is finished there, one that several share leaves partial
//     results in the workspace, which combine_kernel, launched behind, adds up in a fixed order.  cluster_of has the rule and
//     the figures of both.
//   Copies: one warp requests the tiles with TMA (boxes of whole pages, or what a tile takes of one), as far ahead as the ring is deep, across
//     segment borders.  It also fetches page numbers two batches of up to 32 groups of 16 keys ahead, and their scales one.
//   Products: four warps, each with 16 or 32 keys of every tile and online-softmax state of its own (merged when a segment
//     ends), so that nothing in the loop waits for another warp.  S^T = K Q^T and O^T = V^T P^T as m16n8k16 products with the
//     rows as the N side: eight rows fill an instruction, where rows on the M side would leave half of it empty.
//     The channel order of the first product and the key order of the second are free, so every lane takes its
//     operands from shared memory 16 bytes at a time: 16 channels of a key, of which eight make a fragment.
//     E4M3: K's codes are the first product's operand as they are, against the queries in two E4M3 parts (split_queries), which
//     hold all eight of a bf16's digits; V's bytes of two keys are interleaved by a byte permutation and become fp16 (exact), as the
//     weights do.  P^T is S^T's accumulator transposed by movmatrix.
//   Scales: k's multiplies the logits.  v's goes into the exponent: with t = logit + log2(v_scale), the weights of the second
//     product are 2^(t - m), m a running reference of t, and the row sum adds weight / v_scale.  So neither costs a
//     multiplication per element.
// Measured (one new token per sequence; bytes of keys, values and scales that must be read; E4M3, 128 channels and 8 key heads where nothing
// else is said): 64 sequences of up to 8191 keys, 555 MB in 96 us = 5.8 TB/s, 0.90 of a copy's rate, which bounds it; one sequence
// of 131,071 keys, 269 MB in 53 us = 5.0 TB/s, where the second launch and the way of the first tiles, 5 us each, have nothing to
// hide behind; one of 1001 keys 7.1 us, of one key 4.8: latency.  16 sequences of up to 4095 keys, 12 heads, bf16: 206 MB in 42 us = 5.0 TB/s.
// 32 sequences, a window of 1000 keys, 4 heads of 64 channels, pages of 16 keys: 16 MB in 10.5 us, latency again.
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "cache_line.cuh"
#include "tmap.h"

namespace sparkattn {

constexpr int kGroupKeys = 16;
constexpr int kDecodeOver = 4;      // tiles that the beginning and the end of an item take as long as
constexpr int kInfoRing = 32;      // tiles whose groups' notes are kept: a batch of up to 8 and a ring of up to 8 at a time
// CTAs per SM: two, so that one's items begin and end while the other's copies run (64 sequences of up to 8191 keys, 8 key heads, E4M3:
// 96 us, by one 110, by three 98; one sequence of 1001 keys 7.3, 12.5, 7.3; 64 of 1000 keys 31.9, 44.0, 37.4).
constexpr int kDecodePerSM = 2;
constexpr int kSmemOfSM = 227 * 1024;      // that CTAs can have, 1 KB of each taken by the system
constexpr int kComputeWarps = 4, kDecodeThreads = 32 * (kComputeWarps + 1);

// ---------------------------------------------------------------------------------------------------------- fragments
template <bool FP8>
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (FP8)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16832(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Shared memory of a tile as TMA leaves it: slabs of at most 128 bytes a row, 16-byte chunks swizzled within 8 rows.
template <int ROW_BYTES, int TILE_KEYS>
__device__ __forceinline__ uint32_t chunk_offset(int row, int chunk) {
  if constexpr (ROW_BYTES == 64) return row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);
  else return (chunk >> 3) * (TILE_KEYS * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
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

template <int D, bool FP8, int NT>
struct DecodeShape {
  static constexpr int R = 8 * NT;
  static constexpr int kElt = FP8 ? 1 : 2;
  static constexpr int kRowBytes = D * kElt;
  // groups of 16 keys that a warp takes of a tile: two where a K or V tile stays within 16 KB, so that their chains of dependent
  // steps run side by side and the steps that a tile needs once are spread over 32 keys, and where the registers hold it (16 rows of 128
  // channels: 16 sequences of 8000 keys, 64 heads over 4, 42.8 us by one group a warp, 46.2 by two; of 64 channels 28.1 and 23.5)
  static constexpr int kPerWarp = kRowBytes <= 128 && D * NT <= 128 ? 2 : 1;
  static constexpr int kGroups = kComputeWarps * kPerWarp, kTileKeys = kGroups * kGroupKeys;
  static constexpr int kTileBytes = kTileKeys * kRowBytes;       // of K or of V
  static constexpr int kOPitch = D + 4;
  static constexpr int kMergeBytes = kComputeWarps * R * (kOPitch + 2) * 4;
  static constexpr int fixed_bytes(int B, int slots) {
    return Marks<D, R, FP8>::kBytes + kMergeBytes + kInfoRing * kGroups * (int)sizeof(GroupInfo) + slots * 16 + 64 + ((B + 1) * 4 > R * 8 ? (B + 1) * 4 : R * 8) + 64;
  }
};

// Some rows see some of a warp's keys of a tile and others do not: see Marks.  A lane looks at the words of V that it loads next.  (A
// function of its own: in the tile loop its code cost the smallest call 0.7 us.)
template <int D, bool FP8, int NT>
__device__ __noinline__ void mark_tile(const CacheFwdParams& p, const Marks<D, 8 * NT, FP8> marks, int set, const Sequence seq, int row0, int rows, int2 seen,
                                       int key0, int tile_row0, int usable, unsigned char* tile) {
  using S = DecodeShape<D, FP8, NT>;
  constexpr int kVWords = D / 8 * S::kElt / 4;
  const int g8 = (threadIdx.x & 31) >> 2, t4 = threadIdx.x & 3;
#pragma unroll 1
  for (int i = 0; i < S::kPerWarp * 4 * kVWords; ++i) {
    const int u = i / kVWords >> 2, in = u * kGroupKeys + 4 * t4 + (i / kVWords & 3), key = key0 + in, channel = g8 * (D / 8) + i % kVWords * (4 / S::kElt);
    const uint32_t at = chunk_offset<S::kRowBytes, S::kTileKeys>(tile_row0 + in, channel * S::kElt / 16) + channel * S::kElt % 16;
    uint32_t* word = reinterpret_cast<uint32_t*>(tile + at);
    if (key >= seen.x && key < seen.y && (usable >> u & 1) && word_not_finite<FP8>(*word))
      *word = mark_word<D, S::R, FP8>(p, marks, set, seq, row0, rows, key, channel, *word);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // before the tile is released to the next copy
}

// CLUSTER: an item (it has one row tile) belongs to a cluster of CTAs, each takes an equal run of its key tiles, and the CTAs' results
// are added up through distributed shared memory.  Otherwise the line, see cache_line.cuh; cluster_of has the rule.
template <int D, bool FP8, int NT, bool CLUSTER>
__global__ void __launch_bounds__(kDecodeThreads, kDecodePerSM)
cache_decode_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ CacheFwdParams p) {
  using S = DecodeShape<D, FP8, NT>;
  constexpr int R = S::R, kRowBytes = S::kRowBytes, kTileKeys = S::kTileKeys, kGroups = S::kGroups, kPerWarp = S::kPerWarp;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* after = smem + p.slots * S::kTileBytes;
  const Marks<D, R, FP8> marks{reinterpret_cast<uint32_t*>(after)};
  float* s_o = reinterpret_cast<float*>(after + Marks<D, R, FP8>::kBytes);           // [warps][R][pitch]
  float2* s_ml = reinterpret_cast<float2*>(s_o + kComputeWarps * R * S::kOPitch);    // [warps][R]
  GroupInfo* s_info = reinterpret_cast<GroupInfo*>(s_ml + kComputeWarps * R);        // [ring][groups]
  uint64_t* full = reinterpret_cast<uint64_t*>(s_info + kInfoRing * kGroups);
  uint64_t* empty = full + p.slots;
  uint64_t* merged = empty + p.slots;                                               // a segment's parts are in shared memory
  uint64_t* taken = merged + 1;                                                      // ... and have been read
  volatile int* s_abort = reinterpret_cast<volatile int*>(taken + 1);
  int* s_bad = const_cast<int*>(s_abort) + 1;
  int* s_warp = s_bad + 2;
  int* s_prefix = s_warp + 8;                                                        // the line's
  float2* s_cta = reinterpret_cast<float2*>(s_warp + 9);                             // [R], a cluster's CTA: reference and sum of its rows
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
    for (int i = 0; i < p.slots; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, kComputeWarps); }
    mbar_init(merged, kComputeWarps);
    mbar_init(taken, kComputeWarps);
    mbar_fence_init();
    *s_abort = 0;
  }
  marks.clear_all();
  pdl_wait();
  Stretch<R, kTileKeys, kDecodeOver> g;
  int worker = 0;
  if constexpr (CLUSTER) {
    __syncthreads();
    const int cluster = (int)blockIdx.x / p.cluster, rank = (int)blockIdx.x - cluster * p.cluster;
    if (cluster == 0) {
      if (rank == 0) check_call(p, s_bad);
      return;
    }
    const int b = fast_div(cluster - 1, p.by_Hk);
    if (!g.run_of(p, b, cluster - 1 - b * p.Hk, rank, p.cluster)) return;
  } else {
  Line<R, kTileKeys, kDecodeOver>::lay_out(p, s_prefix, s_warp);
  const int total = s_prefix[p.batch.B], share = Line<R, kTileKeys, kDecodeOver>::share_of(p, total);
  if (blockIdx.x == 0) {
    check_call(p, s_bad);
    return;
  }
  worker = blockIdx.x - 1;
  const long long begin = (long long)worker * share;
  const bool works = begin < total;
  const int x0 = (int)begin, x1 = (int)min(begin + share, (long long)total);
  if (works) g.begin(p, s_prefix, x0, x1);
  if (threadIdx.x == 0) note_border(p, worker, works, share, g);
  if (!works) return;
  }

  if (warp == kComputeWarps) {
    // ------------------------------------------------------------------------------------------------------ copies
    // The stretch goes by in batches of a few tiles of a segment, of whose groups of 16 keys every lane looks after one.  Pages are
    // asked for two batches ahead and scales one, across segments, so that only the first batch waits for them.
    constexpr int kBatch = 32 / kGroups;
    int t_next = g.t0;
    bool live = true;
    auto ask_pages = [&] {
      while (live && t_next >= g.t1) {
        live = g.next(p);
        t_next = g.t0;
      }
      GroupBatch b{t_next, 0, 0, -1, 1.0f, 1.0f};
      if (!live) return b;
      b.n = min(kBatch, g.t1 - b.t);
      b.h = g.c.h;
      const int key = b.t * kTileKeys + lane * kGroupKeys;
      if (lane / kGroups < b.n && key < g.c.item.hi && key + kGroupKeys > g.c.item.lo)
        b.page = p.batch.page_table[(int64_t)g.c.b * p.batch.max_pages + (key >> p.batch.page_shift)];
      t_next += b.n;
      return b;
    };
    int slot = 0, use = 0, n = 0;        // K and V tiles take turns in the ring; tiles so far
    bool ok = true;
    const int per_box = kGroups / p.boxes;               // groups of a box
    GroupBatch now = ask_pages(), next = ask_pages();
    ask_scales<FP8>(p, now);
    while (ok && now.n > 0) {
      // a box is copied if somebody sees one of its groups; the lane of its first group copies it
      int page = now.page;
      if (per_box > 1) page = max(page, __shfl_xor_sync(0xffffffffu, page, 1));
      if (per_box > 2) page = max(page, __shfl_xor_sync(0xffffffffu, page, 2));
      if (per_box > 4) page = max(page, __shfl_xor_sync(0xffffffffu, page, 4));
      const bool copies = page >= 0 && lane % per_box == 0;
      const uint32_t going = __ballot_sync(0xffffffffu, copies);
      const int key = now.t * kTileKeys + lane * kGroupKeys, row = key & ((1 << p.batch.page_shift) - 1);
      // (a copy may finish before the barrier has been told to expect it: the phase is not over without that arrival)
      auto copy = [&](int u, int kv, int slot) {
        if (lane / kGroups == u && copies) {
          constexpr int kSlab = kRowBytes > 128 ? 128 : kRowBytes;
          unsigned char* dst = smem + slot * S::kTileBytes + (lane % kGroups) * kGroupKeys * kSlab;
#pragma unroll
          for (int sl = 0; sl < kRowBytes / kSlab; ++sl)
            tma_load_4d(dst + sl * (kTileKeys * kSlab), kv ? &tmap_v : &tmap_k, full + slot, sl * (kSlab / S::kElt), row, now.h, page);
        }
      };
      auto arrive = [&](int u, int slot) {
        if (lane == 0) {
          const int boxes = __popc((going >> (u * kGroups)) & ((1u << kGroups) - 1u));
          if (boxes) mbar_expect_tx(full + slot, boxes * p.box_rows * kRowBytes);
          else mbar_arrive(full + slot);
        }
      };
      // the ring is empty at first: its copies do not wait for the first scales
      const int ahead = n == 0 ? min(now.n, p.slots / 2) : 0;
      for (int u = 0; u < ahead; ++u) {
        copy(u, 0, 2 * u);
        copy(u, 1, 2 * u + 1);
      }
      // the groups' notes (what they write over belongs to tiles that left the ring long ago)
      s_info[(n * kGroups + lane) & (kInfoRing * kGroups - 1)] = info_of<FP8>(now);
      __syncwarp();
      ask_scales<FP8>(p, next);
      const GroupBatch after_next = ask_pages();
      for (int u = 0; ok && u < now.n; ++u) {
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (u >= ahead) {
            if (use > 0) ok = __all_sync(0xffffffffu, pipe_wait(empty + slot, (use - 1) & 1, s_abort, 1));
            if (!ok) break;
            copy(u, kv, slot);
          }
          arrive(u, slot);
          if (++slot == p.slots) { slot = 0; ++use; }
        }
      }
      n += now.n;
      now = next;
      next = after_next;
    }
    // (nobody leaves before the copies have landed: the computing warps wait for every tile)
  } else {
    // ---------------------------------------------------------------------------------------------------- products
    const int g8 = lane >> 2, t4 = lane & 3;
    constexpr int kSteps = D / 16;                     // k-steps of the first product, m-tiles of the second
    constexpr int kChunkCh = 16 / S::kElt;             // channels of a 16-byte chunk
    int slot = 0, use = 0, segments = 0;
    int at_info = warp * kPerWarp;                                // of the tile whose scores come next
    bool ok = true;
    do {
      // the rows' queries as the first product's B operand: lane (g8, t4) has channels of row g8
      constexpr int kQ = FP8 ? D / 32 * 4 : kSteps * 2;
      uint32_t qf[NT][kQ];                             // bf16: k-step j has words 2j, 2j + 1; E4M3: step j's high parts 4j, 4j + 1, low parts 4j + 2, 4j + 3
      float c_row[NT][2];                              // of the accumulators' rows 2 t4 and 2 t4 + 1: logit -> log2 units
      int lo[NT][2], hi[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 8 + g8, row = g.row0 + r;
        const bool there = r < g.rows;
        const int token = there ? fast_div(row, p.by_G) : 0, head = there ? g.c.h * p.G + (row - token * p.G) : 0;
        const __nv_bfloat16* src = p.q + (int64_t)(g.c.seq.start + token) * p.q_stride_t + head * p.q_stride_h;
        float back = 1.0f;
        if constexpr (FP8) {
          uint4 raw[D / 32];
#pragma unroll
          for (int j = 0; j < D / 32; ++j)
            raw[j] = there ? *reinterpret_cast<const uint4*>(src + (t4 + 4 * (j / 2)) * 16 + (j & 1) * 8) : make_uint4(0u, 0u, 0u, 0u);
          float top = 0.0f;
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            const uint32_t x[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) top = largest(top, x[i]);
          }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const QueryScale s = query_scale(top);
          back = s.back;
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            const uint32_t x[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
            for (int i = 0; i < 2; ++i) split_queries(x[2 * i], x[2 * i + 1], s.to, qf[nt][4 * j + i], qf[nt][4 * j + 2 + i]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            const int chunk = t4 + 4 * (j / (kChunkCh / 4));
            const uint2 x = there ? *reinterpret_cast<const uint2*>(src + chunk * kChunkCh + (j % (kChunkCh / 4)) * 4) : make_uint2(0u, 0u);
            qf[nt][2 * j] = x.x;
            qf[nt][2 * j + 1] = x.y;
          }
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
      constexpr int kVWords = D / 8 * S::kElt / 4;      // 32-bit words of a lane's channels: 2, 4 or 8
      const int row0 = warp * (kPerWarp * kGroupKeys);
      auto wait_full = [&] { return __all_sync(0xffffffffu, pipe_wait(full + slot, use & 1, s_abort, 2)) != 0; };
      auto release = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + slot);
        if (++slot == p.slots) { slot = 0; ++use; }
      };
      for (int t = g.t0; t < g.t1; ++t) {
        ok = wait_full();
        if (!ok) break;
        GroupInfo info[kPerWarp];
        float s[kPerWarp][NT][4];
        {
          // S^T: the product's row 2 t + e (of 0..7) is key 4 t + e of the group, row 8 + 2 t + e key 4 t + 2 + e
          const uint32_t at = smem_u32(smem + slot * S::kTileBytes);
          uint4 ka[kPerWarp][kRowBytes / 64], kb[kPerWarp][kRowBytes / 64];
#pragma unroll
          for (int u = 0; u < kPerWarp; ++u) {
            const int key = row0 + u * kGroupKeys + 4 * (g8 >> 1) + (g8 & 1);
#pragma unroll
            for (int c = 0; c < kRowBytes / 64; ++c) {
              ka[u][c] = lds16(at + chunk_offset<kRowBytes, kTileKeys>(key, t4 + 4 * c));
              kb[u][c] = lds16(at + chunk_offset<kRowBytes, kTileKeys>(key + 2, t4 + 4 * c));
            }
            info[u] = s_info[at_info + u];
          }
          at_info = (at_info + kGroups) & (kInfoRing * kGroups - 1);
          release();
          [[maybe_unused]] float s_low[kPerWarp][NT][4];
#pragma unroll
          for (int u = 0; u < kPerWarp; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 4; ++i) s[u][nt][i] = s_low[u][nt][i] = 0.0f;
#pragma unroll
          for (int c = 0; c < kRowBytes / 64; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int u = 0; u < kPerWarp; ++u) {
                const uint32_t a[4] = {j ? ka[u][c].z : ka[u][c].x, j ? kb[u][c].z : kb[u][c].x, j ? ka[u][c].w : ka[u][c].y, j ? kb[u][c].w : kb[u][c].y};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  if constexpr (FP8) {
                    const uint32_t* q = qf[nt] + 4 * (2 * c + j);
                    mma_16832(s[u][nt], a, q[0], q[1]);
                    mma_16832(s_low[u][nt], a, q[2], q[3]);
                  } else {
                    mma_16816<false>(s[u][nt], a, qf[nt][2 * (2 * c + j)], qf[nt][2 * (2 * c + j) + 1]);
                  }
                }
              }
          if constexpr (FP8) {
#pragma unroll
            for (int u = 0; u < kPerWarp; ++u)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[u][nt][i] += s_low[u][nt][i];
          }
        }
        // t = logit + log2(v scale); keys a row does not see get -inf
        const int key0 = t * kTileKeys + row0;
        bool edge = key0 < all_lo || key0 + kPerWarp * kGroupKeys > all_hi;
#pragma unroll
        for (int u = 0; u < kPerWarp; ++u) {
          edge = edge || !info[u].usable;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[u][nt][i] = fmaf(s[u][nt][i], c_row[nt][i & 1] * info[u].k, info[u].v_log2);
        }
        if (edge) {
#pragma unroll
          for (int u = 0; u < kPerWarp; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int key = key0 + u * kGroupKeys + 4 * (g8 >> 1) + (g8 & 1) + (i & 2);
                if (key < lo[nt][i & 1] || key >= hi[nt][i & 1] || !info[u].usable) s[u][nt][i] = -INFINITY;
              }
        }
        float top[NT][2];
        bool moves = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            top[nt][i] = fmaxf(s[0][nt][i], s[0][nt][i + 2]);
            if constexpr (kPerWarp > 1) top[nt][i] = fmaxf(top[nt][i], fmaxf(s[1][nt][i], s[1][nt][i + 2]));
            moves = moves || top[nt][i] > m[nt][i] + kLazy;
          }
        if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
              for (int k = 4; k < 32; k <<= 1) top[nt][i] = fmaxf(top[nt][i], __shfl_xor_sync(0xffffffffu, top[nt][i], k));
              const float to = fmaxf(m[nt][i], top[nt][i]);
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
        // bf16 pages: the weights in two bf16 parts, since one (2^-8) would add as much to the result's error as its own rounding does
        uint32_t pf[kPerWarp][NT][FP8 ? 2 : 4];
#pragma unroll
        for (int u = 0; u < kPerWarp; ++u)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float ref = m[nt][i & 1];
              w[i] = fast_exp2(s[u][nt][i] - (ref == -INFINITY ? 0.0f : ref - kBase));
            }
            l[nt][0] = fmaf(w[0] + w[2], info[u].v_inv, l[nt][0]);
            l[nt][1] = fmaf(w[1] + w[3], info[u].v_inv, l[nt][1]);
            if constexpr (FP8) {
              const __half2 a = __floats2half2_rn(w[0], w[1]), b = __floats2half2_rn(w[2], w[3]);
              pf[u][nt][0] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&a));
              pf[u][nt][1] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&b));
            } else {
              // (the first cut off, so that the second is positive, and at least 2^-18 of the weight: an infinite value then gives its infinity
              // twice, and the weight 0 of a key that the row does not see stays 0)
              uint32_t high[4];
              float low[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                high[i] = __float_as_uint(w[i]) & 0xffff0000u;
                low[i] = fmaxf(w[i] - __uint_as_float(high[i]), w[i] * 3.8e-6f);
              }
              const uint32_t a = __byte_perm(high[0], high[1], 0x7632), b = __byte_perm(high[2], high[3], 0x7632);
              const __nv_bfloat162 la = __floats2bfloat162_rn(low[0], low[1]), lb = __floats2bfloat162_rn(low[2], low[3]);
              pf[u][nt][0] = transpose_8x8(a);
              pf[u][nt][1] = transpose_8x8(b);
              pf[u][nt][2] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&la));
              pf[u][nt][3] = transpose_8x8(*reinterpret_cast<const uint32_t*>(&lb));
            }
          }
        // V of keys 4 t4 .. 4 t4 + 3 of each group, channels D/8 g8 ..
        ok = wait_full();
        if (!ok) break;
        const uint32_t s_v = smem_u32(smem + slot * S::kTileBytes);
        if (edge && (all_lo > g.c.item.lo || all_hi < g.c.item.hi))
          mark_tile<D, FP8, NT>(p, marks, segments, g.c.seq, g.row0, g.rows, make_int2(g.c.item.lo, g.c.item.hi), key0, row0,
                                info[0].usable | info[kPerWarp - 1].usable << 1, smem + slot * S::kTileBytes);
        uint32_t vw[kPerWarp][4][kVWords];
#pragma unroll
        for (int u = 0; u < kPerWarp; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = row0 + u * kGroupKeys + 4 * t4 + i;
            if constexpr (kVWords == 2) {
              const uint2 w = lds8(s_v + chunk_offset<kRowBytes, kTileKeys>(key, g8 >> 1) + (g8 & 1) * 8);
              vw[u][i][0] = w.x; vw[u][i][1] = w.y;
            } else {
#pragma unroll
              for (int c = 0; c < kVWords / 4; ++c) {
                const uint4 w = lds16(s_v + chunk_offset<kRowBytes, kTileKeys>(key, g8 * (kVWords / 4) + c));
                vw[u][i][4 * c] = w.x; vw[u][i][4 * c + 1] = w.y; vw[u][i][4 * c + 2] = w.z; vw[u][i][4 * c + 3] = w.w;
              }
            }
          }
        if (edge) {
          // what no row sees may be anything, and 0 times that need not be 0
#pragma unroll
          for (int u = 0; u < kPerWarp; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = key0 + u * kGroupKeys + 4 * t4 + i;
              if (key < g.c.item.lo || key >= g.c.item.hi || !info[u].usable) {
#pragma unroll
                for (int w = 0; w < kVWords; ++w) vw[u][i][w] = 0u;
              }
            }
        }
        release();
        // O^T: m-tile i has channels D/8 g8 + 2i (rows g8) and + 2i + 1 (rows 8 + g8)
#pragma unroll
        for (int u = 0; u < kPerWarp; ++u)
#pragma unroll
          for (int w = 0; w < kVWords; ++w) {
            const uint32_t* v0 = vw[u][0];
            const uint32_t* v1 = vw[u][1];
            const uint32_t* v2 = vw[u][2];
            const uint32_t* v3 = vw[u][3];
            if constexpr (FP8) {
              uint32_t a[4], b[4];
              e4m3_to_half(__byte_perm(v0[w], v1[w], 0x5140), a[0], a[1]);
              e4m3_to_half(__byte_perm(v2[w], v3[w], 0x5140), a[2], a[3]);
              e4m3_to_half(__byte_perm(v0[w], v1[w], 0x7362), b[0], b[1]);
              e4m3_to_half(__byte_perm(v2[w], v3[w], 0x7362), b[2], b[3]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_16816<true>(o[2 * w][nt], a, pf[u][nt][0], pf[u][nt][1]);
                mma_16816<true>(o[2 * w + 1][nt], b, pf[u][nt][0], pf[u][nt][1]);
              }
            } else {
              const uint32_t a[4] = {__byte_perm(v0[w], v1[w], 0x5410), __byte_perm(v0[w], v1[w], 0x7632),
                                     __byte_perm(v2[w], v3[w], 0x5410), __byte_perm(v2[w], v3[w], 0x7632)};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_16816<false>(o[w][nt], a, pf[u][nt][0], pf[u][nt][1]);
                mma_16816<false>(o[w][nt], a, pf[u][nt][2], pf[u][nt][3]);
              }
            }
          }
      }
      if (!ok) break;
      // ------------------------------------------------------------------------------------- the warps' parts together
      if (segments > 0) ok = __all_sync(0xffffffffu, pipe_wait(taken, (segments - 1) & 1, s_abort, 3));
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
      ok = __all_sync(0xffffffffu, pipe_wait(merged, segments & 1, s_abort, 4));
      if (!ok) break;
      const int slot = 2 * worker + (g.first ? 0 : 1);
      const bool marked = *reinterpret_cast<volatile uint32_t*>(marks.any(segments)) != 0u;
      if (!CLUSTER && warp == 0) marks.clear(segments + 2);    // (last read two segments ago, marked again behind the next segment's end)
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
        if (marked) {
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = marks.add(segments, r, ch + j, acc[j]);
        }
        if (CLUSTER && p.cluster > 1) {
          float4* dst = reinterpret_cast<float4*>(s_o + r * S::kOPitch + ch);       // (in place of the first warp's, which this thread alone reads)
          dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
          dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
          if (ch == 0) s_cta[r] = make_float2(top, sum);
        } else if (CLUSTER || g.whole) {
          const int row = g.row0 + r, of = fast_div(row, p.by_G), token = g.c.seq.start + of, head = g.c.h * p.G + row - of * p.G;
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
      if constexpr (CLUSTER) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(taken);
      ++segments;
    } while (g.next(p));
  }
  if constexpr (CLUSTER) {
    if (p.cluster > 1) {
      // (every thread of the cluster comes here, whatever happened to it)
      cluster_arrive();
      cluster_wait();
      const int rank = (int)blockIdx.x % p.cluster;
      constexpr int kPer = D / 4;                            // threads of a row, four channels each
      if (warp < kComputeWarps) {
        for (int task = rank + p.cluster * (int)threadIdx.x; task < g.rows * kPer; task += p.cluster * 32 * kComputeWarps) {
          const int r = task / kPer, ch = (task % kPer) * 4;
          const uint32_t at_ml = smem_u32(s_cta + r), at_o = smem_u32(s_o + r * S::kOPitch + ch);
          float top = -INFINITY, sum = 0.0f, acc[4] = {};
#pragma unroll 8
          for (int c = 0; c < p.cluster; ++c) {
            const float2 ml = cluster_ld2(at_ml, c);
            const float4 v = cluster_ld4(at_o, c);
            const float to = fmaxf(top, ml.x), f = to == -INFINITY ? 0.0f : fast_exp2(ml.x - to), keep = to == -INFINITY ? 0.0f : fast_exp2(top - to);
            sum = fmaf(ml.y, f, sum * keep);
            acc[0] = fmaf(v.x, f, acc[0] * keep);
            acc[1] = fmaf(v.y, f, acc[1] * keep);
            acc[2] = fmaf(v.z, f, acc[2] * keep);
            acc[3] = fmaf(v.w, f, acc[3] * keep);
            top = to;
          }
          const int row = g.row0 + r, of = fast_div(row, p.by_G), token = g.c.seq.start + of, head = g.c.h * p.G + row - of * p.G;
          const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
          const __nv_bfloat162 a = __floats2bfloat162_rn(acc[0] * inv, acc[1] * inv), b = __floats2bfloat162_rn(acc[2] * inv, acc[3] * inv);
          *reinterpret_cast<uint2*>(p.out + (int64_t)token * p.out_stride_t + head * p.out_stride_h + ch) =
              make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
          if (p.lse && ch == 0) p.lse[(int64_t)token * p.H + head] = sum == 0.0f ? -INFINITY : (top - kBase + log2f(sum)) * 0.6931471805599453f;
        }
      }
      cluster_arrive();
      cluster_wait();                                        // nobody leaves while others read its memory
    }
  }
  if (threadIdx.x == 0) report_abort(p.status, *s_abort);
  if (*s_abort) __nanosleep(200000);      // let copies in flight land before the CTA's memory goes
}

// ------------------------------------------------------------------------------------------------------------ host side
namespace {
constexpr size_t align256(size_t x) { return (x + 255) / 256 * 256; }
// Who splits an item: a cluster of the returned number of CTAs, or (0) the line.
//   A cluster adds up its parts at once (128-key tiles, 8 key heads, one sequence of 500 / 4000 / 16,000 keys: 6.2 / 8.5 / 15.3 us, line 9.4 / 12.1 /
//   16.0), as many CTAs as one wave of two per SM holds, of up to sixteen where that leaves SMs to spare (16 of 8 items: 4000 keys 8.5 us, 8: 9.0;
//   16,000 keys 15.3 and 18.2; more than a wave: 16 sequences of 1000 keys by 2 CTAs an item 10.6 us, by 4 16.0).
//   Two of a long item's where one each would fill a wave: sequences seldom have one length (16 sequences of up to 4000 keys, 12 heads, E4M3:
//   27.0 us, by one CTA 33.1, the line 26.7; all of one length 50.4, 42.5, 42.8).
//   The line takes over where clusters leave SMs idle for long (32,000 keys: 19.2 us, clusters of 16 24.2) and where the
//   items are more than a wave and long, whose lengths may differ (64 sequences of up to 8191 keys, 8 heads: 95 us, clusters of
//   1 / 2 120 / 109; all of one length 171 and 167 / 184; of 2000 keys 56 and 52).  So it does between, from 2304 keys a CTA on: lengths up to
//   the stated one, in parentheses all of it, line / cluster of two, E4M3: 10 sequences of 8 heads, 4000 keys 18.1 / 20.2 us (22.1 / 24.6), 16,000
//   41.8 / 64.7 (61.5 / 78.2); 16 of 8, 4000 20.5 / 20.3 (32.7 / 27.6), 16,000 52.7 / 65.7 (89.2 / 83.2); 16 of 12, 8000 43.0 / 46.1 (71.4 / 87.9); cluster
//   of four: 5 of 8, 16,000 26.0 / 36.1 (36.3 / 43.4).  bf16: 16 of 8, 4000 31.8 / 30.4 (51.5 / 44.1); 8 of 12, 16,000 73.3 / 94.9 (129 / 118); 32 of 8, 8000
//   93.0 / one CTA 105 (169 / 150).
//   Lengths are known on the device only: the table's width stands for them, and one sequence of 1000 keys under a table of 131,072 takes the
//   line (9.8 us; under its own width a cluster, 6.2).  Sixteen CTAs take eight SMs of one GPC: 148 SMs in eight GPCs always leave one with that many.
int cluster_of(const sparkattn_cache_t& c, const sparkattn_batch_t& b, int frame_tokens, int window, int tile_keys, int sms) {
  const long long items = (long long)b.B * c.H;
  long long keys = (long long)b.max_pages * c.page;                       // that an item may have
  if (window > 0) keys = std::min(keys, ((long long)window + 1) * frame_tokens + b.max_new);
  const long long tiles = (keys + tile_keys - 1) / tile_keys;
  int n = items * 16 <= sms ? 16 : 8;
  while (n > 1 && (items * n > std::max(2 * sms, 16) || n / 2 >= tiles)) n /= 2;
  if (n == 1 && items <= 2 * sms && tiles >= 16) n = 2;
  if (items > 2 * sms ? tiles >= 32 : items * n < sms ? tiles > 12 * n : keys > 2304LL * n) return 0;
  return n;
}

// rows of an item, and stretches of the line: up to 16 rows per key head take this file's kernel, more the tensor cores' (cache_chunk.cu)
struct Plan {
  int R, workers;
  size_t borders, ml, o;       // bytes of the workspace's parts behind the header
};
int plan_rows(const sparkattn_cache_t& c, const sparkattn_batch_t& b, int H) {
  const long long rows = (long long)(H / c.H) * b.max_new;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 128 ? 128 : 256;
}
Plan plan_of(const sparkattn_cache_t& c, const sparkattn_batch_t& b, int H) {
  Plan p;
  p.R = plan_rows(c, b, H);
  p.workers = current_sm_count() * (p.R >= 128 ? 1 : kDecodePerSM);
  p.borders = align256((size_t)p.workers * sizeof(Border));
  p.ml = align256((size_t)2 * p.workers * p.R * 8);
  p.o = (size_t)2 * p.workers * p.R * c.d * 4;
  return p;
}
}  // namespace

// The kernels count key tiles of all items in 32 bits.  What the struct allows at most, whatever the lengths are: a sixteenth of this for
// 32,000 tokens of 64 query heads, eight key heads and a million keys.
bool cache_work_fits(const sparkattn_cache_t& c, const sparkattn_batch_t& b, int H) {
  const int R = plan_rows(c, b, H);
  const double items = ((double)b.T * (H / c.H) / R + b.B) * c.H, tiles = (double)b.max_pages * c.page / 64 + 1;
  return items * (tiles + std::max(kDecodeOver, 6)) < 2147418112.0;
}

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
  p.box_rows = c.page < S::kTileKeys ? c.page : S::kTileKeys;
  p.boxes = S::kTileKeys / p.box_rows;
  if ((rc = make_page_map(&mk, k_cache, S::kElt, c, p.box_rows)) != SPARKATTN_OK) return rc;
  if ((rc = make_page_map(&mv, v_cache, S::kElt, c, p.box_rows)) != SPARKATTN_OK) return rc;
  const long long items = (long long)b.B * c.H;
  p.cluster = cluster_of(c, b, p.causal.frame, p.causal.window, S::kTileKeys, p.workers / kDecodePerSM);
  const bool cluster = p.cluster > 0;
  // as deep a ring as the CTAs of an SM leave each other, sixteen tiles at most; fewer CTAs where a great many sequences leave no room
  const int listed = cluster ? 0 : b.B;
  for (int per = kDecodePerSM; per > 0; --per) {
    p.slots = (kSmemOfSM / per - 1024 - S::fixed_bytes(listed, 16)) / S::kTileBytes;
    if (p.slots >= 3) break;
  }
  if (p.slots > 16) p.slots = 16;
  if (p.slots < 3) return SPARKATTN_E_UNSUPPORTED_SHAPE;
  const int smem = p.slots * S::kTileBytes + S::fixed_bytes(listed, p.slots);
  auto kern = cluster ? cache_decode_kernel<D, FP8, NT, true> : cache_decode_kernel<D, FP8, NT, false>;
  // (the kernel's, not the call's: the most that any call asks for, since host threads with other batches set it too)
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemOfSM - 1024) != cudaSuccess) return SPARKATTN_E_CUDA;
  if (cluster) {
    if (p.cluster > 8 && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return SPARKATTN_E_CUDA;
    return launch_clustered(kern, dim3((unsigned)((items + 1) * p.cluster)), kDecodeThreads, smem, true, p.cluster, stream, mk, mv, p);
  }
  if ((rc = launch_kernel(kern, dim3(p.workers + 1), kDecodeThreads, smem, true, stream, mk, mv, p)) != SPARKATTN_OK) return rc;
  return launch_kernel(combine_kernel<D, S::R>, dim3(p.workers - 1), kCombineThreads, 0, true, stream, p);
}

int launch_cache_fwd(const sparkattn_cache_t& c, const sparkattn_batch_t& b, const sparkattn_rows_t& q, int H, const void* k_cache,
                     const void* v_cache, const float* k_scale, const float* v_scale, int frame_tokens, int window, float softmax_scale,
                     const sparkattn_rows_t& out, float* lse, void* workspace, cudaStream_t stream) {
  CacheFwdParams p{};
  p.batch = make_batch_view(c, b);
  p.causal = {frame_tokens, window, make_fast_div(std::max(frame_tokens, 1))};
  p.q = static_cast<const __nv_bfloat16*>(q.data);
  p.out = static_cast<__nv_bfloat16*>(out.data);
  p.q_stride_t = q.stride_t; p.q_stride_h = q.stride_h;
  p.out_stride_t = out.stride_t; p.out_stride_h = out.stride_h;
  p.k_scale = k_scale; p.v_scale = v_scale;
  p.lse = lse;
  p.H = H; p.Hk = c.H; p.G = H / c.H;
  p.by_Hk = make_fast_div(p.Hk);
  p.by_G = make_fast_div(p.G);
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
  if (plan.R >= 128) return launch_cache_chunk(c, plan.R, p, k_cache, v_cache, stream);
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
