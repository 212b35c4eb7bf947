// The line: the key tiles of all items of a call, one behind the other, cut into stretches of equal work.
//
// An item is R query rows (row = token * G + head in its group) of one (sequence, key head); its tiles of TK keys run from
// the first to the last key that any of its rows sees, at least one, so that somebody writes the rows of an empty sequence.
// Every item stands for OVER units more than it has tiles, in front of them: what it takes to begin and to finish one, without which the
// stretches with many short items would take longest (a piece of 2048 tokens of each of four prompts of up to 8000, 32 heads over 8: 540 us
// with six, 660 without; 64 sequences of up to 8191 keys, one token each, 8 heads: 96 us with four, 107 without).
// Stretch w is units [w * share, (w + 1) * share).  What a stretch holds of an item is a segment; an item that lies in one
// stretch is finished there, the others leave partial results that combine_kernel adds up in the line's order.
// Items stand in the order (sequence, key head, row tile).
// SINK: an item's rows also see the sequence's first tokens.  The tiles of these stand in front of the window's in the item's run of tiles, with
// the numbers right below theirs (Item::tile_of), so that everything that counts tiles counts on; the keys between take no part.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "cache.h"

namespace sparkattn {

// The reference m of a row moves when a weight would pass 2^10 times the one that set it; weights are 2^kBase at the reference, so
// that fp16 holds them (2^15 < 65504) and loses only what lies below 2^-30 of it, half of the smallest subnormal number.
constexpr float kBase = 5.0f, kLazy = 10.0f;

struct CacheFwdParams {
  BatchView batch;
  Causal causal;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  int64_t q_stride_t, q_stride_h, out_stride_t, out_stride_h;
  const float* k_scale;
  const float* v_scale;
  float* lse;
  int H, Hk, G;
  FastDiv by_Hk, by_G;           // (divisions took 4 us of the 67 of five drafted tokens of 8 sequences, 64 heads over 8: every role has them in code of its own)
  float scale_log2;
  int box_rows, boxes;           // keys of one TMA box, boxes of a tile
  int least;                     // units a stretch has at least
  int workers;                   // stretches
  int slots;                     // K and V tiles that a CTA's ring holds
  int cluster;                   // CTAs of an item's cluster; 0: the line
  int row_tiles;                 // clusters, SINK: row tiles of a (sequence, key head), each an item
  FastDiv by_row_tiles;
  int32_t* status;
  struct Border* borders;        // [workers]
  float* part_ml;                // [2 workers][R][2] reference, sum
  float* part_o;                 // [2 workers][R][d] unnormalised output (128 rows and more: [2 workers][d / 4][R][4])
};

// What the combining kernel needs to know of the border in front of a stretch: the item that it cuts, if it does.
struct Border {
  int before;                    // units of the item in front of the border; 0: the border cuts none
  int units, share;              // of the item; of a stretch
  int token0, row0, rows, h;     // row r is head h * G + (row0 + r) % G of token token0 + (row0 + r) / G
  int pad;
};

// cache_chunk.cu: items of 128 or 256 rows
int launch_cache_chunk(const sparkattn_cache_t& c, int rows, CacheFwdParams& p, const void* k_cache, const void* v_cache, cudaStream_t stream);

// 16 keys of a tile, as the copying warp has looked them up
struct GroupInfo {
  float k;           // factor of the logits
  float v_log2;      // log2 of the V scale
  float v_inv;       // its inverse
  int usable;        // somebody sees keys of it, and the page exists
};

template <int R, int TK, int OVER, bool SINK>
struct Line {
  struct Item {
    int first, tiles;            // key tiles, counted from the front of the sequence (SINK: see tile_of)
    int lo, hi;                  // keys that any of its rows sees (SINK: besides the first ones)
    int window;                  // SINK: the window's first tile
    __device__ __forceinline__ int units() const { return tiles + OVER; }
    // where tile number t lies in the sequence
    __device__ __forceinline__ int tile_of(int t) const { return SINK && t < window ? t - first : t; }
  };
  static __device__ __forceinline__ int row_tiles(const CacheFwdParams& p, const Sequence& s) { return (s.n * p.G + R - 1) / R; }
  static __device__ __forceinline__ Item item_of(const CacheFwdParams& p, const Sequence& s, int rt) {
    const int last_row = max(min((rt + 1) * R, s.n * p.G) - 1, 0);
    Item it;
    it.lo = visible_keys(p.causal, s.first_pos() + fast_div(rt * R, p.by_G), s.len).x;
    it.hi = visible_keys(p.causal, s.first_pos() + fast_div(last_row, p.by_G), s.len).y;
    it.first = it.lo / TK;
    it.tiles = max((it.hi + TK - 1) / TK - it.first, 1);
    if constexpr (SINK) {
      it.window = it.first;
      const int front = min((p.causal.sink - 1) / TK + 1, it.first);
      it.first -= front;
      it.tiles += front;
    }
    return it;
  }
  // Units of the row tiles of one key head, every lane for a sequence of its own (n = 0: none).  Whole warps: few sequences of many row tiles are
  // taken one after the other by all lanes (three frames of 1560 tokens, one sequence of 19 row tiles: 0.8 us instead of 3.8).
  static __device__ __forceinline__ int units_of(const CacheFwdParams& p, const Sequence& s) {
    const int tiles = row_tiles(p, s);
    int sum = 0;
    if constexpr (R >= 128) {
      const int most = (int)__reduce_max_sync(0xffffffffu, (unsigned)tiles), lane = threadIdx.x & 31;
      uint32_t long_ones = __ballot_sync(0xffffffffu, tiles > 1);
      if (__popc(long_ones) * ((most + 31) / 32) < most) {
        if (tiles == 1) sum = item_of(p, s, 0).units();
        for (; long_ones != 0; long_ones &= long_ones - 1) {
          const int l = __ffs(long_ones) - 1;
          const Sequence its{__shfl_sync(0xffffffffu, s.start, l), __shfl_sync(0xffffffffu, s.n, l), __shfl_sync(0xffffffffu, s.len, l)};
          int part = 0;
          for (int rt = lane; rt < row_tiles(p, its); rt += 32) part += item_of(p, its, rt).units();
          part = (int)__reduce_add_sync(0xffffffffu, (unsigned)part);
          if (lane == l) sum = part;
        }
        return sum;
      }
    }
    for (int rt = 0; rt < tiles; ++rt) sum += item_of(p, s, rt).units();
    return sum;
  }
  // all threads: prefix[b] = units in front of sequence b, prefix[B] = all (shared memory)
  static __device__ __forceinline__ void lay_out(const CacheFwdParams& p, int* prefix, int* s_warp) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    int carry = 0;
    for (int base = 0; base < p.batch.B; base += blockDim.x) {
      const int b = base + threadIdx.x;
      const int mine = units_of(p, b < p.batch.B ? sequence_of(p.batch, b) : Sequence{0, 0, 0}) * p.Hk;
      int x = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) s_warp[warp] = x;
      __syncthreads();
      int before = carry, all = carry;
      for (int w = 0; w < warps; ++w) {
        if (w < warp) before += s_warp[w];
        all += s_warp[w];
      }
      if (b < p.batch.B) prefix[b] = before + x - mine;
      carry = all;
      __syncthreads();
    }
    if (threadIdx.x == 0) prefix[p.batch.B] = carry;
    __syncthreads();
  }
  static __device__ __forceinline__ int share_of(const CacheFwdParams& p, int total) { return max((total + p.workers - 1) / p.workers, p.least); }

  // A place in the line, and the walk along it.  Whole warps.
  struct Place {
    Sequence seq;
    Item item;
    int b, h, rt, row_tiles;
    int at;                      // units of the item in front of the place
  };
  static __device__ __forceinline__ Place find(const CacheFwdParams& p, const int* prefix, int x) {
    Place c;
    int lo = 0, hi = p.batch.B;                   // prefix[lo] <= x; sequences without new tokens have equal entries
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (prefix[mid] <= x) lo = mid; else hi = mid;
    }
    c.b = lo;
    c.seq = sequence_of(p.batch, lo);
    c.row_tiles = row_tiles(p, c.seq);
    const int each = fast_div(prefix[lo + 1] - prefix[lo], p.by_Hk);
    int in = x - prefix[lo];
    c.h = in / each;
    in -= c.h * each;
    // the row tile: 32 of them at a time
    const int lane = threadIdx.x & 31;
    int rt0 = 0;
    c.rt = 0;
    c.at = in;
    if (c.row_tiles > 1) {
      for (;; rt0 += 32) {
        const int mine = rt0 + lane < c.row_tiles ? item_of(p, c.seq, rt0 + lane).units() : 0;
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, sum, o);
          if (lane >= o) sum += y;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, sum > in);
        if (past != 0) {
          const int l = __ffs(past) - 1;
          c.rt = rt0 + l;
          c.at = in - __shfl_sync(0xffffffffu, sum - mine, l);
          break;
        }
        in -= __shfl_sync(0xffffffffu, sum, 31);
        if (rt0 + 32 >= c.row_tiles) break;       // (never: in is smaller than the sum of all)
      }
    }
    c.item = item_of(p, c.seq, c.rt);
    return c;
  }
  // to the front of the next item
  static __device__ __forceinline__ void next_item(const CacheFwdParams& p, Place& c) {
    c.at = 0;
    if (++c.rt == c.row_tiles) {
      c.rt = 0;
      if (++c.h == p.Hk) {
        c.h = 0;
        do ++c.b, c.seq = sequence_of(p.batch, c.b); while (c.seq.n == 0 && c.b < p.batch.B - 1);
        c.row_tiles = row_tiles(p, c.seq);
      }
    }
    c.item = item_of(p, c.seq, c.rt);
  }
};

// A stretch of the line, taken segment by segment.
template <int R, int TK, int OVER, bool SINK>
struct Stretch {
  using L = Line<R, TK, OVER, SINK>;
  typename L::Place c;
  int x, end;
  int t0, t1;                    // the segment's key tiles, numbered as the item's (none, where it is all beginning)
  int row0, rows;                // its rows
  bool whole, first;             // the item lies in this stretch; the stretch's first segment
  __device__ __forceinline__ void begin(const CacheFwdParams& p, const int* prefix, int from, int to) {
    x = from;
    end = to;
    c = L::find(p, prefix, from);
    first = true;
    cut(p);
  }
  __device__ __forceinline__ void cut(const CacheFwdParams& p) {
    const int until = min(c.item.units(), c.at + end - x);
    t0 = c.item.first + max(c.at - OVER, 0);
    t1 = c.item.first + max(until - OVER, 0);
    whole = c.at == 0 && until == c.item.units();
    row0 = c.rt * R;
    rows = min(R, c.seq.n * p.G - row0);
    x += until - c.at;
  }
  // instead: run `rank` of `ranks` equal runs of row tile rt of (b, h), the only one but for SINK; false if it has no rows
  __device__ __forceinline__ bool run_of(const CacheFwdParams& p, int b, int h, int rt, int rank, int ranks) {
    c.b = b;
    c.h = h;
    c.rt = SINK ? rt : 0;
    c.at = 0;
    c.row_tiles = 1;
    c.seq = sequence_of(p.batch, b);
    if (SINK ? c.seq.n * p.G <= c.rt * R : c.seq.n == 0) return false;
    c.item = L::item_of(p, c.seq, c.rt);
    const int each = (c.item.tiles + ranks - 1) / ranks, end_tile = c.item.first + c.item.tiles;
    t0 = min(c.item.first + rank * each, end_tile);
    t1 = min(t0 + each, end_tile);
    row0 = c.rt * R;
    rows = SINK ? min(R, c.seq.n * p.G - row0) : c.seq.n * p.G;
    x = end = 0;
    first = true;
    whole = false;
    return true;
  }
  // false behind the last segment
  __device__ __forceinline__ bool next(const CacheFwdParams& p) {
    if (x >= end) return false;
    L::next_item(p, c);
    first = false;
    cut(p);
    return true;
  }
};

// Queries against E4M3 keys: a row times the power of two that brings its largest entry to [128, 256), as two E4M3 parts,
// high = rne(x) and low = rne(x - high).  A bf16 has eight significant digits and an E4M3 four, so x - high has at most four and
// the sum of the parts is x, but for entries below 2^-9 of the row's largest, whose low part falls into E4M3's subnormal
// numbers: off by at most 2^-10, half of their step, which is 2^-17 of the largest.  Products of two E4M3 numbers are exact in the tensor core and their sums were found to be
// fp32's (off by at most 2^-25 of the sum of the magnitudes, m16n8k32 over 128 channels).  Keys stay codes, and the two products
// take as long as one with 16-bit operands.  A row with an infinity or a NaN in it gives NaN.
struct QueryScale {
  float to, back;
};
__device__ __forceinline__ float largest(float top, uint32_t two_bf16) {
  // (integer order: NaN above infinity above the finite)
  const uint32_t a = (two_bf16 & 0x7fffu) << 16, b = two_bf16 & 0x7fff0000u;
  return __uint_as_float(max(max(a, b), __float_as_uint(top)));
}
__device__ __forceinline__ QueryScale query_scale(float top) {
  const int e = min(max((int)(__float_as_uint(top) >> 23), 8), 254);
  return {__uint_as_float((uint32_t)(261 - e) << 23), __float_as_uint(top) < 0x7f800000u ? __uint_as_float((uint32_t)(e - 7) << 23) : __uint_as_float(0x7fffffffu)};
}
// four channels (two bf16 pairs) as four codes of high parts and four of low parts
__device__ __forceinline__ void split_queries(uint32_t x, uint32_t y, float to, uint32_t& high, uint32_t& low) {
  const float v[4] = {__uint_as_float(x << 16) * to, __uint_as_float(x & 0xffff0000u) * to, __uint_as_float(y << 16) * to, __uint_as_float(y & 0xffff0000u) * to};
  uint32_t h[2], l[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    h[i] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * i], v[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)h[i], __NV_E4M3)));
    l[i] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * i] - f.x, v[2 * i + 1] - f.y), __NV_SATFINITE, __NV_E4M3);
  }
  high = h[0] | h[1] << 16;
  low = l[0] | l[1] << 16;
}

// A batch of tiles as the copying warp asks for it: every lane looks after one group of 16 keys, its page and its scales.
struct GroupBatch {
  int t, n, h;                   // first tile, tiles; key head
  int key;                       // SINK: the group's first
  int page;                      // of the lane's group, -1: nobody sees it, or there is no such page
  float k_scale, v_scale;
};
template <bool FP8>
__device__ __forceinline__ void ask_scales(const CacheFwdParams& p, GroupBatch& b) {
  if ((uint32_t)b.page >= (uint32_t)p.batch.pages) b.page = -1;
  if constexpr (FP8) {
    if (b.page >= 0) {
      b.k_scale = p.k_scale[(int64_t)b.page * p.Hk + b.h];
      b.v_scale = p.v_scale[(int64_t)b.page * p.Hk + b.h];
    }
  }
}
template <bool FP8>
__device__ __forceinline__ GroupInfo info_of(const GroupBatch& b) {
  GroupInfo info{1.0f, 0.0f, 1.0f, b.page >= 0};
  if constexpr (FP8) {
    const float v = fmaxf(b.v_scale, 0x1p-64f);      // a scale of zero stays finite, and so do sums of weights over it
    info.k = b.k_scale;
    info.v_log2 = log2f(v);
    info.v_inv = 1.0f / v;
  }
  return info;
}

// Values that are not finite, under a mask.  In a tile that some rows of an item see only in part, a key has weight 0 for rows that do
// not see it, and 0 times an infinity or a NaN is NaN.  There such a value becomes 0 in the product's operand, and the rows
// that do see its key get it back at the end: a bit per row and channel for what has +infinity (or NaN) and one for -infinity (or NaN)
// coming.  (Tiles that every row sees whole need none of this, nor do keys that no row sees: their values become zeros.)
constexpr int kMarkSets = 4;             // of segments: whoever marks is at most two ahead of who reads
template <int D, int R, bool FP8>
struct Marks {
  static constexpr int kSigns = FP8 ? 1 : 2;         // E4M3 has no infinities
  static constexpr int kWords = D / 32;
  static constexpr int kBytes = kMarkSets * (R * kSigns * kWords + 4) * 4;
  uint32_t* at;
  __device__ __forceinline__ uint32_t* any(int set) const { return at + (set & (kMarkSets - 1)) * (R * kSigns * kWords + 4); }
  __device__ __forceinline__ uint32_t* row(int set, int r) const { return any(set) + 4 + r * kSigns * kWords; }
  // nothing marked: all of a CTA's threads for all sets, a warp for one
  __device__ __forceinline__ void clear_all() const {
    for (int i = threadIdx.x; i < kBytes / 4; i += blockDim.x) at[i] = 0u;
  }
  __device__ __forceinline__ void clear(int set) const {
    for (int i = threadIdx.x & 31; i < R * kSigns * kWords + 4; i += 32) any(set)[i] = 0u;
  }
  // x plus what is marked for it
  __device__ __forceinline__ float add(int set, int r, int channel, float x) const {
    const uint32_t* w = row(set, r) + channel / 32;
    const bool up = w[0] >> (channel % 32) & 1u, down = FP8 ? up : w[(kSigns - 1) * kWords] >> (channel % 32) & 1u;
    return x + (up ? INFINITY : 0.0f) + (down ? -INFINITY : 0.0f);
  }
};
// Whether some value of a word (four E4M3 codes, or two bf16) is not finite.
template <bool FP8>
__device__ __forceinline__ bool word_not_finite(uint32_t w) {
  if constexpr (FP8) return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0u;
  else return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
}
// Such a word of key `key`, channels from `channel` on: its values that are not finite are marked for the rows that see the key, and
// become zeros.  (Inlined, and in loops that stay loops: the operand warps have few registers, and no call may take more.)
template <int D, int R, bool FP8, bool SINK>
__device__ __forceinline__ uint32_t mark_word(const CacheFwdParams& p, const Marks<D, R, FP8> marks, int set, const Sequence seq, int row0, int rows, int key,
                                           int channel, uint32_t w) {
  constexpr int kPer = FP8 ? 4 : 2, kBits = 32 / kPer;
  uint32_t up = 0u, down = 0u, out = w;
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const uint32_t v = w >> (i * kBits) & (FP8 ? 0xffu : 0xffffu);
    const bool bad = FP8 ? (v & 0x7fu) == 0x7fu : (v & 0x7f80u) == 0x7f80u;
    if (!bad) continue;
    const bool nan = FP8 || (v & 0x7fu) != 0u;
    if (nan || !(v & 0x8000u)) up |= 1u << ((channel + i) % 32);
    if (nan || (v & 0x8000u)) down |= 1u << ((channel + i) % 32);
    out &= ~((FP8 ? 0xffu : 0xffffu) << (i * kBits));
  }
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    const int2 seen = visible_keys(p.causal, seq.first_pos() + fast_div(row0 + r, p.by_G), seq.len);
    if (!sees<SINK>(p.causal, seen, key)) continue;
    uint32_t* to = marks.row(set, r) + channel / 32;
    if (up) atomicOr(to, up);
    if (!FP8 && down) atomicOr(to + (Marks<D, R, FP8>::kSigns - 1) * Marks<D, R, FP8>::kWords, down);
    *reinterpret_cast<volatile uint32_t*>(marks.any(set)) = 1u;
  }
  return out;
}

// the status of a call: the first CTA's work
template <bool SINK>
__device__ __forceinline__ void check_call(const CacheFwdParams& p, int* s_bad) {
  check_batch<SINK>(p.batch, s_bad, [&](const Sequence& s) {
    if (s.n == 0) return make_int2(0, 0);
    const int lo = visible_keys(p.causal, s.first_pos(), s.len).x, hi = visible_keys(p.causal, s.len - 1, s.len).y;
    return make_int2(lo >> p.batch.page_shift, (hi + (1 << p.batch.page_shift) - 1) >> p.batch.page_shift);
  }, p.causal.sink);
  leave_status(p.status, s_bad);
}
template <int R, int TK, int OVER, bool SINK>
__device__ __forceinline__ void note_border(const CacheFwdParams& p, int worker, bool works, int share, const Stretch<R, TK, OVER, SINK>& g) {
  Border b{};
  if (works) b = {g.c.at, g.c.item.units(), share, g.c.seq.start, g.row0, g.rows, g.c.h, 0};
  reinterpret_cast<int4*>(p.borders + worker)[0] = reinterpret_cast<const int4*>(&b)[0];
  reinterpret_cast<int4*>(p.borders + worker)[1] = reinterpret_cast<const int4*>(&b)[1];
}

// Adds up what several stretches have left of an item, in the order of the line.  CTA w looks at the border in front of stretch
// w + 1 and does the item if that is the first border inside it.  A warp takes a row, or, of an item of few rows,
// every n-th part of a row, since what this kernel spends is the time of a few loads one after the other.
constexpr int kCombineThreads = 512;
template <int D, int R>
__global__ void __launch_bounds__(kCombineThreads)
combine_kernel(const __grid_constant__ CacheFwdParams p) {
  static_assert(R < 128, "parts of 128 rows and more lie in another order");
  constexpr int kVec = D / 32, kWarps = kCombineThreads / 32;
  __shared__ float s_acc[kWarps][D + 2];
  pdl_wait();
  const int4 b0 = reinterpret_cast<const int4*>(p.borders + blockIdx.x + 1)[0], b1 = reinterpret_cast<const int4*>(p.borders + blockIdx.x + 1)[1];
  const int before = b0.x, units = b0.y, share = b0.z, token0 = b0.w, row0 = b1.x, rows = b1.y, h = b1.z;
  if (before == 0 || before > share) return;
  const int w0 = blockIdx.x, parts = 1 + (units - before + share - 1) / share;
  // the stretch in front holds the item's beginning as its last segment (its only one where it begins with it), the others as their first
  auto slot_of = [&](int i) { return 2 * (w0 + i) + (i > 0 || before == share ? 0 : 1); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = rows >= kWarps ? 1 : kWarps / rows;           // warps of a row
  const int share_of_row = warp % split;
  for (int r = warp / split; r - warp / split < rows; r += kWarps / split) {
    const bool there = r < rows && warp / split < kWarps / split;
    float top = -INFINITY, sum = 0.0f, acc[kVec] = {};
    if (there) {
      for (int i = lane; i < parts; i += 32) top = fmaxf(top, p.part_ml[((int64_t)slot_of(i) * R + r) * 2]);
    }
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
    if (there) {
#pragma unroll 8
      for (int i = share_of_row; i < parts; i += split) {
        const int64_t at = (int64_t)slot_of(i) * R + r;
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + at * 2);
        const float f = top == -INFINITY ? 0.0f : fast_exp2(ml.x - top);
        sum = fmaf(ml.y, f, sum);
        const float* src = p.part_o + at * D + lane * kVec;
        float v[kVec];
        if constexpr (kVec == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(src);
        else *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(src);
#pragma unroll
        for (int j = 0; j < kVec; ++j) acc[j] = ml.x == -INFINITY ? acc[j] : fmaf(v[j], f, acc[j]);      // (a part without keys has left no output)
      }
    }
    if (split > 1) {
#pragma unroll
      for (int j = 0; j < kVec; ++j) s_acc[warp][lane * kVec + j] = acc[j];
      if (lane == 0) s_acc[warp][D] = sum;
      __syncthreads();
      if (there && share_of_row == 0) {
        for (int i = 1; i < split; ++i) {
#pragma unroll
          for (int j = 0; j < kVec; ++j) acc[j] += s_acc[warp + i][lane * kVec + j];
          sum += s_acc[warp + i][D];
        }
      }
      __syncthreads();
    }
    if (!there || share_of_row != 0) continue;
    const int row = row0 + r, of = fast_div(row, p.by_G), token = token0 + of, head = h * p.G + row - of * p.G;
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + (int64_t)token * p.out_stride_t + head * p.out_stride_h + lane * kVec);
#pragma unroll
    for (int j = 0; j < kVec / 2; ++j) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(acc[2 * j] * inv, acc[2 * j + 1] * inv);
      dst[j] = *reinterpret_cast<const uint32_t*>(&v);
    }
    if (p.lse && lane == 0) p.lse[(int64_t)token * p.H + head] = sum == 0.0f ? -INFINITY : (top - kBase + log2f(sum)) * 0.6931471805599453f;
  }
}

// The same for items of 128 rows and more.  A lane has a row and a warp two groups of four channels, as the parts lie in memory (what a softmax
// thread has of its row in registers goes there a line at a time); rows of the output come together in shared memory.
// Pieces are 32 rows by 64 channels, dealt out to the CTAs of all of an item's borders, gridDim.y each, so that an item of many parts has many CTAs; three parts are
// on their way at a time, and the code is one loop without a remainder, since it comes from memory at every call.  Five tokens of 8 heads of one sequence of
// 131,072 keys, 148 parts: 53 us (whole rows by the first border's four CTAs 78; two or four parts at a time 57 and 51); five of 64 heads of 8 sequences,
// 3 parts: 68 (70; 69 and 69); 52 of 8 heads over 2 of 6 sequences of up to 26,175, bf16: 40 (57; 41 and 40); a prompt of 5000 tokens of 4 heads 54 (54; 53 and 55).
constexpr int kCombineRowsThreads = 256, kCombineRowsCtas = 6;
template <int D, int R>
__global__ void __launch_bounds__(kCombineRowsThreads, 4)
combine_rows_kernel(const __grid_constant__ CacheFwdParams p) {
  constexpr int kWarps = kCombineRowsThreads / 32, kGroups = 2, kAtOnce = 3, kPieces = D / 4 / (kWarps * kGroups), kPitch = kWarps * kGroups * 4 + 8;
  __shared__ __align__(16) __nv_bfloat16 s_out[32 * kPitch];
  __shared__ float s_top[kWarps][32];
  pdl_wait();
  const int4 b0 = reinterpret_cast<const int4*>(p.borders + blockIdx.x + 1)[0], b1 = reinterpret_cast<const int4*>(p.borders + blockIdx.x + 1)[1];
  const int units = b0.y, share = b0.z, token0 = b0.w, row0 = b1.x, rows = b1.y, h = b1.z;
  if (b0.x == 0) return;
  const int border = b0.x > share ? (b0.x - 1) / share : 0, before = b0.x - border * share;         // which of the item's this is; units in front of the first one
  const int w0 = (int)blockIdx.x - border, parts = 1 + (units - before + share - 1) / share;
  auto slot_of = [&](int i) { return 2 * (w0 + i) + (i > 0 || before == share ? 0 : 1); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // (items of fewer than 16 rows: every n-th part by itself, then the sums of these, the order that calls of many sequences with few rows have had)
  const int split = rows >= 16 ? 1 : 16 / rows;
  const bool few = split == 1 && parts <= kAtOnce;      // all on their way at once: what the largest is shows from them
#pragma unroll 1
  for (int piece = border * (int)gridDim.y + (int)blockIdx.y; piece < (rows + 31) / 32 * kPieces; piece += (parts - 1) * (int)gridDim.y) {
    const int r0 = piece / kPieces * 32, g0 = piece % kPieces * (kWarps * kGroups);         // first row, first group of four channels
    const int r = r0 + lane;      // (rows behind the item's last are parts' rows all the same, of no meaning)
    float top = -INFINITY;
    if (!few) {
#pragma unroll 4
      for (int i = warp; i < parts; i += kWarps) top = fmaxf(top, p.part_ml[((int64_t)slot_of(i) * R + r) * 2]);
      s_top[warp][lane] = top;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWarps; ++i) top = fmaxf(top, s_top[i][lane]);
    }
    auto add_up = [&](int k, float& sum, float (&acc)[kGroups][4]) {
#pragma unroll 1
      for (int i0 = k; i0 < parts; i0 += kAtOnce * split) {
        float2 ml[kAtOnce];
        float4 v[kAtOnce][kGroups];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int i = i0 + u * split, slot = slot_of(i);
          ml[u] = make_float2(-INFINITY, 0.0f);      // (adds nothing)
          if (i < parts) ml[u] = *reinterpret_cast<const float2*>(p.part_ml + ((int64_t)slot * R + r) * 2);
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            v[u][g] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (i < parts) v[u][g] = *reinterpret_cast<const float4*>(p.part_o + (((int64_t)slot * (D / 4) + g0 + warp + g * kWarps) * R + r) * 4);
          }
        }
        if (few) {
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) top = fmaxf(top, ml[u].x);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const float f = top == -INFINITY ? 0.0f : fast_exp2(ml[u].x - top);
          sum = fmaf(ml[u].y, f, sum);
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            const float x[4] = {v[u][g].x, v[u][g].y, v[u][g].z, v[u][g].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[g][j] = ml[u].x == -INFINITY ? acc[g][j] : fmaf(x[j], f, acc[g][j]);      // (a part without keys has left no output)
          }
        }
      }
    };
    float sum = 0.0f, acc[kGroups][4] = {};
    add_up(0, sum, acc);
#pragma unroll 1
    for (int k = 1; k < split; ++k) {
      float sum_k = 0.0f, acc_k[kGroups][4] = {};
      add_up(k, sum_k, acc_k);
      sum += sum_k;
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[g][j] += acc_k[g][j];
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const __nv_bfloat162 a = __floats2bfloat162_rn(acc[g][0] * inv, acc[g][1] * inv), b = __floats2bfloat162_rn(acc[g][2] * inv, acc[g][3] * inv);
      *reinterpret_cast<uint2*>(s_out + lane * kPitch + (warp + g * kWarps) * 4) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
    if (p.lse && g0 == 0 && warp == 0 && r < rows) {
      const int row = row0 + r, of = fast_div(row, p.by_G);
      p.lse[(int64_t)(token0 + of) * p.H + h * p.G + row - of * p.G] = sum == 0.0f ? -INFINITY : (top - kBase + log2f(sum)) * 0.6931471805599453f;
    }
    __syncthreads();
    constexpr int kLanes = kGroups * kWarps / 2;      // 16 bytes each
#pragma unroll 1
    for (int i = threadIdx.x; i < 32 * kLanes; i += kCombineRowsThreads) {
      const int mine = i / kLanes, c = i % kLanes;
      if (r0 + mine >= rows) continue;
      const int row = row0 + r0 + mine, of = fast_div(row, p.by_G);
      *reinterpret_cast<uint4*>(p.out + (int64_t)(token0 + of) * p.out_stride_t + (h * p.G + row - of * p.G) * p.out_stride_h + g0 * 4 + c * 8) =
          *reinterpret_cast<const uint4*>(s_out + mine * kPitch + c * 8);
    }
    __syncthreads();
  }
}

}  // namespace sparkattn
