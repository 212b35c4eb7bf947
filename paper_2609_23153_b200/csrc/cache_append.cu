// sparkattn_cache_append: new keys and values into a paged cache (bf16, or E4M3 with a scale per page and head), keys and
// queries rotated by their positions on the way.
//
// The rotation is a 2 x 2 product per channel pair; the quantisation of a page needs the largest |x| of its new tokens
// before the first code, so a page's tokens of one head stay in registers between the two: HBM sees every row once.
// A unit is the new tokens of one (sequence, page) and some of its lines; a line is one head of K, of V or of the queries.  Four threads
// per token (at least a warp) work on a unit.  The tokens' cosines and sines, which all heads share, go to shared memory
// once; then the lines are taken one after the other, the next one's rows on their way (asynchronous copies, each thread's own)
// while this one is encoded.
// Bandwidth bounds it.  Measured (128 channels, bytes read and written; a copy's rate is 6.46 TB/s): prompts of up to 4001 tokens,
// 8 sequences, 32 query and 8 key heads, bf16 pages of 64, half the channels rotated: 425 MB in 74 us = 5.8 TB/s, 0.89 of it.  4680
// tokens of 12 heads (three frames of 1560), E4M3 pages of 128, positions of three axes: 74 MB in 19 us = 3.9 TB/s; the
// SMs issue an instruction in six of ten clocks, rotating and encoding, and the one wave has its beginning and end to itself.  One token for each of 128 sequences
// 5.0 us, for one 2.7: latency.  With the norm of keys and queries (NORM) the frames take 24.5 us, a line of a page 3.3 of them, over bf16 pages 20.6, and the
// tokens 6.05 and 5.55.
#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "cache.h"
#include "rows.cuh"
#include "tmap.h"

namespace sparkattn {

struct RowsView {
  __nv_bfloat16* data;
  int64_t stride_t, stride_h;
};
struct AppendParams {
  BatchView batch;
  RotaryView rotary;             // rot = 0: nothing is rotated
  NormView norm;
  RowsView q, k, v, q_out;       // q.data NULL: no queries
  unsigned char* k_cache;
  unsigned char* v_cache;
  float* k_scale;
  float* v_scale;
  int64_t stride_page, stride_h, stride_n;
  int H, Hk;
  int pages_each;                // pages of a sequence that max_new tokens can reach
  FastDiv by_pages_each, by_groups, by_B;
  int lines;                     // of a (sequence, page): K and V of every key head, then the queries
  int groups;                    // units that share them: unit g takes lines g, g + groups, ...
  int units;
  int budget, one;               // budget more than 0: units of a sequence, by whether it reaches one page, of `one` units, or two, of `groups` each (see its_share)
  int32_t* status;
};

// cosines and sines of a unit's tokens as [rows][pairs], from the tables; a pair outside them is turned by nothing
__device__ __forceinline__ void gather_phases(const RotaryView& r, int rows, int t0, int pos0, float* s_cos, float* s_sin, int tid, int threads) {
  const int quads = r.rot / 8;                             // of four pairs
  for (int i = tid; i < rows * quads; i += threads) {
    const int row = i / quads, m = (i - row * quads) * 4;
    const int32_t* at = r.positions + (int64_t)(t0 + row) * r.axes;
    float4 c = make_float4(1.0f, 1.0f, 1.0f, 1.0f), s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (r.axis == nullptr) {
      const uint32_t e = r.positions ? at[0] : pos0 + row;
      if (e < (uint32_t)r.rows) {
        c = *reinterpret_cast<const float4*>(r.cos + (e * (r.rot / 2) + m));
        s = *reinterpret_cast<const float4*>(r.sin + (e * (r.rot / 2) + m));
      }
    } else {
      float* cc = &c.x;
      float* ss = &s.x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t ax = r.axis[m + j];
        const uint32_t e = ax >= (uint32_t)r.axes ? 0xffffffffu : r.positions ? (uint32_t)at[ax] : (uint32_t)(pos0 + row);
        if (e < (uint32_t)r.rows) {
          cc[j] = r.cos[e * (r.rot / 2) + m + j];
          ss[j] = r.sin[e * (r.rot / 2) + m + j];
        }
      }
    }
    *reinterpret_cast<float4*>(s_cos + row * (r.rot / 2) + m) = c;
    *reinterpret_cast<float4*>(s_sin + row * (r.rot / 2) + m) = s;
  }
}
// bits of the largest |x|, NaN aside; or of the finite ones
template <bool FINITE>
__device__ __forceinline__ uint32_t largest_bits(const Chunk& c, uint32_t top) {
  float m = __uint_as_float(top);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float a = fabsf(c.x[j]);
    m = fmaxf(m, FINITE && !(a < INFINITY) ? 0.0f : a);
  }
  return __float_as_uint(m);
}
// smallest power of two s with amax <= 448 s (448 = 1.75 * 2^8), from the bits of amax >= 1e-12
__device__ __forceinline__ float power_scale(uint32_t amax_bits) {
  const uint32_t u = max(amax_bits, __float_as_uint(1e-12f));
  return __uint_as_float(((u >> 23) - 8u + ((u & 0x7fffffu) > 0x600000u ? 1u : 0u)) << 23);
}
__device__ __forceinline__ uint2 encode(const Chunk& c, float inv) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(c.x[2 * j], inv), __fmul_rn(c.x[2 * j + 1], inv)), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
__device__ __forceinline__ Chunk decode(uint2 codes) {
  Chunk c;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t pair = (j < 2 ? codes.x : codes.y) >> (16 * (j & 1));
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3)));
    c.x[2 * j] = f.x;
    c.x[2 * j + 1] = f.y;
  }
  return c;
}

// The new tokens of a (sequence, page).
struct Part {
  int page, held;              // the page, -1: nothing to do; tokens there before
  int rows, t0, pos0;          // new tokens; row of the call and position of the first
};
__device__ __forceinline__ Part part_of(const AppendParams& p, int b, int j, const Sequence& s) {
  Part u{-1, 0, 0, 0, 0};
  const int first = max(s.first_pos(), 0), number = (first >> p.batch.page_shift) + j;
  u.pos0 = max(number << p.batch.page_shift, first);
  u.rows = min((number + 1) << p.batch.page_shift, s.len) - u.pos0;
  if (u.rows <= 0 || number >= p.batch.max_pages) { u.rows = 0; return u; }
  u.held = u.pos0 & ((1 << p.batch.page_shift) - 1);
  u.t0 = s.start + u.pos0 - s.first_pos();
  u.page = p.batch.page_table[(int64_t)b * p.batch.max_pages + number];
  if ((uint32_t)u.page >= (uint32_t)p.batch.pages) u.page = -1;
  return u;
}

// Which page of its sequence a unit takes, and of its lines every groups-th from `first` on.
struct Share {
  int j, first, groups;
};
// Where sequences reach two pages at most, by where they begin in one, each has its units for those that it does reach.  From the first token on: 108 tokens of
// each of 4, pages of 128, 32 + 2 x 8 heads, 5.5 us, with units for two pages of each 7.7; up to 120 of each of 60, 8 + 2 x 8, bf16, 14.3 and 18.6.  From anywhere:
// 60 of each of 20, pages of 64, 8 + 2 x 8 heads, 9.4 and 10.4, where units for one page of each take 13.7; up to 120 of each of 60 18.6 and 17.4 (18.4).
__device__ __forceinline__ Share its_share(const AppendParams& p, int unit, const Sequence& s) {
  const int first = max(s.first_pos(), 0);
  const bool two = s.len > first && (s.len - 1) >> p.batch.page_shift > first >> p.batch.page_shift;
  const int groups = two ? p.groups : p.one, j = unit >= groups;
  return {j + (unit >= 2 * groups), unit - j * groups, groups};
}

template <int D, int ROWS>
struct UnitShape {
  static constexpr int kLanes = D / 8;                             // threads of a row
  static constexpr int U = ROWS * 4 < 32 ? 32 : ROWS * 4;          // threads of a unit
  static constexpr int kThreads = U < 256 ? 256 : U;               // of a CTA
  static constexpr int kRowsAtOnce = U / kLanes;
  static constexpr int C = (ROWS + kRowsAtOnce - 1) / kRowsAtOnce;
  // rows on their way, then cosines and sines
  static constexpr int kRowBytes = kThreads * C * 16;
  static size_t smem(int rot) { return kRowBytes + (size_t)(kThreads / U) * ROWS * rot * sizeof(float); }
  // CTAs per SM: 64 registers a thread, or 80 where norm and codes of a page's 128 channels need them (8 prompts of up to 4706 tokens, 48 + 2 x 4 heads, pages of
  // 32 and 64: 114 and 116 us by three, 127 and 126 by four; without the norm 108 and 102)
  static constexpr int per_sm(bool fp8, bool norm) { return fp8 && norm && D == 128 && U > 32 && kThreads == 256 ? 3 : 1024 / kThreads; }
};

// Lines first, first + step, ... of a unit: the threads hold its up to ROWS new rows of one of them, 16 bytes of a row each at a time.
// NORM: keys and queries are normalised first.
template <int D, bool FP8, int ROWS, bool NORM>
__device__ __forceinline__ void append_lines(const AppendParams& p, const Part& u, int first, int step, int group, uint32_t* s_max,
                                             const float* s_cos, const float* s_sin) {
  using S = UnitShape<D, ROWS>;
  constexpr int U = S::U, C = S::C;
  const int tid = threadIdx.x % U, chunk = tid % S::kLanes, row0 = tid / S::kLanes;
  const RotaryView& rot = p.rotary;
  const int pairs = rot.rot / 2, half = rot.rot / 16;            // chunks per side
  const bool on = chunk * 8 < rot.rot, second = chunk >= half;
  // where this chunk's pairs lie, and (halves) the lane with their other sides: the lanes of a row hold its chunks in order
  const int m0 = rot.interleaved ? chunk * 4 : (second ? chunk - half : chunk) * 8;
  const int partner = (threadIdx.x & 31 & ~(S::kLanes - 1)) + (!on ? chunk : second ? chunk - half : chunk + half);
  const float sign = second ? 1.0f : -1.0f;
  [[maybe_unused]] Chunk weight;                                 // NORM: of the line's head
  // row r's chunk turned (lanes of a row together: halves pass their chunks on)
  auto turned = [&](uint4 v, int r, bool there) {
    const float* c = s_cos + r * pairs + m0;
    const float* s = s_sin + r * pairs + m0;
    if constexpr (NORM) {
      const Chunk x = normed<D>(widen(v), weight, p.norm.eps);
      if (rot.rot == 0) return x;
      if (rot.interleaved) {
        if (!on || !there) return x;
        const float4 cc = *reinterpret_cast<const float4*>(c), ss = *reinterpret_cast<const float4*>(s);
        return turn_pairs_fused({cc.x, cc.y, cc.z, cc.w}, {ss.x, ss.y, ss.z, ss.w}, x);
      }
      const Chunk far = chunk_of(x, partner);
      if (!on || !there) return x;
      const float4 c0 = reinterpret_cast<const float4*>(c)[0], c1 = reinterpret_cast<const float4*>(c)[1];
      const float4 s0 = reinterpret_cast<const float4*>(s)[0], s1 = reinterpret_cast<const float4*>(s)[1];
      return turn_halves_fused({c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w},
                               {s0.x * sign, s0.y * sign, s0.z * sign, s0.w * sign, s1.x * sign, s1.y * sign, s1.z * sign, s1.w * sign}, x, far);
    }
    if (rot.interleaved) return on && there ? turn_pairs(c, s, widen(v)) : widen(v);
    const uint4 far = make_uint4(__shfl_sync(0xffffffffu, v.x, partner), __shfl_sync(0xffffffffu, v.y, partner), __shfl_sync(0xffffffffu, v.z, partner),
                                 __shfl_sync(0xffffffffu, v.w, partner));
    return on && there ? turn_halves(c, s, widen(v), widen(far), sign) : widen(v);
  };
  extern __shared__ __align__(16) unsigned char s_raw[];
  const uint32_t mine = smem_u32(s_raw) + threadIdx.x * 16;      // the thread's places, kThreads * 16 bytes apart
  float old = 0.0f;                                              // E4M3: the scale of the line's page, if it held tokens
  auto scale_of = [&](int n) { return (n < p.Hk ? p.k_scale + n : p.v_scale + n - p.Hk) + (int64_t)u.page * p.Hk; };
  auto fetch = [&](int n) {
    const bool key = n < p.Hk, query = n >= 2 * p.Hk;
    const RowsView& from = key ? p.k : query ? p.q : p.v;
    const int h = key ? n : query ? n - 2 * p.Hk : n - p.Hk;
    const int rows = query || u.page >= 0 ? u.rows : 0;
    const __nv_bfloat16* src = from.data + h * from.stride_h + (int64_t)(u.t0 + row0) * from.stride_t + chunk * 8;
    const int64_t by = S::kRowsAtOnce * from.stride_t;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      if (row0 + i * S::kRowsAtOnce < rows) cp_async16(mine + i * S::kThreads * 16, src);
      src += by;
    }
    cp_async_commit();
    if constexpr (FP8) old = !query && rows > 0 && u.held > 0 ? *scale_of(n) : 0.0f;
  };
  fetch(first);
  [[maybe_unused]] const void* weight_of = nullptr;
  [[maybe_unused]] bool weighted = false;
  int turn_of = 0;                                               // which half of s_max this line takes
#pragma unroll 1
  for (int n = first; n < p.lines; n += step) {
    const bool query = n >= 2 * p.Hk, rotate = (n < p.Hk || query) && (NORM || rot.rot > 0);
    const int h = n < p.Hk ? n : query ? n - 2 * p.Hk : n - p.Hk;
    if constexpr (NORM) {
      // (one head's weights serve the other heads' lines where all heads share them)
      const void* from = query ? p.norm.q_weight : p.norm.k_weight;
      if (rotate && (!weighted || p.norm.stride != 0 || from != weight_of)) {
        weight = norm_weights(p.norm, from, h, chunk * 8);
        weight_of = from;
        weighted = true;
      }
    }
    const int rows = query || u.page >= 0 ? u.rows : 0;
    uint4 raw[C];
    cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < C; ++i)
      raw[i] = row0 + i * S::kRowsAtOnce < rows ? *reinterpret_cast<const uint4*>(s_raw + (threadIdx.x + i * S::kThreads) * 16) : make_uint4(0u, 0u, 0u, 0u);
    const float before = old;
    if (n + step < p.lines) fetch(n + step);
    if (!FP8 || query) {
      // bf16 to bf16
      unsigned char* at = query ? reinterpret_cast<unsigned char*>(p.q_out.data + h * p.q_out.stride_h + (int64_t)(u.t0 + row0) * p.q_out.stride_t + chunk * 8)
                                : (n < p.Hk ? p.k_cache : p.v_cache) + ((int64_t)u.page * p.stride_page + h * p.stride_h + (int64_t)(u.held + row0) * p.stride_n + chunk * 8) * 2;
      const int64_t by = 2 * S::kRowsAtOnce * (query ? p.q_out.stride_t : p.stride_n);
      uint4 y[C];
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const int r = row0 + i * S::kRowsAtOnce;
        y[i] = rotate ? narrow(turned(raw[i], r, r < rows)) : raw[i];
      }
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if (row0 + i * S::kRowsAtOnce < rows) *reinterpret_cast<uint4*>(at) = y[i];
        at += by;
      }
    } else {
      unsigned char* page = (n < p.Hk ? p.k_cache : p.v_cache) + (int64_t)u.page * p.stride_page + h * p.stride_h + chunk * 8;
      Chunk x[C];
      uint32_t amax = 0;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const int r = row0 + i * S::kRowsAtOnce;
        x[i] = rotate ? turned(raw[i], r, r < rows) : widen(raw[i]);
        amax = largest_bits<false>(x[i], amax);
      }
      float* scale_at = scale_of(n);
      amax = __reduce_max_sync(0xffffffffu, amax);
      if (amax >= 0x7f800000u) {                                 // infinities among them: the finite ones count
        amax = 0;
#pragma unroll
        for (int i = 0; i < C; ++i) amax = largest_bits<true>(x[i], amax);
        amax = __reduce_max_sync(0xffffffffu, amax);
      }
      if constexpr (U > 32) {
        uint32_t* s = s_max + turn_of * (S::kThreads / 32);
        turn_of ^= 1;
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = amax;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(U) : "memory");
        amax = __reduce_max_sync(0xffffffffu, s[group * (U / 32) + (threadIdx.x & 31) % (U / 32)]);
      }
      float scale = power_scale(amax);
      if (u.held > 0 && before >= scale) scale = before;
      const float inv = 1.0f / scale;
      if (rows > 0 && u.held > 0 && scale > before) {
        const float again = __fmul_rn(before, inv);
        for (int r = row0; r < u.held; r += S::kRowsAtOnce) {
          uint2* codes = reinterpret_cast<uint2*>(page + (int64_t)r * p.stride_n);
          *codes = encode(decode(*codes), again);
        }
      }
      unsigned char* at = page + (int64_t)(u.held + row0) * p.stride_n;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if (row0 + i * S::kRowsAtOnce < rows) *reinterpret_cast<uint2*>(at) = encode(x[i], inv);
        at += S::kRowsAtOnce * p.stride_n;
      }
      // (every thread of a larger unit has the page's scale of before: it arrived in front of the barrier above)
      __syncwarp();
      if (rows > 0 && tid == 0) *scale_at = scale;
    }
  }
}

template <int D, bool FP8, int ROWS, bool NORM>
__global__ void __launch_bounds__(UnitShape<D, ROWS>::kThreads, UnitShape<D, ROWS>::per_sm(FP8, NORM))
cache_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int kThreads = UnitShape<D, ROWS>::kThreads;
  __shared__ uint32_t s_max[2 * kThreads / 32];
  extern __shared__ __align__(16) unsigned char s_raw[];
  __shared__ int s_bad[2];
  pdl_wait();
  if (blockIdx.x == 0) {
    const int shift = p.batch.page_shift;
    check_batch<false>(p.batch, s_bad, [&](const Sequence& s) { return make_int2(max(s.first_pos(), 0) >> shift, s.n == 0 ? 0 : (s.len + (1 << shift) - 1) >> shift); });
    if (p.rotary.rot > 0) {
      const RotaryView& r = p.rotary;
      auto bad = [&](int detail) { if (atomicExch(s_bad, 1) == 0) s_bad[1] = detail; };
      if (r.positions) {
        // sixteen bytes at a time where they lie so: 105 sequences of up to 2784 tokens, three axes, 10 + 2 x 2 heads of 64 channels take 110 us, which number by
        // number waited for this CTA, 200.  (A few rounds of the other loop by that: a token of each of 100 sequences 3.9 us, and 4.8 by both loops.)
        const long long n = (long long)p.batch.T * r.axes, quads = n > 32 * kThreads && reinterpret_cast<uintptr_t>(r.positions) % 16 == 0 ? n / 4 : 0;
#pragma unroll 1
        for (long long first = threadIdx.x; first < quads; first += 8 * kThreads) {
          int4 at[8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            at[i] = first + i * kThreads < quads ? reinterpret_cast<const int4*>(r.positions)[first + i * kThreads] : make_int4(0, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            for (const int e : {at[i].x, at[i].y, at[i].z, at[i].w})
              if ((uint32_t)e >= (uint32_t)r.rows) bad(e);
        }
#pragma unroll 1
        for (long long first = 4 * quads + threadIdx.x; first < n; first += 8 * kThreads) {
          int at[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) at[i] = first + i * kThreads < n ? r.positions[first + i * kThreads] : 0;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if ((uint32_t)at[i] >= (uint32_t)r.rows) bad(at[i]);
        }
      } else {
        for (int b = threadIdx.x; b < p.batch.B; b += kThreads) {
          const Sequence s = sequence_of(p.batch, b);
          if (s.n > 0 && s.len > r.rows) bad(s.len - 1);
        }
      }
      if (r.axis)
        for (int m = threadIdx.x; m < r.rot / 2; m += kThreads)
          if ((uint32_t)r.axis[m] >= (uint32_t)r.axes) bad(r.axis[m]);
    }
    leave_status(p.status, s_bad);
    return;
  }
  constexpr int U = UnitShape<D, ROWS>::U;
  // (the same in all lanes, which the compiler has to see: with the unit's numbers in vector registers pages of 32 and less spilled, 178 us instead of 127)
  const int group = __shfl_sync(0xffffffffu, (int)threadIdx.x / U, 0);
  const int unit = (int)(blockIdx.x - 1) * (kThreads / U) + group;
  if (unit >= p.units) return;
  // (the sequences' first units, then their second ones and so on: those of less to do come last, and the SMs have as many of them each)
  const bool budget = U > 32 && p.budget > 0;
  const int of = fast_div(unit, budget ? p.by_B : p.by_groups), b = budget ? unit - of * p.batch.B : fast_div(of, p.by_pages_each);
  const Sequence s = sequence_of(p.batch, b);
  const Share share = budget ? its_share(p, of, s) : Share{of - b * p.pages_each, unit - of * p.groups, p.groups};
  const Part u = part_of(p, b, share.j, s);
  if (u.rows <= 0) return;
  float* s_cos = reinterpret_cast<float*>(s_raw + UnitShape<D, ROWS>::kRowBytes) + group * ROWS * p.rotary.rot;
  float* s_sin = s_cos + ROWS * (p.rotary.rot / 2);
  if (p.rotary.rot > 0) {
    gather_phases(p.rotary, u.rows, u.t0, u.pos0, s_cos, s_sin, threadIdx.x % U, U);
    if constexpr (U > 32) asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(U) : "memory");
    else __syncwarp();
  }
  append_lines<D, FP8, ROWS, NORM>(p, u, share.first, share.groups, group, s_max, s_cos, s_sin);
}

template <int D, bool FP8, bool NORM>
static int launch_rows(const AppendParams& given, int rows, cudaStream_t stream) {
  auto go = [&](auto kern, auto shape) {
    constexpr int kThreads = decltype(shape)::kThreads, per = kThreads / decltype(shape)::U;
    AppendParams p = given;
    p.lines = 2 * p.Hk + (p.q.data ? p.H : 0);
    // One wave of CTAs where that leaves a unit at most sixteen lines, else units of eight
    const long long parts = (long long)p.batch.B * p.pages_each, slots = (long long)per * decltype(shape)::per_sm(FP8, NORM) * current_sm_count();
    auto groups_for = [&](long long wave, long long pages) { return (int)std::min<long long>(std::max<long long>(wave / pages, 1), p.lines); };
    auto lines_of = [&](int groups) { return (p.lines + groups - 1) / groups; };
    p.groups = groups_for(slots, parts);
    if (p.lines > 16 * p.groups) {
      p.groups = (p.lines + 7) / 8;
    } else {
      // ... or a wave of the pages that T new tokens reach on average, wherever in a page they begin, and a little more, where that leaves a unit fewer lines.
      // Three frames of 1560 tokens by eight units a page instead of seven 19.5 us for 20.9, and 20.3 for 21.0 where they reach a page more; 16 sequences of up to
      // 400 tokens over pages of 128, 64 channels, 17.4 and 25.0.  The CTAs of pages that are not reached cost what they take to begin, so units of few lines or of four
      // tokens have to get half as many by a third more CTAs at most: two tokens of each of 186, 48 lines, 7.3 us
      // otherwise and 5.8.  (By one page of every sequence less than it could reach: 256 tokens of each of 8 over pages of 128 17.0 instead of 12.4.)
      const int g = groups_for(slots + slots / 32, p.batch.B + (p.batch.T - p.batch.B + (1 << p.batch.page_shift) - 1) / (1 << p.batch.page_shift));
      const int before = lines_of(p.groups), after = lines_of(g);
      if (before >= 4 && rows > 4 ? after < before : 2 * after <= before && 3 * parts * g <= 4 * slots) p.groups = g;
    }
    if (rows > 4 && p.pages_each == 2 && slots >= 4LL * p.batch.B) {
      // a wave of one page of every sequence for those that reach one, and for the others half of that where it is enough
      p.one = groups_for(slots, p.batch.B);
      if (slots >= 4 * parts) p.groups = groups_for(slots / p.batch.B, 2);
      else if (p.lines > 16 * p.one) p.one = p.groups;
      p.budget = std::max(p.one, 2 * p.groups);
    }
    const long long units = p.budget > 0 ? (long long)p.budget * p.batch.B : parts * p.groups;
    if (units > 0x7fffff00LL) return (int)SPARKATTN_E_UNSUPPORTED_SHAPE;
    p.units = (int)units;
    p.by_pages_each = make_fast_div(p.pages_each);
    p.by_groups = make_fast_div(p.groups);
    p.by_B = make_fast_div(p.batch.B);
    const unsigned ctas = 1 + (unsigned)((units + per - 1) / per);
    const size_t smem = decltype(shape)::smem(p.rotary.rot);
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)decltype(shape)::smem(D)) != cudaSuccess) return (int)SPARKATTN_E_CUDA;
    return launch_kernel(kern, dim3(ctas), kThreads, smem, true, stream, p);
  };
  if (rows <= 4) return go(cache_append_kernel<D, FP8, 4, NORM>, UnitShape<D, 4>{});
  if (rows <= 16) return go(cache_append_kernel<D, FP8, 16, NORM>, UnitShape<D, 16>{});
  if (rows <= 32) return go(cache_append_kernel<D, FP8, 32, NORM>, UnitShape<D, 32>{});
  if (rows <= 64) return go(cache_append_kernel<D, FP8, 64, NORM>, UnitShape<D, 64>{});
  return go(cache_append_kernel<D, FP8, 128, NORM>, UnitShape<D, 128>{});
}

int launch_cache_append(const sparkattn_cache_t& c, const sparkattn_batch_t& b, const sparkattn_norm_t* norm, const sparkattn_rotary_t* rotary,
                        const sparkattn_rows_t* q, int H, const sparkattn_rows_t& k, const sparkattn_rows_t& v, void* k_cache, void* v_cache, float* k_scale,
                        float* v_scale, const sparkattn_rows_t* q_out, void* workspace, cudaStream_t stream) {
  AppendParams p{};
  p.batch = make_batch_view(c, b);
  p.rotary = make_rotary_view(rotary);
  p.norm = make_norm_view(norm, c.d);
  auto view = [](const sparkattn_rows_t& r) { return RowsView{static_cast<__nv_bfloat16*>(r.data), r.stride_t, r.stride_h}; };
  if (q) { p.q = view(*q); p.q_out = view(*q_out); }
  p.k = view(k);
  p.v = view(v);
  p.k_cache = static_cast<unsigned char*>(k_cache);
  p.v_cache = static_cast<unsigned char*>(v_cache);
  p.k_scale = k_scale; p.v_scale = v_scale;
  p.stride_page = c.stride_page; p.stride_h = c.stride_h; p.stride_n = c.stride_n;
  p.H = H; p.Hk = c.H;
  p.pages_each = (b.max_new - 1 + c.page - 1) / c.page + 1;
  p.status = static_cast<int32_t*>(workspace);
  const int rows = c.page < b.max_new ? c.page : b.max_new;
  const bool fp8 = c.dtype == SPARKATTN_FP8_E4M3;
  auto go = [&](auto normed) {
    constexpr bool NORM = decltype(normed)::value;
    if (c.d == 128) return fp8 ? launch_rows<128, true, NORM>(p, rows, stream) : launch_rows<128, false, NORM>(p, rows, stream);
    return fp8 ? launch_rows<64, true, NORM>(p, rows, stream) : launch_rows<64, false, NORM>(p, rows, stream);
  };
  return norm ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace sparkattn
