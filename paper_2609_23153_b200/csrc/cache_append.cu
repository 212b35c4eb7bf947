// sparkattn_cache_append: new keys and values into a paged cache (bf16, or E4M3 with a scale per page and head), keys and
// queries rotated by their positions on the way.
//
// The rotation is a 2 x 2 product per channel pair; the quantisation of a page needs the largest |x| of its new tokens
// before the first code, so a page's tokens of one head stay in registers between the two: HBM sees every row once.
// A unit is the new tokens of one (sequence, page, head) of K or of V; 2 threads per token row (at least a warp) hold it.
// The queries, which nothing is reduced over, go row by row: a thread keeps its channels' phases for all heads of a token.
#include <cuda_fp8.h>

#include "cache.h"

namespace sparkattn {

constexpr int kAppendThreads = 256;

struct RowsView {
  __nv_bfloat16* data;
  int64_t stride_t, stride_h;
};
struct RotaryView {
  const float* cos;
  const float* sin;
  const int32_t* positions;
  const int32_t* axis;
  int rot, interleaved, rows, axes;
};
struct AppendParams {
  BatchView batch;
  RotaryView rotary;             // rot = 0: nothing is rotated
  RowsView q, k, v, q_out;       // q.data NULL: no queries
  unsigned char* k_cache;
  unsigned char* v_cache;
  float* k_scale;
  float* v_scale;
  int64_t stride_page, stride_h, stride_n;
  int H, Hk;
  int pages_each;                // pages of a sequence that max_new tokens can reach
  long long units;
  int unit_ctas;                 // CTAs 1 .. unit_ctas work on units, those behind them on query rows
  int q_tokens;                  // tokens per query CTA
  int32_t* status;
};

// eight fp32 channels
struct Chunk {
  float x[8];
};
__device__ __forceinline__ Chunk widen(uint4 v) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
  Chunk c;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = __bfloat1622float2(p[j]);
    c.x[2 * j] = f.x;
    c.x[2 * j + 1] = f.y;
  }
  return c;
}
__device__ __forceinline__ uint4 narrow(const Chunk& c) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(c.x[2 * j], c.x[2 * j + 1]);
    w[j] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The phases of the channels 8c .. 8c+7 of a token.  Interleaved: cosines and sines of its four pairs.  Halves: of
// the eight pairs of which the chunk holds one side.
struct Phases {
  float c[8], s[8];
  bool on;
};
__device__ __forceinline__ Phases phases_of(const RotaryView& r, int t, int pos, int chunk) {
  Phases p;
  p.on = chunk * 8 < r.rot;
  if (!p.on) return p;
  const int pairs = r.rot / 2;
  const int n = r.interleaved ? 4 : 8;
  const int m0 = r.interleaved ? chunk * 4 : (chunk * 8) % pairs;
  if (r.axis == nullptr) {
    const int at = r.positions ? r.positions[(int64_t)t * r.axes] : pos;
    p.on = (uint32_t)at < (uint32_t)r.rows;
    if (!p.on) return p;
    const float4* c = reinterpret_cast<const float4*>(r.cos + (int64_t)at * pairs + m0);
    const float4* s = reinterpret_cast<const float4*>(r.sin + (int64_t)at * pairs + m0);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (4 * j < n) {
        const float4 a = c[j], b = s[j];
        p.c[4 * j] = a.x; p.c[4 * j + 1] = a.y; p.c[4 * j + 2] = a.z; p.c[4 * j + 3] = a.w;
        p.s[4 * j] = b.x; p.s[4 * j + 1] = b.y; p.s[4 * j + 2] = b.z; p.s[4 * j + 3] = b.w;
      }
    return p;
  }
  // a pair whose position lies outside the table is left as it is: turned by nothing
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    p.c[j] = 1.0f;
    p.s[j] = 0.0f;
    if (j < n) {
      const int ax = r.axis[m0 + j];
      const int at = (uint32_t)ax >= (uint32_t)r.axes ? -1 : r.positions ? r.positions[(int64_t)t * r.axes + ax] : pos;
      if ((uint32_t)at < (uint32_t)r.rows) {
        p.c[j] = r.cos[(int64_t)at * pairs + m0 + j];
        p.s[j] = r.sin[(int64_t)at * pairs + m0 + j];
      }
    }
  }
  return p;
}
// The chunk turned, given the raw chunk that holds the other side of its pairs (halves; its own where interleaved).  Each product
// and sum is rounded by itself, so that a cache filled by any route holds the same bits.
__device__ __forceinline__ Chunk turn(const RotaryView& r, const Phases& p, int chunk, const Chunk& x, const Chunk& other) {
  Chunk y = x;
  if (!p.on) return y;
  if (r.interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = x.x[2 * j], b = x.x[2 * j + 1];
      y.x[2 * j] = __fsub_rn(__fmul_rn(a, p.c[j]), __fmul_rn(b, p.s[j]));
      y.x[2 * j + 1] = __fadd_rn(__fmul_rn(a, p.s[j]), __fmul_rn(b, p.c[j]));
    }
  } else if (chunk * 8 < r.rot / 2) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y.x[j] = __fsub_rn(__fmul_rn(x.x[j], p.c[j]), __fmul_rn(other.x[j], p.s[j]));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) y.x[j] = __fadd_rn(__fmul_rn(other.x[j], p.s[j]), __fmul_rn(x.x[j], p.c[j]));
  }
  return y;
}
// the lanes of a row hold its chunks in order: the lane with the other side of this lane's pairs
template <int D>
__device__ __forceinline__ uint4 other_side(const RotaryView& r, int chunk, uint4 v) {
  const int half = r.rot / 16;                             // chunks per side
  const int partner = chunk < half ? chunk + half : chunk < 2 * half ? chunk - half : chunk;
  const int src = (threadIdx.x & 31 & ~(D / 8 - 1)) + partner;
  v.x = __shfl_sync(0xffffffffu, v.x, src);
  v.y = __shfl_sync(0xffffffffu, v.y, src);
  v.z = __shfl_sync(0xffffffffu, v.z, src);
  v.w = __shfl_sync(0xffffffffu, v.w, src);
  return v;
}

__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
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

// U threads hold the up to ROWS new rows of a unit, 16 bytes of a row each at a time.
template <int D, bool FP8, int ROWS>
__device__ __forceinline__ void append_units(const AppendParams& p, uint32_t* s_max) {
  constexpr int kLanes = D / 8;                                    // threads of a row
  constexpr int U = ROWS * 2 < 32 ? 32 : ROWS * 2;
  constexpr int kRowsAtOnce = U / kLanes;
  constexpr int C = (ROWS + kRowsAtOnce - 1) / kRowsAtOnce;
  constexpr int kElt = FP8 ? 1 : 2;
  const int group = threadIdx.x / U, tid = threadIdx.x % U;
  const long long unit = (long long)(blockIdx.x - 1) * (kAppendThreads / U) + group;
  const int chunk = tid % kLanes, row0 = tid / kLanes;
  const bool is_v = unit & 1;
  const long long rest = unit >> 1;
  const int h = (int)(rest % p.Hk);
  const int bj = (int)(rest / p.Hk);
  const int b = bj / p.pages_each;
  const int P = 1 << p.batch.page_shift;
  int rows = 0, held = 0, pos0 = 0, t0 = 0, page = -1;
  if (unit < p.units) {
    const Sequence s = sequence_of(p.batch, b);
    const int first = max(s.first_pos(), 0);
    const int number = (first >> p.batch.page_shift) + bj % p.pages_each;
    pos0 = max(number << p.batch.page_shift, first);
    rows = min((number + 1) << p.batch.page_shift, s.len) - pos0;
    if (rows > 0 && number < p.batch.max_pages) {
      held = pos0 & (P - 1);
      t0 = s.start + pos0 - s.first_pos();
      page = p.batch.page_table[(int64_t)b * p.batch.max_pages + number];
    }
    if ((uint32_t)page >= (uint32_t)p.batch.pages) rows = 0;
  }
  const RowsView& from = is_v ? p.v : p.k;
  const __nv_bfloat16* src = from.data + h * from.stride_h + chunk * 8;
  unsigned char* dst = (is_v ? p.v_cache : p.k_cache) + ((int64_t)page * p.stride_page + h * p.stride_h + chunk * 8) * kElt;
  uint4 raw[C];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int r = row0 + i * kRowsAtOnce;
    raw[i] = r < rows ? *reinterpret_cast<const uint4*>(src + (int64_t)(t0 + r) * from.stride_t) : make_uint4(0u, 0u, 0u, 0u);
  }
  float* scale_at = FP8 && rows > 0 ? (is_v ? p.v_scale : p.k_scale) + (int64_t)page * p.Hk + h : nullptr;
  const float old = FP8 && rows > 0 && held > 0 ? *scale_at : 0.0f;
  const bool rotate = !is_v && p.rotary.rot > 0;
  Chunk x[C];
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int r = row0 + i * kRowsAtOnce;
    x[i] = widen(raw[i]);
    if (__any_sync(0xffffffffu, rotate)) {
      const uint4 far = other_side<D>(p.rotary, chunk, raw[i]);
      if (rotate && r < rows) x[i] = turn(p.rotary, phases_of(p.rotary, t0 + r, pos0 + r, chunk), chunk, x[i], widen(far));
    }
    if constexpr (FP8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = max(amax, finite_bits(x[i].x[j]));
    }
  }
  if constexpr (!FP8) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int r = row0 + i * kRowsAtOnce;
      if (r < rows) *reinterpret_cast<uint4*>(dst + (int64_t)(held + r) * p.stride_n * kElt) = narrow(x[i]);
    }
  } else {
    amax = __reduce_max_sync(0xffffffffu, amax);
    if constexpr (U > 32) {
      if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = amax;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < U / 32; ++w) amax = max(amax, s_max[group * (U / 32) + w]);
    }
    float scale = power_scale(amax);
    if (held > 0 && old >= scale) scale = old;
    const float inv = 1.0f / scale;
    if (rows > 0 && held > 0 && scale > old) {
      const float again = __fmul_rn(old, inv);
      for (int r = row0; r < held; r += kRowsAtOnce) {
        uint2* at = reinterpret_cast<uint2*>(dst + (int64_t)r * p.stride_n);
        *at = encode(decode(*at), again);
      }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int r = row0 + i * kRowsAtOnce;
      if (r < rows) *reinterpret_cast<uint2*>(dst + (int64_t)(held + r) * p.stride_n) = encode(x[i], inv);
    }
    // (every thread of a larger unit has read the old scale: the barrier above is behind that read)
    __syncwarp();
    if (rows > 0 && tid == 0) *scale_at = scale;
  }
}

template <int D>
__device__ __forceinline__ void rotate_queries(const AppendParams& p) {
  constexpr int kLanes = D / 8, kHeadsAtOnce = kAppendThreads / kLanes, kAhead = 4;
  const int chunk = threadIdx.x % kLanes, h0 = threadIdx.x / kLanes;
  const int first = (blockIdx.x - 1 - p.unit_ctas) * p.q_tokens;
  for (int t = first; t < min(first + p.q_tokens, p.batch.T); ++t) {
    // the token's sequence, for its position there
    int pos = 0;
    bool owned = true;
    if (p.rotary.positions == nullptr) {
      int b = 0;
      if (p.batch.q_start == nullptr) {
        b = t / (p.batch.T / p.batch.B);
      } else {
        int hi = p.batch.B;                               // the last sequence that starts at or before t
        while (hi - b > 1) {
          const int mid = (b + hi) >> 1;
          if (p.batch.q_start[mid] <= t) b = mid; else hi = mid;
        }
      }
      const Sequence s = sequence_of(p.batch, b);
      owned = t >= s.start && t < s.start + s.n;
      pos = s.first_pos() + t - s.start;
    }
    Phases ph = phases_of(p.rotary, t, pos, chunk);
    if (!owned) ph.on = false;
    const __nv_bfloat16* src = p.q.data + (int64_t)t * p.q.stride_t + chunk * 8;
    __nv_bfloat16* dst = p.q_out.data + (int64_t)t * p.q_out.stride_t + chunk * 8;
    for (int base = 0; base < p.H; base += kHeadsAtOnce * kAhead) {
      uint4 raw[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = base + h0 + i * kHeadsAtOnce;
        if (h < p.H) raw[i] = *reinterpret_cast<const uint4*>(src + h * p.q.stride_h);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = base + h0 + i * kHeadsAtOnce;
        if (base + i * kHeadsAtOnce >= p.H) break;
        if (h >= p.H) raw[i] = make_uint4(0u, 0u, 0u, 0u);
        const Chunk far = widen(other_side<D>(p.rotary, chunk, raw[i]));
        const uint4 y = narrow(turn(p.rotary, ph, chunk, widen(raw[i]), far));
        if (h < p.H) *reinterpret_cast<uint4*>(dst + h * p.q_out.stride_h) = y;
      }
    }
  }
}

template <int D, bool FP8, int ROWS>
__global__ void __launch_bounds__(kAppendThreads)
cache_append_kernel(const __grid_constant__ AppendParams p) {
  __shared__ uint32_t s_max[kAppendThreads / 32];
  __shared__ int s_bad[2];
  pdl_wait();
  if (blockIdx.x == 0) {
    const int shift = p.batch.page_shift;
    check_batch(p.batch, s_bad, [&](const Sequence& s) { return make_int2(max(s.first_pos(), 0) >> shift, s.n == 0 ? 0 : (s.len + (1 << shift) - 1) >> shift); });
    if (p.rotary.rot > 0) {
      const RotaryView& r = p.rotary;
      auto bad = [&](int detail) { if (atomicExch(s_bad, 1) == 0) s_bad[1] = detail; };
      if (r.positions) {
        for (long long i = threadIdx.x; i < (long long)p.batch.T * r.axes; i += kAppendThreads)
          if ((uint32_t)r.positions[i] >= (uint32_t)r.rows) bad(r.positions[i]);
      } else {
        for (int b = threadIdx.x; b < p.batch.B; b += kAppendThreads) {
          const Sequence s = sequence_of(p.batch, b);
          if (s.n > 0 && s.len > r.rows) bad(s.len - 1);
        }
      }
      if (r.axis)
        for (int m = threadIdx.x; m < r.rot / 2; m += kAppendThreads)
          if ((uint32_t)r.axis[m] >= (uint32_t)r.axes) bad(r.axis[m]);
    }
    leave_status(p.status, s_bad);
  } else if ((int)blockIdx.x <= p.unit_ctas) {
    append_units<D, FP8, ROWS>(p, s_max);
  } else {
    rotate_queries<D>(p);
  }
}

template <int D, bool FP8>
static int launch_rows(const AppendParams& p, int rows, cudaStream_t stream) {
  auto go = [&](auto kern, int unit_threads) {
    AppendParams q = p;
    const int per = kAppendThreads / unit_threads;
    const long long ctas = (p.units + per - 1) / per, q_ctas = p.q.data ? ((long long)p.batch.T + p.q_tokens - 1) / p.q_tokens : 0;
    if (1 + ctas + q_ctas > 0x7fffffffLL) return (int)SPARKATTN_E_UNSUPPORTED_SHAPE;
    q.unit_ctas = (int)ctas;
    return launch_kernel(kern, dim3((unsigned)(1 + ctas + q_ctas)), kAppendThreads, 0, true, stream, q);
  };
  if (rows <= 4) return go(cache_append_kernel<D, FP8, 4>, 32);
  if (rows <= 16) return go(cache_append_kernel<D, FP8, 16>, 32);
  if (rows <= 32) return go(cache_append_kernel<D, FP8, 32>, 64);
  if (rows <= 64) return go(cache_append_kernel<D, FP8, 64>, 128);
  return go(cache_append_kernel<D, FP8, 128>, 256);
}

int launch_cache_append(const sparkattn_cache_t& c, const sparkattn_batch_t& b, const sparkattn_rotary_t* rotary, const sparkattn_rows_t* q,
                        int H, const sparkattn_rows_t& k, const sparkattn_rows_t& v, void* k_cache, void* v_cache, float* k_scale,
                        float* v_scale, const sparkattn_rows_t* q_out, void* workspace, cudaStream_t stream) {
  AppendParams p{};
  p.batch = make_batch_view(c, b);
  if (rotary) p.rotary = {rotary->cos, rotary->sin, rotary->positions, rotary->axis, rotary->rot, rotary->interleaved, rotary->rows, rotary->axes};
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
  p.units = 2LL * b.B * p.pages_each * c.H;
  p.q_tokens = 1;
  p.status = static_cast<int32_t*>(workspace);
  const int rows = c.page < b.max_new ? c.page : b.max_new;
  const bool fp8 = c.dtype == SPARKATTN_FP8_E4M3;
  if (c.d == 128) return fp8 ? launch_rows<128, true>(p, rows, stream) : launch_rows<128, false>(p, rows, stream);
  return fp8 ? launch_rows<64, true>(p, rows, stream) : launch_rows<64, false>(p, rows, stream);
}

}  // namespace sparkattn
