// sparkattn_norm_rotate: RMS norm of each head's queries and keys and their rotation, whole sequences at a time.
//
// y = R(x / sqrt(mean x^2 + eps) * w), row by row; nothing is used twice but the tokens' cosines and sines, which all heads share, and the
// weights, which all tokens share.  So a thread stays with 16 bytes of one token's rows: its pairs' phases and (per tensor) its weights are in
// registers once, and it goes through the heads, four rows asked for at a time.  The sum of squares goes through the D / 8 lanes of a row.
// A CTA is 256 threads: 16 tokens (32 of 64 channels) by a run of the (sample, head) lines of both tensors.
// Bandwidth bounds it, and instructions are near: 40 + 40 heads of 75,600 tokens, 128 channels, 3.10 GB in 497 us = 6.2 TB/s, 0.95 of a copy's rate,
// called for seconds, under the power limit, 530-550; halves, whose other sides go through the lanes, 585-600 and 615-630.  Five CTAs an SM (48 registers)
// take 499, but 540-565 for seconds, and halves spill (711).  Halves as eight bytes of either side a thread: 650.  With scalar instructions and the
// rotation's products rounded one by one 541 us, the SMs issuing in 0.78 of the clocks.  Small calls are latency: phases, then rows; 8 heads
// of two samples of 1201 tokens, 64 channels, 3.5 us.
#include <algorithm>
#include <type_traits>

#include "rows.cuh"
#include "tmap.h"

namespace sparkattn {

constexpr int kNormThreads = 256;

struct HeadRowsView {
  const __nv_bfloat16* in;
  __nv_bfloat16* out;
  int64_t in_b, in_h, in_n, out_b, out_h, out_n;      // strides
  const void* weight;
  int H, lines;                                       // heads; samples * heads
  FastDiv by_H;
};
struct NormRotateParams {
  HeadRowsView x[2];             // queries, keys (lines 0: none)
  RotaryView rotary;             // rot = 0: nothing is rotated
  NormView norm;
  int N;
  int tiles, each;               // tiles of tokens; lines of a CTA
  FastDiv by_tiles;
  int32_t* status;
};

// Whether a pair of token n is turned by an angle of the tables.  (A pair that is not stays as it is and is reported.)
__device__ __forceinline__ uint32_t angle_row(const RotaryView& r, int n, int m) {
  uint32_t axis = 0;
  if (r.axis != nullptr) {
    axis = (uint32_t)r.axis[m];
    if (axis >= (uint32_t)r.axes) return 0xffffffffu;
  }
  return r.positions != nullptr ? (uint32_t)r.positions[(int64_t)n * r.axes + axis] : (uint32_t)n;
}

// U: rows that a thread asks for at a time
template <int D, bool INTERLEAVED, bool NORM, int U>
__global__ void __launch_bounds__(kNormThreads, 4)
norm_rotate_kernel(const __grid_constant__ NormRotateParams p) {
  constexpr int kLanes = D / 8, kRows = kNormThreads / kLanes, kPairs = INTERLEAVED ? 4 : 8;
  const RotaryView& r = p.rotary;
  const int group = fast_div((int)blockIdx.x, p.by_tiles), tile = (int)blockIdx.x - group * p.tiles;
  const int chunk = threadIdx.x % kLanes, n = tile * kRows + threadIdx.x / kLanes;
  const bool there = n < p.N, on = chunk * 8 < r.rot;
  const int half = r.rot / 16;                                    // halves: chunks of a side
  const bool second = chunk >= half;
  const int m0 = INTERLEAVED ? chunk * 4 : (second ? chunk - half : chunk) * 8;
  const int partner = (threadIdx.x & 31 & ~(kLanes - 1)) + (!on ? chunk : second ? chunk - half : chunk + half);
  pdl_wait();
  bool code_there = false;
  if (blockIdx.x == 0 && threadIdx.x == 0) code_there = take_header(p.status);
  float c[kPairs], s[kPairs];
  int bad = 0;
  bool any_bad = false;
#pragma unroll
  for (int j = 0; j < kPairs; ++j) {
    c[j] = 1.0f;
    s[j] = 0.0f;
  }
  if (there && on) {
    if (r.axis == nullptr) {
      // one row of the tables, four pairs at a time
      const uint32_t e = r.positions != nullptr ? (uint32_t)r.positions[(int64_t)n * r.axes] : (uint32_t)n;
      if (e < (uint32_t)r.rows) {
#pragma unroll
        for (int j = 0; j < kPairs; j += 4) {
          const float4 cc = *reinterpret_cast<const float4*>(r.cos + (e * (r.rot / 2) + m0 + j));
          const float4 ss = *reinterpret_cast<const float4*>(r.sin + (e * (r.rot / 2) + m0 + j));
          c[j] = cc.x; c[j + 1] = cc.y; c[j + 2] = cc.z; c[j + 3] = cc.w;
          s[j] = ss.x; s[j + 1] = ss.y; s[j + 2] = ss.z; s[j + 3] = ss.w;
        }
      } else {
        any_bad = true;
        bad = (int)e;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const uint32_t e = angle_row(r, n, m0 + j);
        if (e < (uint32_t)r.rows) {
          c[j] = r.cos[e * (r.rot / 2) + m0 + j];
          s[j] = r.sin[e * (r.rot / 2) + m0 + j];
        } else {
          any_bad = true;
          bad = (int)e;
        }
      }
    }
  }
  if (!INTERLEAVED && !second) {
#pragma unroll
    for (int j = 0; j < kPairs; ++j) s[j] = -s[j];                // a first side takes away what a second side adds
  }
  auto turned = [&](const Chunk& x) {
    Chunk y{};
    if constexpr (NORM && INTERLEAVED) {
      y = turn_pairs_fused(c, s, x);
    } else if constexpr (NORM) {
      y = turn_halves_fused(c, s, x, chunk_of(x, partner));
    } else if constexpr (INTERLEAVED) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y.x[2 * j] = __fsub_rn(__fmul_rn(x.x[2 * j], c[j]), __fmul_rn(x.x[2 * j + 1], s[j]));
        y.x[2 * j + 1] = __fadd_rn(__fmul_rn(x.x[2 * j], s[j]), __fmul_rn(x.x[2 * j + 1], c[j]));
      }
    } else {
      const Chunk far = chunk_of(x, partner);
#pragma unroll
      for (int j = 0; j < 8; ++j) y.x[j] = __fadd_rn(__fmul_rn(x.x[j], c[j]), __fmul_rn(far.x[j], s[j]));
    }
    return y;
  };
  const int from = group * p.each, to = from + p.each;
#pragma unroll 1
  for (int t = 0, base = 0; t < 2; base += p.x[t].lines, ++t) {
    const HeadRowsView& v = p.x[t];
    const int first = max(from - base, 0), last = min(to - base, v.lines);
    if (first >= last) continue;
    Chunk weight;
    if constexpr (NORM) {
      if (p.norm.stride == 0) weight = norm_weights(p.norm, v.weight, 0, chunk * 8);
    }
    const __nv_bfloat16* in = v.in + (int64_t)n * v.in_n + chunk * 8;
    __nv_bfloat16* out = v.out + (int64_t)n * v.out_n + chunk * 8;
#pragma unroll 1
    for (int l0 = first; l0 < last; l0 += U) {
      uint4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int l = l0 + u, b = fast_div(l, v.by_H), h = l - b * v.H;
        raw[u] = l < last && there ? *reinterpret_cast<const uint4*>(in + (b * v.in_b + h * v.in_h)) : make_uint4(0u, 0u, 0u, 0u);
      }
      [[maybe_unused]] float by[U];
      constexpr bool kTogether = NORM && INTERLEAVED && U == 4;      // (halves have the registers' room taken up by the other sides' phases)
      if constexpr (kTogether) {
#pragma unroll
        for (int u = 0; u < U; ++u) by[u] = sum_of_squares(widen(raw[u]));
        norm_factors<D>(by, p.norm.eps);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int l = l0 + u, b = fast_div(l, v.by_H), h = l - b * v.H;
        Chunk x = widen(raw[u]);
        if constexpr (NORM) {
          if (p.norm.stride != 0 && l < last) weight = norm_weights(p.norm, v.weight, h, chunk * 8);
          if constexpr (kTogether) x = scaled(x, weight, by[u]);
          else x = normed<D>(x, weight, p.norm.eps);
        }
        if (r.rot > 0) {
          const Chunk y = turned(x);
          if (on) x = y;
        }
        if (l < last && there) *reinterpret_cast<uint4*>(out + (b * v.out_b + h * v.out_h)) = narrow(x);
      }
    }
  }
  if (r.rot == 0) return;
  if (group == 0 && any_bad) report_early(p.status, SPARKATTN_E_BAD_INDEX, bad);
  if (blockIdx.x == 0 && __syncthreads_or(code_there)) {
    // the word held a code, which may have been one of this call's: see take_header
    any_bad = false;
    // one pass for each axis that some pair turns by (for every run of pairs of one axis: 75,600 tokens, three axes in turns, 1.1 ms)
    uint32_t axes = r.axis == nullptr ? 1u : 0u;
    if (r.axis != nullptr) {
#pragma unroll 1
      for (int m = 0; m < r.rot / 2; ++m) {
        const uint32_t axis = (uint32_t)r.axis[m];
        if (axis < (uint32_t)r.axes) {
          axes |= 1u << axis;
        } else {
          any_bad = true;
          bad = -1;
        }
      }
    }
#pragma unroll 1
    for (; axes != 0; axes &= axes - 1) {
      const int axis = __ffs(axes) - 1;
#pragma unroll 4
      for (int row = threadIdx.x; row < p.N; row += kNormThreads) {
        const uint32_t e = r.positions != nullptr ? (uint32_t)r.positions[(int64_t)row * r.axes + axis] : (uint32_t)row;
        if (e >= (uint32_t)r.rows) {
          any_bad = true;
          bad = (int)e;
        }
      }
    }
    if (any_bad) report_early(p.status, SPARKATTN_E_BAD_INDEX, bad);
  }
}

int launch_norm_rotate(const HeadRows& q, const HeadRows* k, const sparkattn_norm_t* norm, const sparkattn_rotary_t* rotary, void* workspace,
                       cudaStream_t stream) {
  NormRotateParams p{};
  auto view = [](const HeadRows& x, const void* weight) {
    const sparkattn_shape_t &i = *x.in_shape, &o = *x.out_shape;
    return HeadRowsView{static_cast<const __nv_bfloat16*>(x.in), static_cast<__nv_bfloat16*>(x.out), i.stride_b, i.stride_h, i.stride_n, o.stride_b,
                        o.stride_h, o.stride_n, weight, i.H, i.B * i.H, make_fast_div(i.H)};
  };
  const sparkattn_shape_t& s = *q.in_shape;
  p.rotary = make_rotary_view(rotary);
  p.norm = make_norm_view(norm, s.d);
  p.x[0] = view(q, p.norm.q_weight);
  if (k) p.x[1] = view(*k, p.norm.k_weight);
  p.N = s.N;
  p.status = static_cast<int32_t*>(workspace);
  const int rows = kNormThreads / (s.d / 8), sms = current_sm_count();
  if (sms < 1) return SPARKATTN_E_CUDA;
  p.tiles = (s.N + rows - 1) / rows;
  p.by_tiles = make_fast_div(p.tiles);
  // Four rows at a time where that gives every place on the SMs a CTA (40 + 40 heads of 75,600 tokens: 504 us by four, 564 by two), else two, so that more CTAs share the work (8 heads of 1201 tokens of 64 channels: 3.5 us by two, 4.1 by four).
  const long long lines = (long long)p.x[0].lines + p.x[1].lines;
  const int u = (lines + 3) / 4 * p.tiles >= 4LL * sms ? 4 : 2;
  // runs of lines: three CTAs for every place, whole batches of rows (56 + 8 heads of four samples of 715 tokens by four lines a CTA 22.5 us, by five 29.5)
  long long groups = std::min<long long>((12LL * sms + p.tiles - 1) / p.tiles, (lines + u - 1) / u);
  p.each = (int)((lines + groups - 1) / groups + u - 1) / u * u;
  groups = (lines + p.each - 1) / p.each;
  if (groups * p.tiles > 0x7fffff00LL) return SPARKATTN_E_UNSUPPORTED_SHAPE;
  auto go = [&](auto d, auto inter, auto normed) {
    constexpr int D = decltype(d)::value;
    constexpr bool I = decltype(inter)::value, N = decltype(normed)::value;
    return launch_kernel(u == 4 ? norm_rotate_kernel<D, I, N, 4> : norm_rotate_kernel<D, I, N, 2>, dim3((unsigned)(groups * p.tiles)), kNormThreads, 0, true,
                         stream, p);
  };
  auto with = [&](auto d) {
    using std::true_type, std::false_type;
    if (p.rotary.interleaved) return norm ? go(d, true_type{}, true_type{}) : go(d, true_type{}, false_type{});
    return norm ? go(d, false_type{}, true_type{}) : go(d, false_type{}, false_type{});
  };
  return s.d == 128 ? with(std::integral_constant<int, 128>{}) : with(std::integral_constant<int, 64>{});
}

}  // namespace sparkattn
