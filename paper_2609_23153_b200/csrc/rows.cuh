// Rows of bf16 channels, eight to a thread, as the calls that normalise and rotate queries and keys take them: the norm of a row and the
// rotation of its channel pairs.  D / 8 neighbouring lanes of a warp hold a row.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"
#include "launch.h"

namespace sparkattn {

struct RotaryView {
  const float* cos;
  const float* sin;
  const int32_t* positions;
  const int32_t* axis;
  int rot, interleaved, rows, axes;
};
inline RotaryView make_rotary_view(const sparkattn_rotary_t* r) {
  return r ? RotaryView{r->cos, r->sin, r->positions, r->axis, r->rot, r->interleaved, r->rows, r->axes} : RotaryView{};
}
// Weights of the norms: [D], or [heads, D] where stride is D; NULL: ones
struct NormView {
  const void* q_weight;
  const void* k_weight;
  int stride, bf16;
  float eps;
};
inline NormView make_norm_view(const sparkattn_norm_t* n, int d) {
  return n ? NormView{n->q_weight, n->k_weight, n->per_head ? d : 0, n->weight_dtype == SPARKATTN_BF16, n->eps} : NormView{};
}

// eight fp32 channels
struct Chunk {
  float x[8];
};
__device__ __forceinline__ Chunk widen(uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  Chunk c;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    c.x[2 * j] = __uint_as_float(w[j] << 16);
    c.x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
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

// the weights of eight channels of a head
__device__ __forceinline__ Chunk norm_weights(const NormView& n, const void* weight, int head, int channel) {
  Chunk w;
  const int at = head * n.stride + channel;
  if (weight == nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w.x[j] = 1.0f;
  } else if (n.bf16) {
    w = widen(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(weight) + at));
  } else {
    const float4* from = reinterpret_cast<const float4*>(static_cast<const float*>(weight) + at);
    const float4 a = from[0], b = from[1];
    w = {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
  }
  return w;
}
// x / sqrt(mean x^2 + eps) * weight of a row whose chunks the D / 8 lanes hold.  Squares, their sum and the products are fp32; the order of the sum
// is that of the channels, then of the lanes, those D / 16 apart first, so a row has the same bits whatever call it goes through.  In pairs of
// channels: with scalar instructions (and the rotation's products rounded one by one) 40 + 40 heads of 75,600 tokens took 541 us instead of 514.
__device__ __forceinline__ float sum_of_squares(const Chunk& x) {
  uint64_t sum2 = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint64_t pair = pack_f32x2(x.x[2 * j], x.x[2 * j + 1]);
    sum2 = j == 0 ? fmul2(pair, pair) : ffma2(pair, pair, sum2);
  }
  const float2 two = unpack_f32x2(sum2);
  return two.x + two.y;
}
template <int D>
__device__ __forceinline__ float norm_factor(float row_sum, float eps) {
  float by;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(by) : "f"(__fmaf_rn(row_sum, 1.0f / D, eps)));      // (eps is a normal number)
  return by;
}
__device__ __forceinline__ Chunk scaled(const Chunk& x, const Chunk& weight, float by) {
  const uint64_t by2 = pack_f32x2(by, by);
  Chunk r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 y = unpack_f32x2(fmul2(pack_f32x2(x.x[2 * j], x.x[2 * j + 1]), fmul2(pack_f32x2(weight.x[2 * j], weight.x[2 * j + 1]), by2)));
    r.x[2 * j] = y.x;
    r.x[2 * j + 1] = y.y;
  }
  return r;
}
template <int D>
__device__ __forceinline__ Chunk normed(const Chunk& x, const Chunk& weight, float eps) {
  float sum = sum_of_squares(x);
#pragma unroll
  for (int o = D / 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return scaled(x, weight, norm_factor<D>(sum, eps));
}
// The sums of four rows' chunks into the rows' factors: the lanes share the rows out, a quarter of them a row, and pass the factors round.  (Ten
// instructions a row become six.)
template <int D>
__device__ __forceinline__ void norm_factors(float (&x)[4], float eps) {
  constexpr int L = D / 8;
  const int lane = threadIdx.x & 31;
  const bool high = lane & (L / 2), odd = lane & (L / 4);
  float a = high ? x[2] : x[0], b = high ? x[3] : x[1];
  a += __shfl_xor_sync(0xffffffffu, high ? x[0] : x[2], L / 2);
  b += __shfl_xor_sync(0xffffffffu, high ? x[1] : x[3], L / 2);
  float mine = odd ? b : a;
  mine += __shfl_xor_sync(0xffffffffu, odd ? a : b, L / 4);
#pragma unroll
  for (int o = L / 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  mine = norm_factor<D>(mine, eps);
#pragma unroll
  for (int u = 0; u < 4; ++u) x[u] = __shfl_sync(0xffffffffu, mine, (lane & ~(L - 1)) + (u & 2 ? L / 2 : 0) + (u & 1 ? L / 4 : 0));
}
// The rotation behind a norm: a product rounded, the other one and the sum in one step.  Interleaved: the chunk's four pairs by c, s.
__device__ __forceinline__ Chunk turn_pairs_fused(const float (&c)[4], const float (&s)[4], const Chunk& x) {
  Chunk r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    r.x[2 * j] = __fmaf_rn(x.x[2 * j], c[j], -__fmul_rn(x.x[2 * j + 1], s[j]));
    r.x[2 * j + 1] = __fmaf_rn(x.x[2 * j], s[j], __fmul_rn(x.x[2 * j + 1], c[j]));
  }
  return r;
}
// Halves: far holds the other sides, s is negative on the first side
__device__ __forceinline__ Chunk turn_halves_fused(const float (&c)[8], const float (&s)[8], const Chunk& x, const Chunk& far) {
  Chunk r;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const uint64_t other = fmul2(pack_f32x2(far.x[j], far.x[j + 1]), pack_f32x2(s[j], s[j + 1]));
    const float2 y = unpack_f32x2(ffma2(pack_f32x2(x.x[j], x.x[j + 1]), pack_f32x2(c[j], c[j + 1]), other));
    r.x[j] = y.x;
    r.x[j + 1] = y.y;
  }
  return r;
}

// The chunk turned by its share c, s of a row of them.  Interleaved: its own four pairs.  Halves: `y` holds the other sides of its
// eight channels.  Each product and sum is rounded by itself, so that a cache filled by any route holds the same bits.  (Scalar
// instructions: the packed ones want their pairs in neighbouring registers and spend more on moves than they save, and a packed sum
// behind packed products was fused with one of them, which rounds once.)
__device__ __forceinline__ Chunk turn_pairs(const float* c, const float* s, const Chunk& x) {
  const float4 cc = *reinterpret_cast<const float4*>(c), ss = *reinterpret_cast<const float4*>(s);
  const float cv[4] = {cc.x, cc.y, cc.z, cc.w}, sv[4] = {ss.x, ss.y, ss.z, ss.w};
  Chunk r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    r.x[2 * j] = __fsub_rn(__fmul_rn(x.x[2 * j], cv[j]), __fmul_rn(x.x[2 * j + 1], sv[j]));
    r.x[2 * j + 1] = __fadd_rn(__fmul_rn(x.x[2 * j], sv[j]), __fmul_rn(x.x[2 * j + 1], cv[j]));
  }
  return r;
}
__device__ __forceinline__ Chunk turn_halves(const float* c, const float* s, const Chunk& x, const Chunk& y, float sign) {
  Chunk r;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float4 cc = reinterpret_cast<const float4*>(c)[g], ss = reinterpret_cast<const float4*>(s)[g];
    const float cv[4] = {cc.x, cc.y, cc.z, cc.w}, sv[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)      // a first side takes away what a second side adds: x c - y s and x c + y s round alike
      r.x[4 * g + j] = __fadd_rn(__fmul_rn(x.x[4 * g + j], cv[j]), __fmul_rn(y.x[4 * g + j], __fmul_rn(sv[j], sign)));
  }
  return r;
}

// the chunk that another lane holds
__device__ __forceinline__ Chunk chunk_of(const Chunk& x, int lane) {
  Chunk r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r.x[j] = __shfl_sync(0xffffffffu, x.x[j], lane);
  return r;
}

}  // namespace sparkattn
