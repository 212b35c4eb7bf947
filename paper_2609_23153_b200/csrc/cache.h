// What the kernels of the paged cache share: the batch as the device sees it, and the keys that a token may attend to.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "launch.h"

namespace sparkattn {

// A sequence of the batch: rows [start, start + n) of the call, `len` tokens in the cache.  Whatever the caller's numbers
// are, the result stays inside the tensors (the first CTA of a call reports what had to be cut).
struct Sequence {
  int start, n, len;
  __device__ __forceinline__ int first_pos() const { return len - n; }
};
struct BatchView {
  const int32_t* page_table;
  const int32_t* kv_len;
  const int32_t* q_start;
  int B, T, max_new, max_pages, page_shift, pages;
};
inline BatchView make_batch_view(const sparkattn_cache_t& c, const sparkattn_batch_t& b) {
  int shift = 4;
  while ((1 << shift) < c.page) ++shift;
  return {b.page_table, b.kv_len, b.q_start, b.B, b.T, b.max_new, b.max_pages, shift, c.pages};
}
__device__ __forceinline__ int token_capacity(const BatchView& v) {
  return (int)min((long long)v.max_pages << v.page_shift, 0x7fffff00LL);
}
__device__ __forceinline__ Sequence sequence_of(const BatchView& v, int b) {
  Sequence s;
  const int len = v.kv_len[b];
  int stop;
  if (v.q_start != nullptr) {
    s.start = v.q_start[b];
    stop = v.q_start[b + 1];
  } else {
    const int each = v.T / v.B;
    s.start = b * each;
    stop = s.start + each;
  }
  s.start = min(max(s.start, 0), v.T);
  s.n = min(min(max(stop, s.start), v.T) - s.start, v.max_new);
  s.len = min(max(len, 0), token_capacity(v));
  return s;
}

// [lo, hi) of the keys that the token at position pos of a sequence of len tokens sees; in kernels with SINK those of its window, in
// front of which it sees the first `sink` keys
struct Causal {
  int frame, window;      // frame 0: every key; window 0: from the first key on
  FastDiv by_frame;
  int sink;               // more than 0 only where there is a window
};
__device__ __forceinline__ int2 visible_keys(const Causal& c, int pos, int len) {
  if (c.frame == 0) return make_int2(0, len);
  if (pos < 0) return make_int2(0, 0);
  const int f = fast_div(pos, c.by_frame);
  const long long hi = ((long long)f + 1) * c.frame;
  const long long lo = c.window == 0 ? 0 : max((long long)(f - c.window + 1) * c.frame, 0LL);
  return make_int2((int)min(lo, (long long)len), (int)min(hi, (long long)len));
}

template <bool SINK>
__device__ __forceinline__ bool sees(const Causal& c, int2 seen, int key) {
  return key < seen.y && (key >= seen.x || (SINK && key < c.sink));
}

// One CTA looks through the numbers a call was given and leaves the status word: nobody else writes it but a wait that has run
// out, seconds later, so that nothing has to be cleared in front.  reach: pages of the sequence that the call reaches, from the
// first to behind the last; SINK: and those of the first `sink` tokens.  (This CTA is what a call of hundreds of short sequences waits for, or one of long tables
// of small pages: with the first tokens' places worked out in calls that have none, a token of each of 4000 sequences of 50 took 161 us instead of 143.)
template <bool SINK, typename Reach>
__device__ __forceinline__ void check_batch(const BatchView& v, int* s_bad /* [2], shared */, Reach reach, int sink = 0) {
  if (threadIdx.x == 0) { s_bad[0] = 0; s_bad[1] = 0; }
  __syncthreads();
  auto bad = [&](int detail) { if (atomicExch(s_bad, 1) == 0) s_bad[1] = detail; };
  for (int b = threadIdx.x; b < v.B; b += blockDim.x) {
    const int len = v.kv_len[b];
    if (len < 0 || len > token_capacity(v)) bad(len);
    if (v.q_start != nullptr) {
      const int lo = v.q_start[b], hi = v.q_start[b + 1];
      if (lo < 0 || hi < lo || hi > v.T || hi - lo > v.max_new || (long long)hi - lo > len) bad(b);
    } else if (v.T / v.B > len) {
      bad(b);
    }
  }
  // eight lanes per sequence, eight pages each at a time
  const int lanes = 8, lane = threadIdx.x & (lanes - 1);
  for (int b = threadIdx.x / lanes; b < v.B; b += blockDim.x / lanes) {
    const Sequence s = sequence_of(v, b);
    const int2 pages = reach(s);
    const int32_t* row = v.page_table + (int64_t)b * v.max_pages;
    const int last = min(pages.y, v.max_pages);
    // (the first tokens' pages stand in front of the others, `gap` pages nearer to them than they are)
    const int front = SINK ? min(((sink - 1) >> v.page_shift) + 1, pages.x) : 0, gap = pages.x - front;
    for (int i = pages.x - front + lane; i < last; i += lanes * 8) {
      int page[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int at = i + lanes * u;
        page[u] = at < last ? row[SINK && at < pages.x ? at - gap : at] : 0;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if ((uint32_t)page[u] >= (uint32_t)v.pages) bad(page[u]);
    }
  }
}
__device__ __forceinline__ void leave_status(int32_t* status, const int* s_bad) {
  __syncthreads();
  if (threadIdx.x == 0)
    *reinterpret_cast<unsigned long long*>(status) =
        s_bad[0] ? (unsigned long long)(uint32_t)s_bad[1] << 32 | (uint32_t)SPARKATTN_E_BAD_INDEX : 0ull;
}

}  // namespace sparkattn
