// The book of a paged cache: who holds which pages.  sparkattn_pages_fork, _reserve, _trim, _compact keep it, sparkattn_cache_copy_pages moves
// what the pages hold.
//
// The book is a few hundred thousand words at most, so what a step costs is launches and chains of loads; a launch takes 2 us.
//   What has to happen in order, counting pages, handing them out, changing the counts once they are at their other place, is the work of one
//   thread-block cluster of up to sixteen CTAs, whose barrier stands between the steps and through whose shared memory the counts go; a chain of
//   launches would take 2 us a step.  Tables that go to another place are copied meanwhile by the grid's other clusters.
//   A fork changes counts for whole rows, by integer additions, in any order: a launch of its own, since sixteen SMs issue their additions to
//   scattered words a few clocks apart (256 rows of 500 entries: 11.2 us with one cluster, 4.6 with two launches).
// Free pages are handed out in ascending order: the same call gives the same book.
// Measured: a fork of 256 sequences of up to 32,000 tokens, pages of 64, 4.6 us; pages for a token of each of 128 sequences 7.2 us, in place 6.3, with the step's
// lengths 7.4, for prompts of 4000 tokens of each of 32, pages of 16, 10.3, for one of 65,536, whose 4096 entries one warp writes, 31; the 90
// copies of pages of 16 tokens that they share 2.7; a trim of 32 sequences 4.7, with nothing to give back 3.1; compact, 1560 pages, 6.4.  Latency
// bounds all of them.  The copy of 368 pages of 196 KB, K and V, 289 MB read and written: 49 us = 5.9 TB/s, 0.89 of a copy's rate.
#include <algorithm>
#include <type_traits>

#include "cache.h"
#include "tmap.h"

namespace sparkattn {

constexpr int kBookThreads = 512, kBookWarps = kBookThreads / 32, kBookClusterMax = 16;

struct BookView {
  const int32_t* table;        // [B, max_pages]
  const int32_t* refs;         // [pages]
  int32_t* table_out;
  int32_t* refs_out;
  int B, max_pages, pages, shift;
};
inline BookView make_book_view(const sparkattn_book_t& b, int32_t* table_out, int32_t* refs_out) {
  int shift = 0;
  while ((1 << shift) < b.page) ++shift;
  return {b.page_table, b.refs, table_out, refs_out, b.B, b.max_pages, b.pages, shift};
}
__device__ __forceinline__ int pages_of(const BookView& v, int tokens) { return (int)(((long long)tokens + (1 << v.shift) - 1) >> v.shift); }
__device__ __forceinline__ bool fits_table(const BookView& v, int tokens) { return tokens >= 0 && tokens <= (long long)v.max_pages << v.shift; }

// What one cluster knows together
struct BookShared {
  int status[kBookClusterMax][2];      // of the first CTA: what every CTA has found
  int bad[2];                          // what this CTA has found: a code, a number
  int count[kBookWarps];               // per warp
  int scan[kBookWarps];
};
__device__ __forceinline__ int cluster_ld_int(const int* at, int rank) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(cluster_map(smem_u32(at), rank)) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_st_int(const int* at, int rank, int v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(cluster_map(smem_u32(at), rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void found(BookShared& s, int code, int detail) {
  if (atomicCAS(&s.bad[0], 0, code) == 0) s.bad[1] = detail;
}
__device__ __forceinline__ void book_barrier() {
  __syncwarp();
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ void book_begin(BookShared& s) {
  if (threadIdx.x == 0) s.bad[0] = s.bad[1] = 0;
  __syncthreads();
}
// The end of the first cluster's work: its first CTA writes the status word, which nobody else does.  (The barriers before this one say
// that the first CTA is there.)
__device__ __forceinline__ void book_end(BookShared& s, int rank, int ranks, int32_t* status) {
  __syncthreads();
  if (threadIdx.x < 2) cluster_st_int(&s.status[rank][threadIdx.x], 0, s.bad[threadIdx.x]);
  book_barrier();
  if (rank == 0 && threadIdx.x == 0) {
    unsigned long long word = 0;
    for (int i = ranks - 1; i >= 0; --i)
      if (s.status[i][0] != 0) word = (unsigned long long)(uint32_t)s.status[i][1] << 32 | (uint32_t)s.status[i][0];
    *reinterpret_cast<unsigned long long*>(status) = word;
  }
}
// The pool in runs of the cluster's warps, so that ranks within it need one exchange of counts and no further barriers.
struct PoolRun {
  int first, last;
};
__device__ __forceinline__ int run_length(int pages, int ranks) {
  const int warps = ranks * kBookWarps;
  return ((pages + warps - 1) / warps + 31) & ~31;
}
__device__ __forceinline__ PoolRun run_of_warp(int pages, int ranks, int rank) {
  const int each = run_length(pages, ranks), w = rank * kBookWarps + (threadIdx.x >> 5);
  const int first = (int)min((long long)w * each, (long long)pages);
  return {first, (int)min((long long)first + each, (long long)pages)};
}
// Counts of the runs, s.count of every CTA (behind a cluster barrier): (those in front of this warp's run, all).  Whole CTA.
__device__ __forceinline__ int2 in_front(BookShared& s, int rank, int ranks) {
  int mine = 0, all = 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = lane; i < ranks * kBookWarps; i += 32) {
    const int n = cluster_ld_int(&s.count[i % kBookWarps], i / kBookWarps);
    all += n;
    if (i < rank * kBookWarps + warp) mine += n;
  }
  return make_int2((int)__reduce_add_sync(0xffffffffu, (unsigned)mine), (int)__reduce_add_sync(0xffffffffu, (unsigned)all));
}
// refs -> refs_out (or where they are), and the number of pages of the warp's run for which `counts` holds
template <typename Counts>
__device__ __forceinline__ int count_run(const BookView& v, const PoolRun& run, Counts counts) {
  int n = 0;
  const int lane = threadIdx.x & 31;
  const bool copy = v.refs_out != v.refs;
#pragma unroll 1
  for (int p0 = run.first + lane; p0 < run.last; p0 += 32 * 8) {
    int r[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) r[u] = p0 + 32 * u < run.last ? v.refs[p0 + 32 * u] : 0;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (p0 + 32 * u < run.last) {
        n += counts(r[u]);
        if (copy) v.refs_out[p0 + 32 * u] = r[u];
      }
  }
  return (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
}

// Table rows to their other place, a warp taking up to 256 columns of a row: row b from row from(b) (-1: none), an entry of column i as
// entry(b, i, e); keep(b, i): it is not this function's.
constexpr int kCopyColumns = 256;
template <typename From, typename Entry, typename Keep>
__device__ __forceinline__ void copy_table(const BookView& v, int rows, int cta, int ctas, From from, Entry entry, Keep keep) {
  const int segments = (v.max_pages + kCopyColumns - 1) / kCopyColumns, lane = threadIdx.x & 31;
  const long long items = (long long)rows * segments;
  for (long long item = (long long)cta * kBookWarps + (threadIdx.x >> 5); item < items; item += (long long)ctas * kBookWarps) {
    const int b = (int)(item / segments), c0 = (int)(item - (long long)b * segments) * kCopyColumns + lane, source = from(b);
    const int32_t* in = v.table + (int64_t)source * v.max_pages;
    int32_t* out = v.table_out + (int64_t)b * v.max_pages;
    int e[kCopyColumns / 32];
#pragma unroll
    for (int u = 0; u < kCopyColumns / 32; ++u) {
      const int i = c0 + 32 * u;
      e[u] = source >= 0 && i < v.max_pages ? in[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < kCopyColumns / 32; ++u) {
      const int i = c0 + 32 * u;
      if (i < v.max_pages && !keep(b, i)) out[i] = entry(b, i, e[u]);
    }
  }
}

// refs to their other place, CTAs from `cta` on
__device__ __forceinline__ void copy_refs(const BookView& v, int cta, int ctas) {
  if (v.refs_out == v.refs) return;
#pragma unroll 4
  for (long long i = (long long)cta * kBookThreads + threadIdx.x; i < v.pages; i += (long long)ctas * kBookThreads) v.refs_out[i] = v.refs[i];
}
__device__ __forceinline__ void first_status(const BookShared& s, int32_t* status) {
  __syncthreads();
  if (threadIdx.x == 0) *reinterpret_cast<unsigned long long*>(status) = (unsigned long long)(uint32_t)s.bad[1] << 32 | (uint32_t)s.bad[0];
}
// `change` added to the counts of up to 64 entries of a row, a warp's (-1: none); bad(e) for entries that name no page, and where a count falls
// below 0.  (An SM issues additions to scattered words a few clocks apart, so they are dealt out to many: 64 instead of 256 entries a warp took a
// fork of 256 rows of 500 entries from 7.2 us to 4.7, a trim that gives back 12,000 pages from 7.6 to 4.7.)
constexpr int kCountColumns = 64;
template <typename Bad>
__device__ __forceinline__ void add_to_counts(const BookView& v, const int (&e)[kCountColumns / 32], int change, Bad bad) {
  int before[kCountColumns / 32];
  if (change > 0) {
#pragma unroll
    for (int u = 0; u < kCountColumns / 32; ++u) {
      if ((uint32_t)e[u] < (uint32_t)v.pages) atomicAdd(v.refs_out + e[u], change);
      before[u] = 1;
    }
  } else {
#pragma unroll
    for (int u = 0; u < kCountColumns / 32; ++u) before[u] = (uint32_t)e[u] < (uint32_t)v.pages ? atomicAdd(v.refs_out + e[u], change) : 1;
  }
#pragma unroll
  for (int u = 0; u < kCountColumns / 32; ++u)
    if (((uint32_t)e[u] >= (uint32_t)v.pages && e[u] != -1) || before[u] <= 0) bad(e[u]);
}

// ---------------------------------------------------------------------------------------------------------------- fork
struct ForkParams {
  BookView v;
  const int32_t* kv_len;
  const int32_t* parent;
  int32_t* kv_len_out;
  int32_t* uses;                 // workspace [B]: sequences that go on from a row, less one
  int B_out;
  int32_t* status;
};
__global__ void __launch_bounds__(kBookThreads)
pages_fork_kernel(const __grid_constant__ ForkParams p) {
  const BookView& v = p.v;
  pdl_wait();
  if (blockIdx.x > 0) {
    const int cta = blockIdx.x - 1, ctas = gridDim.x - 1;
    copy_table(v, p.B_out, cta, ctas, [&](int b) { const int f = p.parent[b]; return (uint32_t)f < (uint32_t)v.B ? f : -1; }, [](int, int, int e) { return e; },
               [](int, int) { return false; });
    copy_refs(v, cta, ctas);
    return;
  }
  __shared__ BookShared s;
  __shared__ int uses[kCacheMaxSequences];
  for (int b = threadIdx.x; b < v.B; b += kBookThreads) uses[b] = -1;
  book_begin(s);
  for (int b = threadIdx.x; b < p.B_out; b += kBookThreads) {
    const int f = p.parent[b];
    const bool there = (uint32_t)f < (uint32_t)v.B;
    if (there) atomicAdd(&uses[f], 1);
    else if (f != -1) found(s, SPARKATTN_E_BAD_INDEX, f);
    p.kv_len_out[b] = there ? p.kv_len[f] : 0;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < v.B; b += kBookThreads) p.uses[b] = uses[b];
  first_status(s, p.status);
}
// Every row's number of users changes by the sequences that go on from it less one; its pages' counts do with it.
__global__ void __launch_bounds__(kBookThreads)
pages_fork_counts_kernel(const __grid_constant__ ForkParams p) {
  const BookView& v = p.v;
  const int segments = (v.max_pages + kCountColumns - 1) / kCountColumns, lane = threadIdx.x & 31;
  const long long items = (long long)v.B * segments;
  pdl_wait();
  for (long long item = (long long)blockIdx.x * kBookWarps + (threadIdx.x >> 5); item < items; item += (long long)gridDim.x * kBookWarps) {
    const int b = (int)(item / segments), c0 = (int)(item - (long long)b * segments) * kCountColumns + lane, change = p.uses[b];
    int e[kCountColumns / 32];
#pragma unroll
    for (int u = 0; u < kCountColumns / 32; ++u) e[u] = c0 + 32 * u < v.max_pages ? v.table[(int64_t)b * v.max_pages + c0 + 32 * u] : -1;
    if (change != 0) add_to_counts(v, e, change, [&](int page) { report_status(p.status, SPARKATTN_E_BAD_INDEX, page); });
  }
}

// ---------------------------------------------------------------------------------------------------------------- trim
struct TrimParams {
  BookView v;
  const int32_t* kv_len;
  int frame, window, sink, ranks;
  int32_t* status;
};
// Columns of a sequence that no later token reads: [from, to) between the first tokens and the window, and from `end` on
struct Dead {
  int from, to, end;
};
__device__ __forceinline__ Dead dead_of(const TrimParams& p, int b) {
  const int len = p.kv_len[b];
  if (!fits_table(p.v, len)) return {0, 0, p.v.max_pages};
  Dead d{0, 0, pages_of(p.v, len)};
  if (p.window > 0) {
    const long long lo = max(((long long)(len / p.frame) - p.window + 1) * p.frame, 0LL);
    d.from = (int)min((long long)pages_of(p.v, p.sink), (long long)p.v.max_pages);
    d.to = (int)(lo >> p.v.shift);
  }
  return d;
}
__device__ __forceinline__ bool is_dead(const Dead& d, int i) { return i >= d.end || (i >= d.from && i < d.to); }

__global__ void __launch_bounds__(kBookThreads)
pages_trim_kernel(const __grid_constant__ TrimParams p) {
  __shared__ BookShared s;
  const int cluster = (int)blockIdx.x / p.ranks, rank = (int)blockIdx.x - cluster * p.ranks;
  const BookView& v = p.v;
  pdl_wait();
  if (cluster > 0) {
    Dead d{};
    int of = -1;
    copy_table(v, v.B, (int)blockIdx.x - p.ranks, (int)gridDim.x - p.ranks, [&](int b) {
      if (b != of) { of = b; d = dead_of(p, b); }
      return b; }, [&](int, int i, int e) { return is_dead(d, i) ? -1 : e; }, [](int, int) { return false; });
    return;
  }
  book_begin(s);
  copy_refs(v, rank, p.ranks);
  for (int b = rank * kBookThreads + threadIdx.x; b < v.B; b += p.ranks * kBookThreads)
    if (!fits_table(v, p.kv_len[b])) found(s, SPARKATTN_E_BAD_INDEX, p.kv_len[b]);
  const int segments = (v.max_pages + kCountColumns - 1) / kCountColumns, lane = threadIdx.x & 31;
  const bool in_place = v.table_out == v.table;
  const long long items = (long long)v.B * segments, step = p.ranks * kBookWarps;
  bool waited = false;
  for (long long item = rank * kBookWarps + (threadIdx.x >> 5); item - rank * kBookWarps - (threadIdx.x >> 5) < items; item += step) {
    // (the first entries are on their way while the counts are)
    const bool there = item < items;
    const int b = there ? (int)(item / segments) : 0, first = (int)(item - (long long)b * segments) * kCountColumns, c0 = first + lane;
    const Dead d = dead_of(p, b);
    const int64_t row = (int64_t)b * v.max_pages;
    const bool some = there && (first + kCountColumns > d.end || (first < d.to && first + kCountColumns > d.from));
    int e[kCountColumns / 32];
#pragma unroll
    for (int u = 0; u < kCountColumns / 32; ++u) {
      const int i = c0 + 32 * u;
      e[u] = some && i < v.max_pages && is_dead(d, i) ? v.table[row + i] : -1;
    }
    if (!waited) book_barrier();
    waited = true;
    add_to_counts(v, e, -1, [&](int page) { found(s, SPARKATTN_E_BAD_INDEX, page); });
    if (in_place) {
#pragma unroll
      for (int u = 0; u < kCountColumns / 32; ++u)
        if (e[u] != -1) v.table_out[row + c0 + 32 * u] = -1;
    }
  }
  book_end(s, rank, p.ranks, p.status);
}

// ------------------------------------------------------------------------------------------------------------- reserve
struct ReserveParams {
  BookView v;
  const int32_t* kv_len;
  const int32_t* kv_new;
  int32_t* kv_len_out;           // NULL: not asked for
  int32_t* src;
  int32_t* dst;
  int32_t* list;                 // workspace: the free pages that are handed out, in order; then, where columns ask in place of others' pages, the entry that each has taken the place of
  int ranks, slots;              // slots of the hash table: a power of two, twice the sequences or more
  int32_t* status;
};
constexpr int kOwnColumns = 32;      // a sequence that asks for more columns is looked through by the whole CTA
// What a sequence asks for: pages for those of the columns [first, last) that have none, or one that others hold as well (reserved ahead, then
// forked: whoever goes on there would write into the others' tokens, and there is nothing in it to copy), and another page in place of a
// partly filled one, `tail`, that others hold as well.
struct Asks {
  int tail, first, last;         // tail: column of the partly filled page, or first where there is none
  bool fine;                     // the numbers make sense
  __device__ __forceinline__ bool partly() const { return tail < first; }
};
__device__ __forceinline__ Asks asks_of(const ReserveParams& p, int b) {
  const int old = p.kv_len[b], len = p.kv_new[b];
  Asks a{0, 0, 0, old >= 0 && len >= old && fits_table(p.v, len)};
  if (a.fine && len > old) a = {old >> p.v.shift, pages_of(p.v, old), pages_of(p.v, len), true};
  return a;
}
// Dynamic shared memory: prefix[B + 1]; of every sequence the columns that it asks for and the page that it copies; the hash table of partly
// filled pages that several hold: page, sequences that write to it, the first of them.  Every CTA of the first cluster has it all.
__global__ void __launch_bounds__(kBookThreads)
pages_reserve_kernel(const __grid_constant__ ReserveParams p) {
  __shared__ BookShared s;
  __shared__ int s_ahead;              // some column asks for a page in place of one that others hold
  __shared__ uint32_t s_wrong[kCacheMaxSequences / 32];      // a bit for every sequence whose numbers make no sense
  extern __shared__ int s_dynamic[];
  const BookView& v = p.v;
  int* prefix = s_dynamic;
  int* s_tail = prefix + v.B + 1;
  int* s_first = s_tail + v.B;
  int* s_last = s_first + v.B;
  int* s_copy = s_last + v.B;
  int* h_page = s_copy + v.B;
  int* h_writers = h_page + p.slots;
  int* h_first = h_writers + p.slots;
  const int cluster = (int)blockIdx.x / p.ranks, rank = (int)blockIdx.x - cluster * p.ranks;
  pdl_wait();
  if (cluster > 0) {
    Asks a{};
    int of = -1;
    copy_table(v, v.B, (int)blockIdx.x - p.ranks, (int)gridDim.x - p.ranks, [&](int b) {
      if (b != of) { of = b; a = asks_of(p, b); }
      return b; }, [](int, int, int e) { return e; }, [&](int, int i) { return i >= a.tail && i < a.last; });
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < p.slots; i += kBookThreads) { h_page[i] = -1; h_writers[i] = 0; h_first[i] = 0x7fffffff; }
  if (threadIdx.x == 0) s_ahead = 0;
  if (threadIdx.x < kCacheMaxSequences / 32) s_wrong[threadIdx.x] = 0u;
  book_begin(s);
  auto slot_of = [&](int page, bool insert) {
    uint32_t at = (uint32_t)page * 2654435761u >> 7;
    for (int tries = 0; tries < p.slots; ++tries, ++at) {           // (it always ends earlier: there are more slots than pages in it)
      int* k = h_page + (at & (p.slots - 1));
      const int there = insert ? atomicCAS(k, -1, page) : *k;
      if (there == page || (insert && there == -1)) break;
    }
    return (int)(at & (p.slots - 1));
  };
  // who writes to pages that several hold, and the columns that ask for a page
  bool long_one = false, ahead = false;
  auto wrong = [&](int b, int detail) {
    found(s, SPARKATTN_E_BAD_INDEX, detail);
    atomicOr(s_wrong + b / 32, 1u << (b & 31));
  };
  // a page ahead that others hold as well
  auto shared_ahead = [&](int b, int e) {
    if ((uint32_t)e >= (uint32_t)v.pages) return false;
    const int holders = v.refs[e];
    if (holders < 1) wrong(b, e);
    ahead |= holders > 1;
    return holders > 1;
  };
  for (int b = threadIdx.x; b < v.B; b += kBookThreads) {
    const Asks a = asks_of(p, b);
    int shared = -1;
    if (!a.fine) wrong(b, b);
    const int32_t* row = v.table + (int64_t)b * v.max_pages;
    const int e = a.partly() ? row[a.tail] : 0;
    int missing = 0;
    if (a.last - a.first <= kOwnColumns) {
      // (eight on their way at a time; mostly none of them is a page)
      for (int i0 = a.first; i0 < a.last; i0 += 8) {
        int e8[8], pages = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) e8[u] = i0 + u < a.last ? row[i0 + u] : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) pages += (uint32_t)e8[u] < (uint32_t)v.pages ? 1 : 0;
        missing += min(8, a.last - i0) - pages;
        if (pages == 0) continue;
#pragma unroll 1
        for (int i = i0; i < min(i0 + 8, a.last); ++i) missing += shared_ahead(b, row[i]) ? 1 : 0;
      }
    } else {
      long_one = true;
    }
    if (a.partly()) {
      const int holders = (uint32_t)e < (uint32_t)v.pages ? v.refs[e] : 0;
      if (holders < 1) {
        wrong(b, e);
      } else if (holders > 1) {
        shared = e;
        const int at = slot_of(e, true);
        atomicAdd(h_writers + at, 1);
        atomicMin(h_first + at, b);
      }
    }
    prefix[b] = missing;
    s_tail[b] = a.tail;
    s_first[b] = a.first;
    s_last[b] = a.last;
    s_copy[b] = shared;
  }
  if (ahead) s_ahead = 1;
  const PoolRun run = run_of_warp(v.pages, p.ranks, rank);
  const int free_here = count_run(v, run, [](int r) { return r == 0 ? 1 : 0; });
  if (lane == 0) s.count[warp] = free_here;
  if (__syncthreads_or(long_one)) {
    ahead = false;
    // 256 columns at a time, those of a sequence dealt out to the warps
    for (int b0 = 0; b0 < v.B; b0 += 32) {
      const int own = b0 + lane, columns = own < v.B ? s_last[own] - s_first[own] : 0;
      const int chunks = columns > kOwnColumns ? (columns + kCopyColumns - 1) / kCopyColumns : 0;
      for (uint32_t left = __ballot_sync(0xffffffffu, ((warp - own) & (kBookWarps - 1)) < chunks); left != 0; left &= left - 1) {
        const int b = b0 + __ffs(left) - 1, last = s_last[b];
        const int32_t* row = v.table + (int64_t)b * v.max_pages;
        int n = 0;
        for (long long i0 = s_first[b] + (long long)((warp - b) & (kBookWarps - 1)) * kCopyColumns; i0 < last; i0 += kBookWarps * kCopyColumns) {
          int e[kCopyColumns / 32], pages = 0;
#pragma unroll
          for (int u = 0; u < kCopyColumns / 32; ++u) e[u] = i0 + 32 * u + lane < last ? row[i0 + 32 * u + lane] : -1;
#pragma unroll
          for (int u = 0; u < kCopyColumns / 32; ++u) {
            const bool is = (uint32_t)e[u] < (uint32_t)v.pages;
            pages += is ? 1 : 0;
            n += i0 + 32 * u + lane < last && !is ? 1 : 0;
          }
          if (pages == 0) continue;
#pragma unroll 1
          for (long long i = i0 + lane; i < min(i0 + kCopyColumns, (long long)last); i += 32) n += shared_ahead(b, row[i]) ? 1 : 0;
        }
        n = (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
        if (lane == 0) atomicAdd(&prefix[b], n);
      }
    }
    if (ahead) s_ahead = 1;
    __syncthreads();
  }
  int carry = 0;
  for (int base = 0; base < v.B; base += kBookThreads) {
    const int b = base + threadIdx.x;
    int mine = 0;
    if (b < v.B) {
      mine = prefix[b];
      // the first of the sequences that write to a page keeps it, if nobody else holds it
      const int page = s_copy[b];
      if (page >= 0) {
        const int at = slot_of(page, false);
        if (h_writers[at] == v.refs[page] && h_first[at] == b) s_copy[b] = -1;
        else ++mine;
      }
    }
    int x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) s.scan[warp] = x;
    __syncthreads();
    int before = carry;
    for (int w = 0; w < kBookWarps; ++w) {
      if (w < warp) before += s.scan[w];
      carry += s.scan[w];
    }
    if (b < v.B) prefix[b] = before + x - mine;
    __syncthreads();
  }
  book_barrier();
  const int2 free = in_front(s, rank, p.ranks);
  const bool enough = carry <= free.y;
  if (!enough && rank == 0 && threadIdx.x == 0) {      // (goes before what else has been found)
    s.bad[0] = SPARKATTN_E_OUT_OF_PAGES;
    s.bad[1] = carry - free.y;
  }
  if (enough) {
    int k = free.x;
    for (int p0 = run.first; p0 < run.last && k < carry; p0 += 32 * 8) {
      int r[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) r[u] = p0 + 32 * u + lane < run.last ? v.refs[p0 + 32 * u + lane] : 1;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const uint32_t all = __ballot_sync(0xffffffffu, r[u] == 0);
        const int mine = k + __popc(all & ((1u << lane) - 1u)), page = p0 + 32 * u + lane;
        if (r[u] == 0 && mine < carry) {
          p.list[mine] = page;
          v.refs_out[page] = 1;
        }
        k += __popc(all);
      }
    }
  }
  book_barrier();
  // Counts of what is replaced fall at once, or, where columns are looked at for being shared, behind the last barrier, so that every
  // look sees the same; until then the list holds what its pages take the place of.
  const bool later = s_ahead != 0;
  for (int b = rank * kBookWarps + warp; b < v.B; b += p.ranks * kBookWarps) {
    const int tail = s_tail[b], first = s_first[b], last = s_last[b], from = enough ? s_copy[b] : -1;
    int at = prefix[b];
    const int32_t* row = v.table + (int64_t)b * v.max_pages;
    int32_t* out = v.table_out + (int64_t)b * v.max_pages;
    if (lane == 0) {
      const int to = from >= 0 ? p.list[at] : -1;
      if (from >= 0) {
        if (later) p.list[at] = from;
        else atomicSub(v.refs_out + from, 1);
      }
      if (p.kv_len_out != nullptr) p.kv_len_out[b] = (s_wrong[b / 32] >> (b & 31) & 1u) || (!enough && last > tail) ? -1 : p.kv_new[b];      // (last > tail: it asks)
      p.src[b] = from;
      p.dst[b] = to;
      if (tail < first) out[tail] = from >= 0 ? to : row[tail];
    }
    if (from >= 0) ++at;
    auto fill = [&](int i0, auto many) {
      constexpr int U = decltype(many)::value;
      int e[U];
#pragma unroll
      for (int u = 0; u < U; ++u) e[u] = i0 + 32 * u + lane < last ? row[i0 + 32 * u + lane] : -1;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool asks = enough && i0 + 32 * u + lane < last && ((uint32_t)e[u] >= (uint32_t)v.pages || (later && v.refs[e[u]] > 1));
        const uint32_t all = __ballot_sync(0xffffffffu, asks);
        if (asks) {
          int32_t* mine = p.list + at + __popc(all & ((1u << lane) - 1u));
          const int to = *mine;
          if (later) *mine = e[u];
          e[u] = to;
        }
        at += __popc(all);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + 32 * u + lane < last) out[i0 + 32 * u + lane] = e[u];
    };
    if (last - first <= 32) {
      fill(first, std::integral_constant<int, 1>{});
    } else {
      for (int i0 = first; i0 < last; i0 += kCopyColumns) fill(i0, std::integral_constant<int, kCopyColumns / 32>{});
    }
  }
  book_end(s, rank, p.ranks, p.status);
  if (!later || !enough) return;      // (its barrier stands between the last look at a count and what follows)
  for (int i = rank * kBookThreads + threadIdx.x; i < carry; i += p.ranks * kBookThreads) {
    const int e = p.list[i];
    if ((uint32_t)e < (uint32_t)v.pages) atomicSub(v.refs_out + e, 1);
  }
}

// ------------------------------------------------------------------------------------------------------------- compact
struct CompactParams {
  BookView v;
  int32_t* src;
  int32_t* dst;                  // [pages / 2]
  int32_t* to;                   // workspace [pages]: where a page goes, -1: nobody holds it
  int ranks;
  int32_t* status;
};
// With n pages in use, those from n on move, the i-th of them to the i-th free page below n.  A free page at x has x - used(x) free ones in
// front of it, a moving one used(x) - used(n) moving ones.
__global__ void __launch_bounds__(kBookThreads)
pages_compact_kernel(const __grid_constant__ CompactParams p) {
  __shared__ BookShared s;
  __shared__ int s_part;
  const int rank = (int)blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const BookView& v = p.v;
  pdl_wait();
  book_begin(s);
  const PoolRun run = run_of_warp(v.pages, p.ranks, rank);
  int n = 0;
#pragma unroll 8
  for (int i = run.first + lane; i < run.last; i += 32) n += v.refs[i] > 0 ? 1 : 0;
  n = (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
  if (lane == 0) s.count[warp] = n;
  if (threadIdx.x == 0) s_part = 0;
  book_barrier();
  const int2 used = in_front(s, rank, p.ranks);
  // used(n): the runs in front of n's, and a part of that one
  const int border = used.y, each = run_length(v.pages, p.ranks), border_run = border / each;
  int front = 0;
  for (int i = lane; i < min(border_run, p.ranks * kBookWarps); i += 32) front += cluster_ld_int(&s.count[i % kBookWarps], i / kBookWarps);
  front = (int)__reduce_add_sync(0xffffffffu, (unsigned)front);
  int part = 0;
  for (long long i = (long long)border_run * each + threadIdx.x; i < border; i += kBookThreads) part += v.refs[i] > 0 ? 1 : 0;
  part = (int)__reduce_add_sync(0xffffffffu, (unsigned)part);
  if (lane == 0) atomicAdd(&s_part, part);
  __syncthreads();
  const int below = front + s_part, moves = border - below;
  int k = used.x;                                                   // used pages in front
  for (int p0 = run.first; p0 < run.last; p0 += 32 * 8) {
    int r[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) r[u] = p0 + 32 * u + lane < run.last ? v.refs[p0 + 32 * u + lane] : 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int at = p0 + 32 * u + lane;
      const bool there = at < run.last, is = there && r[u] > 0;
      const uint32_t all = __ballot_sync(0xffffffffu, is);
      const int in_use = k + __popc(all & ((1u << lane) - 1u));
      if (there) {
        if (is && at >= border) p.src[in_use - below] = at;
        else p.to[at] = is ? at : -1;
        if (!is && at < border) p.dst[at - in_use] = at;
      }
      k += __popc(all);
    }
  }
  for (int i = moves + rank * kBookThreads + threadIdx.x; i < v.pages / 2; i += p.ranks * kBookThreads) p.src[i] = p.dst[i] = -1;
  book_barrier();
  if (v.refs_out != v.refs) {
    // every page's count where it ends up: what stays, then what moves (whose new places nobody held)
#pragma unroll 8
    for (int p0 = run.first + lane; p0 < run.last; p0 += 32) {
      const int r = v.refs[p0];
      if (p0 < border ? r > 0 : true) v.refs_out[p0] = p0 < border ? r : 0;
    }
  }
#pragma unroll 4
  for (int i = rank * kBookThreads + threadIdx.x; i < moves; i += p.ranks * kBookThreads) {
    const int from = p.src[i], to = p.dst[i];
    p.to[from] = to;
    v.refs_out[to] = v.refs[from];
    if (v.refs_out == v.refs) v.refs_out[from] = 0;
  }
  book_end(s, rank, p.ranks, p.status);
}
__global__ void __launch_bounds__(kBookThreads)
pages_remap_kernel(const __grid_constant__ CompactParams p) {
  pdl_wait();
  const long long entries = (long long)p.v.B * p.v.max_pages, step = (long long)gridDim.x * kBookThreads;
#pragma unroll 4
  for (long long i = (long long)blockIdx.x * kBookThreads + threadIdx.x; i < entries; i += step) {
    const int e = p.v.table[i];
    const int to = (uint32_t)e < (uint32_t)p.v.pages ? p.to[e] : -1;
    if (to < 0 && e != -1) report_status(p.status, SPARKATTN_E_BAD_INDEX, e);
    p.v.table_out[i] = to;
  }
}

// ---------------------------------------------------------------------------------------------------------------- copy
constexpr int kCopyThreads = 256, kCopyUnroll = 8, kCopyPerSM = 4, kCopyPieces = 32 * kCopyUnroll;      // 16-byte pieces of a unit, a warp's
constexpr int kCheckPages = 1 << 16;      // pages that a checking CTA looks after: two bits each in 16 KB

struct CopyPagesParams {
  const uint4* from[2];          // K, V
  uint4* to[2];
  const float* scale_from[2];    // NULL: bf16
  float* scale_to[2];
  int64_t page_from, page_to;    // strides in 16-byte pieces
  int64_t outer_from[2], outer_to[2];      // of a run: (j / runs) * outer[0] + (j % runs) * outer[1]
  FastDiv by_run, by_runs;
  int run, runs, pieces;         // contiguous pieces; runs of the inner dimension; pieces of a page
  int H, pages_from, pages_to, same;       // same: one pool
  const int32_t* src;
  const int32_t* dst;
  int n, split;                  // pairs; units of a page's K or V
  long long units;
  int check_ctas;
  int32_t* status;
};

// Looks through the pairs: numbers outside the pools, a page that is written twice, and one that is written and read.
__device__ __forceinline__ bool check_pairs(const CopyPagesParams& p, int range, uint32_t* bits, int* s_bad) {
  const int first = range * kCheckPages;
  uint32_t* written = bits;
  uint32_t* read = bits + kCheckPages / 32;
  for (int i = threadIdx.x; i < 2 * kCheckPages / 32; i += kCopyThreads) bits[i] = 0u;
  if (threadIdx.x == 0) { s_bad[0] = 0; s_bad[1] = 0; }
  __syncthreads();
  auto bad = [&](int page) { if (atomicExch(s_bad, 1) == 0) s_bad[1] = page; };
  auto look = [&](int a, int b) {
    if (a == -1 && b == -1) return;
    if ((uint32_t)a >= (uint32_t)p.pages_from || (uint32_t)b >= (uint32_t)p.pages_to) {
      bad((uint32_t)a >= (uint32_t)p.pages_from ? a : b);
      return;
    }
    // (whoever marks a page as written looks for it among those read, and the other way round, each after its own mark: one of two finds the other)
    const uint32_t to = (uint32_t)b - (uint32_t)first, from = (uint32_t)a - (uint32_t)first;
    if (to < (uint32_t)kCheckPages) {
      const uint32_t bit = 1u << (to & 31);
      if (atomicOr(written + (to >> 5), bit) & bit) bad(b);
      if (p.same && (atomicOr(read + (to >> 5), 0u) & bit)) bad(b);
    }
    if (p.same && from < (uint32_t)kCheckPages) {
      const uint32_t bit = 1u << (from & 31);
      atomicOr(read + (from >> 5), bit);
      if (atomicOr(written + (from >> 5), 0u) & bit) bad(a);
    }
  };
  // sixteen bytes at a time where the lists lie so (200,000 pairs of -1: 40 us, one by one and in two passes 82)
  const int whole = ((reinterpret_cast<uintptr_t>(p.src) | reinterpret_cast<uintptr_t>(p.dst)) & 15u) == 0 ? p.n / 4 : 0;
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < whole; i0 += 4 * kCopyThreads) {
    int4 a[4], b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool there = whole - i0 > u * kCopyThreads;
      a[u] = there ? reinterpret_cast<const int4*>(p.src)[i0 + u * kCopyThreads] : make_int4(-1, -1, -1, -1);
      b[u] = there ? reinterpret_cast<const int4*>(p.dst)[i0 + u * kCopyThreads] : make_int4(-1, -1, -1, -1);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      look(a[u].x, b[u].x);
      look(a[u].y, b[u].y);
      look(a[u].z, b[u].z);
      look(a[u].w, b[u].w);
    }
  }
#pragma unroll 1
  for (long long i = 4LL * whole + threadIdx.x; i < p.n; i += kCopyThreads) look(p.src[i], p.dst[i]);
  __syncthreads();
  const bool is = s_bad[0] != 0;
  if (threadIdx.x == 0 && is) report_early(p.status, SPARKATTN_E_BAD_INDEX, s_bad[1]);
  __syncthreads();
  return is;
}

// Warps go through the units, 4 KB of a page's K or V each, w, w + warps, ...: 32 of them are looked up at a time, and those with a page to copy
// copied one after the other, eight 16-byte loads of every lane in flight.
__global__ void __launch_bounds__(kCopyThreads, kCopyPerSM)
cache_copy_pages_kernel(const __grid_constant__ CopyPagesParams p) {
  __shared__ uint32_t bits[2 * kCheckPages / 32];
  __shared__ int s_bad[2];
  pdl_wait();
  if ((int)blockIdx.x < p.check_ctas) {
    bool code_there = false;
    if (blockIdx.x == 0 && threadIdx.x == 0) code_there = take_header(p.status);
    check_pairs(p, blockIdx.x, bits, s_bad);
    if (blockIdx.x == 0 && __syncthreads_or(code_there))
      // the word held a code, which may have been another CTA's: see take_header
      for (int range = 1; range < p.check_ctas; ++range) check_pairs(p, range, bits, s_bad);
    return;
  }
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)((int)blockIdx.x - p.check_ctas) * (kCopyThreads / 32) + (threadIdx.x >> 5);
  const long long warps = (long long)((int)gridDim.x - p.check_ctas) * (kCopyThreads / 32);
#pragma unroll 1
  for (long long u0 = warp; u0 < p.units; u0 += 32 * warps) {
    const long long unit = u0 + lane * warps;
    int from = -1, to = -1, part = 0;
    if (unit < p.units) {
      const int pair = (int)(unit / (2 * p.split));
      part = (int)(unit - (long long)pair * 2 * p.split);
      from = p.src[pair];
      to = p.dst[pair];
    }
    uint32_t going = __ballot_sync(0xffffffffu, (uint32_t)from < (uint32_t)p.pages_from && (uint32_t)to < (uint32_t)p.pages_to);
    for (; going != 0; going &= going - 1) {
      const int l = __ffs(going) - 1;
      const int its_from = __shfl_sync(0xffffffffu, from, l), its_to = __shfl_sync(0xffffffffu, to, l), its_part = __shfl_sync(0xffffffffu, part, l);
      const int kv = its_part >= p.split, first = (its_part - kv * p.split) * kCopyPieces + lane;
      const uint4* in = p.from[kv] + its_from * p.page_from;
      uint4* out = p.to[kv] + its_to * p.page_to;
      uint4 x[kCopyUnroll];
      if (p.run == p.pieces) {
        // the whole page side by side
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u)
          if (first + 32 * u < p.pieces) x[u] = in[first + 32 * u];
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u)
          if (first + 32 * u < p.pieces) out[first + 32 * u] = x[u];
      } else {
        int64_t at[kCopyUnroll];
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
          const int piece = first + 32 * u, run = fast_div(piece, p.by_run), in_run = piece - run * p.run;
          const int outer = fast_div(run, p.by_runs), inner = run - outer * p.runs;
          at[u] = outer * p.outer_to[0] + inner * p.outer_to[1] + in_run;
          if (piece < p.pieces) x[u] = in[outer * p.outer_from[0] + inner * p.outer_from[1] + in_run];
        }
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u)
          if (first + 32 * u < p.pieces) out[at[u]] = x[u];
      }
      if (p.scale_from[kv] != nullptr && its_part == kv * p.split)
        for (int h = lane; h < p.H; h += 32) p.scale_to[kv][(int64_t)its_to * p.H + h] = p.scale_from[kv][(int64_t)its_from * p.H + h];
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ host side
namespace {
// CTAs of the first cluster: by the words that it goes through, some 4000 a CTA
int ranks_for(long long words) {
  int n = 1;
  while (n < kBookClusterMax && (long long)n * 4096 < words) n *= 2;
  return n;
}
// CTAs for rows of max_pages entries, a warp for `columns` of them
int ctas_for(long long rows, int max_pages, int columns, int sms) {
  const long long warps = rows * ((max_pages + columns - 1) / columns), ctas = (warps + kBookWarps - 1) / kBookWarps;
  return (int)std::max<long long>(1, std::min<long long>(ctas, 2LL * sms));
}
template <typename Params>
int launch_book(void (*kern)(Params), int clusters, int ranks, size_t smem, cudaStream_t stream, const Params& p) {
  if (ranks > 8 && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return SPARKATTN_E_CUDA;
  return launch_clustered(kern, dim3((unsigned)(clusters * ranks)), kBookThreads, smem, true, ranks, stream, p);
}
}  // namespace

size_t pages_workspace_bytes(const sparkattn_book_t& b) { return kWorkspaceHeaderBytes + ((size_t)std::max(b.pages, b.B) * 4 + 255) / 256 * 256; }

int launch_pages_fork(const sparkattn_book_t& book, const int32_t* kv_len, const int32_t* parent, int B_out, int32_t* table_out, int32_t* kv_len_out,
                      int32_t* refs_out, void* workspace, cudaStream_t stream) {
  int32_t* status = static_cast<int32_t*>(workspace);
  const ForkParams p{make_book_view(book, table_out, refs_out), kv_len, parent, kv_len_out, status + kWorkspaceHeaderBytes / 4, B_out, status};
  const int sms = current_sm_count();
  if (sms < 1) return SPARKATTN_E_CUDA;
  const int rc = launch_kernel(pages_fork_kernel, dim3(1 + ctas_for(B_out, book.max_pages, kCopyColumns, sms)), kBookThreads, 0, true, stream, p);
  if (rc != SPARKATTN_OK) return rc;
  return launch_kernel(pages_fork_counts_kernel, dim3(ctas_for(book.B, book.max_pages, kCountColumns, sms)), kBookThreads, 0, true, stream, p);
}

int launch_pages_trim(const sparkattn_book_t& book, const int32_t* kv_len, int frame, int window, int sink, int32_t* table_out, int32_t* refs_out,
                      void* workspace, cudaStream_t stream) {
  TrimParams p{make_book_view(book, table_out, refs_out), kv_len, std::max(frame, 1), window, sink, 1, static_cast<int32_t*>(workspace)};
  const int sms = current_sm_count();
  if (sms < 1) return SPARKATTN_E_CUDA;
  p.ranks = ranks_for(4LL * book.B * book.max_pages + book.pages);
  const int copiers = table_out != book.page_table ? (ctas_for(book.B, book.max_pages, kCopyColumns, sms) + p.ranks - 1) / p.ranks : 0;
  return launch_book(pages_trim_kernel, 1 + copiers, p.ranks, 0, stream, p);
}

int launch_pages_reserve(const sparkattn_book_t& book, const int32_t* kv_len, const int32_t* kv_new, int32_t* kv_len_out, int32_t* table_out,
                         int32_t* refs_out, int32_t* src, int32_t* dst, void* workspace, cudaStream_t stream) {
  int32_t* status = static_cast<int32_t*>(workspace);
  ReserveParams p{make_book_view(book, table_out, refs_out), kv_len, kv_new, kv_len_out, src, dst, status + kWorkspaceHeaderBytes / 4, 1, 64, status};
  const int sms = current_sm_count();
  if (sms < 1) return SPARKATTN_E_CUDA;
  while (p.slots < 2 * book.B) p.slots *= 2;
  p.ranks = ranks_for((long long)book.pages + 64LL * book.B);
  const size_t smem = (5 * (size_t)book.B + 1 + 3 * (size_t)p.slots) * 4;
  // (the most that any call asks for: host threads with other batches set it too)
  if (cudaFuncSetAttribute(pages_reserve_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (5 * kCacheMaxSequences + 1 + 3 * 2 * kCacheMaxSequences) * 4) != cudaSuccess)
    return SPARKATTN_E_CUDA;
  const int copiers = table_out != book.page_table ? (ctas_for(book.B, book.max_pages, kCopyColumns, sms) + p.ranks - 1) / p.ranks : 0;
  return launch_book(pages_reserve_kernel, 1 + copiers, p.ranks, smem, stream, p);
}

int launch_pages_compact(const sparkattn_book_t& book, int32_t* table_out, int32_t* refs_out, int32_t* src, int32_t* dst, void* workspace, cudaStream_t stream) {
  int32_t* status = static_cast<int32_t*>(workspace);
  CompactParams p{make_book_view(book, table_out, refs_out), src, dst, status + kWorkspaceHeaderBytes / 4, ranks_for(book.pages), status};
  const int sms = current_sm_count();
  if (sms < 1) return SPARKATTN_E_CUDA;
  const int rc = launch_book(pages_compact_kernel, 1, p.ranks, 0, stream, p);
  if (rc != SPARKATTN_OK) return rc;
  const long long entries = (long long)book.B * book.max_pages, ctas = (entries + 4 * kBookThreads - 1) / (4 * kBookThreads);
  return launch_kernel(pages_remap_kernel, dim3((unsigned)std::min<long long>(ctas, 2 * sms)), kBookThreads, 0, true, stream, p);
}

int launch_copy_pages(const sparkattn_cache_t& from, const PagePools& in, const sparkattn_cache_t& to, const PagePools& out, const int32_t* src,
                      const int32_t* dst, int n, void* workspace, cudaStream_t stream) {
  CopyPagesParams p{};
  const int per16 = from.dtype == SPARKATTN_BF16 ? 8 : 16;
  for (int i = 0; i < 2; ++i) {
    p.from[i] = static_cast<const uint4*>(i ? in.v : in.k);
    p.to[i] = static_cast<uint4*>(i ? out.v : out.k);
    p.scale_from[i] = i ? in.v_scale : in.k_scale;
    p.scale_to[i] = i ? out.v_scale : out.k_scale;
  }
  p.page_from = from.stride_page / per16;
  p.page_to = to.stride_page / per16;
  // the page as runs of contiguous bytes: rows, with the tokens of a head or the heads of a token where these lie side by side in both pools, or all
  struct Dim {
    long long count, from, to;
  } token{from.page, from.stride_n, to.stride_n}, head{from.H, from.stride_h, to.stride_h}, in_dim = token, out_dim = head;
  if (!(token.from == from.d && token.to == from.d) && head.from == from.d && head.to == from.d) { in_dim = head; out_dim = token; }
  long long run = from.d;
  auto join = [&](Dim& d) { if (d.from == run && d.to == run) { run *= d.count; d.count = 1; } };
  join(in_dim);
  if (in_dim.count == 1) join(out_dim);
  if (run / per16 > 0x3fffffffLL || (long long)from.H * from.page * from.d / per16 > 0x3fffffffLL) return SPARKATTN_E_UNSUPPORTED_SHAPE;
  p.run = (int)(run / per16);
  p.runs = (int)in_dim.count;
  p.outer_from[0] = out_dim.from / per16; p.outer_from[1] = in_dim.from / per16;
  p.outer_to[0] = out_dim.to / per16; p.outer_to[1] = in_dim.to / per16;
  p.by_run = make_fast_div(p.run);
  p.by_runs = make_fast_div(p.runs);
  p.pieces = (int)((long long)from.H * from.page * from.d / per16);
  p.H = from.H;
  p.pages_from = from.pages;
  p.pages_to = to.pages;
  p.same = in.k == out.k;
  p.src = src; p.dst = dst; p.n = n;
  p.split = (p.pieces + kCopyPieces - 1) / kCopyPieces;
  p.units = 2LL * p.split * n;
  p.check_ctas = (int)(((long long)to.pages + kCheckPages - 1) / kCheckPages);
  p.status = static_cast<int32_t*>(workspace);
  const int sms = current_sm_count();
  if (sms < 1) return SPARKATTN_E_CUDA;
  const unsigned ctas = p.check_ctas + (unsigned)std::min<long long>((p.units + kCopyThreads / 32 - 1) / (kCopyThreads / 32), (long long)kCopyPerSM * sms);
  return launch_kernel(cache_copy_pages_kernel, dim3(ctas), kCopyThreads, 0, true, stream, p);
}

}  // namespace sparkattn
