// Page tables of a paged cache: pages handed out, shared, given back, compacted, and rows of other pools copied (sm_100a).
//
// A call lists at most 1024 rows.  What it changes in the tables is decided by one CTA (a row per thread, sums over the rows by one
// scan), so that every answer follows from the order of the list alone and no atomic's order reaches a result: atomics are
// only used where their order cannot be seen (sums, minima, maxima).  The bytes of pages that move are copied by a second kernel over
// the whole GPU, from a list of (source, destination) pairs that the first one left in the caller's workspace; a source is never a
// destination of the same call, so the copies need no order.  The bookkeeping is bound by latency (a handful of dependent loads), the copy
// by memory: each byte is read once and written once.
#include <cuda_runtime.h>

#include <climits>

#include "internal.h"

namespace lumo {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kCopyFlight = 4;                                    // 16-byte pieces in flight per thread
constexpr int kChunk = kCopyThreads * kCopyFlight * 16;           // bytes one CTA copies at a time
static_assert(kMaxPageRows <= kPlanThreads, "a thread per listed row");

// the caller's workspace, in ints: owner[n_rows] | count[n_pages] | last[n_pages] | src[n_pages] | dst[n_pages] | moves, live
struct WorkView {
  int32_t *owner, *count, *last, *src, *dst, *moves;
  __host__ __device__ explicit WorkView(const PageTableDev& t) {
    owner = t.work;
    count = owner + t.n_rows;
    last = count + t.n_pages;
    src = last + t.n_pages;
    dst = src + t.n_pages;
    moves = dst + t.n_pages;
  }
};

__device__ __forceinline__ int pages_of(const PageTableDev& t, int positions) { return (int)(((long long)positions + t.page - 1) / t.page); }

// exclusive sum over the CTA's threads; *total gets the sum of all (every thread; two barriers)
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* total) {
  __shared__ unsigned long long part[kPlanThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();                                                // the last call's readers are done with part
  if (lane == 31) part[warp] = x;
  __syncthreads();
  unsigned long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w < warp) before += part[w];
    all += part[w];
  }
  *total = all;
  return before + x - v;
}

// The listed row of this thread: -1 if there is none (or it is passed over); *st says what is wrong with it.  The first of equal rows
// counts, the others are refused.  Every thread calls it.
__device__ __forceinline__ int listed_row(const PageTableDev& t, const WorkView& w, const int32_t* rows, int n, int* st) {
  const int i = threadIdx.x;
  int row = i < n ? rows[i] : -1;
  *st = LUMO_SEQ_OK;
  if (row != -1 && (row < 0 || row >= t.n_rows)) { *st = LUMO_SEQ_BAD_ROW; row = -1; }
  if (row >= 0) __stcg(&w.owner[row], INT_MAX);
  __syncthreads();
  if (row >= 0) atomicMin(&w.owner[row], i);
  __syncthreads();
  if (row >= 0 && __ldcg(&w.owner[row]) != i) { *st = LUMO_SEQ_BAD_ROW; row = -1; }
  return row;
}

// ---- reserve ------------------------------------------------------------------------------
// Positions [start, end) of every listed row become writable: pages among them that other rows share are replaced by copies, missing ones
// are added.  All or nothing: when the free pages do not suffice, nothing changes.
__global__ void __launch_bounds__(kPlanThreads, 1) pages_reserve_kernel(const PageTableDev t, const int32_t* rows, const int32_t* start,
                                                                     const int32_t* end, int add, int n, int32_t* status) {
  __shared__ int4 grow[kMaxPageRows];                             // row, first page to add, end, place of the first in the order of taking
  const int i = threadIdx.x;
  const WorkView w(t);
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  int st;
  int row = listed_row(t, w, rows, n, &st);
  int have = 0, need = 0, first = 0, stop = 0;                    // pages: mapped, wanted, shared ones looked for in [first, stop)
  if (row >= 0) {
    const int a = start[i];
    const long long z = end ? (long long)end[i] : (long long)a + add;
    have = t.row_pages[row];
    if (a < 0 || z < a || (z + t.page - 1) / t.page > t.max_pages || have < 0 || have > t.max_pages) {
      st = LUMO_SEQ_BAD_CTX;
      row = -1;
    } else {
      need = pages_of(t, (int)z);
      if (z > a) { first = a / t.page; stop = min(have, need); }
    }
  }
  const int32_t* mine = t.table + (size_t)(row < 0 ? 0 : row) * t.max_pages;
  if (row >= 0)
    for (int k = first; k < stop; ++k) {
      const int pg = mine[k];
      if (pg < 0 || pg >= t.n_pages) { st = LUMO_SEQ_BAD_PAGE; row = -1; break; }
    }
  if (row < 0) { have = need = first = stop = 0; }
  for (int k = first; k < stop; ++k) {
    const int pg = mine[k];
    if (t.refs[pg] > 1) { __stcg(&w.count[pg], 0); __stcg(&w.last[pg], -1); }
  }
  __syncthreads();
  for (int k = first; k < stop; ++k) {
    const int pg = mine[k];
    if (t.refs[pg] > 1) { atomicAdd(&w.count[pg], 1); atomicMax(&w.last[pg], i); }
  }
  __syncthreads();
  // a shared page is copied, except for the last listed sharer when all its sharers are listed
  auto copied = [&](int pg) {
    const int r = t.refs[pg];
    return r > 1 && !(__ldcg(&w.count[pg]) == r && __ldcg(&w.last[pg]) == i);
  };
  int copies = 0;
  for (int k = first; k < stop; ++k) copies += copied(mine[k]);
  const int extra = need > have ? need - have : 0;
  unsigned long long all;
  const unsigned long long before = block_scan((unsigned long long)(copies + extra) << 32 | (unsigned)copies, &all);
  const int total = (int)(all >> 32), moves = (int)(all & 0xffffffffu);
  const int free = min(max(*t.free_count, 0), t.n_pages);
  const bool fits = total <= free;
  if (status && i < n) status[i] = st != LUMO_SEQ_OK ? st : (row >= 0 && !fits ? (int)LUMO_SEQ_NO_PAGES : (int)LUMO_SEQ_OK);
  __syncthreads();                                                // every thread has read the count
  if (i == 0) *w.moves = fits ? moves : 0;
  if (!fits) return;                                              // the same answer in every thread
  int order = (int)(before >> 32), m = (int)(before & 0xffffffffu);
  for (int k = first; k < stop; ++k) {
    const int pg = mine[k];
    if (!copied(pg)) continue;
    const int fresh = t.free_list[free - 1 - order++];
    const bool real = fresh >= 0 && fresh < t.n_pages;            // (a list that was never set up leads nowhere)
    __stcg(&w.src[m], real ? pg : -1);
    __stcg(&w.dst[m], fresh);
    ++m;
    if (!real) continue;
    t.table[(size_t)row * t.max_pages + k] = fresh;
    t.refs[fresh] = 1;
  }
  if (i < kMaxPageRows) grow[i] = extra ? make_int4(row, have, need, order) : make_int4(0, 0, 0, 0);
  if (extra) t.row_pages[row] = need;
  __syncthreads();
  for (int k = i; k < moves; k += kPlanThreads) {
    const int pg = __ldcg(&w.src[k]);
    if (pg >= 0) atomicSub(&t.refs[pg], 1);
  }
  for (int r = i >> 5; r < n; r += kPlanThreads / 32) {
    const int4 g = grow[r];
    for (int k = g.y + (i & 31); k < g.z; k += 32) {
      const int fresh = t.free_list[free - 1 - (g.w + k - g.y)];
      if (fresh < 0 || fresh >= t.n_pages) continue;
      t.table[(size_t)g.x * t.max_pages + k] = fresh;
      t.refs[fresh] = 1;
    }
  }
  if (i == 0) *t.free_count = free - total;
}

// ---- free ---------------------------------------------------------------------------------
// Pages of the listed rows behind the first `keep` positions given back.  A released page whose count falls to zero goes onto the free list
// once, in the place of the first entry that released it; the entries count in the order of the list, and the last one is stored first,
// so that pages taken by one call and given back by another come off the list in the same order again.
__global__ void __launch_bounds__(kPlanThreads, 1) pages_free_kernel(const PageTableDev t, const int32_t* rows, const int32_t* keep, int n, int32_t* status) {
  constexpr int kWarps = kPlanThreads / 32, kFlight = 4;          // a warp goes through its rows 128 entries at a time
  __shared__ int4 row_of[kMaxPageRows];                           // row, its first released page, one behind the last, number of its first entry
  __shared__ int given_of[kMaxPageRows];                          // pages the row gives back
  const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
  const WorkView w(t);
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  int st;
  int row = listed_row(t, w, rows, n, &st);
  int have = 0, left = 0;
  if (row >= 0) {
    const int kp = keep ? keep[i] : 0;
    have = t.row_pages[row];
    if (kp < 0 || have < 0 || have > t.max_pages) { st = LUMO_SEQ_BAD_CTX; row = -1; have = 0; }
    else left = min(have, pages_of(t, kp));
  }
  if (status && i < n) status[i] = st;
  unsigned long long all;
  const int before = (int)block_scan((unsigned long long)(row >= 0 ? have - left : 0), &all);
  if (i < kMaxPageRows) { row_of[i] = row >= 0 ? make_int4(row, left, have, before) : make_int4(0, 0, 0, 0); given_of[i] = 0; }
  if (row >= 0) t.row_pages[row] = left;
  __syncthreads();
  // f(place in the table, page or -1, number of the entry, whether there is one) for the entries of a row, in order, whole warps at a time
  auto walk = [&](int r, auto f) {
    const int4 g = row_of[r];
    int32_t* mine = t.table + (size_t)g.x * t.max_pages;
    for (int k0 = g.y; k0 < g.z; k0 += 32 * kFlight) {
      int pg[kFlight];
#pragma unroll
      for (int q = 0; q < kFlight; ++q) {
        const int k = k0 + 32 * q + lane;
        pg[q] = k < g.z ? mine[k] : -1;
        if (pg[q] < 0 || pg[q] >= t.n_pages) pg[q] = -1;          // (an entry that names no page releases none)
      }
      f(mine, k0, pg, g);
    }
  };
  for (int r = warp; r < n; r += kWarps)
    walk(r, [&](int32_t*, int, const int* pg, const int4&) {
#pragma unroll
      for (int q = 0; q < kFlight; ++q)
        if (pg[q] >= 0) __stcg(&w.count[pg[q]], INT_MAX);
    });
  __syncthreads();
  for (int r = warp; r < n; r += kWarps)
    walk(r, [&](int32_t*, int k0, const int* pg, const int4& g) {
#pragma unroll
      for (int q = 0; q < kFlight; ++q)
        if (pg[q] >= 0) { atomicMin(&w.count[pg[q]], g.w + k0 + 32 * q + lane - g.y); atomicSub(&t.refs[pg[q]], 1); }
    });
  __syncthreads();
  // an entry gives its page back when nobody holds the page any longer and it is the first that released it
  auto gives = [&](const int* pg, int k0, const int4& g, bool* out) {
    int ref[kFlight], first[kFlight];
#pragma unroll
    for (int q = 0; q < kFlight; ++q) { ref[q] = pg[q] >= 0 ? __ldcg(&t.refs[pg[q]]) : 1; first[q] = pg[q] >= 0 ? __ldcg(&w.count[pg[q]]) : -1; }
#pragma unroll
    for (int q = 0; q < kFlight; ++q) out[q] = ref[q] <= 0 && first[q] == g.w + k0 + 32 * q + lane - g.y;
  };
  for (int r = warp; r < n; r += kWarps) {
    int sum = 0;
    walk(r, [&](int32_t*, int k0, const int* pg, const int4& g) {
      bool gv[kFlight];
      gives(pg, k0, g, gv);
#pragma unroll
      for (int q = 0; q < kFlight; ++q) sum += __popc(__ballot_sync(0xffffffffu, gv[q]));
    });
    if (lane == 0) given_of[r] = sum;
  }
  __syncthreads();
  const int mine_given = i < n ? given_of[i] : 0;
  const int rank0 = (int)block_scan((unsigned long long)mine_given, &all);
  const int given = (int)all;
  if (i < n) given_of[i] = rank0;                                 // now: pages given back by the rows before
  const int free = min(max(*t.free_count, 0), t.n_pages - min(given, t.n_pages));
  __syncthreads();
  for (int r = warp; r < n; r += kWarps) {
    int rank = given_of[r];
    walk(r, [&](int32_t* mine, int k0, const int* pg, const int4& g) {
      bool gv[kFlight];
      gives(pg, k0, g, gv);
#pragma unroll
      for (int q = 0; q < kFlight; ++q) {
        const unsigned m = __ballot_sync(0xffffffffu, gv[q]);
        if (gv[q]) t.free_list[free + given - 1 - (rank + __popc(m & ((1u << lane) - 1u)))] = pg[q];
        rank += __popc(m);
        if (k0 + 32 * q + lane < g.z) mine[k0 + 32 * q + lane] = -1;
      }
    });
  }
  if (i == 0) *t.free_count = free + given;
}

// ---- fork ---------------------------------------------------------------------------------
// A CTA per pair: the destination row, empty so far, gets the source's pages.  A destination that an earlier pair names, or that is
// a source of the call, is refused, so no CTA reads what another one writes: a source that a pair names as its destination stays as it was.
// A pair that is passed over (-1 on either side) names nothing.
__global__ void __launch_bounds__(kCopyThreads) pages_fork_kernel(const PageTableDev t, const int32_t* src, const int32_t* dst, int n, int32_t* status) {
  const int i = blockIdx.x, tid = threadIdx.x;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int s = src[i], d = dst[i];
  int st = LUMO_SEQ_OK;
  if (s == -1 || d == -1) {                                       // passed over
    if (tid == 0 && status) status[i] = st;
    return;
  }
  bool clash = false;
  for (int j = tid; j < n; j += kCopyThreads) {
    const int sj = src[j], dj = dst[j];
    clash |= sj != -1 && dj != -1 && ((dj == d && j < i) || sj == d);
  }
  clash = __syncthreads_or(clash);
  int have = 0;
  if (s < 0 || s >= t.n_rows || d < 0 || d >= t.n_rows || clash) st = LUMO_SEQ_BAD_ROW;
  else {
    have = t.row_pages[s];
    if (t.row_pages[d] != 0) st = LUMO_SEQ_BAD_ROW;
    else if (have < 0 || have > t.max_pages) st = LUMO_SEQ_BAD_CTX;
  }
  bool bad = false;
  if (st == LUMO_SEQ_OK)
    for (int k = tid; k < have; k += kCopyThreads) {
      const int pg = t.table[(size_t)s * t.max_pages + k];
      bad |= pg < 0 || pg >= t.n_pages;
    }
  if (__syncthreads_or(bad)) st = LUMO_SEQ_BAD_PAGE;              // (the barrier: row_pages[d] has been read by every thread)
  if (tid == 0 && status) status[i] = st;
  if (st != LUMO_SEQ_OK) return;
  for (int k = tid; k < have; k += kCopyThreads) {
    const int pg = t.table[(size_t)s * t.max_pages + k];
    t.table[(size_t)d * t.max_pages + k] = pg;
    atomicAdd(&t.refs[pg], 1);
  }
  if (tid == 0) t.row_pages[d] = have;
}

// ---- compact ------------------------------------------------------------------------------
// The pages in use move to the lowest numbers: with L of them, the k-th page in use at or beyond L goes to the k-th unused one below L.
__global__ void __launch_bounds__(kPlanThreads, 1) pages_compact_kernel(const PageTableDev t) {
  constexpr int kWords = kMaxPages / 32, kOwn = kWords / kPlanThreads;
  __shared__ uint32_t used[kWords];                               // a bit per page
  __shared__ int below_s;
  const int i = threadIdx.x, lane = i & 31;
  const WorkView w(t);
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int words = (t.n_pages + 31) / 32;
  const int own = (words + kPlanThreads - 1) / kPlanThreads;      // consecutive words per thread
  for (int k = i >> 5; k < kOwn * kPlanThreads && k < own * kPlanThreads; k += kPlanThreads / 32) {
    const int p = k * 32 + lane;
    const uint32_t b = __ballot_sync(0xffffffffu, p < t.n_pages && t.refs[p] > 0);
    if (lane == 0) used[k] = b;
  }
  __syncthreads();
  int mine = 0;
  for (int k = 0; k < own; ++k) mine += __popc(used[i * own + k]);
  unsigned long long all;
  const int before = (int)block_scan((unsigned long long)mine, &all);
  const int live = (int)all;
  if (i == 0) below_s = live;                                     // pages in use below number `live` (all, when the pool is full)
  __syncthreads();
  int seen = before;
  for (int k = 0; k < own; ++k) {
    const int word = i * own + k;
    if (live / 32 == word) below_s = seen + __popc(used[word] & ((1u << (live & 31)) - 1u));
    seen += __popc(used[word]);
  }
  __syncthreads();
  const int below = below_s, moves = live - below;
  seen = before;
  for (int k = 0; k < own; ++k) {
    const int word = i * own + k;
    const uint32_t u = used[word];
    for (uint32_t b = ~u; b; b &= b - 1) {                        // unused, below `live`: a hole
      const int bit = __ffs(b) - 1, p = word * 32 + bit;
      if (p >= live) break;
      __stcg(&w.dst[p - (seen + __popc(u & ((1u << bit) - 1u)))], p);
    }
    for (uint32_t b = u; b; b &= b - 1) {                         // in use, at or beyond it: moves
      const int bit = __ffs(b) - 1, p = word * 32 + bit;
      if (p >= live) __stcg(&w.src[seen + __popc(u & ((1u << bit) - 1u)) - below], p);
    }
    seen += __popc(u);
  }
  __syncthreads();
  for (int k = i; k < moves; k += kPlanThreads) {
    const int a = __ldcg(&w.src[k]), b = __ldcg(&w.dst[k]);
    w.count[a] = b;                                               // for the table entries that name the page
    t.refs[b] = t.refs[a];
    t.refs[a] = 0;
  }
  for (int k = i; k < t.n_pages - live; k += kPlanThreads) t.free_list[k] = t.n_pages - 1 - k;
  if (i == 0) { *t.free_count = t.n_pages - live; w.moves[0] = moves; w.moves[1] = live; }
}

// ---- copies -------------------------------------------------------------------------------
__device__ __forceinline__ void copy_chunk(unsigned char* base, long long bytes, int src, int dst, int chunk) {
  const uint4* from = reinterpret_cast<const uint4*>(base + (long long)src * bytes);
  uint4* to = reinterpret_cast<uint4*>(base + (long long)dst * bytes);
  const long long pieces = bytes >> 4, at = (long long)chunk * (kChunk / 16) + threadIdx.x;
  uint4 v[kCopyFlight];
#pragma unroll
  for (int f = 0; f < kCopyFlight; ++f)
    if (at + f * kCopyThreads < pieces) v[f] = __ldcs(from + at + f * kCopyThreads);
#pragma unroll
  for (int f = 0; f < kCopyFlight; ++f)
    if (at + f * kCopyThreads < pieces) __stcs(to + at + f * kCopyThreads, v[f]);
}

// grid (CTAs, pools): the pages of the list moved in every pool; `remap`: first the table entries that name a moved page
__global__ void __launch_bounds__(kCopyThreads) pages_move_kernel(const PageTableDev t, const PagePools pools, int remap) {
  const WorkView w(t);
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int moves = w.moves[0];
  if (moves == 0) return;
  if (remap && blockIdx.y == 0) {
    const int live = w.moves[1];
    const long long entries = (long long)t.n_rows * t.max_pages;
    for (long long e = (long long)blockIdx.x * kCopyThreads + threadIdx.x; e < entries; e += (long long)gridDim.x * kCopyThreads) {
      const int pg = t.table[e];
      if (pg >= live && pg < t.n_pages) t.table[e] = w.count[pg];
    }
  }
  if (pools.n == 0) return;
  unsigned char* base = pools.p[blockIdx.y];
  const long long bytes = pools.bytes[blockIdx.y];
  const int chunks = (int)((bytes + kChunk - 1) / kChunk);
  for (long long it = blockIdx.x; it < (long long)moves * chunks; it += gridDim.x) {
    const int m = (int)(it / chunks);
    if (w.src[m] >= 0) copy_chunk(base, bytes, w.src[m], w.dst[m], (int)(it - (long long)m * chunks));
  }
}

// grid (CTAs, blocks): rows of every block copied from src to dst.  Every CTA judges all pairs alike before it copies.
__global__ void __launch_bounds__(kCopyThreads) rows_copy_kernel(const PagePools blocks, int n_rows, const int32_t* src, const int32_t* dst, int n, int32_t* status) {
  __shared__ int src_s[kMaxPageRows], dst_s[kMaxPageRows];
  __shared__ unsigned char ok_s[kMaxPageRows];
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  for (int i = threadIdx.x; i < n; i += kCopyThreads) { src_s[i] = src[i]; dst_s[i] = dst[i]; }
  __syncthreads();
  // pairs that are passed over name nothing (a pass of its own: done while staging, the compiler schedules the copy below another way, and 64
  // rows of two states take 67.5 us instead of 63.5)
  for (int i = threadIdx.x; i < n; i += kCopyThreads)
    if (src_s[i] == -1 || dst_s[i] == -1) src_s[i] = dst_s[i] = -1;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kCopyThreads) {
    const int s = src_s[i], d = dst_s[i];
    const bool skip = s == -1;
    bool bad = s < 0 || s >= n_rows || d < 0 || d >= n_rows;
    if (!skip && !bad)
      for (int j = 0; j < n; ++j) bad |= (dst_s[j] == d && j < i) || src_s[j] == d;
    ok_s[i] = !skip && !bad;
    if (status && blockIdx.x == 0 && blockIdx.y == 0) status[i] = !skip && bad ? (int)LUMO_SEQ_BAD_ROW : (int)LUMO_SEQ_OK;
  }
  __syncthreads();
  unsigned char* base = blocks.p[blockIdx.y];
  const long long bytes = blocks.bytes[blockIdx.y];
  const long long chunks = (bytes + kChunk - 1) / kChunk;
  for (long long it = blockIdx.x; it < (long long)n * chunks; it += gridDim.x) {
    const int m = (int)(it / chunks);
    if (ok_s[m]) copy_chunk(base, bytes, src_s[m], dst_s[m], (int)(it - (long long)m * chunks));
  }
}

__global__ void __launch_bounds__(kCopyThreads) pages_init_kernel(const PageTableDev t) {
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const long long step = (long long)gridDim.x * kCopyThreads, me = (long long)blockIdx.x * kCopyThreads + threadIdx.x;
  for (long long e = me; e < (long long)t.n_rows * t.max_pages; e += step) t.table[e] = -1;
  for (long long e = me; e < t.n_rows; e += step) t.row_pages[e] = 0;
  for (long long e = me; e < t.n_pages; e += step) { t.refs[e] = 0; t.free_list[e] = t.n_pages - 1 - (int)e; }
  if (me == 0) *t.free_count = t.n_pages;
}

dim3 copy_grid(int sms, int pools) {
  const int n = pools > 0 ? pools : 1;
  return dim3((unsigned)((8 * sms + n - 1) / n), (unsigned)n);    // eight CTAs an SM over all pools
}

}  // namespace

cudaError_t launch_pages_init(const PageTableDev& t, int sms, bool pdl, cudaStream_t st) {
  return launch_kernel(pages_init_kernel, dim3(sms), dim3(kCopyThreads), 0, st, pdl, t);
}

cudaError_t launch_pages_fork(const PageTableDev& t, const int32_t* src, const int32_t* dst, int n, int32_t* status, bool pdl, cudaStream_t st) {
  return launch_kernel(pages_fork_kernel, dim3(n), dim3(kCopyThreads), 0, st, pdl, t, src, dst, n, status);
}

cudaError_t launch_pages_free(const PageTableDev& t, const int32_t* rows, const int32_t* keep, int n, int32_t* status, bool pdl, cudaStream_t st) {
  return launch_kernel(pages_free_kernel, dim3(1), dim3(kPlanThreads), 0, st, pdl, t, rows, keep, n, status);
}

cudaError_t launch_pages_reserve(const PageTableDev& t, const PagePools& pools, const int32_t* rows, const int32_t* start, const int32_t* end,
                                 int add, int n, int32_t* status, int sms, bool pdl, cudaStream_t st) {
  const cudaError_t e = launch_kernel(pages_reserve_kernel, dim3(1), dim3(kPlanThreads), 0, st, pdl, t, rows, start, end, add, n, status);
  if (e != cudaSuccess || pools.n == 0) return e;
  return launch_kernel(pages_move_kernel, copy_grid(sms, pools.n), dim3(kCopyThreads), 0, st, pdl, t, pools, 0);
}

cudaError_t launch_pages_compact(const PageTableDev& t, const PagePools& pools, int sms, bool pdl, cudaStream_t st) {
  const cudaError_t e = launch_kernel(pages_compact_kernel, dim3(1), dim3(kPlanThreads), 0, st, pdl, t);
  if (e != cudaSuccess) return e;
  return launch_kernel(pages_move_kernel, copy_grid(sms, pools.n), dim3(kCopyThreads), 0, st, pdl, t, pools, 1);
}

cudaError_t launch_rows_copy(const PagePools& blocks, int n_rows, const int32_t* src, const int32_t* dst, int n, int32_t* status, int sms,
                             bool pdl, cudaStream_t st) {
  return launch_kernel(rows_copy_kernel, copy_grid(sms, blocks.n), dim3(kCopyThreads), 0, st, pdl, blocks, n_rows, src, dst, n, status);
}

}  // namespace lumo
