// What the two forms of the attention over the paged 4-bit cache share: waits, staging of a tile, the work decomposition.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "internal.h"
#include "kv4.h"

namespace lumo {

#ifdef __CUDACC__
namespace {      // (one copy per source file that includes this)

constexpr int kDh = 128;
constexpr int kKeys = 128;            // keys per tile
constexpr int kTileBytes = kKeys * 2 * kKv4Entry;   // 18432: keys and values, codes and scales
constexpr int kSeqCache = 64;         // sequences whose context length, cache row and tile count are kept in shared memory
constexpr float kLag = 8.f;           // the reference maximum moves when exceeded by more than this (log2 units)
constexpr float kLift = 6.f;          // probabilities are held as 2^kLift times themselves: at most 2^14 in f16, and what f16 drops is below 2^-30
constexpr uint32_t kSpinLimit = 1u << 22, kSpinLimitDrill = 1u << 10;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(unsigned long long* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(unsigned long long* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(unsigned long long* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
// Bounded wait: false if the phase did not complete within `limit` polls.
__device__ __forceinline__ bool mbar_wait(unsigned long long* bar, uint32_t parity, uint32_t limit) {
  const uint32_t addr = smem_u32(bar);
  for (uint32_t spin = 0; spin < limit; ++spin) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(done) : "r"(addr), "r"(parity) : "memory");
    if (done) return true;
  }
  return false;
}
// untiled bulk copy into shared memory: both addresses 16-byte aligned, a multiple of 16 bytes; completion counted on `bar`
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, unsigned long long* bar, uint64_t policy) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;\n"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)), "l"(policy) : "memory");
}
__device__ __forceinline__ uint64_t l2_evict_first_policy() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;\n" : "=l"(p));
  return p;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// (base-2 log-sum-exp of a row from its reference maximum and lifted sum; a NaN stays one, a row without keys gives -inf)
__device__ __forceinline__ float row_lse2(float m, float l) { return l == 0.f ? -INFINITY : m - kLift + log2f(l); }
__device__ __forceinline__ float row_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }

// The power of two that takes a query row to f16: its largest magnitude becomes 2^14 to 2^15 (less for a row below 2^-46, whose logits are
// zero to fp32; without a bound the way back could underflow).  `top`: that magnitude's bits.
__device__ __forceinline__ int query_exponent(uint32_t top) {
  const int e = (int)(top >> 23) - 127;
  return min(14 - e, 60);
}

// ---- work decomposition ----------------------------------------------------------------
// Units are numbered u = (b * Hkv + hkv) * RT + rt; unit u owns nt(b) tiles (0 for a sequence that fails its check).  Automatic mode: the
// units are laid end to end on a line, each preceded by `cost` idle positions (the price of starting it, in tiles); CTA c owns the
// positions [c * per, (c + 1) * per), works on the tiles among them, and the slot of a segment is u + c (strictly increasing along the line,
// so unique).  Fixed mode (S partitions): CTA c owns partition c mod S of unit c / S, slot c.
struct Segment {
  int b, hkv, rt;     // unit
  int t0, n;          // first tile within the unit, tile count (n = 0 possible in fixed mode)
  int slot;
  int unit, slot0, nslots;   // the unit, and the slots all its segments write (ascending along the key range)
  int ctx, crow;
};
struct WorkState {
  int b, q;           // current sequence, unit within the sequence
  int g, g_end;       // next position on the line, end of this CTA's share (the host bounds the line: kv4_line)
  int g_unit;         // position at which the current unit's stretch (idle prefix, then its tiles) starts
  int nt;             // tiles per unit of the current sequence
  int per;            // automatic mode: positions per CTA
  int parts;          // partitions per unit when CTA c owns partition c mod parts of unit c / parts; 0: shares of the line
  bool fixed_done;
};
// in shared memory: the first sequences, and what one warp has found out for all roles
struct SeqCache {
  int ctx[kSeqCache], row[kSeqCache], nt[kSeqCache];
  WorkState work;     // behind the first segment
  Segment first;
  bool any;           // whether there is a first segment
};

__device__ __forceinline__ int seq_tiles(const Kv4AttnArgs& a, int cx, int cr) {
  return seq_check(cx, cr, a.Ns, a.n_rows, a.max_pos) == LUMO_SEQ_OK ? (cx + a.Ns + kKeys - 1) / kKeys : 0;
}

template <int kCost, int kMinTiles, int kSlack>
struct Work : WorkState {
  static constexpr int kSegmentCost = kCost;
  const Kv4AttnArgs& a;
  const SeqCache& sc;
  bool fresh = true;

  __device__ __forceinline__ int tiles_of(int bb, int* ctx, int* crow) const {
    if (bb < kSeqCache) { *ctx = sc.ctx[bb]; *crow = sc.row[bb]; return sc.nt[bb]; }
    *ctx = a.ctx_len[bb];
    *crow = a.cache_row[bb];
    return seq_tiles(a, *ctx, *crow);
  }

  __device__ __forceinline__ Work(const Kv4AttnArgs& args, const SeqCache& cache) : WorkState(cache.work), a(args), sc(cache) {}

  // Run by one warp, before the roles part: fills the cache, finds the CTA's share, a lane a sequence, and the share's first segment.  (By
  // every warp for itself, sequence after sequence, this took 1700 cycles of each CTA's start; a copy of it takes a few dozen.)
  static __device__ __forceinline__ void set_up(const Kv4AttnArgs& a, SeqCache& sc) {
    const int lane = threadIdx.x & 31;
    const int upb = a.Hkv * a.RT;       // units per sequence
    int total = 0, most = 0, cx, cr;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const int bb = b0 + lane;
      int n = 0;
      if (bb < a.B) {
        cx = a.ctx_len[bb];
        cr = a.cache_row[bb];
        n = seq_tiles(a, cx, cr);
        if (bb < kSeqCache) { sc.ctx[bb] = cx; sc.row[bb] = cr; sc.nt[bb] = n; }
      }
      total += n > 0 ? (n + kCost) * upb : 0;
      most = max(most, n);
    }
    total = __reduce_add_sync(0xffffffffu, total);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) sc.work = {0, 0, 0, 0, 0, 0, 1, a.S, false};
    __syncwarp();
    Work w(a, sc);
    if (w.parts == 0) {
      w.per = (total + (int)gridDim.x - 1) / (int)gridDim.x;
      // Short contexts: when there is a CTA for every unit and no unit is much longer than an even share, units stay whole: nothing
      // is cut, and with one segment per unit the outputs are final when they leave this kernel.
      if (a.B * upb <= (int)gridDim.x && most <= w.per + kSlack) w.parts = 1;
    }
    if (w.parts == 0) {
      if (w.per < kMinTiles) w.per = kMinTiles;
      w.g = (int)blockIdx.x * w.per;
      w.g_end = w.g + w.per < total ? w.g + w.per : total;
      int acc = 0;                      // the sequence whose units hold position g, and where they start
      w.b = a.B;
      for (int b0 = 0; b0 < a.B && w.g < w.g_end; b0 += 32) {
        const int n = b0 + lane < a.B ? w.tiles_of(b0 + lane, &cx, &cr) : 0;
        const int span = n > 0 ? (n + kCost) * upb : 0;
        int upto = span;
#pragma unroll 1
        for (int d = 1; d < 32; d *= 2) {
          const int x = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += x;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, w.g < acc + upto);
        if (hit) {
          const int at = __ffs(hit) - 1;
          acc += __shfl_sync(0xffffffffu, upto - span, at);
          w.nt = __shfl_sync(0xffffffffu, n, at);
          w.b = b0 + at;
          w.q = (w.g - acc) / (w.nt + kCost);
          w.g_unit = acc + w.q * (w.nt + kCost);
          break;
        }
        acc += __shfl_sync(0xffffffffu, upto, 31);
      }
    }
    Segment sg = {};
    const bool any = w.advance(&sg);
    if (lane == 0) { sc.work = w; sc.first = sg; sc.any = any; }
  }

  // next segment of this CTA; false when the share is exhausted
  __device__ __forceinline__ bool next(Segment* s) {
    if (fresh) {
      fresh = false;
      *s = sc.first;
      return sc.any;
    }
    return advance(s);
  }

  __device__ __forceinline__ bool advance(Segment* s) {
    const int upb = a.Hkv * a.RT;
    if (parts > 0) {
      if (fixed_done) return false;
      fixed_done = true;
      const int u = blockIdx.x / parts, part = blockIdx.x - u * parts;
      s->b = u / upb;
      if (s->b >= a.B) return false;
      const int r = u - s->b * upb;
      s->hkv = r / a.RT; s->rt = r - s->hkv * a.RT;
      const int n_all = tiles_of(s->b, &s->ctx, &s->crow);
      s->t0 = (int)(((long long)part * n_all) / parts);
      s->n = (int)(((long long)(part + 1) * n_all) / parts) - s->t0;
      s->slot = blockIdx.x;
      s->unit = u; s->slot0 = u * parts; s->nslots = parts;
      return n_all > 0;
    }
    while (g < g_end && b < a.B) {
      if (nt == 0 || g >= g_unit + nt + kCost) {         // move to the next unit (skipping sequences without tiles)
        if (nt > 0) g_unit += nt + kCost;
        if (nt == 0 || ++q == upb) {
          q = 0;
          int cx, cr;
          do { ++b; nt = b < a.B ? tiles_of(b, &cx, &cr) : 0; } while (b < a.B && nt == 0);
        }
        continue;
      }
      const int first = g_unit + kCost;                  // position of the unit's tile 0
      const int lo = g > first ? g : first;
      const int hi = first + nt < g_end ? first + nt : g_end;
      g = g_unit + nt + kCost < g_end ? g_unit + nt + kCost : g_end;
      if (lo >= hi) continue;                            // only idle positions of this unit fall into the share
      const int u = b * upb + q;
      s->b = b; s->hkv = a.RT == 1 ? q : q / a.RT; s->rt = q - s->hkv * a.RT;
      tiles_of(b, &s->ctx, &s->crow);
      s->t0 = lo - first;
      s->n = hi - lo;
      s->slot = u + blockIdx.x;
      s->unit = u;
      const int c0 = first / per;
      s->slot0 = u + c0;
      s->nslots = (first + nt - 1) / per - c0 + 1;
      return true;
    }
    return false;
  }
};

// The page numbers that a loading warp needs for a segment, a lane a page of the tile, asked for a tile ahead.
struct PageWalk {
  const int32_t* entries;
  int n, per_tile, left, next;        // tiles, pages a tile; pages of the segment's row from its first one on; the number on its way
  __device__ __forceinline__ PageWalk(const Kv4AttnArgs& a, const Segment& sg) {
    const int lane = threadIdx.x & 31, first = (sg.t0 * kKeys) >> a.page_log2;
    entries = a.table + (size_t)sg.crow * a.max_pages + first + lane;
    n = sg.n;
    per_tile = kKeys >> a.page_log2;
    left = ((sg.ctx + a.Ns + (1 << a.page_log2) - 1) >> a.page_log2) - first - lane;
    next = wanted(0) ? __ldg(entries) : -1;
  }
  // whether this lane has a page of tile j that holds positions below ctx + Ns
  __device__ __forceinline__ bool wanted(int j) const { return (int)(threadIdx.x & 31) < per_tile && j < n && j * per_tile < left; }
  __device__ __forceinline__ int take(int j) {
    const int pg = next;
    next = wanted(j + 1) ? __ldg(entries + (j + 1) * per_tile) : -1;
    return pg;
  }
};

// Stages one tile, or its keys (which = 0) or values (1) alone: a bulk copy per page.  A page number out of range sets *bad_page, and nothing
// is copied for it.
template <bool kBoth>
__device__ __forceinline__ void load_tile(const Kv4AttnArgs& a, const Segment& sg, bool wanted, int pg, int which, uint32_t dst, unsigned long long* full,
                                          uint32_t* bad_page, uint64_t policy) {
  const int lane = threadIdx.x & 31, page = 1 << a.page_log2;
  const bool good = wanted && pg >= 0 && pg < a.n_pages;
  const uint32_t bytes = page * (kBoth ? 2 : 1) * kKv4Entry;
  const unsigned loads = __ballot_sync(0xffffffffu, good);
  const bool bad = __any_sync(0xffffffffu, wanted && !good);
  if (lane == 0) {
    if (bad) *reinterpret_cast<volatile uint32_t*>(bad_page) = 1;
    mbar_expect_tx(full, __popc(loads) * bytes);
  }
  __syncwarp();
  if (good) bulk_load(dst + lane * bytes, a.pages + kv4_block(a.Hkv, page, pg, sg.hkv, which), bytes, full, policy);
}

__device__ __forceinline__ bool slot_seen(const uint32_t* row, int s) {        // s: suffix slot; below 0: context
  return s < 0 || (s < kMaxAttnSlots && ((__ldg(row + (s >> 5)) >> (s & 31)) & 1u));
}

}  // namespace
#endif

}  // namespace lumo
