// Attention over the paged 4-bit cache on tcgen05, for units of more than sixteen query rows (sm_100a); kv4_attn.cu says what is computed
// and how the work is dealt out.  A persistent CTA per SM; the query rows of all heads that share the KV head sit in one 128-row tile
// (row = head-in-group * N + node).
//
//   warps 0-7    softmax: two groups of four warps take the tiles in turn, a thread a query row (= tensor-memory lane) of 128 keys, so that on
//                every scheduler one warp looks for its tile's maxima while the other keeps the exponentials' unit busy.  A thread applies
//                visibility by selection, exponentiates against the row's REFERENCE maximum (shared by the groups; it moves, with a
//                rescale of the accumulator, only when exceeded by more than 2^kLag) and stores the probabilities as f16 over logits that
//                it has read: the A operand of the second product, where it lies
//   warps 8-15   codes to operands, four warps for the keys and four for the values: 32 codes and two scales at a time from the staged
//                page blocks to f16 in shared memory ([128 keys x 128 bytes] per half of the head, 128-byte swizzle; two buffers each)
//   warps 16, 17 loaders: bulk copies of a head's page blocks into two rings of three tiles, one of keys and one of values (the values
//                are used two tiles later)
//   warps 18, 19 issuers: S = Q K^T into one of three S buffers (up to two tiles ahead of the probabilities, so that a group finds its next
//                logits ready), and O += P V into an accumulator that stays in tensor memory for the whole segment.  The tensor core takes
//                few instructions ahead, and a wait costs its issuer 150 cycles or more even when nothing is awaited (measured): so there
//                are two, each with one commit and a wait or two a tile, and one issues while the other waits.  Q lies in shared memory: the
//                tensor core reads it from there at the same rate (1024 cycles for both products either way, measured)
//
// What bounds it: a tile takes an SM 1850 cycles once all warps are at work (8 x 28 nodes at 16k; counters by the profiler).  In them the two
// products take 1024, the exponentials 1024 on their units, the arithmetic units 1010 (half of it codes to f16 and back to pairs), and
// each scheduler issues 1390 instructions: no unit is full, but five warps a scheduler find something to issue in three cycles of four at
// best.  The cache's bytes, 18 KB a tile, need 800 cycles of the SM's share of the memory.  Around the tiles a CTA spends 10 thousand cycles
// until its first logits (lengths, page numbers, first copies and first instructions, one after another) and 4 to 6 thousand on the
// read-out.  Measured, with the merge: 4 x 8 nodes at 8k 26.5 to 28 us, 8 x 28 at 16k 71 to 77 us (615 to 665 TFLOP/s, at the power limit's
// edge; 66 in a short run), 64 nodes at 128k 161 to 164 us (840 to 855 TFLOP/s, at 1.64 GHz under the power limit).
#include "f32x2.h"
#include "kv4_attn.h"

namespace lumo {

namespace {

constexpr int kRows = 128;            // query rows per unit = tensor-memory lanes
constexpr int kSoftmaxWarps = 8, kGroupWarps = 4;     // four warps: one softmax group, the keys' or the values' conversion
constexpr int kLoadWarp = kSoftmaxWarps + 2 * kGroupWarps, kIssueWarp = kLoadWarp + 2;   // two of each
constexpr int kThreads = 32 * (kIssueWarp + 2);
constexpr int kStages = 3;            // staged tiles per ring
constexpr int kRawBytes = kKeys * kKv4Entry;            // 9216
constexpr int kBufs = 3;              // S buffers
constexpr int kTmemCols = 512;        // S buffers (and P in them): 0..383; O: 384..511
constexpr int kColO = kBufs * kKeys;
constexpr int kHalfBytes = 16384;     // one dh half of an operand tile: [128 keys x 128 B]
constexpr int kOpBytes = 2 * kHalfBytes;
constexpr int kOffK = 0;              // two K tiles, two V tiles, Q, the ring
constexpr int kOffV = 2 * kOpBytes;
constexpr int kOffQ = 4 * kOpBytes;
constexpr int kOffRaw = 5 * kOpBytes;
constexpr int kOffCtl = kOffRaw + 2 * kStages * kRawBytes;
struct Ctl {
  unsigned long long raw_full[2][kStages], raw_empty[2][kStages];   // [keys, values]
  unsigned long long k_full[2];
  unsigned long long s_full[kBufs];   // logits complete (and the K tile read)
  unsigned long long pv_full[kBufs];  // probabilities and values complete
  // Product of P and V complete.  One per S buffer: whoever waits for tile t's here is itself needed for tile t + 3's, so no phase is missed
  // (with two, the issuer of tile t's logits could come after tile t - 1's product, two phases late, and wait for ever).
  unsigned long long o_done[kBufs];
  unsigned long long v_full[kBufs];   // values (and nan_blocks) written, for softmax threads; three for the same reason
  unsigned long long q_full, o_free, drain[2];
  uint32_t tmem_base;
  uint32_t timed_out;
  uint32_t bad_page[2][16];           // [keys' loader, values' loader], by segment number mod 16: the loader is never that far ahead
  SeqCache seq;
  float ref[kRows];                   // the rows' reference maxima
  float xchg[2][kRows];               // [group][row]: what the two threads of a row tell one another
  uint32_t nan_blocks[2][kRows / 4];  // [V buffer][key], a byte each: blocks of values that are NaN in a suffix position
};
constexpr int kSmemBytes = kOffCtl + (int)sizeof(Ctl);
static_assert(kSmemBytes + 1024 <= 227 * 1024, "one CTA per SM");
// A segment's start and end cost about as much as eight tiles.  Charged 4, 8, 12, us, in one short run: 8 x 28 nodes at 16k 67.4, 66.4, 68.1; 4
// x 8 at 8k 28.8, 27.4, 28.4; 3 x 20 at 5k 21.8, 22.1, 22.7; 12 x 16 at 16k 88.0, 88.2, 90.9; 2 x 64 at 40k 77.8, 76.2, 76.9.
using TcWork = Work<8, 4, 4>;

__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
// shared-memory matrix descriptor, 128-byte swizzle
__device__ __forceinline__ uint64_t umma_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFF) >> 4);
  d |= (uint64_t)(lbo >> 4) << 16;
  d |= (uint64_t)(sbo >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// instruction descriptor: f16 x f16 -> fp32; b_mn = 1 when B is MN-major
__host__ __device__ constexpr uint32_t umma_idesc(int M, int N, int b_mn) {
  return (1u << 4) | ((uint32_t)b_mn << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// product with the A operand in tensor memory (row = lane, two f16 per 32-bit column, K-major)
__device__ __forceinline__ void umma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// product with both operands in shared memory
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
      ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_commit(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void pair_sync(int bar) { asm volatile("barrier.cta.sync %0, 64;\n" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void pair_arrive(int bar) { asm volatile("barrier.cta.arrive %0, 64;\n" ::"r"(bar) : "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Visibility of 64 consecutive keys from suffix slot s0 on (negative: keys of the committed context, always visible), from a
// node's 256-bit row over the suffix.
__device__ __forceinline__ unsigned long long visible64(const uint32_t* row, int s0) {
  if (s0 >= kMaxAttnSlots) return 0ull;
  const int w = s0 > 0 ? s0 >> 5 : 0, off = s0 > 0 ? s0 & 31 : 0;
  unsigned long long v = __ldg(row + w);
  if (w + 1 < 8) v |= (unsigned long long)__ldg(row + w + 1) << 32;
  if (off) {
    v >>= off;
    if (w + 2 < 8) v |= (unsigned long long)__ldg(row + w + 2) << (64 - off);
  }
  if (s0 < 0) v = s0 <= -64 ? ~0ull : v << -s0 | ((1ull << -s0) - 1ull);
  return v;
}

template <bool kDrill>
__global__ void __launch_bounds__(kThreads, 1) kv4_attn_tc_kernel(const Kv4AttnArgs a) {
  auto wait = [](unsigned long long* bar, uint32_t parity) { return mbar_wait(bar, parity, kDrill ? kSpinLimitDrill : kSpinLimit); };
  extern __shared__ __align__(1024) unsigned char smem[];
  Ctl& sm = *reinterpret_cast<Ctl*>(smem + kOffCtl);
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  bool ok = (sbase & 1023u) == 0;     // cannot fail with this file's layout; refuse rather than mis-swizzle

  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&sm.tmem_base)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  if (tid == 0) {
    for (int s = 0; s < 2 * kStages; ++s) { mbar_init(&sm.raw_full[0][s], 1); mbar_init(&sm.raw_empty[0][s], kGroupWarps); }
    for (int s = 0; s < 2; ++s) mbar_init(&sm.k_full[s], kGroupWarps);
    for (int s = 0; s < kBufs; ++s) {
      mbar_init(&sm.s_full[s], 1); mbar_init(&sm.pv_full[s], 2 * kGroupWarps);
      mbar_init(&sm.o_done[s], 1); mbar_init(&sm.v_full[s], kGroupWarps);
    }
    mbar_init(&sm.q_full, kSoftmaxWarps);
    mbar_init(&sm.o_free, kSoftmaxWarps);
    mbar_init(&sm.drain[0], 1);
    mbar_init(&sm.drain[1], 1);
    sm.timed_out = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (tid < 32) sm.bad_page[0][tid] = 0;
  // The set-up above touches nothing of earlier kernels; everything below may.
  pdl_wait();
  pdl_trigger();
  if (warp == 0) TcWork::set_up(a, sm.seq);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;

  TcWork work(a, sm.seq);
  Segment sg;
  uint32_t it = 0;        // tiles this CTA has started, over all segments: ring stage, buffers and phases
  uint32_t nseg = 0;      // segments with tiles so far: phases of q_full and o_free

  if (warp == kLoadWarp || warp == kLoadWarp + 1) {
    // ---------------- loaders: keys (which = 0) and values (1), a lane a page ----------------
    const uint64_t policy = l2_evict_first_policy();
    const int which = warp - kLoadWarp;
    while (work.next(&sg)) {
      PageWalk walk(a, sg);
      for (int j = 0; j < sg.n; ++j, ++it) {
        const uint32_t st = it % kStages, use = it / kStages;
        const bool wanted = walk.wanted(j);
        const int pg = walk.take(j);
        if (use > 0 && ok) ok = wait(&sm.raw_empty[which][st], (use - 1) & 1u);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (j == 0 && lane == 0) sm.bad_page[which][nseg & 15u] = 0;
        if (!kDrill) load_tile<false>(a, sg, wanted, pg, which, sbase + kOffRaw + (which * kStages + st) * kRawBytes, &sm.raw_full[which][st],
                         &sm.bad_page[which][nseg & 15u], policy);
      }
      if (!ok) break;
      if (sg.n > 0) ++nseg;
    }
    // no copy may be on its way when the CTA leaves: the last use of every stage (complete already unless a wait ran out)
    for (uint32_t s = 0; s < kStages && s < it; ++s) wait(&sm.raw_full[which][s], ((it - 1 - s) / kStages) & 1u);
    if (!ok && lane == 0) sm.timed_out = 1u;
  } else if (warp == kIssueWarp) {
    // ---------------- issuer of S = Q K^T: both K-major, 128 rows of 128 B per dh half ----------------
    // (whole warps run these loops, and one lane issues; all lanes take part in electing it, also when a wait has run out for some)
    constexpr uint32_t id = umma_idesc(kRows, kKeys, 0);
    const uint64_t dq = umma_desc(sbase + kOffQ, 16, 1024), dk = umma_desc(sbase + kOffK, 16, 1024);
    while (work.next(&sg)) {
      if (sg.n == 0) continue;
      if (ok) ok = wait(&sm.q_full, nseg & 1u);
      for (int j = 0; j < sg.n; ++j, ++it) {
        if (ok) ok = wait(&sm.k_full[it & 1u], (it >> 1) & 1u);
        // tile t's S buffer is free when tile t - 3's probabilities have been used
        if (it >= kBufs && ok) ok = wait(&sm.o_done[it % kBufs], (it / kBufs - 1) & 1u);
        tc_fence_after();
        const uint64_t kd = dk + (it & 1u) * (kOpBytes >> 4);
        const uint32_t d = tmem + (it % kBufs) * kKeys;
        if (elect_one() && ok && !kDrill) {
#pragma unroll
          for (int ks = 0; ks < kDh / 16; ++ks) {
            constexpr int half16 = kHalfBytes >> 4;
            umma_ss(d, dq + (ks >> 2) * half16 + (ks & 3) * 2, kd + (ks >> 2) * half16 + (ks & 3) * 2, id, ks ? 1u : 0u);
          }
          umma_commit(&sm.s_full[it % kBufs]);
        }
        __syncwarp();
      }
      ++nseg;
    }
    if (!ok) sm.timed_out = 1u;
  } else if (warp == kIssueWarp + 1) {
    // ---------------- issuer of O += P V ----------------
    // A = P in the first half of its S buffer, B = V tile (MN-major: 128 B of dh per key row, the two dh halves kHalfBytes apart, 16 keys =
    // 2048 B per K step)
    constexpr uint32_t id = umma_idesc(kRows, kDh, 1);
    const uint64_t dv = umma_desc(sbase + kOffV, kHalfBytes, 1024);
    while (work.next(&sg)) {
      if (sg.n == 0) continue;
      for (int j = 0; j < sg.n; ++j, ++it) {
        if (j == 0 && nseg > 0 && ok) ok = wait(&sm.o_free, (nseg - 1) & 1u);
        if (ok) ok = wait(&sm.pv_full[it % kBufs], (it / kBufs) & 1u);
        tc_fence_after();
        const uint64_t vd = dv + (it & 1u) * (kOpBytes >> 4);
        const uint32_t p = tmem + (it % kBufs) * kKeys;
        if (elect_one() && ok && !kDrill) {
#pragma unroll
          for (int ks = 0; ks < kKeys / 16; ++ks) umma_ta(tmem + kColO, p + ks * 8, vd + ks * (2048 >> 4), id, (j == 0 && ks == 0) ? 0u : 1u);
          umma_commit(&sm.o_done[it % kBufs]);
        }
        __syncwarp();
      }
      ++nseg;
    }
    if (!ok) sm.timed_out = 1u;
  } else if (warp >= kSoftmaxWarps) {
    // ---------------- codes to operands: keys (which = 0) or values (1) ----------------
    const int which = (warp - kSoftmaxWarps) >> 2, w = warp & 3;
    const int page = 1 << a.page_log2;
    // Lane (r, ch): codes [32 ch, 32 ch + 32) of a key, that is blocks 2 ch and 2 ch + 1.  Eight lanes (two keys, all of their codes) read 128
    // contiguous bytes; the lanes of the head's second half take the key two further, so that the eight write eight different 16-byte columns.
    const int ch = lane & 3, kr = (lane >> 2) ^ (ch & 2);
    while (work.next(&sg)) {
      const uint32_t* usedw = a.used + (size_t)sg.b * 8;
      for (int j = 0; j < sg.n; ++j, ++it) {
        const uint32_t st = it % kStages, buf = it & 1u;
        const int pos0 = (sg.t0 + j) * kKeys;
        const bool tail = pos0 + kKeys > sg.ctx;         // uniform: the tile reaches past the committed context
        const unsigned char* raw = smem + kOffRaw + (which * kStages + st) * kRawBytes;
        if (ok) ok = wait(&sm.raw_full[which][st], (it / kStages) & 1u);
        ok = __all_sync(0xffffffffu, ok);                // (what follows shuffles: all lanes or none)
        uint4 code[4];
        uint32_t sc[4];
        if (ok) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = w * 32 + i * 8 + kr, pi = key >> a.page_log2, r = key & (page - 1);
            const unsigned char* blk = raw + pi * page * kKv4Entry;
            code[i] = *reinterpret_cast<const uint4*>(blk + r * 64 + ch * 16);
            sc[i] = *reinterpret_cast<const unsigned short*>(blk + page * 64 + r * 8 + ch * 2);
          }
        }
        __syncwarp();
        // (the codes are in registers; whoever gave up keeps the stage: its copies may not have landed, and none go on top)
        if (ok && lane == 0) mbar_arrive(&sm.raw_empty[which][st]);
        // the operand buffer is free when the product two tiles back has read it (that of a K tile is announced by its logits)
        if (it >= 2 && ok) {
          const uint32_t b2 = (it - 2) % kBufs;
          ok = wait(which ? &sm.o_done[b2] : &sm.s_full[b2], ((it - 2) / kBufs) & 1u);
        }
        ok = __all_sync(0xffffffffu, ok);
        if (ok) {
          if (which && tail) {
            // Values nobody reads get a scale of zero (0 x NaN), and so does a NaN that some nodes read: the softmax warps, which know
            // who does, hear of it by a bit per block.
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = w * 32 + i * 8 + kr, slot = pos0 + key - sg.ctx;
              uint32_t bits = 0;
              if (slot >= 0) {
                const bool live = slot < a.Ns && ((__ldg(usedw + (slot >> 5)) >> (slot & 31)) & 1u);
                const bool n0 = (sc[i] & 0x7Fu) == 0x7Fu, n1 = (sc[i] & 0x7F00u) == 0x7F00u;
                if (live) bits = ((uint32_t)n0 | (uint32_t)n1 << 1) << (2 * ch);
                if (!live) sc[i] = 0;
                if (n0) sc[i] &= 0xFF00u;
                if (n1) sc[i] &= 0x00FFu;
              }
              // the key's four lanes: two in this group of four, two in the group of the key two further
              bits |= __shfl_xor_sync(0xffffffffu, bits, 1);
              bits |= __shfl_sync(0xffffffffu, bits, (lane ^ 2) ^ 8);
              if (ch == 0) reinterpret_cast<unsigned char*>(sm.nan_blocks[buf])[key] = (unsigned char)bits;
            }
          }
          unsigned char* op = smem + (which ? kOffV : kOffK) + buf * kOpBytes + (ch >> 1) * kHalfBytes;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = w * 32 + i * 8 + kr;
            const uint32_t s2 = e4m3x2_to_half2(sc[i]), s_lo = __byte_perm(s2, 0, 0x1010), s_hi = __byte_perm(s2, 0, 0x3232);
            const uint32_t words[4] = {code[i].x, code[i].y, code[i].z, code[i].w};
            unsigned char* row = op + key * 128;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t s = k & 2 ? s_hi : s_lo;
              uint32_t h[4];
              e2m1x8_to_half2(words[k], h);
              *reinterpret_cast<uint4*>(row + ((((ch & 1) * 4 + k) ^ (kr & 7)) << 4)) =
                  make_uint4(mul_half2(h[0], s), mul_half2(h[1], s), mul_half2(h[2], s), mul_half2(h[3], s));
            }
          }
          fence_async_proxy();                           // for the tensor core's reads
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(which ? &sm.v_full[it % kBufs] : &sm.k_full[buf]);
          if (which) mbar_arrive(&sm.pv_full[it % kBufs]);
        }
      }
    }
    if (!ok) sm.timed_out = 1u;
  } else {
    // ---------------- softmax ----------------
    // Warps w and w + 4 hold the 32 rows of one lane quarter; group `half` = warp / 4 takes the tiles of that parity, and at a segment's end
    // the output columns [64 half, 64 half + 64).
    const int half = warp >> 2;
    const int row = 32 * (warp & 3) + lane;              // tensor-memory lane this warp may touch
    const uint32_t tmem_lane = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const int pair_bar = 1 + (warp & 3);                 // named barriers of the two warps of a lane quarter: both wait ...
    const int chain_bar = 5 + (warp & 3);                // ... (+ 4 parity) the reference maximum is that of the tile before
    const int GN = a.G * a.N;
    // Query tile of a segment into shared memory: this thread's half of its row in f16 (zeros beyond the group); returns what takes the logits
    // back to log2 units.  The S products of the segment before have all completed by then: each group has awaited its own tiles', and
    // the first barrier below is behind the last tiles of both.
    auto store_q = [&](const Segment& g) {
      const int rgq = g.rt * kRows + row;
      const bool okq = rgq < GN;
      const int hq = okq ? rgq / a.N : 0, nq = okq ? rgq - hq * a.N : 0;
      const uint4* qrow = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + ((size_t)g.b * a.N + nq) * a.q_stride +
                                                         ((size_t)g.hkv * a.G + hq) * kDh);
      uint32_t qr[32], top = 0;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 v = okq ? __ldg(qrow + half * 8 + c) : make_uint4(0u, 0u, 0u, 0u);
        qr[4 * c] = v.x; qr[4 * c + 1] = v.y; qr[4 * c + 2] = v.z; qr[4 * c + 3] = v.w;
      }
#pragma unroll
      for (int c = 0; c < 32; ++c) top = max(top, max((qr[c] << 16) & 0x7FFF0000u, qr[c] & 0x7FFF0000u));
      sm.xchg[half][row] = __uint_as_float(top);
      pair_sync(pair_bar);
      top = max(top, __float_as_uint(sm.xchg[half ^ 1][row]));
      pair_sync(pair_bar);                               // both have read before either writes there again
      const int e = query_exponent(top);
      const float up = exp2i(e);
#pragma unroll
      for (int c = 0; c < 32; ++c) qr[c] = pack_half2(__uint_as_float(qr[c] << 16) * up, __uint_as_float(qr[c] & 0xFFFF0000u) * up);
      unsigned char* qd = smem + kOffQ + half * kHalfBytes + row * 128;
#pragma unroll
      for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(qd + ((c ^ (row & 7)) << 4)) = make_uint4(qr[4 * c], qr[4 * c + 1], qr[4 * c + 2], qr[4 * c + 3]);
      fence_async_proxy();                               // for the tensor core's reads
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full);
      return a.scale_log2 * exp2i(-e);
    };
    Segment sgn;
    bool have = work.next(&sg);
    float mul = 0.f, mul_next = 0.f;
    if (have && sg.n > 0) mul = store_q(sg);
    for (; have; sg = sgn, mul = mul_next) {
      const int rg = sg.rt * kRows + row;
      const bool row_ok = rg < GN;
      const bool warp_ok = sg.rt * kRows + 32 * (warp & 3) < GN;     // some row of this warp is one
      const int hl = row_ok ? rg / a.N : 0, node = row_ok ? rg - hl * a.N : 0;
      float4* slot_o = reinterpret_cast<float4*>(a.part_o + (size_t)sg.slot * kRows * kDh) + (size_t)(half * 16) * kRows + row;
      float* slot_l = a.part_lse + (size_t)sg.slot * kRows + row;
      if (tid == 0) a.unit_slots[sg.unit] = make_int2(sg.slot0, sg.nslots);   // for the merge (same pair from every writer)
      if (sg.n == 0) {                                   // empty partition (fixed mode; a CTA's only segment): an empty slot
        if (row_ok) {
          for (int e = 0; e < 16; ++e) slot_o[(size_t)e * kRows] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (half == 0) *slot_l = -INFINITY;
        }
        have = work.next(&sgn);
        continue;
      }
      const uint32_t* visw = a.vis + ((size_t)sg.b * a.N + node) * 8;
      float m = -INFINITY, l = 0.f;                      // reference maximum (log2 units), this thread's part of the row sum
      uint32_t nan_cols = 0;                             // blocks of the output that a NaN value reaches
      for (int j = 0; j < sg.n; ++j, ++it) {
        const uint32_t buf = it & 1u, sb = it % kBufs;
        if ((int)buf != half) continue;                  // the other group's tile
        const int kpos0 = (sg.t0 + j) * kKeys;
        const bool tail = kpos0 + kKeys > sg.ctx;        // uniform: the tile reaches past the committed context
        if (ok) ok = wait(&sm.s_full[sb], (it / kBufs) & 1u);
        tc_fence_after();
        __syncwarp();
        if (warp_ok) {
          const uint32_t s_col = tmem_lane + sb * kKeys;
          unsigned long long vm[2] = {~0ull, ~0ull};
          if (tail) { vm[0] = visible64(visw, kpos0 - sg.ctx); vm[1] = visible64(visw, kpos0 + 64 - sg.ctx); }
          if (tail) {                                    // a masked logit is replaced before anything is computed with it
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
              uint32_t sr[16];
              tmem_ld16(s_col + c * 16, sr);
              tmem_ld_wait();
              const uint32_t v = (uint32_t)(vm[c >> 2] >> (16 * (c & 3)));
#pragma unroll
              for (int e = 0; e < 16; ++e) sr[e] = ((v >> e) & 1u) ? sr[e] : 0xFF800000u;
              tmem_st16(s_col + c * 16, sr);
            }
            tmem_st_wait();
          }
          // ---- the row's maximum
          float mx2[2] = {-INFINITY, -INFINITY};
          uint32_t sr[2][16];                            // two sets of sixteen logits: one in use, one on its way
          tmem_ld16(s_col, sr[0]);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            tmem_ld_wait();
            if (c < 7) tmem_ld16(s_col + (c + 1) * 16, sr[(c + 1) & 1]);
#pragma unroll
            for (int e = 0; e < 16; e += 2) mx2[(e >> 1) & 1] = max3(mx2[(e >> 1) & 1], __uint_as_float(sr[c & 1][e]), __uint_as_float(sr[c & 1][e + 1]));
          }
          const float mx = fmaxf(mx2[0], mx2[1]) * mul;
          // ---- the reference maximum: that of the tile before, unless this tile exceeds it by more than kLag
          float cur = -INFINITY;
          if (j > 0) {
            pair_sync(chain_bar + 4 * (int)(buf ^ 1u));
            cur = sm.ref[row];
          }
          const float mnew = mx > cur + kLag ? mx : cur;
          if (j + 1 < sg.n) {
            sm.ref[row] = mnew;
            pair_arrive(chain_bar + 4 * (int)buf);
          }
          if (__any_sync(0xffffffffu, mnew != m)) {      // some row's reference is not what this thread's sum goes by
            if (j > 0 && __any_sync(0xffffffffu, mnew != cur && cur != -INFINITY)) {
              // O still takes the product of the tile before: wait for it, then scale this row of it
              const float corr = cur == -INFINITY ? 1.f : ex2(cur - mnew);
              if (ok) ok = wait(&sm.o_done[(it - 1) % kBufs], ((it - 1) / kBufs) & 1u);
              tc_fence_after();
              __syncwarp();
#pragma unroll 1
              for (int c = 0; c < kDh; c += 16) {
                uint32_t orr[16];
                tmem_ld16(tmem_lane + kColO + c, orr);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) orr[e] = __float_as_uint(__uint_as_float(orr[e]) * corr);
                tmem_st16(tmem_lane + kColO + c, orr);
              }
              tmem_st_wait();
            }
            if (m != mnew && m != -INFINITY) l *= ex2(m - mnew);
            m = mnew;
          }
          // ---- probabilities, sixteen keys at a time, the next sixteen logits on their way; over logits that have been read
          const float mu = m == -INFINITY ? 0.f : m - kLift;
          const float2 mulx2 = make_float2(mul, mul), mux2 = make_float2(-mu, -mu);
          float2 ls[2] = {make_float2(l, 0.f), make_float2(0.f, 0.f)};
          tmem_ld16(s_col, sr[0]);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            tmem_ld_wait();
            if (c < 7) tmem_ld16(s_col + (c + 1) * 16, sr[(c + 1) & 1]);
            const uint32_t* x = sr[c & 1];
            uint32_t pk[8];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              const float2 y = fma2(make_float2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), mulx2, mux2);
              const float2 p = make_float2(ex2(y.x), ex2(y.y));
              ls[(e >> 1) & 1] = add2(ls[(e >> 1) & 1], p);
              pk[e >> 1] = pack_half2(p.x, p.y);
            }
            tmem_st8(s_col + c * 8, pk);
          }
          ls[0] = add2(ls[0], ls[1]);
          l = ls[0].x + ls[0].y;
          tmem_st_wait();
          if (tail) {                                    // NaN values among the keys this row sees
            if (ok) ok = wait(&sm.v_full[sb], (it / kBufs) & 1u);
            uint32_t any = 0;
#pragma unroll 4
            for (int c = 0; c < 32; ++c) any |= sm.nan_blocks[buf][c];
            if (any)
              for (int e = 0; e < kKeys; ++e)
                if ((vm[e >> 6] >> (e & 63)) & 1ull) nan_cols |= reinterpret_cast<const unsigned char*>(sm.nan_blocks[buf])[e];
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.pv_full[sb]);
      }
      // end of the segment.  First the next segment's queries (its logits then run under this read-out) ...
      have = work.next(&sgn);
      if (have && sgn.n > 0) mul_next = store_q(sgn);
      // ... then the last O product, the two groups' sums, normalise and write the slot
      const bool last = (int)((it - 1) & 1u) == half;    // this group had the last tile: its reference is the accumulator's
      if (last) sm.ref[row] = m;
      pair_sync(pair_bar);
      // (behind the barrier: the last tile's logits are known to be there, hence the product three tiles before, whose phase this wait
      // would otherwise take for the last one's)
      if (ok) ok = wait(&sm.o_done[(it - 1) % kBufs], ((it - 1) / kBufs) & 1u);
      tc_fence_after();
      __syncwarp();
      // (behind the wait: the last tile has been loaded; both loaders see the same pages)
      const bool bad = *reinterpret_cast<volatile uint32_t*>(&sm.bad_page[0][nseg & 15u]) != 0;
      const float mine = m;
      m = sm.ref[row];
      if (m != mine && mine != -INFINITY) l *= ex2(mine - m);
      sm.xchg[half][row] = l;
      pair_sync(pair_bar);
      const float lt = sm.xchg[0][row] + sm.xchg[1][row];
      pair_sync(pair_bar);
      sm.xchg[half][row] = __uint_as_float(nan_cols);
      pair_sync(pair_bar);
      nan_cols |= __float_as_uint(sm.xchg[half ^ 1][row]);
      const float inv = row_inverse(lt) * a.v_mul;
      const bool whole = sg.nslots == 1;                 // the only segment of its unit: these are the final outputs
      const size_t out_row = (((size_t)sg.b * a.N + node) * a.Hq + (size_t)sg.hkv * a.G + hl);
      if (warp_ok) {
#pragma unroll 1
        for (int c = 0; c < 64; c += 32) {
          uint32_t orr[32];
          tmem_ld32(tmem_lane + kColO + half * 64 + c, orr);
          tmem_ld_wait();
          if (!row_ok) continue;
          const uint32_t nan = nan_cols >> (half * 4 + (c >> 4));
          const float f[2] = {nan & 1u ? __uint_as_float(0x7FC00000u) : inv, nan & 2u ? __uint_as_float(0x7FC00000u) : inv};
#pragma unroll
          for (int e = 0; e < 32; ++e) orr[e] = bad ? 0u : __float_as_uint(__uint_as_float(orr[e]) * f[e >> 4]);
          if (whole && a.out_bf16) {
            uint4* o = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out) + out_row * kDh + half * 64 + c);
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              uint32_t w[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(orr[e + 2 * k]), __uint_as_float(orr[e + 2 * k + 1]));
                w[k] = *reinterpret_cast<const uint32_t*>(&v);
              }
              o[e >> 3] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          } else if (whole) {
            uint4* o = reinterpret_cast<uint4*>(reinterpret_cast<float*>(a.out) + out_row * kDh + half * 64 + c);
#pragma unroll
            for (int e = 0; e < 32; e += 4) o[e >> 2] = make_uint4(orr[e], orr[e + 1], orr[e + 2], orr[e + 3]);
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              slot_o[(size_t)((c + e) >> 2) * kRows] = make_float4(__uint_as_float(orr[e]), __uint_as_float(orr[e + 1]), __uint_as_float(orr[e + 2]),
                                                                   __uint_as_float(orr[e + 3]));
          }
        }
        if (row_ok && half == 0) {
          const float l2 = row_lse2(m == -INFINITY ? 0.f : m, lt);
          if (!whole) *slot_l = bad ? INFINITY : l2;
          else if (a.lse) a.lse[out_row] = bad ? 0.f : l2 * kLn2;
        }
      }
      if (whole && tid == 0) a.part_lse[(size_t)sg.slot * kRows] = bad ? INFINITY : 0.f;
      tc_fence_before();
      pair_sync(pair_bar);                               // the partner has read xchg before the next segment writes it
      if (lane == 0) mbar_arrive(&sm.o_free);
      ++nseg;
    }
    if (!ok) sm.timed_out = 1u;
  }

  tc_fence_before();
  __syncthreads();
  if (sm.timed_out) {                 // products may still run that nobody awaited: they end before tensor memory is freed
    if (warp >= kIssueWarp) {
      if (elect_one()) umma_commit(&sm.drain[warp - kIssueWarp]);
      wait(&sm.drain[warp - kIssueWarp], 0);
    }
    __syncthreads();
  }
  if (tid == 0) a.cta_code[blockIdx.x] = (int)sm.timed_out;      // the merge kernel turns this into status words
  if (warp == kIssueWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

}  // namespace

int kv4_segment_cost_tc() { return TcWork::kSegmentCost; }

template <bool kDrill>
static cudaError_t launch_tc(const Kv4Plan& plan, bool pdl, cudaStream_t st) {
  static bool configured[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < kMaxDevices && !configured[dev]) {
    e = cudaFuncSetAttribute(kv4_attn_tc_kernel<kDrill>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  return launch_kernel(kv4_attn_tc_kernel<kDrill>, dim3(plan.a.C), dim3(kThreads), kSmemBytes, st, pdl, plan.a);
}

cudaError_t launch_kv4_attn_tc(const Kv4Plan& plan, bool pdl, cudaStream_t st) {
  return plan.drill ? launch_tc<true>(plan, pdl, st) : launch_tc<false>(plan, pdl, st);       // (the kernel in use does not carry the test aid)
}

}  // namespace lumo
