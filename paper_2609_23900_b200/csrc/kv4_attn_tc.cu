// Attention over the paged 4-bit cache on tcgen05, for units of more than sixteen query rows (sm_100a); kv4_attn.cu says what is computed
// and how the work is dealt out.  A persistent CTA per SM; the query rows of all heads that share the KV head sit in one 128-row tile
// (row = head-in-group * N + node).
//
//   warps 0-7    softmax: a query row (= tensor-memory lane) is shared by two threads (warps w and w + 4), 64 keys each.  A thread reads its
//                logits, applies visibility by selection, exponentiates against a REFERENCE maximum, which moves (with a rescale of the
//                accumulator) only when exceeded by more than 2^kLag, and stores the probabilities as f16 in the first half of the
//                columns its own logits stood in: that is the A operand of the second product, where it lies
//   warps 8-11   codes to operands: 32 codes and two scales at a time from the staged page blocks to f16 in shared memory, K and V tiles
//                alike ([128 keys x 128 bytes] per half of the head, 128-byte swizzle; two buffers each).  Eight lanes read 128
//                contiguous bytes of codes and write eight different 16-byte columns
//   warp 12      loader: bulk copies of a head's page blocks into a ring of five tiles
//   warp 13      issuer: S = Q K^T into one of two S buffers (one tile ahead of the probabilities), O += P V into an accumulator that
//                stays in tensor memory for the whole segment.  Q and P are A operands in tensor memory
//
// What bounds it: shared memory carries 164 KB a tile (codes written and read, operands written and read by the tensor core), 1312 cycles at
// 128 bytes a cycle; the two products take 1024 cycles, the exponentials 1024 on their own units, and the instructions of the softmax and
// of the conversion about 1100 of the four schedulers.  The cache's bytes, 18 KB a tile, need 800 cycles of the SM's share of the
// memory.
#include "kv4_attn.h"

namespace lumo {

namespace {

constexpr int kRows = 128;            // query rows per unit = tensor-memory lanes
constexpr int kSoftmaxWarps = 8, kConvertWarps = 4;
constexpr int kLoadWarp = kSoftmaxWarps + kConvertWarps, kIssueWarp = kLoadWarp + 1;
constexpr int kThreads = 32 * (kIssueWarp + 1);
constexpr int kStages = 5;            // ring of staged tiles
constexpr int kTmemCols = 512;        // S buffers (and P in them): 0..127, 128..255; O: 256..383; Q (f16 pairs): 384..447
constexpr int kColO = 256;
constexpr int kColQ = 384;
constexpr int kHalfBytes = 16384;     // one dh half of an operand tile: [128 keys x 128 B]
constexpr int kOpBytes = 2 * kHalfBytes;
constexpr int kOffK = 0;              // two K tiles, two V tiles, the ring
constexpr int kOffV = 2 * kOpBytes;
constexpr int kOffRaw = 4 * kOpBytes;
constexpr int kOffCtl = kOffRaw + kStages * kTileBytes;
struct Ctl {
  unsigned long long raw_full[kStages], raw_empty[kStages];
  unsigned long long k_full[2], k_empty[2], v_full[2], v_empty[2];
  unsigned long long s_full[2], p_full[2];
  unsigned long long q_full, o_free, drain;
  uint32_t tmem_base;
  uint32_t timed_out;
  uint32_t bad_page[16];              // by segment number mod 16: the loader is never that far ahead
  SeqCache seq;
  float xchg[2][kRows];               // [key half][row]: what the two threads of a row tell one another
  uint32_t nan_blocks[2][kRows / 4];  // [V buffer][key], a byte each: blocks of values that are NaN in a suffix position
};
constexpr int kSmemBytes = kOffCtl + (int)sizeof(Ctl);
static_assert(kSmemBytes + 1024 <= 227 * 1024, "one CTA per SM");
using TcWork = Work<5, 4, 4>;

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
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }
// whether any of the 64 threads of a pair of warps says yes (all of them get the answer)
__device__ __forceinline__ bool pair_any(int bar, bool x) {
  uint32_t r;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %2, 0;\n"
      "barrier.cta.red.or.pred q, %1, 64, p;\n"
      "selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r) : "r"(bar), "r"((uint32_t)x) : "memory");
  return r != 0;
}
__device__ __forceinline__ void pair_sync(int bar) { asm volatile("barrier.cta.sync %0, 64;\n" ::"r"(bar) : "memory"); }

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

__global__ void __launch_bounds__(kThreads, 1) kv4_attn_tc_kernel(const Kv4AttnArgs a) {
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
    for (int s = 0; s < kStages; ++s) { mbar_init(&sm.raw_full[s], 1); mbar_init(&sm.raw_empty[s], kConvertWarps); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.k_full[s], kConvertWarps); mbar_init(&sm.v_full[s], kConvertWarps);
      mbar_init(&sm.k_empty[s], 1); mbar_init(&sm.v_empty[s], 1);
      mbar_init(&sm.s_full[s], 1); mbar_init(&sm.p_full[s], kSoftmaxWarps);
    }
    mbar_init(&sm.q_full, kSoftmaxWarps);
    mbar_init(&sm.o_free, kSoftmaxWarps);
    mbar_init(&sm.drain, 1);
    sm.timed_out = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (tid < 16) sm.bad_page[tid] = 0;
  // The set-up above touches nothing of earlier kernels; everything below may.
  pdl_wait();
  pdl_trigger();
  fill_seq_cache(a, sm.seq);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;

  TcWork work(a, sm.seq);
  Segment sg;
  uint32_t it = 0;        // tiles this CTA has started, over all segments: ring stage, buffers and phases
  uint32_t nseg = 0;      // segments with tiles so far: phases of q_full and o_free

  if (warp == kLoadWarp) {
    // ---------------- loader ----------------
    const uint64_t policy = l2_evict_first_policy();
    while (work.next(&sg)) {
      for (int j = 0; j < sg.n; ++j, ++it) {
        const uint32_t st = it % kStages, use = it / kStages;
        if (use > 0 && ok) ok = mbar_wait(&sm.raw_empty[st], (use - 1) & 1u);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (j == 0 && lane == 0) sm.bad_page[nseg & 15u] = 0;
        load_tile(a, sg, sg.t0 + j, sbase + kOffRaw + st * kTileBytes, &sm.raw_full[st], &sm.bad_page[nseg & 15u], policy);
      }
      if (!ok) break;
      if (sg.n > 0) ++nseg;
    }
    // no copy may be on its way when the CTA leaves: the last use of every stage (complete already unless a wait ran out)
    for (uint32_t s = 0; s < kStages && s < it; ++s) mbar_wait(&sm.raw_full[s], ((it - 1 - s) / kStages) & 1u);
    if (!ok && lane == 0) sm.timed_out = 1u;
  } else if (warp == kIssueWarp) {
    // ---------------- tensor-core issuer ----------------
    if (lane == 0) {
      // S = Q K^T: A = Q in tensor memory, B = K tile (K-major: 128 key rows of 128 B per dh half)
      auto issue_qk = [&](uint32_t t) {
        constexpr uint32_t id = umma_idesc(kRows, kKeys, 0);
        if (ok) ok = mbar_wait(&sm.k_full[t & 1u], (t >> 1) & 1u);
        tc_fence_after();
        if (!ok) return;
        const uint32_t kb = sbase + kOffK + (t & 1u) * kOpBytes;
#pragma unroll
        for (int ks = 0; ks < kDh / 16; ++ks)
          umma_ta(tmem + (t & 1u) * kKeys, tmem + kColQ + ks * 8, umma_desc(kb + (ks >> 2) * kHalfBytes + (ks & 3) * 32, 16, 1024), id, ks ? 1u : 0u);
        umma_commit(&sm.s_full[t & 1u]);
        umma_commit(&sm.k_empty[t & 1u]);
      };
      // O += P V: A = P where the logits of its keys stood, B = V tile (MN-major: 128 B of dh per key row, the two dh halves kHalfBytes
      // apart, 16 keys = 2048 B per K step)
      auto issue_pv = [&](uint32_t t, bool first) {
        constexpr uint32_t id = umma_idesc(kRows, kDh, 1);
        const uint32_t vb = sbase + kOffV + (t & 1u) * kOpBytes, p = tmem + (t & 1u) * kKeys;
#pragma unroll
        for (int ks = 0; ks < kKeys / 16; ++ks)
          umma_ta(tmem + kColO, p + (ks >> 2) * 64 + (ks & 3) * 8, umma_desc(vb + ks * 2048, kHalfBytes, 1024), id, (first && ks == 0) ? 0u : 1u);
        umma_commit(&sm.v_empty[t & 1u]);
      };
      while (work.next(&sg)) {
        if (sg.n == 0) continue;
        if (ok) ok = mbar_wait(&sm.q_full, nseg & 1u);
        issue_qk(it);
        for (int j = 0; j < sg.n; ++j, ++it) {
          // the next tile's logits run under this one's softmax; their buffer's last reader was the product before this one
          if (j + 1 < sg.n) issue_qk(it + 1);
          if (ok) ok = mbar_wait(&sm.v_full[it & 1u], (it >> 1) & 1u);
          if (ok) ok = mbar_wait(&sm.p_full[it & 1u], (it >> 1) & 1u);
          if (j == 0 && nseg > 0 && ok) ok = mbar_wait(&sm.o_free, (nseg - 1) & 1u);
          tc_fence_after();
          if (ok) issue_pv(it, j == 0);
        }
        ++nseg;
      }
      if (!ok) {                      // products may still run: they end before tensor memory is freed
        umma_commit(&sm.drain);
        mbar_wait(&sm.drain, 0);
        sm.timed_out = 1u;
      }
    }
    __syncwarp();
  } else if (warp >= kSoftmaxWarps) {
    // ---------------- codes to operands ----------------
    const int w = warp - kSoftmaxWarps;
    const int page = 1 << a.page_log2;
    const int ch = lane & 3;                             // codes [32 ch, 32 ch + 32) of a key: blocks 2 ch and 2 ch + 1
    const int swap = ch >> 1 ? 2 : 0;                    // the second half of the head in another order: no two lanes meet in a bank
    while (work.next(&sg)) {
      const uint32_t* usedw = a.used + (size_t)sg.b * 8;
      for (int j = 0; j < sg.n; ++j, ++it) {
        const uint32_t st = it % kStages, buf = it & 1u;
        const int pos0 = (sg.t0 + j) * kKeys;
        const bool tail = pos0 + kKeys > sg.ctx;         // uniform: the tile reaches past the committed context
        const unsigned char* raw = smem + kOffRaw + st * kTileBytes;
        if (ok) ok = mbar_wait(&sm.raw_full[st], (it / kStages) & 1u);
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
          unsigned long long* empty = which ? &sm.v_empty[buf] : &sm.k_empty[buf];
          if (it >= 2 && ok) ok = mbar_wait(empty, ((it >> 1) - 1) & 1u);
          ok = __all_sync(0xffffffffu, ok);              // (what follows shuffles: all lanes or none)
          unsigned char* op = smem + (which ? kOffV : kOffK) + buf * kOpBytes + (ch >> 1) * kHalfBytes;
          if (ok) {
            uint4 code[4];
            uint32_t sc[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = w * 32 + i * 8 + (lane >> 2), pi = key >> a.page_log2, r = key & (page - 1);
              const unsigned char* blk = raw + (pi * 2 + which) * page * kKv4Entry;
              code[i] = *reinterpret_cast<const uint4*>(blk + r * 64 + ch * 16);
              sc[i] = *reinterpret_cast<const unsigned short*>(blk + page * 64 + r * 8 + ch * 2);
            }
            if (which && tail) {
              // Values nobody reads get a scale of zero (0 x NaN), and so does a NaN that some nodes read: the softmax warps, which know
              // who does, hear of it by a bit per block.
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int key = w * 32 + i * 8 + (lane >> 2), slot = pos0 + key - sg.ctx;
                uint32_t bits = 0;
                if (slot >= 0) {
                  const bool live = slot < a.Ns && ((__ldg(usedw + (slot >> 5)) >> (slot & 31)) & 1u);
                  const bool n0 = (sc[i] & 0x7Fu) == 0x7Fu, n1 = (sc[i] & 0x7F00u) == 0x7F00u;
                  if (live) bits = ((uint32_t)n0 | (uint32_t)n1 << 1) << (2 * ch);
                  if (!live) sc[i] = 0;
                  if (n0) sc[i] &= 0xFF00u;
                  if (n1) sc[i] &= 0x00FFu;
                }
                bits |= __shfl_xor_sync(0xffffffffu, bits, 1);
                bits |= __shfl_xor_sync(0xffffffffu, bits, 2);
                if (ch == 0) reinterpret_cast<unsigned char*>(sm.nan_blocks[buf])[key] = (unsigned char)bits;
              }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = w * 32 + i * 8 + (lane >> 2);
              const uint32_t s2 = e4m3x2_to_half2(sc[i]), s_lo = __byte_perm(s2, 0, 0x1010), s_hi = __byte_perm(s2, 0, 0x3232);
              unsigned char* row = op + key * 128;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                // word kk = k ^ swap of the four; the two orders differ by exchanging words (0, 2) and (1, 3)
                const uint32_t c0 = k == 0 ? code[i].x : k == 1 ? code[i].y : k == 2 ? code[i].z : code[i].w;
                const uint32_t c1 = k == 0 ? code[i].z : k == 1 ? code[i].w : k == 2 ? code[i].x : code[i].y;
                const uint32_t c = swap ? c1 : c0;
                const int kk = k ^ swap;
                const uint32_t s = (kk & 2) ? s_hi : s_lo;
                uint32_t h[4];
                e2m1x8_to_half2(c, h);
                *reinterpret_cast<uint4*>(row + ((((ch & 1) * 4 + kk) ^ (key & 7)) << 4)) =
                    make_uint4(mul_half2(h[0], s), mul_half2(h[1], s), mul_half2(h[2], s), mul_half2(h[3], s));
              }
            }
            fence_async_proxy();                         // for the tensor core's reads
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(which ? &sm.v_full[buf] : &sm.k_full[buf]);
        }
        if (lane == 0) mbar_arrive(&sm.raw_empty[st]);
      }
    }
    if (!ok) sm.timed_out = 1u;
  } else {
    // ---------------- softmax ----------------
    // Warps w and w + 4 share the 32 rows of one lane quarter; the first takes keys 0..63 of every tile and output columns 0..63, the
    // second the other halves.
    const int half = warp >> 2;
    const int row = 32 * (warp & 3) + lane;              // tensor-memory lane this warp may touch
    const uint32_t tmem_lane = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const int pair_bar = 1 + (warp & 3);                 // named barrier of the two warps of a lane quarter
    const int GN = a.G * a.N;
    // Query tile of a segment into tensor memory: this thread's half of its row, two f16 per column (zeros beyond the group); returns what
    // takes the logits back to log2 units.  Called when the S products of the segment before have all completed (every thread
    // awaited their s_full phases): for the first segment at once, for the others before that segment's read-out.
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
      tmem_st32(tmem_lane + kColQ + half * 32, qr);
      tmem_st_wait();
      tc_fence_before();
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
        const uint32_t buf = it & 1u;
        const int kpos0 = (sg.t0 + j) * kKeys + half * 64;     // first key of this thread's 64
        const bool tail = (sg.t0 + j + 1) * kKeys > sg.ctx;    // uniform: the tile reaches past the committed context
        unsigned long long vm = ~0ull;
        if (tail) vm = visible64(visw, kpos0 - sg.ctx);
        if (ok) ok = mbar_wait(&sm.s_full[buf], (it >> 1) & 1u);
        tc_fence_after();
        __syncwarp();
        if (warp_ok) {
          uint32_t sr[64];
          tmem_ld32(tmem_lane + buf * kKeys + half * 64, sr);
          tmem_ld32(tmem_lane + buf * kKeys + half * 64 + 32, sr + 32);
          tmem_ld_wait();
          if (tail) {                                    // a masked logit is replaced, never computed with
#pragma unroll
            for (int e = 0; e < 64; ++e) sr[e] = ((vm >> e) & 1ull) ? sr[e] : 0xFF800000u;
          }
          float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 64; ++e) mx4[e & 3] = fmaxf(mx4[e & 3], __uint_as_float(sr[e]));
          float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * mul;
          // Both threads of a row take the same decision: the reference moves when either half exceeds it by more than kLag.
          if (pair_any(pair_bar, mx > m + kLag)) {
            sm.xchg[half][row] = mx;
            pair_sync(pair_bar);
            mx = fmaxf(mx, sm.xchg[half ^ 1][row]);
            pair_sync(pair_bar);                         // both have read before either writes there again
            float corr = 1.f;
            if (mx > m + kLag) { corr = m == -INFINITY ? 1.f : ex2(m - mx); m = mx; }
            if (j > 0 && __any_sync(0xffffffffu, corr != 1.f)) {
              // O still takes the product of the tile before: wait for it, then scale this thread's columns
              if (ok) ok = mbar_wait(&sm.v_empty[(it - 1) & 1u], ((it - 1) >> 1) & 1u);
              tc_fence_after();
              __syncwarp();
#pragma unroll 1
              for (int c = 0; c < 64; c += 16) {
                uint32_t orr[16];
                asm volatile(
                    "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                    : "=r"(orr[0]), "=r"(orr[1]), "=r"(orr[2]), "=r"(orr[3]), "=r"(orr[4]), "=r"(orr[5]), "=r"(orr[6]), "=r"(orr[7]),
                      "=r"(orr[8]), "=r"(orr[9]), "=r"(orr[10]), "=r"(orr[11]), "=r"(orr[12]), "=r"(orr[13]), "=r"(orr[14]), "=r"(orr[15])
                    : "r"(tmem_lane + kColO + half * 64 + c) : "memory");
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) orr[e] = __float_as_uint(__uint_as_float(orr[e]) * corr);
                asm volatile(
                    "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n"
                    ::"r"(tmem_lane + kColO + half * 64 + c), "r"(orr[0]), "r"(orr[1]), "r"(orr[2]), "r"(orr[3]), "r"(orr[4]), "r"(orr[5]), "r"(orr[6]),
                      "r"(orr[7]), "r"(orr[8]), "r"(orr[9]), "r"(orr[10]), "r"(orr[11]), "r"(orr[12]), "r"(orr[13]), "r"(orr[14]), "r"(orr[15])
                    : "memory");
              }
              tmem_st_wait();
              l *= corr;
            }
          }
          const float mu = m == -INFINITY ? 0.f : m - kLift;
          uint32_t pk[32];
          float ls4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < 64; c += 2) {
            const float p0 = ex2(fmaf(__uint_as_float(sr[c]), mul, -mu));
            const float p1 = ex2(fmaf(__uint_as_float(sr[c + 1]), mul, -mu));
            ls4[(c >> 1) & 3] += p0 + p1;
            pk[c >> 1] = pack_half2(p0, p1);
          }
          l += (ls4[0] + ls4[1]) + (ls4[2] + ls4[3]);
          tmem_st32(tmem_lane + buf * kKeys + half * 64, pk);
          tmem_st_wait();
          if (tail) {                                    // NaN values among the keys this row sees
            if (ok) ok = mbar_wait(&sm.v_full[buf], (it >> 1) & 1u);
            uint32_t any = 0;
#pragma unroll 4
            for (int c = 0; c < 16; ++c) any |= sm.nan_blocks[buf][half * 16 + c];
            if (any)
              for (int e = 0; e < 64; ++e)
                if ((vm >> e) & 1ull) nan_cols |= reinterpret_cast<const unsigned char*>(sm.nan_blocks[buf])[half * 64 + e];
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[buf]);
      }
      // end of the segment.  First the next segment's queries (its logits then run under this read-out) ...
      have = work.next(&sgn);
      if (have && sgn.n > 0) mul_next = store_q(sgn);
      // ... then the last O product, normalise and write the slot
      if (ok) ok = mbar_wait(&sm.v_empty[(it - 1) & 1u], ((it - 1) >> 1) & 1u);
      tc_fence_after();
      const bool bad = *reinterpret_cast<volatile uint32_t*>(&sm.bad_page[nseg & 15u]) != 0;
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
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const bool nan = (nan_cols >> (half * 4 + (c + e) / 16)) & 1u;
            orr[e] = bad ? 0u : nan ? 0x7FC00000u : __float_as_uint(__uint_as_float(orr[e]) * inv);
          }
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
  if (tid == 0) a.cta_code[blockIdx.x] = (int)sm.timed_out;      // the merge kernel turns this into status words
  if (warp == kIssueWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

}  // namespace

cudaError_t launch_kv4_attn_tc(const Kv4Plan& plan, bool pdl, cudaStream_t st) {
  static bool configured[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < kMaxDevices && !configured[dev]) {
    e = cudaFuncSetAttribute(kv4_attn_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  return launch_kernel(kv4_attn_tc_kernel, dim3(plan.a.C), dim3(kThreads), kSmemBytes, st, pdl, plan.a);
}

}  // namespace lumo
