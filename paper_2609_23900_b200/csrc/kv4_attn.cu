// Ancestry-masked decode attention over the paged 4-bit cache (sm_100a):
//
//   out[b,i,h,:] = sum_p softmax_p(scale q[b,i,h] . k[p]) v[p]  over the context and the node's ancestors and itself
//
// Keys and values come as e2m1 codes and e4m3 scales, 144 bytes a position and KV head.  A code times its scale has at most six
// significant bits, so it is exact in f16: the tensor cores multiply f16 operands whose only roundings are those of the
// probabilities (half a step: 2^-11 relative each).  Against the same formula with fp32 probabilities, bf16 outputs differ by 0.0005 to 0.0009
// of their norm (neighbouring bf16 numbers here and there; the bf16 rounding itself is 0.0017); fp32 ones would cost the second product twice
// over (high and low parts).  A query row is scaled by a power of two to fit f16 (its elements are bf16: eight bits) and the logits are
// scaled back in fp32; sums are fp32.
//
// The work is the list of 128-key tiles of all (sequence, KV head, row tile) units in order; a CTA takes a contiguous share of the list, and
// every piece of its share that lies in one unit is a SEGMENT, whose normalised output and base-2 log-sum-exp go to a slot;
// kv4_merge_kernel combines the slots of a unit in key order.  A tile is staged by bulk copies, one per page: a head's keys and values
// of a page are adjacent.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "internal.h"
#include "kv4_attn.h"

namespace lumo {

namespace {

// ---- register form -----------------------------------------------------------------------
// For up to 8 NT query rows per unit (a token or a short tree of one request times its head group): one warp issues the bulk copies into a ring
// of eight tiles, and the others turn codes into matrix operands in registers, without a second trip through shared memory.  A warp takes 16
// or 32 keys of a tile at a time (NT = 1: 32, two chains of products to overlap), sixteen of them thus:
//
//   S^T [16 keys x 8 rows] = K Q^T, eight m16n8k16 products; lane (g, t) of a warp (g = lane / 4, t = lane % 4) supplies elements
//       [32 t, 32 t + 32) of two keys, one 16-byte read each: which element stands at which place of the inner dimension is free as long as
//       Q's fragments agree
//   O^T [128 x 8 rows] += V^T P^T, eight products (one per 16 elements of the head): lane (g, t) supplies block g of four keys.  The two
//       codes of a byte have to belong to two keys: the nibbles of two keys' words are interleaved (two instructions per eight codes).
//       P^T comes out of S^T's accumulators by an 8 x 8 transposition across the warp.
//
// Every warp has its own reference maximum per row and its own sums; they meet once per segment, through shared memory, in warp order.
// A tile takes each scheduler 720 instructions (90 for 16 keys and scheduler; three quarters turn codes into f16), and the SM's share of the
// memory 800 cycles; four warps a scheduler issue in six cycles of ten, so a tile takes 1170.  Sixteen tokens at 16k: 57 to 58 us, 4.0 TB/s;
// one token at 4k: 12.2 us, of which the attention kernel takes 8.2 (a chain of dependent loads, two tiles and the warps' meeting) and the
// merge the rest.
template <int NT> struct Small {
  static constexpr int kWarps = NT == 1 ? 15 : 11;       // consumers; with the loader a multiple of four: 128 registers a thread, 168 for NT = 2
  static constexpr int kSub = NT == 1 ? 2 : 1;           // groups of sixteen keys a warp takes at a time
  static constexpr int kPieces = kKeys / 16 / kSub;      // pieces of a tile
  static constexpr int kStages = 8;
  static constexpr int kThreads = 32 * (kWarps + 1);
  static constexpr int kRedRow = 132;                    // floats per row of the reduction buffer: the stores of a half warp meet no bank twice
  static constexpr int kOffRed = kStages * kTileBytes;
  static constexpr int kOffCtl = kOffRed + kWarps * 8 * kRedRow * 4;
  struct Ctl {
    // Two per stage, taken in turn: a warp may wait for a tile while the copies of the one before it in that stage are still on their way (it
    // has pieces of every fourth tile or so, and copies may overtake one another), and would take that one's phase for its own.
    unsigned long long full[2 * kStages], empty[kStages];
    SeqCache seq;
    float stat[kWarps][8 * NT][2];                       // a warp's reference maximum and sum of each row
    uint32_t timed_out;
    uint32_t bad_page[16];                               // by segment number mod 16: the loader is never that far ahead
  };
  static constexpr int kBytes = kOffCtl + (int)sizeof(Ctl);
  // A segment costs about as much as twelve tiles.  Charged 6, 12, 18, us: 16 tokens at 16k 58.5, 57.1, 59.8; one at 4k 12.4, 12.4, 12.5; 5
  // at 30k 38.5, 36.8, 37.5; 9 trees of 2 nodes at 7k 27.7, 26.1, 26.8; 12 rows, 6 at 12k 40.1, 39.1, 40.7; 16 rows, 16 at 16k 95.2, 93.8,
  // 97.5.  No share below two tiles (four: one at 4k takes 0.6 us more), and whole units up to three tiles longer than a share.
  using W = Work<12, 2, 3>;
};
static_assert(Small<1>::kBytes <= 227 * 1024 && Small<2>::kBytes <= 227 * 1024, "one CTA per SM");

__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(x));
  return r;
}

template <int NT, bool kDrill>
__global__ void __launch_bounds__(Small<NT>::kThreads, 1) kv4_attn_small_kernel(const Kv4AttnArgs a) {
  using C = Small<NT>;
  auto wait = [](unsigned long long* bar, uint32_t parity) { return mbar_wait(bar, parity, kDrill ? kSpinLimitDrill : kSpinLimit); };
  extern __shared__ __align__(128) unsigned char smem[];
  typename C::Ctl& sm = *reinterpret_cast<typename C::Ctl*>(smem + C::kOffCtl);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < C::kStages; ++s) mbar_init(&sm.empty[s], C::kPieces);
    for (int s = 0; s < 2 * C::kStages; ++s) mbar_init(&sm.full[s], 1);
    sm.timed_out = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (tid < 16) sm.bad_page[tid] = 0;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  if (warp == C::kWarps) C::W::set_up(a, sm.seq);
  __syncthreads();
  typename C::W work(a, sm.seq);
  Segment sg;
  bool ok = true;
  uint32_t it = 0;     // tiles of this CTA so far, over all segments
  uint32_t nseg = 0;

  if (warp == C::kWarps) {
    // ---------------- loader ----------------
    const uint64_t policy = l2_evict_first_policy();
    while (work.next(&sg)) {
      PageWalk walk(a, sg);
      for (int j = 0; j < sg.n; ++j, ++it) {
        const uint32_t st = it % C::kStages, use = it / C::kStages;
        const bool wanted = walk.wanted(j);
        const int pg = walk.take(j);
        if (use > 0 && ok) ok = wait(&sm.empty[st], (use - 1) & 1u);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (j == 0 && lane == 0) sm.bad_page[nseg & 15u] = 0;
        if (!kDrill)
          load_tile<true>(a, sg, wanted, pg, 0, smem_u32(smem) + st * kTileBytes, &sm.full[it % (2 * C::kStages)], &sm.bad_page[nseg & 15u], policy);
      }
      if (!ok) break;
      if (sg.n > 0) ++nseg;
    }
    if (!ok && lane == 0) sm.timed_out = 1;
    // no copy may be on its way when the CTA leaves: the last use of every barrier (complete already unless a wait ran out)
    for (uint32_t s = 0; s < 2 * C::kStages && s < it; ++s) wait(&sm.full[s], ((it - 1 - s) / (2 * C::kStages)) & 1u);
  } else {
    // ---------------- consumers ----------------
    const int g = lane >> 2, t = lane & 3;
    const int GN = a.G * a.N, page = 1 << a.page_log2;
    const int kq = (g >> 1) + (g & 1) * 4;               // position of matrix row g among eight keys: lane t's value keys are t and t + 4
    // where this lane's parts of a group of sixteen keys lie, behind the group's page and its first position in it
    const uint32_t k_codes = kq * 64 + t * 16, k_scales = page * 64 + kq * 8 + t * 2;
    const uint32_t v_codes = page * kKv4Entry + t * 64 + g * 8, v_scales = page * (kKv4Entry + 64) + t * 8 + g;
    float* red = reinterpret_cast<float*>(smem + C::kOffRed);
    while (work.next(&sg)) {
      if (tid == 0) a.unit_slots[sg.unit] = make_int2(sg.slot0, sg.nslots);   // for the merge (same pair from every writer)
      // query fragments: row 8 nt + g, elements [32 t, 32 t + 32)
      uint32_t qf[NT][16];
      float mul[NT][2];                                  // logits of rows 8 nt + 2 t, + 1 back from the scaled queries, in log2 units
      const uint32_t* vis[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = sg.rt * a.R + nt * 8 + g;
        const bool in = r < GN;
        const int hl = in ? r / a.N : 0, node = in ? r - hl * a.N : 0;
        const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + ((size_t)sg.b * a.N + node) * a.q_stride +
                                                          ((size_t)sg.hkv * a.G + hl) * kDh + t * 32);
        uint32_t w[16], top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 v = in ? __ldg(src + i) : make_uint4(0, 0, 0, 0);
          w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, max((w[i] << 16) & 0x7FFF0000u, w[i] & 0x7FFF0000u));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = query_exponent(top);
        const float up = exp2i(e);
#pragma unroll
        for (int i = 0; i < 16; ++i) qf[nt][i] = pack_half2(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xFFFF0000u) * up);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int lr = 2 * t + h;                      // the accumulators' row
          mul[nt][h] = a.scale_log2 * exp2i(-__shfl_sync(0xffffffffu, e, lr * 4));
          const int rr = sg.rt * a.R + nt * 8 + lr;
          vis[nt][h] = a.vis + ((size_t)sg.b * a.N + (rr < GN ? rr % a.N : 0)) * 8;
        }
      }
      const uint32_t* usedw = a.used + (size_t)sg.b * 8;
      float o[NT][8][4], m[NT][2], mu[NT][2], l[NT][2];       // mu: what is taken off the logits (a row without keys: 0)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[nt][j][e] = 0.f;
        m[nt][0] = m[nt][1] = -INFINITY;
        mu[nt][0] = mu[nt][1] = l[nt][0] = l[nt][1] = 0.f;
      }
      // the segment's pieces of 16 kSub keys are dealt out to the warps in turn
      for (int gi = warp; gi < sg.n * C::kPieces; gi += C::kWarps) {
        const uint32_t tt = it + gi / C::kPieces, st = tt % C::kStages;
        const int first = (gi % C::kPieces) * 16 * C::kSub;
        if (ok) ok = wait(&sm.full[tt % (2 * C::kStages)], (tt / (2 * C::kStages)) & 1u);
        ok = __all_sync(0xffffffffu, ok);                // (what follows shuffles: all lanes or none)
        const int pos0 = (sg.t0 + gi / C::kPieces) * kKeys + first;     // the piece's first position
        if (ok && pos0 < sg.ctx + a.Ns) {
          const bool tail = pos0 + 16 * C::kSub > sg.ctx;
          const unsigned char *at_codes[C::kSub], *at_scales[C::kSub];
#pragma unroll
          for (int u = 0; u < C::kSub; ++u) {            // a group of sixteen lies in one page
            const int c0 = first + 16 * u, r0 = c0 & (page - 1);
            const unsigned char* pg = smem + st * kTileBytes + (c0 >> a.page_log2) * (page * 2 * kKv4Entry);
            at_codes[u] = pg + r0 * 64;
            at_scales[u] = pg + r0 * 8;
          }
          // ---- S^T
          float s[C::kSub][NT][4];
#pragma unroll
          for (int u = 0; u < C::kSub; ++u) {
            float s2[NT][4];                             // two chains of four products each
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[u][nt][e] = s2[nt][e] = 0.f;
            const uint4 ka = *reinterpret_cast<const uint4*>(at_codes[u] + k_codes), kb = *reinterpret_cast<const uint4*>(at_codes[u] + k_codes + 8 * 64);
            const uint32_t sa = e4m3x2_to_half2(*reinterpret_cast<const unsigned short*>(at_scales[u] + k_scales));
            const uint32_t sb = e4m3x2_to_half2(*reinterpret_cast<const unsigned short*>(at_scales[u] + k_scales + 8 * 8));
            const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
            const uint32_t fa[2] = {__byte_perm(sa, 0, 0x1010), __byte_perm(sa, 0, 0x3232)}, fb[2] = {__byte_perm(sb, 0, 0x1010), __byte_perm(sb, 0, 0x3232)};
#pragma unroll
            for (int w = 0; w < 4; ++w) {                // 32 t + 8 w ..: block 2 t for w < 2
              uint32_t ha[4], hb[4];
              e2m1x8_to_half2(wa[w], ha);
              e2m1x8_to_half2(wb[w], hb);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t fr[4] = {mul_half2(ha[2 * k], fa[w >> 1]), mul_half2(hb[2 * k], fb[w >> 1]), mul_half2(ha[2 * k + 1], fa[w >> 1]),
                                        mul_half2(hb[2 * k + 1], fb[w >> 1])};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(k ? s2[nt] : s[u][nt], fr, qf[nt][4 * w + 2 * k], qf[nt][4 * w + 2 * k + 1]);
              }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[u][nt][e] = (s[u][nt][e] + s2[nt][e]) * mul[nt][e & 1];
          }
          // ---- softmax: s[u][nt] = (key kq of group u: rows 2 t, 2 t + 1), (key 8 + kq: the same rows).  A masked logit is replaced.
          if (tail) {
#pragma unroll
            for (int u = 0; u < C::kSub; ++u)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (!slot_seen(vis[nt][e & 1], pos0 + 16 * u + kq + 8 * (e >> 1) - sg.ctx)) s[u][nt][e] = -INFINITY;
          }
          bool over = false;
          float top[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = fmaxf(s[0][nt][h], s[0][nt][2 + h]);
#pragma unroll
              for (int u = 1; u < C::kSub; ++u) x = fmaxf(x, fmaxf(s[u][nt][h], s[u][nt][2 + h]));
              top[nt][h] = x;
              over |= x > m[nt][h] + kLag;
            }
          if (__any_sync(0xffffffffu, over)) {           // some row's reference maximum has to move
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float mx = top[nt][h];
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                if (mx > m[nt][h] + kLag) {
                  const float corr = ex2(m[nt][h] - mx); // 0 the first time, when there is nothing to scale
                  m[nt][h] = mx;
                  mu[nt][h] = mx - kLift;
                  l[nt][h] *= corr;
#pragma unroll
                  for (int jj = 0; jj < 8; ++jj) { o[nt][jj][h] *= corr; o[nt][jj][2 + h] *= corr; }
                }
              }
          }
          uint32_t p0[C::kSub][NT], p1[C::kSub][NT];
#pragma unroll
          for (int u = 0; u < C::kSub; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float p[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) p[e] = ex2(s[u][nt][e] - mu[nt][e & 1]);
              l[nt][0] += p[0] + p[2];
              l[nt][1] += p[1] + p[3];
              p0[u][nt] = transpose8(pack_half2(p[0], p[1]));
              p1[u][nt] = transpose8(pack_half2(p[2], p[3]));
            }
          // ---- O^T: block g of keys t, t + 4 and t + 8, t + 12 of a group
#pragma unroll
          for (int u = 0; u < C::kSub; ++u) {
            uint2 vc[4];
            uint32_t b4[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              vc[k] = *reinterpret_cast<const uint2*>(at_codes[u] + v_codes + k * 4 * 64);
              b4[k] = at_scales[u][v_scales + k * 4 * 8];
            }
            if (tail) {
              // Values nobody reads are left out of the product by a scale of zero (0 x NaN), and so is a NaN that some nodes read: it
              // turns block g of those nodes' outputs into NaN by hand.
              const int slot0 = pos0 + 16 * u - sg.ctx;
              uint32_t nan = 0;                          // bit per key of the group
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int slot = slot0 + t + 4 * k;
                if (slot < 0) continue;
                const bool live = slot < a.Ns && ((__ldg(usedw + (slot >> 5)) >> (slot & 31)) & 1u);
                if (live && (b4[k] & 0x7Fu) == 0x7Fu) nan |= 1u << (t + 4 * k);
                if (!live || (b4[k] & 0x7Fu) == 0x7Fu) b4[k] = 0;
              }
              if (__any_sync(0xffffffffu, nan != 0)) {
                nan |= __shfl_xor_sync(0xffffffffu, nan, 1);
                nan |= __shfl_xor_sync(0xffffffffu, nan, 2);     // block g, all sixteen keys
                // the accumulators' rows of lane (g, t) are head elements of block g: its own mask
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int h = 0; h < 2; ++h) {
                    bool hit = false;
#pragma unroll 1
                    for (int k = 0; k < 16; ++k) hit |= ((nan >> k) & 1u) && slot_seen(vis[nt][h], slot0 + k);
                    if (hit)
#pragma unroll
                      for (int jj = 0; jj < 8; ++jj) o[nt][jj][h] = o[nt][jj][2 + h] = __int_as_float(0x7FC00000);
                  }
              }
            }
            const uint32_t sc[2] = {e4m3x2_to_half2(b4[0] | b4[1] << 8), e4m3x2_to_half2(b4[2] | b4[3] << 8)};
#pragma unroll
            for (int w = 0; w < 2; ++w) {                // codes 8 w .. 8 w + 7 of the block
              uint32_t ev[2][4], od[2][4];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t x = w ? vc[2 * k].y : vc[2 * k].x, y = w ? vc[2 * k + 1].y : vc[2 * k + 1].x;
                e2m1x8_to_half2((x & 0x0F0F0F0Fu) | ((y << 4) & 0xF0F0F0F0u), ev[k]);
                e2m1x8_to_half2(((x >> 4) & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u), od[k]);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t fr[4] = {mul_half2(ev[0][i], sc[0]), mul_half2(od[0][i], sc[0]), mul_half2(ev[1][i], sc[1]), mul_half2(od[1][i], sc[1])};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][4 * w + i], fr, p0[u][nt], p1[u][nt]);
              }
            }
          }
        }
        __syncwarp();
        if (ok && lane == 0) mbar_arrive(&sm.empty[st]); // (whoever gave up keeps the stage: its copies may not have landed, and none go on top)
      }
      it += sg.n;
      // ---- the warps' parts meet: maxima and sums, then the outputs of eight rows at a time
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = l[nt][h];
          x += __shfl_xor_sync(0xffffffffu, x, 4);
          x += __shfl_xor_sync(0xffffffffu, x, 8);
          x += __shfl_xor_sync(0xffffffffu, x, 16);
          if (g == 0) { sm.stat[warp][nt * 8 + 2 * t + h][0] = m[nt][h]; sm.stat[warp][nt * 8 + 2 * t + h][1] = x; }
        }
      asm volatile("bar.sync 1, %0;\n" ::"r"(C::kWarps * 32) : "memory");
      const bool whole = sg.nslots == 1;                 // the only segment of its unit: these are the final outputs
      const bool bad = sg.n > 0 && *reinterpret_cast<volatile uint32_t*>(&sm.bad_page[nseg & 15u]) != 0;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int lr = 2 * t + h;
          float mx = -INFINITY;
#pragma unroll
          for (int w = 0; w < C::kWarps; ++w) mx = fmaxf(mx, sm.stat[w][nt * 8 + lr][0]);
          const float f = m[nt][h] == -INFINITY ? (l[nt][h] == 0.f ? 0.f : 1.f) : ex2(m[nt][h] - mx);
#pragma unroll
          for (int jj = 0; jj < 8; ++jj)
            *reinterpret_cast<float2*>(red + (warp * 8 + lr) * C::kRedRow + jj * 16 + g * 2) = make_float2(o[nt][jj][h] * f, o[nt][jj][2 + h] * f);
        }
        asm volatile("bar.sync 1, %0;\n" ::"r"(C::kWarps * 32) : "memory");
        for (int e = tid; e < 8 * 64; e += C::kWarps * 32) {     // row e / 64, elements 2 (e % 64) and the next
          const int lr = e >> 6, pr = e & 63, r = sg.rt * a.R + nt * 8 + lr;
          if (r >= GN) continue;
          float mx = -INFINITY, lt = 0.f;
#pragma unroll
          for (int w = 0; w < C::kWarps; ++w) mx = fmaxf(mx, sm.stat[w][nt * 8 + lr][0]);
          float2 sum = make_float2(0.f, 0.f);
#pragma unroll
          for (int w = 0; w < C::kWarps; ++w) {
            const float mw = sm.stat[w][nt * 8 + lr][0], lw = sm.stat[w][nt * 8 + lr][1];
            lt += lw * (mw == -INFINITY ? 1.f : ex2(mw - mx));
            const float2 v = *reinterpret_cast<const float2*>(red + (w * 8 + lr) * C::kRedRow + (pr & 7) * 16 + (pr >> 3) * 2);
            sum.x += v.x;
            sum.y += v.y;
          }
          const float inv = bad ? 0.f : row_inverse(lt) * a.v_mul;
          const float2 val = bad ? make_float2(0.f, 0.f) : make_float2(sum.x * inv, sum.y * inv);
          const float l2 = row_lse2(mx == -INFINITY ? 0.f : mx, lt);
          if (whole) {
            const int hl = r / a.N, node = r - hl * a.N;
            const size_t row = ((size_t)sg.b * a.N + node) * a.Hq + (size_t)sg.hkv * a.G + hl;
            if (a.out_bf16) {
              const __nv_bfloat162 v = __floats2bfloat162_rn(val.x, val.y);
              reinterpret_cast<__nv_bfloat162*>(a.out)[row * 64 + pr] = v;
            } else {
              reinterpret_cast<float2*>(a.out)[row * 64 + pr] = val;
            }
            if (pr == 0 && a.lse) a.lse[row] = bad ? 0.f : l2 * kLn2;
          } else {
            const int rl = nt * 8 + lr;
            float* slot = a.part_o + (size_t)sg.slot * a.R * kDh;
            *reinterpret_cast<float2*>(slot + ((size_t)(pr >> 1) * a.R + rl) * 4 + (pr & 1) * 2) = val;
            if (pr == 0) a.part_lse[(size_t)sg.slot * a.R + rl] = bad ? INFINITY : l2;
          }
        }
        asm volatile("bar.sync 1, %0;\n" ::"r"(C::kWarps * 32) : "memory");
      }
      if (whole && tid == 0) a.part_lse[(size_t)sg.slot * a.R] = bad ? INFINITY : 0.f;
      if (sg.n > 0) ++nseg;
    }
    if (!ok) sm.timed_out = 1;
  }
  __syncthreads();
  if (tid == 0) a.cta_code[blockIdx.x] = (int)sm.timed_out;      // the merge kernel turns this into status words
}

// ---- combination ---------------------------------------------------------------------------
// An entry is one row of a unit and four columns; a slot holds its rows by groups of four columns, [column group][row][4], so a warp reads 512
// contiguous bytes.  kParts threads take an entry's slots in turn, each four to a flight of loads against a running maximum, and meet through
// shared memory in order: the result for a given decomposition is reproducible.  A slot whose log-sum-exp is +inf (no sum gives that) met a
// page that does not exist.  What it costs is the chain of loads (which slots, their weights and rows) and, with many rows, how many
// threads an SM holds: hence the bound on registers.
template <int kParts>
__global__ void __launch_bounds__(256, 4) kv4_merge_kernel(const Kv4AttnArgs a, int r_log2) {
  constexpr int kBatch = 4, kEntries = 256 / kParts;
  __shared__ float4 acc_s[kParts > 1 ? 256 : 1];
  __shared__ float2 stat_s[kParts > 1 ? 256 : 1];      // maximum, denominator
  const int upb = a.Hkv * a.RT;
  const int per_log2 = r_log2 + 5 - (kParts == 1 ? 8 : 6);               // CTAs per unit (R >= 8: at least one)
  const int u = blockIdx.x >> per_log2, tid = threadIdx.x;
  const int part = kParts == 1 ? 0 : tid / kEntries;
  const int i = (blockIdx.x & ((1 << per_log2) - 1)) * kEntries + (tid & (kEntries - 1));
  const int cg = i >> r_log2, r = i & ((1 << r_log2) - 1);
  const int b = u / upb, rem = u - b * upb;
  const int hkv = rem / a.RT, rt = rem - hkv * a.RT, rg = rt * a.R + r;
  pdl_wait();          // launched as a programmatic dependent of the attention kernel: its slots are complete from here on
  pdl_trigger();
  const int cx = a.ctx_len[b], cr = a.cache_row[b];
  const int2 sl = a.unit_slots[u];       // meaningless for a sequence that fails its check
  const bool reports = rem == 0 && i < 32 && part == 0 && a.status;      // one warp a sequence
  int late = 0;
  if (reports) {
#pragma unroll 5
    for (int c = i; c < a.C; c += 32) late |= a.cta_code[c];
  }
  const int st = seq_check(cx, cr, a.Ns, a.n_rows, a.max_pos);
  const bool row_ok = rg < a.G * a.N;
  const int n = st == LUMO_SEQ_OK ? sl.y : 0;
  const float* lp = a.part_lse + (size_t)sl.x * a.R + (sl.y == 1 || !row_ok ? 0 : r);
  const float4* op = reinterpret_cast<const float4*>(a.part_o) + ((size_t)sl.x * 32 + cg) * a.R + r;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float mx = -INFINITY, den = 0.f;
  bool bad = false;
  if (n > 1 ? row_ok || reports : reports)
    for (int s0 = part; s0 < n; s0 += kParts * kBatch) {
      float4 v[kBatch];
      float w[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const bool in = s0 + k * kParts < n;
        w[k] = in ? lp[(size_t)(s0 + k * kParts) * a.R] : -INFINITY;
        v[k] = in && n > 1 && row_ok ? op[(size_t)(s0 + k * kParts) * 32 * a.R] : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      float top = mx;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) { top = fmaxf(top, w[k]); bad |= w[k] == INFINITY; }
      if (top == INFINITY) continue;
      const float corr = mx == -INFINITY ? 1.f : ex2(mx - top);          // (nothing summed yet, or NaN alone)
      den *= corr; acc.x *= corr; acc.y *= corr; acc.z *= corr; acc.w *= corr;
      mx = top;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (w[k] == -INFINITY) continue;   // none, or a slot without keys for this row
        const float x = mx == -INFINITY ? w[k] : ex2(w[k] - mx);         // (no maximum: every weight is a NaN)
        den += x;
        acc.x = fmaf(x, v[k].x, acc.x); acc.y = fmaf(x, v[k].y, acc.y);
        acc.z = fmaf(x, v[k].z, acc.z); acc.w = fmaf(x, v[k].w, acc.w);
      }
    }
  if constexpr (kParts > 1) {
    acc_s[tid] = acc;
    stat_s[tid] = make_float2(bad ? INFINITY : mx, den);
    __syncthreads();
    if (part) return;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < kParts; ++k) { const float w = stat_s[k * kEntries + tid].x; bad |= w == INFINITY; top = fmaxf(top, w); }
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    den = 0.f;
    mx = top;
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const float2 w = stat_s[k * kEntries + tid];
      const float4 v = acc_s[k * kEntries + tid];
      const float x = w.x == -INFINITY && w.y == 0.f ? 0.f : mx == -INFINITY ? 1.f : ex2(w.x - mx);       // (a part of NaN weights alone keeps its NaN)
      den = fmaf(x, w.y, den);
      acc.x = fmaf(x, v.x, acc.x); acc.y = fmaf(x, v.y, acc.y); acc.z = fmaf(x, v.z, acc.z); acc.w = fmaf(x, v.w, acc.w);
    }
  }
  if (reports) {
    late = __any_sync(0xffffffffu, late);
    if (i == 0) a.status[b] = st != LUMO_SEQ_OK ? st : (late ? (int)LUMO_SEQ_TIMEOUT : (bad ? (int)LUMO_SEQ_BAD_PAGE : (int)LUMO_SEQ_OK));
  }
  if (!row_ok || n == 1) return;         // (a single segment: the attention kernel has written the outputs)
  const int hl = rg / a.N, node = rg - hl * a.N;
  const size_t row = ((size_t)b * a.N + node) * a.Hq + (size_t)hkv * a.G + hl;
  float lse = 0.f;
  if (n == 0 || bad) {
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
  } else {
    const float inv = row_inverse(den);
    acc = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    lse = den == 0.f ? -INFINITY : (mx + log2f(den)) * kLn2;
  }
  if (a.out_bf16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(acc.x, acc.y), y = __floats2bfloat162_rn(acc.z, acc.w);
    reinterpret_cast<uint2*>(a.out)[row * 32 + cg] = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  } else {
    reinterpret_cast<float4*>(a.out)[row * 32 + cg] = acc;
  }
  if (a.lse && cg == 0) a.lse[row] = lse;
}

template <int NT, bool kDrill>
cudaError_t launch_small(const Kv4Plan& plan, bool pdl, cudaStream_t st) {
  static bool configured[kMaxDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < kMaxDevices && !configured[dev]) {
    e = cudaFuncSetAttribute(kv4_attn_small_kernel<NT, kDrill>, cudaFuncAttributeMaxDynamicSharedMemorySize, Small<NT>::kBytes);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  return launch_kernel(kv4_attn_small_kernel<NT, kDrill>, dim3(plan.a.C), dim3(Small<NT>::kThreads), Small<NT>::kBytes, st, pdl, plan.a);
}

// Rows of a row tile: the register form up to sixteen, the tensor-memory form (kv4_attn_tc.cu) beyond.  The latter's 128-row tile costs the same
// however many rows are in use; the register form's work grows with them.  Register form against tensor memory, us: 16 sequences at 16k
// with 4, 8 and 16 rows 57.6, 61.8, 95.2 against 109; 4 at 8k with 20 and 32 rows (in tiles of sixteen) 33.9, 37.5 against 25.6, 26.5; 8
// at 16k with 32 rows 95.3 against 61.4.
int rows_per_tile(int G, int N) { return G * N <= 8 ? 8 : G * N <= 16 ? 16 : 128; }

}  // namespace

long long kv4_units(int B, int N, int Hq, int Hkv) {
  const int G = Hq / Hkv, R = rows_per_tile(G, N);
  return (long long)B * Hkv * ((G * N + R - 1) / R);
}
long long kv4_line(const Kv4Shape& s) {
  const int R = rows_per_tile(s.Hq / s.Hkv, s.N);
  const int cost = R == 8 ? Small<1>::W::kSegmentCost : R == 16 ? Small<2>::W::kSegmentCost : kv4_segment_cost_tc();
  const long long tiles = (((long long)s.max_pages << s.page_log2) + kKeys - 1) / kKeys;
  return kv4_units(s.B, s.N, s.Hq, s.Hkv) * (tiles + cost);
}

// workspace: partial outputs [slots][R][128], log-sum-exps [slots][R], CTA codes, the units' slots
static size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t kv4_work_bytes(int B, int N, int Hq, int Hkv, int n_splits, int sms) {
  const int R = rows_per_tile(Hq / Hkv, N);
  const size_t units = (size_t)kv4_units(B, N, Hq, Hkv), ctas = n_splits > 0 ? units * n_splits : (size_t)sms;
  const size_t slots = n_splits > 0 ? ctas : units + ctas;
  return round256(slots * R * kDh * 4) + round256(slots * R * 4) + round256(ctas * 4) + round256(units * sizeof(int2));
}

void kv4_plan(const Kv4Shape& s, const Kv4AttnPtrs& p, const uint32_t* vis, const uint32_t* used, float scale, long long q_stride, int out_bf16,
              int n_splits, void* work, int sms, bool drill, Kv4Plan* plan) {
  Kv4AttnArgs& a = plan->a;
  a.pages = reinterpret_cast<const unsigned char*>(p.pages); a.q = p.q; a.out = p.out; a.lse = p.lse; a.status = p.status;
  a.ctx_len = s.ctx_len; a.cache_row = s.cache_row; a.table = s.table; a.vis = vis; a.used = used; a.q_stride = q_stride;
  a.B = s.B; a.N = s.N; a.Ns = s.Ns; a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.Hq / s.Hkv;
  a.R = rows_per_tile(a.G, a.N);
  a.RT = (a.G * a.N + a.R - 1) / a.R;
  a.n_rows = s.n_rows; a.max_pages = s.max_pages; a.n_pages = s.n_pages; a.page_log2 = s.page_log2; a.max_pos = s.max_pages << s.page_log2;
  const size_t units = (size_t)s.B * s.Hkv * a.RT, ctas = n_splits > 0 ? units * n_splits : (size_t)sms;
  const size_t slots = n_splits > 0 ? ctas : units + ctas;
  a.S = n_splits; a.C = (int)ctas; a.out_bf16 = out_bf16;
  plan->sms = sms;
  plan->drill = drill;
  a.scale_log2 = ldexpf(scale * kLog2e, s.k_exp);
  a.v_mul = ldexpf(1.f, s.v_exp);
  unsigned char* w = reinterpret_cast<unsigned char*>(work);
  a.part_o = reinterpret_cast<float*>(w); w += round256(slots * a.R * kDh * 4);
  a.part_lse = reinterpret_cast<float*>(w); w += round256(slots * a.R * 4);
  a.cta_code = reinterpret_cast<int32_t*>(w); w += round256(ctas * 4);
  a.unit_slots = reinterpret_cast<int2*>(w);
}

cudaError_t launch_kv4_attn(const Kv4Plan& plan, bool pdl, cudaStream_t st) {
  if (plan.a.R == 128) return launch_kv4_attn_tc(plan, pdl, st);
  if (plan.drill) return plan.a.R == 8 ? launch_small<1, true>(plan, pdl, st) : launch_small<2, true>(plan, pdl, st);
  return plan.a.R == 8 ? launch_small<1, false>(plan, pdl, st) : launch_small<2, false>(plan, pdl, st);
}

// Four threads an entry while all of their CTAs run at once: then the chain of flights is what the merge takes (a token at 4k: 3.7 us, 4.6
// with one); one where four would come in several waves (4 x 8 nodes at 8k: 5.5 us, 7.4 with four).
cudaError_t launch_kv4_merge(const Kv4Plan& plan, bool pdl, cudaStream_t st) {
  const Kv4AttnArgs& a = plan.a;
  const long long units = (long long)a.B * a.Hkv * a.RT;
  const int r_log2 = a.R == 8 ? 3 : a.R == 16 ? 4 : 7;
  if (units * a.R / 2 <= 4LL * plan.sms) return launch_kernel(kv4_merge_kernel<4>, dim3((unsigned)(units * a.R / 2)), dim3(256), 0, st, pdl, a, r_log2);
  return launch_kernel(kv4_merge_kernel<1>, dim3((unsigned)(units * a.R / 8)), dim3(256), 0, st, pdl, a, r_log2);
}

}  // namespace lumo
