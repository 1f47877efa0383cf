// Entries of the paged 4-bit cache: written (the tree's through the slot map, or tokens listed one by one), read back in bf16, and moved
// at publication (sm_100a).  A head's 128 numbers are eight blocks of 16; a block is an e4m3 scale s and sixteen e2m1 codes c, and stands
// for c * s * 2^e (e: the layer's exponent, one for keys and one for values).
//
//   s = e4m3(max|x| 2^-e / 6), nearest, ties to even, at most 448; c = e2m1(x 2^-e / s), nearest, ties to the even code, at most 6;
//   s = 0: codes of zero; a block with a NaN: scale NaN, codes zero.
//
// The values are bf16, so a quotient that is not exactly on a border between two codes (or two scales) is at least 1/255 away from it,
// relatively: a product with a reciprocal that is off by a few ulp, rounded to 11 or 12 bits, lands on a border exactly when the quotient
// does, and no division is needed.
// Likewise c * s has at most six significant bits: reading back in bf16 is exact.
//
// Sixteen lanes a row of 128 numbers, 16 bytes of bf16 a lane.  At a prompt's size neither the bytes nor the instructions (110 for two rows to
// quantise and store, 70 to read back) fill their units: 0.5 issued a cycle and scheduler with 40 % of the warps, most stalls on loads, and in
// the read on the barrier behind which the places are known.  Latency bounds it (8191 tokens of 8 heads, both ways: 23.6 us, 3.6 TB/s); a
// tree's entries take a launch.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "f32x2.h"
#include "internal.h"
#include "kv4.h"

namespace lumo {

namespace {

constexpr int kThreads = 256;
constexpr int kRowLanes = 16;
constexpr int kGroups = kThreads / kRowLanes;

// four bytes of codes (elements 0..7, two a byte, the even one low) and the block's scale of eight values held by this lane; the block's
// other eight are in the neighbouring lane (all 32 lanes call this)
__device__ __forceinline__ uint32_t quantise8(uint4 raw, float down, uint32_t* scale_byte) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  // the largest magnitude by bit pattern: a NaN is above infinity, infinity above everything else
  uint32_t top2 = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
  top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
  const uint32_t top = max(top2 << 16, top2 & 0xFFFF0000u);
  const bool nan = top > 0x7F800000u;
  const float six = fminf(__uint_as_float(top) * down * (1.f / 6.f), 1024.f);          // (beyond 448 is 448; a NaN is seen to below)
  const float wide = six * 4097.f;
  uint32_t sb = e4m3_of(wide - (wide - six));    // to twelve bits first
  if (nan) sb = 0x7Fu;
  *scale_byte = sb;
  const float s = e4m3_value(sb);
  const float r = nan || s == 0.f ? 0.f : down * reciprocal(s);
  const float2 r2 = make_float2(r, r);
  float2 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // to f16's 11 bits first; a value of a block without scale becomes a zero of its sign
    const float2 x = mul2(make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u)), r2);
    q[i] = __half22float2(__floats2half2_rn(x.x, x.y));
  }
  const uint32_t codes = e2m1x8_of(q);
  return nan ? 0u : codes;
}

// One row (a token's keys or values of a head) by sixteen lanes: quantise and store.  Every lane of the warp calls it.
__device__ __forceinline__ void store_row(unsigned char* entry_codes, unsigned char* entry_scales, uint4 raw, float down, int lane16, bool ok) {
  uint32_t sb;
  const uint32_t c = quantise8(raw, down, &sb);
  if (!ok) return;
  reinterpret_cast<uint32_t*>(entry_codes)[lane16] = c;
  if (!(lane16 & 1)) entry_scales[lane16 >> 1] = (unsigned char)sb;
}

// Tree entries: grid (node, sequence, layer).  Node i of sequence b goes to position ctx_len[b] + slot[b][i].  The whole stretch
// [ctx, ctx + Ns) is checked by every CTA of the sequence alike, so a sequence is written whole or not at all.
template <class KL>
__global__ void __launch_bounds__(kThreads) kv4_write_kernel(const KL L, const Kv4Shape s) {
  const int i = blockIdx.x, b = blockIdx.y, l = blockIdx.z;
  const int lane16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int rows = 2 * s.Hkv;                    // keys of all heads, then values
  const long long tok = (long long)b * s.N + i;
  auto src = [&](int r) {
    const int which = r >= s.Hkv, h = which ? r - s.Hkv : r;
    return reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(which ? L.vn[l] : L.kn[l]) + tok * s.kv_stride + h * 128) + lane16;
  };
  uint4 raw = make_uint4(0, 0, 0, 0);            // requested together with the numbers that say where it goes
  if (grp < rows) raw = __ldg(src(grp));
  const int ctx = s.ctx_len[b], crow = s.cache_row[b], slot = s.slot[tok];
  const int bad = kv4_seq_check(s, ctx, crow, true);
  if (L.status[l] && i == 0 && threadIdx.x == 0) L.status[l][b] = bad;
  if (bad != LUMO_SEQ_OK) return;
  const int p = ctx + slot;
  const int pg = s.table[(size_t)crow * s.max_pages + (p >> s.page_log2)];
  const int at = p & (s.page - 1);
  const float down_k = exp2i(-s.k_exp), down_v = exp2i(-s.v_exp);
  for (int r0 = 0; r0 < rows; r0 += kGroups) {   // uniform over the CTA: the shuffles see whole warps
    const int r = r0 + grp;
    const bool ok = r < rows;
    if (r0) raw = ok ? __ldg(src(r)) : make_uint4(0, 0, 0, 0);
    const int which = r >= s.Hkv, h = which ? r - s.Hkv : r;
    unsigned char* blk = reinterpret_cast<unsigned char*>(L.pages[l]) + kv4_block(s.Hkv, s.page, pg, ok ? h : 0, which);
    store_row(blk + at * 64, blk + s.page * 64 + at * 8, raw, which ? down_v : down_k, lane16, ok);
  }
}

// Where the listed tokens of a CTA lie: offset of the page's first block, position in the page, whether there is such a place.
constexpr int kMostTokens = 32;
struct __align__(16) Place { long long page; int at; int ok; };
// How the sixteen-lane groups of a CTA go through n tokens of `rows` rows: a group keeps its row (of every pass of sixteen) and takes every
// `side`-th token, so that addresses run on by a constant; with fewer than sixteen rows, groups beyond the last whole token rest.
struct Walk {
  int side, token, row;      // tokens side by side; this group's first token; its row in the first pass
  __device__ __forceinline__ Walk(int grp, int rows) {
    side = rows >= kGroups ? 1 : kGroups / rows;
    token = rows >= kGroups ? 0 : grp / rows;
    row = grp - token * rows;
  }
};
__device__ __forceinline__ void find_places(const Kv4Shape& s, const Kv4Tokens& t, int t0, int n, bool writes, bool report, Place* p) {
  const int i = threadIdx.x;
  if (i >= n) return;
  const int tok = t0 + i;
  const int row = t.row[tok], pos = t.pos[tok];
  int pg;
  const int st = kv4_token_check(s, row, pos, writes, &pg);
  if (report && t.status) t.status[tok] = st;
  p[i] = {(long long)kv4_block(s.Hkv, s.page, pg < 0 ? 0 : pg, 0, 0), pos & (s.page - 1), st == LUMO_SEQ_OK && pg >= 0};
}

// Tokens listed one by one: entry of token t goes to position pos[t] of row row[t]; row -1 is passed over.  A CTA takes `per` tokens: their
// places are looked up once, by a thread each, while the first rows are on their way; four rows in flight per sixteen lanes.
template <class KL>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(const KL L, const Kv4Shape s, const Kv4Tokens t, int per) {
  constexpr int kFlight = 4;
  __shared__ Place places[kMostTokens];
  const int l = blockIdx.y, t0 = blockIdx.x * per, n = min(per, t.T - t0);
  const int lane16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int rows = 2 * s.Hkv;
  const Walk walk(grp, rows);
  bool known = false;
  for (int r0 = 0; r0 < rows; r0 += kGroups) {   // (uniform over the CTA, like the loop below: the shuffles see whole warps)
    const int r = r0 + walk.row, which = r >= s.Hkv, h = which ? r - s.Hkv : r;      // keys of all heads, then values
    const bool mine = r < rows && walk.token < walk.side;
    const float down = exp2i(which ? -s.v_exp : -s.k_exp);
    const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(which ? L.vn[l] : L.kn[l]) + (t0 + walk.token) * s.kv_stride + h * 128 + lane16 * 8;
    unsigned char* blk = reinterpret_cast<unsigned char*>(L.pages[l]) + (2 * h + which) * (s.page * kKv4Entry);
    const long long step = walk.side * s.kv_stride;
    for (int k0 = 0; k0 < n; k0 += kFlight * walk.side, src += kFlight * step) {
      uint4 raw[kFlight];
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        raw[f] = make_uint4(0, 0, 0, 0);
        if (mine && k0 + f * walk.side + walk.token < n) raw[f] = __ldg(reinterpret_cast<const uint4*>(src + f * step));
      }
      if (!known) {                              // the places are looked up while the first rows are on their way
        find_places(s, t, t0, n, true, l == 0, places);
        __syncthreads();
        known = true;
      }
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        const int k = k0 + f * walk.side + walk.token;
        const bool in = mine && k < n;
        const Place pl = places[in ? k : 0];
        unsigned char* page = blk + pl.page;
        store_row(page + pl.at * 64, page + s.page * 64 + pl.at * 8, raw[f], down, lane16, in && pl.ok);
      }
    }
  }
}

// The way back: entries of the listed tokens in bf16 (exact); zeros for a token that fails its check or has row -1.
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(const unsigned char* pages, const Kv4Shape s, const Kv4Tokens t, __nv_bfloat16* k_out,
                                                            __nv_bfloat16* v_out, int per) {
  constexpr int kFlight = 8;
  __shared__ Place places[kMostTokens];
  const int t0 = blockIdx.x * per, n = min(per, t.T - t0);
  const int lane16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int rows = 2 * s.Hkv;
  const Walk walk(grp, rows);
  find_places(s, t, t0, n, false, true, places);
  __syncthreads();
  if (walk.token >= walk.side) return;
  for (int r = walk.row; r < rows; r += kGroups) {
    const int which = r >= s.Hkv, h = which ? r - s.Hkv : r;
    const float up = exp2i(which ? s.v_exp : s.k_exp);
    const unsigned char* blk = pages + (2 * h + which) * (s.page * kKv4Entry);
    uint4* dst = reinterpret_cast<uint4*>((which ? v_out : k_out) + ((long long)(t0 + walk.token) * s.Hkv + h) * 128) + lane16;
    const int step = walk.side * s.Hkv * 16;
    for (int k0 = walk.token; k0 < n; k0 += kFlight * walk.side, dst += kFlight * (long long)step) {
      uint32_t codes[kFlight], sb[kFlight];
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        const int k = k0 + f * walk.side;
        const Place pl = places[k < n ? k : 0];
        codes[f] = 0; sb[f] = 0;
        if (k < n && pl.ok) {
          const unsigned char* page = blk + pl.page;
          codes[f] = reinterpret_cast<const uint32_t*>(page + pl.at * 64)[lane16];
          sb[f] = page[s.page * 64 + pl.at * 8 + (lane16 >> 1)];
        }
      }
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        if (k0 + f * walk.side >= n) continue;
        const float sc = e4m3_value(sb[f]) * up;
        uint32_t h2[4], w[4];
        e2m1x8_to_half2(codes[f], h2);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 v = mul2(__half22float2(*reinterpret_cast<const __half2*>(&h2[k])), make_float2(sc, sc));
          const __nv_bfloat162 o = __floats2bfloat162_rn(v.x, v.y);
          w[k] = *reinterpret_cast<const uint32_t*>(&o);
        }
        dst[(long long)f * step] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

// Publication: grid (KV head x {K, V}, sequence, layer).  A CTA stages the 72-byte entries of all accepted nodes that have to move in shared
// memory, then writes them: all reads come before any write, and entries of different heads never overlap.
template <class KL>
__global__ void __launch_bounds__(kThreads) kv4_publish_kernel(const KL L, const Kv4Shape s, const int32_t* __restrict__ accepted,
                                                               const int32_t* __restrict__ len, int lmax, int32_t* ctx_len_out) {
  __shared__ uint2 stage[kMaxNodes * 9];         // an entry: eight pieces of codes, one of scales
  __shared__ int acc_s[kMaxNodes], par_s[kMaxNodes], src_s[kMaxNodes];
  __shared__ int st_s;
  const int h = blockIdx.x >> 1, which = blockIdx.x & 1, b = blockIdx.y, l = blockIdx.z;
  const int tid = threadIdx.x;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int ctx = s.ctx_len[b], crow = s.cache_row[b];
  const int n = len[b];
  const int nn = n < 0 ? 0 : (n > lmax ? lmax : n);
  for (int t = tid; t < lmax; t += blockDim.x) {
    const int a = accepted[(size_t)b * lmax + t];
    acc_s[t] = a;
    const bool in = a >= 0 && a < s.N;
    par_s[t] = in ? s.parent[(size_t)b * s.N + a] : -2;
    src_s[t] = in ? s.slot[(size_t)b * s.N + a] : 0;
  }
  __syncthreads();
  const int seq = kv4_seq_check(s, ctx, crow, true);       // the same answer in every thread
  if (tid == 0) {
    int st = seq;
    if (st == LUMO_SEQ_OK) st = check_path_staged(acc_s, par_s, s.N, n, lmax);
    st_s = st;
    const bool lead = blockIdx.x == 0;
    if (lead && L.status[l]) L.status[l][b] = st;
    if (lead && l == 0 && ctx_len_out) ctx_len_out[b] = st == LUMO_SEQ_OK ? ctx + n : ctx;
  }
  __syncthreads();
  if (st_s != LUMO_SEQ_OK) return;
  unsigned char* pages = reinterpret_cast<unsigned char*>(L.pages[l]);
  auto piece = [&](int pos, int j) {
    const int pg = s.table[(size_t)crow * s.max_pages + (pos >> s.page_log2)], at = pos & (s.page - 1);
    unsigned char* blk = pages + kv4_block(s.Hkv, s.page, pg, h, which);
    return reinterpret_cast<uint2*>(j < 8 ? blk + at * 64 + j * 8 : blk + s.page * 64 + at * 8);
  };
  for (int c = tid; c < nn * 9; c += blockDim.x) {
    const int t = c / 9, j = c - t * 9;
    if (src_s[t] != t) stage[c] = *piece(ctx + src_s[t], j);
  }
  __syncthreads();
  for (int c = tid; c < nn * 9; c += blockDim.x) {
    const int t = c / 9, j = c - t * 9;
    if (src_s[t] != t) *piece(ctx + t, j) = stage[c];
  }
}

}  // namespace

cudaError_t launch_kv4_write(const Kv4Layers& L, const Kv4Shape& s, int n_layers, bool pdl, cudaStream_t st) {
  const dim3 grid(s.N, s.B, n_layers);
  if (n_layers <= kFewLayers) return launch_kernel(kv4_write_kernel<FewKv4Layers>, grid, dim3(kThreads), 0, st, pdl, few_layers(L), s);
  return launch_kernel(kv4_write_kernel<Kv4Layers>, grid, dim3(kThreads), 0, st, pdl, L, s);
}

// Tokens a CTA takes: 128 rows' worth (8191 tokens of 8 KV heads appended and read back: 23.6 us; 64 rows: 27.6, 192: 24.9), fewer while the
// GPU is not covered.
static int tokens_per_cta(int T, int Hkv, int sms) {
  int per = 128 / (2 * Hkv);
  per = per < 1 ? 1 : (per > kMostTokens ? kMostTokens : per);
  while (per > 1 && (T + per - 1) / per < 2 * sms) per /= 2;
  return per;
}

cudaError_t launch_kv4_append(const Kv4Layers& L, const Kv4Shape& s, int n_layers, const Kv4Tokens& t, int sms, bool pdl, cudaStream_t st) {
  const int per = tokens_per_cta(t.T, s.Hkv, sms);
  const dim3 grid((t.T + per - 1) / per, n_layers);
  if (n_layers <= kFewLayers) return launch_kernel(kv4_append_kernel<FewKv4Layers>, grid, dim3(kThreads), 0, st, pdl, few_layers(L), s, t, per);
  return launch_kernel(kv4_append_kernel<Kv4Layers>, grid, dim3(kThreads), 0, st, pdl, L, s, t, per);
}

cudaError_t launch_kv4_read(const void* pages, const Kv4Shape& s, const Kv4Tokens& t, void* k_out, void* v_out, int sms,
                            bool pdl, cudaStream_t st) {
  const int per = tokens_per_cta(t.T, s.Hkv, sms);
  return launch_kernel(kv4_read_kernel, dim3((t.T + per - 1) / per), dim3(kThreads), 0, st, pdl, reinterpret_cast<const unsigned char*>(pages), s, t,
                       reinterpret_cast<__nv_bfloat16*>(k_out), reinterpret_cast<__nv_bfloat16*>(v_out), per);
}

cudaError_t launch_kv4_publish(const Kv4Layers& L, const Kv4Shape& s, int n_layers, const int32_t* accepted, const int32_t* len, int lmax,
                               int32_t* ctx_len_out, bool pdl, cudaStream_t st) {
  const dim3 grid(2 * s.Hkv, s.B, n_layers);
  if (n_layers <= kFewLayers)
    return launch_kernel(kv4_publish_kernel<FewKv4Layers>, grid, dim3(kThreads), 0, st, pdl, few_layers(L), s, accepted, len, lmax, ctx_len_out);
  return launch_kernel(kv4_publish_kernel<Kv4Layers>, grid, dim3(kThreads), 0, st, pdl, L, s, accepted, len, lmax, ctx_len_out);
}

}  // namespace lumo
