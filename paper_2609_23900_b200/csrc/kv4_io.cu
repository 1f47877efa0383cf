// Entries of the paged 4-bit cache: written (the tree's through the slot map, or tokens listed one by one), read back in bf16, and moved
// at publication (sm_100a).  A head's 128 numbers are eight blocks of 16; a block is an e4m3 scale s and sixteen e2m1 codes c, and stands
// for c * s * 2^e (e: the layer's exponent, one for keys and one for values).
//
//   s = e4m3(max|x| 2^-e / 6), nearest, ties to even, at most 448; c = e2m1(x 2^-e / s), nearest, ties to the even code, at most 6;
//   s = 0: codes of zero; a block with a NaN: scale NaN, codes zero.
//
// The values are bf16, so a quotient that is not exactly on a border between two codes (or two scales) is at least 1/255 away from it,
// relatively: the product with the scale's reciprocal, rounded to the 11 bits of f16, lands on a border exactly when the quotient does.
// Likewise c * s has at most six significant bits: reading back in bf16 is exact.
//
// All of it is data movement: sixteen lanes a row of 128 numbers, 16 bytes of bf16 a lane.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

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
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max((w[i] << 16) & 0x7FFF0000u, w[i] & 0x7FFF0000u));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const bool nan = top > 0x7F800000u;
  uint32_t sb = e4m3_of(__uint_as_float(top) * down / 6.f);
  if (nan) sb = 0x7Fu;
  *scale_byte = sb;
  const float s = e4m3_value(sb);
  const float r = nan || s == 0.f ? 0.f : down / s;
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // to f16's 11 bits first (above); a value of a block without scale becomes a zero of its sign
    const __half2 q = __floats2half2_rn(__uint_as_float(w[i] << 16) * r, __uint_as_float(w[i] & 0xFFFF0000u) * r);
    codes |= e2m1x2_of(__low2float(q), __high2float(q)) << (8 * i);
  }
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

// Tokens listed one by one: entry of token t goes to position pos[t] of row row[t]; row -1 is passed over.  CTAs go through (token, round
// of rows) pairs, two in flight.
template <class KL>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(const KL L, const Kv4Shape s, const Kv4Tokens t) {
  const int l = blockIdx.y;
  const int lane16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int rows = 2 * s.Hkv;
  const long long items = (long long)t.T * rows; // one row each
  const long long step = (long long)gridDim.x * kGroups;
  const float down_k = exp2i(-s.k_exp), down_v = exp2i(-s.v_exp);
  struct Item { uint4 raw; unsigned char* blk; int at, which; bool ok; };
  auto fetch = [&](long long it) {
    Item x;
    x.ok = it < items;
    x.raw = make_uint4(0, 0, 0, 0);
    x.blk = nullptr; x.at = 0; x.which = 0;
    if (!x.ok) return x;
    const int tok = (int)(it / rows), r = (int)(it - (long long)tok * rows);
    x.which = r >= s.Hkv;
    const int h = x.which ? r - s.Hkv : r;
    x.raw = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(x.which ? L.vn[l] : L.kn[l]) + (long long)tok * s.kv_stride + h * 128) + lane16);
    int pg;
    const int st = kv4_token_check(s, t.row[tok], t.pos[tok], true, &pg);
    if (r == 0 && lane16 == 0 && L.status[l]) L.status[l][tok] = st;
    x.ok = st == LUMO_SEQ_OK && pg >= 0;
    x.at = t.pos[tok] & (s.page - 1);
    if (x.ok) x.blk = reinterpret_cast<unsigned char*>(L.pages[l]) + kv4_block(s.Hkv, s.page, pg, h, x.which);
    return x;
  };
  // uniform over the CTA: the shuffles see whole warps
  for (long long base = (long long)blockIdx.x * kGroups; base < items; base += 2 * step) {
    const Item a = fetch(base + grp), c = fetch(base + step + grp);
    store_row(a.blk + a.at * 64, a.blk + s.page * 64 + a.at * 8, a.raw, a.which ? down_v : down_k, lane16, a.ok);
    store_row(c.blk + c.at * 64, c.blk + s.page * 64 + c.at * 8, c.raw, c.which ? down_v : down_k, lane16, c.ok);
  }
}

// The way back: entries of the listed tokens in bf16 (exact); zeros for a token that fails its check or has row -1.
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(const unsigned char* pages, const Kv4Shape s, const Kv4Tokens t, __nv_bfloat16* k_out,
                                                            __nv_bfloat16* v_out, int32_t* status) {
  const int lane16 = threadIdx.x & 15, grp = threadIdx.x >> 4;
  pdl_wait();          // everything below may belong to earlier kernels
  pdl_trigger();
  const int rows = 2 * s.Hkv;
  const long long items = (long long)t.T * rows;
  const long long step = (long long)gridDim.x * kGroups;
  const float up_k = exp2i(s.k_exp), up_v = exp2i(s.v_exp);
  constexpr int kFlight = 4;
  for (long long base = (long long)blockIdx.x * kGroups + grp; base < items; base += kFlight * step) {
    uint32_t codes[kFlight], sb[kFlight];
    __nv_bfloat16* dst[kFlight];
    float up[kFlight];
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const long long it = base + f * step;
      dst[f] = nullptr; codes[f] = 0; sb[f] = 0; up[f] = 1.f;
      if (it >= items) continue;
      const int tok = (int)(it / rows), r = (int)(it - (long long)tok * rows);
      const int which = r >= s.Hkv, h = which ? r - s.Hkv : r;
      int pg;
      const int st = kv4_token_check(s, t.row[tok], t.pos[tok], false, &pg);
      if (r == 0 && lane16 == 0 && status) status[tok] = st;
      dst[f] = (which ? v_out : k_out) + ((long long)tok * s.Hkv + h) * 128 + lane16 * 8;
      up[f] = which ? up_v : up_k;
      if (st != LUMO_SEQ_OK || pg < 0) continue;
      const int at = t.pos[tok] & (s.page - 1);
      const unsigned char* blk = pages + kv4_block(s.Hkv, s.page, pg, h, which);
      codes[f] = reinterpret_cast<const uint32_t*>(blk + at * 64)[lane16];
      sb[f] = blk[s.page * 64 + at * 8 + (lane16 >> 1)];
    }
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      if (!dst[f]) continue;
      const float sc = e4m3_value(sb[f]) * up[f];
      uint32_t h2[4], w[4];
      e2m1x8_to_half2(codes[f], h2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h2[i]));
        const __nv_bfloat162 o = __floats2bfloat162_rn(v.x * sc, v.y * sc);
        w[i] = *reinterpret_cast<const uint32_t*>(&o);
      }
      *reinterpret_cast<uint4*>(dst[f]) = make_uint4(w[0], w[1], w[2], w[3]);
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

cudaError_t launch_kv4_write(const Kv4Layers& L, const Kv4Shape& s, int n_layers, int, bool pdl, cudaStream_t st) {
  const dim3 grid(s.N, s.B, n_layers);
  if (n_layers <= kFewLayers) return launch_kernel(kv4_write_kernel<FewKv4Layers>, grid, dim3(kThreads), 0, st, pdl, few_layers(L), s);
  return launch_kernel(kv4_write_kernel<Kv4Layers>, grid, dim3(kThreads), 0, st, pdl, L, s);
}

// CTAs for `items` rows: enough to fill the GPU, no more than there is work for
static unsigned row_ctas(long long items, int sms) {
  const long long want = (items + kGroups - 1) / kGroups, most = 8LL * sms;
  return (unsigned)(want < most ? want : most);
}

cudaError_t launch_kv4_append(const Kv4Layers& L, const Kv4Shape& s, int n_layers, const Kv4Tokens& t, int sms, bool pdl, cudaStream_t st) {
  const dim3 grid(row_ctas((long long)t.T * 2 * s.Hkv, sms), n_layers);
  if (n_layers <= kFewLayers) return launch_kernel(kv4_append_kernel<FewKv4Layers>, grid, dim3(kThreads), 0, st, pdl, few_layers(L), s, t);
  return launch_kernel(kv4_append_kernel<Kv4Layers>, grid, dim3(kThreads), 0, st, pdl, L, s, t);
}

cudaError_t launch_kv4_read(const void* pages, const Kv4Shape& s, const Kv4Tokens& t, void* k_out, void* v_out, int32_t* status, int sms,
                            bool pdl, cudaStream_t st) {
  const dim3 grid(row_ctas((long long)t.T * 2 * s.Hkv, sms));
  return launch_kernel(kv4_read_kernel, grid, dim3(kThreads), 0, st, pdl, reinterpret_cast<const unsigned char*>(pages), s, t,
                       reinterpret_cast<__nv_bfloat16*>(k_out), reinterpret_cast<__nv_bfloat16*>(v_out), status);
}

cudaError_t launch_kv4_publish(const Kv4Layers& L, const Kv4Shape& s, int n_layers, const int32_t* accepted, const int32_t* len, int lmax,
                               int32_t* ctx_len_out, bool pdl, cudaStream_t st) {
  const dim3 grid(2 * s.Hkv, s.B, n_layers);
  if (n_layers <= kFewLayers)
    return launch_kernel(kv4_publish_kernel<FewKv4Layers>, grid, dim3(kThreads), 0, st, pdl, few_layers(L), s, accepted, len, lmax, ctx_len_out);
  return launch_kernel(kv4_publish_kernel<Kv4Layers>, grid, dim3(kThreads), 0, st, pdl, L, s, accepted, len, lmax, ctx_len_out);
}

}  // namespace lumo
