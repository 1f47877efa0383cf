// Norm of every query and key head and the position rotation, in one pass (sm_100a).
//
//   y = x * rsqrt(mean(x^2) + eps) * (w + offset);   pairs (a, b) of y's first `rot` elements become
//   (a cos t - b sin t, a sin t + b cos t) * m,      t = position(axis of the pair) * inv_freq[pair]
//
// Bound by memory: each element is read once and written once.  A row (one head of one token) is held by dh / 8 lanes,
// 16 bytes (bf16) or 32 bytes (fp32) each; sums and products are fp32, rounded once at the end.  A warp takes one token and a run of its heads,
// without a barrier in the CTA: it works out the token's angles, in 64 bits (at position 10^6 an fp32 product is off by 0.03 rad), reduced
// to a fraction of a turn and handed to sincospif, keeps its cosines and sines in registers, and goes through its heads with four rows
// per group of lanes on their way.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "f32x2.h"
#include "internal.h"

namespace lumo {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kFlight = 4;                     // rows on their way per group of lanes
constexpr double kInvTwoPi = 0.15915494309189533577;

template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const void* p) { v = *reinterpret_cast<const uint4*>(p); }   // (not the read-only path: outputs may be the inputs)
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ Raw8 from(int lane, int width) const {
    Raw8 r;
    r.v.x = __shfl_sync(0xffffffffu, v.x, lane, width); r.v.y = __shfl_sync(0xffffffffu, v.y, lane, width);
    r.v.z = __shfl_sync(0xffffffffu, v.z, lane, width); r.v.w = __shfl_sync(0xffffffffu, v.w, lane, width);
    return r;
  }
  static __device__ __forceinline__ void store(void* p, const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ Raw8 from(int lane, int width) const {
    Raw8 r;
    r.a.x = __shfl_sync(0xffffffffu, a.x, lane, width); r.a.y = __shfl_sync(0xffffffffu, a.y, lane, width);
    r.a.z = __shfl_sync(0xffffffffu, a.z, lane, width); r.a.w = __shfl_sync(0xffffffffu, a.w, lane, width);
    r.b.x = __shfl_sync(0xffffffffu, b.x, lane, width); r.b.y = __shfl_sync(0xffffffffu, b.y, lane, width);
    r.b.z = __shfl_sync(0xffffffffu, b.z, lane, width); r.b.w = __shfl_sync(0xffffffffu, b.w, lane, width);
    return r;
  }
  static __device__ __forceinline__ void store(void* p, const float* f) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// Warp w of the grid takes token w / chunks and the heads [(w % chunks) * per, + per) of q's and k's heads together.
template <typename T, int DH>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 3 : 2) rope_kernel(const RopeArgs a, int chunks, int per) {
  constexpr int LPR = DH / 8;                 // lanes per row
  constexpr int NG = 32 / LPR;                // rows a warp works on at a time
  __shared__ __align__(16) float cs[kWarps][2][DH / 2];   // cosines, sines of the warp's token
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = a.rot >> 1;
  const int grp = lane / LPR, vi = lane % LPR, e0 = vi * 8;
  pdl_wait();                                 // everything below may belong to earlier kernels
  pdl_trigger();
  const long long w = (long long)blockIdx.x * kWarps + warp;
  const int tok = (int)(w / chunks);
  if (tok >= a.T) return;                     // (whole warps; no barrier follows)
  const int h_lo = (int)(w - (long long)tok * chunks) * per, h_hi = min(a.Hq + a.Hkv, h_lo + per);
  // the angles
  for (int j = lane; j < half; j += 32) {
    int pos;
    if (a.pos) {
      int ax = 0;                             // the pair's axis: blocks of sections, or taking turns while height and width last
      if (a.axes == 3) {
        if (a.turns) { const int r = j % 3; ax = r && j / 3 < a.section[r] ? r : 0; }
        else ax = j < a.section[0] ? 0 : (j < a.section[0] + a.section[1] ? 1 : 2);
      }
      pos = a.pos[(long long)ax * a.T + tok];
    } else {
      pos = a.ctx_len[tok / a.N] + a.depth[tok] - 1;
    }
    const double turn = (double)pos * (double)a.inv_freq[j] * kInvTwoPi;
    float s, c;
    sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
    cs[warp][0][j] = c * a.mscale;
    cs[warp][1][j] = s * a.mscale;
  }
  __syncwarp();
  // Where the other element of this lane's pairs is: style "half": rot / 16 lanes away; style "pairs": in this lane (the neighbour).
  const bool turned = e0 < a.rot;
  const int partner = !turned || a.style == 1 ? vi : (e0 < half ? vi + (half >> 3) : vi - (half >> 3));
  const bool within = a.style == 1;
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {      // queries, then keys
    const int H0 = kind ? a.Hq : 0, lo = max(h_lo, H0), hi = min(h_hi, kind ? a.Hq + a.Hkv : a.Hq);
    if (lo >= hi) continue;
    const long long in_st = kind ? a.k_stride : a.q_stride, out_st = kind ? a.k_out_stride : a.q_out_stride;
    const T* src = reinterpret_cast<const T*>(kind ? a.k : a.q) + tok * in_st + e0;
    T* dst = reinterpret_cast<T*>(kind ? a.k_out : a.q_out) + tok * out_st + e0;
    Raw8<T> raw[kFlight];
    int h = lo + grp - H0;
    const int n = hi - H0;
#pragma unroll
    for (int f = 0; f < kFlight; ++f)
      if (h + f * NG < n) raw[f].load(src + (h + f * NG) * DH);
    // y_i = inv (A_i x_i + B_i x_partner): weights, cosines and sines in one factor each
    float2 A[4], B[4];
    {
      // weights of this lane's elements and of their partners, cosines and signed sines
      float wf[8], wp[8], c[8], sn[8];
      const T* wt = reinterpret_cast<const T*>(a.norm ? (kind ? a.k_weight : a.q_weight) : nullptr);
#pragma unroll
      for (int i = 0; i < 8; ++i) { wf[i] = wp[i] = c[i] = 1.f; sn[i] = 0.f; }
      if (wt) {
        Raw8<T> r;
        r.load(wt + e0);
        r.get(wf);
        r.load(wt + partner * 8);
        r.get(wp);
#pragma unroll
        for (int i = 0; i < 8; ++i) { wf[i] += a.weight_offset; wp[i] += a.weight_offset; }
      }
      if (within) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) { const float x = wp[i]; wp[i] = wp[i + 1]; wp[i + 1] = x; }
      }
      if (turned && within) {
        const float4 cv = *reinterpret_cast<const float4*>(&cs[warp][0][e0 >> 1]), sv = *reinterpret_cast<const float4*>(&cs[warp][1][e0 >> 1]);
        c[0] = c[1] = cv.x; c[2] = c[3] = cv.y; c[4] = c[5] = cv.z; c[6] = c[7] = cv.w;
        sn[0] = -sv.x; sn[1] = sv.x; sn[2] = -sv.y; sn[3] = sv.y; sn[4] = -sv.z; sn[5] = sv.z; sn[6] = -sv.w; sn[7] = sv.w;
      } else if (turned) {
        const int j0 = e0 < half ? e0 : e0 - half;
        const float sign = e0 < half ? -1.f : 1.f;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          const float4 cv = *reinterpret_cast<const float4*>(&cs[warp][0][j0 + i]), sv = *reinterpret_cast<const float4*>(&cs[warp][1][j0 + i]);
          c[i] = cv.x; c[i + 1] = cv.y; c[i + 2] = cv.z; c[i + 3] = cv.w;
          sn[i] = sign * sv.x; sn[i + 1] = sign * sv.y; sn[i + 2] = sign * sv.z; sn[i + 3] = sign * sv.w;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        A[i] = make_float2(wf[2 * i] * c[2 * i], wf[2 * i + 1] * c[2 * i + 1]);
        B[i] = make_float2(wp[2 * i] * sn[2 * i], wp[2 * i + 1] * sn[2 * i + 1]);
      }
    }
    // whole warps go through this: a group beyond its heads works on what it has and stores nothing
    for (; h - grp < n; h += kFlight * NG) {
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        const int hh = h + f * NG;
        float2 x[4], y[4];
        Raw8<T> mine = raw[f];
        mine.get(reinterpret_cast<float*>(x));
        if (hh + kFlight * NG < n) raw[f].load(src + (hh + kFlight * NG) * DH);
        float inv = 1.f;
        if (a.norm) {
          float2 sq = mul2(x[0], x[0]);
#pragma unroll
          for (int i = 1; i < 4; ++i) sq = fma2(x[i], x[i], sq);
          float ss = sq.x + sq.y;
#pragma unroll
          for (int d = LPR / 2; d; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d, LPR);
          inv = rsqrtf(ss * (1.f / DH) + a.eps);
        }
        if (within) {
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = turned ? make_float2(x[i].y, x[i].x) : make_float2(0.f, 0.f);
        } else {
          mine = mine.from(partner, LPR);
          if (!turned) mine.clear();          // (whatever x holds)
          mine.get(reinterpret_cast<float*>(y));
        }
        const float2 inv2 = make_float2(inv, inv);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul2(fma2(B[i], y[i], mul2(A[i], x[i])), inv2);
        if (hh < n) Raw8<T>::store(dst + hh * DH, reinterpret_cast<const float*>(y));
      }
    }
  }
}

template <typename T, int DH>
cudaError_t launch_t(const RopeArgs& a, int sms, bool pdl, cudaStream_t st) {
  constexpr int NG = 32 * 8 / DH;
  const int H = a.Hq + a.Hkv;
  // Few tokens: as many warps a token as give the GPU sixteen an SM, down to one round of loads each.  Many tokens: a warp goes through all
  // heads of its token, and its angles are worked out once.
  const long long rows_per_warp = ((long long)a.T * H + 16LL * sms - 1) / (16LL * sms);
  int per = (int)(rows_per_warp < H ? rows_per_warp : H);
  per = (per + NG - 1) / NG * NG;
  const int chunks = (H + per - 1) / per;
  const long long warps = (long long)a.T * chunks;
  return launch_kernel(rope_kernel<T, DH>, dim3((unsigned)((warps + kWarps - 1) / kWarps)), dim3(kThreads), 0, st, pdl, a, chunks, per);
}

template <typename T>
cudaError_t launch_dh(const RopeArgs& a, int sms, bool pdl, cudaStream_t st) {
  if (a.dh == 64) return launch_t<T, 64>(a, sms, pdl, st);
  if (a.dh == 128) return launch_t<T, 128>(a, sms, pdl, st);
  return launch_t<T, 256>(a, sms, pdl, st);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, int dtype, int sms, bool pdl, cudaStream_t st) {
  return dtype == LUMO_BF16 ? launch_dh<__nv_bfloat16>(a, sms, pdl, st) : launch_dh<float>(a, sms, pdl, st);
}

}  // namespace lumo
