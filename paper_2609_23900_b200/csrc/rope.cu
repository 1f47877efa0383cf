// Norm of every query and key head and the position rotation, in one pass (sm_100a).
//
//   y = x * rsqrt(mean(x^2) + eps) * (w + offset);   pairs (a, b) of y's first `rot` elements become
//   (a cos t - b sin t, a sin t + b cos t) * m,      t = position(axis of the pair) * inv_freq[pair]
//
// Bound by memory: each element is read once and written once.  A row (one head of one token) is held by dh / 8 lanes,
// 16 bytes (bf16) or 32 bytes (fp32) each; sums and products are fp32, rounded once at the end.  The angles of a token are the
// same for all its heads: they are worked out once per token into shared memory, in 64 bits (at position 10^6 an fp32
// product is off by 0.03 rad), reduced to a fraction of a turn and handed to sincospif; a group of lanes then keeps its
// cosines and sines in registers while it goes through its heads.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "internal.h"

namespace lumo {

namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 4;                     // most tokens of a CTA
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
  static __device__ __forceinline__ void store(void* p, const float* f) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// grid (token groups, head chunks); a CTA covers tokens [x * tpc, ...) and heads [y * chunk, ...) of q's and k's heads together
template <typename T, int DH>
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeArgs a, int tpc, int chunk) {
  constexpr int LPR = DH / 8;                 // lanes per row
  constexpr int NG = kThreads / LPR;          // rows in flight per CTA
  __shared__ __align__(16) float cs[2][kTokens][DH / 2];       // cosines, sines: [token of the CTA][pair]
  const int tid = threadIdx.x, half = a.rot >> 1;
  pdl_wait();                                 // everything below may belong to earlier kernels
  pdl_trigger();
  const int t0 = blockIdx.x * tpc;
  const int H = a.Hq + a.Hkv;
  const int h_end = min(H, (int)(blockIdx.y + 1) * chunk);
  // this group's token and first head; its first row is requested ahead of the angles
  const int grp = tid / LPR, vi = tid % LPR;
  const int gpt = NG / tpc;                   // groups per token (tpc divides NG)
  const int tok_l = grp / gpt, tok = t0 + tok_l;
  int h = blockIdx.y * chunk + grp % gpt;
  const bool mine = tok < a.T;
  auto src = [&](int hh) {
    return hh < a.Hq ? reinterpret_cast<const T*>(a.q) + (long long)tok * a.q_stride + hh * DH + vi * 8
                     : reinterpret_cast<const T*>(a.k) + (long long)tok * a.k_stride + (hh - a.Hq) * DH + vi * 8;
  };
  Raw8<T> next;
  if (mine && h < h_end) next.load(src(h));
  for (int i = tid; i < tpc * half; i += kThreads) {
    const int tl = i / half, j = i - tl * half, t = t0 + tl;
    if (t < a.T) {
      int pos;
      if (a.pos) {
        int ax = 0;                           // the pair's axis: blocks of sections, or taking turns while height and width last
        if (a.axes == 3) {
          if (a.turns) { const int r = j % 3; ax = r && j / 3 < a.section[r] ? r : 0; }
          else ax = j < a.section[0] ? 0 : (j < a.section[0] + a.section[1] ? 1 : 2);
        }
        pos = a.pos[(long long)ax * a.T + t];
      } else {
        pos = a.ctx_len[t / a.N] + a.depth[t] - 1;
      }
      const double turn = (double)pos * (double)a.inv_freq[j] * kInvTwoPi;
      float s, c;
      sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
      cs[0][tl][j] = c * a.mscale;
      cs[1][tl][j] = s * a.mscale;
    }
  }
  __syncthreads();
  if (!mine) return;                          // whole groups leave; the shuffles below name their own group's lanes only
  const unsigned lanes = LPR == 32 ? 0xffffffffu : ((1u << LPR) - 1u) << ((tid & 31) / LPR * LPR);
  // this lane's part of the head: 0 first elements of the pairs, 1 second, 2 (style "pairs") both, 3 not rotated
  const int e0 = vi * 8;
  const int part = e0 >= a.rot ? 3 : (a.style == 1 ? 2 : (e0 < half ? 0 : 1));
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = 0.f; }
  if (part == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { c[i] = cs[0][tok_l][(e0 >> 1) + i]; s[i] = cs[1][tok_l][(e0 >> 1) + i]; }
  } else if (part < 2) {
    const int j0 = part ? e0 - half : e0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = cs[0][tok_l][j0 + i]; s[i] = part ? cs[1][tok_l][j0 + i] : -cs[1][tok_l][j0 + i]; }
  }
  // style "half": the other element of this lane's pairs is rot / 16 lanes away
  const int partner = part == 0 ? vi + (half >> 3) : (part == 1 ? vi - (half >> 3) : vi);
  for (; h < h_end; h += gpt) {
    const Raw8<T> raw = next;
    if (h + gpt < h_end) next.load(src(h + gpt));
    const bool is_q = h < a.Hq;
    float x[8];
    raw.get(x);
    if (a.norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
      for (int d = LPR / 2; d; d >>= 1) ss += __shfl_xor_sync(lanes, ss, d, LPR);
      const float inv = rsqrtf(ss * (1.f / DH) + a.eps);
      const T* w = reinterpret_cast<const T*>(is_q ? a.q_weight : a.k_weight);
      if (w) {
        float wf[8];
        Raw8<T> wr;
        wr.load(w + e0);
        wr.get(wf);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * (wf[i] + a.weight_offset);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= inv;
      }
    }
    if (a.style == 1) {
      if (part == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = x[2 * i], v = x[2 * i + 1];
          x[2 * i] = u * c[i] - v * s[i];
          x[2 * i + 1] = u * s[i] + v * c[i];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = __shfl_sync(lanes, x[i], partner, LPR);
        if (part < 2) x[i] = fmaf(y, s[i], x[i] * c[i]);
      }
    }
    T* dst = is_q ? reinterpret_cast<T*>(a.q_out) + (long long)tok * a.q_out_stride + h * DH + e0
                  : reinterpret_cast<T*>(a.k_out) + (long long)tok * a.k_out_stride + (h - a.Hq) * DH + e0;
    Raw8<T>::store(dst, x);
  }
}

template <typename T, int DH>
cudaError_t launch_t(const RopeArgs& a, int sms, bool pdl, cudaStream_t st) {
  constexpr int NG = kThreads * 8 / DH;
  const int H = a.Hq + a.Hkv;
  // Few tokens: one a CTA, and as many CTAs a token as its heads fill, so that a call of one token is one round of loads.  Many
  // tokens: four a CTA, each group of lanes keeping its angles through its share of the heads.
  const long long ctas1 = (long long)a.T * ((H + NG - 1) / NG);
  int tpc = 1, chunk = NG;
  if (ctas1 > 4LL * sms) {
    chunk = H;
    tpc = kTokens;
  }
  const dim3 grid((unsigned)((a.T + tpc - 1) / tpc), (unsigned)((H + chunk - 1) / chunk));
  return launch_kernel(rope_kernel<T, DH>, grid, dim3(kThreads), 0, st, pdl, a, tpc, chunk);
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
