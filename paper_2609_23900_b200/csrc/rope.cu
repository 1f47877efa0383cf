// Norm of every query and key head and the position rotation, in one pass (sm_100a).
//
//   y = x * rsqrt(mean(x^2) + eps) * (w + offset);   pairs (a, b) of y's first `rot` elements become
//   (a cos t - b sin t, a sin t + b cos t) * m,      t = position(axis of the pair) * inv_freq[pair]
//
// Each element is read once and written once; what bounds the kernel at a prompt's size is that traffic together with the instructions (97
// for two rows of 128, angles included).  A row (one head of one token) is held by dh / 8 lanes, so that both elements of a pair are in one
// lane; sums and products are fp32, rounded once at the end.  A warp takes one token and a run of its heads, without a barrier in the CTA: it
// works out the token's angles, in 64 bits (at position 10^6 an fp32 product is off by 0.03 rad), reduced to a fraction of a turn and
// handed to sincospif in fp32 (off by 2^-26 of a turn, 1e-7 rad, at most: what fp32 sines are good for), keeps cosines, sines and weights in registers as one factor an element, and goes through its heads with four rows
// per group of lanes on their way.
// Measured: 8192 tokens of 32 + 8 heads of 128 in bf16, 30.7 us, 5.5 TB/s (with partners fetched by shuffles 36.2, with a branch for elements
// that are not rotated 34.2); one token, and 224, 4.3 us (a launch).  The same bytes in the other forms: heads of 64 and 256 30.1 and 31.7,
// pairs 30.0 to 31.9 (heads of 64, 128, 256), fp32 (4096 tokens) 29.8 to 31.2, in pairs 30.4 to 32.0.
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

// a b + c where `on`, else c: one predicated instruction (as a branch it made the lanes of a warp part company in every row)
__device__ __forceinline__ float2 fma2_if(bool on, float2 a, float2 b, float2 c) {
  asm("{\n.reg .pred p;\nsetp.ne.u32 p, %3, 0;\n@p fma.rn.f32x2 %0, %1, %2, %0;\n}\n"
      : "+l"(reinterpret_cast<unsigned long long&>(c))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "r"((uint32_t)on));
  return c;
}

// two runs of four elements
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint2 a, b;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, const __nv_bfloat16* q) {       // (not the read-only path: outputs may be the inputs)
    a = *reinterpret_cast<const uint2*>(p);
    b = *reinterpret_cast<const uint2*>(q);
  }
  __device__ __forceinline__ void get(float2* f) const {
    const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, __nv_bfloat16* q, const float2* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(f[i].x, f[i].y);
      w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    *reinterpret_cast<uint2*>(q) = make_uint2(w[2], w[3]);
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, const float* q) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(q);
  }
  __device__ __forceinline__ void get(float2* f) const {
    f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
  }
  static __device__ __forceinline__ void store(float* p, float* q, const float2* f) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    *reinterpret_cast<float4*>(q) = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
  }
};

template <typename T> constexpr int kCtas = sizeof(T) == 2 ? 4 : 2;      // per SM (bf16: 31.4 us at 8192 tokens, three: 34.4)

// Warp w of the grid takes token w / chunks and the heads [(w % chunks) * per, + per) of q's and k's heads together.
template <typename T, int DH, bool kPairs>
__global__ void __launch_bounds__(kThreads, kCtas<T>) rope_kernel(const RopeArgs a, int chunks, int per) {
  constexpr int LPR = DH / 8;                 // lanes per row
  constexpr int NG = 32 / LPR;                // rows a warp works on at a time
  __shared__ __align__(16) float cs[kWarps][2][DH / 2];   // cosines, sines of the warp's token
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = a.rot >> 1;
  const int grp = lane / LPR, vi = lane % LPR;
  // This lane's elements: four from p0 on and four from p1 on.  Style "half": four of the first half and the four that they form pairs with;
  // style "pairs", and elements that are not rotated: eight in a row.
  const bool split = !kPairs && 4 * vi < half;
  const int p0 = split ? 4 * vi : 8 * vi;
  const int gap = split ? half : 4;
  const bool turned = p0 < a.rot;
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
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {      // queries, then keys
    const int H0 = kind ? a.Hq : 0, lo = max(h_lo, H0), hi = min(h_hi, kind ? a.Hq + a.Hkv : a.Hq);
    if (lo >= hi) continue;
    const long long in_st = kind ? a.k_stride : a.q_stride, out_st = kind ? a.k_out_stride : a.q_out_stride;
    const T* src = reinterpret_cast<const T*>(kind ? a.k : a.q) + tok * in_st + p0;
    T* dst = reinterpret_cast<T*>(kind ? a.k_out : a.q_out) + tok * out_st + p0;
    Raw8<T> raw[kFlight];
    int left = hi - lo - grp;                 // rows from this group's next one on
    src += (lo - H0 + grp) * DH;
    dst += (lo - H0 + grp) * DH;
    const T* src1 = src + gap;
    T* dst1 = dst + gap;
#pragma unroll
    for (int f = 0; f < kFlight; ++f)
      if (f * NG < left) raw[f].load(src + f * NG * DH, src1 + f * NG * DH);
    // y_i = inv (A_i x_i + B_i x_partner): weights, cosines and signed sines in one factor each
    float2 A[4], B[4];
    {
      float2 w[4], c[4], sn[4];
      const T* wt = reinterpret_cast<const T*>(a.norm ? (kind ? a.k_weight : a.q_weight) : nullptr);
#pragma unroll
      for (int i = 0; i < 4; ++i) { w[i] = c[i] = make_float2(1.f, 1.f); sn[i] = make_float2(0.f, 0.f); }
      if (wt) {
        Raw8<T> r;
        r.load(wt + p0, wt + p0 + gap);
        r.get(w);
        const float2 off = make_float2(a.weight_offset, a.weight_offset);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = add2(w[i], off);
      }
      if (turned) {
        const int j0 = kPairs ? p0 >> 1 : p0;
        const float4 cv = *reinterpret_cast<const float4*>(&cs[warp][0][j0]), sv = *reinterpret_cast<const float4*>(&cs[warp][1][j0]);
        if (kPairs) {
          c[0] = make_float2(cv.x, cv.x); c[1] = make_float2(cv.y, cv.y); c[2] = make_float2(cv.z, cv.z); c[3] = make_float2(cv.w, cv.w);
          sn[0] = make_float2(-sv.x, sv.x); sn[1] = make_float2(-sv.y, sv.y); sn[2] = make_float2(-sv.z, sv.z); sn[3] = make_float2(-sv.w, sv.w);
        } else {
          c[0] = c[2] = make_float2(cv.x, cv.y); c[1] = c[3] = make_float2(cv.z, cv.w);
          sn[2] = make_float2(sv.x, sv.y); sn[3] = make_float2(sv.z, sv.w);
          sn[0] = make_float2(-sv.x, -sv.y); sn[1] = make_float2(-sv.z, -sv.w);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        A[i] = mul2(w[i], c[i]);
        B[i] = mul2(kPairs ? make_float2(w[i].y, w[i].x) : w[i ^ 2], sn[i]);
      }
    }
    // whole warps go through this: a group beyond its heads works on what it has and stores nothing
    for (; left + grp > 0; left -= kFlight * NG, src += kFlight * NG * DH, src1 += kFlight * NG * DH, dst += kFlight * NG * DH, dst1 += kFlight * NG * DH) {
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        float2 x[4], y[4];
        raw[f].get(x);
        if ((kFlight + f) * NG < left) raw[f].load(src + (kFlight + f) * NG * DH, src1 + (kFlight + f) * NG * DH);
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
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[i] = mul2(A[i], x[i]);
          y[i] = fma2_if(turned, B[i], kPairs ? make_float2(x[i].y, x[i].x) : x[i ^ 2], y[i]);      // (not with factors of zero: x may be infinite)
        }
        const float2 inv2 = make_float2(inv, inv);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], inv2);
        if (f * NG < left) Raw8<T>::store(dst + f * NG * DH, dst1 + f * NG * DH, y);
      }
    }
  }
}

template <typename T, int DH>
cudaError_t launch_t(const RopeArgs& a, int sms, bool pdl, cudaStream_t st) {
  constexpr int NG = 32 * 8 / DH;
  const int H = a.Hq + a.Hkv;
  // Few tokens: as many warps a token as give the GPU sixteen an SM, down to one round of loads each.  Many tokens: a warp goes through all
  // heads of its token, and its angles are worked out once (two warps a token: 33.2 us instead of 30.7 at 8192 tokens of 40 heads; rows
  // dealt out evenly over a resident grid: no gain either).
  const long long rows_per_warp = ((long long)a.T * H + 16LL * sms - 1) / (16LL * sms);
  int per = (int)(rows_per_warp < H ? rows_per_warp : H);
  per = (per + NG - 1) / NG * NG;
  const int chunks = (H + per - 1) / per;
  const long long warps = (long long)a.T * chunks;
  const dim3 grid((unsigned)((warps + kWarps - 1) / kWarps));
  if (a.style == 1) return launch_kernel(rope_kernel<T, DH, true>, grid, dim3(kThreads), 0, st, pdl, a, chunks, per);
  return launch_kernel(rope_kernel<T, DH, false>, grid, dim3(kThreads), 0, st, pdl, a, chunks, per);
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
