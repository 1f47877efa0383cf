// Device helpers shared by the kernels of the paged 4-bit cache.
#pragma once
#include <cuda_fp16.h>

#include "internal.h"

namespace lumo {

#ifdef __CUDACC__
__device__ __forceinline__ float exp2i(int e) {          // 2^e for |e| <= 126
  return __int_as_float((e + 127) << 23);
}
// e4m3 bits of a value >= 0: nearest, ties to even, at most 448
__device__ __forceinline__ uint32_t e4m3_of(float x) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(r) : "f"(0.f), "f"(x));
  return r & 0xFFu;
}
// two e4m3 numbers (low byte first) as f16 pair, exact
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(r) : "h"((unsigned short)two));
  return r;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  const uint32_t h = e4m3x2_to_half2(byte & 0xFFu);
  return __low2float(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float reciprocal(float x) {   // to about an ulp
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}
// eight e2m1 codes (the first in the lowest four bits): nearest, ties to the even code, at most 6
__device__ __forceinline__ uint32_t e2m1x8_of(const float2* x) {
  uint32_t r;
  asm("{\n.reg .b8 a, b, c, d;\n"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\ncvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\ncvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\nmov.b32 %0, {a, b, c, d};\n}\n"
      : "=r"(r) : "f"(x[0].x), "f"(x[0].y), "f"(x[1].x), "f"(x[1].y), "f"(x[2].x), "f"(x[2].y), "f"(x[3].x), "f"(x[3].y));
  return r;
}
// eight codes -> four f16 pairs, exact
__device__ __forceinline__ void e2m1x8_to_half2(uint32_t codes, uint32_t* h) {
  asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, a;\ncvt.rn.f16x2.e2m1x2 %1, b;\ncvt.rn.f16x2.e2m1x2 %2, c;\ncvt.rn.f16x2.e2m1x2 %3, d;\n}\n"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
}

// offset of the block of keys (which = 0) or values (1) of head h in page pg
__device__ __forceinline__ size_t kv4_block(int Hkv, int page, int pg, int h, int which) {
  return (((size_t)pg * Hkv + h) * 2 + which) * (size_t)(page * kKv4Entry);
}

// Row, length and pages of a sequence: the row exists, context plus suffix fit it, and every page of [ctx, ctx + Ns) exists (`writes`: and
// is this row's alone).  A pure function of its arguments: every thread, CTA and call reaches the same answer.
__device__ __forceinline__ int kv4_seq_check(const Kv4Shape& s, int ctx, int crow, bool writes) {
  const int st = seq_check(ctx, crow, s.Ns, s.n_rows, s.max_pages << s.page_log2);
  if (st != LUMO_SEQ_OK) return st;
  const int first = ctx >> s.page_log2, last = (ctx + s.Ns - 1) >> s.page_log2;
  int bad = 0;
  for (int i = first; i <= last; ++i) {                  // at most 17
    const int pg = s.table[(size_t)crow * s.max_pages + i];
    if (pg < 0 || pg >= s.n_pages || (writes && s.refs && s.refs[pg] != 1)) bad = 1;
  }
  return bad ? LUMO_SEQ_BAD_PAGE : LUMO_SEQ_OK;
}
// The same for one listed token; *pg is its page, -1 for a token that is passed over (row -1).
__device__ __forceinline__ int kv4_token_check(const Kv4Shape& s, int row, int pos, bool writes, int* pg) {
  *pg = -1;
  if (row == -1) return LUMO_SEQ_OK;
  if (row < 0 || row >= s.n_rows) return LUMO_SEQ_BAD_ROW;
  if (pos < 0 || (pos >> s.page_log2) >= s.max_pages) return LUMO_SEQ_BAD_CTX;
  const int p = s.table[(size_t)row * s.max_pages + (pos >> s.page_log2)];
  if (p < 0 || p >= s.n_pages || (writes && s.refs && s.refs[p] != 1)) return LUMO_SEQ_BAD_PAGE;
  *pg = p;
  return LUMO_SEQ_OK;
}
#endif

}  // namespace lumo
