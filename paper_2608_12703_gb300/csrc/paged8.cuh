// A paged K/V cache held in 8 bits: e4m3 codes and one scale for each group of
// 16 slots and head.
#pragma once

#include "paged.cuh"

namespace asrspec {

constexpr float E4M3_MAX = 448.f;

// The cache as the kernels see it: the view of its codes (one byte an element)
// and where the scales lie, in elements.
struct Paged8View {
  PagedView c;
  float *k_scale, *v_scale;
  long long s_page, s_head;
  int dim;
  __device__ __forceinline__ long long scale_at(int pid, int kvh, int grp) const {
    const int in_page = grp - (int)(c.groups.div((uint32_t)grp) * c.groups.d);
    return pid * s_page + kvh * s_head + in_page;
  }
};

// Two floats to e4m3 (nearest even, magnitudes above 448 become 448, NaN its code): lo in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t v;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(hi), "f"(lo));
  return v;
}
// The values of two codes, exact.
__device__ __forceinline__ float2 e4m3x2_value(uint32_t v) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)v));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}

// Two codes of the low half of w to fp16: .x the low byte.
__device__ __forceinline__ uint32_t half2_of(uint32_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
  return h;
}
// Two fp16 numbers as they are, infinities as NaN: 0 x + x.  A row of q with an infinity in it then has no score but NaN;
// left as it is, a row whose scores are all -inf would look like one that sees no slot.
__device__ __forceinline__ uint32_t nan_for_inf(uint32_t x) {
  uint32_t y;
  asm("fma.rn.f16x2 %0, %1, %2, %1;" : "=r"(y) : "r"(x), "r"(0));
  return y;
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127
// Bytes of x that are a NaN code, as a mask.
__device__ __forceinline__ uint32_t nan_codes(uint32_t x) {
  const uint32_t top = ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (top >> 7) * 0xffu;
}

// ---- Host: argument checks and launches shared by the entry points -----------
int paged8_view(const asr_paged8_cache* c, Paged8View* v);
int paged8_writable(const asr_paged8_cache* c);   // of checked ones: whether rows may be appended
int paged8_rows(const asr_paged8_cache* c, const asr_paged_rows* r, int dtype, PagedRows* v);
cudaError_t launch_append8(const Paged8View& c, const PagedRows& r, int dtype, cudaStream_t st);
// Attention of many rows (dtype 1 or 2), whose K/V are in the pages.  counts: 2, zero between calls.
cudaError_t launch_prompt8(const Paged8View& c, const PagedRows& r, int dtype, void* out, float* lse, int* counts, bool appended,
                           cudaStream_t st);

}  // namespace asrspec
