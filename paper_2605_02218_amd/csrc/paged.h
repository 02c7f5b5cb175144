// Pieces shared by the kernels that work on a paged cache: the sequence of a row, the place of a position, 16-bit rows and 8-bit codes.
#pragma once
#include "common.h"
#include "kernels.h"

namespace covspec {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// The sequence that row t belongs to: the last s with start[s] <= t; -1 in front of the first one, S behind the last one.
__device__ __forceinline__ int seq_of(const int32_t* start, int S, int t) {
  int lo = 0, hi = S + 1;                       // the first index whose start is beyond t lies in lo .. hi
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= t) lo = mid + 1; else hi = mid;
  }
  return lo - 1;
}

// The same for a whole wave, lanes asking for tokens of their own: GROUPS runs of neighbouring lanes, one token each.  64 starts are compared at a
// time, so that up to 256 sequences take one or a few loads that do not wait for one another; beyond, halving takes fewer.
template <int GROUPS>
__device__ __forceinline__ int seq_of_wave(const int32_t* start, int S, int t) {
  if (S > 256) return seq_of(start, S, t);
  const int lane = threadIdx.x & 63, group = lane / (64 / GROUPS);
  int s = -1;
  for (int s0 = 0; s0 <= S; s0 += 64) {
    const int v = s0 + lane <= S ? start[s0 + lane] : 0x7FFFFFFF;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int n = __popcll(__ballot(v <= __builtin_amdgcn_readlane(t, g * (64 / GROUPS))));
      s += group == g ? n : 0;
    }
  }
  return s;
}

// Place of position `pos` of sequence s, counted in tokens of one key head's slots: (page * H + head) << shift | place.  -1: it does not exist.
__device__ __forceinline__ long place_of(const Paged& c, int s, long pos, int head) {
  if (pos < 0 || (pos >> c.page_shift) >= c.max_pages) return -1;
  const int page = c.pages[(long)s * c.max_pages + (pos >> c.page_shift)];
  if (page < 0 || page >= c.n_pages) return -1;
  return (((long)page * c.H + head) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
}

// Two values of a 16-bit type, to and from fp32; rounding to the nearest even.
template <int DT> struct Half;
template <> struct Half<DT_BF16> {
  static __device__ __forceinline__ f32x2_t unpack(uint32_t w) { return (f32x2_t){bf16lo_to_f32(w), bf16hi_to_f32(w)}; }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)a, (__bf16)b}); }
};
template <> struct Half<DT_F16> {
  static __device__ __forceinline__ f32x2_t unpack(uint32_t w) {
    const f16x2_t h = __builtin_bit_cast(f16x2_t, w);
    return (f32x2_t){(float)h[0], (float)h[1]};
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, (f16x2_t){(_Float16)a, (_Float16)b}); }
};

// Four 8-bit codes of a word to fp32.
template <int KEPT>
__device__ __forceinline__ f32x4_t decode4(uint32_t w) {
  if constexpr (KEPT == DT_I8) {
    return (f32x4_t){(float)(int8_t)(w & 0xFF), (float)(int8_t)(w >> 8 & 0xFF), (float)(int8_t)(w >> 16 & 0xFF), (float)(int8_t)(w >> 24)};
  } else {
    const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return (f32x4_t){a[0], a[1], b[0], b[1]};
  }
}

// Codes of a row: x ((1 / amax) Q) to the nearest, ties to even.
constexpr float kTiny = 0x1p-100f;              // smaller maxima: (1 / amax) Q and the products with it would leave the range of fp32

template <int KEPT> constexpr float kTop = KEPT == DT_I8 ? 127.f : 448.f;

template <int KEPT>
__device__ __forceinline__ uint32_t encode4(const float (&y)[4]) {
  if constexpr (KEPT == DT_I8) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)rintf(y[e]) & 0xFFu) << (8 * e);
    return w;
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  }
}

// 1 / step and step of a row's codes, from its largest magnitude as the bits of a float (NaN above infinity above the finite ones); false: not finite.
template <int KEPT>
__device__ __forceinline__ bool code_step(uint32_t top, float& inv, float& scale) {
  const float amax = __uint_as_float(top);
  const bool finite = top < 0x7F800000u;
  inv = finite && amax >= kTiny ? (1.f / amax) * kTop<KEPT> : 0.f;
  scale = !finite ? __uint_as_float(0x7FC00000u) : amax >= kTiny ? amax / kTop<KEPT> : 0.f;
  return finite;
}
template <int KEPT>
__device__ __forceinline__ uint32_t encode_row4(const float* x, float inv, bool finite) {
  float y[4];
#pragma unroll
  // three roundings: the largest may come out some parts in 2^23 above Q
  for (int e = 0; e < 4; ++e) y[e] = finite ? __builtin_amdgcn_fmed3f(x[e] * inv, -kTop<KEPT>, kTop<KEPT>) : 0.f;
  return encode4<KEPT>(y);
}

}  // namespace covspec
