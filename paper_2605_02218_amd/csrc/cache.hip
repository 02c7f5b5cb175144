// Paged cache of keys and values: rows of new tokens into it, in 16 bits or quantised to 8, and positions back out of it.
//
// A row is the D values of one token and key head.  In 8 bits amax = max |x|, scale = amax / Q, code = x (Q / amax) to the nearest, ties to even
// (Q = 127 for integers, 448 for e4m3): a code is off by at most half a step, so |x - scale code| <= scale / 2 for integers.
//
// D / 8 lanes take a row of k and the same row of v, 16 bytes of each, so that the maximum is four exchanges inside a row of 16 lanes and every
// access is whole: 2 D bytes of a row in, D or 2 D out.  Both kernels only move data.
#include <type_traits>

#include "paged.h"

namespace covspec {

namespace {

constexpr int CT = 256;

// lanes of a row: a power of two, so that exchanges stay inside; head dimension 96 leaves a quarter of them without work
constexpr int row_lanes(int D) { return D == 64 ? 8 : 16; }
constexpr float kTiny = 0x1p-100f;              // smaller maxima: Q / amax and the products with it would leave the range of fp32

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

// Codes of the row that LANES neighbouring lanes hold eight values of each; the scale is the same in all of them.
template <int DT, int KEPT, int LANES>
__device__ __forceinline__ u32x2_t quantise(const u32x4_t& raw, float& scale) {
  float x[8];
  uint32_t top = 0;                              // |x| as integers: NaN above infinity above the finite ones
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x2_t p = Half<DT>::unpack(raw[e]);
    x[2 * e] = p[0];
    x[2 * e + 1] = p[1];
    top = max(top, max(__float_as_uint(p[0]) & 0x7FFFFFFFu, __float_as_uint(p[1]) & 0x7FFFFFFFu));
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  const float amax = __uint_as_float(top);
  const bool finite = top < 0x7F800000u;
  const float inv = finite && amax >= kTiny ? kTop<KEPT> / amax : 0.f;
  scale = !finite ? __uint_as_float(0x7FC00000u) : amax >= kTiny ? amax / kTop<KEPT> : 0.f;
  u32x2_t out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float y[4];
#pragma unroll
    // inv has one rounding and the product another: the largest may come out one part in 2^23 above Q
    for (int e = 0; e < 4; ++e) y[e] = finite ? __builtin_amdgcn_fmed3f(x[4 * h + e] * inv, -kTop<KEPT>, kTop<KEPT>) : 0.f;
    out[h] = encode4<KEPT>(y);
  }
  return out;
}

template <int DT, int KEPT, int D>
__global__ __launch_bounds__(CT) void cache_write_kernel(Paged c, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, long pitch,
                                                         void* __restrict__ kc, void* __restrict__ vc, float* __restrict__ ks, float* __restrict__ vs) {
  constexpr int LANES = row_lanes(D);
  const int lane = threadIdx.x & (LANES - 1);
  const long row = (long)blockIdx.x * (CT / LANES) + threadIdx.x / LANES;
  const int t = (int)(row / c.H), h = (int)(row % c.H);
  long to = -1;
  if (t < c.T) {
    const int s = seq_of(c.start, c.S, t);
    if (s >= 0 && s < c.S) to = place_of(c, s, (long)c.length[s] - c.start[s + 1] + t, h);
  }
  // the lanes of a row take part in its exchanges together
  const bool has = to >= 0, mine = has && lane * 8 < D;
  const long from = t * pitch + h * D + lane * 8;
  u32x4_t a = {}, b = {};
  if (mine) {
    a = *(const u32x4_t*)(k + from);
    b = *(const u32x4_t*)(v + from);
  }
  if constexpr (KEPT == DT) {
    if (mine) {
      *(u32x4_t*)((uint16_t*)kc + to * D + lane * 8) = a;
      *(u32x4_t*)((uint16_t*)vc + to * D + lane * 8) = b;
    }
  } else {
    float sa, sb;
    const u32x2_t ca = quantise<DT, KEPT, LANES>(a, sa), cb = quantise<DT, KEPT, LANES>(b, sb);
    if (mine) {
      *(u32x2_t*)((uint8_t*)kc + to * D + lane * 8) = ca;
      *(u32x2_t*)((uint8_t*)vc + to * D + lane * 8) = cb;
      if (lane == 0) { ks[to] = sa; vs[to] = sb; }
    }
  }
}

template <int DT, int KEPT, int D>
__device__ __forceinline__ u32x4_t read8(const void* codes, const float* scale, long at, int lane) {
  if (at < 0) return (u32x4_t){};
  if constexpr (KEPT == DT) {
    return *(const u32x4_t*)((const uint16_t*)codes + at * D + lane * 8);
  } else {
    const u32x2_t w = *(const u32x2_t*)((const uint8_t*)codes + at * D + lane * 8);
    const float s = scale[at];
    const f32x4_t a = decode4<KEPT>(w[0]), b = decode4<KEPT>(w[1]);
    return (u32x4_t){Half<DT>::pack(a[0] * s, a[1] * s), Half<DT>::pack(a[2] * s, a[3] * s), Half<DT>::pack(b[0] * s, b[1] * s),
                     Half<DT>::pack(b[2] * s, b[3] * s)};
  }
}

template <int DT, int KEPT, int D>
__global__ __launch_bounds__(CT) void cache_read_kernel(Paged c, const void* __restrict__ kc, const void* __restrict__ vc, const float* __restrict__ ks,
                                                        const float* __restrict__ vs, uint16_t* __restrict__ k, uint16_t* __restrict__ v, long pitch) {
  constexpr int LANES = row_lanes(D);
  const int lane = threadIdx.x & (LANES - 1);
  const long row = (long)blockIdx.x * (CT / LANES) + threadIdx.x / LANES;
  const int t = (int)(row / c.H), h = (int)(row % c.H);
  if (t >= c.T || lane * 8 >= D) return;
  const int s = seq_of(c.start, c.S, t);
  if (s < 0 || s >= c.S) return;                // a padding row
  const long at = place_of(c, s, (long)c.length[s] - c.start[s + 1] + t, h);
  const u32x4_t a = read8<DT, KEPT, D>(kc, ks, at, lane), b = read8<DT, KEPT, D>(vc, vs, at, lane);
  const long to = t * pitch + h * D + lane * 8;
  *(u32x4_t*)(k + to) = a;
  *(u32x4_t*)(v + to) = b;
}

}  // namespace

// f(kind of 16-bit type, kind of cache, head dimension) with the three as constants
template <typename F>
static hipError_t with_forms(const Paged& c, F f) {
  auto dims = [&](auto dt, auto kept) {
    if (c.D == 64) return f(dt, kept, std::integral_constant<int, 64>{});
    if (c.D == 96) return f(dt, kept, std::integral_constant<int, 96>{});
    if (c.D == 128) return f(dt, kept, std::integral_constant<int, 128>{});
    return hipErrorInvalidValue;
  };
  auto kinds = [&](auto dt) {
    if (c.kept == dt.value) return dims(dt, dt);
    if (c.kept == DT_I8) return dims(dt, std::integral_constant<int, DT_I8>{});
    if (c.kept == DT_E4M3) return dims(dt, std::integral_constant<int, DT_E4M3>{});
    return hipErrorInvalidValue;
  };
  if (c.dtype == DT_BF16) return kinds(std::integral_constant<int, DT_BF16>{});
  if (c.dtype == DT_F16) return kinds(std::integral_constant<int, DT_F16>{});
  return hipErrorInvalidValue;
}

hipError_t launch_cache_write(const Paged& c, const void* k, const void* v, long pitch, void* kc, void* vc, float* ks, float* vs, hipStream_t stream) {
  return with_forms(c, [&](auto dt, auto kept, auto dim) {
    constexpr int rows = CT / row_lanes(dim.value);
    const unsigned grid = (unsigned)(((long)c.T * c.H + rows - 1) / rows);
    hipLaunchKernelGGL((cache_write_kernel<dt.value, kept.value, dim.value>), dim3(grid), dim3(CT), 0, stream, c, (const uint16_t*)k, (const uint16_t*)v,
                       pitch, kc, vc, ks, vs);
    return hipGetLastError();
  });
}

hipError_t launch_cache_read(const Paged& c, const void* kc, const void* vc, const float* ks, const float* vs, void* k, void* v, long pitch,
                             hipStream_t stream) {
  return with_forms(c, [&](auto dt, auto kept, auto dim) {
    constexpr int rows = CT / row_lanes(dim.value);
    const unsigned grid = (unsigned)(((long)c.T * c.H + rows - 1) / rows);
    hipLaunchKernelGGL((cache_read_kernel<dt.value, kept.value, dim.value>), dim3(grid), dim3(CT), 0, stream, c, kc, vc, ks, vs, (uint16_t*)k, (uint16_t*)v,
                       pitch);
    return hipGetLastError();
  });
}

}  // namespace covspec
