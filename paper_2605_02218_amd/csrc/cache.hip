// Paged cache of keys and values: rows of new tokens into it, in 16 bits or quantised to 8, and positions back out of it.
//
// A row is the D values of one token and key head.  In 8 bits amax = max |x|, scale = amax / Q, code = x ((1 / amax) Q) to the nearest, ties to even
// (Q = 127 for integers, 448 for e4m3): a code is off by at most half a step, so |x - scale code| <= scale / 2 for integers.
//
// D / 8 lanes take a row of k and the same row of v, 16 bytes of each, so that the maximum is four exchanges inside a row of 16 lanes and every
// access is whole: 2 D bytes of a row in, D or 2 D out.  Both kernels only move data.
#include <type_traits>

#include "paged.h"

namespace covspec {

namespace {

constexpr int CT = 256;
// Neighbouring heads of a token that a lane takes.  us: 16 caches of 1500 to 6000 tokens read from 8 bits (8 heads, head dimension 128) 88 with one head,
// 71.5 with two, 75 with four, 113 with eight; 8 x 3008 tokens written to e4m3 36.6, 33.8, 34.1, 35.5.
constexpr int HEADS = 2;

// lanes of a row: a power of two, so that exchanges stay inside; head dimension 96 leaves a quarter of them without work
constexpr int row_lanes(int D) { return D == 64 ? 8 : 16; }
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
  float inv;
  const bool finite = code_step<KEPT>(top, inv, scale);
  u32x2_t out;
#pragma unroll
  for (int h = 0; h < 2; ++h) out[h] = encode_row4<KEPT>(x + 4 * h, inv, finite);
  return out;
}

// Which heads of which token the lanes of a row take: HEADS neighbouring heads, so that the sequence and the page are looked up once for them and
// their rows are on their way together.
struct Mine { int token, head0; long place; bool padding; };
template <int LANES>
__device__ __forceinline__ Mine find(const Paged& c, int groups) {
  const long x = (long)blockIdx.x * (CT / LANES) + threadIdx.x / LANES;
  Mine m;
  m.token = (int)(x / groups);
  m.head0 = (int)(x % groups) * HEADS;
  const int s = seq_of_wave<64 / LANES>(c.start, c.S, m.token < c.T ? m.token : 0x7FFFFFFF);
  m.padding = m.token >= c.T || s < 0 || s >= c.S;
  m.place = m.padding ? -1 : place_of(c, s, (long)c.length[s] - c.start[s + 1] + m.token, m.head0);
  return m;
}

template <int DT, int KEPT, int D>
__global__ __launch_bounds__(CT) void cache_write_kernel(Paged c, int groups, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, long pitch,
                                                         void* __restrict__ kc, void* __restrict__ vc, float* __restrict__ ks, float* __restrict__ vs) {
  constexpr int LANES = row_lanes(D);
  const int lane = threadIdx.x & (LANES - 1);
  const Mine m = find<LANES>(c, groups);
  // the lanes of a row take part in its exchanges together
  const bool mine = m.place >= 0 && lane * 8 < D;
  const long from = m.token * pitch + m.head0 * D + lane * 8;
  u32x4_t a[HEADS], b[HEADS];
#pragma unroll
  for (int h = 0; h < HEADS; ++h) {
    a[h] = b[h] = (u32x4_t){};
    if (mine && m.head0 + h < c.H) {
      a[h] = *(const u32x4_t*)(k + from + h * D);
      b[h] = *(const u32x4_t*)(v + from + h * D);
    }
  }
#pragma unroll
  for (int h = 0; h < HEADS; ++h) {
    const bool has = mine && m.head0 + h < c.H;
    const long to = m.place + ((long)h << c.page_shift);
    if constexpr (KEPT == DT) {
      if (has) {
        *(u32x4_t*)((uint16_t*)kc + to * D + lane * 8) = a[h];
        *(u32x4_t*)((uint16_t*)vc + to * D + lane * 8) = b[h];
      }
    } else {
      float sa, sb;
      const u32x2_t ca = quantise<DT, KEPT, LANES>(a[h], sa), cb = quantise<DT, KEPT, LANES>(b[h], sb);
      if (has) {
        *(u32x2_t*)((uint8_t*)kc + to * D + lane * 8) = ca;
        *(u32x2_t*)((uint8_t*)vc + to * D + lane * 8) = cb;
        if (lane == 0) { ks[to] = sa; vs[to] = sb; }
      }
    }
  }
}

template <int DT, int KEPT>
__device__ __forceinline__ u32x4_t decode8(u32x2_t w, float s) {
  const f32x4_t a = decode4<KEPT>(w[0]), b = decode4<KEPT>(w[1]);
  return (u32x4_t){Half<DT>::pack(a[0] * s, a[1] * s), Half<DT>::pack(a[2] * s, a[3] * s), Half<DT>::pack(b[0] * s, b[1] * s),
                   Half<DT>::pack(b[2] * s, b[3] * s)};
}

template <int DT, int KEPT, int D>
__global__ __launch_bounds__(CT) void cache_read_kernel(Paged c, int groups, const void* __restrict__ kc, const void* __restrict__ vc,
                                                        const float* __restrict__ ks, const float* __restrict__ vs, uint16_t* __restrict__ k,
                                                        uint16_t* __restrict__ v, long pitch) {
  constexpr int LANES = row_lanes(D);
  typedef std::conditional_t<KEPT == DT, u32x4_t, u32x2_t> raw_t;
  typedef std::conditional_t<KEPT == DT, uint16_t, uint8_t> code_t;
  const int lane = threadIdx.x & (LANES - 1);
  const Mine m = find<LANES>(c, groups);
  if (m.padding || lane * 8 >= D) return;
  raw_t a[HEADS], b[HEADS];
  float sa[HEADS], sb[HEADS];
#pragma unroll
  for (int h = 0; h < HEADS; ++h) {
    a[h] = b[h] = (raw_t){};
    sa[h] = sb[h] = 0.f;
    if (m.place >= 0 && m.head0 + h < c.H) {
      const long at = m.place + ((long)h << c.page_shift);
      a[h] = *(const raw_t*)((const code_t*)kc + at * D + lane * 8);
      b[h] = *(const raw_t*)((const code_t*)vc + at * D + lane * 8);
      if constexpr (KEPT != DT) { sa[h] = ks[at]; sb[h] = vs[at]; }
    }
  }
  const long to = m.token * pitch + m.head0 * D + lane * 8;
#pragma unroll
  for (int h = 0; h < HEADS; ++h)
    if (m.head0 + h < c.H) {
      if constexpr (KEPT == DT) {
        *(u32x4_t*)(k + to + h * D) = a[h];
        *(u32x4_t*)(v + to + h * D) = b[h];
      } else {
        *(u32x4_t*)(k + to + h * D) = decode8<DT, KEPT>(a[h], sa[h]);
        *(u32x4_t*)(v + to + h * D) = decode8<DT, KEPT>(b[h], sb[h]);
      }
    }
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
    const int groups = (c.H + HEADS - 1) / HEADS;
    const unsigned grid = (unsigned)(((long)c.T * groups + rows - 1) / rows);
    hipLaunchKernelGGL((cache_write_kernel<dt.value, kept.value, dim.value>), dim3(grid), dim3(CT), 0, stream, c, groups, (const uint16_t*)k, (const uint16_t*)v,
                       pitch, kc, vc, ks, vs);
    return hipGetLastError();
  });
}

hipError_t launch_cache_read(const Paged& c, const void* kc, const void* vc, const float* ks, const float* vs, void* k, void* v, long pitch,
                             hipStream_t stream) {
  return with_forms(c, [&](auto dt, auto kept, auto dim) {
    constexpr int rows = CT / row_lanes(dim.value);
    const int groups = (c.H + HEADS - 1) / HEADS;
    const unsigned grid = (unsigned)(((long)c.T * groups + rows - 1) / rows);
    hipLaunchKernelGGL((cache_read_kernel<dt.value, kept.value, dim.value>), dim3(grid), dim3(CT), 0, stream, c, groups, kc, vc, ks, vs, (uint16_t*)k, (uint16_t*)v,
                       pitch);
    return hipGetLastError();
  });
}

}  // namespace covspec
