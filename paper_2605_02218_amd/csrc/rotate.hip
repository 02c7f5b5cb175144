// Rotary positions: rows of q and k turned, to new rows, in place, or with v straight into the paged cache.
//
// Pair (x1, x2) number i of a row at position pos: y1 = x1 c - x2 s, y2 = x2 c + x1 s, (c, s) = magnitude (cos, sin)(2 pi u), u = frac(pos step_i).
// step_i is a 64-bit binary fraction of a turn, so pos step_i mod 2^64 is u itself, exact but for the last bits of step_i (2^-33 of a turn at position 2^31).
// Of u the upper 32 bits go on (1.5e-9 of an angle): an eighth of a turn to both sides of the nearest quarter, where short series are good to 2^-28.
//
// D / 16 lanes take a row, 16 elements each: eight pairs, two pieces of 16 bytes.  A lane's cosines and sines serve all rows of a token it takes, every
// `step`-th of its heads; lanes of neighbouring groups take neighbouring heads.  Bound by memory; single tokens by latency: all heads at once.
#include <type_traits>

#include "paged.h"

namespace covspec {

namespace {

constexpr int RT = 256;
// Rows of a lane, about, where there are rows enough to fill the device: its angles serve them all, and fewer rows even out better.  us with two, four and eight: 20480 tokens
// of 32 heads with three axes 77.9, 73.4, 76.8; 8 x 3008 tokens of 32 + 8 heads of 128 into a 16-bit cache -, 118, 123; 16000 of 64 + 8 heads -, 128, 134; 24064 of 16 + 16 heads
// of 64 39.4, 36.8, 36.2; of 8 + 1 heads with one row 22.1, with three 18.2.
constexpr int EACH = 4;

struct Turn { float c, s; };
// Cosine and sine of a 64-bit fraction of a turn: series around the nearest quarter, |x| <= pi / 4, errors below 2^-28 of 1.  What the conversion to a float, the product with
// 2 pi 2^-32 and the square lose goes into the last sums, so that these are all that is rounded: 2^-24 at most, in the mean 1.05 times the error of a number that is rounded once
// (without these parts 1.4 times; prompts into the cache take 114 us with and without, image tokens with three axes 2 more).
__device__ __forceinline__ Turn turn_of(uint64_t u, float magnitude) {
  constexpr double kUnit = 6.283185307179586476925 / 4294967296.0;
  constexpr float kHigh = (float)kUnit, kLow = (float)(kUnit - (double)kHigh);
  const uint32_t hi = (uint32_t)(u >> 32), quarter = (hi + 0x20000000u) >> 30;
  const int32_t i = (int32_t)(hi - (quarter << 30));                   // up to 2^29 to both sides
  const float f = (float)i, x = f * kHigh, y = x * x;
  const float rest = __builtin_fmaf(f, kHigh, -x) + __builtin_fmaf(f, kLow, (float)(i - (int32_t)f) * kHigh);        // x + rest is the angle
  float c = __builtin_fmaf(y, -1.f / 3628800.f, 1.f / 40320.f);
  c = __builtin_fmaf(y, c, -1.f / 720.f);
  c = __builtin_fmaf(y, c, 1.f / 24.f);
  c = __builtin_fmaf(y, c, -0.5f);
  c = 1.f + __builtin_fmaf(y, c, -__builtin_fmaf(x, rest, 0.5f * __builtin_fmaf(x, x, -y)));
  float s = __builtin_fmaf(y, 1.f / 362880.f, -1.f / 5040.f);
  s = __builtin_fmaf(y, s, 1.f / 120.f);
  s = __builtin_fmaf(y, s, -1.f / 6.f);
  s = x + __builtin_fmaf(x * y, s, rest * c);
  const bool odd = quarter & 1;
  const float a = odd ? s : c, b = odd ? c : s;
  return Turn{quarter == 1 || quarter == 2 ? -a * magnitude : a * magnitude, quarter >= 2 ? -b * magnitude : b * magnitude};
}

__device__ __forceinline__ void load16(const uint16_t* from, int a, int b, u32x4_t (&w)[2]) {
  w[0] = *(const u32x4_t*)(from + a);
  w[1] = *(const u32x4_t*)(from + b);
}
template <int DT>
__device__ __forceinline__ void unpack16(const u32x4_t (&w)[2], float (&x)[16]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const f32x2_t p = Half<DT>::unpack(w[e / 4][e % 4]);
    x[2 * e] = p[0];
    x[2 * e + 1] = p[1];
  }
}
template <int DT>
__device__ __forceinline__ void store16(uint16_t* to, int a, int b, const float (&x)[16]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    *(u32x4_t*)(to + (h == 0 ? a : b)) = (u32x4_t){Half<DT>::pack(x[8 * h], x[8 * h + 1]), Half<DT>::pack(x[8 * h + 2], x[8 * h + 3]),
                                                   Half<DT>::pack(x[8 * h + 4], x[8 * h + 5]), Half<DT>::pack(x[8 * h + 6], x[8 * h + 7])};
}

// KEPT: what k and v are kept as in the cache; -1: rows, no cache.  FAR: pairs (i, i + R / 2), else (2i, 2i + 1).
template <int DT, int KEPT, int D, bool FAR>
__global__ __launch_bounds__(RT) void rotate_kernel(Paged c, Rotate r) {
  constexpr bool CACHE = KEPT >= 0, CODES = CACHE && KEPT != DT;
  constexpr int LANES = D == 64 ? 4 : 8;                               // head dimension 96 leaves two of eight without work
  const long x = (long)blockIdx.x * (RT / LANES) + threadIdx.x / LANES;
  const int lane = threadIdx.x & (LANES - 1), t = (int)(x / r.step), first = (int)(x % r.step);
  const bool inside = t < c.T && lane * 16 < D;
  bool mine = inside;
  int pos = 0;
  long place = -1;                                                     // of head 0
  if (c.start) {
    const int s = seq_of_wave<64 / LANES>(c.start, c.S, t < c.T ? t : 0x7FFFFFFF);
    mine = inside && s >= 0 && s < c.S;
    if (mine) {
      const long at = (long)c.length[s] - c.start[s + 1] + t;
      pos = (int)at;
      if constexpr (CACHE) place = place_of(c, s, at, 0);
    }
  }
  // which elements: eight at a and eight at b, neighbouring lanes' next to each other; eight pairs, across the two (FAR) or four in each, or 16 that are not turned
  const bool turns = lane * 16 < r.R;
  const int at = turns ? lane : lane - r.R / 16, a = (turns ? 0 : r.R) + 8 * at, b = a + (turns ? r.R : D - r.R) / 2;
  Turn w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = Turn{1.f, 0.f};
  if (turns && mine) {
    int p[4] = {pos, pos, pos, pos};
    if (r.positions) {
#pragma unroll
      for (int x = 0; x < 4; ++x) p[x] = r.positions[(long)min(x, r.n_axes - 1) * c.T + t];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int pair = FAR ? 8 * lane + 4 * h : 4 * lane + h * (r.R / 4);       // and three behind it
      int axis[4] = {0, 0, 0, 0};
      if (r.axis) {
#pragma unroll
        for (int e = 0; e < 4; ++e) axis[e] = r.axis[pair + e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = axis[e] <= 0 ? p[0] : axis[e] == 1 ? p[1] : axis[e] == 2 ? p[2] : p[3];      // beyond the last axis p repeats it
        w[4 * h + e] = turn_of((uint64_t)(int64_t)at * r.steps[pair + e], r.magnitude);
      }
    }
  }
  auto turned = [&](float (&y)[16]) {
    if (!turns) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = FAR ? e : 2 * e, j = FAR ? e + 8 : 2 * e + 1;
      const float x1 = y[i], x2 = y[j];
      y[i] = __builtin_fmaf(x1, w[e].c, -(x2 * w[e].s));
      y[j] = __builtin_fmaf(x2, w[e].c, x1 * w[e].s);
    }
  };
  // a row of codes: the lanes of the row exchange their maxima, so all of them come here
  auto keep = [&](const float (&y)[16], bool has, long to, void* codes, float* scales) {
    if constexpr (CODES) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(y[e]) & 0x7FFFFFFFu);
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
      float inv, scale;
      const bool finite = code_step<KEPT>(top, inv, scale);
      if (has) {
        uint8_t* const row = (uint8_t*)codes + to * D;
        *(u32x2_t*)(row + a) = (u32x2_t){encode_row4<KEPT>(y, inv, finite), encode_row4<KEPT>(y + 4, inv, finite)};
        *(u32x2_t*)(row + b) = (u32x2_t){encode_row4<KEPT>(y + 8, inv, finite), encode_row4<KEPT>(y + 12, inv, finite)};
        if (lane == 0) scales[to] = scale;
      }
    } else {
      if (has) store16<DT>((uint16_t*)codes + to * D, a, b, y);
    }
  };
  const int rows_q = r.q ? r.heads : 0, rows = rows_q + (r.k ? c.H : 0);
  const bool goes = CACHE ? mine && place >= 0 : mine;                 // rows of k and v
  // row h of q, or, behind those, of k, and of v for a cache
  struct Raw { u32x4_t x[2], v[2]; };
  auto request = [&](int h, Raw& f) {
    f.x[0] = f.x[1] = f.v[0] = f.v[1] = (u32x4_t){};
    const bool far = h >= rows_q;
    const long row = far ? t * r.k_pitch + (long)(h - rows_q) * D : t * r.q_pitch + (long)h * D;
    if (h < rows && (far ? goes : mine)) {
      load16((far ? r.k : r.q) + row, a, b, f.x);
      if constexpr (CACHE)
        if (far) load16(r.v + row, a, b, f.v);
    }
  };
  Raw now;
  request(first, now);
  // all lanes of a wave stay to the end of the loop, where rows exchange their maxima; a row is on its way while the one before is turned
  for (int h0 = 0; h0 < rows; h0 += r.step) {
    const int h = h0 + first;
    Raw next;
    request(h + r.step, next);
    float y[16];
    unpack16<DT>(now.x, y);
    turned(y);
    if (h < rows_q) {
      if (mine) store16<DT>(r.q_out + t * r.q_out_pitch + (long)h * D, a, b, y);
    } else {
      const bool has = goes && h < rows;
      const int g = h - rows_q;
      if constexpr (CACHE) {
        const long to = place + ((long)g << c.page_shift);
        keep(y, has, to, r.kc, r.ks);
        if constexpr (CODES) {
          unpack16<DT>(now.v, y);
          keep(y, has, to, r.vc, r.vs);
        } else if (has) {
          *(u32x4_t*)((uint16_t*)r.vc + to * D + a) = now.v[0];
          *(u32x4_t*)((uint16_t*)r.vc + to * D + b) = now.v[1];
        }
      } else if (has) {
        store16<DT>(r.k_out + t * r.k_out_pitch + (long)g * D, a, b, y);
      }
    }
    now = next;
  }
}

template <int DT, int KEPT, int D>
hipError_t launch_dim(const Paged& c, Rotate r, hipStream_t stream) {
  constexpr int LANES = D == 64 ? 4 : 8;
  const int rows = (r.q ? r.heads : 0) + (r.k ? c.H : 0);
  r.step = rows;
  while (r.step > (rows + EACH - 1) / EACH && (long)c.T * r.step * LANES > 256l * 2048) r.step = (r.step + 1) / 2;
  const unsigned grid = (unsigned)(((long)c.T * r.step * LANES + RT - 1) / RT);
  if (r.interleaved)
    hipLaunchKernelGGL((rotate_kernel<DT, KEPT, D, false>), dim3(grid), dim3(RT), 0, stream, c, r);
  else
    hipLaunchKernelGGL((rotate_kernel<DT, KEPT, D, true>), dim3(grid), dim3(RT), 0, stream, c, r);
  return hipGetLastError();
}

template <int DT, int KEPT>
hipError_t launch_kept(const Paged& c, const Rotate& r, hipStream_t stream) {
  if (c.D == 64) return launch_dim<DT, KEPT, 64>(c, r, stream);
  if (c.D == 96) return launch_dim<DT, KEPT, 96>(c, r, stream);
  if (c.D == 128) return launch_dim<DT, KEPT, 128>(c, r, stream);
  return hipErrorInvalidValue;
}

template <int DT>
hipError_t launch_type(const Paged& c, const Rotate& r, hipStream_t stream) {
  if (!r.kc) return launch_kept<DT, -1>(c, r, stream);
  if (c.kept == DT) return launch_kept<DT, DT>(c, r, stream);
  if (c.kept == DT_I8) return launch_kept<DT, DT_I8>(c, r, stream);
  if (c.kept == DT_E4M3) return launch_kept<DT, DT_E4M3>(c, r, stream);
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_rotate(const Paged& c, const Rotate& r, hipStream_t stream) {
  if (c.dtype == DT_BF16) return launch_type<DT_BF16>(c, r, stream);
  if (c.dtype == DT_F16) return launch_type<DT_F16>(c, r, stream);
  return hipErrorInvalidValue;
}

}  // namespace covspec
