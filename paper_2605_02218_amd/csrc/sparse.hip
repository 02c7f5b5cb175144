// Attention over the pages that a cheap score selects for each row: summaries of pages, scores, the choice, attention over it.
//
// A page's summary is, channel by channel, the largest and the smallest of its keys as int8 codes with one scale.  For codes c of a query, which are those of
// an 8-bit row, sum_d max(c_d largest_d, c_d smallest_d) = sum_d max(c_d, 0) largest_d + min(c_d, 0) smallest_d is a product over 2 D terms, exact in
// int32 whatever its order, and fewer than 2^24; two fp32 products with the scales follow.  So the scores are defined to the bit, and with them
// the choice, on any machine.  A block costs 2 D + 4 bytes to score and page_size 2 D e to attend to.
#include <algorithm>
#include <type_traits>

#include "host_cache.h"
#include "parting.h"
#include "tiles.h"

namespace covspec {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

// Rows and lengths as covspec_attend takes them.  t uniform in the wave; false: a padding row.  The sequence is the last one that begins at or in front of t: of 64
// starts at a time, every 64th part's first while there are more, then all of them with their lengths, so that up to 63 sequences take one load's time.
struct Row { int s, row0, n, old; };
__device__ __forceinline__ bool row_of(const Paged& c, int t, Row& r) {
  const int lane = threadIdx.x & 63;
  int first = 0, n = c.S + 1;                     // it is one of these
  while (n > 64) {
    const int step = (n + 63) / 64, i = lane * step;
    const int at = __popcll(__ballot(i < n && c.start[first + min(i, n - 1)] <= t)) - 1;
    if (at < 0) return false;
    first += at * step;
    n = min(step, n - at * step);
  }
  const int s = min(first + lane, c.S), start = c.start[s], len = c.length[min(s, c.S - 1)];
  const int at = __popcll(__ballot(lane < n && start <= t)) - 1;
  r.s = first + at;
  if (at < 0 || r.s >= c.S || t >= c.T) return false;
  r.row0 = min(max(__builtin_amdgcn_readlane(start, at), 0), c.T);
  const int end = at == 63 ? c.start[r.s + 1] : __builtin_amdgcn_readlane(start, at + 1);
  r.n = max(min(end, c.T), r.row0) - r.row0;
  r.old = (int)max((long)__builtin_amdgcn_readlane(len, at) - r.n, -(1l << 30));
  return true;
}
// End of what row i of the chunk sees.
__device__ __forceinline__ int seen_end(const Paged& c, const Row& r, int i, int max_len, bool tree) {
  const long cap = min((long)max_len, (long)c.max_pages << c.page_shift), hi = (long)r.old + (tree ? min(r.n, 64) : i + 1);
  return (int)max(min(hi, cap), 0l);
}
__device__ __forceinline__ int blocks_up_to(const Paged& c, int end) { return (int)(((long)end + (1 << c.page_shift) - 1) >> c.page_shift); }

// ---- summaries

__device__ __forceinline__ uint32_t wave_top(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));      // row_shr 1, 2, 4, 8
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, true));      // row_bcast 15, 31
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, true));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

template <int DT, int KEPT, int D> struct Piece {
  static constexpr bool CODES = KEPT != DT;
  static constexpr int N = CODES ? 16 : 8;             // channels of a lane: 16 bytes
  static constexpr int LANES = D / N <= 4 ? 4 : D / N <= 8 ? 8 : 16;       // of a row; head dimension 96 leaves a quarter without work
};

// Over the lanes that are `LANES` apart.
template <int LANES, typename F>
__device__ __forceinline__ float over_rows(float x, F f) {
  if constexpr (LANES <= 4) x = f(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x124, 0xf, 0xf, true)));      // row_ror 4
  if constexpr (LANES <= 8) x = f(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x128, 0xf, 0xf, true)));      // row_ror 8
  return over_groups<16>(x, f);
}

// Bound by memory for prompts in 16 bits (8 x 3008 tokens of 8 heads of 128 11.4 us, 4.3 TB/s), by latency for those in 8 (11.8 us for half the bytes) and for single tokens (64 in
// 16 bits 5.1 us, in 8 7.9): start and length, the page's number, its rows and the reduction, one behind the other.
// A wave takes a page of a key head, or (WAVES = 4) a workgroup a large one: four waves on a page of 64 took 20 us instead of 11 for 256 single tokens.  BY_ROW: an item is a row, the first of its sequence's on the page does the work;
// else items are the pages that each sequence's rows touch, one sequence behind the other.
template <int DT, int KEPT, int D, int WAVES, bool BY_ROW>
__global__ __launch_bounds__(256) void summary_kernel(Paged c, long items, const void* __restrict__ kc, const float* __restrict__ ks, int8_t* __restrict__ summary,
                                                      float* __restrict__ scales) {
  typedef Piece<DT, KEPT, D> P;
  constexpr int N = P::N, LANES = P::LANES, ROWS = 64 / LANES;
  __shared__ float shared[WAVES > 1 ? WAVES : 1][WAVES > 1 ? 2 * D + 1 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long item = WAVES > 1 ? blockIdx.x : (long)blockIdx.x * 4 + wave;
  if (item >= items) return;
  const int x = (int)(item / c.H), g = (int)(item % c.H);
  const int shift = c.page_shift, cap = c.max_pages << shift;
  int s = -1, block = 0, len = 0;
  if constexpr (BY_ROW) {
    Row r;
    if (!row_of(c, x, r)) return;
    const long pos = (long)r.old + (x - r.row0);
    if (pos < 0 || pos >= cap || (x != r.row0 && (pos & ((1 << shift) - 1)) != 0)) return;
    s = r.s;
    block = (int)(pos >> shift);
    len = r.old + r.n;
  } else {
    int left = x;
    for (int s0 = 0; s0 < c.S && s < 0; s0 += 64) {
      const int mine = min(s0 + lane, c.S - 1), row0 = min(max(c.start[mine], 0), c.T), n = max(min(c.start[mine + 1], c.T), row0) - row0, length = c.length[mine];
      const int lo = (int)max((long)length - n, 0l), hi = min(length, cap);
      const int own = s0 + lane < c.S && n > 0 && lo < hi ? ((hi - 1) >> shift) - (lo >> shift) + 1 : 0, upto = wave_inscan(own);
      const unsigned long long over = __ballot(upto > left);
      if (over) {
        const int at = __ffsll((long long)over) - 1;
        s = s0 + at;
        len = __builtin_amdgcn_readlane(length, at);
        block = (__builtin_amdgcn_readlane(lo, at) >> shift) + left - __builtin_amdgcn_readlane(upto, at) + __builtin_amdgcn_readlane(own, at);
      }
      left -= __builtin_amdgcn_readlane(upto, 63);
    }
    if (s < 0) return;
  }
  const int page = c.pages[(long)s * c.max_pages + block];
  if (page < 0 || page >= c.n_pages) return;
  const int count = min(min(len, cap) - (block << shift), 1 << shift);          // positions of the page: at least one, if `start` ascends
  if (count < 1) return;
  const long first = ((long)page * c.H + g) << shift;
  const int piece = lane % LANES, row = lane / LANES;
  float top[N], low[N];
  float bad = 0.f;                                // NaN once a number is not finite
#pragma unroll
  for (int e = 0; e < N; ++e) { top[e] = -INFINITY; low[e] = INFINITY; }
  if (piece * N < D) {
    constexpr int AHEAD = 8;
    for (int j0 = (WAVES > 1 ? wave * ROWS : 0); j0 < count; j0 += AHEAD * ROWS * WAVES) {
      u32x4_t raw[AHEAD];
      float scale[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const long at = first + min(j0 + i * ROWS * WAVES + row, count - 1);           // the last row again behind it
        raw[i] = *(const u32x4_t*)((const char*)kc + (at * D + piece * N) * (P::CODES ? 1 : 2));
        if constexpr (P::CODES) scale[i] = ks[at];
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        float v[N];
        if constexpr (P::CODES) {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const f32x4_t f = decode4<KEPT>(raw[i][w]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * w + e] = f[e] * scale[i];
          }
        } else {
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const f32x2_t f = Half<DT>::unpack(raw[i][w]);
            v[2 * w] = f[0];
            v[2 * w + 1] = f[1];
          }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
          top[e] = fmaxf(top[e], v[e]);
          low[e] = fminf(low[e], v[e]);
          bad = __builtin_fmaf(v[e], 0.f, bad);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    top[e] = over_rows<LANES>(top[e], [](float x, float y) { return fmaxf(x, y); });
    low[e] = over_rows<LANES>(low[e], [](float x, float y) { return fminf(x, y); });
  }
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (piece * N < D) most = fmaxf(most, fmaxf(top[e], -low[e]));
  uint32_t size = wave_top(__any(bad != 0.f || bad != bad) ? 0x7FC00000u : __float_as_uint(most));     // largest magnitude, as bits
  if constexpr (WAVES > 1) {
    if (row == 0 && piece * N < D) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        shared[wave][piece * N + e] = top[e];
        shared[wave][D + piece * N + e] = low[e];
      }
    }
    if (lane == 0) shared[wave][2 * D] = __uint_as_float(size);
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      size = max(size, __float_as_uint(shared[w][2 * D]));
      if (piece * N < D) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          top[e] = fmaxf(top[e], shared[w][piece * N + e]);
          low[e] = fminf(low[e], shared[w][D + piece * N + e]);
        }
      }
    }
  }
  float inv, scale;
  const bool finite = code_step<DT_I8>(size, inv, scale);
  const long to = (long)page * c.H + g;
  if (row == 0 && piece * N < D) {
#pragma unroll
    for (int w = 0; w < N / 4; ++w) {
      *(uint32_t*)(summary + to * 2 * D + piece * N + 4 * w) = encode_row4<DT_I8>(top + 4 * w, inv, finite);
      *(uint32_t*)(summary + to * 2 * D + D + piece * N + 4 * w) = encode_row4<DT_I8>(low + 4 * w, inv, finite);
    }
  }
  if (lane == 0) scales[to] = scale;
}

// ---- scores

// A score as an integer of the same order.  A NaN comes above all others if it is positive, as the canonical one; kAbsent, a NaN of all ones, becomes 0, for a block
// that is not there (kNone): as a block's scale it goes through its products (a NaN among the factors comes out as it is, before one in the summand).  The largest key
// (kAlways) is left for blocks that are taken whatever their score.
constexpr uint32_t kAbsent = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t score_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

// Blocks are rows of the product, 16 at a time, (token, query head) its columns; the terms are max(c, 0) largest, then min(c, 0) smallest, 64 a step.  A lane has
// column lane % 16 of a product and 16 neighbouring terms of each step.
// The largest over runs of gp neighbouring lanes, a power of two, up to 16.
template <int N>
__device__ __forceinline__ void over_run(uint32_t (&v)[N], int gp) {
  auto over = [&](auto step) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = max(v[i], (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v[i], step.value, 0xf, 0xf, true));
  };
  if (gp >= 2) over(std::integral_constant<int, 0xB1>{});              // quad_perm 1 0 3 2
  if (gp >= 4) over(std::integral_constant<int, 0x4E>{});              // quad_perm 2 3 0 1
  if (gp >= 8) over(std::integral_constant<int, 0x141>{});             // row_half_mirror
  if (gp >= 16) over(std::integral_constant<int, 0x140>{});            // row_mirror
}

template <int D> constexpr int kSteps = 2 * D / 64;

template <int D> constexpr int kOwn = D == 96 ? kSteps<D> : kSteps<D> / 2;          // a lane's terms below and above zero are the same elements but for D = 96
template <int D, int NT> struct Queries {
  u32x4_t raw[NT][kOwn<D>][2];
  bool real[NT];
};
template <int D, int NT> struct Codes {
  i32x4_t q[NT][kSteps<D>];
  float scale[NT], bias[NT];                      // bias: 0; -infinity for a column of no query; NaN for a query that is none of numbers, whose scale is then 0
};
// from(n): the query of the lane's column 16 n + lane % 16, or null
template <int D, int NT, typename F>
__device__ __forceinline__ void load_queries(F from, Queries<D, NT>& r) {
  const int quad = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const uint16_t* const x = from(n);
    r.real[n] = x != nullptr;
#pragma unroll
    for (int k = 0; k < kOwn<D>; ++k) {
      const int k0 = 64 * k + 16 * quad, d = k0 >= D ? k0 - D : k0;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        r.raw[n][k][p] = (u32x4_t){};
        if (x) r.raw[n][k][p] = *(const u32x4_t*)(x + d + 8 * p);
      }
    }
  }
}
// Four int8 codes: beside 1.5 2^23 the nearest whole number, ties to even, is the low byte; at most 127 (1 + 3 2^-24) before, so 127 behind.
__device__ __forceinline__ uint32_t int_codes(const float (&y)[4], float inv) {
#pragma clang fp contract(off)
  uint32_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = y[e] * inv;                                        // rounded on its own
    b[e] = __float_as_uint(x + 12582912.f);
  }
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
}
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
template <int DT, int D, int NT>
__device__ __forceinline__ void query_codes(const Queries<D, NT>& r, int columns, Codes<D, NT>& c) {
  constexpr int OWN = kOwn<D>;
  const int quad = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (16 * n >= columns) break;
    u16x2_t most = {0, 0};                        // magnitudes of both types are in the order of their bits
#pragma unroll
    for (int k = 0; k < OWN; ++k)
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, r.raw[n][k][p][e] & 0x7FFF7FFFu));
    uint32_t top = max(most[0], most[1]);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
    float inv;
    const bool finite = code_step<DT_I8>(__float_as_uint(Half<DT>::unpack(top)[0]), inv, c.scale[n]);
    const uint32_t keep = finite ? ~0u : 0u;
    if (!finite) c.scale[n] = 0.f;
    c.bias[n] = !r.real[n] ? -INFINITY : finite ? 0.f : __uint_as_float(0x7FC00000u);
#pragma unroll
    for (int k = 0; k < OWN; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const f32x2_t f0 = Half<DT>::unpack(r.raw[n][k][w / 2][2 * (w & 1)]), f1 = Half<DT>::unpack(r.raw[n][k][w / 2][2 * (w & 1) + 1]);
        const float y[4] = {f0[0], f0[1], f1[0], f1[1]};
        const uint32_t code = int_codes(y, inv) & keep, sign = code >> 7 & 0x01010101u, below = (sign << 8) - sign;       // bytes of codes below zero
        if constexpr (D == 96) {
          c.q[n][k][w] = (int)(64 * k + 16 * quad >= D ? code & below : code & ~below);
        } else {
          c.q[n][k][w] = (int)(code & ~below);
          c.q[n][k + OWN][w] = (int)(code & below);
        }
      }
  }
}

// 64 blocks of a sequence, block b0 + lane in a lane: on their way, then their scores.
template <int D> struct Scored {
  i32x4_t m[4][kSteps<D>];
  float scale;
};
__device__ __forceinline__ int block_id(const Paged& c, int s, int b, int nb) { return b < nb ? c.pages[(long)s * c.max_pages + b] : -1; }
template <int D>
__device__ __forceinline__ void load_blocks(const Paged& c, int g, const int8_t* summary, const float* scales, int id, Scored<D>& r) {
  const int lane = threadIdx.x & 63;
  const bool there = id >= 0 && id < c.n_pages;
  id = there ? id : 0;
  r.scale = scales[(long)id * c.H + g];
  r.scale = __uint_as_float(!there ? kAbsent : r.scale != r.scale ? 0x7FC00000u : __float_as_uint(r.scale));       // a NaN of any sign and payload as the canonical one
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const long from = ((long)__shfl(id, 16 * j + (lane & 15), 64) * c.H + g) * 2 * D + 16 * (lane >> 4);
#pragma unroll
    for (int k = 0; k < kSteps<D>; ++k) r.m[j][k] = *(const i32x4_t*)(summary + from + 64 * k);
  }
}
// put(n, j, keys): those of blocks 16 j + 4 (lane / 16) + 0 .. 3 for the token whose first column is 16 n + lane % 16, in those lanes; gp columns a token, a power of two
// up to 16 NT, `columns` in all
template <int D, int NT, typename F>
__device__ __forceinline__ void score_blocks(const Scored<D>& b, const Codes<D, NT>& q, int gp, int columns, F put) {
  const int lane = threadIdx.x & 63, quad = lane >> 4, parts = gp <= 16 ? 1 : gp >> 4;
  const bool first = (lane & 15 & (gp - 1)) == 0;
  float ksc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) ksc[i] = __shfl(b.scale, 16 * (i / 4) + 4 * quad + i % 4, 64);
  uint32_t best[16];                              // blocks 16 (i / 4) + 4 quad + i % 4
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (16 * n >= columns) break;
    const bool more = (n & (parts - 1)) != 0;     // heads of the same token
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      i32x4_t acc = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < kSteps<D>; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b.m[j][k], q.q[n][k], acc, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t key = score_key(__builtin_fmaf((float)acc[e] * ksc[4 * j + e], q.scale[n], q.bias[n]));       // a product's rounding: what is added is 0
        best[4 * j + e] = more ? max(best[4 * j + e], key) : key;
      }
    }
    if ((n & (parts - 1)) != parts - 1 && 16 * (n + 1) < columns) continue;
    over_run(best, gp);
    if (first) {
#pragma unroll
      for (int j = 0; j < 4; ++j) put(n & ~(parts - 1), j, (u32x4_t){best[4 * j], best[4 * j + 1], best[4 * j + 2], best[4 * j + 3]});
    }
  }
}

// Scores in a launch of their own, the blocks spread over the device: a workgroup takes 256 blocks for as many tokens of a sequence as 16 NT columns hold; of 64 columns each wave
// makes the codes of 16 for all (with every wave making all of them 24 us instead of 19 below).  Bound by vector instructions, 9 for a score, where the columns are full (8 tokens
// of 8 heads for each key head, 16 sequences of 375 to 1500 blocks: 19 us, 31 MB of summaries), else by latency: 5 us for a token's 2001 blocks, 7.5 for four tokens' 15626.
constexpr int SCORED = 256;
template <int DT, int D, int NT>
__global__ __launch_bounds__(256, 2) void score_kernel(Paged c, Attend a, int gp, int chunks, int pitch, const int8_t* __restrict__ summary,
                                                    const float* __restrict__ scales, uint32_t* __restrict__ keys) {
  static_assert(NT == 1 || NT == 4, "a wave makes the codes of 16 columns");
  __shared__ i32x4_t made[NT > 1 ? NT : 1][kSteps<D>][NT > 1 ? 64 : 1];
  __shared__ f32x2_t factors[NT > 1 ? NT : 1][NT > 1 ? 64 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.heads / c.H, tokens = 16 * NT / gp;
  const long item = blockIdx.x / c.H;
  const int g = blockIdx.x % c.H, chunk = (int)(item % chunks);
  // groups of `tokens` rows of a sequence, one sequence behind the other
  int left = (int)(item / chunks), s = -1, row0 = 0, n = 0, len = 0, i0 = 0;
  for (int s0 = 0; s0 < c.S && s < 0; s0 += 64) {
    const int mine = min(s0 + lane, c.S - 1), first = min(max(c.start[mine], 0), c.T), rows = max(min(c.start[mine + 1], c.T), first) - first, length = c.length[mine];
    const int own = s0 + lane < c.S ? (rows + tokens - 1) / tokens : 0, upto = wave_inscan(own);
    const unsigned long long over = __ballot(upto > left);
    if (over) {
      const int at = __ffsll((long long)over) - 1;
      s = s0 + at;
      row0 = __builtin_amdgcn_readlane(first, at);
      n = __builtin_amdgcn_readlane(rows, at);
      len = __builtin_amdgcn_readlane(length, at);
      i0 = (left - __builtin_amdgcn_readlane(upto, at) + __builtin_amdgcn_readlane(own, at)) * tokens;
    }
    left -= __builtin_amdgcn_readlane(upto, 63);
  }
  if (s < 0) return;
  const Row r = {s, row0, n, (int)max((long)len - n, -(1l << 30))};
  const int i1 = min(i0 + tokens, n), nb = blocks_up_to(c, seen_end(c, r, i1 - 1, a.max_len, a.visible != nullptr)), b0 = chunk * SCORED + wave * 64;
  if (chunk * SCORED >= nb) return;
  const int id = block_id(c, s, b0 + lane, nb);
  const int shift = __builtin_ctz(gp), columns = (i1 - i0) * gp;
  auto query = [&](int y) -> const uint16_t* {
    const int x = 16 * y + (lane & 15), i = i0 + (x >> shift), h = x & (gp - 1);
    return i < i1 && h < G ? (const uint16_t*)a.q + (long)(row0 + i) * a.q_pitch + (long)(g * G + h) * D : nullptr;
  };
  Queries<D, 1> raw;
  load_queries<D, 1>([&](int) { return query(NT > 1 ? wave : 0); }, raw);
  Scored<D> b;
  load_blocks<D>(c, g, summary, scales, id, b);                        // of the pool's first page where there are no more blocks
  Codes<D, NT> q;
  if constexpr (NT > 1) {
    Codes<D, 1> own;
    query_codes<DT, D, 1>(raw, 16, own);
#pragma unroll
    for (int k = 0; k < kSteps<D>; ++k) made[wave][k][lane] = own.q[0][k];
    factors[wave][lane] = (f32x2_t){own.scale[0], own.bias[0]};
    __syncthreads();
    if (b0 >= nb) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (16 * n >= columns) break;
#pragma unroll
      for (int k = 0; k < kSteps<D>; ++k) q.q[n][k] = made[n][k][lane];
      const f32x2_t f = factors[n][lane];
      q.scale[n] = f[0];
      q.bias[n] = f[1];
    }
  } else {
    if (b0 >= nb) return;
    query_codes<DT, D, 1>(raw, columns, q);
  }
  score_blocks<D, NT>(b, q, gp, columns, [&](int y, int j, u32x4_t key) {
    const int i = i0 + ((16 * y + (lane & 15)) >> shift);
    if (i < i1) *(u32x4_t*)(keys + ((long)(row0 + i) * c.H + g) * pitch + b0 + 16 * j + 4 * (lane >> 4)) = key;
  });
}

// ---- the choice

// The keys of a row's blocks lie in LDS, `count` of them with zeros behind the last up to a multiple of 256; a lane takes four neighbours.  The key that parts those
// taken from the others is found by counting keys in 1024 equal parts of the range where it must lie, then in the part that holds it (parting.h), at most four times,
// twice as a rule; then the blocks above it and the first ones at it, in order.
constexpr int BINS = 1024, PASSES = 4, GROUPS = 128;       // 256 neighbouring blocks a group
struct ChoiceLds {
  int bins[PASSES][BINS];
  int above[GROUPS];
  int counts[16][4], found[PASSES][4];
};
template <int THREADS>
__device__ __forceinline__ void clear_bins(ChoiceLds& l) {
  for (int i = threadIdx.x; i < PASSES * BINS / 4; i += THREADS) ((i32x4_t*)l.bins)[i] = (i32x4_t){0, 0, 0, 0};
}
// Where the `need`-th largest of counted keys lies: the part, how many are beyond it, how many in it.  N parts for each lane, `own`, in the order of the lanes.
template <int N>
__device__ __forceinline__ Part part_of(const int (&own)[N], int need) {
  int sum = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) sum += own[i];
  const int upto = wave_inscan(sum), over = __builtin_amdgcn_readlane(upto, 63) - upto;    // keys in the parts of later lanes
  const int from = 63 - __builtin_clzll(__ballot(over < need && over + sum >= need));      // one lane
  int bin = 0, before = over, here = 0;
#pragma unroll
  for (int i = N - 1; i >= 0; --i) {
    const bool past = before + here >= need;      // found in a part above
    before += past ? 0 : here;
    here = past ? here : own[i];
    bin = past ? bin : i;
  }
  return Part{from * N + __builtin_amdgcn_readlane(bin, from), __builtin_amdgcn_readlane(before, from), __builtin_amdgcn_readlane(here, from)};
}
// What a thread has seen of the keys.
struct Seen { uint32_t lo = kAlways, hi = 0; int always = 0, there = 0; };
__device__ __forceinline__ void see(Seen& s, const u32x4_t& k) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t x = k[e];
    s.always += x == kAlways;
    s.there += x != kNone;
    s.lo = min(s.lo, x - 1 < kAlways - 1 ? x : kAlways);
    s.hi = max(s.hi, x == kAlways ? 0u : x);
  }
}
__device__ __forceinline__ Seen over_wave(const Seen& s) {
  Seen r;
  r.lo = ~wave_top(~s.lo);
  r.hi = wave_top(s.hi);
  r.always = __builtin_amdgcn_readlane(wave_inscan(s.always), 63);
  r.there = __builtin_amdgcn_readlane(wave_inscan(s.there), 63);
  return r;
}
// Of a lane's four keys those above `at` and, 16 bits further up, those at it.
__device__ __forceinline__ int above_and_at(const u32x4_t& k, uint32_t at, bool ties) {
  int n = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) n += k[e] > at ? 1 : ties && k[e] == at ? 1 << 16 : 0;
  return n;
}
// The lane's taken ones of blocks b .. b + 3, with `ups` above `at` and `eqs` at it in front of them.  No place behind the list's last
// is written, whatever was counted (by a comparison in the place of the outer minimum choose_rows_kernel takes 10.3 us instead of 8.7).
template <typename F>
__device__ __forceinline__ void put_taken(const u32x4_t& k, int b, uint32_t at, bool ties, int more, int top, int ups, int eqs, F put) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool is_up = k[e] > at, is_eq = ties && k[e] == at;
    if (is_up || (is_eq && eqs < more)) put(min(ups + min(eqs, more), top - 1), b + e);
    ups += is_up;
    eqs += is_eq;
  }
}
// Blocks taken, ascending, through put(place, block); their number is returned.  All threads, with what they have seen of all keys between them.
template <int THREADS, typename F>
__device__ __forceinline__ int choose(const uint32_t* keys, int count, const Seen& seen, int top, ChoiceLds& l, F put) {
  constexpr int WAVES = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), groups = count >> 8;
  const u32x4_t* const mine = (const u32x4_t*)keys + lane;             // of group x: mine[64 x]
  Seen all = over_wave(seen);
  if (lane == 0) *(i32x4_t*)l.counts[wave] = (i32x4_t){all.always, all.there, (int)all.lo, (int)all.hi};
  __syncthreads();                                                     // the keys are there as well
  all = Seen();
  if (lane < WAVES) {
    const i32x4_t v = *(const i32x4_t*)l.counts[lane];
    all.always = v[0];
    all.there = v[1];
    all.lo = (uint32_t)v[2];
    all.hi = (uint32_t)v[3];
  }
  all = over_wave(all);
  Parting part = {0, 0};
  if (all.there - all.always > top - all.always) {
    part = parting_key<10>(all.lo, all.hi, top - all.always, [&](int pass, uint32_t lo, uint32_t width, int shift, int need) {
      for (int x = wave; x < groups; x += WAVES) {
        const u32x4_t k = mine[64 * x];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k[e] - lo <= width) atomicAdd(&l.bins[pass][(k[e] - lo) >> shift], 1);
      }
      __syncthreads();
      Part p = {};
      if (WAVES <= 4 || wave == 0) {              // four waves do it each for itself, more would be in one another's way
        int own[BINS / 64];
#pragma unroll
        for (int i = 0; i < BINS / 256; ++i) {
          const i32x4_t v = ((const i32x4_t*)l.bins[pass])[lane * (BINS / 256) + i];
#pragma unroll
          for (int e = 0; e < 4; ++e) own[4 * i + e] = v[e];
        }
        p = part_of(own, need);
      }
      if (WAVES > 4) {
        if (threadIdx.x == 0) *(i32x4_t*)l.found[pass] = (i32x4_t){p.bin, p.before, p.here, 0};
        __syncthreads();
        const i32x4_t v = *(const i32x4_t*)l.found[pass];
        p = Part{__builtin_amdgcn_readfirstlane(v[0]), __builtin_amdgcn_readfirstlane(v[1]), __builtin_amdgcn_readfirstlane(v[2])};
      }
      return p;
    });
  }
  // in order
  const uint32_t at = part.at;
  const int more = part.more;
  const bool ties = at != 0 && more > 0;
  for (int x = wave; x < groups; x += WAVES) {
    const int n = wave_inscan(above_and_at(mine[64 * x], at, ties));
    if (lane == 63) l.above[x] = n;
  }
  __syncthreads();
  int ups = 0, eqs = 0;                           // in front of the 64 groups at hand
  for (int x0 = 0; x0 < groups; x0 += 64) {
    const int n = x0 + lane < groups ? l.above[x0 + lane] : 0, up = n & 0xFFFF, eq = n >> 16, up_upto = wave_inscan(up), eq_upto = wave_inscan(eq);
    for (int i = wave; i < 64 && x0 + i < groups; i += WAVES) {
      const u32x4_t k = mine[64 * (x0 + i)];
      const int own = above_and_at(k, at, ties), front = wave_inscan(own) - own;
      put_taken(k, ((x0 + i) * 64 + lane) * 4, at, ties, more, top, ups + __builtin_amdgcn_readlane(up_upto - up, i) + (front & 0xFFFF),
                eqs + __builtin_amdgcn_readlane(eq_upto - eq, i) + (front >> 16), put);
    }
    ups += __builtin_amdgcn_readlane(up_upto, 63);
    eqs += __builtin_amdgcn_readlane(eq_upto, 63);
  }
  return ups + min(eqs, more);
}

// Keys of a lane's four blocks b .. b + 3 of nb as the choice takes them.  Those from +0 on go down by one: with that -0, a negative score below half of the smallest number, is
// equal to +0, and kAlways is left to the first and recent ones, so that no more than `top` are taken whatever lies there.  (By a comparison with -0's key 2.5 us of 37 to 58
// with groups of more than 16 heads of 128 over codes, where registers are short.)
__device__ __forceinline__ u32x4_t keys_of(const Sparse& sp, int nb, int b, u32x4_t scored) {
  u32x4_t k;
#pragma unroll
  for (int e = 0; e < 4; ++e) k[e] = b + e >= nb ? kNone : b + e < sp.first || b + e >= nb - sp.recent ? kAlways : scored[e] - (scored[e] >> 31);
  return k;
}
// A row's scores of an earlier launch into LDS, four loads on their way at a time.
template <int THREADS>
__device__ __forceinline__ Seen take_scores(const Sparse& sp, const uint32_t* scored, int nb, int count, uint32_t* keys) {
  Seen seen;
  for (int b0 = 4 * threadIdx.x; b0 < count; b0 += 16 * THREADS) {
    u32x4_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = b0 + 4 * THREADS * i;
      k[i] = (u32x4_t){0, 0, 0, 0};
      if (b < nb) k[i] = *(const u32x4_t*)(scored + b);                // their pitch is a multiple of 64
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = b0 + 4 * THREADS * i;
      if (b < count) {
        k[i] = keys_of(sp, nb, b, k[i]);
        see(seen, k[i]);
        *(u32x4_t*)(keys + b) = k[i];
      }
    }
  }
  return seen;
}
size_t choice_lds(int blocks) { return sizeof(ChoiceLds) + ((size_t)blocks + 255) / 256 * 256 * sizeof(uint32_t); }

// A workgroup for each row and key head: for few rows of many blocks.
constexpr int CHOOSERS = 1024;
__global__ __launch_bounds__(CHOOSERS) void choose_kernel(Paged c, int max_len, bool tree, Sparse sp, int pitch, const uint32_t* __restrict__ scores) {
  extern __shared__ __align__(1024) char smem[];
  const int t = blockIdx.x / c.H;
  Row r;
  if (!row_of(c, t, r)) return;
  const int nb = blocks_up_to(c, seen_end(c, r, t - r.row0, max_len, tree)), count = (nb + 255) & ~255;
  ChoiceLds& choice = *(ChoiceLds*)smem;
  uint32_t* const keys = (uint32_t*)(smem + sizeof(ChoiceLds));
  int32_t* const list = sp.blocks + (long)blockIdx.x * sp.top;
  clear_bins<CHOOSERS>(choice);
  const Seen seen = take_scores<CHOOSERS>(sp, scores + (long)blockIdx.x * pitch, nb, count, keys);
  const int taken = choose<CHOOSERS>(keys, count, seen, sp.top, choice, [&](int at, int b) { list[at] = b; });
  for (int e = taken + (int)threadIdx.x; e < sp.top; e += CHOOSERS) list[e] = -1;
}

// A wave for each row and key head: for many rows of up to 2048 blocks, 32 keys in a lane.  The same steps with 256 parts; nobody waits for others (1024 rows of up to
// 1500 blocks 8.6 us, by workgroups of four waves 9.7).
constexpr int ROW_BLOCKS = 2048;
__global__ __launch_bounds__(256) void choose_rows_kernel(Paged c, int max_len, bool tree, Sparse sp, int pitch, const uint32_t* __restrict__ scores) {
  constexpr int TRIPS = ROW_BLOCKS / 256;
  __shared__ __align__(16) int bins[4][256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long item = (long)blockIdx.x * 4 + wave;
  const int t = (int)(item / c.H);
  Row r;
  if (!row_of(c, t, r)) return;
  const int nb = blocks_up_to(c, seen_end(c, r, t - r.row0, max_len, tree));
  const uint32_t* const scored = scores + item * pitch;
  u32x4_t k[TRIPS];
#pragma unroll
  for (int i = 0; i < TRIPS; ++i) {
    const int b = 256 * i + 4 * lane;
    k[i] = (u32x4_t){0, 0, 0, 0};
    if (b < nb) k[i] = *(const u32x4_t*)(scored + b);
  }
  Seen all;
#pragma unroll
  for (int i = 0; i < TRIPS; ++i) {
    k[i] = keys_of(sp, nb, 256 * i + 4 * lane, k[i]);
    if (256 * i < nb) see(all, k[i]);
  }
  all = over_wave(all);
  Parting part = {0, 0};
  int* const mine = bins[wave];
  if (all.there - all.always > sp.top - all.always) {
    part = parting_key<8>(all.lo, all.hi, sp.top - all.always, [&](int, uint32_t lo, uint32_t width, int shift, int need) {
      ((i32x4_t*)mine)[lane] = (i32x4_t){0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < TRIPS; ++i)
        if (256 * i < nb) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (k[i][e] - lo <= width) atomicAdd(&mine[(k[i][e] - lo) >> shift], 1);
        }
      const i32x4_t v = ((const i32x4_t*)mine)[lane];                  // a wave's accesses to LDS keep their order
      const int own[4] = {v[0], v[1], v[2], v[3]};
      return part_of(own, need);
    });
  }
  const uint32_t at = part.at;
  const int more = part.more;
  const bool ties = at != 0 && more > 0;
  int32_t* const list = sp.blocks + item * sp.top;
  int ups = 0, eqs = 0;
#pragma unroll
  for (int i = 0; i < TRIPS; ++i)
    if (256 * i < nb) {
      const int own = above_and_at(k[i], at, ties), upto = wave_inscan(own), front = upto - own, sum = __builtin_amdgcn_readlane(upto, 63);
      put_taken(k[i], 256 * i + 4 * lane, at, ties, more, sp.top, ups + (front & 0xFFFF), eqs + (front >> 16), [&](int place, int b) { list[place] = b; });
      ups += sum & 0xFFFF;
      eqs += sum >> 16;
    }
  for (int e = ups + min(eqs, more) + lane; e < sp.top; e += 64) list[e] = -1;
}

// ---- attention over the choice

// Bound by memory: 64 single tokens of 2048 positions each over e4m3, scores and choice included, 75 us, 350 MB, 4.7 TB/s; trees of eight tokens, 1536 positions each over bf16,
// 105 us, 7.7 TB/s with what rows of a sequence have in common.  Few items: by the chain of a tile's instructions, 2500 cycles.  An item is the query heads of one key head of one
// row, M of them, over its blocks one behind the other: positions v = 0 .. top page_size - 1 of a list.  They all see the same.  The list is the caller's (GIVEN), or chosen
// first: by scores of an earlier launch (SCORES), or by the workgroup's own (WHOLE), for whom keys and values of the choice and all summaries are read at once.  KW waves take
// every KW-th tile of 32; `pieces` workgroups share a long list, sparse_join_kernel adds them up.  Forms of tiles, products and softmax as in the attention over whole caches
// (attend.hip); what the row does not see is -infinity among the scores and zeros in V.
// A wave has two tiles in LDS, one on its way while the other is computed; 16-bit rows of more than 64 elements one, whose keys are replaced by the next once they are in
// registers, and its values then: two waves on each unit instead of one that holds twice as much (us of a call, 1024 items of 1536 positions 158 and 149, 512 of 2048 137 and
// 128, 1024 of 2048 229 and 215).  Four tiles of codes for a wave measured the same for few items.
constexpr int KT = 32;
enum { GIVEN, SCORES, WHOLE };
struct Listed {
  int pieces, span;                    // span: positions of a piece, a multiple of 128
  int from, pitch;                     // from: GIVEN, SCORES, WHOLE; pitch: of the scores of an item
  const uint32_t* scores;
};
constexpr int OWN_BLOCKS = 4096;       // of a choice by a workgroup of the attention


template <int DT, int KEPT, int D, int M, int KW> struct Sizes {
  typedef Form<DT, KEPT, D> F;
  static constexpr bool CODES = KEPT != DT;
  static constexpr int TILE = KT * F::ROWB, STAGE = 2 * TILE + (CODES ? 8 * KT : 0), SLOT = D * M * 4 + 512;
  static constexpr bool ONE = !CODES && D > 64;       // room for one tile of a wave, else for two
  static constexpr int TILES = KW * (ONE ? 1 : 2) * STAGE, JOIN = (KW - 1) * SLOT;
  static constexpr int LDS = TILES > JOIN ? TILES : JOIN;
};

template <int DT, int KEPT, int D, int M, int KW>
__global__ __launch_bounds__(64 * KW, 2) void sparse_attend_kernel(Paged c, Attend a, Sparse sp, Listed ls, float* __restrict__ part, f32x2_t* __restrict__ stat) {
  typedef Sizes<DT, KEPT, D, M, KW> Z;
  constexpr int THREADS = 64 * KW;
  typedef Form<DT, KEPT, D> F;
  constexpr bool CODES = KEPT != DT, ONE = Z::ONE;
  constexpr int VDT = CODES ? DT_BF16 : DT;
  // p (v_scale) in two 16-bit parts, as single tokens of the whole cache have it
  constexpr bool SPLIT_P = CODES || DT == DT_BF16;
  typedef Operand<DT, M> P1;
  typedef Operand<VDT, M> P2;
  typedef typename P1::vec vec;
  typedef typename P2::vec vvec;
  typedef typename P1::acc acc;
  constexpr int NG = 64 / M, KM = 8 * NG, CA = M * M / 64;
  constexpr int DM = D / M, KS = D / KM, ST = KT / M, NX = KT / KM;
  constexpr int TILE = Z::TILE, STAGE = Z::STAGE, LOADS = KT / F::RPI;
  extern __shared__ __align__(1024) char smem[];
  __shared__ int list_page[1024], list_block[1024], list_end;
  const int tid = threadIdx.x, lane = tid & 63, kw = __builtin_amdgcn_readfirstlane(tid >> 6), grp = lane / M;
  const int G = a.heads / c.H, shift = c.page_shift, page_mask = (1 << shift) - 1;
  const int g = blockIdx.x % c.H, x = blockIdx.x / c.H, t = x % c.T, piece = x / c.T, h0 = blockIdx.y * M;
  // what goes by the row's number alone is on its way first: a given list, the queries
  const int begin = piece * ls.span, end = min(begin + ls.span, sp.top << shift);
  const int e0 = begin >> shift, entries = ((end - 1) >> shift) - e0 + 1;
  int32_t* const list = sp.blocks + ((long)t * c.H + g) * sp.top;
  int listed = -1;
  if (ls.from == GIVEN && tid < entries) listed = list[e0 + tid];
  const int in_tile = lane % M, rg = h0 + in_tile, head = g * G + rg;
  const bool has = rg < G;
  const float unit = fmaxf(fabsf(a.scale), 1.2e-38f), c2 = unit * kLog2E;
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;             // a negative scale negates the query
  u32x4_t raw_q[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    raw_q[k] = (u32x4_t){};
    if (has) raw_q[k] = *(const u32x4_t*)((const uint16_t*)a.q + t * a.q_pitch + (long)head * D + KM * k + 8 * grp);
  }

  Row row;
  if (!row_of(c, t, row)) return;
  const int hi = seen_end(c, row, t - row.row0, a.max_len, a.visible != nullptr);
  const int always = a.visible ? min(row.old, hi) : hi;                // below this every position is seen
  const unsigned long long bits = a.visible ? (unsigned long long)a.visible[t] : 0;

  // ---- the piece's blocks
  if (tid == 0) list_end = 0;
  if (ls.from == GIVEN) {
    for (int e = tid; e < entries; e += THREADS) list_block[e] = e == tid ? listed : list[e0 + e];
  } else {
    const int nb = blocks_up_to(c, hi), count = (nb + 255) & ~255;
    ChoiceLds& choice = *(ChoiceLds*)smem;
    uint32_t* const keys = (uint32_t*)(smem + sizeof(ChoiceLds));
    Seen seen;
    clear_bins<THREADS>(choice);
    if (ls.from == SCORES) {
      seen = take_scores<THREADS>(sp, ls.scores + ((long)t * c.H + g) * ls.pitch, nb, count, keys);
    } else {
      constexpr int NT = M == 16 ? 1 : 4;
      Scored<D> next;
      int id = block_id(c, row.s, kw * 64 + lane, nb);
      Queries<D, NT> raw;
      load_queries<D, NT>([&](int y) -> const uint16_t* {
        const int h = 16 * y + (lane & 15);
        return h < G ? (const uint16_t*)a.q + t * a.q_pitch + (long)(g * G + h) * D : nullptr;
      }, raw);
      if (kw * 64 < nb) load_blocks<D>(c, g, sp.summary, sp.scales, id, next);
      id = block_id(c, row.s, THREADS + kw * 64 + lane, nb);
      Codes<D, NT> codes;
      query_codes<DT, D, NT>(raw, G, codes);
      for (int b0 = kw * 64; b0 < count; b0 += THREADS) {
        const Scored<D> now = next;
        if (b0 + THREADS < nb) load_blocks<D>(c, g, sp.summary, sp.scales, id, next);
        id = block_id(c, row.s, b0 + 2 * THREADS + lane, nb);
        if (b0 < nb) {
          score_blocks<D, NT>(now, codes, 16 * NT, G, [&](int, int j, u32x4_t scored) {
            const int b = b0 + 16 * j + 4 * (lane >> 4);
            scored = keys_of(sp, nb, b, scored);
            see(seen, scored);
            *(u32x4_t*)(keys + b) = scored;
          });
        } else {
          keys[b0 + lane] = kNone;
        }
      }
    }
    const bool writes = piece == 0 && blockIdx.y == 0;
    const int taken = choose<THREADS>(keys, count, seen, sp.top, choice, [&](int at, int b) {
      if (at >= e0 && at < e0 + entries) list_block[at - e0] = b;
      if (writes) list[at] = b;
    });
    for (int e = tid; e < sp.top; e += THREADS)
      if (e >= taken) {
        if (e >= e0 && e < e0 + entries) list_block[e - e0] = -1;
        if (writes) list[e] = -1;
      }
  }
  __syncthreads();
  for (int e = tid; e < entries; e += THREADS) {
    const int b = list_block[e];
    int page = -1;
    if (b >= 0 && b < c.max_pages && ((long)b << shift) < hi) page = c.pages[(long)row.s * c.max_pages + b];
    if (page >= c.n_pages) page = -1;
    list_page[e] = page;
    if (page >= 0) atomicMax(&list_end, e + 1);
  }
  __syncthreads();
  const int stop = min(end, (e0 + __builtin_amdgcn_readfirstlane(list_end)) << shift);
  const int count = max(stop - begin + KT - 1, 0) / KT, mine = kw < count ? (count - kw + KW - 1) / KW : 0;

  vec q[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) q[k] = __builtin_bit_cast(vec, raw_q[k] ^ flip);

  // ---- tiles into LDS
  const unsigned base = (unsigned)(uintptr_t)(lds_char*)smem + kw * (ONE ? 1 : 2) * STAGE;
  // 16 positions of the list from v on: their page (-1: nothing there) and block
  struct Groups { int page[2], block[2]; };
  auto look_up = [&](int tile) {
    Groups r;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int v = begin + tile * KT + 16 * u, e = min(v >> shift, (stop - 1) >> shift) - e0;
      r.page[u] = __builtin_amdgcn_readfirstlane(v < stop ? list_page[e] : -1);
      r.block[u] = __builtin_amdgcn_readfirstlane(list_block[e]);
    }
    return r;
  };
  // a tile's keys, values or both (with the scales of codes)
  auto fetch = [&](int tile, const Groups& w, int stage, bool keys, bool values) __attribute__((always_inline)) {
    const unsigned to = base + stage * STAGE;
    long at[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) at[u] = (((long)max(w.page[u], 0) * c.H + g) << shift) + ((begin + tile * KT + 16 * u) & page_mask);
    if constexpr (CODES) {
      const int y = lane & 31;
      load4_lds(to + 2 * TILE, (lane < 32 ? a.ks : a.vs) + (y < 16 ? at[0] : at[1]) + (y & 15));
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int x0 = i * F::RPI, xr = (x0 & 15) + lane / F::CH, part_of = (lane % F::CH) ^ F::turn(xr);
      if (F::PIECES == F::CH || part_of < F::PIECES) {
        const long where = uniform(at[x0 / 16]);
        const unsigned off = (unsigned)xr * (D * F::ESZ) + part_of * 16;
        if (keys) load16_lds(to + x0 * F::ROWB, (const char*)a.kc + where * (D * F::ESZ), off);
        if (values) load16_lds(to + TILE + x0 * F::ROWB, (const char*)a.vc + where * (D * F::ESZ), off);
      }
    }
  };
  // bit x: the row sees position x of the tile
  auto seen_in = [&](int tile, const Groups& w) {
    uint32_t see = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const long j0 = ((long)w.block[u] << shift) + ((begin + tile * KT + 16 * u) & page_mask);
      auto below = [](long k) { return k <= 0 ? 0ull : k >= 64 ? ~0ull : (1ull << k) - 1; };
      unsigned long long m = below(always - j0);
      if (a.visible && j0 + 16 > row.old) {
        const long by = row.old - j0;
        m |= (by >= 64 || by <= -64 ? 0ull : by >= 0 ? bits << by : bits >> -by) & below(hi - j0);
      }
      see |= (w.page[u] >= 0 ? (uint32_t)m & 0xFFFFu : 0u) << (16 * u);
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)see);
  };

  acc o[DM];
#pragma unroll
  for (int d = 0; d < DM; ++d)
#pragma unroll
    for (int e = 0; e < CA; ++e) o[d][e] = 0.f;
  float m = -INFINITY, ref = 0.f, sum = 0.f;
  bool far = false;

  int kbase[M == 16 ? 2 : 1];
#pragma unroll
  for (int b = 0; b < (M == 16 ? 2 : 1); ++b) {
    const int y = M == 16 ? (lane & 3) | (lane & 12) << 1 | b << 2 : (lane & 3) | (lane & 8) >> 1 | (lane & 4) << 1 | (lane & 16);
    kbase[b] = y * F::ROWB + (CODES ? ((grp >> 1) ^ F::turn(y)) * 16 + 8 * (grp & 1) : (grp ^ F::turn(y)) * 16);
  }
  const int vcol = M == 16 ? 0 : lane >> 4 & 1, vj = lane & 15;
  int vbase[CODES ? 1 : 2];
  if constexpr (CODES) {
    const int y = 8 * grp + vj / 2;
    vbase[0] = y * F::ROWB + (vcol ^ F::turn(y)) * 16 + 8 * (vj & 1);
  } else {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int y = 8 * grp + 4 * b + vj / 4;
      vbase[b] = y * F::ROWB + ((2 * vcol + (vj >> 1 & 1)) ^ F::turn(y)) * 16 + 8 * (vj & 1);
    }
  }
  typedef std::conditional_t<CODES, u32x2_t, u32x4_t> raw_t;

  // ONE: with the keys of the tile there and its values behind them; `next` is the tile to come, if there is one
  auto work = [&](uint32_t see, int stage, int tile, const Groups& next, bool more) __attribute__((always_inline)) {
    const lds_char* const kt = (const lds_char*)(base + stage * STAGE);
    lds_char* const vt = (lds_char*)(base + stage * STAGE + TILE);
    const __attribute__((address_space(3))) float* const scales = (const __attribute__((address_space(3))) float*)(base + stage * STAGE + 2 * TILE);
    const bool partial = see != ~0u;
    auto clear_unseen = [&] {                                          // 0 * v is NaN where v is not finite
#pragma unroll
      for (int i = 0; i < KT * F::CH / 64; ++i) {
        const int y = (i * 64 + lane) / F::CH;
        if (!(see >> y & 1)) *(__attribute__((address_space(3))) u32x4_t*)(vt + (i * 64 + lane) * 16) = (u32x4_t){};
      }
    };
    if (!ONE && partial) clear_unseen();
    raw_t kf[ST][KS];
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int k = 0; k < KS; ++k)
        kf[st][k] = *(const __attribute__((address_space(3))) raw_t*)(kt + (M == 16 ? st / 2 : st) * 32 * F::ROWB + (kbase[M == 16 ? st & 1 : 0] ^ k * KM * F::ESZ));
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (ONE) {
      wait_lds();
      if (more) fetch(tile, next, 0, true, false);
    }
    acc sc[ST];
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int e = 0; e < CA; ++e) sc[st][e] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int st = 0; st < ST; ++st) {
        u32x4_t w;
        if constexpr (CODES) w = widen8<DT, KEPT>(kf[st][k]); else w = kf[st][k];
        sc[st] = P1::mfma(__builtin_bit_cast(vec, w), q[k], sc[st]);
      }
    float z[NX][8];                                                    // position KM x + 8 group + e
#pragma unroll
    for (int y = 0; y < NX; ++y)
#pragma unroll
      for (int e = 0; e < 8; ++e) z[y][e] = M == 16 ? sc[2 * y + e / 4][e % 4] : sc[y / 2][8 * (y & 1) + e];
    if constexpr (CODES) {
#pragma unroll
      for (int y = 0; y < NX; ++y)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const f32x4_t w = *(const __attribute__((address_space(3))) f32x4_t*)(scales + KM * y + 8 * grp + 4 * f);
#pragma unroll
          for (int e = 0; e < 4; ++e) z[y][4 * f + e] *= w[e];
        }
    }
    if (partial) {
#pragma unroll
      for (int y = 0; y < NX; ++y) {
        const uint32_t w = see >> (8 * grp) >> (KM * y);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[y][e] = w & (1u << e) ? z[y][e] : -INFINITY;
      }
    }
    float top = z[0][0];
#pragma unroll
    for (int y = 0; y < NX; ++y)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, z[y][e]);
    top = row_max<M>(top);
    const bool grow = (top - m) * c2 > kSlack;                         // m = -infinity: whenever something is seen
    if (__any(grow)) {
      const float next = grow ? top : m;
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - next) * c2);
      sum *= keep;
#pragma unroll
      for (int d = 0; d < DM; ++d)
#pragma unroll
        for (int e = 0; e < CA; ++e) o[d][e] *= keep;
      m = next;
      ref = m == -INFINITY ? 0.f : m * c2;
      far = __any(fabsf(ref) > 1e38f);
    }
    raw_t vf[2][DM];
    auto load_v = [&](int y) {
#pragma unroll
      for (int d = 0; d < DM; ++d) {
        if constexpr (CODES) {
          typedef __attribute__((address_space(3))) i32x2_t L;
          vf[y & 1][d] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((L*)(vt + y * KM * F::ROWB + (vbase[0] ^ d * M))));
        } else {
          typedef __attribute__((address_space(3))) s16x4_t L;
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const u32x2_t raw = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(vt + y * KM * F::ROWB + (vbase[b] ^ d * 2 * M))));
            vf[y & 1][d][2 * b] = raw[0];
            vf[y & 1][d][2 * b + 1] = raw[1];
          }
        }
      }
    };
    if constexpr (!ONE) load_v(0);
    if (__builtin_expect(far, 0)) {
      const float from = m == -INFINITY ? 0.f : m;                     // then all scores are -infinity or NaN: zeros or NaN
#pragma unroll
      for (int y = 0; y < NX; ++y)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[y][e] = __builtin_amdgcn_exp2f((z[y][e] - from) * c2);
    } else {
#pragma unroll
      for (int y = 0; y < NX; ++y)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[y][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[y][e], c2, -ref));
    }
    float part_sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int y = 0; y < NX; ++y)
#pragma unroll
      for (int e = 0; e < 8; ++e) part_sum[e & 3] += z[y][e];
    sum += (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
    if constexpr (CODES) {
#pragma unroll
      for (int y = 0; y < NX; ++y)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const f32x4_t w = *(const __attribute__((address_space(3))) f32x4_t*)(scales + KT + KM * y + 8 * grp + 4 * f);
#pragma unroll
          for (int e = 0; e < 4; ++e) {                                // the scale of a row that is not seen may be anything
            const bool unseen = partial && !(see >> (8 * grp) >> (KM * y + 4 * f + e) & 1);
            z[y][4 * f + e] = unseen ? 0.f : z[y][4 * f + e] * w[e];
          }
        }
    }
    u32x4_t prob[NX], rest[SPLIT_P ? NX : 1];
#pragma unroll
    for (int y = 0; y < NX; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a0 = z[y][2 * e], a1 = z[y][2 * e + 1];
        if constexpr (SPLIT_P && !CODES) {
          // cut, not rounded, and the second part a little larger: both are above zero, and an infinity in v times them is one
          constexpr float more = 1.f + 0x1p-20f;
          const uint32_t f0 = __float_as_uint(a0) & 0xFFFF0000u, f1 = __float_as_uint(a1) & 0xFFFF0000u;
          prob[y][e] = f0 >> 16 | f1;
          rest[y][e] = Half<VDT>::pack(__builtin_fmaf(a0, more, -__uint_as_float(f0)), __builtin_fmaf(a1, more, -__uint_as_float(f1)));
        } else {
          prob[y][e] = Half<VDT>::pack(a0, a1);
          if constexpr (SPLIT_P) rest[y][e] = Half<VDT>::pack(a0 - bf16lo_to_f32(prob[y][e]), a1 - bf16hi_to_f32(prob[y][e]));
        }
      }
    if constexpr (ONE) {
      __builtin_amdgcn_sched_barrier(0);
      if (more) wait_loads<LOADS>(); else wait_loads<0>();
      __builtin_amdgcn_sched_barrier(0);
      if (partial) clear_unseen();
      load_v(0);
    }
#pragma unroll
    for (int y = 0; y < NX; ++y) {
      if (y + 1 < NX) load_v(y + 1);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (ONE) {
        if (y + 1 == NX) {
          wait_lds();
          if (more) fetch(tile, next, 0, false, true);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int d = 0; d < DM; ++d) {
        u32x4_t w;
        if constexpr (CODES) w = widen8<VDT, KEPT>(vf[y & 1][d]); else w = vf[y & 1][d];
        o[d] = P2::mfma(__builtin_bit_cast(vvec, w), __builtin_bit_cast(vvec, prob[y]), o[d]);
        if constexpr (SPLIT_P) o[d] = P2::mfma(__builtin_bit_cast(vvec, w), __builtin_bit_cast(vvec, rest[y]), o[d]);
      }
    }
  };

  if (mine > 0) {
    Groups now = look_up(kw), next = {};
    fetch(kw, now, 0, true, !ONE);
    if constexpr (ONE) fetch(kw, now, 0, false, true);
    if (mine > 1) next = look_up(kw + KW);
    for (int i = 0; i < mine; ++i) {
      const Groups here = now;
      const bool more = i + 1 < mine;
      const int behind = kw + (i + 1) * KW;                            // the tile to come
      if constexpr (ONE) {
        const uint32_t see = seen_in(kw + i * KW, here);
        wait_loads<LOADS>();                                           // the keys
        __builtin_amdgcn_sched_barrier(0);
        if (see != 0) {
          work(see, 0, behind, next, more);
        } else {
          wait_loads<0>();
          if (more) {
            fetch(behind, next, 0, true, false);
            fetch(behind, next, 0, false, true);
          }
        }
        now = next;
        if (i + 2 < mine) next = look_up(behind + KW);
      } else {
        if (more) {
          fetch(behind, next, (i + 1) & 1, true, true);
          now = next;
          if (i + 2 < mine) next = look_up(behind + KW);
          wait_loads<2 * LOADS + (CODES ? 1 : 0)>();
        } else {
          wait_loads<0>();
        }
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t see = seen_in(kw + i * KW, here);
        if (see != 0) work(see, i & 1, 0, next, false);
        __builtin_amdgcn_sched_barrier(0);
        wait_lds();                                                    // nothing reads the stage that is filled next
      }
    }
  }
  sum = row_sum<M>(sum);
  m *= unit;                                                           // in units of the scores

  // ---- the waves
  __syncthreads();
  if (kw > 0) {
    char* const to = smem + (kw - 1) * Z::SLOT;
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int b = 0; b < CA / 4; ++b) *(f32x4_t*)(to + (d * (CA / 4) + b) * 1024 + lane * 16) = (f32x4_t){o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
    *(float*)(to + D * M * 4 + lane * 4) = m;
    *(float*)(to + D * M * 4 + 256 + lane * 4) = sum;
  }
  __syncthreads();
  if (kw > 0) return;
#pragma unroll
  for (int w = 0; w < KW - 1; ++w) {
    const char* const other = smem + w * Z::SLOT;
    const float m2 = *(const float*)(other + D * M * 4 + lane * 4), s2 = *(const float*)(other + D * M * 4 + 256 + lane * 4);
    const float top = fmaxf(m, m2), zero = top == -INFINITY ? 0.f : top;
    const float f1 = __builtin_amdgcn_exp2f((m - zero) * kLog2E), f2 = __builtin_amdgcn_exp2f((m2 - zero) * kLog2E);
    sum = sum * f1 + s2 * f2;
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int b = 0; b < CA / 4; ++b) {
        const f32x4_t v = *(const f32x4_t*)(other + (d * (CA / 4) + b) * 1024 + lane * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][4 * b + e] = o[d][4 * b + e] * f1 + v[e] * f2;
      }
    m = top;
  }
  if (!has) return;
  if (ls.pieces == 1) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t* const out = (uint16_t*)a.out + t * a.out_pitch + (long)head * D;
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int b = 0; b < CA / 4; ++b)
        *(u32x2_t*)(out + M * d + 8 * b + 4 * grp) = (u32x2_t){Half<DT>::pack(o[d][4 * b] * inv, o[d][4 * b + 1] * inv), Half<DT>::pack(o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv)};
    if (a.lse && grp == 0) a.lse[(long)t * a.heads + head] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
  } else {
    const long to = ((long)t * a.heads + head) * ls.pieces + piece;
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int b = 0; b < CA / 4; ++b) *(f32x4_t*)(part + to * D + M * d + 8 * b + 4 * grp) = (f32x4_t){o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
    if (grp == 0) stat[to] = (f32x2_t){m, sum};
  }
}

// Adds up the pieces of a row and head, 32 lanes a row, eight pieces on their way at once.
constexpr int JT = 256;
template <int DT, int D>
__global__ __launch_bounds__(JT) void sparse_join_kernel(Paged c, Attend a, int pieces, const float* __restrict__ part, const f32x2_t* __restrict__ stat) {
  const long row = (long)blockIdx.x * (JT / 32) + threadIdx.x / 32;
  const int at = threadIdx.x & 31;
  if (row >= (long)c.T * a.heads) return;
  const int t = (int)(row / a.heads), head = (int)(row % a.heads);
  if (t < c.start[0] || t >= c.start[c.S]) return;
  float m = -INFINITY;
  for (int k = at; k < pieces; k += 32) m = fmaxf(m, stat[row * pieces + k][0]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float zero = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < pieces; k0 += 8) {
    f32x2_t st[8];
    f32x4_t v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long from = row * pieces + min(k0 + k, pieces - 1);
      st[k] = stat[from];
      v[k] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
      if (at * 4 < D) v[k] = *(const f32x4_t*)(part + from * D + at * 4);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const bool has = k0 + k < pieces;
      const float f = has ? __builtin_amdgcn_exp2f((st[k][0] - zero) * kLog2E) : 0.f;
      sum += has ? st[k][1] * f : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += has ? v[k][e] * f : 0.f;
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (at * 4 < D)
    *(u32x2_t*)((uint16_t*)a.out + t * a.out_pitch + (long)head * D + at * 4) = (u32x2_t){Half<DT>::pack(o[0] * inv, o[1] * inv), Half<DT>::pack(o[2] * inv, o[3] * inv)};
  if (a.lse && at == 0) a.lse[(long)t * a.heads + head] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
}

// ---- launches

int blocks_of(const Paged& c, int max_len) { return (int)(((long)max_len + (1 << c.page_shift) - 1) >> c.page_shift); }
int key_pitch(const Paged& c, int max_len) { return (blocks_of(c, max_len) + 63) / 64 * 64; }
int run_of(int G) {
  int gp = 1;
  while (gp < G) gp *= 2;
  return gp;
}

// Workgroups that lists are cut for: two to a compute unit, or one where tiles are 16 KB and two share its loads (192 items of 2048 positions, us of a call: 50.2, cut for 512 53.7).
int slots_of(const Paged& c) { return c.kept == c.dtype && c.D > 64 ? 256 : 512; }

// Where the items would not fill half of the device their lists are cut, into up to 16 pieces of 256 positions or more.  us of a call in a graph, one token of 8 key heads over
// bf16: 1536 positions in one piece 29.9, in six 24.7; 2048 in four 26.2, in eight 25.0; 4096 in eight 26.6, in 16 26.1; 8192 in 16 29.4, in 32 31.0.  1024 positions 26.7 and in
// four pieces 24.5, but the launch that joins them takes the host 3 us, which calls from Python wait for: only tiles of 32 heads, in four waves, are cut there (34.1 and 28.3).
struct Pieces { int pieces, span; };
Pieces pieces_of(const Paged& c, int heads, int top) {
  const int G = heads / c.H, M = G <= 16 ? 16 : 32;
  const long items = (long)c.T * c.H * ((G + M - 1) / M), positions = (long)top << c.page_shift;
  const int slots = slots_of(c);
  long pieces = 2 * items > slots || positions < (M == 16 ? 1536 : 1024) ? 1 : std::min<long>(slots / items, std::min<long>(positions / 256, 16));
  long span = ((positions + pieces - 1) / pieces + 127) / 128 * 128;
  pieces = (positions + span - 1) / span;
  return Pieces{(int)pieces, (int)span};
}

int choice_from(const Paged& c, int max_len, const Sparse& sp);
size_t key_bytes(const Paged& c, int max_len, const Sparse& sp) {
  return choice_from(c, max_len, sp) == SCORES ? ((size_t)c.T * c.H * key_pitch(c, max_len) * sizeof(uint32_t) + 255) / 256 * 256 : 0;
}

// Which way the choice goes.  An item's own workgroup scores, chooses and attends (WHOLE) where there is a workgroup for each compute unit and rows do not share their
// sequence's summaries, or these are little beside the keys and values and all items are at work at once.  us of a call and its summaries with the choice in one launch, in two
// (SCORES), in three (apart, below): 64 single tokens behind 9000 to 61000 positions over bf16 136, 149, 152, of head dimension 64 67, 76, 80, over e4m3 85, 99, 103; 256 behind
// 2000 to 20000 over e4m3 254, 271, 269; 12 rows of 32 heads of their own 34.5, 35.8, 37.8; but 4 tokens each of 64 sequences (2048 items) over bf16 184, 182, 176.  With fewer
// items it does so where a workgroup scores a sequence in one or two steps: one token of 32 heads in one launch and in three behind 120 blocks 26.9 and 27.5 (codes 30.4 and
// 31.2), 250 blocks 27.7 and 28.5 (31.3 and 32.1), 500 blocks 29.9 and 28.6 (33.5 and 31.9), 1000 blocks 33.6 and 28.4; 8 tokens behind 250 blocks 29.7 and 30.8, 500 blocks
// 32.0 and 30.7 (with four waves each; eight take 2 to 3 us less of all).
int choice_from(const Paged& c, int max_len, const Sparse& sp) {
  if (sp.given) return GIVEN;
  const long nb = blocks_of(c, max_len), row = (long)c.D * (c.kept == c.dtype ? 2 : 1);
  const bool alone = 2l * c.T <= 3l * c.S, cheap = (long)c.T * c.H <= slots_of(c) && nb * (2 * c.D + 4) * 4 <= ((long)sp.top << c.page_shift) * 2 * row;
  return (long)c.T * c.H < 256 ? (nb <= 256 ? WHOLE : SCORES) : (nb <= OWN_BLOCKS && (alone || cheap) ? WHOLE : SCORES);
}

template <int DT, int D>
hipError_t launch_scores(const Paged& c, const Attend& a, const Sparse& sp, uint32_t* keys, hipStream_t stream) {
  const int nb = blocks_of(c, a.max_len), pitch = key_pitch(c, a.max_len), gp = run_of(a.heads / c.H), chunks = (nb + SCORED - 1) / SCORED;
  const bool one = gp <= 16 && (long)c.T * gp <= 16l * c.S;            // 16 columns hold the rows of a sequence, in the mean
  const int tokens = (one ? 16 : 64) / gp;
  const dim3 grid((unsigned)(std::min<long>(c.T, c.T / tokens + (long)c.S) * c.H * chunks));
  if (one)
    hipLaunchKernelGGL((score_kernel<DT, D, 1>), grid, dim3(256), 0, stream, c, a, gp, chunks, pitch, sp.summary, sp.scales, keys);
  else
    hipLaunchKernelGGL((score_kernel<DT, D, 4>), grid, dim3(256), 0, stream, c, a, gp, chunks, pitch, sp.summary, sp.scales, keys);
  return hipGetLastError();
}

PerDeviceInt raised_choose;
hipError_t launch_choice(const Paged& c, const Attend& a, const Sparse& sp, int pitch, const uint32_t* scores, hipStream_t stream) {
  const int nb = blocks_of(c, a.max_len);
  const long rows = (long)c.T * c.H;
  if (nb <= ROW_BLOCKS && rows >= 128) {
    hipLaunchKernelGGL(choose_rows_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, c, a.max_len, a.visible != nullptr, sp, pitch, scores);
    return hipGetLastError();
  }
  hipError_t e = ensure_dynamic_lds(raised_choose, (const void*)choose_kernel, choice_lds(nb));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(choose_kernel, dim3((unsigned)rows), dim3(CHOOSERS), choice_lds(nb), stream, c, a.max_len, a.visible != nullptr, sp, pitch, scores);
  return hipGetLastError();
}

template <int DT, int KEPT, int D, int M, int KW>
hipError_t launch_form(const Paged& c, const Attend& a, const Sparse& sp, void* ws, hipStream_t stream) {
  const Pieces pc = pieces_of(c, a.heads, sp.top);
  int from = choice_from(c, a.max_len, sp);
  const int nb = blocks_of(c, a.max_len), pitch = key_pitch(c, a.max_len);
  // A launch of its own chooses where many pieces, or some thousand workgroups at a compute unit each or two, would do it beside their loads.  us of a call inside and apart:
  // 2048 items over e4m3 125 and 116, over bf16 182 and 176, 1024 over bf16 114 and 113, 768 over e4m3 68.7 and 68.1; but 512 over bf16 62.1 and 64.4, 256 41.7 and 44.0.  The
  // attention alone for 16 items in 16 pieces of 15626 blocks: 104, and 13 + 12 apart.
  const bool apart = from == SCORES && (nb > OWN_BLOCKS || (long)pc.pieces * nb > 8192 || (long)c.T * c.H * pc.pieces >= 1024);
  const size_t lds = std::max<size_t>(Sizes<DT, KEPT, D, M, KW>::LDS, from == GIVEN || apart ? 0 : choice_lds(nb));
  static PerDeviceInt raised;
  hipError_t e = ensure_dynamic_lds(raised, (const void*)sparse_attend_kernel<DT, KEPT, D, M, KW>, lds);
  if (e != hipSuccess) return e;
  if (from == SCORES && (e = launch_scores<DT, D>(c, a, sp, (uint32_t*)ws, stream)) != hipSuccess) return e;
  if (apart) {
    e = launch_choice(c, a, sp, pitch, (const uint32_t*)ws, stream);
    if (e != hipSuccess) return e;
    from = GIVEN;
  }
  float* part = (float*)((char*)ws + key_bytes(c, a.max_len, sp));
  f32x2_t* stat = (f32x2_t*)(part + (size_t)c.T * a.heads * pc.pieces * D);
  const Listed ls{pc.pieces, pc.span, from, pitch, (const uint32_t*)ws};
  const int G = a.heads / c.H;
  hipLaunchKernelGGL((sparse_attend_kernel<DT, KEPT, D, M, KW>), dim3((unsigned)((long)c.T * c.H * pc.pieces), (G + M - 1) / M), dim3(64 * KW), lds, stream, c, a, sp, ls, part, stat);
  if ((e = hipGetLastError()) != hipSuccess || pc.pieces == 1) return e;
  const long rows = (long)c.T * a.heads;
  hipLaunchKernelGGL((sparse_join_kernel<DT, D>), dim3((unsigned)((rows + JT / 32 - 1) / (JT / 32))), dim3(JT), 0, stream, c, a, pc.pieces, (const float*)part, (const f32x2_t*)stat);
  return hipGetLastError();
}

// f(16-bit type, kind of cache, head dimension) with the three as constants
template <typename F>
hipError_t with_forms(const Paged& c, F f) {
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

}  // namespace

size_t sparse_workspace_bytes(const Paged& c, int heads, int max_len, const Sparse& sp) {
  const Pieces pc = pieces_of(c, heads, sp.top);
  const size_t parts = pc.pieces == 1 ? 0 : (size_t)c.T * heads * pc.pieces * (c.D + 2) * sizeof(float);
  return std::max<size_t>(key_bytes(c, max_len, sp) + parts, 256);
}

// A launch has fewer than 2^32 threads.
bool sparse_fits(const Paged& c, int heads, int max_len, int top) {
  const long nb = blocks_of(c, max_len);
  if (nb > 32768) return false;
  const double rows = (double)c.T * c.H;
  const Pieces pc = pieces_of(c, heads, top);
  return rows * ((nb + SCORED - 1) / SCORED) * 256 < 4e9 && rows * pc.pieces * 256 < 4e9 && rows * 1024 < 4e9 && (double)c.T * heads * 32 < 4e9;
}

// Pages that the rows of a call touch, at most, and whether its rows are fewer.
static long touched_pages(const Paged& c, bool* by_row) {
  const long touched = ((long)c.T >> c.page_shift) + 2l * c.S;
  *by_row = c.T <= touched;
  return std::min<long>(c.T, touched);
}

bool summary_fits(const Paged& c) {
  bool by_row;
  return (double)touched_pages(c, &by_row) * c.H * 256 < 4e9;
}

hipError_t launch_summary(const Paged& c, const void* kc, const float* ks, int8_t* summary, float* scales, hipStream_t stream) {
  return with_forms(c, [&](auto dt, auto kept, auto dim) {
    bool by_row;
    const long items = touched_pages(c, &by_row) * c.H;
    // pages of 128 as well where those that the sequences end in and fill are no more than the compute units (us of 256 items 6.8 and 5.9, over e4m3 8.7 and 8.0; of 320 8.7 and 9.8)
    const bool large = c.page_shift >= 8 || (c.page_shift == 7 && std::min<long>(c.T, (c.T >> 7) + c.S) * c.H <= 256);
    auto go = [&](auto kernel, int per) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((items + per - 1) / per)), dim3(256), 0, stream, c, items, kc, ks, summary, scales);
      return hipGetLastError();
    };
    if (large && by_row) return go((summary_kernel<dt.value, kept.value, dim.value, 4, true>), 1);
    if (large) return go((summary_kernel<dt.value, kept.value, dim.value, 4, false>), 1);
    if (by_row) return go((summary_kernel<dt.value, kept.value, dim.value, 1, true>), 4);
    return go((summary_kernel<dt.value, kept.value, dim.value, 1, false>), 4);
  });
}

hipError_t launch_sparse(const Paged& c, const Attend& a, const Sparse& sp, void* ws, hipStream_t stream) {
  return with_forms(c, [&](auto dt, auto kept, auto dim) {
    const int G = a.heads / c.H;
    // Eight waves, two on each unit of a compute unit, where there is half a workgroup for each: a tile is 2500 cycles of instructions that wait for one another.  us of a call
    // with four waves and with eight: a token of 32 / 8 heads 28.7 and 26.1 (head dimension 64 23.7 and 21.2, e4m3 32.3 and 29.2), 16 tokens 28.3 and 26.0; but 32 tokens 40.1
    // and 41.6, and with tiles of 32 heads 16 tokens of two key heads 35.7 and 40.4.
    if (G <= 16 && (long)c.T * c.H * pieces_of(c, a.heads, sp.top).pieces <= 128) return launch_form<dt.value, kept.value, dim.value, 16, 8>(c, a, sp, ws, stream);
    if (G <= 16) return launch_form<dt.value, kept.value, dim.value, 16, 4>(c, a, sp, ws, stream);
    return launch_form<dt.value, kept.value, dim.value, 32, 4>(c, a, sp, ws, stream);
  });
}

}  // namespace covspec
