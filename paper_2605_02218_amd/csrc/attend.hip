// Attention of a batch's rows over a paged cache: prompts, drafted segments and single tokens.
//
// o = sum_j p_j v_j / sum_j p_j, p_j = 2^(y_j - m), y_j = scale log2(e) q . k_j, in one pass over the positions with a running reference m: when m
// grows, what was summed so far is scaled by 2^(m_old - m_new).  (m, sum p, sum p v) of disjoint sets of positions join the same way, so that
// waves, and workgroups, may share a long sequence.
//
// Rows: the group's query heads of one token are rows of the same key head, so a sequence with n tokens and G heads for each key head has n G rows,
// r = token * G + head, which one read of its keys and values serves.  A wave takes 32 rows; a workgroup RW waves with rows of their own,
// which share the tiles of keys and values in LDS, times KW waves that take every KW-th tile.  Few rows (single tokens, segments) are bound by
// the bytes of the cache: all waves on different tiles; many rows are bound by the matrix pipes: waves on different rows.
//
// A tile of KT positions is 2 KT rows of the pool, 16 bytes a lane straight into LDS, the next tile's while this one is computed.  S^T = K Q^T
// leaves row r of the queries in the lanes r and r + 32 (16 positions each of 32), so the softmax statistics of a row are plain
// registers of its lanes, the factors of a rescaling too, and the probabilities already lie as the operand of O^T = V^T P^T wants them:
// the k-th slot of an operand may be any position as long as both operands agree.  V^T comes out of LDS by transposing reads.
#include <type_traits>

#include "host_cache.h"
#include "paged.h"

namespace covspec {

namespace {

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));

constexpr float kLog2E = 1.44269502f, kLn2 = 0.693147182f;
constexpr float kSlack = 8.f;         // the reference may stay 2^8 behind the largest score: p <= 256 is as good in 16 bits

// Forms of a tile in LDS.  A row of the pool takes CH pieces of 16 bytes (a power of two: head dimension 96 leaves a quarter unused); piece c of
// row x lies in slot c ^ turn(x), so that reads of one piece of many rows (K) and of a few pieces of neighbouring rows (V) meet all banks.
template <int DT, int KEPT, int D> struct Form {
  static constexpr int ESZ = KEPT == DT ? 2 : 1;
  static constexpr int PIECES = D * ESZ / 16;
  static constexpr int CH = PIECES <= 4 ? 4 : PIECES <= 8 ? 8 : 16;
  static constexpr int ROWB = CH * 16;                 // bytes of a row in LDS
  static constexpr int RPI = 64 / CH;                  // rows a wave loads at a time
  static __device__ __forceinline__ int turn(int x) {
    if constexpr (CH == 16) return (x & 3) << 2 | (x >> 2 & 3);
    if constexpr (CH == 8) return (x >> 1 & 1) << 2 | (x >> 2 & 3);
    return x >> 2 & 3;
  }
};

template <int DT> struct Operand;
template <> struct Operand<DT_BF16> {
  typedef bf16x8_t vec;
  static __device__ __forceinline__ f32x16_t mfma(vec a, vec b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<DT_F16> {
  typedef f16x8_t vec;
  static __device__ __forceinline__ f32x16_t mfma(vec a, vec b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// Eight codes to a 16-bit type, exactly: integers up to 127 and e4m3's four bits of significand fit both.
template <int DT, int KEPT>
__device__ __forceinline__ u32x4_t widen8(u32x2_t w) {
  u32x4_t r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (KEPT == DT_E4M3 && DT == DT_BF16) {
      r[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[h], 1.f, false));
      r[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[h], 1.f, true));
    } else if constexpr (KEPT == DT_E4M3) {
      r[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[h], 1.f, false));
      r[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[h], 1.f, true));
    } else if constexpr (DT == DT_F16) {
      // 0x64uu is 1024 + u: u = code + 128 in the low byte, less 1152
      const uint32_t u = w[h] ^ 0x80808080u;
      const f16x2_t less = {(_Float16)1152.f, (_Float16)1152.f};
      r[2 * h] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - less);
      r[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - less);
    } else {
      const f32x4_t f = decode4<DT_I8>(w[h]);
      r[2 * h] = Half<DT_BF16>::pack(f[0], f[1]);
      r[2 * h + 1] = Half<DT_BF16>::pack(f[2], f[3]);
    }
  }
  return r;
}

// max over the two lanes of a row (lane, lane ^ 32)
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Pool to LDS, 16 or 4 bytes a lane: to `lds` + lane * 16 (4).  Written out because the compiler, where it knows of such a load, waits for all
// of them in front of the first transposing read; here the waits are the kernel's own (wait_loads).  No register is loaded.  s_nop: five cycles
// between a vector instruction that wrote the address' scalar registers and this, one behind m0, which nothing else here uses.
__device__ __forceinline__ void load16_lds(unsigned lds, const void* base, unsigned off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load4_lds(unsigned lds, const void* from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(from) : "memory");
}
// Waits that no access to memory is moved across.
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }

// How the positions are split over workgroups: chunks of `clen` positions, a multiple of 128.
struct Split { int chunks, clen; };

// Row t of the batch and its range of positions, for whoever needs it row by row: [lo, hi) holds all it can see.
struct Range { int lo, hi; };
__device__ __forceinline__ Range seen_range(const Paged& c, const Attend& a, int old, int n, int i0, int i1) {
  const long cap = min((long)a.max_len, (long)c.max_pages << c.page_shift);
  long hi = a.visible ? (long)old + min(n, 64) : (long)old + i1 + 1, lo = a.visible || a.window == 0 ? 0 : (long)old + i0 + 1 - a.window;
  return Range{(int)max(lo, 0l), (int)max(min(hi, cap), 0l)};
}
__device__ __forceinline__ int tokens_before(int length, int n) { return (int)max((long)length - n, -(1l << 30)); }

template <int DT, int KEPT, int D, int RW, int KW, int KT>
__global__ __launch_bounds__(64 * RW * KW, RW * KW == 4 && RW == 1 ? 1 : 2) void attend_kernel(Paged c, Attend a, Split sp, int tiles, float* __restrict__ part, f32x2_t* __restrict__ stat) {
  typedef Form<DT, KEPT, D> F;
  constexpr bool CODES = KEPT != DT;
  constexpr int VDT = CODES ? DT_BF16 : DT;              // type of the products with v
  constexpr bool SPLIT_P = CODES && DT == DT_F16;        // p v_scale in two bf16 parts: fp16 has not the range for it, one bf16 not the bits
  constexpr int TR = 32 * RW, DT32 = D / 32, KS = D / 16, ST = KT / 32;
  constexpr int TILE = KT * F::ROWB, STAGE = 2 * TILE + (CODES ? 8 * KT : 0), GROUP = 2 * STAGE;
  constexpr int LOADS = KT / F::RPI / RW;                // of a wave, for one of K and V
  static_assert(LOADS >= 1 && 2 * LOADS + 1 < 63, "");
  typedef typename Operand<DT>::vec vec;
  typedef typename Operand<VDT>::vec vvec;
  extern __shared__ __align__(1024) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW, half = lane >> 5;
  const int G = a.heads / c.H;

  // ---- which rows: key heads next to each other (an XCD each, for eight of them, so that row tiles of one head meet in its L2), then chunks, then
  // row tiles from the last to the first, which see most
  const int g = blockIdx.x % c.H, chunk = blockIdx.x / c.H % sp.chunks;
  int tile = tiles - 1 - (int)(blockIdx.x / c.H / sp.chunks), s = -1, row0 = 0, n = 0;
  for (int s0 = 0; s0 < c.S && s < 0; s0 += 64) {
    const int mine = s0 + lane;
    const int b = mine < c.S ? min(max(c.start[mine], 0), c.T) : c.T, e = mine < c.S ? max(min(c.start[mine + 1], c.T), b) : c.T;
    const int own = mine < c.S ? (int)(((long)(e - b) * G + TR - 1) / TR) : 0;
    int upto = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int w = __shfl_up(upto, o, 64);
      if (lane >= o) upto += w;
    }
    const unsigned long long over = __ballot(upto > tile);
    if (over) {
      const int l = __ffsll((long long)over) - 1;
      s = __builtin_amdgcn_readfirstlane(s0 + l);
      row0 = __builtin_amdgcn_readlane(b, l);
      n = __builtin_amdgcn_readlane(e, l) - row0;
      tile -= __builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(own, l);
    } else {
      tile -= __builtin_amdgcn_readlane(upto, 63);
    }
  }
  if (s < 0) return;
  tile = __builtin_amdgcn_readfirstlane(tile);
  const int old = __builtin_amdgcn_readfirstlane(tokens_before(c.length[s], n));
  const int rows = n * G, r0 = tile * TR;                             // T heads < 2^30
  const int i0 = r0 / G, i1 = (min(r0 + TR, rows) - 1) / G;
  const Range range = seen_range(c, a, old, n, i0, i1);
  const int lo = __builtin_amdgcn_readfirstlane(max(range.lo, chunk * sp.clen) & ~15), hi = __builtin_amdgcn_readfirstlane(min(range.hi, (chunk + 1) * sp.clen));
  if (lo >= hi && sp.chunks > 1) return;
  const int count = lo < hi ? (hi - lo + KT - 1) / KT : 0;            // tiles; this wave's are kw, kw + KW, ...

  // ---- the lane's row and what it sees: positions [klo, khi), and bits of the chunk.  Rows beyond the last count as seeing all, of a query of zeros.
  const int r = r0 + 32 * rw + (lane & 31);
  const bool has = r < rows;
  const int token = has ? r / G : 0, head = g * G + (has ? r - token * G : 0), t_row = row0 + token;
  int klo = 0, khi = 0x7FFFFFFF;
  unsigned long long bits = 0;
  if (has) {
    if (a.visible) { khi = old; bits = (unsigned long long)a.visible[t_row]; }
    else { khi = old + token + 1; klo = a.window ? khi - a.window : 0; }
  }
  const int khi_min = __builtin_amdgcn_readfirstlane(wave_min(khi)), klo_max = __builtin_amdgcn_readfirstlane(wave_max(klo));
  const int khi_max = a.visible ? 0x7FFFFFFF : __builtin_amdgcn_readfirstlane(wave_max(has ? khi : 0));
  const int klo_min = __builtin_amdgcn_readfirstlane(wave_min(has ? klo : 0x7FFFFFFF));

  // p = 2^((z - m) c2): z the product q . k, in 8 bits times the scales of the key and of the softmax.  c2 is above zero, so that -infinity stays
  // what it is.  `unit` brings m back to the scores' own units.
  const float unit = CODES ? 1.f : fmaxf(fabsf(a.scale), 1.2e-38f), c2 = unit * kLog2E, kscale = fabsf(a.scale);
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;             // a negative scale negates the query
  vec q[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    u32x4_t w = {};
    if (has) w = *(const u32x4_t*)((const uint16_t*)a.q + t_row * a.q_pitch + (long)head * D + 16 * k + 8 * half) ^ flip;
    q[k] = __builtin_bit_cast(vec, w);
  }

  // ---- tiles into LDS
  const unsigned base = (unsigned)(uintptr_t)(lds_char*)smem + kw * GROUP;
  const __attribute__((address_space(4))) int32_t* const table = (const __attribute__((address_space(4))) int32_t*)(c.pages + (long)s * c.max_pages);
  const int page_mask = (1 << c.page_shift) - 1;
  struct Pages { int id[KT / 16]; };
  auto look_up = [&](int t) {                                          // page of every 16 positions of tile t
    Pages p;
#pragma unroll
    for (int u = 0; u < KT / 16; ++u) p.id[u] = table[min(lo + t * KT + 16 * u, hi - 1) >> c.page_shift];
    return p;
  };
  // bit u: positions 16 u .. of the tile are on a page that exists
  auto exist = [&](const Pages& p) {
    unsigned ok = 0;
#pragma unroll
    for (int u = 0; u < KT / 16; ++u) ok |= (unsigned)(p.id[u] >= 0 && p.id[u] < c.n_pages) << u;
    return ok;
  };
  auto fetch = [&](int t, const Pages& p, int stage) {
    const unsigned to = base + stage * STAGE;
    const int j0 = lo + t * KT;
    long at[KT / 16];                                                  // where 16 positions' rows begin, in tokens
    int last[KT / 16];
#pragma unroll
    for (int u = 0; u < KT / 16; ++u) {
      const int id = p.id[u] >= 0 && p.id[u] < c.n_pages ? p.id[u] : 0, j = min(j0 + 16 * u, (hi - 1) & ~15);
      at[u] = (((long)id * c.H + g) << c.page_shift) + (j & page_mask);
      last[u] = min(hi - 1 - j, 15);                                   // rows behind the last position are copies of its row
    }
    if constexpr (CODES) {
      // scales of K, then of V, a float each; every wave a part of them
      constexpr int PART = 2 * KT / RW;
      if (lane < PART) {
        const int x = rw * PART + lane, y = x % KT, u = y / 16;
        long place = at[0];
        int l = last[0];
#pragma unroll
        for (int w = 1; w < KT / 16; ++w) { place = u == w ? at[w] : place; l = u == w ? last[w] : l; }
        const float* from = (x < KT ? a.ks : a.vs) + place + min(y & 15, l);
        load4_lds(to + 2 * TILE + rw * PART * 4, from);
      }
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int x0 = (rw * LOADS + i) * F::RPI;                        // rows x0 .. x0 + RPI - 1 of the tile: within 16
      const int u = x0 / 16;
      long where = at[0];
      int l = last[0];
      if constexpr (RW == 1) { where = at[u]; l = last[u]; }
      else {
#pragma unroll
        for (int w = 1; w < KT / 16; ++w) { where = u == w ? at[w] : where; l = u == w ? last[w] : l; }
      }
      const int x = (x0 & 15) + lane / F::CH, piece = (lane % F::CH) ^ F::turn(x);
      if (F::PIECES == F::CH || piece < F::PIECES) {
        const unsigned off = (unsigned)min(x, l) * (D * F::ESZ) + piece * 16;
        load16_lds(to + x0 * F::ROWB, (const char*)a.kc + where * (D * F::ESZ), off);
        load16_lds(to + TILE + x0 * F::ROWB, (const char*)a.vc + where * (D * F::ESZ), off);
      }
    }
  };

  f32x16_t o[DT32];
#pragma unroll
  for (int d = 0; d < DT32; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float m = -INFINITY, ref = 0.f, sum = 0.f;             // ref = m c2, or zero
  bool far = false;                                      // m c2 is beyond the range of fp32 in some lane

  // K: row 4 h + 8 b + ... of an S^T tile is position 16 t + 8 h + 4 b + i, so that a lane's values 8 t .. 8 t + 7 are eight positions in a row
  const int krow = (lane & 3) | (lane & 8) >> 1 | (lane & 4) << 1 | (lane & 16);
  const int kbase = krow * F::ROWB + (CODES ? F::turn(krow) * 16 + 8 * half : (half ^ F::turn(krow)) * 16);
  // V: a group of 16 lanes reads 4 (8, codes) positions x 16 columns, which come out as a column for each lane
  const int vgrp = lane >> 4, vj = lane & 15;
  int vbase[CODES ? 1 : 2];
  if constexpr (CODES) {
    const int x = 8 * (vgrp >> 1) + vj / 2;
    vbase[0] = x * F::ROWB + ((vgrp & 1) ^ F::turn(x)) * 16 + 8 * (vj & 1);
  } else {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int x = 8 * (vgrp >> 1) + 4 * b + vj / 4;
      vbase[b] = x * F::ROWB + ((2 * (vgrp & 1) + (vj >> 1 & 1)) ^ F::turn(x)) * 16 + 8 * (vj & 1);
    }
  }

  auto compute = [&](int t, unsigned ok, int stage) {
    const lds_char* const kt = (const lds_char*)(base + stage * STAGE);
    const lds_char* const vt = kt + TILE;
    const int j0 = lo + t * KT;
    if (j0 >= khi_max || j0 + KT <= klo_min) return;                   // no row of this wave sees any of it
    // all pieces of K on their way before the first product
    typedef std::conditional_t<CODES, u32x2_t, u32x4_t> raw_t;
    raw_t kf[ST][KS];
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int k = 0; k < KS; ++k) kf[st][k] = *(const __attribute__((address_space(3))) raw_t*)(kt + st * 32 * F::ROWB + (kbase ^ k * (CODES ? 16 : 32)));
    __builtin_amdgcn_sched_barrier(0);
    f32x16_t z[ST];
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int e = 0; e < 16; ++e) z[st][e] = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int st = 0; st < ST; ++st) {
        u32x4_t w;
        if constexpr (CODES) w = widen8<DT, KEPT>(kf[st][k]); else w = kf[st][k];
        z[st] = Operand<DT>::mfma(__builtin_bit_cast(vec, w), q[k], z[st]);
      }
    // V of step x: 16 positions
    raw_t vf[2][DT32];
    auto load_v = [&](int x) {
#pragma unroll
      for (int d = 0; d < DT32; ++d) {
        if constexpr (CODES) {
          typedef __attribute__((address_space(3))) i32x2_t L;
          vf[x & 1][d] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((L*)(vt + x * 16 * F::ROWB + (vbase[0] ^ d * 32))));
        } else {
          typedef __attribute__((address_space(3))) s16x4_t L;
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const u32x2_t raw = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(vt + x * 16 * F::ROWB + (vbase[b] ^ d * 64))));
            vf[x & 1][d][2 * b] = raw[0];
            vf[x & 1][d][2 * b + 1] = raw[1];
          }
        }
      }
    };
    const __attribute__((address_space(3))) float* const scales = (const __attribute__((address_space(3))) float*)(vt + TILE);
    if constexpr (CODES) {
#pragma unroll
      for (int st = 0; st < ST; ++st)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const f32x4_t w = *(const __attribute__((address_space(3))) f32x4_t*)(scales + 32 * st + 16 * (f / 2) + 8 * half + 4 * (f & 1));
#pragma unroll
          for (int e = 0; e < 4; ++e) z[st][4 * f + e] *= w[e] * kscale;
        }
    }
    const bool partial = j0 + KT > min(khi_min, hi) || j0 < klo_max || ok != (1u << KT / 16) - 1;
    if (partial) {
      // bit x: the lane's row sees position j0 + x
      auto below = [](int x) { return x <= 0 ? 0ull : x >= 64 ? ~0ull : (1ull << x) - 1; };
      unsigned long long see = below(khi - j0) & ~below(klo - j0);
      if (a.visible && j0 + KT > old) {
        const int by = old - j0;                                       // of the chunk's first position
        see |= by >= 64 || by <= -64 ? 0ull : by >= 0 ? bits << by : bits >> -by;
      }
      see &= below(hi - j0);
      unsigned long long there = 0;
#pragma unroll
      for (int u = 0; u < KT / 16; ++u) there |= (ok >> u & 1 ? 0xFFFFull : 0ull) << (16 * u);
      see = (see & there) >> (8 * half);
#pragma unroll
      for (int st = 0; st < ST; ++st) {
        const uint32_t w = (uint32_t)(see >> (32 * st));
#pragma unroll
        for (int e = 0; e < 16; ++e) z[st][e] = w & (1u << (16 * (e / 8) + e % 8)) ? z[st][e] : -INFINITY;
      }
    }
    float top = z[0][0];
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, z[st][e]);
    top = pair_max(top);
    const bool grow = (top - m) * c2 > kSlack;                         // m = -infinity: whenever something is seen
    if (__any(grow)) {
      const float next = grow ? top : m;
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - next) * c2);
      sum *= keep;
#pragma unroll
      for (int d = 0; d < DT32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= keep;
      m = next;
      ref = m == -INFINITY ? 0.f : m * c2;
      far = __any(fabsf(ref) > 1e38f);
    }
    load_v(0);
    float part_sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (__builtin_expect(far, 0)) {
#pragma unroll
      for (int st = 0; st < ST; ++st)
#pragma unroll
        for (int e = 0; e < 16; ++e) z[st][e] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((z[st][e] - m) * c2);
    } else {
#pragma unroll
      for (int st = 0; st < ST; ++st)
#pragma unroll
        for (int e = 0; e < 16; ++e) z[st][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[st][e], c2, -ref));
    }
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int e = 0; e < 16; ++e) part_sum[e & 3] += z[st][e];
    sum += (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
    if constexpr (CODES) {
#pragma unroll
      for (int st = 0; st < ST; ++st)
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          const f32x4_t w = *(const __attribute__((address_space(3))) f32x4_t*)(scales + KT + 32 * st + 16 * (f / 2) + 8 * half + 4 * (f & 1));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = z[st][4 * f + e], y = p * w[e];
            z[st][4 * f + e] = partial && p == 0.f ? 0.f : y;          // the scale of an unseen row may be anything
          }
        }
    }
#pragma unroll
    for (int x = 0; x < KT / 16; ++x) {
      u32x4_t p, rest;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a0 = z[x / 2][8 * (x & 1) + 2 * e], a1 = z[x / 2][8 * (x & 1) + 2 * e + 1];
        p[e] = Half<VDT>::pack(a0, a1);
        if constexpr (SPLIT_P) rest[e] = Half<VDT>::pack(a0 - bf16lo_to_f32(p[e]), a1 - bf16hi_to_f32(p[e]));
      }
      if (x + 1 < KT / 16) load_v(x + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < DT32; ++d) {
        u32x4_t w;
        if constexpr (CODES) w = widen8<VDT, KEPT>(vf[x & 1][d]); else w = vf[x & 1][d];
        o[d] = Operand<VDT>::mfma(__builtin_bit_cast(vvec, w), __builtin_bit_cast(vvec, p), o[d]);
        if constexpr (SPLIT_P) o[d] = Operand<VDT>::mfma(__builtin_bit_cast(vvec, w), __builtin_bit_cast(vvec, rest), o[d]);
      }
    }
  };

  if (count > 0) {
    // tile t of the group's: fetched while the one before is computed.  All waves of a workgroup meet as often as the group with most tiles needs.
    const int mine = kw < count ? (count - kw + KW - 1) / KW : 0, most = (count + KW - 1) / KW;
    Pages now, next;
    if (mine > 0) { now = look_up(kw); fetch(kw, now, 0); }
    if (mine > 1) next = look_up(kw + KW);
    for (int t = 0; t < most; ++t) {
      const bool work = t < mine, more = t + 1 < mine;
      unsigned ok = 0;
      if (work) ok = exist(now);
      if (more) {
        fetch(kw + (t + 1) * KW, next, (t + 1) & 1);
        now = next;
        if (t + 2 < mine) next = look_up(kw + (t + 2) * KW);
        wait_loads<2 * LOADS + (CODES ? 1 : 0)>();
      } else {
        wait_loads<0>();
      }
      if constexpr (RW > 1) meet();                                    // the others' parts of the tile are there as well
      __builtin_amdgcn_sched_barrier(0);
      if (work) compute(kw + t * KW, ok, t & 1);
      __builtin_amdgcn_sched_barrier(0);
      wait_lds();                                                      // nothing reads the stage that is filled next
      if constexpr (RW > 1) meet();
    }
  }

  // ---- NaN: 0 * v of a position that some row of the tile does not see may have made it, if that v is not finite.  The rows are summed again,
  // term by term with the products left out.
  bool nan = false;
#pragma unroll
  for (int d = 0; d < DT32; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) nan |= o[d][e] != o[d][e];
  if (__any(nan)) {
#pragma unroll
    for (int d = 0; d < DT32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    for (int t = kw; t < count; t += KW)
      for (int j = lo + t * KT; j < min(lo + t * KT + KT, hi); ++j) {
        const long x = place_of(c, s, j, g);
        bool see = has && x >= 0 && j >= klo && j < khi;
        if (a.visible && j >= old) see = has && x >= 0 && j - old < 64 && (bits >> (j - old) & 1);
        if (!__any(see)) continue;
        float y = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const u32x4_t w = __builtin_bit_cast(u32x4_t, q[k]);
          u32x4_t kk;
          if constexpr (CODES) kk = widen8<DT, KEPT>(*(const u32x2_t*)((const char*)a.kc + x * D + 16 * k + 8 * half));
          else kk = *(const u32x4_t*)((const char*)a.kc + (x * D + 16 * k + 8 * half) * 2);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x2_t u = Half<DT>::unpack(w[e]), v = Half<DT>::unpack(kk[e]);
            y += u[0] * v[0] + u[1] * v[1];
          }
        }
        y = pair_sum(y);
        if constexpr (CODES) y *= a.ks[x] * kscale;
        float p = __builtin_amdgcn_exp2f((y - m) * c2);
        if constexpr (CODES) p *= a.vs[x];
#pragma unroll
        for (int d = 0; d < DT32; ++d)
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const long from = x * D + 32 * d + 8 * b + 4 * half;
            float v[4];
            if constexpr (CODES) {
              const f32x4_t f = decode4<KEPT>(*(const uint32_t*)((const char*)a.vc + from));
              v[0] = f[0]; v[1] = f[1]; v[2] = f[2]; v[3] = f[3];
            } else {
              const u32x2_t w = *(const u32x2_t*)((const char*)a.vc + from * 2);
              const f32x2_t f0 = Half<DT>::unpack(w[0]), f1 = Half<DT>::unpack(w[1]);
              v[0] = f0[0]; v[1] = f0[1]; v[2] = f1[0]; v[3] = f1[1];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[d][4 * b + e] = see ? __builtin_fmaf(p, v[e], o[d][4 * b + e]) : o[d][4 * b + e];
          }
      }
  }
  sum = pair_sum(sum);
  m *= unit;                                             // in units of the scores

  // ---- the waves that shared the rows
  if constexpr (KW > 1) {
    constexpr int SLOT = D * 32 * 4 + 512;                             // sums, then references and sums of p of a wave's lanes
    __syncthreads();
    if (kw > 0) {
      char* const to = smem + ((kw - 1) * RW + rw) * SLOT;
#pragma unroll
      for (int d = 0; d < DT32; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) *(f32x4_t*)(to + (d * 4 + b) * 1024 + lane * 16) = (f32x4_t){o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
      *(float*)(to + D * 128 + lane * 4) = m;
      *(float*)(to + D * 128 + 256 + lane * 4) = sum;
    }
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int w = 0; w < KW - 1; ++w) {
      const char* const from = smem + (w * RW + rw) * SLOT;
      const float m2 = *(const float*)(from + D * 128 + lane * 4), s2 = *(const float*)(from + D * 128 + 256 + lane * 4);
      const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
      const float f1 = __builtin_amdgcn_exp2f((m - ref) * kLog2E), f2 = __builtin_amdgcn_exp2f((m2 - ref) * kLog2E);
      sum = sum * f1 + s2 * f2;
#pragma unroll
      for (int d = 0; d < DT32; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const f32x4_t v = *(const f32x4_t*)(from + (d * 4 + b) * 1024 + lane * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][4 * b + e] = o[d][4 * b + e] * f1 + v[e] * f2;
        }
      m = top;
    }
  }
  if (!has) return;
  if (sp.chunks > 1) {
    const long row = ((long)chunk * c.T + t_row) * a.heads + head;
#pragma unroll
    for (int d = 0; d < DT32; ++d)
#pragma unroll
      for (int b = 0; b < 4; ++b) *(f32x4_t*)(part + row * D + 32 * d + 8 * b + 4 * half) = (f32x4_t){o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
    if (half == 0) stat[row] = (f32x2_t){m, sum};
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* const out = (uint16_t*)a.out + t_row * a.out_pitch + (long)head * D;
#pragma unroll
  for (int d = 0; d < DT32; ++d)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      *(u32x2_t*)(out + 32 * d + 8 * b + 4 * half) = (u32x2_t){Half<DT>::pack(o[d][4 * b] * inv, o[d][4 * b + 1] * inv), Half<DT>::pack(o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv)};
  if (a.lse && half == 0) a.lse[(long)t_row * a.heads + head] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
}

// Joins the chunks of a row, a wave per row and head; the chunks that touch what the row can see are the ones that were written for it.
template <int DT, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(Paged c, Attend a, Split sp, const float* __restrict__ part, const f32x2_t* __restrict__ stat) {
  const int lane = threadIdx.x & 63;
  const long x = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (x >= (long)c.T * a.heads) return;
  const int t = (int)(x / a.heads), head = (int)(x % a.heads);
  const int s = seq_of(c.start, c.S, t);
  if (s < 0 || s >= c.S) return;
  const int n = c.start[s + 1] - c.start[s], i = t - c.start[s];
  const Range range = seen_range(c, a, tokens_before(c.length[s], n), n, i, i);
  const int first = range.lo / sp.clen, last = range.lo < range.hi ? (range.hi - 1) / sp.clen : first - 1;
  float m = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
  for (int k = first; k <= last; ++k) {
    const long row = ((long)k * c.T + t) * a.heads + head;
    const f32x2_t w = stat[row];
    const float p0 = lane * 2 < D ? part[row * D + lane * 2] : 0.f, p1 = lane * 2 < D ? part[row * D + lane * 2 + 1] : 0.f;
    const float top = fmaxf(m, w[0]), ref = top == -INFINITY ? 0.f : top;
    const float f1 = __builtin_amdgcn_exp2f((m - ref) * kLog2E), f2 = __builtin_amdgcn_exp2f((w[0] - ref) * kLog2E);
    sum = sum * f1 + w[1] * f2;
    o0 = o0 * f1 + p0 * f2;
    o1 = o1 * f1 + p1 * f2;
    m = top;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (lane * 2 < D) *(uint32_t*)((uint16_t*)a.out + t * a.out_pitch + (long)head * D + lane * 2) = Half<DT>::pack(o0 * inv, o1 * inv);
  if (a.lse && lane == 0) a.lse[x] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
}

// ---- the rule for the form of the workgroups and the split
struct Plan { int rw, tiles; Split sp; };

Plan plan_of(const Paged& c, int heads, int max_len) {
  const long G = heads / c.H, rows = (long)c.T * G, mean = (rows + c.S - 1) / c.S;
  Plan p;
  p.rw = mean <= 32 ? 1 : mean <= 64 ? 2 : 4;
  const int TR = 32 * p.rw;
  p.tiles = (int)(rows / TR + c.S);
  const long groups = (long)p.tiles * c.H;
  const long want = p.rw == 4 ? 512 : 2048, least = p.rw == 4 ? 1024 : 512;
  long chunks = (want + groups - 1) / groups;
  const long most = (max_len + least - 1) / least;
  chunks = chunks < most ? chunks : most;
  const long clen = ((max_len + chunks - 1) / chunks + 127) / 128 * 128;
  p.sp.clen = (int)clen;
  p.sp.chunks = (int)((max_len + clen - 1) / clen);
  return p;
}

size_t part_bytes(const Paged& c, int heads, const Split& sp) { return ((size_t)sp.chunks * c.T * heads * c.D * sizeof(float) + 255) / 256 * 256; }

template <int DT, int KEPT, int D, int RW, int KW, int KT>
hipError_t launch_form(const Paged& c, const Attend& a, const Plan& p, void* ws, hipStream_t stream) {
  typedef Form<DT, KEPT, D> F;
  constexpr size_t stage = 2 * KT * F::ROWB + (KEPT != DT ? 8 * KT : 0), slots = (size_t)(KW - 1) * RW * (D * 128 + 512);
  constexpr size_t lds = 2 * KW * stage > slots ? 2 * KW * stage : slots;
  static PerDeviceInt raised;
  hipError_t e = ensure_dynamic_lds(raised, (const void*)attend_kernel<DT, KEPT, D, RW, KW, KT>, lds);
  if (e != hipSuccess) return e;
  float* part = (float*)ws;
  f32x2_t* stat = (f32x2_t*)((char*)ws + part_bytes(c, a.heads, p.sp));
  const unsigned grid = (unsigned)p.tiles * c.H * p.sp.chunks;
  hipLaunchKernelGGL((attend_kernel<DT, KEPT, D, RW, KW, KT>), dim3(grid), dim3(64 * RW * KW), lds, stream, c, a, p.sp, p.tiles, part, stat);
  if ((e = hipGetLastError()) != hipSuccess || p.sp.chunks == 1) return e;
  const unsigned joins = (unsigned)(((long)c.T * a.heads + 3) / 4);
  hipLaunchKernelGGL((attend_join_kernel<DT, D>), dim3(joins), dim3(256), 0, stream, c, a, p.sp, (const float*)part, (const f32x2_t*)stat);
  return hipGetLastError();
}

template <int DT, int KEPT, int D>
hipError_t launch_attend_d(const Paged& c, const Attend& a, void* ws, hipStream_t stream) {
  const Plan p = plan_of(c, a.heads, a.max_len);
  if (p.rw == 1) return launch_form<DT, KEPT, D, 1, 4, 32>(c, a, p, ws, stream);
  if (p.rw == 2) return launch_form<DT, KEPT, D, 2, 2, 32>(c, a, p, ws, stream);
  return launch_form<DT, KEPT, D, 4, 1, 64>(c, a, p, ws, stream);
}

template <int DT, int KEPT>
hipError_t launch_attend_k(const Paged& c, const Attend& a, void* ws, hipStream_t stream) {
  if (c.D == 64) return launch_attend_d<DT, KEPT, 64>(c, a, ws, stream);
  if (c.D == 96) return launch_attend_d<DT, KEPT, 96>(c, a, ws, stream);
  if (c.D == 128) return launch_attend_d<DT, KEPT, 128>(c, a, ws, stream);
  return hipErrorInvalidValue;
}

template <int DT>
hipError_t launch_attend_t(const Paged& c, const Attend& a, void* ws, hipStream_t stream) {
  if (c.kept == DT) return launch_attend_k<DT, DT>(c, a, ws, stream);
  if (c.kept == DT_I8) return launch_attend_k<DT, DT_I8>(c, a, ws, stream);
  if (c.kept == DT_E4M3) return launch_attend_k<DT, DT_E4M3>(c, a, ws, stream);
  return hipErrorInvalidValue;
}

}  // namespace

size_t attend_workspace_bytes(const Paged& c, int heads, int max_len) {
  const Plan p = plan_of(c, heads, max_len);
  if (p.sp.chunks == 1) return 256;
  return part_bytes(c, heads, p.sp) + (size_t)p.sp.chunks * c.T * heads * sizeof(f32x2_t);
}

hipError_t launch_attend(const Paged& c, const Attend& a, void* ws, hipStream_t stream) {
  if (c.dtype == DT_BF16) return launch_attend_t<DT_BF16>(c, a, ws, stream);
  if (c.dtype == DT_F16) return launch_attend_t<DT_F16>(c, a, ws, stream);
  return hipErrorInvalidValue;
}

}  // namespace covspec
