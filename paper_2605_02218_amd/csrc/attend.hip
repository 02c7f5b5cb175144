// Attention of a batch's rows over a paged cache: prompts, drafted segments and single tokens.
//
// o = sum_j p_j v_j / sum_j p_j, p_j = 2^(y_j - m), y_j = scale log2(e) q . k_j, in one pass over the positions with a running reference m: when m
// grows, what was summed so far is scaled by 2^(m_old - m_new).  (m, sum p, sum p v) of disjoint sets of positions join the same way, so that
// waves, and workgroups, may share a long sequence.
//
// Rows: the group's query heads of one token are rows of the same key head, so a sequence with n tokens and G heads for each key head has n G rows,
// r = token * G + head, which one read of its keys and values serves.  A wave takes 16 or 32 rows (M); a workgroup RW waves with rows of
// their own, which share the tiles of keys and values in LDS, times KW waves that take every KW-th tile.  Few rows (single tokens, segments) are bound by
// the bytes of the cache: all waves on different tiles; many rows are bound by the matrix pipes: waves on different rows.
//
// A tile of KT positions is 2 KT rows of the pool, 16 bytes a lane straight into LDS, the next tile's while this one is computed.  S^T = K Q^T
// leaves row r of the queries in the lanes r and r + 32 (16 positions each of 32; with M = 16 in four lanes, r + 16 i), so the softmax statistics of a row are plain
// registers of its lanes, the factors of a rescaling too, and the probabilities already lie as the operand of O^T = V^T P^T wants them:
// the k-th slot of an operand may be any position as long as both operands agree.  V^T comes out of LDS by transposing reads.
#include <type_traits>

#include "host_cache.h"
#include "tiles.h"

namespace covspec {

namespace {

// What rows i0 .. i1 of a sequence see lies in [lo, hi).
struct Range { int lo, hi; };
__device__ __forceinline__ Range seen_range(const Paged& c, const Attend& a, int old, int n, int i0, int i1) {
  const long cap = min((long)a.max_len, (long)c.max_pages << c.page_shift);
  long hi = a.visible ? (long)old + min(n, 64) : (long)old + i1 + 1, lo = a.visible || a.window == 0 ? 0 : (long)old + i0 + 1 - a.window;
  return Range{(int)max(lo, 0l), (int)max(min(hi, cap), 0l)};
}
__device__ __forceinline__ int tokens_before(int length, int n) { return (int)max((long)length - n, -(1l << 30)); }

// The work: an item is a tile of `rows` rows of a sequence and a key head, a unit `unit` of its positions.  Items lie one behind the other, by sequence,
// head and tile, all of a sequence counted with the units of its longest.
//   shares > 0: that many workgroups at most take equal pieces of the sequence of units, so that long and short sequences together keep all of them
//     busy to the end; an item that a piece does not hold whole goes to `part`, and attend_join_kernel adds its pieces up.
//   shares == 0: a workgroup per item, and no join: many items even out by themselves.
struct Split { int rows, unit, shares, least, tiles, joins; };

// The sequences, 64 at a time, a lane each: rows, length, tiles, units of an item, units in all and up to here.
struct Block { int row0, n, len, tiles, units, own, upto, items_upto; };
template <bool ITEMS>                                 // ITEMS: a unit is a tile, of one head
__device__ __forceinline__ Block block_of(const Paged& c, const Attend& a, const Split& sp, int s0) {
  const int mine = s0 + (threadIdx.x & 63), safe = min(mine, c.S - 1), G = a.heads / c.H;
  Block v;
  v.row0 = min(max(c.start[safe], 0), c.T);
  v.n = max(min(c.start[safe + 1], c.T), v.row0) - v.row0;
  v.len = c.length[safe];
  v.tiles = mine < c.S ? (int)(((long)v.n * G + sp.rows - 1) / sp.rows) : 0;
  v.units = 1;
  if constexpr (!ITEMS) {
    long most = seen_range(c, a, tokens_before(v.len, v.n), v.n, 0, v.n - 1).hi;
    if (a.window > 0) most = min(most, (long)a.window + sp.rows / G + 17);       // first and last row of a tile, rounding to 16
    v.units = max(1, (int)((most + sp.unit - 1) / sp.unit));
  }
  v.own = ITEMS ? v.tiles : v.tiles * v.units * c.H;
  v.upto = wave_inscan(v.own);
  v.items_upto = ITEMS ? 0 : wave_inscan(v.tiles * c.H);
  return v;
}
// at: where the unit asked for lies among the sequence's own; items: items in front of the sequence; s < 0: nowhere
struct Place { int s, row0, n, len, tiles, units, at, items; };
// Unit x of the block, which begins at sequence s0, behind `items` items of heads H.
__device__ __forceinline__ Place place_in(const Block& v, int s0, int x, int items, int H) {
  Place p;
  p.s = -1;
  const unsigned long long over = __ballot(v.upto > x);
  if (over) {
    const int at = __ffsll((long long)over) - 1, own = __builtin_amdgcn_readlane(v.own, at);
    p.s = s0 + at;
    p.row0 = __builtin_amdgcn_readlane(v.row0, at);
    p.n = __builtin_amdgcn_readlane(v.n, at);
    p.len = __builtin_amdgcn_readlane(v.len, at);
    p.tiles = __builtin_amdgcn_readlane(v.tiles, at);
    p.units = __builtin_amdgcn_readlane(v.units, at);
    p.items = items + __builtin_amdgcn_readlane(v.items_upto, at) - p.tiles * H;
    p.at = x - __builtin_amdgcn_readlane(v.upto, at) + own;
    if (p.at < 0 || p.at >= own) p.s = -1;                     // `start` does not ascend
  }
  return p;
}
__device__ __forceinline__ int block_total(const Block& v) { return __builtin_amdgcn_readlane(v.upto, 63); }
template <bool ITEMS>
__device__ __forceinline__ Place find(const Paged& c, const Attend& a, const Split& sp, int x) {
  Place p;
  p.s = -1;
  int items = 0;
  for (int s0 = 0; s0 < c.S && p.s < 0; s0 += 64) {
    const Block v = block_of<ITEMS>(c, a, sp, s0);
    p = place_in(v, s0, x, items, c.H);
    x -= block_total(v);
    items += __builtin_amdgcn_readlane(v.items_upto, 63);
  }
  return p;
}
// Shares of `total` units: the first `more` have one unit more than the others.
struct Shares {
  int n = 0, each = 0, more = 0;
  __device__ __forceinline__ Shares() {}
  __device__ __forceinline__ Shares(const Split& sp, int total) : n(min(sp.shares, max(1, total / sp.least))), each(total / n), more(total - each * n) {}
  __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
  __device__ __forceinline__ int of(int x) const { return x < more * (each + 1) ? x / (each + 1) : more + (x - more * (each + 1)) / each; }
};
// For the join, by the item's number: its pieces (0: it is in one), the first one's share; first row of the sequence in the batch, first query head, first row
// of the tile among the sequence's, their count.  Written by the share in which the item begins.
struct Joined { int pieces, share, row0, head0, r0, rows; };

template <int DT, int KEPT, int D, int M, int RW, int KW, int KT>
__global__ __launch_bounds__(64 * RW * KW, 2) void attend_kernel(Paged c, Attend a, Split sp, float* __restrict__ part, f32x2_t* __restrict__ stat, Joined* __restrict__ joined, int* __restrict__ joined_count) {
  typedef Form<DT, KEPT, D> F;
  // 8-bit codes: a single wave widens what it multiplies; waves that share tiles widen each tile once, in LDS, between them.  Their scales, in fp32:
  // of K times the scores, of V times p, which bf16 has the range for.  fp16 has not; there p v_scale goes in as two bf16 parts (one has not the bits:
  // with v = code * scale rounded to fp16 instead the error against 64 bits was 1.65 times that of the output's own rounding, a tree
  // of 88 rows behind 120001 tokens took 74 us instead of 83).
  constexpr bool CODES = KEPT != DT, WIDE = CODES && RW > 1;
  constexpr int VDT = CODES ? DT_BF16 : DT;              // type of the products with v
  // In bf16, p (v_scale) goes into its products in two parts as well, 16 bits of significand, wherever that costs 3 % or less: where a wave has tiles of its own,
  // and in 16-bit caches up to 64 rows.  Error against 64 bits with one part 1.45 times the rounding of the output for 64 single tokens over e4m3, 1.37 for 32
  // segments, with two 1.00.  us with one and two: 64 single tokens over e4m3 124 and 126, over bf16 behind 8192 positions each 352 to 358 and 358 to 363, segments of 64
  // rows 392 and 399; but those over e4m3 299 and 344, 88 rows 400 and 468, prompts of 4 x 3008 tokens 750 and 943.  fp16 caches have p's 11 bits.
  constexpr bool SPLIT_P = CODES ? DT == DT_F16 || RW == 1 : DT == DT_BF16 && RW <= 2;
  typedef Form<DT, WIDE ? DT : KEPT, D> W;               // of the tiles that are multiplied
  constexpr bool RAW = CODES && !WIDE;
  constexpr bool TURNS = RW == 8;                        // see the loop over the tiles
  constexpr bool AGAIN = KEPT != DT_I8 && RW > 1, CLEAR = KEPT != DT_I8 && RW == 1;      // v that is not finite: see in front of sums
  static_assert(!TURNS || (KW == 1 && KT == 64 && !CODES), "");
  typedef Operand<DT, M> P1;
  typedef Operand<VDT, M> P2;
  typedef typename P1::vec vec;
  typedef typename P2::vec vvec;
  typedef typename P1::acc acc;
  constexpr int NG = 64 / M, KM = 8 * NG, CA = M * M / 64;               // lanes of a row; terms of a product; values of a result in a lane
  constexpr int TR = M * RW, DM = D / M, KS = D / KM, ST = KT / M, NX = KT / KM;
  constexpr int TILE = KT * F::ROWB, STAGE = 2 * TILE + (CODES ? 8 * KT : 0);
  constexpr int WTILE = KT * W::ROWB, GROUP = (TURNS ? 4 : 2) * STAGE + (WIDE ? 2 * WTILE : 0);
  constexpr int LOADS = KT / F::RPI / RW;                // of a wave, for one of K and V
  static_assert(LOADS >= 1 && 2 * LOADS + 1 < 63 && D % KM == 0 && KT % KM == 0 && KT % 32 == 0 && KT <= 64, "");
  extern __shared__ __align__(1024) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW, grp = lane / M;
  const int G = a.heads / c.H;

  // ---- which work.  Items: key heads next to each other (an XCD each, for eight of them, so that row tiles of one head meet in its L2), row tiles
  // from the last to the first, which see most.  Shares: neighbours on one XCD.
  int x = 0, x_end = 1, share = 0;
  Shares share_of_unit;
  Place p;
  if (sp.shares > 0) {
    const Block first = block_of<false>(c, a, sp, 0);                  // in most calls all sequences
    int total = block_total(first), items = __builtin_amdgcn_readlane(first.items_upto, 63);
    for (int s0 = 64; s0 < c.S; s0 += 64) {
      const Block v = block_of<false>(c, a, sp, s0);
      total += block_total(v);
      items += __builtin_amdgcn_readlane(v.items_upto, 63);
    }
    const Shares shares(sp, total);
    const int each = (shares.n + 7) / 8;
    share = (blockIdx.x % 8) * each + blockIdx.x / 8;
    if (blockIdx.x == 0 && tid == 0) *joined_count = items;
    if ((int)(blockIdx.x / 8) >= each || share >= shares.n) return;
    x = shares.begin(share);
    x_end = shares.begin(share + 1);
    if (x >= x_end) return;
    p = c.S <= 64 ? place_in(first, 0, x, 0, c.H) : find<false>(c, a, sp, x);
    share_of_unit = shares;
  } else {
    p = find<true>(c, a, sp, sp.tiles - 1 - (int)(blockIdx.x / c.H));
  }
  while (true) {
  if (p.s < 0) return;
  const int s = p.s, row0 = p.row0, n = p.n;
  int tile = p.at, g = blockIdx.x % c.H, from = 0, upto = 1;
  bool whole = true;
  if (sp.shares > 0) {
    const int item = p.at / p.units;
    from = p.at - item * p.units;
    upto = min(p.units, from + x_end - x);
    whole = from == 0 && upto == p.units;
    g = item / p.tiles;
    tile = item - g * p.tiles;
    const int number = p.items + item;
    if (tid == 0 && from == 0 && number >= 0 && number < sp.joins) {
      Joined j = {};
      if (!whole) {
        j.pieces = share_of_unit.of(x + p.units - 1) - share + 1;
        j.share = share;
        j.row0 = p.row0;
        j.head0 = g * G;
        j.r0 = tile * TR;
        j.rows = p.n * G;
      }
      joined[number] = j;
    }
    x += upto - from;
  } else {
    x = x_end;
  }
  const int old = tokens_before(p.len, n), rows = n * G, r0 = tile * TR;   // T heads < 2^30
  const int i0 = r0 / G, i1 = (min(r0 + TR, rows) - 1) / G;
  const Range range = seen_range(c, a, old, n, i0, i1);
  const int low = range.lo & ~15;
  const int lo = (int)min((long)low + (long)from * sp.unit, 0x7FFFFFF0l), hi = whole ? range.hi : (int)min((long)range.hi, (long)low + (long)upto * sp.unit);
  const int count = lo < hi ? (hi - lo + KT - 1) / KT : 0;            // tiles; this wave's are kw, kw + KW, ...

  // ---- the lane's row and what it sees: positions [klo, khi), and bits of the chunk.  Rows beyond the last count as seeing all, of a query of zeros.
  const int rfirst = r0 + M * rw, r = rfirst + lane % M;
  const bool has = r < rows;
  const int token = has ? r / G : 0, head = g * G + (has ? r - token * G : 0), t_row = row0 + token;
  int klo = 0, khi = 0x7FFFFFFF;
  unsigned long long bits = 0;
  if (has) {
    if (a.visible) { khi = old; bits = (unsigned long long)a.visible[t_row]; }
    else { khi = old + token + 1; klo = a.window ? khi - a.window : 0; }
  }
  // of the wave's rows, which see more from one to the next: what all see is [klo_max, khi_min), what any [klo_min, khi_max)
  int khi_min = 0, khi_max = 0, klo_min = 0, klo_max = 0;
  if (rfirst < rows) {
    const int tfirst = rfirst / G, tlast = (min(rfirst + M, rows) - 1) / G;
    khi_min = a.visible ? old : old + tfirst + 1;
    khi_max = a.visible ? 0x7FFFFFFF : old + tlast + 1;
    klo_min = a.window ? khi_min - a.window : 0;
    klo_max = a.window ? khi_max - a.window : 0;
  }

  // p = 2^((z - m) c2): z the product q . k, in 8 bits times the scale of the key.  c2 is above zero, so that -infinity stays
  // what it is.  `unit` brings m back to the scores' own units.
  const float unit = fmaxf(fabsf(a.scale), 1.2e-38f), c2 = unit * kLog2E;
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;             // a negative scale negates the query
  vec q[KS];
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    u32x4_t w = {};
    if (has) w = *(const u32x4_t*)((const uint16_t*)a.q + t_row * a.q_pitch + (long)head * D + KM * k + 8 * grp) ^ flip;
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
        where = uniform(where);
        const unsigned off = (unsigned)min(x, l) * (D * F::ESZ) + piece * 16;
        load16_lds(to + x0 * F::ROWB, (const char*)a.kc + where * (D * F::ESZ), off);
        load16_lds(to + TILE + x0 * F::ROWB, (const char*)a.vc + where * (D * F::ESZ), off);
      }
    }
  };

  acc o[DM];
#pragma unroll
  for (int d = 0; d < DM; ++d)
#pragma unroll
    for (int e = 0; e < CA; ++e) o[d][e] = 0.f;
  float m = -INFINITY, ref = 0.f, sum = 0.f;             // ref = m c2, or zero
  bool far = false;                                      // m c2 is beyond the range of fp32 in some lane

  // K: which position is which column of S^T is chosen so that a lane's values 8 x .. 8 x + 7 are the eight positions KM x + 8 group + 0 .. 7
  int kbase[M == 16 ? 2 : 1];
#pragma unroll
  for (int b = 0; b < (M == 16 ? 2 : 1); ++b) {
    const int x = M == 16 ? (lane & 3) | (lane & 12) << 1 | b << 2 : (lane & 3) | (lane & 8) >> 1 | (lane & 4) << 1 | (lane & 16);
    kbase[b] = x * W::ROWB + (RAW ? ((grp >> 1) ^ W::turn(x)) * 16 + 8 * (grp & 1) : (grp ^ W::turn(x)) * 16);
  }
  // V: 16 lanes read 4 (8, codes) positions x 16 columns, which come out as a column for each lane
  const int vcol = M == 16 ? 0 : lane >> 4 & 1, vj = lane & 15;
  int vbase[RAW ? 1 : 2];
  if constexpr (RAW) {
    const int x = 8 * grp + vj / 2;
    vbase[0] = x * W::ROWB + (vcol ^ W::turn(x)) * 16 + 8 * (vj & 1);
  } else {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int x = 8 * grp + 4 * b + vj / 4;
      vbase[b] = x * W::ROWB + ((2 * vcol + (vj >> 1 & 1)) ^ W::turn(x)) * 16 + 8 * (vj & 1);
    }
  }

  // The codes of a stage to 16 bits, by the waves that share them.
  auto widen = [&](int stage) {
    const lds_char* const raw = (const lds_char*)(base + stage * STAGE);
    lds_char* const wide = (lds_char*)(base + 2 * STAGE);
    const int me = rw * 64 + lane;
#pragma unroll
    for (int i = 0; i < KT * F::CH / (64 * RW); ++i) {
      const int y = i * 64 * RW + me, row = y / F::CH, piece = y % F::CH;
      if (F::PIECES == F::CH || piece < F::PIECES) {
        const int from = row * F::ROWB + (piece ^ F::turn(row)) * 16, to = row * W::ROWB + ((2 * piece) ^ W::turn(row)) * 16;
        const u32x4_t kk = *(const __attribute__((address_space(3))) u32x4_t*)(raw + from);
        const u32x4_t vv = *(const __attribute__((address_space(3))) u32x4_t*)(raw + TILE + from);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = h == 0 ? to : to ^ 16;                        // the next piece
          *(__attribute__((address_space(3))) u32x4_t*)(wide + at) = widen8<DT, KEPT>((u32x2_t){kk[2 * h], kk[2 * h + 1]});
          *(__attribute__((address_space(3))) u32x4_t*)(wide + WTILE + at) = widen8<VDT, KEPT>((u32x2_t){vv[2 * h], vv[2 * h + 1]});
        }
      }
    }
  };

  // A tile in three steps: the scores, the probabilities, the sums of v.
  typedef std::conditional_t<RAW, u32x2_t, u32x4_t> raw_t;
  float z[NX][8];                                                      // position KM x + 8 group + e
  u32x4_t prob[NX], rest[SPLIT_P ? NX : 1];
  auto seen = [&](int t) { const int j0 = lo + t * KT; return j0 < khi_max && j0 + KT > klo_min; };       // by any row of this wave
  raw_t kf[ST][KS];
  auto load_k = [&](int stage, int st) {
    const lds_char* const kt = (const lds_char*)(base + (WIDE ? 2 * STAGE : stage * STAGE));
#pragma unroll
    for (int k = 0; k < KS; ++k) kf[st][k] = *(const __attribute__((address_space(3))) raw_t*)(kt + (M == 16 ? st / 2 : st) * 32 * W::ROWB + (kbase[M == 16 ? st & 1 : 0] ^ k * KM * W::ESZ));
  };
  acc sc[ST];
  auto multiply_k = [&](int st, int k) {
    u32x4_t w;
    if constexpr (RAW) w = widen8<DT, KEPT>(kf[st][k]); else w = kf[st][k];
    sc[st] = P1::mfma(__builtin_bit_cast(vec, w), q[k], sc[st]);
  };
  auto clear_scores = [&] {
#pragma unroll
    for (int st = 0; st < ST; ++st)
#pragma unroll
      for (int e = 0; e < CA; ++e) sc[st][e] = 0.f;
  };
  auto take_scores = [&] {
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
      for (int e = 0; e < 8; ++e) z[x][e] = M == 16 ? sc[2 * x + e / 4][e % 4] : sc[x / 2][8 * (x & 1) + e];
  };
  auto scores = [&](int stage) {
    // all pieces of K on their way before the first product
#pragma unroll
    for (int st = 0; st < ST; ++st) load_k(stage, st);
    __builtin_amdgcn_sched_barrier(0);
    clear_scores();
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int st = 0; st < ST; ++st) multiply_k(st, k);
    take_scores();
  };
  raw_t vf[2][DM];                                                     // V of step x, KM positions, and of the next
  auto load_v = [&](int stage, int x) {
    const lds_char* const vt = (const lds_char*)(base + (WIDE ? 2 * STAGE : stage * STAGE)) + WTILE;
#pragma unroll
    for (int d = 0; d < DM; ++d) {
      if constexpr (RAW) {
        typedef __attribute__((address_space(3))) i32x2_t L;
        vf[x & 1][d] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((L*)(vt + x * KM * W::ROWB + (vbase[0] ^ d * M))));
      } else {
        typedef __attribute__((address_space(3))) s16x4_t L;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const u32x2_t raw = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((L*)(vt + x * KM * W::ROWB + (vbase[b] ^ d * 2 * M))));
          vf[x & 1][d][2 * b] = raw[0];
          vf[x & 1][d][2 * b + 1] = raw[1];
        }
      }
    }
  };
  bool partial = false;                                                // some row of the wave does not see all of the tile
  bool again = false, left = false;                                    // AGAIN: second pass over the tiles; the products of the last one with v are left out
  auto seen_in_part = [&](int j0, unsigned ok) { return j0 + KT > min(khi_min, hi) || j0 < klo_max || ok != (1u << KT / 16) - 1; };
  auto probabilities = [&](int t, unsigned ok, int stage, auto early) {
    const int j0 = lo + t * KT;
    const __attribute__((address_space(3))) float* const scales = (const __attribute__((address_space(3))) float*)(base + stage * STAGE + 2 * TILE);
    if constexpr (CODES) {
#pragma unroll
      for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const f32x4_t w = *(const __attribute__((address_space(3))) f32x4_t*)(scales + KM * x + 8 * grp + 4 * f);
#pragma unroll
          for (int e = 0; e < 4; ++e) z[x][4 * f + e] *= w[e];
        }
    }
    partial = seen_in_part(j0, ok);
    if constexpr (AGAIN) left = partial && again;
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
      see = (see & there) >> (8 * grp);
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const uint32_t w = (uint32_t)(see >> (KM * x));
#pragma unroll
        for (int e = 0; e < 8; ++e) z[x][e] = w & (1u << e) ? z[x][e] : -INFINITY;
      }
    }
    float top = z[0][0];
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, z[x][e]);
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
    early();                                                           // what is loaded while the exponentials are taken
    float part_sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (__builtin_expect(far, 0)) {
      const float from = m == -INFINITY ? 0.f : m;                     // then all scores are -infinity or NaN: zeros or NaN
#pragma unroll
      for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[x][e] = __builtin_amdgcn_exp2f((z[x][e] - from) * c2);
    } else {
#pragma unroll
      for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[x][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[x][e], c2, -ref));
    }
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
      for (int e = 0; e < 8; ++e) part_sum[e & 3] += z[x][e];
    sum += (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
    if constexpr (CODES) {
      auto scale = [&](auto some) {                                    // the scale of a row that is not seen may be anything
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            const f32x4_t w = *(const __attribute__((address_space(3))) f32x4_t*)(scales + KT + KM * x + 8 * grp + 4 * f);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[x][4 * f + e] = some.value && z[x][4 * f + e] == 0.f ? 0.f : z[x][4 * f + e] * w[e];
          }
      };
      if (partial) scale(std::true_type{}); else scale(std::false_type{});
    }
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a0 = z[x][2 * e], a1 = z[x][2 * e + 1];
        if constexpr (SPLIT_P && !CODES) {
          // cut, not rounded, and the second part a little larger: both are above zero, and an infinity in v times them is one
          constexpr float more = 1.f + 0x1p-20f;
          const uint32_t f0 = __float_as_uint(a0) & 0xFFFF0000u, f1 = __float_as_uint(a1) & 0xFFFF0000u;
          prob[x][e] = f0 >> 16 | f1;
          rest[x][e] = Half<VDT>::pack(__builtin_fmaf(a0, more, -__uint_as_float(f0)), __builtin_fmaf(a1, more, -__uint_as_float(f1)));
        } else {
          prob[x][e] = Half<VDT>::pack(a0, a1);
          if constexpr (SPLIT_P) rest[x][e] = Half<VDT>::pack(a0 - bf16lo_to_f32(prob[x][e]), a1 - bf16hi_to_f32(prob[x][e]));
        }
      }
  };
  auto multiply_v = [&](int x) {
#pragma unroll
    for (int d = 0; d < DM; ++d) {
      u32x4_t w;
      if constexpr (RAW) w = widen8<VDT, KEPT>(vf[x & 1][d]); else w = vf[x & 1][d];
      o[d] = P2::mfma(__builtin_bit_cast(vvec, w), __builtin_bit_cast(vvec, prob[x]), o[d]);
      if constexpr (SPLIT_P) o[d] = P2::mfma(__builtin_bit_cast(vvec, w), __builtin_bit_cast(vvec, rest[x]), o[d]);
    }
  };
  // A position that a row does not see has p = 0 for it, but 0 * v is NaN if that v is not finite (of codes only e4m3 has such: its NaN).
  //   CLEAR, waves with tiles of their own: in tiles that are not seen whole such numbers are replaced by zeros in front of the products, in the
  //     registers of the operand, and added afterwards to the rows that see them (infinity times any p > 0 is infinity, NaN is NaN).
  //   AGAIN, waves that share tiles and that the test costs more: a workgroup whose sums have come out NaN goes over its tiles again, without the products
  //     with v of those that are not seen whole, and adds these term by term.  us, without either / with the test in the operands or while a tile is
  //     widened / so: prompts of 4 x 3008 tokens 731, 782, 745; 88 rows behind 8192 positions 384, 396, 386; 2048 tokens behind 14336 of an e4m3 cache
  //     1459, 1527, 1468.
  constexpr uint32_t TOP = CODES ? 0x7F7F7F7Fu : VDT == DT_BF16 ? 0x7F807F80u : 0x7C007C00u, ONE = CODES ? 0x01010101u : VDT == DT_BF16 ? 0x00800080u : 0x04000400u;
  constexpr uint32_t SIGN = CODES ? 0x80808080u : 0x80008000u;
  constexpr int FIELD = CODES ? 8 : 16;
  auto infinite_in = [](uint32_t w) { return ((w & TOP) + ONE) & SIGN; };                  // the sign bits of those fields
  auto cleared = [](uint32_t w, uint32_t hit) { return w & ~(hit | (hit - (hit >> (FIELD - 1)))); };
  auto clear_infinite = [&](int i) __attribute__((always_inline)) {                        // of the operand vf[i]: any in the wave?
    uint32_t hit = 0;
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int w = 0; w < (RAW ? 2 : 4); ++w) hit |= infinite_in(vf[i][d][w]);
    if (!__any(hit != 0)) return false;
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int w = 0; w < (RAW ? 2 : 4); ++w) vf[i][d][w] = cleared(vf[i][d][w], infinite_in(vf[i][d][w]));
    return true;
  };
  auto row_sees = [&](int t, unsigned ok, int x) __attribute__((always_inline)) {           // the lane's row, position x of tile t
    const int j = lo + t * KT + x;
    const bool see = a.visible && j >= old ? j - old < 64 && (bits >> (j - old) & 1) : j >= klo && j < khi;
    return see && has && j < hi && (ok >> (x >> 4) & 1);
  };
  auto add_infinite = [&](int t, unsigned ok, int stage) __attribute__((always_inline)) {
    const lds_char* const vt = (const lds_char*)(base + stage * STAGE + TILE);
#pragma unroll 1
    for (int x = 0; x < KT; ++x) {
      const bool see = row_sees(t, ok, x);
#pragma unroll
      for (int d = 0; d < DM; ++d)
#pragma unroll
        for (int b = 0; b < CA / 4; ++b) {
          const int col = M * d + 8 * b + 4 * grp, piece = CODES ? col >> 4 : col >> 3;       // the first of the lane's four columns
          const lds_char* const from = vt + x * F::ROWB + (piece ^ F::turn(x)) * 16 + (CODES ? col & 15 : (col & 7) * 2);
          f32x4_t v;
          if constexpr (CODES) {
            v = decode4<KEPT>(*(const __attribute__((address_space(3))) uint32_t*)from);
          } else {
            const u32x2_t w = *(const __attribute__((address_space(3))) u32x2_t*)from;
            const f32x2_t f0 = Half<DT>::unpack(w[0]), f1 = Half<DT>::unpack(w[1]);
            v = (f32x4_t){f0[0], f0[1], f1[0], f1[1]};
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][4 * b + e] += see && !(fabsf(v[e]) < INFINITY) ? v[e] : 0.f;
        }
    }
  };
  auto sums = [&](int t, unsigned ok, int stage) __attribute__((always_inline)) {          // the first step is on its way
    bool infinite = false;
#pragma unroll
    for (int x = 0; x < NX; ++x) {
      if (x + 1 < NX) load_v(stage, x + 1);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (CLEAR)
        if (partial) infinite |= clear_infinite(x & 1);
      multiply_v(x);
    }
    if constexpr (CLEAR)
      if (__builtin_expect(infinite, 0)) add_infinite(t, ok, stage);
  };

  // AGAIN: behind the first pass, whether there is a second one; all waves of the workgroup together.
  __attribute__((address_space(3))) int* const vote = (__attribute__((address_space(3))) int*)(lds_char*)(smem + KW * GROUP);
  auto once_more = [&]() __attribute__((always_inline)) {
    if (!AGAIN || again) return false;
    bool nan = false;
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int e = 0; e < CA; ++e) nan |= o[d][e] != o[d][e];
    if (nan && has) *vote = 1;
    wait_lds();
    meet();
    again = __builtin_amdgcn_readfirstlane(*vote) != 0;
    if (!again) return false;
    wait_lds();                                                        // all have read it
    meet();
#pragma unroll
    for (int d = 0; d < DM; ++d)
#pragma unroll
      for (int e = 0; e < CA; ++e) o[d][e] = 0.f;
    m = -INFINITY;
    ref = sum = 0.f;
    far = left = false;
    return true;
  };
  auto add_left_out = [&]() __attribute__((always_inline)) {
    if (!AGAIN || !again) return;
    for (int t = kw; t < count; t += KW) {
      const int j0 = lo + t * KT;
      if (!seen(t) || !seen_in_part(j0, exist(look_up(t)))) continue;
#pragma unroll 1
      for (int j = j0; j < min(j0 + KT, hi); ++j) {
        const long x = place_of(c, s, j, g);
        const bool see = has && x >= 0 && (a.visible && j >= old ? j - old < 64 && (bits >> (j - old) & 1) : j >= klo && j < khi);
        if (!__any(see)) continue;
        float y = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          u32x4_t w = __builtin_bit_cast(u32x4_t, q[k]), kk;
          if constexpr (TURNS) {                                       // read again: with it kept to here prompts take 1 % longer
            w = (u32x4_t){};
            if (has) w = *(const u32x4_t*)((const uint16_t*)a.q + t_row * a.q_pitch + (long)head * D + KM * k + 8 * grp) ^ flip;
          }
          if constexpr (CODES) kk = widen8<DT, KEPT>(*(const u32x2_t*)((const char*)a.kc + x * D + KM * k + 8 * grp));
          else kk = *(const u32x4_t*)((const char*)a.kc + (x * D + KM * k + 8 * grp) * 2);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const f32x2_t u = Half<DT>::unpack(w[e]), v = Half<DT>::unpack(kk[e]);
            y += u[0] * v[0] + u[1] * v[1];
          }
        }
        y = row_sum<M>(y);
        if constexpr (CODES) y *= a.ks[x];
        float p = __builtin_amdgcn_exp2f((y - m) * c2);
        if constexpr (CODES) p *= a.vs[x];
#pragma unroll
        for (int d = 0; d < DM; ++d)
#pragma unroll
          for (int b = 0; b < CA / 4; ++b) {
            const long from = x * D + M * d + 8 * b + 4 * grp;
            f32x4_t v;
            if constexpr (CODES) {
              v = decode4<KEPT>(*(const uint32_t*)((const char*)a.vc + from));
            } else {
              const u32x2_t w = *(const u32x2_t*)((const char*)a.vc + from * 2);
              const f32x2_t f0 = Half<DT>::unpack(w[0]), f1 = Half<DT>::unpack(w[1]);
              v = (f32x4_t){f0[0], f0[1], f1[0], f1[1]};
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[d][4 * b + e] = see ? __builtin_fmaf(p, v[e], o[d][4 * b + e]) : o[d][4 * b + e];
          }
      }
    }
  };

  if constexpr (TURNS) {
    // Two waves on every SIMD, one of each half of the workgroup, take turns: while one multiplies (the sums of a tile, the scores of the next), the
    // other exponentiates.  Slot 2 t: the first half multiplies for tile t, the second has the probabilities of tile t - 1; then the other way round.
    // Tile t is read in the slots 2 t .. 2 t + 3 and sent for in slot 2 t - 4, when the tile four before it has been used.
    const bool second = rw >= RW / 2;
    Pages next;
    unsigned ring = 0;                                                 // what exists of the tiles in the four stages
    int sent = 0;
    auto send = [&] {
      if (sent < count) {
        ring = (ring & ~(15u << 4 * (sent & 3))) | exist(next) << 4 * (sent & 3);
        fetch(sent, next, sent & 3);
        ++sent;
        if (sent < count) next = look_up(sent);
      }
    };
    auto arrived = [&](int t) {                                        // tile t, of which at most the next one is sent behind it
      if (sent > t + 1) wait_loads<2 * LOADS>(); else wait_loads<0>();
    };
    auto slot = [&] {
      __builtin_amdgcn_sched_barrier(0);
      wait_lds();                                                      // nothing of a stage is still being read
      meet();
      __builtin_amdgcn_sched_barrier(0);
    };
    while (count > 0) {
      if (tid == 0) *vote = 0;                                         // all meet behind it and in front of its use
      ring = sent = 0;
      next = look_up(0);
      send();
      send();
      arrived(0);
      slot();
      if (second) {
        send();
        slot();
      }
      for (int t = 0; t < count; ++t) {
        if (!second) send();
        // the first half of K on its way before the products with V, the second before those with the first
        load_k(t & 3, 0);
        if (t > 0 && seen(t - 1) && !left) {
          load_v((t - 1) & 3, 0);
          sums(t - 1, 0, (t - 1) & 3);
        }
        load_k(t & 3, 1);
        __builtin_amdgcn_sched_barrier(0);
        clear_scores();
#pragma unroll
        for (int st = 0; st < ST; ++st)
#pragma unroll
          for (int k = 0; k < KS; ++k) multiply_k(st, k);
        take_scores();
        if (second) arrived(t + 1);
        slot();
        if (second) send();
        if (seen(t)) probabilities(t, ring >> 4 * (t & 3) & 15, t & 3, [] {});
        if (!second) arrived(t + 1);
        slot();
      }
      if (!second) slot();
      if (seen(count - 1) && !left) {
        load_v((count - 1) & 3, 0);
        sums(count - 1, 0, (count - 1) & 3);
      }
      if (!once_more()) break;
    }
    add_left_out();
  } else if (count > 0) {
    // tile t of the group's: fetched while the one before is computed.  All waves of a workgroup meet as often as the group with most tiles needs.
    const int mine = kw < count ? (count - kw + KW - 1) / KW : 0, most = (count + KW - 1) / KW;
    do {
    Pages now, next;
    if (AGAIN && tid == 0) *vote = 0;                                  // all meet behind it and in front of its use
    if (mine > 0) { now = look_up(kw); fetch(kw, now, 0); }
    if (mine > 1) next = look_up(kw + KW);
    for (int t = 0; t < most; ++t) {
      const bool work = t < mine, more = t + 1 < mine;
      unsigned ok = 0;
      if (work) ok = exist(now);
      auto ahead = [&] {
        fetch(kw + (t + 1) * KW, next, (t + 1) & 1);
        now = next;
        if (t + 2 < mine) next = look_up(kw + (t + 2) * KW);
      };
      if constexpr (WIDE) {
        wait_loads<0>();
        meet();                                                        // the tile is there, and the one before has been used
        if (more) ahead();
        if (work) widen(t & 1);
        wait_lds();
        meet();
      } else {
        if (more) {
          ahead();
          wait_loads<2 * LOADS + (CODES ? 1 : 0)>();
        } else {
          wait_loads<0>();
        }
        if constexpr (RW > 1) meet();                                  // the others' parts of the tile are there as well
      }
      __builtin_amdgcn_sched_barrier(0);
      if (work && seen(kw + t * KW)) {
        scores(t & 1);
        probabilities(kw + t * KW, ok, t & 1, [&] { load_v(t & 1, 0); });
        if (!left) sums(kw + t * KW, ok, t & 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_lds();                                                      // nothing reads the stage that is filled next
      if constexpr (RW > 1 && !WIDE) meet();
    }
    } while (once_more());
    add_left_out();
  }

  sum = row_sum<M>(sum);
  m *= unit;                                             // in units of the scores

  // ---- the waves that shared the rows
  if constexpr (KW > 1) {
    constexpr int SLOT = D * M * 4 + 512;                              // sums, then references and sums of p of a wave's lanes
    __syncthreads();
    if (kw > 0) {
      char* const to = smem + ((kw - 1) * RW + rw) * SLOT;
#pragma unroll
      for (int d = 0; d < DM; ++d)
#pragma unroll
        for (int b = 0; b < CA / 4; ++b) *(f32x4_t*)(to + (d * (CA / 4) + b) * 1024 + lane * 16) = (f32x4_t){o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
      *(float*)(to + D * M * 4 + lane * 4) = m;
      *(float*)(to + D * M * 4 + 256 + lane * 4) = sum;
    }
    __syncthreads();
    if (kw == 0) {
#pragma unroll
      for (int w = 0; w < KW - 1; ++w) {
        const char* const other = smem + (w * RW + rw) * SLOT;
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
    }
  }
  if (kw == 0 && has) {
    if (whole) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint16_t* const out = (uint16_t*)a.out + t_row * a.out_pitch + (long)head * D;
#pragma unroll
      for (int d = 0; d < DM; ++d)
#pragma unroll
        for (int b = 0; b < CA / 4; ++b)
          *(u32x2_t*)(out + M * d + 8 * b + 4 * grp) = (u32x2_t){Half<DT>::pack(o[d][4 * b] * inv, o[d][4 * b + 1] * inv), Half<DT>::pack(o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv)};
      if (a.lse && grp == 0) a.lse[(long)t_row * a.heads + head] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
    } else {
      // a share begins inside at most one item and ends inside at most one other
      const long row = (long)(2 * share + (from > 0 ? 0 : 1)) * TR + (r - r0);
#pragma unroll
      for (int d = 0; d < DM; ++d)
#pragma unroll
        for (int b = 0; b < CA / 4; ++b) *(f32x4_t*)(part + row * D + M * d + 8 * b + 4 * grp) = (f32x4_t){o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
      if (grp == 0) stat[row] = (f32x2_t){m, sum};
    }
  }
  if (x >= x_end) return;
  __syncthreads();                                                     // the tiles' LDS is used again
  p = find<false>(c, a, sp, x);
  }
}

// Adds up the items in several pieces, 32 lanes a row's sums from one piece: ROWS = 8, a row each for few pieces; ROWS = 1, every eighth piece of the
// same row for many.  Eight pieces are on their way at once.
constexpr int JT = 256;
template <int DT, int D, int ROWS>
__global__ __launch_bounds__(JT) void attend_join_kernel(Attend a, int T, int G, int tile_rows, int shares, const float* __restrict__ part, const f32x2_t* __restrict__ stat,
                                                         const Joined* __restrict__ joined, const int* __restrict__ joined_count) {
  constexpr int PARTS = JT / 32 / ROWS;
  __shared__ f32x4_t sums[PARTS][32];
  __shared__ float totals[PARTS];
  const int at = threadIdx.x & 31, group = threadIdx.x / 32, in_tile = blockIdx.y * ROWS + (ROWS == 1 ? 0 : group), mine = ROWS == 1 ? group : 0;
  if ((int)blockIdx.x >= *joined_count) return;
  const Joined it = joined[blockIdx.x];
  const int r = it.r0 + in_tile;
  if (it.pieces == 0 || r >= it.rows) return;          // ROWS == 1: all threads alike
  const int t = it.row0 + r / G, head = it.head0 + r % G;
  // a record that nobody wrote, where `start` does not ascend, leads nowhere
  if (it.pieces < 0 || it.share < 0 || it.pieces > shares - it.share || r < 0 || t < 0 || t >= T || it.head0 < 0 || it.head0 > a.heads - G) return;
  auto row_of = [&](int k) { return (long)(2 * (it.share + k) + (k == 0 ? 1 : 0)) * tile_rows + in_tile; };
  float m = -INFINITY;
  for (int k = at; k < it.pieces; k += 32) m = fmaxf(m, stat[row_of(k)][0]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float zero = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = mine; k0 < it.pieces; k0 += 8 * PARTS) {
    f32x2_t st[8];
    f32x4_t v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const long row = row_of(min(k0 + k * PARTS, it.pieces - 1));
      st[k] = stat[row];
      v[k] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
      if (at * 4 < D) v[k] = *(const f32x4_t*)(part + row * D + at * 4);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const bool has = k0 + k * PARTS < it.pieces;
      const float f = has ? __builtin_amdgcn_exp2f((st[k][0] - zero) * kLog2E) : 0.f;
      sum += has ? st[k][1] * f : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += has ? v[k][e] * f : 0.f;
    }
  }
  if constexpr (PARTS > 1) {
    sums[mine][at] = o;
    if (at == 0) totals[mine] = sum;
    __syncthreads();
    if (mine > 0) return;
#pragma unroll
    for (int k = 1; k < PARTS; ++k) {
      sum += totals[k];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += sums[k][at][e];
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (at * 4 < D)
    *(u32x2_t*)((uint16_t*)a.out + t * a.out_pitch + (long)head * D + at * 4) = (u32x2_t){Half<DT>::pack(o[0] * inv, o[1] * inv), Half<DT>::pack(o[2] * inv, o[3] * inv)};
  if (a.lse && at == 0) a.lse[(long)t * a.heads + head] = sum == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(sum) * kLn2;
}

// ---- the rule for the form of the workgroups and the split, by the rows of a sequence (tokens x heads for each key head) in the mean.
// Tiles of 16 rows up to 16, of 32 (64, 128) up to 32 (64, any more); us for 64 x 8192 positions of a 16-bit cache, 8 key heads: 4 rows for each in
// 16-row tiles 352, in 32-row tiles 372; 64 rows 357, 88 rows 397, all near the 370 that the bytes take at 5.8 TB/s.
// 256 rows whose waves take turns (16-bit caches) from 512 on, where the workgroups, one on a compute unit, are shares or many: 512 tokens behind 32256
// 587 instead of 658 with 128 rows, 1024 behind 15360 565 instead of 626, prompts of 6000 (1500 items) 668 and 686, of 4096 (1024) 329 and 334.  Between 257 and
// 1023 items, of the larger size, it goes by how the last round of 256 is filled, which lengths decide that the host does not know: prompts of 272 items 53 and 46,
// 376 113 and 107, 512 100 and 106, 640 160 and 151, 768 202 and 197 (1090 and 1167 with 9000 positions in front), 896 262 and 263; 128 rows there.
// The rows are the mean over the sequences, padding and empty ones included: one long chunk among single tokens gives each token a tile of its size.
// Shares where a workgroup per item would leave half of the device idle: 256 tokens behind 32512 (128 items of 128 rows) 361 instead of 909, single tokens
// of 8 sequences 40 instead of 70, 8 drafted tokens of 4 sequences 37 instead of 128, a tree behind 120001 positions 84 instead of 5450; 32 segments
// behind 900 to 6100 (256 items) 119.5 and 121.5.  With more items there is nothing to gain, as those that still run have the memory to themselves: 64
// single tokens behind 700 to 7900 (512 items) 126 by shares and 123 by items; and a share's way from one item to the next is not hidden: 96 segments
// (768 items) 184 and 151, 256 single tokens of a 16-bit cache 408 and 280, of an 8-bit one 202 and 165; 544 items of a window over several
// sequences 181 and 112, as shares do not read the same positions at the same time.
struct Plan { int width, rw; Split sp; unsigned grid; bool many; };     // many: pieces for an item

Plan plan_of(const Paged& c, int heads, int max_len) {
  const long G = heads / c.H, rows = (long)c.T * G, mean = (rows + c.S - 1) / c.S;
  auto about = [&](long tile) { return (mean + tile - 1) / tile * c.S * c.H; };       // items, if the sequences were alike
  Plan p;
  p.width = mean <= 16 ? 16 : 32;
  p.rw = mean <= 32 ? 1 : mean <= 64 ? 2 : c.kept == c.dtype && mean >= 512 && (about(256) <= 256 || about(256) >= 1024) ? 8 : 4;
  const int TR = p.width * p.rw;
  p.sp.rows = TR;
  p.sp.unit = p.rw == 1 ? 128 : 64;                  // a tile for each wave that takes tiles of its own
  p.sp.least = 2;                                    // a share's own beginning and end cost some units' time
  p.sp.tiles = (int)(rows / TR + c.S);               // at most: a sequence begins a tile
  // As many shares as are at work at once: one or two on each of 256 compute units, by the LDS of the form; four waves with two stages of 16-bit tiles of
  // their own, in rows of 256 bytes, take 128 of its 160 KB, as do eight that take turns.  us for 8 tokens of 4 heads for each of 8 key heads of 128, 256 shares
  // and 512: one sequence of 30000 positions 39 and 50, 8 of 900 to 6100 36 and 49, 16 71 and 79, 32 (no shares with the one, shares with the other) 105 and 118.
  const bool alone = p.rw == 8 || (p.rw == 1 && c.kept == c.dtype && c.D > 64);
  const int slots = alone ? 256 : 512;
  const long items = (long)p.sp.tiles * c.H, units = (max_len + p.sp.unit - 1) / p.sp.unit;
  const bool share = 2 * about(TR) <= slots && (double)items * units < 2e9;       // units are counted in 32 bits
  p.sp.shares = share ? slots : 0;
  p.sp.joins = (int)items;                           // of shares at most `slots`: rows / TR + S is at most twice what `about` says
  p.many = slots >= 8 * items;
  p.grid = share ? slots : (unsigned)items;
  return p;
}

size_t part_bytes(const Paged& c, const Split& sp) { return (size_t)2 * sp.shares * sp.rows * c.D * sizeof(float); }

template <int DT, int KEPT, int D, int M, int RW, int KW, int KT>
hipError_t launch_form(const Paged& c, const Attend& a, const Plan& p, void* ws, hipStream_t stream) {
  typedef Form<DT, KEPT, D> F;
  constexpr size_t stage = 2 * KT * F::ROWB + (KEPT != DT ? 8 * KT : 0), wide = KEPT != DT && RW > 1 ? 2 * KT * Form<DT, DT, D>::ROWB : 0, slots = (size_t)(KW - 1) * RW * (D * M * 4 + 512);
  constexpr size_t tiles = KW * ((RW == 8 ? 4 : 2) * stage + wide) + (KEPT != DT_I8 && RW > 1 ? 16 : 0), lds = tiles > slots ? tiles : slots;
  static PerDeviceInt raised;
  hipError_t e = ensure_dynamic_lds(raised, (const void*)attend_kernel<DT, KEPT, D, M, RW, KW, KT>, lds);
  if (e != hipSuccess) return e;
  float* part = (float*)ws;
  f32x2_t* stat = (f32x2_t*)((char*)ws + part_bytes(c, p.sp));
  Joined* joined = (Joined*)(stat + (size_t)2 * p.sp.shares * p.sp.rows);
  int* joined_count = (int*)(joined + p.sp.joins);
  hipLaunchKernelGGL((attend_kernel<DT, KEPT, D, M, RW, KW, KT>), dim3(p.grid), dim3(64 * RW * KW), lds, stream, c, a, p.sp, part, stat, joined, joined_count);
  if ((e = hipGetLastError()) != hipSuccess || p.sp.shares == 0) return e;
  const int G = a.heads / c.H;
  if (p.many)
    hipLaunchKernelGGL((attend_join_kernel<DT, D, 1>), dim3((unsigned)p.sp.joins, p.sp.rows), dim3(JT), 0, stream, a, c.T, G, p.sp.rows, p.sp.shares, (const float*)part, (const f32x2_t*)stat,
                       (const Joined*)joined, (const int*)joined_count);
  else
    hipLaunchKernelGGL((attend_join_kernel<DT, D, 8>), dim3((unsigned)p.sp.joins, p.sp.rows / 8), dim3(JT), 0, stream, a, c.T, G, p.sp.rows, p.sp.shares, (const float*)part, (const f32x2_t*)stat,
                       (const Joined*)joined, (const int*)joined_count);
  return hipGetLastError();
}

template <int DT, int KEPT, int D>
hipError_t launch_attend_d(const Paged& c, const Attend& a, void* ws, hipStream_t stream) {
  const Plan p = plan_of(c, a.heads, a.max_len);
  if (p.width == 16) return launch_form<DT, KEPT, D, 16, 1, 4, 32>(c, a, p, ws, stream);
  if (p.rw == 1) return launch_form<DT, KEPT, D, 32, 1, 4, 32>(c, a, p, ws, stream);
  if (p.rw == 2) return launch_form<DT, KEPT, D, 32, 2, 2, 32>(c, a, p, ws, stream);
  if constexpr (DT == KEPT)
    if (p.rw == 8) return launch_form<DT, KEPT, D, 32, 8, 1, 64>(c, a, p, ws, stream);
  return launch_form<DT, KEPT, D, 32, 4, 1, 64>(c, a, p, ws, stream);
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
  return p.sp.shares == 0 ? 256 : part_bytes(c, p.sp) + (size_t)2 * p.sp.shares * p.sp.rows * sizeof(f32x2_t) + p.sp.joins * sizeof(Joined) + sizeof(int);
}

// A launch has fewer than 2^32 threads.
bool attend_fits(const Paged& c, int heads, int max_len) {
  const Plan p = plan_of(c, heads, max_len);
  return (double)(c.S + (long)c.T * (heads / c.H) / p.sp.rows) * c.H * 512 < 4e9 || p.sp.shares > 0;
}

hipError_t launch_attend(const Paged& c, const Attend& a, void* ws, hipStream_t stream) {
  if (c.dtype == DT_BF16) return launch_attend_t<DT_BF16>(c, a, ws, stream);
  if (c.dtype == DT_F16) return launch_attend_t<DT_F16>(c, a, ws, stream);
  return hipErrorInvalidValue;
}

}  // namespace covspec
