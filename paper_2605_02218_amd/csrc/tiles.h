// Pieces shared by the kernels that attend over a paged cache: forms of a tile of keys or values in LDS, the matrix products, loads into LDS and the
// waits for them, exchanges between the lanes of a row.
#pragma once
#include "paged.h"

namespace covspec {

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

// A product of M columns (positions for S^T, columns of v for O^T) with M rows over KM terms; a lane has eight neighbouring terms of an operand, those
// of its group of M lanes, and CA values of the result: column 8 b + 4 group + i for value 4 b + i.
template <int DT, int M> struct Operand;
template <> struct Operand<DT_BF16, 32> {
  typedef bf16x8_t vec;
  typedef f32x16_t acc;
  static __device__ __forceinline__ acc mfma(vec a, vec b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<DT_F16, 32> {
  typedef f16x8_t vec;
  typedef f32x16_t acc;
  static __device__ __forceinline__ acc mfma(vec a, vec b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<DT_BF16, 16> {
  typedef bf16x8_t vec;
  typedef f32x4_t acc;
  static __device__ __forceinline__ acc mfma(vec a, vec b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<DT_F16, 16> {
  typedef f16x8_t vec;
  typedef f32x4_t acc;
  static __device__ __forceinline__ acc mfma(vec a, vec b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
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

// Over the lanes of a row, one in each group of M.
template <int M, typename F>
__device__ __forceinline__ float over_groups(float x, F f) {
  if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int M> __device__ __forceinline__ float row_max(float x) { return over_groups<M>(x, [](float a, float b) { return fmaxf(a, b); }); }
template <int M> __device__ __forceinline__ float row_sum(float x) { return over_groups<M>(x, [](float a, float b) { return a + b; }); }

// Pool to LDS, 16 or 4 bytes a lane: to `lds` + lane * 16 (4).  Written out because the compiler, where it knows of such a load, waits for all
// of them in front of the first transposing read; here the waits are the kernel's own (wait_loads).  No register is loaded.  s_nop: five cycles
// between a vector instruction that wrote the address' scalar registers and this, one behind m0, which nothing else here uses.
__device__ __forceinline__ void load16_lds(unsigned lds, const void* base, unsigned off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load4_lds(unsigned lds, const void* from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(from) : "memory");
}
__device__ __forceinline__ long uniform(long v) {
  return (long)(((unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)v));
}
// Waits that no access to memory is moved across.
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void meet() { asm volatile("s_barrier" ::: "memory"); }

}  // namespace covspec
