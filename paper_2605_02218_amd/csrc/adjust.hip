// What a sampler does to logits before they are verified: penalties for words that were said, biases, temperature, a grammar's mask.
//
// For a word with n occurrences in what the model has said, x = z F + A with F = (said or asked ? (z > 0 ? 1 / r : r) : 1) / T and
// A = (bias - (f n + (n > 0 ? c : 0))) / T, -infinity where the mask says so.  One workgroup takes a chunk of the vocabulary, a vector of words a thread, for all positions of a
// sequence: the history is counted once in LDS (a word of it lands in one of the chunks), a thread then keeps the counts of its words in
// registers, and from one position to the next only the drafted word between them is added.
#include "vocab.h"

namespace covspec {

namespace {

// Threads of a workgroup, rows on their way; us for 64 x 8 rows of 151936 bf16 words with histories, biases and masks: 512 threads and one row 79.2,
// two 74, three 74.4, four 75.2; two rows with 256 threads 80, with 1024 75.
constexpr int AT = 512;
constexpr int AHEAD = 2;

template <int DT>
__device__ __forceinline__ void store_logits(void* p, long i, const float (&x)[LogitVec<DT>::N]) {
  u32x4_t w;
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(x[e]);
    *(u32x4_t*)((float*)p + i) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (DT == DT_BF16) {
        typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
        w[e] = __builtin_bit_cast(uint32_t, (pair_t){(__bf16)x[2 * e], (__bf16)x[2 * e + 1]});
      } else {
        typedef _Float16 pair_t __attribute__((ext_vector_type(2)));
        w[e] = __builtin_bit_cast(uint32_t, (pair_t){(_Float16)x[2 * e], (_Float16)x[2 * e + 1]});
      }
    }
    *(u32x4_t*)((uint16_t*)p + i) = w;
  }
}

template <int DT>
__global__ __launch_bounds__(AT) void adjust_kernel(Adjust a, int L, int V) {
#pragma clang fp contract(off)
  constexpr int N = LogitVec<DT>::N;
  __shared__ alignas(16) int seen[AT * N];       // bit 0: in the prompt; above it: occurrences behind the prompt
  __shared__ alignas(16) int entry[AT * N];      // index of the word's last bias, counted from 1 within the sequence's
  const int s = blockIdx.y, w0 = blockIdx.x * AT * N, tid = threadIdx.x;
  const int mine = w0 + tid * N;                 // V % N == 0: whole vectors only
  const bool has = mine < V;
  const long row0 = (long)s * L;
  // The rows on their way with their masks, the first ones while the history is counted.  Loads come back in order: nothing else is loaded in
  // the loop over the rows, or it would wait for all of these.
  const int pitch = (V + 31) / 32;
  u32x4_t next[AHEAD];
  uint32_t mask[AHEAD];
  auto fetch = [&](int t, int u) {
    if (has && t < L) {
      next[u] = LogitVec<DT>::load_raw(a.z, (row0 + t) * V + mine);
      if (a.allowed) mask[u] = a.allowed[(row0 + t) * pitch + (mine >> 5)];        // N divides 32: one word holds them all
    }
  };
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) {
    next[t] = (u32x4_t){};
    mask[t] = 0;
    fetch(t, t);
  }
  const int lane = tid & 63, word_of = a.drafted && lane < L - 1 ? a.drafted[row0 + lane] : -1;      // no row lies behind the last
#pragma unroll
  for (int e = 0; e < N; e += 4) *(u32x4_t*)(seen + tid * N + e) = (u32x4_t){};
  if (a.bias_start) {
#pragma unroll
    for (int e = 0; e < N; e += 4) *(u32x4_t*)(entry + tid * N + e) = (u32x4_t){};
  }
  __syncthreads();
  // counted from the history's own beginning: a prompt_len of any size, the largest there is included, only ever means the words in front of it
  const int h0 = a.history_start[s], asked = a.prompt_len ? a.prompt_len[s] : 0;
  const unsigned words = (unsigned)max(a.history_start[s + 1] - h0, 0);
#pragma unroll 4
  for (unsigned i = tid; i < words; i += AT) {
    const int w = a.history[h0 + (int)i];
    const unsigned at = (unsigned)w - (unsigned)w0;
    if (w >= 0 && w < V && at < (unsigned)(AT * N)) {
      if ((int)i < asked) atomicOr(seen + at, 1); else atomicAdd(seen + at, 2);
    }
  }
  int b0 = 0;
  if (a.bias_start) {
    b0 = a.bias_start[s];
    const int b1 = a.bias_start[s + 1];
    for (int i = b0 + tid; i < b1; i += AT) {
      const int w = a.bias_word[i];
      const unsigned at = (unsigned)w - (unsigned)w0;
      if (w >= 0 && w < V && at < (unsigned)(AT * N)) atomicMax(entry + at, i - b0 + 1);
    }
  }
  __syncthreads();
  if (!has) return;
  const float rep = a.penalties[4 * s], pres = a.penalties[4 * s + 1], freq = a.penalties[4 * s + 2], temp = a.penalties[4 * s + 3];
  const float irep = 1.f / rep, itemp = temp > 0.f ? 1.f / temp : 1.f;
  // x F + A: a word's F above and below zero, and A, for the n occurrences in `seen`.  Without a bias the zero is the negative one, and A with it where
  // nothing is subtracted either: x + -0 is x for both zeros.
  float up[N], down[N], add[N];
  auto word = [&](int e, int n, int i) {
    const float bias = i > 0 ? a.bias_value[b0 + i - 1] : -0.f;
    const int said = n >> 1;
    up[e] = n == 0 ? itemp : irep * itemp;
    down[e] = n == 0 ? itemp : rep * itemp;
    const float less = freq * (float)said + (said > 0 ? pres : 0.f);
    add[e] = (bias - less) * itemp;
  };
#pragma unroll
  for (int e = 0; e < N; ++e) word(e, seen[tid * N + e], a.bias_start ? entry[tid * N + e] : 0);
  for (int t0 = 0; t0 < L; t0 += AHEAD)
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    const int t = t0 + u;
    if (t >= L) break;
    float x[N];
    LogitVec<DT>::unpack(next[u], x);
    const uint32_t bits = mask[u] >> (mine & 31);
    fetch(t + AHEAD, u);
    if (t > 0) {
      const unsigned at = (unsigned)__builtin_amdgcn_readlane(word_of, t - 1) - (unsigned)mine;
      if (at < (unsigned)N) {                    // one thread of the row's
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (at == (unsigned)e) word(e, seen[tid * N + e] += 2, a.bias_start ? entry[tid * N + e] : 0);
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = __builtin_fmaf(x[e], x[e] > 0.f ? up[e] : down[e], add[e]);
    if (a.allowed) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint32_t keep = (uint32_t)((int32_t)(bits << (31 - e)) >> 31);
        x[e] = __uint_as_float((__float_as_uint(x[e]) & keep) | (0xFF800000u & ~keep));
      }
    }
    store_logits<DT>(a.out, (row0 + t) * V + mine, x);
  }
}

template <int DT>
hipError_t launch_adjust_t(const Adjust& a, int S, int L, int V, hipStream_t stream) {
  constexpr int words = AT * LogitVec<DT>::N;
  hipLaunchKernelGGL((adjust_kernel<DT>), dim3((V + words - 1) / words, S), dim3(AT), 0, stream, a, L, V);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adjust(const Adjust& a, int S, int L, int V, int dtype, hipStream_t stream) {
  if (S < 1 || L < 1 || V < 2 || S > 65535) return hipErrorInvalidValue;
  if (dtype == DT_BF16) return launch_adjust_t<DT_BF16>(a, S, L, V, stream);
  if (dtype == DT_F16) return launch_adjust_t<DT_F16>(a, S, L, V, stream);
  return launch_adjust_t<DT_F32>(a, S, L, V, stream);
}

}  // namespace covspec
