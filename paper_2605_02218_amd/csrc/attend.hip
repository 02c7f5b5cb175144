// Attention of a batch's rows over a paged cache.
#include "paged.h"

namespace covspec {

namespace {

// A row's statistics and sums over the positions it sees, one wave per row and head: a lane takes a position in turn for the scores, then all
// lanes two or fewer columns of v.
template <int DT, int KEPT, int D>
__global__ __launch_bounds__(64) void attend_rows_kernel(Paged c, Attend a) {
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  const int s = seq_of(c.start, c.S, t);
  if (s < 0 || s >= c.S) return;
  const int g = h / (a.heads / c.H);
  const int first = c.start[s], n = c.start[s + 1] - first, i = t - first;
  const long old = (long)c.length[s] - n, pos = old + i;
  const long seen_end = a.visible ? min(old + n, old + 64) : pos + 1;
  const long k1 = min(seen_end, (long)a.max_len), k0 = max(0l, a.window > 0 ? pos + 1 - a.window : 0l);
  const long long bits = a.visible ? a.visible[t] : 0;
  __shared__ float q[D];
  __shared__ float p[64];
  __shared__ long at[64];
  for (int d = lane; d < D; d += 64) q[d] = Half<DT>::unpack(((const uint16_t*)a.q)[t * a.q_pitch + h * D + d])[0];
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
  auto value = [&](const void* codes, const float* scale, long x, int d) {
    if constexpr (KEPT == DT) return Half<DT>::unpack(((const uint16_t*)codes)[x * D + d])[0];
    else return decode4<KEPT>(((const uint8_t*)codes)[x * D + d])[0] * scale[x];
  };
  for (long j0 = k0; j0 < k1; j0 += 64) {
    const long j = j0 + lane;
    bool see = j < k1;
    if (a.visible && j >= old) see = see && (bits >> (j - old) & 1);
    const long x = see ? place_of(c, s, j, g) : -1;
    float z = -INFINITY;
    if (x >= 0) {
      z = 0.f;
      for (int d = 0; d < D; ++d) z += q[d] * value(a.kc, a.ks, x, d);
      z *= a.scale;
    }
    const float top = fmaxf(m, wave_max(z));
    const float ref = top == -INFINITY ? 0.f : top, keep = expf(m - ref);
    const float e = x >= 0 ? expf(z - ref) : 0.f;
    m = top;
    l = l * keep + wave_sum(e);
    __syncthreads();
    p[lane] = e;
    at[lane] = x;
    __syncthreads();
    for (int k = 0; k < 2; ++k) o[k] *= keep;
    for (int y = 0; y < 64; ++y)
      if (at[y] >= 0)
        for (int k = 0; k < 2; ++k)
          if (lane + 64 * k < D) o[k] += p[y] * value(a.vc, a.vs, at[y], lane + 64 * k);
  }
  for (int k = 0; k < 2; ++k)
    if (lane + 64 * k < D) ((uint16_t*)a.out)[t * a.out_pitch + h * D + lane + 64 * k] = (uint16_t)Half<DT>::pack(l == 0.f ? 0.f : o[k] / l, 0.f);
  if (a.lse && lane == 0) a.lse[(long)t * a.heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

template <int DT, int KEPT>
hipError_t launch_attend_d(const Paged& c, const Attend& a, hipStream_t stream) {
  const dim3 grid(c.T, a.heads), block(64);
  if (c.D == 64) hipLaunchKernelGGL((attend_rows_kernel<DT, KEPT, 64>), grid, block, 0, stream, c, a);
  else if (c.D == 96) hipLaunchKernelGGL((attend_rows_kernel<DT, KEPT, 96>), grid, block, 0, stream, c, a);
  else if (c.D == 128) hipLaunchKernelGGL((attend_rows_kernel<DT, KEPT, 128>), grid, block, 0, stream, c, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

template <int DT>
hipError_t launch_attend_t(const Paged& c, const Attend& a, hipStream_t stream) {
  if (c.kept == DT) return launch_attend_d<DT, DT>(c, a, stream);
  if (c.kept == DT_I8) return launch_attend_d<DT, DT_I8>(c, a, stream);
  if (c.kept == DT_E4M3) return launch_attend_d<DT, DT_E4M3>(c, a, stream);
  return hipErrorInvalidValue;
}

}  // namespace

size_t attend_workspace_bytes(const Paged&, int, int) { return 256; }

hipError_t launch_attend(const Paged& c, const Attend& a, void*, hipStream_t stream) {
  if (c.dtype == DT_BF16) return launch_attend_t<DT_BF16>(c, a, stream);
  if (c.dtype == DT_F16) return launch_attend_t<DT_F16>(c, a, stream);
  return hipErrorInvalidValue;
}

}  // namespace covspec
