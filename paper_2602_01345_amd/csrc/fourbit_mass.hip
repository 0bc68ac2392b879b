// What the rows of the 4-bit cache collect of the queries' attention.
#include "fourbit.h"

namespace {

// One thread per key.
template <typename T, int DH>
__global__ __launch_bounds__(64) void mass_kernel(const T* __restrict__ q, int64_t q_sb, int64_t q_sr, int64_t q_sh, FourBitView c,
                                                  int heads, int n, const int32_t* __restrict__ n_rows, int P,
                                                  const int32_t* __restrict__ kv_rows, float scale_log2,
                                                  const float* __restrict__ lse, const float* __restrict__ mass_in,
                                                  float* __restrict__ mass) {
  const int b = blockIdx.y, lane = threadIdx.x, j = blockIdx.x;
  const int len = image_prior(kv_rows, b, P), nq = image_count(n_rows, b, n);
  constexpr int GPR = DH / kGroup;
  const int64_t at = (int64_t)b * c.cap + j;
  if (j >= len) {
    if (lane == 0) mass[at] = -1.0f;
    return;
  }
  float sum = 0.f;
  for (int64_t i = lane; i < (int64_t)nq * heads; i += 64) {
    const int s = (int)(i / heads), h = (int)(i % heads);
    const T* qp = q + b * q_sb + s * q_sr + h * q_sh;
    const int64_t r = ((int64_t)b * c.hk + h / (heads / c.hk)) * c.cap + j;
    float sc = 0.f;
    for (int g = 0; g < GPR; ++g) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(c.codes[0] + (r * GPR + g) * 16);
      const float ks = fourbit_scale(c.scales[0][r * GPR + g]);
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const bf16x8 kv = fourbit_eight(w[jj], ks);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc = fmaf((float)qp[g * kGroup + jj * 8 + e], (float)kv[e], sc);
      }
    }
    sum += __builtin_amdgcn_exp2f(fmaf(sc, scale_log2, -lse[((int64_t)b * n + s) * heads + h] * 1.4426950408889634f));
  }
  sum = wave_sum(sum);
  if (lane == 0) {
    const float m0 = mass_in ? mass_in[at] : 0.f;
    mass[at] = (m0 > 0.f ? m0 : 0.f) + sum;
  }
}

}  // namespace

size_t fourbit_mass_workspace_bytes(const nova_fourbit_cache&, int, int, int) { return 0; }

hipError_t launch_fourbit_mass(const nova_ctx*, hipStream_t st, int dtype, const nova_fourbit_cache& c, int heads, int n,
                               const nova_rows& q, const int32_t* n_rows, int P, const int32_t* kv_rows, float scale_log2,
                               const float* lse, const float* mass_in, float* mass, void*) {
  if (c.capacity == 0) return hipSuccess;
  const dim3 grid(c.capacity, c.B);
#define GO(T, DH)                                                                                                    \
  mass_kernel<T, DH><<<grid, 64, 0, st>>>(static_cast<const T*>(q.data), q.stride_b, q.stride_row, q.stride_head, \
                                          fourbit_view(c), heads, n, n_rows, P, kv_rows, scale_log2, lse, mass_in, mass)
  if (dtype == NOVA_BF16) { if (c.dh == 64) GO(bf16_t, 64); else GO(bf16_t, 128); }
  else { if (c.dh == 64) GO(float, 64); else GO(float, 128); }
#undef GO
  return hipGetLastError();
}
