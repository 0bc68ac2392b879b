// Rows into and out of the key/value cache in 4 bits: quantise and append, read back, evict.  All three are copies with a
// conversion on the way, bound by HBM (or, for a token per image, by the launch).
#include <algorithm>

#include "fourbit.h"

namespace {

constexpr int kThreads = 256;

struct RowsView {                        // caller's rows of K and of V (data may be null: that half is skipped)
  void* data[2];
  int64_t sb[2], sr[2], sh[2], sc[2];
};

// One thread per group of 32 channels; groups of a row are neighbours.
template <typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(RowsView in, FourBitView c, int dh, int B, int n, int P,
                                                          const int32_t* __restrict__ n_rows, const int32_t* __restrict__ kv_rows,
                                                          int32_t* __restrict__ kv_next) {
  const int gpr = dh / kGroup, which = blockIdx.y;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (kv_next && which == 0 && i < B) kv_next[i] = image_prior(kv_rows, (int)i, P) + image_count(n_rows, (int)i, n);
  if (i >= (int64_t)B * n * c.hk * gpr) return;
  const int g = (int)(i % gpr);
  const int64_t r = i / gpr;
  const int h = (int)(r % c.hk), s = (int)(r / c.hk % n), b = (int)(r / c.hk / n);
  if (s >= image_count(n_rows, b, n)) return;
  const T* x = static_cast<const T*>(in.data[which]) + b * in.sb[which] + s * in.sr[which] + h * in.sh[which] +
               g * kGroup * in.sc[which];
  float v[kGroup], a = 0.f;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < kGroup; ++e) {
    v[e] = (float)x[e * in.sc[which]];
    bad |= !(fabsf(v[e]) < INFINITY);
    a = fmaxf(a, fabsf(v[e]));
  }
  // a = m 2^t with 1 <= m < 2: 2^e >= a / 6 from e = t - 2 on if m <= 1.5, else from t - 1 on
  const uint32_t bits = __float_as_uint(a);
  int e = (int)(bits >> 23) - 127 - 2 + ((bits & 0x7FFFFFu) > 0x400000u);
  e = min(max(e, -124), 125);
  const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  if (!bad) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], v[8 * j + 0], v[8 * j + 1], scale, 0);
      w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], v[8 * j + 2], v[8 * j + 3], scale, 1);
      w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], v[8 * j + 4], v[8 * j + 5], scale, 2);
      w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], v[8 * j + 6], v[8 * j + 7], scale, 3);
    }
  }
  const int64_t row = ((int64_t)b * c.hk + h) * c.cap + image_prior(kv_rows, b, P) + s;
  *reinterpret_cast<u32x4*>(const_cast<uint8_t*>(c.codes[which]) + (row * gpr + g) * 16) = u32x4{w[0], w[1], w[2], w[3]};
  const_cast<uint8_t*>(c.scales[which])[row * gpr + g] = bad ? 255 : (uint8_t)(e + 127);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void unpack_kernel(RowsView out, FourBitView c, int dh, int B, int n, int first,
                                                          const int32_t* __restrict__ first_rows,
                                                          const int32_t* __restrict__ n_rows) {
  const int gpr = dh / kGroup, which = blockIdx.y;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (!out.data[which] || i >= (int64_t)B * n * c.hk * gpr) return;
  const int g = (int)(i % gpr);
  const int64_t r = i / gpr;
  const int h = (int)(r % c.hk), s = (int)(r / c.hk % n), b = (int)(r / c.hk / n);
  T* x = static_cast<T*>(out.data[which]) + b * out.sb[which] + s * out.sr[which] + h * out.sh[which] +
         g * kGroup * out.sc[which];
  u32x4 w = {0u, 0u, 0u, 0u};
  float scale = 1.0f;
  if (s < image_count(n_rows, b, n)) {
    const int64_t row = ((int64_t)b * c.hk + h) * c.cap + image_prior(first_rows, b, first) + s;
    w = *reinterpret_cast<const u32x4*>(c.codes[which] + (row * gpr + g) * 16);
    scale = fourbit_scale(c.scales[which][row * gpr + g]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x8 v = fourbit_eight(w[j], scale);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[(j * 8 + e) * out.sc[which]] = (T)(float)v[e];
  }
}

__global__ __launch_bounds__(kThreads) void evict_kernel(FourBitView src, FourBitView dst, int gpr, int B, int k, int slots, int P,
                                                         const int32_t* __restrict__ idx, const int32_t* __restrict__ k_rows,
                                                         const int32_t* __restrict__ kv_rows, int32_t* __restrict__ kv_next,
                                                         const float* __restrict__ mass_src, float* __restrict__ mass_dst) {
  const int b = blockIdx.z, h = blockIdx.y >> 1, which = blockIdx.y & 1;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int g = (int)(i % gpr);
  const int64_t s = i / gpr;
  if (s >= slots) return;
  const int len = image_prior(kv_rows, b, P), m = min(image_count(k_rows, b, k), len);
  if (kv_next && blockIdx.y == 0 && i == 0) kv_next[b] = m;
  const bool mass = mass_src && blockIdx.y == 0 && g == 0;
  if (s >= m) {
    if (mass && s < dst.cap) mass_dst[(int64_t)b * dst.cap + s] = -1.0f;
    return;
  }
  const int j = idx[(int64_t)b * k + s];
  const bool have = j >= 0 && j < len;
  const int64_t bh = (int64_t)b * src.hk + h, to = (bh * dst.cap + s) * gpr + g, from = (bh * src.cap + j) * gpr + g;
  *reinterpret_cast<u32x4*>(const_cast<uint8_t*>(dst.codes[which]) + to * 16) =
      have ? *reinterpret_cast<const u32x4*>(src.codes[which] + from * 16) : u32x4{0u, 0u, 0u, 0u};
  const_cast<uint8_t*>(dst.scales[which])[to] = have ? src.scales[which][from] : 127;
  if (mass) mass_dst[(int64_t)b * dst.cap + s] = have ? mass_src[(int64_t)b * src.cap + j] : 0.0f;
}

RowsView rows_view(const nova_rows* k, const nova_rows* v) {
  RowsView r = {};
  const nova_rows* p[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    if (!p[i]) continue;
    r.data[i] = p[i]->data;
    r.sb[i] = p[i]->stride_b; r.sr[i] = p[i]->stride_row; r.sh[i] = p[i]->stride_head; r.sc[i] = p[i]->stride_channel;
  }
  return r;
}

}  // namespace

hipError_t launch_fourbit_append(hipStream_t st, int dtype, const nova_fourbit_cache& c, int n, const nova_rows* k,
                                 const nova_rows* v, const int32_t* n_rows, int P, const int32_t* kv_rows, int32_t* kv_next) {
  const int64_t items = std::max((int64_t)c.B * n * c.kv_heads * (c.dh / kGroup), kv_next ? (int64_t)c.B : 0);
  if (items == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + kThreads - 1) / kThreads), 2);
  if (dtype == NOVA_BF16)
    append_kernel<bf16_t><<<grid, kThreads, 0, st>>>(rows_view(k, v), fourbit_view(c), c.dh, c.B, n, P, n_rows, kv_rows, kv_next);
  else
    append_kernel<float><<<grid, kThreads, 0, st>>>(rows_view(k, v), fourbit_view(c), c.dh, c.B, n, P, n_rows, kv_rows, kv_next);
  return hipGetLastError();
}

hipError_t launch_fourbit_unpack(hipStream_t st, int dtype, const nova_fourbit_cache& c, int first, int n,
                                 const int32_t* first_rows, const int32_t* n_rows, const nova_rows* k, const nova_rows* v) {
  const int64_t items = (int64_t)c.B * n * c.kv_heads * (c.dh / kGroup);
  const dim3 grid((unsigned)((items + kThreads - 1) / kThreads), 2);
  if (dtype == NOVA_BF16)
    unpack_kernel<bf16_t><<<grid, kThreads, 0, st>>>(rows_view(k, v), fourbit_view(c), c.dh, c.B, n, first, first_rows, n_rows);
  else
    unpack_kernel<float><<<grid, kThreads, 0, st>>>(rows_view(k, v), fourbit_view(c), c.dh, c.B, n, first, first_rows, n_rows);
  return hipGetLastError();
}

hipError_t launch_fourbit_evict(hipStream_t st, const nova_fourbit_cache& src, const nova_fourbit_cache& dst, int k,
                                const int32_t* idx, const int32_t* k_rows, int P, const int32_t* kv_rows, int32_t* kv_next,
                                const float* mass_src, float* mass_dst) {
  const int gpr = src.dh / kGroup, slots = std::max({k, mass_src ? dst.capacity : 0, kv_next ? 1 : 0});
  if (slots == 0) return hipSuccess;
  const dim3 grid((unsigned)(((int64_t)slots * gpr + kThreads - 1) / kThreads), 2 * src.kv_heads, src.B);
  evict_kernel<<<grid, kThreads, 0, st>>>(fourbit_view(src), fourbit_view(dst), gpr, src.B, k, slots, P, idx, k_rows, kv_rows, kv_next, mass_src,
                                          mass_dst);
  return hipGetLastError();
}
