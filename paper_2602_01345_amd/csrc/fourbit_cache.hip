// Rows into and out of the key/value cache in 4 bits: quantise and append, read back, evict.  All three are copies with a
// conversion on the way, bound by HBM (or, for a token per image, by the launch).
//
// A workgroup has one image, one head, K or V, and kBlockRows rows.  Where the caller's channels lie side by side (and
// everything is a multiple of 16 bytes) a thread takes eight channels, four neighbours a group: loads and stores of whole
// lines on both sides.  Otherwise (values key-minor, say) a thread takes a group of one row and neighbouring lanes neighbouring
// rows, so that the caller's side is read or written along the rows.
//
// Measured: 6425 rows of 2 images, 16 heads of 128 in bf16 in 34.6 us (133 MB, 3.8 TB/s; the values key-minor with an odd pitch) and
// out again in 21.4 (6.2 TB/s); a row of 8 images in 3; 8192 of 32768 rows of 4 images, 8 heads of 128, moved in 25 us (71 MB: lines of
// 128 bytes are fetched for rows of 64).
#include <algorithm>

#include "fourbit.h"

namespace {

constexpr int kThreads = 256;
template <int DH> constexpr int kBlockRows = kThreads * kGroup / DH;     // a thread per group: 64 rows of 128, 128 of 64

struct RowsView {                        // caller's rows of K and of V (data may be null: that half is skipped)
  void* data[2];
  int64_t sb[2], sr[2], sh[2], sc[2];
  int vec[2];                            // channels side by side, 16-byte aligned
};

// largest of four neighbouring lanes
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, dpp_or<0xB1, 0xF>(v, 0.0f));
  return fmaxf(v, dpp_or<0x4E, 0xF>(v, 0.0f));
}
// Scale byte of a group with largest magnitude a = m 2^t, 1 <= m < 2: the smallest e with a <= 6 2^e is t - 2 up to m = 1.5 and
// t - 1 from there on.
__device__ __forceinline__ uint32_t scale_byte(float a) {
  const uint32_t bits = __float_as_uint(a);
  const int e = (int)(bits >> 23) - 127 - 2 + ((bits & 0x7FFFFFu) > 0x400000u);
  return (uint32_t)(min(max(e, -124), 125) + 127);
}
// Codes of eight channels: the conversion rounds to the nearest level, of two to the even one, and saturates.
__device__ __forceinline__ uint32_t encode_eight(const float* v, float scale) {
  uint32_t w = 0u;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void append_kernel(RowsView in, FourBitView c, int n, int P,
                                                          const int32_t* __restrict__ n_rows, const int32_t* __restrict__ kv_rows,
                                                          int32_t* __restrict__ kv_next) {
  constexpr int GPR = DH / kGroup, LPR = DH / 8, ROWS = kBlockRows<DH>;
  const int b = blockIdx.z, h = blockIdx.y >> 1, which = blockIdx.y & 1, tid = threadIdx.x;
  const int count = image_count(n_rows, b, n), prior = image_prior(kv_rows, b, P);
  if (kv_next && blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) kv_next[b] = prior + count;
  const int row0 = blockIdx.x * ROWS;
  const T* x = static_cast<const T*>(in.data[which]) + b * in.sb[which] + h * in.sh[which];
  const int64_t base = ((int64_t)b * c.hk + h) * c.cap + prior;
  uint8_t* codes = const_cast<uint8_t*>(c.codes[which]) + base * (DH / 2);
  uint8_t* scales = const_cast<uint8_t*>(c.scales[which]) + base * GPR;
  if (in.vec[which]) {
    constexpr int IT = ROWS * LPR / kThreads;
    float v[IT][8];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int s = row0 + i * (kThreads / LPR) + tid / LPR;
      if (s >= count) continue;
      const T* p = x + s * in.sr[which] + tid % LPR * 8;
      if constexpr (sizeof(T) == 2) {
        const bf16x8 w = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = (float)w[e];
      } else {
        const f32x4 w0 = *reinterpret_cast<const f32x4*>(p), w1 = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[i][e] = w0[e]; v[i][4 + e] = w1[e]; }
      }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int s = row0 + i * (kThreads / LPR) + tid / LPR;
      if (s >= count) continue;                            // all lanes of a group, or none
      float a = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) a = fmaxf(a, fabsf(v[i][e]) < INFINITY ? fabsf(v[i][e]) : INFINITY);     // NaN as infinity
      a = quad_max(a);
      const bool bad = a == INFINITY;
      const uint32_t byte = scale_byte(a);
      *reinterpret_cast<uint32_t*>(codes + s * (DH / 2) + tid % LPR * 4) = bad ? 0u : encode_eight(v[i], fourbit_scale(byte));
      if (tid % 4 == 0) scales[s * GPR + tid % LPR / 4] = bad ? 255 : (uint8_t)byte;
    }
    return;
  }
  const int s = row0 + tid % ROWS, g = tid / ROWS;
  if (s >= count) return;
  x += s * in.sr[which] + g * kGroup * in.sc[which];
  float v[kGroup], a = 0.f;
#pragma unroll
  for (int e = 0; e < kGroup; ++e) v[e] = (float)x[e * in.sc[which]];
#pragma unroll
  for (int e = 0; e < kGroup; ++e) a = fmaxf(a, fabsf(v[e]) < INFINITY ? fabsf(v[e]) : INFINITY);
  const bool bad = a == INFINITY;
  const uint32_t byte = scale_byte(a);
  u32x4 w = {0u, 0u, 0u, 0u};
  if (!bad)
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = encode_eight(v + 8 * e, fourbit_scale(byte));
  *reinterpret_cast<u32x4*>(codes + s * (DH / 2) + g * 16) = w;
  scales[s * GPR + g] = bad ? 255 : (uint8_t)byte;
}

template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void unpack_kernel(RowsView out, FourBitView c, int n, int first,
                                                          const int32_t* __restrict__ first_rows,
                                                          const int32_t* __restrict__ n_rows) {
  constexpr int GPR = DH / kGroup, LPR = DH / 8, ROWS = kBlockRows<DH>;
  const int b = blockIdx.z, h = blockIdx.y >> 1, which = blockIdx.y & 1, tid = threadIdx.x;
  if (!out.data[which]) return;
  const int count = image_count(n_rows, b, n), row0 = blockIdx.x * ROWS;
  T* x = static_cast<T*>(out.data[which]) + b * out.sb[which] + h * out.sh[which];
  const int64_t base = ((int64_t)b * c.hk + h) * c.cap + image_prior(first_rows, b, first);
  const uint8_t* codes = c.codes[which] + base * (DH / 2);
  const uint8_t* scales = c.scales[which] + base * GPR;
  if (out.vec[which]) {
    constexpr int IT = ROWS * LPR / kThreads;
    uint32_t w[IT], byte[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int s = row0 + i * (kThreads / LPR) + tid / LPR;
      w[i] = 0u;
      byte[i] = 127u;
      if (s < count) {
        w[i] = *reinterpret_cast<const uint32_t*>(codes + s * (DH / 2) + tid % LPR * 4);
        byte[i] = scales[s * GPR + tid % LPR / 4];
      }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int s = row0 + i * (kThreads / LPR) + tid / LPR;
      if (s >= n) continue;
      const bf16x8 v = fourbit_eight(w[i], fourbit_scale(byte[i]));
      T* p = x + s * out.sr[which] + tid % LPR * 8;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<bf16x8*>(p) = v;
      } else {
        *reinterpret_cast<f32x4*>(p) = f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{(float)v[4], (float)v[5], (float)v[6], (float)v[7]};
      }
    }
    return;
  }
  const int s = row0 + tid % ROWS, g = tid / ROWS;
  if (s >= n) return;
  u32x4 w = {0u, 0u, 0u, 0u};
  uint32_t byte = 127u;
  if (s < count) {
    w = *reinterpret_cast<const u32x4*>(codes + s * (DH / 2) + g * 16);
    byte = scales[s * GPR + g];
  }
  x += s * out.sr[which] + g * kGroup * out.sc[which];
#pragma unroll
  for (int e4 = 0; e4 < 4; ++e4) {
    const bf16x8 v = fourbit_eight(w[e4], fourbit_scale(byte));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[(e4 * 8 + e) * out.sc[which]] = (T)(float)v[e];
  }
}

template <int DH>
__global__ __launch_bounds__(kThreads) void evict_kernel(FourBitView src, FourBitView dst, int k, int slots, int P,
                                                         const int32_t* __restrict__ idx, const int32_t* __restrict__ k_rows,
                                                         const int32_t* __restrict__ kv_rows, int32_t* __restrict__ kv_next,
                                                         const float* __restrict__ mass_src, float* __restrict__ mass_dst) {
  constexpr int GPR = DH / kGroup, ROWS = kBlockRows<DH>;
  const int b = blockIdx.z, h = blockIdx.y >> 1, which = blockIdx.y & 1, tid = threadIdx.x;
  const int s = blockIdx.x * ROWS + tid / GPR, g = tid % GPR;
  const int len = image_prior(kv_rows, b, P), m = min(image_count(k_rows, b, k), len);
  if (kv_next && blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) kv_next[b] = m;
  const bool mass = mass_src && blockIdx.y == 0 && g == 0;
  if (s >= m) {
    if (mass && s < slots) mass_dst[(int64_t)b * dst.cap + s] = -1.0f;
    return;
  }
  const int j = idx[(int64_t)b * k + s];
  const bool have = j >= 0 && j < len;
  const int64_t bh = (int64_t)b * src.hk + h, to = (bh * dst.cap + s) * GPR + g, from = (bh * src.cap + j) * GPR + g;
  u32x4 w = {0u, 0u, 0u, 0u};
  uint8_t byte = 127;
  if (have) {
    w = *reinterpret_cast<const u32x4*>(src.codes[which] + from * 16);
    byte = src.scales[which][from];
  }
  *reinterpret_cast<u32x4*>(const_cast<uint8_t*>(dst.codes[which]) + to * 16) = w;
  const_cast<uint8_t*>(dst.scales[which])[to] = byte;
  if (mass) mass_dst[(int64_t)b * dst.cap + s] = have ? mass_src[(int64_t)b * src.cap + j] : 0.0f;
}

RowsView rows_view(int dtype, const nova_rows* k, const nova_rows* v) {
  RowsView r = {};
  const nova_rows* p[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    if (!p[i]) continue;
    r.data[i] = p[i]->data;
    r.sb[i] = p[i]->stride_b; r.sr[i] = p[i]->stride_row; r.sh[i] = p[i]->stride_head; r.sc[i] = p[i]->stride_channel;
    const int64_t per = dtype == NOVA_BF16 ? 8 : 4;                          // elements in 16 bytes
    r.vec[i] = r.sc[i] == 1 && (reinterpret_cast<uintptr_t>(r.data[i]) & 15) == 0 && r.sb[i] % per == 0 && r.sr[i] % per == 0 &&
               r.sh[i] % per == 0;
  }
  return r;
}

}  // namespace

hipError_t launch_fourbit_append(hipStream_t st, int dtype, const nova_fourbit_cache& c, int n, const nova_rows* k,
                                 const nova_rows* v, const int32_t* n_rows, int P, const int32_t* kv_rows, int32_t* kv_next) {
  if (n == 0 && !kv_next) return hipSuccess;
  const RowsView in = rows_view(dtype, k, v);
  const FourBitView to = fourbit_view(c);
#define GO(T, DH)                                                                                                                  \
  append_kernel<T, DH><<<dim3((std::max(n, 1) + kBlockRows<DH> - 1) / kBlockRows<DH>, 2 * c.kv_heads, c.B), kThreads, 0, st>>>(    \
      in, to, n, P, n_rows, kv_rows, kv_next)
  if (dtype == NOVA_BF16) { if (c.dh == 64) GO(bf16_t, 64); else GO(bf16_t, 128); }
  else { if (c.dh == 64) GO(float, 64); else GO(float, 128); }
#undef GO
  return hipGetLastError();
}

hipError_t launch_fourbit_unpack(hipStream_t st, int dtype, const nova_fourbit_cache& c, int first, int n,
                                 const int32_t* first_rows, const int32_t* n_rows, const nova_rows* k, const nova_rows* v) {
  const RowsView out = rows_view(dtype, k, v);
  const FourBitView from = fourbit_view(c);
#define GO(T, DH)                                                                                                                  \
  unpack_kernel<T, DH><<<dim3((n + kBlockRows<DH> - 1) / kBlockRows<DH>, 2 * c.kv_heads, c.B), kThreads, 0, st>>>(                 \
      out, from, n, first, first_rows, n_rows)
  if (dtype == NOVA_BF16) { if (c.dh == 64) GO(bf16_t, 64); else GO(bf16_t, 128); }
  else { if (c.dh == 64) GO(float, 64); else GO(float, 128); }
#undef GO
  return hipGetLastError();
}

hipError_t launch_fourbit_evict(hipStream_t st, const nova_fourbit_cache& src, const nova_fourbit_cache& dst, int k,
                                const int32_t* idx, const int32_t* k_rows, int P, const int32_t* kv_rows, int32_t* kv_next,
                                const float* mass_src, float* mass_dst) {
  const int slots = mass_src ? dst.capacity : k;               // k <= capacity
  if (slots == 0 && !kv_next) return hipSuccess;
#define GO(DH)                                                                                                                     \
  evict_kernel<DH><<<dim3((std::max(slots, 1) + kBlockRows<DH> - 1) / kBlockRows<DH>, 2 * src.kv_heads, src.B), kThreads, 0, st>>>(\
      fourbit_view(src), fourbit_view(dst), k, slots, P, idx, k_rows, kv_rows, kv_next, mass_src, mass_dst)
  if (src.dh == 64) GO(64); else GO(128);
#undef GO
  return hipGetLastError();
}

hipError_t launch_fourbit_block_attention(const nova_ctx* ctx, hipStream_t st, const nova_block_shape& s, const RowCounts& rc,
                                          const FourBitBlock& fb, const void* q, float scale_log2, void* out) {
  const int64_t dh = s.C / s.heads, rows = (int64_t)s.heads * fb.pitch * dh;
  const nova_rows k = {fb.k_new, rows, dh, fb.pitch * dh, 1}, v = {fb.v_new, rows, 1, fb.pitch * dh, fb.pitch};
  const nova_rows qv = {const_cast<void*>(q), (int64_t)s.k * s.C, s.C, dh, 1};
  const int total = s.kv_len + s.k;
  hipError_t e = launch_fourbit_append(st, s.dtype, fb.cache, s.k, &k, &v, rc.k_rows, s.kv_len, rc.kv_rows, fb.kv_after);
  if (e != hipSuccess) return e;
  const int32_t* after = rc.k_rows || rc.kv_rows ? fb.kv_after : nullptr;     // every image has `total` rows otherwise
  e = launch_fourbit_attention(ctx, st, s.dtype, fb.cache, s.heads, s.k, qv, rc.k_rows, total, after, scale_log2, out,
                               fb.mass ? fb.lse : nullptr, fb.work);
  if (e != hipSuccess || !fb.mass) return e;
  return launch_fourbit_mass(ctx, st, s.dtype, fb.cache, s.heads, s.k, qv, rc.k_rows, total, after, scale_log2, fb.lse, fb.mass_in,
                             fb.mass, fb.work);
}
