// The key/value cache in 4 bits (format: include/nova.h), for its kernels and for the host side that launches them.
#pragma once
#include "common.h"
#include "nova_internal.h"

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kGroup = 32;               // channels that share a scale byte

// Two codes, byte SEL of four, times 2^(scale's exponent): exact in bf16, NaN where the scale byte is 255 (the conversion
// reads nothing of the scale but its exponent).
template <int SEL>
__device__ __forceinline__ bf16x2 fourbit_pair(uint32_t codes, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL);
}
// Eight consecutive channels of a row: the operand of one MFMA.
__device__ __forceinline__ bf16x8 fourbit_eight(uint32_t codes, float scale) {
  const bf16x2 a = fourbit_pair<0>(codes, scale), b = fourbit_pair<1>(codes, scale), c = fourbit_pair<2>(codes, scale),
               d = fourbit_pair<3>(codes, scale);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float fourbit_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Rows of one head as a buffer of `bytes`: loads from there on give zeros, codes and scales that read as zero.
__device__ __forceinline__ auto head_buffer(const uint8_t* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, bytes, 0x00020000);
}

// A cache as the kernels take it.  Rows of K and of V lie alike: row j of head bh has its codes at (bh * cap + j) * dh / 2.
struct FourBitView {
  const uint8_t* codes[2];               // K, V
  const uint8_t* scales[2];
  int hk, cap;
};
inline FourBitView fourbit_view(const nova_fourbit_cache& c) {
  FourBitView v = {};
  v.codes[0] = static_cast<const uint8_t*>(c.k_codes);
  v.codes[1] = static_cast<const uint8_t*>(c.v_codes);
  v.scales[0] = static_cast<const uint8_t*>(c.k_scales);
  v.scales[1] = static_cast<const uint8_t*>(c.v_scales);
  v.hk = c.kv_heads;
  v.cap = c.capacity;
  return v;
}
