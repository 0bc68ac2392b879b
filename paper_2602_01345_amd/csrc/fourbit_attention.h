// What the attention kernels over the 4-bit cache share: arguments, the rows of a key head, operands, the joining of key runs.
#pragma once
#include "fourbit.h"

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kBig = 1024.0f;          // sum of a lane's probabilities of one tile above which the softmax reference moves

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// An operand of the caller's type as bf16 numbers whose sum it is.  Cached values are bf16 as they are, so a bf16 operand
// takes one MFMA and an fp32 one three: 3 x 8 bits of significand are all 24 of it.  Each part is the leading bits of what is
// left, cut off and not rounded: the largest fp32 numbers round to an infinity.
template <typename T> constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

__device__ __forceinline__ bf16_t leading(float x) { return __builtin_bit_cast(bf16_t, (uint16_t)(__float_as_uint(x) >> 16)); }
__device__ __forceinline__ void split(float x, bf16_t (&p)[1]) { p[0] = (bf16_t)x; }       // rounded: why, at many_kernel's head
__device__ __forceinline__ void split(float x, bf16_t (&p)[3]) {
  p[0] = leading(x);
  const float r = x - (float)p[0];
  p[1] = leading(r);
  p[2] = leading(r - (float)p[1]);
}
template <typename T>
__device__ __forceinline__ void load_eight(const T* src, bf16x8 (&f)[kParts<T>]) {
  if constexpr (kParts<T> == 1) {
    f[0] = *reinterpret_cast<const bf16x8*>(src);
  } else {
    const f32x4 a = *reinterpret_cast<const f32x4*>(src), b = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bf16_t p[3];
      split(e < 4 ? a[e & 3] : b[e & 3], p);
#pragma unroll
      for (int i = 0; i < 3; ++i) f[i][e] = p[i];
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_four(T* dst, f32x4 v, float f) {
  if constexpr (kParts<T> == 1) {
    *reinterpret_cast<bf16x4*>(dst) = bf16x4{(bf16_t)(v[0] * f), (bf16_t)(v[1] * f), (bf16_t)(v[2] * f), (bf16_t)(v[3] * f)};
  } else {
    *reinterpret_cast<f32x4*>(dst) = v * f;
  }
}

// Byte offset of 16-byte chunk c of row r in an LDS tile of rows of ROWB bytes: chunk c lies in place c ^ f(r).  f is a sum of
// r's bits chosen so that none of these meets a bank twice, whether 128 or 256 bytes are served at a time: one chunk of 8 or 16
// rows running (operands read along the rows, rows written); two neighbouring chunks of rows 4 i .. 4 i + 3 and of the 4 behind
// them, four chunks of 4 rows (transposing reads by 16 or 32 lanes).  The top bit of c goes into the lowest place bit, for eight
// lanes that write a chunk each of the groups of two or four rows.  With the usual f(r) = r mod 16 transposing reads take
// twice the time: 57 % of the LDS cycles with many rows of 128 channels were conflicts.  f repeats after 16 rows.
template <int ROWB>
__device__ __forceinline__ int swz(int r, int c) {
  const int f = 2 * (r & 3) ^ 3 * ((r >> 2) & 1) ^ (ROWB == 256 ? 8 * ((r ^ (r >> 3)) & 1) ^ c >> 3 : ((r >> 3) & 1) ^ c >> 2);
  return r * ROWB + ((c ^ f) << 4);
}

// Four rows by sixteen channels of an LDS tile, transposed on the way: sixteen neighbouring lanes name four rows' 8-byte pieces
// (lane i: row i / 4, piece i % 4) and get lane i's channel of the four rows.
typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4_t;
__device__ __forceinline__ bf16x4 read_transposed(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t)p);
}
__device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b) { return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }

// The queries that read one key head are its rows: query s of head j G + g is row s G + g (G heads share a key head).
template <typename T>
struct AttentionArgs {
  const T* q;
  int64_t q_sb, q_sr, q_sh;
  FourBitView c;
  int heads, G, n, P;
  const int32_t *n_rows, *kv_rows;
  float scale_log2;
  T* out;
  float* lse;
  // Pieces: item i (a block of rows of one key head) is one workgroup below n_whole and nsplit of them, runs of key tiles, from
  // there on; the latter leave sums against their own reference to be joined: part_o [run][row of the block][dh] and part_ml
  // [run][row of the block] (reference in log2 units, sum)
  int blocks, items;     // of rows per key head; in all
  int dealt;             // items of key heads that come in eights
  uint32_t blocks_inv, hk_inv, G_inv, nsplit_inv;
  int n_whole, nsplit;
  int run_tiles;         // tiles per run; 0: an item's tiles divided by nsplit
  int ranked;            // > 0: items come by falling length of their images, this many (64 at most)
  float* part_o;
  float* part_ml;

  // Key head (of all images') and block of rows of an item.  Workgroups are dealt to the 8 XCDs in turn: the blocks of one key
  // head go to one XCD and share its L2, eight key heads running to the eight XCDs, so that images of different lengths load
  // them alike.  What is left of the key heads goes as it comes.
  __device__ __forceinline__ void place(int item, int& b, int& j, int& block) const {
    int bh;
    if (item < dealt) {
      bh = div_by(item >> 3, blocks, blocks_inv, block) * 8 + (item & 7);
    } else {
      bh = div_by(item, blocks, blocks_inv, block);
    }
    b = div_by(bh, c.hk, hk_inv, j);
  }
  // The image of rank b by length (of two alike the earlier one first), for all lanes of a wave at once.
  __device__ __forceinline__ int by_length(int b) const {
    const int lane = threadIdx.x & 63, mine = lane < ranked ? image_prior(kv_rows, lane, P) : 0;
    int rank = lane < ranked ? 0 : lane;
    for (int i = 0; i < ranked; ++i) {
      const int other = __builtin_amdgcn_readlane(mine, i);
      if (lane < ranked) rank += other > mine || (other == mine && i < lane);
    }
    return __shfl(__builtin_amdgcn_ds_permute(rank * 4, lane), b, NOVA_WAVE);
  }
  __device__ __forceinline__ const T* query(int b, int j, int row) const {
    int g;
    const int s = div_by(row, G, G_inv, g);
    return q + b * q_sb + s * q_sr + (j * G + g) * q_sh;
  }
  __device__ __forceinline__ int64_t out_row(int b, int j, int row) const {
    int g;
    const int s = div_by(row, G, G_inv, g);
    return ((int64_t)b * n + s) * heads + j * G + g;
  }
};

// fourbit_few.hip: blocks of 16 mt rows, 4 or 8 waves that each take key tiles of their own (8: mt 1)
template <typename T>
hipError_t launch_fourbit_few(hipStream_t st, int dh, int mt, int waves, unsigned grid, const AttentionArgs<T>& a);
