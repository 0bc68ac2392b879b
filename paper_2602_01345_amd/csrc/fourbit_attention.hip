// Attention over the 4-bit cache for many rows per key head (whole scales, prompts); which kernel takes which shape; the
// joining of key runs.
//
// As in attention_bf16.hip everything is computed transposed, a lane owning one row (query):
//   S^T = K Q^T    A operand = key rows from LDS, B operand = the row's channels, held in registers
//   O^T += V^T P^T A operand = value rows from LDS, read transposed, B operand = the probabilities as they come out of the
//                  softmax: the order of the keys in that product is free, so the values follow the scores' lane layout
// A workgroup is four waves of 32 rows.  Tiles of 64 keys are converted to bf16 (exactly: a level times a power of two) by
// all of its threads on the way from registers into LDS, once for the 128 rows; the codes of the tile after next are
// on the way meanwhile.  Two stages of LDS, two workgroups per CU (three with bf16 heads of 64), so that one wave's softmax runs
// next to another's MFMAs; a wave asks for priority while it issues MFMAs, or two waves of a SIMD fall into step and take turns
// at everything (385 us without, 340 with: 2458 queries of 2 images, 16 heads of 128, 8883 keys).  1.06 PFLOP/s there (a library
// product x W^T of 8192^3 1.60, with both operands by rows 1.36); with heads of 64 the softmax's vector instructions add to the
// MFMAs' time (1024 queries of 4 images, 32 heads, 4096 keys 160 us, 0.86 PFLOP/s).
// Probabilities of bf16 calls go into the second product as bf16: one rounding each (half a step, 2^-8 at most) instead of three
// MFMAs per operand.  The sum they are divided by is that of the fp32 ones.  One token, 424 keys: rms error 1.93e-3 of the
// result against 1.67e-3 for its own rounding to bf16 alone.
#include <algorithm>
#include <cfloat>

#include "fourbit_attention.h"

namespace {

constexpr int kWaves = 4, kTile = 64, kRows = kWaves * 32;

template <typename T, int DH>
__global__ __launch_bounds__(kWaves * 64, DH == 64 && sizeof(T) == 2 ? 3 : 2) void many_kernel(AttentionArgs<T> a) {
  constexpr int NP = kParts<T>;
  constexpr int GPR = DH / kGroup;
  constexpr int ROWB = DH * 2;
  constexpr int HALF = kTile * ROWB, STAGE = 2 * HALF;     // K rows, V rows
  constexpr int KS = DH / 16;                  // MFMAs along dh for a score block
  constexpr int DB = DH / 32;                  // 32-channel blocks of the output
  constexpr int CW = DH / 32;                  // dwords of codes per thread and tile: a quarter of a row of K and of V
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const bool whole = (int)blockIdx.x < a.n_whole;
  const int run = blockIdx.x - a.n_whole;
  const int split_i = whole ? 0 : run % a.nsplit;
  const int nparts = whole ? 1 : a.nsplit;
  int b, j, block;
  a.place(whole ? blockIdx.x : a.n_whole + run / a.nsplit, b, j, block);
  if (a.ranked) b = __builtin_amdgcn_readfirstlane(a.by_length(b));
  const int64_t bh = (int64_t)b * a.c.hk + j;
  const int row0 = block * kRows;
  const int rows = a.n * a.G, live = image_count(a.n_rows, b, a.n) * a.G, len = image_prior(a.kv_rows, b, a.P);
  const int ntiles = row0 < live ? (len + kTile - 1) / kTile : 0;
  const int per = (ntiles + nparts - 1) / nparts;
  const int t0 = split_i * per, t1 = min(ntiles, t0 + per);

  const uint8_t* codes[2] = {a.c.codes[0] + bh * a.c.cap * (DH / 2), a.c.codes[1] + bh * a.c.cap * (DH / 2)};
  const uint8_t* scales[2] = {a.c.scales[0] + bh * a.c.cap * GPR, a.c.scales[1] + bh * a.c.cap * GPR};

  // this thread's quarter (the wave's) of row lane of a tile, so that neighbouring lanes write one chunk of neighbouring rows; rows
  // past the last take the last one's place (their scores are set to -inf below, their values are those of a row that counts)
  const int frow = lane, fq = wave;
  uint32_t cw[2][CW], cb[2];
  auto request = [&](int t) {
    const uint32_t r = min(t * kTile + frow, len - 1);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      if constexpr (DH == 128) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(codes[w] + r * 64 + fq * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) cw[w][e] = x[e];
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(codes[w] + r * 32 + fq * 8);
        cw[w][0] = x[0];
        cw[w][1] = x[1];
      }
      cb[w] = scales[w][r * GPR + fq * GPR / 4];
    }
  };
  auto convert = [&](int stage) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float scale = fourbit_scale(cb[w]);
#pragma unroll
      for (int e = 0; e < CW; ++e)
        *reinterpret_cast<bf16x8*>(lds + stage * STAGE + w * HALF + swz<ROWB>(frow, fq * CW + e)) = fourbit_eight(cw[w][e], scale);
    }
  };
  // waits for this wave's LDS traffic only: requested codes stay on the way
  auto barrier = [] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  if (t0 < t1) request(t0);
  const int row = row0 + wave * 32 + col;
  bf16x8 qf[KS][NP];                                       // channels 16 t + 8 half .. + 7 of this lane's row
  {
    // past the last live row its copies: what lies in padding (NaN, say) is nobody's
    const T* qp = a.query(b, j, max(min(row, live - 1), 0)) + half * 8;
#pragma unroll
    for (int t = 0; t < KS; ++t) load_eight(qp + t * 16, qf[t]);
  }
  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  // probabilities are 2^(score - m_run); m_run is a reference, not necessarily the largest score (-inf: none yet)
  float m_run = -INFINITY, l_run = 0.f;
  const bool wave_live = row0 + wave * 32 < live;
  // this lane's places in a tile: its key's chunks, and for transposed reads of values the 8-byte piece lane % 4 of 16 channels of
  // key 4 half + (lane % 16) / 4 and of the one 8 behind it.  The swizzle repeats after 16 rows.
  int ka[KS], va[DB][2];
#pragma unroll
  for (int t = 0; t < KS; ++t) ka[t] = swz<ROWB>(col, t * 2 + half);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int x = 0; x < 2; ++x)
      va[d][x] = swz<ROWB>(4 * half + ((lane & 15) >> 2) + 8 * x, 4 * d + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8;

  if (t0 < t1) {
    convert(0);
    if (t0 + 1 < t1) request(t0 + 1);
    barrier();
  }
  for (int t = t0; t < t1; ++t) {
    const int stage = (t - t0) & 1;
    const char* sk = lds + stage * STAGE;
    const char* sv = sk + HALF;
    f32x16 s[2];
    if (wave_live) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 kf = *reinterpret_cast<const bf16x8*>(sk + kb * 32 * ROWB + ka[ks]);
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) s[kb] = mfma32(kf, qf[ks][p], s[kb]);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if (t + 1 < t1) {
      convert(stage ^ 1);
      if (t + 2 < t1) request(t + 2);
    }
    if (wave_live) {
      // ---- softmax: register r of block kb is key 64 t + 32 kb + 8 (r / 4) + 4 half + r % 4
      if ((t + 1) * kTile > len) {
        const float dead = a.scale_log2 < 0.f ? INFINITY : -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (t * kTile + kb * 32 + 8 * (r >> 2) + 4 * half + (r & 3) >= len) s[kb][r] = dead;
      }
      float e[2][16], psum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          e[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale_log2, -m_run));
          psum += e[kb][r];
        }
      if (__any(!(psum <= kBig))) {
        // some score lies far above the reference, or there is none yet: it moves to the largest score, and the sums with it
        float tmax = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, s[kb][r] * a.scale_log2);
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32, NOVA_WAVE));
        const float m_new = fmaxf(m_run, tmax);
        const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
        m_run = m_new;
        const float ref = m_new == -INFINITY ? 0.f : m_new;           // nothing but scores of -inf so far
        psum = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            e[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale_log2, -ref));
            psum += e[kb][r];
          }
      }
      l_run += psum;
      if constexpr (NP > 1 && DH == 128) {
        // in the scores' place: with three operands per row registers are short (2458 queries of 2 images, 16 heads of 128, 8883
        // keys 892 -> 811 us; with 64 channels 2-6 % slower, in bf16 2 %)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = e[kb][r];
      }
      __builtin_amdgcn_s_setprio(1);
      // ---- O^T += V^T P^T, 16 keys per MFMA: the lane's keys 16 u + 4 half .. + 3 and 8 behind them
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        bf16x8 pf[NP];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          bf16_t p[NP];
          split(NP > 1 && DH == 128 ? s[u >> 1][(u & 1) * 8 + i] : e[u >> 1][(u & 1) * 8 + i], p);
#pragma unroll
          for (int x = 0; x < NP; ++x) pf[x][i] = p[x];
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const char* at = sv + u * 16 * ROWB;
          const bf16x8 vf = join(read_transposed(at + va[d][0]), read_transposed(at + va[d][1]));
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) o[d] = mfma32(vf, pf[p], o[d]);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    barrier();
  }

  if (row >= rows) return;
  const float l = l_run + __shfl_xor(l_run, 32, NOVA_WAVE);
  if (nparts == 1) {
    const bool some = row < live && len > 0;
    const int64_t to = a.out_row(b, j, row);
    const float inv = some ? 1.0f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (some) v = f32x4{o[d][r4 * 4], o[d][r4 * 4 + 1], o[d][r4 * 4 + 2], o[d][r4 * 4 + 3]};
        store_four(a.out + to * DH + d * 32 + r4 * 8 + half * 4, v, inv);
      }
    if (a.lse && half == 0)
      a.lse[to] = some ? ((m_run == -INFINITY ? 0.f : m_run) + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  } else {
    const int64_t to = (int64_t)run * kRows + (row - row0);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<f32x4*>(a.part_o + to * DH + d * 32 + r4 * 8 + half * 4) =
            f32x4{o[d][r4 * 4], o[d][r4 * 4 + 1], o[d][r4 * 4 + 2], o[d][r4 * 4 + 3]};
    if (half == 0) {
      a.part_ml[to * 2] = m_run;
      a.part_ml[to * 2 + 1] = l;
    }
  }
}

// The runs of the cut items joined: out = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m).  A thread has four channels of
// one row and every SL-th run; with many runs per row (SL = 8: from five on) the threads of a row join through LDS.
template <typename T, int DH, int SL>
__global__ __launch_bounds__(256) void join_kernel(AttentionArgs<T> a, int block_rows, int used_rows) {
  constexpr int C4 = DH / 4, RPW = 256 / (C4 * SL);
  __shared__ f32x4 part_o[SL > 1 ? 256 : 1];
  __shared__ float part_m[SL > 1 ? 256 / C4 : 1], part_l[SL > 1 ? 256 / C4 : 1];
  const int tid = threadIdx.x, c4 = tid % C4, sl = tid / C4 % SL;
  const int64_t r = (int64_t)blockIdx.x * RPW + tid / (C4 * SL);
  const int ci = (int)(r / used_rows), rr = (int)(r - (int64_t)ci * used_rows);
  int b, j, block;
  a.place(min(a.n_whole + ci, a.items - 1), b, j, block);
  if (a.ranked) b = a.by_length(b);
  const int row = block * block_rows + rr;
  const int len = image_prior(a.kv_rows, b, a.P);
  const bool there = a.n_whole + ci < a.items && row < a.n * a.G;
  const bool some = there && row < image_count(a.n_rows, b, a.n) * a.G && len > 0;
  const int runs = !some ? 0 : a.run_tiles ? min(a.nsplit, ((len + kTile - 1) / kTile + a.run_tiles - 1) / a.run_tiles) : a.nsplit;
  const int64_t p0 = (int64_t)ci * a.nsplit * block_rows + rr;
  // a run without a finite score has reference -inf and sum 0 or NaN, and 0 or NaN in its results: it is added as it is
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int s = sl; s < runs; s += SL) {
    const int64_t p = p0 + (int64_t)s * block_rows;
    const float ms = a.part_ml[p * 2], ls = a.part_ml[p * 2 + 1];
    const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + p * DH + c4 * 4);
    const float mn = fmaxf(m, ms);
    const float w0 = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn), w1 = ms == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ms - mn);
    l = l * w0 + ls * w1;
    acc = acc * w0 + o * w1;
    m = mn;
  }
  if constexpr (SL > 1) {
    part_o[tid] = acc;
    if (c4 == 0) {
      part_m[tid / C4] = m;
      part_l[tid / C4] = l;
    }
    __syncthreads();
    if (sl > 0 || !there) return;
    const int g = tid / C4;
    for (int s = 1; s < SL; ++s) m = fmaxf(m, part_m[g + s]);
    l = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < SL; ++s) {
      const float w = part_m[g + s] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(part_m[g + s] - m);
      l = fmaf(w, part_l[g + s], l);
      acc += w * part_o[tid + s * C4];
    }
  }
  if (!there) return;
  const int64_t to = a.out_row(b, j, row);
  store_four(a.out + to * DH + c4 * 4, acc, some ? 1.0f / l : 0.f);
  if (a.lse && c4 == 0) a.lse[to] = some ? ((m == -INFINITY ? 0.f : m) + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// How a call is divided: mt > 0: blocks of 16 mt rows (fourbit_few.hip), else blocks of kRows; items below n_whole are one
// workgroup each, the others nsplit.
struct Plan {
  int mt, waves, block_rows, blocks, items, n_whole, nsplit, run_tiles, ranked;
  int64_t runs() const { return nsplit > 1 ? (int64_t)(items - n_whole) * nsplit : 0; }
};
constexpr int kCus = 256;
// Tiles up to which a block of 16 rows stays whole, eight waves of one workgroup with up to three each, and nothing is joined by a
// second launch.  One line for both types and head sizes, between the places where it would lie for each (us in one launch / in
// runs and joined, 32 key heads: bf16, 64 channels 8 tiles 4.9 / 6.2, 16 5.9 / 6.5, 24 6.9 / 6.8, 40 8.7 / 8.0; 128 channels 8
// 6.0 / 6.8, 16 7.6 / 7.3, 24 9.1 / 7.3; fp32, 128 channels 8 7.8 / 7.9, 24 12.5 / 8.4; 128 key heads: bf16 24 7.7 / 9.7 and 10.3 /
// 12.2, 40 9.8 / 11.5 and 13.7 / 15.3, fp32, 128 channels 24 13.8 / 16.3).  With 512 key heads the other side is one launch of
// four waves per block, and faster (128 channels 8 tiles 12.9 / 9.9, 24 24.3 / 22.2).
constexpr int kFewWhole = 24;
constexpr int kRanked = 32;          // most images that are ranked: every workgroup does it for itself, a step per image
Plan plan(const nova_fourbit_cache& c, int heads, int n, int kv_len, bool ragged) {
  const int rows = n * (heads / c.kv_heads), ntiles = (kv_len + kTile - 1) / kTile;
  Plan p = {};
  p.mt = rows <= 16 ? 1 : rows <= 32 ? 2 : 0;
  // More rows, but no more than two workgroups per CU in blocks of 32, and no wave with more than eight tiles: no tile waits for
  // the others, and nothing is joined afterwards (us in blocks of 128 / of 32; 16 heads of 64, one image: 205 queries, 629 keys
  // 9.1 + 3.9 / 7.9; 64, 155 6.4 / 5.9; two images, 30 heads, 128 queries, 2000 keys 13.3 + 6.5 / 13.9; of 128 channels: 256
  // queries, 521 keys 13.0 + 4.0 / 12.2; but 100 queries, 3100 keys 14.3 + 4.5 / 25.1).
  const int64_t blocks32 = (int64_t)c.B * c.kv_heads * ((rows + 31) / 32);
  const bool spread = p.mt == 0 && blocks32 <= 2 * kCus && ntiles <= 32;
  if (spread) p.mt = 2;
  p.waves = 4;
  p.block_rows = p.mt ? 16 * p.mt : kRows;
  p.blocks = (rows + p.block_rows - 1) / p.block_rows;
  p.items = c.B * c.kv_heads * p.blocks;
  p.n_whole = p.items;
  p.nsplit = 1;
  p.run_tiles = 0;
  if (p.mt) {
    const int want = std::min((12 * kCus + p.items - 1) / p.items, ntiles);      // waves per item: twelve per CU, a tile each
    p.run_tiles = ntiles;
    if (want > 4 && p.mt == 1 && ntiles <= kFewWhole) {
      p.waves = 8;
    } else if (want > 4 && !spread) {
      p.run_tiles = std::max((ntiles + want / 4 - 1) / (want / 4), 4);
      p.nsplit = (ntiles + p.run_tiles - 1) / p.run_tiles;
      if (p.nsplit > 1) p.n_whole = 0;
    }
    return p;
  }
  const int slots = 2 * kCus, rest = p.items % slots;
  // Images with lengths of their own: the longest first, so that short ones fill up the end; from two rounds of items on that is
  // enough and none is cut (us without / with, lengths falling, rising, mixed, equal: 8 images of 512 queries, 36 heads of 64, up
  // to 1728 keys 71, 69, 69, 82 / 65, 64, 62, 84; 24 of 300, 16 heads, 1200 keys 45, 45, 49, 57 / 42, 42, 41, 58; 6 of 1000, 16 heads
  // of 128, 3000 keys, cut as ever, 121, 122, 123, 150 / 123, 117, 116, 152).
  p.ranked = ragged && p.items > slots && c.B > 1 && c.B <= kRanked ? c.B : 0;
  if (rest == 0 || (p.ranked && p.items >= 2 * slots)) return p;
  // A few more items than CUs, and long ones: most CUs would have one, which is little to hide anything behind, and the others two
  // (us whole / in three: 264 items, 8000 keys 135 / 110 of 64 channels, 204 / 176 of 128; 320 136 / 117, 214 / 195; images of
  // different lengths 115 / 94, 181 / 149; but 400 140 / 143, 235 / 246, and 320 of 3000 keys 57 / 55, 87 / 93).
  const bool in_three = p.items > kCus && p.items <= kCus + kCus / 4 && ntiles >= 64;
  const int s = in_three ? 3 : std::min(slots / rest, ntiles / 4);
  if (s >= 2) {
    p.n_whole = p.items - rest;
    p.nsplit = s;
  }
  return p;
}

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

template <typename T>
hipError_t attend(hipStream_t st, const nova_fourbit_cache& c, int heads, int n, const nova_rows& q, const int32_t* n_rows, int P,
                  const int32_t* kv_rows, float scale_log2, void* out, float* lse, void* workspace) {
  const Plan p = plan(c, heads, n, P, kv_rows != nullptr);
  AttentionArgs<T> a = {};
  a.q = static_cast<const T*>(q.data);
  a.q_sb = q.stride_b; a.q_sr = q.stride_row; a.q_sh = q.stride_head;
  a.c = fourbit_view(c);
  a.heads = heads; a.G = heads / c.kv_heads; a.n = n; a.P = P;
  a.n_rows = n_rows; a.kv_rows = kv_rows;
  // Rows past the last have scores of -inf, which a scale of 0 would make NaN.  The smallest positive fp32 number (2^-149) in its
  // place leaves less than 2^-21 of any finite score: no two weights differ by more than that.
  a.scale_log2 = scale_log2 == 0.f ? FLT_TRUE_MIN : scale_log2;
  a.out = static_cast<T*>(out);
  a.lse = lse;
  a.blocks = p.blocks; a.items = p.items; a.dealt = p.items / (8 * p.blocks) * 8 * p.blocks;
  a.blocks_inv = div_inv(p.blocks); a.hk_inv = div_inv(c.kv_heads); a.G_inv = div_inv(a.G); a.nsplit_inv = div_inv(p.nsplit);
  a.n_whole = p.n_whole; a.nsplit = p.nsplit; a.run_tiles = p.run_tiles; a.ranked = p.ranked;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + up256((size_t)p.runs() * p.block_rows * c.dh * 4));
  const unsigned grid = (unsigned)(p.n_whole + p.runs());
  hipError_t e;
  if (p.mt) {
    e = launch_fourbit_few<T>(st, c.dh, p.mt, p.waves, grid, a);
  } else {
    if (c.dh == 64) many_kernel<T, 64><<<grid, kWaves * 64, 0, st>>>(a);
    else many_kernel<T, 128><<<grid, kWaves * 64, 0, st>>>(a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.nsplit == 1) return e;
  const int used = std::min(p.block_rows, n * a.G);            // rows of a block that there are, where it is the only one
  const int64_t rows = (int64_t)(p.items - p.n_whole) * used;
#define GO(DH, SL) join_kernel<T, DH, SL><<<(unsigned)((rows * (DH / 4 * SL) + 255) / 256), 256, 0, st>>>(a, p.block_rows, used)
  if (c.dh == 64) { if (p.nsplit > 4) GO(64, 8); else GO(64, 1); }
  else { if (p.nsplit > 4) GO(128, 8); else GO(128, 1); }
#undef GO
  return hipGetLastError();
}

}  // namespace

size_t fourbit_attention_workspace_bytes(const nova_fourbit_cache& c, int heads, int n, int kv_len) {
  const Plan p = plan(c, heads, n, kv_len, false);           // of the two the one that asks for more
  if (p.nsplit == 1) return 0;
  const size_t rows = (size_t)p.runs() * p.block_rows;
  return up256(rows * c.dh * 4) + up256(rows * 8);
}

hipError_t launch_fourbit_attention(const nova_ctx*, hipStream_t st, int dtype, const nova_fourbit_cache& c, int heads, int n,
                                    const nova_rows& q, const int32_t* n_rows, int P, const int32_t* kv_rows, float scale_log2,
                                    void* out, float* lse, void* workspace) {
  if (dtype == NOVA_BF16) return attend<bf16_t>(st, c, heads, n, q, n_rows, P, kv_rows, scale_log2, out, lse, workspace);
  return attend<float>(st, c, heads, n, q, n_rows, P, kv_rows, scale_log2, out, lse, workspace);
}
