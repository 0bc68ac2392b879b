// Attention over the 4-bit cache for few rows per key head (a row: a query of one of the heads that share it): single tokens,
// a handful of queries, small scales.  What bounds it is reading the cache once.
//
// A workgroup is four or eight waves and one block of up to 16 MT rows; tiles of 64 keys are dealt to the waves, which share nothing
// until their results are joined at the end, so no tile waits at a barrier.  Everything is computed transposed, a lane owning
// one row of 16 (col) and the four lane groups (grp) parts of the keys:
//   S^T = K Q^T    16 keys x 16 rows per MFMA.  The order of the channels in that product is free, so a lane takes them as they
//                  lie in the cache: dh / 4 neighbouring channels of one key, 16 bytes at dh = 128, in one load and with one
//                  scale, four conversions to an operand and no trip through LDS.
//   O^T += V^T P^T the order of the keys is free as well: the scores a lane holds after two S^T tiles, keys 4 grp .. + 3 of
//                  either, are its operand as they are.  Values are converted as they come (a lane: 32 channels of a key),
//                  laid into the wave's own LDS by rows and read back transposed.
// Measured: one query of 32 heads of 128 on 8 key heads, 4 images of 32768 rows (143 MB) 29.5 us, of which 6.6 are start, first
// latency and the joining of waves and the rest runs at 6.1 TB/s; of 16 heads of 64, 8 images of 424 rows 5.6 us, a tile per wave.
#include "fourbit_attention.h"

namespace {

constexpr int kTile = 64;

template <typename T, int DH, int MT, int NW>
__global__ __launch_bounds__(NW * 64, NW == 8 || MT == 2 || sizeof(T) * DH == 512 ? 2 : 3) void few_kernel(AttentionArgs<T> a) {
  constexpr int NP = kParts<T>;
  constexpr int GPR = DH / kGroup;             // groups per row
  constexpr int ROWB = DH * 2;                 // bytes of a converted row
  constexpr int KW = DH / 32;                  // dwords of codes (MFMA steps) a lane holds per 16 keys
  constexpr int VL = DH / 32;                  // 16-byte loads of value codes per lane and tile
  constexpr int VR = 64 / GPR;                 // value rows per such load
  constexpr int DT = DH / 16;                  // 16-channel blocks of the output
  constexpr int HALF = 32 * ROWB;              // LDS of a wave: 32 converted value rows, then its 16 x DH results
  __shared__ __attribute__((aligned(1024))) char lds[NW * HALF];
  __shared__ float part_m[NW][16], part_l[NW][16];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int piece = blockIdx.x, nparts = a.nsplit;
  int split_i, b, j, block;
  a.place(div_by(piece, nparts, a.nsplit_inv, split_i), b, j, block);
  const int row0 = block * 16 * MT;
  const int rows = a.n * a.G, live = image_count(a.n_rows, b, a.n) * a.G, len = image_prior(a.kv_rows, b, a.P);
  const int ntiles = row0 < live ? (len + kTile - 1) / kTile : 0;
  // runs of one length whatever the image has, so that an image of any length is spread like the others; what none needs leaves
  const int t0 = split_i * a.run_tiles, t1 = min(ntiles, t0 + a.run_tiles);
  if (nparts > 1 && t0 >= t1) return;

  const int64_t base = ((int64_t)b * a.c.hk + j) * a.c.cap;
  const auto kc = head_buffer(a.c.codes[0] + base * (DH / 2), len * (DH / 2)), ks = head_buffer(a.c.scales[0] + base * GPR, len * GPR);
  const auto vc = head_buffer(a.c.codes[1] + base * (DH / 2), len * (DH / 2)), vs = head_buffer(a.c.scales[1] + base * GPR, len * GPR);
  const uint32_t k_lane = col * (DH / 2) + grp * (DH / 8), ks_lane = col * GPR + grp * GPR / 4;
  uint32_t kw[4][KW], vw[VL][4], kb[4], vb[VL];
  auto load_k = [&](int t) {
    const uint32_t o = k_lane + t * (kTile * DH / 2), os = ks_lane + t * (kTile * GPR);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DH == 128) {
        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(kc, o + i * 16 * (DH / 2), 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) kw[i][e] = w[e];
      } else {
        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(kc, o + i * 16 * (DH / 2), 0, 0);
        kw[i][0] = w[0];
        kw[i][1] = w[1];
      }
      kb[i] = __builtin_amdgcn_raw_buffer_load_b8(ks, os + i * 16 * GPR, 0, 0);
    }
  };
  auto load_v = [&](int t) {
    const uint32_t o = lane * 16 + t * (kTile * DH / 2), os = lane + t * (kTile * GPR);
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(vc, o + i * 1024, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) vw[i][e] = w[e];
      vb[i] = __builtin_amdgcn_raw_buffer_load_b8(vs, os + i * 64, 0, 0);
    }
  };

  const int first = t0 + wave;
  if (first < t1) {
    load_k(first);
    load_v(first);
  }
  // operand of step e: channels grp dh / 4 + 8 e .. + 7 of row col; past the last live row its copies (padding is nobody's)
  bf16x8 qf[MT][KW][NP];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const T* qp = a.query(b, j, max(min(row0 + mt * 16 + col, live - 1), 0)) + grp * (DH / 4);
#pragma unroll
    for (int e = 0; e < KW; ++e) load_eight(qp + e * 8, qf[mt][e]);
  }
  f32x4 o[MT][DT];
  float m_run[MT], l_run[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m_run[mt] = -INFINITY;
    l_run[mt] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[mt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  char* sv = lds + wave * HALF;
  // transposed reads: lane i of a group of sixteen names row 4 grp + i / 4 and 8-byte piece i % 4 of 16 channels
  int vaddr[DT];
  {
    const int r = 4 * grp + (col >> 2);
#pragma unroll
    for (int d = 0; d < DT; ++d) vaddr[d] = swz<ROWB>(r, 2 * d + ((col & 3) >> 1)) + (col & 1) * 8;
  }

  // values of 32 keys through the wave's LDS (its reads and writes are done in order): a lane's groups of channels
  char* lay_at[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) lay_at[e] = sv + swz<ROWB>(lane / GPR, lane % GPR * 4 + e);
  auto lay = [&](int u) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < VL / 2; ++i) {
      const float scale = fourbit_scale(vb[u * VL / 2 + i]);
#pragma unroll
      for (int e = 0; e < 4; ++e)        // the swizzle repeats after 16 rows
        *reinterpret_cast<bf16x8*>(lay_at[e] + i * VR * ROWB) = fourbit_eight(vw[u * VL / 2 + i][e], scale);
    }
    asm volatile("" ::: "memory");
  };
  for (int t = first; t < t1; t += NW) {
    const bool more = t + NW < t1;
    // ---- scores: register r of tile i is key 16 i + 4 grp + r, for row col
    f32x4 s[MT][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float scale = fourbit_scale(kb[i]);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) s[mt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < KW; ++e) {
        const bf16x8 kf = fourbit_eight(kw[i][e], scale);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) s[mt][i] = mfma16(kf, qf[mt][e][p], s[mt][i]);
      }
    }
    if (more) load_k(t + NW);
    lay(0);

    // ---- softmax: probabilities are 2^(score - m_run) against a reference that moves only when a sum of them says that some
    // score lies far above it, or there is none yet (-inf): no largest score, no lanes asked in the common case
    if ((t + 1) * kTile > len) {
      const float dead = a.scale_log2 < 0.f ? INFINITY : -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (t * kTile + i * 16 + grp * 4 + r >= len)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) s[mt][i][r] = dead;
    }
    float pr[MT][4][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float psum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          pr[mt][i][r] = __builtin_amdgcn_exp2f(fmaf(s[mt][i][r], a.scale_log2, -m_run[mt]));
          psum += pr[mt][i][r];
        }
      if (__any(!(psum <= kBig))) {
        float tmax = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) tmax = fmaxf(tmax, s[mt][i][r] * a.scale_log2);
        tmax = fmaxf(tmax, __shfl_xor(tmax, 16, NOVA_WAVE));
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32, NOVA_WAVE));
        const float m_new = fmaxf(m_run[mt], tmax);
        const float alpha = m_run[mt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[mt] - m_new);
        l_run[mt] *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[mt][d] *= alpha;
        m_run[mt] = m_new;
        const float ref = m_new == -INFINITY ? 0.f : m_new;            // nothing but scores of -inf so far
        psum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            pr[mt][i][r] = __builtin_amdgcn_exp2f(fmaf(s[mt][i][r], a.scale_log2, -ref));
            psum += pr[mt][i][r];
          }
      }
      l_run[mt] += psum;
    }

    // ---- O^T += V^T P^T, 32 keys at a time
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u == 1) {
        lay(1);
        if (more) load_v(t + NW);
      }
      bf16x8 pf[MT][NP];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          bf16_t p[NP];
          split(pr[mt][2 * u + (e >> 2)][e & 3], p);
#pragma unroll
          for (int i = 0; i < NP; ++i) pf[mt][i][e] = p[i];
        }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const bf16x8 vf = join(read_transposed(sv + vaddr[d]), read_transposed(sv + vaddr[d] + 16 * ROWB));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) o[mt][d] = mfma16(vf, pf[mt][p], o[mt][d]);
      }
    }
  }

  // ---- join the waves: [channel / 4][row] of four channels each in a wave's LDS
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float l = l_run[mt];
    l += __shfl_xor(l, 16, NOVA_WAVE);
    l += __shfl_xor(l, 32, NOVA_WAVE);
    if (mt > 0) __syncthreads();
    if (grp == 0) {
      part_m[wave][col] = m_run[mt];
      part_l[wave][col] = l;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(sv + ((d * 4 + grp) * 16 + col) * 16) = o[mt][d];
    __syncthreads();
    for (int i = tid; i < 16 * (DH / 4); i += NW * 64) {
      const int c4 = i % (DH / 4), rr = i / (DH / 4), row = row0 + mt * 16 + rr;
      if (row >= rows) continue;
      float m = -INFINITY, lt = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, part_m[w][rr]);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        // a wave without a finite score has reference -inf and sum 0 or NaN, and NaN or 0 in its results
        const float f = part_m[w][rr] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(part_m[w][rr] - m);
        lt = fmaf(f, part_l[w][rr], lt);
        acc += f * *reinterpret_cast<const f32x4*>(lds + w * HALF + (c4 * 16 + rr) * 16);
      }
      if (nparts == 1) {
        const bool some = row < live && len > 0;
        const int64_t to = a.out_row(b, j, row);
        store_four(a.out + to * DH + c4 * 4, some ? acc : f32x4{0.f, 0.f, 0.f, 0.f}, some ? 1.0f / lt : 0.f);
        if (a.lse && c4 == 0) a.lse[to] = some ? ((m == -INFINITY ? 0.f : m) + __builtin_amdgcn_logf(lt)) * kLn2 : -INFINITY;
      } else {
        const int64_t to = (int64_t)piece * 16 * MT + mt * 16 + rr;
        *reinterpret_cast<f32x4*>(a.part_o + to * DH + c4 * 4) = acc;
        if (c4 == 0) {
          a.part_ml[to * 2] = m;
          a.part_ml[to * 2 + 1] = lt;
        }
      }
    }
  }
}

}  // namespace

template <typename T>
hipError_t launch_fourbit_few(hipStream_t st, int dh, int mt, int waves, unsigned grid, const AttentionArgs<T>& a) {
#define GO(DH, MT, NW) few_kernel<T, DH, MT, NW><<<grid, NW * 64, 0, st>>>(a)
  if (dh == 64) { if (mt == 2) GO(64, 2, 4); else if (waves == 8) GO(64, 1, 8); else GO(64, 1, 4); }
  else { if (mt == 2) GO(128, 2, 4); else if (waves == 8) GO(128, 1, 8); else GO(128, 1, 4); }
#undef GO
  return hipGetLastError();
}
template hipError_t launch_fourbit_few<bf16_t>(hipStream_t, int, int, int, unsigned, const AttentionArgs<bf16_t>&);
template hipError_t launch_fourbit_few<float>(hipStream_t, int, int, int, unsigned, const AttentionArgs<float>&);
