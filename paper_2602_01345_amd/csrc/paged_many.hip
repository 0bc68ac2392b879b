// Attention over a cache in pages for many rows per key head (whole scales, chunks of prompts).
//
// As in fourbit_attention.hip everything is computed transposed, a lane owning one row (query):
//   S^T = K Q^T    A operand = key rows from LDS, B operand = the row's channels, held in registers
//   O^T += V^T P^T A operand = value rows from LDS, read transposed, B operand = the probabilities as they come out of the softmax
// A workgroup is four waves of 32 rows.  Tiles of 64 keys go from the pages into LDS without passing through registers, each wave its
// 16 keys (which lie in one page, wherever pages end) of K and of V, a line per row, the swizzle made by which chunk of its row a lane
// asks for.  Two stages of LDS, two workgroups per CU (three with heads of 64), so that one wave's softmax runs next to another's
// MFMAs; a wave asks for priority while it issues MFMAs (below: 930 us; in the softmax instead 966, for the second product only 951; heads
// of 64, 4 images of 1024 over 4096 172 / 199 / 172).  What bounds it is that and power: two images, 2048 queries behind 14 336 rows,
// 32 heads of 128 on 8 (1.03 TFLOP) 930 to 1050 us by card, 1.0 to 1.1 PFLOP/s with the matrix cores busy 55 % of the cycles; 8 images of
// 512, 36 heads of 64 (44 GFLOP) 65 to 73, MFMA busy 32 % of the cycles, where 32 exponentials stand next to 16 MFMAs.
// Probabilities go into the second product as bf16, here and for bf16 in paged_few.hip and paged_chosen.hip: one rounding each (half a step,
// 2^-8 at most) instead of two or three MFMAs for the parts of an fp32 number.  The sum they are divided by is that of the fp32 ones.  The
// result's error against 64 bits goes from 1.7e-3 of it, which is its own rounding to bf16, to 1.8e-3 (the sizes above).
// A weight of 0 times a value that is no number is NaN, so what a row does not see could show in its result.  A workgroup whose sums
// end as anything but finite numbers goes over its tiles again, and takes those with such values in them key by key.
#include <type_traits>

#include "paged.h"

namespace {

constexpr int kWaves = 4, kTile = 64, kRows = kPagedRows;

__device__ __forceinline__ void wait_all() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);                      // vmcnt(0) lgkmcnt(0): own loads into LDS have landed, own reads are done
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int DH>
__global__ __launch_bounds__(kWaves * 64, DH == 64 ? 3 : 2) void many_kernel(PagedArgs<bf16_t> a) {
  constexpr int ROWB = DH * 2;
  constexpr int HALF = kTile * ROWB, STAGE = 2 * HALF;     // K rows, V rows
  constexpr int KS = DH / 16;                  // MFMAs along dh for a score block
  constexpr int DB = DH / 32;                  // 32-channel blocks of the output
  constexpr int NL = 16 * ROWB / 1024, RPL = 1024 / ROWB;  // loads of a wave's 16 rows, rows per load
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  __shared__ uint32_t odd_waves[kWaves];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const bool whole = (int)blockIdx.x < a.n_whole;
  const int run = blockIdx.x - a.n_whole;
  const int split_i = whole ? 0 : run % a.nsplit;
  const int nparts = whole ? 1 : a.nsplit;
  int b, j, block, unused;
  a.place_block(whole ? blockIdx.x : a.n_whole + run / a.nsplit, b, j, block);
  b = __builtin_amdgcn_readfirstlane(b);
  const int row0 = block * kRows;
  const int rows = a.n * a.G, count = image_count(a.n_rows, b, a.n), live = count * a.G, len = image_prior(a.kv_rows, b, a.P);
  const int last = min(row0 + kRows, live) - 1;            // last live row of the block
  const int seen_block = last < row0 ? 0 : visible_keys(a.causal, len, count, div_by(last, a.G, a.G_inv, unused));
  const int gshift = a.shift - 4, gmask = (1 << gshift) - 1;     // groups of 16 keys of a page
  const int groups = (seen_block + 15) / 16;
  const int ntiles = (groups + 3) / 4;
  const int per = (ntiles + nparts - 1) / nparts;
  const int t0 = split_i * per, t1 = min(ntiles, t0 + per);
  // keys that the wave's first and last live row see
  const int wrow = row0 + wave * 32, wlast = min(wrow + 31, live - 1);
  const bool wave_live = wrow < live;
  const int s_wave = div_by(min(wrow, max(live - 1, 0)), a.G, a.G_inv, unused), s_wlast = div_by(max(wlast, 0), a.G, a.G_inv, unused);
  const int seen_least = wave_live ? visible_keys(a.causal, len, count, s_wave) : 0;
  const int seen_most = wave_live ? visible_keys(a.causal, len, count, s_wlast) : 0;

  // this lane's part of a load of RPL rows: the chunk of its row that the swizzle puts where the lane's 16 bytes go
  uint32_t part[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) part[i] = swizzled_source<ROWB>(i * RPL + lane / (64 / RPL), lane % (64 / RPL));
  const int32_t* table = a.table + (int64_t)b * a.pitch;
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((lptr_t)lds);
  // The wave's 16 keys of a tile lie in one page, the u-th of the image; lanes hold 64 tiles' places in the pool.
  int held = 0, held_first = 0;
  auto hold = [&](int t) {
    held_first = t;
    held = groups > 0 ? table[min((t + lane) * 4 + wave, groups - 1) >> gshift] : -1;
  };
  auto look_up = [&](int t) {
    if (t - held_first >= 64) hold(t);
    return __builtin_amdgcn_readlane(held, t - held_first);
  };
  auto request = [&](int t, int page) {
    const int x = t * 4 + wave, u = x >> gshift, at_row = (x & gmask) * 16;
    const int there = x < groups ? min(max(len - (u << a.shift) - at_row, 0), (1 << a.shift) - at_row) : 0;
    const u32x4 ks = page_words<bf16_t, DH>(a.keys, page, a.pages, a.hk, j, a.shift, at_row, there);
    const u32x4 vs = page_words<bf16_t, DH>(a.values, page, a.pages, a.hk, j, a.shift, at_row, there);
    const uint32_t to = lds0 + (t & 1) * STAGE + wave * 16 * ROWB;
    load_to_lds(ks, to, part);
    load_to_lds(vs, to + HALF, part);
  };

  hold(t0);
  int next = look_up(t0);
  if (t0 < t1) {
    request(t0, next);
    next = look_up(t0 + 1);
  }
  const int row = wrow + col;
  bf16x8 qf[KS];                                           // channels 16 t + 8 half .. + 7 of this lane's row
  const int row_live = max(min(row, live - 1), 0);         // past the last live row its copies: what lies in padding is nobody's
  {
    const bf16_t* qp = a.query(b, j, row_live) + half * 8;
#pragma unroll
    for (int t = 0; t < KS; ++t) qf[t] = *reinterpret_cast<const bf16x8*>(qp + t * 16);
  }
  const int s_row = div_by(row_live, a.G, a.G_inv, unused);
  const int seen = visible_keys(a.causal, len, count, s_row);
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

  f32x16 o[DB];
  // probabilities are 2^(score - m_run); m_run is a reference, not necessarily the largest score
  float m_run, l_run;
  auto clear = [&] {
    m_run = kNone;
    l_run = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  };
  clear();

  auto over_tiles = [&](auto strict_tag) {
  constexpr bool STRICT = decltype(strict_tag)::value;     // the second time
  for (int t = t0; t < t1; ++t) {
    wait_all();                                            // tile t has landed, and nobody reads the other stage any more
    const int key0 = t * kTile;
    const bool mine = key0 < seen_most;
    // the next tile is asked for behind the first MFMAs, which then start at once (67 us at the barrier, 65 here: 8 images of 512
    // queries, 36 heads of 64)
    auto ahead = [&] {
      if (t + 1 < t1) {
        request(t + 1, next);
        next = look_up(t + 2);
      }
    };
    if (!mine) ahead();
    if (mine) {                                            // (a whole wave's) something that its rows see
    const char* sk = lds + (t & 1) * STAGE;
    const char* sv = sk + HALF;
    f32x16 s[2];
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[kb] = mfma32(*reinterpret_cast<const bf16x8*>(sk + kb * 32 * ROWB + ka[ks]), qf[ks], s[kb]);
    }
    __builtin_amdgcn_s_setprio(0);
    ahead();
    // ---- softmax: register r of block kb is key 64 t + 32 kb + 8 (r / 4) + 4 half + r % 4
    bool careful = false;
    if (key0 + kTile > seen_least) {                       // keys that not all of its rows see
      const float dead = a.scale_log2 < 0.f ? INFINITY : -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + kb * 32 + 8 * (r >> 2) + 4 * half + (r & 3) >= seen) s[kb][r] = dead;
      if constexpr (STRICT) {
        uint32_t odd = 0u;
#pragma unroll 1
        for (int i = 0; i < ROWB / 16; ++i) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(sv + (i * 64 + lane) * 16);
#pragma unroll
          for (int c = 0; c < 4; ++c) odd |= odd_pair(w[c]);
        }
        careful = __any(odd != 0u);
      }
    }
    float e[2][16], psum = 0.f;
    auto probabilities = [&] {
      psum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          e[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale_log2, -m_run));
          psum += e[kb][r];
        }
    };
    auto largest = [&] {
      float tmax = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, s[kb][r] * a.scale_log2);
      return max_across_32(tmax);
    };
    auto move = [&](float tmax) {
      const float m_new = fmaxf(m_run, tmax);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      m_run = m_new;
    };
    probabilities();
    if (__any(!(psum <= kBig))) {
      // some score lies far above the reference, as any does above the first one: it moves to the largest score, and the sums with it
      move(largest());
      probabilities();
    }
    l_run += psum;
    __builtin_amdgcn_s_setprio(1);
    // ---- O^T += V^T P^T, 16 keys per MFMA: the lane's keys 16 u + 4 half .. + 3 and 8 behind them
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      bf16x8 pf;
#pragma unroll
      for (int i = 0; i < 8; ++i) pf[i] = (bf16_t)e[u >> 1][(u & 1) * 8 + i];
      const char* at = sv + u * 16 * ROWB;
      if (!STRICT || !careful) {
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = mfma32(join(read_transposed(at + va[d][0]), read_transposed(at + va[d][1])), pf, o[d]);
      } else {
        // one key at a time: element i of the lanes of half x.  Rows whose weight for it is 0 take nothing of it.
#pragma unroll 1
        for (int ix = 0; ix < 16; ++ix) {
          const int i = ix >> 1, x = ix & 1;
          const uint32_t bits = half == x ? (i & 1 ? 0xFFFF0000u : 0xFFFFu) : 0u;
          u32x4 only;
#pragma unroll
          for (int c = 0; c < 4; ++c) only[c] = c == i >> 1 ? bits : 0u;
          const u32x4 w = __builtin_bit_cast(u32x4, pf) & only;
          const uint32_t weight = __shfl(w[0] | w[1] | w[2] | w[3], col + 32 * x, NOVA_WAVE);
          asm volatile("" ::: "memory");
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            f32x16 one;
#pragma unroll
            for (int r = 0; r < 16; ++r) one[r] = 0.f;
            const bf16x8 vf = join(read_transposed(at + va[d][0]), read_transposed(at + va[d][1]));
            one = mfma32(__builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, vf) & only), __builtin_bit_cast(bf16x8, w), one);
            if (weight)
#pragma unroll
              for (int r = 0; r < 16; ++r) o[d][r] += one[r];
          }
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    }
  }
  };
  over_tiles(std::false_type{});
  if (t0 < t1) {
    float sum = 0.f;                                       // 0, or NaN where some number is none
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum = fmaf(o[d][r], 0.f, sum);
    odd_waves[wave] = __any(sum != 0.f);
    wait_all();
    if (odd_waves[0] | odd_waves[1] | odd_waves[2] | odd_waves[3]) {
      clear();
      hold(t0);
      request(t0, look_up(t0));
      next = look_up(t0 + 1);
      over_tiles(std::true_type{});
    }
  }

  if (row >= rows) return;
  const float l = l_run + __shfl_xor(l_run, 32, NOVA_WAVE);
  if (nparts == 1) {
    const bool some = row < live && seen > 0;
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
      a.lse[to] = some ? (m_run + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
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

}  // namespace

hipError_t launch_paged_many(hipStream_t st, int dh, unsigned grid, const PagedArgs<bf16_t>& a) {
  if (dh == 64) many_kernel<64><<<grid, kWaves * 64, 0, st>>>(a);
  else many_kernel<128><<<grid, kWaves * 64, 0, st>>>(a);
  return hipGetLastError();
}
