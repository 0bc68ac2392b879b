// Attention over a cache in pages where queries have chosen pages each for themselves, many rows per key head (chunks of prompts).
//
// A block goes over the union of its queries' lists, and most tiles of it are some rows' alone.  So a workgroup is eight waves of 16 rows,
// the fewest that an MFMA takes: tiles of 64 keys go from the pages into LDS once for all of them, and a wave does those that one of its
// own queries has chosen, each row masked where it has not.  Computed transposed, as in paged_few.hip, a lane owning one row (col) and the
// four lane groups (grp) parts of the keys:
//   S^T = K Q^T    16 keys x 16 rows per MFMA, keys and channels from LDS by rows, the row's channels in registers
//   O^T += V^T P^T the scores a lane holds after two S^T products are its operand as they are, values read transposed
// Two stages of LDS, two workgroups per CU, so that the waves that have nothing to do in one tile leave the SIMD to others.
// What bounds it is the longest wave's way through each tile: 1024 queries, 32 heads of 128 on 8, 32 of 512 pages each, take 247 us with
// the join, of which 32 queries' unions (264 pages on average) loaded and nothing else are 145, and computed without a load 240.
// Waves of 32 rows, which do 1.6 times as many tiles' rows in vain, take 324, tiles of 32 keys in four stages 341; masks by comparing
// every key 280.
// Values that are no numbers in rows that a query does not see: a weight of 0 times such a value is NaN, and a score of what has not been
// chosen may be one too.  A workgroup whose sums end as anything but finite numbers goes over its tiles again, every key masked for
// itself; a tile's values that are no numbers are taken out of it then and their kinds put beside it, a number for each, so that a second
// product with 1 for every weight above 0 counts what a row takes of each kind.
#include "paged.h"

namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
constexpr int kWaves = 8, kTile = 64, kRows = kPagedRows;
static_assert(kWaves * 16 == kRows, "");

__device__ __forceinline__ void wait_all() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);                      // vmcnt(0) lgkmcnt(0): own loads into LDS have landed, own reads are done
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int DH>
__global__ __launch_bounds__(kWaves * 64, 4) void chosen_kernel(PagedArgs<bf16_t> a) {
  constexpr int ROWB = DH * 2;
  constexpr int HALF = kTile * ROWB, STAGE = 2 * HALF;     // K rows, V rows
  constexpr int KC = DH / 32;                  // MFMAs along dh for 16 keys
  constexpr int DT = DH / 16;                  // 16-channel blocks of the output
  constexpr int NL = 16 * ROWB / 1024, RPL = 1024 / ROWB;  // loads of 16 rows, rows per load
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  __shared__ uint32_t odd_waves[kWaves];
  static_assert(sizeof(lds) + sizeof(odd_waves) == paged_chosen_lds(DH), "");
  extern __shared__ uint32_t lists[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
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
  const int s_first = div_by(row0, a.G, a.G_inv, unused), s_last = last < row0 ? s_first : div_by(last, a.G, a.G_inv, unused);
  const int seen_block = last < row0 ? 0 : visible_keys(a.causal, len, count, s_last);
  const int gshift = a.shift - 4, gmask = (1 << gshift) - 1;     // groups of 16 keys of a page
  const ChosenPages list =
      list_chosen<bf16_t, kWaves * 64, kWaves / 2>(a, lists, b, j, row0, s_first, s_last, (seen_block + (1 << a.shift) - 1) >> a.shift);
  const int groups = list.count << gshift;
  const int ntiles = (groups + 3) / 4;
  const int per = (ntiles + nparts - 1) / nparts;
  const int t0 = split_i * per, t1 = min(ntiles, t0 + per);
  // the wave's queries, as bits of the words that two waves share
  const int wrow = row0 + wave * 16, wlast = min(wrow + 15, live - 1);
  const bool wave_live = wrow < live;
  const int s_word = div_by(row0 + (wave >> 1) * 32, a.G, a.G_inv, unused);
  const int s_wave = div_by(min(wrow, max(live - 1, 0)), a.G, a.G_inv, unused), s_wlast = div_by(max(wlast, 0), a.G, a.G_inv, unused);
  const int seen_least = wave_live ? visible_keys(a.causal, len, count, s_wave) : 0;
  const int seen_most = wave_live ? visible_keys(a.causal, len, count, s_wlast) : 0;
  const uint32_t all = wave_live ? 0xFFFFFFFFu >> (31 - (s_wlast - s_wave)) << (s_wave - s_word) : 0u;

  // four waves load keys and four values, 16 rows each, which lie in one page: a lane asks for the chunk of its row that the swizzle puts
  // where its 16 bytes go
  uint32_t part[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) part[i] = swizzled_source<ROWB>(i * RPL + lane / (64 / RPL), lane % (64 / RPL));
  const uint64_t pool = reinterpret_cast<uint64_t>(wave < 4 ? a.keys : a.values);
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((lptr_t)lds) + wave * 16 * ROWB;
  // Lanes hold what is to be known of 64 groups of 16 keys, those of 16 tiles: first key, which of the wave's queries have chosen its page,
  // where its rows begin in the wave's pool, and how many bytes of rows of its page there are from there on.
  struct Groups { int key0; uint32_t who, lo, hi, bytes; } held = {};
  int held_first = 0;
  auto hold = [&](int t) {
    held_first = t;
    const int x = t * 4 + lane, u = min(x, groups - 1) >> gshift, page = list.page[u], at_row = (x & gmask) * 16;
    const bool there = x < groups && (unsigned)page < (unsigned)a.pages;
    held.key0 = ((int)list.listed[u] << a.shift) + at_row;
    held.who = x < groups ? list.member[u * (kWaves / 2) + (wave >> 1)] & all : 0u;
    const uint64_t at = pool + (uint64_t)(((((int64_t)(there ? page : 0) * a.hk + j) << a.shift) + at_row) * ROWB);
    held.lo = (uint32_t)at;
    held.hi = (uint32_t)(at >> 32) & 0xFFFFu;
    held.bytes = there ? min(max(len - held.key0, 0), (1 << a.shift) - at_row) * ROWB : 0;
  };
  int key0_next[4];
  uint32_t who_next[4];
  auto request = [&](int t) {                              // and what the wave has to know of tile t
    if (t - held_first >= 16) hold(t);
    const int i = (t - held_first) * 4;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      key0_next[g] = __builtin_amdgcn_readlane(held.key0, i + g);
      who_next[g] = (uint32_t)__builtin_amdgcn_readlane((int)held.who, i + g);
    }
    const int w = i + (wave & 3);
    const u32x4 buffer = {(uint32_t)__builtin_amdgcn_readlane((int)held.lo, w), (uint32_t)__builtin_amdgcn_readlane((int)held.hi, w),
                          (uint32_t)__builtin_amdgcn_readlane((int)held.bytes, w), 0x00020000u};
    load_to_lds(buffer, lds0 + (t & 1) * STAGE, part);
  };
  auto begin = [&] {
    hold(t0);
    request(t0);
  };
  if (t0 < t1) begin();
  const int row = wrow + col;
  const int row_live = max(min(row, live - 1), 0);         // past the last live row its copies: what lies in padding is nobody's
  bf16x8 qf[KC];                                           // chunk grp + 4 e of this lane's row
  {
    const bf16_t* qp = a.query(b, j, row_live) + grp * 8;
#pragma unroll
    for (int e = 0; e < KC; ++e) qf[e] = *reinterpret_cast<const bf16x8*>(qp + e * 32);
  }
  const int s_row = div_by(row_live, a.G, a.G_inv, unused);
  const int seen = visible_keys(a.causal, len, count, s_row);
  const uint32_t bit = 1u << ((s_row - s_word) & 31);
  // this lane's places in a tile: its key's chunks, and for transposed reads of values the 8-byte piece lane % 4 of 16 channels of key
  // 4 grp + col / 4.  The swizzle repeats after 16 rows.
  int ka[KC], va[DT];
#pragma unroll
  for (int e = 0; e < KC; ++e) ka[e] = swz<ROWB>(col, e * 4 + grp);
#pragma unroll
  for (int d = 0; d < DT; ++d) va[d] = swz<ROWB>(4 * grp + (col >> 2), 2 * d + ((col & 3) >> 1)) + (col & 1) * 8;

  f32x4 o[DT];
  // probabilities are 2^(score - m_run); m_run is a reference, not necessarily the largest score
  float m_run, l_run;
  auto clear = [&] {
    m_run = kNone;
    l_run = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  clear();

  bool strict = false;                                     // the second time over the tiles
  for (;;) {
  for (int t = t0; t < t1; ++t) {
    wait_all();                                            // tile t has landed, and nobody reads the other stage any more
    const int stage = (t & 1) * STAGE, other = STAGE - stage;
    if (strict) {
#pragma unroll 1
      for (int i = tid * 16; i < HALF; i += kWaves * 64 * 16) {
        u16x8 v = *reinterpret_cast<const u16x8*>(lds + stage + HALF + i), kinds;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool odd = (v[e] & 0x7F80) == 0x7F80;
          kinds[e] = !odd ? 0 : v[e] & 0x7F ? 0x4680 : v[e] & 0x8000 ? 0x4300 : 0x3F80;           // bf16 2^14, 2^7, 1
          v[e] = odd ? 0 : v[e];
        }
        *reinterpret_cast<u16x8*>(lds + stage + HALF + i) = v;
        *reinterpret_cast<u16x8*>(lds + other + HALF + i) = kinds;
      }
      wait_all();
    }
    int key0[4];
    uint32_t who[4], any = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      key0[i] = key0_next[i];
      who[i] = who_next[i];
      any |= who[i];
    }
    const bool mine = key0[0] < seen_most && any != 0u;
    auto ahead = [&] {
      if (t + 1 < t1 && !strict) request(t + 1);
    };
    if (!mine) ahead();
    if (mine) {                                            // (a whole wave's) something that its rows see
    auto keys = [&](int i, int e) { return *reinterpret_cast<const bf16x8*>(lds + stage + i * 16 * ROWB + ka[e]); };
    auto values = [&](int at, int u, int d) {
      const char* p = lds + at + HALF + u * 32 * ROWB + va[d];
      return join(read_transposed(p), read_transposed(p + 16 * ROWB));
    };
    // ---- scores: register r of group i is key 4 grp + r of it, for row col
    f32x4 s[4];
    __builtin_amdgcn_s_setprio(1);                         // others wait for it (through the tile 247 us, for the products alone 252, without 255)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < KC; ++e) s[i] = mfma16(keys(i, e), qf[e], s[i]);
      if (i & 1) __builtin_amdgcn_sched_barrier(0);        // keys of two groups on their way at a time: registers
    }
    ahead();
    // What a row has not chosen has no weight: -inf in place of its reference, which leaves scores that are no numbers to the second time.
    const float dead = a.scale_log2 < 0.f ? INFINITY : -INFINITY;
    if (strict || key0[3] + 16 > seen_least) {             // keys that not all of its rows see
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int sees = who[i] & bit ? seen - key0[i] - 4 * grp : 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r >= sees) s[i][r] = dead;
      }
    }
    float pr[4][4], psum = 0.f;
    auto probabilities = [&] {
      float sums[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float from = who[i] & bit ? -m_run : -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) pr[i][r] = __builtin_amdgcn_exp2f(fmaf(s[i][r], a.scale_log2, from));
        sums[i] = (pr[i][0] + pr[i][1]) + (pr[i][2] + pr[i][3]);
      }
      psum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    };
    auto largest = [&] {
      float tmax = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) tmax = fmaxf(tmax, who[i] & bit ? s[i][r] * a.scale_log2 : -INFINITY);
      return max_across_32(max_across_16(tmax));
    };
    probabilities();
    if (__any(!(psum <= kBig))) {
      // some score lies far above the reference, as any does above the first one: it moves to the largest score, and the sums with it
      const float m_new = fmaxf(m_run, largest());
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= alpha;
      m_run = m_new;
      probabilities();
    }
    l_run += psum;
    // ---- O^T += V^T P^T, 32 keys per MFMA
    bf16x8 pf[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[u][e] = (bf16_t)pr[2 * u + (e >> 2)][e & 3];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        o[d] = mfma16(values(stage, u, d), pf[u], o[d]);
        if ((d & 3) == 3) __builtin_amdgcn_sched_barrier(0);                                    // four operands on their way at a time
      }
    __builtin_amdgcn_s_setprio(0);
    if (strict) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[u][e] = pf[u][e] == (bf16_t)0.f ? (bf16_t)0.f : (bf16_t)1.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        f32x4 counts = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) counts = mfma16(values(other, u, d), pf[u], counts);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int c = (int)counts[r];
          if (c & 0x7F) o[d][r] += INFINITY;
          if (c & 0x3F80) o[d][r] -= INFINITY;
          if (c >> 14) o[d][r] = NAN;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    }
    if (strict && t + 1 < t1) {
      wait_all();
      request(t + 1);
    }
  }
  if (t0 >= t1 || strict) break;
  float sum = 0.f;                                         // 0, or NaN where some number is none
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) sum = fmaf(o[d][r], 0.f, sum);
  odd_waves[wave] = __any(sum != 0.f);
  wait_all();
  uint32_t odd = 0u;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) odd |= odd_waves[w];
  if (__builtin_expect(odd == 0u, 1)) break;
  strict = true;
  clear();
  begin();
  }

  if (row >= rows) return;
  float l = l_run + __shfl_xor(l_run, 16, NOVA_WAVE);
  l += __shfl_xor(l, 32, NOVA_WAVE);
  if (nparts == 1) {
    bool some = row < live && seen > 0;
    if (__builtin_expect(l == 0.f, 0)) {
      int again = row;
      asm("" : "+v"(again));                               // divided once more: the quotient would be held through the loop
      some = some && sees_chosen(a, b, j, div_by(again, a.G, a.G_inv, unused), seen);
    }
    const int64_t to = a.out_row(b, j, row);
    const float inv = some ? 1.0f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) store_four(a.out + to * DH + d * 16 + grp * 4, some ? o[d] : f32x4{0.f, 0.f, 0.f, 0.f}, inv);
    if (a.lse && grp == 0) a.lse[to] = some ? (m_run + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  } else {
    const int64_t to = (int64_t)run * kRows + (row - row0);
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(a.part_o + to * DH + d * 16 + grp * 4) = o[d];
    if (grp == 0) {
      a.part_ml[to * 2] = m_run;
      a.part_ml[to * 2 + 1] = l;
    }
  }
}

}  // namespace

hipError_t launch_paged_chosen(hipStream_t st, int dh, unsigned grid, const PagedArgs<bf16_t>& a) {
  const size_t lists = (chosen_bytes(a.most_pages, a.most_listed, kWaves / 2) + 15) / 16 * 16;
  if (dh == 64) chosen_kernel<64><<<grid, kWaves * 64, lists, st>>>(a);
  else chosen_kernel<128><<<grid, kWaves * 64, lists, st>>>(a);
  return hipGetLastError();
}
