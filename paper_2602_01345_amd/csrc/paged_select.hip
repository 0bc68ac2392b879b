// Which pages of a cache a query reads: a score per page from the page's mean key, and the k best pages of every (query, key head).
//
// Means and queries are whole numbers of at most 127 times a power of two (the means as nova_paged_summarise writes them, the
// queries rounded here), so a score is a sum of whole numbers under 2^21 times a power of two: exact in fp32 in whatever order it
// is taken, and a query chooses the same pages alone, in a chunk of any size and on any tiling.
//
// A workgroup has up to 16 queries of one key head.  Scores on the matrix cores, 16 pages x 16 queries per MFMA, one after the other
// for the heads that share the key head, their largest kept; as order-preserving 32-bit keys in LDS.  Then a wave per query: the
// k-th largest key bit by bit, by counting, and the pages above it and the first of those that equal it, in ascending order.
// What bounds it: issuing the count, per 64 keys and bit a comparison on the vector unit and a population count and an addition on the
// scalar one, for many queries: 1024 of 32 heads of 128 on 8 and 512 pages 32 us, vector instructions in 51 % of the cycles, scalar ones in
// 33 %, MFMA busy 6 %; for one the chain table, means, 32 bits, 13 us.  Registers are bounded so that two
// workgroups share a CU, for some spills outside of the loops (bf16, heads of 128: 47 -> 37 us with the means; fp32 4000 queries, 16
// heads of 128 171 -> 129, 1024 of 32 on 8 63 -> 62, but one token over four images 18.1 -> 21.3).
#include <algorithm>

#include "paged.h"

namespace {

constexpr int kWaves = 8;
constexpr int kHeads = 4;                // heads whose queries are held in registers at a time
constexpr int kAhead = 2;                // groups of 16 pages whose means a wave asks for at a time
constexpr int kMostKeys = 32;            // keys a lane holds while the k-th largest is looked for
constexpr uint32_t kTaken = 0xFFFFFFFFu; // key of a `first` or `recent` page, whatever its score; 0: of one that the query does not see
constexpr uint32_t kOdd = 0xFFFFFFFEu;   // of a page with a mean of NaN: in front of every score, behind those that are taken

struct SelectArgs {
  const void* q;
  int64_t q_sb, q_sr, q_sh;
  const bf16_t* means;
  const int32_t* table;
  int pitch, pages, hk, G, shift, n, P, causal, first, recent, k, queries, row;     // queries per workgroup, keys of one in LDS
  const int32_t *n_rows, *kv_rows;
  int32_t* chosen;
  int sharing;                           // waves that choose for one query together
};

__device__ __forceinline__ uint32_t score_key(float s) {
  uint32_t b = __float_as_uint(s);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return kOdd;              // a page that holds a NaN or an infinity shows in the result
  if (b == 0x80000000u) b = 0u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// R: keys a lane holds
template <typename T, int DH, int R>
__global__ __launch_bounds__(kWaves * 64, 4) void select_kernel(SelectArgs a) {
  constexpr int KC = DH / 32;                  // MFMAs per score: chunk 4 e + grp of eight channels
  extern __shared__ uint32_t keys[];           // [queries][row]
  __shared__ int counts[2][kWaves], equals[kWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int b = blockIdx.z, j = blockIdx.y, s0 = blockIdx.x * a.queries;
  const int count = image_count(a.n_rows, b, a.n), len = image_prior(a.kv_rows, b, a.P);
  const int up = (1 << a.shift) - 1;
  const int mine = min(s0 + min(col, a.queries - 1), max(count, 1) - 1);        // dead queries: the last live one's copies
  const int s_last = min(s0 + a.queries, count) - 1;
  const int npages = s_last < s0 ? 0 : (visible_keys(a.causal, len, count, s_last) + up) >> a.shift;
  const int seen = (visible_keys(a.causal, len, count, mine) + up) >> a.shift;  // pages this lane's query sees

  if (npages > 0) {
    const int32_t* table = a.table + (int64_t)b * a.pitch;
    // means of kAhead groups of pages: places in the pool first, asked for one round ahead
    int page[kAhead];
    auto look_up = [&](int x0) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) page[i] = table[min((x0 + i * kWaves) * 16 + col, npages - 1)];
    };
    look_up(wave);
    // the query's scale: one for all heads that share the key head
    const T* q = static_cast<const T*>(a.q) + b * a.q_sb + mine * a.q_sr + (int64_t)j * a.G * a.q_sh + grp * 8;
    uint32_t top = 0u;                         // largest magnitude, as the bits of an fp32 number: those that are none come last
    bf16x8 qf[kHeads][KC];                     // queries as they are (bf16), then rounded
    // (a head's fp32 numbers at a time: the compiler would have all of them in registers at once, for half the waves)
    auto load_heads = [&](int g0, auto use) {
      if constexpr (sizeof(T) == 2)
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
          if (g0 + g >= a.G) break;
#pragma unroll
          for (int e = 0; e < KC; ++e) qf[g][e] = *reinterpret_cast<const bf16x8*>(q + (g0 + g) * a.q_sh + e * 32);
        }
#pragma unroll
      for (int g = 0; g < kHeads; ++g) {
        if (g0 + g >= a.G) break;
        f32x4 w[KC][2];
        if constexpr (sizeof(T) == 4)
#pragma unroll
          for (int e = 0; e < KC; ++e)
#pragma unroll
            for (int c = 0; c < 2; ++c) w[e][c] = *reinterpret_cast<const f32x4*>(q + (g0 + g) * a.q_sh + e * 32 + c * 4);
#pragma unroll
        for (int e = 0; e < KC; ++e)
#pragma unroll
          for (int i = 0; i < 8; ++i) use(g, e, i, sizeof(T) == 2 ? (float)qf[g][e][i] : w[e][i >> 2][i & 3]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    for (int g0 = 0; g0 < a.G; g0 += kHeads)
      load_heads(g0, [&](int, int, int, float v) { top = max(top, __float_as_uint(v) & 0x7FFFFFFFu); });
    top = max(top, (uint32_t)__shfl_xor((int)top, 16, NOVA_WAVE));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, NOVA_WAVE));
    // the smallest power of two of which 127 reach the largest: as in summarise_kernel
    const int e2 = (int)(top >> 23) - 127 - 6 + ((top & 0x7FFFFFu) > 0x7E0000u);                // 127 / 64 = 1.984375
    const bool odd = top >= 0x7F800000u, held = !odd && e2 <= 100;                              // held: nothing passes 127
    const float unit = __uint_as_float((uint32_t)(127 - min(max(e2, -100), 100)) << 23);

    for (int g0 = 0; g0 < a.G; g0 += kHeads) {
      auto rounded = [&](int g, int e, int i, float v) { qf[g][e][i] = (bf16_t)rintf(v * unit); };
      if (sizeof(T) == 4 || a.G > kHeads) {
        load_heads(g0, rounded);
      } else {
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
          if (g0 + g >= a.G) break;
#pragma unroll
          for (int e = 0; e < KC; ++e)
#pragma unroll
            for (int i = 0; i < 8; ++i) rounded(g, e, i, (float)qf[g][e][i]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (__any(!held))                        // (rare) a query with a NaN or an infinity: zeros; past 127 * 2^100: that
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
          if (g0 + g >= a.G) break;
#pragma unroll
          for (int e = 0; e < KC; ++e)
#pragma unroll
            for (int i = 0; i < 8; ++i) qf[g][e][i] = odd ? (bf16_t)0.f : (bf16_t)fminf(fmaxf((float)qf[g][e][i], -127.f), 127.f);
          __builtin_amdgcn_sched_barrier(0);
        }
      if (g0 > 0) look_up(wave);
      for (int x0 = wave; x0 * 16 < npages; x0 += kAhead * kWaves) {
        bf16x8 means[kAhead][KC];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const bool there = (unsigned)page[i] < (unsigned)a.pages;
          const bf16_t* mp = a.means + ((int64_t)(there ? page[i] : 0) * a.hk + j) * DH + grp * 8;
#pragma unroll
          for (int e = 0; e < KC; ++e) {
            means[i][e] = bf16x8{};
            if (there) means[i][e] = *reinterpret_cast<const bf16x8*>(mp + e * 32);
          }
        }
        look_up(x0 + kAhead * kWaves);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
        const int x = x0 + i * kWaves;
        if (x * 16 >= npages) break;
        const auto& m = means[i];
        f32x4 best;
#pragma unroll
        for (int g = 0; g < kHeads; ++g) {
          if (g0 + g >= a.G) break;
          f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < KC; ++e) s = mfma16(m[e], qf[g][e], s);
#pragma unroll
          for (int r = 0; r < 4; ++r) best[r] = g == 0 ? s[r] : fmaxf(best[r], s[r]);
        }
        // register r is page 16 x + 4 grp + r, for query col
        u32x4 key;
        uint32_t* at = keys + col * a.row + x * 16 + grp * 4;
        const bool keep = col < a.queries;
        const u32x4 before = g0 > 0 && keep ? *reinterpret_cast<const u32x4*>(at) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at_page = x * 16 + grp * 4 + r;
          const bool taken = at_page < a.first || at_page >= seen - a.recent;
          const uint32_t w = max(score_key(best[r]), before[r]);
          key[r] = at_page >= seen ? 0u : taken ? kTaken : w;
        }
        if (keep) *reinterpret_cast<u32x4*>(at) = key;
        }
      }
    }
  }
  __syncthreads();

  // `sharing` waves per query, each with R keys per lane running.  The k-th largest key bit by bit from the top: the largest t of
  // which at least `take` keys are none the smaller, or, earlier, a t of which exactly `take` are.
  const int part = wave % a.sharing;
  const uint64_t below = (1ull << lane) - 1;
  for (int i0 = 0; i0 < a.queries; i0 += kWaves / a.sharing) {
    const int i = i0 + wave / a.sharing, s = s0 + i;
    const bool live = i < a.queries && s < a.n;
    const int sees = live && s < count ? (visible_keys(a.causal, len, count, s) + up) >> a.shift : 0;
    const int take = min(a.k, sees), x0 = part * R * 64 + lane;
    uint32_t w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = x0 + r * 64 < sees ? keys[i * a.row + x0 + r * 64] : 0u;
    auto at_least = [&](uint32_t t) {
      int c = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) c += (int)__popcll(__ballot(w[r] >= t));
      return c;
    };
    uint32_t t = 0u;
    int over = sees;                                             // pages with a key of at least t
    if (a.sharing == 1) {
      if (take < sees)
        for (int bit = 31; bit >= 0 && over != take; --bit) {
          const uint32_t higher = t | 1u << bit;
          const int c = at_least(higher);
          if (c >= take) { t = higher; over = c; }
        }
    } else {
      for (int bit = 31; bit >= 0; --bit) {                      // all waves alike: they meet at a barrier for every bit
        const uint32_t higher = t | 1u << bit;
        const int own = at_least(higher);                        // of all lanes of the wave
        if (lane == 0) counts[bit & 1][wave] = own;
        __syncthreads();
        int c = 0;
        for (int p = 0; p < a.sharing; ++p) c += counts[bit & 1][wave - part + p];
        if (take < sees && over != take && c >= take) { t = higher; over = c; }
      }
    }
    t = max(t, 1u);                                              // 0: every page that is seen
    // pages above t, of those that equal it the first ones
    int above = 0, equal = 0, in_front = 0, equal_in_front = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      above += (int)__popcll(__ballot(w[r] > t));
      equal += (int)__popcll(__ballot(w[r] == t));
    }
    int more = take - above;                                     // pages of key t that are taken
    if (a.sharing > 1) {
      __syncthreads();
      if (lane == 0) { counts[0][wave] = above; equals[wave] = equal; }
      __syncthreads();
      int all = 0;
      for (int p = 0; p < a.sharing; ++p) {
        all += counts[0][wave - part + p];
        if (p < part) { in_front += counts[0][wave - part + p]; equal_in_front += equals[wave - part + p]; }
      }
      more = take - all;
      __syncthreads();
    }
    if (!live) continue;
    int32_t* to = a.chosen + (((int64_t)b * a.n + s) * a.hk + j) * a.k;
    int at = in_front + min(equal_in_front, more), left = max(more - equal_in_front, 0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t same = __ballot(w[r] == t);
      const bool taken = w[r] > t || (w[r] == t && (int)__popcll(same & below) < left);
      const uint64_t all = __ballot(taken);
      const int place = at + (int)__popcll(all & below);
      if (taken && place < take) to[place] = x0 + r * 64;        // `take` pages are
      at += (int)__popcll(all);
      left = max(left - (int)__popcll(same), 0);
    }
    if (part == 0)
      for (int x = take + lane; x < a.k; x += 64) to[x] = -1;
  }
}

}  // namespace

hipError_t launch_paged_select(hipStream_t st, const PagedSelect& s) {
  SelectArgs a = {};
  a.q = s.q.data;
  a.q_sb = s.q.stride_b; a.q_sr = s.q.stride_row; a.q_sh = s.q.stride_head;
  a.means = static_cast<const bf16_t*>(s.means);
  a.table = s.table; a.pitch = s.pitch; a.pages = s.pages; a.hk = s.hk; a.G = s.heads / s.hk; a.shift = s.shift;
  a.n = s.n; a.P = s.kv_len; a.causal = s.causal; a.first = s.first; a.recent = s.recent; a.k = s.k;
  a.n_rows = s.n_rows; a.kv_rows = s.kv_rows; a.chosen = s.chosen;
  const int pages = (s.kv_len + (1 << s.shift) - 1) >> s.shift;
  a.row = (pages + 63) / 64 * 64 + 4;                            // four more, so that the queries of a wave meet different banks
  // as many queries as there are, and have room in a part of a CU's LDS
  a.queries = 16;
  while (a.queries > 1 && ((size_t)a.queries * a.row * 4 > 65536 || a.queries / 2 >= s.n)) a.queries /= 2;
  // Keys a lane holds: the fewest that do (us with 4 / 8 / 16 / 32 of them: 1024 queries, 64 pages 25.6 / 30.2 / - / 57, 512 pages - /
  // 36 / - / 63, 1024 pages - / - / 70 / 88; one query, 256 pages 13.8 / 15.0 / - / 23, 1024 pages - / - / 24 / 29).  Several waves per
  // query only where one cannot hold its keys: they meet at a barrier for every bit (one query, 1024 pages, two waves 29 / one 24).
  a.sharing = 1;
  while (pages > a.sharing * kMostKeys * 64) a.sharing *= 2;     // 2048 pages per wave, 16384 in all
  const int each = (pages + a.sharing - 1) / a.sharing;
  const dim3 grid((s.n + a.queries - 1) / a.queries, s.hk, s.B);
  const size_t lds = (size_t)a.queries * a.row * 4;
#define GO(T, DH)                                                                                                 \
  do {                                                                                                            \
    if (each <= 256) select_kernel<T, DH, 4><<<grid, kWaves * 64, lds, st>>>(a);                                  \
    else if (each <= 512) select_kernel<T, DH, 8><<<grid, kWaves * 64, lds, st>>>(a);                             \
    else if (each <= 1024) select_kernel<T, DH, 16><<<grid, kWaves * 64, lds, st>>>(a);                           \
    else select_kernel<T, DH, kMostKeys><<<grid, kWaves * 64, lds, st>>>(a);                                      \
  } while (0)
  if (s.dtype == NOVA_BF16) { if (s.dh == 64) GO(bf16_t, 64); else GO(bf16_t, 128); }
  else { if (s.dh == 64) GO(float, 64); else GO(float, 128); }
#undef GO
  return hipGetLastError();
}
