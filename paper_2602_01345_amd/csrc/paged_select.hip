// Which pages of a cache a query reads: a score per page from the page's mean key, and the k best pages of every (query, key head).
//
// Means and queries are whole numbers of at most 127 times a power of two (the means as nova_paged_summarise writes them, the
// queries rounded here), so a score is a sum of whole numbers under 2^21 times a power of two: exact in fp32 in whatever order it
// is taken, and a query chooses the same pages alone, in a chunk of any size and on any tiling.
//
// A workgroup has up to 16 queries of one key head.  Scores on the matrix cores, 16 pages x 16 queries per MFMA, one after the other
// for the heads that share the key head, their largest kept; as order-preserving 32-bit keys in LDS.  Then a wave per query: the
// k-th largest key bit by bit, by counting, and the pages above it and the first of those that equal it, in ascending order.
#include <algorithm>

#include "paged.h"

namespace {

constexpr int kWaves = 8;
constexpr int kHeads = 4;                // heads whose queries are held in registers at a time
constexpr uint32_t kTaken = 0xFFFFFFFFu; // key of a page that is taken whatever its score; 0: one that the query does not see

struct SelectArgs {
  const void* q;
  int64_t q_sb, q_sr, q_sh;
  const bf16_t* means;
  const int32_t* table;
  int pitch, pages, hk, G, shift, n, P, causal, first, recent, k, queries, row;     // queries per workgroup, keys of one in LDS
  const int32_t *n_rows, *kv_rows;
  int32_t* chosen;
};

__device__ __forceinline__ uint32_t score_key(float s) {
  uint32_t b = __float_as_uint(s);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return kTaken;            // a page that holds a NaN or an infinity shows in the result
  if (b == 0x80000000u) b = 0u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <typename T, int DH>
__global__ __launch_bounds__(kWaves * 64, 2) void select_kernel(SelectArgs a) {
  constexpr int KC = DH / 32;                  // MFMAs per score: chunk 4 e + grp of eight channels
  extern __shared__ uint32_t keys[];           // [queries][row]
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
    // the query's scale: one for all heads that share the key head
    const T* q = static_cast<const T*>(a.q) + b * a.q_sb + mine * a.q_sr + (int64_t)j * a.G * a.q_sh + grp * 8;
    float top = 0.f;
    bool odd = false;
    for (int g = 0; g < a.G; ++g)
#pragma unroll
      for (int e = 0; e < KC; ++e)
#pragma unroll
        for (int c = 0; c < 8; c += Vec16<T>::N) {
          Vec16<T> v;
          v.load(q + g * a.q_sh + e * 32 + c);
#pragma unroll
          for (int i = 0; i < Vec16<T>::N; ++i) {
            top = fmaxf(top, fabsf(v.get(i)));
            odd |= !(fabsf(v.get(i)) < INFINITY);
          }
        }
    top = fmaxf(top, __shfl_xor(top, 16, NOVA_WAVE));
    top = fmaxf(top, __shfl_xor(top, 32, NOVA_WAVE));
    odd |= __shfl_xor((int)odd, 16, NOVA_WAVE);
    odd |= __shfl_xor((int)odd, 32, NOVA_WAVE);
    // the smallest power of two of which 127 reach the largest: as in summarise_kernel
    const uint32_t bits = __float_as_uint(top);
    int e2 = (int)(bits >> 23) - 127 - 6 + ((bits & 0x7FFFFFu) > 0x7E0000u);    // 127 / 64 = 1.984375
    e2 = min(max(e2, -100), 100);
    const float unit = odd ? 0.f : __uint_as_float((uint32_t)(127 - e2) << 23);

    for (int g0 = 0; g0 < a.G; g0 += kHeads) {
      bf16x8 qf[kHeads][KC];
#pragma unroll
      for (int g = 0; g < kHeads; ++g)
#pragma unroll
        for (int e = 0; e < KC; ++e)
#pragma unroll
          for (int c = 0; c < 8; c += Vec16<T>::N) {
            Vec16<T> v;
            v.load(q + min(g0 + g, a.G - 1) * a.q_sh + e * 32 + c);
#pragma unroll
            for (int i = 0; i < Vec16<T>::N; ++i) {
              const float w = odd ? 0.f : fminf(fmaxf(rintf(v.get(i) * unit), -127.f), 127.f);
              qf[g][e][c + i] = (bf16_t)w;
            }
          }
      for (int x = wave; x * 16 < npages; x += kWaves) {
        const int ordinal = min(x * 16 + col, npages - 1), page = a.table[(int64_t)b * a.pitch + ordinal];
        const bool there = (unsigned)page < (unsigned)a.pages;
        bf16x8 m[KC];
        const bf16_t* mp = a.means + ((int64_t)(there ? page : 0) * a.hk + j) * DH + grp * 8;
#pragma unroll
        for (int e = 0; e < KC; ++e) {
          m[e] = *reinterpret_cast<const bf16x8*>(mp + e * 32);
          if (!there) m[e] = bf16x8{};
        }
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
          const int i = x * 16 + grp * 4 + r;
          const bool taken = i < a.first || i >= seen - a.recent;
          const uint32_t w = max(score_key(best[r]), before[r]);
          key[r] = i >= seen ? 0u : taken ? kTaken : w;
        }
        if (keep) *reinterpret_cast<u32x4*>(at) = key;
      }
    }
  }
  __syncthreads();

  for (int i = wave; i < a.queries; i += kWaves) {
    const int s = s0 + i;
    if (s >= a.n) break;
    int32_t* to = a.chosen + (((int64_t)b * a.n + s) * a.hk + j) * a.k;
    const int sees = s < count ? (visible_keys(a.causal, len, count, s) + up) >> a.shift : 0;
    const int take = min(a.k, sees);
    const uint32_t* key = keys + i * a.row;
    // pages with a key of at least t
    auto at_least = [&](uint32_t t) {
      int c = 0;
      for (int x = lane; x < (sees + 63) / 64 * 64; x += 64) c += __popcll(__ballot(x < sees && key[x] >= t));
      return c;
    };
    uint32_t t = 0u;
    int over = sees;                                             // pages with a key of at least t
    if (take < sees)
      for (int bit = 31; bit >= 0 && over != take; --bit) {
        const uint32_t higher = t | 1u << bit;
        const int c = at_least(higher);
        if (c >= take) { t = higher; over = c; }
      }
    // t is the take-th largest key, or `take` pages have one of at least t
    int equal = 0;                                               // pages of key t that are taken
    if (over > take) equal = take - (t == kTaken ? 0 : at_least(t + 1));
    else equal = over;
    int at = 0;
    for (int x0 = 0; x0 < sees; x0 += 64) {
      const int x = x0 + lane;
      const uint32_t w = x < sees ? key[x] : 0u;
      const bool above = x < sees && w > t, same = x < sees && w == t;
      const uint64_t sames = __ballot(same), below = (1ull << lane) - 1;
      const bool mine_too = above || (same && (int)__popcll(sames & below) < equal);
      const uint64_t all = __ballot(mine_too);
      if (mine_too) to[at + (int)__popcll(all & below)] = x;
      at += (int)__popcll(all);
      equal -= min(equal, (int)__popcll(sames));
    }
    for (int x = at + lane; x < a.k; x += 64) to[x] = -1;
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
  const dim3 grid((s.n + a.queries - 1) / a.queries, s.hk, s.B);
  const size_t lds = (size_t)a.queries * a.row * 4;
#define GO(T, DH) select_kernel<T, DH><<<grid, kWaves * 64, lds, st>>>(a)
  if (s.dtype == NOVA_BF16) { if (s.dh == 64) GO(bf16_t, 64); else GO(bf16_t, 128); }
  else { if (s.dh == 64) GO(float, 64); else GO(float, 128); }
#undef GO
  return hipGetLastError();
}
