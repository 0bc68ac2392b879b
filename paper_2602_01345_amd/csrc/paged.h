// The key/value cache in pages (include/nova.h) as its kernels take it.
#pragma once
#include "attention_core.h"
#include "nova_internal.h"

// The first reference of a softmax: no finite score lies below it, and a row that sees nothing stays there with a sum of 0.
constexpr float kNone = -3.40282347e38f;
constexpr int kPageGroup = 16;           // rows that never lie in two pages: pages have 2^shift rows, 16 at least

// A (page, key head)'s rows from `row` on as the four words of a buffer for loads that go into LDS: `rows` of them exist, loads from
// there on give zeros.  A page that is none of the pool has no rows, so that no table leads a load out of it.  Where the rows begin
// stands in the buffer's base and never in a load's scalar offset: whether that one counts against the buffer's length, and what comes of
// a length that is less than it, is not said alike everywhere.
template <typename T, int DH>
__device__ __forceinline__ u32x4 page_words(const T* pool, int page, int pages, int hk, int j, int shift, int row, int rows) {
  const bool there = (unsigned)page < (unsigned)pages;
  const uint64_t base = reinterpret_cast<uint64_t>(pool + (((((int64_t)(there ? page : 0) * hk + j) << shift) + row) * DH));
  return u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, there ? rows * (uint32_t)(DH * sizeof(T)) : 0u, 0x00020000u};
}
// Loads that go into LDS are written in assembly: the compiler, which cannot tell which LDS a transposed read may meet, would make every
// such read wait for all of them.  They have no output registers, and who reads what they bring waits for vmcnt(0) and at a
// barrier first.
// 16 bytes per lane from lane_off[e] of the buffer to the e-th KB of LDS from `to` on (to: of the whole wave).  The waits in front of the
// loads are those that the hardware asks for: five states after a vector instruction that wrote a scalar register which a load
// reads (the compiler does not look for that here), one after a write of m0.
template <int N>
__device__ __forceinline__ void load_to_lds(u32x4 buffer, uint32_t to, const uint32_t (&lane_off)[N]) {
  static_assert(N == 2 || N == 4 || N == 8, "");
  if constexpr (N == 8) {
    load_to_lds(buffer, to, {lane_off[0], lane_off[1], lane_off[2], lane_off[3]});
    load_to_lds(buffer, to + 4096, {lane_off[4], lane_off[5], lane_off[6], lane_off[7]});
  } else if constexpr (N == 4) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds"
                 :: "s"(to), "v"(lane_off[0]), "v"(lane_off[1]), "v"(lane_off[2]), "v"(lane_off[3]), "s"(buffer)
                 : "memory", "scc");
  } else {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds"
                 :: "s"(to), "v"(lane_off[0]), "v"(lane_off[1]), "s"(buffer) : "memory", "scc");
  }
}

// Query s of an image (the last `count` of its `len` rows) sees this many keys from the front.
__device__ __forceinline__ int visible_keys(int causal, int len, int count, int s) {
  if (!causal) return len;
  const int v = len - count + s + 1;
  return v < 0 ? 0 : (v > len ? len : v);
}

template <typename T>
struct PagedArgs : AttentionItems<T> {
  const T* keys;                         // pools [pages, hk, 2^shift, dh]
  const T* values;
  const int32_t* table;                  // [B, pitch]
  int pitch, pages, shift, causal;
  const int32_t* chosen;                 // [B, n, hk, take], or nullptr: all rows
  int take, most_pages, most_listed;     // pages an image has at most; entries of the list of chosen pages of a block of rows
  uint32_t take_inv;

  // Image, key head and block of rows of an item: as AttentionItems::place, images by falling length where they are ranked, and the
  // blocks that see most first.
  __device__ __forceinline__ void place_block(int item, int& b, int& j, int& block) const {
    this->place(item, b, j, block);
    if (this->ranked) b = this->by_length(b);
    if (causal) block = this->blocks - 1 - block;
  }
};

// Query s of image b, which sees `visible` keys, has chosen a page with some of them.  Asked only of queries whose weights sum to 0: scores
// that are all -inf leave that too, and a result that is no number, as they do where nothing is chosen.
template <typename T>
__device__ __forceinline__ bool sees_chosen(const PagedArgs<T>& a, int b, int j, int s, int visible) {
  const int32_t* chosen = a.chosen + (((int64_t)b * a.n + s) * a.hk + j) * a.take;
  const unsigned npages = (unsigned)(visible + (1 << a.shift) - 1) >> a.shift;
  for (int i = 0; i < a.take; ++i)
    if ((unsigned)chosen[i] < npages) return true;
  return false;
}

// The larger of a lane's number and that of the lane 32, or 16, away, on the vector unit.
__device__ __forceinline__ float max_across_32(float v) {
  const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float max_across_16(float v) {
  const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}

// some bf16 number of the two in w is no finite one: an exponent of ones carries into the bit above it
__device__ __forceinline__ uint32_t odd_pair(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t odd_one(uint32_t w) { return ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u; }

// The pages that a block's queries have chosen, as ascending ordinals, with a word per page for every 32 rows of the block: bit s says
// that query s (counted from the first of these rows) has chosen it.  Made in LDS by all threads of the workgroup, as a bitmap over
// the image's pages: the order of the lists, repeats, and entries that are no pages of the image do not matter.
struct ChosenPages {
  const uint16_t* listed;
  const int32_t* page;                   // the listed pages' places in the pool
  const uint32_t* member;                // [listed][WORDS]
  int count;
};
inline size_t chosen_bytes(int most_pages, int most_listed, int words) {
  return ((size_t)(most_pages + 31) / 32 * 2 + 1 + (size_t)most_listed * (words + 1)) * 4 + (size_t)most_listed * 2;
}
template <typename T, int THREADS, int WORDS>
__device__ __forceinline__ ChosenPages list_chosen(const PagedArgs<T>& a, uint32_t* lds, int b, int j, int row0, int s_first, int s_last,
                                                   int npages) {
  const int tid = threadIdx.x, lane = tid & 63, words = (npages + 31) / 32, most_words = (a.most_pages + 31) / 32;
  uint32_t* bits = lds;
  uint32_t* before = lds + most_words;   // listed pages in front of a word
  uint32_t* member = lds + 2 * most_words + 1;
  int32_t* page = reinterpret_cast<int32_t*>(member + a.most_listed * WORDS);
  uint16_t* listed = reinterpret_cast<uint16_t*>(page + a.most_listed);
  const int32_t* chosen = a.chosen + (((int64_t)b * a.n + s_first) * a.hk + j) * a.take;
  const int entries = npages > 0 ? (s_last - s_first + 1) * a.take : 0;
  auto entry = [&](int i, int& s) {
    int at;
    s = div_by(i, a.take, a.take_inv, at);
    return chosen[(int64_t)s * a.hk * a.take + at];
  };
  for (int w = tid; w < words; w += THREADS) bits[w] = 0u;
  for (int w = tid; w < a.most_listed * WORDS; w += THREADS) member[w] = 0u;
  __syncthreads();
  for (int i = tid; i < entries; i += THREADS) {
    int s;
    const int c = entry(i, s);
    if ((unsigned)c < (unsigned)npages) atomicOr(&bits[c >> 5], 1u << (c & 31));
  }
  __syncthreads();
  if (tid < 64) {
    int base = 0;
    for (int w0 = 0; w0 < words; w0 += 64) {
      const int mine = w0 + lane < words ? __popc(bits[w0 + lane]) : 0;
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(inc, o, NOVA_WAVE);
        if (lane >= o) inc += t;
      }
      if (w0 + lane < words) before[w0 + lane] = base + inc - mine;
      base += __shfl(inc, 63, NOVA_WAVE);
    }
    if (lane == 0) before[words] = base;
  }
  __syncthreads();
  for (int w = tid; w < words; w += THREADS) {
    uint32_t m = bits[w];
    for (int at = before[w]; m; m &= m - 1, ++at) {
      const int i = w * 32 + __ffs(m) - 1;
      listed[at] = (uint16_t)i;
      page[at] = a.table[(int64_t)b * a.pitch + i];
    }
  }
  for (int i = tid; i < entries; i += THREADS) {
    int s;
    const int c = entry(i, s);
    if ((unsigned)c >= (unsigned)npages) continue;
    uint32_t* to = member + (before[c >> 5] + __popc(bits[c >> 5] & ((1u << (c & 31)) - 1))) * WORDS;
    if constexpr (WORDS == 1) {
      atomicOr(to, 1u << s);
    } else {
      // the 32-row parts of the block that hold rows of this query
      const int first = max((s_first + s) * a.G - row0, 0) >> 5, last = min(((s_first + s + 1) * a.G - 1 - row0) >> 5, WORDS - 1);
      for (int w = first; w <= last; ++w) {
        int unused;
        atomicOr(to + w, 1u << (s_first + s - div_by(row0 + w * 32, a.G, a.G_inv, unused)));
      }
    }
  }
  __syncthreads();
  return {listed, page, member, (int)before[words]};
}

// Which 16-byte chunk of row r (as a byte offset from row 0) the LDS tile of swz has in place p of that row: its inverse.
template <int ROWB>
__device__ __forceinline__ uint32_t swizzled_source(int r, int p) {
  const int x = p ^ ((swz<ROWB>(r, 0) - r * ROWB) >> 4);
  return r * ROWB + ((x ^ x >> (ROWB == 256 ? 3 : 2)) << 4);
}

// paged_few.hip: blocks of 16 mt rows, 4 or 8 waves (8: mt 1) that each take tiles of so many keys of their own
template <typename T> constexpr int paged_few_tile(int dh) { return 8192 / (dh * (int)sizeof(T)); }
template <typename T>
hipError_t launch_paged_few(hipStream_t st, int dh, int mt, int waves, unsigned grid, const PagedArgs<T>& a);

// paged_many.hip: blocks of so many rows, bf16
constexpr int kPagedRows = 128;
hipError_t launch_paged_many(hipStream_t st, int dh, unsigned grid, const PagedArgs<bf16_t>& a);

// paged_chosen.hip: the same, chosen pages.  LDS besides the list: two stages of keys and of values, a word per wave
constexpr int paged_chosen_lds(int dh) { return 2 * 2 * 64 * dh * 2 + 8 * 4; }
hipError_t launch_paged_chosen(hipStream_t st, int dh, unsigned grid, const PagedArgs<bf16_t>& a);
