// The key/value cache in pages (include/nova.h) as its kernels take it.
#pragma once
#include "attention_core.h"
#include "nova_internal.h"

constexpr int kPageGroup = 16;           // rows that never lie in two pages: pages have 2^shift rows, 16 at least

// A (page, key head)'s rows as a buffer: `rows` of them exist, loads from there on give zeros.  A page that is none of the pool
// has no rows, so that no table leads a load out of it.
template <typename T, int DH>
__device__ __forceinline__ auto page_buffer(const T* pool, int page, int pages, int hk, int j, int shift, int rows) {
  const bool there = (unsigned)page < (unsigned)pages;
  const T* base = pool + ((((int64_t)(there ? page : 0) * hk + j) << shift) * DH);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, there ? rows * (int)(DH * sizeof(T)) : 0, 0x00020000);
}

// The same as the four words of a buffer, for loads that go into LDS.  They are written in assembly: the compiler, which cannot tell
// which LDS a transposed read may meet, would make every such read wait for all of them.  They have no output registers, and who
// reads what they bring waits for vmcnt(0) and at a barrier first.
template <typename T, int DH>
__device__ __forceinline__ u32x4 page_words(const T* pool, int page, int pages, int hk, int j, int shift, int rows) {
  const bool there = (unsigned)page < (unsigned)pages;
  const uint64_t base = reinterpret_cast<uint64_t>(pool + ((((int64_t)(there ? page : 0) * hk + j) << shift) * DH));
  return u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, there ? rows * (uint32_t)(DH * sizeof(T)) : 0u, 0x00020000u};
}
// 16 bytes per lane of keys and of values from lane_off + off (off, to_k, to_v: of the whole wave) to 1 KB of LDS each.  The waits in
// front of the loads are those that the hardware asks for: five states after a vector instruction that wrote a scalar register
// which a load reads (the compiler does not look for that here), one after a write of m0.
__device__ __forceinline__ void load_to_lds(u32x4 keys, u32x4 values, uint32_t to_k, uint32_t to_v, uint32_t lane_off, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, %5 offen lds\n\t"
               "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %4, %5 offen lds"
               :: "s"(to_k), "s"(to_v), "v"(lane_off), "s"(keys), "s"(values), "s"(off) : "memory");
}
// A number of a list that all lanes of a wave ask for alike, by a scalar load.
__device__ __forceinline__ int load_scalar(const int32_t* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p));
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

  // Image, key head and block of rows of an item: as AttentionItems::place, images by falling length where they are ranked, and the
  // blocks that see most first.
  __device__ __forceinline__ void place_block(int item, int& b, int& j, int& block) const {
    this->place(item, b, j, block);
    if (this->ranked) b = this->by_length(b);
    if (causal) block = this->blocks - 1 - block;
  }
};

// some bf16 number of the two in w is no finite one: an exponent of ones carries into the bit above it
__device__ __forceinline__ uint32_t odd_pair(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t odd_one(uint32_t w) { return ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u; }

// Which 16-byte chunk of row r (as a byte offset from row 0) the LDS tile of swz has in place p of that row: its inverse.
template <int ROWB>
__device__ __forceinline__ uint32_t swizzled_source(int r, int p) {
  const int x = p ^ ((swz<ROWB>(r, 0) - r * ROWB) >> 4);
  return r * ROWB + ((x ^ x >> (ROWB == 256 ? 3 : 2)) << 4);
}

// paged_few.hip: blocks of 16 mt rows, four waves that each take tiles of so many keys of their own
template <typename T> constexpr int paged_few_tile(int dh) { return 8192 / (dh * (int)sizeof(T)); }
template <typename T>
hipError_t launch_paged_few(hipStream_t st, int dh, int mt, unsigned grid, const PagedArgs<T>& a);

// paged_many.hip: blocks of so many rows, bf16
constexpr int kPagedRows = 128;
hipError_t launch_paged_many(hipStream_t st, int dh, unsigned grid, const PagedArgs<bf16_t>& a);
