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
};

// paged_few.hip: blocks of 16 mt rows, four waves that each take tiles of so many keys of their own
template <typename T> constexpr int paged_few_tile(int dh) { return 8192 / (dh * (int)sizeof(T)); }
template <typename T>
hipError_t launch_paged_few(hipStream_t st, int dh, int mt, unsigned grid, const PagedArgs<T>& a);
