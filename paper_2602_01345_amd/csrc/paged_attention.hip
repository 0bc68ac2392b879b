// Attention over a cache in pages: how a call is divided over workgroups, and the joining of key runs.
#include <algorithm>
#include <cfloat>

#include "paged.h"

namespace {

// The runs of the cut items joined: out = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m).  A thread has four channels of
// one row and every SL-th run; with many runs per row the threads of a row join through LDS.  Runs that had no tiles have
// left a sum of 0 and nothing else.
template <typename T, int DH, int SL>
__global__ __launch_bounds__(256) void join_kernel(PagedArgs<T> a, int block_rows, int used_rows) {
  constexpr int C4 = DH / 4, RPW = 256 / (C4 * SL);
  __shared__ f32x4 part_o[SL > 1 ? 256 : 1];
  __shared__ float part_m[SL > 1 ? 256 / C4 : 1], part_l[SL > 1 ? 256 / C4 : 1];
  const int tid = threadIdx.x, c4 = tid % C4, sl = tid / C4 % SL;
  const int64_t r = (int64_t)blockIdx.x * RPW + tid / (C4 * SL);
  const int ci = (int)(r / used_rows), rr = (int)(r - (int64_t)ci * used_rows);
  int b, j, block, g_unused;
  a.place_block(min(a.n_whole + ci, a.items - 1), b, j, block);
  const int row = block * block_rows + rr;
  const bool there = a.n_whole + ci < a.items && row < a.n * a.G;
  const int count = image_count(a.n_rows, b, a.n), len = image_prior(a.kv_rows, b, a.P);
  const int s_row = div_by(there ? row : 0, a.G, a.G_inv, g_unused);
  const int visible = visible_keys(a.causal, len, count, s_row);
  bool some = there && s_row < count && visible > 0;
  const int64_t p0 = (int64_t)ci * a.nsplit * block_rows + rr;
  float m = kNone, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s = sl; some && s < a.nsplit; s += SL) {
    const int64_t p = p0 + (int64_t)s * block_rows;
    const float ms = a.part_ml[p * 2], ls = a.part_ml[p * 2 + 1];
    if (ls == 0.f) continue;
    const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + p * DH + c4 * 4);
    const float mn = fmaxf(m, ms);
    const float w0 = __builtin_amdgcn_exp2f(m - mn), w1 = __builtin_amdgcn_exp2f(ms - mn);
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
      const float w = __builtin_amdgcn_exp2f(part_m[g + s] - m);
      l = fmaf(w, part_l[g + s], l);
      acc += w * part_o[tid + s * C4];
    }
  }
  if (!there) return;
  if (a.chosen && l == 0.f) some = some && sees_chosen(a, b, j, s_row, visible);
  const int64_t to = a.out_row(b, j, row);
  store_four(a.out + to * DH + c4 * 4, some ? acc : f32x4{0.f, 0.f, 0.f, 0.f}, some ? 1.0f / l : 0.f);
  if (a.lse && c4 == 0) a.lse[to] = some ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// How a call is divided: mt > 0: blocks of 16 mt rows (paged_few.hip), else blocks of kPagedRows (paged_many.hip); items below n_whole
// are one workgroup each, the others nsplit runs (of run_tiles tiles where that is not 0).
struct Plan {
  int mt, waves, block_rows, blocks, items, n_whole, nsplit, run_tiles, ranked, listed;
  int64_t runs() const { return nsplit > 1 ? (int64_t)(items - n_whole) * nsplit : 0; }
};
constexpr int kCus = 256;
constexpr size_t kMostList = 160 * 1024 / 2 - paged_chosen_lds(128);
constexpr int kRanked = 32;          // most images that are ranked: every workgroup does it for itself, a step per image
Plan plan(const nova_paged_cache& c, int B, int heads, int n, int kv_len, int take, bool ragged) {
  const int G = heads / c.kv_heads, rows = n * G;
  const bool wide = c.dtype == NOVA_F32;
  Plan p = {};
  const int pages = (kv_len + c.page_rows - 1) / c.page_rows;
  // pages that the queries of a block of so many rows may have chosen
  auto listed = [&](int block_rows) {
    return take > 0 ? (int)std::min<int64_t>(pages, (int64_t)std::min({block_rows, (block_rows - 1) / G + 2, n}) * take) : 0;
  };
  // Rows that share what is read of a page, and registers of rows against waves:
  //   fp32   16 with heads of 128 and where pages are chosen, else up to 32 (us in blocks of 16 / of 32; 1024 queries, 4096 keys, 16 heads
  //          of 128 320 / 352, of 64 178 / 150; 512 queries over 16 of 128 pages, 32 heads of 128 on 8 227 / 329, of 64 130 / 152)
  //   bf16   128 from 33 on, but with heads of 64 up to two blocks of 32 per CU over up to 2048 keys are left as they are: no tile waits
  //          for the others, and nothing is joined afterwards (us in blocks of 32 / of 128; 8 images of 128 queries, 16 heads of 64:
  //          256 keys 9.5 / 9.2, 512 12.0 / 17.4, 1024 17.0 / 21.9, 2048 26.7 / 29.0, 4096 47.3 / 41.5; 4 images of 256, 16 heads of 128:
  //          256 16.4 / 12.9, 512 20.9 / 22.6, 1024 30.7 / 30.0, 2048 47.9 / 38.8)
  //   bf16, chosen pages   128 (paged_chosen.hip) where the lists of a block's queries together hold half as many pages as there are, so
  //          that they share some, if there are blocks for a quarter of the CUs and the list leaves room for a second workgroup with
  //          heads of 128 in the LDS (16 heads of 128, 1024 queries, 32 of so many pages of 16 rows: 732 106 / 102, 736, whose list does not,
  //          100 / 159; heads of 64 have room for longer ones, which gain with long pages alone: 1024 pages of 16 rows 69 / 88, of 64 295 /
  //          263, 2048 of 16 78 / 105) (us in blocks of 32 / of 128; 32 heads of 128 on 8, 1024 queries, of 512 pages 128 chosen 853 / 439, 32 352 / 252, 8
  //          113 / 107, 4 60 / 64; 4 images of 64, 8 of 128 pages, 64 blocks of 128, 39 / 45; 2 of 500, 12 heads on 4, 20 of 256 pages, 96
  //          blocks, 74 / 67; 16 heads of 64, 2000 queries, 32 of 256 pages 224 / 174); 16 where blocks are few (in blocks of 16 / of 32;
  //          32 heads of 128 on 8, 2 images of 20 queries, 16 of 512 pages 25 / 31; 128 queries, 32 of 512 66 / 62)
  const int64_t heads_all = (int64_t)B * c.kv_heads, blocks32 = heads_all * ((rows + 31) / 32);
  if (rows <= 16 || (wide && (c.dh == 128 || take > 0))) p.mt = 1;
  else if (rows <= 32 || wide) p.mt = 2;
  else if (take == 0) p.mt = c.dh == 64 && blocks32 <= 2 * kCus && kv_len <= 2048 ? 2 : 0;
  else if (blocks32 <= kCus / 4) p.mt = 1;
  else
    p.mt = heads_all * ((rows + kPagedRows - 1) / kPagedRows) > kCus / 4 &&
           2 * (int64_t)std::min((kPagedRows - 1) / G + 2, n) * take >= (int64_t)pages &&
           chosen_bytes(pages, listed(kPagedRows), kPagedRows / 32) <= kMostList ? 0 : 2;
  p.block_rows = p.mt ? 16 * p.mt : kPagedRows;
  p.blocks = (rows + p.block_rows - 1) / p.block_rows;
  p.items = B * c.kv_heads * p.blocks;
  p.n_whole = p.items;
  p.nsplit = 1;
  p.waves = 4;
  p.listed = listed(p.block_rows);
  if (p.mt) {
    const int tile = wide ? paged_few_tile<float>(c.dh) : paged_few_tile<bf16_t>(c.dh);
    // most keys a block goes over: all, or what its queries may have chosen
    const int64_t keys = take > 0 ? (int64_t)p.listed * c.page_rows : kv_len;
    const int ntiles = (int)((keys + tile - 1) / tile);
    p.run_tiles = ntiles;
    const int want = std::min((8 * kCus + p.items - 1) / p.items, ntiles);       // waves per item: eight per CU, a tile each
    // Blocks of 16 rows that stay whole, eight waves of one workgroup, so that nothing is joined by a second launch: up to 12 tiles,
    // more of them the more blocks there are, whose tiles the chip can only read one after the other anyway (us in runs and joined /
    // in one launch, tiles of 32 keys, heads of 128 in bf16: 32 blocks 8 tiles 8.0 / 6.5, 16 9.2 / 8.1, 24 7.9 / 10.2; 128 blocks 16
    // 11.8 / 8.9, 48 22.3 / 19.2, 96 35.9 / 33.2; fp32, tiles of 16: 32 blocks 8 8.3 / 7.0, 16 9.7 / 10.0; 128 blocks 48 23.8 / 22.4, 96
    // 37.7 / 38.1)
    if (want > 4 && p.mt == 1 && ntiles <= std::max(12, p.items * 3 / 8)) {
      p.waves = 8;
    } else if (want > 4) {
      p.run_tiles = std::max((ntiles + want / 4 - 1) / (want / 4), 4);
      p.nsplit = (ntiles + p.run_tiles - 1) / p.run_tiles;
      if (p.nsplit > 1) p.n_whole = 0;
    }
    return p;
  }
  const int ntiles = (int)(((take > 0 ? (int64_t)p.listed * c.page_rows : kv_len) + 63) / 64), slots = 2 * kCus, rest = p.items % slots;
  // Images with lengths of their own: the longest first, so that short ones fill up the end; from two rounds of items on that is
  // enough and none is cut (us in this order / in that of the images, the rest cut; 8 images of 512 queries, 36 heads of 64, up to 2048
  // keys 84 / 90; of 700, 16 heads of 128, up to 8000 303 / 302; 16 of 300, 32 heads of 128 on 8, up to 8000 460 / 452).
  p.ranked = ragged && p.items > slots && B > 1 && B <= kRanked ? B : 0;
  if (rest == 0 || (p.ranked && p.items >= 2 * slots)) return p;
  // A few more items than CUs, and long ones: most CUs would have one, which is little to hide anything behind, and the others two
  // (us in three runs each / whole; 272 items of 8000 keys, heads of 128, 174 / 201, 306 186 / 230, 280 of 16 000 318 / 399; heads of 64,
  // of which three items share a CU: 272 of 4096 72 / 71; chosen pages, heads of 128: 272 items, 32 of 512 pages of 64 rows 462 / 636, of
  // 16 rows 186 / 206, 8 of 512 of 64 248 / 301, 304 items, 32 of 256 of 64 315 / 411, 320, 16 of 128 of 64 187 / 215).
  const bool in_three = c.dh == 128 && p.items > kCus && p.items <= kCus + kCus / 4 && ntiles >= 64;
  const int s = in_three ? 3 : std::min(slots / rest, ntiles / 4);
  if (s >= 2) {
    p.n_whole = p.items - rest;
    p.nsplit = s;
  }
  return p;
}

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

template <typename T>
hipError_t attend(hipStream_t st, const PagedCall& call) {
  const nova_paged_cache& c = *call.cache;
  const Plan p = plan(c, call.B, call.heads, call.n, call.kv_len, call.take, call.kv_rows != nullptr);
  PagedArgs<T> a = {};
  a.q = static_cast<const T*>(call.q.data);
  a.q_sb = call.q.stride_b; a.q_sr = call.q.stride_row; a.q_sh = call.q.stride_head;
  a.heads = call.heads; a.hk = c.kv_heads; a.G = call.heads / c.kv_heads; a.n = call.n; a.P = call.kv_len;
  a.n_rows = call.n_rows; a.kv_rows = call.kv_rows;
  // Keys that a row does not see have scores of -inf, which a scale of 0 would make NaN.  The smallest positive fp32 number
  // (2^-149) in its place leaves less than 2^-21 of any finite score: no two weights differ by more than that.
  a.scale_log2 = call.scale_log2 == 0.f ? FLT_TRUE_MIN : call.scale_log2;
  a.out = static_cast<T*>(call.out);
  a.lse = call.lse;
  a.keys = static_cast<const T*>(c.k_pages);
  a.values = static_cast<const T*>(c.v_pages);
  a.table = call.table; a.pitch = call.pitch; a.pages = c.pages; a.shift = __builtin_ctz(c.page_rows); a.causal = call.causal;
  a.chosen = call.chosen; a.take = call.take;
  a.most_pages = (call.kv_len + c.page_rows - 1) / c.page_rows;
  a.most_listed = p.listed;
  a.take_inv = div_inv(call.take);
  a.blocks = p.blocks; a.items = p.items; a.dealt = p.items / (8 * p.blocks) * 8 * p.blocks;
  a.blocks_inv = div_inv(p.blocks); a.hk_inv = div_inv(c.kv_heads); a.G_inv = div_inv(a.G); a.nsplit_inv = div_inv(p.nsplit);
  a.n_whole = p.n_whole; a.nsplit = p.nsplit; a.run_tiles = p.run_tiles; a.ranked = p.ranked;
  a.part_o = static_cast<float*>(call.workspace);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(call.workspace) + up256((size_t)p.runs() * p.block_rows * c.dh * 4));
  const unsigned grid = (unsigned)(p.n_whole + p.runs());
  hipError_t e;
  if constexpr (sizeof(T) == 4) e = launch_paged_few<T>(st, c.dh, p.mt, p.waves, grid, a);
  else if (p.mt) e = launch_paged_few<T>(st, c.dh, p.mt, p.waves, grid, a);
  else e = a.chosen ? launch_paged_chosen(st, c.dh, grid, a) : launch_paged_many(st, c.dh, grid, a);
  if (e != hipSuccess || p.nsplit == 1) return e;
  const int used = std::min(p.block_rows, call.n * a.G);         // rows of a block that there are, where it is the only one
  const int64_t rows = (int64_t)(p.items - p.n_whole) * used;
#define GO(DH, SL) join_kernel<T, DH, SL><<<(unsigned)((rows * (DH / 4 * SL) + 255) / 256), 256, 0, st>>>(a, p.block_rows, used)
  if (c.dh == 64) { if (p.nsplit > 4) GO(64, 8); else GO(64, 1); }
  else { if (p.nsplit > 4) GO(128, 8); else GO(128, 1); }
#undef GO
  return hipGetLastError();
}

}  // namespace

size_t paged_attention_workspace_bytes(const nova_paged_cache& c, int B, int heads, int n, int kv_len, int take) {
  const Plan p = plan(c, B, heads, n, kv_len, take, false);      // of the two the one that asks for more
  if (p.nsplit == 1) return 0;
  const size_t rows = (size_t)p.runs() * p.block_rows;
  return up256(rows * c.dh * 4) + up256(rows * 8);
}

hipError_t launch_paged_attention(hipStream_t st, const PagedCall& call) {
  return call.cache->dtype == NOVA_BF16 ? attend<bf16_t>(st, call) : attend<float>(st, call);
}
