// Attention over a cache in pages, blocks of 16 or 32 rows (a row: a query of one of the heads that share a key head): single
// tokens, a handful of queries, and queries that have chosen pages each for themselves.  What bounds it is reading the keys and
// values once: a token of four images, 32 heads of 128 on 8, up to 32 768 rows, 386 MB, 72 us or 5.4 TB/s; 41 MB of fp32 (two images of
// 2521 rows, 16 heads of 64, 5 queries) 13 us, which is the first latency and the joins.
//
// A workgroup is four or eight waves and one block of rows; tiles of keys are dealt to the waves, which share nothing until their results
// are joined at the end, so no tile waits at a barrier.  A tile is made of groups of 16 keys; a group lies in one page, wherever a
// page ends.  Everything is computed transposed, a lane owning one row of 16 (col) and the four lane groups (grp) parts of the keys:
//   S^T = K Q^T    16 keys x 16 rows per MFMA.  The order of the channels in that product is free, so the four lanes of a key take
//                  neighbouring 16 bytes of it, a line per key, straight into operands.
//   O^T += V^T P^T the order of the keys is free as well: the scores a lane holds after two S^T tiles (bf16), or one (fp32, whose
//                  operands are single numbers), are its operand as they are.  Values go from the pages into the wave's own LDS by
//                  rows, two tiles of it, and come back transposed (bf16), or four neighbouring channels a lane (fp32).
// Chosen pages: the block goes over the union of its queries' lists; where a row has not chosen a page its reference is -inf, which
// takes its weights to 0 and leaves scores that are no numbers to the second time (every key compared for itself: 59.4 -> 58.0 us, 1024
// queries, 32 heads of 128 on 8, 4 of 512 pages each; fp32, 512 queries, 16 of 128 pages, 64 channels 124 -> 121).
// A weight of 0 times a value that is no number is NaN, so what a row does not see could show in its result.  A wave whose sums end
// as anything but finite numbers goes over its tiles again, and takes those with such values in them key by key.
#include "paged.h"

namespace {

template <typename T, int DH, int MT, int NW, bool CHOSEN>
__global__ __launch_bounds__(NW * 64, 2) void few_kernel(PagedArgs<T> a) {
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr int TG = paged_few_tile<T>(DH) / kPageGroup;         // groups per tile
  constexpr int TG_SHIFT = TG == 4 ? 2 : TG == 2 ? 1 : 0;
  constexpr int ROWB = DH * (int)sizeof(T);
  constexpr int KC = ROWB / 64;                // 16-byte chunks of a key per lane
  constexpr int VG = 16 * ROWB / 1024, RPL = 1024 / ROWB > 0 ? 1024 / ROWB : 1;      // loads of values per group, rows per load
  constexpr int DT = DH / 16;                  // 16-channel blocks of the output
  constexpr int TILE = TG * 16 * ROWB, MINE = 2 * TILE;          // values of a tile; LDS of a wave, in the end its 16 x DH results
  static_assert(TILE == 8192 && TG * (KC + VG) == 16, "the wait for values counts sixteen loads behind them");
  __shared__ __attribute__((aligned(1024))) char lds[NW * MINE];
  __shared__ float part_m[NW][16], part_l[NW][16];
  extern __shared__ uint32_t lists[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int piece = blockIdx.x, nparts = a.nsplit;
  int split_i, b, j, block;
  a.place_block(div_by(piece, nparts, a.nsplit_inv, split_i), b, j, block);
  b = __builtin_amdgcn_readfirstlane(b);
  const int row0 = block * 16 * MT;
  const int rows = a.n * a.G, count = image_count(a.n_rows, b, a.n), live = count * a.G, len = image_prior(a.kv_rows, b, a.P);
  const int last = min(row0 + 16 * MT, live) - 1;                // last live row of the block
  int g_unused;
  const int s_first = div_by(row0, a.G, a.G_inv, g_unused), s_last = last < row0 ? s_first : div_by(last, a.G, a.G_inv, g_unused);
  // keys the first and the last query see
  const int seen_least = visible_keys(a.causal, len, count, s_first);
  const int seen_most = last < row0 ? 0 : visible_keys(a.causal, len, count, s_last);
  const int gshift = a.shift - 4, gmask = (1 << gshift) - 1;     // groups of a page
  const int32_t* table = a.table + (int64_t)b * a.pitch;

  ChosenPages list = {};
  int groups = (seen_most + 15) / 16;
  if constexpr (CHOSEN) {
    list = list_chosen<T, NW * 64, 1>(a, lists, b, j, row0, s_first, s_last, (seen_most + (1 << a.shift) - 1) >> a.shift);
    groups = list.count << gshift;
  }
  const int ntiles = (groups + TG - 1) / TG;
  // runs of one length whatever the image has, so that an image of any length is spread like the others; lists of chosen pages in
  // equal parts, since how long the union of several is nobody knows beforehand
  const int run = CHOSEN ? (ntiles + nparts - 1) / nparts : a.run_tiles;
  const int t0 = split_i * run, t1 = min(ntiles, t0 + run);
  if (nparts > 1 && t0 >= t1) {                                  // nothing for this one: nothing to be joined
    for (int rr = tid; rr < 16 * MT; rr += NW * 64) {
      const int64_t to = (int64_t)piece * 16 * MT + rr;
      a.part_ml[to * 2] = kNone;
      a.part_ml[to * 2 + 1] = 0.f;
    }
    return;
  }

  // A tile's groups, one per lane: first key (one that nobody sees where there is no such group), where its rows begin in a pool, and
  // how many bytes of rows of its page there are from there on (none where the page is none).  Looked up a tile ahead of the loads.
  struct Groups { int key0; uint32_t bytes, lo, hi; };
  const int64_t page_bytes = ((int64_t)a.hk << a.shift) * ROWB, head_at = ((int64_t)j << a.shift) * ROWB;
  auto look_up = [&](int t) {
    const int x = t * TG + (lane & (TG - 1)), u = min(x, max(groups, 1) - 1) >> gshift;
    Groups g = {1 << 30, 0u, 0u, 0u};
    int ordinal = u, page = -1;
    if (groups > 0) {
      if constexpr (CHOSEN) {
        page = list.page[u];
        ordinal = list.listed[u];
      } else {
        page = table[u];
      }
    }
    const int row = (x & gmask) * 16;
    const bool there = (unsigned)page < (unsigned)a.pages;
    const int64_t at = (there ? page : 0) * page_bytes + head_at + row * ROWB;
    if (x < groups) {
      g.key0 = (ordinal << a.shift) + row;
      if (there) g.bytes = min(max(len - g.key0, 0), (1 << a.shift) - row) * ROWB;
    }
    g.lo = (uint32_t)at;
    g.hi = (uint32_t)(at >> 32);
    return g;
  };
  // group i of a tile as a buffer: loads from where its page's rows end give zeros
  auto from = [&](const T* pool, const Groups& g, int i) {
    const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(g.hi, i) << 32 | (uint32_t)__builtin_amdgcn_readlane(g.lo, i);
    const uint64_t base = reinterpret_cast<uint64_t>(pool) + at;
    return u32x4{(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, (uint32_t)__builtin_amdgcn_readlane(g.bytes, i), 0x00020000u};
  };
  u32x4 kw[TG][KC];
  int key0[TG];                                                  // first keys of the tile's groups
  auto keys_of = [&](const Groups& g) {
#pragma unroll
    for (int i = 0; i < TG; ++i) key0[i] = __builtin_amdgcn_readlane(g.key0, i);
  };
  // that of the group behind i - 1's: in a tile of one page 16 rows further on
  const bool one_page = gshift >= TG_SHIFT;
  auto following = [&](u32x4 w, const T* pool, const Groups& g, int i) {
    if (!one_page) return from(pool, g, i);
    const uint64_t base = ((uint64_t)w[1] << 32 | w[0]) + 16 * ROWB;
    return u32x4{(uint32_t)base, (uint32_t)(base >> 32), (uint32_t)__builtin_amdgcn_readlane(g.bytes, i), 0x00020000u};
  };
  auto load_k = [&](const Groups& g) {
    u32x4 w = from(a.keys, g, 0);
#pragma unroll
    for (int i = 0; i < TG; ++i) {
      if (i > 0) w = following(w, a.keys, g, i);
      const auto buffer = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)w[1] << 32 | w[0]), 0, w[2], w[3]);
#pragma unroll
      for (int e = 0; e < KC; ++e) kw[i][e] = __builtin_amdgcn_raw_buffer_load_b128(buffer, col * ROWB + (e * 4 + grp) * 16, 0, 0);
    }
  };
  // bf16: the swizzle is made by which chunk of its row a lane asks for; fp32: rows as they are
  char* mine = lds + wave * MINE;
  const uint32_t mine0 = (uint32_t)reinterpret_cast<uintptr_t>((lptr_t)mine);
  uint32_t part[VG];
#pragma unroll
  for (int e = 0; e < VG; ++e) {
    if constexpr (WIDE) part[e] = e * 1024 + lane * 16;
    else part[e] = swizzled_source<ROWB>(e * RPL + lane / (64 / RPL), lane % (64 / RPL));
  }
  auto load_v = [&](int stage, const Groups& g) {
    u32x4 w = from(a.values, g, 0);
#pragma unroll
    for (int i = 0; i < TG; ++i) {
      if (i > 0) w = following(w, a.values, g, i);
      load_to_lds(w, mine0 + stage * TILE + i * VG * 1024, part);
    }
  };

  const int first = t0 + wave;
  Groups next = look_up(first);
  keys_of(next);
  if (first < t1) {
    load_v(0, next);
    load_k(next);
    next = look_up(first + NW);
  }
  // chunk grp + 4 e of row col; past the last live row its copies (padding is nobody's)
  u32x4 qf[MT][KC];
  int seen[MT], bit[MT];                                         // keys this lane's rows see, their queries' places in a word
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = max(min(row0 + mt * 16 + col, live - 1), 0);
    const T* qp = a.query(b, j, row) + grp * (16 / (int)sizeof(T));
#pragma unroll
    for (int e = 0; e < KC; ++e) qf[mt][e] = *reinterpret_cast<const u32x4*>(qp + e * (64 / (int)sizeof(T)));
    const int s = div_by(row, a.G, a.G_inv, g_unused);
    seen[mt] = visible_keys(a.causal, len, count, s);
    bit[mt] = s - s_first;
  }
  f32x4 o[MT][DT];
  float m_run[MT], l_run[MT];
  auto clear = [&] {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m_run[mt] = kNone;
      l_run[mt] = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[mt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  clear();
  // transposed reads: lane i of a group of sixteen names row 4 grp + i / 4 and 8-byte piece i % 4 of 16 channels
  int vaddr[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
    vaddr[d] = WIDE ? 0 : swz<WIDE ? 256 : ROWB>(4 * grp + (col >> 2), 2 * d + ((col & 3) >> 1)) + (col & 1) * 8;

  bool strict = false;                                           // the second time over the tiles
  int stage = 0;
  for (int t = first; t < t1;) {
    const bool more = t + NW < t1;
    const char* sv = mine + stage * TILE;
    uint32_t who[TG];
    if constexpr (CHOSEN)
#pragma unroll
      for (int i = 0; i < TG; ++i) who[i] = list.member[min(t * TG + i, groups - 1) >> gshift];
    // ---- scores: register r of group i is key 4 grp + r of it, for row col
    f32x4 s[MT][TG];
#pragma unroll
    for (int i = 0; i < TG; ++i)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        s[mt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < KC; ++e) {
          if constexpr (WIDE) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
              s[mt][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[i][e][c]), __uint_as_float(qf[mt][e][c]), s[mt][i], 0, 0, 0);
          } else {
            s[mt][i] = mfma16(__builtin_bit_cast(bf16x8, kw[i][e]), __builtin_bit_cast(bf16x8, qf[mt][e]), s[mt][i]);
          }
        }
      }
    if (more) {
      load_v(stage ^ 1, next);
      load_k(next);
    }

    // ---- keys that not every row of the block sees
    const bool masked = key0[TG - 1] >= (1 << 30) || key0[TG - 1] + 16 > seen_least;
    if (masked || (CHOSEN && strict)) {
      const float dead = a.scale_log2 < 0.f ? INFINITY : -INFINITY;
#pragma unroll
      for (int i = 0; i < TG; ++i)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const bool mine = !CHOSEN || ((who[i] >> bit[mt]) & 1u);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if ((CHOSEN && !mine) || key0[i] + 4 * grp + r >= seen[mt]) s[mt][i][r] = dead;
        }
    }
    bool careful = false;
    // the tile's values have landed: at most the sixteen loads of the next tile are still on the way
    asm volatile("" ::: "memory");
    if (more) __builtin_amdgcn_s_waitcnt(0x4F70);                // vmcnt(16)
    else __builtin_amdgcn_s_waitcnt(0x0F70);                     // vmcnt(0)
    asm volatile("" ::: "memory");
    if (strict && (masked || CHOSEN)) {
      uint32_t odd = 0u;
#pragma unroll 1
      for (int i = 0; i < TILE / 1024; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(sv + i * 1024 + lane * 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) odd |= WIDE ? odd_one(w[c]) : odd_pair(w[c]);
      }
      careful = __any(odd != 0u);
    }

    // ---- softmax: probabilities are 2^(score - m_run) against a reference that moves only when a sum of them says that some
    // score lies far above it, as any does above the first one
    float pr[MT][TG][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float psum = 0.f;
      auto probabilities = [&] {
        psum = 0.f;
#pragma unroll
        for (int i = 0; i < TG; ++i) {
          const float from = !CHOSEN || ((who[i] >> bit[mt]) & 1u) ? -m_run[mt] : -INFINITY;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            pr[mt][i][r] = __builtin_amdgcn_exp2f(fmaf(s[mt][i][r], a.scale_log2, from));
            psum += pr[mt][i][r];
          }
        }
      };
      auto largest = [&] {
        float tmax = -INFINITY;
#pragma unroll
        for (int i = 0; i < TG; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            tmax = fmaxf(tmax, !CHOSEN || ((who[i] >> bit[mt]) & 1u) ? s[mt][i][r] * a.scale_log2 : -INFINITY);
        return max_across_32(max_across_16(tmax));
      };
      auto move = [&](float tmax) {
        const float m_new = fmaxf(m_run[mt], tmax);
        const float alpha = __builtin_amdgcn_exp2f(m_run[mt] - m_new);
        l_run[mt] *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[mt][d] *= alpha;
        m_run[mt] = m_new;
      };
      probabilities();
      if (__any(!(psum <= kBig))) {
        move(largest());
        probabilities();
      }
      l_run[mt] += psum;
    }

    // ---- O^T += V^T P^T
    if constexpr (WIDE) {
      // register c of the d4-th four blocks of channels: channels 64 d4 + 4 row + c of the output's rows
      auto values = [&](int i, int r, int d4) {
        return *reinterpret_cast<const f32x4*>(sv + (i * 16 + 4 * grp + r) * ROWB + d4 * 256 + col * 16);
      };
      if (!careful) {
#pragma unroll
        for (int i = 0; i < TG; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int d4 = 0; d4 < DT / 4; ++d4) {
              const f32x4 v = values(i, r, d4);
#pragma unroll
              for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                  o[mt][d4 * 4 + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[c], pr[mt][i][r], o[mt][d4 * 4 + c], 0, 0, 0);
            }
      } else {
        // one key at a time: that of the lanes of group x.  Rows whose weight for it is 0 take nothing of it.
#pragma unroll
        for (int i = 0; i < TG; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll 1
            for (int x = 0; x < 4; ++x) {
              asm volatile("" ::: "memory");
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                const bool some = __shfl(pr[mt][i][r], col + 16 * x, NOVA_WAVE) != 0.f;
#pragma unroll
                for (int d4 = 0; d4 < DT / 4; ++d4) {
                  const f32x4 v = values(i, r, d4);
#pragma unroll
                  for (int c = 0; c < 4; ++c) {
                    const f32x4 one = __builtin_amdgcn_mfma_f32_16x16x4f32(grp == x ? v[c] : 0.f, grp == x ? pr[mt][i][r] : 0.f,
                                                                           f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                    if (some) o[mt][d4 * 4 + c] += one;
                  }
                }
              }
            }
      }
    } else {
#pragma unroll
      for (int u = 0; u < TG / 2; ++u) {                         // 32 keys at a time
        const char* at = sv + u * 32 * ROWB;
        bf16x8 pf[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < 8; ++e) pf[mt][e] = (bf16_t)pr[mt][2 * u + (e >> 2)][e & 3];
        if (!careful) {
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const bf16x8 vf = join(read_transposed(at + vaddr[d]), read_transposed(at + vaddr[d] + 16 * ROWB));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][d] = mfma16(vf, pf[mt], o[mt][d]);
          }
        } else {
          // one key at a time: element e of the lanes of group x
#pragma unroll 1
          for (int ex = 0; ex < 32; ++ex) {
            const int e = ex >> 2, x = ex & 3;
            asm volatile("" ::: "memory");                       // read the values again: held in registers they would be spilled
            const uint32_t half = grp == x ? (e & 1 ? 0xFFFF0000u : 0xFFFFu) : 0u;
            u32x4 only;
#pragma unroll
            for (int c = 0; c < 4; ++c) only[c] = c == e >> 1 ? half : 0u;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              const u32x4 w = __builtin_bit_cast(u32x4, pf[mt]) & only;
              const uint32_t weight = __shfl(w[0] | w[1] | w[2] | w[3], col + 16 * x, NOVA_WAVE);
#pragma unroll
              for (int d = 0; d < DT; ++d) {
                const bf16x8 vf = join(read_transposed(at + vaddr[d]), read_transposed(at + vaddr[d] + 16 * ROWB));
                const f32x4 one = mfma16(__builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, vf) & only), __builtin_bit_cast(bf16x8, w),
                                         f32x4{0.f, 0.f, 0.f, 0.f});
                if (weight) o[mt][d] += one;
              }
            }
          }
        }
      }
    }
    keys_of(next);
    if (t + 2 * NW < t1) next = look_up(t + 2 * NW);
    t += NW;
    stage ^= 1;
    if (t >= t1 && !strict) {
      float sum = 0.f;                                           // 0, or NaN where some number is none
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) sum = fmaf(o[mt][d][r], 0.f, sum);
      if (__any(sum != 0.f)) {
        strict = true;
        clear();
        t = first;
        next = look_up(first);
        keys_of(next);
        load_v(stage, next);
        load_k(next);
        next = look_up(first + NW);
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
    for (int d = 0; d < DT; ++d) {
      // fp32: register r of block d is channel 64 (d / 4) + 16 grp + 4 r + d % 4
      const int c4 = WIDE ? d / 4 * 16 + grp * 4 + d % 4 : d * 4 + grp;
      f32x4 v = o[mt][d];
      if constexpr (WIDE)
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = o[mt][d / 4 * 4 + c][d % 4];
      *reinterpret_cast<f32x4*>(mine + (c4 * 16 + col) * 16) = v;
    }
    __syncthreads();
    for (int i = tid; i < 16 * (DH / 4); i += NW * 64) {
      const int c4 = i % (DH / 4), rr = i / (DH / 4), row = row0 + mt * 16 + rr;
      if (row >= rows) continue;
      float m = kNone, lt = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, part_m[w][rr]);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = __builtin_amdgcn_exp2f(part_m[w][rr] - m);
        lt = fmaf(f, part_l[w][rr], lt);
        acc += f * *reinterpret_cast<const f32x4*>(lds + w * MINE + (c4 * 16 + rr) * 16);
      }
      if (nparts == 1) {
        const int s = div_by(row, a.G, a.G_inv, g_unused), visible = visible_keys(a.causal, len, count, s);
        bool some = row < live && visible > 0;
        if (CHOSEN && lt == 0.f) some = some && sees_chosen(a, b, j, s, visible);
        const int64_t to = a.out_row(b, j, row);
        store_four(a.out + to * DH + c4 * 4, some ? acc : f32x4{0.f, 0.f, 0.f, 0.f}, some ? 1.0f / lt : 0.f);
        if (a.lse && c4 == 0) a.lse[to] = some ? (m + __builtin_amdgcn_logf(lt)) * kLn2 : -INFINITY;
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
hipError_t launch_paged_few(hipStream_t st, int dh, int mt, int waves, unsigned grid, const PagedArgs<T>& a) {
  const size_t lists = a.chosen ? chosen_bytes(a.most_pages, a.most_listed, 1) : 0;
#define GO(DH, MT, NW, CHOSEN) few_kernel<T, DH, MT, NW, CHOSEN><<<grid, NW * 64, CHOSEN ? (lists + 15) / 16 * 16 : 0, st>>>(a)
#define ONE(DH, CHOSEN) do { if (waves == 8) GO(DH, 1, 8, CHOSEN); else GO(DH, 1, 4, CHOSEN); } while (0)
  if (mt == 1) {
    if (dh == 64) { if (a.chosen) ONE(64, true); else ONE(64, false); }
    else { if (a.chosen) ONE(128, true); else ONE(128, false); }
  } else if constexpr (sizeof(T) == 4) {
    if (dh != 64 || a.chosen) return hipErrorInvalidValue;       // 16 rows there
    GO(64, 2, 4, false);
  } else {
    if (dh == 64) { if (a.chosen) GO(64, 2, 4, true); else GO(64, 2, 4, false); }
    else { if (a.chosen) GO(128, 2, 4, true); else GO(128, 2, 4, false); }
  }
#undef ONE
#undef GO
  return hipGetLastError();
}
template hipError_t launch_paged_few<bf16_t>(hipStream_t, int, int, int, unsigned, const PagedArgs<bf16_t>&);
template hipError_t launch_paged_few<float>(hipStream_t, int, int, int, unsigned, const PagedArgs<float>&);
