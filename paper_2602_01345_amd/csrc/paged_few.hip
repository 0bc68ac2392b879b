// Attention over a cache in pages, blocks of 16 or 32 rows (a row: a query of one of the heads that share a key head): single
// tokens, a handful of queries, and queries that have chosen pages each for themselves.  What bounds it is reading the keys and
// values once.
//
// A workgroup is four waves and one block of rows; tiles of keys are dealt to the waves, which share nothing until their results
// are joined at the end, so no tile waits at a barrier.  A tile is made of groups of 16 keys; a group lies in one page, wherever a
// page ends.  Everything is computed transposed, a lane owning one row of 16 (col) and the four lane groups (grp) parts of the keys:
//   S^T = K Q^T    16 keys x 16 rows per MFMA.  The order of the channels in that product is free, so the four lanes of a key take
//                  neighbouring 16 bytes of it, a line per key, straight into operands.
//   O^T += V^T P^T the order of the keys is free as well: the scores a lane holds after two S^T tiles (bf16), or one (fp32, whose
//                  operands are single numbers), are its operand as they are.  bf16 values pass through the wave's own LDS, laid by
//                  rows and read back transposed; fp32 values come from memory as operands, four neighbouring channels a lane.
// Chosen pages: the block's list is the union of its queries' lists, made in LDS as a bitmap over the image's pages (so that the
// order of the lists, repeats and entries that are no pages do not matter), with a word per listed page that says which queries chose it.
#include "paged.h"

namespace {

constexpr int kWaves = 4;

template <typename T, int DH, int MT, bool CHOSEN>
__global__ __launch_bounds__(kWaves * 64, 2) void few_kernel(PagedArgs<T> a) {
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr int TG = paged_few_tile<T>(DH) / kPageGroup;         // groups per tile
  constexpr int ROWB = DH * (int)sizeof(T);
  constexpr int KC = ROWB / 64;                // 16-byte chunks of a key per lane
  constexpr int RPL = WIDE ? 4 : 1024 / ROWB;  // rows of values per load of the wave (fp32: each of 64 channels)
  constexpr int VG = 16 * ROWB / 1024;         // loads of values per group
  constexpr int DT = DH / 16;                  // 16-channel blocks of the output
  constexpr int HALF = 16 * DH * 4;            // LDS of a wave: 32 rows of bf16 values, then its 16 x DH results
  __shared__ __attribute__((aligned(1024))) char lds[kWaves * HALF];
  __shared__ float part_m[kWaves][16], part_l[kWaves][16];
  extern __shared__ uint32_t lists[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int piece = blockIdx.x, nparts = a.nsplit;
  int split_i, b, j, block;
  a.place_block(div_by(piece, nparts, a.nsplit_inv, split_i), b, j, block);
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

  // ---- the block's list of chosen pages: ascending ordinals, and who chose them
  uint16_t* listed = nullptr;
  uint32_t* member = nullptr;
  int groups = (seen_most + 15) / 16;
  if constexpr (CHOSEN) {
    const int npages = (seen_most + (1 << a.shift) - 1) >> a.shift, words = (npages + 31) / 32, most_words = (a.most_pages + 31) / 32;
    uint32_t* bits = lists;
    uint32_t* before = lists + most_words;                       // listed pages in front of a word
    member = lists + 2 * most_words + 1;
    listed = reinterpret_cast<uint16_t*>(member + a.most_listed);
    const int entries = (s_last - s_first + 1) * a.take;
    const int32_t* chosen = a.chosen + (((int64_t)b * a.n + s_first) * a.hk + j) * a.take;
    auto entry = [&](int i, int& s) {
      s = i / a.take;
      return chosen[(int64_t)s * a.hk * a.take + (i - s * a.take)];
    };
    for (int w = tid; w < words; w += kWaves * 64) bits[w] = 0u;
    for (int w = tid; w < a.most_listed; w += kWaves * 64) member[w] = 0u;
    __syncthreads();
    for (int i = tid; npages > 0 && i < entries; i += kWaves * 64) {
      int s;
      const int c = entry(i, s);
      if ((unsigned)c < (unsigned)npages) atomicOr(&bits[c >> 5], 1u << (c & 31));
    }
    __syncthreads();
    if (wave == 0) {
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
    groups = (int)before[words] << gshift;
    for (int w = tid; w < words; w += kWaves * 64) {
      uint32_t m = bits[w];
      for (int at = before[w]; m; m &= m - 1) listed[at++] = (uint16_t)(w * 32 + __ffs(m) - 1);
    }
    for (int i = tid; npages > 0 && i < entries; i += kWaves * 64) {
      int s;
      const int c = entry(i, s);
      if ((unsigned)c < (unsigned)npages)
        atomicOr(&member[before[c >> 5] + __popc(bits[c >> 5] & ((1u << (c & 31)) - 1))], 1u << s);
    }
    __syncthreads();
  }
  const int ntiles = (groups + TG - 1) / TG;
  // runs of one length whatever the image has, so that an image of any length is spread like the others
  const int t0 = split_i * a.run_tiles, t1 = min(ntiles, t0 + a.run_tiles);
  if (nparts > 1 && t0 >= t1) {                                  // nothing for this one: nothing to be joined
    for (int rr = tid; rr < 16 * MT; rr += kWaves * 64) {
      const int64_t to = (int64_t)piece * 16 * MT + rr;
      a.part_ml[to * 2] = -INFINITY;
      a.part_ml[to * 2 + 1] = 0.f;
    }
    return;
  }

  // Pages of a tile, one lane per group: loaded a tile ahead of what is loaded through them.
  struct Pages { int ordinal, page; };
  auto look_up = [&](int t) {
    const int x = min(t * TG + (lane & (TG - 1)), max(groups, 1) - 1);
    Pages p;
    p.ordinal = x >> gshift;
    if constexpr (CHOSEN) p.ordinal = groups > 0 ? listed[p.ordinal] : 0;
    p.page = groups > 0 ? table[p.ordinal] : -1;
    return p;
  };
  u32x4 kw[TG][KC], vw[TG * VG];
  int key0[TG];                                                  // first key of the tile's groups
  auto group_key = [&](const Pages& p, int t, int i) {
    const int x = t * TG + i;
    const int first = (__builtin_amdgcn_readlane(p.ordinal, i) << a.shift) + ((x & gmask) << 4);
    return x < groups ? first : 1 << 30;                         // no such group: its keys are seen by nobody
  };
  auto buffer = [&](const T* pool, const Pages& p, int t, int i, uint32_t& at) {
    const int x = t * TG + i, ordinal = __builtin_amdgcn_readlane(p.ordinal, i);
    const int there = x < groups ? min(max(len - (ordinal << a.shift), 0), 1 << a.shift) : 0;
    at = (x & gmask) * 16 * ROWB;
    return page_buffer<T, DH>(pool, __builtin_amdgcn_readlane(p.page, i), a.pages, a.hk, j, a.shift, there);
  };
  auto load_k = [&](int t, const Pages& p) {
#pragma unroll
    for (int i = 0; i < TG; ++i) {
      uint32_t at;
      const auto from = buffer(a.keys, p, t, i, at);
#pragma unroll
      for (int e = 0; e < KC; ++e)
        kw[i][e] = __builtin_amdgcn_raw_buffer_load_b128(from, col * ROWB + (e * 4 + grp) * 16, at, 0);
    }
  };
  auto load_v = [&](int t, const Pages& p) {
#pragma unroll
    for (int i = 0; i < TG; ++i) {
      uint32_t at;
      const auto from = buffer(a.values, p, t, i, at);
#pragma unroll
      for (int e = 0; e < VG; ++e) {
        if constexpr (WIDE)                                      // row 4 grp + r, channels 64 d + 4 col .. + 3; e = r DH / 64 + d
          vw[i * VG + e] = __builtin_amdgcn_raw_buffer_load_b128(from, (4 * grp + e / (DH / 64)) * ROWB + (e % (DH / 64)) * 256 + col * 16, at, 0);
        else
          vw[i * VG + e] = __builtin_amdgcn_raw_buffer_load_b128(from, lane * 16, at + e * 1024, 0);
      }
    }
  };

  const int first = t0 + wave;
  Pages pages = look_up(first), pages_next = look_up(first + kWaves);
  if (first < t1) {
    load_k(first, pages);
    load_v(first, pages);
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
  if constexpr (!WIDE) {
    const int r = 4 * grp + (col >> 2);
#pragma unroll
    for (int d = 0; d < DT; ++d) vaddr[d] = swz<ROWB>(r, 2 * d + ((col & 3) >> 1)) + (col & 1) * 8;
  }
  // values of 32 keys through the wave's LDS (its reads and writes are done in order)
  auto lay = [&](int u) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 2 * VG; ++i)
      *reinterpret_cast<u32x4*>(sv + swz<WIDE ? 256 : ROWB>(i * RPL + lane / (64 / RPL), lane % (64 / RPL))) = vw[u * 2 * VG + i];
    asm volatile("" ::: "memory");
  };

  for (int t = first; t < t1; t += kWaves) {
    const bool more = t + kWaves < t1;
#pragma unroll
    for (int i = 0; i < TG; ++i) key0[i] = group_key(pages, t, i);
    uint32_t who[TG];
    if constexpr (CHOSEN)
#pragma unroll
      for (int i = 0; i < TG; ++i) who[i] = member[min((t * TG + i), groups - 1) >> gshift];
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
    if (more) load_k(t + kWaves, pages_next);

    // ---- keys that not every row of the block sees
    bool masked = CHOSEN || key0[TG - 1] >= (1 << 30) || key0[TG - 1] + 16 > seen_least;
    if (masked) {
      const float dead = a.scale_log2 < 0.f ? INFINITY : -INFINITY;
#pragma unroll
      for (int i = 0; i < TG; ++i)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const bool mine = !CHOSEN || ((who[i] >> bit[mt]) & 1u);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!mine || key0[i] + 4 * grp + r >= seen[mt]) s[mt][i][r] = dead;
        }
      // a weight of 0 times a value that is no number would be one of NaN: such tiles take their values key by key below
      uint32_t odd = 0u;
#pragma unroll
      for (int i = 0; i < TG * VG; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) odd |= WIDE ? odd_one(vw[i][c]) : odd_pair(vw[i][c]);
      masked = __any(odd != 0u);
    }
    const bool careful = masked;
    if constexpr (!WIDE) lay(0);

    // ---- softmax: probabilities are 2^(score - m_run) against a reference that moves only when a sum of them says that some
    // score lies far above it, or there is none yet (-inf)
    float pr[MT][TG][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float psum = 0.f;
#pragma unroll
      for (int i = 0; i < TG; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          pr[mt][i][r] = __builtin_amdgcn_exp2f(fmaf(s[mt][i][r], a.scale_log2, -m_run[mt]));
          psum += pr[mt][i][r];
        }
      if (__any(!(psum <= kBig))) {
        float tmax = -INFINITY;
#pragma unroll
        for (int i = 0; i < TG; ++i)
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
        for (int i = 0; i < TG; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            pr[mt][i][r] = __builtin_amdgcn_exp2f(fmaf(s[mt][i][r], a.scale_log2, -ref));
            psum += pr[mt][i][r];
          }
      }
      l_run[mt] += psum;
    }

    // ---- O^T += V^T P^T
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < TG; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const float v = __uint_as_float(vw[i * VG + r * (DH / 64) + d / 4][d % 4]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              if (!careful) {
                o[mt][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, pr[mt][i][r], o[mt][d], 0, 0, 0);
              } else {
#pragma unroll 1
                for (int x = 0; x < 4; ++x) {
                  const f32x4 one = __builtin_amdgcn_mfma_f32_16x16x4f32(grp == x ? v : 0.f, grp == x ? pr[mt][i][r] : 0.f,
                                                                         f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                  if (__shfl(pr[mt][i][r], col + 16 * x, NOVA_WAVE) != 0.f) o[mt][d] += one;
                }
              }
            }
          }
      if (more) load_v(t + kWaves, pages_next);
    } else {
#pragma unroll
      for (int u = 0; u < TG / 2; ++u) {                         // 32 keys at a time
        if (u > 0) lay(u);
        if (u == TG / 2 - 1 && more) load_v(t + kWaves, pages_next);
        bf16x8 pf[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < 8; ++e) pf[mt][e] = (bf16_t)pr[mt][2 * u + (e >> 2)][e & 3];
        if (!careful) {
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const bf16x8 vf = join(read_transposed(sv + vaddr[d]), read_transposed(sv + vaddr[d] + 16 * ROWB));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][d] = mfma16(vf, pf[mt], o[mt][d]);
          }
        } else {
          // one key at a time: element e of the lanes of group x.  Rows whose weight for it is 0 take nothing of it.
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
                const bf16x8 vf = join(read_transposed(sv + vaddr[d]), read_transposed(sv + vaddr[d] + 16 * ROWB));
                const f32x4 one = mfma16(__builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, vf) & only), __builtin_bit_cast(bf16x8, w),
                                         f32x4{0.f, 0.f, 0.f, 0.f});
                if (weight) o[mt][d] += one;
              }
            }
          }
        }
      }
    }
    pages = pages_next;
    if (t + 2 * kWaves < t1) pages_next = look_up(t + 2 * kWaves);
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
      *reinterpret_cast<f32x4*>(sv + (c4 * 16 + col) * 16) = v;
    }
    __syncthreads();
    for (int i = tid; i < 16 * (DH / 4); i += kWaves * 64) {
      const int c4 = i % (DH / 4), rr = i / (DH / 4), row = row0 + mt * 16 + rr;
      if (row >= rows) continue;
      float m = -INFINITY, lt = 0.f;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, part_m[w][rr]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        // a wave that has seen nothing of a row has reference -inf and sum 0
        const float f = part_m[w][rr] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(part_m[w][rr] - m);
        lt = fmaf(f, part_l[w][rr], lt);
        acc += f * *reinterpret_cast<const f32x4*>(lds + w * HALF + (c4 * 16 + rr) * 16);
      }
      if (nparts == 1) {
        const int s = div_by(row, a.G, a.G_inv, g_unused);
        const bool some = row < live && visible_keys(a.causal, len, count, s) > 0 && !(CHOSEN && lt == 0.f);
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
hipError_t launch_paged_few(hipStream_t st, int dh, int mt, unsigned grid, const PagedArgs<T>& a) {
  const size_t lists = a.chosen ? ((size_t)(a.most_pages + 31) / 32 * 2 + 1) * 4 + (size_t)a.most_listed * 6 : 0;
#define GO(DH, MT)                                                                                     \
  do {                                                                                                 \
    if (a.chosen) few_kernel<T, DH, MT, true><<<grid, kWaves * 64, (lists + 15) / 16 * 16, st>>>(a);   \
    else few_kernel<T, DH, MT, false><<<grid, kWaves * 64, 0, st>>>(a);                                \
  } while (0)
  if (dh == 64) { if (mt == 2) GO(64, 2); else GO(64, 1); }
  else { if (mt == 2) GO(128, 2); else GO(128, 1); }
#undef GO
  return hipGetLastError();
}
template hipError_t launch_paged_few<bf16_t>(hipStream_t, int, int, unsigned, const PagedArgs<bf16_t>&);
template hipError_t launch_paged_few<float>(hipStream_t, int, int, unsigned, const PagedArgs<float>&);
