// What the rows of the 4-bit cache collect of the queries' attention: mass_j = sum over rows of 2^(score - lse), a row being a
// query of one of the heads that share a key head.  Half the products of the attention and as many exponentials, no values.
//
// S = Q K^T, 32 rows x 32 keys per MFMA, a lane owning one key of either of two blocks: the sum over rows stays in the lane.  A
// wave has 64 keys, converted once into the operands it holds in registers (the order of the channels in the product is free:
// a lane takes half a row of the cache as it lies); the rows come in tiles of 32 or 64 through LDS, shared by the four waves.
// A launch leaves sums per key head (and run of rows, where there are few keys); a second one adds them up in a fixed order.
//
// Bound by vector instructions, an fma, an exp2 and an add per score: 1640 queries of 2 images, 16 heads of 128, 8065 keys 133 us,
// 0.82 PFLOP/s.
//
// Few rows (single tokens, a handful of queries): reading the keys once bounds it, and launches.  The waves of a workgroup take
// 64 keys of several key heads and add up among themselves, one launch and no workspace.  16 x 16 MFMAs, the keys from the cache
// into registers, as in fourbit_few.hip.  32 heads of 128 on 8, 4 images of 32768 rows (71 MB) 17.8 us, launch and start included.
#include <algorithm>

#include "fourbit_attention.h"

namespace {

constexpr int kWaves = 4, kKeys = kWaves * 64, kSubRows = 32;
constexpr int kTallRows = 512;       // rows per key head from which a bf16 tile has 64 of them (both measured at the launch)

// What a row has collected after a call.  A sum that is no number (one query or key of NaN is enough) adds nothing: a NaN would be
// ranked behind the rows that do not exist (-1), which would then be kept in place of the image's own.
__device__ __forceinline__ float collected(float before, float sum) {
  return (before > 0.f ? before : 0.f) + (sum == sum ? sum : 0.f);
}

template <typename T>
struct MassArgs {
  const T* q;
  int64_t q_sb, q_sr, q_sh;
  FourBitView c;
  int heads, G, n, P;
  uint32_t G_inv;
  const int32_t *n_rows, *kv_rows;
  float scale_log2;
  const float* lse;
  int chunks, nsplit;    // key chunks per key head, runs of row tiles
  float* part;           // [B][hk][nsplit][pitch]
  int pitch;
};

template <typename T, int DH, int SUBS>
__global__ __launch_bounds__(kWaves * 64, 2) void mass_kernel(MassArgs<T> a) {
  constexpr int NP = kParts<T>, kTileRows = SUBS * kSubRows;
  constexpr int GPR = DH / kGroup, ROWB = DH * 2, KS = DH / 16;
  constexpr int PLANE = kTileRows * ROWB, STAGE = NP * PLANE;
  constexpr int QL = kTileRows * DH / 8 / (kWaves * 64);       // runs of eight channels per thread and tile
  constexpr int CPR = DH / 8;                                  // of them per row
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
  __shared__ __attribute__((aligned(16))) float neg_lse[2][kTileRows];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int split_i = blockIdx.x % a.nsplit, ic = blockIdx.x / a.nsplit;
  const int chunk = ic % a.chunks, bh = ic / a.chunks;
  const int b = bh / a.c.hk, j = bh - b * a.c.hk;
  const int live = image_count(a.n_rows, b, a.n) * a.G, len = image_prior(a.kv_rows, b, a.P);
  const int key0 = chunk * kKeys + wave * 64;
  if (chunk * kKeys >= len) return;                            // the whole workgroup: nothing is read of these keys' sums
  const int ntiles = (live + kTileRows - 1) / kTileRows, per = (ntiles + a.nsplit - 1) / a.nsplit;
  const int t0 = split_i * per, t1 = min(ntiles, t0 + per);

  // ---- rows of a tile: past the last one its copies, which weigh nothing (lse = inf).  A thread walks its rows in steps of a
  // tile: row s G + g goes on by 32 / G queries and 32 % G heads, with one query more and G heads fewer where that passes G.
  // (Dividing anew for every tile was 70 of the loop's 200 vector instructions.)
  struct Walk {
    int row, g;
    const T* p;
  };
  int step_g;
  const int64_t step_s = div_by(kTileRows, a.G, a.G_inv, step_g);
  const int64_t step = step_s * a.q_sr + step_g * a.q_sh, wrap = a.q_sr - a.G * a.q_sh;
  const T* q_head = a.q + b * a.q_sb + (int64_t)j * a.G * a.q_sh;
  Walk walk[QL];
  const T* last;
  const float *lse_p, *lse_end;
  int lse_g;
  {
    int g;
    const int s = div_by(max(live - 1, 0), a.G, a.G_inv, g);
    last = q_head + s * a.q_sr + g * a.q_sh;
    const int sl = div_by(t0 * kTileRows + tid % kTileRows, a.G, a.G_inv, lse_g);
    const float* l = a.lse + (int64_t)b * a.n * a.heads + j * a.G;
    lse_p = l + (int64_t)sl * a.heads + lse_g;
    lse_end = l + (int64_t)s * a.heads + g;                      // the last live row's, and nothing behind it is read
  }
#pragma unroll
  for (int i = 0; i < QL; ++i) {
    const int x = tid + i * kWaves * 64;
    walk[i].row = t0 * kTileRows + x / CPR;
    const int s = div_by(walk[i].row, a.G, a.G_inv, walk[i].g);
    walk[i].p = q_head + s * a.q_sr + walk[i].g * a.q_sh;
  }
  T qr[QL][8];
  float lse_r = 0.f;
  auto request = [&]() {                                         // the next tile's
#pragma unroll
    for (int i = 0; i < QL; ++i) {
      Walk& w = walk[i];
      const T* p = (w.row < live ? w.p : last) + (tid + i * kWaves * 64) % CPR * 8;
      if constexpr (NP == 1) {
        *reinterpret_cast<u32x4*>(qr[i]) = *reinterpret_cast<const u32x4*>(p);
      } else {
        *reinterpret_cast<f32x4*>(qr[i]) = *reinterpret_cast<const f32x4*>(p);
        *reinterpret_cast<f32x4*>(qr[i] + 4) = *reinterpret_cast<const f32x4*>(p + 4);
      }
      w.row += kTileRows;
      w.g += step_g;
      w.p += step;
      if (w.g >= a.G) {
        w.g -= a.G;
        w.p += wrap;
      }
    }
    if (tid < kTileRows) {
      lse_r = lse_p <= lse_end ? -kAttnLog2e * *lse_p : -INFINITY;
      lse_g += step_g;
      lse_p += step_s * a.heads + step_g;
      if (lse_g >= a.G) {
        lse_g -= a.G;
        lse_p += a.heads - a.G;
      }
    }
  };
  auto place = [&](int stage) {
#pragma unroll
    for (int i = 0; i < QL; ++i) {
      const int x = tid + i * kWaves * 64;
      bf16x8 f[NP];
      load_eight(qr[i], f);
#pragma unroll
      for (int p = 0; p < NP; ++p) *reinterpret_cast<bf16x8*>(lds + stage * STAGE + p * PLANE + swz<ROWB>(x / CPR, x % CPR)) = f[p];
    }
    if (tid < kTileRows) neg_lse[stage][tid] = lse_r;
  };
  auto barrier = [] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);                        // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  if (t0 < t1) request();

  // ---- this lane's keys: channels half dh / 2 + 8 t of key col of block kb
  bf16x8 kf[2][KS];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int64_t r = (int64_t)bh * a.c.cap + min(key0 + kb * 32 + col, len - 1);
    const uint8_t* w = a.c.codes[0] + r * (DH / 2) + half * (DH / 4);
    const uint8_t* sc = a.c.scales[0] + r * GPR + half * (GPR / 2);
#pragma unroll
    for (int x = 0; x < GPR / 2; ++x) {
      const u32x4 c = *reinterpret_cast<const u32x4*>(w + x * 16);
      const float scale = fourbit_scale(sc[x]);
#pragma unroll
      for (int e = 0; e < 4; ++e) kf[kb][x * 4 + e] = fourbit_eight(c[e], scale);
    }
  }
  int qa[KS];
#pragma unroll
  for (int t = 0; t < KS; ++t) qa[t] = swz<ROWB>(col, half * KS + t);

  float acc[2] = {0.f, 0.f};
  if (t0 < t1) {
    place(0);
    if (t0 + 1 < t1) request();
    barrier();
  }
  for (int t = t0; t < t1; ++t) {
    const int stage = (t - t0) & 1;
    const char* sq = lds + stage * STAGE;
    auto next = [&] {
      if (t + 1 < t1) {
        place(stage ^ 1);
        if (t + 2 < t1) request();
      }
    };
    float sum[2] = {0.f, 0.f};
    if constexpr (SUBS > 1) next();
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) {
          const bf16x8 qf = *reinterpret_cast<const bf16x8*>(sq + p * PLANE + sub * kSubRows * ROWB + qa[ks]);
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) s[kb] = mfma32(qf, kf[kb][ks], s[kb]);
        }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (SUBS == 1) next();
      // register r is row 8 (r / 4) + 4 half + r % 4 of the 32
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const f32x4 nl = *reinterpret_cast<const f32x4*>(&neg_lse[stage][sub * kSubRows + 8 * r4 + 4 * half]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) sum[kb] += __builtin_amdgcn_exp2f(fmaf(s[kb][r4 * 4 + e], a.scale_log2, nl[e]));
      }
    }
    acc[0] += sum[0];
    acc[1] += sum[1];
    barrier();
  }
  float* to = a.part + ((int64_t)bh * a.nsplit + split_i) * a.pitch;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const float v = acc[kb] + __shfl_xor(acc[kb], 32, NOVA_WAVE);
    const int key = key0 + kb * 32 + col;
    if (half == 0 && key < len) to[key] = v;
  }
}

// 32 keys per workgroup, every eighth part to one eighth of its threads: with few keys there are many parts (runs of rows), and
// one thread per key would fetch them one after the other (1174 queries of 18 heads, three keys: the call 25 us so, 13.7 now).
constexpr int kAddKeys = 32, kAddGroups = 8;
__global__ __launch_bounds__(kAddKeys* kAddGroups) void add_kernel(const float* __restrict__ part, int pitch, int parts, int cap, int P,
                                                                   const int32_t* __restrict__ kv_rows, const float* mass_in,
                                                                   float* mass) {
  __shared__ float sums[kAddGroups][kAddKeys];
  const int b = blockIdx.y, x = threadIdx.x % kAddKeys, g = threadIdx.x / kAddKeys, k = blockIdx.x * kAddKeys + x;
  const int len = image_prior(kv_rows, b, P);
  float sum = 0.f;
  if (k < len) {
    const float* p = part + (int64_t)b * parts * pitch + k;
#pragma unroll 8
    for (int i = g; i < parts; i += kAddGroups) sum += p[(int64_t)i * pitch];
  }
  sums[g][x] = sum;
  __syncthreads();
  if (g > 0 || k >= cap) return;
  const int64_t at = (int64_t)b * cap + k;
  if (k >= len) {
    mass[at] = -1.0f;
    return;
  }
  const float m0 = mass_in ? mass_in[at] : 0.f;
#pragma unroll
  for (int i = 1; i < kAddGroups; ++i) sum += sums[i][x];
  mass[at] = collected(m0, sum);
}

// HW waves of a workgroup share NT tiles of 64 keys, each with every HW-th key head; kFewWaves / HW such groups.
constexpr int kFewWaves = 8;
constexpr int kFewRows = 32;         // rows per key head up to which this kernel is taken

template <typename T, int DH, int HW, int NT>
__global__ __launch_bounds__(kFewWaves * 64) void mass_few_kernel(MassArgs<T> a, const float* mass_in, float* mass) {
  constexpr int NP = kParts<T>, GPR = DH / kGroup, KW = DH / 32, GROUPS = kFewWaves / HW, KEYS = NT * 64;
  __shared__ float part[kFewWaves][KEYS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int b = blockIdx.y, key0 = (blockIdx.x * GROUPS + wave / HW) * KEYS;
  const int live = image_count(a.n_rows, b, a.n) * a.G, len = image_prior(a.kv_rows, b, a.P);
  float acc[NT][4];                                          // key 64 t + 16 i + col, rows 4 grp .. + 3 of every sixteen
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[t][i] = 0.f;
  if (key0 < len) {
    for (int j = wave % HW; j < a.c.hk; j += HW) {
      const int64_t base = ((int64_t)b * a.c.hk + j) * a.c.cap;
      const auto kc = head_buffer(a.c.codes[0] + base * (DH / 2), len * (DH / 2)), ks = head_buffer(a.c.scales[0] + base * GPR, len * GPR);
      const uint32_t o = (key0 + col) * (DH / 2) + grp * (DH / 8), os = (key0 + col) * GPR + grp * GPR / 4;
      for (int row0 = 0; row0 < live; row0 += 16) {
        uint32_t kw[2][4][KW], kb[2][4];
        auto request = [&](int t) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (DH == 128) {
              const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(kc, o + (t * 64 + i * 16) * (DH / 2), 0, 0);
#pragma unroll
              for (int e = 0; e < 4; ++e) kw[t & 1][i][e] = w[e];
            } else {
              const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(kc, o + (t * 64 + i * 16) * (DH / 2), 0, 0);
              kw[t & 1][i][0] = w[0];
              kw[t & 1][i][1] = w[1];
            }
            kb[t & 1][i] = __builtin_amdgcn_raw_buffer_load_b8(ks, os + (t * 64 + i * 16) * GPR, 0, 0);
          }
        };
        int g;
        const int s = div_by(min(row0 + col, live - 1), a.G, a.G_inv, g);
        const T* qp = a.q + b * a.q_sb + s * a.q_sr + (j * a.G + g) * a.q_sh + grp * (DH / 4);
        bf16x8 qf[KW][NP];
#pragma unroll
        for (int e = 0; e < KW; ++e) load_eight(qp + e * 8, qf[e]);
        float nl[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = row0 + 4 * grp + r;
          const int sr = div_by(min(row, live - 1), a.G, a.G_inv, g);
          nl[r] = row < live ? -kAttnLog2e * a.lse[((int64_t)b * a.n + sr) * a.heads + j * a.G + g] : -INFINITY;
        }
        request(0);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (t + 1 < NT) request(t + 1);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < KW; ++e) {
              const bf16x8 kf = fourbit_eight(kw[t & 1][i][e], fourbit_scale(kb[t & 1][i]));
#pragma unroll
              for (int p = NP - 1; p >= 0; --p) sc = mfma16(qf[e][p], kf, sc);
            }
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale_log2, nl[r]));
            acc[t][i] += sum;
          }
          __builtin_amdgcn_sched_barrier(0);                   // one tile's operands at a time
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      acc[t][i] += __shfl_xor(acc[t][i], 16, NOVA_WAVE);
      acc[t][i] += __shfl_xor(acc[t][i], 32, NOVA_WAVE);
    }
    part[wave][t * 64 + lane] = grp == 0 ? acc[t][0] : grp == 1 ? acc[t][1] : grp == 2 ? acc[t][2] : acc[t][3];
  }
  __syncthreads();
  for (int x = tid; x < GROUPS * KEYS; x += kFewWaves * 64) {
    const int k = blockIdx.x * GROUPS * KEYS + x;
    if (k >= a.c.cap) return;
    const int64_t at = (int64_t)b * a.c.cap + k;
    if (k >= len) {
      mass[at] = -1.0f;
      continue;
    }
    const float m0 = mass_in ? mass_in[at] : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < HW; ++w) sum += part[x / KEYS * HW + w][x % KEYS];
    mass[at] = collected(m0, sum);
  }
}

struct Plan {
  int few;               // waves that share keys, or 0: mass_kernel
  int chunks, nsplit, pitch;
};
constexpr int kCus = 256;
Plan plan(const nova_fourbit_cache& c, int heads, int n, int kv_len) {
  Plan p = {};
  if ((int64_t)n * (heads / c.kv_heads) <= kFewRows) {
    p.few = c.kv_heads >= 8 ? 8 : c.kv_heads >= 4 ? 4 : c.kv_heads >= 2 ? 2 : 1;
    return p;
  }
  p.chunks = (kv_len + kKeys - 1) / kKeys;
  p.pitch = (kv_len + 63) / 64 * 64;
  const int64_t items = std::max((int64_t)c.B * c.kv_heads * p.chunks, (int64_t)1);
  const int tiles = (int)(((int64_t)n * (heads / c.kv_heads) + kSubRows - 1) / kSubRows);
  // Up to two workgroups per CU, as many as fit (one run per item from 257 items on; tiles are counted in 32 rows, so that of
  // taller ones some runs may get none); eight, so that they end together, where a run still has 512 rows: its start, the conversion of
  // its keys, is then little (us with two / eight: 280 items of 30360 rows 765 / 368; 423 of 1887 77 / 72; 1024 of 1640 the same; but
  // 1024 of 512 in runs of 256 46 / 49, 192 of 600 in runs of 128 19 / 21).
  const int64_t two = std::min((int64_t)tiles, 2 * kCus / items), eight = std::min((int64_t)tiles / 16, (8 * kCus + items - 1) / items);
  p.nsplit = (int)std::max({(int64_t)1, two, eight});
  return p;
}

template <typename T>
hipError_t collect(hipStream_t st, const nova_fourbit_cache& c, int heads, int n, const nova_rows& q, const int32_t* n_rows, int P,
                   const int32_t* kv_rows, float scale_log2, const float* lse, const float* mass_in, float* mass, void* workspace) {
  const Plan p = plan(c, heads, n, P);
  MassArgs<T> a = {};
  a.q = static_cast<const T*>(q.data);
  a.q_sb = q.stride_b; a.q_sr = q.stride_row; a.q_sh = q.stride_head;
  a.c = fourbit_view(c);
  a.heads = heads; a.G = heads / c.kv_heads; a.n = n; a.P = P;
  a.G_inv = div_inv(a.G);
  a.n_rows = n_rows; a.kv_rows = kv_rows;
  a.scale_log2 = scale_log2;
  a.lse = lse;
  a.chunks = p.chunks; a.nsplit = p.nsplit; a.pitch = p.pitch;
  a.part = static_cast<float*>(workspace);
  if (p.few) {
    // Two tiles per wave once that leaves two workgroups per CU: the rows are read once for them, and the next keys on the way
    // meanwhile (us with one / two / four: 4 images, 32 heads of 128 on 8, 32768 rows 21.9 / 17.8 / 18.4; 16 images, 16 heads
    // of 64, 4096 rows 12.5 / 10.9 / 11.0; 8 images, 600 rows 9.2 / 9.9 / 9.8).  The capacity decides, which the grid has to cover:
    // rows behind an image's are marked.  A long cache with few rows in it pays for that (the first of these shapes with one /
    // two: 300 rows of 32768 6.6 / 7.7, 2000 7.5 / 8.0, 8000 10.2 / 9.5).
    const int tile_groups = kFewWaves / p.few * 64;
    const bool two = (int64_t)c.B * c.capacity / tile_groups >= 4 * kCus;
    const int keys = tile_groups * (two ? 2 : 1);
    const dim3 grid((c.capacity + keys - 1) / keys, c.B);
#define GO(DH, HW) if (two) mass_few_kernel<T, DH, HW, 2><<<grid, kFewWaves * 64, 0, st>>>(a, mass_in, mass); \
                   else mass_few_kernel<T, DH, HW, 1><<<grid, kFewWaves * 64, 0, st>>>(a, mass_in, mass)
#define GO_DH(DH) if (p.few == 8) { GO(DH, 8); } else if (p.few == 4) { GO(DH, 4); } else if (p.few == 2) { GO(DH, 2); } else { GO(DH, 1); }
    if (c.dh == 64) { GO_DH(64) } else { GO_DH(128) }
#undef GO_DH
#undef GO
    return hipGetLastError();
  }
  int parts = 0;
  if (P > 0) {
    parts = c.kv_heads * p.nsplit;
    const unsigned grid = (unsigned)((int64_t)c.B * c.kv_heads * p.chunks * p.nsplit);
    // Tiles of 64 rows halve the barriers and give the softmax of one half the products of the other to run beside (us with 32 /
    // 64, bf16: 2 images of 1640 queries, 16 heads of 128 140.9 / 136.8; 8 of 512, 36 heads of 64 50.4 / 46.9).  Few rows would
    // be padding (40 of them 20.5 / 22.7), and in fp32 the LDS then holds one workgroup per CU (500 rows 53 / 70).
    constexpr int kTall = sizeof(T) == 2 ? 2 : 1;
    const bool tall = (int64_t)n * a.G >= kTallRows;
    if (c.dh == 64) {
      if (tall) mass_kernel<T, 64, kTall><<<grid, kWaves * 64, 0, st>>>(a);
      else mass_kernel<T, 64, 1><<<grid, kWaves * 64, 0, st>>>(a);
    } else {
      if (tall) mass_kernel<T, 128, kTall><<<grid, kWaves * 64, 0, st>>>(a);
      else mass_kernel<T, 128, 1><<<grid, kWaves * 64, 0, st>>>(a);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  add_kernel<<<dim3((c.capacity + kAddKeys - 1) / kAddKeys, c.B), kAddKeys * kAddGroups, 0, st>>>(
      a.part, p.pitch, parts, c.capacity, P, kv_rows, mass_in, mass);
  return hipGetLastError();
}

}  // namespace

size_t fourbit_mass_workspace_bytes(const nova_fourbit_cache& c, int heads, int n, int kv_len) {
  const Plan p = plan(c, heads, n, kv_len);
  return (size_t)c.B * c.kv_heads * p.nsplit * p.pitch * sizeof(float);
}

hipError_t launch_fourbit_mass(const nova_ctx*, hipStream_t st, int dtype, const nova_fourbit_cache& c, int heads, int n,
                               const nova_rows& q, const int32_t* n_rows, int P, const int32_t* kv_rows, float scale_log2,
                               const float* lse, const float* mass_in, float* mass, void* workspace) {
  if (dtype == NOVA_BF16) return collect<bf16_t>(st, c, heads, n, q, n_rows, P, kv_rows, scale_log2, lse, mass_in, mass, workspace);
  return collect<float>(st, c, heads, n, q, n_rows, P, kv_rows, scale_log2, lse, mass_in, mass, workspace);
}
