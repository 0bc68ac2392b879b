// The key/value cache in pages: page lists and slots from the images' lengths, rows into pages, means of pages.
//
// Page lists are integer work on a few numbers per image: every workgroup takes the prefix sums over all images for itself (what an
// image gives back, what it needs), after which every entry of a list, slot and place of the stack of free pages has a
// formula of its own and nothing waits for anything: a chain of dependent loads, 3 us for 256 images that get a row each; 131 072 slots
// in two launches 10 us, four slots a thread one after the other with a chain of loads each, on 128 of the CUs, and 3.  Appends
// are copies of whole lines, bound by HBM (134 MB, read with the stride of a joint projection, 22 us; a row each for 64 images 2.7).  Means: a
// wave per page and key head, sums in 64 bits, in which the sum of a page's rows is as good as exact in any order (one page per image and key head 5 us: the latency of table, length and rows).
#include <algorithm>

#include "paged.h"

namespace {

constexpr int kThreads = 256;

// ---- page lists and slots ----------------------------------------------------------------------------------------
struct ImageRows {
  int keep, rows, held, want;            // rows that stay; rows wanted; pages before and after
};
__device__ __forceinline__ ImageRows image_rows(const PagedReserve& r, int b) {
  const int now = image_prior(r.kv_rows, b, r.kv_len), count = image_count(r.n_rows, b, r.n), up = (1 << r.shift) - 1;
  ImageRows x;
  x.keep = r.keep_rows ? min(max(r.keep_rows[b], 0), now) : now;
  x.rows = x.keep + count;
  x.held = (now + up) >> r.shift;
  x.want = (x.rows + up) >> r.shift;
  return x;
}

// largest i of [0, n] with at[i] <= v (at[0] = 0, ascending)
__device__ __forceinline__ int find(const int32_t* at, int n, int v) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (at[mid] <= v) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <int NT>
__global__ __launch_bounds__(NT) void reserve_kernel(PagedReserve r, uint32_t n_inv, int write_state, int write_lists) {
  extern __shared__ int32_t sums[];
  int32_t* gone = sums;                  // [B + 1] pages given back by the images in front
  int32_t* need = sums + r.B + 1;        // [B + 1] pages that those of them want that grow
  __shared__ int32_t wave_gone[NT / 64], wave_need[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int base_gone = 0, base_need = 0;
  for (int b0 = 0; b0 < r.B; b0 += NT) {
    const int b = b0 + tid;
    int g = 0, w = 0;
    if (b < r.B) {
      const ImageRows x = image_rows(r, b);
      g = max(x.held - x.want, 0);
      w = max(x.want - x.held, 0);
    }
    int gi = g, wi = w;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int tg = __shfl_up(gi, o, NOVA_WAVE), tw = __shfl_up(wi, o, NOVA_WAVE);
      if (lane >= o) { gi += tg; wi += tw; }
    }
    __syncthreads();                     // the sums of the last images have been read
    if (lane == 63) { wave_gone[wave] = gi; wave_need[wave] = wi; }
    __syncthreads();
    int all_gone = 0, all_need = 0;
    for (int i = 0; i < NT / 64; ++i) {
      if (i < wave) { gi += wave_gone[i]; wi += wave_need[i]; }
      all_gone += wave_gone[i];
      all_need += wave_need[i];
    }
    if (b < r.B) {
      gone[b] = base_gone + gi - g;
      need[b] = base_need + wi - w;
    }
    base_gone += all_gone;
    base_need += all_need;
  }
  if (tid == 0) {
    gone[r.B] = base_gone;
    need[r.B] = base_need;
  }
  const int stack = min(max(r.free_count[0], 0), r.pages);
  const int height = stack + base_gone;
  __syncthreads();
  // Images are served in order up to the first that asks for more than is left: those in front of `served` with need[b + 1] <=
  // height.  Pages handed out: `out`.
  int served = r.B, out = base_need;
  if (base_need > height) {
    served = find(need, r.B, height);    // need[served] <= height < need[served + 1]
    out = need[served];
  }
  // page that the stack hands out as the i-th
  auto handed = [&](int i) {
    const int at = height - 1 - i;
    if (at < stack) return r.free_pages[at];
    const int b = find(gone, r.B - 1, at - stack);
    return r.table[(int64_t)b * r.pitch + image_rows(r, b).want + (at - stack - gone[b])];
  };
  if (write_lists) {
    const int64_t step = (int64_t)gridDim.x * NT, t0 = (int64_t)blockIdx.x * NT + tid;
    if (r.slots)
      for (int64_t i = t0; i < (int64_t)r.B * r.n; i += step) {
        int s;
        const int b = div_by((int)i, r.n, n_inv, s);
        const ImageRows x = image_rows(r, b);
        const int after = b < served || x.want <= x.held ? x.rows : min(x.rows, x.held << r.shift);
        const int row = x.keep + s, page = row >> r.shift;
        int slot = -1;
        if (row < after) {
          const int id = page < x.held ? r.table[(int64_t)b * r.pitch + page] : handed(need[b] + page - x.held);
          // an entry that is no page of the pool has no slots
          slot = (unsigned)id < (unsigned)r.pages ? (id << r.shift) + (row & ((1 << r.shift) - 1)) : -1;
        }
        r.slots[i] = slot;
      }
    for (int64_t i = t0; i < out; i += step) {
      // the last image with need[b] <= i has pages to get
      const int b = find(need, r.B - 1, (int)i);
      const ImageRows x = image_rows(r, b);
      r.table[(int64_t)b * r.pitch + x.held + ((int)i - need[b])] = handed((int)i);
    }
    for (int64_t i = t0; i < base_gone - out && stack + i < r.pages; i += step) {
      const int b = find(gone, r.B - 1, (int)i);
      r.free_pages[stack + i] = r.table[(int64_t)b * r.pitch + image_rows(r, b).want + ((int)i - gone[b])];
    }
  }
  if (write_state) {
    // the lengths and the stack's height may be the arrays read above (and by the loops in front of this, in this workgroup)
    constexpr int PER = 4096 / NT;
    int after[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = i * NT + tid;
      after[i] = 0;
      if (b < r.B) {
        const ImageRows x = image_rows(r, b);
        after[i] = b < served || x.want <= x.held ? x.rows : min(x.rows, x.held << r.shift);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i * NT + tid < r.B) r.kv_next[i * NT + tid] = after[i];
    if (tid == 0) r.free_next[0] = min(height - out, r.pages);
  }
}

// ---- rows into pages ----------------------------------------------------------------------------------------------
struct AppendArgs {
  const void* from[2];
  void* to[2];
  int64_t sb[2], sr[2], sh[2], sc[2];
  int vec[2];                            // channels side by side, 16-byte aligned
  const int32_t* slots;
  int64_t rows;                          // B n
  int n, hk, shift, most;                // most: slots of the pool
  uint32_t n_inv;
};

// Eight channels (four of fp32) per thread and row.  Where the caller's channels lie side by side neighbouring threads have
// neighbouring chunks of a row, otherwise neighbouring rows.
template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  constexpr int E = 16 / (int)sizeof(T), CPR = DH / E, ROWS = kThreads / CPR;
  const int which = blockIdx.z, j = blockIdx.y, tid = threadIdx.x;
  const bool vec = a.vec[which];
  const int chunk = vec ? tid % CPR : tid / ROWS;
  const int64_t i = (int64_t)blockIdx.x * ROWS + (vec ? tid / CPR : tid % ROWS);
  if (i >= a.rows) return;
  const int slot = a.slots[i];
  if ((unsigned)slot >= (unsigned)a.most) return;
  int s;
  const int b = div_by((int)i, a.n, a.n_inv, s);
  const T* x = static_cast<const T*>(a.from[which]) + b * a.sb[which] + s * a.sr[which] + j * a.sh[which];
  const int mask = (1 << a.shift) - 1;
  T* to = static_cast<T*>(a.to[which]) + ((((int64_t)(slot >> a.shift) * a.hk + j) << a.shift) + (slot & mask)) * DH + chunk * E;
  if (vec) {
    *reinterpret_cast<u32x4*>(to) = *reinterpret_cast<const u32x4*>(x + chunk * E);
    return;
  }
  Vec16<T> v;
#pragma unroll
  for (int e = 0; e < E; ++e) v.v[e] = x[(chunk * E + e) * a.sc[which]];
  *reinterpret_cast<decltype(v.v)*>(to) = v.v;
}

// ---- means of pages -----------------------------------------------------------------------------------------------
__device__ __forceinline__ double two_to(int e) { return __longlong_as_double((long long)(e + 1023) << 52); }

// A wave has one page of one key head: E channels per lane, the lanes of a channel every so many rows.
template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void summarise_kernel(const T* __restrict__ keys, const int32_t* __restrict__ table, int pitch,
                                                             int pages, int hk, int shift, int n, const int32_t* n_rows,
                                                             int kv_len, const int32_t* kv_rows, bf16_t* means) {
  constexpr int E = 16 / (int)sizeof(T), CPR = DH / E, RPL = 64 / CPR;          // chunks of a row, rows per load
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.z, j = blockIdx.y;
  const int len = image_prior(kv_rows, b, kv_len), from = max(len - image_count(n_rows, b, n), 0);
  const int ordinal = (from >> shift) + blockIdx.x * (kThreads / 64) + wave;
  if (from >= len || ordinal << shift >= len) return;
  const int page = table[(int64_t)b * pitch + ordinal], rows = min(len - (ordinal << shift), 1 << shift);
  if ((unsigned)page >= (unsigned)pages) return;
  const T* x = keys + (((int64_t)page * hk + j) << shift) * DH + lane % CPR * E;
  double sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.0;
  for (int r0 = 0; r0 < rows; r0 += 4 * RPL) {
    Vec16<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + i * RPL + lane / CPR;
      if (r < rows) v[i].load(x + r * DH);
      else
#pragma unroll
        for (int e = 0; e < E; ++e) v[i].set(e, 0.f);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += (double)v[i].get(e);
  }
#pragma unroll
  for (int o = CPR; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += __shfl_xor(sum[e], o, NOVA_WAVE);
  // all lanes of a channel hold the same sum
  double top = 0.0;
  bool odd = false;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    sum[e] /= (double)rows;
    odd |= !(fabs(sum[e]) < (double)INFINITY);
    top = fmax(top, fabs(sum[e]));
  }
#pragma unroll
  for (int o = 1; o < CPR; o <<= 1) top = fmax(top, __shfl_xor(top, o, NOVA_WAVE));
  odd = __any(odd);
  // the smallest e with top <= 127 2^e: top = m 2^x, 1 <= m < 2, gives x - 6 up to m = 127 / 64 and x - 5 from there on
  const int exponent = (int)((__double_as_longlong(top) >> 52) & 0x7FF) - 1023;
  int e2 = exponent - 6 + (top * two_to(min(max(-exponent, -1022), 1023)) > 127.0 / 64.0);
  e2 = top == 0.0 ? -100 : min(max(e2, -100), 100);
  if (lane >= CPR) return;
  bf16_t* to = means + ((int64_t)page * hk + j) * DH + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const double w = fmin(fmax(rint(sum[e] * two_to(-e2)), -127.0), 127.0);
    to[e] = odd ? (bf16_t)NAN : (bf16_t)(float)(w * two_to(e2));
  }
}

}  // namespace

hipError_t launch_paged_reserve(hipStream_t st, const PagedReserve& r) {
  const size_t lds = (size_t)(r.B + 1) * 8;
  const uint32_t n_inv = div_inv(r.n);
  // One workgroup does it all in one launch; many entries are dealt to many, and a second launch writes what the first has read (us in one /
  // in two launches: 256 images of one new row 5.2 / 7.4, 4096 of one 15.7 / 29.9, 16 of 256 rows 6.6 / 8.5, 32 of 256 9.1 / 8.8, 64 of
  // 2048 80 / 9.0).  With thousands of images the prefix sums, taken twice in two launches, count more than the entries do, which the rule
  // does not look at: 2048 images of four rows 13.1 / 19.1, 4096 of two 17.9 / 30.9, in two launches both.
  const int64_t entries = std::max<int64_t>((int64_t)r.B * r.n, r.B);
  if (entries <= 4096) {
    reserve_kernel<1024><<<1, 1024, lds, st>>>(r, n_inv, 1, 1);
    return hipGetLastError();
  }
  const unsigned grid = (unsigned)std::min<int64_t>((entries + 1023) / 1024, 512);
  reserve_kernel<256><<<grid, 256, lds, st>>>(r, n_inv, 0, 1);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  reserve_kernel<1024><<<1, 1024, lds, st>>>(r, n_inv, 1, 0);
  return hipGetLastError();
}

hipError_t launch_paged_append(hipStream_t st, const nova_paged_cache& c, int B, int n, const nova_rows& k, const nova_rows& v,
                               const int32_t* slots) {
  AppendArgs a = {};
  const nova_rows* in[2] = {&k, &v};
  const int per = c.dtype == NOVA_BF16 ? 8 : 4;                  // elements in 16 bytes
  for (int i = 0; i < 2; ++i) {
    a.from[i] = in[i]->data;
    a.sb[i] = in[i]->stride_b; a.sr[i] = in[i]->stride_row; a.sh[i] = in[i]->stride_head; a.sc[i] = in[i]->stride_channel;
    a.vec[i] = a.sc[i] == 1 && (reinterpret_cast<uintptr_t>(in[i]->data) & 15) == 0 && a.sb[i] % per == 0 && a.sr[i] % per == 0 &&
               a.sh[i] % per == 0;
  }
  a.to[0] = c.k_pages;
  a.to[1] = c.v_pages;
  a.slots = slots;
  a.rows = (int64_t)B * n;
  a.n = n; a.hk = c.kv_heads; a.shift = __builtin_ctz(c.page_rows); a.most = c.pages * c.page_rows;
  a.n_inv = div_inv(n);
#define GO(T, DH)                                                                                                    \
  append_kernel<T, DH><<<dim3((unsigned)((a.rows * (DH * (int)sizeof(T) / 16) + kThreads - 1) / kThreads), c.kv_heads, 2), kThreads, 0, st>>>(a)
  if (c.dtype == NOVA_BF16) { if (c.dh == 64) GO(bf16_t, 64); else GO(bf16_t, 128); }
  else { if (c.dh == 64) GO(float, 64); else GO(float, 128); }
#undef GO
  return hipGetLastError();
}

hipError_t launch_paged_summarise(hipStream_t st, const nova_paged_cache& c, int B, const int32_t* table, int pitch, int n,
                                  const int32_t* n_rows, int kv_len, const int32_t* kv_rows, void* means) {
  const int shift = __builtin_ctz(c.page_rows);
  const int most = ((int)std::min<int64_t>(n, kv_len) + c.page_rows - 2) / c.page_rows + 1;      // pages so many rows lie in at most
  const dim3 grid((most + 3) / 4, c.kv_heads, B);
#define GO(T, DH)                                                                                                                \
  summarise_kernel<T, DH><<<grid, kThreads, 0, st>>>(static_cast<const T*>(c.k_pages), table, pitch, c.pages, c.kv_heads, shift,  \
                                                     n, n_rows, kv_len, kv_rows, static_cast<bf16_t*>(means))
  if (c.dtype == NOVA_BF16) { if (c.dh == 64) GO(bf16_t, 64); else GO(bf16_t, 128); }
  else { if (c.dh == 64) GO(float, 64); else GO(float, 128); }
#undef GO
  return hipGetLastError();
}
