// C ABI of the library (declared in include/nova.h): argument checks on the host,
// then dispatch to the kernel launchers.  No allocation, no synchronisation.
#include <algorithm>
#include <cstdlib>
#include <new>

#include "nova_internal.h"

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline size_t esize(int dtype) { return dtype == NOVA_BF16 ? 2 : 4; }
inline bool valid_dtype(int dtype) { return dtype == NOVA_F32 || dtype == NOVA_BF16; }
inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

int shape_error(const nova_block_shape* s) {
  if (!s) return NOVA_ERR_INVALID_ARG;
  if (!valid_dtype(s->dtype)) return NOVA_ERR_UNSUPPORTED;
  if (s->B < 0 || s->N < 0 || s->C < 1 || s->heads < 1 || s->ffn_mult < 1 || s->kv_len < 0 || s->k < 0)
    return NOVA_ERR_INVALID_ARG;
  if (s->k > s->N) return NOVA_ERR_INVALID_ARG;
  if (s->C % s->heads != 0) return NOVA_ERR_INVALID_ARG;
  if ((int64_t)s->kv_len + s->k > s->kv_capacity) return NOVA_ERR_INVALID_ARG;
  const int dh = s->C / s->heads;
  if (s->dtype == NOVA_BF16) {
    if (s->C % 64 != 0 || (dh != 64 && dh != 128) || s->kv_capacity % 64 != 0) return NOVA_ERR_UNSUPPORTED;
  } else {
    if (s->C % 4 != 0 || dh > 256) return NOVA_ERR_UNSUPPORTED;
    // the fp32 attention keeps one score per cached key in LDS, and behind them dh floats or the eight that its waves
    // exchange: 64 KiB, and up to 28 bytes more with heads of fewer than eight channels (a CU has 160 KiB)
    if ((int64_t)s->kv_len + s->k + dh > 16384) return NOVA_ERR_UNSUPPORTED;
  }
  if ((int64_t)s->B * s->k * (int64_t)s->C * s->ffn_mult > (int64_t)1 << 40) return NOVA_ERR_UNSUPPORTED;
  return NOVA_OK;
}

int set_device(const nova_ctx* ctx) {
  int cur = -1;
  if (hipGetDevice(&cur) != hipSuccess) return NOVA_ERR_HIP;
  if (cur != ctx->device && hipSetDevice(ctx->device) != hipSuccess) return NOVA_ERR_HIP;
  return NOVA_OK;
}

// Makes the context's device current for a call and puts the caller's back afterwards.
struct DeviceScope {
  int before = -1;
  int rc = NOVA_OK;
  explicit DeviceScope(const nova_ctx* ctx) {
    int cur = -1;
    if (hipGetDevice(&cur) != hipSuccess) { rc = NOVA_ERR_HIP; return; }
    if (cur == ctx->device) return;
    if (hipSetDevice(ctx->device) != hipSuccess) { rc = NOVA_ERR_HIP; return; }
    before = cur;
  }
  ~DeviceScope() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Two arrays share a byte.
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// A cache in 4 bits.  At most 2^24 rows: a head's codes are 1 GiB, offsets within a head have 32 bits (between heads 64).
int fourbit_sizes_error(const nova_fourbit_cache* c) {
  if (!c) return NOVA_ERR_INVALID_ARG;
  if (c->B < 0 || c->kv_heads < 1 || c->capacity < 0) return NOVA_ERR_INVALID_ARG;
  if (c->dh != 64 && c->dh != 128) return NOVA_ERR_UNSUPPORTED;
  if (c->B > 65535 || c->kv_heads > 32767 || c->capacity > 1 << 24) return NOVA_ERR_UNSUPPORTED;
  return NOVA_OK;
}
int fourbit_error(const nova_fourbit_cache* c) {
  if (int rc = fourbit_sizes_error(c)) return rc;
  if (c->B == 0 || c->capacity == 0) return NOVA_OK;
  for (const void* p : {c->k_codes, c->k_scales, c->v_codes, c->v_scales})
    if (!p || !aligned16(p)) return NOVA_ERR_INVALID_ARG;
  return NOVA_OK;
}

int counts_error(std::initializer_list<const void*> arrays) {
  for (const void* p : arrays)
    if (!aligned(p, 4)) return NOVA_ERR_INVALID_ARG;
  return NOVA_OK;
}

// Rows [B, n, heads, dh] of the caller's.  vector: channels side by side, everything else a multiple of 16 bytes.
int rows_error(const nova_rows* r, int dtype, int B, int n, int heads, bool vector) {
  if (!r->data || !aligned(r->data, vector ? 16 : esize(dtype))) return NOVA_ERR_INVALID_ARG;
  const int64_t stride[4] = {r->stride_b, r->stride_row, r->stride_head, r->stride_channel};
  const int64_t extent[4] = {B, n, heads, 2};
  for (int i = 0; i < 4; ++i) {
    if (extent[i] <= 1) continue;
    if (stride[i] < 0 || stride[i] > (int64_t)1 << 40) return NOVA_ERR_INVALID_ARG;
    if (vector && (i == 3 ? stride[i] != 1 : stride[i] * (int64_t)esize(dtype) % 16 != 0)) return NOVA_ERR_INVALID_ARG;
  }
  return NOVA_OK;
}

// Strides of extents of 1 mean nothing and may be anything: zero, so that no kernel multiplies by them.
nova_rows settled(const nova_rows& r, int B, int n, int heads) {
  nova_rows s = r;
  if (B <= 1) s.stride_b = 0;
  if (n <= 1) s.stride_row = 0;
  if (heads <= 1) s.stride_head = 0;
  return s;
}

// n queries per image of `heads` heads over kv_len rows of a cache: at most 2^30 queries of one head in all, looked at factor by
// factor, since the product of three ints may pass 64 bits.
int query_sizes_error(const nova_fourbit_cache& c, int heads, int n, int kv_len) {
  if (heads < 1 || n < 0 || kv_len < 0 || kv_len > c.capacity || heads % c.kv_heads != 0) return NOVA_ERR_INVALID_ARG;
  constexpr int kMost = 1 << 30;
  if (c.B > 0 && (heads > kMost / c.B || n > kMost / (c.B * heads))) return NOVA_ERR_UNSUPPORTED;
  return NOVA_OK;
}
// Such a call has work to do, so that it may need a workspace.
bool query_has_work(const nova_fourbit_cache* c, int heads, int n, int kv_len) {
  return fourbit_sizes_error(c) == NOVA_OK && c->B > 0 && n > 0 && query_sizes_error(*c, heads, n, kv_len) == NOVA_OK;
}

// What nova_fourbit_attention and nova_fourbit_mass check alike.
int fourbit_query_error(int dtype, const nova_fourbit_cache* cache, int heads, int n, const nova_rows* q, int kv_len) {
  if (!valid_dtype(dtype)) return NOVA_ERR_UNSUPPORTED;
  if (int rc = fourbit_error(cache)) return rc;
  if (int rc = query_sizes_error(*cache, heads, n, kv_len)) return rc;
  if (cache->B == 0 || n == 0) return NOVA_OK;
  if (!q) return NOVA_ERR_INVALID_ARG;
  return rows_error(q, dtype, cache->B, n, heads, true);
}

// What the block calls check of everything but the cache and the workspace; `plain`: the shape to hold against the kernels'
// limits.  Sets `var`.  Returns 1 where there is nothing to do.
int block_error(const nova_block_shape* plain, const nova_block_weights* weights, const nova_block_variant* variant,
                const RowCounts& rows, const void* x, const int32_t* kept_idx, const void* y_kept, nova_block_variant* var) {
  if (!weights) return NOVA_ERR_INVALID_ARG;
  for (const void* p : {(const void*)rows.k_rows, (const void*)rows.kv_rows, (const void*)rows.kv_next})
    if (reinterpret_cast<uintptr_t>(p) & 3) return NOVA_ERR_INVALID_ARG;
  *var = {};
  if (variant) *var = *variant;
  if ((var->gelu_tanh != 0 && var->gelu_tanh != 1) || (var->qk_norm != 0 && var->qk_norm != 1))
    return NOVA_ERR_INVALID_ARG;
  if (var->qk_norm && (!var->qk_scale || (reinterpret_cast<uintptr_t>(var->qk_scale) & 3) != 0))
    return NOVA_ERR_INVALID_ARG;
  if (var->ada && !aligned16(var->ada)) return NOVA_ERR_INVALID_ARG;
  if (int rc = shape_error(plain)) return rc;
  if (var->w_cq) {
    if (!var->w_co || !var->k_text || !var->v_text) return NOVA_ERR_INVALID_ARG;
    if (var->text_len < 1 || var->text_len > var->text_capacity) return NOVA_ERR_INVALID_ARG;
    const void* cptrs[] = {var->w_cq, var->b_cq, var->w_co, var->b_co, var->k_text, var->v_text};
    for (const void* p : cptrs)
      if (p && !aligned16(p)) return NOVA_ERR_INVALID_ARG;
    const int dh = plain->C / plain->heads;
    if (plain->dtype == NOVA_BF16 ? var->text_capacity % 64 != 0 : (int64_t)var->text_len + dh > 16384)
      return NOVA_ERR_UNSUPPORTED;
  }
  if (plain->k == 0 || plain->B == 0) return 1;
  if (!x || !kept_idx || !y_kept) return NOVA_ERR_INVALID_ARG;
  if (!weights->w_qkv || !weights->w_o || !weights->w_fc1 || !weights->w_fc2) return NOVA_ERR_INVALID_ARG;
  const void* ptrs[] = {x, y_kept, weights->w_qkv, weights->w_o, weights->w_fc1, weights->w_fc2,
                        weights->b_qkv, weights->b_o, weights->b_fc1, weights->b_fc2};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return NOVA_ERR_INVALID_ARG;
  return NOVA_OK;
}

// The shape of a block whose cache is held in 4 bits as the other kernels see it: kept rows in a cache of their own.
nova_block_shape fourbit_plain_shape(const nova_block_shape& s) {
  nova_block_shape p = s;
  p.kv_len = 0;
  p.kv_capacity = s.k > 0 && s.k <= INT32_MAX - 63 ? (s.k + 63) / 64 * 64 : 64;
  return p;
}
int fourbit_shape_error(const nova_block_shape* s) {
  if (!s) return NOVA_ERR_INVALID_ARG;
  const nova_block_shape p = fourbit_plain_shape(*s);
  if (int rc = shape_error(&p)) return rc;
  if (s->kv_len < 0 || (int64_t)s->kv_len + s->k > s->kv_capacity) return NOVA_ERR_INVALID_ARG;
  const int dh = s->C / s->heads;
  if ((dh != 64 && dh != 128) || s->kv_capacity > 1 << 24 || s->B > 65535 || s->heads > 32767 ||
      (int64_t)s->B * s->heads * std::max(s->k, 1) > (int64_t)1 << 30)
    return NOVA_ERR_UNSUPPORTED;
  return NOVA_OK;
}
// Its workspace: that of the block, then the kept rows' keys and values, lengths, logarithms, and the attention's own.
size_t carve_fourbit(const nova_block_shape& s, void* base, FourBitBlock* fb) {
  const nova_block_shape p = fourbit_plain_shape(s);
  const size_t rows = (size_t)s.B * s.heads, dh = s.C / s.heads, total = (size_t)s.kv_len + s.k;
  const nova_fourbit_cache c = {nullptr, nullptr, nullptr, nullptr, s.B, s.heads, s.kv_capacity, (int32_t)dh};
  size_t off = up256(carve_workspace(p, nullptr).total);
  char* b = static_cast<char*>(base);
  const size_t half = up256(rows * p.kv_capacity * dh * esize(s.dtype));
  fb->pitch = p.kv_capacity;
  fb->k_new = b + off; off += half;
  fb->v_new = b + off; off += half;
  fb->kv_after = reinterpret_cast<int32_t*>(b + off); off += up256((size_t)s.B * 4);
  fb->lse = reinterpret_cast<float*>(b + off); off += up256(rows * s.k * 4);
  fb->work = b + off;
  off += up256(std::max(fourbit_attention_workspace_bytes(c, s.heads, s.k, (int)total),
                        fourbit_mass_workspace_bytes(c, s.heads, s.k, (int)total)));
  return off;
}

}  // namespace

BlockWorkspace carve_workspace(const nova_block_shape& s, void* base) {
  const size_t M = (size_t)s.B * s.k, C = s.C, F = (size_t)s.C * s.ffn_mult, e = esize(s.dtype);
  BlockWorkspace w;
  char* p = static_cast<char*>(base);
  size_t off = 0;
  w.u = p + off;    off += up256(M * C * e);
  w.q = p + off;    off += up256(M * C * e);
  w.attn = p + off; off += up256(M * C * e);
  w.x1 = p + off;   off += up256(M * C * e);
  w.hid = p + off;  off += up256(M * F * e);
  w.part_o = w.part_ml = nullptr;
  w.part_floats = 0;
  if (s.dtype == NOVA_BF16) {
    // One region serves two users, one after the other: the partial results of the attention items that are cut
    // into key runs (only the items of the last, partly filled round over the workgroup slots are: at most
    // kAttentionMaxPieces runs of up to 256 queries x dh floats, or attention_max_split() per item when the call
    // is small), and the fp32 K-slice sums of the projections back to C (slices x rows x C for launches whose tiles
    // fill at most half of the compute units: at most 128 tiles of 256 x 256).
    const size_t dh = (size_t)(s.C / s.heads);
    const size_t Mp = (size_t)s.B * (((size_t)s.k + 255) / 256 * 256);
    const size_t attn = std::min((size_t)attention_max_split() * Mp * C, (size_t)kAttentionMaxPieces * 256 * dh);
    const size_t kslice = std::min((size_t)4 * M * C, (size_t)128 * 256 * 256);
    w.part_floats = (int64_t)std::max(attn, kslice);
    w.part_o = p + off;  off += up256((size_t)w.part_floats * 4);
    w.part_ml = p + off; off += up256((size_t)w.part_floats / dh * 2 * 4);     // (reference, sum) per query and run
  }
  w.total = off;
  return w;
}

extern "C" {

int nova_create(nova_ctx** out, int device_id) {
  if (!out) return NOVA_ERR_INVALID_ARG;
  *out = nullptr;
  int n = 0;
  if (hipGetDeviceCount(&n) != hipSuccess) return NOVA_ERR_HIP;
  if (device_id < 0 || device_id >= n) return NOVA_ERR_INVALID_ARG;
  hipDeviceProp_t prop;
  if (hipGetDeviceProperties(&prop, device_id) != hipSuccess) return NOVA_ERR_HIP;
  // the allocation-free entry point's scratch is a static device array: resolve its address on this device now
  if (head_entropy_static_init(device_id) != hipSuccess) return NOVA_ERR_HIP;
  nova_ctx* c = new (std::nothrow) nova_ctx;
  if (!c) return NOVA_ERR_HIP;
  c->device = device_id;
  c->num_cus = prop.multiProcessorCount;
  c->lds_per_block = prop.sharedMemPerBlock;
  c->prof_mask = 0;
  const char* g = getenv("NOVA_GEMM_CFG");
  const char* a = getenv("NOVA_ATTN_CFG");
  c->gemm_cfg = g ? atoi(g) : -1;
  c->attn_cfg = a ? atoi(a) : -1;
  const char* sp = getenv("NOVA_ATTN_SPLIT");
  c->attn_split = sp ? atoi(sp) : -1;
  const char* gp = getenv("NOVA_GEMM_PARTS");
  c->gemm_parts = gp ? atoi(gp) : -1;
  const char* gs = getenv("NOVA_GEMM_PERSIST");
  c->gemm_persist = gs ? atoi(gs) : -1;
  const char* gk = getenv("NOVA_GEMM_KSPLIT");
  c->gemm_ksplit = gk ? atoi(gk) : -1;
  *out = c;
  return NOVA_OK;
}

int nova_destroy(nova_ctx* ctx) {
  if (ctx) {
    for (ProfRecord& r : ctx->prof) {
      (void)hipEventDestroy(r.start);
      (void)hipEventDestroy(r.stop);
    }
  }
  delete ctx;
  return NOVA_OK;
}

int nova_probe(nova_ctx* ctx, void* stream, int kind, const void* src, void* dst, int64_t bytes, int iters,
               float* sink, double* work) {
  if (!ctx || !sink || !work) return NOVA_ERR_INVALID_ARG;
  if (int rc = set_device(ctx)) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  switch (kind) {
    case NOVA_PROBE_READ:
      if (!src || bytes < 16 || reinterpret_cast<uintptr_t>(src) % 16) return NOVA_ERR_INVALID_ARG;
      e = launch_probe_read(st, ctx->num_cus, src, bytes, sink);
      *work = (double)(bytes / 16 * 16);
      break;
    case NOVA_PROBE_COPY:
      if (!src || !dst || bytes < 16 || reinterpret_cast<uintptr_t>(src) % 16 || reinterpret_cast<uintptr_t>(dst) % 16)
        return NOVA_ERR_INVALID_ARG;
      e = launch_probe_copy(st, ctx->num_cus, src, dst, bytes);
      *work = 2.0 * (double)(bytes / 16 * 16);
      break;
    case NOVA_PROBE_MFMA:
      if (iters < 1) return NOVA_ERR_INVALID_ARG;
      e = launch_probe_mfma(st, ctx->num_cus, iters, sink);
      // workgroups x waves x rounds x MFMAs x flops of one 32x32x16 MFMA
      *work = (double)ctx->num_cus * 8.0 * (double)iters * 32.0 * (2.0 * 32 * 32 * 16);
      break;
    case NOVA_PROBE_MFMA_DATA:
      // every lane reads 128 bytes of operands: num_cus workgroups of 512 lanes
      if (iters < 1 || !src || reinterpret_cast<uintptr_t>(src) % 16 || bytes < (int64_t)ctx->num_cus * 512 * 128)
        return NOVA_ERR_INVALID_ARG;
      e = launch_probe_mfma_data(st, ctx->num_cus, src, iters, sink);
      *work = (double)ctx->num_cus * 8.0 * (double)iters * 32.0 * (2.0 * 32 * 32 * 16);
      break;
    default: return NOVA_ERR_INVALID_ARG;
  }
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_profile_stages(nova_ctx* ctx, uint32_t stage_mask) {
  if (!ctx || (stage_mask >> NOVA_STAGE_COUNT) != 0) return NOVA_ERR_INVALID_ARG;
  ctx->prof_mask = stage_mask;
  return NOVA_OK;
}

int nova_profile_collect(nova_ctx* ctx, int stage, double* total_ms, int64_t* launches) {
  if (!ctx || stage < 0 || stage >= NOVA_STAGE_COUNT) return NOVA_ERR_INVALID_ARG;
  double ms = 0.0;
  int64_t n = 0;
  int rc = NOVA_OK;
  std::vector<ProfRecord> keep;
  for (ProfRecord& r : ctx->prof) {
    if (r.stage != stage) { keep.push_back(r); continue; }
    float t = 0.f;
    if (hipEventSynchronize(r.stop) != hipSuccess || hipEventElapsedTime(&t, r.start, r.stop) != hipSuccess)
      rc = NOVA_ERR_HIP;
    else { ms += t; ++n; }
    (void)hipEventDestroy(r.start);
    (void)hipEventDestroy(r.stop);
  }
  ctx->prof.swap(keep);
  if (total_ms) *total_ms = ms;
  if (launches) *launches = n;
  return rc;
}

const char* nova_strerror(int code) {
  switch (code) {
    case NOVA_OK: return "ok";
    case NOVA_ERR_INVALID_ARG: return "invalid argument";
    case NOVA_ERR_UNSUPPORTED: return "unsupported shape or dtype";
    case NOVA_ERR_WORKSPACE: return "workspace too small or misaligned";
    case NOVA_ERR_HIP: return "HIP runtime error";
    case NOVA_ERR_STATIC_SCRATCH: return "request exceeds the static scratch of the allocation-free entry point";
    default: return "unknown error code";
  }
}

size_t nova_workspace_bytes(const nova_block_shape* shape) {
  if (shape_error(shape) != NOVA_OK || shape->k == 0 || shape->B == 0) return 0;
  return carve_workspace(*shape, nullptr).total;
}

int nova_entropy(nova_ctx* ctx, void* stream, const void* logits, int logits_dtype, int64_t rows_per_batch,
                 int batch, int V, int64_t row_stride_elems, float* entropy, float* mean_entropy) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (!valid_dtype(logits_dtype)) return NOVA_ERR_UNSUPPORTED;
  if (rows_per_batch < 0 || batch < 0 || V < 1 || row_stride_elems < V) return NOVA_ERR_INVALID_ARG;
  if (rows_per_batch == 0 || batch == 0) return NOVA_OK;
  if (!logits || !entropy) return NOVA_ERR_INVALID_ARG;
  return nova_entropy_blocks(ctx, stream, 1, &logits, logits_dtype, rows_per_batch, batch, V, row_stride_elems, &entropy,
                             mean_entropy ? &mean_entropy : nullptr);
}

int nova_entropy_blocks(nova_ctx* ctx, void* stream, int n_blocks, const void* const* logits, int logits_dtype,
                        int64_t rows_per_batch, int batch, int V, int64_t row_stride_elems, float* const* entropy,
                        float* const* mean_entropy) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (!valid_dtype(logits_dtype)) return NOVA_ERR_UNSUPPORTED;
  if (n_blocks < 0 || rows_per_batch < 0 || batch < 0 || V < 1 || row_stride_elems < V) return NOVA_ERR_INVALID_ARG;
  if (n_blocks == 0 || rows_per_batch == 0 || batch == 0) return NOVA_OK;
  if (!logits || !entropy) return NOVA_ERR_INVALID_ARG;
  if (rows_per_batch * batch > ((int64_t)1 << 31) - 8) return NOVA_ERR_UNSUPPORTED;
  for (int i = 0; i < n_blocks; ++i) {
    if (!logits[i] || !entropy[i] || (mean_entropy && !mean_entropy[i])) return NOVA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(logits[i]) % esize(logits_dtype)) != 0) return NOVA_ERR_INVALID_ARG;
  }
  if (int rc = set_device(ctx)) return rc;
  StageTimer timer(ctx, static_cast<hipStream_t>(stream), NOVA_STAGE_ENTROPY);
  hipError_t e = launch_entropy(static_cast<hipStream_t>(stream), ctx->num_cus, n_blocks, logits, logits_dtype, rows_per_batch,
                                batch, V, row_stride_elems, entropy, mean_entropy);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_entropy_bits(nova_ctx* ctx, void* stream, const void* bit_logits, int logits_dtype,
                      int64_t rows_per_batch, int batch, int d, float* entropy, float* mean_entropy) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (!valid_dtype(logits_dtype)) return NOVA_ERR_UNSUPPORTED;
  if (rows_per_batch < 0 || batch < 0 || d < 1) return NOVA_ERR_INVALID_ARG;
  if (rows_per_batch == 0 || batch == 0) return NOVA_OK;
  if (!bit_logits || !entropy) return NOVA_ERR_INVALID_ARG;
  if (rows_per_batch * batch > ((int64_t)1 << 31) - 8) return NOVA_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(bit_logits) % esize(logits_dtype)) != 0) return NOVA_ERR_INVALID_ARG;
  if (int rc = set_device(ctx)) return rc;
  hipError_t e = launch_entropy_bits(static_cast<hipStream_t>(stream), bit_logits, logits_dtype, rows_per_batch,
                                     batch, d, entropy, mean_entropy);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

size_t nova_head_entropy_workspace_bytes(int64_t rows_per_batch, int batch, int V) {
  if (rows_per_batch <= 0 || batch <= 0 || V < 1 || rows_per_batch * batch > ((int64_t)1 << 24)) return 0;
  return head_entropy_workspace_bytes((int)(rows_per_batch * batch), V);
}

int nova_head_entropy(nova_ctx* ctx, void* stream, const void* hidden, const void* w_head, const void* b_head,
                      int dtype, int64_t rows_per_batch, int batch, int C, int V, float* entropy,
                      float* mean_entropy, void* workspace, size_t workspace_bytes) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (dtype != NOVA_BF16) return NOVA_ERR_UNSUPPORTED;
  if (rows_per_batch < 0 || batch < 0 || V < 1 || C < 1) return NOVA_ERR_INVALID_ARG;
  if (rows_per_batch == 0 || batch == 0) return NOVA_OK;
  if (rows_per_batch * batch > ((int64_t)1 << 24)) return NOVA_ERR_UNSUPPORTED;
  if (C % 64 != 0) return NOVA_ERR_UNSUPPORTED;
  if (!hidden || !w_head || !entropy || !workspace) return NOVA_ERR_INVALID_ARG;
  for (const void* p : {hidden, w_head, b_head, (const void*)workspace})
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return NOVA_ERR_INVALID_ARG;
  if (workspace_bytes < nova_head_entropy_workspace_bytes(rows_per_batch, batch, V)) return NOVA_ERR_WORKSPACE;
  if (int rc = set_device(ctx)) return rc;
  hipError_t e = launch_head_entropy(ctx, static_cast<hipStream_t>(stream), hidden, w_head, b_head,
                                     (int)rows_per_batch, batch, C, V, entropy, mean_entropy, workspace);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_head_entropy_static(nova_ctx* ctx, void* stream, const void* hidden, const void* w_head,
                             const void* b_head, int dtype, int64_t rows_per_batch, int batch, int C, int V,
                             float* entropy, float* mean_entropy) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (dtype != NOVA_BF16) return NOVA_ERR_UNSUPPORTED;
  if (rows_per_batch < 0 || batch < 0 || V < 1 || C < 1) return NOVA_ERR_INVALID_ARG;
  if (rows_per_batch == 0 || batch == 0) return NOVA_OK;
  if (rows_per_batch * batch > ((int64_t)1 << 24)) return NOVA_ERR_UNSUPPORTED;
  if (C % 64 != 0) return NOVA_ERR_UNSUPPORTED;
  if (!hidden || !w_head || !entropy) return NOVA_ERR_INVALID_ARG;
  for (const void* p : {hidden, w_head, b_head})
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return NOVA_ERR_INVALID_ARG;
  if (head_entropy_partial_bytes(ctx, (int)(rows_per_batch * batch), V, C) > head_entropy_static_capacity())
    return NOVA_ERR_STATIC_SCRATCH;
  void* scratch_ptr = head_entropy_static_scratch(ctx->device);     // resolved by nova_create on this device
  if (!scratch_ptr) return NOVA_ERR_HIP;
  if (int rc = set_device(ctx)) return rc;
  hipError_t e = launch_head_entropy(ctx, static_cast<hipStream_t>(stream), hidden, w_head, b_head,
                                     (int)rows_per_batch, batch, C, V, entropy, mean_entropy, scratch_ptr);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_select(nova_ctx* ctx, void* stream, const float* entropy, int B, int N, int k, const int32_t* k_per_row,
                int32_t* kept_idx, uint8_t* keep_mask) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (B < 0 || N < 0 || k < 0 || k > N) return NOVA_ERR_INVALID_ARG;
  if (N > 65536) return NOVA_ERR_UNSUPPORTED;
  if (B == 0 || N == 0) return NOVA_OK;
  if (!entropy || !keep_mask || (k > 0 && !kept_idx)) return NOVA_ERR_INVALID_ARG;
  if (int rc = set_device(ctx)) return rc;
  StageTimer timer(ctx, static_cast<hipStream_t>(stream), NOVA_STAGE_SELECT);
  hipError_t e = launch_select(static_cast<hipStream_t>(stream), 1, &entropy, B, N, &k, k_per_row, &kept_idx, &keep_mask);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_select_blocks(nova_ctx* ctx, void* stream, int n_blocks, const float* const* entropy, int B, int N, const int32_t* k,
                       int32_t* const* kept_idx, uint8_t* const* keep_mask) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (n_blocks < 0 || B < 0 || N < 0 || (n_blocks > 0 && !k)) return NOVA_ERR_INVALID_ARG;
  for (int i = 0; i < n_blocks; ++i)
    if (k[i] < 0 || k[i] > N) return NOVA_ERR_INVALID_ARG;
  if (N > 65536) return NOVA_ERR_UNSUPPORTED;
  if (n_blocks == 0 || B == 0 || N == 0) return NOVA_OK;
  if (!entropy || !kept_idx || !keep_mask) return NOVA_ERR_INVALID_ARG;
  for (int i = 0; i < n_blocks; ++i)
    if (!entropy[i] || !keep_mask[i] || (k[i] > 0 && !kept_idx[i])) return NOVA_ERR_INVALID_ARG;
  if (int rc = set_device(ctx)) return rc;
  StageTimer timer(ctx, static_cast<hipStream_t>(stream), NOVA_STAGE_SELECT);
  hipError_t e = launch_select(static_cast<hipStream_t>(stream), n_blocks, entropy, B, N, k, nullptr, kept_idx, keep_mask);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_layer_ratio(nova_ctx* ctx, void* stream, const float* mean_entropy, float* entropy_sum,
                     const float* ratio_t, int j, int B, int N, float* ratio_tj, int32_t* k_per_row) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (j < 1 || B < 0 || N < 0 || N > (1 << 24)) return NOVA_ERR_INVALID_ARG;
  if (B == 0) return NOVA_OK;
  if (!mean_entropy || !entropy_sum || !ratio_t || !ratio_tj || !k_per_row) return NOVA_ERR_INVALID_ARG;
  if (int rc = set_device(ctx)) return rc;
  hipError_t e = launch_layer_ratio(static_cast<hipStream_t>(stream), mean_entropy, entropy_sum, ratio_t, j, B, N,
                                    ratio_tj, k_per_row);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_pruned_block(nova_ctx* ctx, void* stream, const nova_block_shape* shape,
                      const nova_block_weights* weights, const void* x, const int32_t* kept_idx, void* k_cache,
                      void* v_cache, void* y_kept, void* workspace, size_t workspace_bytes) {
  return nova_pruned_block_variant(ctx, stream, shape, weights, nullptr, x, kept_idx, k_cache, v_cache, y_kept,
                                   workspace, workspace_bytes);
}

int nova_pruned_block_variant(nova_ctx* ctx, void* stream, const nova_block_shape* shape,
                              const nova_block_weights* weights, const nova_block_variant* variant,
                              const void* x, const int32_t* kept_idx, void* k_cache, void* v_cache, void* y_kept,
                              void* workspace, size_t workspace_bytes) {
  return nova_pruned_block_rows(ctx, stream, shape, weights, variant, nullptr, nullptr, nullptr, x, kept_idx, k_cache,
                                v_cache, y_kept, workspace, workspace_bytes);
}

int nova_pruned_block_rows(nova_ctx* ctx, void* stream, const nova_block_shape* shape,
                           const nova_block_weights* weights, const nova_block_variant* variant,
                           const int32_t* k_per_row, const int32_t* kv_len_per_row, int32_t* kv_len_next,
                           const void* x, const int32_t* kept_idx, void* k_cache, void* v_cache, void* y_kept,
                           void* workspace, size_t workspace_bytes) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  const RowCounts rows = {k_per_row, kv_len_per_row, kv_len_next};
  nova_block_variant var;
  if (int rc = block_error(shape, weights, variant, rows, x, kept_idx, y_kept, &var)) return rc == 1 ? NOVA_OK : rc;
  if (!k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache)) return NOVA_ERR_INVALID_ARG;
  const size_t need = carve_workspace(*shape, nullptr).total;
  if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
    return NOVA_ERR_WORKSPACE;
  if (int rc = set_device(ctx)) return rc;
  const BlockWorkspace ws = carve_workspace(*shape, workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (shape->dtype == NOVA_BF16)
    e = launch_block_bf16(ctx, st, *shape, *weights, var, rows, x, kept_idx, k_cache, v_cache, y_kept, ws);
  else
    e = launch_block_f32(ctx, st, *shape, *weights, var, rows, static_cast<const float*>(x), kept_idx,
                         static_cast<float*>(k_cache), static_cast<float*>(v_cache), static_cast<float*>(y_kept), ws);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_merge_cache(nova_ctx* ctx, void* stream, int dtype, int B, int C, int h, int w, int hp, int wp, int k,
                     const void* x, const void* y_kept, const int32_t* kept_idx, const uint8_t* keep_mask,
                     const void* cache_prev, void* out, void* cache_new) {
  return nova_merge_cache_interp(ctx, stream, dtype, NOVA_INTERP_BILINEAR, B, C, h, w, hp, wp, k, x, y_kept, kept_idx,
                                 keep_mask, cache_prev, out, cache_new);
}

int nova_merge_cache_interp(nova_ctx* ctx, void* stream, int dtype, int interp, int B, int C, int h, int w, int hp,
                            int wp, int k, const void* x, const void* y_kept, const int32_t* kept_idx,
                            const uint8_t* keep_mask, const void* cache_prev, void* out, void* cache_new) {
  return nova_merge_cache_rows(ctx, stream, dtype, interp, B, C, h, w, hp, wp, k, nullptr, x, y_kept, kept_idx,
                               keep_mask, cache_prev, out, cache_new);
}

int nova_merge_cache_rows(nova_ctx* ctx, void* stream, int dtype, int interp, int B, int C, int h, int w, int hp,
                          int wp, int k, const int32_t* k_per_row, const void* x, const void* y_kept,
                          const int32_t* kept_idx, const uint8_t* keep_mask, const void* cache_prev, void* out,
                          void* cache_new) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(k_per_row) & 3) return NOVA_ERR_INVALID_ARG;
  if (interp != NOVA_INTERP_BILINEAR && interp != NOVA_INTERP_NEAREST && interp != NOVA_INTERP_BICUBIC)
    return NOVA_ERR_INVALID_ARG;
  if (!valid_dtype(dtype)) return NOVA_ERR_UNSUPPORTED;
  if (B < 0 || C < 1 || h < 0 || w < 0 || k < 0) return NOVA_ERR_INVALID_ARG;
  const int64_t N = (int64_t)h * w;
  if (k > N || N > ((int64_t)1 << 30)) return NOVA_ERR_INVALID_ARG;
  if (B == 0 || N == 0) return NOVA_OK;
  if (C % (16 / (int)esize(dtype)) != 0) return NOVA_ERR_UNSUPPORTED;
  if (!x || !out || !keep_mask || out == x) return NOVA_ERR_INVALID_ARG;
  if (k > 0 && (!y_kept || !kept_idx)) return NOVA_ERR_INVALID_ARG;
  // with per-image counts some image may keep fewer than k tokens: the prior cache is needed whatever k is
  if ((k < N || k_per_row) && (!cache_prev || hp < 1 || wp < 1)) return NOVA_ERR_INVALID_ARG;
  if (hp < 1 || wp < 1) cache_prev = nullptr;   // only reachable with k == N: an empty prior grid is never sampled
  const void* ptrs[] = {x, y_kept, cache_prev, out, cache_new};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return NOVA_ERR_INVALID_ARG;
  if (int rc = set_device(ctx)) return rc;
  StageTimer timer(ctx, static_cast<hipStream_t>(stream), NOVA_STAGE_MERGE);
  hipError_t e = launch_merge(static_cast<hipStream_t>(stream), dtype, interp, B, C, h, w, hp, wp, k, x, y_kept, kept_idx,
                              keep_mask, cache_prev, out, cache_new, k_per_row);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_fourbit_append(nova_ctx* ctx, void* stream, int dtype, const nova_fourbit_cache* cache, int n, const nova_rows* k,
                        const nova_rows* v, const int32_t* n_per_row, int kv_len, const int32_t* kv_len_per_row,
                        int32_t* kv_len_next) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (!valid_dtype(dtype)) return NOVA_ERR_UNSUPPORTED;
  if (int rc = fourbit_error(cache)) return rc;
  if (n < 0 || kv_len < 0 || (int64_t)kv_len + n > cache->capacity) return NOVA_ERR_INVALID_ARG;
  if (int rc = counts_error({n_per_row, kv_len_per_row, kv_len_next})) return rc;
  const int B = cache->B, hk = cache->kv_heads;
  for (const void* p : {n_per_row, kv_len_per_row})
    if (overlap(kv_len_next, (size_t)B * 4, p, (size_t)B * 4)) return NOVA_ERR_INVALID_ARG;
  if ((int64_t)B * hk * n > (int64_t)1 << 36) return NOVA_ERR_UNSUPPORTED;
  if (B == 0) return NOVA_OK;
  nova_rows ks = {}, vs = {};
  if (n > 0) {
    if (!k || !v) return NOVA_ERR_INVALID_ARG;
    for (const nova_rows* r : {k, v})
      if (int rc = rows_error(r, dtype, B, n, hk, false)) return rc;
    ks = settled(*k, B, n, hk);
    vs = settled(*v, B, n, hk);
  }
  const DeviceScope device(ctx);
  if (device.rc) return device.rc;
  return launch_fourbit_append(static_cast<hipStream_t>(stream), dtype, *cache, n, &ks, &vs, n_per_row, kv_len, kv_len_per_row,
                               kv_len_next) == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_fourbit_unpack(nova_ctx* ctx, void* stream, int dtype, const nova_fourbit_cache* cache, int first, int n,
                        const int32_t* first_per_row, const int32_t* n_per_row, const nova_rows* k, const nova_rows* v) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (!valid_dtype(dtype)) return NOVA_ERR_UNSUPPORTED;
  if (int rc = fourbit_error(cache)) return rc;
  if (n < 0 || first < 0 || (int64_t)first + n > cache->capacity) return NOVA_ERR_INVALID_ARG;
  if (int rc = counts_error({first_per_row, n_per_row})) return rc;
  const int B = cache->B, hk = cache->kv_heads;
  if ((int64_t)B * hk * n > (int64_t)1 << 36) return NOVA_ERR_UNSUPPORTED;
  if (B == 0 || n == 0 || (!k && !v)) return NOVA_OK;
  nova_rows out[2] = {};
  const nova_rows* in[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    if (!in[i]) continue;
    if (int rc = rows_error(in[i], dtype, B, n, hk, false)) return rc;
    out[i] = settled(*in[i], B, n, hk);
    if (out[i].stride_channel == 0 || (n > 1 && out[i].stride_row == 0) || (hk > 1 && out[i].stride_head == 0) ||
        (B > 1 && out[i].stride_b == 0))
      return NOVA_ERR_INVALID_ARG;
  }
  const DeviceScope device(ctx);
  if (device.rc) return device.rc;
  return launch_fourbit_unpack(static_cast<hipStream_t>(stream), dtype, *cache, first, n, first_per_row, n_per_row, &out[0],
                               &out[1]) == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

size_t nova_fourbit_attention_workspace_bytes(const nova_fourbit_cache* cache, int heads, int n, int kv_len) {
  return query_has_work(cache, heads, n, kv_len) ? fourbit_attention_workspace_bytes(*cache, heads, n, kv_len) : 0;
}

int nova_fourbit_attention(nova_ctx* ctx, void* stream, int dtype, const nova_fourbit_cache* cache, int heads, int n,
                           const nova_rows* q, const int32_t* n_per_row, int kv_len, const int32_t* kv_len_per_row, float scale,
                           void* out, float* lse, void* workspace, size_t workspace_bytes) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (int rc = fourbit_query_error(dtype, cache, heads, n, q, kv_len)) return rc;
  if (int rc = counts_error({n_per_row, kv_len_per_row, lse})) return rc;
  if (cache->B == 0 || n == 0) return NOVA_OK;
  if (!out || !aligned16(out) || out == q->data) return NOVA_ERR_INVALID_ARG;
  const size_t need = nova_fourbit_attention_workspace_bytes(cache, heads, n, kv_len);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace))) return NOVA_ERR_WORKSPACE;
  const DeviceScope device(ctx);
  if (device.rc) return device.rc;
  return launch_fourbit_attention(ctx, static_cast<hipStream_t>(stream), dtype, *cache, heads, n,
                                  settled(*q, cache->B, n, heads), n_per_row, kv_len, kv_len_per_row, scale * kAttnLog2e, out,
                                  lse, workspace) == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

size_t nova_fourbit_mass_workspace_bytes(const nova_fourbit_cache* cache, int heads, int n, int kv_len) {
  return query_has_work(cache, heads, n, kv_len) ? fourbit_mass_workspace_bytes(*cache, heads, n, kv_len) : 0;
}

int nova_fourbit_mass(nova_ctx* ctx, void* stream, int dtype, const nova_fourbit_cache* cache, int heads, int n,
                      const nova_rows* q, const int32_t* n_per_row, int kv_len, const int32_t* kv_len_per_row, float scale,
                      const float* lse, const float* mass_in, float* mass, void* workspace, size_t workspace_bytes) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (int rc = fourbit_query_error(dtype, cache, heads, n, q, kv_len)) return rc;
  if (int rc = counts_error({n_per_row, kv_len_per_row, lse, mass_in, mass})) return rc;
  if (cache->B == 0 || cache->capacity == 0) return NOVA_OK;
  if (!mass || (n > 0 && !lse)) return NOVA_ERR_INVALID_ARG;
  const size_t mass_bytes = (size_t)cache->B * cache->capacity * 4;
  if (mass_in != mass && overlap(mass_in, mass_bytes, mass, mass_bytes)) return NOVA_ERR_INVALID_ARG;
  const size_t need = nova_fourbit_mass_workspace_bytes(cache, heads, n, kv_len);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace))) return NOVA_ERR_WORKSPACE;
  const DeviceScope device(ctx);
  if (device.rc) return device.rc;
  const nova_rows none = {};
  return launch_fourbit_mass(ctx, static_cast<hipStream_t>(stream), dtype, *cache, heads, n,
                             n > 0 ? settled(*q, cache->B, n, heads) : none, n_per_row, kv_len, kv_len_per_row,
                             scale * kAttnLog2e, lse, mass_in, mass, workspace) == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

int nova_fourbit_evict(nova_ctx* ctx, void* stream, const nova_fourbit_cache* src, const nova_fourbit_cache* dst, int k,
                       const int32_t* kept_idx, const int32_t* k_per_row, int kv_len, const int32_t* kv_len_per_row,
                       int32_t* kv_len_next, const float* mass_src, float* mass_dst) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  for (const nova_fourbit_cache* c : {src, dst})
    if (int rc = fourbit_error(c)) return rc;
  if (src->B != dst->B || src->kv_heads != dst->kv_heads || src->dh != dst->dh) return NOVA_ERR_INVALID_ARG;
  if (k < 0 || k > dst->capacity || kv_len < 0 || kv_len > src->capacity || !mass_src != !mass_dst) return NOVA_ERR_INVALID_ARG;
  if (int rc = counts_error({kept_idx, k_per_row, kv_len_per_row, kv_len_next, mass_src, mass_dst})) return rc;
  const size_t B = (size_t)src->B, rows_src = B * src->kv_heads * src->capacity, rows_dst = B * src->kv_heads * dst->capacity;
  if (B == 0) return NOVA_OK;
  if (k > 0 && !kept_idx) return NOVA_ERR_INVALID_ARG;
  for (const void* p : {k_per_row, kv_len_per_row})
    if (overlap(kv_len_next, B * 4, p, B * 4)) return NOVA_ERR_INVALID_ARG;
  if (overlap(kv_len_next, B * 4, kept_idx, B * k * 4) ||
      overlap(mass_src, B * src->capacity * 4, mass_dst, B * dst->capacity * 4))
    return NOVA_ERR_INVALID_ARG;
  const size_t row_codes = src->dh / 2, row_scales = src->dh / 32;
  for (const void* s : {src->k_codes, src->v_codes})
    for (const void* d : {dst->k_codes, dst->v_codes})
      if (overlap(s, rows_src * row_codes, d, rows_dst * row_codes)) return NOVA_ERR_INVALID_ARG;
  for (const void* s : {src->k_scales, src->v_scales})
    for (const void* d : {dst->k_scales, dst->v_scales})
      if (overlap(s, rows_src * row_scales, d, rows_dst * row_scales)) return NOVA_ERR_INVALID_ARG;
  const DeviceScope device(ctx);
  if (device.rc) return device.rc;
  return launch_fourbit_evict(static_cast<hipStream_t>(stream), *src, *dst, k, kept_idx, k_per_row, kv_len, kv_len_per_row,
                              kv_len_next, mass_src, mass_dst) == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

size_t nova_fourbit_block_workspace_bytes(const nova_block_shape* shape) {
  if (fourbit_shape_error(shape) != NOVA_OK || shape->k == 0 || shape->B == 0) return 0;
  FourBitBlock fb = {};
  return carve_fourbit(*shape, nullptr, &fb);
}

int nova_pruned_block_fourbit(nova_ctx* ctx, void* stream, const nova_block_shape* shape, const nova_block_weights* weights,
                              const nova_block_variant* variant, const int32_t* k_per_row, const int32_t* kv_len_per_row,
                              int32_t* kv_len_next, const void* x, const int32_t* kept_idx, const nova_fourbit_cache* cache,
                              const float* mass_in, float* mass, void* y_kept, void* workspace, size_t workspace_bytes) {
  if (!ctx) return NOVA_ERR_INVALID_ARG;
  if (int rc = fourbit_shape_error(shape)) return rc;
  if (int rc = fourbit_error(cache)) return rc;
  if (cache->B != shape->B || cache->kv_heads != shape->heads || cache->dh != shape->C / shape->heads ||
      cache->capacity != shape->kv_capacity)
    return NOVA_ERR_INVALID_ARG;
  if (int rc = counts_error({mass_in, mass})) return rc;
  if (mass_in && !mass) return NOVA_ERR_INVALID_ARG;
  const size_t mass_bytes = (size_t)cache->B * cache->capacity * 4;
  if (mass_in != mass && overlap(mass_in, mass_bytes, mass, mass_bytes)) return NOVA_ERR_INVALID_ARG;
  const RowCounts rows = {k_per_row, kv_len_per_row, kv_len_next};
  nova_block_variant var;
  const nova_block_shape plain = fourbit_plain_shape(*shape);
  if (int rc = block_error(&plain, weights, variant, rows, x, kept_idx, y_kept, &var)) return rc == 1 ? NOVA_OK : rc;
  FourBitBlock fb = {};
  const size_t need = carve_fourbit(*shape, nullptr, &fb);
  if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
    return NOVA_ERR_WORKSPACE;
  const DeviceScope device(ctx);
  if (device.rc) return device.rc;
  carve_fourbit(*shape, workspace, &fb);
  fb.cache = *cache;
  fb.mass_in = mass_in;
  fb.mass = mass;
  const BlockWorkspace ws = carve_workspace(plain, workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (shape->dtype == NOVA_BF16)
    e = launch_block_bf16(ctx, st, *shape, *weights, var, rows, x, kept_idx, nullptr, nullptr, y_kept, ws, &fb);
  else
    e = launch_block_f32(ctx, st, *shape, *weights, var, rows, static_cast<const float*>(x), kept_idx, nullptr, nullptr,
                         static_cast<float*>(y_kept), ws, &fb);
  return e == hipSuccess ? NOVA_OK : NOVA_ERR_HIP;
}

}  // extern "C"
