// Host part of the paged 4-bit cache: argument checks, contexts, launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <string>

#include "kv.h"

struct wf_kv_ctx {
  int device = 0;
  int dtype = 0;
  wfkv::Geo g{};
  int n_cu = 0;
  char* areas = nullptr;             // kAreas work areas: sums, then the two arrays of counts
  void* owner[wfkv::kAreas] = {};    // the streams that have them
  int owners = 0;
  char err[256] = "";
};

namespace {

thread_local char g_kv_err[256] = "";

wf_status fail(wf_kv_ctx* ctx, wf_status st, const char* fmt, ...) __attribute__((format(printf, 3, 4)));
wf_status fail(wf_kv_ctx* ctx, wf_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(ctx ? ctx->err : g_kv_err, sizeof(g_kv_err), fmt, ap);
  va_end(ap);
  return st;
}

wf_status check_desc(const wf_kv_desc* d) {
  if (!d) return fail(nullptr, WF_EINVAL, "desc is NULL");
  if (d->kv_heads < 1 || d->q_heads < 1 || d->q_heads > WF_KV_MAX_HEADS || d->q_heads % d->kv_heads)
    return fail(nullptr, WF_EINVAL, "q_heads=%d must be a multiple of kv_heads=%d in [1, %d]", d->q_heads,
                d->kv_heads, WF_KV_MAX_HEADS);
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
    return fail(nullptr, WF_EUNSUPPORTED, "head_dim=%d is not 64, 128 or 256", d->head_dim);
  const int b = d->block_tokens;
  if (b < 16 || b > 256 || (b & (b - 1)))
    return fail(nullptr, WF_EUNSUPPORTED, "block_tokens=%d is not 16, 32, 64, 128 or 256", b);
  if (d->n_blocks < 1 || d->n_blocks > WF_KV_MAX_BLOCKS)
    return fail(nullptr, WF_EINVAL, "n_blocks=%d outside [1, %d]", d->n_blocks, WF_KV_MAX_BLOCKS);
  if (d->max_blocks < 1 || d->max_blocks > WF_KV_MAX_WIDTH || (int64_t)d->max_blocks * b > (1ll << 30))
    return fail(nullptr, WF_EINVAL, "max_blocks=%d outside [1, %d] or rows above 2^30 tokens", d->max_blocks,
                WF_KV_MAX_WIDTH);
  if (d->dtype != WF_KV_BF16 && d->dtype != WF_KV_F16)
    return fail(nullptr, WF_EINVAL, "dtype=%d is not WF_KV_BF16 or WF_KV_F16", d->dtype);
  return WF_OK;
}

int64_t cell_bytes(const wf_kv_desc* d) { return (int64_t)d->block_tokens * (d->head_dim + 4); }

// Makes the context's device the current one for a scope.
struct OnDevice {
  int prev = 0;
  hipError_t e;
  explicit OnDevice(int device) {
    e = hipGetDevice(&prev);
    if (e == hipSuccess && prev != device) e = hipSetDevice(device);
    changed = e == hipSuccess && prev != device;
  }
  ~OnDevice() {
    if (changed) (void)hipSetDevice(prev);
  }
  bool changed = false;
};

template <class F>
wf_status launch(wf_kv_ctx* ctx, const char* what, F&& f) {
  OnDevice on(ctx->device);
  hipError_t e = on.e;
  if (e == hipSuccess) e = f();
  if (e != hipSuccess) return fail(ctx, WF_EHIP, "%s: %s", what, hipGetErrorString(e));
  return WF_OK;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The work area of a stream, for good; none for those that come when all are given.
wfkv::AttendWork area_of(wf_kv_ctx* ctx, void* stream) {
  int i = 0;
  while (i < ctx->owners && ctx->owner[i] != stream) ++i;
  if (i == wfkv::kAreas) return wfkv::AttendWork{ctx->n_cu, nullptr, 0, nullptr, nullptr, 0};
  if (i == ctx->owners) ctx->owner[ctx->owners++] = stream;
  char* at = ctx->areas + i * wfkv::kAreaBytes;
  char* counts = at + wfkv::kPartBytes;
  return wfkv::AttendWork{ctx->n_cu, reinterpret_cast<float*>(at), wfkv::kPartBytes, reinterpret_cast<int32_t*>(counts),
                          reinterpret_cast<int32_t*>(counts + wfkv::kCountBytes), wfkv::kCountBytes};
}

wf_status null_ctx() { return fail(nullptr, WF_EINVAL, "ctx is NULL"); }

}  // namespace

extern "C" {

wf_status wf_kv_cache_bytes(const wf_kv_desc* desc, int64_t* bytes) {
  const wf_status st = check_desc(desc);
  if (st != WF_OK) return st;
  if (!bytes) return fail(nullptr, WF_EINVAL, "bytes is NULL");
  *bytes = (int64_t)desc->n_blocks * desc->kv_heads * cell_bytes(desc);
  return WF_OK;
}

wf_status wf_kv_ctx_create(int hip_device, const wf_kv_desc* desc, wf_kv_ctx** out) {
  if (!out) return fail(nullptr, WF_EINVAL, "out is NULL");
  *out = nullptr;
  const wf_status st = check_desc(desc);
  if (st != WF_OK) return st;
  int n = 0;
  const hipError_t e = hipGetDeviceCount(&n);
  if (e != hipSuccess || n <= 0) return fail(nullptr, WF_EHIP, "no HIP device: %s", hipGetErrorString(e));
  if (hip_device < 0 || hip_device >= n) return fail(nullptr, WF_EINVAL, "hip_device out of range");
  wf_kv_ctx* ctx = new (std::nothrow) wf_kv_ctx();
  if (!ctx) return fail(nullptr, WF_ENOMEM, "out of host memory");
  ctx->device = hip_device;
  ctx->dtype = desc->dtype;
  wfkv::Geo& g = ctx->g;
  g.hq = desc->q_heads;
  g.hk = desc->kv_heads;
  g.d = desc->head_dim;
  g.group = g.hq / g.hk;
  g.b = desc->block_tokens;
  g.b_log2 = __builtin_ctz((unsigned)g.b);
  g.n_blocks = desc->n_blocks;
  g.width = desc->max_blocks;
  g.cell = (int)cell_bytes(desc);
  wf_status made = launch(ctx, "wf_kv_ctx_create", [&] {
    hipError_t e = hipDeviceGetAttribute(&ctx->n_cu, hipDeviceAttributeMultiprocessorCount, hip_device);
    if (e == hipSuccess) e = hipMalloc(&ctx->areas, wfkv::kAreas * wfkv::kAreaBytes);
    if (e != hipSuccess) return e;
    e = hipMemset2D(ctx->areas + wfkv::kPartBytes, wfkv::kAreaBytes, 0, 2 * wfkv::kCountBytes, wfkv::kAreas);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) (void)hipFree(ctx->areas);
    return e;
  });
  if (made != WF_OK) {
    const wf_status st = fail(nullptr, made, "%s", ctx->err);
    delete ctx;
    return st;
  }
  *out = ctx;
  return WF_OK;
}

void wf_kv_ctx_destroy(wf_kv_ctx* ctx) {
  if (!ctx) return;
  {
    OnDevice on(ctx->device);
    (void)hipFree(ctx->areas);
  }
  delete ctx;
}

const char* wf_kv_last_error(const wf_kv_ctx* ctx) { return ctx ? ctx->err : g_kv_err; }

wf_status wf_kv_step(wf_kv_ctx* ctx, const int32_t* new_tokens, int32_t n_rows, int32_t n_tokens,
                     const int32_t* len_in, int32_t* len_out, const int32_t* pool_in, int32_t* pool_out,
                     int32_t* ring, int32_t* table, int32_t* q_off, int64_t* slot, int32_t* pos,
                     uint8_t* granted, void* hip_stream) {
  if (!ctx) return null_ctx();
  if (n_rows < 0 || n_rows > WF_KV_MAX_ROWS)
    return fail(ctx, WF_EINVAL, "n_rows=%d outside [0, %d]", n_rows, WF_KV_MAX_ROWS);
  if (n_tokens < 0 || n_tokens > WF_KV_MAX_TOKENS)
    return fail(ctx, WF_EINVAL, "n_tokens=%d outside [0, %d]", n_tokens, WF_KV_MAX_TOKENS);
  if (!pool_in || !pool_out || !ring || !q_off) return fail(ctx, WF_EINVAL, "pool_in, pool_out, ring or q_off is NULL");
  if (n_rows && (!new_tokens || !len_in || !len_out || !table || !granted))
    return fail(ctx, WF_EINVAL, "a row array (new_tokens, len_in, len_out, table, granted) is NULL");
  if (n_tokens && (!slot || !pos)) return fail(ctx, WF_EINVAL, "slot or pos is NULL");
  if ((n_rows && len_in == len_out) || pool_in == pool_out)
    return fail(ctx, WF_EINVAL, "len_out and pool_out must not be len_in and pool_in");
  const wfkv::StepArgs a{new_tokens, n_rows, n_tokens, len_in, len_out, pool_in, pool_out,
                         ring, table, q_off, slot, pos, granted};
  return launch(ctx, "wf_kv_step", [&] { return wfkv::launch_step(ctx->g, a, (hipStream_t)hip_stream); });
}

wf_status wf_kv_store(wf_kv_ctx* ctx, const void* q, const void* k, const void* v, int64_t q_stride,
                      int64_t k_stride, int64_t v_stride, int32_t n_tokens, const wf_kv_norm_rope* how,
                      const int32_t* pos, const int64_t* slot, void* q_out, uint8_t* cache,
                      void* hip_stream) {
  if (!ctx) return null_ctx();
  const wfkv::Geo& g = ctx->g;
  if (n_tokens < 0 || n_tokens > WF_KV_MAX_TOKENS)
    return fail(ctx, WF_EINVAL, "n_tokens=%d outside [0, %d]", n_tokens, WF_KV_MAX_TOKENS);
  if (!how) return fail(ctx, WF_EINVAL, "how is NULL");
  if (!std::isfinite(how->eps) || how->eps < 0) return fail(ctx, WF_EINVAL, "eps must be finite and >= 0");
  if (how->rot_dim < 0 || how->rot_dim > g.d || how->rot_dim % 16)
    return fail(ctx, WF_EINVAL, "rot_dim=%d is not a multiple of 16 in [0, %d]", how->rot_dim, g.d);
  if (how->interleaved != 0 && how->interleaved != 1) return fail(ctx, WF_EINVAL, "interleaved is not 0 or 1");
  if (how->rot_dim && (!how->cos_sin || how->n_pos < 1))
    return fail(ctx, WF_EINVAL, "cos_sin is NULL or has no rows");
  if (n_tokens == 0) return WF_OK;
  if (!q || !k || !v || !slot || !q_out || !cache || (how->rot_dim && !pos))
    return fail(ctx, WF_EINVAL, "q, k, v, pos, slot, q_out or cache is NULL");
  if (q_stride < (int64_t)g.hq * g.d || k_stride < (int64_t)g.hk * g.d || v_stride < (int64_t)g.hk * g.d ||
      q_stride % 8 || k_stride % 8 || v_stride % 8)
    return fail(ctx, WF_EINVAL, "a token stride is below its heads' channels or not a multiple of 8");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(cache, 16) ||
      !aligned(how->q_weight, 16) || !aligned(how->k_weight, 16) || !aligned(how->cos_sin, 16))
    return fail(ctx, WF_EINVAL, "q, k, v, q_out, cache, weights and cos_sin must be aligned to 16 bytes");
  const wfkv::StoreArgs a{q, k, v, q_stride, k_stride, v_stride, n_tokens, *how, pos, slot, q_out, cache};
  return launch(ctx, "wf_kv_store", [&] { return wfkv::launch_store(g, ctx->dtype, a, (hipStream_t)hip_stream); });
}

wf_status wf_kv_load(wf_kv_ctx* ctx, const uint8_t* cache, const int64_t* slot, int32_t n_tokens, void* k_out,
                     void* v_out, void* hip_stream) {
  if (!ctx) return null_ctx();
  if (n_tokens < 0 || n_tokens > WF_KV_MAX_TOKENS)
    return fail(ctx, WF_EINVAL, "n_tokens=%d outside [0, %d]", n_tokens, WF_KV_MAX_TOKENS);
  if (n_tokens == 0) return WF_OK;
  if (!cache || !slot || !k_out || !v_out) return fail(ctx, WF_EINVAL, "cache, slot, k_out or v_out is NULL");
  if (!aligned(cache, 16) || !aligned(k_out, 16) || !aligned(v_out, 16))
    return fail(ctx, WF_EINVAL, "cache, k_out and v_out must be aligned to 16 bytes");
  const wfkv::LoadArgs a{cache, slot, n_tokens, k_out, v_out};
  return launch(ctx, "wf_kv_load", [&] { return wfkv::launch_load(ctx->g, ctx->dtype, a, (hipStream_t)hip_stream); });
}

wf_status wf_kv_attend(wf_kv_ctx* ctx, const void* q, int64_t q_stride, int32_t n_tokens, const uint8_t* cache,
                       const int32_t* table, const int32_t* kv_len, const int32_t* q_off, const int32_t* pos,
                       int32_t n_rows, float scale, int32_t window, int32_t max_q, int32_t max_kv, void* out,
                       void* hip_stream) {
  if (!ctx) return null_ctx();
  const wfkv::Geo& g = ctx->g;
  if (n_rows < 0 || n_rows > WF_KV_MAX_ROWS)
    return fail(ctx, WF_EINVAL, "n_rows=%d outside [0, %d]", n_rows, WF_KV_MAX_ROWS);
  if (n_tokens < 0 || n_tokens > WF_KV_MAX_TOKENS)
    return fail(ctx, WF_EINVAL, "n_tokens=%d outside [0, %d]", n_tokens, WF_KV_MAX_TOKENS);
  if (!std::isfinite(scale)) return fail(ctx, WF_EINVAL, "scale must be finite");
  if (window < 0 || max_q < 0 || max_kv < 0) return fail(ctx, WF_EINVAL, "window, max_q and max_kv must be >= 0");
  if (n_rows == 0 || n_tokens == 0) return WF_OK;
  if (!q || !cache || !table || !kv_len || !q_off || !pos || !out)
    return fail(ctx, WF_EINVAL, "q, cache, table, kv_len, q_off, pos or out is NULL");
  if (q_stride < (int64_t)g.hq * g.d || q_stride % 8)
    return fail(ctx, WF_EINVAL, "q_stride is below the heads' channels or not a multiple of 8");
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(cache, 16))
    return fail(ctx, WF_EINVAL, "q, out and cache must be aligned to 16 bytes");
  const wfkv::AttendArgs a{q, q_stride, n_tokens, cache, table, kv_len, q_off, pos, n_rows, scale,
                           window, max_q, max_kv, out};
  const wfkv::AttendWork work = area_of(ctx, hip_stream);
  return launch(ctx, "wf_kv_attend", [&] { return wfkv::launch_attend(g, ctx->dtype, a, work, (hipStream_t)hip_stream); });
}

}  // extern "C"
