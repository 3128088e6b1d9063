// C-ABI of liblsv (declared in include/lsv.h): host-side validation, then launches.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "lsv_attn.h"
#include "lsv_device.h"
#include "lsv_gemm.h"
#include "lsv_internal.h"
#include "lsv_ops.h"

namespace {

thread_local char g_err[512] = "";

struct TimingHook {
  int kernel = 0, n = 0;
  unsigned flags = 0;
  hipEvent_t ev[2 * LSV_MAX_TIMING_SLOTS];
} g_timing;

int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return code;
}
int ok() {
  g_err[0] = 0;
  return LSV_OK;
}
int hip_rc(int rc, const char* what) {
  if (rc == LSV_ERR_HIP && strncmp(g_err, "timing event", 12) == 0) return rc;
  if (rc == LSV_ERR_HIP) return fail(LSV_ERR_HIP, "%s: %s", what, hipGetErrorString(hipGetLastError()));
  if (rc == LSV_ERR_UNSUPPORTED) return fail(rc, "%s: unsupported shape", what);
  if (rc != LSV_OK) return fail(rc, "%s failed", what);
  return ok();
}

int check_config(const lsv_model_config* c) {
  if (!c) return fail(LSV_ERR_INVALID_ARG, "cfg is NULL");
  if (c->n_layers < 1 || c->d_model < 64 || c->d_model % 64 || c->n_q_heads < 1 || c->n_kv_heads < 1 ||
      c->n_q_heads % c->n_kv_heads || c->d_ff < 4 || c->d_ff % 4 || c->vocab < 1)
    return fail(LSV_ERR_INVALID_ARG, "bad model dimensions (d_model %% 64, n_q %% n_kv, d_ff %% 4 required)");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(LSV_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (c->d_model > 8192) return fail(LSV_ERR_UNSUPPORTED, "d_model must be <= 8192");
  if (c->dtype != LSV_DTYPE_F32 && c->dtype != LSV_DTYPE_BF16) return fail(LSV_ERR_INVALID_ARG, "bad dtype");
  if (!(c->rms_eps > 0.f) || !(c->rope_base > 0.0) || !isfinite(c->rope_base) || c->reserved0 != 0.f)
    return fail(LSV_ERR_INVALID_ARG, "bad rms_eps / rope_base / reserved0");
  // the weight streams address a packed matrix with 32-bit byte offsets
  const lsv::ModelLayout ml = lsv::model_layout(lsv::shape_of(c));
  for (const lsv::PackedMat* p : {&ml.lm_head, &ml.qkv, &ml.o, &ml.gateup, &ml.down})
    if ((size_t)p->Nt * p->Kt * 1024 >= ((size_t)1 << 32))
      return fail(LSV_ERR_UNSUPPORTED, "a packed projection of %zu bytes reaches 4 GiB", (size_t)p->Nt * p->Kt * 1024);
  return LSV_OK;
}

}  // namespace

extern "C" {

const char* lsv_status_string(int s) {
  switch (s) {
    case LSV_OK: return "ok";
    case LSV_ERR_INVALID_ARG: return "invalid argument";
    case LSV_ERR_UNSUPPORTED: return "unsupported configuration";
    case LSV_ERR_HIP: return "HIP runtime error";
    case LSV_ERR_CAPACITY: return "KV-cache capacity exceeded";
    case LSV_ERR_NONFINITE: return "non-finite value";
  }
  return "unknown status";
}

const char* lsv_last_error(void) { return g_err; }
int lsv_abi_version(void) { return 3; }

size_t lsv_packed_model_bytes(const lsv_model_config* cfg) {
  if (check_config(cfg) != LSV_OK) return 0;
  return lsv::model_layout(lsv::shape_of(cfg)).total;
}

int lsv_pack_globals(const lsv_model_config* cfg, const void* d_embed, const void* d_final_norm, const void* d_lm_head,
                     void* d_packed, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!d_embed || !d_final_norm || !d_lm_head || !d_packed) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  const lsv::Shape s = lsv::shape_of(cfg);
  const lsv::ModelLayout ml = lsv::model_layout(s);
  hipStream_t st = (hipStream_t)stream;
  char* P = (char*)d_packed;
  if (hipMemcpyAsync(P + ml.embed, d_embed, (size_t)s.V * s.d * s.es, hipMemcpyDeviceToDevice, st) != hipSuccess)
    return fail(LSV_ERR_HIP, "copy: %s", hipGetErrorString(hipGetLastError()));
  if ((rc = lsv::launch_pack(s, lsv::PACK_PLAIN, ml.lm_head, d_lm_head, nullptr, nullptr, P, st)) ||
      (rc = lsv::launch_gain(s, d_final_norm, P + ml.final_norm, st)))
    return hip_rc(rc, "pack globals");
  return ok();
}

int lsv_pack_layer(const lsv_model_config* cfg, int32_t layer, const void* d_wq, const void* d_wk, const void* d_wv,
                   const void* d_wo, const void* d_wg, const void* d_wu, const void* d_wd, const void* d_attn_norm,
                   const void* d_ffn_norm, void* d_packed, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (layer < 0 || layer >= cfg->n_layers) return fail(LSV_ERR_INVALID_ARG, "layer %d out of range", layer);
  if (!d_wq || !d_wk || !d_wv || !d_wo || !d_wg || !d_wu || !d_wd || !d_attn_norm || !d_ffn_norm || !d_packed)
    return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  const lsv::Shape s = lsv::shape_of(cfg);
  const lsv::ModelLayout ml = lsv::model_layout(s);
  hipStream_t st = (hipStream_t)stream;
  char* LB = (char*)d_packed + ml.layer_base + (size_t)layer * ml.layer_stride;
  if ((rc = lsv::launch_pack(s, lsv::PACK_QKV, ml.qkv, d_wq, d_wk, d_wv, LB, st)) ||
      (rc = lsv::launch_pack(s, lsv::PACK_PLAIN, ml.o, d_wo, nullptr, nullptr, LB, st)) ||
      (rc = lsv::launch_pack(s, lsv::PACK_GATEUP, ml.gateup, d_wg, d_wu, nullptr, LB, st)) ||
      (rc = lsv::launch_pack(s, lsv::PACK_PLAIN, ml.down, d_wd, nullptr, nullptr, LB, st)) ||
      (rc = lsv::launch_gain(s, d_attn_norm, LB + ml.attn_norm, st)) ||
      (rc = lsv::launch_gain(s, d_ffn_norm, LB + ml.ffn_norm, st)))
    return hip_rc(rc, "pack layer");
  return ok();
}

size_t lsv_kv_cache_bytes(const lsv_model_config* cfg, int32_t batch, int32_t capacity) {
  if (check_config(cfg) != LSV_OK || batch < 1 || capacity < 1 || capacity % LSV_KV_ALIGN) return 0;
  const lsv::Shape s = lsv::shape_of(cfg);
  return (size_t)s.L * 2 * batch * s.nkv * (size_t)capacity * s.hd * s.es;
}

size_t lsv_verify_workspace_bytes(const lsv_model_config* cfg, int32_t batch, int32_t max_rows, int32_t max_ctx) {
  if (check_config(cfg) != LSV_OK || batch < 1 || max_rows < 1 || max_rows > LSV_MAX_ROWS || max_ctx < 1) return 0;
  return lsv::verify_workspace_bytes(lsv::shape_of(cfg), batch, max_rows, max_ctx);
}

__global__ void lsv_clear_kernel(uint4* p, size_t n16) {
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += (size_t)gridDim.x * blockDim.x)
    p[i] = make_uint4(0, 0, 0, 0);
}

int lsv_workspace_clear(void* d_workspace, size_t bytes, void* stream) {
  if (!d_workspace || bytes % 16 || ((uintptr_t)d_workspace & 15))
    return fail(LSV_ERR_INVALID_ARG, "workspace must be non-NULL, 16-byte aligned and a multiple of 16 bytes");
  const size_t n16 = bytes / 16;
  unsigned blocks = (unsigned)((n16 + 255) / 256);
  blocks = blocks > 4096 ? 4096 : (blocks == 0 ? 1 : blocks);
  hipLaunchKernelGGL(lsv_clear_kernel, dim3(blocks), dim3(256), 0, (hipStream_t)stream, (uint4*)d_workspace, n16);
  return hip_rc(hipGetLastError() == hipSuccess ? LSV_OK : LSV_ERR_HIP, "workspace clear");
}

namespace {
// Host checks of a cache description: a slab cache (pages NULL: capacity positions per sequence) or a
// page pool (n_pages pages of LSV_KV_PAGE positions, a page table of max_pages entries per sequence).
int check_kv(const lsv::Shape& s, const lsv::KvLayout& kvl) {
  if (!kvl.pages) {
    if (kvl.capacity < 1 || kvl.capacity % LSV_KV_ALIGN)
      return fail(LSV_ERR_INVALID_ARG, "capacity %d is not a positive multiple of %d", kvl.capacity, (int)LSV_KV_ALIGN);
    // offsets inside a sequence's blocks are 32-bit in the kernels
    if ((size_t)s.nkv * kvl.capacity * s.hd * s.es >= ((size_t)1 << 31))
      return fail(LSV_ERR_INVALID_ARG, "capacity %d: a sequence's KV block of %d x %d x %d elements reaches 2 GiB",
                  kvl.capacity, s.nkv, kvl.capacity, s.hd);
    return LSV_OK;
  }
  if (kvl.n_pages < 1 || kvl.max_pages < 1 || kvl.max_pages > (1 << 20))
    return fail(LSV_ERR_INVALID_ARG, "need n_pages >= 1 and 1 <= max_pages <= 2^20");
  // the attention reads a layer's pool through 32-bit offsets, one page past the end included
  if (((size_t)kvl.n_pages + 1) * s.nkv * LSV_KV_PAGE * s.hd * s.es >= ((size_t)1 << 31))
    return fail(LSV_ERR_INVALID_ARG, "a layer's K pool of %d pages reaches 2 GiB", kvl.n_pages);
  return LSV_OK;
}

int verify(const lsv_model_config* cfg, const void* d_packed, void* d_kv, const lsv::KvLayout& kvl, int32_t batch,
           const int32_t* d_seq_len, const int32_t* d_tokens, const int32_t* d_row_offsets, const int32_t* d_parents,
           int32_t max_rows, int32_t max_ctx, float* d_logits, int32_t* d_status, void* d_workspace,
           size_t workspace_bytes, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!d_packed || !d_kv || !d_seq_len || !d_tokens || !d_row_offsets || !d_logits || !d_workspace)
    return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if (batch < 1 || batch > LSV_MAX_BATCH) return fail(LSV_ERR_INVALID_ARG, "batch %d not in [1, %d]", batch, LSV_MAX_BATCH);
  if (max_rows < 1 || max_rows > LSV_MAX_ROWS)
    return fail(LSV_ERR_INVALID_ARG, "max_rows %d not in [1, %d]", max_rows, LSV_MAX_ROWS);
  const int capacity = kvl.pages ? kvl.max_pages * LSV_KV_PAGE : kvl.capacity;  // positions per sequence
  if (capacity < 1 || max_ctx < 1 || max_ctx > capacity)
    return fail(LSV_ERR_INVALID_ARG, "need 1 <= max_ctx (%d) <= capacity (%d)", max_ctx, capacity);
  const lsv::Shape s = lsv::shape_of(cfg);
  if ((rc = check_kv(s, kvl)) != LSV_OK) return rc;
  if (s.dtype == LSV_DTYPE_F32 && max_ctx > 16384)
    return fail(LSV_ERR_UNSUPPORTED, "fp32 models support max_ctx <= 16384");
  const size_t need = lsv::verify_workspace_bytes(s, batch, max_rows, max_ctx);
  if (workspace_bytes < need)
    return fail(LSV_ERR_INVALID_ARG, "workspace %zu bytes < %zu required", workspace_bytes, need);
  const lsv::ModelLayout ml = lsv::model_layout(s);
  rc = lsv::launch_verify(s, ml, d_packed, d_kv, kvl, batch, d_seq_len, d_tokens, d_row_offsets, d_parents,
                          max_rows, max_ctx, d_logits, d_status, d_workspace, workspace_bytes, (hipStream_t)stream);
  return hip_rc(rc, "verify");
}

lsv::KvLayout slab_kv(int capacity) { return lsv::KvLayout{capacity, nullptr, 0, 0}; }
lsv::KvLayout paged_kv(const int32_t* pages, int max_pages, int n_pages) {
  return lsv::KvLayout{max_pages * LSV_KV_PAGE, pages, max_pages, n_pages};
}
}  // namespace

int lsv_verify_block(const lsv_model_config* cfg, const void* d_packed, void* d_kv, int32_t capacity, int32_t batch,
                     const int32_t* d_seq_len, const int32_t* d_tokens, const int32_t* d_row_offsets, int32_t max_rows,
                     int32_t max_ctx, float* d_logits, int32_t* d_status, void* d_workspace, size_t workspace_bytes,
                     void* stream) {
  return verify(cfg, d_packed, d_kv, slab_kv(capacity), batch, d_seq_len, d_tokens, d_row_offsets, nullptr, max_rows,
                max_ctx, d_logits, d_status, d_workspace, workspace_bytes, stream);
}

size_t lsv_kv_pool_bytes(const lsv_model_config* cfg, int32_t n_pages) {
  if (check_config(cfg) != LSV_OK || n_pages < 1) return 0;
  const lsv::Shape s = lsv::shape_of(cfg);
  return (size_t)s.L * 2 * (size_t)n_pages * s.nkv * LSV_KV_PAGE * s.hd * s.es;
}

int lsv_verify_paged(const lsv_model_config* cfg, const void* d_packed, void* d_kv_pool, int32_t n_pages,
                     const int32_t* d_page_table, int32_t max_pages, int32_t batch, const int32_t* d_seq_len,
                     const int32_t* d_tokens, const int32_t* d_row_offsets, const int32_t* d_parents, int32_t max_rows,
                     int32_t max_ctx, float* d_logits, int32_t* d_status, void* d_workspace, size_t workspace_bytes,
                     void* stream) {
  if (!d_page_table) return fail(LSV_ERR_INVALID_ARG, "NULL page table");
  return verify(cfg, d_packed, d_kv_pool, paged_kv(d_page_table, max_pages, n_pages), batch, d_seq_len, d_tokens,
                d_row_offsets, d_parents, max_rows, max_ctx, d_logits, d_status, d_workspace, workspace_bytes, stream);
}

int lsv_verify_tree(const lsv_model_config* cfg, const void* d_packed, void* d_kv, int32_t capacity, int32_t batch,
                    const int32_t* d_seq_len, const int32_t* d_tokens, const int32_t* d_row_offsets,
                    const int32_t* d_parents, int32_t max_rows, int32_t max_ctx, float* d_logits, int32_t* d_status,
                    void* d_workspace, size_t workspace_bytes, void* stream) {
  if (!d_parents) return fail(LSV_ERR_INVALID_ARG, "NULL parents");
  return verify(cfg, d_packed, d_kv, slab_kv(capacity), batch, d_seq_len, d_tokens, d_row_offsets, d_parents, max_rows,
                max_ctx, d_logits, d_status, d_workspace, workspace_bytes, stream);
}

int lsv_accept_tree(int32_t batch, int32_t vocab, const float* d_logits, const int32_t* d_row_offsets,
                    const int32_t* d_parents, const int32_t* d_tokens, int32_t max_rows, int32_t width,
                    int32_t* d_accept_len, int32_t* d_out_tokens, int32_t* d_path, int32_t* d_seq_len,
                    int32_t* d_status, void* d_workspace, size_t workspace_bytes, void* stream) {
  if (batch < 1 || batch > LSV_MAX_BATCH || vocab < 1) return fail(LSV_ERR_INVALID_ARG, "bad batch or vocab");
  if (max_rows < 1 || max_rows > LSV_MAX_ROWS || width < 1 || width > LSV_MAX_SEQ_ROWS)
    return fail(LSV_ERR_INVALID_ARG, "bad max_rows %d (<= %d) / width %d (<= %d)", max_rows, (int)LSV_MAX_ROWS, width,
                (int)LSV_MAX_SEQ_ROWS);
  if (!d_logits || !d_row_offsets || !d_parents || !d_tokens || !d_accept_len || !d_out_tokens || !d_path ||
      !d_workspace)
    return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if (workspace_bytes < lsv::accept_workspace_bytes(batch, max_rows, vocab))
    return fail(LSV_ERR_INVALID_ARG, "accept workspace too small");
  return hip_rc(lsv::launch_accept_tree(batch, vocab, d_logits, d_row_offsets, d_parents, d_tokens, max_rows, width,
                                        d_accept_len, d_out_tokens, d_path, d_seq_len, d_status, d_workspace,
                                        (hipStream_t)stream),
                "accept_tree");
}

namespace {
int commit_tree(const lsv_model_config* cfg, void* d_kv, const lsv::KvLayout& kvl, int32_t batch,
                const int32_t* d_seq_len, const int32_t* d_accept_len, const int32_t* d_path, int32_t width,
                const int32_t* d_status, void* stream) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (!d_kv || !d_seq_len || !d_accept_len || !d_path) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if (batch < 1 || batch > LSV_MAX_BATCH) return fail(LSV_ERR_INVALID_ARG, "batch %d not in [1, %d]", batch, LSV_MAX_BATCH);
  if (width < 1 || width > LSV_MAX_SEQ_ROWS)
    return fail(LSV_ERR_INVALID_ARG, "width %d not in [1, %d]", width, (int)LSV_MAX_SEQ_ROWS);
  const lsv::Shape s = lsv::shape_of(cfg);
  if ((rc = check_kv(s, kvl)) != LSV_OK) return rc;
  return hip_rc(lsv::launch_commit_tree(s, d_kv, kvl, batch, d_seq_len, d_accept_len, d_path, width, d_status,
                                        (hipStream_t)stream),
                "commit_tree");
}
}  // namespace

int lsv_commit_tree(const lsv_model_config* cfg, void* d_kv, int32_t capacity, int32_t batch, const int32_t* d_seq_len,
                    const int32_t* d_accept_len, const int32_t* d_path, int32_t width, const int32_t* d_status,
                    void* stream) {
  return commit_tree(cfg, d_kv, slab_kv(capacity), batch, d_seq_len, d_accept_len, d_path, width, d_status, stream);
}

int lsv_commit_tree_paged(const lsv_model_config* cfg, void* d_kv_pool, int32_t n_pages, const int32_t* d_page_table,
                          int32_t max_pages, int32_t batch, const int32_t* d_seq_len, const int32_t* d_accept_len,
                          const int32_t* d_path, int32_t width, const int32_t* d_status, void* stream) {
  if (!d_page_table) return fail(LSV_ERR_INVALID_ARG, "NULL page table");
  return commit_tree(cfg, d_kv_pool, paged_kv(d_page_table, max_pages, n_pages), batch, d_seq_len, d_accept_len, d_path,
                     width, d_status, stream);
}

// ---------------------------------------------------------------- attention layer on the paged cache
namespace {
int check_rope(const lsv_rope* r, int head_dim) {
  if ((r->layout != LSV_ROPE_HALF && r->layout != LSV_ROPE_INTERLEAVED) || r->rot_dim < 2 || r->rot_dim % 2 ||
      r->rot_dim > LSV_ROPE_MAX_DIM || r->rot_dim > head_dim || !isfinite(r->amplitude) || r->reserved0 != 0.f)
    return fail(LSV_ERR_INVALID_ARG, "bad rope: layout %d, rot_dim %d (even, 2..%d, <= head_dim %d), amplitude %g",
                r->layout, r->rot_dim, (int)LSV_ROPE_MAX_DIM, head_dim, (double)r->amplitude);
  for (int j = 0; j < r->rot_dim / 2; ++j)
    if (!isfinite(r->freq[j] * 0x1p31))  // the angle of the last position
      return fail(LSV_ERR_INVALID_ARG, "rope: freq[%d] is not finite, or its angles are not", j);
  return LSV_OK;
}

lsv::RopeArgs rope_args(const lsv_rope* r) {
  lsv::RopeArgs a;
  a.layout = r ? r->layout : LSV_ROPE_HALF;
  a.rot = r ? r->rot_dim : 0;
  a.amplitude = r ? r->amplitude : 1.f;
  for (int j = 0; j < a.rot / 2; ++j) a.half_turns[j] = r->freq[j] * M_1_PI;  // those behind are not read
  return a;
}

// Host checks that the append and the attention share.
int check_paged_layer(const lsv_model_config* cfg, int32_t layer, const void* d_kv_pool, int32_t n_pages,
                      const int32_t* d_page_table, int32_t max_pages, int32_t batch, const int32_t* d_seq_len,
                      const int32_t* d_row_offsets, int32_t max_rows, int32_t max_ctx) {
  int rc = check_config(cfg);
  if (rc) return rc;
  if (layer < 0 || layer >= cfg->n_layers) return fail(LSV_ERR_INVALID_ARG, "layer %d out of range", layer);
  if (cfg->n_kv_heads > 65535) return fail(LSV_ERR_UNSUPPORTED, "n_kv_heads %d > 65535", cfg->n_kv_heads);
  if (!d_kv_pool || !d_page_table || !d_seq_len || !d_row_offsets) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if ((uintptr_t)d_kv_pool & 15) return fail(LSV_ERR_INVALID_ARG, "the pool must be 16-byte aligned");
  if (n_pages < 1 || max_pages < 1 || max_pages > (1 << 20))
    return fail(LSV_ERR_INVALID_ARG, "need n_pages >= 1 and 1 <= max_pages <= 2^20");
  if (batch < 1 || batch > LSV_MAX_BATCH) return fail(LSV_ERR_INVALID_ARG, "batch %d not in [1, %d]", batch, LSV_MAX_BATCH);
  if (max_rows < 1 || max_rows > LSV_MAX_CHUNK_ROWS)
    return fail(LSV_ERR_INVALID_ARG, "max_rows %d not in [1, %d]", max_rows, LSV_MAX_CHUNK_ROWS);
  if (max_ctx < 1 || max_ctx > max_pages * LSV_KV_PAGE)
    return fail(LSV_ERR_INVALID_ARG, "need 1 <= max_ctx (%d) <= max_pages * %d (%d)", max_ctx, (int)LSV_KV_PAGE,
                max_pages * LSV_KV_PAGE);
  return LSV_OK;
}

int check_rows(const char* what, const void* p, int es, int64_t stride, int64_t width) {
  if (!p || (uintptr_t)p % es) return fail(LSV_ERR_INVALID_ARG, "%s: NULL or misaligned pointer", what);
  if (stride < width)
    return fail(LSV_ERR_INVALID_ARG, "%s: stride %lld < %lld elements of a row", what, (long long)stride, (long long)width);
  return LSV_OK;
}
}  // namespace

int lsv_rope_init(lsv_rope* rope, int32_t layout, int32_t rot_dim, double base, int32_t scaling, double factor,
                  double low, double high, int32_t original_ctx, double amplitude) {
  if (!rope) return fail(LSV_ERR_INVALID_ARG, "rope is NULL");
  if (layout != LSV_ROPE_HALF && layout != LSV_ROPE_INTERLEAVED) return fail(LSV_ERR_INVALID_ARG, "bad layout %d", layout);
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > LSV_ROPE_MAX_DIM)
    return fail(LSV_ERR_INVALID_ARG, "rot_dim %d is not even in [2, %d]", rot_dim, (int)LSV_ROPE_MAX_DIM);
  if (scaling < LSV_ROPE_PLAIN || scaling > LSV_ROPE_RAMP) return fail(LSV_ERR_INVALID_ARG, "bad scaling %d", scaling);
  if (!(base > 0.0) || !isfinite(base) || !((float)amplitude > 0.f) || !isfinite((float)amplitude))
    return fail(LSV_ERR_INVALID_ARG, "base and amplitude must be finite and positive");
  if (scaling != LSV_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor)))
    return fail(LSV_ERR_INVALID_ARG, "factor must be finite and positive");
  if (scaling == LSV_ROPE_NTK && rot_dim < 4) return fail(LSV_ERR_INVALID_ARG, "LSV_ROPE_NTK needs rot_dim > 2");
  if (scaling == LSV_ROPE_RAMP && !(base > 1.0)) return fail(LSV_ERR_INVALID_ARG, "LSV_ROPE_RAMP needs base > 1");
  const bool blend = scaling == LSV_ROPE_BANDS || scaling == LSV_ROPE_RAMP;
  if (blend && (original_ctx < 1 || !(low > 0.0) || !(high > low) || !isfinite(high)))
    return fail(LSV_ERR_INVALID_ARG, "need original_ctx >= 1 and 0 < low < high");
  lsv_rope r = {layout, rot_dim, (float)amplitude, 0.f, {}};
  if (scaling == LSV_ROPE_NTK) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  auto index_of = [&](double turns) { return rot_dim * log(original_ctx / (2.0 * M_PI * turns)) / (2.0 * log(base)); };
  double first = 0.0, width = 1.0;
  if (scaling == LSV_ROPE_RAMP) {
    first = fmax(floor(index_of(high)), 0.0);
    width = fmax(fmin(ceil(index_of(low)), rot_dim - 1.0) - first, 1e-3);
  }
  for (int j = 0; j < LSV_ROPE_MAX_DIM / 2; ++j) {
    double f = j < rot_dim / 2 ? pow(base, -2.0 * j / rot_dim) : 0.0;
    if (scaling == LSV_ROPE_LINEAR) f /= factor;
    if (blend) {
      const double at = scaling == LSV_ROPE_BANDS ? (original_ctx * f / (2.0 * M_PI) - low) / (high - low)
                                                  : 1.0 - (j - first) / width;
      const double keep = fmin(fmax(at, 0.0), 1.0);
      f = keep * f + (1.0 - keep) * f / factor;
    }
    r.freq[j] = f;
  }
  if (!isfinite(base)) return fail(LSV_ERR_INVALID_ARG, "the stretched base is not finite");
  const int rc = check_rope(&r, LSV_ROPE_MAX_DIM);
  if (rc) return rc;
  *rope = r;
  return ok();
}

int lsv_apply_rope(const lsv_rope* rope, int32_t dtype, int32_t n_heads, int32_t head_dim, int32_t batch,
                   const int32_t* d_seq_len, const int32_t* d_row_offsets, const int32_t* d_positions,
                   int32_t max_rows, const void* d_x, int64_t x_stride, void* d_y, int64_t y_stride, void* stream) {
  if (!rope) return fail(LSV_ERR_INVALID_ARG, "rope is NULL");
  if (dtype != LSV_DTYPE_F32 && dtype != LSV_DTYPE_BF16) return fail(LSV_ERR_INVALID_ARG, "bad dtype");
  if (n_heads < 1 || n_heads > 65535 || head_dim < 8 || head_dim % 8 || head_dim > LSV_ROPE_MAX_DIM)
    return fail(LSV_ERR_INVALID_ARG, "bad n_heads %d or head_dim %d (a multiple of 8 up to %d)", n_heads, head_dim,
                (int)LSV_ROPE_MAX_DIM);
  int rc = check_rope(rope, head_dim);
  if (rc) return rc;
  if (max_rows < 1 || max_rows > LSV_MAX_CHUNK_ROWS)
    return fail(LSV_ERR_INVALID_ARG, "max_rows %d not in [1, %d]", max_rows, LSV_MAX_CHUNK_ROWS);
  if (!d_positions && (!d_seq_len || !d_row_offsets))
    return fail(LSV_ERR_INVALID_ARG, "need positions, or sequence lengths and row offsets");
  if ((d_row_offsets || !d_positions) && (batch < 1 || batch > LSV_MAX_BATCH))
    return fail(LSV_ERR_INVALID_ARG, "batch %d not in [1, %d]", batch, LSV_MAX_BATCH);
  const int64_t width = (int64_t)n_heads * head_dim;
  const int es = dtype == LSV_DTYPE_BF16 ? 2 : 4;
  if ((rc = check_rows("x", d_x, es, x_stride, width)) || (rc = check_rows("y", d_y, es, y_stride, width))) return rc;
  if (d_x == d_y && x_stride != y_stride) return fail(LSV_ERR_INVALID_ARG, "in place needs equal strides");
  const lsv::RowArgs rows{d_seq_len, d_row_offsets, d_positions, batch, max_rows, max_rows, INT32_MAX};
  return hip_rc(lsv::launch_rope(rope_args(rope), dtype, n_heads, head_dim, rows, d_x, x_stride, d_y, y_stride,
                                 (hipStream_t)stream),
                "apply_rope");
}

int lsv_append_paged(const lsv_model_config* cfg, int32_t layer, void* d_kv_pool, int32_t n_pages,
                     const int32_t* d_page_table, int32_t max_pages, int32_t batch, const int32_t* d_seq_len,
                     const int32_t* d_row_offsets, const int32_t* d_positions, int32_t max_rows, int32_t max_ctx,
                     const lsv_rope* rope, const void* d_q, int64_t q_stride, void* d_q_out, int64_t q_out_stride,
                     const void* d_k, int64_t k_stride, const void* d_v, int64_t v_stride, int32_t* d_status,
                     void* stream) {
  int rc = check_paged_layer(cfg, layer, d_kv_pool, n_pages, d_page_table, max_pages, batch, d_seq_len, d_row_offsets,
                             max_rows, max_ctx);
  if (rc) return rc;
  const lsv::Shape s = lsv::shape_of(cfg);
  if (rope && (rc = check_rope(rope, s.hd))) return rc;
  if (!d_q != !d_q_out) return fail(LSV_ERR_INVALID_ARG, "d_q and d_q_out go together");
  if (d_q && ((rc = check_rows("q", d_q, s.es, q_stride, (int64_t)s.nq * s.hd)) ||
              (rc = check_rows("q_out", d_q_out, s.es, q_out_stride, (int64_t)s.nq * s.hd))))
    return rc;
  if (d_q && d_q == d_q_out && q_stride != q_out_stride)
    return fail(LSV_ERR_INVALID_ARG, "in place needs equal strides");
  if ((rc = check_rows("k", d_k, s.es, k_stride, (int64_t)s.nkv * s.hd)) ||
      (rc = check_rows("v", d_v, s.es, v_stride, (int64_t)s.nkv * s.hd)))
    return rc;
  lsv::AppendArgs a;
  a.rows = lsv::RowArgs{d_seq_len, d_row_offsets, d_positions, batch, max_rows, max_rows, max_ctx};
  a.kv = paged_kv(d_page_table, max_pages, n_pages);
  const size_t blk = lsv::kv_layer_block(a.kv, batch, s.nkv, s.hd) * s.es;
  a.k_pool = (char*)d_kv_pool + 2 * (size_t)layer * blk;
  a.v_pool = (char*)a.k_pool + blk;
  a.nq = d_q ? s.nq : 0;
  a.nkv = s.nkv;
  a.hd = s.hd;
  a.q = d_q, a.k = d_k, a.v = d_v, a.q_out = d_q_out;
  a.qs = q_stride, a.qos = q_out_stride, a.ks = k_stride, a.vs = v_stride;
  a.status = d_status;
  return hip_rc(lsv::launch_append(rope_args(rope), s.dtype, a, (hipStream_t)stream), "append_paged");
}

size_t lsv_attend_workspace_bytes(const lsv_model_config* cfg, int32_t batch, int32_t max_rows,
                                  int32_t max_rows_per_seq, int32_t max_ctx) {
  if (check_config(cfg) != LSV_OK || batch < 1 || batch > LSV_MAX_BATCH || max_rows < 1 ||
      max_rows > LSV_MAX_CHUNK_ROWS || max_rows_per_seq < 1 || max_rows_per_seq > max_rows || max_ctx < 1 ||
      max_ctx > (1 << 20) * LSV_KV_PAGE || cfg->n_kv_heads > 65535)
    return 0;
  if (!lsv::attend_fits(lsv::shape_of(cfg), batch, max_rows, max_rows_per_seq, max_ctx)) return 0;
  return lsv::attend_workspace_bytes(lsv::shape_of(cfg), batch, max_rows, max_rows_per_seq, max_ctx);
}

int lsv_attend_paged(const lsv_model_config* cfg, int32_t layer, const void* d_kv_pool, int32_t n_pages,
                     const int32_t* d_page_table, int32_t max_pages, int32_t batch, const int32_t* d_seq_len,
                     const int32_t* d_row_offsets, int32_t max_rows, int32_t max_rows_per_seq, int32_t max_ctx,
                     const lsv_attend_options* options, const void* d_q, int64_t q_stride, void* d_out,
                     int64_t out_stride, float* d_lse, int32_t* d_status, void* d_workspace, size_t workspace_bytes,
                     void* stream) {
  int rc = check_paged_layer(cfg, layer, d_kv_pool, n_pages, d_page_table, max_pages, batch, d_seq_len, d_row_offsets,
                             max_rows, max_ctx);
  if (rc) return rc;
  if (max_rows_per_seq < 1 || max_rows_per_seq > max_rows)
    return fail(LSV_ERR_INVALID_ARG, "max_rows_per_seq %d not in [1, max_rows %d]", max_rows_per_seq, max_rows);
  const lsv::Shape s = lsv::shape_of(cfg);
  if (!lsv::attend_fits(s, batch, max_rows, max_rows_per_seq, max_ctx))
    return fail(LSV_ERR_UNSUPPORTED, "max_rows %d and max_ctx %d: the pages of all query tiles, or the query vectors, reach 2^30; split the block",
                max_rows, max_ctx);
  const lsv_attend_options plain = {};
  const lsv_attend_options& o = options ? *options : plain;
  const bool cap_ok = o.softcap == 0.f || (o.softcap >= 1e-15f && o.softcap <= 1e15f);  // finite in log2 units too
  if (!(fabsf(o.scale) <= 1e15f) || !cap_ok || o.window < 0 || o.reserved0 != 0)
    return fail(LSV_ERR_INVALID_ARG, "bad attention options (scale %g, softcap %g, window %d)", (double)o.scale,
                (double)o.softcap, o.window);
  const int64_t width = (int64_t)s.nq * s.hd;
  if ((rc = check_rows("q", d_q, s.es, q_stride, width)) || (rc = check_rows("out", d_out, s.es, out_stride, width))) return rc;
  if ((((uintptr_t)d_q | (uintptr_t)d_out) & 15) || (q_stride * s.es) % 16 || (out_stride * s.es) % 16)
    return fail(LSV_ERR_INVALID_ARG, "q and out must be 16-byte aligned with strides of whole 16-byte pieces");
  if (d_q == d_out && q_stride != out_stride) return fail(LSV_ERR_INVALID_ARG, "in place needs equal strides");
  const size_t need = lsv::attend_workspace_bytes(s, batch, max_rows, max_rows_per_seq, max_ctx);
  if (!d_workspace || ((uintptr_t)d_workspace & 15) || workspace_bytes < need)
    return fail(LSV_ERR_INVALID_ARG, "attend workspace: %zu bytes at a 16-byte boundary required, got %zu", need,
                workspace_bytes);
  lsv::AttendArgs a;
  a.rows = lsv::RowArgs{d_seq_len, d_row_offsets, nullptr, batch, max_rows, max_rows_per_seq, max_ctx};
  a.kv = paged_kv(d_page_table, max_pages, n_pages);
  const size_t blk = lsv::kv_layer_block(a.kv, batch, s.nkv, s.hd) * s.es;
  a.k_pool = (const char*)d_kv_pool + 2 * (size_t)layer * blk;
  a.v_pool = (const char*)a.k_pool + blk;
  a.nq = s.nq;
  a.nkv = s.nkv;
  a.hd = s.hd;
  a.q = d_q, a.out = d_out, a.qs = q_stride, a.os = out_stride;
  a.lse = d_lse;
  a.status = d_status;
  a.scale = o.scale != 0.f ? o.scale : 1.f / sqrtf((float)s.hd);
  a.softcap = o.softcap;
  a.window = o.window < max_ctx ? o.window : 0;  // a window of every position hides none
  a.slopes = o.d_slopes;
  a.key_start = o.d_key_start;
  a.prefix_len = o.d_prefix_len;
  return hip_rc(lsv::launch_attend(s.dtype, a, d_workspace, (hipStream_t)stream), "attend_paged");
}

size_t lsv_accept_workspace_bytes(int32_t batch, int32_t max_rows, int32_t vocab) {
  if (batch < 1 || max_rows < 1 || vocab < 1) return 0;
  return lsv::accept_workspace_bytes(batch, max_rows, vocab);
}

int lsv_accept(int32_t mode, int32_t batch, int32_t vocab, const float* d_logits, const int32_t* d_row_offsets,
               int32_t max_rows, int32_t max_rows_per_seq, const int32_t* d_tokens, const float* d_draft_probs,
               float temperature, uint64_t seed, uint64_t round, int32_t* d_accept_len, int32_t* d_out_tokens,
               int32_t* d_seq_len, int32_t* d_status, void* d_workspace, size_t workspace_bytes, void* stream) {
  if (mode != LSV_ACC_GREEDY && mode != LSV_ACC_SAMPLE) return fail(LSV_ERR_INVALID_ARG, "bad accept mode %d", mode);
  if (batch < 1 || batch > LSV_MAX_BATCH || vocab < 1) return fail(LSV_ERR_INVALID_ARG, "bad batch or vocab");
  if (max_rows < 1 || max_rows > LSV_MAX_ROWS || max_rows_per_seq < 1 || max_rows_per_seq > LSV_MAX_SEQ_ROWS)
    return fail(LSV_ERR_INVALID_ARG, "bad max_rows %d (<= %d) / max_rows_per_seq %d (<= %d)", max_rows,
                (int)LSV_MAX_ROWS, max_rows_per_seq, (int)LSV_MAX_SEQ_ROWS);
  if (!d_logits || !d_row_offsets || !d_tokens || !d_accept_len || !d_out_tokens || !d_workspace)
    return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if (mode == LSV_ACC_SAMPLE && (!d_draft_probs || !(temperature > 0.f) || !isfinite(temperature)))
    return fail(LSV_ERR_INVALID_ARG, "sampling needs draft probabilities and a finite temperature > 0");
  if (workspace_bytes < lsv::accept_workspace_bytes(batch, max_rows, vocab))
    return fail(LSV_ERR_INVALID_ARG, "accept workspace too small");
  int rc = lsv::launch_accept(mode, batch, vocab, d_logits, d_row_offsets, max_rows, max_rows_per_seq, d_tokens,
                              d_draft_probs, temperature, seed, round, d_accept_len, d_out_tokens, d_seq_len, d_status,
                              d_workspace, (hipStream_t)stream);
  return hip_rc(rc, "accept");
}

int lsv_accept_noalloc(int32_t mode, int32_t batch, int32_t vocab, const float* d_logits,
                       const int32_t* d_row_offsets, int32_t max_rows, int32_t max_rows_per_seq,
                       const int32_t* d_tokens, const float* d_draft_probs, float temperature, uint64_t seed,
                       uint64_t round, int32_t* d_accept_len, int32_t* d_out_tokens, int32_t* d_seq_len,
                       int32_t* d_status, void* stream) {
  if (mode != LSV_ACC_GREEDY && mode != LSV_ACC_SAMPLE) return fail(LSV_ERR_INVALID_ARG, "bad accept mode %d", mode);
  if (batch < 1 || batch > LSV_MAX_BATCH || vocab < 1) return fail(LSV_ERR_INVALID_ARG, "bad batch or vocab");
  if (max_rows < 1 || max_rows > LSV_MAX_ROWS || max_rows_per_seq < 1 || max_rows_per_seq > LSV_MAX_SEQ_ROWS)
    return fail(LSV_ERR_INVALID_ARG, "bad max_rows %d (<= %d) / max_rows_per_seq %d (<= %d)", max_rows,
                (int)LSV_MAX_ROWS, max_rows_per_seq, (int)LSV_MAX_SEQ_ROWS);
  if (!d_logits || !d_row_offsets || !d_tokens || !d_accept_len || !d_out_tokens)
    return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if (mode == LSV_ACC_SAMPLE && (!d_draft_probs || !(temperature > 0.f) || !isfinite(temperature)))
    return fail(LSV_ERR_INVALID_ARG, "sampling needs draft probabilities and a finite temperature > 0");
  const size_t need = lsv::accept_workspace_bytes(batch, max_rows, vocab);
  if (need > lsv::kAcceptStaticBytes)
    return fail(LSV_ERR_UNSUPPORTED, "scratch of %zu bytes needed, the library's holds %zu (LSV_ACCEPT_NOALLOC_BYTES)",
                need, lsv::kAcceptStaticBytes);
  void* ws = nullptr;
  int rc = lsv::accept_scratch(&ws);
  if (rc != LSV_OK) return hip_rc(rc, "accept_noalloc scratch");
  rc = lsv::launch_accept(mode, batch, vocab, d_logits, d_row_offsets, max_rows, max_rows_per_seq, d_tokens,
                          d_draft_probs, temperature, seed, round, d_accept_len, d_out_tokens, d_seq_len, d_status, ws,
                          (hipStream_t)stream);
  return hip_rc(rc, "accept_noalloc");
}

int lsv_select_length(int32_t mode, int32_t batch, int32_t G, const float* d_conf, const double* d_cost, int32_t d_init,
                      int32_t d_max, double alpha, int32_t block_n, uint32_t flags, int32_t* d_gamma, int32_t* d_aux,
                      int32_t* d_row_offsets, int32_t* d_status, void* stream) {
  if (mode != LSV_SEL_MARGINAL && mode != LSV_SEL_EXHAUSTIVE && mode != LSV_SEL_ALG1)
    return fail(LSV_ERR_INVALID_ARG, "bad selector mode %d", mode);
  if (batch < 1 || G < 1 || G > LSV_MAX_G) return fail(LSV_ERR_INVALID_ARG, "need batch >= 1 and 1 <= G <= %d", LSV_MAX_G);
  if (d_max < 1 || d_max > G) return fail(LSV_ERR_INVALID_ARG, "need 1 <= d_max (%d) <= G (%d)", d_max, G);
  if (!d_conf || !d_gamma) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if (flags & ~(uint32_t)(LSV_SEL_BONUS | LSV_SEL_DRAFTED)) return fail(LSV_ERR_INVALID_ARG, "unknown flags");
  if ((flags & LSV_SEL_DRAFTED) && (mode != LSV_SEL_ALG1 || !d_aux))
    return fail(LSV_ERR_INVALID_ARG, "LSV_SEL_DRAFTED needs LSV_SEL_ALG1 and d_aux (blocks drafted)");
  if (d_row_offsets && batch > LSV_MAX_BATCH)
    return fail(LSV_ERR_INVALID_ARG, "row offsets need batch <= %d", LSV_MAX_BATCH);
  if (mode == LSV_SEL_ALG1) {
    if (block_n < 1) return fail(LSV_ERR_INVALID_ARG, "block_n must be >= 1");
    if (!(alpha > 0.0) || !(alpha <= 1.0e6)) return fail(LSV_ERR_INVALID_ARG, "alpha must be in (0, 1e6]");
  } else {
    if (!d_cost) return fail(LSV_ERR_INVALID_ARG, "cost table required");
    if (mode == LSV_SEL_MARGINAL && d_init < 1) return fail(LSV_ERR_INVALID_ARG, "d_init must be >= 1");
  }
  int rc = lsv::launch_select(mode, batch, G, d_conf, d_cost, d_init, d_max, alpha, block_n, flags, d_gamma, d_aux,
                              d_row_offsets, d_status, (hipStream_t)stream);
  return hip_rc(rc, "select");
}

int lsv_select_joint(int32_t batch, int32_t G, const float* d_conf, const double* d_cost, int32_t d_max, uint32_t flags,
                     int32_t* d_gamma, int32_t* d_total, int32_t* d_row_offsets, int32_t* d_status, void* stream) {
  if (batch < 1 || batch > LSV_MAX_BATCH) return fail(LSV_ERR_INVALID_ARG, "need 1 <= batch <= %d", LSV_MAX_BATCH);
  if (G < 1 || G > LSV_MAX_G) return fail(LSV_ERR_INVALID_ARG, "need 1 <= G <= %d", LSV_MAX_G);
  if (d_max < 1 || d_max > G) return fail(LSV_ERR_INVALID_ARG, "need 1 <= d_max (%d) <= G (%d)", d_max, G);
  if (flags & ~(uint32_t)LSV_SEL_BONUS) return fail(LSV_ERR_INVALID_ARG, "unknown flags");
  if (!d_conf || !d_cost || !d_gamma) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  return hip_rc(lsv::launch_select_joint(batch, G, d_conf, d_cost, d_max, flags, d_gamma, d_total, d_row_offsets,
                                         d_status, (hipStream_t)stream),
                "select_joint");
}

int lsv_next_length_g4(int32_t batch, const int32_t* d_gamma, const int32_t* d_accept_len, const int32_t* d_status,
                       int32_t d_min, int32_t d_max, int32_t* d_gamma_next, int32_t* d_row_offsets, int32_t* d_err,
                       void* stream) {
  if (batch < 1) return fail(LSV_ERR_INVALID_ARG, "need batch >= 1");
  if (d_min < 1 || d_min > d_max || d_max > LSV_MAX_SEQ_ROWS - 1)
    return fail(LSV_ERR_INVALID_ARG, "need 1 <= d_min (%d) <= d_max (%d) <= %d", d_min, d_max, LSV_MAX_SEQ_ROWS - 1);
  if (!d_gamma || !d_accept_len || !d_gamma_next) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  if (d_row_offsets && batch > LSV_MAX_BATCH)
    return fail(LSV_ERR_INVALID_ARG, "row offsets need batch <= %d", LSV_MAX_BATCH);
  int rc = lsv::launch_next_length_g4(batch, d_gamma, d_accept_len, d_status, d_min, d_max, d_gamma_next,
                                      d_row_offsets, d_err, (hipStream_t)stream);
  return hip_rc(rc, "next_length_g4");
}

int lsv_pack_block(int32_t batch, int32_t G, const int32_t* d_row_offsets, int32_t max_rows, const int32_t* d_roots,
                   const int32_t* d_drafts, int32_t* d_tokens, int32_t* d_status, void* stream) {
  if (batch < 1 || batch > LSV_MAX_BATCH) return fail(LSV_ERR_INVALID_ARG, "need 1 <= batch <= %d", LSV_MAX_BATCH);
  if (G < 0 || G > LSV_MAX_SEQ_ROWS - 1) return fail(LSV_ERR_INVALID_ARG, "need 0 <= G <= %d", LSV_MAX_SEQ_ROWS - 1);
  if (max_rows < 1 || max_rows > LSV_MAX_ROWS) return fail(LSV_ERR_INVALID_ARG, "need 1 <= max_rows <= %d", LSV_MAX_ROWS);
  if (!d_row_offsets || !d_roots || !d_tokens || (G > 0 && !d_drafts)) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  return hip_rc(lsv::launch_pack_block(batch, G, d_row_offsets, max_rows, d_roots, d_drafts, d_tokens, d_status,
                                       (hipStream_t)stream),
                "pack_block");
}

int lsv_next_roots(int32_t batch, const int32_t* d_accept_len, const int32_t* d_out_tokens, int32_t width,
                   const int32_t* d_status, int32_t* d_roots, void* stream) {
  if (batch < 1) return fail(LSV_ERR_INVALID_ARG, "need batch >= 1");
  if (width < 1 || width > LSV_MAX_SEQ_ROWS) return fail(LSV_ERR_INVALID_ARG, "need 1 <= width <= %d", LSV_MAX_SEQ_ROWS);
  if (!d_accept_len || !d_out_tokens || !d_roots) return fail(LSV_ERR_INVALID_ARG, "NULL pointer");
  return hip_rc(lsv::launch_next_roots(batch, d_accept_len, d_out_tokens, width, d_status, d_roots, (hipStream_t)stream),
                "next_roots");
}

int lsv_set_timing_events(int32_t kernel, void* const* events, int32_t n_slots, uint32_t record_flags) {
  if (kernel < LSV_KERNEL_QKV || kernel > LSV_KERNEL_ATTENTION) return fail(LSV_ERR_INVALID_ARG, "bad kernel class");
  if (n_slots < 0 || n_slots > LSV_MAX_TIMING_SLOTS || (n_slots > 0 && !events))
    return fail(LSV_ERR_INVALID_ARG, "n_slots must be in [0, %d] with a non-NULL event array", LSV_MAX_TIMING_SLOTS);
  g_timing.kernel = kernel;
  g_timing.n = n_slots;
  g_timing.flags = record_flags;
  for (int i = 0; i < 2 * n_slots; ++i) g_timing.ev[i] = (hipEvent_t)events[i];
  return ok();
}

}  // extern "C"

namespace lsv {
// Events are recorded with the caller's flags (hipEventRecordExternal while capturing
// a graph).  Failures are reported through the sticky error that the surrounding
// launch checks.
static void timing_record(hipEvent_t ev, hipStream_t st) {
  const hipError_t e = hipEventRecordWithFlags(ev, st, g_timing.flags);
  if (e != hipSuccess) fail(LSV_ERR_HIP, "timing event record (flags %u): %s", g_timing.flags, hipGetErrorString(e));
}
void timing_before(int kernel, int index, hipStream_t st) {
  if (g_timing.n > 0 && kernel == g_timing.kernel && index < g_timing.n) timing_record(g_timing.ev[2 * index], st);
}
void timing_after(int kernel, int index, hipStream_t st) {
  if (g_timing.n > 0 && kernel == g_timing.kernel && index < g_timing.n) timing_record(g_timing.ev[2 * index + 1], st);
}
}  // namespace lsv
