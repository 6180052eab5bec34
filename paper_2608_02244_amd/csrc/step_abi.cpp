// C ABI of the operators of a step: argument checks and workspaces.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>

#include "abi_internal.hpp"
#include "fsched.h"
#include "step_common.hpp"

namespace {

bool pow2(int32_t x) { return x > 0 && (x & (x - 1)) == 0; }

int shift_of(int32_t x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool stride_ok(int64_t s) { return s >= 0 && (s & 7) == 0; }

constexpr int32_t kMaxPage = 65536, kMaxHeads = 1024;
constexpr int64_t kMaxStride = (int64_t)1 << 40, kMaxInPage = (int64_t)1 << 27;

int check_flags(uint32_t flags) {
  if (!(flags & FSCHED_F_DEVICE_PTRS)) return FSCHED_EINVAL;
  if (flags & ~(uint32_t)(FSCHED_F_DEVICE_PTRS | FSCHED_F_SYNC)) return FSCHED_EINVAL;
  return FSCHED_OK;
}

// Shape and strides of a cache (its pointers are checked by the callers, which
// know whether they are used).
int check_cache(const fsched_kv_cache* c) {
  if (!c || c->reserved != 0) return FSCHED_EINVAL;
  if (c->n_pages < 0 || !pow2(c->page_size) || c->kv_heads < 1) return FSCHED_EINVAL;
  if (c->dtype != FSCHED_BF16 && c->dtype != FSCHED_F16) return FSCHED_EINVAL;
  if (c->head_dim < 1) return FSCHED_EINVAL;
  for (int i = 0; i < 3; ++i)
    if (!stride_ok(c->k_stride[i]) || !stride_ok(c->v_stride[i])) return FSCHED_EINVAL;
  if (!aligned16(c->k) || !aligned16(c->v)) return FSCHED_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return FSCHED_ENOTIMPL;
  if (c->page_size > kMaxPage || c->kv_heads > kMaxHeads) return FSCHED_ETOOLARGE;
  // kernels take byte offsets within a page in 32 bits
  for (int i = 0; i < 3; ++i)
    if (c->k_stride[i] > kMaxStride || c->v_stride[i] > kMaxStride) return FSCHED_ETOOLARGE;
  if (c->k_stride[2] * c->page_size > kMaxInPage || c->v_stride[2] * c->page_size > kMaxInPage)
    return FSCHED_ETOOLARGE;
  return FSCHED_OK;
}

fs::CacheRef cache_ref(const fsched_kv_cache* c) {
  fs::CacheRef r;
  r.k = c->k;
  r.v = c->v;
  r.k_page = c->k_stride[0];
  r.k_head = c->k_stride[1];
  r.k_slot = c->k_stride[2];
  r.v_page = c->v_stride[0];
  r.v_head = c->v_stride[1];
  r.v_slot = c->v_stride[2];
  r.n_pages = c->n_pages;
  r.page_shift = shift_of(c->page_size);
  r.kv_heads = c->kv_heads;
  return r;
}

int finish(hipError_t e, uint32_t flags, hipStream_t s) {
  if (e == hipSuccess && (flags & FSCHED_F_SYNC)) e = hipStreamSynchronize(s);
  return e == hipSuccess ? FSCHED_OK : fs::record_hip_error(e);
}

int check_attn(const fsched_attn_params* p, const fsched_kv_cache* kv) {
  if (!p) return FSCHED_EINVAL;
  int rc = check_flags(p->flags);
  if (rc) return rc;
  rc = check_cache(kv);
  if (rc) return rc;
  if (p->n_req < 0 || p->n_tok < 0 || p->q_heads < 1 || p->q_heads % kv->kv_heads != 0 ||
      p->table_width < 0 || p->window < 0 || p->n_sink < 0 || p->prefix_len < 0)
    return FSCHED_EINVAL;
  if (p->max_q < 1 || (p->n_tok > 0 && p->max_q > p->n_tok)) return FSCHED_EINVAL;
  if (!(p->scale > 0.0f) || !std::isfinite(p->scale)) return FSCHED_EINVAL;
  if (!stride_ok(p->q_token_stride) || !stride_ok(p->q_head_stride) ||
      !stride_ok(p->out_token_stride) || !stride_ok(p->out_head_stride))
    return FSCHED_EINVAL;
  if (p->q_heads > kMaxHeads || p->n_req > FSCHED_MAX_REQ || p->n_tok > FSCHED_MAX_STEP_TOKENS)
    return FSCHED_ETOOLARGE;
  // positions are 32-bit, and a window's ends are computed around them
  if ((int64_t)p->table_width * kv->page_size + p->prefix_len > (1 << 30)) return FSCHED_ETOOLARGE;
  return FSCHED_OK;
}

fs::AttnArgs attn_args(const fsched_attn_params* p, const fsched_kv_cache* kv) {
  fs::AttnArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_req = p->n_req;
  a.n_tok = p->n_tok;
  a.q_heads = p->q_heads;
  a.group = p->q_heads / kv->kv_heads;
  a.max_q = p->max_q;
  a.width = p->table_width;
  // a window of 2^30 or more hides nothing (positions end below)
  a.window = p->window >= (1 << 30) ? 0 : p->window;
  a.n_sink = p->n_sink > (1 << 30) ? (1 << 30) : p->n_sink;
  a.prefix_len = p->prefix_len;
  a.scale_log2 = (float)((double)p->scale * 1.4426950408889634);
  a.q_token = p->q_token_stride;
  a.q_head = p->q_head_stride;
  a.o_token = p->out_token_stride;
  a.o_head = p->out_head_stride;
  a.kv = cache_ref(kv);
  return a;
}

int attend_entry(const fsched_attn_params* p, const fsched_kv_cache* kv, const void* q,
                 const int32_t* prefix_pages, const int32_t* table, const int32_t* q_start,
                 const int32_t* kv_len, void* out, float* lse, void* workspace,
                 int64_t workspace_bytes, void* stream) {
  int rc = check_attn(p, kv);
  if (rc) return rc;
  if (p->n_tok == 0 || p->n_req == 0) return FSCHED_OK;
  if (!q || !q_start || !kv_len || !out) return FSCHED_EINVAL;
  if (p->table_width > 0 && !table) return FSCHED_EINVAL;
  if (p->prefix_len > 0 && !prefix_pages) return FSCHED_EINVAL;
  if (kv->n_pages > 0 && (!kv->k || !kv->v)) return FSCHED_EINVAL;
  if (!aligned16(q) || !aligned16(out)) return FSCHED_EINVAL;
  fs::AttnArgs a = attn_args(p, kv);
  a.q = q;
  a.prefix_pages = p->prefix_len > 0 ? prefix_pages : nullptr;
  a.table = table;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.out = out;
  a.lse = lse;
  hipStream_t s = (hipStream_t)stream;
  const int n_cu = fs::compute_units();
  const size_t need = fs::attend_workspace(a, kv->head_dim, n_cu);
  void* mine = nullptr;
  if (workspace) {
    if (((uintptr_t)workspace & 255) != 0) return FSCHED_EINVAL;
    if (workspace_bytes < 0 || (size_t)workspace_bytes < need) return FSCHED_ESCRATCH;
  } else if (need) {
    mine = workspace = fs::pool_alloc(need, s);
    if (!workspace) return FSCHED_ENOMEM;
  }
  const hipError_t e = fs::launch_attend(a, kv->dtype, kv->head_dim, n_cu, workspace, s);
  if (mine) fs::pool_free(mine, s);
  return finish(e, p->flags, s);
}

}  // namespace

extern "C" {

int fsched_kv_layout(const fsched_layout_params* p, const int32_t* old_len,
                     const int32_t* new_len, const int32_t* free_pages, int32_t* table,
                     int32_t* slots, int32_t* positions, int32_t* q_start, int32_t* kv_len,
                     int32_t* used, void* stream) {
  if (!p || p->reserved != 0) return FSCHED_EINVAL;
  int rc = check_flags(p->flags);
  if (rc) return rc;
  if (p->n_req < 0 || p->n_tok < 0 || !pow2(p->page_size) || p->table_width < 0 ||
      p->n_free < 0 || p->first_pos < 0)
    return FSCHED_EINVAL;
  if (p->page_size > kMaxPage || p->n_req > FSCHED_MAX_REQ || p->n_tok > FSCHED_MAX_STEP_TOKENS)
    return FSCHED_ETOOLARGE;
  if ((int64_t)p->table_width * p->page_size + p->first_pos > (1 << 30)) return FSCHED_ETOOLARGE;
  if (!q_start || !used) return FSCHED_EINVAL;
  if (p->n_req > 0 && (!old_len || !new_len || !kv_len)) return FSCHED_EINVAL;
  if (p->n_req > 0 && p->table_width > 0 && !table) return FSCHED_EINVAL;
  if (p->n_free > 0 && !free_pages) return FSCHED_EINVAL;
  if (p->n_tok > 0 && (!slots || !positions)) return FSCHED_EINVAL;
  fs::LayoutArgs a;
  a.n_req = p->n_req;
  a.n_tok = p->n_tok;
  a.page_shift = shift_of(p->page_size);
  a.width = p->table_width;
  a.n_free = p->n_free;
  a.first_pos = p->first_pos;
  a.old_len = old_len;
  a.new_len = new_len;
  a.free_pages = free_pages;
  a.table = table;
  a.slots = slots;
  a.positions = positions;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.used = used;
  return finish(fs::launch_kv_layout(a, (hipStream_t)stream), p->flags, (hipStream_t)stream);
}

int fsched_qk_norm_rope(const fsched_rope_params* p, const fsched_kv_cache* kv, const void* qkv,
                        const int32_t* positions, const int32_t* slots, const float* cos_sin,
                        const void* q_weight, const void* k_weight, void* q_out, void* stream) {
  if (!p || p->reserved != 0) return FSCHED_EINVAL;
  int rc = check_flags(p->flags);
  if (rc) return rc;
  rc = check_cache(kv);
  if (rc) return rc;
  if (p->n_tok < 0 || p->q_heads < 1 || p->rot_dim < 0 || p->rot_dim > kv->head_dim ||
      p->rot_dim % 16 != 0 || p->n_pos < 0 || (p->interleaved & ~1) != 0 || !(p->eps >= 0.0f) ||
      !std::isfinite(p->eps))
    return FSCHED_EINVAL;
  if (!stride_ok(p->qkv_stride) || !stride_ok(p->q_token_stride) || !stride_ok(p->q_head_stride))
    return FSCHED_EINVAL;
  if (p->q_heads > kMaxHeads || p->n_tok > FSCHED_MAX_STEP_TOKENS) return FSCHED_ETOOLARGE;
  if (p->n_tok == 0) return FSCHED_OK;
  if (!qkv || !q_out || !aligned16(qkv) || !aligned16(q_out)) return FSCHED_EINVAL;
  if (p->rot_dim > 0 && (!positions || !cos_sin || !aligned16(cos_sin))) return FSCHED_EINVAL;
  if (slots && kv->n_pages > 0 && (!kv->k || !kv->v)) return FSCHED_EINVAL;
  if (!aligned16(q_weight) || !aligned16(k_weight)) return FSCHED_EINVAL;
  fs::RopeArgs a;
  a.n_tok = p->n_tok;
  a.q_heads = p->q_heads;
  a.rot_dim = p->rot_dim;
  a.n_pos = p->n_pos;
  a.interleaved = p->interleaved;
  a.eps = p->eps;
  a.qkv_stride = p->qkv_stride;
  a.q_token = p->q_token_stride;
  a.q_head = p->q_head_stride;
  a.kv = cache_ref(kv);
  a.qkv = qkv;
  a.positions = positions;
  a.slots = slots;
  a.cos_sin = cos_sin;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.q_out = q_out;
  hipStream_t s = (hipStream_t)stream;
  return finish(fs::launch_qk_rope(a, kv->dtype, kv->head_dim, fs::compute_units(), s), p->flags,
                s);
}

int fsched_attend_workspace(const fsched_attn_params* p, const fsched_kv_cache* kv,
                            int64_t* bytes) {
  if (!bytes) return FSCHED_EINVAL;
  int rc = check_attn(p, kv);
  if (rc) return rc;
  *bytes = 0;
  if (p->n_tok == 0 || p->n_req == 0) return FSCHED_OK;
  *bytes = (int64_t)fs::attend_workspace(attn_args(p, kv), kv->head_dim, fs::compute_units());
  return FSCHED_OK;
}

int fsched_attend(const fsched_attn_params* p, const fsched_kv_cache* kv, const void* q,
                  const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* out,
                  float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  if (p && p->prefix_len != 0) return FSCHED_EINVAL;
  return attend_entry(p, kv, q, nullptr, table, q_start, kv_len, out, lse, workspace,
                      workspace_bytes, stream);
}

int fsched_attend_shared(const fsched_attn_params* p, const fsched_kv_cache* kv, const void* q,
                         const int32_t* prefix_pages, const int32_t* table,
                         const int32_t* q_start, const int32_t* kv_len, void* out, float* lse,
                         void* workspace, int64_t workspace_bytes, void* stream) {
  return attend_entry(p, kv, q, prefix_pages, table, q_start, kv_len, out, lse, workspace,
                      workspace_bytes, stream);
}

}  // extern "C"
