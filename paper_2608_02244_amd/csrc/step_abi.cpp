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

int check_cache4(const fsched_kv4_cache* c) {
  if (!c || c->reserved != 0) return FSCHED_EINVAL;
  if (c->n_pages < 0 || !pow2(c->page_size) || c->page_size < 16 || c->kv_heads < 1)
    return FSCHED_EINVAL;
  if (c->dtype != FSCHED_BF16 && c->dtype != FSCHED_F16) return FSCHED_EINVAL;
  if (c->head_dim < 1) return FSCHED_EINVAL;
  for (int i = 0; i < 3; ++i)
    if (c->stride[i] < 0 || (c->stride[i] & 15) != 0) return FSCHED_EINVAL;
  if (!aligned16(c->data)) return FSCHED_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return FSCHED_ENOTIMPL;
  if (c->page_size > kMaxPage || c->kv_heads > kMaxHeads) return FSCHED_ETOOLARGE;
  for (int i = 0; i < 3; ++i)
    if (c->stride[i] > kMaxStride) return FSCHED_ETOOLARGE;
  return FSCHED_OK;
}

fs::CacheRef cache4_ref(const fsched_kv4_cache* c) {
  fs::CacheRef r;
  std::memset(&r, 0, sizeof(r));
  r.k = c->data;
  r.k_page = c->stride[0];
  r.k_head = c->stride[1];
  r.k_slot = c->stride[2];
  r.n_pages = c->n_pages;
  r.page_shift = shift_of(c->page_size);
  r.kv_heads = c->kv_heads;
  return r;
}

// What the calls over either kind of cache need of it.
struct AnyCache {
  bool fp4;
  int32_t n_pages, page_size, kv_heads, head_dim, dtype;
  fs::CacheRef ref;
  bool held;  // its pointers are there
};

int any_cache(const fsched_kv_cache* c, bool values, AnyCache* r) {
  const int rc = check_cache(c);
  if (rc) return rc;
  *r = AnyCache{false, c->n_pages, c->page_size, c->kv_heads, c->head_dim, c->dtype,
                cache_ref(c), c->k && (c->v || !values)};
  return FSCHED_OK;
}

int any_cache(const fsched_kv4_cache* c, bool, AnyCache* r) {
  const int rc = check_cache4(c);
  if (rc) return rc;
  *r = AnyCache{true, c->n_pages, c->page_size, c->kv_heads, c->head_dim, c->dtype,
                cache4_ref(c), c->data != nullptr};
  return FSCHED_OK;
}

int finish(hipError_t e, uint32_t flags, hipStream_t s) {
  if (e == hipSuccess && (flags & FSCHED_F_SYNC)) e = hipStreamSynchronize(s);
  return e == hipSuccess ? FSCHED_OK : fs::record_hip_error(e);
}

template <class Cache>
int check_attn(const fsched_attn_params* p, const Cache* kv, bool values, AnyCache* c) {
  if (!p) return FSCHED_EINVAL;
  int rc = check_flags(p->flags);
  if (rc) return rc;
  rc = any_cache(kv, values, c);
  if (rc) return rc;
  if (p->n_req < 0 || p->n_tok < 0 || p->q_heads < 1 || p->q_heads % c->kv_heads != 0 ||
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
  if ((int64_t)p->table_width * c->page_size + p->prefix_len > (1 << 30)) return FSCHED_ETOOLARGE;
  return FSCHED_OK;
}

fs::AttnArgs attn_args(const fsched_attn_params* p, const AnyCache& c) {
  fs::AttnArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_req = p->n_req;
  a.n_tok = p->n_tok;
  a.q_heads = p->q_heads;
  a.group = p->q_heads / c.kv_heads;
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
  a.kv = c.ref;
  return a;
}

// A call's workspace: the caller's, or the library's for the call.
class Workspace {
 public:
  int take(void* given, int64_t bytes, size_t need, hipStream_t s) {
    at_ = given;
    stream_ = s;
    if (given) {
      if (((uintptr_t)given & 255) != 0) return FSCHED_EINVAL;
      return bytes < 0 || (size_t)bytes < need ? FSCHED_ESCRATCH : FSCHED_OK;
    }
    if (need) {
      at_ = mine_ = fs::pool_alloc(need, s);
      if (!at_) return FSCHED_ENOMEM;
    }
    return FSCHED_OK;
  }
  ~Workspace() {
    if (mine_) fs::pool_free(mine_, stream_);
  }
  void* get() const { return at_; }

 private:
  void *at_ = nullptr, *mine_ = nullptr;
  hipStream_t stream_ = nullptr;
};

template <class Cache>
int attend_entry(const fsched_attn_params* p, const Cache* kv, const void* q,
                 const int32_t* prefix_pages, const int32_t* table, const int32_t* q_start,
                 const int32_t* kv_len, void* out, float* lse, void* workspace,
                 int64_t workspace_bytes, void* stream) {
  AnyCache c;
  int rc = check_attn(p, kv, true, &c);
  if (rc) return rc;
  if (p->n_tok == 0 || p->n_req == 0) return FSCHED_OK;
  if (!q || !q_start || !kv_len || !out) return FSCHED_EINVAL;
  if (p->table_width > 0 && !table) return FSCHED_EINVAL;
  if (p->prefix_len > 0 && !prefix_pages) return FSCHED_EINVAL;
  if (c.n_pages > 0 && !c.held) return FSCHED_EINVAL;
  if (!aligned16(q) || !aligned16(out)) return FSCHED_EINVAL;
  fs::AttnArgs a = attn_args(p, c);
  a.q = q;
  a.prefix_pages = p->prefix_len > 0 ? prefix_pages : nullptr;
  a.table = table;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.out = out;
  a.lse = lse;
  hipStream_t s = (hipStream_t)stream;
  const int n_cu = fs::compute_units();
  hipError_t e;
  {
    Workspace ws;
    rc = ws.take(workspace, workspace_bytes, fs::attend_workspace(a, c.fp4, c.head_dim, n_cu), s);
    if (rc) return rc;
    e = fs::launch_attend(a, c.fp4, c.dtype, c.head_dim, n_cu, ws.get(), s);
  }
  return finish(e, p->flags, s);
}

template <class Cache>
int attend_bytes(const fsched_attn_params* p, const Cache* kv, int64_t* bytes) {
  if (!bytes) return FSCHED_EINVAL;
  AnyCache c;
  const int rc = check_attn(p, kv, true, &c);
  if (rc) return rc;
  *bytes = 0;
  if (p->n_tok == 0 || p->n_req == 0) return FSCHED_OK;
  *bytes = (int64_t)fs::attend_workspace(attn_args(p, c), c.fp4, c.head_dim, fs::compute_units());
  return FSCHED_OK;
}

// Rows of a request and key head (its tokens times the query heads) are counted in 32 bits,
// and 64 of them are addressed by 32-bit offsets from the first one's token.
bool rows_fit(const fsched_attn_params* p, const AnyCache& c) {
  const int64_t group = p->q_heads / c.kv_heads;
  if (p->max_q * group > (1 << 30)) return false;
  if (p->q_token_stride > kMaxStride || p->q_head_stride > kMaxStride) return false;
  return (64 / group + 2) * p->q_token_stride + group * p->q_head_stride + c.head_dim <= (1 << 30);
}

template <class Cache>
int weight_entry(const fsched_attn_params* p, const Cache* kv, const void* q, const float* lse,
                 const int32_t* table, const int32_t* q_start, const int32_t* kv_len,
                 float* weight, int64_t weight_stride, void* workspace, int64_t workspace_bytes,
                 void* stream) {
  AnyCache c;
  int rc = check_attn(p, kv, false, &c);
  if (rc) return rc;
  if (weight_stride < (int64_t)p->table_width * c.page_size) return FSCHED_EINVAL;
  if (weight_stride > kMaxStride) return FSCHED_ETOOLARGE;
  if (!rows_fit(p, c)) return FSCHED_ETOOLARGE;
  if (p->n_tok == 0 || p->n_req == 0 || p->table_width == 0) return FSCHED_OK;
  if (!q || !lse || !table || !q_start || !kv_len || !weight) return FSCHED_EINVAL;
  if (c.n_pages > 0 && !c.held) return FSCHED_EINVAL;
  if (!aligned16(q)) return FSCHED_EINVAL;
  fs::WeightArgs a;
  a.at = attn_args(p, c);
  a.at.q = q;
  a.at.table = table;
  a.at.q_start = q_start;
  a.at.kv_len = kv_len;
  a.group.set(a.at.group);
  a.lse = lse;
  a.weight = weight;
  a.weight_stride = weight_stride;
  hipStream_t s = (hipStream_t)stream;
  const int n_cu = fs::compute_units();
  hipError_t e;
  {
    Workspace ws;
    rc = ws.take(workspace, workspace_bytes, fs::weight_workspace(a, c.head_dim, n_cu), s);
    if (rc) return rc;
    e = fs::launch_weight(a, c.fp4, c.dtype, c.head_dim, n_cu, ws.get(), s);
  }
  return finish(e, p->flags, s);
}

template <class Cache>
int weight_bytes(const fsched_attn_params* p, const Cache* kv, int64_t* bytes) {
  if (!bytes) return FSCHED_EINVAL;
  AnyCache c;
  const int rc = check_attn(p, kv, false, &c);
  if (rc) return rc;
  if (!rows_fit(p, c)) return FSCHED_ETOOLARGE;
  *bytes = 0;
  if (p->n_tok == 0 || p->n_req == 0 || p->table_width == 0) return FSCHED_OK;
  fs::WeightArgs a;
  std::memset(&a, 0, sizeof(a));
  a.at = attn_args(p, c);
  *bytes = (int64_t)fs::weight_workspace(a, c.head_dim, fs::compute_units());
  return FSCHED_OK;
}

int check_evict(const fsched_evict_params* p) {
  if (!p || p->reserved != 0) return FSCHED_EINVAL;
  const int rc = check_flags(p->flags);
  if (rc) return rc;
  if (p->n_req < 0 || p->table_width < 0 || !pow2(p->page_size) || p->n_sink < 0 ||
      p->n_recent < 0 || p->n_freed < 0)
    return FSCHED_EINVAL;
  if (p->page_size > kMaxPage || p->n_req > FSCHED_MAX_REQ) return FSCHED_ETOOLARGE;
  const int64_t row = (int64_t)p->table_width * p->page_size;
  // pages of all requests are counted in 32 bits
  if (row > (1 << 30) || (int64_t)p->n_req * p->table_width > INT32_MAX) return FSCHED_ETOOLARGE;
  if (p->weight_stride < row) return FSCHED_EINVAL;
  return p->weight_stride > kMaxStride ? FSCHED_ETOOLARGE : FSCHED_OK;
}

fs::EvictArgs evict_args(const fsched_evict_params* p) {
  fs::EvictArgs a;
  std::memset(&a, 0, sizeof(a));
  a.n_req = p->n_req;
  a.width = p->table_width;
  a.page_shift = shift_of(p->page_size);
  a.n_sink = p->n_sink;
  a.n_recent = p->n_recent;
  a.n_freed = p->n_freed;
  a.weight_stride = p->weight_stride;
  return a;
}

template <class Cache>
int rope_entry(const fsched_rope_params* p, const Cache* kv, const void* qkv,
               const int32_t* positions, const int32_t* slots, const float* cos_sin,
               const void* q_weight, const void* k_weight, void* q_out, void* stream) {
  if (!p || p->reserved != 0) return FSCHED_EINVAL;
  int rc = check_flags(p->flags);
  if (rc) return rc;
  AnyCache c;
  rc = any_cache(kv, true, &c);
  if (rc) return rc;
  if (p->n_tok < 0 || p->q_heads < 1 || p->rot_dim < 0 || p->rot_dim > c.head_dim ||
      p->rot_dim % 16 != 0 || p->n_pos < 0 || (p->interleaved & ~1) != 0 || !(p->eps >= 0.0f) ||
      !std::isfinite(p->eps))
    return FSCHED_EINVAL;
  if (!stride_ok(p->qkv_stride) || !stride_ok(p->q_token_stride) || !stride_ok(p->q_head_stride))
    return FSCHED_EINVAL;
  if (p->q_heads > kMaxHeads || p->n_tok > FSCHED_MAX_STEP_TOKENS) return FSCHED_ETOOLARGE;
  if (p->n_tok == 0) return FSCHED_OK;
  if (!qkv || !q_out || !aligned16(qkv) || !aligned16(q_out)) return FSCHED_EINVAL;
  if (p->rot_dim > 0 && (!positions || !cos_sin || !aligned16(cos_sin))) return FSCHED_EINVAL;
  if (slots && c.n_pages > 0 && !c.held) return FSCHED_EINVAL;
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
  a.kv = c.ref;
  a.qkv = qkv;
  a.positions = positions;
  a.slots = slots;
  a.cos_sin = cos_sin;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.q_out = q_out;
  hipStream_t s = (hipStream_t)stream;
  const int n_cu = fs::compute_units();
  return finish(c.fp4 ? fs::launch_qk_rope4(a, c.dtype, c.head_dim, n_cu, s)
                      : fs::launch_qk_rope(a, c.dtype, c.head_dim, n_cu, s),
                p->flags, s);
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
  return rope_entry(p, kv, qkv, positions, slots, cos_sin, q_weight, k_weight, q_out, stream);
}

int fsched_qk_norm_rope4(const fsched_rope_params* p, const fsched_kv4_cache* kv,
                         const void* qkv, const int32_t* positions, const int32_t* slots,
                         const float* cos_sin, const void* q_weight, const void* k_weight,
                         void* q_out, void* stream) {
  return rope_entry(p, kv, qkv, positions, slots, cos_sin, q_weight, k_weight, q_out, stream);
}

int fsched_kv4_read(const fsched_read_params* p, const fsched_kv4_cache* kv,
                    const int32_t* slots, void* k_out, void* v_out, void* stream) {
  if (!p) return FSCHED_EINVAL;
  int rc = check_flags(p->flags);
  if (rc) return rc;
  rc = check_cache4(kv);
  if (rc) return rc;
  if (p->n_tok < 0 || !stride_ok(p->token_stride) || !stride_ok(p->head_stride))
    return FSCHED_EINVAL;
  if (p->n_tok > FSCHED_MAX_STEP_TOKENS) return FSCHED_ETOOLARGE;
  if (p->n_tok == 0) return FSCHED_OK;
  if (!slots || !k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return FSCHED_EINVAL;
  if (kv->n_pages > 0 && !kv->data) return FSCHED_EINVAL;
  fs::Read4Args a;
  a.n_tok = p->n_tok;
  a.token = p->token_stride;
  a.head = p->head_stride;
  a.kv = cache4_ref(kv);
  a.slots = slots;
  a.k_out = k_out;
  a.v_out = v_out;
  hipStream_t s = (hipStream_t)stream;
  return finish(fs::launch_kv4_read(a, kv->dtype, kv->head_dim, s), p->flags, s);
}

int fsched_attend_workspace(const fsched_attn_params* p, const fsched_kv_cache* kv,
                            int64_t* bytes) {
  return attend_bytes(p, kv, bytes);
}

int fsched_attend4_workspace(const fsched_attn_params* p, const fsched_kv4_cache* kv,
                             int64_t* bytes) {
  return attend_bytes(p, kv, bytes);
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

int fsched_attend4(const fsched_attn_params* p, const fsched_kv4_cache* kv, const void* q,
                   const int32_t* prefix_pages, const int32_t* table, const int32_t* q_start,
                   const int32_t* kv_len, void* out, float* lse, void* workspace,
                   int64_t workspace_bytes, void* stream) {
  return attend_entry(p, kv, q, prefix_pages, table, q_start, kv_len, out, lse, workspace,
                      workspace_bytes, stream);
}

int fsched_attend_weight(const fsched_attn_params* p, const fsched_kv_cache* kv, const void* q,
                         const float* lse, const int32_t* table, const int32_t* q_start,
                         const int32_t* kv_len, float* weight, int64_t weight_stride,
                         void* workspace, int64_t workspace_bytes, void* stream) {
  return weight_entry(p, kv, q, lse, table, q_start, kv_len, weight, weight_stride, workspace,
                      workspace_bytes, stream);
}

int fsched_attend4_weight(const fsched_attn_params* p, const fsched_kv4_cache* kv, const void* q,
                          const float* lse, const int32_t* table, const int32_t* q_start,
                          const int32_t* kv_len, float* weight, int64_t weight_stride,
                          void* workspace, int64_t workspace_bytes, void* stream) {
  return weight_entry(p, kv, q, lse, table, q_start, kv_len, weight, weight_stride, workspace,
                      workspace_bytes, stream);
}

int fsched_attend_weight_workspace(const fsched_attn_params* p, const fsched_kv_cache* kv,
                                   int64_t* bytes) {
  return weight_bytes(p, kv, bytes);
}

int fsched_attend4_weight_workspace(const fsched_attn_params* p, const fsched_kv4_cache* kv,
                                    int64_t* bytes) {
  return weight_bytes(p, kv, bytes);
}

int fsched_kv_evict(const fsched_evict_params* p, const float* weight, const int32_t* kv_len,
                    const int32_t* table, const int32_t* budget, int32_t* new_table,
                    float* new_weight, int32_t* new_len, int32_t* freed, int32_t* count,
                    void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_evict(p);
  if (rc) return rc;
  if (!count || (p->n_freed > 0 && !freed)) return FSCHED_EINVAL;
  if (p->n_req > 0 && (!kv_len || !budget || !new_len)) return FSCHED_EINVAL;
  if (p->n_req > 0 && p->table_width > 0 && (!weight || !table || !new_table || !new_weight))
    return FSCHED_EINVAL;
  fs::EvictArgs a = evict_args(p);
  a.weight = weight;
  a.kv_len = kv_len;
  a.table = table;
  a.budget = budget;
  a.new_table = new_table;
  a.new_weight = new_weight;
  a.new_len = new_len;
  a.freed = freed;
  a.count = count;
  hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  {
    Workspace ws;
    rc = ws.take(workspace, workspace_bytes, fs::evict_workspace(a), s);
    if (rc) return rc;
    e = fs::launch_evict(a, fs::compute_units(), ws.get(), s);
  }
  return finish(e, p->flags, s);
}

int fsched_kv_evict_workspace(const fsched_evict_params* p, int64_t* bytes) {
  if (!bytes) return FSCHED_EINVAL;
  const int rc = check_evict(p);
  if (rc) return rc;
  *bytes = (int64_t)fs::evict_workspace(evict_args(p));
  return FSCHED_OK;
}

}  // extern "C"
