// Launch descriptors and host checks shared by the operators of a step
// (kv_layout.hip, qk_rope.hip, attend*.hip, kv_evict.hip, step_abi.cpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fsched.h"

namespace fs {

struct LayoutArgs {
  int32_t n_req, n_tok, page_shift, width, n_free, first_pos;
  const int32_t* old_len;
  const int32_t* new_len;
  const int32_t* free_pages;
  int32_t* table;
  int32_t* slots;
  int32_t* positions;
  int32_t* q_start;
  int32_t* kv_len;
  int32_t* used;
};

// Device view of an fsched_kv_cache, or of an fsched_kv4_cache: then k is its data and
// k_page, k_head and k_slot (of a group of 16 tokens) are bytes; the v fields are unused.
struct CacheRef {
  const void* k;
  const void* v;
  int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
  int32_t n_pages, page_shift, kv_heads;
};

struct RopeArgs {
  int32_t n_tok, q_heads, rot_dim, n_pos, interleaved;
  float eps;
  int64_t qkv_stride, q_token, q_head;
  CacheRef kv;
  const void* qkv;
  const int32_t* positions;
  const int32_t* slots;
  const float* cos_sin;
  const void* q_weight;
  const void* k_weight;
  void* q_out;
};

struct Read4Args {
  int32_t n_tok;
  int64_t token, head;
  CacheRef kv;
  const int32_t* slots;
  void* k_out;
  void* v_out;
};

struct AttnArgs {
  int32_t n_req, n_tok, q_heads, group, max_q, width, window, n_sink, prefix_len;
  float scale_log2;  // scale * log2(e): exponentials are taken in base 2
  int64_t q_token, q_head, o_token, o_head;
  CacheRef kv;
  const void* q;
  const int32_t* prefix_pages;  // null without a prefix
  const int32_t* table;
  const int32_t* q_start;
  const int32_t* kv_len;
  void* out;
  float* lse;  // nullable
};

// Division of whole numbers below 2^31 by a divisor d that a launch knows:  with
// 2^l >= d > 2^(l - 1) and m = floor(2^(31 + l) / d) + 1, which fits 32 bits,
// floor(n / d) = floor(n m / 2^(31 + l)).
struct Divisor {
  uint32_t m;
  int32_t shift;  // l - 1; -1: d is 1
  void set(int32_t d) {
    shift = -1;
    while ((int64_t)1 << (shift + 1) < d) ++shift;
    m = shift < 0 ? 0 : (uint32_t)(((uint64_t)1 << (32 + shift)) / (uint32_t)d + 1);
  }
  __device__ __forceinline__ int divide(int n) const {
    return shift < 0 ? n : (int)(__umulhi((uint32_t)n, m) >> shift);
  }
};

// The attention weight of held tokens: of `at` q, the tables and the cache's keys.
struct WeightArgs {
  AttnArgs at;
  Divisor group;
  const float* lse;
  float* weight;
  int64_t weight_stride;
};

struct EvictArgs {
  int32_t n_req, width, page_shift, n_sink, n_recent, n_freed;
  int64_t weight_stride;
  const float* weight;
  const int32_t* kv_len;
  const int32_t* table;
  const int32_t* budget;
  int32_t* new_table;
  float* new_weight;
  int32_t* new_len;
  int32_t* freed;
  int32_t* count;
};

hipError_t launch_kv_layout(const LayoutArgs& a, hipStream_t s);
hipError_t launch_qk_rope(const RopeArgs& a, int dtype, int head_dim, int n_cu, hipStream_t s);
hipError_t launch_qk_rope4(const RopeArgs& a, int dtype, int head_dim, int n_cu, hipStream_t s);
hipError_t launch_kv4_read(const Read4Args& a, int dtype, int head_dim, hipStream_t s);

// Workspace bytes of one attention call on a device of n_cu compute units.  fp4: over a
// cache of 4 bits.
size_t attend_workspace(const AttnArgs& a, bool fp4, int head_dim, int n_cu);
hipError_t launch_attend(const AttnArgs& a, bool fp4, int dtype, int head_dim, int n_cu,
                         void* workspace, hipStream_t s);

size_t weight_workspace(const WeightArgs& a, int head_dim, int n_cu);
hipError_t launch_weight(const WeightArgs& a, bool fp4, int dtype, int head_dim, int n_cu,
                         void* workspace, hipStream_t s);

size_t evict_workspace(const EvictArgs& a);
hipError_t launch_evict(const EvictArgs& a, int n_cu, void* workspace, hipStream_t s);

}  // namespace fs
