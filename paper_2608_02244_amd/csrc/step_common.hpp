// Launch descriptors and host checks shared by the operators of a step
// (kv_layout.hip, qk_rope.hip, attend*.hip, step_abi.cpp).
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

struct CacheRef {  // device view of an fsched_kv_cache
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

hipError_t launch_kv_layout(const LayoutArgs& a, hipStream_t s);
hipError_t launch_qk_rope(const RopeArgs& a, int dtype, int head_dim, int n_cu, hipStream_t s);

// Workspace bytes of one attention call on a device of n_cu compute units.
size_t attend_workspace(const AttnArgs& a, int head_dim, int n_cu);
hipError_t launch_attend(const AttnArgs& a, int dtype, int head_dim, int n_cu, void* workspace,
                         hipStream_t s);

}  // namespace fs
