// Attention of a step's new tokens over the paged cache (fsched_attend,
// fsched_attend_shared): one wave per token and query head, one pass over the
// keys with the running maximum and sum of the softmax.
#include <hip/hip_runtime.h>

#include "half.hpp"
#include "step_common.hpp"

namespace fs {
namespace {

constexpr float NEG = -INFINITY;

template <class T, int D>
__global__ __launch_bounds__(64) void attend_simple(AttnArgs a) {
  constexpr int LANES = D / 8, KEYS = 64 / LANES;
  using elem = typename T::elem;
  using x8 = typename T::x8;
  const int lane = threadIdx.x, sub = lane & (LANES - 1), grp = lane / LANES;
  const int h = blockIdx.x % a.q_heads;
  const int t = blockIdx.x / a.q_heads;
  int lo = 0, hi = a.n_req;  // last request with q_start <= t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.q_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int r = lo;
  const int q0 = max(0, a.q_start[r]), q1 = min(a.n_tok, a.q_start[r + 1]);
  if (t < q0 || t >= q1 || t - q0 >= a.max_q) return;
  const int own = min(max(0, a.kv_len[r]), a.width << a.kv.page_shift);
  const int pos = a.prefix_len + own - (q1 - q0) + (t - q0);
  const int total = min(a.prefix_len + own, pos + 1);
  const int kh = h / a.group;
  const int mask = (1 << a.kv.page_shift) - 1;

  float q[8];
  const x8 qr = *(const x8*)((const elem*)a.q + t * a.q_token + h * a.q_head + sub * 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = (float)qr[i] * a.scale_log2;
  float m = NEG, l = 0.0f, o[8] = {};
  for (int j = grp; j < total; j += KEYS) {
    const bool in_window = a.window == 0 || j > pos - a.window || j < a.n_sink;
    if (!in_window) continue;
    const bool pre = j < a.prefix_len;
    const int x = pre ? j : j - a.prefix_len;
    const int page = pre ? a.prefix_pages[x >> a.kv.page_shift]
                         : a.table[(int64_t)r * a.width + (x >> a.kv.page_shift)];
    if (page < 0 || page >= a.kv.n_pages) continue;
    const x8 kr = *(const x8*)((const elem*)a.kv.k + page * a.kv.k_page + kh * a.kv.k_head +
                               (x & mask) * a.kv.k_slot + sub * 8);
    const x8 vr = *(const x8*)((const elem*)a.kv.v + page * a.kv.v_page + kh * a.kv.v_head +
                               (x & mask) * a.kv.v_slot + sub * 8);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(q[i], (float)kr[i], s);
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) s += __shfl_xor(s, d);
    const float m2 = fmaxf(m, s);
    const float f = m2 == NEG ? 1.0f : exp2f(m - m2), p = m2 == NEG ? 0.0f : exp2f(s - m2);
    m = m2;
    l = l * f + p;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = o[i] * f + p * (float)vr[i];
  }
#pragma unroll
  for (int d = LANES; d < 64; d <<= 1) {
    const float mo = __shfl_xor(m, d), lo2 = __shfl_xor(l, d);
    const float m2 = fmaxf(m, mo);
    const float f = m == NEG ? 0.0f : exp2f(m - m2), g = mo == NEG ? 0.0f : exp2f(mo - m2);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = o[i] * f + __shfl_xor(o[i], d) * g;
    l = l * f + lo2 * g;
    m = m2;
  }
  if (grp == 0) {
    x8 res;
#pragma unroll
    for (int i = 0; i < 8; ++i) res[i] = (elem)(l > 0.0f ? o[i] / l : 0.0f);
    *(x8*)((elem*)a.out + t * a.o_token + h * a.o_head + sub * 8) = res;
    if (a.lse && sub == 0)
      a.lse[(int64_t)t * a.q_heads + h] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : NEG;
  }
}

template <class T>
hipError_t launch(const AttnArgs& a, int head_dim, hipStream_t s) {
  const dim3 grid((unsigned)(a.n_tok * a.q_heads));
  switch (head_dim) {
    case 64: attend_simple<T, 64><<<grid, 64, 0, s>>>(a); break;
    case 128: attend_simple<T, 128><<<grid, 64, 0, s>>>(a); break;
    default: attend_simple<T, 256><<<grid, 64, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace(const AttnArgs&, int, int, int) { return 0; }

hipError_t launch_attend(const AttnArgs& a, int dtype, int head_dim, int, void*, hipStream_t s) {
  return dtype == FSCHED_BF16 ? launch<Bf16>(a, head_dim, s) : launch<F16>(a, head_dim, s);
}

}  // namespace fs
