// Attention weight of held tokens: which kernels a call runs (attend_weight.hpp).
#include "attend_weight.hpp"

namespace fs {
namespace {

// What a call of this shape launches.
struct Shape {
  bool few, many;  // requests of either kind are possible
  WeightPlan plan;
  size_t bytes;
};

size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

int64_t most_rows(const WeightArgs& a) {  // of one request and key head
  return (int64_t)a.at.max_q * a.at.group;
}

Shape shape_of(const WeightArgs& a, int head_dim, int n_cu, char* ws) {
  Shape s;
  __builtin_memset((void*)&s, 0, sizeof(s));
  s.few = a.at.group <= WEIGHT_FEW;
  s.many = most_rows(a) > WEIGHT_FEW;
  if (s.many) {
    const int keys = head_dim == 256 ? WeightTileOf<256>::KEYS : WeightTileOf<128>::KEYS;
    s.plan.blocks = 2 * n_cu;
    const size_t parts = round256((size_t)2 * s.plan.blocks * keys * sizeof(float));
    s.plan.part = (float*)ws;
    s.plan.tiles = (WeightTile*)(ws ? ws + parts : nullptr);
    s.bytes = parts + round256((size_t)s.plan.blocks * sizeof(WeightTile));
  }
  return s;
}

// Row tiles of the rows kernel: one if no request can have more than 16 rows, else two, with
// fewer blocks per compute unit.  One row tile for all steps and requests of 17 to 32 rows in the
// tiles kernel / as it is, us, caches of 16 bits and of 4:
//   drafts of 1 to 4 tokens, 64 requests, 8 heads per key head
//     heads of 64    40 / 16,  37 / 13
//     heads of 128   70 / 45,  52 / 28
//     heads of 256   59 / 44,  45 / 28
//   chunks of up to 512 tokens beside 43 decoding requests, 4 heads per key head (128: 4, 8)
//     heads of 64    75 / 76,  65 / 70  (window of 2,048)
//     heads of 128   89 / 92,  72 / 75;  113 / 117,  97 / 100
//     heads of 256   76 / 82,  59 / 64
// (Beside chunks, where the tiles kernel runs anyway, one row tile is faster by 1 to 7 %: a rule
// for those steps alone would have the tiles kernel's least number of rows follow it.)
template <class T, int D, int KIND>
hipError_t launch_kind(const WeightArgs& a, const Shape& p, int n_cu, hipStream_t s) {
  const size_t line = (size_t)(ATT_WAVES + a.at.n_req + 1) * sizeof(int64_t);
  constexpr bool FP4 = KIND == FP4_PAGES;
  if (p.few) {
    if (most_rows(a) <= 16)
      weight_rows_kernel<T, D, 1, KIND>
          <<<(unsigned)(weight_occupancy(D, 1, FP4) * n_cu), ATT_THREADS, line, s>>>(a);
    else
      weight_rows_kernel<T, D, 2, KIND>
          <<<(unsigned)(weight_occupancy(D, 2, FP4) * n_cu), ATT_THREADS, line, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.many) return e;
  }
  using L = WeightTileOf<D>;
  const size_t lds = L::LDS + line;
  void (*kernel)(WeightArgs, WeightPlan) = weight_tiles_kernel<T, D, FP4>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(
        (const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<p.plan.blocks, ATT_THREADS, lds, s>>>(a, p.plan);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;  // the join would read what was not written
  weight_join_kernel<L::KEYS><<<p.plan.blocks, L::KEYS, 0, s>>>(a, p.plan);
  return hipGetLastError();
}

template <class T, int D>
hipError_t launch(const WeightArgs& a, bool fp4, const Shape& p, int n_cu, hipStream_t s) {
  if (fp4) return launch_kind<T, D, FP4_PAGES>(a, p, n_cu, s);
  return a.at.kv.page_shift >= WIDE_SHIFT ? launch_kind<T, D, WIDE_PAGES>(a, p, n_cu, s)
                                          : launch_kind<T, D, SMALL_PAGES>(a, p, n_cu, s);
}

template <class T>
hipError_t launch_dim(const WeightArgs& a, bool fp4, int head_dim, const Shape& p, int n_cu,
                      hipStream_t s) {
  switch (head_dim) {
    case 64: return launch<T, 64>(a, fp4, p, n_cu, s);
    case 128: return launch<T, 128>(a, fp4, p, n_cu, s);
    default: return launch<T, 256>(a, fp4, p, n_cu, s);
  }
}

}  // namespace

size_t weight_workspace(const WeightArgs& a, int head_dim, int n_cu) {
  return shape_of(a, head_dim, n_cu > 0 ? n_cu : 256, nullptr).bytes;
}

hipError_t launch_weight(const WeightArgs& a, bool fp4, int dtype, int head_dim, int n_cu,
                         void* workspace, hipStream_t s) {
  if (n_cu <= 0) n_cu = 256;
  if (a.at.kv.n_pages == 0) return hipSuccess;  // no key is held
  const Shape p = shape_of(a, head_dim, n_cu, (char*)workspace);
  return dtype == FSCHED_BF16 ? launch_dim<Bf16>(a, fp4, head_dim, p, n_cu, s)
                              : launch_dim<F16>(a, fp4, head_dim, p, n_cu, s);
}

}  // namespace fs
