// Joins sums over parts of a contraction.  The parts are added in their order, so the result does not depend on which
// workgroup ended first (atomic additions would).
#include "device_utils.h"
#include "products.h"
#include "tiles.h"

namespace ccld {
namespace {

// four neighbouring columns to a thread where rows allow it; memory-bound: 4 bytes per split and value read, 2 written
template <class T, int V>
__global__ __launch_bounds__(256) void k_join(const float* __restrict__ part, u32 splits, u64 rows, u64 cols, T* __restrict__ out,
                                              i64 ldo) {
  const u64 pieces = rows * cols / V;
  for (u64 p = (u64)blockIdx.x * 256 + threadIdx.x; p < pieces; p += (u64)gridDim.x * 256) {
    const u64 at = p * V, r = at / cols, c = at - r * cols;
    float sum[V] = {};
    for (u32 s = 0; s < splits; ++s) {
      const float* q = part + (u64)s * rows * cols + at;
      if constexpr (V == 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(q);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += v[i];
      } else sum[0] += *q;
    }
    T* o = out + r * ldo + c;
    if constexpr (V == 4) store4(o, f32x4{sum[0], sum[1], sum[2], sum[3]}, 4, true);
    else *o = (T)sum[0];
  }
}

template <class T>
void join(const float* part, u32 splits, u64 rows, u64 cols, T* out, i64 ldo, hipStream_t stream) {
  const bool wide = cols % 4 == 0 && ldo % 4 == 0 && aligned(out, 4 * sizeof(T));
  const u64 n = rows * cols / (wide ? 4 : 1), groups = (n + 255) / 256;
  const u32 grid = (u32)(groups < 4096 ? groups : 4096);
  if (wide) k_join<T, 4><<<grid, 256, 0, stream>>>(part, splits, rows, cols, out, ldo);
  else k_join<T, 1><<<grid, 256, 0, stream>>>(part, splits, rows, cols, out, ldo);
}
}  // namespace

void launch_join(const float* part, uint32_t splits, uint64_t rows, uint64_t cols, void* out, int64_t ldo, int32_t dtype,
                 hipStream_t stream) {
  if (!rows || !cols) return;
  if (dtype == CCLD_BF16) join(part, splits, rows, cols, static_cast<__bf16*>(out), ldo, stream);
  else join(part, splits, rows, cols, static_cast<_Float16*>(out), ldo, stream);
}
}  // namespace ccld
