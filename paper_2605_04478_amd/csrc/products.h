// What the operators of a training step's computation share on the host: limits, alignment, the join of split sums.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ccld.h"

namespace ccld {

constexpr int DEPTH = 64;              // contractions are divided in whole multiples of it
constexpr uint64_t COMPUTE_UNITS = 256;
constexpr uint64_t MAX_GROUPS = (uint64_t)1 << 22;      // workgroups of up to 1,024 threads in a launch
constexpr int64_t MAX_ROWS = (int64_t)1 << 31, MAX_EXPERTS = (int64_t)1 << 20, MAX_WIDTH = (int64_t)1 << 22;
// a tile's last row starts below 2^31 bytes from its first: 256 rows (or DEPTH of them) of this many 16-bit elements, and a row
constexpr int64_t MAX_LD = ((int64_t)1 << 22) - ((int64_t)1 << 14);

inline bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline ccld_status launched() { return hipGetLastError() == hipSuccess ? CCLD_OK : CCLD_E_HIP; }

// out[r][c] = sum over the splits, in their order, of part[s][r][c] (join.hip)
void launch_join(const float* part, uint32_t splits, uint64_t rows, uint64_t cols, void* out, int64_t ldo, int32_t dtype,
                 hipStream_t stream);

}  // namespace ccld
