// What the operators around a step's products share: elements' types, loads of vectors at any alignment, sums and maxima over a wavefront.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_utils.h"
#include "products.h"

namespace ccld {

// N values of 16 bytes and less, at addresses that are aligned to one value: the card loads and stores them in one instruction wherever they start.
template <class T, int N>
struct Vector {
  typedef T type __attribute__((ext_vector_type(N)));
  typedef T loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <class T, int N>
using Vec = typename Vector<T, N>::type;
template <int N, class T>
__device__ __forceinline__ Vec<T, N> load_vec(const T* p) {
  if constexpr (N == 1) return Vec<T, 1>{*p};
  else return *reinterpret_cast<const typename Vector<T, N>::loose*>(p);
}
template <int N, class T>
__device__ __forceinline__ void store_vec(T* p, Vec<T, N> v) {
  if constexpr (N == 1) *p = v[0];
  else *reinterpret_cast<typename Vector<T, N>::loose*>(p) = v;
}

// The same past the caches where they can: for what is not read again before much else has been.
template <int N, class T>
__device__ __forceinline__ Vec<T, N> load_once(const T* p) {
  if constexpr (N == 1) return Vec<T, 1>{*p};
  else return __builtin_nontemporal_load(reinterpret_cast<const typename Vector<T, N>::loose*>(p));
}
template <int N, class T>
__device__ __forceinline__ void store_once(T* p, Vec<T, N> v) {
  if constexpr (N == 1) *p = v[0];
  else __builtin_nontemporal_store(v, reinterpret_cast<typename Vector<T, N>::loose*>(p));
}

// Maxima and sums over a wavefront's lanes, in all of them.  Neighbours by DPP shifts within rows of 16 lanes, then the rows' results (a shuffle
// through the LDS crossbar takes many times as long).
template <int CTRL>
__device__ __forceinline__ float dpp(float v, float outside) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, outside), __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float read_lane(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }
// (NaN is ignored)
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp<0x121>(v, v));      // row_ror: 1, 2, 4, 8
  v = fmaxf(v, dpp<0x122>(v, v));
  v = fmaxf(v, dpp<0x124>(v, v));
  v = fmaxf(v, dpp<0x128>(v, v));
  return fmaxf(fmaxf(read_lane(v, 0), read_lane(v, 16)), fmaxf(read_lane(v, 32), read_lane(v, 48)));
}
__device__ __forceinline__ float wave_total(float v) {
  v += dpp<0x121>(v, v);
  v += dpp<0x122>(v, v);
  v += dpp<0x124>(v, v);
  v += dpp<0x128>(v, v);
  return (read_lane(v, 0) + read_lane(v, 16)) + (read_lane(v, 32) + read_lane(v, 48));
}

constexpr float LOWEST = -__builtin_huge_valf();

inline i64 blocks_for(i64 n, i64 each) { return (n + each - 1) / each; }
inline int32_t size_of(int32_t dtype) { return dtype == CCLD_FP32 ? 4 : 2; }
inline bool known_type(int32_t dtype) { return dtype == CCLD_BF16 || dtype == CCLD_FP16 || dtype == CCLD_FP32; }

// f(T()) for the elements' type
template <class F>
auto with_type(int32_t dtype, F f) {
  return dtype == CCLD_BF16 ? f(__bf16()) : dtype == CCLD_FP16 ? f(_Float16()) : f(float());
}

}  // namespace ccld
