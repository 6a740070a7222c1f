// A step of AdamW over many tensors at once, with states in 32 or in 8 bits (ccld_adamw).
//
//   t = ++count      g' = scale g      m = b1 m + (1 - b1) g'      v = b2 v + (1 - b2) g'^2
//   p = p - lr wd p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Memory bounds it: thirty operations, or sixty with states in 8 bits, to the 10 to 30 bytes of an element.  The tensors of a launch are listed in its arguments, so that nothing has to
// be copied to the device and a captured launch keeps its list; a workgroup finds its tensor by a ballot over the list.  What depends on
// the count is computed once, on the device, by a launch of one thread: a replayed graph counts on.
//
// States in 8 bits: blocks of 256 elements (32 lanes with 8 each) share a scale.  m is an e4m3, v an e5m2 number: a block in which one gradient is
// thousands of times the others' must not lift the others' v, for which its 32 powers of two matter more than a bit of precision.  Rounding to nearest would not
// follow b2 = 0.999, whose steps are a hundredth of what two or three bits tell apart; values are rounded up or down at random, with the odds that keep
// the mean.  The card converts and rounds both formats.
//
// Measured (a copy of 2 GB moves 4.9 TB/s here, x + 1 6.1): 200 tensors, 90M elements in bfloat16 with masters 408 us = 6.2 TB/s; 320M in bfloat16 with 8-bit states 560 us = 5.7 TB/s, where the 61 instructions
// of an element take 532 by themselves (575 where an eps is so small that roots of subnormal numbers count; 732 with conversions and rounding by hand, exact root and quotient), with 32-bit states 1,094 = 6.4, with
// masters and 8-bit states 986, and gradients in 32 bits 1,120; six small tensors 2 + 4 us of a call's 8.8.
#include <algorithm>

#include <math.h>

#include "ccld_internal.h"
#include "operators.h"

using namespace ccld;

namespace {

constexpr int BLOCK = CCLD_ADAMW_BLOCK, ADAMW_THREADS = 128;
// neighbouring elements of a thread: 16 bytes of a 32-bit state, 8 of one in 8 bits
constexpr int each_of(int bits) { return bits == 32 ? 4 : 8; }
// elements of a workgroup: one vector to a thread, or two of 8 bits, which have more to compute.  (90M elements with masters: 406 us; 413 in workgroups of 256 threads, 444 with two vectors to
// a thread, 465 with four, 491 with eight.  320M with 8-bit states: 561; 577 with one vector, 586 with four.)
constexpr int chunk_of(int bits) { return bits == 32 ? 512 : 2048; }
typedef u32 Words __attribute__((ext_vector_type(2), aligned(4)));      // 8-bit values
constexpr int LISTED = 112;                              // tensors of a launch: its arguments have 4 KB

// What a step's elements share.
struct Step { float step_size, root, decay, scale; u32 key; };

struct Tensor { void* p; const void* g; i64 n; u32 start, chunk0; };      // start: in blocks; chunk0: its first workgroup
struct AdamwJob {
  Tensor tensors[LISTED];
  const Step* step;
  void *m, *v;
  float *m_scale, *v_scale, *master;
  float b1, b2, c1, c2, eps;
  int n_tensors;
  bool small_eps, far_eps;       // roots of subnormal numbers count; the card has no reciprocal of eps
};
static_assert(sizeof(AdamwJob) <= 4096, "arguments of a launch");

// 32 bits of a number from 32 bits of another, each of which depends on all of them
__device__ __forceinline__ u32 mix(u32 x) {
  x = (x ^ x >> 16) * 0x9E3779B1u;
  x = (x ^ x >> 15) * 0xBB67AE85u;
  return x ^ x >> 16;
}

struct BeginJob {
  i64* count;
  const float* scale_by;
  Step* step;
  double lr, b1, b2, weight_decay, scale;
  u64 seed;
};
__global__ void k_adamw_begin(BeginJob j) {
  const i64 t = ++*j.count;
  Step s;
  s.step_size = (float)(j.lr / (1.0 - pow(j.b1, (double)t)));
  s.root = (float)(1.0 / sqrt(1.0 - pow(j.b2, (double)t)));
  // (1 - lr wd would lose most of lr wd's bits in 32 of them)
  s.decay = (float)(j.lr * j.weight_decay);
  s.scale = (float)(j.scale_by ? j.scale * (double)*j.scale_by : j.scale);
  s.key = mix(mix(mix(mix((u32)j.seed) ^ (u32)(j.seed >> 32)) ^ (u32)t) ^ (u32)(t >> 32));
  *j.step = s;
}

constexpr float FIRST_MOST = 448.0f, SECOND_MOST = 57344.0f;            // the largest values of e4m3 and e5m2
constexpr float SECOND_LEAST = 0x1p-16f;                               // the smallest of e5m2 but zero

// |x| / scale rounded towards zero, whose reciprocal is at hand: a step of the division's remainder makes it the nearest quotient, the sign of what then remains says whether that is
// too large.  What random bits are added to is then not rounded before: a value goes up or down as the exact quotient says.
__device__ __forceinline__ float quotient(float x, float scale, float reciprocal) {
  const float a = fabsf(x), first = a * reciprocal, q = fmaf(fmaf(-first, scale, a), reciprocal, first);
  return __builtin_bit_cast(float, __builtin_bit_cast(u32, q) - (fmaf(-q, scale, a) < 0 ? 1u : 0u));
}
// The card's rounding to 8 bits by random bits adds those of `random` from the top on to what is cut off, below the smallest normal values too (it was compared with an addition
// to the bits of a float for 2 million values in all of both formats' binades: equal).  16 random bits, and the middle of the interval that they leave: at most 8 (16) short of a step, so that the block's largest
// value, which the scale's rounding may leave 2 units in the last place above the format's, stays.
template <int TO>
__device__ __forceinline__ u32 put_first(float q, u32 random, u32 word) {
  return (u32)__builtin_amdgcn_cvt_sr_fp8_f32(q, (int)(random << 16 | 0x8000), (int)word, TO);
}
// (never zero for what is not)
template <int TO>
__device__ __forceinline__ u32 put_second(float q, float v, u32 random, u32 word) {
  return (u32)__builtin_amdgcn_cvt_sr_bf8_f32(fmaxf(q, v > 0 ? SECOND_LEAST : 0.0f), (int)((random & 0xFFFF0000u) | 0x8000), (int)word, TO);
}

// The largest of 32 lanes' values, which are not negative: as whole numbers these have the same order, with NaN above all others.
template <int CTRL>
__device__ __forceinline__ u32 max_with(u32 v) { return max(v, (u32)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false)); }
__device__ __forceinline__ u32 half_max(u32 v) {
  v = max_with<0x128>(max_with<0x124>(max_with<0x122>(max_with<0x121>(v))));      // row_ror: 1, 2, 4, 8
  return max(v, (u32)__shfl_xor((int)v, 16, 32));
}
__device__ __forceinline__ float scale_of(u32 largest, float most) { return fmaxf(__builtin_bit_cast(float, largest), 0x1p-80f) * (1.0f / most); }

// each operation rounded by itself, as a program that takes them one after another has them: 8-bit values next to one of the random borders then go the same way
__device__ __forceinline__ void next_moments(float& m, float& v, float g, const AdamwJob& j) {
#pragma clang fp contract(off)
  m = j.b1 * m + j.c1 * g;
  v = j.b2 * v + j.c2 * g * g;
}

template <class T, class G, int BITS, bool MASTERS>
__global__ __launch_bounds__(ADAMW_THREADS) void k_adamw(AdamwJob j) {
  constexpr int EACH = each_of(BITS), CHUNK = chunk_of(BITS), PASSES = CHUNK / (ADAMW_THREADS * EACH);
  // the last tensor that starts at or before this workgroup
  int mine = -1;
  for (int i = 0; i < j.n_tensors; i += CCLD_WAVE) {
    const int at = i + (int)lane_id();
    mine += __builtin_popcountll(ballot64(at < j.n_tensors && j.tensors[at < j.n_tensors ? at : 0].chunk0 <= blockIdx.x));
  }
  const Tensor x = j.tensors[__builtin_amdgcn_readfirstlane(mine)];
  const Step s = *j.step;
  const i64 chunk = (i64)(blockIdx.x - x.chunk0) * CHUNK, padded = (x.n + BLOCK - 1) / BLOCK * BLOCK, start = (i64)x.start * BLOCK;
#pragma unroll
  for (int pass = 0; pass < PASSES; ++pass) {
    // (whole blocks: 32 lanes are in or out together)
    const i64 at = chunk + (i64)pass * (ADAMW_THREADS * EACH) + threadIdx.x * EACH;
    if (at >= padded) break;
    const i64 state = start + at;
    float g[EACH], p[EACH], m[EACH], v[EACH];
    T* const to = static_cast<T*>(x.p) + at;
    const G* const from = static_cast<const G*>(x.g) + at;
    const bool whole = at + EACH <= x.n;
    if (whole) {
      const Vec<G, EACH> q = load_once<EACH>(from);
#pragma unroll
      for (int i = 0; i < EACH; ++i) g[i] = s.scale * (float)q[i];
    } else {
#pragma unroll
      for (int i = 0; i < EACH; ++i) g[i] = at + i < x.n ? s.scale * (float)from[i] : 0.0f;
    }
    if constexpr (MASTERS) {
      const Vec<float, EACH> q = load_once<EACH>(j.master + state);
#pragma unroll
      for (int i = 0; i < EACH; ++i) p[i] = q[i];
    } else if (whole) {
      const Vec<T, EACH> q = load_once<EACH>(to);
#pragma unroll
      for (int i = 0; i < EACH; ++i) p[i] = (float)q[i];
    } else {
#pragma unroll
      for (int i = 0; i < EACH; ++i) p[i] = at + i < x.n ? (float)to[i] : 0.0f;
    }
    const i64 block = state / BLOCK;
    if constexpr (BITS == 32) {
      const Vec<float, EACH> qm = load_once<EACH>(static_cast<const float*>(j.m) + state), qv = load_once<EACH>(static_cast<const float*>(j.v) + state);
#pragma unroll
      for (int i = 0; i < EACH; ++i) { m[i] = qm[i]; v[i] = qv[i]; }
    } else {
      const float sm = j.m_scale[block], sv = j.v_scale[block];
      const Words qm = __builtin_nontemporal_load(reinterpret_cast<const Words*>(static_cast<const uint8_t*>(j.m) + state)),
                  qv = __builtin_nontemporal_load(reinterpret_cast<const Words*>(static_cast<const uint8_t*>(j.v) + state));
#pragma unroll
      for (int i = 0; i < EACH; i += 4) {
        const auto m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)qm[i / 4], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)qm[i / 4], true);
        const auto v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)qv[i / 4], false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)qv[i / 4], true);
        m[i] = sm * m0[0]; m[i + 1] = sm * m0[1]; m[i + 2] = sm * m1[0]; m[i + 3] = sm * m1[1];
        v[i] = sv * v0[0]; v[i + 1] = sv * v0[1]; v[i + 2] = sv * v1[0]; v[i + 3] = sv * v1[1];
      }
    }
    float most_m = 0;
    u32 most_v = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      next_moments(m[i], v[i], g[i], j);
      if constexpr (BITS == 8) {
        most_m = fmaxf(most_m, fabsf(m[i]));
        most_v = max(most_v, __builtin_bit_cast(u32, v[i]));
      }
    }
    auto step_by = [&](auto root, auto over) {
#pragma unroll
      for (int i = 0; i < EACH; ++i) p[i] = p[i] - s.decay * p[i] - s.step_size * over(m[i], fmaf(root(v[i]), s.root, j.eps));
    };
    // The card's square root and reciprocal, off by a step each, take subnormal numbers for zero and give none: where those count, what is next to them is moved up for the root, and
    // quotients are divisions.
    auto root = [](float x) { return __builtin_amdgcn_sqrtf(x); };
    auto over = [](float x, float by) { return x * __builtin_amdgcn_rcpf(by); };
    if (j.far_eps) step_by([](float x) { return sqrtf(x); }, [](float x, float by) { return x / by; });
    else if (j.small_eps) step_by([&](float x) {
      const bool low = x < 0x1p-96f;
      return root(x * (low ? 0x1p32f : 1.0f)) * (low ? 0x1p-16f : 1.0f);
    }, over);
    else step_by(root, over);
    if constexpr (MASTERS) {
      // (behind the last element: zeros stay)
      Vec<float, EACH> q;
#pragma unroll
      for (int i = 0; i < EACH; ++i) q[i] = at + i < x.n ? p[i] : 0.0f;
      store_once<EACH>(j.master + state, q);
    }
    if (whole) {
      Vec<T, EACH> q;
#pragma unroll
      for (int i = 0; i < EACH; ++i) q[i] = (T)p[i];
      store_once<EACH>(to, q);
    } else {
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (at + i < x.n) to[i] = (T)p[i];
    }
    if constexpr (BITS == 32) {
      Vec<float, EACH> qm, qv;
#pragma unroll
      for (int i = 0; i < EACH; ++i) { qm[i] = m[i]; qv[i] = v[i]; }
      store_once<EACH>(static_cast<float*>(j.m) + state, qm);
      store_once<EACH>(static_cast<float*>(j.v) + state, qv);
    } else {
      // a gradient that is not finite leaves a v that is not, which is larger as a whole number than all that are (m's largest may hide one): NaN for the block
      const u32 largest = half_max(most_v);
      const bool finite = largest < 0x7F800000u;
      const float sm = finite ? scale_of(half_max(__builtin_bit_cast(u32, most_m)), FIRST_MOST) : __builtin_nanf("");
      const float sv = finite ? scale_of(largest, SECOND_MOST) : __builtin_nanf("");
      const float im = 1.0f / sm, iv = 1.0f / sv;
      const u32 key = mix(s.key ^ (u32)((u64)state >> 32));
      u32 r[EACH];
#pragma unroll
      for (int i = 0; i < EACH; ++i) r[i] = mix(key + (u32)state + i);
      Words qm, qv;
#pragma unroll
      for (int i = 0; i < EACH; i += 4) {
        auto first = [&](int n) { return copysignf(quotient(m[i + n], sm, im), m[i + n]); };
        auto second = [&](int n) { return quotient(v[i + n], sv, iv); };
        qm[i / 4] = put_first<3>(first(3), r[i + 3], put_first<2>(first(2), r[i + 2], put_first<1>(first(1), r[i + 1], put_first<0>(first(0), r[i], 0))));
        qv[i / 4] = put_second<3>(second(3), v[i + 3], r[i + 3], put_second<2>(second(2), v[i + 2], r[i + 2], put_second<1>(second(1), v[i + 1], r[i + 1],
                                  put_second<0>(second(0), v[i], r[i], 0))));
      }
      __builtin_nontemporal_store(qm, reinterpret_cast<Words*>(static_cast<uint8_t*>(j.m) + state));
      __builtin_nontemporal_store(qv, reinterpret_cast<Words*>(static_cast<uint8_t*>(j.v) + state));
      if (threadIdx.x % (BLOCK / EACH) == 0) {
        j.m_scale[block] = sm;
        j.v_scale[block] = sv;
      }
    }
  }
}

template <class T, class G>
void launch(const AdamwJob& j, u32 groups, int bits, hipStream_t stream) {
  const bool masters = j.master != nullptr;
  if constexpr (sizeof(T) == 2) {
    if (masters) {
      if (bits == 32) k_adamw<T, G, 32, true><<<groups, ADAMW_THREADS, 0, stream>>>(j);
      else k_adamw<T, G, 8, true><<<groups, ADAMW_THREADS, 0, stream>>>(j);
      return;
    }
  }
  if (bits == 32) k_adamw<T, G, 32, false><<<groups, ADAMW_THREADS, 0, stream>>>(j);
  else k_adamw<T, G, 8, false><<<groups, ADAMW_THREADS, 0, stream>>>(j);
}

ccld_status check(const ccld_adamw_args* a) {
  if (!a) return CCLD_E_NULL;
  if (!known_type(a->dtype) || (a->grad_dtype != a->dtype && a->grad_dtype != CCLD_FP32) || (a->bits != 8 && a->bits != 32)) return CCLD_E_BAD_ARG;
  if (!isfinite(a->lr) || !isfinite(a->weight_decay) || !isfinite(a->scale) || !(a->eps >= 0) || !isfinite(a->eps)) return CCLD_E_BAD_ARG;
  if (!(a->beta1 >= 0 && a->beta1 < 1 && a->beta2 >= 0 && a->beta2 < 1)) return CCLD_E_BAD_ARG;
  if (a->n_tensors < 0 || a->total < 0 || a->total % BLOCK || (a->master && a->dtype == CCLD_FP32)) return CCLD_E_BAD_ARG;
  if (a->total / BLOCK >= (i64)1 << 32) return CCLD_E_CAPACITY;
  if (!a->count || (a->n_tensors && !a->tensors) || (a->total && (!a->m || !a->v || (a->bits == 8 && (!a->m_scale || !a->v_scale))))) return CCLD_E_NULL;
  if (!aligned(a->count, 8) || !aligned(a->m, 4) || !aligned(a->v, 4) || !aligned(a->m_scale, 4) || !aligned(a->v_scale, 4) || !aligned(a->master, 4) ||
      !aligned(a->scale_by, 4)) return CCLD_E_BAD_ARG;
  if (a->workspace_bytes < CCLD_ADAMW_WORKSPACE || !a->workspace || !aligned(a->workspace, 256)) return CCLD_E_WORKSPACE;
  for (i64 i = 0; i < a->n_tensors; ++i) {
    const ccld_adamw_tensor& t = a->tensors[i];
    if (t.n < 0 || t.start < 0 || t.start % BLOCK || t.start > a->total || t.n > a->total - t.start) return CCLD_E_BAD_ARG;
    if (t.n && (!t.p || !t.g)) return CCLD_E_NULL;
    if (!aligned(t.p, size_of(a->dtype)) || !aligned(t.g, size_of(a->grad_dtype))) return CCLD_E_BAD_ARG;
  }
  return CCLD_OK;
}

}  // namespace

extern "C" ccld_status ccld_adamw(const ccld_adamw_args* a, void* stream) {
  const ccld_status st = check(a);
  if (st != CCLD_OK) return st;
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  Step* const step = static_cast<Step*>(a->workspace);
  k_adamw_begin<<<1, 1, 0, hs>>>(BeginJob{a->count, a->scale_by, step, a->lr, a->beta1, a->beta2, a->weight_decay, a->scale, a->seed});
  AdamwJob j{};
  j.step = step;
  j.m = a->m; j.v = a->v; j.m_scale = a->m_scale; j.v_scale = a->v_scale; j.master = a->master;
  j.b1 = (float)a->beta1; j.b2 = (float)a->beta2; j.c1 = (float)(1.0 - a->beta1); j.c2 = (float)(1.0 - a->beta2); j.eps = (float)a->eps;
  // an eps that 32 bits do not have is still no zero: what never had a gradient stays where it is
  if (a->eps > 0) j.eps = std::max(j.eps, 0x1p-149f);
  // What stands beside eps is the root over sqrt(1 - b2^t), at least sqrt(1 - b2): of a subnormal v up to 2^-63 / sqrt(1 - b2).  From here on that is at most a 2^-25th of eps.
  j.small_eps = a->eps * sqrt(1.0 - a->beta2) < 0x1p-38;
  // (the root of the smallest v is 2^-74.5, of the largest over sqrt(1 - b2) below 2^91: by themselves these have reciprocals)
  j.far_eps = (a->eps > 0 && a->eps < 0x1p-126) || a->eps > 0x1p125;
  u32 groups = 0;
  auto flush = [&] {
    if (!groups) return;
    if (a->dtype == CCLD_FP32) launch<float, float>(j, groups, a->bits, hs);
    else if (a->dtype == CCLD_BF16) a->grad_dtype == CCLD_FP32 ? launch<__bf16, float>(j, groups, a->bits, hs) : launch<__bf16, __bf16>(j, groups, a->bits, hs);
    else a->grad_dtype == CCLD_FP32 ? launch<_Float16, float>(j, groups, a->bits, hs) : launch<_Float16, _Float16>(j, groups, a->bits, hs);
    groups = 0;
    j.n_tensors = 0;
  };
  const i64 most = most_groups(ADAMW_THREADS), chunk = chunk_of(a->bits);
  for (i64 i = 0; i < a->n_tensors; ++i) {
    const ccld_adamw_tensor& t = a->tensors[i];
    // (a tensor that is too long for a launch is taken in pieces)
    for (i64 done = 0; done < t.n;) {
      if (j.n_tensors == LISTED || groups == (u32)most) flush();
      const i64 n = std::min(t.n - done, (most - groups) * chunk);
      j.tensors[j.n_tensors++] = Tensor{static_cast<uint8_t*>(t.p) + done * size_of(a->dtype), static_cast<const uint8_t*>(t.g) + done * size_of(a->grad_dtype), n,
                                        (u32)((t.start + done) / BLOCK), groups};
      groups += (u32)blocks_for(n, chunk);
      done += n;
    }
  }
  flush();
  return launched();
}
