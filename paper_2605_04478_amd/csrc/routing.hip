// The choice of every token's experts, its gradient, and the order of the chosen entries by expert (ccld_route*, ccld_expert_order).
//
//   chosen: the k largest of a row, equal ones by the lower expert      w_j = exp(s_j - m) / sum exp(s - m), over the chosen or over all
//   ds[e_j] = w_j dw_j (of each chosen one)  -  p_e sum_j w_j dw_j      p: the same softmax
//   place[n] = entries of lower experts + earlier entries of the same expert: a stable counting sort
//
// A row of scores belongs to one wavefront and stays in its registers: lane l holds the experts from l V on, so that the lowest
// lane with the largest value has the lowest expert.  A choice is a maximum over the lanes, a ballot and its removal.
#include <algorithm>

#include "ccld_internal.h"
#include "operators.h"

using namespace ccld;

namespace {

struct RouteJob {
  const void* scores;
  int32_t* experts;
  float* weights;
  const float* dweights;
  void* dscores;
  i64 ld, ldd, tokens;
  int n, k, over_all;
};

constexpr int ROUTE_THREADS = 256, ROUTE_TOKENS = ROUTE_THREADS / CCLD_WAVE;

// scores that cannot be chosen (switched off, NaN, behind the last expert) are the lowest value
template <int V, class T>
__device__ __forceinline__ void load_scores(float (&z)[V], const T* row, int lane, int n) {
  const int first = lane * V;
  if (first + V <= n) {
    const Vec<T, V> v = load_vec<V>(row + first);
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = (float)v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = first + i < n ? (float)row[first + i] : LOWEST;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) z[i] = z[i] != z[i] ? LOWEST : z[i];
}
template <int V>
__device__ __forceinline__ float largest_of(const float (&z)[V]) {
  float m = z[0];
#pragma unroll
  for (int i = 1; i < V; ++i) m = fmaxf(m, z[i]);
  return m;
}
// (the largest counts one also where it is infinite)
__device__ __forceinline__ float share(float z, float m) { return z == m ? 1.0f : expf(z - m); }

template <class T, int V>
__global__ __launch_bounds__(ROUTE_THREADS) void k_route(RouteJob j) {
  const int lane = (int)lane_id();
  const i64 first = (i64)blockIdx.x * ROUTE_TOKENS + __builtin_amdgcn_readfirstlane(threadIdx.x / CCLD_WAVE);
  for (i64 t = first; t < j.tokens; t += (i64)gridDim.x * ROUTE_TOKENS) {
    float z[V];
    load_scores<V>(z, static_cast<const T*>(j.scores) + t * j.ld, lane, j.n);
    float total = 0, m0 = LOWEST, value = LOWEST;
    int mine = -1;
    for (int c = 0; c < j.k; ++c) {
      const float best = largest_of(z), m = wave_max(best);
      if (m == LOWEST) break;
      if (c == 0) {
        m0 = m;
        if (j.over_all) {
          float e = 0;
#pragma unroll
          for (int i = 0; i < V; ++i) e += share(z[i], m0);
          total = wave_total(e);
        }
      }
      const int who = (int)__builtin_ctzll(ballot64(best == m));
      int at = V;
#pragma unroll
      for (int i = V - 1; i >= 0; --i) at = z[i] == m ? i : at;
#pragma unroll
      for (int i = 0; i < V; ++i) z[i] = lane == who && i == at ? LOWEST : z[i];
      const int expert = who * V + __builtin_amdgcn_readlane(at, who);
      if (lane == c) { mine = expert; value = m; }
    }
    const float e = mine < 0 ? 0.0f : share(value, m0);
    if (!j.over_all) total = wave_total(e);
    if (lane < j.k) {
      j.experts[t * j.k + lane] = mine;
      j.weights[t * j.k + lane] = mine < 0 ? 0.0f : e / total;
    }
  }
}

template <class T, int V>
__global__ __launch_bounds__(ROUTE_THREADS) void k_route_grad(RouteJob j) {
  const int lane = (int)lane_id();
  const i64 first = (i64)blockIdx.x * ROUTE_TOKENS + __builtin_amdgcn_readfirstlane(threadIdx.x / CCLD_WAVE);
  for (i64 t = first; t < j.tokens; t += (i64)gridDim.x * ROUTE_TOKENS) {
    int expert = -1;
    float w = 0, each = 0;
    if (lane < j.k) {
      expert = j.experts[t * j.k + lane];
      if ((u32)expert < (u32)j.n) {
        w = j.weights[t * j.k + lane];
        each = w * j.dweights[t * j.k + lane];
      }
    }
    float d[V] = {};
    const float common = wave_total(each);
    if (j.over_all) {
      load_scores<V>(d, static_cast<const T*>(j.scores) + t * j.ld, lane, j.n);
      const float m = wave_max(largest_of(d));
      float sum = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        d[i] = m == LOWEST ? 0.0f : share(d[i], m);
        sum += d[i];
      }
      const float scale = m == LOWEST ? 0.0f : common / wave_total(sum);
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] *= -scale;
    } else {
      each -= common * w;
    }
    for (int c = 0; c < j.k; ++c) {
      const int e = __builtin_amdgcn_readlane(expert, c);
      if ((u32)e >= (u32)j.n) continue;
      const float more = read_lane(each, c);
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] = lane * V + i == e ? d[i] + more : d[i];
    }
    T* const row = static_cast<T*>(j.dscores) + t * j.ldd + lane * V;
    if (lane * V + V <= j.n) {
      Vec<T, V> v;
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = (T)d[i];
      store_vec<V>(row, v);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (lane * V + i < j.n) row[i] = (T)d[i];
    }
  }
}

template <bool GRAD, class T, int V>
void launch_route(const RouteJob& j, hipStream_t stream) {
  const u32 grid = (u32)std::min<i64>(blocks_for(j.tokens, ROUTE_TOKENS), 64 * COMPUTE_UNITS);
  if constexpr (GRAD) k_route_grad<T, V><<<grid, ROUTE_THREADS, 0, stream>>>(j);
  else k_route<T, V><<<grid, ROUTE_THREADS, 0, stream>>>(j);
}
template <bool GRAD>
ccld_status launch_route(const RouteJob& j, int32_t dtype, hipStream_t stream) {
  with_type(dtype, [&](auto zero) {
    using T = decltype(zero);
    if (j.n <= 64) launch_route<GRAD, T, 1>(j, stream);
    else if (j.n <= 128) launch_route<GRAD, T, 2>(j, stream);
    else if (j.n <= 256) launch_route<GRAD, T, 4>(j, stream);
    else if (j.n <= 512) launch_route<GRAD, T, 8>(j, stream);
    else launch_route<GRAD, T, 16>(j, stream);
  });
  return launched();
}

ccld_status check_route(const ccld_route_args* a, bool grad) {
  if (!a) return CCLD_E_NULL;
  if (!known_type(a->dtype) || a->tokens < 0 || a->n_experts < 1 || a->k < 1 || a->k > a->n_experts) return CCLD_E_BAD_ARG;
  if (a->tokens >= MAX_ROWS || a->n_experts > CCLD_ROUTE_EXPERTS || a->k > CCLD_ROUTE_MOST) return CCLD_E_CAPACITY;
  const bool reads = !grad || a->over_all;
  if (a->tokens && ((reads && !a->scores) || !a->experts || !a->weights || (grad && (!a->dweights || !a->dscores)))) return CCLD_E_NULL;
  if ((reads && a->ldscores < a->n_experts) || (grad && a->lddscores < a->n_experts)) return CCLD_E_BAD_ARG;
  if ((reads && !aligned(a->scores, size_of(a->dtype))) || !aligned(a->experts, 4) || !aligned(a->weights, 4)) return CCLD_E_BAD_ARG;
  if (grad && (!aligned(a->dweights, 4) || !aligned(a->dscores, size_of(a->dtype)))) return CCLD_E_BAD_ARG;
  return CCLD_OK;
}
RouteJob route_job(const ccld_route_args* a) {
  return RouteJob{a->scores, a->experts, a->weights, a->dweights, a->dscores, a->ldscores, a->lddscores, a->tokens, (int)a->n_experts, (int)a->k,
                  a->over_all != 0};
}

// ---- entries by expert ---------------------------------------------------------------------------------------------
// Chunks of entries, one to a workgroup, whose wavefronts take a stretch of it each.  Counts per chunk first (where there is more than one), then every workgroup
// finds what lies before its own entries of each expert, and a wavefront ranks 64 entries at a time: those of one expert are found by ballots over the bits
// of its number, the lowest of their lanes takes as many places from the wavefront's counter.
struct OrderJob {
  const void* experts;
  int32_t *places, *offsets;
  u32* counts;                   // [chunks][n]
  u32 entries, chunks, stretch;  // stretch: a wavefront's entries
  int n;
};
constexpr int ORDER_THREADS = 256;
constexpr u32 MOST_CHUNKS = 256, LEAST_STRETCH = 512, SINGLE_CHUNK = 8192;

template <class I>
__device__ __forceinline__ u32 expert_at(const OrderJob& j, u32 at, u32 end) {
  if (at >= end) return (u32)j.n;
  const I e = static_cast<const I*>(j.experts)[at];
  return e >= 0 && e < (I)j.n ? (u32)e : (u32)j.n;
}

template <class I>
__global__ __launch_bounds__(ORDER_THREADS) void k_order_count(OrderJob j) {
  __shared__ u32 counts[CCLD_ROUTE_EXPERTS];
  for (int e = threadIdx.x; e < j.n; e += ORDER_THREADS) counts[e] = 0;
  __syncthreads();
  const u64 chunk = (u64)j.stretch * (ORDER_THREADS / CCLD_WAVE), start = blockIdx.x * chunk;
  const u32 end = (u32)min((u64)j.entries, start + chunk);
  for (u64 at = start + threadIdx.x; at < end; at += ORDER_THREADS) {
    const u32 e = expert_at<I>(j, (u32)at, end);
    if (e < (u32)j.n) atomicAdd(&counts[e], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < j.n; e += ORDER_THREADS) j.counts[(u64)blockIdx.x * j.n + e] = counts[e];
}

template <class I, int THREADS>
__global__ __launch_bounds__(THREADS) void k_order_place(OrderJob j) {
  constexpr int WAVES = THREADS / CCLD_WAVE, EACH = CCLD_ROUTE_EXPERTS / THREADS;
  __shared__ u32 counter[WAVES][CCLD_ROUTE_EXPERTS], all[CCLD_ROUTE_EXPERTS], s_wave[WAVES];
  const u32 lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / CCLD_WAVE), n = j.n;
  const u64 start = ((u64)blockIdx.x * WAVES + wave) * j.stretch;
  const u32 end = (u32)min((u64)j.entries, start + j.stretch);
  for (int e = lane; e < n; e += CCLD_WAVE) counter[wave][e] = 0;
  for (u64 at = start + lane; at < end; at += CCLD_WAVE) {
    const u32 e = expert_at<I>(j, (u32)at, end);
    if (e < (u32)n) atomicAdd(&counter[wave][e], 1u);
  }
  __syncthreads();
  // what lies before this chunk's entries of an expert, and how many there are in all
  for (int e = threadIdx.x; e < n; e += THREADS) {
    u32 before = 0, sum = 0;
    if (j.chunks == 1) {
      for (int w = 0; w < WAVES; ++w) sum += counter[w][e];
    } else {
#pragma unroll 8
      for (u32 c = 0; c < j.chunks; ++c) {
        const u32 x = j.counts[(u64)c * n + e];
        sum += x;
        before += c < blockIdx.x ? x : 0;
      }
    }
    all[e] = sum;
    for (int w = 0; w < WAVES; ++w) {
      const u32 x = counter[w][e];
      counter[w][e] = before;
      before += x;
    }
  }
  __syncthreads();
  u32 own[EACH], sum = 0, total;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int e = threadIdx.x * EACH + i;
    own[i] = e < n ? all[e] : 0;
    sum += own[i];
  }
  u32 base = block_exclusive_sum<THREADS>(sum, s_wave, &total);
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int e = threadIdx.x * EACH + i;
    if (e < n) {
      all[e] = base;
      if (blockIdx.x == 0) j.offsets[e] = (int32_t)base;
    }
    base += own[i];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) j.offsets[n] = (int32_t)total;
  __syncthreads();
  const int bits = 32 - __builtin_clz((u32)n);
  for (u64 at0 = start; at0 < end; at0 += CCLD_WAVE) {
    const u64 at = at0 + lane;
    const u32 e = at < end ? expert_at<I>(j, (u32)at, end) : (u32)n;
    u64 same = ~0ull;
    for (int b = 0; b < bits; ++b) {
      const bool set = e >> b & 1;
      const u64 m = ballot64(set);
      same &= set ? m : ~m;
    }
    const u32 rank = mbcnt64(same);
    u32 taken = 0;
    if (rank == 0 && e < (u32)n) taken = atomicAdd(&counter[wave][e], (u32)__builtin_popcountll(same));
    taken = lane_read(taken, (u32)__builtin_ctzll(same));
    if (at < end) j.places[at] = e < (u32)n ? (int32_t)(all[e] + taken + rank) : -1;
  }
}

OrderJob order_job(const ccld_order_args* a, uint64_t* bytes) {
  OrderJob j{a->experts, a->places, a->offsets, static_cast<u32*>(a->workspace), (u32)(a->tokens * a->k), 1, 0, (int)a->n_experts};
  if (j.entries <= SINGLE_CHUNK) {
    j.stretch = (u32)blocks_for(std::max<u32>(j.entries, 1), 1024) * CCLD_WAVE;
    *bytes = 0;
  } else {
    const u64 waves = MOST_CHUNKS * (ORDER_THREADS / CCLD_WAVE);
    j.stretch = std::max<u32>(LEAST_STRETCH, (u32)((((u64)j.entries + waves - 1) / waves + CCLD_WAVE - 1) / CCLD_WAVE * CCLD_WAVE));
    j.chunks = (u32)blocks_for(j.entries, (i64)j.stretch * (ORDER_THREADS / CCLD_WAVE));
    *bytes = (uint64_t)j.chunks * (uint64_t)a->n_experts * 4;
  }
  return j;
}
template <class I>
void launch_order(const OrderJob& j, hipStream_t stream) {
  if (j.chunks == 1) {
    k_order_place<I, 1024><<<1, 1024, 0, stream>>>(j);
  } else {
    k_order_count<I><<<j.chunks, ORDER_THREADS, 0, stream>>>(j);
    k_order_place<I, ORDER_THREADS><<<j.chunks, ORDER_THREADS, 0, stream>>>(j);
  }
}

ccld_status check_order(const ccld_order_args* a) {
  if (!a) return CCLD_E_NULL;
  if ((a->expert_bits != 32 && a->expert_bits != 64) || a->tokens < 0 || a->k < 1 || a->n_experts < 1) return CCLD_E_BAD_ARG;
  if (a->tokens >= MAX_ROWS || a->k >= MAX_ROWS || a->tokens * a->k >= MAX_ROWS || a->n_experts > CCLD_ROUTE_EXPERTS) return CCLD_E_CAPACITY;
  return CCLD_OK;
}

}  // namespace

extern "C" ccld_status ccld_route(const ccld_route_args* a, void* stream) {
  const ccld_status s = check_route(a, false);
  if (s != CCLD_OK || a->tokens == 0) return s;
  return launch_route<false>(route_job(a), a->dtype, static_cast<hipStream_t>(stream));
}
extern "C" ccld_status ccld_route_grad(const ccld_route_args* a, void* stream) {
  const ccld_status s = check_route(a, true);
  if (s != CCLD_OK || a->tokens == 0) return s;
  return launch_route<true>(route_job(a), a->dtype, static_cast<hipStream_t>(stream));
}

extern "C" ccld_status ccld_order_workspace(const ccld_order_args* a, uint64_t* bytes) {
  if (!bytes) return CCLD_E_NULL;
  const ccld_status s = check_order(a);
  if (s == CCLD_OK) order_job(a, bytes);
  return s;
}
extern "C" ccld_status ccld_expert_order(const ccld_order_args* a, void* stream) {
  const ccld_status s = check_order(a);
  if (s != CCLD_OK) return s;
  if (!a->offsets || (a->tokens && (!a->experts || !a->places))) return CCLD_E_NULL;
  if (!aligned(a->experts, a->expert_bits / 8) || !aligned(a->places, 4) || !aligned(a->offsets, 4)) return CCLD_E_BAD_ARG;
  uint64_t need;
  const OrderJob j = order_job(a, &need);
  if (need && (need > a->workspace_bytes || !a->workspace || !aligned(a->workspace, 256))) return CCLD_E_WORKSPACE;
  if (a->expert_bits == 32) launch_order<int32_t>(j, static_cast<hipStream_t>(stream));
  else launch_order<int64_t>(j, static_cast<hipStream_t>(stream));
  return launched();
}
