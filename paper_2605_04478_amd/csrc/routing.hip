// The choice of every token's experts, its gradient, and the order of the chosen entries by expert (ccld_route*, ccld_expert_order).
//
//   chosen: the k largest of a row, equal ones by the lower expert      w_j = exp(s_j - m) / sum exp(s - m), over the chosen or over all
//   ds[e_j] = w_j dw_j (of each chosen one)  -  p_e sum_j w_j dw_j      p: the same softmax
//   place[n] = entries of lower experts + earlier entries of the same expert: a stable counting sort
//
// The choice is bound by its instructions, not by memory: k times a maximum over a row and its removal.  A row therefore belongs to as few lanes as hold it in 16 registers
// each, 16 lanes for up to 256 experts, so that a wavefront's instructions serve four tokens; maxima over 16 lanes take four instructions.
//
// Measured (a copy of 2 GB moves 4.9 TB/s here, x + 1 6.1): 65,536 x 256 in 32 bits, 8 experts, weights over all: 34 us (57 with a wavefront to a token; the scores are 67 MB, 14 us), of which the 1,241 instructions to four tokens
// take 33; gradient 24 us = 5.5 TB/s.  In bfloat16 31 and 18, over the chosen 27 and 10 (8 us of bytes each way); 32,768 x 512 with 16 in 32 bits 51 and 24, in bfloat16 49 and 19.  7 tokens: 3 us of a call's 5.  262,144 entries of 128 experts in order: 3 + 3 + 5 us; 16,384 of 8: 2.5 + 4.5; 20: 3.3.
#include <algorithm>
#include <type_traits>

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

constexpr int ROUTE_THREADS = 256;

// A token's scores in L lanes, V to each, in pieces of up to 4 neighbours: index(i) is the expert of value i.
template <int L, int V>
struct Scores {
  static constexpr int P = V < 4 ? V : 4;
  float z[V];
  static __device__ __forceinline__ int index(int lane, int i) { return (i / P * L + lane) * P + i % P; }
  // scores that cannot be chosen (switched off, NaN, behind the last expert) are the lowest value
  template <class T>
  __device__ __forceinline__ Scores(const T* row, int lane, int n, bool there) {
#pragma unroll
    for (int i = 0; i < V; i += P) {
      const int first = index(lane, i);
      if (there && first + P <= n) {
        const Vec<T, P> v = load_vec<P>(row + first);
#pragma unroll
        for (int p = 0; p < P; ++p) z[i + p] = (float)v[p];
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) z[i + p] = there && first + p < n ? (float)row[first + p] : LOWEST;
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = z[i] != z[i] ? LOWEST : z[i];
  }
  __device__ __forceinline__ float largest() const {
    float m = z[0];
#pragma unroll
    for (int i = 1; i < V; ++i) m = fmaxf(m, z[i]);
    return m;
  }
};

// Over the L lanes of a token, in all of them: pairs, fours, eights and so on exchange what they have, so that every lane adds the same two numbers and all have the same bits.
template <int L, class T, class F>
__device__ __forceinline__ T over_lanes(T v, F f) {
  auto with = [&](auto ctrl) {
    const int x = __builtin_bit_cast(int, v);
    v = f(v, __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xF, 0xF, false)));
  };
  with(std::integral_constant<int, 0xB1>());           // quad_perm: 1, 0, 3, 2
  with(std::integral_constant<int, 0x4E>());           // quad_perm: 2, 3, 0, 1
  with(std::integral_constant<int, 0x141>());          // row_half_mirror: 7 - i of eight
  with(std::integral_constant<int, 0x140>());          // row_mirror: 15 - i
  if constexpr (L > 16) v = f(v, __shfl_xor(v, 16, CCLD_WAVE));
  if constexpr (L > 32) v = f(v, __shfl_xor(v, 32, CCLD_WAVE));
  return v;
}
template <int L>
__device__ __forceinline__ float max_over(float v) { return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int L>
__device__ __forceinline__ float sum_over(float v) { return over_lanes<L>(v, [](float a, float b) { return a + b; }); }
template <int L>
__device__ __forceinline__ int min_over(int v) { return over_lanes<L>(v, [](int a, int b) { return a < b ? a : b; }); }

// exp(z - m) by the card's power of two, whose argument's rounding is made good; the largest counts one also where it is infinite
__device__ __forceinline__ float share(float z, float m) {
  const float d = z - m, t = d * 0x1.715476p+0f, r = fmaf(d, 0x1.715476p+0f, -t) + d * 0x1.4ae0c0p-26f;
  const float e = __builtin_amdgcn_exp2f(t);
  return z == m ? 1.0f : d < -150.0f ? 0.0f : fmaf(e, r * 0x1.62e430p-1f, e);
}

template <class T, int L, int V>
__global__ __launch_bounds__(ROUTE_THREADS) void k_route(RouteJob j) {
  constexpr int TOKENS = ROUTE_THREADS / L;
  struct Pick { float value; int expert; };
  __shared__ Pick picks[TOKENS][CCLD_ROUTE_MOST];
  const int lane = threadIdx.x % L, mine = threadIdx.x / L;
  for (i64 t0 = (i64)blockIdx.x * TOKENS; t0 < j.tokens; t0 += (i64)gridDim.x * TOKENS) {
    const i64 t = t0 + mine;
    const bool there = t < j.tokens;                   // (lanes without a token go along)
    Scores<L, V> s(static_cast<const T*>(j.scores) + t * j.ld, lane, j.n, there);
    float total = 0, m0 = LOWEST;
    for (int c = 0; c < j.k; ++c) {
      const float m = max_over<L>(s.largest());
      if (c == 0) {
        m0 = m;
        if (j.over_all) {
          float e = 0;
#pragma unroll
          for (int i = 0; i < V; ++i) e += s.z[i] == LOWEST ? 0.0f : share(s.z[i], m0);
          total = sum_over<L>(e);
        }
      }
      // the lowest expert with this score, and its removal
      int at = 0x7FFFFFFF;
#pragma unroll
      for (int i = V - 1; i >= 0; --i) at = s.z[i] == m ? s.index(lane, i) : at;
      const int expert = min_over<L>(at);
#pragma unroll
      for (int i = 0; i < V; ++i) s.z[i] = s.index(lane, i) == expert ? LOWEST : s.z[i];
      if (lane == 0) picks[mine][c] = Pick{m, m == LOWEST ? -1 : expert};
    }
    // (a token's lanes are of one wavefront, whose accesses to LDS are in order)
    __builtin_amdgcn_wave_barrier();
    float sum = 0;
    for (int c = lane; c < j.k; c += L) {
      const Pick p = picks[mine][c];
      sum += p.expert < 0 ? 0.0f : share(p.value, m0);
    }
    if (!j.over_all) total = sum_over<L>(sum);
    for (int c = lane; there && c < j.k; c += L) {
      const Pick p = picks[mine][c];
      j.experts[t * j.k + c] = p.expert;
      j.weights[t * j.k + c] = p.expert < 0 ? 0.0f : share(p.value, m0) / total;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The same lanes.  What is added at a token's choices goes through a row of LDS, which its lanes read beside one another and clear again.  (A wavefront to a token that
// compared each choice with its own experts took 34 us for 65,536 x 256 in 32 bits over all experts, this 24.)
template <class T, int L, int V>
__global__ __launch_bounds__(ROUTE_THREADS) void k_route_grad(RouteJob j) {
  constexpr int TOKENS = ROUTE_THREADS / L;
  typedef Scores<L, V> S;
  constexpr int P = S::P;
  __shared__ float rows[TOKENS][L * V];
  const int lane = threadIdx.x % L, mine = threadIdx.x / L;
  for (int i = lane; i < L * V; i += L) rows[mine][i] = 0;
  for (i64 t0 = (i64)blockIdx.x * TOKENS; t0 < j.tokens; t0 += (i64)gridDim.x * TOKENS) {
    const i64 t = t0 + mine;
    const bool there = t < j.tokens;                   // (lanes without a token go along)
    float sum = 0, p[V];
    for (int c = lane; there && c < j.k; c += L) {
      const int e = j.experts[t * j.k + c];
      if ((u32)e < (u32)j.n) sum += j.weights[t * j.k + c] * j.dweights[t * j.k + c];
    }
    const float common = sum_over<L>(sum);
    if (j.over_all) {
      const S s(static_cast<const T*>(j.scores) + t * j.ld, lane, j.n, there);
      const float m = max_over<L>(s.largest());
      float all = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        p[i] = s.z[i] == LOWEST ? 0.0f : share(s.z[i], m);
        all += p[i];
      }
      const float scale = m == LOWEST ? 0.0f : common / sum_over<L>(all);
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] *= -scale;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = 0;
    }
    // (a token's lanes are of one wavefront, whose accesses to LDS are in order; an expert that stands twice in a row counts twice)
    for (int c = lane; there && c < j.k; c += L) {
      const int e = j.experts[t * j.k + c];
      if ((u32)e >= (u32)j.n) continue;
      const float w = j.weights[t * j.k + c], each = w * j.dweights[t * j.k + c];
      atomicAdd(&rows[mine][e], j.over_all ? each : each - common * w);
    }
    __builtin_amdgcn_wave_barrier();
    T* const row = static_cast<T*>(j.dscores) + t * j.ldd;
#pragma unroll
    for (int i = 0; i < V; i += P) {
      const int at = S::index(lane, i);
      Vec<T, P> v;
#pragma unroll
      for (int q = 0; q < P; ++q) {
        v[q] = (T)(p[i + q] + rows[mine][at + q]);
        rows[mine][at + q] = 0;
      }
      if (there && at + P <= j.n) store_once<P>(row + at, v);
      else
#pragma unroll
        for (int q = 0; q < P; ++q)
          if (there && at + q < j.n) row[at + q] = v[q];
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <bool GRAD, class T, int L, int V>
void launch_lanes(const RouteJob& j, hipStream_t stream) {
  const u32 grid = (u32)std::min<i64>(blocks_for(j.tokens, ROUTE_THREADS / L), 64 * COMPUTE_UNITS);
  if constexpr (GRAD) k_route_grad<T, L, V><<<grid, ROUTE_THREADS, 0, stream>>>(j);
  else k_route<T, L, V><<<grid, ROUTE_THREADS, 0, stream>>>(j);
}
template <bool GRAD>
ccld_status launch_route(const RouteJob& j, int32_t dtype, hipStream_t stream) {
  with_type(dtype, [&](auto zero) {
    using T = decltype(zero);
    if (j.n <= 16) launch_lanes<GRAD, T, 16, 1>(j, stream);
    else if (j.n <= 64) launch_lanes<GRAD, T, 16, 4>(j, stream);
    else if (j.n <= 128) launch_lanes<GRAD, T, 16, 8>(j, stream);
    else if (j.n <= 256) launch_lanes<GRAD, T, 16, 16>(j, stream);
    else if (j.n <= 512) launch_lanes<GRAD, T, 32, 16>(j, stream);
    else launch_lanes<GRAD, T, 64, 16>(j, stream);
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
// finds what lies before its own entries of each expert, from all chunks' counts or, where there are many, from a scan of them, and a wavefront ranks 64 entries at a time: those of one expert are found by ballots over the bits
// of its number, the lowest of their lanes takes as many places from the wavefront's counter.
struct OrderJob {
  const void* experts;
  int32_t *places, *offsets;
  u32 *counts, *totals;          // [chunks][n]; [n], where counts are turned into what lies before
  u32 entries, chunks, stretch;  // stretch: a wavefront's entries
  int n;
};
constexpr int ORDER_THREADS = 256;
// Stretches of 256 entries, all of which are on their way at once; longer ones where there would be more than 256 chunks.
constexpr int AT_ONCE = 4;
constexpr u32 MOST_CHUNKS = 256, LEAST_STRETCH = AT_ONCE * CCLD_WAVE, SINGLE_CHUNK = 16 * LEAST_STRETCH;
constexpr u32 FEW_ENTRIES = 4 * LEAST_STRETCH;          // one workgroup of four wavefronts, up to SINGLE_CHUNK one of sixteen

// the experts of a wavefront's next entries, n for those that have none
template <class I>
__device__ __forceinline__ void next_experts(const OrderJob& j, u64 at0, u32 end, u32 (&e)[AT_ONCE]) {
#pragma unroll
  for (int i = 0; i < AT_ONCE; ++i) {
    const u64 at = at0 + i * CCLD_WAVE + lane_id();
    I x = -1;
    if (at < end) x = static_cast<const I*>(j.experts)[at];
    e[i] = x >= 0 && x < (I)j.n ? (u32)x : (u32)j.n;
  }
}

template <class I>
__global__ __launch_bounds__(ORDER_THREADS) void k_order_count(OrderJob j) {
  __shared__ u32 counts[CCLD_ROUTE_EXPERTS];
  for (int e = threadIdx.x; e < j.n; e += ORDER_THREADS) counts[e] = 0;
  __syncthreads();
  const u64 start = ((u64)blockIdx.x * (ORDER_THREADS / CCLD_WAVE) + threadIdx.x / CCLD_WAVE) * j.stretch;
  const u32 end = (u32)min((u64)j.entries, start + j.stretch);
  for (u64 at = start; at < end; at += LEAST_STRETCH) {
    u32 e[AT_ONCE];
    next_experts<I>(j, at, end, e);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
      if (e[i] < (u32)j.n) atomicAdd(&counts[e[i]], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < j.n; e += ORDER_THREADS) j.counts[(u64)blockIdx.x * j.n + e] = counts[e];
}

// Where there are many chunks: each expert's counts become what lies before them, by one wavefront.
constexpr u32 MANY_CHUNKS = 32;
__global__ __launch_bounds__(ORDER_THREADS) void k_order_scan(OrderJob j) {
  constexpr int EACH = MOST_CHUNKS / CCLD_WAVE;
  const int e = blockIdx.x * (ORDER_THREADS / CCLD_WAVE) + threadIdx.x / CCLD_WAVE;
  if (e >= j.n) return;
  const u32 first = lane_id() * EACH;
  u32 x[EACH], sum = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) x[i] = first + i < j.chunks ? j.counts[(u64)(first + i) * j.n + e] : 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) sum += x[i];
  const u32 upto = wave_inclusive_sum(sum);
  u32 before = upto - sum;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (first + i < j.chunks) j.counts[(u64)(first + i) * j.n + e] = before;
    before += x[i];
  }
  if (lane_id() == CCLD_WAVE - 1) j.totals[e] = upto;
}

template <class I, int THREADS>
__global__ __launch_bounds__(THREADS) void k_order_place(OrderJob j) {
  constexpr int WAVES = THREADS / CCLD_WAVE, EACH = CCLD_ROUTE_EXPERTS / THREADS;
  __shared__ u32 counter[WAVES][CCLD_ROUTE_EXPERTS], all[CCLD_ROUTE_EXPERTS], earlier[CCLD_ROUTE_EXPERTS], s_wave[WAVES];
  const u32 lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / CCLD_WAVE), n = j.n;
  const u64 start = ((u64)blockIdx.x * WAVES + wave) * j.stretch;
  const u32 end = (u32)min((u64)j.entries, start + j.stretch);
  for (int e = lane; e < n; e += CCLD_WAVE) counter[wave][e] = 0;
  for (int e = threadIdx.x; e < n; e += THREADS) all[e] = earlier[e] = 0;
  u32 first[AT_ONCE];
  next_experts<I>(j, start, end, first);
  for (u64 at = start; at < end; at += LEAST_STRETCH) {
    u32 e[AT_ONCE];
    if (at == start) __builtin_memcpy(e, first, sizeof e);
    else next_experts<I>(j, at, end, e);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
      if (e[i] < (u32)n) atomicAdd(&counter[wave][e[i]], 1u);
  }
  __syncthreads();
  // what lies before this chunk's entries of an expert, and how many there are in all
  if (j.totals) {
    for (int e = threadIdx.x; e < n; e += THREADS) {
      all[e] = j.totals[e];
      earlier[e] = j.counts[(u64)blockIdx.x * n + e];
    }
    __syncthreads();
  } else if (j.chunks > 1) {
    // the chunks shared by as many threads to an expert as there are, eight at a time
    const int parts = max(THREADS / n, 1);
    for (int i = threadIdx.x; i < n * parts; i += THREADS) {
      const int e = i % n;
      u32 sum = 0, before = 0;
      for (u32 c = i / n; c < j.chunks; c += 8 * parts) {
        u32 x[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = j.counts[(u64)min(c + q * parts, j.chunks - 1) * n + e];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const u32 at = c + q * parts;
          sum += at < j.chunks ? x[q] : 0;
          before += at < min(j.chunks, blockIdx.x) ? x[q] : 0;
        }
      }
      atomicAdd(&all[e], sum);
      atomicAdd(&earlier[e], before);
    }
    __syncthreads();
  }
  for (int e = threadIdx.x; e < n; e += THREADS) {
    u32 before = earlier[e];
    for (int w = 0; w < WAVES; ++w) {
      const u32 x = counter[w][e];
      counter[w][e] = before;
      before += x;
    }
    if (j.chunks == 1) all[e] = before;
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
  for (u64 at0 = start; at0 < end; at0 += LEAST_STRETCH) {
    u32 e[AT_ONCE];
    if (at0 == start) __builtin_memcpy(e, first, sizeof e);
    else next_experts<I>(j, at0, end, e);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      u64 same = ~0ull;
      for (int b = 0; b < bits; ++b) {
        const bool set = e[i] >> b & 1;
        const u64 m = ballot64(set);
        same &= set ? m : ~m;
      }
      const u32 rank = mbcnt64(same);
      u32 taken = 0;
      if (rank == 0 && e[i] < (u32)n) taken = atomicAdd(&counter[wave][e[i]], (u32)__builtin_popcountll(same));
      taken = lane_read(taken, (u32)__builtin_ctzll(same));
      const u64 at = at0 + i * CCLD_WAVE + lane;
      if (at < end) j.places[at] = e[i] < (u32)n ? (int32_t)(all[e[i]] + taken + rank) : -1;
    }
  }
}

OrderJob order_job(const ccld_order_args* a, uint64_t* bytes) {
  OrderJob j{a->experts, a->places, a->offsets, static_cast<u32*>(a->workspace), nullptr, (u32)(a->tokens * a->k), 1, 0, (int)a->n_experts};
  if (j.entries <= SINGLE_CHUNK) {
    j.stretch = (u32)blocks_for(std::max<u32>(j.entries, 1), j.entries <= FEW_ENTRIES ? ORDER_THREADS : 1024) * CCLD_WAVE;
    *bytes = 0;
  } else {
    const u64 waves = MOST_CHUNKS * (ORDER_THREADS / CCLD_WAVE);
    j.stretch = std::max<u32>(LEAST_STRETCH, (u32)((((u64)j.entries + waves - 1) / waves + CCLD_WAVE - 1) / CCLD_WAVE * CCLD_WAVE));
    j.chunks = (u32)blocks_for(j.entries, (i64)j.stretch * (ORDER_THREADS / CCLD_WAVE));
    const uint64_t counts = (uint64_t)j.chunks * (uint64_t)a->n_experts;
    const bool many = j.chunks > MANY_CHUNKS;
    if (many && j.counts) j.totals = j.counts + counts;
    *bytes = 4 * (counts + (many ? (uint64_t)a->n_experts : 0));
  }
  return j;
}
template <class I>
void launch_order(const OrderJob& j, hipStream_t stream) {
  if (j.entries <= FEW_ENTRIES) {
    k_order_place<I, ORDER_THREADS><<<1, ORDER_THREADS, 0, stream>>>(j);
  } else if (j.chunks == 1) {
    k_order_place<I, 1024><<<1, 1024, 0, stream>>>(j);
  } else {
    k_order_count<I><<<j.chunks, ORDER_THREADS, 0, stream>>>(j);
    if (j.totals) k_order_scan<<<(u32)blocks_for(j.n, ORDER_THREADS / CCLD_WAVE), ORDER_THREADS, 0, stream>>>(j);
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
