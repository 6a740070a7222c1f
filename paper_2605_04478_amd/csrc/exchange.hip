// Rows of tokens sorted by expert and back, with their weights, and the gradients of both ways (ccld_dispatch*, ccld_combine*).
//
//   rows[place[t, j]] = x[t]                               dx[t] = sum_j drows[place[t, j]]
//   out[t] = sum_j w[t, j] y[place[t, j]]                  dy[place[t, j]] = w[t, j] dout[t]      dw[t, j] = dout[t] . y[place[t, j]]
//
// Memory bounds all four.  A token belongs to a team of threads, so that its own row is moved once however many experts it has: spreading writes
// one loaded vector to k rows, gathering adds k rows up in registers in the order of j, rounded once.  A place outside the rows is
// never followed.
//
// Measured (a copy of 2 GB moves 4.9 TB/s here, x + 1 6.1): 32,768 x 4,096 in bfloat16 with 8 experts: dispatch 462 us = 5.2 TB/s, combine and dispatch's gradient 445 = 5.4, combine's gradient 899 =
// 5.1; 8,192 x 2,048 with 2: 15 to 17 and 26; 3,001 x 1,001 in half precision with 3, whose rows start anywhere: 5 to 7 and 10.  5 tokens: 3 us each.
// Rows at odd addresses that the caches do not hold: every vector lies across two lines (18,289 x 997 in bfloat16 with 7 experts, other data each time: dispatch, combine, its gradient and dispatch's 76, 92, 188 and 89 us; x 1,000 69, 54, 118 and 54; a copy's rate
// would be 60 and 112 for the gradient).
#include <algorithm>

#include "ccld_internal.h"
#include "operators.h"

using namespace ccld;

namespace {

// Entries of a token that are on their way at once.  Two are enough, with as many tokens to a compute unit as its wavefronts hold; eight ask for six
// rows in vain where there are two (8,192 x 2,048 with 2 experts: combine 18 and 20 us).
constexpr int AT_ONCE = 2;

struct ExchangeJob {
  const int32_t *places, *used;
  const float* weights;
  const void *x, *y;
  void *x_out, *y_out;
  float* dweights;
  i64 ldx, ldy, ldx_out, ldy_out, tokens;
  u32 rows;                      // tokens x k
  int k, d;
};

// a team is a workgroup, or one of the four wavefronts of one
constexpr int threads_of(int team) { return team == CCLD_WAVE ? 256 : team; }

// A token's places and weights.  A team's token is the same for all of its lanes, so these are scalar loads, which no lane has to be active for.
struct Places {
  const __attribute__((address_space(4))) int32_t* place;
  const __attribute__((address_space(4))) float* weight;
  u32 rows;
  __device__ __forceinline__ Places(const ExchangeJob& j, i64 t)
      : place((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(j.places + t * j.k)),
        weight((const __attribute__((address_space(4))) float*)(uintptr_t)(j.weights + t * j.k)), rows(j.rows) {}
  __device__ __forceinline__ int at(int i) const { return (u32)place[i] < rows ? place[i] : -1; }
  __device__ __forceinline__ float weight_at(int i) const { return weight[i]; }
};

// the rows that no entry has, zeroed by the tokens of the same numbers
template <int TEAM, class T>
__device__ __forceinline__ void clear_unused(const ExchangeJob& j, i64 t, int me, u32 used) {
  constexpr int N = 16 / sizeof(T);
  for (u32 r = max((u32)(t * j.k), used); r < (u32)(t * j.k) + (u32)j.k; ++r) {
    T* const row = static_cast<T*>(j.y_out) + (i64)r * j.ldy_out;
    int c = me * N;
    for (; c + N <= j.d; c += TEAM * N) store_once<N>(row + c, Vec<T, N>{});
    for (; c < j.d; ++c) row[c] = (T)0.0f;
  }
}

// (a thread that the end of the row falls on takes what is left of it value by value)
template <class T, int TEAM, bool ONCE>
__global__ __launch_bounds__(threads_of(TEAM)) void k_dispatch(ExchangeJob j) {
  constexpr int N = 16 / sizeof(T), TEAMS = threads_of(TEAM) / TEAM;
  const int me = threadIdx.x % TEAM;
  const u32 used = (u32)max(*j.used, 0);
  i64 t = (i64)blockIdx.x * TEAMS + (TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
  for (; t < j.tokens; t += (i64)gridDim.x * TEAMS) {
    const Places p(j, t);
    const T* const x = static_cast<const T*>(j.x) + t * j.ldx;
    T* const y = static_cast<T*>(j.y_out);
    int c = me * N;
    for (; c + N <= j.d; c += TEAM * N) {
      const Vec<T, N> v = load_vec<N>(x + c);
#pragma unroll 4
      for (int i = 0; i < j.k; ++i) {
        const int at = p.at(i);
        if (at < 0) continue;
        if constexpr (ONCE) store_once<N>(y + at * j.ldy_out + c, v);
        else store_vec<N>(y + at * j.ldy_out + c, v);
      }
    }
    for (; c < j.d; ++c) {
      for (int i = 0; i < j.k; ++i) {
        const int at = p.at(i);
        if (at >= 0) y[at * j.ldy_out + c] = x[c];
      }
    }
    clear_unused<TEAM, T>(j, t, me, used);
  }
}

// WEIGHTED: combine, else the gradient of dispatch
template <class T, int TEAM, bool WEIGHTED>
__global__ __launch_bounds__(threads_of(TEAM)) void k_gather(ExchangeJob j) {
  constexpr int N = 16 / sizeof(T), TEAMS = threads_of(TEAM) / TEAM;
  const int me = threadIdx.x % TEAM;
  i64 t = (i64)blockIdx.x * TEAMS + (TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
  for (; t < j.tokens; t += (i64)gridDim.x * TEAMS) {
    const Places p(j, t);
    const T* const y = static_cast<const T*>(j.y);
    T* const out = static_cast<T*>(j.x_out) + t * j.ldx_out;
    int c = me * N;
    for (; c + N <= j.d; c += TEAM * N) {
      float sum[N] = {};
      for (int i0 = 0; i0 < j.k; i0 += AT_ONCE) {
        // (the first row stands for those that are not there: loads without a branch are all on their way at once)
        Vec<T, N> v[AT_ONCE];
        bool there[AT_ONCE];
        float w[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          const int at = i0 + i < j.k ? p.at(i0 + i) : -1;
          there[i] = at >= 0;
          w[i] = !there[i] ? 0.0f : WEIGHTED ? p.weight_at(i0 + i) : 1.0f;
          v[i] = load_vec<N>(y + max(at, 0) * j.ldy + c);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
          for (int n = 0; n < N; ++n) sum[n] += there[i] ? w[i] * (float)v[i][n] : 0.0f;
      }
      Vec<T, N> o;
#pragma unroll
      for (int n = 0; n < N; ++n) o[n] = (T)sum[n];
      store_once<N>(out + c, o);
    }
    for (; c < j.d; ++c) {
      float sum = 0;
      for (int i = 0; i < j.k; ++i) {
        const int at = p.at(i);
        if (at >= 0) sum += (WEIGHTED ? p.weight_at(i) : 1.0f) * (float)y[at * j.ldy + c];
      }
      out[c] = (T)sum;
    }
  }
}

// The gradient of combine: AT_ONCE entries in a pass over the row, their products with y summed over the team.
template <class T, int TEAM>
__global__ __launch_bounds__(threads_of(TEAM)) void k_combine_grad(ExchangeJob j) {
  constexpr int N = 16 / sizeof(T), TEAMS = threads_of(TEAM) / TEAM, WAVES = TEAM / CCLD_WAVE;
  __shared__ float sums[2][WAVES][AT_ONCE];
  const int me = threadIdx.x % TEAM;
  const u32 used = (u32)max(*j.used, 0);
  int turn = 0;
  i64 t = (i64)blockIdx.x * TEAMS + (TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
  for (; t < j.tokens; t += (i64)gridDim.x * TEAMS) {
    const Places p(j, t);
    const T* const x = static_cast<const T*>(j.x) + t * j.ldx;
    const T* const y = static_cast<const T*>(j.y);
    T* const dy = static_cast<T*>(j.y_out);
    for (int i0 = 0; i0 < j.k; i0 += AT_ONCE) {
      float dot[AT_ONCE] = {};
      int c = me * N;
      for (; c + N <= j.d; c += TEAM * N) {
        const Vec<T, N> v = load_vec<N>(x + c);
        Vec<T, N> q[AT_ONCE];
        if (j.dweights)
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) q[i] = load_vec<N>(y + (i0 + i < j.k ? max(p.at(i0 + i), 0) : 0) * j.ldy + c);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          if (i0 + i >= j.k || p.at(i0 + i) < 0) continue;
          const float w = p.weight_at(i0 + i);
          Vec<T, N> o;
#pragma unroll
          for (int n = 0; n < N; ++n) o[n] = (T)(w * (float)v[n]);
          store_once<N>(dy + p.at(i0 + i) * j.ldy_out + c, o);
          if (j.dweights)
#pragma unroll
            for (int n = 0; n < N; ++n) dot[i] += (float)v[n] * (float)q[i][n];
        }
      }
      for (; c < j.d; ++c) {
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          if (i0 + i >= j.k || p.at(i0 + i) < 0) continue;
          dy[p.at(i0 + i) * j.ldy_out + c] = (T)(p.weight_at(i0 + i) * (float)x[c]);
          if (j.dweights) dot[i] += (float)x[c] * (float)y[p.at(i0 + i) * j.ldy + c];
        }
      }
      if (j.dweights) {
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) dot[i] = wave_total(dot[i]);
        if constexpr (WAVES > 1) {
          // (the place is written again by the pass after the next: one barrier is enough)
          const int wave = threadIdx.x / CCLD_WAVE;
          if (lane_id() == 0)
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) sums[turn][wave][i] = dot[i];
          __syncthreads();
#pragma unroll
          for (int i = 0; i < AT_ONCE; ++i) {
            dot[i] = 0;
            for (int w = 0; w < WAVES; ++w) dot[i] += sums[turn][w][i];
          }
          turn ^= 1;
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
          if (me == 0 && i0 + i < j.k) j.dweights[t * j.k + i0 + i] = p.at(i0 + i) < 0 ? 0.0f : dot[i];
      }
    }
    clear_unused<TEAM, T>(j, t, me, used);
  }
}

enum Way { DISPATCH, DISPATCH_GRAD, COMBINE, COMBINE_GRAD };

template <class T, int TEAM>
void launch(const ExchangeJob& j, Way way, hipStream_t stream) {
  constexpr int THREADS = threads_of(TEAM);
  const u32 grid = (u32)std::min<i64>(blocks_for(j.tokens, THREADS / TEAM), 64 * COMPUTE_UNITS);
  if (way == DISPATCH) {
    // Past the caches, but for rows of whole vectors that share lines with their neighbours: a line then goes to memory in two pieces.  What is left in the caches is there for who reads the rows next, or
    // is written back while another kernel runs: 18,289 x 1,000 in bfloat16 with 7 experts, past and through the caches, takes 73 and 69 us call after call, 128 and 103 with a gather of the same rows behind it, 88 and 99 beside an addition to 256 MB;
    // 4,000 x 1,000 17 and 12, 29 and 24, 20 and 32; 30,000 x 2,056 with 8 284 and 250, 486 and 479, 314 and 287.  (x 1,024 51 and 49; x 997, whose vectors lie across lines, 76 and 87; 32,768 x 4,096 with 8 460 and 470.)
    auto made_of = [&](i64 bytes) { return aligned(j.y_out, bytes) && j.ldy_out * (i64)sizeof(T) % bytes == 0; };
    if (made_of(128) || !made_of(16)) k_dispatch<T, TEAM, true><<<grid, THREADS, 0, stream>>>(j);
    else k_dispatch<T, TEAM, false><<<grid, THREADS, 0, stream>>>(j);
  }
  else if (way == DISPATCH_GRAD) k_gather<T, TEAM, false><<<grid, THREADS, 0, stream>>>(j);
  else if (way == COMBINE) k_gather<T, TEAM, true><<<grid, THREADS, 0, stream>>>(j);
  else k_combine_grad<T, TEAM><<<grid, THREADS, 0, stream>>>(j);
}

ccld_status exchange(const ccld_exchange_args* a, Way way, void* stream) {
  if (!a) return CCLD_E_NULL;
  const bool reads_x = way == DISPATCH || way == COMBINE_GRAD, weighted = way == COMBINE || way == COMBINE_GRAD;
  const bool reads_y = !reads_x || (way == COMBINE_GRAD && a->dweights);
  if (!known_type(a->dtype) || a->tokens < 0 || a->k < 1 || a->d < 1) return CCLD_E_BAD_ARG;
  if (a->tokens >= MAX_ROWS || a->k > CCLD_ROUTE_MOST || a->tokens * a->k >= MAX_ROWS || a->d >= (i64)1 << 28) return CCLD_E_CAPACITY;
  if (a->tokens && (!a->places || (weighted && !a->weights) || (reads_x && (!a->x || !a->y_out || !a->used)) || (!reads_x && !a->x_out) || (reads_y && !a->y)))
    return CCLD_E_NULL;
  auto matrix = [&](const void* p, i64 ld) { return ld >= a->d && aligned(p, size_of(a->dtype)); };
  if (reads_x ? !matrix(a->x, a->ldx) || !matrix(a->y_out, a->ldy_out) : !matrix(a->x_out, a->ldx_out)) return CCLD_E_BAD_ARG;
  if ((reads_y && !matrix(a->y, a->ldy)) || !aligned(a->places, 4) || (weighted && !aligned(a->weights, 4)) || (reads_x && !aligned(a->used, 4)) ||
      (way == COMBINE_GRAD && !aligned(a->dweights, 4))) return CCLD_E_BAD_ARG;
  if (a->tokens == 0) return CCLD_OK;
  const ExchangeJob j{a->places, a->used, weighted ? a->weights : nullptr, a->x, a->y, a->x_out, a->y_out, way == COMBINE_GRAD ? a->dweights : nullptr,
                      a->ldx, a->ldy, a->ldx_out, a->ldy_out, a->tokens, (u32)(a->tokens * a->k), (int)a->k, (int)a->d};
  const hipStream_t st = static_cast<hipStream_t>(stream);
  with_type(a->dtype, [&](auto zero) {
    using T = decltype(zero);
    // a vector to a thread: dispatch, combine, its gradient and dispatch's of 8,192 x 4,096 in bfloat16 with 8 experts each take 104, 112, 223 and 111 us in teams of 512 threads, 108, 118, 233
    // and 118 in teams of 256, 118, 137, 272 and 135 in wavefronts; of 8,192 x 1,024 with 2 experts 9.6, 10.4, 25 and 10 in teams of 512 and 9.0, 9.0, 15 and 9.2 in teams of 128; of 8,192 x 4,096 in 32 bits with 2 experts 73, 70, 123 and 70 in teams of 1,024 and
    // 75, 74, 129 and 74 in teams of 512
    const i64 vectors = blocks_for(a->d, 16 / (i64)sizeof(T));
    if (vectors <= 64) launch<T, CCLD_WAVE>(j, way, st);
    else if (vectors <= 128) launch<T, 128>(j, way, st);
    else if (vectors <= 256) launch<T, 256>(j, way, st);
    else if (vectors <= 512) launch<T, 512>(j, way, st);
    else launch<T, 1024>(j, way, st);
  });
  return launched();
}

}  // namespace

extern "C" ccld_status ccld_dispatch(const ccld_exchange_args* a, void* stream) { return exchange(a, DISPATCH, stream); }
extern "C" ccld_status ccld_dispatch_grad(const ccld_exchange_args* a, void* stream) { return exchange(a, DISPATCH_GRAD, stream); }
extern "C" ccld_status ccld_combine(const ccld_exchange_args* a, void* stream) { return exchange(a, COMBINE, stream); }
extern "C" ccld_status ccld_combine_grad(const ccld_exchange_args* a, void* stream) { return exchange(a, COMBINE_GRAD, stream); }
