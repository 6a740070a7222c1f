// Log probabilities of given tokens under whole rows of logits, their entropy, the largest logits, and the gradient (ccld_token_logprobs*).
//
//   z = logits / T      S = sum exp(z - m)      lse = m + log S      logp = z[token] - lse      entropy = log S + sum exp(z - m) (m - z) / S
//   dlogits = (dlogp ([v = token] - p) - dentropy p (log p + entropy)) / T,  p = exp(z - lse)
//
// Memory bounds both: a row is read once (again for the alternatives, which the caches answer), a few operations and one exponential to a logit.  Largest logit, sum and
// entropy's sum are taken in one pass: every thread takes a batch of values, moves to the batch's maximum if that is larger than its own, and
// adds up relative to it.  The entropy's terms all have one sign, so nothing cancels.
//
// Alternatives: the `top` largest of 64 maxima of a row's parts are each at least as large as the smallest of them, which therefore bounds the row's `top` largest
// logits from below; a second pass collects what reaches the bound (a few more than `top`, as a rule) and ranks it.  Rows of which more reaches it than there is room for, equal
// logits by the thousand, are searched once for each alternative.
#include <algorithm>

#include "ccld_internal.h"
#include "operators.h"

using namespace ccld;

namespace {

struct LogprobJob {
  const void *logits, *tokens;
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_ids;
  const float *dlogp, *dentropy;
  void* dlogits;
  i64 ld, ldd, dlogp_stride, dentropy_stride, rows, vocab;
  float temperature;
  int top, token_bits;
  u32 parts;                     // workgroups to a row (gradient)
};

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
// below 2^-200 of the largest nothing is left of a value (and a masked one stays finite)
constexpr float NOTHING = -200.0f;

__device__ __forceinline__ i64 token_of(const LogprobJob& j, i64 row) {
  const i64 t = j.token_bits == 32 ? static_cast<const int32_t*>(j.tokens)[row] : static_cast<const i64*>(j.tokens)[row];
  return t >= 0 && t < j.vocab ? t : -1;
}

// Sums of exp2((z - m) c) and of exp2((z - m) c) (m - z) c.
struct Sums {
  float m = LOWEST, s = 0, b = 0;
  // the same relative to a maximum that is at least as large
  __device__ __forceinline__ void move(float to, float c) {
    if (to == LOWEST) return;
    const float d = m == LOWEST ? 0.0f : (m - to) * c, f = exp2f(d);
    b = f * (b - s * fmaxf(d, NOTHING));
    s *= f;
    m = to;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&z)[N], float c) {
    float most = m;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, z[i]);
    if (most > m) move(most, c);
    const float from = m == LOWEST ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = (z[i] - from) * c, e = __builtin_amdgcn_exp2f(d);
      s += e;
      b -= e * fmaxf(d, NOTHING);
    }
  }
  __device__ __forceinline__ void join(const Sums& o, float c) {
    const float to = fmaxf(m, o.m);
    Sums other = o;
    move(to, c);
    other.move(to, c);
    s += other.s;
    b += other.b;
  }
};

// The row's values that belong to this thread of so many, in batches: f(values, first column of each vector).
template <class T, int THREADS, class F>
__device__ __forceinline__ void each_batch(const T* row, i64 vocab, int me, F f) {
  constexpr int N = 16 / sizeof(T), BATCH = 4;
  i64 at = (i64)me * N;
  for (; at + (i64)(BATCH - 1) * THREADS * N + N <= vocab; at += (i64)BATCH * THREADS * N) {
    Vec<T, N> v[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) v[i] = load_vec<N>(row + at + (i64)i * THREADS * N);
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      float z[N];
#pragma unroll
      for (int n = 0; n < N; ++n) z[n] = (float)v[i][n];
      f(z, at + (i64)i * THREADS * N);
    }
  }
  for (; at < vocab; at += (i64)THREADS * N) {
    float z[N];
    if (at + N <= vocab) {
      const Vec<T, N> v = load_vec<N>(row + at);
#pragma unroll
      for (int n = 0; n < N; ++n) z[n] = (float)v[n];
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) z[n] = at + n < vocab ? (float)row[at + n] : LOWEST;
    }
    f(z, at);
  }
}

template <int THREADS>
__device__ __forceinline__ Sums join_all(Sums x, float c, float (&place)[THREADS / CCLD_WAVE][3]) {
  const float m = wave_max(x.m);
  x.move(m, c);
  x.s = wave_total(x.s);
  x.b = wave_total(x.b);
  x.m = m;
  constexpr int WAVES = THREADS / CCLD_WAVE;
  const int wave = threadIdx.x / CCLD_WAVE;
  if (lane_id() == 0) { place[wave][0] = x.m; place[wave][1] = x.s; place[wave][2] = x.b; }
  __syncthreads();
  Sums all;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    Sums o;
    o.m = place[w][0]; o.s = place[w][1]; o.b = place[w][2];
    all.join(o, c);
  }
  return all;
}

constexpr int ROOM = 1024;

template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_logprobs(LogprobJob j) {
  __shared__ float place[THREADS / CCLD_WAVE][3];
  __shared__ float maxima[THREADS], value[ROOM];
  __shared__ int id[ROOM];
  __shared__ u32 found;
  __shared__ float bound;
  const float c = LOG2E / j.temperature;
  const int me = threadIdx.x;
  for (i64 r = blockIdx.x; r < j.rows; r += gridDim.x) {
    const T* const row = static_cast<const T*>(j.logits) + r * j.ld;
    Sums x;
    float most = LOWEST;
    each_batch<T, THREADS>(row, j.vocab, me, [&](const auto& z, i64) { x.add(z, c); });
    most = x.m;
    __syncthreads();                        // the row before is done with
    if (me == 0) found = 0;
    maxima[me] = most;
    const Sums all = join_all<THREADS>(x, c, place);
    const bool none = all.m == LOWEST && all.s == 0;
    // (a row that is not empty has a finite lse, at a low temperature too, by which the gradient knows it; NaN stays)
    const float log_s = logf(all.s);
    float lse = none ? LOWEST : all.m / j.temperature + log_s;
    if (!none && fabsf(lse) > __FLT_MAX__) lse = copysignf(__FLT_MAX__, lse);
    if (me == 0) {
      const i64 t = token_of(j, r);
      float logp = 0;
      if (t >= 0) {
        const float z = (float)row[t];
        logp = z == LOWEST && all.s == all.s ? LOWEST : (z - all.m) / j.temperature - log_s;
      }
      j.logp[r] = logp;
      j.lse[r] = lse;
      j.entropy[r] = none ? 0.0f : log_s + all.b * LN2 / all.s;
    }
    if (j.top == 0) continue;
    // 64 maxima: the bound is the one with top - 1 before it
    if (me < CCLD_WAVE) {
      float mine = LOWEST;
      for (int i = me; i < THREADS; i += CCLD_WAVE) mine = fmaxf(mine, maxima[i]);
      int before = 0;
      for (int l = 0; l < CCLD_WAVE; ++l) {
        const float o = read_lane(mine, l);
        before += o > mine || (o == mine && l < me);
      }
      if (before == j.top - 1) bound = mine;
    }
    __syncthreads();
    const float least = bound;
    each_batch<T, THREADS>(row, j.vocab, me, [&](const auto& z, i64 at) {
      constexpr int N = 16 / sizeof(T);
      float most = z[0];
#pragma unroll
      for (int n = 1; n < N; ++n) most = fmaxf(most, z[n]);
      if (most >= least && most > LOWEST) {
        for (int n = 0; n < N; ++n)
          if (z[n] >= least && z[n] > LOWEST) {
            const u32 to = atomicAdd(&found, 1u);
            if (to < ROOM) { value[to] = z[n]; id[to] = (int)(at + n); }
          }
      }
    });
    __syncthreads();
    const u32 n = found;
    int32_t* const ids = j.top_ids + r * j.top;
    float* const logps = j.top_logp + r * j.top;
    auto put = [&](int rank, float z, int at) {
      ids[rank] = at;
      logps[rank] = at < 0 ? LOWEST : (z - all.m) / j.temperature - log_s;
    };
    if (n <= ROOM) {
      for (u32 i = me; i < n; i += THREADS) {
        const float z = value[i];
        const int at = id[i];
        int rank = 0;
        for (u32 o = 0; o < n; ++o) rank += value[o] > z || (value[o] == z && id[o] < at);
        if (rank < j.top) put(rank, z, at);
      }
      for (int i = me; i < j.top; i += THREADS)
        if (i >= (int)n) put(i, 0, -1);
    } else {
      // one after another: the largest of those that come after the one before
      float last = __builtin_huge_valf();
      i64 last_at = -1;
      for (int k = 0; k < j.top; ++k) {
        float best = LOWEST;
        i64 best_at = j.vocab;
        each_batch<T, THREADS>(row, j.vocab, me, [&](const auto& z, i64 at) {
          constexpr int N = 16 / sizeof(T);
#pragma unroll
          for (int n = 0; n < N; ++n)
            if ((z[n] < last || (z[n] == last && at + n > last_at)) && z[n] > best) { best = z[n]; best_at = at + n; }
        });
        __syncthreads();
        maxima[me] = best;
        id[me] = (int)best_at;
        __syncthreads();
        for (int half = THREADS / 2; half >= 1; half /= 2) {
          if (me < half) {
            const float o = maxima[me + half];
            const int at = id[me + half];
            if (o > maxima[me] || (o == maxima[me] && at < id[me])) { maxima[me] = o; id[me] = at; }
          }
          __syncthreads();
        }
        last = maxima[0];
        last_at = id[0];
        if (me == 0) put(k, last, last == LOWEST ? -1 : (int)last_at);
      }
    }
  }
}

// lse of a row far from zero has too few bits behind the point to take exp(z - lse) with (at 64 p is off by 2^-18): the row's maximum and sum are taken
// again there.
constexpr float FAR = 64.0f;

template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_logprobs_grad(LogprobJob j) {
  constexpr int N = 16 / sizeof(T);
  __shared__ float place[THREADS / CCLD_WAVE][3];
  const float c = LOG2E / j.temperature, per = 1.0f / j.temperature;
  const i64 all = j.rows * j.parts;
  for (i64 b = blockIdx.x; b < all; b += gridDim.x) {
    const i64 r = b / j.parts;
    const u32 part = (u32)(b - r * j.parts);
    const T* const row = static_cast<const T*>(j.logits) + r * j.ld;
    T* const out = static_cast<T*>(j.dlogits) + r * j.ldd;
    const float lse = j.lse[r], entropy = j.entropy[r];
    const i64 t = token_of(j, r);
    const float dl = t >= 0 && j.dlogp ? j.dlogp[r * j.dlogp_stride] : 0.0f, de = j.dentropy ? j.dentropy[r * j.dentropy_stride] : 0.0f;
    // log p = (z - base) c2 - rest, in powers of two
    float base = 0, rest = lse * LOG2E;
    const bool none = lse == LOWEST;
    if (fabsf(lse) >= FAR && !none) {
      Sums x;
      each_batch<T, THREADS>(row, j.vocab, threadIdx.x, [&](const auto& z, i64) { x.add(z, c); });
      __syncthreads();
      const Sums sums = join_all<THREADS>(x, c, place);
      base = sums.m;
      rest = log2f(sums.s);
    }
    auto gradient = [&](float z, bool target) {
      if (none) return 0.0f;
      const float d = (z - base) * c - rest, p = __builtin_amdgcn_exp2f(d);
      const float g = (target ? dl : 0.0f) - p * (dl + de * (fmaxf(d, NOTHING) * LN2 + entropy));
      return g * per;
    };
    for (i64 at = ((i64)part * THREADS + threadIdx.x) * N; at < j.vocab; at += (i64)j.parts * THREADS * N) {
      if (at + N <= j.vocab) {
        const Vec<T, N> v = load_vec<N>(row + at);
        Vec<T, N> o;
#pragma unroll
        for (int n = 0; n < N; ++n) o[n] = (T)gradient((float)v[n], at + n == t);
        store_vec<N>(out + at, o);
      } else {
        for (i64 k = at; k < j.vocab; ++k) out[k] = (T)gradient((float)row[k], k == t);
      }
    }
  }
}

ccld_status check(const ccld_logprob_args* a) {
  if (!a) return CCLD_E_NULL;
  if (!known_type(a->dtype) || (a->token_bits != 32 && a->token_bits != 64) || a->rows < 0 || a->vocab < 1) return CCLD_E_BAD_ARG;
  if (!(a->temperature >= 0x1p-64f && a->temperature <= 0x1p64f) || a->top < 0 || a->top > CCLD_TOP_MOST) return CCLD_E_BAD_ARG;
  if (a->rows >= MAX_ROWS || a->vocab >= MAX_ROWS) return CCLD_E_CAPACITY;
  return CCLD_OK;
}
LogprobJob make_job(const ccld_logprob_args* a) {
  return LogprobJob{a->logits, a->tokens, a->logp, a->entropy, a->lse, a->top_logp, a->top_ids, a->dlogp, a->dentropy, a->dlogits, a->ldlogits, a->lddlogits,
                    a->dlogp_stride, a->dentropy_stride, a->rows, a->vocab, a->temperature, a->top, a->token_bits, 1};
}
bool all_aligned(const ccld_logprob_args* a) {
  for (const void* p : {static_cast<const void*>(a->logp), static_cast<const void*>(a->entropy), static_cast<const void*>(a->lse), static_cast<const void*>(a->top_ids),
                        static_cast<const void*>(a->top_logp), static_cast<const void*>(a->dlogp), static_cast<const void*>(a->dentropy)})
    if (!aligned(p, 4)) return false;
  return aligned(a->logits, size_of(a->dtype)) && aligned(a->dlogits, size_of(a->dtype)) && aligned(a->tokens, a->token_bits / 8);
}

}  // namespace

extern "C" ccld_status ccld_logprob_workspace(const ccld_logprob_args* a, uint64_t* bytes) {
  if (!bytes) return CCLD_E_NULL;
  *bytes = 0;
  return check(a);
}

extern "C" ccld_status ccld_token_logprobs(const ccld_logprob_args* a, void* stream) {
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  if (a->rows && (!a->logits || !a->tokens || !a->logp || !a->entropy || !a->lse || (a->top && (!a->top_ids || !a->top_logp)))) return CCLD_E_NULL;
  if (a->ldlogits < a->vocab || !all_aligned(a)) return CCLD_E_BAD_ARG;
  if (a->rows == 0) return CCLD_OK;
  const LogprobJob j = make_job(a);
  const u32 grid = (u32)std::min<i64>(a->rows, 1 << 20);
  with_type(a->dtype, [&](auto zero) {
    using T = decltype(zero);
    if (a->rows < (i64)2 * COMPUTE_UNITS) k_logprobs<T, 1024><<<grid, 1024, 0, static_cast<hipStream_t>(stream)>>>(j);
    else k_logprobs<T, 256><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(j);
  });
  return launched();
}

extern "C" ccld_status ccld_token_logprobs_grad(const ccld_logprob_args* a, void* stream) {
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  if (a->rows && (!a->logits || !a->tokens || !a->entropy || !a->lse || !a->dlogits)) return CCLD_E_NULL;
  if (a->ldlogits < a->vocab || a->lddlogits < a->vocab || !all_aligned(a)) return CCLD_E_BAD_ARG;
  if (a->rows == 0) return CCLD_OK;
  LogprobJob j = make_job(a);
  constexpr int THREADS = 256;
  // eight workgroups to a compute unit, and two vectors to a thread at least
  const i64 vectors = blocks_for(a->vocab, 16 / size_of(a->dtype));
  j.parts = (u32)std::max<i64>(1, std::min<i64>(blocks_for(8 * COMPUTE_UNITS, a->rows), vectors / (2 * THREADS)));
  const u32 grid = (u32)std::min<i64>(a->rows * j.parts, 1 << 20);
  with_type(a->dtype, [&](auto zero) { k_logprobs_grad<decltype(zero), THREADS><<<grid, THREADS, 0, static_cast<hipStream_t>(stream)>>>(j); });
  return launched();
}
