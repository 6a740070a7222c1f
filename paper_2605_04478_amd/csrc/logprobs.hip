// Log probabilities of given tokens under whole rows of logits, their entropy, the largest logits, and the gradient (ccld_token_logprobs*).
//
//   z = logits / T      S = sum exp(z - m)      lse = m + log S      logp = z[token] - lse      entropy = log S + sum exp(z - m) (m - z) / S
//   dlogits = (dlogp ([v = token] - p) - dentropy p (log p + entropy)) / T,  p = exp(z - lse)
//
// Memory bounds both, the exponentials and their dozen of operations to a logit come next.  Largest logit, sum and entropy's sum are taken in one pass: a thread
// adds up relative to a value next to the largest that it has seen, so that the entropy's terms do not cancel.  Few
// long rows are cut into parts, one to a workgroup, which a second launch joins in their order.
//
// Alternatives: of the threads' maxima the `top` largest are as many different logits, so the smallest of them bounds the row's `top` largest logits from
// below.  A second pass, over a row that the caches still hold, collects what reaches the bound (a few more than `top`, as a rule) and ranks it.  Rows of which more reaches it than
// there is room for, equal logits by the thousand, are searched once for each alternative.
//
// Gradient: 1 - p of a sure target needs more bits than lse has, so the sum is taken again.  Rows are held in registers in between, where they fit (131,072 values of
// 16 bits: half of a compute unit's registers), and the next row's vectors are asked for as this row's are written, so that a row is read once and loads do
// not stop while it is computed.
//
// Measured (a copy of 2 GB moves 4.9 TB/s here, x + 1 6.1): 8,192 x 128,000 in bfloat16 356 us = 5.9 TB/s, with 20 alternatives 462, the gradient 775 = 5.4 (951 without the next row's loads); 1,003 x 50,021 in 32 bits 48 and
// 65; rows that registers do not hold are read twice: 8,192 x 151,936 in bfloat16 425 and 1,430, 4,096 x 262,144 364 and 1,210, 2,000 x 128,000 in 32 bits 177 and 605; 3 x 128,000 with 20 alternatives 8 + 5 us, without 4.5 + 2.7.
#include <algorithm>
#include <type_traits>

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
  i64 parts, span;               // of a row, and their columns
  int held;                      // vectors of a thread, where a row is cut into parts
  float *part_sums, *part_values;        // [rows][parts][3], [rows][parts][top]
  int* part_ids;
};

constexpr int JOIN_THREADS = 256;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
// below 2^-200 of the largest nothing is left of a value (and a masked one stays finite)
constexpr float NOTHING = -200.0f;

__device__ __forceinline__ i64 token_of(const LogprobJob& j, i64 row) {
  const i64 t = j.token_bits == 32 ? static_cast<const int32_t*>(j.tokens)[row] : static_cast<const i64*>(j.tokens)[row];
  return t >= 0 && t < j.vocab ? t : -1;
}

template <int N>
__device__ __forceinline__ float largest_of(const float (&z)[N]) {
  float m = z[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, z[i]);
  return m;
}

// sum += x, where sum is `over` above what was added to it: with the rounding of one addition made good by the next, a sum of any length is off by two roundings
__device__ __forceinline__ void add_to(float& sum, float& over, float x) {
  const float y = x - over, t = sum + y;
  over = (t - sum) - y;
  sum = t;
}

// Sums of exp2((z - m) c) and of exp2((z - m) c) (m - z) c.  m follows the largest value seen where that is more than 2^8 times as large: a wavefront then moves a few times in a
// row and not with almost every vector.  The second sum's terms below zero are at most 8 times the first's, and its roundings with them: additions one after another, whose roundings may
// all go one way, would cost the entropy up to 0.0002 with 1,024 values to a thread (and lse 0.00002).  A vector is therefore summed by itself and added to a sum that knows its
// rounding: a vector's eight roundings and three more are left, 2^-18 in the entropy where all terms are at the far end (0.000002 was the most in either length, 512 or 1,024 values).
constexpr float LEEWAY = 8.0f;
struct Sums {
  float m = LOWEST, s = 0, b = 0, s_over = 0, b_over = 0, most = LOWEST;
  // the same relative to another value, above m or some way below
  __device__ __forceinline__ void move(float to, float c) {
    if (to == LOWEST) return;
    const float d = m == LOWEST ? 0.0f : (m - to) * c, f = __builtin_amdgcn_exp2f(d), by = fmaxf(d, NOTHING);
    b = f * fmaf(-by, s, b);
    b_over = f * fmaf(-by, s_over, b_over);
    s *= f;
    s_over *= f;
    m = to;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&z)[N], float c) {
    most = fmaxf(most, largest_of(z));
    if ((most - m) * c > LEEWAY) move(most, c);
    const float from = m == LOWEST ? 0.0f : m;
    float own_s = 0, own_b = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = (z[i] - from) * c, e = __builtin_amdgcn_exp2f(d);
      own_s += e;
      own_b -= e * fmaxf(d, NOTHING);
    }
    add_to(s, s_over, own_s);
    add_to(b, b_over, own_b);
  }
};

// Rows that are read as often as they are gone through, BATCH vectors of 16 bytes to a thread at a time, with the next ones on their way.
// each(f) calls f(values, first column); values that do not fill a vector go to the first threads, one each.
template <class T, int THREADS>
struct Streamed {
  static constexpr int N = 16 / sizeof(T), BATCH = 4;
  static constexpr u32 STEP = BATCH * THREADS * N;
  const T* row;
  u32 vocab;
  __device__ __forceinline__ Streamed(const T* row_, i64 vocab_) : row(row_), vocab((u32)vocab_) {}
  __device__ __forceinline__ u32 whole() const { return vocab - vocab % N; }
  // (columns behind the last vector load that one: without a branch the loads of a batch are all on their way at once)
  __device__ __forceinline__ void load(Vec<T, N> (&v)[BATCH], u32 at) const {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) v[i] = load_vec<N>(row + min(at + i * THREADS * N, vocab - N));
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    const u32 end = whole();
    if (end) {
      u32 at = threadIdx.x * N;
      Vec<T, N> now[BATCH];
      load(now, at);
      for (u32 done = 0; done < end; done += STEP, at += STEP) {
        Vec<T, N> next[BATCH];
        if (done + STEP < end) load(next, at + STEP);
        auto use = [&](int i) {
          float z[N];
#pragma unroll
          for (int n = 0; n < N; ++n) z[n] = (float)now[i][n];
          f(z, (i64)(at + i * THREADS * N));
        };
        if (end - done >= STEP) {
#pragma unroll
          for (int i = 0; i < BATCH; ++i) use(i);
        } else {
#pragma unroll
          for (int i = 0; i < BATCH; ++i)
            if (at + i * THREADS * N < end) use(i);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) now[i] = next[i];
      }
    }
    if (threadIdx.x < vocab - end) {
      const float z[1] = {(float)row[end + threadIdx.x]};
      f(z, (i64)(end + threadIdx.x));
    }
  }
  // each(f) with the results stored to the same columns of `out`; `next` is not needed
  template <class F>
  __device__ __forceinline__ void write(T* out, const T*, F f) const {
    each([&](const auto& z, i64 at) {
      constexpr int S = sizeof(z) / sizeof(float);
      Vec<T, S> o;
      f(z, o);
      store_once<S>(out + at, o);
    });
  }
  // the thread that stores a column
  __device__ __forceinline__ int owner(int at) const { return (u32)at < whole() ? at / N % THREADS : at - (int)whole(); }
};

// Rows that stay in registers.  Vectors and values behind the row's end are the lowest.
typedef u32 words4 __attribute__((ext_vector_type(4)));
template <class T, int THREADS, int VECS>
struct Held {
  static constexpr int N = 16 / sizeof(T);
  words4 v[VECS];
  float rest;                       // one of the values that do not fill a vector
  int vocab;
  __device__ __forceinline__ int whole() const { return vocab - vocab % N; }
  __device__ __forceinline__ bool inside(int i) const {
    return (i + 1) * THREADS * N <= vocab || (i * THREADS + (int)threadIdx.x) * N < whole();       // (the first is known to the whole workgroup)
  }
  // (a scalar base and 32 bits of offset: with a pointer to each vector the registers would not suffice)
  template <class P>
  static __device__ __forceinline__ auto place(P* row, int i) {
    typedef typename std::conditional<std::is_const<P>::value, const char, char>::type byte;
    return reinterpret_cast<P*>(reinterpret_cast<byte*>(row) + i * THREADS * 16 + (u32)(threadIdx.x * 16));
  }
  __device__ __forceinline__ void load(const T* row, int i) {
    if (inside(i)) v[i] = __builtin_bit_cast(words4, load_once<N>(place(row, i)));
  }
  __device__ __forceinline__ void load_rest(const T* row) {
    if ((int)threadIdx.x < vocab - whole()) rest = (float)row[whole() + threadIdx.x];
  }
  __device__ __forceinline__ Held(const T* row, i64 vocab_) : rest(LOWEST), vocab((int)vocab_) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      Vec<T, N> x;
#pragma unroll
      for (int n = 0; n < N; ++n) x[n] = (T)LOWEST;
      v[i] = __builtin_bit_cast(words4, x);
      load(row, i);
    }
    load_rest(row);
  }
  // The values of vector i.  (They stay packed from one time to the next: the compiler would unpack them once for all, into twice the registers.)
  __device__ __forceinline__ void values(int i, float (&z)[N]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      u32 x = v[i][w];
      asm volatile("" : "+v"(x));
      v[i][w] = x;
    }
    const Vec<T, N> x = __builtin_bit_cast(Vec<T, N>, v[i]);
#pragma unroll
    for (int n = 0; n < N; ++n) z[n] = (float)x[n];
  }
  template <class F>
  __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      float z[N];
      values(i, z);
      f(z, (i * THREADS + (int)threadIdx.x) * N);
      __builtin_amdgcn_sched_barrier(0);          // one vector after another: what they need together would not fit
    }
    const float z[1] = {rest};
    f(z, (int)threadIdx.x < vocab - whole() ? whole() + (int)threadIdx.x : vocab);
  }
  // Results stored to the same columns of `out`; each vector makes room for the next row's, if there is one.
  template <class F>
  __device__ __forceinline__ void write(T* out, const T* next, F f) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      float z[N];
      values(i, z);
      Vec<T, N> o;
      f(z, o);
      if (inside(i)) store_once<N>(place(out, i), o);
      if (next) load(next, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    const float z[1] = {rest};
    Vec<T, 1> o;
    f(z, o);
    if ((int)threadIdx.x < vocab - whole()) out[whole() + threadIdx.x] = o[0];
    if (next) load_rest(next);
  }
  __device__ __forceinline__ int owner(int at) const { return at < whole() ? at / N % THREADS : at - whole(); }
};
template <class T, int THREADS, int VECS>
struct RowOf { typedef Held<T, THREADS, VECS> type; };
template <class T, int THREADS>
struct RowOf<T, THREADS, 0> { typedef Streamed<T, THREADS> type; };

// The largest of the workgroup's values and their sum.  place: of this call alone between two barriers of the caller's.
template <int THREADS>
__device__ __forceinline__ float max_of_all(float v, float (&place)[16]) {
  v = wave_max(v);
  if (lane_id() == 0) place[threadIdx.x / CCLD_WAVE] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / CCLD_WAVE; ++w) v = fmaxf(v, place[w]);
  return v;
}
template <int THREADS>
__device__ __forceinline__ float sum_of_all(float v, float (&place)[16]) {
  v = wave_total(v);
  if (lane_id() == 0) place[threadIdx.x / CCLD_WAVE] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < THREADS / CCLD_WAVE; ++w) v += place[w];
  return v;
}

// A value and its column as a number that is larger for larger values and, where these are equal, for lower columns.
__device__ __forceinline__ u64 key_of(float z, int at) {
  const u32 bits = __builtin_bit_cast(u32, z + 0.0f);           // one zero
  return (u64)(bits ^ (bits >> 31 ? ~0u : 0x80000000u)) << 32 | (u32)~at;
}
__device__ __forceinline__ float value_of(u64 key) {
  const u32 bits = (u32)(key >> 32);
  return __builtin_bit_cast(float, bits ^ (bits >> 31 ? 0x80000000u : ~0u));
}
__device__ __forceinline__ int column_of(u64 key) { return (int)~(u32)key; }

// The `top` largest values of a row, equal ones by the lower column: put(rank, value, column), column -1 for what is not there.
template <int THREADS>
struct Alternatives {
  static constexpr int ROOM = 1024;
  uint4 maxima[THREADS / 4];
  u64 key[ROOM], best[THREADS / CCLD_WAVE];
  u32 found;

  // all threads call this; most: the largest of the thread's values
  template <class ROW, class PUT>
  __device__ __forceinline__ void find(ROW& row, float most, int top, PUT put) {
    static_assert(THREADS == 4 * CCLD_WAVE && THREADS >= CCLD_TOP_MOST, "four maxima to a lane, as many as alternatives");
    const int me = threadIdx.x;
    __syncthreads();                        // the row before is done with
    if (me == 0) found = 0;
    reinterpret_cast<u32*>(maxima)[me] = (u32)(key_of(most, 0) >> 32);
    __syncthreads();
    // The largest number of 16 bits that at least `top` maxima reach, bit by bit, in every wavefront by itself (counting for each maximum those before it took 3 us).
    const uint4 o = maxima[lane_id()];
    u32 reached = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
      const u32 more = reached | 1u << bit;
      const int n = __builtin_popcountll(ballot64(o.x >= more)) + __builtin_popcountll(ballot64(o.y >= more)) +
                    __builtin_popcountll(ballot64(o.z >= more)) + __builtin_popcountll(ballot64(o.w >= more));
      reached = n >= top ? more : reached;
    }
    const float least = reached <= (u32)(key_of(LOWEST, 0) >> 32) ? LOWEST : value_of((u64)reached << 32);
    if (most >= least && most > LOWEST)
      row.each([&](const auto& z, i64 at) {
        const float largest = largest_of(z);
        if (largest >= least && largest > LOWEST) {
#pragma unroll
          for (int n = 0; n < (int)(sizeof(z) / sizeof(float)); ++n)
            if (z[n] >= least && z[n] > LOWEST) {
              const u32 to = atomicAdd(&found, 1u);
              if (to < ROOM) key[to] = key_of(z[n], (int)at + n);
            }
        }
      });
    __syncthreads();
    const u32 n = found;
    if (n <= ROOM) {
      for (u32 i = me; i < n; i += THREADS) {
        const u64 mine = key[i];
        int rank = 0;
#pragma unroll 8
        for (u32 o = 0; o < n; ++o) rank += key[o] > mine;
        if (rank < top) put(rank, value_of(mine), column_of(mine));
      }
      for (int i = me; i < top; i += THREADS)
        if (i >= (int)n) put(i, LOWEST, -1);
    } else {
      // one after another: the largest of those that come after the one before
      u64 last = ~0ull;
      for (int k = 0; k < top; ++k) {
        u64 next = 0;
        row.each([&](const auto& z, i64 at) {
#pragma unroll
          for (int n = 0; n < (int)(sizeof(z) / sizeof(float)); ++n) {
            const u64 x = key_of(z[n], (int)at + n);
            if (z[n] > LOWEST && x < last && x > next) next = x;
          }
        });
        next = wave_max_u64(next);
        __syncthreads();
        if (lane_id() == 0) best[me / CCLD_WAVE] = next;
        __syncthreads();
        for (int w = 0; w < THREADS / CCLD_WAVE; ++w) next = max(next, best[w]);
        last = next;
        if (me == 0) put(k, next ? value_of(next) : LOWEST, next ? column_of(next) : -1);
      }
    }
  }
};

// what a row's sums say
struct Values {
  float m, per, log_s, lse, entropy;
  bool nan;
  __device__ __forceinline__ Values(const Sums& x, float temperature) : m(x.m), nan(x.s != x.s) {
    const bool none = x.m == LOWEST && x.s == 0;
    per = temperature;
    log_s = logf(x.s);
    // (a row that is not empty has a finite lse, at a low temperature too, by which the gradient knows it; NaN stays)
    lse = none ? LOWEST : m / temperature + log_s;
    if (!none && fabsf(lse) > __FLT_MAX__) lse = copysignf(__FLT_MAX__, lse);
    entropy = none ? 0.0f : log_s + x.b * LN2 / x.s;
  }
  __device__ __forceinline__ float logp(float z) const { return z == LOWEST && !nan ? LOWEST : (z - m) / per - log_s; }
};
template <class T>
__device__ __forceinline__ void put_values(const LogprobJob& j, i64 r, const Values& v) {
  const i64 t = token_of(j, r);
  j.logp[r] = t < 0 ? 0.0f : v.logp((float)static_cast<const T*>(j.logits)[r * j.ld + t]);
  j.lse[r] = v.lse;
  j.entropy[r] = v.entropy;
}

// A row, or (j.parts > 1) a part of one, to a workgroup.
// VECS: the parts are held in registers; 0: read as often as they are gone through
template <class T, int THREADS, int VECS>
__global__ __launch_bounds__(THREADS) void k_logprobs(LogprobJob j) {
  __shared__ float places[3][16];
  __shared__ Alternatives<THREADS> alternatives;
  const float c = LOG2E / j.temperature;
  for (i64 b = blockIdx.x; b < j.rows * j.parts; b += gridDim.x) {
    const i64 r = b / j.parts, start = (b - r * j.parts) * j.span;
    typename RowOf<T, THREADS, VECS>::type row(static_cast<const T*>(j.logits) + r * j.ld + start, min(j.span, j.vocab - start));
    Sums x;
    row.each([&](const auto& z, auto) { x.add(z, c); });
    const float most = x.most;
    __syncthreads();                        // the row before is done with
    x.move(max_of_all<THREADS>(most, places[0]), c);
    x.s = sum_of_all<THREADS>(x.s - x.s_over, places[1]);
    x.b = sum_of_all<THREADS>(x.b - x.b_over, places[2]);
    if (j.parts > 1) {
      if (threadIdx.x == 0) { j.part_sums[3 * b] = x.m; j.part_sums[3 * b + 1] = x.s; j.part_sums[3 * b + 2] = x.b; }
      if (j.top)
        alternatives.find(row, most, j.top, [&](int rank, float z, int at) {
          j.part_values[b * j.top + rank] = z;
          j.part_ids[b * j.top + rank] = at < 0 ? -1 : (int)start + at;
        });
    } else {
      const Values v(x, j.temperature);
      if (threadIdx.x == 0) put_values<T>(j, r, v);
      if (j.top)
        alternatives.find(row, most, j.top, [&](int rank, float z, int at) {
          j.top_ids[r * j.top + rank] = at;
          j.top_logp[r * j.top + rank] = at < 0 ? LOWEST : v.logp(z);
        });
    }
  }
}

// The alternatives of a row's parts, as a row.
struct Candidates {
  const float* value;
  const int* id;
  int n;
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    for (int i = threadIdx.x; i < n; i += JOIN_THREADS) {
      const float z[1] = {value[i]};
      f(z, (i64)id[i]);
    }
  }
};
template <class T>
__global__ __launch_bounds__(JOIN_THREADS) void k_logprobs_join(LogprobJob j) {
  __shared__ Alternatives<JOIN_THREADS> alternatives;
  const float c = LOG2E / j.temperature;
  for (i64 r = blockIdx.x; r < j.rows; r += gridDim.x) {
    // every wavefront by itself: a part to a lane
    Sums x;
    const u32 part = lane_id();
    if (part < j.parts) {
      const float* const at = j.part_sums + 3 * (r * j.parts + part);
      x.m = at[0]; x.s = at[1]; x.b = at[2];
    }
    x.move(wave_max(x.m), c);
    x.s = wave_total(x.s);
    x.b = wave_total(x.b);
    const Values v(x, j.temperature);
    if (threadIdx.x == 0) put_values<T>(j, r, v);
    if (!j.top) continue;
    const i64 first = r * j.parts * j.top;
    Candidates row{j.part_values + first, j.part_ids + first, (int)j.parts * j.top};
    float most = LOWEST;
    row.each([&](const auto& z, i64) { most = fmaxf(most, z[0]); });
    alternatives.find(row, most, j.top, [&](int rank, float z, int at) {
      j.top_ids[r * j.top + rank] = at;
      j.top_logp[r * j.top + rank] = at < 0 ? LOWEST : v.logp(z);
    });
  }
}

// lse says where to measure from.  Beyond 2^20 it does not say it well enough and the largest logit is looked for.
constexpr float FAR = 0x1p20f;

template <class T, int THREADS, int VECS>
__global__ __launch_bounds__(THREADS) void k_logprobs_grad(LogprobJob j) {
  __shared__ float places[2][2][16];
  const float c = LOG2E / j.temperature, per = 1.0f / j.temperature;
  int turn = 0;
  i64 r = blockIdx.x;
  const T* logits = static_cast<const T*>(j.logits) + r * j.ld;
  typename RowOf<T, THREADS, VECS>::type held(logits, j.vocab);
  for (; r < j.rows; r += gridDim.x) {
    const T* const next = r + gridDim.x < j.rows ? logits + gridDim.x * j.ld : nullptr;
    T* const out = static_cast<T*>(j.dlogits) + r * j.ldd;
    const float lse = j.lse[r], entropy = j.entropy[r];
    const int t = (int)token_of(j, r);
    const bool none = lse == LOWEST;
    const float dl = !none && t >= 0 && j.dlogp ? j.dlogp[r * j.dlogp_stride] : 0.0f, de = !none && j.dentropy ? j.dentropy[r * j.dentropy_stride] : 0.0f;
    float from = none ? 0.0f : lse * j.temperature, s = 0, over = 0, rest = 0;
    if (!none) {
      if (!(fabsf(lse) < FAR)) {
        float m = LOWEST;
        held.each([&](const auto& z, auto) { m = fmaxf(m, largest_of(z)); });
        from = max_of_all<THREADS>(m, places[turn][1]);
      }
      held.each([&](const auto& z, auto) {
        float own = 0;
#pragma unroll
        for (int n = 0; n < (int)(sizeof(z) / sizeof(float)); ++n) own += __builtin_amdgcn_exp2f((z[n] - from) * c);
        if constexpr (VECS == 0) add_to(s, over, own);
        else s += own;                      // (17 of them at most)
      });
      rest = log2f(sum_of_all<THREADS>(s - over, places[turn][0]));
      turn ^= 1;                            // (a place is written again behind the next row's barrier)
    }
    // dlogits without the target's own: -p (k0 + k1 log2 p)
    const float k0 = -(none ? 0.0f : dl + de * entropy) * per, k1 = -de * LN2 * per;
    auto gradient = [&](float z) {
      const float d = (z - from) * c - rest;
      return __builtin_amdgcn_exp2f(d) * (k1 * fmaxf(d, NOTHING) + k0);
    };
    held.write(out, next, [&](const auto& z, auto& o) {
#pragma unroll
      for (int n = 0; n < (int)(sizeof(z) / sizeof(float)); ++n) o[n] = (T)gradient(z[n]);
    });
    // (behind the same thread's store to the same place)
    if (t >= 0 && (int)threadIdx.x == held.owner(t)) out[t] = (T)(dl * per + gradient((float)logits[t]));
    if constexpr (VECS == 0) held.row = next;
    logits = next;
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
                    a->dlogp_stride, a->dentropy_stride, a->rows, a->vocab, a->temperature, a->top, a->token_bits, 1, a->vocab, 0};
}
// Few long rows are cut into parts of 4 or 8 vectors to a thread, which stay in registers (longer ones, where there would be more than MOST_PARTS, do not).  With 20 alternatives,
// in parts of 4, of 8, and whole, bfloat16: 3 x 128,000 13.0, 14.3 and 23 us; 64 x 128,000 16.5, 16.5 and 32.6; 256 x 128,000 33.9, 29.1 and 38.1; 400 x 128,000 46.9, 40.1 and 44.6; 600 x 128,000 64.8, 53.0 and 54.1;
// 64 x 20,000 13.3, 15.0 and 12.5; 128 x 32,000 14.0, 15.2 and 15.1; 600 x 32,000 24.7, 24.3 and 19.9.
constexpr i64 MOST_PARTS = CCLD_WAVE, LEAST_PARTS = 5;
constexpr int THREADS = 256;
void cut_rows(LogprobJob& j, int32_t dtype, uint8_t* workspace, uint64_t* bytes) {
  const i64 n = 16 / size_of(dtype);
  auto parts = [&](int vecs) { return blocks_for(j.vocab, vecs * THREADS * n); };
  auto fits = [&](int vecs, i64 groups) { return parts(vecs) <= MOST_PARTS && j.rows * parts(vecs) <= groups * (i64)COMPUTE_UNITS; };
  *bytes = 0;
  if (parts(4) < LEAST_PARTS) return;
  j.held = fits(4, 4) ? 4 : fits(8, 16) ? 8 : 0;
  if (j.held) j.span = j.held * THREADS * n;
  else if (parts(8) > MOST_PARTS) j.span = blocks_for(blocks_for(j.vocab, n), std::max<i64>(1, std::min(MOST_PARTS, 2 * (i64)COMPUTE_UNITS / std::max<i64>(j.rows, 1)))) * n;
  j.parts = blocks_for(j.vocab, j.span);
  if (j.parts == 1) return;
  auto take = [&](i64 each) {
    uint8_t* const at = workspace ? workspace + *bytes : nullptr;
    *bytes += ((uint64_t)(j.rows * j.parts * each) + 255) & ~(uint64_t)255;
    return at;
  };
  j.part_sums = reinterpret_cast<float*>(take(12));
  j.part_values = reinterpret_cast<float*>(take(4 * j.top));
  j.part_ids = reinterpret_cast<int*>(take(4 * j.top));
}

template <class T, int THREADS, int VECS>
void launch_grad(const LogprobJob& j, hipStream_t stream) {
  // 16 wavefronts to a compute unit, each workgroup with rows one after another
  const i64 most = VECS >= 8 ? (i64)COMPUTE_UNITS * 1024 / THREADS : 1 << 20;
  k_logprobs_grad<T, THREADS, VECS><<<(u32)std::min(j.rows, most), THREADS, 0, stream>>>(j);
}
// the smallest form that holds a row
template <class T>
void launch_grad(const LogprobJob& j, hipStream_t stream) {
  constexpr i64 N = 16 / sizeof(T);
  const i64 vectors = blocks_for(j.vocab, N);
  if (vectors <= 256) launch_grad<T, 256, 1>(j, stream);
  else if (vectors <= 256 * 4) launch_grad<T, 256, 4>(j, stream);
  else if (vectors <= 256 * 8) launch_grad<T, 256, 8>(j, stream);
  else if (vectors <= 256 * 16) launch_grad<T, 256, 16>(j, stream);
  else if (vectors <= 512 * 16) launch_grad<T, 512, 16>(j, stream);
  else if (vectors <= 1024 * 16) launch_grad<T, 1024, 16>(j, stream);
  else if (j.rows < 2 * (i64)COMPUTE_UNITS) launch_grad<T, 1024, 0>(j, stream);
  else launch_grad<T, 256, 0>(j, stream);
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
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  LogprobJob j = make_job(a);
  cut_rows(j, a->dtype, nullptr, bytes);
  return CCLD_OK;
}

extern "C" ccld_status ccld_token_logprobs(const ccld_logprob_args* a, void* stream) {
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  if (a->rows && (!a->logits || !a->tokens || !a->logp || !a->entropy || !a->lse || (a->top && (!a->top_ids || !a->top_logp)))) return CCLD_E_NULL;
  if (a->ldlogits < a->vocab || !all_aligned(a)) return CCLD_E_BAD_ARG;
  if (a->rows == 0) return CCLD_OK;
  LogprobJob j = make_job(a);
  uint64_t need;
  cut_rows(j, a->dtype, static_cast<uint8_t*>(a->workspace), &need);
  if (need && (need > a->workspace_bytes || !a->workspace || !aligned(a->workspace, 256))) return CCLD_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const u32 grid = (u32)std::min<i64>(j.rows * j.parts, 1 << 20);
  with_type(a->dtype, [&](auto zero) {
    using T = decltype(zero);
    if (j.held == 4) k_logprobs<T, THREADS, 4><<<grid, THREADS, 0, st>>>(j);
    else if (j.held == 8) k_logprobs<T, THREADS, 8><<<grid, THREADS, 0, st>>>(j);
    else k_logprobs<T, THREADS, 0><<<grid, THREADS, 0, st>>>(j);
    if (j.parts > 1) k_logprobs_join<T><<<(u32)j.rows, JOIN_THREADS, 0, st>>>(j);
  });
  return launched();
}

extern "C" ccld_status ccld_token_logprobs_grad(const ccld_logprob_args* a, void* stream) {
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  if (a->rows && (!a->logits || !a->tokens || !a->entropy || !a->lse || !a->dlogits)) return CCLD_E_NULL;
  if (a->ldlogits < a->vocab || a->lddlogits < a->vocab || !all_aligned(a)) return CCLD_E_BAD_ARG;
  if (a->rows == 0) return CCLD_OK;
  with_type(a->dtype, [&](auto zero) { launch_grad<decltype(zero)>(make_job(a), static_cast<hipStream_t>(stream)); });
  return launched();
}
