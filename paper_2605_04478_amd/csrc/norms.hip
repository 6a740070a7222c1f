// The norms before and after a block, fused with its gate and the scale of the residual stream, and their gradient (ccld_norm_*).
//
//   r1 = 1 / sqrt(mean(b^2) + eps)     n = b r1 w_post     x = scale h + gate n     (h' = x rounded)
//   r2 = 1 / sqrt(mean(x^2) + eps)     u = x r2 w_pre
//
//   dx = dh' + r2 (du w_pre - x r2^2 mean(du w_pre x))      dh = scale dx      dgate = sum dx n
//   dn = dx gate      db = r1 (dn w_post - b r1^2 mean(dn w_post b))      dw_post = sum dn b r1      dw_pre = sum du x r2
//
// Memory bounds both: a dozen operations per element, each row read once and kept in registers between its two reductions.  A
// row belongs to one wavefront where it is short, else to a workgroup.  The gradient takes x from h and b again, which costs no more
// bytes than reading h' and is exact; its sums over rows are kept in registers by teams that take many rows each, and joined by a
// second kernel in the teams' order.
//
// Measured (a copy of 2 GB moves 4.9 TB/s here, an elementwise sum 6.0): 32,768 x 8,192 in bfloat16 372 us = 5.8 TB/s; 16,384 x 4,096 92 us = 5.8 TB/s
// forward and 163 us = 5.0 TB/s of the bytes that the gradient needs (6 reads and writes of a row), with 6 us for the join; 3,003 x 2,500 in 32 bits 21, 35
// and 6 us.  One row: 3 us of a call's 6.
#include <algorithm>

#include "ccld_internal.h"
#include "products.h"
#include "tiles.h"

using namespace ccld;

namespace {

// A thread has PIECES x 8 of a row's columns, in vectors of VEC: 16 bytes (VEC 8 or 4) where rows are made of whole words, else single
// values.  The vectors of a team's TEAM threads lie side by side.
template <class T>
using Piece = T __attribute__((ext_vector_type(8)));

template <int TEAM, int VEC>
__device__ __forceinline__ int column(int t, int p, int i) { return ((p * (8 / VEC) + i / VEC) * TEAM + t) * VEC + i % VEC; }

// A row as a buffer of its d values: columns beyond them load zeros and are not stored, without a branch (words of 32 bits are checked one by
// one, so that a vector may reach over the end).  Every value of a row that is not
// there (no pointer) is zero.
template <class T>
__device__ __forceinline__ auto row_buffer(const T* row, int d) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(row), 0, row ? d * (int)sizeof(T) : 0, 0x00027000);
}
typedef u32 u32x4 __attribute__((ext_vector_type(4)));

template <int TEAM, int VEC, class T>
__device__ __forceinline__ Piece<T> load_piece(const T* row, int t, int p, int d) {
  Piece<T> v;
  const auto buffer = row_buffer(row, d);
#pragma unroll
  for (int i = 0; i < 8; i += VEC) {
    const int at = column<TEAM, VEC>(t, p, i) * (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(VEC)));
    vec q;
    if constexpr (VEC > 1) q = __builtin_bit_cast(vec, __builtin_amdgcn_raw_buffer_load_b128(buffer, at, 0, 0));
    else if constexpr (sizeof(T) == 4) q = __builtin_bit_cast(vec, __builtin_amdgcn_raw_buffer_load_b32(buffer, at, 0, 0));
    else q = __builtin_bit_cast(vec, __builtin_amdgcn_raw_buffer_load_b16(buffer, at, 0, 0));
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[i + e] = q[e];
  }
  return v;
}
template <int TEAM, int VEC, class T>
__device__ __forceinline__ void store_piece(T* row, const float (&v)[8], int t, int p, int d) {
  const auto buffer = row_buffer(row, d);
  if constexpr (VEC > 1) {
    constexpr int N = 16 / sizeof(T);            // values of the stored type to 16 bytes: fewer than VEC where sums of 32 bits leave
#pragma unroll
    for (int i = 0; i < 8; i += N) {
      typedef T vec __attribute__((ext_vector_type(N)));
      vec q;
#pragma unroll
      for (int e = 0; e < N; ++e) q[e] = (T)v[i + e];
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, q), buffer, column<TEAM, VEC>(t, p, i) * (int)sizeof(T), 0, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = column<TEAM, 1>(t, p, i) * (int)sizeof(T);
      const T x = (T)v[i];
      if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(u32, x), buffer, at, 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, x), buffer, at, 0, 0);
    }
  }
}

// The sums of N values over a row's threads.  Teams of several wavefronts are workgroups: a call's place in LDS is written
// again by the call after the next, so one barrier is enough.
template <int TEAM, int N>
__device__ __forceinline__ void team_sums(float (&v)[N], float (&place)[16][4]) {
#pragma unroll
  for (int m = CCLD_WAVE / 2; m >= 1; m >>= 1)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += __shfl_xor(v[n], m, CCLD_WAVE);
  if constexpr (TEAM > CCLD_WAVE) {
    if (lane_id() == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) place[threadIdx.x / CCLD_WAVE][n] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = 0;
#pragma unroll
    for (int i = 0; i < TEAM / CCLD_WAVE; ++i)
#pragma unroll
      for (int n = 0; n < N; ++n) v[n] += place[i][n];
  }
}

struct NormJob {
  const void *h, *b, *gate, *w_post, *w_pre, *dh_out, *du;
  void *h_out, *u, *dh, *db, *dgate;
  float *rstd_post, *rstd_pre;
  i64 ldh, ldb, ldgate, ldh_out, ldu, lddh_out, lddu, lddh, lddb;
  i64 rows, rows_per_gate;
  i64 row0;                      // first row of the launch (forward)
  int d;
  float scale, eps;
  // gradient: the rows in chunks that lie within a gate's, and where sums go
  i64 chunks, chunk_rows;
  u32 chunks_per_gate;
  float *part_post, *part_pre;   // [teams][d]
  float* part_gate;              // [chunks][d], or null: a gate's rows are one chunk and its sum leaves at once
};

// a team of one wavefront shares a workgroup with three others
template <int TEAM>
constexpr int threads_of() { return TEAM == CCLD_WAVE ? 256 : TEAM; }

template <class T, int TEAM, int PIECES, int VEC>
__global__ __launch_bounds__(threads_of<TEAM>()) void k_norm(NormJob j) {
  __shared__ float places[2][16][4];
  const int t = threadIdx.x % TEAM;
  i64 row = blockIdx.x;
  if (threads_of<TEAM>() > TEAM) row = row * (threads_of<TEAM>() / TEAM) + __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM);
  row += j.row0;
  if (row >= j.rows) return;                       // whole teams
  Piece<T> pb[PIECES], ph[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    pb[p] = load_piece<TEAM, VEC>(static_cast<const T*>(j.b) + row * j.ldb, t, p, j.d);
    ph[p] = load_piece<TEAM, VEC>(static_cast<const T*>(j.h) + row * j.ldh, t, p, j.d);
  }
  float sum[1] = {0};
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[0] += (float)pb[p][i] * (float)pb[p][i];
  team_sums<TEAM>(sum, places[0]);
  const float r1 = 1.0f / sqrtf(sum[0] / (float)j.d + j.eps);
  const T* gate = j.gate ? static_cast<const T*>(j.gate) + row / j.rows_per_gate * j.ldgate : nullptr;
  float x[PIECES][8];
  sum[0] = 0;
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const Piece<T> w = load_piece<TEAM, VEC>(static_cast<const T*>(j.w_post), t, p, j.d);
    Piece<T> g;
    if (gate) g = load_piece<TEAM, VEC>(gate, t, p, j.d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float n = (float)pb[p][i] * r1 * (float)w[i];
      x[p][i] = j.scale * (float)ph[p][i] + (gate ? (float)g[i] * n : n);
      sum[0] += x[p][i] * x[p][i];
    }
    store_piece<TEAM, VEC>(static_cast<T*>(j.h_out) + row * j.ldh_out, x[p], t, p, j.d);
  }
  team_sums<TEAM>(sum, places[1]);
  const float r2 = 1.0f / sqrtf(sum[0] / (float)j.d + j.eps);
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const Piece<T> w = load_piece<TEAM, VEC>(static_cast<const T*>(j.w_pre), t, p, j.d);
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = x[p][i] * r2 * (float)w[i];
    store_piece<TEAM, VEC>(static_cast<T*>(j.u) + row * j.ldu, u, t, p, j.d);
  }
  if (t == 0) {
    j.rstd_post[row] = r1;
    j.rstd_pre[row] = r2;
  }
}

// Values that stay packed in registers: the compiler cannot unpack them once for all rows, which would take twice the registers.
template <class T>
__device__ __forceinline__ void keep_packed(Piece<T>& v) {
  typedef u32 words __attribute__((ext_vector_type(sizeof(Piece<T>) / 4)));
  words w = __builtin_bit_cast(words, v);
#pragma unroll
  for (int i = 0; i < (int)sizeof(Piece<T>) / 4; ++i) {
    u32 x = w[i];
    asm volatile("" : "+v"(x));
    w[i] = x;
  }
  v = __builtin_bit_cast(Piece<T>, w);
}

// With e = du w_pre and q = gate w_post b both means follow from sums that need neither, so that a row has one reduction:
//   mean(du w_pre x) = sum(e x) / d      sum(dn w_post b) = sum(q (dh' + r2 e)) - m2 sum(q x)      (m2 = r2^3 mean(e x))
// 128 registers for 16-bit vectors, so that 16 wavefronts run on a compute unit (8 otherwise), each with its next row on the way while it
// computes one (ROWS_AHEAD).  Where that does not fit, a row is kept and the weights are loaded for each (ROWS_KEPT: 4,097 to 8,192 columns of
// 32 bits), or the row is read again, from the caches, after its reduction (ROWS_AGAIN: more than 8,192 columns).
enum { ROWS_AHEAD, ROWS_KEPT, ROWS_AGAIN };
template <class T, int TEAM, int PIECES, int VEC, int ROWS>
__global__ __launch_bounds__(threads_of<TEAM>(), TEAM == 1024 || (sizeof(T) == 2 && VEC > 1) ? 4 : 2) void k_norm_grad(NormJob j) {
  constexpr int PER_GROUP = threads_of<TEAM>() / TEAM;
  __shared__ float places[2][16][4];
  const int t = threadIdx.x % TEAM;
  // (rows are known to be the same for a wavefront: their addresses stay in scalar registers)
  const i64 team = PER_GROUP == 1 ? (i64)blockIdx.x : (i64)blockIdx.x * PER_GROUP + __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM);
  const i64 teams = (i64)gridDim.x * PER_GROUP;
  float s_post[PIECES][8] = {}, s_pre[PIECES][8] = {}, s_gate[PIECES][8] = {};
  const float per_d = 1.0f / (float)j.d;
  struct Columns { Piece<T> b, h, dh, du; };
  struct Rstd { float post, pre; };
  struct Weights { Piece<T> post, pre, gate; };
  auto load = [&](i64 row, int p, bool there = true) {
    Columns c;
    c.b = load_piece<TEAM, VEC>(there ? static_cast<const T*>(j.b) + row * j.ldb : nullptr, t, p, j.d);
    c.h = load_piece<TEAM, VEC>(there ? static_cast<const T*>(j.h) + row * j.ldh : nullptr, t, p, j.d);
    c.dh = load_piece<TEAM, VEC>(there && j.dh_out ? static_cast<const T*>(j.dh_out) + row * j.lddh_out : nullptr, t, p, j.d);
    c.du = load_piece<TEAM, VEC>(there && j.du ? static_cast<const T*>(j.du) + row * j.lddu : nullptr, t, p, j.d);
    return c;
  };
  auto load_rstd = [&](i64 row) { return Rstd{j.rstd_post[row], j.rstd_pre[row]}; };
  auto load_weights = [&](const T* gate, int p) {
    Weights w;
    w.post = load_piece<TEAM, VEC>(static_cast<const T*>(j.w_post), t, p, j.d);
    w.pre = load_piece<TEAM, VEC>(static_cast<const T*>(j.w_pre), t, p, j.d);
    if (gate) w.gate = load_piece<TEAM, VEC>(gate, t, p, j.d);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) w.gate[i] = (T)1.0f;
    return w;
  };
  // x and y = dh' + r2 e of a thread's columns
  auto values = [&](const Columns& c, const Weights& w, float r1, float r2, float (&x)[8], float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = j.scale * (float)c.h[i] + (float)w.gate[i] * (float)w.post[i] * (float)c.b[i] * r1;
      y[i] = (float)c.dh[i] + r2 * ((float)c.du[i] * (float)w.pre[i]);
    }
  };
  int turn = 0;
  for (i64 chunk = team; chunk < j.chunks; chunk += teams) {
    const i64 g = chunk / j.chunks_per_gate, in = chunk - g * j.chunks_per_gate;
    const i64 row0 = g * j.rows_per_gate + in * j.chunk_rows;
    const i64 row1 = min(row0 + j.chunk_rows, (g + 1) * j.rows_per_gate);
    const T* gate = j.gate ? static_cast<const T*>(j.gate) + g * j.ldgate : nullptr;
    if (row0 >= row1) continue;
    Columns next[PIECES];
    Weights w[PIECES];
    Rstd next_rstd = load_rstd(row0);
    if constexpr (ROWS == ROWS_AHEAD) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        w[p] = load_weights(gate, p);
        next[p] = load(row0, p);
      }
    }
    for (i64 row = row0; row < row1; ++row) {
      // (the row after the last is loaded as zeros: a branch would make the compiler wait for loads that it cannot count)
      const float r1 = next_rstd.post, r2 = next_rstd.pre;
      const bool more = row + 1 < row1;
      next_rstd = load_rstd(more ? row + 1 : row);
      Columns now[PIECES];
      float x[PIECES][8], y[PIECES][8], sum[3] = {0, 0, 0};
      if constexpr (ROWS == ROWS_AHEAD) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
          now[p] = next[p];
          next[p] = load(row + 1, p, more);
          keep_packed<T>(w[p].post);
          keep_packed<T>(w[p].pre);
          keep_packed<T>(w[p].gate);
        }
      }
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        if constexpr (ROWS != ROWS_AHEAD) { now[p] = load(row, p); w[p] = load_weights(gate, p); }
        values(now[p], w[p], r1, r2, x[p], y[p]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float q = (float)w[p].gate[i] * (float)w[p].post[i] * (float)now[p].b[i], du = (float)now[p].du[i];
          s_pre[p][i] += du * x[p][i] * r2;
          sum[0] += du * (float)w[p].pre[i] * x[p][i];
          sum[1] += q * y[p][i];
          sum[2] += q * x[p][i];
        }
      }
      team_sums<TEAM>(sum, places[turn]);
      turn ^= 1;
      const float m2 = sum[0] * per_d * r2 * r2 * r2, m1 = (sum[1] - m2 * sum[2]) * per_d * r1 * r1;
      i64 again = row;
      asm volatile("" : "+s"(again));           // not the values from before the reduction
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        if constexpr (ROWS == ROWS_KEPT) w[p] = load_weights(gate, p);
        if constexpr (ROWS == ROWS_AGAIN) { now[p] = load(again, p); w[p] = load_weights(gate, p); values(now[p], w[p], r1, r2, x[p], y[p]); }
        float dh[8], db[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float b = (float)now[p].b[i], w1 = (float)w[p].post[i], dx = y[p][i] - x[p][i] * m2, nb = b * r1;
          const float dn = dx * (float)w[p].gate[i];
          dh[i] = j.scale * dx;
          s_gate[p][i] += dx * nb * w1;
          s_post[p][i] += dn * nb;
          db[i] = r1 * (dn * w1 - b * m1);
        }
        store_piece<TEAM, VEC>(static_cast<T*>(j.dh) + row * j.lddh, dh, t, p, j.d);
        store_piece<TEAM, VEC>(static_cast<T*>(j.db) + row * j.lddb, db, t, p, j.d);
      }
    }
    if (j.dgate) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        if (j.part_gate) store_piece<TEAM, VEC>(j.part_gate + chunk * j.d, s_gate[p], t, p, j.d);
        else store_piece<TEAM, VEC>(static_cast<T*>(j.dgate) + g * j.d, s_gate[p], t, p, j.d);
#pragma unroll
        for (int i = 0; i < 8; ++i) s_gate[p][i] = 0;
      }
    }
  }
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    store_piece<TEAM, VEC>(j.part_post + team * j.d, s_post[p], t, p, j.d);
    store_piece<TEAM, VEC>(j.part_pre + team * j.d, s_pre[p], t, p, j.d);
  }
}

struct SumJob {
  const float *part_post, *part_pre, *part_gate;
  void *dw_post, *dw_pre, *dgate;
  i64 teams;
  u32 chunks_per_gate;
  u32 sums;                      // two weights, and the gates whose rows are in several chunks (or in none)
  int d;
};

// Sums over the teams, 64 columns to a workgroup: a wavefront's rows one after another, then the wavefronts' sums.
constexpr int SUM_THREADS = 1024;
template <class T>
__global__ __launch_bounds__(SUM_THREADS) void k_norm_sums(SumJob j) {
  __shared__ float sums[SUM_THREADS / CCLD_WAVE][CCLD_WAVE];
  const int lane = (int)lane_id(), wave = threadIdx.x / CCLD_WAVE, c = blockIdx.x * CCLD_WAVE + lane;
  for (u32 what = blockIdx.y; what < j.sums; what += gridDim.y) {
    const float* p = what == 0 ? j.part_post : what == 1 ? j.part_pre : j.part_gate + (i64)(what - 2) * j.chunks_per_gate * j.d;
    T* out = static_cast<T*>(what == 0 ? j.dw_post : what == 1 ? j.dw_pre : j.dgate) + (what < 2 ? 0 : (i64)(what - 2) * j.d);
    const i64 n = what < 2 ? j.teams : j.chunks_per_gate;
    float s = 0;
    if (c < j.d) {
      i64 r = wave;
      constexpr int AT_ONCE = 8;
      for (; r + (AT_ONCE - 1) * (SUM_THREADS / CCLD_WAVE) < n; r += AT_ONCE * (SUM_THREADS / CCLD_WAVE)) {
        float v[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) v[i] = p[(r + i * (SUM_THREADS / CCLD_WAVE)) * j.d + c];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) s += v[i];
      }
      for (; r < n; r += SUM_THREADS / CCLD_WAVE) s += p[r * j.d + c];
    }
    __syncthreads();                   // the sums before are read
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < j.d) {
      s = 0;
#pragma unroll
      for (int i = 0; i < SUM_THREADS / CCLD_WAVE; ++i) s += sums[i][lane];
      out[c] = (T)s;
    }
  }
}

i64 div_up(i64 a, i64 b) { return (a + b - 1) / b; }

// Threads to a row of the gradient, which keeps three sums per column in registers: 8 columns each, 16 of the widest rows.
int grad_team(i64 d) { return d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024; }

struct Plan { int team; i64 groups, teams, chunks, chunk_rows; u32 chunks_per_gate; float *part_post, *part_pre, *part_gate; u64 bytes; };

Plan make_plan(const ccld_norm_args* a, uint8_t* base) {
  Plan p{};
  p.team = grad_team(a->d);
  const i64 per_group = p.team == CCLD_WAVE ? 4 : 1, gates = a->gate ? a->groups : 1;
  // 16 wavefronts to a compute unit, 8 of teams of one; as many chunks, so that each team has one, or one for each gate
  const i64 want = std::max<i64>(1, std::min<i64>(a->rows, (i64)COMPUTE_UNITS * (p.team == CCLD_WAVE ? 8 : 1024 / p.team)));
  const i64 per_gate = a->rows / gates;
  p.chunks_per_gate = (u32)std::max<i64>(1, std::min(per_gate, want / gates));
  p.chunk_rows = div_up(per_gate, p.chunks_per_gate);
  p.chunks_per_gate = (u32)std::max<i64>(1, p.chunk_rows ? div_up(per_gate, p.chunk_rows) : 1);
  p.chunks = a->rows ? gates * p.chunks_per_gate : 0;
  p.groups = div_up(std::min(p.chunks, want), per_group);
  p.teams = p.groups * per_group;
  auto take = [&](i64 rows) {
    float* at = base ? reinterpret_cast<float*>(base + p.bytes) : nullptr;
    p.bytes += ((u64)rows * a->d * 4 + 255) & ~(u64)255;
    return at;
  };
  p.part_post = take(p.teams);
  p.part_pre = take(p.teams);
  if (a->gate && a->dgate && p.chunks_per_gate > 1) p.part_gate = take(p.chunks);
  return p;
}

i64 element_bytes(const ccld_norm_args* a) { return a->dtype == CCLD_FP32 ? 4 : 2; }

ccld_status check(const ccld_norm_args* a) {
  if (!a) return CCLD_E_NULL;
  if (a->dtype != CCLD_BF16 && a->dtype != CCLD_FP16 && a->dtype != CCLD_FP32) return CCLD_E_BAD_ARG;
  if (a->rows < 0 || a->d < 1 || a->groups < 1 || (a->gate && a->rows % a->groups)) return CCLD_E_BAD_ARG;
  if (a->rows >= MAX_ROWS || a->groups >= MAX_ROWS || a->d > CCLD_NORM_MAX) return CCLD_E_CAPACITY;
  if (!(a->eps >= 0)) return CCLD_E_BAD_ARG;
  return CCLD_OK;
}

template <class... P>
bool all_aligned(uintptr_t bytes, P... p) { return (aligned(p, bytes) && ...); }
template <class... L>
bool all_at_least(i64 d, L... l) { return ((l >= d) && ...); }
// Vectors of 16 bytes need rows that are made of whole words of 32 bits: buffers are checked, and may be aligned, by the word.
bool wide(const ccld_norm_args* a, bool grad) {
  const i64 word = 4 / element_bytes(a);
  auto words = [&](i64 ld, const void* p) { return !p || (ld % word == 0 && aligned(p, 4)); };
  const bool w = a->d % word == 0 && words(a->ldh, a->h) && words(a->ldb, a->b) && words(a->ldgate, a->gate) && words(0, a->w_post) && words(0, a->w_pre);
  if (!grad) return w && words(a->ldh_out, a->h_out) && words(a->ldu, a->u);
  return w && words(a->lddh, a->dh) && words(a->lddb, a->db) && words(0, a->dgate) && words(a->lddh_out, a->dh_out) && words(a->lddu, a->du);
}

NormJob make_job(const ccld_norm_args* a) {
  NormJob j{};
  j.h = a->h; j.b = a->b; j.gate = a->gate; j.w_post = a->w_post; j.w_pre = a->w_pre; j.dh_out = a->dh_out; j.du = a->du;
  j.h_out = a->h_out; j.u = a->u; j.dh = a->dh; j.db = a->db; j.dgate = a->gate ? a->dgate : nullptr;
  j.rstd_post = a->rstd_post; j.rstd_pre = a->rstd_pre;
  j.ldh = a->ldh; j.ldb = a->ldb; j.ldgate = a->ldgate; j.ldh_out = a->ldh_out; j.ldu = a->ldu; j.lddh_out = a->lddh_out;
  j.lddu = a->lddu; j.lddh = a->lddh; j.lddb = a->lddb;
  j.rows = a->rows;
  j.rows_per_gate = a->gate ? std::max<i64>(a->rows / a->groups, 1) : std::max<i64>(a->rows, 1);
  j.d = (int)a->d;
  j.scale = a->scale; j.eps = a->eps;
  return j;
}

template <class T, int TEAM, int PIECES>
void launch_forward(NormJob j, bool w, hipStream_t stream) {
  constexpr int THREADS = threads_of<TEAM>(), VEC = 16 / sizeof(T), PER_GROUP = THREADS / TEAM;
  const auto kernel = w ? &k_norm<T, TEAM, PIECES, VEC> : &k_norm<T, TEAM, PIECES, 1>;
  for (; j.row0 < j.rows; j.row0 += most_groups(THREADS) * PER_GROUP)
    kernel<<<(u32)std::min(div_up(j.rows - j.row0, PER_GROUP), most_groups(THREADS)), THREADS, 0, stream>>>(j);
}
// a wavefront to a row of up to 1,024 columns, a workgroup beyond
template <class T>
ccld_status forward(const ccld_norm_args* a, hipStream_t stream) {
  const NormJob j = make_job(a);
  const bool w = wide(a, false);
  if (a->d <= 512) launch_forward<T, 64, 1>(j, w, stream);
  else if (a->d <= 1024) launch_forward<T, 64, 2>(j, w, stream);
  else if (a->d <= 2048) launch_forward<T, 256, 1>(j, w, stream);
  else if (a->d <= 4096) launch_forward<T, 256, 2>(j, w, stream);
  else if (a->d <= 8192) launch_forward<T, 512, 2>(j, w, stream);
  else launch_forward<T, 1024, 2>(j, w, stream);
  return launched();
}

template <class T, int TEAM, int PIECES>
void launch_gradient(const NormJob& j, const Plan& p, bool w, hipStream_t stream) {
  constexpr int ROWS = PIECES > 1 ? ROWS_AGAIN : TEAM == 1024 && sizeof(T) == 4 ? ROWS_KEPT : ROWS_AHEAD;
  const auto kernel = w ? &k_norm_grad<T, TEAM, PIECES, (int)(16 / sizeof(T)), ROWS> : &k_norm_grad<T, TEAM, PIECES, 1, ROWS>;
  kernel<<<(u32)p.groups, threads_of<TEAM>(), 0, stream>>>(j);
}
template <class T>
ccld_status gradient(const ccld_norm_args* a, hipStream_t stream) {
  NormJob j = make_job(a);
  const Plan p = make_plan(a, static_cast<uint8_t*>(a->workspace));
  j.chunks = p.chunks; j.chunk_rows = p.chunk_rows; j.chunks_per_gate = p.chunks_per_gate;
  j.part_post = p.part_post; j.part_pre = p.part_pre; j.part_gate = p.part_gate;
  const bool w = wide(a, true);
  if (p.groups) {
    if (p.team == 64) launch_gradient<T, 64, 1>(j, p, w, stream);
    else if (p.team == 128) launch_gradient<T, 128, 1>(j, p, w, stream);
    else if (p.team == 256) launch_gradient<T, 256, 1>(j, p, w, stream);
    else if (p.team == 512) launch_gradient<T, 512, 1>(j, p, w, stream);
    else if (a->d <= 8192) launch_gradient<T, 1024, 1>(j, p, w, stream);
    else launch_gradient<T, 1024, 2>(j, p, w, stream);
  }
  SumJob s{p.part_post, p.part_pre, p.part_gate, a->dw_post, a->dw_pre, a->dgate, p.teams, a->rows ? p.chunks_per_gate : 0, 2, j.d};
  if (j.dgate && (p.part_gate || a->rows == 0)) s.sums += (u32)a->groups;
  k_norm_sums<T><<<dim3((u32)div_up(a->d, CCLD_WAVE), std::min(s.sums, 65535u)), SUM_THREADS, 0, stream>>>(s);
  return launched();
}

}  // namespace

extern "C" ccld_status ccld_norm_workspace(const ccld_norm_args* a, uint64_t* bytes) {
  if (!bytes) return CCLD_E_NULL;
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  *bytes = make_plan(a, nullptr).bytes;
  return CCLD_OK;
}

extern "C" ccld_status ccld_norm_residual(const ccld_norm_args* a, void* stream) {
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  if (!a->w_post || !a->w_pre || (a->rows && (!a->h || !a->b || !a->h_out || !a->u || !a->rstd_post || !a->rstd_pre))) return CCLD_E_NULL;
  if (!all_at_least(a->d, a->ldh, a->ldb, a->ldh_out, a->ldu) || (a->gate && a->ldgate < a->d)) return CCLD_E_BAD_ARG;
  if (!all_aligned(element_bytes(a), a->h, a->b, a->gate, a->w_post, a->w_pre, a->h_out, a->u) || !all_aligned(4, a->rstd_post, a->rstd_pre))
    return CCLD_E_BAD_ARG;
  if (a->rows == 0) return CCLD_OK;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return a->dtype == CCLD_BF16 ? forward<__bf16>(a, st) : a->dtype == CCLD_FP16 ? forward<_Float16>(a, st) : forward<float>(a, st);
}

extern "C" ccld_status ccld_norm_residual_grad(const ccld_norm_args* a, void* stream) {
  const ccld_status s = check(a);
  if (s != CCLD_OK) return s;
  if (!a->w_post || !a->w_pre || !a->dw_post || !a->dw_pre ||
      (a->rows && (!a->h || !a->b || !a->dh || !a->db || !a->rstd_post || !a->rstd_pre))) return CCLD_E_NULL;
  if (!all_at_least(a->d, a->ldh, a->ldb, a->lddh, a->lddb) || (a->gate && a->ldgate < a->d) || (a->dh_out && a->lddh_out < a->d) ||
      (a->du && a->lddu < a->d)) return CCLD_E_BAD_ARG;
  if (!all_aligned(element_bytes(a), a->h, a->b, a->gate, a->w_post, a->w_pre, a->dh_out, a->du, a->dh, a->db, a->dgate, a->dw_post, a->dw_pre) ||
      !all_aligned(4, a->rstd_post, a->rstd_pre)) return CCLD_E_BAD_ARG;
  if (make_plan(a, nullptr).bytes > a->workspace_bytes || (a->rows && !a->workspace) || !aligned(a->workspace, 256)) return CCLD_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return a->dtype == CCLD_BF16 ? gradient<__bf16>(a, st) : a->dtype == CCLD_FP16 ? gradient<_Float16>(a, st) : gradient<float>(a, st);
}
