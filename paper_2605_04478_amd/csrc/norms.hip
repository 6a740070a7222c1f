// The norms before and after a block, fused with its gate and the scale of the residual stream, and their gradient (ccld_norm_*).
//
//   r1 = 1 / sqrt(mean(b^2) + eps)     n = b r1 w_post     x = scale h + gate n     (h' = x rounded)
//   r2 = 1 / sqrt(mean(x^2) + eps)     u = x r2 w_pre
//
//   dx = dh' + r2 (du w_pre - x r2^2 mean(du w_pre x))      dh = scale dx      dgate = sum dx n
//   dn = dx gate      db = r1 (dn w_post - b r1^2 mean(dn w_post b))      dw_post = sum dn b r1      dw_pre = sum du x r2
//
// Memory bounds both: a dozen operations per element, each row read once and kept in registers between its two reductions.  A
// row belongs to one wavefront where it fits, else to a workgroup.  The gradient takes x from h and b again, which costs no more
// bytes than reading h' and is exact; its sums over rows are kept in registers by teams that take many rows each, and joined by a
// second kernel in the teams' order.
#include <algorithm>

#include "ccld_internal.h"
#include "products.h"
#include "tiles.h"

using namespace ccld;

namespace {

// PIECES x 8 columns to each of a row's TEAM threads: neighbours of 8 where rows are aligned to that (WIDE), else one by one
template <int TEAM, bool WIDE>
__device__ __forceinline__ int first_column(int t, int p) { return WIDE ? (p * TEAM + t) * 8 : p * 8 * TEAM + t; }
template <int TEAM, bool WIDE>
constexpr int column_step() { return WIDE ? 1 : TEAM; }

template <class T, int TEAM, bool WIDE>
__device__ __forceinline__ void load8(float* v, const T* p, int c, int d) {
  if constexpr (WIDE) {
    typedef __attribute__((ext_vector_type(16 / sizeof(T)))) T piece;
    if (c < d) {
#pragma unroll
      for (int k = 0; k < 8; k += 16 / (int)sizeof(T)) {
        const piece q = *reinterpret_cast<const piece*>(p + c + k);
#pragma unroll
        for (int i = 0; i < 16 / (int)sizeof(T); ++i) v[k + i] = (float)q[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i * TEAM < d ? (float)p[c + i * TEAM] : 0.0f;
  }
}

template <class T, int TEAM, bool WIDE>
__device__ __forceinline__ void store8(T* p, const float* v, int c, int d) {
  if constexpr (WIDE) {
    typedef __attribute__((ext_vector_type(16 / sizeof(T)))) T piece;
    if (c < d) {
#pragma unroll
      for (int k = 0; k < 8; k += 16 / (int)sizeof(T)) {
        piece q;
#pragma unroll
        for (int i = 0; i < 16 / (int)sizeof(T); ++i) q[i] = (T)v[k + i];
        *reinterpret_cast<piece*>(p + c + k) = q;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i * TEAM < d) p[c + i * TEAM] = (T)v[i];
  }
}

// the sum over a row's threads; every call of a kernel that has a workgroup to a row takes another of its two slots in LDS
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float (&slot)[16]) {
#pragma unroll
  for (int m = CCLD_WAVE / 2; m >= 1; m >>= 1) v += __shfl_xor(v, m, CCLD_WAVE);
  if constexpr (TEAM > CCLD_WAVE) {
    if (lane_id() == 0) slot[threadIdx.x / CCLD_WAVE] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < TEAM / CCLD_WAVE; ++i) v += slot[i];
  }
  return v;
}

struct NormJob {
  const void *h, *b, *gate, *w_post, *w_pre, *dh_out, *du;
  void *h_out, *u, *dh, *db, *dgate;
  float *rstd_post, *rstd_pre;
  i64 ldh, ldb, ldgate, ldh_out, ldu, lddh_out, lddu, lddh, lddb;
  i64 rows, rows_per_gate;
  int d;
  float scale, eps;
  // gradient: the rows in chunks that lie within a gate's, and where sums go
  i64 chunks, chunk_rows;
  u32 chunks_per_gate;
  float *part_post, *part_pre;   // [teams][d]
  float* part_gate;              // [chunks][d], or null: a gate's rows are one chunk and its sum leaves at once
};

template <class T, int TEAM, int PIECES, bool WIDE>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_norm(NormJob j) {
  constexpr int PER_GROUP = TEAM < 256 ? 256 / TEAM : 1;
  __shared__ float slots[2][16];
  const int t = threadIdx.x % TEAM;
  const i64 row = (i64)blockIdx.x * PER_GROUP + threadIdx.x / TEAM;
  if (row >= j.rows) return;                       // whole teams: those of several wavefronts are whole workgroups
  const T* b = static_cast<const T*>(j.b) + row * j.ldb;
  const T* h = static_cast<const T*>(j.h) + row * j.ldh;
  float vb[PIECES][8], vx[PIECES][8];
  float sum = 0;
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = first_column<TEAM, WIDE>(t, p);
    load8<T, TEAM, WIDE>(vb[p], b, c, j.d);
    load8<T, TEAM, WIDE>(vx[p], h, c, j.d);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += vb[p][i] * vb[p][i];
  }
  const float r1 = 1.0f / sqrtf(team_sum<TEAM>(sum, slots[0]) / (float)j.d + j.eps);
  const T* gate = j.gate ? static_cast<const T*>(j.gate) + row / j.rows_per_gate * j.ldgate : nullptr;
  sum = 0;
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = first_column<TEAM, WIDE>(t, p);
    float w[8], g[8];
    load8<T, TEAM, WIDE>(w, static_cast<const T*>(j.w_post), c, j.d);
    if (gate) load8<T, TEAM, WIDE>(g, gate, c, j.d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float n = vb[p][i] * r1 * w[i];
      vx[p][i] = j.scale * vx[p][i] + (gate ? g[i] * n : n);
      sum += vx[p][i] * vx[p][i];
    }
    store8<T, TEAM, WIDE>(static_cast<T*>(j.h_out) + row * j.ldh_out, vx[p], c, j.d);
  }
  const float r2 = 1.0f / sqrtf(team_sum<TEAM>(sum, slots[1]) / (float)j.d + j.eps);
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = first_column<TEAM, WIDE>(t, p);
    float w[8];
    load8<T, TEAM, WIDE>(w, static_cast<const T*>(j.w_pre), c, j.d);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] *= vx[p][i] * r2;
    store8<T, TEAM, WIDE>(static_cast<T*>(j.u) + row * j.ldu, w, c, j.d);
  }
  if (t == 0) {
    j.rstd_post[row] = r1;
    j.rstd_pre[row] = r2;
  }
}

template <class T, int TEAM, int PIECES, bool WIDE>
__global__ __launch_bounds__(TEAM < 256 ? 256 : TEAM) void k_norm_grad(NormJob j) {
  constexpr int PER_GROUP = TEAM < 256 ? 256 / TEAM : 1;
  __shared__ float slots[2][16];
  const int t = threadIdx.x % TEAM;
  const i64 team = (i64)blockIdx.x * PER_GROUP + threadIdx.x / TEAM, teams = (i64)gridDim.x * PER_GROUP;
  float s_post[PIECES][8] = {}, s_pre[PIECES][8] = {}, s_gate[PIECES][8] = {};
  const float per_d = 1.0f / (float)j.d;
  for (i64 chunk = team; chunk < j.chunks; chunk += teams) {
    const i64 g = chunk / j.chunks_per_gate, in = chunk - g * j.chunks_per_gate;
    const i64 row0 = g * j.rows_per_gate + in * j.chunk_rows;
    const i64 row1 = min(row0 + j.chunk_rows, (g + 1) * j.rows_per_gate);
    const T* gate = j.gate ? static_cast<const T*>(j.gate) + g * j.ldgate : nullptr;
    for (i64 row = row0; row < row1; ++row) {
      const float r1 = j.rstd_post[row], r2 = j.rstd_pre[row];
      float vb[PIECES][8], vx[PIECES][8], vd[PIECES][8], vu[PIECES][8];
      float sum = 0;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int c = first_column<TEAM, WIDE>(t, p);
        load8<T, TEAM, WIDE>(vb[p], static_cast<const T*>(j.b) + row * j.ldb, c, j.d);
        load8<T, TEAM, WIDE>(vx[p], static_cast<const T*>(j.h) + row * j.ldh, c, j.d);
        if (j.du) load8<T, TEAM, WIDE>(vu[p], static_cast<const T*>(j.du) + row * j.lddu, c, j.d);
        if (j.dh_out) load8<T, TEAM, WIDE>(vd[p], static_cast<const T*>(j.dh_out) + row * j.lddh_out, c, j.d);
      }
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int c = first_column<TEAM, WIDE>(t, p);
        float w1[8], w2[8], gt[8];
        load8<T, TEAM, WIDE>(w1, static_cast<const T*>(j.w_post), c, j.d);
        load8<T, TEAM, WIDE>(w2, static_cast<const T*>(j.w_pre), c, j.d);
        if (gate) load8<T, TEAM, WIDE>(gt, gate, c, j.d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float n = vb[p][i] * r1 * w1[i];
          vx[p][i] = j.scale * vx[p][i] + (gate ? gt[i] * n : n);
          const float du = j.du ? vu[p][i] : 0;
          s_pre[p][i] += du * vx[p][i] * r2;
          vu[p][i] = du * w2[i];
          sum += vu[p][i] * vx[p][i];
        }
      }
      const float m2 = team_sum<TEAM>(sum, slots[0]) * per_d * r2 * r2;
      sum = 0;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int c = first_column<TEAM, WIDE>(t, p);
        float w1[8], gt[8], out[8];
        load8<T, TEAM, WIDE>(w1, static_cast<const T*>(j.w_post), c, j.d);
        if (gate) load8<T, TEAM, WIDE>(gt, gate, c, j.d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float dx = (j.dh_out ? vd[p][i] : 0) + r2 * (vu[p][i] - vx[p][i] * m2);
          out[i] = j.scale * dx;
          const float nb = vb[p][i] * r1, dn = gate ? dx * gt[i] : dx;
          s_gate[p][i] += dx * nb * w1[i];
          s_post[p][i] += dn * nb;
          vd[p][i] = dn * w1[i];
          sum += vd[p][i] * vb[p][i];
        }
        store8<T, TEAM, WIDE>(static_cast<T*>(j.dh) + row * j.lddh, out, c, j.d);
      }
      const float m1 = team_sum<TEAM>(sum, slots[1]) * per_d * r1 * r1;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int c = first_column<TEAM, WIDE>(t, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) vd[p][i] = r1 * (vd[p][i] - vb[p][i] * m1);
        store8<T, TEAM, WIDE>(static_cast<T*>(j.db) + row * j.lddb, vd[p], c, j.d);
      }
    }
    if (j.dgate) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int c = first_column<TEAM, WIDE>(t, p);
        if (j.part_gate) store8<float, TEAM, WIDE>(j.part_gate + chunk * j.d, s_gate[p], c, j.d);
        else store8<T, TEAM, WIDE>(static_cast<T*>(j.dgate) + g * j.d, s_gate[p], c, j.d);
#pragma unroll
        for (int i = 0; i < 8; ++i) s_gate[p][i] = 0;
      }
    }
  }
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = first_column<TEAM, WIDE>(t, p);
    store8<float, TEAM, WIDE>(j.part_post + team * j.d, s_post[p], c, j.d);
    store8<float, TEAM, WIDE>(j.part_pre + team * j.d, s_pre[p], c, j.d);
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
    if (c < j.d)
      for (i64 r = wave; r < n; r += SUM_THREADS / CCLD_WAVE) s += p[r * j.d + c];
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

// Threads to a row of the gradient, which keeps three sums per column in registers: 8 to 32 columns each.
int grad_team(i64 d) { return d <= 512 ? 64 : d <= 4096 ? 256 : 512; }

struct Plan { int team; i64 groups, teams, chunks, chunk_rows; u32 chunks_per_gate; float *part_post, *part_pre, *part_gate; u64 bytes; };

Plan make_plan(const ccld_norm_args* a, uint8_t* base) {
  Plan p{};
  p.team = grad_team(a->d);
  const i64 per_group = p.team < 256 ? 256 / p.team : 1, gates = a->gate ? a->groups : 1;
  // two workgroups to a compute unit; as many chunks, so that each team has one, or one for each gate
  const i64 want = std::max<i64>(1, std::min<i64>(a->rows, 2 * (i64)COMPUTE_UNITS * per_group));
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
template <class... L>
bool all_eights(L... l) { return ((l % 8 == 0) && ...); }

// pieces of 8 columns start on 16 bytes in every row
bool wide(const ccld_norm_args* a, bool grad) {
  bool w = a->d % 8 == 0 && all_eights(a->ldh, a->ldb) && all_aligned(16, a->h, a->b, a->w_post, a->w_pre, a->gate) &&
           (!a->gate || a->ldgate % 8 == 0);
  if (grad)
    w = w && all_eights(a->lddh, a->lddb) && all_aligned(16, a->dh, a->db, a->dgate, a->dh_out, a->du) &&
        (!a->dh_out || a->lddh_out % 8 == 0) && (!a->du || a->lddu % 8 == 0);
  else w = w && all_eights(a->ldh_out, a->ldu) && all_aligned(16, a->h_out, a->u);
  return w;
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
void launch_forward(const NormJob& j, bool w, hipStream_t stream) {
  constexpr int THREADS = TEAM < 256 ? 256 : TEAM;
  const u32 grid = (u32)div_up(j.rows, THREADS / TEAM);
  const auto kernel = w ? &k_norm<T, TEAM, PIECES, true> : &k_norm<T, TEAM, PIECES, false>;
  kernel<<<grid, THREADS, 0, stream>>>(j);
}
// a wavefront to a row of up to 2,048 columns, a workgroup of four beyond
template <class T>
ccld_status forward(const ccld_norm_args* a, hipStream_t stream) {
  const NormJob j = make_job(a);
  const bool w = wide(a, false);
  if (a->d <= 512) launch_forward<T, 64, 1>(j, w, stream);
  else if (a->d <= 1024) launch_forward<T, 64, 2>(j, w, stream);
  else if (a->d <= 2048) launch_forward<T, 256, 1>(j, w, stream);
  else if (a->d <= 4096) launch_forward<T, 256, 2>(j, w, stream);
  else if (a->d <= 8192) launch_forward<T, 256, 4>(j, w, stream);
  else launch_forward<T, 512, 4>(j, w, stream);
  return launched();
}

template <class T, int TEAM, int PIECES>
void launch_gradient(const NormJob& j, const Plan& p, bool w, hipStream_t stream) {
  const auto kernel = w ? &k_norm_grad<T, TEAM, PIECES, true> : &k_norm_grad<T, TEAM, PIECES, false>;
  kernel<<<(u32)p.groups, TEAM < 256 ? 256 : TEAM, 0, stream>>>(j);
}
template <class T>
ccld_status gradient(const ccld_norm_args* a, hipStream_t stream) {
  NormJob j = make_job(a);
  const Plan p = make_plan(a, static_cast<uint8_t*>(a->workspace));
  j.chunks = p.chunks; j.chunk_rows = p.chunk_rows; j.chunks_per_gate = p.chunks_per_gate;
  j.part_post = p.part_post; j.part_pre = p.part_pre; j.part_gate = p.part_gate;
  const bool w = wide(a, true);
  if (p.groups) {
    if (a->d <= 512) launch_gradient<T, 64, 1>(j, p, w, stream);
    else if (a->d <= 2048) launch_gradient<T, 256, 1>(j, p, w, stream);
    else if (a->d <= 4096) launch_gradient<T, 256, 2>(j, p, w, stream);
    else if (a->d <= 8192) launch_gradient<T, 512, 2>(j, p, w, stream);
    else launch_gradient<T, 512, 4>(j, p, w, stream);
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
