// Softmax cross entropy over a large vocabulary and its gradient (ccld_vocab_*), without the matrix of logits.
//
//   z = h w^T     lse = log sum_v exp z_v     loss = lse - z_label
//   dz = g (exp(z - lse) - [v = label])     dh = dz w     dw = dz^T h
//
// Loss: every output tile of the product reduces its logits to a running maximum and a sum of exponentials per row, and
// one kernel joins a row's tiles.  Gradient: the logits of a piece of the vocabulary are taken again, turned into dz where they
// are, and two more products bring the piece's share of dh and its rows of dw; dz is kept for one piece at a time.
//
// Rows without a target are dropped first: the others' h rows are copied side by side, so that what a masked row holds
// reaches no sum (zero times infinity would) and costs no work.  How many there are is known on the device only: grids are laid
// out for all rows, and workgroups beyond the last row end at once.
//
// Exponentials are 2^(x log2 e) in 32 bits: for x down to -30 off by 30 roundings of 2^-24 at most, a thousandth of a step of the
// 16-bit types that gradients leave in.  dz is rounded to the operands' type for the matrix cores, after a scaling by the power of two that
// brings the largest finite |g| just under 2^15: half-precision gradients of 10^-9 keep their bits.  What the rounding leaves of a row's target, which is most of
// dz where a model is unsure, is kept for itself and added to both gradients (Targets, k_input_rows); up to 128 kept rows the whole of dz
// is kept in two 16-bit parts (dz_parts).
//
// What bounds it: the matrix cores, with the logits taken twice (4 products for the 3 of an implementation that keeps them); for a handful of rows
// reading the vocabulary's weights, and then its launches.  Measured, on different cards: 8,192 rows x 4,096 x 128,000 in bfloat16, loss and gradients, 26.8 to 28.5 ms =
// 1,200 to 1,280 TFLOP/s of the four products; 4,096 x 2,048 x 65,536, the loss alone, 0.92 to 1.03 ms = 1,070 to 1,180 TFLOP/s, where the exponentials take what the
// product does not hide; 5 rows x 2,048 x 32,000 34 to 41 us, of which 22 read the weights at 6 TB/s, three launches and their gaps are the rest.
#include <algorithm>

#include "ccld_internal.h"
#include "products.h"
#include "tiles.h"

using namespace ccld;

namespace {

extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

constexpr float LOG2E = 1.4426950408889634f;
constexpr int USED_THREADS = 1024;

// what the kernels share in the workspace
struct Rows {
  u32* count;          // rows with a target; then the exponent of the scaling of dz
  i32* row;            // [rows] which they are
  i32* place;          // [rows] a row's place among them, or -1
  i32* label;          // [rows] of the kept rows, as are the following
  float* target;       // [rows] z_label
  float* lse;          // [rows] (gradient)
  float* scale;        // [rows] dloss (gradient), scaled
  float* rest;         // [rows] what rounding leaves of the target's dz (gradient, where dz has one part)
  void* h;             // [kept rows][dp], for each part of dz
};

// Up to 128 kept rows dz is two 16-bit parts, its rounding and what that left, so that it costs no bits: with few rows any one value's rounding
// can be all that a row of dw is off by (one row in bfloat16: 0.0031 beside 0.0017).  The products of so few rows are bound by the vocabulary's weights: 9 rows
// x 2,504 x 10,082 take 73 us instead of 70, 57 x 1,432 x 55,406 202 instead of 174.  With more rows the products would take half as long again; there
// the rest of each row's target alone is kept, one value to a row.  A word's row of dw that is no row's target may still be off by
// dz's rounding and its own (a half step each), and so may dh of a row that is sure of a wrong word.
constexpr u32 TWO_PARTS = 128;
__host__ __device__ __forceinline__ u32 dz_parts(u32 kept) { return kept <= TWO_PARTS ? 2 : 1; }

__device__ __forceinline__ i64 label_at(const void* p, int bits, i64 i) {
  return bits == 64 ? static_cast<const i64*>(p)[i] : (i64)static_cast<const i32*>(p)[i];
}

// A kept row's values, padded with zeros to dp columns, V at a time; and, for the gradient, its lse and scaled dloss.
template <class T, int V>
__device__ __forceinline__ void gather_piece(const Rows& w, i64 i, i64 kept, i64 step, i64 at, int c, i64 r, const T* h, i64 ldh, int d, const float* lse,
                                             const float* dloss, i64 dloss_stride, float scale) {
  const u32 parts = dloss ? dz_parts((u32)kept) : 1;
  for (u32 part = 0; part < parts; ++part, i += step) {
    if constexpr (V == 8) reinterpret_cast<s16x8*>(w.h)[i] = *reinterpret_cast<const s16x8*>(h + r * ldh + c);
    else static_cast<T*>(w.h)[i] = c < d ? h[r * ldh + c] : (T)0.0f;
  }
  if (c == 0 && dloss) {
    w.lse[at] = lse[r];
    w.scale[at] = dloss[r * dloss_stride] * scale;
  }
}

// Which rows have a target, in order; zeros for the loss of the others; the largest finite |dloss|.  One workgroup: the labels of 8,192
// rows are 64 KB.  GATHER: there are no more rows than threads, and every workgroup finds them by itself and copies its share of them too
// (a launch less: 5 us of a handful of rows' 45).
template <class T, int V, bool GATHER>
__global__ __launch_bounds__(USED_THREADS) void k_used_rows(Rows w, const void* labels, int bits, i64 rows, i64 vocab, float* loss, float* lse_out,
                                                            const T* h, i64 ldh, int d, int dp, const float* lse, const float* dloss, i64 dloss_stride) {
  __shared__ u32 sums[USED_THREADS / CCLD_WAVE];
  __shared__ float tops[USED_THREADS / CCLD_WAVE];
  __shared__ i32 list[GATHER ? USED_THREADS : 1];
  const u32 lane = lane_id(), wave = threadIdx.x / CCLD_WAVE;
  const bool writes = blockIdx.x == 0;
  u32 before = 0;
  float top = 0;
  for (i64 base = 0; base < rows; base += USED_THREADS) {
    const i64 r = base + threadIdx.x;
    const i64 l = r < rows ? label_at(labels, bits, r) : -1;
    const bool used = l >= 0 && l < vocab;
    const u64 mask = ballot64(used);
    if (lane == 0) sums[wave] = (u32)__popcll(mask);
    __syncthreads();
    u32 at = before;
    for (u32 i = 0; i < USED_THREADS / CCLD_WAVE; ++i) {
      if (i < wave) at += sums[i];
      before += sums[i];
    }
    __syncthreads();
    at += mbcnt64(mask);
    if (used && dloss) {
      const float size = fabsf(dloss[r * dloss_stride]);
      if (size < __builtin_inff()) top = fmaxf(top, size);      // (an infinite row's dz is infinite at any scale)
    }
    if (GATHER && used) list[at] = (i32)r;
    if (writes && r < rows) {
      if (used) {
        w.row[at] = (i32)r;
        w.label[at] = (i32)l;
      } else if (loss) {
        loss[r] = 0;
        lse_out[r] = 0;
      }
      w.place[r] = used ? (i32)at : -1;
    }
  }
  for (int m = CCLD_WAVE / 2; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, CCLD_WAVE));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  for (u32 i = 0; i < USED_THREADS / CCLD_WAVE; ++i) top = fmaxf(top, tops[i]);
  int e = 0;
  if (top > 0) (void)frexpf(top, &e);
  // top 2^(15 - e) lies in [2^14, 2^15); the scale and its inverse stay within 32-bit floats
  const int scaling = top > 0 ? min(15 - e, 120) : 0;
  if (writes && threadIdx.x == 0) {
    w.count[0] = before;
    reinterpret_cast<i32*>(w.count)[1] = scaling;
  }
  if constexpr (GATHER) {
    const int pieces = dp / V;
    for (i64 i = (i64)blockIdx.x * USED_THREADS + threadIdx.x; i < (i64)before * pieces; i += (i64)gridDim.x * USED_THREADS) {
      const i64 at = i / pieces;
      gather_piece<T, V>(w, i, before, (i64)before * pieces, at, (int)(i - at * pieces) * V, list[at], h, ldh, d, lse, dloss, dloss_stride, ldexpf(1.0f, scaling));
    }
  }
}

// The kept rows side by side.
template <class T, int V>
__global__ __launch_bounds__(256) void k_gather_rows(Rows w, const T* __restrict__ h, i64 ldh, int d, int dp, const float* lse,
                                                     const float* dloss, i64 dloss_stride) {
  const i64 n = w.count[0];
  const int pieces = dp / V;
  const float scale = ldexpf(1.0f, reinterpret_cast<const i32*>(w.count)[1]);
  for (i64 i = (i64)blockIdx.x * 256 + threadIdx.x; i < n * pieces; i += (i64)gridDim.x * 256) {
    const i64 at = i / pieces;
    gather_piece<T, V>(w, i, n, n * pieces, at, (int)(i - at * pieces) * V, w.row[at], h, ldh, d, lse, dloss, dloss_stride, scale);
  }
}

struct LogitJob {
  Rows rows;
  const void* w;           // first row of the piece
  i64 ldw;
  int d, dp;
  int first, cols;         // the piece of the vocabulary
  u32 col_tiles;
  float2* part;            // [rows][col_tiles] (maximum, sum of exponentials) of a row's tiles
  void* dz;                // [rows][lddz] (gradient)
  i64 lddz;
};

// the tile of this workgroup among those of the kept rows, or false
template <class C>
__device__ __forceinline__ bool logit_tile(u32 kept, u32 col_tiles, int& m0, int& n0) {
  const u32 tm = (kept + C::BM - 1) / C::BM;
  if (blockIdx.x >= tm * col_tiles) return false;
  const uint2 t = grouped_order(xcd_order(blockIdx.x, tm * col_tiles), tm, col_tiles, 8);
  m0 = (int)t.x * C::BM;
  n0 = (int)t.y * C::BN;
  return true;
}

// (maximum, sum of exp(x - maximum)) of two sets; the maximum is -inf where all are, 0 where one is +inf.  A factor is 2^-126 at least: an
// infinite sum stays one beside a maximum of hundreds (a factor of zero would make it NaN), and finite sums, below 2^32, add nothing to
// the other set's, which is one at least.
__device__ __forceinline__ float2 join_sums(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x);
  const float ref = top == -__builtin_inff() ? 0 : top;
  auto share = [&](float2 s) { return s.y * fmaxf(__builtin_amdgcn_exp2f((s.x - ref) * LOG2E), 0x1p-126f); };
  return make_float2(top, share(a) + share(b));
}

template <class C, class T, bool DIRECT>
__global__ __launch_bounds__(C::THREADS) void k_logit_sums(LogitJob j) {
  int m0, n0;
  const int kept = (int)j.rows.count[0];
  if (!logit_tile<C>(kept, j.col_tiles, m0, n0)) return;
  const int rows = min(C::BM, kept - m0), cols = min(C::BN, j.cols - n0);
  TileProduct<C, T, false, false, DIRECT> prod;
  prod.run(lds, static_cast<const T*>(j.rows.h) + (i64)m0 * j.dp, j.dp, rows, static_cast<const T*>(j.w) + (i64)n0 * j.ldw, j.ldw,
           cols, j.d);
  __syncthreads();                                      // the stages' place is taken over
  float2* sums = reinterpret_cast<float2*>(lds);        // [WN][BM]
  const u32 lane = lane_id(), wave = threadIdx.x / CCLD_WAVE;
  const int left = cols - (int)(prod.wave_n() + 4 * (lane / 16));
#pragma unroll
  for (int i = 0; i < C::MI; ++i) {
    const int m = (int)prod.wave_m() + 16 * i + (int)(lane % 16);
    const int want = m < rows ? j.rows.label[m0 + m] - j.first - n0 - (int)(prod.wave_n() + 4 * (lane / 16)) : -1;
    float top = -__builtin_inff();
#pragma unroll
    for (int b = 0; b < C::NI; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * b + r < left) {
          top = fmaxf(top, prod.acc[i][b][r]);
          if (16 * b + r == want) j.rows.target[m0 + m] = prod.acc[i][b][r];
        }
#pragma unroll
    for (int x = 16; x < CCLD_WAVE; x *= 2) top = fmaxf(top, __shfl_xor(top, x, CCLD_WAVE));
    if (top == __builtin_inff()) top = 0;
    const float ref = top == -__builtin_inff() ? 0 : top;
    float sum = 0;
#pragma unroll
    for (int b = 0; b < C::NI; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (16 * b + r < left) sum += __builtin_amdgcn_exp2f((prod.acc[i][b][r] - ref) * LOG2E);
#pragma unroll
    for (int x = 16; x < CCLD_WAVE; x *= 2) sum += __shfl_xor(sum, x, CCLD_WAVE);
    if (lane < 16) sums[wave % C::WN * C::BM + m] = make_float2(top, sum);
  }
  __syncthreads();
  for (int m = threadIdx.x; m < rows; m += C::THREADS) {
    float2 s = sums[m];
#pragma unroll
    for (int i = 1; i < C::WN; ++i) s = join_sums(s, sums[i * C::BM + m]);
    j.part[(i64)(m0 + m) * j.col_tiles + n0 / C::BN] = s;
  }
}

// a wavefront to a row, from the kept row `first` on: its tiles' sums
__global__ __launch_bounds__(256) void k_loss(Rows w, i64 first, const float2* __restrict__ part, u32 col_tiles, float* loss, float* lse) {
  const i64 n = w.count[0];
  const i64 at = first + (i64)blockIdx.x * 4 + threadIdx.x / CCLD_WAVE;
  if (at >= n) return;
  float2 s = make_float2(-__builtin_inff(), 0);
  for (u32 i = lane_id(); i < col_tiles; i += CCLD_WAVE) s = join_sums(s, part[at * col_tiles + i]);
#pragma unroll
  for (int x = 1; x < CCLD_WAVE; x *= 2)
    s = join_sums(s, make_float2(__shfl_xor(s.x, x, CCLD_WAVE), __shfl_xor(s.y, x, CCLD_WAVE)));
  if (lane_id() == 0) {
    // (the largest logit and the target's first: where they are one, the loss keeps bits that lse has not)
    const float top = s.x == -__builtin_inff() ? 0 : s.x, more = logf(s.y);
    lse[w.row[at]] = top + more;
    loss[w.row[at]] = (top - w.target[at]) + more;
  }
}

// what rounding to T leaves of a value, exactly; nothing of an infinite one (infinity less itself would make the products NaN)
template <class T>
__device__ __forceinline__ float rest_of(float v) {
  const float rest = v - (float)(T)v;
  return fabsf(rest) < __builtin_inff() ? rest : 0;
}

template <class C, class T, bool DIRECT>
__global__ __launch_bounds__(C::THREADS) void k_logit_grad(LogitJob j) {
  int m0, n0;
  const int kept = (int)j.rows.count[0];
  if (!logit_tile<C>(kept, j.col_tiles, m0, n0)) return;
  const int rows = min(C::BM, kept - m0), cols = min(C::BN, j.cols - n0);
  TileProduct<C, T, false, false, DIRECT> prod;
  prod.run(lds, static_cast<const T*>(j.rows.h) + (i64)m0 * j.dp, j.dp, rows, static_cast<const T*>(j.w) + (i64)n0 * j.ldw, j.ldw,
           cols, j.d);
  const u32 lane = lane_id(), n1 = prod.wave_n() + 4 * (lane / 16), parts = dz_parts((u32)kept);
#pragma unroll
  for (int i = 0; i < C::MI; ++i) {
    const int m = (int)prod.wave_m() + 16 * i + (int)(lane % 16);
    const bool in = m < rows;
    const float lse = in ? j.rows.lse[m0 + m] : 0, scale = in ? j.rows.scale[m0 + m] : 0;
    const int want = in ? j.rows.label[m0 + m] - j.first - n0 - (int)n1 : -1;
    float target = 0;
#pragma unroll
    for (int b = 0; b < C::NI; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float p = __builtin_amdgcn_exp2f((prod.acc[i][b][r] - lse) * LOG2E);
        if (16 * b + r == want) {
          p -= 1;
          target = p * scale;
        }
        prod.acc[i][b][r] = (int)n1 + 16 * b + r < cols ? p * scale : 0;      // columns beyond the piece are zeros that products may read
      }
    const bool mine = want >= 0 && want < 16 * C::NI && want % 16 < 4 && (int)n1 + want < cols;
    if (mine && parts == 1) j.rows.rest[m0 + m] = rest_of<T>(target);
  }
  T* dz = static_cast<T*>(j.dz) + (i64)m0 * j.lddz + n0;
  prod.store(lds, dz, j.lddz, rows, C::BN, true, true, 1.0f);
  if (parts > 1) {                     // what that rounding left, exactly
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int b = 0; b < C::NI; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) prod.acc[i][b][r] = rest_of<T>(prod.acc[i][b][r]);
    __builtin_amdgcn_wave_barrier();
    prod.store(lds, dz + (i64)kept * j.lddz, j.lddz, rows, C::BN, true, true, 1.0f);
  }
}

struct InputJob {            // dh: dz [kept][width] times w [width][d]
  Rows rows;
  const void *dz, *w;
  i64 lddz, ldw;
  int d, width, full_width;  // this piece of the vocabulary's, and all but the last one's
  u32 col_tiles;
  float* sum;                // [splits][kept rows][d]
  bool more;                 // add to what an earlier piece left
};

// the parts of dh's contraction, the same for all pieces
template <class C>
__device__ __forceinline__ u32 input_splits(u32 kept, u32 col_tiles, int full_width) {
  return splits_of<C>((kept + C::BM - 1) / C::BM * col_tiles, (u32)full_width / 32);
}

template <class C, class T, bool DIRECT>
__global__ __launch_bounds__(C::THREADS) void k_input_grad(InputJob j) {
  const int kept = (int)(j.rows.count[0] * dz_parts(j.rows.count[0]));
  const u32 tm = (u32)(kept + C::BM - 1) / C::BM, tiles = tm * j.col_tiles, splits = input_splits<C>((u32)kept, j.col_tiles, j.full_width);
  if (blockIdx.x >= tiles * splits) return;
  const u32 id = xcd_order(blockIdx.x, tiles * splits), split = id / tiles;
  const uint2 place = grouped_order(id - split * tiles, tm, j.col_tiles, 8);
  const int m0 = (int)place.x * C::BM, n0 = (int)place.y * C::BN;
  const int split_width = (int)((j.full_width / 64 + splits - 1) / splits * 64), c0 = (int)split * split_width;
  const int depth = max(0, min(split_width, j.width - c0));
  const int rows = min(C::BM, kept - m0), cols = min(C::BN, j.d - n0);
  TileProduct<C, T, false, true, DIRECT> prod;
  prod.run(lds, static_cast<const T*>(j.dz) + (i64)m0 * j.lddz + c0, j.lddz, rows, static_cast<const T*>(j.w) + (i64)(depth ? c0 : 0) * j.ldw + n0,
           j.ldw, cols, depth);
  float* o = j.sum + ((i64)split * kept + m0) * j.d + n0;
  prod.each([&](u32 m, u32 n, f32x4 v) {
    if ((int)m >= rows || (int)n >= cols) return;
    float* q = o + (i64)m * j.d + n;
    if (j.d % 4 == 0) {
      if (j.more) v += *reinterpret_cast<const f32x4*>(q);
      *reinterpret_cast<f32x4*>(q) = v;
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if ((int)n + r < cols) q[r] = j.more ? q[r] + v[r] : v[r];
    }
  });
}

// dh leaves: the splits' sums in their order, what rounding left of the target's dz, rows back in their places, zeros for rows without a target.  V
// neighbouring columns to a thread where rows allow it.
template <class C, class T, int V>
__global__ __launch_bounds__(256) void k_input_rows(Rows w, const float* __restrict__ sum, u32 col_tiles, int full_width, i64 rows, int d,
                                                    const T* __restrict__ words, i64 ldw, T* dh, i64 lddh) {
  const u32 parts = dz_parts(w.count[0]);
  const i64 kept = w.count[0], all = kept * parts;
  const u32 splits = input_splits<C>((u32)all, col_tiles, full_width);
  const float back = ldexpf(1.0f, -reinterpret_cast<const i32*>(w.count)[1]);
  const int pieces = d / V;
  for (i64 i = (i64)blockIdx.x * 256 + threadIdx.x; i < rows * pieces; i += (i64)gridDim.x * 256) {
    const i64 r = i / pieces, c = (i - r * pieces) * V, at = w.place[r];
    typedef float vec __attribute__((ext_vector_type(V)));
    vec v = 0;
    const bool has_rest = parts == 1 && at >= 0;
    const float rest = has_rest ? w.rest[at] : 0;
    T word[V];                                           // on its way with the sums
    __builtin_memcpy(word, words + (has_rest ? w.label[at] * ldw : 0) + c, sizeof(word));
    for (i64 of = at; of >= 0 && of < all; of += kept) {
      const float* q = sum + of * d + c;
      const i64 step = all * d;
      u32 s = 0;
      for (; s + 8 <= splits; s += 8) {              // eight on their way at once: a load after the other took 15 us of 64 parts
        vec x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = *reinterpret_cast<const vec*>(q + (s + e) * step);
#pragma unroll
        for (int e = 0; e < 8; ++e) v += x[e];
      }
      for (; s < splits; ++s) v += *reinterpret_cast<const vec*>(q + s * step);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float more = rest * (float)word[e];
      if (fabsf(more) < __builtin_inff()) v[e] += more;      // (beside an infinite product a rest says nothing)
    }
    if constexpr (V == 4) store4(dh + r * lddh + c, v * back, 4, true);
    else dh[r * lddh + c] = (T)(v[0] * back);
  }
}

struct WeightJob {           // dw of a piece: dz^T [width][kept] times h [kept][d]
  Rows rows;
  const void* dz;
  i64 lddz;
  void* dw;                  // first row of the piece
  i64 lddw;
  int first;                 // word of the piece's first row
  int d, dp, width;
  u32 n_tiles, k_tiles;
  float* part;               // [splits][width][d] or null
  bool whole;                // rows of dw are aligned to 16 bytes
};

// Adds to a tile's sums what rounding left of the targets' dz: rest times h for every kept row whose word is one of the tile's.  Each wavefront looks
// through its share of the labels; what all found is the contraction of further steps, whose matrix of dz has one value to a row.
// Rows are added in an order that their places decide.  The first labels are loaded before the tile's product, and rows while those before them are
// multiplied: nothing else runs beside the largest tiles, and each load that is waited for costs them a microsecond.  Measured, dw alone, without and with: 8,192 rows x
// 4,096 x 32,000 1,660 and 1,680 us; 1,200 rows x 1,536 x 50,021 180 and 191, 196 where half of the rows have one tile's words, 221 where all have; 700 rows x
// 800 x 5,000, half of them of one tile's words, 15 and 23.
template <class C, class T>
struct Targets {
  static constexpr int WAVES = C::THREADS / CCLD_WAVE, SHARE = C::BM == 256 ? 512 : 256, AT_ONCE = WAVES * SHARE;
  static constexpr int STEPS = std::is_same_v<C, Short> ? 1 : 2, ROWS = 32 * STEPS;      // of a contraction, by the room in LDS
  static constexpr int TURN = 4 * CCLD_WAVE;           // labels that a wavefront loads at once
  typedef __attribute__((ext_vector_type(4))) int i32x4;
  typedef Operand<T, C::BN, ROWS, C::THREADS, true, false> H;
  struct Place { u32 list[WAVES][SHARE], count[WAVES]; };
  static constexpr int DZ = C::BM * ROWS * 2, STAGE = DZ + C::BN * ROWS * 2;        // a round's dz and h
  static_assert(AT_ONCE <= 1 << 16 && C::BM <= 1 << 16 && ROWS <= C::THREADS, "a row and a word to an entry");
  static_assert(2 * STAGE + sizeof(Place) <= C::LDS_BYTES, "room");

  i32x4 first;                                         // of the product's time

  // a lane's labels of a turn, or none (beyond the last are no rows': the workspace goes on behind them)
  __device__ __forceinline__ static int at_of(int turn) {
    return (turn * WAVES + (int)__builtin_amdgcn_readfirstlane(threadIdx.x / CCLD_WAVE)) * TURN + 4 * (int)lane_id();
  }
  __device__ __forceinline__ static i32x4 labels(const WeightJob& j, i64 base, int turn, int kept) {
    const i64 at = base + at_of(turn);
    return at < kept ? *reinterpret_cast<const i32x4*>(j.rows.label + at) : i32x4{-1, -1, -1, -1};
  }
  __device__ __forceinline__ void start(const WeightJob& j, int kept) { first = labels(j, 0, 0, kept); }

  template <class P>
  __device__ __forceinline__ void add(P& prod, const WeightJob& j, int kept, int n0, int ns, int k0) {
    Place& place = *reinterpret_cast<Place*>(lds + 2 * STAGE);
    const u32 lane = lane_id(), wave = threadIdx.x / CCLD_WAVE;
    const T* h = static_cast<const T*>(j.rows.h) + k0;
    H oh;
    oh.start(h, j.dp, min(C::BN, j.dp - k0));
    Fragments<C::BM, C::MI, ROWS, true> fz;
    Fragments<C::BN, C::NI, ROWS, true> fh;
    fz.start(prod.wave_m());
    fh.start(prod.wave_n());
    // dz's places are zeros but for one value to a row, which the row's thread takes back
    const s16x8 zeros = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int i = (int)threadIdx.x * 16; i < DZ; i += C::THREADS * 16) {
      *reinterpret_cast<s16x8*>(lds + i) = zeros;
      *reinterpret_cast<s16x8*>(lds + STAGE + i) = zeros;
    }
    short* mine[2] = {nullptr, nullptr};
    u32 turn = 0;
    const int from = j.first + n0;
    for (i64 base = 0; base < kept; base += AT_ONCE) {
      i32x4 label = base ? labels(j, base, 0, kept) : first;
      u32 n = 0;
      for (int turn = 0; turn < SHARE / TURN && base + turn * (WAVES * TURN) < kept; ++turn) {
        const i32x4 then = labels(j, turn + 1 < SHARE / TURN ? base : kept, turn + 1, kept);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = at_of(turn) + e, word = label[e] - from;
          const bool in = base + at < kept && word >= 0 && word < ns;
          const u64 mask = ballot64(in);
          if (in) place.list[wave][n + mbcnt64(mask)] = (u32)at << 16 | (u32)word;
          n += (u32)__popcll(mask);
        }
        label = then;
      }
      if (lane == 0) place.count[wave] = n;
      __syncthreads();
      u32 found = 0, before[WAVES];
#pragma unroll
      for (int i = 0; i < WAVES; ++i) {
        before[i] = found;
        found += (u32)__builtin_amdgcn_readfirstlane((int)place.count[i]);
      }
      // entry k of all that were found, or none
      auto entry = [&](u32 k) {
        u32 at = k;
#pragma unroll
        for (int i = 1; i < WAVES; ++i) at = k >= before[i] ? i * SHARE + k - before[i] : at;
        return k < found ? (&place.list[0][0])[at] : 0xFFFFFFFFu;
      };
      s16x8 next[H::PIECES];
      int next_word = -1;
      float next_rest = 0;
      auto fetch = [&](u32 at) {
#pragma unroll
        for (int i = 0; i < H::PIECES; ++i) {
          const u32 e = entry(at + oh.row + i * H::ROW_STEP);
          const int x = (int)oh.column(i);
          next[i] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
          if (e != 0xFFFFFFFFu && x < oh.left) next[i] = *reinterpret_cast<const s16x8*>(h + (base + (e >> 16)) * j.dp + x);
        }
        if (threadIdx.x < ROWS) {
          const u32 e = entry(at + threadIdx.x);
          next_word = e != 0xFFFFFFFFu ? (int)(e & 0xFFFF) : -1;
          next_rest = e != 0xFFFFFFFFu ? j.rows.rest[base + (e >> 16)] : 0;
        }
      };
      if (found) fetch(0);
      // a place is written again two rounds on, when all have passed the barrier of the round between
      for (u32 at = 0; at < found; at += ROWS, turn ^= 1) {
        unsigned char *dz = lds + turn * STAGE, *rows = dz + DZ;
#pragma unroll
        for (int i = 0; i < H::PIECES; ++i) H::put(rows, i, next[i]);
        if (threadIdx.x < ROWS) {
          short*& place_of = turn ? mine[1] : mine[0];
          if (place_of) *place_of = 0;
          place_of = nullptr;
          if (next_word >= 0) {
            const u32 c = threadIdx.x, x = (u32)next_word;
            place_of = reinterpret_cast<short*>(dz + c * (C::BM * 2) + ((x / 16) ^ across_key<C::BM>(c)) * 32 + x % 16 * 2);
            *place_of = __builtin_bit_cast(short, (T)next_rest);
          }
        }
        __syncthreads();
        if (at + ROWS < found) fetch(at + ROWS);
        for (int step = 0; step < STEPS && at + 32 * step < found; ++step) {
          s16x8 vh[C::NI];
#pragma unroll
          for (int b = 0; b < C::NI; ++b) vh[b] = fh.read(rows, b, step);
#pragma unroll
          for (int i = 0; i < C::MI; ++i) {
            const s16x8 v = fz.read(dz, i, step);
#pragma unroll
            for (int b = 0; b < C::NI; ++b) prod.acc[i][b] = mma(vh[b], v, prod.acc[i][b], T());
          }
        }
      }
      __syncthreads();               // the lists and places are read
    }
  }
};

template <class C, class T>
__global__ __launch_bounds__(C::THREADS, C::WAVES) void k_weight_grad(WeightJob j) {
  const u32 id = xcd_order(blockIdx.x, gridDim.x);
  const uint2 t = grouped_order(id, j.n_tiles, j.k_tiles, 8);
  const int n0 = (int)t.x * C::BM, k0 = (int)t.y * C::BN;
  const u32 parts = dz_parts(j.rows.count[0]);
  const int kept = (int)(j.rows.count[0] * parts);
  const int share = ((kept + (int)gridDim.y - 1) / (int)gridDim.y + C::DEPTH - 1) / C::DEPTH * C::DEPTH;
  const i64 first = (i64)blockIdx.y * share;
  const int depth = (int)max((i64)0, min((i64)share, kept - first));
  const i64 at = depth ? first : 0;
  // dz has whole tiles of columns, h rows padded to 16 bytes
  const int ns = min(C::BM, j.width - n0), ks = min(C::BN, j.d - k0);
  const bool has_targets = parts == 1 && blockIdx.y == 0;
  Targets<C, T> targets;
  if (has_targets) targets.start(j, kept);
  TileProduct<C, T, true, true, true> prod;
  prod.run(lds, static_cast<const T*>(j.dz) + at * j.lddz + n0, j.lddz, C::BM, static_cast<const T*>(j.rows.h) + at * j.dp + k0, j.dp,
           min(C::BN, j.dp - k0), depth);
  if (has_targets) targets.add(prod, j, kept, n0, ns, k0);
  if (j.part) {
    float* q = j.part + ((i64)blockIdx.y * j.width + n0) * j.d + k0;
    prod.each([&](u32 m, u32 n, f32x4 v) { if ((int)m < ns) store4(q + (i64)m * j.d + n, v, ks - (int)n, j.d % 4 == 0); });
  } else {
    const float back = ldexpf(1.0f, -reinterpret_cast<const i32*>(j.rows.count)[1]);
    // (beyond a few rows a stream whatever the lines: the vocabulary's weights, which are read again, stay in the memory's cache.  148 rows,
    // 1,392 x 109,201: 430 us for the whole step and 455; 57 rows, 1,432 x 55,406: 190 and 174)
    const bool stream = !std::is_same_v<C, Short> || streams(j.lddw, depth);
    prod.store(lds, static_cast<T*>(j.dw) + (i64)n0 * j.lddw + k0, j.lddw, ns, ks, j.whole, stream, back);
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_weight_rows(Rows w, const float* __restrict__ part, u32 splits, i64 width, int d, T* dw, i64 lddw) {
  const float back = ldexpf(1.0f, -reinterpret_cast<const i32*>(w.count)[1]);
  for (i64 i = (i64)blockIdx.x * 256 + threadIdx.x; i < width * d; i += (i64)gridDim.x * 256) {
    const i64 r = i / d, c = i - r * d;
    float v = 0;
    for (u32 s = 0; s < splits; ++s) v += part[(i64)s * width * d + i];
    dw[r * lddw + c] = (T)(v * back);
  }
}


i64 div_up(i64 a, i64 b) { return (a + b - 1) / b; }
i64 round_up(i64 a, i64 b) { return div_up(a, b) * b; }

// rows of dz, all parts, at most: how many rows are kept is known on the device
i64 dz_rows(const ccld_vocab_args* a) { return std::max(a->rows, std::min<i64>(a->rows, TWO_PARTS) * 2); }

// The vocabulary's weights are loaded to LDS directly where pieces of 16 bytes lie wholly inside or outside them and start on 16 bytes, else through
// registers, which the largest tiles have none to spare for: tiles go by addresses too.  The workspace does not: it serves both.
bool whole_pieces(const ccld_vocab_args* a) { return a->d % 8 == 0 && a->ldw % 8 == 0; }
bool is_direct(const ccld_vocab_args* a) { return whole_pieces(a) && aligned(a->w, 16); }

// for rows x cols of results; less than 48 rows are bound by reading the vocabulary's weights
Tile choose_tile(i64 rows, i64 cols, i64 depth, bool direct, u32 most_splits) {
  return rows < 48 ? FEW : choose_cut((u64)rows, (u64)cols, (u64)depth, direct, most_splits).tile;
}
// Logits cannot be split along their contraction: where there are few tiles, smaller ones, so that more compute units read the weights.  60 rows, a vocabulary
// of 3,047, 1,976 deep: 16.1 us in tiles of 32 x 32, 20.9 of 32 x 128, 25.5 of 128 x 128; 345 rows, 2,232, 944 deep: 20.1, 16.9 and 21.0; 100 rows,
// 20,000, 1,000 deep: 41, 30 and 24.5.
Tile logit_tiles(i64 rows, i64 cols, i64 depth, bool direct) {
  const i64 few = div_up(rows, Few::BM) * div_up(cols, Few::BN);
  return few < (i64)COMPUTE_UNITS / 2 ? NARROW : few <= (i64)COMPUTE_UNITS ? FEW : choose_tile(rows, cols, depth, direct, 1);
}

// dz of a piece, both of its parts, is 2^28 values (512 MB) and a line of 256 to a row at most, up to 65,536 rows; more rows have pieces of 4,096 columns all the same,
// 8 KB to a row.  A piece has 2^21 columns at most: a tile of dz is reached by 32-bit offsets.
i64 piece_width(const ccld_vocab_args* a) {
  const i64 w = std::min<i64>(std::max<i64>(round_up(((i64)1 << 28) / std::max<i64>(dz_rows(a), 1), 256), 4096), (i64)1 << 21);
  const i64 pieces = div_up(a->vocab, w);
  return round_up(div_up(a->vocab, pieces), 256);
}
static_assert(((i64)1 << 21) + 256 < MAX_LD, "dz's rows");

struct Carver {
  uint8_t* base; u64 off;
  template <class V> V* take(u64 count) {
    off = (off + 255) & ~(u64)255;
    V* p = base ? reinterpret_cast<V*>(base + off) : nullptr;
    off += count * sizeof(V);
    return p;
  }
};

struct Plan {
  bool direct;
  Rows rows;
  int dp;
  // loss
  Tile logits;
  u32 col_tiles;
  float2* part;
  // gradient
  i64 width;
  uint16_t* dz;
  Tile input;
  u32 pieces;              // workgroups for dh at most
  float* sum;
  Tile weight;
  u32 weight_splits;
  float* weight_part;
};

Plan make_plan(const ccld_vocab_args* a, bool grad, bool direct, Carver& c) {
  Plan p{};
  p.direct = direct;
  const u64 rows = (u64)a->rows;
  p.dp = (int)round_up(a->d, 8);
  const u64 all = grad ? (u64)dz_rows(a) : rows;
  p.rows.count = c.take<u32>(2);
  p.rows.row = c.take<i32>(rows);
  p.rows.place = c.take<i32>(rows);
  p.rows.label = c.take<i32>(rows);
  p.rows.target = c.take<float>(rows);
  p.rows.lse = c.take<float>(rows);
  p.rows.scale = c.take<float>(rows);
  p.rows.rest = c.take<float>(rows);
  p.rows.h = c.take<uint16_t>(all * p.dp);
  if (!grad) {
    p.logits = logit_tiles(a->rows, a->vocab, a->d, direct);
    p.col_tiles = (u32)div_up(a->vocab, tile_n(p.logits));
    p.part = c.take<float2>(rows * p.col_tiles);
    return p;
  }
  p.width = piece_width(a);
  p.logits = logit_tiles(a->rows, p.width, a->d, direct);
  p.col_tiles = (u32)div_up(p.width, tile_n(p.logits));
  p.dz = c.take<uint16_t>(all * p.width);
  if (a->dh) {
    // the parts of the contraction are chosen on the device, by the rows that have a target: pieces are bounded, not parts
    p.input = choose_tile((i64)all, a->d, p.width, direct, MOST_SPLITS);
    const u64 tiles = (u64)div_up((i64)all, tile_m(p.input)) * div_up(a->d, tile_n(p.input));
    p.pieces = (u32)std::max<u64>(tiles, MOST_PIECES);
    p.sum = c.take<float>(std::max<u64>(all * a->d, (u64)MOST_PIECES * tile_m(p.input) * tile_n(p.input)));
  }
  if (a->dw) {
    const Cut w = choose_weight_cut((u64)p.width, (u64)a->d, all, true);
    p.weight = w.tile;
    p.weight_splits = w.splits;
    if (p.weight_splits > 1) p.weight_part = c.take<float>((u64)p.weight_splits * p.width * a->d);
  }
  return p;
}

ccld_status check(const ccld_vocab_args* a, bool grad) {
  if (!a) return CCLD_E_NULL;
  if ((a->dtype != CCLD_BF16 && a->dtype != CCLD_FP16) || (a->label_bits != 32 && a->label_bits != 64)) return CCLD_E_BAD_ARG;
  if (a->rows < 0 || a->d < 1 || a->vocab < 1) return CCLD_E_BAD_ARG;
  if (a->rows >= MAX_ROWS || a->vocab >= MAX_ROWS - 512 || a->d >= MAX_LD) return CCLD_E_CAPACITY;
  if (a->ldh < a->d || a->ldw < a->d) return CCLD_E_BAD_ARG;
  if (a->ldw >= MAX_LD) return CCLD_E_CAPACITY;
  if (grad && (a->dloss_stride < 0 || (a->dh && a->lddh < a->d) || (a->dw && a->lddw < a->d))) return CCLD_E_BAD_ARG;
  const i64 cols = grad ? piece_width(a) : a->vocab;
  auto fits = [](Tile t, i64 m, i64 n) { return launches(t, (u64)div_up(m, tile_m(t)) * div_up(n, tile_n(t))); };
  const i64 all = dz_rows(a);
  for (bool direct : {false, true}) {
    if (!fits(logit_tiles(a->rows, cols, a->d, direct), a->rows, cols)) return CCLD_E_CAPACITY;
    if (grad && !fits(choose_tile(all, a->d, cols, direct, MOST_SPLITS), all, a->d)) return CCLD_E_CAPACITY;
  }
  if (grad && !fits(choose_weight_cut((u64)cols, (u64)a->d, (u64)all, true).tile, cols, a->d)) return CCLD_E_CAPACITY;
  return CCLD_OK;
}

ccld_status check_pointers(const ccld_vocab_args* a, bool grad) {
  if (!a->w || (a->rows && (!a->h || !a->labels))) return CCLD_E_NULL;
  if (a->rows && (grad ? !a->lse || !a->dloss : !a->loss || !a->lse)) return CCLD_E_NULL;
  if (!aligned(a->labels, a->label_bits / 8)) return CCLD_E_BAD_ARG;
  for (const void* p : {a->h, a->w, (const void*)a->dh, (const void*)a->dw})
    if (!aligned(p, 2)) return CCLD_E_BAD_ARG;
  for (const void* p : {(const void*)a->dloss, (const void*)a->loss, (const void*)a->lse})
    if (!aligned(p, 4)) return CCLD_E_BAD_ARG;
  uint64_t need = 0;
  const ccld_status s = ccld_vocab_workspace(a, grad, &need);
  if (s != CCLD_OK) return s;
  if (!a->workspace || !aligned(a->workspace, 256) || a->workspace_bytes < need) return CCLD_E_WORKSPACE;
  return CCLD_OK;
}

u32 stream_groups(i64 threads) { return (u32)std::min<i64>(std::max<i64>(div_up(threads, 256), 1), 4096); }

template <class T, int V>
void start_rows(const ccld_vocab_args* a, const Plan& p, bool grad, hipStream_t stream) {
  const T* h = static_cast<const T*>(a->h);
  const float *lse = grad ? a->lse : nullptr, *dloss = grad ? a->dloss : nullptr;
  float *loss = grad ? nullptr : a->loss, *lse_out = grad ? nullptr : a->lse;
  const i64 pieces = a->rows * (p.dp / V);
  const bool few = a->rows <= USED_THREADS;
  const auto used = few ? &k_used_rows<T, V, true> : &k_used_rows<T, V, false>;
  used<<<few ? (u32)std::min<i64>(std::max<i64>(div_up(pieces, USED_THREADS), 1), (i64)COMPUTE_UNITS) : 1, USED_THREADS, 0, stream>>>(
      p.rows, a->labels, a->label_bits, a->rows, a->vocab, loss, lse_out, h, a->ldh, (int)a->d, p.dp, lse, dloss, a->dloss_stride);
  if (!few) k_gather_rows<T, V><<<stream_groups(pieces), 256, 0, stream>>>(p.rows, h, a->ldh, (int)a->d, p.dp, lse, dloss, a->dloss_stride);
}
template <class T>
void start(const ccld_vocab_args* a, const Plan& p, bool grad, hipStream_t stream) {
  if (a->d % 8 == 0 && a->ldh % 8 == 0 && aligned(a->h, 16)) start_rows<T, 8>(a, p, grad, stream);
  else start_rows<T, 1>(a, p, grad, stream);
}

// whether a tiling's kernels that are not direct are: the largest tiles, which no plan through registers takes, have the direct ones alone
template <class C>
constexpr bool ELSE_DIRECT = std::is_same_v<C, Large>;

template <class C, class T>
void launch_logit_sums(const ccld_vocab_args* a, const Plan& p, const LogitJob& j, hipStream_t stream) {
  const u32 grid = (u32)(div_up(a->rows, C::BM) * j.col_tiles);
  const auto kernel = p.direct ? &k_logit_sums<C, T, true> : &k_logit_sums<C, T, ELSE_DIRECT<C>>;
  kernel<<<grid, C::THREADS, C::LDS_BYTES, stream>>>(j);
}
template <class C, class T>
void launch_logit_grad(const ccld_vocab_args* a, const Plan& p, LogitJob j, hipStream_t stream) {
  j.col_tiles = (u32)div_up(j.cols, C::BN);
  const u32 grid = (u32)(div_up(a->rows, C::BM) * j.col_tiles);
  const auto kernel = p.direct ? &k_logit_grad<C, T, true> : &k_logit_grad<C, T, ELSE_DIRECT<C>>;
  kernel<<<grid, C::THREADS, C::LDS_BYTES, stream>>>(j);
}
template <class C, class T>
void launch_input_grad(const Plan& p, InputJob j, hipStream_t stream) {
  j.col_tiles = (u32)div_up(j.d, C::BN);
  const auto kernel = p.direct ? &k_input_grad<C, T, true> : &k_input_grad<C, T, ELSE_DIRECT<C>>;
  kernel<<<p.pieces, C::THREADS, C::LDS_BYTES, stream>>>(j);
}
template <class C, class T>
void launch_input_rows(const ccld_vocab_args* a, const Plan& p, hipStream_t stream) {
  const int d = (int)a->d;
  const bool wide = d % 4 == 0 && a->lddh % 4 == 0 && aligned(a->dh, 8);
  const auto kernel = wide ? &k_input_rows<C, T, 4> : &k_input_rows<C, T, 1>;
  kernel<<<stream_groups(a->rows * a->d / (wide ? 4 : 1)), 256, 0, stream>>>(p.rows, p.sum, (u32)div_up(d, C::BN), (int)p.width, a->rows, d,
                                                                            static_cast<const T*>(a->w), a->ldw, static_cast<T*>(a->dh), a->lddh);
}
template <class C, class T>
void launch_weight_grad(const Plan& p, WeightJob j, hipStream_t stream) {
  j.n_tiles = (u32)div_up(j.width, C::BM);
  j.k_tiles = (u32)div_up(j.d, C::BN);
  const auto kernel = &k_weight_grad<C, T>;
  kernel<<<dim3(j.n_tiles * j.k_tiles, p.weight_splits), C::THREADS, C::LDS_BYTES, stream>>>(j);
}

template <class T>
ccld_status loss(const ccld_vocab_args* a, const Plan& p, hipStream_t stream) {
  start<T>(a, p, false, stream);
  const LogitJob j{p.rows, a->w, a->ldw, (int)a->d, p.dp, 0, (int)a->vocab, p.col_tiles, p.part, nullptr, 0};
  if (p.logits == LARGE) launch_logit_sums<Large, T>(a, p, j, stream);
  else if (p.logits == MEDIUM) launch_logit_sums<Medium, T>(a, p, j, stream);
  else if (p.logits == FEW) launch_logit_sums<Few, T>(a, p, j, stream);
  else launch_logit_sums<Narrow, T>(a, p, j, stream);
  for (i64 first = 0; first < a->rows; first += 4 * most_groups(256))
    k_loss<<<(u32)std::min(div_up(a->rows - first, 4), most_groups(256)), 256, 0, stream>>>(p.rows, first, p.part, p.col_tiles, a->loss, a->lse);
  return launched();
}

template <class T>
ccld_status gradient(const ccld_vocab_args* a, const Plan& p, hipStream_t stream) {
  start<T>(a, p, true, stream);
  for (i64 first = 0; first < a->vocab; first += p.width) {
    const i64 cols = std::min<i64>(p.width, a->vocab - first);
    const T* w = static_cast<const T*>(a->w) + first * a->ldw;
    if (a->rows) {
      const LogitJob j{p.rows, w, a->ldw, (int)a->d, p.dp, (int)first, (int)cols, 0, nullptr, p.dz, p.width};
      if (p.logits == LARGE) launch_logit_grad<Large, T>(a, p, j, stream);
      else if (p.logits == MEDIUM) launch_logit_grad<Medium, T>(a, p, j, stream);
      else if (p.logits == FEW) launch_logit_grad<Few, T>(a, p, j, stream);
      else launch_logit_grad<Narrow, T>(a, p, j, stream);
    }
    if (a->dh && a->rows) {
      const InputJob j{p.rows, p.dz, w, p.width, a->ldw, (int)a->d, (int)cols, (int)p.width, 0, p.sum, first > 0};
      if (p.input == LARGE) launch_input_grad<Large, T>(p, j, stream);
      else if (p.input == MEDIUM) launch_input_grad<Medium, T>(p, j, stream);
      else launch_input_grad<Few, T>(p, j, stream);
    }
    if (a->dw) {
      T* dw = static_cast<T*>(a->dw) + first * a->lddw;
      const WeightJob j{p.rows, p.dz, p.width, dw, a->lddw, (int)first, (int)a->d, p.dp, (int)cols, 0, 0, p.weight_part,
                        a->lddw % 8 == 0 && aligned(dw, 16)};
      if (p.weight == LARGE) launch_weight_grad<Large, T>(p, j, stream);
      else if (p.weight == MEDIUM) launch_weight_grad<Medium, T>(p, j, stream);
      else launch_weight_grad<Short, T>(p, j, stream);
      if (p.weight_part)
        k_weight_rows<T><<<stream_groups(cols * a->d), 256, 0, stream>>>(p.rows, p.weight_part, p.weight_splits, cols, (int)a->d, dw, a->lddw);
    }
  }
  if (a->dh && a->rows) {
    if (p.input == LARGE) launch_input_rows<Large, T>(a, p, stream);
    else if (p.input == MEDIUM) launch_input_rows<Medium, T>(a, p, stream);
    else launch_input_rows<Few, T>(a, p, stream);
  }
  return launched();
}

template <class C, class T>
hipError_t allow_tiling() {
  hipError_t e = hipSuccess;
  auto allow = [&](auto k) { if (e == hipSuccess) e = allow_lds(reinterpret_cast<const void*>(k), C::LDS_BYTES); };
  if constexpr (!std::is_same_v<C, Short>) {
    allow(&k_logit_sums<C, T, true>);
    allow(&k_logit_sums<C, T, ELSE_DIRECT<C>>);
    allow(&k_logit_grad<C, T, true>);
    allow(&k_logit_grad<C, T, ELSE_DIRECT<C>>);
  }
  if constexpr (C::BN > 32 && !std::is_same_v<C, Short>) {
    allow(&k_input_grad<C, T, true>);
    allow(&k_input_grad<C, T, ELSE_DIRECT<C>>);
  }
  if constexpr (C::BM > 32) allow(&k_weight_grad<C, T>);
  return e;
}

}  // namespace

namespace ccld {
hipError_t allow_lds_vocab() {
  for (hipError_t e : {allow_tiling<Large, __bf16>(), allow_tiling<Large, _Float16>(), allow_tiling<Medium, __bf16>(),
                       allow_tiling<Medium, _Float16>(), allow_tiling<Short, __bf16>(), allow_tiling<Short, _Float16>(), allow_tiling<Few, __bf16>(),
                       allow_tiling<Few, _Float16>(), allow_tiling<Narrow, __bf16>(), allow_tiling<Narrow, _Float16>()})
    if (e != hipSuccess) return e;
  return hipSuccess;
}
}  // namespace ccld

extern "C" ccld_status ccld_vocab_workspace(const ccld_vocab_args* a, int32_t grad, uint64_t* bytes) {
  if (!bytes) return CCLD_E_NULL;
  const ccld_status s = check(a, grad != 0);
  if (s != CCLD_OK) return s;
  u64 need = 0;
  for (bool direct : {false, true}) {
    if (direct && !whole_pieces(a)) continue;
    Carver c{nullptr, 0};
    (void)make_plan(a, grad != 0, direct, c);
    need = std::max(need, c.off);
  }
  *bytes = (need + 255) & ~(u64)255;
  return CCLD_OK;
}

extern "C" ccld_status ccld_vocab_loss(const ccld_vocab_args* a, void* stream) {
  ccld_status s = check(a, false);
  if (s == CCLD_OK) s = check_pointers(a, false);
  if (s == CCLD_OK) s = ccld_device_init();
  if (s != CCLD_OK || a->rows == 0) return s;
  Carver c{static_cast<uint8_t*>(a->workspace), 0};
  const Plan p = make_plan(a, false, is_direct(a), c);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return a->dtype == CCLD_BF16 ? loss<__bf16>(a, p, st) : loss<_Float16>(a, p, st);
}

extern "C" ccld_status ccld_vocab_loss_grad(const ccld_vocab_args* a, void* stream) {
  ccld_status s = check(a, true);
  if (s == CCLD_OK) s = check_pointers(a, true);
  if (s == CCLD_OK) s = ccld_device_init();
  if (s != CCLD_OK) return s;
  Carver c{static_cast<uint8_t*>(a->workspace), 0};
  const Plan p = make_plan(a, true, is_direct(a), c);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return a->dtype == CCLD_BF16 ? gradient<__bf16>(a, p, st) : gradient<_Float16>(a, p, st);
}
