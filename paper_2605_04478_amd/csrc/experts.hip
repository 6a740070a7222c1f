// Matrix products grouped by expert, with ragged numbers of rows, and their gradients (ccld_expert_*).
//
//   y[r] = x[r] w_e^T      dx[r] = dy[r] w_e      dw_e = sum over e's rows of dy[r]^T x[r]
//
// One launch for all experts: the host knows how many rows there are but not whose, so it launches as many workgroups as the
// worst division of the rows needs and each finds its tile in the offsets (a prefix sum over the experts' tile counts by a
// wavefront); those beyond the last tile end at once.  What bounds the kernels: the matrix cores from about 500 rows for an expert on, moving
// the experts' weights below 128, both and the start and end of a tile's work between.
//
// Measured (bfloat16 unless said, on one of several cards, whose matrix cores differ by 7 %; a copy of 2 GB moves 4.9 TB/s here, reads alone more): 37 rows of 16 experts, 4,096 x 2,048 each, 37 us = 7.3 TB/s where
// the weights lie in the memory's cache, 48 us = 5.6 TB/s where not; 32,768 rows of 32 experts, 4,096 x 4,096, 3.0 ms for the three products = 1,090
// TFLOP/s, 1,230 with the ragged ends of the tiles, which are 13 % of the work; 8,192 rows of 64 experts, 1,024 x 2,048, half precision, 265 us = 390
// TFLOP/s and 2.4 TB/s; 5,003 rows of 12 experts, 1,336 x 1,000, 28, 29 and 41 us.
#include <algorithm>

#include "ccld_internal.h"
#include "products.h"
#include "tiles.h"

using namespace ccld;

namespace {

extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

struct Offsets {
  const void* at; int bits; int rows; u32 n_experts;
  __device__ __forceinline__ int get(u32 e) const {
    const i64 v = bits == 64 ? static_cast<const i64*>(at)[e] : (i64)static_cast<const i32*>(at)[e];
    return v < 0 ? 0 : v > rows ? rows : (int)v;
  }
  // rows of a part: the experts, then the rows before the first and after the last one, which are nobody's
  __device__ __forceinline__ int2 range(u32 e) const {
    if (e < n_experts) { const int a = get(e), b = get(e + 1); return make_int2(a, b > a ? b : a); }
    return e == n_experts ? make_int2(0, get(0)) : make_int2(get(n_experts), rows);
  }
};

struct RowJob {              // y or dx
  const void *a, *w;         // x or dy; the weights
  void* out;
  float* part;               // [splits][rows][cols] sums of the splits, or null: `out` is written
  Offsets off;
  i64 lda, ldw, estride, ldo;
  int cols, depth, split_depth;
  u32 col_tiles;
  bool whole;                // rows of out are aligned to 16 bytes
};

struct WeightJob {           // dw
  const void *dy, *x;
  void* out;
  float* part;               // [splits][n_experts][n][k]
  Offsets off;
  i64 lddy, ldx;
  int n, k;
  u32 n_tiles, k_tiles;
  bool whole;
};

// The tile of a workgroup: the part that it belongs to, that part's first m-tile (of BM rows, counted over all parts), number of m-tiles and
// rows, and the tile's number within it.  part is n_experts + 2 for workgroups beyond the last tile.  Every wavefront finds it by
// itself, 64 parts at a time: once for the number of tiles, which the XCDs share evenly, and once for its own.
struct Place { u32 part, at, tiles; int2 range; };
template <int BM>
__device__ __forceinline__ Place find_tile(const Offsets& off, u32 block, u32 col_tiles) {
  const u32 parts = off.n_experts + 2, lane = lane_id();
  auto part_tiles = [&](u32 e, int2& r) {
    r = e < parts ? off.range(e) : make_int2(0, 0);
    return (u32)(r.y - r.x + BM - 1) / BM;
  };
  int2 r;
  u32 total = 0;
  for (u32 base = 0; base < parts; base += CCLD_WAVE)
    total += __builtin_amdgcn_readlane((int)wave_inclusive_sum(part_tiles(base + lane, r)), CCLD_WAVE - 1);
  const Place none{parts, 0, 0, make_int2(0, 0)};
  if (block >= total * col_tiles) return none;
  const u32 id = xcd_order(block, total * col_tiles);
  u32 before = 0;
  for (u32 base = 0; base < parts; base += CCLD_WAVE) {
    const u32 t = part_tiles(base + lane, r), incl = before + wave_inclusive_sum(t);
    const u64 hit = ballot64(id < incl * col_tiles);
    if (hit) {
      const int src = __builtin_ctzll(hit);
      Place p;
      p.part = base + src;
      p.tiles = __builtin_amdgcn_readlane((int)t, src);
      p.at = id - (__builtin_amdgcn_readlane((int)incl, src) - p.tiles) * col_tiles;
      p.range = make_int2(__builtin_amdgcn_readlane(r.x, src), __builtin_amdgcn_readlane(r.y, src));
      return p.at < p.tiles * col_tiles ? p : none;     // (offsets that decrease can make the counts pass 32 bits)
    }
    before = __builtin_amdgcn_readlane((int)incl, CCLD_WAVE - 1);
  }
  return none;
}

template <class C, class T, bool W_ACROSS, bool DIRECT>
__global__ __launch_bounds__(C::THREADS) void k_expert_rows(RowJob j) {
  const Place p = find_tile<C::BM>(j.off, blockIdx.x, j.col_tiles);
  if (p.part >= j.off.n_experts + 2) return;
  const uint2 t = grouped_order(p.at, p.tiles, j.col_tiles, 8);
  const int row0 = p.range.x + (int)t.x * C::BM, col0 = (int)t.y * C::BN;
  const int c0 = (int)blockIdx.y * j.split_depth;
  int depth = min(j.split_depth, j.depth - c0);
  if (p.part >= j.off.n_experts || depth < 0) depth = 0;       // nobody's rows: zeros
  const u32 e = p.part < j.off.n_experts ? p.part : 0;
  const int rows = min(C::BM, p.range.y - row0), cols = min(C::BN, j.cols - col0);
  const T* w = static_cast<const T*>(j.w) + (i64)e * j.estride + (W_ACROSS ? (i64)c0 * j.ldw + col0 : (i64)col0 * j.ldw + c0);
  TileProduct<C, T, false, W_ACROSS, DIRECT> prod;
  prod.run(lds, static_cast<const T*>(j.a) + (i64)row0 * j.lda + c0, j.lda, rows, w, j.ldw, cols, depth);
  if (j.part) {
    float* o = j.part + ((i64)blockIdx.y * j.off.rows + row0) * j.cols + col0;
    prod.each([&](u32 m, u32 n, f32x4 v) { if ((int)m < rows) store4(o + (i64)m * j.cols + n, v, cols - (int)n, j.cols % 4 == 0); });
  } else {
    prod.store(lds, static_cast<T*>(j.out) + (i64)row0 * j.ldo + col0, j.ldo, rows, cols, j.whole, streams(j.ldo, j.depth), 1.0f);
  }
}

template <class C, class T, bool DIRECT>
__global__ __launch_bounds__(C::THREADS, C::WAVES) void k_expert_weights(WeightJob j) {
  // every expert's tiles are divided among the XCDs, since experts differ in their rows (an expert after another to an XCD: 1.5
  // times the time at 32 experts whose rows spread like exp(0.7 N)).  Workgroups of the same number modulo 8 share an XCD within an
  // expert too, whichever its first one has.
  const u32 tiles = j.n_tiles * j.k_tiles, e = blockIdx.x / tiles;
  const uint2 t = grouped_order(xcd_order(blockIdx.x - e * tiles, tiles), j.n_tiles, j.k_tiles, 8);
  const int n0 = (int)t.x * C::BM, k0 = (int)t.y * C::BN;
  const int2 r = j.off.range(e);
  // this split's rows: an equal share, in whole stages
  const int share = ((r.y - r.x + (int)gridDim.y - 1) / (int)gridDim.y + C::DEPTH - 1) / C::DEPTH * C::DEPTH;
  const i64 first = r.x + (i64)blockIdx.y * share;
  const int depth = (int)max((i64)0, min((i64)share, r.y - first));
  const i64 at = depth ? first : 0;
  const int ns = min(C::BM, j.n - n0), ks = min(C::BN, j.k - k0);
  TileProduct<C, T, true, true, DIRECT> prod;
  prod.run(lds, static_cast<const T*>(j.dy) + at * j.lddy + n0, j.lddy, ns, static_cast<const T*>(j.x) + at * j.ldx + k0, j.ldx,
           ks, depth);
  const i64 o = ((i64)e * j.n + n0) * j.k + k0;
  if (j.part) {
    float* q = j.part + (i64)blockIdx.y * j.off.n_experts * j.n * j.k + o;
    prod.each([&](u32 m, u32 n, f32x4 v) { if ((int)m < ns) store4(q + (i64)m * j.k + n, v, ks - (int)n, j.k % 4 == 0); });
  } else {
    prod.store(lds, static_cast<T*>(j.out) + o, j.k, ns, ks, j.whole, streams(j.k, depth), 1.0f);
  }
}


u64 div_up(u64 a, u64 b) { return (a + b - 1) / b; }

// How the rows' products are cut.  Experts with less than 48 rows on average are bound by reading their weights: tiles of 32 rows.
struct RowPlan { Tile tile; u32 col_tiles; u64 groups; u32 splits; int split_depth; };
RowPlan plan_rows(u64 rows, u64 experts, int cols, int depth, bool whole) {
  RowPlan p;
  const u64 busy = std::min(rows, experts), mean = rows / std::max<u64>(experts, 1), steps = div_up(depth, DEPTH);
  u64 s = 1;
  if (mean < 48) {
    p.tile = FEW;
    const u64 tiles = std::max<u64>(div_up(rows, 32), busy) * div_up(cols, 128);
    while (tiles * s < COMPUTE_UNITS && steps / (2 * s) >= 8) s *= 2;
  } else {
    // a part's last tile is half full on average
    const double m256 = std::max<double>(busy, rows / 256.0 + busy * 0.5), m128 = std::max<double>(busy, rows / 128.0 + busy * 0.5);
    const Cut c = choose_cut(m256 * div_up(cols, 256), m128 * div_up(cols, 128), 2 * steps, (double)rows * cols, busy == 1, whole);
    p.tile = c.tile;
    s = c.splits;
  }
  p.col_tiles = (u32)div_up(cols, tile_n(p.tile));
  // tiles of the worst division: every part may end in a tile of its own
  p.groups = (rows / tile_m(p.tile) + std::min(rows, experts + 2)) * p.col_tiles;
  p.split_depth = (int)(div_up(steps, s) * DEPTH);
  p.splits = (u32)div_up(steps, div_up(steps, s));
  return p;
}

struct WeightPlan { Tile tile; u32 n_tiles, k_tiles, splits; };
WeightPlan plan_weights(u64 rows, u64 experts, int n, int k, bool whole) {
  const Cut c = choose_weight_cut((u64)n, (u64)k, div_up(rows, experts), whole, experts);
  return WeightPlan{c.tile, (u32)div_up(n, tile_m(c.tile)), (u32)div_up(k, tile_n(c.tile)), c.splits};
}

// Pieces of 16 bytes lie wholly inside or outside the operands: x, dy, the weights.  Where they also start on 16 bytes they are loaded to LDS directly, else
// through registers, which the largest and the short tiles have none to spare for: tiles go by addresses too.  The workspace does not: it
// serves both.
bool whole_pieces(const ccld_expert_args* a, i64 ld) { return a->k % 8 == 0 && a->n % 8 == 0 && a->ldw % 8 == 0 && a->expert_stride % 8 == 0 && ld % 8 == 0; }
bool rows_whole(const ccld_expert_args* a, bool grad) { return whole_pieces(a, grad ? a->lddy : a->ldx); }
bool rows_direct(const ccld_expert_args* a, bool grad) { return rows_whole(a, grad) && aligned(a->w, 16) && aligned(grad ? a->dy : a->x, 16); }
bool weights_whole(const ccld_expert_args* a) { return a->n % 8 == 0 && a->k % 8 == 0 && a->lddy % 8 == 0 && a->ldx % 8 == 0; }
bool weights_direct(const ccld_expert_args* a) { return weights_whole(a) && aligned(a->dy, 16) && aligned(a->x, 16); }

RowPlan row_plan(const ccld_expert_args* a, bool grad, bool direct) {
  return plan_rows((u64)a->rows, (u64)a->n_experts, (int)(grad ? a->k : a->n), (int)(grad ? a->n : a->k), direct);
}
WeightPlan weight_plan(const ccld_expert_args* a, bool direct) { return plan_weights((u64)a->rows, (u64)a->n_experts, (int)a->n, (int)a->k, direct); }

ccld_status check(const ccld_expert_args* a, bool grad) {
  if (!a) return CCLD_E_NULL;
  if ((a->dtype != CCLD_BF16 && a->dtype != CCLD_FP16) || (a->offsets_bits != 32 && a->offsets_bits != 64)) return CCLD_E_BAD_ARG;
  if (a->rows < 0 || a->k < 1 || a->n < 1 || a->n_experts < 1) return CCLD_E_BAD_ARG;
  if (a->rows >= MAX_ROWS || a->n_experts >= MAX_EXPERTS || a->k >= MAX_WIDTH || a->n >= MAX_WIDTH) return CCLD_E_CAPACITY;
  if (a->ldw < a->k || a->expert_stride < 0 || a->ldx < a->k) return CCLD_E_BAD_ARG;
  if (a->ldw >= MAX_LD || a->ldx >= MAX_LD) return CCLD_E_CAPACITY;
  if (grad) {
    if (a->lddy < a->n || (a->dx && a->lddx < a->k)) return CCLD_E_BAD_ARG;
    if (a->lddy >= MAX_LD) return CCLD_E_CAPACITY;
  } else if (a->ldy < a->n) return CCLD_E_BAD_ARG;
  for (bool direct : {false, true}) {
    const RowPlan p = row_plan(a, grad, direct);
    if ((!grad || a->dx) && !launches(p.tile, p.groups)) return CCLD_E_CAPACITY;
    const WeightPlan w = weight_plan(a, direct);
    if (grad && a->dw && !launches(w.tile, (u64)a->n_experts * w.n_tiles * w.k_tiles)) return CCLD_E_CAPACITY;
  }
  return CCLD_OK;
}

ccld_status check_pointers(const ccld_expert_args* a, bool grad) {
  if (!a->offsets || !a->w) return CCLD_E_NULL;
  if (a->rows && (grad ? !a->dy || (a->dw && !a->x) : !a->x || !a->y)) return CCLD_E_NULL;
  if (!aligned(a->offsets, a->offsets_bits / 8)) return CCLD_E_BAD_ARG;
  for (const void* p : {a->x, a->w, a->dy, (const void*)a->y, (const void*)a->dx, (const void*)a->dw})
    if (!aligned(p, 2)) return CCLD_E_BAD_ARG;
  uint64_t need = 0;
  const ccld_status s = ccld_expert_workspace(a, grad, &need);
  if (s != CCLD_OK) return s;
  if (need && (!a->workspace || !aligned(a->workspace, 256) || a->workspace_bytes < need)) return CCLD_E_WORKSPACE;
  return CCLD_OK;
}

u64 row_part_bytes(const RowPlan& p, u64 rows, u64 cols) { return p.splits > 1 ? 4 * p.splits * rows * cols : 0; }
u64 weight_part_bytes(const WeightPlan& p, u64 experts, u64 n, u64 k) { return p.splits > 1 ? 4 * p.splits * experts * n * k : 0; }

template <class C, class T, bool W_ACROSS, bool DIRECT>
void launch_rows(const RowJob& j, const RowPlan& p, hipStream_t stream) {
  k_expert_rows<C, T, W_ACROSS, DIRECT><<<dim3((u32)p.groups, p.splits), C::THREADS, C::LDS_BYTES, stream>>>(j);
}
template <class T, bool W_ACROSS, bool DIRECT>
void launch_rows(const RowJob& j, const RowPlan& p, hipStream_t stream) {
  if constexpr (DIRECT)
    if (p.tile == LARGE) return launch_rows<Large, T, W_ACROSS, true>(j, p, stream);
  if (p.tile == MEDIUM) launch_rows<Medium, T, W_ACROSS, DIRECT>(j, p, stream);
  else launch_rows<Few, T, W_ACROSS, DIRECT>(j, p, stream);
}

template <class T>
ccld_status product_of_rows(const ccld_expert_args* a, bool grad, hipStream_t stream) {
  const int cols = (int)(grad ? a->k : a->n), depth = (int)(grad ? a->n : a->k);
  const bool d = rows_direct(a, grad);
  const RowPlan p = row_plan(a, grad, d);
  RowJob j{};
  j.a = grad ? a->dy : a->x;
  j.lda = grad ? a->lddy : a->ldx;
  j.w = a->w;
  j.out = grad ? a->dx : a->y;
  j.ldo = grad ? a->lddx : a->ldy;
  j.part = p.splits > 1 ? static_cast<float*>(a->workspace) : nullptr;
  j.off = Offsets{a->offsets, a->offsets_bits, (int)a->rows, (u32)a->n_experts};
  j.ldw = a->ldw; j.estride = a->expert_stride;
  j.cols = cols; j.depth = depth; j.split_depth = p.split_depth; j.col_tiles = p.col_tiles;
  j.whole = j.ldo % 8 == 0 && aligned(j.out, 16);
  if (grad) d ? launch_rows<T, true, true>(j, p, stream) : launch_rows<T, true, false>(j, p, stream);
  else d ? launch_rows<T, false, true>(j, p, stream) : launch_rows<T, false, false>(j, p, stream);
  if (j.part) launch_join(j.part, p.splits, (u64)a->rows, (u64)cols, j.out, j.ldo, a->dtype, stream);
  return launched();
}

template <class C, class T, bool DIRECT>
void launch_weights(const WeightJob& j, const WeightPlan& p, hipStream_t stream) {
  k_expert_weights<C, T, DIRECT><<<dim3(j.off.n_experts * p.n_tiles * p.k_tiles, p.splits), C::THREADS, C::LDS_BYTES, stream>>>(j);
}

template <class T>
ccld_status product_of_weights(const ccld_expert_args* a, hipStream_t stream) {
  const bool d = weights_direct(a);
  const WeightPlan p = weight_plan(a, d);
  WeightJob j{};
  j.dy = a->dy; j.x = a->x; j.out = a->dw;
  j.part = p.splits > 1 ? static_cast<float*>(a->workspace) : nullptr;
  j.off = Offsets{a->offsets, a->offsets_bits, (int)a->rows, (u32)a->n_experts};
  j.lddy = a->lddy; j.ldx = a->ldx; j.n = (int)a->n; j.k = (int)a->k;
  j.n_tiles = p.n_tiles; j.k_tiles = p.k_tiles;
  j.whole = a->k % 8 == 0 && aligned(a->dw, 16);
  if (!d) launch_weights<Medium, T, false>(j, p, stream);
  else if (p.tile == LARGE) launch_weights<Large, T, true>(j, p, stream);
  else if (p.tile == MEDIUM) launch_weights<Medium, T, true>(j, p, stream);
  else launch_weights<Short, T, true>(j, p, stream);
  if (j.part) launch_join(j.part, p.splits, (u64)a->n_experts * a->n, (u64)a->k, j.out, a->k, a->dtype, stream);
  return launched();
}

template <class C, class T>
hipError_t allow_tiling() {
  hipError_t e = hipSuccess;
  auto allow = [&](auto k) { if (e == hipSuccess) e = allow_lds(reinterpret_cast<const void*>(k), C::LDS_BYTES); };
  if constexpr (!std::is_same_v<C, Short>) {
    allow(&k_expert_rows<C, T, false, true>);
    allow(&k_expert_rows<C, T, true, true>);
  }
  if constexpr (std::is_same_v<C, Medium> || std::is_same_v<C, Few>) {
    allow(&k_expert_rows<C, T, false, false>);
    allow(&k_expert_rows<C, T, true, false>);
  }
  if constexpr (C::BM > 32) allow(&k_expert_weights<C, T, true>);
  if constexpr (std::is_same_v<C, Medium>) allow(&k_expert_weights<C, T, false>);
  return e;
}

}  // namespace

namespace ccld {
hipError_t allow_lds_experts() {
  for (hipError_t e : {allow_tiling<Large, __bf16>(), allow_tiling<Large, _Float16>(), allow_tiling<Medium, __bf16>(),
                       allow_tiling<Medium, _Float16>(), allow_tiling<Short, __bf16>(), allow_tiling<Short, _Float16>(), allow_tiling<Few, __bf16>(),
                       allow_tiling<Few, _Float16>()})
    if (e != hipSuccess) return e;
  return hipSuccess;
}
}  // namespace ccld

extern "C" ccld_status ccld_expert_workspace(const ccld_expert_args* a, int32_t grad, uint64_t* bytes) {
  if (!bytes) return CCLD_E_NULL;
  const ccld_status s = check(a, grad != 0);
  if (s != CCLD_OK) return s;
  u64 need = 0;
  auto rows = [&](bool direct) { need = std::max(need, row_part_bytes(row_plan(a, grad, direct), a->rows, grad ? a->k : a->n)); };
  auto weights = [&](bool direct) { need = std::max(need, weight_part_bytes(weight_plan(a, direct), a->n_experts, a->n, a->k)); };
  if (!grad || a->dx) rows(false);
  if ((!grad || a->dx) && rows_whole(a, grad)) rows(true);
  if (grad && a->dw) weights(false);                       // the two gradients follow one another: one workspace serves both
  if (grad && a->dw && weights_whole(a)) weights(true);
  *bytes = (need + 255) & ~(u64)255;
  return CCLD_OK;
}

extern "C" ccld_status ccld_expert_product(const ccld_expert_args* a, void* stream) {
  ccld_status s = check(a, false);
  if (s == CCLD_OK) s = check_pointers(a, false);
  if (s == CCLD_OK) s = ccld_device_init();
  if (s != CCLD_OK || a->rows == 0) return s;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return a->dtype == CCLD_BF16 ? product_of_rows<__bf16>(a, false, st) : product_of_rows<_Float16>(a, false, st);
}

extern "C" ccld_status ccld_expert_product_grad(const ccld_expert_args* a, void* stream) {
  ccld_status s = check(a, true);
  if (s == CCLD_OK) s = check_pointers(a, true);
  if (s == CCLD_OK) s = ccld_device_init();
  if (s != CCLD_OK) return s;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const bool bf = a->dtype == CCLD_BF16;
  if (a->dx && a->rows) s = bf ? product_of_rows<__bf16>(a, true, st) : product_of_rows<_Float16>(a, true, st);
  if (s == CCLD_OK && a->dw) s = bf ? product_of_weights<__bf16>(a, st) : product_of_weights<_Float16>(a, st);
  return s;
}
