// Products of matrices in 16-bit types on the matrix cores: one output tile by one workgroup.
//
//   C[m, n] = sum over c of A(m, c) B(n, c)
//
// Either operand lies in memory with the contraction c along its rows ("along", A[m * ld + c]) or across them ("across",
// A[c * ld + m]).  The forward product of a linear layer has both along, its input's gradient has the weights across, its
// weights' gradient has both across; no operand is transposed in memory for any of them.
//
// A stage of DEPTH values of c is brought to LDS by loads that bypass the registers (16 bytes per lane, a wavefront's 1,024
// bytes side by side).  The fragments of the stage that is multiplied are in registers, and are replaced by the next stage's as they
// are used up.  Fragments of operands that lie along c are read 16 bytes at a time; those that lie across by the
// transposing read, which gives a lane four values of c of its own column.  LDS positions are permuted so that neither meets a
// bank twice: the loads fetch, for a fixed position, the piece that belongs there.
//
// Rows of a stage of 32 values are half a cache line of an operand that lies along c.  Stages are therefore loaded in pairs, both
// of A's in one step and both of B's in the next: the second half of a line is asked for right after the first, and does not
// travel from the L2 again.
//
// The matrix instruction is given B as its first operand, so that a lane ends up with four neighbouring n of one m:
// value r of block (i, j) in lane l is C[16 i + l % 16, 16 j + 4 (l / 16) + r].
//
// Lanes whose piece lies outside the operand load from an offset beyond the buffer's range, which the hardware answers with
// zeros: ragged edges need no branch, and a product's sums are those of the valid part.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "device_utils.h"
#include "products.h"

namespace ccld {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

// sums in 32 bits; products of 16-bit values are exact in them
__device__ __forceinline__ f32x4 mma(s16x8 a, s16x8 b, f32x4 c, __bf16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(s16x8 a, s16x8 b, f32x4 c, _Float16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

constexpr u32 OUTSIDE = 0x80000000u;           // an offset beyond every buffer's range
constexpr u32 BUFFER_RANGE = 0x7FFFFFF0u;

// 16 bytes of every lane, from `offset` bytes behind base, to LDS from p on, the lanes' side by side.  In assembly, because the compiler
// waits for all loads to LDS that it knows of before every transposing read; who reads waits in stage_barrier.  No register is
// written.  (M0 holds the place; what uses it may follow its write after one instruction.)
__device__ __forceinline__ void load_to_lds(const void* base, unsigned char* p, u32 offset) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef __attribute__((ext_vector_type(4))) u32 u32x4;
  const u64 at = (u64)(uintptr_t)base;
  const u32x4 buffer = {(u32)at, (u32)(at >> 32) & 0xFFFF, BUFFER_RANGE, 0x00027000};
  const u32 place = (u32)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)p;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(place), "v"(offset), "s"(buffer) : "memory");
#endif
}

// A workgroup's tile of BM x BN, divided among WM x WN wavefronts, and its stages.
template <int BM_, int BN_, int WM_, int WN_, int DEPTH_, int STAGES_>
struct Tiling {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, DEPTH = DEPTH_, STAGES = STAGES_;
  static constexpr int THREADS = WM * WN * CCLD_WAVE;
  static constexpr int TM = BM / WM, TN = BN / WN;       // a wavefront's share
  static constexpr int MI = TM / 16, NI = TN / 16;
  static constexpr int STAGE_BYTES = (BM + BN) * DEPTH * 2;
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
  static constexpr int WAVES = THREADS / CCLD_WAVE * (163840 / LDS_BYTES) / 4;       // to a SIMD, as many workgroups as the LDS holds
  static_assert(TM % 16 == 0 && TN % 16 == 0, "blocks of 16 x 16");
};

// Large: the matrix cores' time for a step equals the LDS's (128 KB moved for 256 x 256 x 32), 4 stages ahead, one workgroup to a compute unit: 8192^3 in
//   bfloat16 at 1,260 to 1,400 TFLOP/s (a library's 1,380).
// Medium: two workgroups to a compute unit, one computes while the other starts or ends; the LDS bounds it: 1,084 TFLOP/s.
// Short: three small workgroups, for gradients of weights from few rows, which writing the results bounds (products.h).
// Few: up to 32 rows against a stream of weights, 16 KB of them to a step, which reading the weights bounds (5.5 TB/s at 16 experts of 4,096 x 2,048).
// Narrow: the same for so few columns that tiles of 128 would leave compute units without work; seven steps of 4 KB ahead.
using Large = Tiling<256, 256, 2, 4, 32, 5>;
using Medium = Tiling<128, 128, 2, 4, 32, 5>;
using Short = Tiling<128, 128, 2, 2, 32, 3>;
using Few = Tiling<32, 128, 1, 4, 64, 4>;
using Narrow = Tiling<32, 32, 2, 1, 64, 8>;

// Which 32-byte piece of an operand that lies across c is kept at a position of row c in LDS: the wavefront's transposing
// reads touch rows c .. c + 3 and c + 8 .. c + 11 at once, 32 bytes of each.
template <int ROWS>
__device__ __forceinline__ u32 across_key(u32 c) {
  if constexpr (ROWS >= 128) return (c & 3) | (((c >> 3) & 1) << 2);
  else if constexpr (ROWS == 64) return ((c >> 1) & 1) | (((c >> 3) & 1) << 1);
  else return (c >> 3) & 1;
}

// The same for operands that lie along c: reads touch eight rows at once, 16 bytes of each.
template <int DEPTH>
__device__ __forceinline__ u32 along_key(u32 row) { return DEPTH == 64 ? row & 7 : (row >> 1) & 3; }

__device__ const unsigned char ZEROS[16] __attribute__((aligned(16))) = {};

// One operand's share of the stages: ROWS of its output index by DEPTH of c.
// DIRECT loads need 16-byte pieces to be aligned and wholly inside or outside the operand; otherwise they pass through registers (load()).
template <class T, int ROWS, int DEPTH, int THREADS, bool ACROSS, bool DIRECT>
struct Operand {
  static constexpr int PIECES = ROWS * DEPTH / 8 / THREADS;      // 16-byte pieces per thread and stage
  static_assert(ROWS * DEPTH / 8 % THREADS == 0, "whole pieces");
  static constexpr int PER_ROW = ACROSS ? ROWS / 8 : DEPTH / 8;  // pieces in a row of the LDS tile
  static constexpr int ROW_STEP = THREADS / PER_ROW;             // rows between a thread's pieces

  const T* base;          // first value of the current stage
  i64 ld;                 // values between rows in memory
  u32 row, col;           // of the thread's first piece: row of the LDS tile, first value within it
  int left;               // rows (along) or columns (across) that the operand has from base on
  u32 offset[PIECES];     // in bytes from base, or OUTSIDE

  __device__ __forceinline__ void start(const T* p, i64 ld_, int left_) {
    base = p; ld = ld_; left = left_;
    const u32 tid = threadIdx.x;
    row = tid / PER_ROW;
    const u32 at = tid % PER_ROW;
    if constexpr (ACROSS) col = 8 * ((((at >> 1) ^ across_key<ROWS>(row)) << 1) | (at & 1));
    else col = 8 * (at ^ along_key<DEPTH>(row));
    static_assert(ACROSS ? ROW_STEP % 16 == 0 || PIECES == 1 || (ROW_STEP == 8 && ROWS >= 128) : ROW_STEP % 8 == 0, "column()");
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const u32 r = row + i * ROW_STEP, x = column(i);
      const bool in = ACROSS ? (int)x < left : (int)r < left;
      offset[i] = in ? (u32)((i64)r * ld + x) * 2 : OUTSIDE;
    }
  }
  // first value of piece i within its row: a thread's rows are permuted alike, but for those that differ by an odd multiple of 8
  __device__ __forceinline__ u32 column(int i) const { return ACROSS && ROW_STEP == 8 ? col ^ ((i & 1) * 64) : col; }

  // Loads one of the thread's pieces of the stage that starts at base to the operand's place in it; `depth` values of c are left.
  __device__ __forceinline__ void fetch(unsigned char* tile, int i, int depth) const {
    if constexpr (DIRECT) {
      const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / CCLD_WAVE);
      const int c = ACROSS ? (int)(row + i * ROW_STEP) : (int)col;
      load_to_lds(base, tile + (i * THREADS + wave * CCLD_WAVE) * 16, c < depth ? offset[i] : OUTSIDE);
    } else put(tile, i, load(i, depth));
  }
  // The same through registers.  Every lane loads 16 bytes, from ZEROS where its piece is outside, so that the compiler can count the loads that are on
  // their way.  A piece that reaches over the edge is loaded so that it ends there, and shifted; one at the start of a row's stage or tile,
  // before which nothing may lie, value by value.
  __device__ __forceinline__ s16x8 load(int i, int depth) const {
    const u32 r = row + i * ROW_STEP;
    const int x = (int)column(i), inside = ACROSS ? ((int)r < depth ? left - x : 0) : ((int)r < left ? depth - x : 0);
    const bool over = inside > 0 && inside < 8;
    const int back = over && x > 0 ? 8 - inside : 0;
    const unsigned char* p = reinterpret_cast<const unsigned char*>(base) + offset[i];
    s16x8 v;
    __builtin_memcpy(&v, inside >= 8 || back ? p - 2 * back : ZEROS, 16);              // loads need no alignment
    if (ballot64(over)) {
      u64 part[2];
      __builtin_memcpy(part, &v, 16);
      const int bits = 16 * back;
      if (bits >= 64) {
        part[0] = part[1] >> (bits - 64);
        part[1] = 0;
      } else if (bits) {
        part[0] = part[0] >> bits | part[1] << (64 - bits);
        part[1] >>= bits;
      }
      __builtin_memcpy(&v, part, 16);
      if (over && !back) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (e < inside) v[e] = reinterpret_cast<const short*>(p)[e];
      }
    }
    return v;
  }
  __device__ __forceinline__ static void put(unsigned char* tile, int i, s16x8 v) {
    *reinterpret_cast<s16x8*>(tile + (i * THREADS + threadIdx.x) * 16) = v;
  }
  __device__ __forceinline__ void next_stage() { base += ACROSS ? ld * DEPTH : (i64)DEPTH; }
};

// Where a wavefront finds its fragments of an operand: COUNT blocks of 16 from row0 on.
template <int ROWS, int COUNT, int DEPTH, bool ACROSS>
struct Fragments {
  u32 at[ACROSS ? COUNT : DEPTH / 32];

  __device__ __forceinline__ void start(u32 row0) {
    const u32 lane = threadIdx.x % CCLD_WAVE, g = lane / 16, t = lane % 16;
    if constexpr (ACROSS) {
      const u32 c = 8 * g + t / 4;
#pragma unroll
      for (int j = 0; j < COUNT; ++j)
        at[j] = c * (ROWS * 2) + (((row0 / 16 + j) ^ across_key<ROWS>(c)) * 32) + (t % 4) * 8;
    } else {
#pragma unroll
      for (int k = 0; k < DEPTH / 32; ++k) at[k] = (row0 + t) * (DEPTH * 2) + (((4 * k + g) ^ along_key<DEPTH>(t)) * 16);
    }
  }
  // block j, part k of the stage: eight values of c from 32 k + 8 (lane / 16) on, of row row0 + 16 j + lane % 16
  __device__ __forceinline__ s16x8 read(const unsigned char* tile, int j, int k) const {
    if constexpr (ACROSS) {
      typedef __attribute__((address_space(3))) s16x4* lds_ptr;
      const unsigned char* p = tile + at[j] + k * 32 * ROWS * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * ROWS * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return *reinterpret_cast<const s16x8*>(tile + at[k] + j * 16 * DEPTH * 2);
    }
  }
};

// waits until all but the newest NEWER of this wavefront's loads are in LDS and its LDS accesses are done, then for the others
template <int NEWER>
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(NEWER) : "memory");
}

// Whether results leave as a stream, which the L2 does not keep: rows that are made of whole lines (1 % of 8192^3, whose operands need the L2).  Where
// workgroups share lines, these leave whole only from the L2 (64 experts' dw of 1,024 x 2,040 from 2 rows each: 156 us as a stream, 71 so), which
// matters less than the operands in long contractions (8 experts of 4,000 x 4,000 and 2,000 rows each: 500 and 510 us).
__device__ __forceinline__ bool streams(i64 ldo, int depth) { return ldo % 64 == 0 || depth > 1024; }

template <class C, class T, bool A_ACROSS, bool B_ACROSS, bool DIRECT>
struct TileProduct {
  f32x4 acc[C::MI][C::NI];

  __device__ __forceinline__ static u32 wave_m() { return (threadIdx.x / CCLD_WAVE) / C::WN * C::TM; }
  __device__ __forceinline__ static u32 wave_n() { return (threadIdx.x / CCLD_WAVE) % C::WN * C::TN; }

  static constexpr int PARTS = C::DEPTH / 32, A_BYTES = C::BM * C::DEPTH * 2;
  typedef Operand<T, C::BM, C::DEPTH, C::THREADS, A_ACROSS, DIRECT> A;
  typedef Operand<T, C::BN, C::DEPTH, C::THREADS, B_ACROSS, DIRECT> B;
  static constexpr int LOADS = A::PIECES + B::PIECES;
  // a, b: the tile's first values; rows_a, rows_b: outputs that the operands have from there on (more than zero); depth: values
  // of c (zero leaves the sums zero).  All of the workgroup's threads take part; lds has C::LDS_BYTES, which are free afterwards.
  __device__ __forceinline__ void run(unsigned char* lds, const T* a, i64 lda, int rows_a, const T* b, i64 ldb, int rows_b,
                                      int depth) {
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    if (depth <= 0) return;
    A oa;
    B ob;
    oa.start(a, lda, rows_a);
    ob.start(b, ldb, rows_b);
    Fragments<C::BM, C::MI, C::DEPTH, A_ACROSS> fa;
    Fragments<C::BN, C::NI, C::DEPTH, B_ACROSS> fb;
    fa.start(wave_m());
    fb.start(wave_n());
    constexpr bool PAIRS = C::DEPTH == 32 && C::STAGES >= 5;            // (fewer stages have no two free places)
    constexpr int STAGES_AHEAD = PAIRS ? C::STAGES - 1 : C::STAGES;      // a pair needs two free places
    constexpr int A_TURN = PAIRS ? 2 * A::PIECES : A::PIECES, B_TURN = PAIRS ? 2 * B::PIECES : B::PIECES;
    auto after = [](u32 p) { return p + C::STAGE_BYTES == C::LDS_BYTES ? 0 : p + C::STAGE_BYTES; };
    int left_a = depth, left_b = depth;        // of the stages that are not on their way yet
#pragma unroll
    for (int s = 0; s < STAGES_AHEAD; ++s) {
#pragma unroll
      for (int i = 0; i < A::PIECES; ++i) oa.fetch(lds + s * C::STAGE_BYTES, i, left_a);
#pragma unroll
      for (int i = 0; i < B::PIECES; ++i) ob.fetch(lds + s * C::STAGE_BYTES + A_BYTES, i, left_b);
      oa.next_stage();
      ob.next_stage();
      left_a -= C::DEPTH;
      left_b -= C::DEPTH;
    }
    stage_barrier<DIRECT ? LOADS * (STAGES_AHEAD - 1) : 0>();
    s16x8 va[PARTS][C::MI], even[PARTS][C::NI], odd[PARTS][C::NI];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
#pragma unroll
      for (int j = 0; j < C::NI; ++j) even[k][j] = fb.read(lds + A_BYTES, j, k);
#pragma unroll
      for (int i = 0; i < C::MI; ++i) va[k][i] = fa.read(lds, i, k);
    }
    // A step multiplies the stage that is in registers and reads the next one.  Its first turns need nothing from LDS; then the
    // wavefronts wait for one another: the next stage has arrived everywhere, and the place of the stage in registers is free.
    // Stages beyond the last are zeros.
    u32 next = C::STAGE_BYTES, free = PAIRS ? (C::STAGES - 1) * C::STAGE_BYTES : 0;
    // (through registers: what a step loads is written to LDS when the next one ends, so that it has the time of two)
    constexpr int EVEN_LOADS = DIRECT ? 1 : PAIRS ? A_TURN : LOADS, ODD_LOADS = DIRECT ? 1 : PAIRS ? B_TURN : LOADS;
    s16x8 held_even[EVEN_LOADS], held_odd[ODD_LOADS];
    u32 held_free = 0, held_second = 0;
    bool held = false;
    constexpr int TURNS = PARTS * C::MI, HOLD = TURNS / 4 < 1 ? 1 : TURNS / 4;
    // Tiles of few rows have registers to spare: their sums are held in four, a part of a step each, which are off by a quarter as much.
    constexpr int CHAINS = C::BM == 32 ? 2 * PARTS : 1;
    f32x4 chain[CHAINS][C::MI][C::NI] = {};
    auto step = [&](const s16x8 (&vb)[PARTS][C::NI], s16x8 (&then)[PARTS][C::NI], auto is_odd) {
      constexpr bool ODD = decltype(is_odd)::value;
      auto multiply = [&](int turn) {
#pragma unroll
        for (int j = 0; j < C::NI; ++j) {
          f32x4& sum = CHAINS == 1 ? acc[turn % C::MI][j] : chain[ODD * PARTS + turn / C::MI][turn % C::MI][j];
          sum = mma(vb[turn / C::MI][j], va[turn / C::MI][turn % C::MI], sum, T());
        }
      };
#pragma unroll
      for (int turn = 0; turn < HOLD; ++turn) multiply(turn);
      __builtin_amdgcn_sched_barrier(0);
      stage_barrier<!DIRECT ? 63 : !PAIRS ? LOADS * (C::STAGES - 2) : ODD ? A_TURN : A_TURN + B_TURN>();
      const unsigned char* s = lds + next;
      // loads of this step: a stage, or both stages of a pair for one operand
      constexpr int FIRST = !PAIRS || !ODD ? A_TURN : 0, ALL = FIRST + (!PAIRS || ODD ? B_TURN : 0);
      const u32 second = after(free);
      auto load = [&](int i) {
        if (i < FIRST) {
          if (i == A::PIECES) oa.next_stage();
          const int n = i % A::PIECES, left = i < A::PIECES ? left_a : left_a - C::DEPTH;
          if constexpr (DIRECT) oa.fetch(lds + (i < A::PIECES ? free : second), n, left);
          else (ODD ? held_odd : held_even)[i] = oa.load(n, left);
        } else {
          const int k = i - FIRST;
          if (k == B::PIECES) ob.next_stage();
          const int n = k % B::PIECES, left = k < B::PIECES ? left_b : left_b - C::DEPTH;
          if constexpr (DIRECT) ob.fetch(lds + (k < B::PIECES ? free : second) + A_BYTES, n, left);
          else (ODD ? held_odd : held_even)[i] = ob.load(n, left);
        }
      };
      if constexpr (!DIRECT) {
#pragma unroll
        for (int i = 0; i < ALL; ++i) load(i);
      }
      int loaded = 0, read_b = 0;
#pragma unroll
      for (int turn = HOLD; turn < TURNS; ++turn) {
        const int share = turn + 1 - HOLD, of = TURNS - HOLD;
#pragma unroll
        for (; read_b < PARTS * C::NI * share / of; ++read_b) then[read_b / C::NI][read_b % C::NI] = fb.read(s + A_BYTES, read_b % C::NI, read_b / C::NI);
        if (turn - HOLD < HOLD) va[(turn - HOLD) / C::MI][(turn - HOLD) % C::MI] = fa.read(s, (turn - HOLD) % C::MI, (turn - HOLD) / C::MI);
        if constexpr (DIRECT) {
#pragma unroll
          for (; loaded < ALL * share / of; ++loaded) load(loaded);
        }
        multiply(turn);
        va[turn / C::MI][turn % C::MI] = fa.read(s, turn % C::MI, turn / C::MI);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (!DIRECT) {
        if (held) {
          constexpr int A_HELD = !PAIRS || ODD ? A_TURN : 0, OTHERS = ODD ? EVEN_LOADS : ODD_LOADS;      // the other step's loads
#pragma unroll
          for (int i = 0; i < OTHERS; ++i) {
            const int k = i < A_HELD ? i : i - A_HELD, pieces = i < A_HELD ? A::PIECES : B::PIECES;
            unsigned char* stage = lds + (k < pieces ? held_free : held_second);
            const s16x8 v = (ODD ? held_even : held_odd)[i];
            if (i < A_HELD) A::put(stage, k % pieces, v);
            else B::put(stage + A_BYTES, k % pieces, v);
          }
        }
        held = true;
        held_free = free;
        held_second = second;
      }
      constexpr int MOVED = PAIRS ? 2 * C::DEPTH : C::DEPTH;
      if (!PAIRS || !ODD) { oa.next_stage(); left_a -= MOVED; }
      if (!PAIRS || ODD) { ob.next_stage(); left_b -= MOVED; free = PAIRS ? after(second) : second; }
      next = after(next);
    };
    for (int done = 0; done < depth; done += 2 * C::DEPTH) {
      step(even, odd, std::false_type());
      step(odd, even, std::true_type());
    }
    if constexpr (CHAINS > 1) {
      static_assert(CHAINS == 4, "pairs of pairs");
#pragma unroll
      for (int i = 0; i < C::MI; ++i)
#pragma unroll
        for (int j = 0; j < C::NI; ++j) acc[i][j] = (chain[0][i][j] + chain[1][i][j]) + (chain[2][i][j] + chain[3][i][j]);
    }
    stage_barrier<0>();
  }

  // Writes the tile, scaled, to out: rows x cols of it exist.  Sums are rounded once, to nearest even.  A wavefront turns its share
  // round in LDS, so that rows leave in whole cache lines (as the sums lie, a store would touch 16 rows, 32 bytes each); whole:
  // rows are aligned to 16 bytes; stream: they are not kept in the L2 (see streams()).  Follows run().
  __device__ __forceinline__ void store(unsigned char* lds, T* out, i64 ldo, int rows, int cols, bool whole, bool stream, float scale) const {
    typedef __attribute__((ext_vector_type(4))) T t4;
    const u32 lane = threadIdx.x % CCLD_WAVE;
    unsigned char* own = lds + threadIdx.x / CCLD_WAVE * (C::TM * C::TN * 2);
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NI; ++j) {
        const u32 m = 16 * i + lane % 16, n = 16 * j + 4 * (lane / 16);
        const f32x4 v = acc[i][j] * scale;
        *reinterpret_cast<t4*>(own + m * (C::TN * 2) + (((n / 8) ^ along_key<C::TN>(m)) * 16) + n % 8 * 2) = t4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
      }
    __builtin_amdgcn_wave_barrier();
    if (whole && stream) store_rows<true>(own, out, ldo, rows, cols, true);
    else store_rows<false>(own, out, ldo, rows, cols, whole);
  }
  template <bool STREAM>
  __device__ __forceinline__ static void store_rows(const unsigned char* own, T* out, i64 ldo, int rows, int cols, bool whole) {
    constexpr int PIECES = C::TN / 8;
    const int lane = (int)(threadIdx.x % CCLD_WAVE), m0 = (int)wave_m(), n0 = (int)wave_n();
#pragma unroll
    for (int i = 0; i < C::TM * PIECES / CCLD_WAVE; ++i) {
      const int m = i * (CCLD_WAVE / PIECES) + lane / PIECES, p = lane % PIECES, n = n0 + 8 * p;
      const s16x8 v = *reinterpret_cast<const s16x8*>(own + m * (C::TN * 2) + ((p ^ along_key<C::TN>(m)) * 16));
      if (m0 + m < rows) {
        T* q = out + (i64)(m0 + m) * ldo + n;
        if (whole && n + 8 <= cols) {
          if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<s16x8*>(q));
          else *reinterpret_cast<s16x8*>(q) = v;
        } else if (n + 8 <= cols) __builtin_memcpy(q, &v, 16);
        else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const short x = v[e];              // (a bit cast of a vector's element itself takes the vector's first one)
            if (n + e < cols) q[e] = __builtin_bit_cast(T, x);
          }
        }
      }
    }
  }

  // f(m, n, four sums of n .. n + 3) for every block, m and n within the tile
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    const u32 lane = threadIdx.x % CCLD_WAVE;
    const u32 m = wave_m() + lane % 16, n = wave_n() + 4 * (lane / 16);
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NI; ++j) f(m + 16 * i, n + 16 * j, acc[i][j]);
  }
};

// Writes four neighbouring values, `left` of which exist; WIDE: rows are aligned to 8 bytes.
// Sums are rounded once, to nearest even, when they leave.
template <class T>
__device__ __forceinline__ void store4(T* p, f32x4 v, int left, bool wide) {
  typedef __attribute__((ext_vector_type(4))) T t4;
  if (wide && left >= 4) {
    *reinterpret_cast<t4*>(p) = t4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < left) p[r] = (T)v[r];
  }
}

// In how many parts the contraction of `tiles` tiles is computed: the least time in nanoseconds, by choose_cut's figures for a step (0.25 us in tiles of 32
// rows) and 10 us for every tile's start and end, with no more than MOST_PIECES pieces.  steps: of 32 along the contraction.  A lane of the
// wavefront weighs each number.
template <class C>
__device__ __forceinline__ u32 splits_of(u32 tiles, u32 steps) {
  static_assert(MOST_SPLITS == CCLD_WAVE, "one to a lane");
  constexpr u32 AT_ONCE = (C::BM == 256 ? 1 : 2) * (u32)COMPUTE_UNITS, STEP_NS = C::BM == 256 ? 770 : C::BM == 128 ? 500 : 250;
  const u32 s = lane_id() + 1;
  const bool may = s == 1 || (tiles * s <= MOST_PIECES && steps >= 16 * s);
  const u32 rounds = (tiles * s + AT_ONCE - 1) / AT_ONCE, depth = (steps + s - 1) / s;
  u64 best = may ? ((u64)rounds * (10000 + (u64)depth * STEP_NS) + (u64)tiles * s * (C::BM * C::BN) / 560) * CCLD_WAVE + lane_id() : ~(u64)0;
#pragma unroll
  for (int x = 1; x < CCLD_WAVE; x *= 2) {
    const u64 other = __shfl_xor(best, x, CCLD_WAVE);
    best = other < best ? other : best;
  }
  return (u32)__builtin_amdgcn_readfirstlane((int)(best % CCLD_WAVE)) + 1;
}

// Workgroups are handed to the eight XCDs in turn, each with an L2 of its own: this gives each XCD a contiguous share of n
// pieces of work.
__device__ __forceinline__ u32 xcd_order(u32 id, u32 n) {
  const u32 xcd = id % 8, at = id / 8, each = n / 8, more = n % 8;
  return xcd * each + (xcd < more ? xcd : more) + at;
}

// The place of piece `at` of tm x tn tiles: columns of up to GROUP m-tiles, so that the workgroups that run together in an
// XCD share rows and columns.
__device__ __forceinline__ uint2 grouped_order(u32 at, u32 tm, u32 tn, u32 group) {
  const u32 g = at / (group * tn), first = g * group, size = tm - first < group ? tm - first : group, in = at - g * group * tn;
  return make_uint2(first + in % size, in / size);
}

}  // namespace ccld
