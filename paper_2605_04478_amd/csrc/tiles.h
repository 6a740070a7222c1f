// Products of matrices in 16-bit types on the matrix cores: one output tile by one workgroup.
//
//   C[m, n] = sum over c of A(m, c) B(n, c)
//
// Either operand lies in memory with the contraction c along its rows ("along", A[m * ld + c]) or across them ("across",
// A[c * ld + m]).  The forward product of a linear layer has both along, its input's gradient has the weights across, its
// weights' gradient has both across; no operand is transposed in memory for any of them.
//
// A tile of DEPTH values of c is brought to LDS by loads that bypass the registers (16 bytes per lane, a wavefront's 1,024
// bytes side by side), STAGES - 1 tiles ahead of the one that is multiplied.  Fragments of operands that lie along c are read
// 16 bytes at a time; those that lie across by the transposing read, which gives a lane four values of c of its own
// column.  LDS positions are permuted so that neither meets a bank twice: the loads fetch, for a fixed position, the
// piece that belongs there.
//
// The matrix instruction is given B as its first operand, so that a lane ends up with four neighbouring n of one m:
// value r of block (i, j) in lane l is C[16 i + l % 16, 16 j + 4 (l / 16) + r].
//
// Lanes whose piece lies outside the operand load from an offset beyond the buffer's range, which the hardware answers with
// zeros: ragged edges need no branch, and a product's sums are those of the valid part.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_utils.h"

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

constexpr int DEPTH = 64;                      // values of c in a stage
constexpr u32 OUTSIDE = 0x80000000u;           // an offset beyond every buffer's range
constexpr u32 BUFFER_RANGE = 0x7FFFFFF0u;

// 16 bytes of every lane, from `offset` bytes behind base, to LDS from p on, the lanes' side by side.  (The host's pass over this file
// knows no loads of 16 bytes to LDS, which only gfx950 has.)
__device__ __forceinline__ void load_to_lds(const void* base, unsigned char* p, u32 offset) {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, BUFFER_RANGE, 0x00027000),
                                           (__attribute__((address_space(3))) void*)p, 16, offset, 0, 0, 0);
#endif
}

// A workgroup's tile of BM x BN, divided among WM x WN wavefronts.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct Tiling {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int THREADS = WM * WN * CCLD_WAVE;
  static constexpr int TM = BM / WM, TN = BN / WN;       // a wavefront's share
  static constexpr int MI = TM / 16, NI = TN / 16;
  static constexpr int STAGE_BYTES = (BM + BN) * DEPTH * 2;
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
  static_assert(TM % 16 == 0 && TN % 16 == 0, "blocks of 16 x 16");
};

// Which 32-byte piece of an operand that lies across c is kept at a position of row c in LDS: the wavefront's transposing
// reads touch rows c .. c + 3 and c + 8 .. c + 11 at once, 32 bytes of each.
template <int ROWS>
__device__ __forceinline__ u32 across_key(u32 c) {
  if constexpr (ROWS >= 128) return (c & 3) | (((c >> 3) & 1) << 2);
  else if constexpr (ROWS == 64) return ((c >> 1) & 1) | (((c >> 3) & 1) << 1);
  else return (c >> 3) & 1;
}

// One operand's share of the stages: ROWS of its output index by DEPTH of c.
// DIRECT loads need 16-byte pieces to be aligned and wholly inside or outside the operand; otherwise single values are loaded
// with a check each and written to LDS from registers.
template <class T, int ROWS, int THREADS, bool ACROSS, bool DIRECT>
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
    else col = 8 * (at ^ (row & 7));
    // the permutation is the same for all of a thread's pieces: their rows differ by multiples of 16 or 8
    static_assert(ACROSS ? ROW_STEP % 16 == 0 || PIECES == 1 : ROW_STEP % 8 == 0, "one permutation per thread");
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const u32 r = row + i * ROW_STEP;
      const bool in = ACROSS ? (int)col < left : (int)r < left;
      offset[i] = in ? (u32)((i64)r * ld + col) * 2 : OUTSIDE;
    }
  }

  // Brings the stage that starts at base to LDS and moves on; `depth` values of c are left.  tile: the operand's place in the
  // stage.
  __device__ __forceinline__ void fetch(unsigned char* tile, int depth) {
    if constexpr (DIRECT) {
      const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / CCLD_WAVE);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        u32 o = offset[i];
        if (depth < DEPTH) {
          const int c = ACROSS ? (int)(row + i * ROW_STEP) : (int)col;
          o = c < depth ? o : OUTSIDE;
        }
        load_to_lds(base, tile + (i * THREADS + wave * CCLD_WAVE) * 16, o);
      }
    } else {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const u32 r = row + i * ROW_STEP;
        s16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int x = (int)col + e;
          const bool in = ACROSS ? x < left && (int)r < depth : (int)r < left && x < depth;
          v[e] = in ? __builtin_bit_cast(short, base[(i64)r * ld + x]) : (short)0;
        }
        *reinterpret_cast<s16x8*>(tile + (i * THREADS + threadIdx.x) * 16) = v;
      }
    }
    base += ACROSS ? ld * DEPTH : (i64)DEPTH;
  }
};

// A wavefront's fragments of an operand: COUNT blocks of 16 from row0 on.
template <int ROWS, int COUNT, bool ACROSS>
struct Fragments {
  u32 at[ACROSS ? COUNT : 2];

  __device__ __forceinline__ void start(u32 row0) {
    const u32 lane = threadIdx.x % CCLD_WAVE, g = lane / 16, t = lane % 16;
    if constexpr (ACROSS) {
      const u32 c = 8 * g + t / 4;
#pragma unroll
      for (int j = 0; j < COUNT; ++j)
        at[j] = c * (ROWS * 2) + (((row0 / 16 + j) ^ across_key<ROWS>(c)) * 32) + (t % 4) * 8;
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) at[k] = (row0 + t) * (DEPTH * 2) + (((4 * k + g) ^ (t & 7)) * 16);
    }
  }
  // block j, half k of the stage: eight values of c from 32 k + 8 (lane / 16) on, of row row0 + 16 j + lane % 16
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

// waits until all but the newest `newer` of this wavefront's loads are in LDS and its LDS reads are done, then for the others
template <int NEWER>
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(NEWER) : "memory");
}

template <class C, class T, bool A_ACROSS, bool B_ACROSS, bool DIRECT>
struct TileProduct {
  f32x4 acc[C::MI][C::NI];

  __device__ __forceinline__ static u32 wave_m() { return (threadIdx.x / CCLD_WAVE) / C::WN * C::TM; }
  __device__ __forceinline__ static u32 wave_n() { return (threadIdx.x / CCLD_WAVE) % C::WN * C::TN; }

  // a, b: the tile's first values; rows_a, rows_b: outputs that the operands have from there on (more than zero); depth: values
  // of c (zero leaves the sums zero).  All of the workgroup's threads take part; lds has C::LDS_BYTES.
  __device__ __forceinline__ void run(unsigned char* lds, const T* a, i64 lda, int rows_a, const T* b, i64 ldb, int rows_b,
                                      int depth) {
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    Operand<T, C::BM, C::THREADS, A_ACROSS, DIRECT> oa;
    Operand<T, C::BN, C::THREADS, B_ACROSS, DIRECT> ob;
    oa.start(a, lda, rows_a);
    ob.start(b, ldb, rows_b);
    Fragments<C::BM, C::MI, A_ACROSS> fa;
    Fragments<C::BN, C::NI, B_ACROSS> fb;
    fa.start(wave_m());
    fb.start(wave_n());
    constexpr int A_BYTES = C::BM * DEPTH * 2;
    constexpr int LOADS = DIRECT ? decltype(oa)::PIECES + decltype(ob)::PIECES : 0;
    const int steps = (depth + DEPTH - 1) / DEPTH;
    auto fetch = [&](int step) {
      unsigned char* s = lds + step % C::STAGES * C::STAGE_BYTES;
      oa.fetch(s, depth - step * DEPTH);
      ob.fetch(s + A_BYTES, depth - step * DEPTH);
    };
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s)
      if (s < steps) fetch(s);
    for (int step = 0; step < steps; ++step) {
      // the oldest stage has arrived, and everybody is done with the one before it, whose place the next fetch takes
      if (step + C::STAGES - 2 < steps) stage_barrier<LOADS * (C::STAGES - 2)>();
      else stage_barrier<0>();
      if (step + C::STAGES - 1 < steps) fetch(step + C::STAGES - 1);
      const unsigned char* s = lds + step % C::STAGES * C::STAGE_BYTES;
#pragma unroll
      for (int k = 0; k < DEPTH / 32; ++k) {
        s16x8 va[C::MI], vb[C::NI];
#pragma unroll
        for (int j = 0; j < C::NI; ++j) vb[j] = fb.read(s + A_BYTES, j, k);
#pragma unroll
        for (int i = 0; i < C::MI; ++i) va[i] = fa.read(s, i, k);
#pragma unroll
        for (int i = 0; i < C::MI; ++i)
#pragma unroll
          for (int j = 0; j < C::NI; ++j) acc[i][j] = mma(vb[j], va[i], acc[i][j], T());
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
