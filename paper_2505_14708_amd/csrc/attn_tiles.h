// Tiles, operands and products that the dense attention kernels (k_dense_fwd.hip, k_dense_bwd.hip) share.
//
// A wave works on 32 columns at a time: 32 rows of one operand (queries, or keys in the kernel for the gradients of K and V), one to a
// lane l % 32, that stay in registers, while tiles of rows of the others come through LDS.  Two products make up every kernel:
//
//   scores   C = X Y^T     X: 32 rows of an LDS tile, Y: the wave's 32 rows; contraction over the channels
//   mix      Z += X^T C    X: the same kind of tile, read transposed; contraction over its 32 rows
//
// Lane l of the 64 holds in C's 16 registers the rows 16(a / 8) + 8(l / 32) + a % 8 of column l % 32 (a = 0..15): X's rows are fed in
// the order sigma (bits 2 and 3 of the row number change places), so that 8 registers in a row are 8 rows in a row and C goes into
// the second product without leaving its lane.  A softmax over rows of C is a lane's own registers and one exchange with lane l ^ 32.
// Z's registers are the channels 32 dt + 8(a / 4) + 4(l / 32) + a % 4 of the same column.
//
// bf16: v_mfma_f32_32x32x16_bf16, X read in 16-byte pieces for the scores and by ds_read_b64_tr_b16 (four rows of 16 channels become
// 16 columns of four) for the mix.  float32: v_mfma_f32_32x32x2_f32, a lane's 16-byte piece of X feeds four of them, and the mix reads
// single words, whose transposition is a matter of addresses.
//
// Tiles are row major in LDS, 16-byte pieces of row r stored at piece number p ^ swizzle(r), and arrive by 16-byte direct-to-LDS loads: the
// lane that fills position p of row r fetches piece p ^ swizzle(r).  The swizzles let both kinds of reads touch all banks.
#pragma once
#include <float.h>
#include <math.h>
#include "da_internal.h"
#include "dense_attn.h"

namespace da {
namespace dense {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
typedef __attribute__((address_space(3))) float lds_f32;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <class T> struct Type;
template <> struct Type<__bf16> {
  typedef bf16x8 piece;
  static constexpr int PER = 8;      // elements of a 16-byte piece
};
template <> struct Type<float> {
  typedef f32x4 piece;
  static constexpr int PER = 4;
};

template <class T, int D> constexpr int kRowBytes = D * (int)sizeof(T);

template <class T, int D> __device__ __forceinline__ int swizzle(int row) {
  if constexpr (sizeof(T) == 4) return row & 15;
  else if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  else return ((row & 2) << 1) | ((row >> 2) & 3);
}

__device__ __forceinline__ int sigma(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

__device__ __forceinline__ f32x16 zero16() {
  return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// 16 bytes a lane from global memory to LDS: lane i's land at lds + 16 i.  (m0 holds the LDS address; it is put back.)
__device__ __forceinline__ void dma16(const void* g, unsigned lds) {
  unsigned keep;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
      : "=&s"(keep) : "v"(g), "s"(lds) : "memory");
}
// the same with a uniform base and a 32-bit offset of the lane's own
__device__ __forceinline__ void dma16(const void* base, unsigned off, unsigned lds) {
  unsigned keep;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
      : "=&s"(keep) : "v"(off), "s"(base), "s"(lds) : "memory");
}
// 4 bytes a lane
__device__ __forceinline__ void dma4(const void* g, unsigned lds) {
  unsigned keep;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
      : "=&s"(keep) : "v"(g), "s"(lds) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// the lane number, in a way that the compiler neither moves nor keeps: what follows from it is made anew in each trip of a loop, where
// registers are short
__device__ __forceinline__ int opaque_lane() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

// workgroup barrier behind which LDS written by the loads above may be read (each wave has waited for its own)
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ float max_across_halves(float x) {
  u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_across_halves(float x) {
  u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// ---------------------------------------------------------------------------------- tiles
// ROWS rows of D elements, row j of the tile being row min(first + j, last) of `base` (rows `stride` bytes apart), into LDS at `lds`, by the NW
// waves of the workgroup.  (Rows behind the last one repeat it: every address is one of a row that is there.)
template <class T, int D, int ROWS, int NW>
__device__ __forceinline__ void load_tile(const unsigned char* base, long long stride, int first, int last, unsigned lds, int wave) {
  constexpr int RB = kRowBytes<T, D>, CPR = RB / 16, RPS = 64 / CPR, STEPS = ROWS / RPS;
  static_assert(STEPS % NW == 0, "whole steps per wave");
  const int lane = opaque_lane();
  const int r_in = lane / CPR, p = lane % CPR;
  if (first + ROWS - 1 <= last && stride < (1LL << 24)) {
    const unsigned char* at = base + (long long)first * stride;
#pragma unroll
    for (int k = 0; k < STEPS / NW; ++k) {
      const int it = k * NW + wave, row = it * RPS + r_in;
      dma16(at + (long long)(it * RPS) * stride, (unsigned)(r_in * (int)stride + ((p ^ swizzle<T, D>(row)) << 4)), lds + it * 1024);
    }
  } else {
#pragma unroll
    for (int k = 0; k < STEPS / NW; ++k) {
      const int it = k * NW + wave, row = it * RPS + r_in;
      dma16(base + (long long)min(first + row, last) * stride + ((p ^ swizzle<T, D>(row)) << 4), lds + it * 1024);
    }
  }
}

// ---------------------------------------------------------------------------------- products
// A wave's own 32 rows: piece 2t + l / 32 of row l % 32.
template <class T, int D> struct Own {
  static constexpr int N = kRowBytes<T, D> / 32;
  typename Type<T>::piece x[N];
  __device__ __forceinline__ void load(const unsigned char* row, int hi) {
#pragma unroll
    for (int t = 0; t < N; ++t) x[t] = *(const typename Type<T>::piece*)(row + (2 * t + hi) * 16);
  }
};

// LDS address (less the tile's) of the piece that this lane feeds to step 0 of `scores`; that of step t is at ^ 32 t
template <class T, int D> __device__ __forceinline__ unsigned scores_lane(int lane) {
  const int row = sigma(lane & 31);
  return row * kRowBytes<T, D> + (((lane >> 5) ^ swizzle<T, D>(row)) << 4);
}

// NQ sets of 32 columns against 32 rows of the tile, added to what c holds
template <class T, int D, int NQ>
__device__ __forceinline__ void add_scores(unsigned at, const Own<T, D> (&own)[NQ], f32x16 (&c)[NQ]) {
  // Operands arrive AHEAD steps before their use: more of them in flight do not fit the registers of 64 queries (40 heads of 75600 by 512, forward:
  // three 1020 us, two 950 us).
  constexpr int N = Own<T, D>::N, AHEAD = 2;
  typename Type<T>::piece x[N];
  auto fetch = [&](int t) { x[t] = *(const __attribute__((address_space(3))) typename Type<T>::piece*)(uintptr_t)(at ^ (32 * t)); };
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) fetch(t);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int t = 0; t < N; ++t) {
    if (t + AHEAD < N) fetch(t + AHEAD);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < NQ; ++h) c[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[t], own[h].x[t], c[h], 0, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < NQ; ++h) c[h] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[t][i], own[h].x[t][i], c[h], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// bf16, with the wave's own 32 rows in LDS as well, where registers are short: piece t of lane l at own_at + 1024 t, own_at + 16 l being the lane's
template <int D>
__device__ __forceinline__ void add_scores_lds(unsigned at, unsigned own_at, f32x16& c) {
  constexpr int N = Own<__bf16, D>::N, AHEAD = 2;
  bf16x8 x[N], y[N];
  auto fetch = [&](int t) {
    x[t] = *(lds_bf16x8*)(uintptr_t)(at ^ (32 * t));
    y[t] = *(lds_bf16x8*)(uintptr_t)(own_at + 1024 * t);
  };
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) fetch(t);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int t = 0; t < N; ++t) {
    if (t + AHEAD < N) fetch(t + AHEAD);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[t], y[t], c, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <class T, int D, int NQ>
__device__ __forceinline__ void scores(unsigned at, const Own<T, D> (&own)[NQ], f32x16 (&c)[NQ]) {
#pragma unroll
  for (int h = 0; h < NQ; ++h) c[h] = zero16();
  add_scores<T, D, NQ>(at, own, c);
}

// LDS address (less the tile's) of this lane's part of the transposed operands: bf16: rows 8(l/32) + 0..3 of step 0, channel group 0; channel
// group dt is at ^ 64 dt, step t 16 rows further, rows + 4: row + 4 and pieces ^ 1.  float32: row 8(l/32), channel l % 32.
template <class T, int D> __device__ __forceinline__ unsigned mix_lane(int lane) {
  const int hi = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    const int l = lane & 15, row = 8 * hi + (l >> 2), piece = 2 * ((lane >> 4) & 1) + ((l >> 1) & 1);
    return row * kRowBytes<T, D> + ((piece ^ swizzle<T, D>(row)) << 4) + (l & 1) * 8;
  } else {
    const int m = lane & 31, row = 8 * hi;
    return row * kRowBytes<T, D> + (((m >> 2) ^ swizzle<T, D>(row)) << 4) + (m & 3) * 4;
  }
}

// c as the right operand of `mix`.  bf16: rounded to nearest; a probability or its gradient enters the product with 8 bits, as every bf16
// operand does, and is summed in 32.
template <class T> struct Mixed;
template <> struct Mixed<__bf16> {
  bf16x8 x[2];
  Mixed() = default;
  __device__ __forceinline__ explicit Mixed(const f32x16& c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16x2 p = __builtin_convertvector((f32x2{c[2 * i], c[2 * i + 1]}), bf16x2);
      x[i >> 2][(2 * i) & 7] = p[0];
      x[i >> 2][(2 * i + 1) & 7] = p[1];
    }
  }
};
template <> struct Mixed<float> {
  f32x16 x;
  Mixed() = default;
  __device__ __forceinline__ explicit Mixed(const f32x16& c) : x(c) {}
};

template <class T, int D, int NQ>
__device__ __forceinline__ void mix(unsigned at, const Mixed<T> (&c)[NQ], f32x16 (&z)[NQ][D / 32]) {
  constexpr int RB = kRowBytes<T, D>, G = D / 32;
  if constexpr (sizeof(T) == 2) {
    constexpr int N = 2 * G, AHEAD = 2;
    s16x8 x[N];
    auto fetch = [&](int i) {
      const int t = i / G, dt = i % G;
      const unsigned a0 = (at ^ (64 * dt)) + t * 16 * RB, a1 = (at ^ (64 * dt + 16)) + (t * 16 + 4) * RB;
      const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)a0);
      const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)a1);
      x[i] = __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i + AHEAD < N) fetch(i + AHEAD);
#pragma unroll
      for (int h = 0; h < NQ; ++h)
        z[h][i % G] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[i]), c[h].x[i / G], z[h][i % G], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  } else {
#pragma unroll
    for (int a = 0; a < 16; ++a) {
#pragma unroll
      for (int dt = 0; dt < G; ++dt) {
        const unsigned w = (at ^ (((a & 7) << 4) | (dt << 7))) + (16 * (a >> 3) + (a & 7)) * RB;
        const float x = *(lds_f32*)(uintptr_t)w;
#pragma unroll
        for (int h = 0; h < NQ; ++h) z[h][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, c[h].x[a], z[h][dt], 0, 0, 0);
      }
      if (a % 2) __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// row of C that register a of a lane holds
__device__ __forceinline__ int c_row(int a, int hi) { return 16 * (a >> 3) + 8 * hi + (a & 7); }

// A column of Z (D channels of one row of the result) to its place, in the result's type: 16 bytes a lane where two lanes of a row
// exchange halves first.
template <class T, int D>
__device__ __forceinline__ void store_column(unsigned char* row, int hi, const f32x16 (&z)[D / 32], float f, bool there) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{z[dt][8 * k + 2 * i] * f, z[dt][8 * k + 2 * i + 1] * f}), bf16x2));
        // w[0..1]: channels 16k + 4hi + 0..3, w[2..3]: 16k + 8 + 4hi + 0..3; afterwards the lane has 16k + 8hi + 0..7
        const u32x2 s0 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const u32x2 s1 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        if (there) *(u32x4*)(row + (32 * dt + 16 * k + 8 * hi) * 2) = u32x4{s0[0], s1[0], s0[1], s1[1]};
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (there)
          *(f32x4*)(row + (32 * dt + 8 * k + 4 * hi) * 4) =
              f32x4{z[dt][4 * k] * f, z[dt][4 * k + 1] * f, z[dt][4 * k + 2] * f, z[dt][4 * k + 3] * f};
    }
  }
}

// ---------------------------------------------------------------------------------- relative position bias
// The bias of a head by r = key - query - q_pos, times log2(e), in LDS: r from -(cut + kBiasPad) to cut + kBiasPad, what lies beyond `cut`
// having the outermost buckets' values.  A square of 32 x 32 that touches -cut < r < cut reaches no further than kBiasPad past it.
constexpr int kBiasPad = 64;
constexpr float kMasks = -0x1p100f;
__host__ __device__ inline int bias_entries(int cut) { return 2 * (cut + kBiasPad) + 1; }

template <class T>
__device__ __forceinline__ void fill_bias(float* lds, const RelRule& rule, const T* table, int H, int h, int thread, int threads) {
  const int n = bias_entries(rule.cut);
  for (int i = thread; i < n; i += threads) {
    const float b = (float)table[(long long)rel_bucket(rule, i - rule.cut - kBiasPad) * H + h];
    // A mask of the type's lowest value is minus infinity here: a row that only such entries reach has nothing to attend, and with a score
    // added they could be minus infinity or not.
    lds[i] = b <= kMasks ? -INFINITY : b * kLog2e;
  }
}

// a square's bias: the wave's columns are queries (SIGN +1: r grows with the register's row) or keys (-1)
template <int SIGN>
__device__ __forceinline__ void read_bias(unsigned at, f32x16& b) {
#pragma unroll
  for (int a = 0; a < 16; ++a) b[a] = *(lds_f32*)(uintptr_t)(at + SIGN * 4 * (16 * (a >> 3) + (a & 7)));
}

// Workgroups are dealt to the 8 XCDs in turn.  The `each` pieces of work of a head go to one XCD, whose L2 then holds the rows that they share, and
// the heads to the XCDs in turn, so that batch elements of different lengths are spread over all of them (64 heads of 512 queries, keys of 512, 336, 160 and
// 444: the three kernels of a training step 155 us with an eighth of the list to each XCD, 141 us so).  Heads beyond a multiple of 8: an eighth of their pieces each.
__device__ __forceinline__ long long xcd_order(long long id, long long total, long long each) {
  const long long turns = total / each / 8, most = turns * 8 * each, x = id % 8, n = id / 8;
  if (id < most) return (n / each * 8 + x) * each + n % each;
  const long long rest = total - most, part = rest / 8, more = rest % 8, i = (id - most) / 8;
  return most + x * part + min(x, more) + i;                // (most is a multiple of 8)
}

// Rows of a tile.  Waves that have each 32 or 64 columns of their own share tiles of 16 KB at most, so that two workgroups of two pairs of
// buffers fit a CU.  Where there are too few columns for that, JW waves have the same 32 columns and take the 32 rows of JW in turn
// (their sums are put together at the end, join_waves): tiles of 32 JW rows.
template <class T, int D, int JW> constexpr int kTileRows = JW > 1 ? 32 * JW : kRowBytes<T, D> > 256 ? 32 : 64;
// the most waves that may join: tiles of K and V, twice, in 128 KB
template <class T, int D> constexpr int kJoin = kRowBytes<T, D> > 256 ? 2 : 4;

// Z of JW waves over the same 32 columns, each times its wave's f, added up in the order of the waves; `put(row, channel, x)` gets 8 channels
// of a row at a time.  The tiles' memory is free by then (every wave behind the first barrier).
template <int D, int JW, class Put>
__device__ __forceinline__ void join_waves(float* buf, int wave, int lane, const f32x16 (&z)[D / 32], float f, Put put) {
  constexpr int S = D + 4;         // row stride: 16 lanes' pieces in 64 banks
  tile_barrier();
  float* mine = buf + (wave * 32 + (lane & 31)) * S + 4 * (lane >> 5);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int k = 0; k < 4; ++k) *(f32x4*)(mine + 32 * dt + 8 * k) = f32x4{z[dt][4 * k] * f, z[dt][4 * k + 1] * f, z[dt][4 * k + 2] * f, z[dt][4 * k + 3] * f};
  tile_barrier();
  for (int i = wave * 64 + lane; i < 32 * (D / 8); i += 64 * JW) {
    const int row = i / (D / 8), c = i % (D / 8) * 8;
    f32x4 x[2] = {};
#pragma unroll
    for (int w = 0; w < JW; ++w) {
      x[0] += *(const f32x4*)(buf + (w * 32 + row) * S + c);
      x[1] += *(const f32x4*)(buf + (w * 32 + row) * S + c + 4);
    }
    put(row, c, x);
  }
}

// 8 channels to their place in the result's type
template <class T> __device__ __forceinline__ void store8(unsigned char* at, const f32x4 (&x)[2], float f) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)(x[i >> 2][i & 3] * f);
    *(bf16x8*)at = y;
  } else {
    *(f32x4*)at = x[0] * f;
    *(f32x4*)(at + 16) = x[1] * f;
  }
}

// What a launch is made for: its queries' rows are those of single heads, the same with a bias, or those of several heads (dense_packed).
enum Mode { PLAIN, BIAS, PACKED };
template <int MODE> __device__ __forceinline__ int heads_of(const DenseGeo& q) { return MODE == PACKED ? q.Hk : q.H; }
template <int MODE> __device__ __forceinline__ int kv_head(const DenseGeo& q, int hd) { return MODE == PACKED || q.group == 1 ? hd : hd / q.group; }

// where row rr of head `hd` (of those the kernels see) of batch element b lives
template <int MODE>
__device__ __forceinline__ long long query_offset(const DenseGeo& q, const Rows& r, int b, int hd, int rr) {
  if constexpr (MODE != PACKED) return b * r.sb + hd * r.sh + (long long)rr * r.sn;
  const int g = rr / q.N, n = rr - g * q.N;
  return b * r.sb + (long long)(hd * q.group + g) * r.sh + (long long)n * r.sn;
}

// s c2 + add.  float32: the rounding of c2 alone would be off by |s c2| 2^-25, and is made good.
template <class T> __device__ __forceinline__ float biased(const DenseGeo& q, float s, float add) {
  if constexpr (sizeof(T) == 4) add = __builtin_fmaf(fmaxf(s, q.s_low), q.c2_lo, add);     // (a score of minus infinity stays one)
  return __builtin_fmaf(s, q.c2, add);
}
template <class T> __device__ __forceinline__ float power_of(const DenseGeo& q, float s, float add) { return exp2_fast(biased<T>(q, s, add)); }

// What a row's exponentials are taken against: `top`, one of the row's largest x with a bias, of its scores without.  There, with r = top c2
// rounded, exp2(fma(s, c2, -r)) has the rounding of its result only; the largest score's exponent is what r was rounded by, up to 2^-25 |r|, which all of the
// row have in common, so that it divides out.  But where |r| reaches 2^31 the powers would be infinite, or all of them zero.  So beyond kNear it
// is the differences of scores that are scaled: they are exact for the scores that count.
constexpr float kNear = 0x1p24f;
struct Ref { float score, x; };          // x of a score s against it: (s - score) c2 - x
template <int MODE> __device__ __forceinline__ bool is_distant(const DenseGeo& q, float top) { return MODE != BIAS && fabsf(top * q.c2) > kNear; }
template <int MODE> __device__ __forceinline__ Ref ref_of(const DenseGeo& q, float top) {
  if constexpr (MODE == BIAS) return Ref{0.f, top};
  return is_distant<MODE>(q, top) ? Ref{top, 0.f} : Ref{0.f, top * q.c2};
}
// what sums against `from` have to be multiplied by to be against `to`
template <int MODE> __device__ __forceinline__ float moved(const DenseGeo& q, float from, float to) {
  const Ref a = ref_of<MODE>(q, from), b = ref_of<MODE>(q, to);
  return exp2_fast(__builtin_fmaf(a.score - b.score, q.c2, a.x - b.x));
}

}  // namespace dense

constexpr int kCUs = 256;

inline dim3 grid_of(long long n) {     // n workgroups of at most 256 threads, in as many rows as the limit of 2^32 threads along x makes
  const long long x = n < (1LL << 23) ? n : (1LL << 23);
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

// Into how many pieces each of `wgs` workgroups is cut that go through `units` tiles (unit_us each, with two workgroups to a CU), where the
// sums of the pieces have to be written and read again (join_mb, for each piece).  A launch takes whole rounds of `slots` workgroups, so the
// rounds times a piece's tiles (and one for its beginning and end) are weighed against the join, at 4 TB/s and 6 us for its launch.
inline int cut(long long wgs, long long units, int slots, double unit_us, double join_mb) {
  int best = 1;
  double least = 0;
  for (int n = 1; n <= 64 && (n == 1 || units / n >= 4); ++n) {
    const double rounds = (double)((wgs * n + slots - 1) / slots);
    const double us = rounds * (double)((units + n - 1) / n + 1) * unit_us + (n > 1 ? 6.0 + 0.5 * n * join_mb : 0.0);
    if (n == 1 || us < least) least = us, best = n;
  }
  return best;
}
// us of a tile for one product, two workgroups of four waves to a CU (as all rules count; with 64 channels registers and LDS let in three to five of
// some kernels): bf16 64 rows, float32 64 rows of 64 or 32 of 128 channels
inline double product_us(const DenseGeo& q) { return q.dtype == DA_F32 ? 3.4 : q.d == 128 ? 0.85 : 0.5; }

}  // namespace da
