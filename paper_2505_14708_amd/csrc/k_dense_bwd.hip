// Dense attention of N queries to M keys, backward.
//
// With x = scale q.k + bias, p = exp(x - lse), delta_i = dO_i . O_i and ds = p (dO.v - delta):
//     dQ = scale ds K      dK = scale ds^T Q      dV = p^T dO      dtable[c] = sum of ds over the pairs whose bucket is c
// Two kernels, each of which makes p and dO V^T anew (seven products of N x M x d instead of five, but no sums shared between
// workgroups: no atomics, the same bits every time, and the sums stay in registers; bfloat16 has an eighth, p K):
//   dense_dq_kernel   32 queries a wave on the lane axis, tiles of K and V pass by
//   dense_dkv_kernel  32 keys a wave on the lane axis, tiles of Q and dO pass by, with lse and delta of their rows; also the sums for dtable
// Where one side is short the other is cut and the pieces' sums are put together by a third launch, in a fixed order.
//
// delta.  O is stored with the type's rounding (bfloat16: 2^-8), and dO . O inherits it.  But sum_j ds_ij = 0 for the delta that belongs to p and dO V^T,
// so what the first kernel's rows of ds add up to is what its delta is off by.  Its dQ has that times the row's sum of p K too much, which in bfloat16 it
// sums beside (dQ's error in norm, 512 keys, scores with a deviation of 1, 2, 4: 2.4e-3, 2.6e-3, 3.5e-3 without, 2.4e-3 with, which is what the roundings
// of ds and dQ are; 24 heads of 32760 by 512, both gradient kernels: 785 us without, 840 with; a round over the keys for delta alone ahead of
// the other would be 1040).  The second kernel, and dtable with it, gets the corrected delta.  (dtable was off by 2.9e-3 in norm with 64 heads of 512 by 512;
// by about its final rounding's 1.7e-3 so.)
//
// Bounds: one wave's chain of products and exponentials at two waves per SIMD.  24 heads of 32760 by 512, 128 channels: dQ 425 us, matrix pipe 47 %, vector
// pipe 43 %, LDS 17 % of the cycles; dK and dV 394 us, 50 %, 37 % and 31 %.  With 64 channels half the matrix work beside as many vector instructions.
#include <type_traits>
#include "attn_tiles.h"

namespace da {
namespace dense {

struct BwdArgs {
  const unsigned char *Q, *K, *V, *O, *dO;
  const void* table;
  const float* lse;
  unsigned char *dQ, *dK, *dV;
  void* dtable;
  float *start, *delta;            // [heads][padded rows]: where a row's scores start (start_of), -delta
  float *top, *log_l;              // the same: of rows in a far tile (kFarLse) the largest score and log2(sum) against it
  float *dq_part, *r_part, *dkv_part;  // sums of pieces: dQ, rows of ds, dK and dV
  unsigned char* k_part;           // the same: scale p K, in bfloat16 (it is for a correction of some thousandths)
  float* bias_part;                // [work item][buckets]
  long long rows, padded;          // rows of a head as the kernels see them, and rounded up to 32
  long long items;                 // work items of the launch
  int tiles, splits;               // dq: tiles of queries, pieces of the keys; dkv: tiles of keys, pieces of the queries
  int row_tiles, per_head;         // dkv: tiles of queries of a head, pieces of a head
};

// The sums of a square by r = key - query, keys on the lanes (32, twice) and queries in the registers: a register's halves are put into two, each
// with zeros in the upper lanes (v_permlane32_swap), and added up query by query, with a step of one lane between them (wave_shr): after 16
// queries lane l holds the sum of key - query = l - 15.  Two chains, queries 0..15 and 16..31, with an array each in LDS.
// (24 heads of 4099 by 4099, 128 channels, gradients of K and V: 734 us by way of a square in LDS, whose room also kept a second workgroup off
// the CU.  Straight into LDS with its own addition, ds_add_f32: 64 heads of 512 by 512 193 us instead of 73.)
__device__ __forceinline__ void add_diagonals(const f32x16& x, float* at, int n_bias, int lane) {
  auto next = [](float sum, unsigned y) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, sum), 0x138, 0xf, 0xf, true)) + __uint_as_float(y);
  };
  unsigned up[2][8];
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2 y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[8 * i + a]), 0u, false, false);
      sum[i] = next(sum[i], y[0]);
      up[i][a] = y[1];
    }
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int i = 0; i < 2; ++i) sum[i] = next(sum[i], up[i][a]);
  if (lane < 47) {
    at[lane - 15] += sum[0];
    at[n_bias + lane - 31] += sum[1];
  }
}

template <class T> __device__ __forceinline__ float dot_piece(const typename Type<T>::piece& x, const typename Type<T>::piece& y, float s) {
#pragma unroll
  for (int i = 0; i < Type<T>::PER; ++i) s = __builtin_fmaf((float)x[i], (float)y[i], s);
  return s;
}

// entries of the expanded bias row that belong to bucket c: first and last (last < first: none)
__device__ __forceinline__ void bucket_range(const RelRule& t, int c, int& first, int& last) {
  const bool ahead = t.bidirectional && c >= t.n;
  const int k = ahead ? c - t.n : c, zero = t.cut + kBiasPad;
  int lo, hi;                      // distances
  if (k < t.e) {
    lo = hi = k;
  } else {
    const int i = k - t.e;
    lo = i == 0 ? t.e : t.border[i - 1];
    hi = i == t.n_border ? zero : t.border[i] - 1;
  }
  if (ahead) {
    first = zero + max(lo, 1);
    last = zero + hi;
  } else {
    first = zero - hi;
    last = zero - lo;
    if (!t.bidirectional && k == 0) last = 2 * zero;   // one way: everything at or ahead of the query
  }
}

// What is added to a row's scores in the second kernel.  bf16: the sums of the matrix product start from -lse / scale, which costs nothing.
// float32: subtracted at the end, -lse log2(e) (from the start it would add its own roundings, of the size of lse, to every step's).
// Minus infinity where a row has nothing to attend or is padding: p is 0.
template <class T> __device__ __forceinline__ float start_of(const DenseGeo& q, float lse2) {
  const float x = sizeof(T) == 2 ? -lse2 / q.c2 : -lse2;
  return fabsf(x) < FLT_MIN ? 0.f : x;
}

// lse holds log(sum) beside the largest score in one float.  What it was rounded by, and its product with log2(e), scale all probabilities of a row by
// 1 +- |lse| 2^-23.6 (a single score is known no better, but they would no longer add up to 1): beside the operands' rounding that is small up to kFarLse
// (bfloat16: 8e-5 of 2e-3; float32: 1e-5, as its scores' own), and from 2^24 on it is everything.  So a workgroup with a row beyond makes its
// rows' largest scores and sums again, in a round of its own ahead of the others, takes the probabilities from those, and leaves them for the second
// kernel, with a mark in `start`.  (The mark is no ordinary row's start, and nothing beside a score where sums start from it.)
template <class T> constexpr float kFarLse = sizeof(T) == 2 ? 1024.f : 128.f;
constexpr int kFarMark = 1;
template <class T> __device__ __forceinline__ bool is_far_lse(float l) { return fabsf(l) > kFarLse<T> && l > -FLT_MAX; }

// The largest x (with a bias) or score (without) of each of the wave's 32 queries among all keys, and the sum of exp2(x - that), of waves that share
// their queries a wave's part of both; through the first tile's memory, one tile at a time.
template <class T, int D, int KB, int NW, int JW, int MODE>
__device__ __forceinline__ void far_sums(const DenseGeo& q, const Own<T, D> (&own)[1], const unsigned char* kb, long long ks, int len, int n_tiles,
                                         unsigned lds, unsigned s_lane, int wave, int lane, const float* bias_row, int first_row, int last_row,
                                         float& top, float& sum) {
  constexpr int RB = kRowBytes<T, D>;
  const int hi = lane >> 5;
  top = -FLT_MAX;
  sum = 0.f;
  for (int t = 0; t < n_tiles; ++t) {
    tile_barrier();
    load_tile<T, D, KB, NW>(kb, ks, t * KB, len - 1, lds, wave);
    wait_loads();
    tile_barrier();
    if (first_row > last_row) continue;
    for (int i = 0; i < KB / 32 / JW; ++i) {
      const int sub = JW > 1 ? wave : i, key0 = t * KB + 32 * sub;
      if (key0 >= len) break;
      f32x16 s[1];
      scores<T, D, 1>(lds + sub * 32 * RB + s_lane, own, s);
      const int left = len - key0 - 8 * hi, low = MODE == BIAS ? key0 - first_row - q.q_pos : 0, wide = MODE == BIAS ? q.rule.cut + kBiasPad : 0;
      float m = -FLT_MAX;
#pragma unroll
      for (int a = 0; a < 16; ++a) {
        const int r = 16 * (a >> 3) + (a & 7);
        if constexpr (MODE == BIAS) s[0][a] = biased<T>(q, s[0][a], bias_row[min(max(low + 8 * hi + r - (lane & 31) + wide, 0), 2 * wide)]);
        s[0][a] = r < left ? s[0][a] : -INFINITY;
        m = fmaxf(m, s[0][a]);
      }
      m = fmaxf(top, max_across_halves(m));
      sum *= exp2_fast(MODE == BIAS ? top - m : (top - m) * q.c2);
#pragma unroll
      for (int a = 0; a < 16; ++a) sum += MODE == BIAS ? exp2_fast(s[0][a] - m) : power_of<T>(q, s[0][a] - m, 0.f);
      top = m;
    }
  }
  sum = sum_across_halves(sum);
}

template <class T, int D, int JW> constexpr int kDqWaves = JW > 1 || kRowBytes<T, D> > 256 ? 1 : 2;

// bf16, 128 channels: the two sums are 128 registers, Q's and dO's rows 64 and the two squares 32, of 256.  With a bias 20 would be spilled; there dO's rows are
// in LDS, 8 KB a wave, and the tiles of 32 rows so that two workgroups still fit a CU (24 heads of 4099 by 4099, both gradient kernels: 950 us
// spilled, 916 so; without a bias, 24 heads of 32760 by 512, 840 and 860 us).
template <class T, int D, int JW, int MODE> constexpr bool kGradInLds = sizeof(T) == 2 && D == 128 && JW == 1 && MODE == BIAS;
template <class T, int D, int JW, int MODE> constexpr int kDqRows = kGradInLds<T, D, JW, MODE> ? 32 : kTileRows<T, D, JW>;

template <class T, int D, int NW, int JW, int MODE>
__global__ __launch_bounds__(64 * NW, (kDqWaves<T, D, JW>)) void dense_dq_kernel(DenseGeo q, BwdArgs g) {
  constexpr int KB = kDqRows<T, D, JW, MODE>, RB = kRowBytes<T, D>, TILE = KB * RB, RT = 32 * (NW / JW);
  constexpr bool GRAD_IN_LDS = kGradInLds<T, D, JW, MODE>;
  constexpr int NZ = sizeof(T) == 2 ? 2 : 1;           // sums of ds K; of p K
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[4 * TILE + (GRAD_IN_LDS ? NW * 32 * RB : 0)];
  __shared__ float parts[NW * 32];
  extern __shared__ __attribute__((aligned(16))) float bias_row[];
  const long long id = blockIdx.y * (long long)gridDim.x + blockIdx.x;
  if (id >= g.items) return;
  const long long item = xcd_order(id, g.items, (long long)g.tiles * g.splits);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hi = lane >> 5;
  const int split = (int)(item % g.splits);
  const long long bht = item / g.splits;
  const int tile = (int)(bht % g.tiles);
  const long long bh = bht / g.tiles;
  const int heads = heads_of<MODE>(q);
  const int b = (int)(bh / heads), hd = (int)(bh - (long long)b * heads), hk = kv_head<MODE>(q, hd);
  const int len = q.kv_len ? min(max(q.kv_len[b], 0), q.M) : q.M;
  const int first_row = tile * RT + (JW > 1 ? 0 : wave * 32), last_row = (int)g.rows - 1;
  const int n_tiles = (len + KB - 1) / KB, each = (n_tiles + g.splits - 1) / g.splits;
  const int t0 = min(split * each, n_tiles), t1 = min(t0 + each, n_tiles);
  const long long ks = q.k.sn * (long long)sizeof(T), vs = q.v.sn * (long long)sizeof(T);
  const unsigned char* kb = g.K + (b * q.k.sb + hk * q.k.sh) * (long long)sizeof(T);
  const unsigned char* vb = g.V + (b * q.v.sb + hk * q.v.sh) * (long long)sizeof(T);
  const unsigned lds = (unsigned)(uintptr_t)(lds_f32*)tiles;
  const int rr = first_row + (lane & 31), rc = min(rr, last_row);
  // lse of the wave's and of all of the workgroup's rows, ahead of the longer loads
  const float l = g.lse[bh * g.rows + rc];
  float all_l[RT > 64 ? RT / 64 : 1];
#pragma unroll
  for (int i = 0; i < RT; i += 64) all_l[i / 64] = g.lse[bh * g.rows + min(tile * RT + i + lane % (RT < 64 ? RT : 64), last_row)];
  if (t0 < t1) {
    load_tile<T, D, KB, NW>(kb, ks, t0 * KB, len - 1, lds, wave);
    load_tile<T, D, KB, NW>(vb, vs, t0 * KB, len - 1, lds + TILE, wave);
  }
  if constexpr (MODE == BIAS) fill_bias<T>(bias_row, q.rule, (const T*)g.table, q.H, hd, threadIdx.x, 64 * NW);

  Own<T, D> own[1], grad[1];
  f32x16 z[NZ][D / 32];
  own[0].load(g.Q + query_offset<MODE>(q, q.q, b, hd, rc) * (long long)sizeof(T), hi);
  grad[0].load(g.dO + query_offset<MODE>(q, q.dout, b, hd, rc) * (long long)sizeof(T), hi);
  float delta = 0.f;
  {
    Own<T, D> out;
    out.load(g.O + query_offset<MODE>(q, q.o, b, hd, rc) * (long long)sizeof(T), hi);
#pragma unroll
    for (int t = 0; t < Own<T, D>::N; ++t) delta = dot_piece<T>(grad[0].x[t], out.x[t], delta);
    delta = sum_across_halves(delta);
    if constexpr (GRAD_IN_LDS) {
#pragma unroll
      for (int t = 0; t < Own<T, D>::N; ++t) *(bf16x8*)(tiles + 4 * TILE + wave * 32 * RB + t * 1024 + lane * 16) = grad[0].x[t];
    }
  }
  float lse2 = rr <= last_row && l != -INFINITY ? l * kLog2e : INFINITY;   // far: log2(sum)
  bool far = false;                // the same for all waves of the workgroup
  for (float x : all_l) far = far || is_far_lse<T>(x);
  far = __builtin_amdgcn_readfirstlane(__any(far));
  float off = 0.f;                 // this lane's part of the row's sum of ds
#pragma unroll
  for (int n = 0; n < NZ; ++n)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) z[n][dt] = zero16();
  const unsigned s_lane = scores_lane<T, D>(lane), m_lane = mix_lane<T, D>(lane);
  const unsigned bias_lds = MODE == BIAS ? (unsigned)(uintptr_t)(lds_f32*)bias_row : 0u;

  float top = 0.f;
  if (__builtin_expect(far, 0)) {
    wait_loads();
    float sum;
    far_sums<T, D, KB, NW, JW, MODE>(q, own, kb, ks, len, n_tiles, lds, s_lane, wave, lane, bias_row, first_row, last_row, top, sum);
    if constexpr (JW > 1) {
      if (hi == 0) parts[wave * 32 + lane] = top;
      __syncthreads();
      float most = -FLT_MAX;
#pragma unroll
      for (int w = 0; w < NW; ++w) most = fmaxf(most, parts[w * 32 + (lane & 31)]);
      sum *= exp2_fast(MODE == BIAS ? top - most : (top - most) * q.c2);
      __syncthreads();
      if (hi == 0) parts[wave * 32 + lane] = sum;
      __syncthreads();
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) sum += parts[w * 32 + (lane & 31)];
      __syncthreads();
      top = most;
    }
    lse2 = rr <= last_row && sum > 0.f ? __builtin_log2f(sum) : INFINITY;
    tile_barrier();
    if (t0 < t1) {
      load_tile<T, D, KB, NW>(kb, ks, t0 * KB, len - 1, lds, wave);
      load_tile<T, D, KB, NW>(vb, vs, t0 * KB, len - 1, lds + TILE, wave);
    }
  }
  for (int t = t0; t < t1; ++t) {
    const unsigned buf = lds + ((t - t0) & 1) * (2 * TILE);
    wait_loads();
    tile_barrier();
    if (t + 1 < t1) {
      const unsigned next = lds + ((t + 1 - t0) & 1) * (2 * TILE);
      load_tile<T, D, KB, NW>(kb, ks, (t + 1) * KB, len - 1, next, wave);
      load_tile<T, D, KB, NW>(vb, vs, (t + 1) * KB, len - 1, next + TILE, wave);
    }
    if (first_row > last_row) continue;
#pragma unroll
    for (int i = 0; i < KB / 32 / JW; ++i) {
      const int sub = JW > 1 ? wave : i;
      const int key0 = t * KB + 32 * sub;
      if (key0 >= len) break;
      f32x16 s[1], dp[1];
      scores<T, D, 1>(buf + sub * 32 * RB + s_lane, own, s);
      if constexpr (GRAD_IN_LDS) {
        dp[0] = zero16();
        add_scores_lds<D>(buf + TILE + sub * 32 * RB + s_lane, lds + 4 * TILE + wave * 32 * RB + lane * 16, dp[0]);
      } else {
        scores<T, D, 1>(buf + TILE + sub * 32 * RB + s_lane, grad, dp);
      }
      const int left = len - key0 - 8 * hi;
      if constexpr (MODE == BIAS) {
        const int low = key0 - first_row - q.q_pos;          // r of key 0 and query 0 of the square
        if (low - 31 >= q.rule.cut || low + 31 <= -q.rule.cut) {
          const float out = bias_row[low > 0 ? 2 * (q.rule.cut + kBiasPad) : 0];
          if (__builtin_expect(far, 0)) {
#pragma unroll
            for (int a = 0; a < 16; ++a) s[0][a] = exp2_fast((biased<T>(q, s[0][a], out) - top) - lse2);
          } else {
#pragma unroll
            for (int a = 0; a < 16; ++a) s[0][a] = power_of<T>(q, s[0][a], out - lse2);
          }
        } else {
          f32x16 bs;
          read_bias<1>(bias_lds + 4 * (low + 8 * hi - (lane & 31) + q.rule.cut + kBiasPad), bs);
          if (__builtin_expect(far, 0)) {
#pragma unroll
            for (int a = 0; a < 16; ++a) s[0][a] = exp2_fast((biased<T>(q, s[0][a], bs[a]) - top) - lse2);
          } else {
#pragma unroll
            for (int a = 0; a < 16; ++a) s[0][a] = power_of<T>(q, s[0][a], bs[a] - lse2);
          }
        }
      } else {
        if (far || key0 + 32 > len) {
#pragma unroll
          for (int a = 0; a < 16; ++a) s[0][a] = 16 * (a >> 3) + (a & 7) < left ? s[0][a] - top : -INFINITY;
        }
#pragma unroll
        for (int a = 0; a < 16; ++a) s[0][a] = power_of<T>(q, s[0][a], -lse2);
      }
      if (MODE == BIAS && key0 + 32 > len) {
#pragma unroll
        for (int a = 0; a < 16; ++a) s[0][a] = 16 * (a >> 3) + (a & 7) < left ? s[0][a] : 0.f;
      }
      Mixed<T> c[NZ];
      if constexpr (NZ == 2) c[1] = Mixed<T>(s[0]);
#pragma unroll
      for (int a = 0; a < 16; ++a) {
        s[0][a] *= dp[0][a] - delta;
        off += s[0][a];
      }
      c[0] = Mixed<T>(s[0]);
      mix<T, D, NZ>(buf + sub * 32 * RB + m_lane, c, z);
    }
  }
  off = sum_across_halves(off);
  if constexpr (JW > 1) {
    if (hi == 0) parts[wave * 32 + lane] = off;
    __syncthreads();
    off = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) off += parts[w * 32 + (lane & 31)];
  }
  const bool there = rr <= last_row;
  const float f = g.splits == 1 ? off : 0.f;           // (pieces: dense_sum_dq_kernel)
  if constexpr (NZ == 2) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int a = 0; a < 16; ++a) z[0][dt][a] = __builtin_fmaf(z[1][dt][a], -f, z[0][dt][a]);
  }
  if constexpr (JW > 1) {
    float* buf = (float*)tiles;
    join_waves<D, NW>(buf, wave, lane, z[0], q.scale, [&](int row, int c, f32x4 (&x)[2]) {
      if (first_row + row > last_row) return;
      if (g.splits == 1) store8<T>(g.dQ + (query_offset<MODE>(q, q.dq, b, hd, first_row + row) + c) * (long long)sizeof(T), x, 1.f);
      else store8<float>((unsigned char*)(g.dq_part + (item * RT + row) * D + c), x, 1.f);
    });
    if constexpr (NZ == 2) {
      if (g.splits > 1)
        join_waves<D, NW>(buf, wave, lane, z[1], q.scale, [&](int row, int c, f32x4 (&x)[2]) {
          if (first_row + row <= last_row) store8<T>(g.k_part + ((item * RT + row) * D + c) * (long long)sizeof(T), x, 1.f);
        });
    }
    if (wave != 0) return;
    if (g.splits > 1 && there && hi == 0) g.r_part[item * RT + lane] = off;
  } else if (g.splits == 1) {
    store_column<T, D>(g.dQ + query_offset<MODE>(q, q.dq, b, hd, rc) * (long long)sizeof(T), hi, z[0], q.scale, there);
  } else {
    const long long at = item * RT + wave * 32 + (lane & 31);
    store_column<float, D>((unsigned char*)(g.dq_part + at * D), hi, z[0], q.scale, there);
    if constexpr (NZ == 2) store_column<T, D>(g.k_part + at * RB, hi, z[1], q.scale, there);
    if (there && hi == 0) g.r_part[at] = off;
  }
  if (split == 0 && hi == 0 && rr < g.padded) {
    g.start[bh * g.padded + rr] = far ? __int_as_float(kFarMark) : start_of<T>(q, lse2);
    if (__builtin_expect(far, 0)) {
      g.top[bh * g.padded + rr] = top;
      g.log_l[bh * g.padded + rr] = lse2;
    }
    g.delta[bh * g.padded + rr] = there ? -(g.splits == 1 ? delta + off : delta) : 0.f;
  }
}

// Probabilities of a square (keys on the lanes) whose queries are in a far tile: rows r of top and log_l for the registers of row r.  (None is above 1:
// the scores are sums in another order here.)  r0: key - query of the lane's key and the square's row 8 (l / 32).
template <class T, int MODE>
__device__ __forceinline__ void far_powers(const DenseGeo& q, f32x16& s, const float* top, const float* log_l, const float* bias_row, int r0) {
  const int wide = MODE == BIAS ? q.rule.cut + kBiasPad : 0;
#pragma unroll
  for (int a = 0; a < 16; ++a) {
    const int r = 16 * (a >> 3) + (a & 7);
    float x;
    if constexpr (MODE == BIAS) x = biased<T>(q, s[a], bias_row[min(max(r0 - r + wide, 0), 2 * wide)]) - top[r];
    else x = biased<T>(q, s[a] - top[r], 0.f);
    s[a] = exp2_fast(fminf(x, 0.f) - log_l[r]);
    if (a % 4 == 3) __builtin_amdgcn_sched_barrier(0);            // (a few rows' numbers at a time: registers)
  }
}

// waves to a SIMD that the kernel below is made for
template <class T, int D, int JW> constexpr int kDkvWaves = JW > 1 || kRowBytes<T, D> > 256 ? 1 : 2;

// bf16, 128 channels: the sums of 32 keys are 128 registers, K's and V's rows 64 and the squares of scores and of dO V^T 32, of 256.  With a bias
// that is too much by a few, which would be spilled, and their way back waits, in the order of all loads, for the next tiles (24 heads of 4099 by
// 4099: 545 us).  There V's rows are in LDS, 8 KB a wave, and the tiles are of 32 rows so that two workgroups still fit a CU (511 us).
template <class T, int D, int JW, int MODE> constexpr bool kVInLds = sizeof(T) == 2 && D == 128 && JW == 1 && MODE == BIAS;
template <class T, int D, int JW, int MODE> constexpr int kDkvRows = kVInLds<T, D, JW, MODE> ? 32 : kTileRows<T, D, JW>;

template <class T, int D, int NW, int JW, int MODE>
__global__ __launch_bounds__(64 * NW, (kDkvWaves<T, D, JW>)) void dense_dkv_kernel(DenseGeo q, BwdArgs g) {
  constexpr int QB = kDkvRows<T, D, JW, MODE>, RB = kRowBytes<T, D>, TILE = QB * RB, STAGE = 2 * TILE + 1024, KT = 32 * (NW / JW);
  constexpr bool V_IN_LDS = kVInLds<T, D, JW, MODE>;
  // twice: Q, dO, where their rows start from and delta; the waves' own rows of V
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[2 * STAGE + (V_IN_LDS ? NW * 32 * RB : 0)];
  extern __shared__ __attribute__((aligned(16))) float bias_row[];           // then each wave's sums of ds by r
  const long long id = blockIdx.y * (long long)gridDim.x + blockIdx.x;
  if (id >= g.items) return;
  const long long item = xcd_order(id, g.items, (long long)g.tiles * g.splits);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hi = lane >> 5;
  // the tiles of keys of one piece of the queries are neighbours: they read the same rows
  const int tile = (int)(item % g.tiles);
  const long long rest = item / g.tiles;
  const int split = (int)(rest % g.splits);
  const long long bh = rest / g.splits;
  const int b = (int)(bh / q.Hk), hk = (int)(bh - (long long)b * q.Hk);
  const int len = q.kv_len ? min(max(q.kv_len[b], 0), q.M) : q.M;
  const int key0 = tile * KT + (JW > 1 ? 0 : wave * 32);
  const int hd = MODE == PACKED || q.group == 1 ? hk : hk * q.group + split / g.per_head;
  const int piece = MODE == PACKED || q.group == 1 ? split : split % g.per_head;
  const long long stat = ((long long)b * heads_of<MODE>(q) + hd) * g.padded;
  const int each = (g.row_tiles + g.per_head - 1) / g.per_head;
  const int t0 = min(piece * each, g.row_tiles), t1 = tile * KT < len ? min(t0 + each, g.row_tiles) : t0;
  const int last_row = (int)g.rows - 1;
  const unsigned lds = (unsigned)(uintptr_t)(lds_f32*)tiles;

  // a tile of queries and of dO, and what goes with their rows
  auto load_rows = [&](int t, unsigned to) {
    const int first = t * QB, last = min(first + QB - 1, last_row);
    if constexpr (MODE != PACKED) {
      load_tile<T, D, QB, NW>(g.Q + (b * q.q.sb + hd * q.q.sh) * (long long)sizeof(T), q.q.sn * (long long)sizeof(T), first, last, to, wave);
      load_tile<T, D, QB, NW>(g.dO + (b * q.dout.sb + hd * q.dout.sh) * (long long)sizeof(T), q.dout.sn * (long long)sizeof(T), first, last,
                              to + TILE, wave);
    } else {
      constexpr int CPR = RB / 16, RPS = 64 / CPR;
      const int lane = opaque_lane();
#pragma unroll
      for (int k = 0; k < QB / RPS / NW; ++k) {
        const int it = k * NW + wave, row = it * RPS + lane / CPR, rr = min(first + row, last);
        const unsigned p = ((lane % CPR) ^ swizzle<T, D>(row)) << 4;
        dma16(g.Q + query_offset<MODE>(q, q.q, b, hd, rr) * (long long)sizeof(T) + p, to + it * 1024);
        dma16(g.dO + query_offset<MODE>(q, q.dout, b, hd, rr) * (long long)sizeof(T) + p, to + TILE + it * 1024);
      }
    }
    constexpr int CH = QB > 64 ? QB / 64 : 1;        // 64 rows' numbers at a time
#pragma unroll
    for (int i = 0; i < 2 * CH; ++i) {
      if (i % NW != wave) continue;
      const long long rr = stat + min((long long)first + 64 * (i % CH) + lane, g.padded - 1);
      dma4((i / CH ? g.delta : g.start) + rr, to + 2 * TILE + 512 * (i / CH) + 256 * (i % CH));
    }
  };
  if (t0 < t1) load_rows(t0, lds);
  const int n_bias = MODE == BIAS ? (bias_entries(q.rule.cut) + 3) & ~3 : 0;
  float* diag = bias_row + n_bias + wave * (2 * n_bias);         // this wave's sums by r, as the bias row: two arrays
  float far_sum[2] = {0.f, 0.f};
  if constexpr (MODE == BIAS) {
    fill_bias<T>(bias_row, q.rule, (const T*)g.table, q.H, hd, threadIdx.x, 64 * NW);
    for (int i = lane; i < 2 * n_bias; i += 64) diag[i] = 0.f;
  }

  Own<T, D> own_k[1], own_v[1];
  f32x16 zk[1][D / 32], zv[1][D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) zk[0][dt] = zv[0][dt] = zero16();
  if (t0 < t1) {
    const long long kc = min(key0 + (lane & 31), len - 1);
    own_k[0].load(g.K + (b * q.k.sb + hk * q.k.sh + kc * q.k.sn) * (long long)sizeof(T), hi);
    own_v[0].load(g.V + (b * q.v.sb + hk * q.v.sh + kc * q.v.sn) * (long long)sizeof(T), hi);
    if constexpr (V_IN_LDS) {
#pragma unroll
      for (int t = 0; t < Own<T, D>::N; ++t) *(bf16x8*)(tiles + 2 * STAGE + wave * 32 * RB + t * 1024 + lane * 16) = own_v[0].x[t];
    }
  }
  const unsigned s_lane = scores_lane<T, D>(lane), m_lane = mix_lane<T, D>(lane);
  const unsigned bias_lds = MODE == BIAS ? (unsigned)(uintptr_t)(lds_f32*)bias_row : 0u;

  for (int t = t0; t < t1; ++t) {
    const unsigned buf = lds + ((t - t0) & 1) * STAGE;
    wait_loads();
    tile_barrier();
    if (t + 1 < t1) load_rows(t + 1, lds + ((t + 1 - t0) & 1) * STAGE);
    if (key0 >= len) continue;
#pragma unroll
    for (int i = 0; i < QB / 32 / JW; ++i) {
      const int sub = JW > 1 ? wave : i;
      const int row0 = t * QB + 32 * sub;
      if (row0 > last_row) break;
      // Sums start from what belongs to their rows (start_of, -delta): registers 4i .. 4i + 3 have rows 16(i / 2) + 8 hi + 4(i % 2) + 0..3.
      constexpr bool kLate = sizeof(T) == 4;
      f32x16 s[1], dp[1], late;
      int mark = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned at = buf + 2 * TILE + 4 * (32 * sub + 16 * (i >> 1) + 8 * hi + 4 * (i & 1));
        const f32x4 l = *(lds_f32x4*)(uintptr_t)at, dl = *(lds_f32x4*)(uintptr_t)(at + 512);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          late[4 * i + e] = kLate ? l[e] : 0.f;
          s[0][4 * i + e] = kLate ? 0.f : l[e];
          dp[0][4 * i + e] = dl[e];
        }
        if (i == 0) mark = __builtin_amdgcn_readfirstlane(__float_as_int(l[0]));
      }
      add_scores<T, D, 1>(buf + sub * 32 * RB + s_lane, own_k, s);
      if constexpr (V_IN_LDS) add_scores_lds<D>(buf + TILE + sub * 32 * RB + s_lane, lds + 2 * STAGE + wave * 32 * RB + lane * 16, dp[0]);
      else add_scores<T, D, 1>(buf + TILE + sub * 32 * RB + s_lane, own_v, dp);
      const int low = MODE == BIAS ? key0 - row0 - q.q_pos : 0;      // r of key 0 and query 0 of the square
      const bool is_far = MODE == BIAS && (low - 31 >= q.rule.cut || low + 31 <= -q.rule.cut);
      if (__builtin_expect(mark == kFarMark, 0)) {
        far_powers<T, MODE>(q, s[0], g.top + stat + row0 + 8 * hi, g.log_l + stat + row0 + 8 * hi, bias_row, low + (lane & 31) - 8 * hi);
      } else if constexpr (MODE == BIAS) {
        if (is_far) {
          const float far = bias_row[low > 0 ? 2 * (q.rule.cut + kBiasPad) : 0];
#pragma unroll
          for (int a = 0; a < 16; ++a) s[0][a] = power_of<T>(q, s[0][a], kLate ? far + late[a] : far);
        } else {
          f32x16 bs;
          read_bias<-1>(bias_lds + 4 * (low + (lane & 31) - 8 * hi + q.rule.cut + kBiasPad), bs);
#pragma unroll
          for (int a = 0; a < 16; ++a) s[0][a] = power_of<T>(q, s[0][a], kLate ? bs[a] + late[a] : bs[a]);
        }
      } else {
        // (A branch that is always taken: in one block with the products the exponentials cost 16 to 48 spilled registers, in one of their own none.
        // 24 heads of 32760 by 512: 540 and 427 us.)
        int always = 1;
        asm volatile("" : "+s"(always));
        if (always)
#pragma unroll
        for (int a = 0; a < 16; ++a) s[0][a] = kLate ? power_of<T>(q, s[0][a], late[a]) : exp2_fast(s[0][a] * q.c2);
      }
      const Mixed<T> p[1] = {Mixed<T>(s[0])};
#pragma unroll
      for (int a = 0; a < 16; ++a) dp[0][a] *= s[0][a];
      const Mixed<T> ds[1] = {Mixed<T>(dp[0])};
      if constexpr (MODE == BIAS) {
        if (key0 + 32 > len) {
          const bool is_there = key0 + (lane & 31) < len;
#pragma unroll
          for (int a = 0; a < 16; ++a) dp[0][a] = is_there ? dp[0][a] : 0.f;
        }
        if (is_far) {
          float x = 0.f;
#pragma unroll
          for (int a = 0; a < 16; ++a) x += dp[0][a];
          far_sum[0] += low > 0 ? 0.f : x;
          far_sum[1] += low > 0 ? x : 0.f;
        } else {
          add_diagonals(dp[0], diag + low + q.rule.cut + kBiasPad, n_bias, lane);
        }
      }
      mix<T, D, 1>(buf + TILE + sub * 32 * RB + m_lane, p, zv);
      mix<T, D, 1>(buf + sub * 32 * RB + m_lane, ds, zk);
    }
  }
  const long long bhs = (long long)q.B * q.Hk;
  float* part = g.dkv_part + (split * bhs + bh) * q.M * D;               // K's, and V's behind all of K's
  const long long v_part = g.splits * bhs * q.M * D;
  unsigned char* dk = g.dK + (b * q.dk.sb + hk * q.dk.sh) * (long long)sizeof(T);
  unsigned char* dv = g.dV + (b * q.dv.sb + hk * q.dv.sh) * (long long)sizeof(T);
  if constexpr (JW > 1) {
    auto put = [&](unsigned char* out, long long stride, float* parts, int row, int c, f32x4 (&x)[2]) {
      const int key = key0 + row;
      if (key >= len) x[0] = x[1] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (g.splits > 1 ? key >= len : key >= q.M) return;
      if (g.splits > 1) store8<float>((unsigned char*)(parts + (long long)key * D + c), x, 1.f);
      else store8<T>(out + (key * stride + c) * (long long)sizeof(T), x, 1.f);
    };
    float* buf = (float*)tiles;
    join_waves<D, NW>(buf, wave, lane, zk[0], q.scale, [&](int row, int c, f32x4 (&x)[2]) { put(dk, q.dk.sn, part, row, c, x); });
    join_waves<D, NW>(buf, wave, lane, zv[0], 1.f, [&](int row, int c, f32x4 (&x)[2]) { put(dv, q.dv.sn, part + v_part, row, c, x); });
  } else {
    const int key = key0 + (lane & 31);
    const long long kc = min(key, q.M - 1);
    if (g.splits == 1) {
      if (key >= len) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) zk[0][dt] = zv[0][dt] = zero16();
      }
      store_column<T, D>(dk + kc * q.dk.sn * (long long)sizeof(T), hi, zk[0], q.scale, key < q.M);
      store_column<T, D>(dv + kc * q.dv.sn * (long long)sizeof(T), hi, zv[0], 1.f, key < q.M);
    } else {
      store_column<float, D>((unsigned char*)(part + kc * D), hi, zk[0], q.scale, key < len);
      store_column<float, D>((unsigned char*)(part + v_part + kc * D), hi, zv[0], 1.f, key < len);
    }
  }
  if constexpr (MODE == BIAS) {
    // the waves' sums by r, added up bucket by bucket: eight lanes to a bucket
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x = far_sum[i];
#pragma unroll
      for (int w = 32; w >= 1; w >>= 1) x += __shfl_xor(x, w);
      if (lane == 0) diag[(i ? 2 * (q.rule.cut + kBiasPad) : 0)] += x;
    }
    __syncthreads();
    for (int c0 = 0; c0 < q.buckets; c0 += 8 * NW) {
      const int c = c0 + (threadIdx.x >> 3);
      float x = 0.f;
      if (c < q.buckets) {
        int first, last;
        bucket_range(q.rule, c, first, last);
        for (int i = first + (threadIdx.x & 7); i <= last; i += 8)
#pragma unroll
          for (int w = 0; w < 2 * NW; ++w) x += bias_row[n_bias + w * n_bias + i];
      }
#pragma unroll
      for (int w = 4; w >= 1; w >>= 1) x += __shfl_xor(x, w);
      if (c < q.buckets && (threadIdx.x & 7) == 0) g.bias_part[item * q.buckets + c] = x;
    }
  }
}

// Sums over the pieces, D / 4 threads to a row, in the order of the pieces.
template <class T, int D>
__device__ __forceinline__ void sum_pieces(const float* part, long long step, int n, T* out, int c) {
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < n; ++s) x += *(const f32x4*)(part + s * step + 4 * c);
  if constexpr (sizeof(T) == 2) *(bf16x4*)(out + 4 * c) = __builtin_convertvector(x, bf16x4);
  else *(f32x4*)(out + 4 * c) = x;
}

template <class T, int D, int MODE>
__global__ __launch_bounds__(256) void dense_sum_dq_kernel(DenseGeo q, BwdArgs g, int RT) {
  constexpr int P = D / 4;
  const long long row = (blockIdx.y * (long long)gridDim.x + blockIdx.x) * (256 / P) + threadIdx.x / P;
  const int heads = heads_of<MODE>(q);
  if (row >= (long long)q.B * heads * g.rows) return;
  const long long bh = row / g.rows;
  const int rr = (int)(row - bh * g.rows), b = (int)(bh / heads), hd = (int)(bh - (long long)b * heads), c = threadIdx.x % P;
  const int tile = rr / RT;
  const long long first = ((bh * g.tiles + tile) * g.splits) * RT + (rr - tile * RT);
  T* out = (T*)g.dQ + query_offset<MODE>(q, q.dq, b, hd, rr) + 4 * c;
  float off = 0.f;                 // what delta is off by
  f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < g.splits; ++s) {
    const long long at = first + (long long)s * RT;
    off += g.r_part[at];
    x += *(const f32x4*)(g.dq_part + at * D + 4 * c);
    if constexpr (sizeof(T) == 2) y += __builtin_convertvector(*(const bf16x4*)(g.k_part + (at * D + 4 * c) * 2), f32x4);
  }
  if constexpr (sizeof(T) == 2) *(bf16x4*)out = __builtin_convertvector(x - y * off, bf16x4);
  else *(f32x4*)out = x;
  if (c == 0) g.delta[bh * g.padded + rr] -= off;
}

template <class T, int D>
__global__ __launch_bounds__(256) void dense_sum_dkv_kernel(DenseGeo q, BwdArgs g) {
  constexpr int P = D / 4;
  const long long n = (long long)q.B * q.Hk * q.M;
  long long row = (blockIdx.y * (long long)gridDim.x + blockIdx.x) * (256 / P) + threadIdx.x / P;
  if (row >= 2 * n) return;
  const bool v = row >= n;
  if (v) row -= n;
  const long long bh = row / q.M;
  const int key = (int)(row - bh * q.M), b = (int)(bh / q.Hk), hk = (int)(bh - (long long)b * q.Hk);
  const int len = q.kv_len ? min(max(q.kv_len[b], 0), q.M) : q.M;
  const Rows& r = v ? q.dv : q.dk;
  sum_pieces<T, D>(g.dkv_part + ((v ? g.splits * n : 0) + row) * D, n * D, key < len ? g.splits : 0,
                   (T*)(v ? g.dV : g.dK) + (b * r.sb + hk * r.sh + key * r.sn), threadIdx.x % P);
}

// dtable[c][h]: the work items of head h in order, a few stretches of them at a time
template <class T>
__global__ __launch_bounds__(256) void dense_sum_bias_kernel(DenseGeo q, BwdArgs g) {
  __shared__ float sums[256];
  const long long h = blockIdx.y * (long long)gridDim.x + blockIdx.x;
  if (h >= q.H) return;
  const int c = threadIdx.x % q.buckets, slice = threadIdx.x / q.buckets, slices = 256 / q.buckets;
  const long long run = (long long)g.per_head * g.tiles, n = run * q.B, per_batch = run * q.H;   // (a batch element's heads follow each other)
  float x = 0.f;
  if (slice < slices) {
    const long long each = (n + slices - 1) / slices, i0 = slice * each, i1 = min(i0 + each, n);
#pragma unroll 8
    for (long long i = i0; i < i1; ++i) {
      const long long b = i / run;
      x += g.bias_part[(b * per_batch + h * run + (i - b * run)) * q.buckets + c];
    }
  }
  sums[threadIdx.x] = x;
  __syncthreads();
  if (threadIdx.x < q.buckets) {
    float y = 0.f;
    for (int s = 0; s < slices; ++s) y += sums[s * q.buckets + threadIdx.x];
    ((T*)g.dtable)[(long long)threadIdx.x * q.H + h] = (T)y;
  }
}

}  // namespace dense

namespace {

constexpr size_t kLds = 160 * 1024;

struct BwdPlan {
  int join, row_tile, tiles, splits;                                            // dq
  int kv_join, kv_tiles, kv_splits, per_head, row_tiles, q_tile;                // dkv
  size_t start, delta, top, log_l, k_part, dq_part, r_part, dkv_part, bias_part, total;
};

inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

// LDS of the second kernel beside its tiles: bias and sums by r of `waves` waves
inline size_t dkv_bias_lds(const DenseGeo& q, int waves) {
  if (!q.bias) return 0;
  const size_t n = (dense::bias_entries(q.rule.cut) + 3) & ~3;
  return (n + 2 * waves * n) * sizeof(float);
}

// Workgroups of four waves with 32 queries (keys) each, or, where they are too few, of waves that share 32 and take the other side in turn.  Either is cut
// where that fills its rounds.  The waves also join where there are many workgroups but three of the four waves would have nothing, if the other side is
// four of their tiles or more (960 heads of 32 by 32, 128 channels: 29 us, joining 65).  Not in bfloat16 with 128 channels, where two workgroups
// fit a CU and one that joins (960 heads of 513 queries by 16 keys: 180 us, joining 196).
// 192 heads of 32760 queries by 16 keys, 128 channels, bfloat16: 2602 us uncut with one wave of four at work, 1951 in 8 pieces, 1948 in 4 joining; float32,
// 8190 queries: 3232, 2731 and 2032.  By 64 keys: 2765, 2221 and 2464; 3699, 3220 and 3363.
BwdPlan plan_bwd(const DenseGeo& q) {
  BwdPlan p;
  const long long rows = dense_rows(q), heads = (long long)q.B * dense_heads(q), kv_heads = (long long)q.B * q.Hk;
  const bool f32 = q.dtype == DA_F32;
  const int row_bytes = q.d * (f32 ? 4 : 2), tile = row_bytes > 256 ? 32 : 64, enough = kCUs / 4 * 3;
  const int kv_tile = !f32 && q.d == 128 && q.bias ? 32 : tile;
  const int joined = row_bytes > 256 ? 64 : 128, join_slots = row_bytes == 128 ? 2 * kCUs : kCUs;      // rows of a joining workgroup's tile
  const int few = f32 || q.d == 64 ? 32 : 0;
  const int slots = row_bytes > 256 ? kCUs : 2 * kCUs;                                                 // (one wave to a SIMD there)
  auto pieces_joined = [&](long long wgs, long long units, double join_mb) {
    if (2 * wgs > join_slots) return cut(wgs, units, join_slots, 2 * product_us(q), join_mb);
    long long n = join_slots / wgs;
    n = n > units / 2 ? units / 2 : n;
    return (int)(n < 1 ? 1 : n);
  };
  long long wgs = heads * ((rows + 127) / 128);
  p.join = 0;
  p.splits = rows > 64 || wgs >= enough ? cut(wgs, (q.M + tile - 1) / tile, slots, 3 * product_us(q), 128.0 * wgs * q.d * 4e-6) : 1;
  if (wgs * p.splits < enough || (rows <= few && q.M >= 4 * joined)) {
    const long long n = heads * ((rows + 31) / 32);
    p.join = 1;
    p.splits = pieces_joined(n, (q.M + joined - 1) / joined, 32.0 * n * q.d * 4e-6);
  }
  p.row_tile = p.join ? 32 : 128;
  p.tiles = (int)((rows + p.row_tile - 1) / p.row_tile);
  const int stretches = dense_packed(q) ? 1 : q.group;   // a piece stays within the rows of a head
  wgs = kv_heads * stretches * ((q.M + 127) / 128);
  p.kv_join = 0;
  const double kv_mb = 2.0 * kv_heads * q.M * q.d * 4e-6;
  p.per_head = q.M > 64 || wgs >= enough ? cut(wgs, (rows + tile - 1) / tile, slots, 4 * product_us(q), kv_mb) : 1;
  const size_t tiles_lds = 2 * (2 * (size_t)joined * row_bytes + 1024);
  if ((wgs * p.per_head < enough || (q.M <= few && rows >= 4 * joined)) && tiles_lds + dkv_bias_lds(q, row_bytes > 256 ? 2 : 4) <= kLds) {
    p.kv_join = 1;
    p.per_head = pieces_joined(kv_heads * stretches * ((q.M + 31) / 32), (rows + joined - 1) / joined, kv_mb);
  }
  const int kt = p.kv_join ? 32 : 128;
  p.q_tile = p.kv_join ? joined : kv_tile;
  p.kv_tiles = (q.M + kt - 1) / kt;
  p.row_tiles = (int)((rows + p.q_tile - 1) / p.q_tile);
  p.kv_splits = p.per_head * stretches;
  const size_t padded = (size_t)(rows + 31) / 32 * 32;
  size_t off = 0;
  p.start = off; off += align_up(heads * padded * sizeof(float));
  p.delta = off; off += align_up(heads * padded * sizeof(float));
  p.top = off; off += align_up(heads * padded * sizeof(float));
  p.log_l = off; off += align_up(heads * padded * sizeof(float));
  p.dq_part = off; off += p.splits > 1 ? align_up((size_t)heads * p.tiles * p.splits * p.row_tile * q.d * sizeof(float)) : 0;
  p.k_part = off; off += p.splits > 1 && !f32 ? align_up((size_t)heads * p.tiles * p.splits * p.row_tile * q.d * 2) : 0;
  p.r_part = off; off += p.splits > 1 ? align_up((size_t)heads * p.tiles * p.splits * p.row_tile * sizeof(float)) : 0;
  p.dkv_part = off; off += p.kv_splits > 1 ? align_up(2 * (size_t)p.kv_splits * kv_heads * q.M * q.d * sizeof(float)) : 0;
  p.bias_part = off; off += q.bias ? align_up((size_t)kv_heads * p.kv_tiles * p.kv_splits * q.buckets * sizeof(float)) : 0;
  p.total = off;
  return p;
}

template <class T, int D, int NW, int JW, int MODE>
hipError_t run_dq(const DenseGeo& q, const BwdPlan& p, const dense::BwdArgs& a, hipStream_t s) {
  const size_t lds = MODE == dense::BIAS ? dense::bias_entries(q.rule.cut) * sizeof(float) : 0;
  dense::dense_dq_kernel<T, D, NW, JW, MODE><<<grid_of(a.items), 64 * NW, lds, s>>>(q, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const long long rows = (long long)q.B * dense_heads(q) * a.rows;
  constexpr int R = 256 / (D / 4);
  dense::dense_sum_dq_kernel<T, D, MODE><<<grid_of((rows + R - 1) / R), 256, 0, s>>>(q, a, 32 * (NW / JW));
  return hipGetLastError();
}

template <class T, int D, int NW, int JW, int MODE>
hipError_t run_dkv(const DenseGeo& q, const BwdPlan& p, const dense::BwdArgs& a, hipStream_t s) {
  dense::dense_dkv_kernel<T, D, NW, JW, MODE><<<grid_of(a.items), 64 * NW, dkv_bias_lds(q, NW), s>>>(q, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (MODE == dense::BIAS) {
    dense::dense_sum_bias_kernel<T><<<grid_of(q.H), 256, 0, s>>>(q, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (p.kv_splits == 1) return e;
  constexpr int R = 256 / (D / 4);
  dense::dense_sum_dkv_kernel<T, D><<<grid_of((2LL * q.B * q.Hk * q.M + R - 1) / R), 256, 0, s>>>(q, a);
  return hipGetLastError();
}

template <class T, int D, int MODE>
hipError_t run_bwd(const DenseGeo& q, const BwdPlan& p, dense::BwdArgs a, hipStream_t s) {
  constexpr int J = dense::kJoin<T, D>;
  a.tiles = p.tiles; a.splits = p.splits;
  a.items = (long long)q.B * dense_heads(q) * p.tiles * p.splits;
  hipError_t e = p.join ? run_dq<T, D, J, J, MODE>(q, p, a, s) : run_dq<T, D, 4, 1, MODE>(q, p, a, s);
  if (e != hipSuccess) return e;
  a.tiles = p.kv_tiles; a.splits = p.kv_splits; a.per_head = p.per_head; a.row_tiles = p.row_tiles;
  a.items = (long long)q.B * q.Hk * p.kv_tiles * p.kv_splits;
  return p.kv_join ? run_dkv<T, D, J, J, MODE>(q, p, a, s) : run_dkv<T, D, 4, 1, MODE>(q, p, a, s);
}

}  // namespace

size_t dense_bwd_workspace(const DenseGeo& q) { return plan_bwd(q).total; }

hipError_t launch_dense_bwd(const DenseGeo& q, const void* Q, const void* K, const void* V, const void* table, const void* O,
                            const float* lse, const void* dO, void* dQ, void* dK, void* dV, void* dtable, void* ws, hipStream_t s) {
  const BwdPlan p = plan_bwd(q);
  dense::BwdArgs a;
  a.Q = (const unsigned char*)Q; a.K = (const unsigned char*)K; a.V = (const unsigned char*)V;
  a.O = (const unsigned char*)O; a.dO = (const unsigned char*)dO;
  a.table = table; a.lse = lse;
  a.dQ = (unsigned char*)dQ; a.dK = (unsigned char*)dK; a.dV = (unsigned char*)dV; a.dtable = dtable;
  char* base = (char*)ws;
  a.start = (float*)(base + p.start); a.delta = (float*)(base + p.delta);
  a.top = (float*)(base + p.top); a.log_l = (float*)(base + p.log_l);
  a.dq_part = (float*)(base + p.dq_part); a.r_part = (float*)(base + p.r_part); a.dkv_part = (float*)(base + p.dkv_part);
  a.bias_part = (float*)(base + p.bias_part);
  a.k_part = (unsigned char*)(base + p.k_part);
  a.rows = dense_rows(q);
  a.padded = (a.rows + 31) / 32 * 32;
  a.tiles = a.splits = a.per_head = a.row_tiles = 0;
  a.items = 0;
  auto pick = [&](auto t, auto d) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value;
    if (q.bias) return run_bwd<T, D, dense::BIAS>(q, p, a, s);
    return dense_packed(q) ? run_bwd<T, D, dense::PACKED>(q, p, a, s) : run_bwd<T, D, dense::PLAIN>(q, p, a, s);
  };
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  if (q.dtype == DA_BF16) return q.d == 128 ? pick((__bf16)0.f, d128) : pick((__bf16)0.f, d64);
  return q.d == 128 ? pick(0.f, d128) : pick(0.f, d64);
}

}  // namespace da
