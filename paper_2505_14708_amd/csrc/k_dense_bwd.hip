// Dense attention of N queries to M keys, backward.
//
// With x = scale q.k + bias, p = exp(x - lse), delta_i = dO_i . O_i and ds = p (dO.v - delta):
//     dQ = scale ds K      dK = scale ds^T Q      dV = p^T dO      dtable[c] = sum of ds over the pairs whose bucket is c
// Two kernels, each of which makes p and dO V^T anew (seven products of N x M x d instead of five, but no sums shared between
// workgroups: no atomics, the same bits every time, and the sums stay in registers):
//   dense_dq_kernel   32 queries a wave on the lane axis, tiles of K and V pass by; also delta, and the sums for dtable
//   dense_dkv_kernel  32 keys a wave on the lane axis, tiles of Q and dO pass by, with lse and delta of their rows
// Where one side is short the other is cut and the pieces' sums are put together by a third launch, in a fixed order.
#include "attn_tiles.h"

namespace da {
namespace dense {

struct BwdArgs {
  const unsigned char *Q, *K, *V, *O, *dO;
  const void* table;
  const float* lse;
  unsigned char *dQ, *dK, *dV;
  void* dtable;
  float *lse2, *delta;             // [heads][padded rows]: lse log2(e) (+inf where a row has nothing to attend or is padding), delta
  float *dq_part, *dkv_part;       // sums of pieces
  float* bias_part;                // [work item][buckets]
  long long rows, padded;          // rows of a head as the kernels see them, and rounded up to 32
  long long items;                 // work items of the launch
  int tiles, splits;               // dq: tiles of queries, pieces of the keys; dkv: tiles of keys, pieces of the queries
  int row_tiles, per_head;         // dkv: tiles of queries of a head, pieces of a head
};

constexpr int kScratch = 36;       // row stride, in words, of the square that a wave's ds goes through for its diagonals

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

template <class T, int D, int NQ, int NW, bool BIAS>
__global__ __launch_bounds__(64 * NW, NQ == 1 && NW > 1 ? 2 : 1) void dense_dq_kernel(DenseGeo q, BwdArgs g) {
  constexpr int KB = kKeys<T, D>, RB = kRowBytes<T, D>, TILE = KB * RB, RT = 32 * NQ * NW;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[4 * TILE];
  extern __shared__ __attribute__((aligned(16))) float more[];       // bias row; then per wave its diagonals and its square
  const long long id = blockIdx.y * (long long)gridDim.x + blockIdx.x;
  if (id >= g.items) return;
  const long long item = xcd_order(id, g.items);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hi = lane >> 5;
  const int split = (int)(item % g.splits);
  const long long bht = item / g.splits;
  const int tile = (int)(bht % g.tiles);
  const long long bh = bht / g.tiles;
  const int heads = BIAS ? q.H : q.Hk;
  const int b = (int)(bh / heads), hd = (int)(bh - (long long)b * heads), hk = BIAS ? hd / q.group : hd;
  const int len = q.kv_len ? min(max(q.kv_len[b], 0), q.M) : q.M;
  const int first_row = tile * RT + wave * (32 * NQ), last_row = (int)g.rows - 1;
  const int n_tiles = (len + KB - 1) / KB, each = (n_tiles + g.splits - 1) / g.splits;
  const int t0 = min(split * each, n_tiles), t1 = min(t0 + each, n_tiles);
  const long long ks = q.k.sn * (long long)sizeof(T), vs = q.v.sn * (long long)sizeof(T);
  const unsigned char* kb = g.K + (b * q.k.sb + hk * q.k.sh) * (long long)sizeof(T);
  const unsigned char* vb = g.V + (b * q.v.sb + hk * q.v.sh) * (long long)sizeof(T);
  const unsigned lds = (unsigned)(uintptr_t)(lds_f32*)tiles;
  if (t0 < t1) {
    load_tile<T, D, KB, NW>(kb, ks, t0 * KB, len - 1, lds, wave, lane);
    load_tile<T, D, KB, NW>(vb, vs, t0 * KB, len - 1, lds + TILE, wave, lane);
  }
  const int n_bias = BIAS ? (bias_entries(q.rule.cut) + 3) & ~3 : 0;
  float* diag = more + n_bias + wave * (n_bias + 32 * kScratch);
  if constexpr (BIAS) {
    fill_bias<T>(more, q.rule, (const T*)g.table, q.H, hd, threadIdx.x, 64 * NW);
    for (int i = lane; i < n_bias; i += 64) diag[i] = 0.f;
  }

  Own<T, D> own[NQ], grad[NQ];
  f32x16 z[NQ][D / 32];
  float lse2[NQ], delta[NQ];
#pragma unroll
  for (int h = 0; h < NQ; ++h) {
    const int rr = first_row + 32 * h + (lane & 31), rc = min(rr, last_row);
    own[h].load(g.Q + query_offset<BIAS>(q, q.q, b, hd, rc) * (long long)sizeof(T), hi);
    grad[h].load(g.dO + query_offset<BIAS>(q, q.dout, b, hd, rc) * (long long)sizeof(T), hi);
    Own<T, D> out;
    out.load(g.O + query_offset<BIAS>(q, q.o, b, hd, rc) * (long long)sizeof(T), hi);
    float s = 0.f;
#pragma unroll
    for (int t = 0; t < Own<T, D>::N; ++t) s = dot_piece<T>(grad[h].x[t], out.x[t], s);
    delta[h] = rr <= last_row ? sum_across_halves(s) : 0.f;
    const float l = g.lse[bh * g.rows + rc];
    lse2[h] = rr <= last_row && l != -INFINITY ? l * kLog2e : INFINITY;
    if (split == 0 && hi == 0 && rr < g.padded) {
      g.lse2[bh * g.padded + rr] = lse2[h];
      g.delta[bh * g.padded + rr] = delta[h];
    }
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) z[h][dt] = zero16();
  }
  const unsigned s_lane = scores_lane<T, D>(lane), m_lane = mix_lane<T, D>(lane);
  const unsigned bias_lds = BIAS ? (unsigned)(uintptr_t)(lds_f32*)more : 0u;
  float far_sum[2] = {0.f, 0.f};

  for (int t = t0; t < t1; ++t) {
    const unsigned buf = lds + ((t - t0) & 1) * (2 * TILE);
    wait_loads();
    tile_barrier();
    if (t + 1 < t1) {
      const unsigned next = lds + ((t + 1 - t0) & 1) * (2 * TILE);
      load_tile<T, D, KB, NW>(kb, ks, (t + 1) * KB, len - 1, next, wave, lane);
      load_tile<T, D, KB, NW>(vb, vs, (t + 1) * KB, len - 1, next + TILE, wave, lane);
    }
    if (NW > 1 && first_row > last_row) continue;
#pragma unroll
    for (int sub = 0; sub < KB / 32; ++sub) {
      const int key0 = t * KB + 32 * sub;
      if (key0 >= len) break;
      f32x16 s[NQ], dp[NQ];
      scores<T, D, NQ>(buf + sub * 32 * RB + s_lane, own, s);
      scores<T, D, NQ>(buf + TILE + sub * 32 * RB + s_lane, grad, dp);
      const int left = len - key0 - 8 * hi;
#pragma unroll
      for (int h = 0; h < NQ; ++h) {
        const int low = BIAS ? key0 - (first_row + 32 * h) - q.q_pos : 0;
        const bool is_far = BIAS && (low - 31 >= q.rule.cut || low + 31 <= -q.rule.cut);
        if constexpr (BIAS) {
          if (is_far) {
            const float far = more[low > 0 ? 2 * (q.rule.cut + kBiasPad) : 0] - lse2[h];
#pragma unroll
            for (int a = 0; a < 16; ++a) s[h][a] = exp2_fast(__builtin_fmaf(s[h][a], q.c2, far));
          } else {
            f32x16 bs;
            read_bias<1>(bias_lds + 4 * (low + 8 * hi - (lane & 31) + q.rule.cut + kBiasPad), bs);
#pragma unroll
            for (int a = 0; a < 16; ++a) s[h][a] = exp2_fast(__builtin_fmaf(s[h][a], q.c2, bs[a]) - lse2[h]);
          }
        } else {
#pragma unroll
          for (int a = 0; a < 16; ++a) s[h][a] = exp2_fast(__builtin_fmaf(s[h][a], q.c2, -lse2[h]));
        }
        if (key0 + 32 > len) {
#pragma unroll
          for (int a = 0; a < 16; ++a) s[h][a] = 16 * (a >> 3) + (a & 7) < left ? s[h][a] : 0.f;
        }
#pragma unroll
        for (int a = 0; a < 16; ++a) s[h][a] *= dp[h][a] - delta[h];
        if constexpr (BIAS) {
          if (is_far) {
            float x = 0.f;
#pragma unroll
            for (int a = 0; a < 16; ++a) x += s[h][a];
            far_sum[0] += low > 0 ? 0.f : x;
            far_sum[1] += low > 0 ? x : 0.f;
          } else {
            // Diagonals of the square (query n, key m; r = low + m - n): by way of LDS lane c reads the keys (n + c) mod 32 of half
            // the queries, whose sum before the wrap belongs to r = low + c and behind it to low + c - 32.
            float* sq = diag + n_bias;
            f32x4* row = (f32x4*)(sq + (lane & 31) * kScratch + 8 * hi);
            row[0] = f32x4{s[h][0], s[h][1], s[h][2], s[h][3]};
            row[1] = f32x4{s[h][4], s[h][5], s[h][6], s[h][7]};
            row[4] = f32x4{s[h][8], s[h][9], s[h][10], s[h][11]};
            row[5] = f32x4{s[h][12], s[h][13], s[h][14], s[h][15]};
            __builtin_amdgcn_wave_barrier();
            const int c = lane & 31;
            float straight = 0.f, wrapped = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int n = 2 * i + hi, m = n + c;
              const float x = sq[n * kScratch + (m & 31)];
              straight += m < 32 ? x : 0.f;
              wrapped += m < 32 ? 0.f : x;
            }
            const float d0 = sum_across_halves(straight), d1 = sum_across_halves(wrapped);
            const int at = low + (hi ? c - 32 : c) + q.rule.cut + kBiasPad;
            diag[at] += hi ? d1 : d0;
            __builtin_amdgcn_wave_barrier();
          }
        }
      }
      if constexpr (NQ == 1) {
        const Mixed<T> p[1] = {Mixed<T>(s[0])};
        mix<T, D, 1>(buf + sub * 32 * RB + m_lane, p, z);
      } else {
        const Mixed<T> p[2] = {Mixed<T>(s[0]), Mixed<T>(s[1])};
        mix<T, D, 2>(buf + sub * 32 * RB + m_lane, p, z);
      }
    }
  }
#pragma unroll
  for (int h = 0; h < NQ; ++h) {
    const int rr = first_row + 32 * h + (lane & 31);
    const bool there = rr <= last_row;
    if (g.splits == 1)
      store_column<T, D>(g.dQ + query_offset<BIAS>(q, q.dq, b, hd, min(rr, last_row)) * (long long)sizeof(T), hi, z[h], q.scale, there);
    else
      store_column<float, D>((unsigned char*)(g.dq_part + (item * RT + wave * (32 * NQ) + 32 * h + (lane & 31)) * D), hi, z[h], q.scale, there);
  }
  if constexpr (BIAS) {
    // the waves' diagonals, added up bucket by bucket: eight lanes to a bucket
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x = far_sum[i];
#pragma unroll
      for (int w = 32; w >= 1; w >>= 1) x += __shfl_xor(x, w);
      if (lane == 0) diag[i ? 2 * (q.rule.cut + kBiasPad) : 0] += x;
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
          for (int w = 0; w < NW; ++w) x += more[n_bias + w * (n_bias + 32 * kScratch) + i];
      }
#pragma unroll
      for (int w = 4; w >= 1; w >>= 1) x += __shfl_xor(x, w);
      if (c < q.buckets && (threadIdx.x & 7) == 0) g.bias_part[item * q.buckets + c] = x;
    }
  }
}

template <class T, int D, int NW, bool BIAS>
__global__ __launch_bounds__(64 * NW, NW == 1 ? 1 : 2) void dense_dkv_kernel(DenseGeo q, BwdArgs g) {
  constexpr int QB = kKeys<T, D>, RB = kRowBytes<T, D>, TILE = QB * RB, STAGE = 2 * TILE + 1024, KT = 32 * NW;
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[2 * STAGE];  // twice: Q, dO, lse2 and delta of their rows
  extern __shared__ __attribute__((aligned(16))) float bias_row[];
  const long long id = blockIdx.y * (long long)gridDim.x + blockIdx.x;
  if (id >= g.items) return;
  const long long item = xcd_order(id, g.items);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hi = lane >> 5;
  // the tiles of keys of one piece of the queries are neighbours: they read the same rows
  const int tile = (int)(item % g.tiles);
  const long long rest = item / g.tiles;
  const int split = (int)(rest % g.splits);
  const long long bh = rest / g.splits;
  const int b = (int)(bh / q.Hk), hk = (int)(bh - (long long)b * q.Hk);
  const int len = q.kv_len ? min(max(q.kv_len[b], 0), q.M) : q.M;
  const int key0 = tile * KT + wave * 32, key = key0 + (lane & 31);
  const int hd = BIAS ? hk * q.group + split / g.per_head : hk, piece = BIAS ? split % g.per_head : split;
  const long long stat = ((long long)b * (BIAS ? q.H : q.Hk) + hd) * g.padded;
  const int each = (g.row_tiles + g.per_head - 1) / g.per_head;
  const int t0 = min(piece * each, g.row_tiles), t1 = tile * KT < len ? min(t0 + each, g.row_tiles) : t0;
  const int last_row = (int)g.rows - 1;
  const unsigned lds = (unsigned)(uintptr_t)(lds_f32*)tiles;

  // a tile of queries and of dO, and what goes with their rows
  auto load_rows = [&](int t, unsigned to) {
    const int first = t * QB, last = min(first + QB - 1, last_row);
    if (BIAS || q.group == 1 || first / q.N == last / q.N) {
      const int g0 = BIAS || q.group == 1 ? 0 : first / q.N, n0 = first - g0 * q.N, n1 = last - g0 * q.N;
      const int h0 = BIAS || q.group == 1 ? hd : hd * q.group + g0;
      load_tile<T, D, QB, NW>(g.Q + (b * q.q.sb + h0 * q.q.sh) * (long long)sizeof(T), q.q.sn * (long long)sizeof(T), n0, n1, to, wave, lane);
      load_tile<T, D, QB, NW>(g.dO + (b * q.dout.sb + h0 * q.dout.sh) * (long long)sizeof(T), q.dout.sn * (long long)sizeof(T), n0, n1,
                              to + TILE, wave, lane);
    } else {
      constexpr int CPR = RB / 16, RPS = 64 / CPR;
#pragma unroll
      for (int k = 0; k < QB / RPS / NW; ++k) {
        const int it = k * NW + wave, row = it * RPS + lane / CPR, rr = min(first + row, last);
        const unsigned p = ((lane % CPR) ^ swizzle<T, D>(row)) << 4;
        dma16(g.Q + query_offset<BIAS>(q, q.q, b, hd, rr) * (long long)sizeof(T) + p, to + it * 1024);
        dma16(g.dO + query_offset<BIAS>(q, q.dout, b, hd, rr) * (long long)sizeof(T) + p, to + TILE + it * 1024);
      }
    }
    const long long rr = stat + min((long long)first + lane, g.padded - 1);
    if (wave == 0) dma4(g.lse2 + rr, to + 2 * TILE);
    if (wave == (NW > 1 ? 1 : 0)) dma4(g.delta + rr, to + 2 * TILE + 256);
  };
  if (t0 < t1) load_rows(t0, lds);
  if constexpr (BIAS) fill_bias<T>(bias_row, q.rule, (const T*)g.table, q.H, hd, threadIdx.x, 64 * NW);

  Own<T, D> own_k[1], own_v[1];
  f32x16 zk[1][D / 32], zv[1][D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) zk[0][dt] = zv[0][dt] = zero16();
  if (t0 < t1) {
    const long long kc = min(key, len - 1);
    own_k[0].load(g.K + (b * q.k.sb + hk * q.k.sh + kc * q.k.sn) * (long long)sizeof(T), hi);
    own_v[0].load(g.V + (b * q.v.sb + hk * q.v.sh + kc * q.v.sn) * (long long)sizeof(T), hi);
  }
  const unsigned s_lane = scores_lane<T, D>(lane), m_lane = mix_lane<T, D>(lane);
  const unsigned bias_lds = BIAS ? (unsigned)(uintptr_t)(lds_f32*)bias_row : 0u;

  for (int t = t0; t < t1; ++t) {
    const unsigned buf = lds + ((t - t0) & 1) * STAGE;
    wait_loads();
    tile_barrier();
    if (t + 1 < t1) load_rows(t + 1, lds + ((t + 1 - t0) & 1) * STAGE);
    if (NW > 1 && key0 >= len) continue;
#pragma unroll
    for (int sub = 0; sub < QB / 32; ++sub) {
      const int row0 = t * QB + 32 * sub;
      if (row0 > last_row) break;
      f32x16 s[1], dp[1];
      scores<T, D, 1>(buf + sub * 32 * RB + s_lane, own_k, s);
      scores<T, D, 1>(buf + TILE + sub * 32 * RB + s_lane, own_v, dp);
      f32x4 l[4], dl[4];           // of the rows of registers 4i .. 4i + 3
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned at = buf + 2 * TILE + 4 * (32 * sub + 16 * (i >> 1) + 8 * hi + 4 * (i & 1));
        l[i] = *(lds_f32x4*)(uintptr_t)at;
        dl[i] = *(lds_f32x4*)(uintptr_t)(at + 256);
      }
      if constexpr (BIAS) {
        const int low = key0 - row0 - q.q_pos;       // r of key 0 and query 0 of the square
        if (low - 31 >= q.rule.cut || low + 31 <= -q.rule.cut) {
          const float far = bias_row[low > 0 ? 2 * (q.rule.cut + kBiasPad) : 0];
#pragma unroll
          for (int a = 0; a < 16; ++a) s[0][a] = __builtin_fmaf(s[0][a], q.c2, far);
        } else {
          f32x16 bs;
          read_bias<-1>(bias_lds + 4 * (low + (lane & 31) - 8 * hi + q.rule.cut + kBiasPad), bs);
#pragma unroll
          for (int a = 0; a < 16; ++a) s[0][a] = __builtin_fmaf(s[0][a], q.c2, bs[a]);
        }
#pragma unroll
        for (int a = 0; a < 16; ++a) s[0][a] = exp2_fast(s[0][a] - l[a >> 2][a & 3]);
      } else {
#pragma unroll
        for (int a = 0; a < 16; ++a) s[0][a] = exp2_fast(__builtin_fmaf(s[0][a], q.c2, -l[a >> 2][a & 3]));
      }
      const Mixed<T> p[1] = {Mixed<T>(s[0])};
#pragma unroll
      for (int a = 0; a < 16; ++a) dp[0][a] = s[0][a] * (dp[0][a] - dl[a >> 2][a & 3]);
      const Mixed<T> ds[1] = {Mixed<T>(dp[0])};
      mix<T, D, 1>(buf + TILE + sub * 32 * RB + m_lane, p, zv);
      mix<T, D, 1>(buf + sub * 32 * RB + m_lane, ds, zk);
    }
  }
  if (g.splits == 1) {
    if (key >= len) {
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) zk[0][dt] = zv[0][dt] = zero16();
    }
    const long long kc = min(key, q.M - 1);
    store_column<T, D>(g.dK + (b * q.dk.sb + hk * q.dk.sh + kc * q.dk.sn) * (long long)sizeof(T), hi, zk[0], q.scale, key < q.M);
    store_column<T, D>(g.dV + (b * q.dv.sb + hk * q.dv.sh + kc * q.dv.sn) * (long long)sizeof(T), hi, zv[0], 1.f, key < q.M);
  } else {
    const long long bhs = (long long)q.B * q.Hk;
    float* at = g.dkv_part + ((split * bhs + bh) * q.M + min(key, q.M - 1)) * D;
    store_column<float, D>((unsigned char*)at, hi, zk[0], q.scale, key < len);
    store_column<float, D>((unsigned char*)(at + g.splits * bhs * q.M * D), hi, zv[0], 1.f, key < len);
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

template <class T, int D, bool BIAS>
__global__ __launch_bounds__(256) void dense_sum_dq_kernel(DenseGeo q, BwdArgs g, int RT) {
  constexpr int P = D / 4;
  const long long row = (blockIdx.y * (long long)gridDim.x + blockIdx.x) * (256 / P) + threadIdx.x / P;
  const int heads = BIAS ? q.H : q.Hk;
  if (row >= (long long)q.B * heads * g.rows) return;
  const long long bh = row / g.rows;
  const int rr = (int)(row - bh * g.rows), b = (int)(bh / heads), hd = (int)(bh - (long long)b * heads);
  const int tile = rr / RT;
  const long long first = ((bh * g.tiles + tile) * g.splits) * RT + (rr - tile * RT);
  sum_pieces<T, D>(g.dq_part + first * D, (long long)RT * D, g.splits, (T*)g.dQ + query_offset<BIAS>(q, q.dq, b, hd, rr), threadIdx.x % P);
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

// dtable[c][h]: the work items of head h in order, a few of their stretches at a time
template <class T>
__global__ __launch_bounds__(256) void dense_sum_bias_kernel(DenseGeo q, BwdArgs g) {
  __shared__ float sums[256];
  const int h = blockIdx.x, c = threadIdx.x % q.buckets, slice = threadIdx.x / q.buckets, slices = 256 / q.buckets;
  const long long run = (long long)g.tiles * g.splits, n = run * q.B;
  float x = 0.f;
  if (slice < slices) {
    const long long each = (n + slices - 1) / slices, i0 = slice * each, i1 = min(i0 + each, n);
#pragma unroll 8
    for (long long i = i0; i < i1; ++i) {
      const long long b = i / run;
      x += g.bias_part[((b * q.H + h) * run + (i - b * run)) * q.buckets + c];
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

struct BwdPlan {
  int waves, sets, tiles, splits;                    // dq
  int kv_waves, kv_tiles, kv_splits, per_head, row_tiles;  // dkv
  size_t lse2, delta, dq_part, dkv_part, bias_part, total;
};

inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

BwdPlan plan_bwd(const DenseGeo& q) {
  BwdPlan p;
  const long long rows = dense_rows(q), heads = (long long)q.B * dense_heads(q), kv_heads = (long long)q.B * q.Hk;
  const int tile = q.dtype == DA_F32 && q.d == 128 ? 32 : 64;
  p.waves = rows <= 64 ? 1 : 4;
  p.sets = 1;
  const int rt = 32 * p.sets * p.waves;
  p.tiles = (int)((rows + rt - 1) / rt);
  const long long want = 2 * kCUs, key_tiles = (q.M + tile - 1) / tile;
  auto pieces = [&](long long wgs, long long units) {
    long long n = wgs >= want ? 1 : (want + wgs - 1) / wgs;
    n = n > units / 4 ? units / 4 : n;
    return (int)(n < 1 ? 1 : n);
  };
  p.splits = pieces(heads * p.tiles, key_tiles);
  p.kv_waves = q.M <= 32 ? 1 : 4;
  const int kt = 32 * p.kv_waves;
  p.kv_tiles = (q.M + kt - 1) / kt;
  p.row_tiles = (int)((rows + tile - 1) / tile);
  const int stretches = q.bias ? q.group : 1;        // with a bias a piece stays within a head
  p.per_head = pieces(kv_heads * p.kv_tiles * stretches, p.row_tiles);
  p.kv_splits = p.per_head * stretches;
  const size_t padded = (size_t)(rows + 31) / 32 * 32;
  size_t off = 0;
  p.lse2 = off; off += align_up(heads * padded * sizeof(float));
  p.delta = off; off += align_up(heads * padded * sizeof(float));
  p.dq_part = off; off += p.splits > 1 ? align_up((size_t)heads * p.tiles * p.splits * rt * q.d * sizeof(float)) : 0;
  p.dkv_part = off; off += p.kv_splits > 1 ? align_up(2 * (size_t)p.kv_splits * kv_heads * q.M * q.d * sizeof(float)) : 0;
  p.bias_part = off; off += q.bias ? align_up((size_t)heads * p.tiles * p.splits * q.buckets * sizeof(float)) : 0;
  p.total = off;
  return p;
}

template <class T, int D, int NW, bool BIAS>
hipError_t run_dq(const DenseGeo& q, const BwdPlan& p, const dense::BwdArgs& a, hipStream_t s) {
  const size_t n = (dense::bias_entries(q.rule.cut) + 3) & ~3;
  const size_t lds = BIAS ? (n + NW * (n + 32 * dense::kScratch)) * sizeof(float) : 0;
  dense::dense_dq_kernel<T, D, 1, NW, BIAS><<<grid_of(a.items), 64 * NW, lds, s>>>(q, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const long long rows = (long long)q.B * dense_heads(q) * a.rows;
  constexpr int R = 256 / (D / 4);
  dense::dense_sum_dq_kernel<T, D, BIAS><<<grid_of((rows + R - 1) / R), 256, 0, s>>>(q, a, 32 * NW);
  return hipGetLastError();
}

template <class T, int D, int NW, bool BIAS>
hipError_t run_dkv(const DenseGeo& q, const BwdPlan& p, const dense::BwdArgs& a, hipStream_t s) {
  const size_t lds = BIAS ? dense::bias_entries(q.rule.cut) * sizeof(float) : 0;
  dense::dense_dkv_kernel<T, D, NW, BIAS><<<grid_of(a.items), 64 * NW, lds, s>>>(q, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.kv_splits == 1) return e;
  constexpr int R = 256 / (D / 4);
  dense::dense_sum_dkv_kernel<T, D><<<grid_of((2LL * q.B * q.Hk * q.M + R - 1) / R), 256, 0, s>>>(q, a);
  return hipGetLastError();
}

template <class T, int D, bool BIAS>
hipError_t run_bwd(const DenseGeo& q, const BwdPlan& p, dense::BwdArgs a, hipStream_t s) {
  a.tiles = p.tiles; a.splits = p.splits;
  a.items = (long long)q.B * dense_heads(q) * p.tiles * p.splits;
  hipError_t e = p.waves == 1 ? run_dq<T, D, 1, BIAS>(q, p, a, s) : run_dq<T, D, 4, BIAS>(q, p, a, s);
  if (e != hipSuccess) return e;
  if (BIAS) {
    dense::dense_sum_bias_kernel<T><<<q.H, 256, 0, s>>>(q, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  a.tiles = p.kv_tiles; a.splits = p.kv_splits; a.per_head = p.per_head; a.row_tiles = p.row_tiles;
  a.items = (long long)q.B * q.Hk * p.kv_tiles * p.kv_splits;
  return p.kv_waves == 1 ? run_dkv<T, D, 1, BIAS>(q, p, a, s) : run_dkv<T, D, 4, BIAS>(q, p, a, s);
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
  a.lse2 = (float*)(base + p.lse2); a.delta = (float*)(base + p.delta);
  a.dq_part = (float*)(base + p.dq_part); a.dkv_part = (float*)(base + p.dkv_part);
  a.bias_part = (float*)(base + p.bias_part);
  a.rows = dense_rows(q);
  a.padded = (a.rows + 31) / 32 * 32;
  const bool bias = q.bias != 0;
  if (q.dtype == DA_BF16) {
    if (q.d == 128) return bias ? run_bwd<__bf16, 128, true>(q, p, a, s) : run_bwd<__bf16, 128, false>(q, p, a, s);
    return bias ? run_bwd<__bf16, 64, true>(q, p, a, s) : run_bwd<__bf16, 64, false>(q, p, a, s);
  }
  if (q.d == 128) return bias ? run_bwd<float, 128, true>(q, p, a, s) : run_bwd<float, 128, false>(q, p, a, s);
  return bias ? run_bwd<float, 64, true>(q, p, a, s) : run_bwd<float, 64, false>(q, p, a, s);
}

}  // namespace da
