// Dense attention of N queries to M keys, forward: softmax(scale Q K^T + bias) V in one pass over the keys.
//
// Per set of 32 queries and 32 keys a wave computes S^T = K Q^T, the running maximum and sum of the softmax, and O^T += V^T P^T, with the
// two products of attn_tiles.h; the queries lie on the lane axis.  Tiles of K and V come through LDS, twice buffered and shared by the waves
// of the workgroup.
//
// Bounds: 40 heads of 75600 by 512, 128 channels, bf16: 866 us, 0.92 PFLOP/s (a large library product reaches 1.23 on this card); in a counted run of 980 us the
// matrix pipe is busy 42 % and the vector pipe 50 % of the cycles, with little of it at the same time, LDS 10 %.  One query of 32768 keys at 32 heads: K and V at
// 4.5 TB/s.
#include <type_traits>
#include "attn_tiles.h"

namespace da {
namespace dense {

constexpr float kLazy = 8.0f;          // the reference of the exponentials moves when a score exceeds it by more than this many powers of two

struct FwdArgs {
  const unsigned char *Q, *K, *V;
  const void* table;
  unsigned char* O;
  float* lse;
  float* part;           // splits > 1: [work item][rows of the tile][D] sums of P V, then [work item][rows of the tile][2] top (ref_of) and sum of P
  int tiles, splits;
  long long rows, items; // queries of a head, work items
};

// natural log of a sum l against `top`
template <int MODE> __device__ __forceinline__ float log_sum(const DenseGeo& q, float top, float l) {
  constexpr float kLn2Lo = 0.6931471805599453 - (double)kLn2;
  const Ref r = ref_of<MODE>(q, top);
  return l > 0.f ? __builtin_fmaf(r.score, q.scale, __builtin_fmaf(r.x, kLn2, __builtin_fmaf(r.x, kLn2Lo, logf(l)))) : -INFINITY;
}

// NW waves, JW of which share their columns (1, or all)
template <class T, int D, int NQ, int NW, int JW, int MODE>
__global__ __launch_bounds__(64 * NW, JW > 1 ? 1 : 2) void dense_fwd_kernel(DenseGeo q, FwdArgs g) {
  static_assert(JW == 1 || (JW == NW && NQ == 1), "one set of columns to join");
  constexpr int KB = kTileRows<T, D, JW>, RB = kRowBytes<T, D>, TILE = KB * RB, RT = 32 * NQ * (NW / JW);
  __shared__ __attribute__((aligned(1024))) unsigned char tiles[4 * TILE];   // K, V, K, V
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
  const int first_row = tile * RT + (JW > 1 ? 0 : wave * (32 * NQ)), last_row = (int)g.rows - 1;

  // this split's keys
  const int n_tiles = (len + KB - 1) / KB, each = (n_tiles + g.splits - 1) / g.splits;
  const int t0 = min(split * each, n_tiles), t1 = min(t0 + each, n_tiles);
  const long long ks = q.k.sn * (long long)sizeof(T), vs = q.v.sn * (long long)sizeof(T);
  const unsigned char* kb = g.K + (b * q.k.sb + hk * q.k.sh) * (long long)sizeof(T);
  const unsigned char* vb = g.V + (b * q.v.sb + hk * q.v.sh) * (long long)sizeof(T);
  const unsigned lds = (unsigned)(uintptr_t)(lds_f32*)tiles;
  if (t0 < t1) {
    load_tile<T, D, KB, NW>(kb, ks, t0 * KB, len - 1, lds, wave);
    load_tile<T, D, KB, NW>(vb, vs, t0 * KB, len - 1, lds + TILE, wave);
  }
  if constexpr (MODE == BIAS) fill_bias<T>(bias_row, q.rule, (const T*)g.table, q.H, hd, threadIdx.x, 64 * NW);

  Own<T, D> own[NQ];
  f32x16 z[NQ][D / 32];
  float ref[NQ], top[NQ], sum[NQ];                     // ref: Ref's x of top, with a bias the top itself
#pragma unroll
  for (int h = 0; h < NQ; ++h) {
    own[h].load(g.Q + query_offset<MODE>(q, q.q, b, hd, min(first_row + 32 * h + (lane & 31), last_row)) * (long long)sizeof(T), hi);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) z[h][dt] = zero16();
    // below every finite score, so that scores of minus infinity weigh nothing from the start
    ref[h] = top[h] = -FLT_MAX;
    sum[h] = 0.f;
  }
  const unsigned s_lane = scores_lane<T, D>(lane), m_lane = mix_lane<T, D>(lane);
  const unsigned bias_lds = MODE == BIAS ? (unsigned)(uintptr_t)(lds_f32*)bias_row : 0u;

  auto top_of = [&](int h) { return MODE == BIAS ? ref[h] : top[h]; };
  unsigned long long distant = 0;                      // lanes with a distant row

  for (int t = t0; t < t1; ++t) {
    const unsigned buf = lds + ((t - t0) & 1) * (2 * TILE);
    wait_loads();
    tile_barrier();
    if (t + 1 < t1) {
      const unsigned next = lds + ((t + 1 - t0) & 1) * (2 * TILE);
      load_tile<T, D, KB, NW>(kb, ks, (t + 1) * KB, len - 1, next, wave);
      load_tile<T, D, KB, NW>(vb, vs, (t + 1) * KB, len - 1, next + TILE, wave);
    }
    if (first_row > last_row) continue;                // (a wave of padding only helps to load)
#pragma unroll
    for (int i = 0; i < KB / 32 / JW; ++i) {
      const int sub = JW > 1 ? wave : i;
      const int key0 = t * KB + 32 * sub;
      if (key0 >= len) break;
      f32x16 s[NQ];
      scores<T, D, NQ>(buf + sub * 32 * RB + s_lane, own, s);
      float mx[NQ];
      bool moves = false;
      const int left = len - key0 - 8 * hi;
#pragma unroll
      for (int h = 0; h < NQ; ++h) {
        if constexpr (MODE == BIAS) {
          const int low = key0 - (first_row + 32 * h) - q.q_pos;          // r of key 0 and query 0 of the square
          if (low - 31 >= q.rule.cut || low + 31 <= -q.rule.cut) {
            const float far = bias_row[low > 0 ? 2 * (q.rule.cut + kBiasPad) : 0];
#pragma unroll
            for (int a = 0; a < 16; ++a) s[h][a] = biased<T>(q, s[h][a], far);
          } else {
            f32x16 bs;
            read_bias<1>(bias_lds + 4 * (low + 8 * hi - (lane & 31) + q.rule.cut + kBiasPad), bs);
#pragma unroll
            for (int a = 0; a < 16; ++a) s[h][a] = biased<T>(q, s[h][a], bs[a]);
          }
        }
        if (key0 + 32 > len) {
#pragma unroll
          for (int a = 0; a < 16; ++a) s[h][a] = 16 * (a >> 3) + (a & 7) < left ? s[h][a] : -INFINITY;
        }
        float m = s[h][0];
#pragma unroll
        for (int a = 1; a < 16; ++a) m = fmaxf(m, s[h][a]);
        m = max_across_halves(m);
        mx[h] = m;
        moves = moves || (MODE == BIAS ? m : m * q.c2) - ref[h] > kLazy;
      }
      if (__builtin_amdgcn_ballot_w64(moves) | distant) {     // (a distant row: its differences are taken in here)
        bool any = false;
        float score[NQ];
#pragma unroll
        for (int h = 0; h < NQ; ++h) {
          const float to = fmaxf(top_of(h), mx[h]), f = moved<MODE>(q, top_of(h), to);
          const Ref r = ref_of<MODE>(q, to);
          top[h] = to;
          ref[h] = r.x;
          any = any || is_distant<MODE>(q, to);
          sum[h] *= f;
          score[h] = r.score;
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int a = 0; a < 16; ++a) z[h][dt][a] *= f;
        }
        distant = __builtin_amdgcn_ballot_w64(any);
        if (distant) {
#pragma unroll
          for (int h = 0; h < NQ; ++h)
#pragma unroll
            for (int a = 0; a < 16; ++a) s[h][a] -= score[h];
        }
      }
#pragma unroll
      for (int h = 0; h < NQ; ++h) {
#pragma unroll
        for (int a = 0; a < 16; ++a) {
          s[h][a] = MODE == BIAS ? exp2_fast(s[h][a] - ref[h]) : power_of<T>(q, s[h][a], -ref[h]);
          sum[h] += s[h][a];
        }
      }
      if constexpr (NQ == 1) {
        const Mixed<T> p[1] = {Mixed<T>(s[0])};
        mix<T, D, 1>(buf + TILE + sub * 32 * RB + m_lane, p, z);
      } else {
        const Mixed<T> p[2] = {Mixed<T>(s[0]), Mixed<T>(s[1])};
        mix<T, D, 2>(buf + TILE + sub * 32 * RB + m_lane, p, z);
      }
    }
  }
  if constexpr (JW > 1) {
    // the waves' tops and sums, then their sums of P V against the largest top
    float* buf = (float*)tiles;
    f32x2* stat = (f32x2*)(buf + NW * 32 * (D + 4));
    const float own_sum = sum_across_halves(sum[0]);
    tile_barrier();
    if (hi == 0) stat[wave * 32 + lane] = f32x2{top_of(0), own_sum};
    tile_barrier();
    float most = -FLT_MAX;
#pragma unroll
    for (int w = 0; w < NW; ++w) most = fmaxf(most, stat[w * 32 + (lane & 31)][0]);
    join_waves<D, NW>(buf, wave, lane, z[0], moved<MODE>(q, top_of(0), most), [&](int row, int c, f32x4 (&x)[2]) {
      const int rr = first_row + row;
      if (rr > last_row) return;
      float t = -FLT_MAX, l = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) t = fmaxf(t, stat[w * 32 + row][0]);
#pragma unroll
      for (int w = 0; w < NW; ++w) l = __builtin_fmaf(stat[w * 32 + row][1], moved<MODE>(q, stat[w * 32 + row][0], t), l);
      if (g.splits == 1) {
        store8<T>(g.O + (query_offset<MODE>(q, q.o, b, hd, rr) + c) * (long long)sizeof(T), x, l > 0.f ? 1.f / l : 0.f);
        if (g.lse && c == 0) g.lse[bh * g.rows + rr] = log_sum<MODE>(q, t, l);
      } else {
        const long long at = item * RT + row;
        store8<float>((unsigned char*)(g.part + at * D + c), x, 1.f);
        if (c == 0) *(f32x2*)(g.part + g.items * RT * D + at * 2) = f32x2{t, l};
      }
    });
    return;
  }
#pragma unroll
  for (int h = 0; h < NQ; ++h) {
    const int rr = first_row + 32 * h + (lane & 31);
    const bool there = rr <= last_row;
    const float l = sum_across_halves(sum[h]);
    if (g.splits == 1) {
      const int rc = min(rr, last_row);
      store_column<T, D>(g.O + query_offset<MODE>(q, q.o, b, hd, rc) * (long long)sizeof(T), hi, z[h], l > 0.f ? 1.f / l : 0.f, there);
      if (g.lse && there && hi == 0) g.lse[bh * g.rows + rr] = log_sum<MODE>(q, top_of(h), l);
    } else {
      const long long at = item * RT + wave * (32 * NQ) + 32 * h + (lane & 31);
      store_column<float, D>((unsigned char*)(g.part + at * D), hi, z[h], 1.f, there);
      if (there && hi == 0) *(f32x2*)(g.part + g.items * RT * D + at * 2) = f32x2{top_of(h), l};
    }
  }
}

// The pieces of a row put together, in an order that depends on their number alone: W waves to a row, each with every W-th piece.
template <class T, int D, int W, int MODE>
__global__ __launch_bounds__(256) void dense_join_kernel(DenseGeo q, FwdArgs g, int RT) {
  __shared__ float sums[4][D];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, w = wave % W;
  const long long rows = (long long)q.B * heads_of<MODE>(q) * g.rows;
  const long long id = (blockIdx.y * (long long)gridDim.x + blockIdx.x) * (4 / W) + wave / W;
  const long long row = min(id, rows - 1);
  const int heads = heads_of<MODE>(q);
  const long long bh = row / g.rows;
  const int rr = (int)(row - bh * g.rows), b = (int)(bh / heads), hd = (int)(bh - (long long)b * heads);
  const int tile = rr / RT;
  const long long first = ((bh * g.tiles + tile) * g.splits) * RT + (rr - tile * RT);
  const float* stat = g.part + g.items * RT * D + first * 2;
  const float* part = g.part + first * D;
  float top = -FLT_MAX, l = 0.f;
  for (int s = lane; s < g.splits; s += 64) {
    const f32x2 x = *(const f32x2*)(stat + (long long)s * RT * 2);
    top = fmaxf(top, x[0]);            // (of a piece without keys: -FLT_MAX, with sums of 0)
  }
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
  for (int s = lane; s < g.splits; s += 64) {
    const f32x2 x = *(const f32x2*)(stat + (long long)s * RT * 2);
    l = __builtin_fmaf(x[1], moved<MODE>(q, x[0], top), l);
  }
#pragma unroll
  for (int i = 32; i >= 1; i >>= 1) l += __shfl_xor(l, i);
  constexpr int E = D / 64;
  float o[E] = {};
#pragma unroll 8
  for (int s = w; s < g.splits; s += W) {
    const f32x2 x = *(const f32x2*)(stat + (long long)s * RT * 2);
    const float f = moved<MODE>(q, x[0], top);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = __builtin_fmaf(part[(long long)s * RT * D + lane * E + e], f, o[e]);
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) sums[wave][lane * E + e] = o[e];
    __syncthreads();
    if (w == 0) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        for (int i = 1; i < W; ++i) o[e] += sums[wave + i][lane * E + e];
    }
  }
  if (w != 0 || id >= rows) return;
  T* out = (T*)g.O + query_offset<MODE>(q, q.o, b, hd, rr);
#pragma unroll
  for (int e = 0; e < E; ++e) out[lane * E + e] = (T)(l > 0.f ? o[e] / l : 0.f);
  if (g.lse && lane == 0) g.lse[row] = log_sum<MODE>(q, top, l);
}

}  // namespace dense

namespace {

template <class T, int D, int NQ, int NW, int JW, int MODE>
hipError_t run_fwd(const DenseGeo& q, const FwdPlan& p, dense::FwdArgs a, hipStream_t s) {
  const size_t lds = MODE == dense::BIAS ? dense::bias_entries(q.rule.cut) * sizeof(float) : 0;
  dense::dense_fwd_kernel<T, D, NQ, NW, JW, MODE><<<grid_of(a.items), 64 * NW, lds, s>>>(q, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const long long rows = (long long)q.B * dense_heads(q) * a.rows;
  const int rt = 32 * NQ * (NW / JW);
  // (a wave to a row needs thousands of rows to fill the card)
  if (rows <= 2048) dense::dense_join_kernel<T, D, 4, MODE><<<grid_of(rows), 256, 0, s>>>(q, a, rt);
  else dense::dense_join_kernel<T, D, 1, MODE><<<grid_of((rows + 3) / 4), 256, 0, s>>>(q, a, rt);
  return hipGetLastError();
}

template <class T, int D, int MODE>
hipError_t pick_fwd(const DenseGeo& q, const FwdPlan& p, const dense::FwdArgs& a, hipStream_t s) {
  constexpr int J = dense::kJoin<T, D>;
  if (p.join) return run_fwd<T, D, 1, J, J, MODE>(q, p, a, s);
  if constexpr (sizeof(T) == 2)
    if (p.sets == 2) return run_fwd<T, D, 2, 4, 1, MODE>(q, p, a, s);
  return run_fwd<T, D, 1, 4, 1, MODE>(q, p, a, s);
}

}  // namespace

// Workgroups of four waves with 64 queries each (bf16, where they fill the card: each operand from LDS feeds two products), with 32 each, or of
// waves that share 32 queries and take the keys in turn: where there are few workgroups, and, with at most 64 queries, where those that join fit the card at once or, with
// 64 channels, their tiles of 128 keys are several.  (192 heads of 16 queries by 2000 keys, bf16, 128 channels: joining 36 us, else 56, in two pieces 38; 960
// heads: 182 and 171; of 64 queries by 64 keys 46 and 17.  float32, 64 channels, 960 heads of 16 by 2000: 273 and 386, by 64 keys 27 and 22; bf16, 64 channels,
// 384 heads of 64 by 2000: 41 and 49, by 300 keys 13 and 11; 720 heads by 2000 91 and 71.)
FwdPlan plan_dense_fwd(const DenseGeo& q) {
  FwdPlan p;
  const long long rows = dense_rows(q), heads = (long long)q.B * dense_heads(q);
  const bool f32 = q.dtype == DA_F32, wide = q.d * (f32 ? 4 : 2) > 256;
  const long long wgs = heads * ((rows + 127) / 128), units = (q.M + (wide ? 31 : 63)) / (wide ? 32 : 64);
  const long long small = heads * ((rows + 31) / 32);
  const int enough = kCUs / 4 * 3, slots = q.d * (f32 ? 4 : 2) == 128 ? 2 * kCUs : kCUs;     // (of workgroups that join)
  p.join = 0; p.sets = 1; p.splits = 1;
  if (!f32 && rows > 128 && heads * ((rows + 255) / 256) >= kCUs / 2 * 3) {   // three quarters of the places, two to a CU
    p.sets = 2;
  } else if (wgs < enough || rows <= 64) {
    p.splits = rows > 64 || wgs >= enough ? cut(wgs, units, 2 * kCUs, 2 * product_us(q), 128.0 * wgs * q.d * 4e-6) : 1;
    const bool many_keys = q.d == 64 && (f32 ? q.M >= 256 : rows <= 32 ? q.M >= 512 : q.M >= 1000 && small <= 2 * slots);
    if (wgs * p.splits < enough || (rows <= 64 && (small <= slots || many_keys))) {
      p.join = 1;
      const int n = wide ? 64 : 128;
      const long long tiles = (q.M + n - 1) / n;
      long long s = slots / small;
      if (s > tiles / 2) s = tiles / 2;
      p.splits = s < 1 ? 1 : (int)s;
    }
  }
  p.row_tile = p.join ? 32 : 128 * p.sets;
  p.tiles = (int)((rows + p.row_tile - 1) / p.row_tile);
  return p;
}

size_t dense_fwd_workspace(const DenseGeo& q) {
  const FwdPlan p = plan_dense_fwd(q);
  if (p.splits == 1) return 0;
  return (size_t)q.B * dense_heads(q) * p.tiles * p.splits * p.row_tile * (q.d + 2) * sizeof(float);
}

hipError_t launch_dense_fwd(const DenseGeo& q, const void* Q, const void* K, const void* V, const void* table, void* O, float* lse,
                            void* ws, hipStream_t s) {
  const FwdPlan p = plan_dense_fwd(q);
  dense::FwdArgs a;
  a.Q = (const unsigned char*)Q; a.K = (const unsigned char*)K; a.V = (const unsigned char*)V;
  a.table = table; a.O = (unsigned char*)O; a.lse = lse; a.part = (float*)ws;
  a.tiles = p.tiles; a.splits = p.splits;
  a.rows = dense_rows(q);
  a.items = (long long)q.B * dense_heads(q) * p.tiles * p.splits;
  auto pick = [&](auto t, auto d) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value;
    if (q.bias) return pick_fwd<T, D, dense::BIAS>(q, p, a, s);
    return dense_packed(q) ? pick_fwd<T, D, dense::PACKED>(q, p, a, s) : pick_fwd<T, D, dense::PLAIN>(q, p, a, s);
  };
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  if (q.dtype == DA_BF16) return q.d == 128 ? pick((__bf16)0.f, d128) : pick((__bf16)0.f, d64);
  return q.d == 128 ? pick(0.f, d128) : pick(0.f, d64);
}

}  // namespace da
