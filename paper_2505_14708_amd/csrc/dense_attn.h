// One problem of the dense attention kernels (attention to an encoder's states, attention with a relative position bias), host and device.
#pragma once
#include "da_internal.h"
#include "rel_buckets.h"

namespace da {

struct DenseGeo {
  int B, H, Hk, group, N, M, d, dtype;
  float c2, c2_lo;       // scale * log2(e), and what its rounding left: the softmax works in powers of two
  float s_low;           // the lowest score whose product with c2_lo is finite
  float scale;
  Rows q, k, v, o, dout, dq, dk, dv;
  const int32_t* kv_len; // keys of each batch element (NULL: M)
  // with a bias
  int bias, buckets, q_pos;
  RelRule rule;
};

// Rows of queries as the kernels see them: each head's own, or, where heads share keys and have few queries each, those of all heads that share
// a head of K and V as one list (queries of one position in several heads fill a tile, and K and V are read once for them).  A bias is per
// head, so its queries stay apart; from kPackBelow queries on a head fills its tiles by itself.
constexpr int kPackBelow = 256;
inline bool dense_packed(const DenseGeo& q) { return !q.bias && q.group > 1 && q.N < kPackBelow; }
inline int dense_heads(const DenseGeo& q) { return dense_packed(q) ? q.Hk : q.H; }
inline long long dense_rows(const DenseGeo& q) { return dense_packed(q) ? (long long)q.group * q.N : q.N; }

// How the work of the forward pass is cut (host rule; the reasons stand at the function)
struct FwdPlan {
  int join, sets;        // waves share their queries; else sets of 32 queries of a wave
  int row_tile, tiles, splits;   // queries of a workgroup, tiles of them of a head, pieces of the keys
};
FwdPlan plan_dense_fwd(const DenseGeo& q);
size_t dense_fwd_workspace(const DenseGeo& q);
size_t dense_bwd_workspace(const DenseGeo& q);

hipError_t launch_dense_fwd(const DenseGeo& q, const void* Q, const void* K, const void* V, const void* table, void* O, float* lse,
                            void* ws, hipStream_t s);
hipError_t launch_dense_bwd(const DenseGeo& q, const void* Q, const void* K, const void* V, const void* table, const void* O,
                            const float* lse, const void* dO, void* dQ, void* dK, void* dV, void* dtable, void* ws, hipStream_t s);

}  // namespace da
