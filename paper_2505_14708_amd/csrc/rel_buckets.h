// Buckets of relative positions (host arithmetic; no HIP, so that it compiles for the CPU by itself).
#pragma once
#include <math.h>
#include <stdint.h>

namespace da {

constexpr int kMaxBuckets = 256;
constexpr int kMaxDistance = 1024;

// r = key position - query position.  A direction has n buckets (half of them, and the upper half for r > 0, if bidirectional); of its
// distances a, those below e = n / 2 have one each, and the others share n - e: number k of those begins at the smallest a with
//     (a / e)^(n - e) >= (max_distance / e)^k
// which is e + floor((n - e) log(a / e) / log(max_distance / e)) without a logarithm to round; the last one has no end.
struct RelRule {
  int n, e;                          // buckets of a direction, distances with one of their own
  int bidirectional;
  int cut;                           // the distance from which on there is only one bucket
  int n_border;
  int16_t border[kMaxBuckets / 2 + 1];   // where shared bucket 1, 2, .. begins
};

// a^p >= b^(p - k) c^k, exactly (numbers of up to 11 bits, powers of up to kMaxBuckets)
inline bool power_reaches(int a, int p, int b, int c, int k) {
  constexpr int kWords = (11 * kMaxBuckets + 31) / 32 + 1;
  struct Number {
    uint32_t w[kWords];
    int n;
    void times(uint32_t f) {
      uint64_t carry = 0;
      for (int i = 0; i < n; ++i) {
        carry += (uint64_t)w[i] * f;
        w[i] = (uint32_t)carry;
        carry >>= 32;
      }
      if (carry) w[n++] = (uint32_t)carry;
    }
  } l, r;
  l.w[0] = r.w[0] = 1u;
  l.n = r.n = 1;
  for (int i = 0; i < p; ++i) l.times((uint32_t)a);
  for (int i = 0; i < p; ++i) r.times((uint32_t)(i < k ? c : b));
  if (l.n != r.n) return l.n > r.n;
  for (int i = l.n; i-- > 0;)
    if (l.w[i] != r.w[i]) return l.w[i] > r.w[i];
  return true;
}

// false: not a rule (too few or too many buckets, or distances that end before the shared buckets begin)
inline bool make_rel_rule(int buckets, int max_distance, int bidirectional, RelRule* out) {
  if (bidirectional != 0 && bidirectional != 1) return false;
  if (buckets < 1 || buckets > kMaxBuckets || (bidirectional && buckets % 2 != 0)) return false;
  RelRule t;
  t.bidirectional = bidirectional;
  t.n = bidirectional ? buckets / 2 : buckets;
  t.e = t.n / 2;
  if (t.e < 1 || max_distance <= t.e || max_distance > kMaxDistance) return false;
  t.n_border = t.n - t.e - 1;
  for (int k = 1; k <= t.n_border; ++k) {
    // in doubles, whose error is below 1e-11 here, unless a whole number lies nearer than 1e-6: then exactly
    const double at = t.e * pow((double)max_distance / t.e, (double)k / (t.n - t.e));
    const int near = (int)floor(at + 0.5);
    int lo = (int)ceil(at);
    if (fabs(at - near) < 1e-6) lo = power_reaches(near, t.n - t.e, t.e, max_distance, k) ? near : near + 1;
    t.border[k - 1] = (int16_t)lo;
  }
  for (int k = t.n_border; k <= kMaxBuckets / 2; ++k) t.border[k] = 0;
  t.cut = t.n_border > 0 ? t.border[t.n_border - 1] : t.e;
  *out = t;
  return true;
}

#ifdef __HIP__
__host__ __device__
#endif
inline int rel_bucket(const RelRule& t, int r) {
  int a = t.bidirectional ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
  if (a >= t.e) {
    int k = t.e;
    for (int i = 0; i < t.n_border; ++i) k += a >= t.border[i] ? 1 : 0;
    a = k;
  }
  return a + (t.bidirectional && r > 0 ? t.n : 0);
}

}  // namespace da
