// Host side of the relative position bias: bucket maps and the plan of block
// offsets (see relpos.h).
#include "relpos.h"

#include <algorithm>
#include <cmath>
#include <cstdint>

namespace pf {

std::string build_relpos(pf_relpos &R, int64_t seq, int32_t n_buckets, const int32_t *bucket) {
  R.seq = seq;
  R.nb = (int32_t)(seq / 64);
  R.n_buckets = n_buckets;
  R.bucket.assign(2 * seq, -1);
  for (int64_t i = 0; i < 2 * seq - 1; ++i) {
    if (bucket[i] < -1 || bucket[i] >= n_buckets)
      return "bucket of distance " + std::to_string(i - (seq - 1)) + " is " + std::to_string(bucket[i]) +
             ", not -1 .. n_buckets - 1";
    R.bucket[i + 1] = bucket[i];
  }
  const int32_t nb = R.nb;
  R.info.assign(2 * nb - 1, -1);
  R.omin = 1;
  R.omax = 0;
  bool any = false;
  for (int32_t d = -(nb - 1); d <= nb - 1; ++d) {
    // Distances 64 d - 64 (never in the block) .. 64 d + 63 at w[0 .. 127].
    const int32_t *w = R.bucket.data() + (int64_t)d * 64 + seq - 64;
    const bool one = std::all_of(w + 2, w + 128, [&](int32_t x) { return x == w[1]; });
    int32_t &info = R.info[d + nb - 1];
    if (one) {
      info = w[1];
      if (w[1] < 0) continue;
    } else {
      info = kRelposMixed + (int32_t)(R.order.size() / 64);
      // Ascending by bucket, then by distance.  Position 0 and masked
      // distances carry sums of zero: bucket 0 takes them.
      int32_t pos[128];
      for (int32_t i = 0; i < 128; ++i) pos[i] = i;
      auto id = [&](int32_t i) { return i == 0 || w[i] < 0 ? 0 : w[i]; };
      std::stable_sort(pos, pos + 128, [&](int32_t x, int32_t y) { return id(x) < id(y); });
      for (int l = 0; l < 64; ++l) {
        const uint32_t a = pos[2 * l], b = pos[2 * l + 1];
        R.order.push_back(a | b << 8 | (uint32_t)id(a) << 16 | (uint32_t)id(b) << 24);
      }
    }
    if (!any) R.omin = d;
    R.omax = d;
    any = true;
  }
  return "";
}

namespace {
// Unsigned integers of any size, least significant word first.
using Big = std::vector<uint32_t>;
void mul(Big &x, uint32_t m) {
  uint64_t carry = 0;
  for (uint32_t &w : x) {
    carry += (uint64_t)w * m;
    w = (uint32_t)carry;
    carry >>= 32;
  }
  if (carry) x.push_back((uint32_t)carry);
}
Big power(uint32_t base, int n, Big x = {1}) {
  for (int i = 0; i < n; ++i) mul(x, base);
  return x;
}
bool less(const Big &x, const Big &y) {
  if (x.size() != y.size()) return x.size() < y.size();
  for (size_t i = x.size(); i-- > 0;)
    if (x[i] != y[i]) return x[i] < y[i];
  return false;
}
}  // namespace

std::string log_buckets(int64_t seq, int32_t n_buckets, int64_t max_distance, bool bidirectional,
                        std::vector<int32_t> &bucket) {
  const int32_t n = bidirectional ? n_buckets / 2 : n_buckets, e = n / 2;
  if (n < 2 || (bidirectional && n_buckets % 2))
    return bidirectional ? "n_buckets must be even and at least 4" : "n_buckets must be at least 2";
  if (max_distance <= e || max_distance > 0x7fffffff)
    return "max_distance must exceed the buckets of one distance each and fit 31 bits";
  // Smallest distance of the buckets 1 .. n - 1 of one direction.  From e on,
  // d lies in bucket e + k as soon as (d / e)^(n - e) >= (max_distance / e)^k: an
  // estimate in floating point, settled in integers.
  std::vector<int64_t> steps;
  for (int32_t d = 1; d <= e && d < n; ++d) steps.push_back(d);
  const int m = n - e;
  for (int k = 1; k < m; ++k) {
    const Big bound = power((uint32_t)e, m - k, power((uint32_t)max_distance, k));
    auto in = [&](int64_t d) { return !less(power((uint32_t)d, m), bound); };
    int64_t d = (int64_t)std::llround((double)e * std::pow((double)max_distance / e, (double)k / m));
    d = std::min<int64_t>(std::max<int64_t>(d, e), max_distance);
    while (d > e && in(d - 1)) --d;
    while (!in(d)) ++d;
    steps.push_back(d);
  }
  bucket.resize(2 * seq - 1);
  for (int64_t i = 0; i < 2 * seq - 1; ++i) {
    const int64_t dist = i - (seq - 1), a = dist < 0 ? -dist : dist;
    const int32_t c = (int32_t)(std::upper_bound(steps.begin(), steps.end(), a) - steps.begin());
    bucket[i] = dist <= 0 ? c : bidirectional ? n + c : -1;
  }
  return "";
}

}  // namespace pf
