// Plan of a relative position bias: the bucket of every distance, and what the
// kernels need to know of every 64 x 64 block of distances.
#pragma once

#include <string>
#include <vector>

#include "pf_internal.h"
#include "pixelfly.h"

struct pf_relpos {
  int64_t seq = 0;  // a multiple of 64
  int32_t nb = 0, n_buckets = 0;
  std::vector<int32_t> bucket;  // [2 seq]: distance e - seq; entry 0 is -1
  std::vector<int32_t> info;    // [2 nb - 1], see pf::RelposArgs
  std::vector<uint32_t> order;  // 64 words per mixed block offset
  int32_t omin = 1, omax = 0;   // block offsets with an attended distance (none: 1, 0)

  int device = -1;
  void *dev_mem = nullptr;
  const int32_t *d_bucket = nullptr, *d_info = nullptr;
  const uint32_t *d_order = nullptr;
};

namespace pf {
// Fill the plan from bucket[seq - 1 + distance], distance = -(seq - 1) .. seq - 1.
// Returns "" or an error.
std::string build_relpos(pf_relpos &R, int64_t seq, int32_t n_buckets, const int32_t *bucket);
// Buckets of the logarithmic map by distance, as build_relpos takes them.
std::string log_buckets(int64_t seq, int32_t n_buckets, int64_t max_distance, bool bidirectional,
                        std::vector<int32_t> &bucket);
}  // namespace pf
