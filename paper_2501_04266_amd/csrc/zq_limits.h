// zq_limits.h -- how large a call and a launch may be: host arithmetic, without HIP.
#pragma once

#include <stdint.h>

namespace zq {

constexpr int64_t kMaxGrid = 0x7fffffff;  // workgroups of a call
// A launch has fewer than 2^32 work items a dimension.  The runtime does not refuse
// more: it launches their number modulo 2^32.
constexpr uint64_t kMaxItems = 0xffffffffu;
constexpr unsigned most_groups(unsigned block) { return (unsigned)(kMaxItems / block); }

}  // namespace zq
