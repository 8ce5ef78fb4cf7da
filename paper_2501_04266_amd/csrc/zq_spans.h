// zq_spans.h -- the memory of a table of tensors: what a call writes must not overlap
// anything else of the table.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <vector>

#include "zq.h"

namespace zq {

struct Span {
  uintptr_t from, to;
  bool out;
};
inline void put_span(std::vector<Span>& spans, const void* p, int64_t bytes, bool out) {
  if (p && bytes > 0) spans.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, out});
}
// The ranges in the order of their addresses, each output against what starts before its end.
inline int check_spans(std::vector<Span>& spans) {
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  // the furthest end of outputs, and of anything, among the spans before
  uintptr_t out_to = 0, any_to = 0;
  for (const Span& s : spans) {
    if (s.from < out_to || (s.out && s.from < any_to)) return ZQ_E_ALIAS;
    any_to = std::max(any_to, s.to);
    if (s.out) out_to = std::max(out_to, s.to);
  }
  return ZQ_OK;
}

}  // namespace zq
