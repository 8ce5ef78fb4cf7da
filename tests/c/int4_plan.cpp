// For each line "M N K block" of the standard input, the plan of the product with an
// INT4 weight: its kernel in words (no spaces), then the workgroups in x, y and z, the
// codes of a slice, the groups of weight tiles, the bytes of LDS asked for at the launch
// and of the workspace, and whether the sizes are taken at all.
#include <cstdint>
#include <cstdio>
#include <string>

#include "zq_int4_plan.h"

using namespace zq;

int main() {
  long long M, N, K, block;
  while (std::scanf("%lld %lld %lld %lld", &M, &N, &K, &block) == 4) {
    const Int4Plan p = int4_plan(M, N, K);
    const std::string g = ",G" + std::to_string(int4_codes_a_scale(K, (int32_t)block));
    std::string name;
    switch (p.way) {
      case Int4Way::few: name = "few:" + std::to_string(p.MR); break;
      case Int4Way::lds: name = "lds" + g; break;
      case Int4Way::wide: name = "wide:" + std::to_string(p.MT) + g; break;
      default: name = "regs:" + std::to_string(p.MT) + "x" + std::to_string(p.GB) + g; break;
    }
    if (p.slices > 1) name += ",slices";
    std::printf("%s %lld %lld %lld %lld %lld %lld %lld %d\n", name.c_str(), (long long)p.grid, (long long)p.mgroups,
                (long long)p.slices, (long long)p.each, (long long)p.groups, (long long)p.lds,
                (long long)workspace_of(p, M, N), (int)int4_sizes_ok(M, N, K));
  }
  return 0;
}
