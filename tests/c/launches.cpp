// Stands in for the HIP runtime's kernel launch: notes every launch's grid, workgroup
// size and first argument (as 32 bits), and says that it worked.  No GPU.
#include <cstdint>
#include <vector>

struct Dim {
  uint32_t x, y, z;
};
struct Launch {
  uint64_t kernel, x, y, z, threads, first;
};
static std::vector<Launch> launches;

extern "C" int hipLaunchKernel(const void* kernel, Dim grid, Dim block, void** args, std::size_t, void*) {
  launches.push_back({(uint64_t)(uintptr_t)kernel, grid.x, grid.y, grid.z, (uint64_t)block.x * block.y * block.z,
                      *static_cast<const uint32_t*>(args[0])});
  return 0;
}

// the launches since the last call, at most `most`; their number
extern "C" int take_launches(Launch* out, int most) {
  const int n = (int)launches.size();
  for (int i = 0; i < n && i < most; ++i) out[i] = launches[i];
  launches.clear();
  return n;
}
