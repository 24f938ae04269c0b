// Stands in front of the runtime's launch functions, for a test on a machine without a GPU: launches are written down, not made.
#include <cstddef>
#include <cstdint>
#include <vector>

struct Dim3 {
  uint32_t x, y, z;
};
struct Launch {
  uint64_t grid, threads, lds, first;  // first: the 32 bits that the kernel's argument begins with
};
static Dim3 g_grid, g_block;
static size_t g_lds;
static std::vector<Launch> g_launches;

extern "C" {
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void*) {
  g_grid = grid; g_block = block; g_lds = lds;
  return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* lds, void** stream) {
  *grid = g_grid; *block = g_block; *lds = g_lds; *stream = nullptr;
  return 0;
}
int hipLaunchKernel(const void*, Dim3 grid, Dim3 block, void** args, size_t lds, void*) {
  g_launches.push_back({(uint64_t)grid.x * grid.y * grid.z, (uint64_t)block.x * block.y * block.z, lds, *static_cast<const uint32_t*>(args[0])});
  return 0;
}
int hipGetLastError() { return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }

// the launches since the last call
uint64_t recorded(Launch* out, uint64_t room) {
  const uint64_t n = g_launches.size();
  for (uint64_t i = 0; i < n && i < room; ++i) out[i] = g_launches[i];
  g_launches.clear();
  return n;
}
}
