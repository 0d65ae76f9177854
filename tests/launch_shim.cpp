// Stands between the library and the HIP runtime in a process without a GPU: kernel
// launches succeed and do nothing; they are counted, and the arguments of
// some are looked at.  Preloaded by test_host_launches.py.
#include <dlfcn.h>

#include <algorithm>
#include <map>
#include <string>

#include "hwkv_internal.h"

namespace {
std::map<const void *, std::string> &names() {
  static auto *m = new std::map<const void *, std::string>;
  return *m;
}
std::map<std::string, int> &counts() {
  static auto *m = new std::map<std::string, int>;
  return *m;
}
struct {
  dim3 grid, block;
  size_t shared;
  hipStream_t stream;
} launch;
std::string fault;

// Every entry that the kernel would touch lies in the row of its sequence.
void check_table_move(const hwkv::TableMoveArgs &a, dim3 grid) {
  for (int r = 0; r < a.part[a.n_parts] * hwkv::kMoveRound; ++r) {
    if (a.pages[r] == 0) continue;
    const bool rows = (a.src[r] == hwkv::kMoveCarry || a.src[r] < a.batch) &&
                      (a.dst[r] == hwkv::kMoveCarry || a.dst[r] < a.batch);
    // (a thread an entry, as many as the grid has)
    const int64_t pages = std::min<int64_t>(a.pages[r], (int64_t)grid.x * 256);
    if (!rows || pages > a.max_pages)
      fault = "table_move: " + std::to_string(a.pages[r]) + " entries of rows of " + std::to_string(a.max_pages);
  }
}
}  // namespace

extern "C" {

int shim_launches(const char *kernel) {
  int n = 0;
  for (const auto &c : counts())
    if (c.first.find(kernel) != std::string::npos) n += c.second;
  return n;
}
const char *shim_fault() { return fault.c_str(); }

void __hipRegisterFunction(void **modules, const void *host, char *device, const char *name, unsigned limit, void *tid,
                           void *bid, void *block, void *grid, int *size) {
  using F = void (*)(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *);
  static const F next = (F)dlsym(RTLD_NEXT, "__hipRegisterFunction");
  names()[host] = name;
  next(modules, host, device, name, limit, tid, bid, block, grid, size);
}

hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t stream) {
  launch = {grid, block, shared, stream};
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *stream) {
  *grid = launch.grid;
  *block = launch.block;
  *shared = launch.shared;
  *stream = launch.stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3, void **args, size_t, hipStream_t) {
  const std::string &name = names()[f];
  ++counts()[name];
  if (name.find("table_move") != std::string::npos)
    check_table_move(*static_cast<const hwkv::TableMoveArgs *>(args[0]), grid);
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }

}  // extern "C"
