// Stands between the library and the HIP runtime in a process without a GPU: kernel
// launches succeed and do nothing, and are counted.  Preloaded by
// test_host_launches.py.
#include <dlfcn.h>

#include <map>
#include <string>

#include <hip/hip_runtime.h>

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
}  // namespace

extern "C" {

int shim_launches(const char *kernel) {
  int n = 0;
  for (const auto &c : counts())
    if (c.first.find(kernel) != std::string::npos) n += c.second;
  return n;
}

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
hipError_t hipLaunchKernel(const void *f, dim3, dim3, void **, size_t, hipStream_t) {
  ++counts()[names()[f]];
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }

}  // extern "C"
