// Checks of the launches of head.hip and logits.hip on the host, without a device: a program that stands in for the part of the HIP runtime
// that they use.  A kernel that may take much dynamic LDS has been given room for it on every device that it is launched on, and a
// device that refuses the room is an error of the call.
#include <dlfcn.h>
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>
#include <utility>

#include "../include/xgm.h"

namespace {
int device = 0, n_launches = 0, n_asked = 0, failures = 0;
bool refuse = false;
std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> m;
  return m;
}
std::map<std::pair<const void*, int>, size_t> room;  // of a kernel on a device
struct { dim3 grid, block; size_t shared; hipStream_t stream; } pushed;
void check(bool ok, const std::string& what) {
  if (ok) return;
  ++failures;
  std::printf("FAILED: %s\n", what.c_str());
}
}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned int, void*, void*, void*, void*, int*) { names()[host] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t stream) { pushed = {grid, block, shared, stream}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = pushed.grid; *block = pushed.block; *shared = pushed.shared; *stream = pushed.stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3, dim3, void**, size_t shared, hipStream_t) {
  ++n_launches;
  const std::string& name = names()[f];
  const bool much = name.find("q4_few_kernel") != std::string::npos || name.find("draw_cut_kernel") != std::string::npos;
  const auto at = room.find({f, device});
  if (much) check(at != room.end() && at->second >= shared, name + " launched with " + std::to_string(shared) + " bytes on device " + std::to_string(device));
  return hipSuccess;
}
hipError_t hipExtLaunchKernel(const void* f, dim3 g, dim3 b, void** a, size_t s, hipStream_t st, hipEvent_t, hipEvent_t, int) { return hipLaunchKernel(f, g, b, a, s, st); }
hipError_t hipFuncSetAttribute(const void* f, hipFuncAttribute what, int value) {
  check(what == hipFuncAttributeMaxDynamicSharedMemorySize, "no other attribute is set");
  ++n_asked;
  if (refuse) return hipErrorInvalidValue;
  room[{f, device}] = (size_t)value;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "an error of the stand-in"; }
hipError_t hipGetDeviceCount(int* n) { *n = 100; return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { *p = std::malloc(n); return *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
hipError_t hipMemsetAsync(void*, int, size_t, hipStream_t) { return hipSuccess; }
}

int main(int, char** argv) {
  void* const library = dlopen(argv[1], RTLD_NOW | RTLD_GLOBAL);
  if (!library) { std::fprintf(stderr, "%s\n", dlerror()); return 2; }
#define XGM(name) reinterpret_cast<decltype(name)*>(dlsym(library, #name))
  alignas(16) static char memory[64];  // (never read: there is no kernel)
  const uint8_t* const codes = reinterpret_cast<const uint8_t*>(memory);
  const int32_t* const words = reinterpret_cast<const int32_t*>(memory);
  xgm_sampler* s = nullptr;
  check(XGM(xgm_sampler_create)(2, 1000, nullptr, &s) == XGM_OK, "sampler");
  xgm_logit_rules rules{};
  rules.d_tokens = rules.d_n_tokens = words;
  rules.token_stride = 8;
  xgm_draw_rules draw{};
  draw.d_uniform = reinterpret_cast<const double*>(memory);
  draw.d_top_p = reinterpret_cast<const float*>(memory);
  auto project = [&] { return XGM(xgm_q4_logits)(memory, XGM_BF16, 4, 16384, 16384, codes, memory, nullptr, 1000, 128, memory, XGM_F32, 1000, nullptr, nullptr); };
  auto sample = [&] { return XGM(xgm_sample)(s, memory, XGM_BF16, 2, 1000, 1000, &rules, &draw, reinterpret_cast<int32_t*>(memory), nullptr, nullptr); };

  refuse = true;
  check(project() == XGM_ERR_HIP && n_launches == 0, "a projection whose room is refused");
  check(sample() == XGM_ERR_HIP && n_launches == 0, "a draw whose room is refused");
  refuse = false;
  for (int d : {0, 1, 7, 63, 64, 99, 1, 0}) {
    device = d;
    const int before = n_launches;
    check(project() == XGM_OK && n_launches == before + 1, "a projection on device " + std::to_string(d));
    check(sample() == XGM_OK && n_launches == before + 4, "a draw on device " + std::to_string(d));
  }
  const int asked = n_asked;
  for (int k = 0; k < 10; ++k) check(project() == XGM_OK && sample() == XGM_OK, "again");
  check(n_asked == asked, "a device is asked once");
  refuse = true;
  device = 2;
  const int before = n_launches;
  check(project() == XGM_ERR_HIP && sample() == XGM_ERR_HIP && n_launches == before, "another device that refuses");
  refuse = false;
  check(project() == XGM_OK && sample() == XGM_OK, "and no longer does");
  XGM(xgm_sampler_destroy)(s);
  std::printf("%d failures\n", failures);
  return failures ? 1 : 0;
}
