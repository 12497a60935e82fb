// Checks of the launches of the calls around the mask at the ends of their ranges, on the host, without a device: a program that stands in for the part of the
// HIP runtime that they use.  What the calls accept has to be something that can be launched: in no direction 2^32 threads or more, nor more than 65535
// workgroups beside the first one, nor more than 1024 threads a workgroup.
#include <dlfcn.h>
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>

#include "../include/xgm.h"

namespace {
int n_launches = 0, failures = 0;
std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> m;
  return m;
}
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
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t shared, hipStream_t) {
  ++n_launches;
  const auto fits = [](uint64_t groups, uint64_t threads) { return groups > 0 && threads > 0 && groups * threads < 1ull << 32; };
  check(fits(grid.x, block.x) && fits(grid.y, block.y) && fits(grid.z, block.z) && grid.y <= 65535 && grid.z <= 65535 &&
            (uint64_t)block.x * block.y * block.z <= 1024 && shared <= 160 * 1024,
        names()[f] + " launched with " + std::to_string(grid.x) + " x " + std::to_string(grid.y) + " x " + std::to_string(grid.z) + " workgroups of " +
            std::to_string(block.x) + " threads");
  return hipSuccess;
}
hipError_t hipExtLaunchKernel(const void* f, dim3 g, dim3 b, void** a, size_t s, hipStream_t st, hipEvent_t, hipEvent_t, int) { return hipLaunchKernel(f, g, b, a, s, st); }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "an error of the stand-in"; }
hipError_t hipGetDeviceCount(int* n) { *n = 1; return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipMalloc(void** p, size_t) { *p = std::malloc(256); return hipSuccess; }  // (never read: there is no kernel)
hipError_t hipFree(void* p) { std::free(p); return hipSuccess; }
hipError_t hipMemsetAsync(void*, int, size_t, hipStream_t) { return hipSuccess; }
}

int main(int, char** argv) {
  void* const library = dlopen(argv[1], RTLD_NOW | RTLD_GLOBAL);
  if (!library) { std::fprintf(stderr, "%s\n", dlerror()); return 2; }
  const std::string what = argv[2];
#define XGM(name) reinterpret_cast<decltype(name)*>(dlsym(library, #name))
  // Addresses that no two arrays share (none is read or written).
  auto at = [](uint64_t k) { return reinterpret_cast<char*>(k << 52); };
  auto words = [&](uint64_t k) { return reinterpret_cast<int32_t*>(at(k)); };
  auto floats = [&](uint64_t k) { return reinterpret_cast<float*>(at(k)); };
  auto codes = [&](uint64_t k) { return reinterpret_cast<uint8_t*>(at(k)); };
  auto ran = [&](int status, const std::string& call) {
    check(status == XGM_OK && n_launches > 0, call + ": " + std::to_string(status) + " " + XGM(xgm_last_error)());
    n_launches = 0;
  };
  if (what == "lookups") {
    for (int32_t K : {32, 2048, 2080, (int)XGM_MAX_HIDDEN})
      for (xgm_dtype out : {XGM_F32, XGM_BF16})
        for (int32_t n : {1, (1 << 24) - 1, 1 << 24}) {
          const std::string sizes = std::to_string(n) + " rows of " + std::to_string(K);
          ran(XGM(xgm_f8_embed)(words(1), n, codes(2), floats(3), XGM_MAX_COLUMNS, K, 1.0f, at(4), out, K, nullptr), "f8 " + sizes);
          ran(XGM(xgm_q4_embed)(words(1), n, codes(2), at(3), XGM_BF16, nullptr, XGM_MAX_COLUMNS, K, 32, 1.0f, at(4), out, K, nullptr), "q4 " + sizes);
        }
  } else if (what == "rows") {
    xgm_row_data d[XGM_MAX_ROW_DATA]{};
    for (int64_t parts : {1 << 10, 1 << 20, (1 << 24) - 64, 1 << 24, 1 << 27})
      for (int n : {1, (int)XGM_MAX_ROW_DATA})
        for (int64_t bytes : {1, 16, 4096, 1 << 24}) {
          for (int k = 0; k < n; ++k) {
            d[k].d_data = at(k + 1);
            d[k].part_bytes = d[k].part_stride = bytes;
            d[k].n_parts = (int32_t)(parts >= 1 << 20 ? parts >> 6 : parts);
            d[k].n_outer = (int32_t)(parts / d[k].n_parts);
            d[k].row_stride = bytes * d[k].n_parts;
            d[k].outer_stride = 2 * d[k].row_stride;
          }
          ran(XGM(xgm_reorder_rows)(d, n, words(100), 2, nullptr), std::to_string(n) + " arrays of " + std::to_string(parts) + " parts of " + std::to_string(bytes));
        }
  } else if (what == "projection") {
    for (int32_t B : {1, 64, 65, 129, (int)XGM_MAX_ROWS})
      for (int32_t K : {16, 4096, (int)XGM_MAX_HIDDEN})
        for (int32_t V : {1, 1 << 20, (int)XGM_MAX_COLUMNS})
          for (xgm_dtype out : {XGM_F32, XGM_BF16})
            for (const int32_t* mask : {(const int32_t*)nullptr, (const int32_t*)words(6)}) {
              const std::string sizes = std::to_string(B) + " x " + std::to_string(K) + " x " + std::to_string(V);
              ran(XGM(xgm_f8_logits)(at(1), XGM_BF16, nullptr, B, K, K, codes(3), floats(4), V, at(5), out, V, mask, V, at(7), nullptr), "bf16 " + sizes);
              ran(XGM(xgm_f8_logits)(at(1), XGM_F8, floats(2), B, K, K, codes(3), floats(4), V, at(5), out, V, mask, V, at(7), nullptr), "f8 " + sizes);
            }
    ran(XGM(xgm_f8_quantize)(at(1), XGM_F32, XGM_MAX_ROWS, XGM_MAX_HIDDEN, XGM_MAX_HIDDEN, codes(2), XGM_MAX_HIDDEN, floats(3), nullptr), "to 8 bits");
  } else if (what == "beams") {
    xgm_beams* s = nullptr;
    check(XGM(xgm_beams_create)(XGM_MAX_ROWS, XGM_MAX_LOGITS, nullptr, &s) == XGM_OK, "beams");
    for (int32_t beams : {1, (int)XGM_MAX_BEAMS})
      for (int32_t V : {1, (int)XGM_MAX_LOGITS})
        for (xgm_dtype dt : {XGM_F32, XGM_BF16})
          ran(XGM(xgm_beam_select)(s, at(1) + 4, dt, XGM_MAX_ROWS / beams, beams, V, V + 1, nullptr, floats(2), words(3), XGM_MAX_CONTINUATIONS, 0, words(4), words(5),
                                   floats(6), nullptr), "continuations of " + std::to_string(beams) + " beams of " + std::to_string(V));
    XGM(xgm_beams_destroy)(s);
  } else {
    return 2;
  }
  return failures ? 1 : 0;
}
