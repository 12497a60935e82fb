// Device-side views and launchers of what lies around the mask in a decode
// step: 4-bit output projection (head.hip), rules on
// logits, drawing tokens (logits.hip).
#pragma once
#include <hip/hip_runtime_api.h>

#include <atomic>
#include <cstddef>
#include <cstdint>

namespace xgm {

// Gives a kernel `bytes` of dynamic LDS at most on the current device, beyond what it may take by itself: once on each device,
// since that is where the limit belongs.
class LdsRoom {
 public:
  hipError_t operator()(const void* kernel, size_t bytes) {
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = device >= 0 && device < 64 ? 1ull << device : 0;  // (devices past the 64th are asked every time)
    if (given_.load(std::memory_order_relaxed) & bit) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess) given_.fetch_or(bit, std::memory_order_relaxed);
    return e;
  }

 private:
  std::atomic<uint64_t> given_{0};
};

enum class Elem : int32_t { kF32 = 0, kBF16 = 1, kF16 = 2 };

// the rules on the logits of a batch, in device memory (see xgm_logit_rules)
struct LogitRules {
  const uint32_t* mask;  // null: everything is allowed
  int32_t W_mask, V_mask;
  const int32_t* tokens;  // null: no history
  int64_t token_stride;
  const int32_t *n_tokens, *n_prompt;
  const float *repetition, *frequency, *presence;
  const int32_t* bias_ids;  // null: no biases
  const float* bias;
  const int32_t* bias_offsets;
  int32_t n_bias;
};

struct DrawRules {
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  const double* uniform;
};

struct Head {
  const void* hidden;
  int64_t hidden_stride;
  const uint8_t* codes;
  const void* scales;
  const uint8_t* zeros;  // null: 8
  void* logits;
  int64_t logits_stride;
  const uint32_t* mask;  // null: everything is allowed
  int32_t B, K, V, group, W_mask, V_mask;
};
hipError_t launch_q4_logits(const Head& h, Elem hidden_type, Elem logits_type, hipStream_t stream);

struct Logits {
  const void* at;
  int64_t stride;
  int32_t V;
};
hipError_t launch_process_logits(const Logits& in, Elem type, int32_t B, const LogitRules& rules, void* out, int64_t out_stride, hipStream_t stream);

size_t sampler_bytes(int32_t max_rows, int32_t V);
hipError_t launch_sample(const Logits& in, Elem type, int32_t B, const LogitRules& rules, const DrawRules& draw, void* memory, int32_t max_rows, int32_t max_V,
                         int32_t* ids, float* logprobs, hipStream_t stream);  // memory: sampler_bytes(max_rows, max_V), zeros at first

}  // namespace xgm
