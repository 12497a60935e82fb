// Device-side views and launchers of what lies around the mask in a decode
// step: 4-bit output projection (head.hip), 8-bit output projection and rows of
// both as hidden states (f8.hip), rules on logits, drawing tokens (logits.hip),
// beams and what they keep (beam.hip).
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

// Hidden states, or what they are made from; in 8 bits (scales not null) they have a scale for each 128 columns.
struct F8States {
  const void* at;
  int64_t stride;  // elements
  const float* scales;
};
struct F8Head {
  F8States hidden;
  const uint8_t* codes;
  const float* scales;  // of blocks of 128 rows and 128 columns
  void* logits;
  int64_t logits_stride;
  const uint32_t* mask;  // null: everything is allowed
  int32_t B, K, V, W_mask, V_mask;
};
__host__ __device__ inline int32_t f8_blocks(int32_t n) { return (int32_t)(((int64_t)n + 127) / 128); }
size_t f8_work_bytes(int32_t B, int32_t K);
hipError_t launch_f8_quantize(const void* x, Elem type, int32_t B, int32_t K, int64_t stride, uint8_t* codes, int64_t codes_stride, float* scales, hipStream_t stream);
// hidden_type is not looked at where the states have scales; `work`: f8_work_bytes(B, K) bytes where they have none
hipError_t launch_f8_logits(const F8Head& h, Elem hidden_type, Elem logits_type, void* work, hipStream_t stream);

// Rows of an output matrix as hidden states.
struct Embed {
  const int32_t* ids;
  const uint8_t* codes;
  const void* scales;
  const uint8_t* zeros;  // null: 8
  void* out;
  int64_t out_stride;
  int32_t n, V, K, group;
  float factor;
};
hipError_t launch_q4_embed(const Embed& e, Elem scales_type, Elem out_type, hipStream_t stream);
hipError_t launch_f8_embed(const Embed& e, Elem out_type, hipStream_t stream);

struct Logits {
  const void* at;
  int64_t stride;
  int32_t V;
};
hipError_t launch_process_logits(const Logits& in, Elem type, int32_t B, const LogitRules& rules, void* out, int64_t out_stride, hipStream_t stream);

size_t sampler_bytes(int32_t max_rows, int32_t V);
hipError_t launch_sample(const Logits& in, Elem type, int32_t B, const LogitRules& rules, const DrawRules& draw, void* memory, int32_t max_rows, int32_t max_V,
                         int32_t* ids, float* logprobs, hipStream_t stream);  // memory: sampler_bytes(max_rows, max_V), zeros at first

// Continuations of beams.
constexpr int32_t kMaxBeams = 64, kMaxContinuations = 128;
struct BeamSearch {
  const float* scores;
  const int32_t* ended;  // null: none
  int32_t requests, beams, n_out;
  int32_t placed;
  int32_t *rows, *ids;
  float* out_scores;
};
size_t beam_bytes(int32_t max_rows, int32_t V);
hipError_t launch_beam_select(const Logits& in, Elem type, const LogitRules& rules, const BeamSearch& beams, void* memory, int32_t max_rows, int32_t max_V,
                              hipStream_t stream);  // memory: beam_bytes(max_rows, max_V), zeros at first

// What rows keep, to be moved between them (see xgm_row_data).
struct RowData {
  void* data;
  int64_t row_stride, outer_stride, part_stride, part_bytes;
  const int32_t* used;
  int64_t used_bytes;
  int32_t n_outer, n_parts;
};
constexpr int kMaxRowData = 8;
hipError_t launch_reorder_rows(const RowData* data, int n, const int32_t* source, int32_t B, hipStream_t stream);

}  // namespace xgm
