// Device-side views and launchers of what lies around the mask in a decode
// step: 4-bit output projection (head.hip), rules on
// logits, drawing tokens (logits.hip).
#pragma once
#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace xgm {

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
void launch_q4_logits(const Head& h, Elem hidden_type, Elem logits_type, hipStream_t stream);

struct Logits {
  const void* at;
  int64_t stride;
  int32_t V;
};
void launch_process_logits(const Logits& in, Elem type, int32_t B, const LogitRules& rules, void* out, int64_t out_stride, hipStream_t stream);

size_t sampler_bytes(int32_t max_rows, int32_t V);
void launch_sample(const Logits& in, Elem type, int32_t B, const LogitRules& rules, const DrawRules& draw, void* memory, int32_t max_rows, int32_t max_V,
                   int32_t* ids, float* logprobs, hipStream_t stream);  // memory: sampler_bytes(max_rows, max_V), zeros at first

}  // namespace xgm
