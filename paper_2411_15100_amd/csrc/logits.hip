// What lies behind the mask in a decode step (sections 2.1 and 3.5: the mask goes
// to masked sampling): rules on logits, and drawing one token a row.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "elements.hpp"
#include "logits.hpp"

namespace xgm {

namespace {

// --------------------------------------------------------------- rules on logits
constexpr int kRuleThreads = 256;
constexpr int kRuleTokens = 8192;  // of one workgroup

// The history and the biases of row b in the tokens [first, first + kRuleTokens), as two tables: how often a token was
// generated, with the top bit if it occurs in the prompt, and which entry of the row's biases is the token's (0: none).
// Counts are whole numbers and of the entries the last wins, so the order of the atomics does not matter.
__device__ void gather_rules(const LogitRules& r, int32_t b, int32_t first, uint32_t* counts, uint32_t* entries) {
  for (int32_t i = (int32_t)threadIdx.x; i < kRuleTokens; i += (int32_t)blockDim.x) {
    if (r.tokens) counts[i] = 0;
    if (r.bias_ids) entries[i] = 0;
  }
  __syncthreads();
  if (r.tokens) {
    const int64_t n64 = r.n_tokens[b];
    const int32_t n = (int32_t)(n64 < r.token_stride ? n64 : r.token_stride), prompt = r.n_prompt ? r.n_prompt[b] : 0;
    const int32_t* tokens = r.tokens + (int64_t)b * r.token_stride;
    for (int32_t i = (int32_t)threadIdx.x; i < n; i += (int32_t)blockDim.x) {
      const int64_t at = (int64_t)tokens[i] - first;
      if (at < 0 || at >= kRuleTokens) continue;
      if (i < prompt) atomicOr(&counts[at], 0x80000000u);
      else atomicAdd(&counts[at], 1u);
    }
  }
  if (r.bias_ids) {
    const int32_t e0 = max(r.bias_offsets[b], 0), e1 = min(r.bias_offsets[b + 1], r.n_bias);
    for (int32_t e = e0 + (int32_t)threadIdx.x; e < e1; e += (int32_t)blockDim.x) {
      const int64_t at = (int64_t)r.bias_ids[e] - first;
      if (at >= 0 && at < kRuleTokens) atomicMax(&entries[at], (uint32_t)(e + 1));
    }
  }
  __syncthreads();
}
// What the rules make of a logit: in 64 bits, where neither the product of a factor and a count nor the order of a
// compiler's contractions can change a bit of the 32 that are kept.
struct RowRules {
  double repetition, frequency, presence;
  const float* bias;
  __device__ RowRules(const LogitRules& r, int32_t b)
      : repetition(r.repetition ? (double)r.repetition[b] : 1.0), frequency(r.frequency ? (double)r.frequency[b] : 0.0),
        presence(r.presence ? (double)r.presence[b] : 0.0), bias(r.bias) {}
  __device__ float operator()(float x, uint32_t count, uint32_t entry) const {
    double y = (double)x;
    if (count) y = y > 0.0 ? y / repetition : y * repetition;
    if (count & 0x7fffffffu) y = y - frequency * (double)(count & 0x7fffffffu) - presence;
    if (entry) y += (double)bias[entry - 1];
    return (float)y;
  }
};
__device__ __forceinline__ bool allowed(const LogitRules& r, int32_t b, int32_t v) {
  return !r.mask || (v < r.V_mask && (r.mask[(size_t)b * r.W_mask + (v >> 5)] >> (v & 31) & 1u));
}

// One workgroup per (row, kRuleTokens tokens).
template <Elem E, Elem O>
__global__ __launch_bounds__(kRuleThreads) void process_logits_kernel(Logits in, LogitRules r, typename Type<O>::bits* out, int64_t out_stride) {
  extern __shared__ uint32_t tables[];
  uint32_t *counts = tables, *entries = tables + (r.tokens ? kRuleTokens : 0);
  const int32_t b = (int32_t)blockIdx.y, first = (int32_t)blockIdx.x * kRuleTokens;
  if (r.tokens || r.bias_ids) gather_rules(r, b, first, counts, entries);
  const RowRules rule(r, b);
  const typename Type<E>::bits* x = static_cast<const typename Type<E>::bits*>(in.at) + (int64_t)b * in.stride;
  for (int32_t i = (int32_t)threadIdx.x; i < kRuleTokens && first + i < in.V; i += kRuleThreads) {
    const int32_t v = first + i;
    float y = -__builtin_inff();
    if (allowed(r, b, v)) y = rule(widened<E>(x[v]), r.tokens ? counts[i] : 0u, r.bias_ids ? entries[i] : 0u);
    out[(int64_t)b * out_stride + v] = narrowed<O>(y);
  }
}
size_t rule_table_bytes(const LogitRules& r) { return (size_t)kRuleTokens * 4 * ((r.tokens ? 1 : 0) + (r.bias_ids ? 1 : 0)); }

template <Elem E, Elem O>
void launch_process(const Logits& in, int32_t B, const LogitRules& r, void* out, int64_t out_stride, hipStream_t stream) {
  hipLaunchKernelGGL((process_logits_kernel<E, O>), dim3((in.V + kRuleTokens - 1) / kRuleTokens, B), dim3(kRuleThreads), rule_table_bytes(r), stream, in, r,
                     static_cast<typename Type<O>::bits*>(out), out_stride);
}

// ------------------------------------------------------------------ drawing
constexpr int kDrawThreads = 1024;

// floats in their order as whole numbers; NaN lies with -inf, +inf with the largest finite number
__device__ __forceinline__ uint32_t key_of(float y) {
  if (y != y) y = -__builtin_inff();
  y = fminf(y, FLT_MAX);
  const uint32_t u = __float_as_uint(y == 0.0f ? 0.0f : y);  // (both zeros are one)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }
constexpr uint32_t kNoKey = 0x007fffffu;  // of -inf

struct RowState {
  u64 sum[kDrawThreads / 64];
  u64 mass[256];
  uint32_t count[256];
  uint32_t best[2];
  u64 found[2];
};
// Sums over the workgroup; every thread gets the result.
__device__ u64 sum_all(u64 x, RowState& s) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  __syncthreads();
  if ((threadIdx.x & 63u) == 0) s.sum[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
  for (int w = 0; w < kDrawThreads / 64; ++w) x += s.sum[w];
  return x;
}
// w in whole numbers of 2^-43: a row's sum stays below 2^63, and sums do not depend on their order
__device__ __forceinline__ u64 weight(uint32_t key, double top, double per) {
  return key <= kNoKey ? 0 : (u64)__double2ull_rn(exp(((double)value_of(key) - top) * per) * 8796093022208.0);
}

// The end of the kept prefix: tokens with a larger key, and of those with `key` the ones up to id `id`.
struct Cut {
  uint32_t key;
  int32_t id;
  __device__ bool keeps(uint32_t k, int32_t i) const { return k > key || (k == key && i <= id); }
};

// One row: the logits under the rules lie in y.
__global__ __launch_bounds__(kDrawThreads) void draw_kernel(const float* __restrict__ ys, int32_t V, DrawRules d, int32_t* __restrict__ ids, float* __restrict__ logprobs) {
  __shared__ RowState s;
  const int32_t b = (int32_t)blockIdx.x, tid = (int32_t)threadIdx.x;
  const float* y = ys + (size_t)b * V;
  uint32_t top = 0;
  int32_t top_id = 0;
  for (int32_t v = tid; v < V; v += kDrawThreads) {
    const uint32_t k = key_of(y[v]);
    if (k > top) { top = k; top_id = v; }
  }
  if (tid == 0) { s.best[0] = 0; s.best[1] = ~0u; }
  __syncthreads();
  atomicMax(&s.best[0], top);
  __syncthreads();
  if (top == s.best[0]) atomicMin(&s.best[1], (uint32_t)top_id);
  __syncthreads();
  top = s.best[0];
  top_id = (int32_t)s.best[1];
  if (top <= kNoKey) {
    if (tid == 0) {
      ids[b] = -1;
      if (logprobs) logprobs[b] = -__builtin_inff();
    }
    return;
  }
  const float t = d.uniform ? (d.temperature ? d.temperature[b] : 1.0f) : 0.0f;
  const bool greedy = !(t > 0.0f);
  const double y0 = (double)value_of(top), per = greedy ? 1.0 : 1.0 / (double)t;
  u64 whole = 0;
  for (int32_t v = tid; v < V; v += kDrawThreads) whole += weight(key_of(y[v]), y0, per);
  whole = sum_all(whole, s);
  int32_t drawn = top_id;
  if (!greedy) {
    Cut cut{0, 0};
    u64 total = whole;
    const int32_t k = d.top_k ? d.top_k[b] : 0;
    const float p = d.top_p ? d.top_p[b] : 1.0f, floor_p = d.min_p ? d.min_p[b] : 0.0f;
    // the cut behind the first k tokens, then the one where the sum reaches p of theirs: digit by digit of the key, then
    // of the id among equal keys
    for (int what = 0; what < 2; ++what) {
      if (what == 0 ? !(k > 0 && k < V) : !(p < 1.0f)) continue;
      const Cut before = cut;
      u64 left = what == 0 ? (u64)k : (u64)__double2ull_ru((double)p * (double)total);  // what the rest of the prefix has to reach
      if (left == 0 || (what == 1 && !(p > 0.0f))) left = 1;
      uint32_t key = 0, id = 0;
      u64 above = 0;  // sum of the tokens in front
      for (int digit = 0; digit < 7; ++digit) {  // 4 digits of the key, 3 of the id
        for (int i = tid; i < 256; i += kDrawThreads) { s.mass[i] = 0; s.count[i] = 0; }
        __syncthreads();
        const uint32_t shift = digit < 4 ? 24u - 8u * digit : 16u - 8u * (digit - 4);
        const uint32_t key_mask = digit == 0 ? 0u : digit < 4 ? ~0u << (shift + 8) : ~0u, id_mask = digit <= 4 ? 0u : ~0u << (shift + 8);
        for (int32_t v = tid; v < V; v += kDrawThreads) {
          const uint32_t q = key_of(y[v]);
          if ((q & key_mask) != key || ((uint32_t)v & id_mask) != id || !before.keeps(q, v)) continue;
          const uint32_t at = digit < 4 ? 255u - (q >> shift & 255u) : (uint32_t)v >> shift & 255u;
          atomicAdd(&s.count[at], 1u);
          atomicAdd(&s.mass[at], weight(q, y0, per));
        }
        __syncthreads();
        uint32_t at = 0;
        for (; at < 255; ++at) {
          const u64 x = what == 0 ? (u64)s.count[at] : s.mass[at];
          if (x >= left) break;
          left -= x;
          above += s.mass[at];
        }
        if (digit < 4) key |= (255u - at) << shift;
        else id |= at << shift;
        if (digit == 6) above += s.mass[at];
        __syncthreads();
      }
      cut = Cut{key, (int32_t)id};
      total = above;
    }
    const double least = (double)floor_p < 1.0 ? (double)floor_p : 1.0;
    auto kept = [&](int32_t v) -> u64 {
      const uint32_t q = key_of(y[v]);
      if (q <= kNoKey || !cut.keeps(q, v)) return 0;
      if (floor_p > 0.0f && exp(((double)value_of(q) - y0) * per) < least) return 0;
      return weight(q, y0, per);
    };
    total = 0;
    for (int32_t v = tid; v < V; v += kDrawThreads) total += kept(v);
    total = sum_all(total, s);
    double u = d.uniform[b];
    if (!(u >= 0.0)) u = 0.0;
    u64 target = u < 1.0 ? (u64)(u * (double)total) : total;
    if (target >= total) target = total - 1;
    // the first token at which the running sum exceeds the target
    int32_t v0 = 0;
    for (;; v0 += kDrawThreads) {
      const u64 here = sum_all(v0 + tid < V ? kept(v0 + tid) : 0, s);
      if (target < here || v0 + kDrawThreads >= V) break;
      target -= here;
    }
    u64 w = v0 + tid < V ? kept(v0 + tid) : 0, run = w;
    for (int e = 1; e < 64; e <<= 1) {
      const u64 other = __shfl_up(run, e);
      if ((tid & 63) >= e) run += other;
    }
    __syncthreads();
    if ((tid & 63) == 63) s.sum[tid >> 6] = run;
    __syncthreads();
    for (int i = 0; i < tid >> 6; ++i) run += s.sum[i];
    if (run > target && run - w <= target) s.found[0] = (u64)(v0 + tid);
    __syncthreads();
    drawn = (int32_t)s.found[0];
  }
  if (tid == 0) {
    ids[b] = drawn;
    if (logprobs) logprobs[b] = (float)(((double)value_of(key_of(y[drawn])) - y0) * per - log((double)whole * (1.0 / 8796093022208.0)));
  }
}

template <template <Elem> class Launch, class... Args>
void by_type(Elem e, const Args&... args) {
  if (e == Elem::kF32) Launch<Elem::kF32>::run(args...);
  else if (e == Elem::kBF16) Launch<Elem::kBF16>::run(args...);
  else Launch<Elem::kF16>::run(args...);
}
template <Elem E> struct Process {
  static void run(const Logits& in, const int32_t& B, const LogitRules& r, void* const& out, const int64_t& out_stride, const bool& wide, const hipStream_t& stream) {
    if (wide) launch_process<E, Elem::kF32>(in, B, r, out, out_stride, stream);
    else launch_process<E, E>(in, B, r, out, out_stride, stream);
  }
};
}  // namespace

void launch_process_logits(const Logits& in, Elem type, int32_t B, const LogitRules& rules, void* out, int64_t out_stride, hipStream_t stream) {
  by_type<Process>(type, in, B, rules, out, out_stride, false, stream);
}

size_t sampler_bytes(int32_t max_rows, int32_t V) { return (size_t)max_rows * (size_t)V * sizeof(float); }

void launch_sample(const Logits& in, Elem type, int32_t B, const LogitRules& rules, const DrawRules& draw, void* memory, int32_t* ids, float* logprobs,
                   hipStream_t stream) {
  by_type<Process>(type, in, B, rules, memory, (int64_t)in.V, true, stream);
  hipLaunchKernelGGL(draw_kernel, dim3(B), dim3(kDrawThreads), 0, stream, static_cast<const float*>(memory), in.V, draw, ids, logprobs);
}

}  // namespace xgm
