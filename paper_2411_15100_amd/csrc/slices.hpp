// What kernels that go over the logits of a row share: slices of a row, the rules on their logits, weights 2^t in 64 bits, and what
// workgroups of one kernel hand to each other.  (In the anonymous namespace of every file that includes it.)
#pragma once
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstddef>
#include <cstdint>

#include "elements.hpp"
#include "logits.hpp"

namespace xgm {

namespace {

// ------------------------------------------------------------ a slice of a row
// A workgroup takes kSliceTokens tokens of a row, a thread two groups of 8 neighbours.  A slice begins on 16 bytes, up to a group less
// one token in front of a row that does not, so that a group is one load of 16 bytes (two of them in 32 bits); groups that reach over
// an end of the row are taken token by token.
constexpr int kSliceThreads = 512, kSliceTokens = 8192, kGroups = kSliceTokens / 8 / kSliceThreads, kTokens = 8 * kGroups;

typedef float Tokens __attribute__((ext_vector_type(kTokens)));  // of a thread; a vector, so that it never leaves the registers

template <Elem E> struct Row {
  const typename Type<E>::bits* at;
  int32_t V;
  __device__ Row(const Logits& in, int32_t b) : at(static_cast<const typename Type<E>::bits*>(in.at) + (int64_t)b * in.stride), V(in.V) {}
  __device__ int32_t first_token(int32_t slice) const {
    return slice * kSliceTokens - (int32_t)((uint32_t)reinterpret_cast<uintptr_t>(at) % 16u / sizeof(*at));
  }
};
template <Elem E> struct Group {  // 8 tokens as they lie in memory
  uint32_t word[sizeof(typename Type<E>::bits) * 2];
  __device__ __forceinline__ typename Type<E>::bits operator[](int i) const {
    if constexpr (sizeof(typename Type<E>::bits) == 4) return word[i];
    else return (uint16_t)(word[i / 2] >> (16 * (i & 1)));
  }
  __device__ __forceinline__ void set(int i, typename Type<E>::bits v) {
    if constexpr (sizeof(typename Type<E>::bits) == 4) word[i] = v;
    else word[i / 2] = i & 1 ? (word[i / 2] & 0xffffu) | (uint32_t)v << 16 : (word[i / 2] & 0xffff0000u) | v;
  }
};
// which of the tokens [t, t + 8) lie in the row and are allowed
__device__ __forceinline__ uint32_t allowed_of(const LogitRules& r, int32_t b, int32_t t, int32_t V) {
  uint32_t bits = 255u;
  if (r.mask) {
    const uint32_t* words = r.mask + (size_t)b * r.W_mask;
    const int32_t w = t >> 5;
    const uint32_t lo = w >= 0 && w < r.W_mask ? words[w] : 0u;
    const uint32_t hi = (t & 31) > 24 && w + 1 < r.W_mask ? words[w + 1] : 0u;
    bits = __builtin_amdgcn_alignbit(hi, lo, (uint32_t)t & 31u) & 255u;
    if (t + 8 > r.V_mask) bits &= t < r.V_mask ? (1u << (r.V_mask - t)) - 1u : 0u;
  }
  if (t < 0) bits &= t > -8 ? ~0u << -t : 0u;
  if (t + 8 > V) bits &= t < V ? (1u << (V - t)) - 1u : 0u;
  return bits;
}
template <Elem E> __device__ __forceinline__ Group<E> load_group(const Row<E>& row, int32_t t) {
  typedef typename Type<E>::bits bits;
  Group<E> g{};
  if (t >= 0 && t + 8 <= row.V) {
#pragma unroll
    for (int k = 0; k < (int)sizeof(bits) / 2; ++k) {
      const uint4 x = reinterpret_cast<const uint4*>(row.at + t)[k];
      g.word[4 * k] = x.x; g.word[4 * k + 1] = x.y; g.word[4 * k + 2] = x.z; g.word[4 * k + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (t + i >= 0 && t + i < row.V) g.set(i, row.at[t + i]);
  }
  return g;
}

// --------------------------------------------------------------- rules on logits
// What the history and the biases of a row say about the tokens of a slice, a word each: how often the token was generated, a bit if it
// occurs in the prompt, and which of the row's biases it has (one more; the highest number: one from there on, to be looked for).  Biases
// are entered first, of those of a token the last wins; counts are whole numbers: the order of the atomics does not matter.
// Nothing behind a history's length is read (the last row's memory may end there).
constexpr uint32_t kInPrompt = 0x80000000u, kCount = 0xfffffu;  // (a history is shorter than 2^20)
constexpr int kBiasShift = 20;
constexpr uint32_t kBiasMask = 0x7ffu;
struct RuleTable {
  uint32_t word[kSliceTokens];
};
constexpr int kHistoryAhead = 4;
struct History {
  int32_t token[kHistoryAhead], n, prompt, bias_begin, bias_end;
};
__device__ __forceinline__ History history_ahead(const LogitRules& r, int32_t b) {
  History h{};
  if (r.bias_ids) {
    h.bias_begin = max(r.bias_offsets[b], 0);
    h.bias_end = min(r.bias_offsets[b + 1], r.n_bias);
  }
  if (!r.tokens) return h;
  const int32_t* tokens = r.tokens + (int64_t)b * r.token_stride;
  h.n = (int32_t)min((int64_t)r.n_tokens[b], r.token_stride);
  h.prompt = r.n_prompt ? r.n_prompt[b] : 0;
#pragma unroll
  for (int k = 0; k < kHistoryAhead; ++k) {
    const int32_t i = (int32_t)threadIdx.x + k * kSliceThreads;
    h.token[k] = i < h.n ? tokens[i] : -1;
  }
  return h;
}
__host__ __device__ inline bool has_rules(const LogitRules& r) { return r.tokens || r.bias_ids; }
__device__ __forceinline__ void gather_rules(const LogitRules& r, int32_t b, int32_t first, const History& h, RuleTable& table) {
  uint4* const words = reinterpret_cast<uint4*>(table.word);
#pragma unroll
  for (int i = 0; i < kSliceTokens / 4 / kSliceThreads; ++i) words[i * kSliceThreads + (int32_t)threadIdx.x] = uint4{0, 0, 0, 0};
  __syncthreads();
  if (r.bias_ids) {
    for (int32_t e = h.bias_begin + (int32_t)threadIdx.x; e < h.bias_end; e += kSliceThreads) {
      const int32_t token = r.bias_ids[e];
      const int64_t at = (int64_t)token - first;
      if (token >= 0 && at >= 0 && at < kSliceTokens) atomicMax(&table.word[at], min((uint32_t)(e - h.bias_begin + 1), kBiasMask) << kBiasShift);
    }
    __syncthreads();
  }
  if (r.tokens) {
    auto enter = [&](int32_t i, int32_t token) {
      const int64_t at = (int64_t)token - first;
      if (i >= h.n || token < 0 || at < 0 || at >= kSliceTokens) return;
      if (i < h.prompt) atomicOr(&table.word[at], kInPrompt);
      else atomicAdd(&table.word[at], 1u);
    };
#pragma unroll
    for (int k = 0; k < kHistoryAhead; ++k) enter((int32_t)threadIdx.x + k * kSliceThreads, h.token[k]);
    const int32_t* tokens = r.tokens + (int64_t)b * r.token_stride;
#pragma unroll 4
    for (int32_t i = (int32_t)threadIdx.x + kHistoryAhead * kSliceThreads; i < h.n; i += kSliceThreads) enter(i, tokens[i]);
  }
  __syncthreads();
}
// What the rules make of a logit: in 64 bits, rounded once where it is kept.  Neither the product of a factor and a count nor the order of a
// compiler's contractions can change a bit of the 32 or fewer that are.
struct RowRules {
  double repetition, inverse, frequency, presence;
  const LogitRules& r;
  int32_t begin, end;  // of the row's biases
  __device__ RowRules(const LogitRules& rules, const History& h, int32_t b)
      : repetition(rules.repetition ? (double)rules.repetition[b] : 1.0), inverse(1.0 / repetition), frequency(rules.frequency ? (double)rules.frequency[b] : 0.0),
        presence(rules.presence ? (double)rules.presence[b] : 0.0), r(rules), begin(h.bias_begin), end(h.bias_end) {}
  // The penalties alone.  A quotient is the product with the inverse and what that leaves of it, rounded as the division is; where the
  // rest is none (infinite quotients, factors of 0) the product is the quotient.  frequency * count is exact.
  __device__ __forceinline__ double penalised(float x, uint32_t word) const {
    double y = (double)x;
    const bool divided = y > 0.0;
    const double near = y * (divided ? inverse : repetition), rest = fma(-near, repetition, y);
    y = divided && rest == rest ? fma(rest, inverse, near) : near;
    return word & kCount ? y - frequency * (double)(word & kCount) - presence : y;
  }
  __device__ double biased(float x, uint32_t word, int32_t token) const {
    double y = word & (kInPrompt | kCount) ? penalised(x, word) : (double)x;
    const uint32_t entry = word >> kBiasShift & kBiasMask;
    int32_t e = begin + (int32_t)entry - 1;
    if (entry == kBiasMask)
      for (int32_t k = end - 1; k > e; --k)
        if (r.bias_ids[k] == token) { e = k; break; }
    return y + (double)r.bias[e];
  }
};
__device__ __forceinline__ int32_t place_of(int k) { return (k / 8 * kSliceThreads + (int32_t)threadIdx.x) * 8 + k % 8; }
// The rules on the thread's tokens: get(k) and set(k, logit) for those that a rule touches.  Tokens of a text lie close together where
// ids are given out by frequency, so that many of a wave's are touched or none; biases are few and taken one by one.
template <class Get, class Set> __device__ __forceinline__ void apply_rules(const RuleTable& table, const RowRules& rule, const uint32_t (&ok)[kGroups], int32_t first, Get&& get, Set&& set) {
  uint32_t with_bias = 0;
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
    const uint4 a = *reinterpret_cast<const uint4*>(table.word + place_of(8 * j)), b = *reinterpret_cast<const uint4*>(table.word + place_of(8 * j) + 4);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (!ok[j] || !(a.x | a.y | a.z | a.w | b.x | b.y | b.z | b.w)) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (!w[i] || !(ok[j] >> i & 1u)) continue;
      if (w[i] >> kBiasShift & kBiasMask) with_bias |= 1u << (8 * j + i);
      else set(8 * j + i, rule.penalised(get(8 * j + i), w[i]));
    }
  }
#pragma unroll 1
  for (; with_bias; with_bias &= with_bias - 1) {
    const int k = __builtin_ctz(with_bias);
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < kTokens; ++i)
      if (i == k) v = get(i);
    const double y = rule.biased(v, table.word[place_of(k)], first + place_of(k));
#pragma unroll
    for (int i = 0; i < kTokens; ++i)
      if (i == k) set(i, y);
  }
}

size_t rule_table_bytes(const LogitRules& r) { return has_rules(r) ? sizeof(RuleTable) : 0; }
// slices of a row, wherever it begins
template <Elem E> int32_t slices_of(const Logits& in) {
  constexpr int32_t size = sizeof(typename Type<E>::bits);
  const bool anywhere = reinterpret_cast<uintptr_t>(in.at) % 16 != 0 || in.stride * size % 16 != 0;
  return (int32_t)(((int64_t)in.V + (anywhere ? 16 / size - 1 : 0) + kSliceTokens - 1) / kSliceTokens);
}

// ---------------------------------------------------------------- weights
constexpr int kWaves = kSliceThreads / 64;
constexpr int kBinsAnOctave = 4;
constexpr int kMassBits = 35;

// floats in their order as whole numbers; NaN lies with -inf, +inf with the largest finite number
__device__ __forceinline__ float drawable(float y) { return y > -__builtin_inff() ? fminf(y, FLT_MAX) : -__builtin_inff(); }
__device__ __forceinline__ uint32_t key_of(float y) {
  const uint32_t u = __float_as_uint(y == 0.0f ? 0.0f : y);  // (both zeros are one)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// t of a logit.  The product is rounded by itself: contracted with what is subtracted from it, it would not be the t whose octave was
// taken, which for logits of 1e38 is another number altogether.
__device__ __forceinline__ double octaves(float y, double per) {
#pragma clang fp contract(off)
  return (double)y * per;
}
// 2^t relative to 2^E, E a whole number: sixteenths of an octave come from a table in LDS (its 16 entries lie in different banks), the
// rest from the polynomial that meets the exponential function at the seven Chebyshev points of a sixteenth, which leaves less of it than
// 64 bits hold: with the rounding of t a weight is off by (2 + |y| / temperature) 2^-52 of itself at most.  (A polynomial over a whole octave
// takes eleven terms and as many instructions again.)
__constant__ const double kRoots[16] = {1, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916,
                                        1.189207115002721, 1.241857812073484, 1.2968395546510096, 1.3542555469368927,
                                        1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543,
                                        1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474};
__device__ __forceinline__ void fill_roots(double* roots) {
  if (threadIdx.x < 16) roots[threadIdx.x] = kRoots[threadIdx.x];
}
struct Power {
  int32_t i;      // whole sixteenths above E; far down: a large negative number
  double number;  // 2^t relative to its own octave
  __device__ __forceinline__ Power(double t, double E, const double* roots) {
    const double sixteenths = t * 16.0, whole = floor(sixteenths), r = sixteenths - whole;
    i = (int32_t)fmax(whole - E * 16.0, -1e6);
    double p = 9.382399669764206e-12;
    p = fma(p, r, 1.2713095335610576e-09);
    p = fma(p, r, 1.467611928836712e-07);
    p = fma(p, r, 1.3550807713052586e-05);
    p = fma(p, r, 0.0009383847928200675);
    p = fma(p, r, 0.043321698784995886);
    p = fma(p, r, 1.0);
    number = p * roots[i & 15];
  }
  __device__ __forceinline__ double weight() const { return ldexp(number, i >> 4); }
  __device__ __forceinline__ u64 mass() const {  // in 2^-kMassBits of the octave
    return (u64)__double_as_longlong(fma(number, (double)(1ull << kMassBits), 4503599627370496.0)) - (u64)__double_as_longlong(4503599627370496.0);
  }
  // the bin under the octave E, kBins or more: too far down
  __device__ __forceinline__ int32_t bin() const { return kBinsAnOctave - 1 - (i >> 2); }
};
static_assert(kBinsAnOctave == 4, "four sixteenths to a bin");

// ------------------------------------------- between the workgroups of a kernel
template <class T> __device__ __forceinline__ void put_out(T* to, T v) { __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class T> __device__ __forceinline__ T take_in(const T* from) { return __hip_atomic_load(const_cast<T*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this workgroup is the last of the row's n to come here; what the others have put out before can be taken in then.
__device__ bool last_of(uint32_t* arrived, uint32_t n, uint32_t& flag) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0);  // (everything put out has arrived)
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == n - 1) put_out(arrived, 0u);
    flag = before == n - 1;
  }
  __syncthreads();
  return flag != 0;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// The logits of a slice under the rules, whose table may lie where other things of the workgroup lie: with rules it is called
// only when all threads have read what they need of those, behind a barrier.
template <Elem E>
__device__ __forceinline__ void load_slice(const Row<E>& row, const LogitRules& r, int32_t b, int32_t first, RuleTable& table, Tokens& y) {
  const bool ruled = has_rules(r);
  const History h = history_ahead(r, b);
  Group<E> x[kGroups];
  uint32_t ok[kGroups];
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
    const int32_t t = first + (j * kSliceThreads + (int32_t)threadIdx.x) * 8;
    ok[j] = allowed_of(r, b, t, row.V);
    x[j] = Group<E>{};
    if (ok[j]) x[j] = load_group(row, t);
  }
  const RowRules rule(r, h, b);  // (read before the barriers of the next)
  if (ruled) gather_rules(r, b, first, h, table);
#pragma unroll
  for (int k = 0; k < kTokens; ++k) y[k] = ok[k / 8] >> (k % 8) & 1u ? widened<E>(x[k / 8][k % 8]) : -__builtin_inff();
  if (ruled) apply_rules(table, rule, ok, first, [&](int k) { return y[k]; }, [&](int k, double v) { y[k] = (float)v; });
#pragma unroll
  for (int k = 0; k < kTokens; ++k) y[k] = drawable(y[k]);
  if (ruled) __syncthreads();  // (other things lie where the tables were)
}
}  // namespace

}  // namespace xgm
