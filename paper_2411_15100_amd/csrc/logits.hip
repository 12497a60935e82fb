// What lies behind the mask in a decode step (sections 2.1 and 3.5: the mask goes
// to masked sampling): rules on logits, and drawing one token a row.
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

// One workgroup per slice.  A logit that nothing touches is copied as it is, one that is masked is not read; the table takes 32 KB of LDS, so
// that four workgroups run on a compute unit.  128 rows x 151936 (bf16, histories to 2048, 5 rows of 13 open) take 20 us, 2.8 TB/s: half
// of it instruction issue, half the chain length - history - table - logits in 2.4 rounds of workgroups.  One row of 32000: 6.7 us.
template <Elem E>
__global__ __launch_bounds__(kSliceThreads) void process_logits_kernel(Logits in, LogitRules r, typename Type<E>::bits* out, int64_t out_stride) {
  typedef typename Type<E>::bits bits;
  extern __shared__ __align__(16) char lds[];
  RuleTable& table = *reinterpret_cast<RuleTable*>(lds);
  const int32_t b = (int32_t)blockIdx.y;
  const Row<E> row(in, b);
  const int32_t first = row.first_token((int32_t)blockIdx.x);
  if (first >= in.V) return;
  const bool ruled = has_rules(r);
  const History h = history_ahead(r, b);
  Group<E> x[kGroups];
  uint32_t ok[kGroups];
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
    const int32_t t = first + (j * kSliceThreads + (int32_t)threadIdx.x) * 8;
    ok[j] = allowed_of(r, b, t, in.V);
    x[j] = Group<E>{};
    if (ok[j]) x[j] = load_group(row, t);
  }
  const RowRules rule(r, h, b);  // (read before the barriers of the next)
  if (ruled) gather_rules(r, b, first, h, table);
  bits* const to = out + (int64_t)b * out_stride;
  if (ruled)
    apply_rules(table, rule, ok, first, [&](int k) { return widened<E>(x[k / 8][k % 8]); }, [&](int k, double v) { x[k / 8].set(k % 8, narrowed<E>(v)); });
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
    const int32_t t = first + place_of(8 * j);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!(ok[j] >> i & 1u)) x[j].set(i, narrowed<E>(-__builtin_inff()));
    if (t >= 0 && t + 8 <= in.V && reinterpret_cast<uintptr_t>(to + t) % 16 == 0) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(bits) / 2; ++k)
        reinterpret_cast<uint4*>(to + t)[k] = uint4{x[j].word[4 * k], x[j].word[4 * k + 1], x[j].word[4 * k + 2], x[j].word[4 * k + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (t + i >= 0 && t + i < in.V) to[t + i] = x[j][i];
    }
  }
}
size_t rule_table_bytes(const LogitRules& r) { return has_rules(r) ? sizeof(RuleTable) : 0; }
// slices of a row, wherever it begins
template <Elem E> int32_t slices_of(const Logits& in) {
  constexpr int32_t size = sizeof(typename Type<E>::bits);
  const bool anywhere = reinterpret_cast<uintptr_t>(in.at) % 16 != 0 || in.stride * size % 16 != 0;
  return (int32_t)(((int64_t)in.V + (anywhere ? 16 / size - 1 : 0) + kSliceTokens - 1) / kSliceTokens);
}

// ------------------------------------------------------------------ drawing
// A row's tokens have weights 2^t with t = y log2(e) / temperature, in 64 bits: a wrong token is drawn where a sum is off by
// as much as a random number is close to a border, and a row has 150000 of them.  Sums are taken relative to 2^E, E the octave of the
// largest t of the row or the slice.
// First kernel, one workgroup per slice: logits are read once, the rules and the octave, the largest logit and the sum of the
// slice go into the row's memory; where the row is cut off (top-k, top-p, min-p) also its bins: a quarter of an octave each, 64 octaves
// down, with the number of tokens and the sum of their weights in whole numbers (2^-35 of the bin's octave), which do not depend on
// the order of the atomics.  (That is 2^-36 of a weight at most; more bits, and 8192 tokens of them beside their number, would not fit one atomic of
// 64 bits.)  The workgroup that finishes last for its row puts the slices together.  Without a cut it then
// knows the slice of the drawn token and goes through that one again; with a cut it knows the few bins in which the cuts lie.
// Second kernel, for rows with a cut, one workgroup per slice: the tokens of those bins are listed.  Third, one workgroup per row: it finds the
// cuts among them (where there are too many for the list it goes through the row again each time), the slice and the token.
// What workgroups of one kernel hand to each other goes through atomics of the device, which no cache of an XCD holds back.
// 128 rows x 151936 (top-p, 5 rows of 13 open): 49, 22 and 42 us; instruction issue in 64 bits is 32 of the first's, and the third goes several
// times through the tokens of bins that hold thousands.  One row (top-k, top-p): 18, 8 and 10 us, chains of loads, barriers and selections.  48 rows
// without a cut: 31 us, of which the last slice of a row is done after 17.
constexpr int kWaves = kSliceThreads / 64;
constexpr int kBins = 256, kBinsAnOctave = 4;
constexpr int kMassBits = 35;
constexpr int kCountShift = 50;  // a bin of a slice: number of tokens above, sum of weights below (8192 tokens of less than 2^36)
constexpr u64 kMassMask = (1ull << kCountShift) - 1;
constexpr int kMostCandidates = 16384;

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

struct Slot {  // what a slice leaves
  double E, sum;
  float top;     // -inf: nothing can be drawn
  int32_t top_id;
};
struct RowTotal {  // of a row: its octave, sum, largest logit and its lowest id
  double E, sum;
  float top;
  int32_t top_id;
};
struct RowPlan {  // what the first kernel leaves of a row for the others
  u64 wanted[kBins / 64];  // bins of which they need the tokens
  RowTotal total;
  int32_t cut;       // 0: the row is done
  uint32_t min_key;  // tokens with a smaller key weigh less than min_p
  int32_t reach;     // kept tokens lie in no lighter bin than this one; -1: too many to list them all
  int32_t k_bin, k_need;  // where top-k ends and how many of its tokens there (0: all); k_bin = kBins: nowhere
  double before[kBins + 1];  // mass in front of each bin, in 2^E
};
struct DrawMemory {
  uint32_t *arrived, *n_candidates;  // [rows]: zero between calls
  RowPlan* plans;
  Slot* slots;       // [rows][slices]
  u64* bins;         // [rows][slices][kBins]
  u64* candidates;   // [rows][kMostCandidates]: key, bin, id
  int32_t slices;
};
size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }
int32_t most_slices(int32_t V) { return (V + 7 + kSliceTokens - 1) / kSliceTokens; }
DrawMemory memory_at(void* at, int32_t rows, int32_t V, size_t* bytes) {
  DrawMemory m{};
  m.slices = most_slices(V);
  char* p = static_cast<char*>(at);
  auto take = [&](size_t n) { char* q = p; p += rounded(n); return q; };
  m.arrived = reinterpret_cast<uint32_t*>(take((size_t)rows * 4));
  m.n_candidates = reinterpret_cast<uint32_t*>(take((size_t)rows * 4));
  m.plans = reinterpret_cast<RowPlan*>(take((size_t)rows * sizeof(RowPlan)));
  m.slots = reinterpret_cast<Slot*>(take((size_t)rows * m.slices * sizeof(Slot)));
  m.bins = reinterpret_cast<u64*>(take((size_t)rows * m.slices * kBins * 8));
  m.candidates = reinterpret_cast<u64*>(take((size_t)rows * kMostCandidates * 8));
  *bytes = (size_t)(p - static_cast<char*>(at));
  return m;
}

template <class T> __device__ __forceinline__ void put_out(T* to, T v) { __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class T> __device__ __forceinline__ T take_in(const T* from) { return __hip_atomic_load(const_cast<T*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put_out(Slot* to, const Slot& s) {
  put_out(&to->E, s.E);
  put_out(&to->sum, s.sum);
  put_out(&to->top, s.top);
  put_out(&to->top_id, s.top_id);
}
__device__ __forceinline__ Slot take_in(const Slot* from) { return Slot{take_in(&from->E), take_in(&from->sum), take_in(&from->top), take_in(&from->top_id)}; }

constexpr int kMostSlices = (1 << 20) / kSliceTokens + 1;
constexpr int kFew = 2048;    // candidates that are kept in LDS
constexpr int kRanked = 256;  // and so many are compared each with each
constexpr uint32_t kAtOnce = 1024;  // workgroups of slices that run at once, four to a compute unit
struct Shared {
  double sum[kGroups][kWaves];
  u64 part[kWaves], mass_part[kWaves];
  float top[kWaves];
  int32_t id[kWaves];
  u64 bins[1024];  // of the slice, the row, or a selection
  uint32_t counts[1024];
  double before_mass[kBins + 1];
  uint32_t before_count[kBins + 1];
  Slot slots[kMostSlices];
  double slice_sum[kMostSlices];
  u64 slice_more[kMostSlices];
  uint32_t flag[2];
  int32_t found[2];
  double rest;
  int32_t slice;
  int32_t pick;
  float own[kTokens];  // logits of a thread
  u64 few[kFew];        // (not in the first kernel)
  u64 ranked[kRanked];  // (only in the third)
};

// Whether this workgroup is the last of the row's n to come here; what the others have put out before can be taken in then.
__device__ bool last_of(uint32_t* arrived, uint32_t n, Shared& s) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0);  // (everything put out has arrived)
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before == n - 1) put_out(arrived, 0u);
    s.flag[0] = before == n - 1;
  }
  __syncthreads();
  return s.flag[0] != 0;
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
// v[k], by the steps of a tree (the compiler's own way takes three instructions for each of the 16)
__device__ __forceinline__ float picked(const float (&v)[kTokens], int k) {
  static_assert(kTokens == 16, "four steps");
  float x[kTokens];
#pragma unroll
  for (int i = 0; i < kTokens; ++i) x[i] = v[i];
#pragma unroll
  for (int n = kTokens / 2; n; n >>= 1) {
    const bool upper = k & n;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      float high = x[i + n];
      asm("" : "+v"(high));  // (two elements of one vector are two values here)
      x[i] = upper ? high : x[i];
    }
  }
  return x[0];
}
__device__ __forceinline__ int32_t token_of(int32_t first, int k) { return first + place_of(k); }

// Calls f(logit, token) for the thread's tokens of a slice in order of their ids.  The logits go round in their registers instead of the
// loop being unrolled: what a single workgroup does once costs as much for fetching its instructions as for carrying them out.
template <class F> __device__ __forceinline__ void for_tokens(Tokens& y, int32_t first, F&& f) {
#pragma unroll 1
  for (int k = 0; k < kTokens; ++k) {
    const float v = y[0];
    y = __builtin_shufflevector(y, y, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 0);
    f(v, token_of(first, k), k / 8);
  }
}

// The token of a slice at which the running sum of weights (w of a token's logit and id) first exceeds `rest`, and its logit; the
// last one with a weight if rounding leaves none; -1 if none has any.  The thread in whose eight tokens it lies hands them to eight
// lanes, a token each (one after the other they took 7000 clocks of 15000).
template <class W> __device__ int32_t find_token(Tokens& y, int32_t first, double rest, float* logit, Shared& s, W&& w) {
  static_assert(kGroups == 2, "two groups a thread");
  const int32_t lane = (int32_t)threadIdx.x & 63, wave = (int32_t)threadIdx.x >> 6;
  double run0 = 0.0, run1 = 0.0;
  int32_t last = -1;
#pragma unroll 1
  for (int h = 0; h < kTokens / 4; ++h) {
    double x[4], run = h < 2 ? run0 : run1;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w(y[i], token_of(first, 4 * h + i));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      run += x[i];
      if (x[i] > 0.0) last = token_of(first, 4 * h + i);
    }
    if (h < 2) run0 = run;
    else run1 = run;
    y = __builtin_shufflevector(y, y, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 0, 1, 2, 3);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double other0 = __shfl_up(run0, d), other1 = __shfl_up(run1, d);
    if (lane >= d) { run0 += other0; run1 += other1; }
  }
  __syncthreads();
  if (threadIdx.x == 0) { s.found[0] = INT32_MAX; s.found[1] = -1; }
  if (lane == 63) { s.sum[0][wave] = run0; s.sum[1][wave] = run1; }
  __syncthreads();
  if (last >= 0) atomicMax(&s.found[1], last);
  double base = 0.0, before0 = 0.0, before1 = 0.0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    if (k == wave) before0 = base;
    base += s.sum[0][k];
  }
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    if (k == wave) before1 = base;
    base += s.sum[1][k];
  }
  const double up0 = __shfl_up(run0, 1), up1 = __shfl_up(run1, 1);
  const double at0 = lane ? before0 + up0 : before0, at1 = lane ? before1 + up1 : before1;
  const bool in0 = at0 <= rest && rest < before0 + run0, in1 = at1 <= rest && rest < before1 + run1;
  if (in0 || in1) {  // (one thread: each stretch ends where the next begins)
    s.found[0] = token_of(first, in0 ? 0 : 8);
    s.pick = in0 ? 0 : 8;
    s.rest = in0 ? at0 : at1;
#pragma unroll
    for (int k = 0; k < kTokens; ++k) s.own[k] = y[k];
  }
  __syncthreads();
  const int32_t eight = s.found[0];
  int32_t id = s.found[1];
  if (eight != INT32_MAX) {
    const float v = s.own[s.pick + (lane & 7)];
    const double x = lane < 8 ? w(v, eight + lane) : 0.0;
    double run = x;
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
      const double other = __shfl_up(run, d);
      if (lane >= d) run += other;
    }
    const double up = __shfl_up(run, 1), at = lane ? s.rest + up : s.rest;
    const u64 some = __ballot(x > 0.0), begun = __ballot(x > 0.0 && at <= rest);  // the last whose stretch begins at or before
    const int k = begun ? 63 - __builtin_clzll(begun) : __builtin_ctzll(some | 1ull << 63);
    if (some) id = eight + k;
    *logit = __shfl(v, k);
    if (some) return id;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kTokens; ++k)
    if (token_of(first, k) == id) s.top[0] = y[k];
  __syncthreads();
  *logit = s.top[0];
  return id;
}

struct RowDraw {  // how a row is drawn
  double per, u;  // log2(e) / temperature
  float temperature, top_p, min_p;
  int32_t top_k;
  bool greedy, cut;
  __device__ RowDraw(const DrawRules& d, int32_t b, int32_t V) {
    temperature = d.uniform ? (d.temperature ? d.temperature[b] : 1.0f) : 0.0f;
    greedy = !(temperature > 0.0f);
    if (greedy) temperature = 1.0f;
    per = 1.4426950408889634074 / (double)temperature;
    top_k = d.top_k && d.top_k[b] > 0 && d.top_k[b] < V ? d.top_k[b] : 0;
    top_p = d.top_p && d.top_p[b] < 1.0f ? fmaxf(d.top_p[b], 0.0f) : 1.0f;
    min_p = d.min_p && d.min_p[b] > 0.0f ? fminf(d.min_p[b], 1.0f) : 0.0f;
    cut = !greedy && (top_k > 0 || top_p < 1.0f || min_p > 0.0f);
    u = d.uniform && !greedy ? d.uniform[b] : 0.0;
    if (!(u >= 0.0)) u = 0.0;
    if (u > 1.0) u = 1.0;
  }
};

// The row's largest logit, its lowest id, octave and sum (thread by thread the same), from its slots, which are brought to s.slots;
// the slices' sums relative to the row's octave lie in s.slice_sum.
__device__ RowTotal row_total(const Slot* slots, int32_t n, Shared& s) {
  const int32_t lane = (int32_t)threadIdx.x & 63;
  if ((int32_t)threadIdx.x < n) s.slots[threadIdx.x] = take_in(slots + threadIdx.x);
  __syncthreads();
  RowTotal r{-__builtin_inf(), 0.0, -__builtin_inff(), INT32_MAX};
  for (int32_t i = lane; i < n; i += 64)
    if (s.slots[i].top > -__builtin_inff()) {
      r.top = fmaxf(r.top, s.slots[i].top);
      r.E = fmax(r.E, s.slots[i].E);
    }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    r.top = fmaxf(r.top, __shfl_xor(r.top, d));
    r.E = fmax(r.E, __shfl_xor(r.E, d));
  }
  for (int32_t i = lane; i < n; i += 64) {
    const Slot& one = s.slots[i];
    const bool some = one.top > -__builtin_inff();
    const double d = one.E - r.E, x = some && d > -1000.0 ? ldexp(one.sum, (int)d) : 0.0;
    if (some && one.top == r.top) r.top_id = min(r.top_id, one.top_id);
    r.sum += x;
    if (threadIdx.x < 64) s.slice_sum[i] = x;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) r.top_id = min(r.top_id, __shfl_xor(r.top_id, d));
  r.sum = wave_sum(r.sum);
  __syncthreads();
  return r;
}
// Which slice the random number falls into and what is left of it there.  All threads have read it from `s` when it returns (a last
// barrier sees to that): the tables of the rules may go over it.
struct Place {
  int32_t slice;
  double rest;
};
__device__ Place find_slice(double u, int32_t n, Shared& s) {
  constexpr int kEach = (kMostSlices + 63) / 64;  // neighbours a lane
  const int32_t lane = (int32_t)threadIdx.x;
  if (lane < 64) {
    double x[kEach], run = 0.0;
    int32_t last = -1;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int32_t i = lane * kEach + k;
      x[k] = i < n ? s.slice_sum[i] : 0.0;
      run += x[k];
      if (x[k] > 0.0) last = i;
    }
    double all = run;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double other = __shfl_up(all, d);
      if (lane >= d) all += other;
    }
    const double rest = u * __shfl(all, 63), up = __shfl_up(all, 1), front = lane ? up : 0.0;
    // the last slice with a weight that begins at or before the number
    int32_t at = -1;
    double begin = front, left = 0.0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (x[k] > 0.0 && begin <= rest) { at = lane * kEach + k; left = rest - begin; }
      begin += x[k];
    }
    const u64 who = __ballot(at >= 0), some = __ballot(last >= 0);
    const int owner = who ? 63 - __builtin_clzll(who) : some ? __builtin_ctzll(some) : 0;
    if (lane == owner) {
      s.slice = at >= 0 ? at : max(last, 0);
      s.rest = at >= 0 ? left : 0.0;
    }
  }
  __syncthreads();
  const Place place{s.slice, s.rest};
  __syncthreads();
  return place;
}
// (the sum is taken relative to the weight of the likeliest token as it went into the sum: a token that is alone has logprob 0)
__device__ __forceinline__ void write_out(const RowDraw& d, const RowTotal& r, int32_t id, float y, const double* roots, int32_t* to_id, float* to_logprob) {
  *to_id = id;
  if (to_logprob)
    *to_logprob = id < 0 ? -__builtin_inff()
                         : (float)(((double)y - (double)r.top) / (double)d.temperature - log(r.sum / Power(octaves(r.top, d.per), r.E, roots).weight()));
}

// The row's bins from its slices' into s.bins and s.counts, relative to the octave E, and what lies in front of each (s.before_*;
// masses in 2^E).  All threads, after row_total: half of them take the even slices and half the odd ones.
__device__ void row_bins(const u64* bins, int32_t n, double E, Shared& s) {
  static_assert(kSliceThreads == 2 * kBins, "two threads a bin");
  const int32_t tid = (int32_t)threadIdx.x, bin = tid & (kBins - 1);
  __syncthreads();
  u64 mass = 0;
  uint32_t count = 0;
#pragma unroll 8
  for (int32_t i = tid / kBins; i < n; i += 2) {
    const double d = s.slots[i].top > -__builtin_inff() ? (E - s.slots[i].E) * kBinsAnOctave : (double)kBins;
    const bool some = d <= (double)bin;
    const u64* at = bins + (size_t)i * kBins + (some ? bin - (int32_t)d : 0);
    u64 x = take_in(at);
    if (!some) x = 0;
    mass += x & kMassMask;
    count += (uint32_t)(x >> kCountShift);
  }
  if (tid < kBins) { s.bins[tid] = mass; s.counts[tid] = count; }
  __syncthreads();
  if (tid >= kBins) { s.bins[bin] += mass; s.counts[bin] += count; }
  __syncthreads();
  if (tid < 64) {  // one wave: four bins a lane, an octave
    const double scale = ldexp(1.0, -kMassBits - tid);
    double m[4], run = 0.0;
    uint32_t c[4], total = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = run;
      c[k] = total;
      run += (double)s.bins[tid * 4 + k] * scale;
      total += s.counts[tid * 4 + k];
    }
    double all = run;
    uint32_t all_count = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double other = __shfl_up(all, d);
      const uint32_t other_count = __shfl_up(all_count, d);
      if (tid >= d) { all += other; all_count += other_count; }
    }
    double in_front = __shfl_up(all, 1);
    uint32_t count_in_front = __shfl_up(all_count, 1);
    if (tid == 0) { in_front = 0.0; count_in_front = 0; }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s.before_mass[tid * 4 + k] = in_front + m[k];
      s.before_count[tid * 4 + k] = count_in_front + c[k];
    }
    if (tid == 63) { s.before_mass[kBins] = all; s.before_count[kBins] = all_count; }
  }
  __syncthreads();
}
// the first bin up to and with which at least `count` tokens, or `mass`, lie; kBins - 1 if there are fewer
__device__ int32_t bin_of_count(const Shared& s, uint32_t count) {
  int32_t lo = 0, hi = kBins - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi) / 2;
    if (s.before_count[mid + 1] >= count) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}
__device__ int32_t bin_of_mass(const Shared& s, double mass) {
  mass = fmax(mass, DBL_MIN);  // (at least one token)
  int32_t lo = 0, hi = kBins - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi) / 2;
    if (s.before_mass[mid + 1] >= mass) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}
// The smallest key whose weight is min_p of the largest or more: the logarithm says about where, the exponential function where.  The
// first guess is a key or two off, unless the border lies near a logit of 0, where many keys have one weight: steps that
// double, then halves.
__device__ uint32_t key_of_min(const RowDraw& d, float top) {
  if (!(d.min_p > 0.0f)) return 0;
  const double t = (double)d.temperature;
  auto enough = [&](uint32_t key) { return exp(((double)value_of(key) - (double)top) / t) >= (double)d.min_p; };
  const uint32_t most = key_of(top);
  const uint32_t guess = min(key_of((float)fmax((double)top + t * log((double)d.min_p), -(double)FLT_MAX)), most);
  const bool down = enough(guess);
  uint32_t good = down ? guess : most, bad = down ? key_of(-FLT_MAX) - 1 : guess, step = 1;
  bool doubling = true;
#pragma unroll 1
  while (good - bad > 1) {
    const uint32_t width = good - bad, at = !doubling || step >= width ? bad + width / 2 : down ? good - step : bad + step;
    const bool is = enough(at);
    if (is) good = at;
    else bad = at;
    doubling = doubling && is == down && step < width;
    step *= 2;
  }
  return good;
}

template <Elem E>
__global__ __launch_bounds__(kSliceThreads, 8) void draw_slices_kernel(Logits in, LogitRules r, DrawRules dr, DrawMemory m, int32_t n_slices, int32_t* __restrict__ ids,
                                                                    float* __restrict__ logprobs) {
  extern __shared__ __align__(16) char lds[];
  RuleTable& table = *reinterpret_cast<RuleTable*>(lds);
  Shared& s = *reinterpret_cast<Shared*>(lds);
  __shared__ double roots[16];
  const int32_t b = (int32_t)blockIdx.y, slice = (int32_t)blockIdx.x, tid = (int32_t)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Row<E> row(in, b);
  const RowDraw d(dr, b, in.V);
  Slot* const slots = m.slots + (size_t)b * m.slices;
  u64* const bins = m.bins + (size_t)b * m.slices * kBins;
  int32_t first = row.first_token(slice);
  Tokens y;
  fill_roots(roots);
  load_slice<E>(row, r, b, first, table, y);

  float top = -__builtin_inff();
  int at = -1;
#pragma unroll
  for (int k = 0; k < kTokens; ++k)
    if (y[k] > top) { top = y[k]; at = k; }
  int32_t top_id = at < 0 ? -1 : token_of(first, at);
#pragma unroll
  for (int k = 32; k; k >>= 1) {
    const float other = __shfl_xor(top, k);
    const int32_t other_id = __shfl_xor(top_id, k);
    if (other > top || (other == top && (uint32_t)other_id < (uint32_t)top_id)) { top = other; top_id = other_id; }
  }
  if (lane == 0) { s.top[wave] = top; s.id[wave] = top_id; }
  if (d.cut && tid < kBins) s.bins[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWaves; ++k)
    if (s.top[k] > top || (s.top[k] == top && (uint32_t)s.id[k] < (uint32_t)top_id)) { top = s.top[k]; top_id = s.id[k]; }
  Slot slot{0.0, 0.0, top, top_id};
  if (top > -__builtin_inff()) {
    slot.E = floor(octaves(top, d.per));
    double sum = 0.0;
    auto add = [&](float v) {
      if (!(v > -__builtin_inff())) return;
      const double t = octaves(v, d.per);
      const Power w(t, slot.E, roots);
      sum += w.weight();
      if (d.cut) {
        const int32_t bin = w.bin();
        if (bin < kBins) atomicAdd(&s.bins[bin], w.mass() + (1ull << kCountShift));
      }
    };
#pragma unroll 1
    for (int h = 0; h < kTokens / 4; ++h) {
      add(y[0]); add(y[1]); add(y[2]); add(y[3]);
      y = __builtin_shufflevector(y, y, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 0, 1, 2, 3);
    }
    sum = wave_sum(sum);
    if (lane == 0) s.sum[0][wave] = sum;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) slot.sum += s.sum[0][k];
  }
  if (tid == 0) put_out(slots + slice, slot);
  if (d.cut && tid < kBins) put_out(bins + (size_t)slice * kBins + tid, s.bins[tid]);
  if (!last_of(m.arrived + b, (uint32_t)n_slices, s)) return;

  const RowTotal total = row_total(slots, n_slices, s);
  const bool empty = total.top == -__builtin_inff();
  if (empty || !d.cut) {
    int32_t id = empty ? -1 : total.top_id;
    float logit = total.top;
    if (!empty && !d.greedy) {
      const Place place = find_slice(d.u, n_slices, s);
      first = row.first_token(place.slice);
      load_slice<E>(row, r, b, first, table, y);
      id = find_token(y, first, place.rest, &logit, s, [&](float v, int32_t) { return v > -__builtin_inff() ? Power(octaves(v, d.per), total.E, roots).weight() : 0.0; });
    }
    if (tid == 0) {
      write_out(d, total, id, logit, roots, ids + b, logprobs ? logprobs + b : nullptr);
      m.plans[b].cut = 0;
    }
    return;
  }
  // the bins in which a cut can lie: that of the k-th token unless it ends there, those of p of what lies up to it, that of min_p
  row_bins(bins, n_slices, total.E, s);
  if (tid == 0) {
    RowPlan plan;
    plan.k_need = 0;
    plan.total = total;
    plan.cut = 1;
    plan.k_bin = kBins;
    plan.min_key = key_of_min(d, total.top);
    int32_t from = kBins, to = -1, k_bin = -1, low = -1;
    double least = s.before_mass[kBins], most = least;
    int32_t last = kBins - 1;
    if (d.top_k && (uint32_t)d.top_k < s.before_count[kBins]) {
      last = plan.k_bin = bin_of_count(s, (uint32_t)d.top_k);
      most = s.before_mass[last + 1];
      least = most;
      if ((uint32_t)d.top_k != s.before_count[last + 1]) {
        k_bin = last;
        plan.k_need = d.top_k - (int32_t)s.before_count[last];
        least = s.before_mass[last];
      }
    }
    if (d.top_p < 1.0f) {
      from = bin_of_mass(s, (double)d.top_p * least * (1.0 - 1e-9));
      to = min(last, bin_of_mass(s, fmin((double)d.top_p * most * (1.0 + 1e-9), s.before_mass[kBins])));
      from = min(from, to);
    }
    if (plan.min_key) {
      low = Power(octaves(value_of(plan.min_key), d.per), total.E, roots).bin();
    }
    // Where few tokens are kept they are listed, all of them, and one is drawn from the list: one row of 151936 with top-k 50 takes 37 us
    // that way and 44 by the slices' sums.  Not where the batch has more slices than run at once: the list is then bound by how many slices
    // have something to list (128 rows, top-p: 116 us and 111).
    plan.reach = min(last, min(d.top_p < 1.0f ? to : kBins - 1, plan.min_key ? min(low, kBins - 1) : kBins - 1));
    if (s.before_count[plan.reach + 1] > kRanked || gridDim.x * gridDim.y > kAtOnce) plan.reach = -1;
#pragma unroll
    for (int k = 0; k < kBins / 64; ++k) {
      const int32_t lo = max(from - 64 * k, 0), hi = min(to - 64 * k, 63);
      u64 bits = lo <= hi ? (~0ull << lo) & (~0ull >> (63 - hi)) : 0;
      if (plan.reach >= 64 * k) bits |= ~0ull >> (63 - min(plan.reach - 64 * k, 63));
      if (k_bin >= 0 && k_bin / 64 == k) bits |= 1ull << (k_bin & 63);
      if (low >= 0 && low / 64 == k) bits |= 1ull << (low & 63);
      plan.wanted[k] = bits;
    }
    RowPlan& out = m.plans[b];
#pragma unroll
    for (int k = 0; k < kBins / 64; ++k) out.wanted[k] = plan.wanted[k];
    out.total = plan.total;
    out.cut = 1;
    out.min_key = plan.min_key;
    out.k_bin = plan.k_bin;
    out.k_need = plan.k_need;
    out.reach = plan.reach;
  }
  if (tid <= kBins) m.plans[b].before[tid] = s.before_mass[tid];
}

// A range of keys that holds the tokens of the bins first .. last: where the bins' borders lie, and two keys more at both ends for
// what the divisions round.
struct KeyRange { uint32_t lo, hi; };
__device__ KeyRange keys_of_bins(int32_t first, int32_t last, double E, double per) {
  if (!(per > 0.0)) return KeyRange{0, ~0u};
  const double t_hi = E + 1.0 - (double)first / kBinsAnOctave, t_lo = E + 1.0 - (double)(last + 1) / kBinsAnOctave;
  const float hi = (float)fmin(fmax(t_hi / per, -(double)FLT_MAX), (double)FLT_MAX), lo = (float)fmin(fmax(t_lo / per, -(double)FLT_MAX), (double)FLT_MAX);
  const uint32_t a = key_of(lo), b = key_of(hi);
  return KeyRange{a > 2 ? a - 2 : 0, b < ~0u - 2 ? b + 2 : ~0u};
}

// Goes through the tokens of the wanted bins: f(key, bin, id).  All threads; `listed` of them, a few in s.few, or more than the list holds.
template <Elem E, class F>
__device__ __forceinline__ void for_candidates(const Row<E>& row, const LogitRules& r, const RowDraw& d, const RowPlan& plan, int32_t b, int32_t n_slices, const u64* list,
                                               uint32_t listed, RuleTable& table, const Shared& s, const uint32_t* wanted, const double* roots, F&& f) {
  if (listed <= kMostCandidates) {
    constexpr int kAhead = 4;
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < listed; i += kAhead * kSliceThreads) {
      u64 x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint32_t at = min(i + k * kSliceThreads, listed - 1);
        x[k] = listed <= kFew ? s.few[at] : list[at];
      }
#pragma unroll 1
      for (uint32_t at = i; at < i + kAhead * kSliceThreads && at < listed; at += kSliceThreads) {
        f((uint32_t)(x[0] >> 32), (int32_t)(x[0] >> 24 & 255u), (int32_t)(x[0] & 0xffffffu));
#pragma unroll
        for (int k = 1; k < kAhead; ++k) x[k - 1] = x[k];
      }
    }
    return;
  }
  for (int32_t slice = 0; slice < n_slices; ++slice) {
    const int32_t first = row.first_token(slice);
    Tokens y;
    __syncthreads();  // (the tables of the last slice have been read)
    load_slice<E>(row, r, b, first, table, y);
    for_tokens(y, first, [&](float v, int32_t id, int) {
      if (!(v > -__builtin_inff())) return;
      const int32_t bin = Power(octaves(v, d.per), plan.total.E, roots).bin();
      if (bin < kBins && (wanted[bin / 32] >> (bin & 31) & 1u)) f(key_of(v), bin, id);
    });
  }
}

// The end of a beginning of the row's order: tokens of heavier bins, and of `bin` those with a larger key and of those with `key`
// the ones up to `id`.
struct Cut {
  int32_t bin;
  uint32_t key;
  int32_t id;
  __device__ __forceinline__ bool keeps(int32_t in, uint32_t k, int32_t i) const { return (in < bin) | ((in == bin) & ((k > key) | ((k == key) & (i <= id)))); }
};

template <Elem E>
__global__ __launch_bounds__(kSliceThreads) void draw_list_kernel(Logits in, LogitRules r, DrawRules dr, DrawMemory m) {
  extern __shared__ __align__(16) char lds[];
  RuleTable& table = *reinterpret_cast<RuleTable*>(lds);
  __shared__ uint32_t wanted[kBins / 32];
  __shared__ double roots[16];
  Shared& s = *reinterpret_cast<Shared*>(lds);
  const int32_t b = (int32_t)blockIdx.y, slice = (int32_t)blockIdx.x, tid = (int32_t)threadIdx.x;
  const RowPlan& plan = m.plans[b];
  if (!plan.cut) return;
  const Row<E> row(in, b);
  const RowDraw d(dr, b, in.V);
  u64* const list = m.candidates + (size_t)b * kMostCandidates;
  Tokens y;

  // the tokens of the wanted bins, if the slice has any
  fill_roots(roots);
  if (tid == 0) s.flag[1] = 0;
  if (tid < kBins / 32) wanted[tid] = reinterpret_cast<const uint32_t*>(plan.wanted)[tid];
  const double E_row = plan.total.E;
  const Slot slot = m.slots[(size_t)b * m.slices + slice];
  __syncthreads();
  if (slot.top > -__builtin_inff() && tid < kBins && (wanted[tid / 32] >> (tid & 31) & 1u)) {
    const double at = (double)tid - (E_row - slot.E) * kBinsAnOctave;
    if (at >= 0.0 && m.bins[((size_t)b * m.slices + slice) * kBins + (int32_t)at] >> kCountShift) s.flag[1] = 1;
  }
  __syncthreads();
  if (!s.flag[1]) return;
  int32_t lightest = -1, heaviest = kBins;
#pragma unroll
  for (int k = 0; k < kBins / 64; ++k) {
    const u64 bits = plan.wanted[k];
    if (bits) lightest = k * 64 + 63 - __builtin_clzll(bits);
    if (bits && heaviest == kBins) heaviest = k * 64 + __builtin_ctzll(bits);
  }
  const KeyRange range = keys_of_bins(heaviest, lightest, E_row, d.per);
  const int32_t first = row.first_token(slice);
  __syncthreads();
  load_slice<E>(row, r, b, first, table, y);
  if (tid == 0) s.flag[0] = 0;
  __syncthreads();
  // (two comparisons a token; the few in the range one by one)
  const float least = value_of(max(range.lo, key_of(-FLT_MAX))), most = value_of(min(range.hi, key_of(FLT_MAX)));
  uint32_t in_range = 0;
  float all[kTokens];
#pragma unroll
  for (int k = 0; k < kTokens; ++k) {
    all[k] = y[k];
    in_range |= (all[k] >= least) & (all[k] <= most) ? 1u << k : 0u;
  }
#pragma unroll 1
  for (; in_range; in_range &= in_range - 1) {
    const int k = __builtin_ctz(in_range);
    const float v = picked(all, k);
    const uint32_t key = key_of(v);
    const int32_t id = token_of(first, k), bin = Power(octaves(v, d.per), E_row, roots).bin();
    if (bin >= kBins || !(wanted[bin / 32] >> (bin & 31) & 1u)) continue;
    const u64 x = (u64)key << 32 | (u64)bin << 24 | (u64)(uint32_t)id;
    const uint32_t at = atomicAdd(&s.flag[0], 1u);
    if (at < kFew) {
      s.few[at] = x;
    } else {  // (more than the workgroup collects: one by one)
      const uint32_t place = atomicAdd(m.n_candidates + b, 1u);
      if (place < kMostCandidates) list[place] = x;
    }
  }
  __syncthreads();
  const uint32_t n = min(s.flag[0], (uint32_t)kFew);
  if (tid == 0 && n) s.counts[0] = atomicAdd(m.n_candidates + b, n);
  __syncthreads();
  for (uint32_t i = (uint32_t)tid; i < n; i += kSliceThreads)
    if (s.counts[0] + i < kMostCandidates) list[s.counts[0] + i] = s.few[i];
}

// One workgroup per row with a cut: the cuts among the listed tokens, the slice and the token.
template <Elem E>
__global__ __launch_bounds__(kSliceThreads) void draw_cut_kernel(Logits in, LogitRules r, DrawRules dr, DrawMemory m, int32_t n_slices, int32_t* __restrict__ ids,
                                                                 float* __restrict__ logprobs) {
  extern __shared__ __align__(16) char lds[];
  RuleTable& table = *reinterpret_cast<RuleTable*>(lds);
  __shared__ Shared s;
  __shared__ uint32_t wanted[kBins / 32];
  __shared__ double roots[16];
  const int32_t b = (int32_t)blockIdx.x, tid = (int32_t)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const RowPlan& plan = m.plans[b];
  const Row<E> row(in, b);
  const RowDraw d(dr, b, in.V);
  const Slot* const slots = m.slots + (size_t)b * m.slices;
  const u64* const bins = m.bins + (size_t)b * m.slices * kBins;
  const u64* const list = m.candidates + (size_t)b * kMostCandidates;
  const RowTotal total = plan.total;
  const uint32_t min_key = plan.min_key, listed = m.n_candidates[b];
  const double in_front = plan.before[min(tid, kBins)];
  const uint32_t some = reinterpret_cast<const uint32_t*>(plan.wanted)[min(tid, kBins / 32 - 1)];
  const Slot slot = slots[min(tid, n_slices - 1)];
  u64 few[kFew / kSliceThreads];  // (all are read, so that it need not be known how many there are)
#pragma unroll
  for (int k = 0; k < kFew / kSliceThreads; ++k) few[k] = list[k * kSliceThreads + tid];
  if (!plan.cut) return;
  Tokens y;
  fill_roots(roots);
  if (tid <= kBins) s.before_mass[tid] = in_front;
  if (tid < n_slices) s.slots[tid] = slot;
  if (tid < kBins / 32) wanted[tid] = some;
#pragma unroll
  for (int k = 0; k < kFew / kSliceThreads; ++k) s.few[k * kSliceThreads + tid] = few[k];
  const int32_t reach = plan.reach;
  int32_t k_bin = plan.k_bin, in_bin = plan.k_need ? k_bin : -1;  // in_bin: where the cut of a selection lies
  u64 need = (u64)plan.k_need;  // what the rest of the kept beginning has to reach there: tokens, or mass in the bin's whole numbers
  Cut cut{k_bin, 0, INT32_MAX};
  __syncthreads();
  if (tid == 0) m.n_candidates[b] = 0;
  double up_to = s.before_mass[min(k_bin, kBins - 1) + 1];
  k_bin = min(k_bin, kBins - 1);
  const int32_t low = min_key ? Power(octaves(value_of(min_key), d.per), total.E, roots).bin() : kBins;
  auto kept = [&](uint32_t key, int32_t bin, int32_t id) { return (key >= min_key) & cut.keeps(bin, key, id); };

  // Two selections, top-k and top-p of what it keeps, then the sums of the slices.  A selection goes through the tokens of its bin that
  // are kept so far: passes that sort them into 1024 stretches of their range of keys, and then of ids among the tokens with one
  // key, and narrow the range to the stretch in which the need is reached, until few are left; each of those is then compared with all others.
  // (where few tokens are kept, they are collected and one of them drawn instead of the sums)
  enum { kKeys, kIds, kRank, kSums, kKept };
  int mode = kKeys, what = 0;
  bool begins = true, divided = false;
  Cut within = cut;
  uint32_t lo = 0, hi = 0, left = 0;
  int32_t first_id = 0, last_id = 0, shift = 0, edge = kBins;
  u64 up_to_key = 0, key_mass = 0;
  const int32_t row_first = row.first_token(0);
#pragma unroll 1
  for (int step = 0; step < 32; ++step) {  // (a selection takes 4 + 3 + 1 at most)
    if (begins) {
      begins = false;
      if (what == 0 && in_bin < 0) what = 1;
      if (what == 1) {
        in_bin = -1;
        if (d.top_p < 1.0f) {
          const double target = (double)d.top_p * up_to;
          const int32_t p_bin = min(k_bin, bin_of_mass(s, target));
          const double inside = ldexp(target - s.before_mass[p_bin], kMassBits + p_bin / kBinsAnOctave);
          need = inside >= 1.0 ? (u64)ceil(inside) : 1u;
          if (wanted[p_bin / 32] >> (p_bin & 31) & 1u) in_bin = p_bin;
        }
        if (in_bin < 0) what = 2;
      }
      __syncthreads();
      if (what < 2) {
        const KeyRange range = keys_of_bins(in_bin, in_bin, total.E, d.per);
        lo = range.lo;
        hi = range.hi;
        first_id = 0;
        last_id = in.V - 1;
        within = cut;
        up_to_key = 0;
        mode = kKeys;
        left = listed;
      } else {
        // bins in front of the edge count as they are, the edge's tokens one by one if it is divided
        mode = kSums;
        edge = min(cut.bin, low);
        if (reach >= 0) {
          mode = kKept;
          if (tid == 0) s.flag[0] = 0;
          if (tid < kRanked) { s.ranked[tid] = ~0ull; s.bins[tid] = 0; }
        } else {
          divided = edge < kBins && (edge == low || cut.key != 0 || cut.id != INT32_MAX);
          for (int32_t i = tid; i < n_slices; i += kSliceThreads) s.slice_more[i] = 0;
          if (!divided) break;
        }
      }
    }
    if (mode < kSums && left <= kRanked) {
      mode = kRank;
      if (tid == 0) { s.flag[0] = 0; s.found[0] = -1; }
      if (tid < kRanked) { s.ranked[tid] = ~0ull; s.bins[tid] = 0; }
    } else if (mode < kSums) {
      s.bins[tid] = s.bins[tid + kSliceThreads] = 0;
      s.counts[tid] = s.counts[tid + kSliceThreads] = 0;
      const uint32_t width = mode == kKeys ? hi - lo : (uint32_t)(last_id - first_id);
      shift = width < 1024 ? 0 : 22 - __clz((int)width);
    }
    __syncthreads();
    for_candidates<E>(row, r, d, plan, b, n_slices, list, listed, table, s, wanted, roots, [&](uint32_t key, int32_t bin, int32_t id) {
      if (mode == kKept) {
        if ((bin <= reach) & kept(key, bin, id)) {  // (kRanked of them at most: so many lie in these bins)
          const uint32_t at = atomicAdd(&s.flag[0], 1u);
          s.ranked[at] = (u64)(uint32_t)id << 32 | key;
          s.bins[at] = (u64)(Power(octaves(value_of(key), d.per), total.E, roots).weight() * 4503599627370496.0);
        }
        return;
      }
      if (mode == kSums) {
        if (bin == edge && kept(key, bin, id)) atomicAdd(&s.slice_more[(uint32_t)(id - row_first) / kSliceTokens], Power(octaves(value_of(key), d.per), total.E, roots).mass());
        return;
      }
      if (bin != in_bin || !within.keeps(bin, key, id) || key > hi || key < lo || id < first_id || id > last_id) return;
      const u64 mass = mode != kIds ? Power(octaves(value_of(key), d.per), total.E, roots).mass() : 0;
      if (mode == kRank) {
        const uint32_t at = atomicAdd(&s.flag[0], 1u);
        s.ranked[at] = (u64)~key << 32 | (uint32_t)id;
        s.bins[at] = mass;
        return;
      }
      const uint32_t at = mode == kKeys ? (hi - key) >> shift : (uint32_t)(id - first_id) >> shift;
      atomicAdd(&s.counts[at], 1u);
      if (mode == kKeys) atomicAdd(&s.bins[at], mass);
    });
    if (mode >= kSums) break;
    __syncthreads();
    if (mode == kRank) {
      const uint32_t n = s.flag[0];
      if (n > 0 && (uint32_t)tid < n) {
        const u64 mine = s.ranked[tid], own = s.bins[tid];
        u64 before = 0, whole = 0;
        uint32_t rank = 0;
#pragma unroll 1
        for (uint32_t i = 0; i < n; i += 8) {
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k) {
            const u64 x = s.bins[i + k];
            const bool front = s.ranked[i + k] < mine;
            before += front ? x : 0;
            rank += front ? 1 : 0;
            whole += x;
          }
        }
        // (rounding can leave a need above what there is: the last token then)
        const u64 wanted = min(max(need, (u64)1), what == 0 ? (u64)n : whole), at = what == 0 ? (u64)rank : before;
        if (at < wanted && wanted <= at + (what == 0 ? 1 : own)) {
          s.found[0] = tid;
          s.part[0] = before + own;
        }
      }
      __syncthreads();
      const int32_t at = s.found[0];
      if (at >= 0) {
        cut = Cut{in_bin, ~(uint32_t)(s.ranked[at] >> 32), (int32_t)(uint32_t)s.ranked[at]};
        up_to = s.before_mass[in_bin] + ldexp((double)(up_to_key + s.part[0]), -kMassBits - in_bin / kBinsAnOctave);
      }
      ++what;
      begins = true;
      continue;
    }
    // the stretch with the need: two neighbours a thread
    const bool counted = what == 0 || mode == kIds;
    const u64 m0 = s.bins[2 * tid], m1 = s.bins[2 * tid + 1];
    const uint32_t c0 = s.counts[2 * tid], c1 = s.counts[2 * tid + 1];
    const u64 v0 = counted ? (u64)c0 : m0, v1 = counted ? (u64)c1 : m1;
    u64 all = v0 + v1, all_mass = m0 + m1;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) {
      const u64 other = __shfl_up(all, e), other_mass = __shfl_up(all_mass, e);
      if (lane >= e) { all += other; all_mass += other_mass; }
    }
    if (lane == 63) { s.part[wave] = all; s.mass_part[wave] = all_mass; }
    if (tid == 0) s.found[0] = -1;
    __syncthreads();
    u64 whole = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      if (k < wave) { all += s.part[k]; all_mass += s.mass_part[k]; }
      whole += s.part[k];
    }
    need = min(max(need, (u64)1), whole);
    const u64 begin = all - v0 - v1;
    __syncthreads();
    if (begin < need && need <= all) {
      const bool second = need > begin + v0;
      s.found[0] = 2 * tid + (second ? 1 : 0);
      s.part[0] = begin + (second ? v0 : 0);  // in front of the stretch
      s.part[1] = all_mass - m0 - m1 + (second ? m0 : 0);
      s.part[2] = second ? m1 : m0;
      s.flag[0] = second ? c1 : c0;
    }
    __syncthreads();
    const int32_t at = s.found[0];
    if (at < 0) {  // (no token at all)
      ++what;
      begins = true;
      continue;
    }
    left = s.flag[0];
    if (mode == kKeys) {
      need -= s.part[0];
      up_to_key += s.part[1];
      const uint32_t floor_key = lo;
      hi -= (uint32_t)at << shift;
      lo = shift == 0 ? hi : max(floor_key, hi - ((1u << shift) - 1u));
      if (hi == lo && left > kRanked) {
        // one key: of its tokens the first so many
        key_mass = s.part[2] / left;
        if (what == 1) need = (need + key_mass - 1) / max(key_mass, (u64)1);
        need = min(max(need, (u64)1), (u64)left);
        mode = kIds;
      }
    } else {
      need -= s.part[0];
      up_to_key += s.part[0] * key_mass;
      first_id += at << shift;
      last_id = min(last_id, first_id + (1 << shift) - 1);
      if (left <= kRanked && what == 1) need *= key_mass;  // (in mass again for the comparison)
    }
    __syncthreads();
  }
  __syncthreads();
  if (reach >= 0) {
    // weights in whole numbers of 2^-52 of the octave, so that the order in which they were collected does not matter
    const uint32_t n = s.flag[0];
    if (tid == 0) s.found[0] = -1;
    __syncthreads();
    if ((uint32_t)tid < n) {
      const u64 mine = s.ranked[tid], own = s.bins[tid];
      u64 before = 0, whole = 0;
      bool last = true;  // of those with a weight
#pragma unroll 1
      for (uint32_t i = 0; i < n; i += 8) {
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
          const u64 x = s.bins[i + k];
          const bool front = s.ranked[i + k] < mine;
          before += front ? x : 0;
          whole += x;
          last &= (s.ranked[i + k] <= mine) | (x == 0);
        }
      }
      const u64 rest = (u64)(d.u * (double)whole);
      if (own != 0 && before <= rest && (rest < before + own || last)) s.found[0] = tid;
    }
    __syncthreads();
    if (tid == 0) {
      const u64 it = s.found[0] >= 0 ? s.ranked[s.found[0]] : (u64)(uint32_t)total.top_id << 32 | key_of(total.top);
      write_out(d, total, (int32_t)(it >> 32), value_of((uint32_t)it), roots, ids + b, logprobs ? logprobs + b : nullptr);
    }
    return;
  }
  const double up_to_bin = (double)(divided ? edge : min(edge + 1, kBins));
  constexpr int kTogether = 3;  // slices of a wave whose bins are on their way together
#pragma unroll 1
  for (int32_t begin = wave; begin < n_slices; begin += kTogether * kWaves) {
    u64 x[kTogether][kBins / 64];
#pragma unroll
    for (int j = 0; j < kTogether; ++j)
#pragma unroll
      for (int k = 0; k < kBins / 64; ++k) x[j][k] = bins[(size_t)min(begin + j * kWaves, n_slices - 1) * kBins + k * 64 + lane];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int32_t i = begin + j * kWaves;
      if (i >= n_slices) break;
      double sum = 0.0;
      if (s.slots[i].top > -__builtin_inff()) {
        const double off = (total.E - s.slots[i].E) * kBinsAnOctave;  // of the slice's bins in the row's
#pragma unroll
        for (int k = 0; k < kBins / 64; ++k) {
          const double at = off + (double)(k * 64 + lane);
          if (at < up_to_bin) sum += ldexp((double)(x[j][k] & kMassMask), -kMassBits - (int32_t)at / kBinsAnOctave);
        }
      }
      sum = wave_sum(sum);
      if (lane == 0) s.slice_sum[i] = sum + (divided ? ldexp((double)s.slice_more[i], -kMassBits - edge / kBinsAnOctave) : 0.0);
    }
  }
  __syncthreads();
  const Place place = find_slice(d.u, n_slices, s);
  const int32_t first = row.first_token(place.slice);
  load_slice<E>(row, r, b, first, table, y);
  float logit = 0.0f;
  // of what is kept, all of which is above -inf
  const uint32_t least_key = max(max(max(min_key, cut.key), keys_of_bins(edge, min(edge, kBins - 1), total.E, d.per).lo), key_of(-FLT_MAX));
  const int32_t id = find_token(y, first, place.rest, &logit, s, [&](float v, int32_t token) {
    const uint32_t key = key_of(v);
    double x = 0.0;
    if (key >= least_key) {
      const Power w(octaves(v, d.per), total.E, roots);
      const int32_t bin = w.bin();
      x = (bin < kBins) & kept(key, bin, token) ? w.weight() : 0.0;
    }
    return x;
  });
  if (tid == 0) write_out(d, total, id, logit, roots, ids + b, logprobs ? logprobs + b : nullptr);
}

template <template <Elem> class Launch, class... Args>
hipError_t by_type(Elem e, const Args&... args) {
  if (e == Elem::kF32) return Launch<Elem::kF32>::run(args...);
  if (e == Elem::kBF16) return Launch<Elem::kBF16>::run(args...);
  return Launch<Elem::kF16>::run(args...);
}
template <Elem E> struct Process {
  static hipError_t run(const Logits& in, const int32_t& B, const LogitRules& r, void* const& out, const int64_t& out_stride, const hipStream_t& stream) {
    hipLaunchKernelGGL(process_logits_kernel<E>, dim3(slices_of<E>(in), B), dim3(kSliceThreads), rule_table_bytes(r), stream, in, r,
                       static_cast<typename Type<E>::bits*>(out), out_stride);
    return hipGetLastError();
  }
};
// LDS of a kernel that has no use for its tables any more when it needs the first `bytes` of Shared
size_t lds_with(const LogitRules& r, size_t bytes) { return bytes < rule_table_bytes(r) ? rule_table_bytes(r) : bytes; }
template <Elem E> struct Draw {
  static hipError_t run(const Logits& in, const int32_t& B, const LogitRules& r, const DrawRules& d, const DrawMemory& m, int32_t* const& ids, float* const& logprobs,
                        const hipStream_t& stream) {
    // (the only one of the three that takes a table and Shared at once, 70 KB)
    static LdsRoom room;
    if (const hipError_t e = room(reinterpret_cast<const void*>(&draw_cut_kernel<E>), sizeof(RuleTable)); e != hipSuccess) return e;
    const int32_t n = slices_of<E>(in);
    hipLaunchKernelGGL(draw_slices_kernel<E>, dim3(n, B), dim3(kSliceThreads), lds_with(r, offsetof(Shared, few)), stream, in, r, d, m, n, ids, logprobs);
    if (!d.uniform || !(d.top_k || d.top_p || d.min_p)) return hipGetLastError();
    hipLaunchKernelGGL(draw_list_kernel<E>, dim3(n, B), dim3(kSliceThreads), lds_with(r, offsetof(Shared, ranked)), stream, in, r, d, m);
    hipLaunchKernelGGL(draw_cut_kernel<E>, dim3(B), dim3(kSliceThreads), rule_table_bytes(r), stream, in, r, d, m, n, ids, logprobs);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_process_logits(const Logits& in, Elem type, int32_t B, const LogitRules& rules, void* out, int64_t out_stride, hipStream_t stream) {
  return by_type<Process>(type, in, B, rules, out, out_stride, stream);
}

size_t sampler_bytes(int32_t max_rows, int32_t V) {
  size_t bytes = 0;
  memory_at(nullptr, max_rows, V, &bytes);
  return bytes;
}

hipError_t launch_sample(const Logits& in, Elem type, int32_t B, const LogitRules& rules, const DrawRules& draw, void* memory, int32_t max_rows, int32_t max_V,
                         int32_t* ids, float* logprobs, hipStream_t stream) {
  size_t bytes = 0;
  return by_type<Draw>(type, in, B, rules, draw, memory_at(memory, max_rows, max_V, &bytes), ids, logprobs, stream);
}

}  // namespace xgm
