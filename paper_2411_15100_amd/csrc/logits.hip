// What lies behind the mask in a decode step (sections 2.1 and 3.5: the mask goes
// to masked sampling): rules on logits, and drawing one token a row.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cstdint>

#include "elements.hpp"
#include "logits.hpp"

namespace xgm {

namespace {

// ------------------------------------------------------------ a slice of a row
// A workgroup takes kSliceTokens tokens of a row, a thread two groups of 8 neighbours.  A slice begins on 16 bytes, up to a group less
// one token in front of a row that does not, so that a group is one load of 16 bytes (two of them in 32 bits); groups that reach over
// an end of the row are taken token by token.
constexpr int kSliceThreads = 512, kSliceTokens = 8192, kGroups = kSliceTokens / 8 / kSliceThreads;

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
// The history and the biases of row b in the tokens [first, first + kSliceTokens), as two tables: how often a token was
// generated, with the top bit if it occurs in the prompt, and which entry of the row's biases is the token's (0: none).
// Counts are whole numbers and of the entries the last wins, so the order of the atomics does not matter.
// The first tokens of the history are read before its length is known (they lie in the row's memory whatever it is).
constexpr int kHistoryAhead = 4;
struct History {
  int32_t token[kHistoryAhead], n, prompt;
};
__device__ __forceinline__ History history_ahead(const LogitRules& r, int32_t b) {
  History h{};
  if (!r.tokens) return h;
  const int32_t* tokens = r.tokens + (int64_t)b * r.token_stride;
  h.n = (int32_t)min((int64_t)r.n_tokens[b], r.token_stride);
  h.prompt = r.n_prompt ? r.n_prompt[b] : 0;
#pragma unroll
  for (int k = 0; k < kHistoryAhead; ++k) {
    const int32_t i = (int32_t)threadIdx.x + k * kSliceThreads;
    h.token[k] = i < r.token_stride ? tokens[i] : -1;
  }
  return h;
}
__device__ __forceinline__ void gather_rules(const LogitRules& r, int32_t b, int32_t first, const History& h, uint32_t* counts, uint32_t* entries) {
  uint4* const tables = reinterpret_cast<uint4*>(counts);
  const int32_t words = ((r.tokens ? 1 : 0) + (r.bias_ids ? 1 : 0)) * kSliceTokens / 4;
  for (int32_t i = (int32_t)threadIdx.x; i < words; i += kSliceThreads) tables[i] = uint4{0, 0, 0, 0};
  __syncthreads();
  if (r.tokens) {
    auto enter = [&](int32_t i, int32_t token) {
      const int64_t at = (int64_t)token - first;
      if (i >= h.n || token < 0 || at < 0 || at >= kSliceTokens) return;
      if (i < h.prompt) atomicOr(&counts[at], 0x80000000u);
      else atomicAdd(&counts[at], 1u);
    };
#pragma unroll
    for (int k = 0; k < kHistoryAhead; ++k) enter((int32_t)threadIdx.x + k * kSliceThreads, h.token[k]);
    const int32_t* tokens = r.tokens + (int64_t)b * r.token_stride;
    for (int32_t i = (int32_t)threadIdx.x + kHistoryAhead * kSliceThreads; i < h.n; i += kSliceThreads) enter(i, tokens[i]);
  }
  if (r.bias_ids) {
    const int32_t e0 = max(r.bias_offsets[b], 0), e1 = min(r.bias_offsets[b + 1], r.n_bias);
    for (int32_t e = e0 + (int32_t)threadIdx.x; e < e1; e += kSliceThreads) {
      const int64_t at = (int64_t)r.bias_ids[e] - first;
      if (r.bias_ids[e] >= 0 && at >= 0 && at < kSliceTokens) atomicMax(&entries[at], (uint32_t)(e + 1));
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
// calls f(i, count, entry) for those of the 8 tokens from `at` on in the tables that a rule touches
template <class F> __device__ __forceinline__ void touched(const LogitRules& r, const uint32_t* counts, const uint32_t* entries, int32_t at, F&& f) {
  uint32_t c[8] = {}, e[8] = {};
  if (r.tokens) {
    const uint4 a = *reinterpret_cast<const uint4*>(counts + at), b = *reinterpret_cast<const uint4*>(counts + at + 4);
    c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w; c[4] = b.x; c[5] = b.y; c[6] = b.z; c[7] = b.w;
  }
  if (r.bias_ids) {
    const uint4 a = *reinterpret_cast<const uint4*>(entries + at), b = *reinterpret_cast<const uint4*>(entries + at + 4);
    e[0] = a.x; e[1] = a.y; e[2] = a.z; e[3] = a.w; e[4] = b.x; e[5] = b.y; e[6] = b.z; e[7] = b.w;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c[i] | e[i]) f(i, c[i], e[i]);
}

// One workgroup per slice.  Bound by the bytes where the batch is large (a logit that nothing touches is copied as it is, one that
// is masked is not read); the tables cost 64 KB of LDS at most, two workgroups a compute unit.
template <Elem E>
__global__ __launch_bounds__(kSliceThreads) void process_logits_kernel(Logits in, LogitRules r, typename Type<E>::bits* out, int64_t out_stride) {
  typedef typename Type<E>::bits bits;
  extern __shared__ __align__(16) uint32_t tables[];
  uint32_t *counts = tables, *entries = tables + (r.tokens ? kSliceTokens : 0);
  const int32_t b = (int32_t)blockIdx.y;
  const Row<E> row(in, b);
  const int32_t first = row.first_token((int32_t)blockIdx.x);
  if (first >= in.V) return;
  const bool ruled = r.tokens || r.bias_ids;
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
  if (ruled) gather_rules(r, b, first, h, counts, entries);
  const RowRules rule(r, b);
  bits* const to = out + (int64_t)b * out_stride;
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
    const int32_t at = (j * kSliceThreads + (int32_t)threadIdx.x) * 8, t = first + at;
    if (ruled && ok[j])
      touched(r, counts, entries, at, [&](int i, uint32_t count, uint32_t entry) { x[j].set(i, narrowed<E>(rule(widened<E>(x[j][i]), count, entry))); });
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
size_t rule_table_bytes(const LogitRules& r) { return (size_t)kSliceTokens * 4 * ((r.tokens ? 1 : 0) + (r.bias_ids ? 1 : 0)); }
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
// the order of the atomics.  The workgroup that finishes last for its row puts the slices together.  Without a cut it then
// knows the slice of the drawn token and goes through that one again; with a cut it knows the few bins in which the cuts lie.
// Second kernel, for rows with a cut: the tokens of those bins are listed (where there are too many, gone through again each time);
// the workgroup that finishes last finds the cuts in them, the slice and the token.
// What workgroups of one kernel hand to each other goes through atomics of the device, which no cache of an XCD holds back.
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
// 2^t as a whole octave and a number in [1, 2): the series of the exponential function around the middle of the octave, whose eleven
// terms leave 2.2e-13 of it.
struct Power {
  double octave, number;
  __device__ __forceinline__ explicit Power(double t) {
    octave = floor(t);
    const double x = (t - octave - 0.5) * 0.69314718055994530942;
    double p = 1.0 / 3628800.0;
    p = fma(p, x, 1.0 / 362880.0);
    p = fma(p, x, 1.0 / 40320.0);
    p = fma(p, x, 1.0 / 5040.0);
    p = fma(p, x, 1.0 / 720.0);
    p = fma(p, x, 1.0 / 120.0);
    p = fma(p, x, 1.0 / 24.0);
    p = fma(p, x, 1.0 / 6.0);
    p = fma(p, x, 0.5);
    p = fma(p, x, 1.0);
    p = fma(p, x, 1.0);
    number = p * 1.41421356237309504880;
  }
  // relative to 2^E
  __device__ __forceinline__ double weight(double E) const {
    const double d = octave - E;
    return d > -1000.0 ? ldexp(number, (int)d) : 0.0;
  }
  __device__ __forceinline__ u64 mass() const {  // in 2^-kMassBits of the octave
    return (u64)__double_as_longlong(fma(number, (double)(1ull << kMassBits), 4503599627370496.0)) - (u64)__double_as_longlong(4503599627370496.0);
  }
  // the bin under the octave E, kBins or more: too far down
  __device__ __forceinline__ int32_t bin(double t, double E) const {
    const double d = E - octave;
    return d < kBins / kBinsAnOctave ? (int32_t)d * kBinsAnOctave + (kBinsAnOctave - 1) - (int32_t)((t - octave) * kBinsAnOctave) : kBins;
  }
};

struct Slot {  // what a slice leaves
  double E, sum;
  float top;     // -inf: nothing can be drawn
  int32_t top_id;
};
struct RowPlan {  // what the first kernel leaves of a row for the second
  u64 wanted[kBins / 64];  // bins of which it needs the tokens
  double E;
  float top;
  int32_t cut;  // 0: the row is done
};
struct DrawMemory {
  uint32_t *arrived, *n_candidates;  // [2][rows], [rows]: zero between calls
  RowPlan* plans;
  Slot* slots;       // [rows][slices]
  u64* bins;         // [rows][slices][kBins]
  u64* candidates;   // [rows][kMostCandidates]: key, bin, id
  int32_t rows, slices;
};
size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }
int32_t most_slices(int32_t V) { return (V + 7 + kSliceTokens - 1) / kSliceTokens; }
DrawMemory memory_at(void* at, int32_t rows, int32_t V, size_t* bytes) {
  DrawMemory m{};
  m.rows = rows;
  m.slices = most_slices(V);
  char* p = static_cast<char*>(at);
  auto take = [&](size_t n) { char* q = p; p += rounded(n); return q; };
  m.arrived = reinterpret_cast<uint32_t*>(take((size_t)rows * 8));
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

struct Shared {
  double sum[2][kWaves];
  u64 part[kWaves];
  float top[kWaves];
  int32_t id[kWaves];
  u64 bins[1024];       // of the slice, the row, or a selection
  uint32_t counts[1024];
  double before_mass[kBins + 1];
  uint32_t before_count[kBins + 1];
  double slice_sum[(1 << 20) / kSliceTokens + 2];
  u64 slice_more[(1 << 20) / kSliceTokens + 2];
  uint32_t flag[2];
  int32_t found[2];
  double rest;
  int32_t slice;
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

// The logits of a slice under the rules.
template <Elem E>
__device__ __forceinline__ void load_slice(const Row<E>& row, const LogitRules& r, int32_t b, int32_t first, uint32_t* tables, float (&y)[kGroups][8]) {
  uint32_t *counts = tables, *entries = tables + (r.tokens ? kSliceTokens : 0);
  const bool ruled = r.tokens || r.bias_ids;
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
  if (ruled) gather_rules(r, b, first, h, counts, entries);
  const RowRules rule(r, b);
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[j][i] = ok[j] >> i & 1u ? widened<E>(x[j][i]) : -__builtin_inff();
    if (ruled && ok[j])
      touched(r, counts, entries, (j * kSliceThreads + (int32_t)threadIdx.x) * 8,
              [&](int i, uint32_t count, uint32_t entry) { if (ok[j] >> i & 1u) y[j][i] = rule(y[j][i], count, entry); });
#pragma unroll
    for (int i = 0; i < 8; ++i) y[j][i] = drawable(y[j][i]);
  }
}
template <Elem E> __device__ __forceinline__ int32_t token_of(int32_t first, int j, int i) { return first + (j * kSliceThreads + (int32_t)threadIdx.x) * 8 + i; }

// The token of a slice at which the running sum of weights (w of a token's logit and id) first exceeds `rest`; the last one
// with a weight if rounding leaves none; -1 if none has any.
template <Elem E, class W> __device__ int32_t find_token(const float (&y)[kGroups][8], int32_t first, double rest, Shared& s, W&& w) {
  const int32_t lane = (int32_t)threadIdx.x & 63, wave = (int32_t)threadIdx.x >> 6;
  double run[kGroups];
  int32_t last = -1;
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
    run[j] = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double x = w(y[j][i], token_of<E>(first, j, i));
      run[j] += x;
      if (x > 0.0) last = token_of<E>(first, j, i);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const double other = __shfl_up(run[j], d);
      if (lane >= d) run[j] += other;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) { s.found[0] = INT32_MAX; s.found[1] = -1; }
  if (lane == 63) {
#pragma unroll
    for (int j = 0; j < kGroups; ++j) s.sum[j][wave] = run[j];
  }
  __syncthreads();
  if (last >= 0) atomicMax(&s.found[1], last);
  double base = 0.0;
#pragma unroll
  for (int j = 0; j < kGroups; ++j) {
    double before = base;
    for (int k = 0; k < kWaves; ++k) {
      if (k == wave) before = base;
      base += s.sum[j][k];
    }
    const double end = before + run[j];
    double at = __shfl_up(run[j], 1);
    at = lane ? before + at : before;
    if (at <= rest && rest < end) {
      int32_t token = -1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double x = w(y[j][i], token_of<E>(first, j, i));
        at += x;
        if (x > 0.0 && (token < 0 || at - x <= rest)) token = token_of<E>(first, j, i);  // (the last whose stretch begins at or before)
      }
      if (token >= 0) atomicMin(&s.found[0], token);
    }
  }
  __syncthreads();
  return s.found[0] != INT32_MAX ? s.found[0] : s.found[1];
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

// The row's largest logit, its lowest id, octave and sum (thread by thread the same), from its slots; slices lie in s.slice_sum.
struct RowTotal {
  double E, sum;
  float top;
  int32_t top_id;
};
__device__ RowTotal row_total(const Slot* slots, int32_t n, Shared& s) {
  RowTotal r{0.0, 0.0, -__builtin_inff(), -1};
  const int32_t lane = (int32_t)threadIdx.x & 63;
  // (every wave by itself: at most three slots a lane)
  Slot mine[3];
  int32_t k = 0;
  float top = -__builtin_inff();
  double E = -__builtin_inf();
#pragma unroll
  for (k = 0; k < 3; ++k) {
    const int32_t i = lane + 64 * k;
    mine[k] = i < n ? take_in(slots + i) : Slot{0.0, 0.0, -__builtin_inff(), -1};
    if (mine[k].top > -__builtin_inff()) { top = fmaxf(top, mine[k].top); E = fmax(E, mine[k].E); }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) { top = fmaxf(top, __shfl_xor(top, d)); E = fmax(E, __shfl_xor(E, d)); }
  r.top = top;
  r.E = E;
  int32_t id = INT32_MAX;
  double sum = 0.0;
#pragma unroll
  for (k = 0; k < 3; ++k) {
    if (mine[k].top == top && mine[k].top_id >= 0) id = min(id, mine[k].top_id);
    const double d = mine[k].E - E;
    const double x = mine[k].top > -__builtin_inff() && d > -1000.0 ? ldexp(mine[k].sum, (int)d) : 0.0;
    sum += x;
    if (threadIdx.x < 64 && lane + 64 * k < n) s.slice_sum[lane + 64 * k] = x;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) id = min(id, __shfl_xor(id, d));
  r.top_id = id;
  r.sum = wave_sum(sum);
  __syncthreads();
  return r;
}
// Which slice the random number falls into and what is left of it there: s.slice, s.rest.
__device__ void find_slice(double u, int32_t n, Shared& s) {
  if (threadIdx.x == 0) {
    double total = 0.0;
    for (int32_t i = 0; i < n; ++i) total += s.slice_sum[i];
    double rest = u * total;
    int32_t at = -1;
    for (int32_t i = 0; i < n; ++i) {
      const double x = s.slice_sum[i];
      if (!(x > 0.0)) continue;
      if (at >= 0) {
        if (rest < s.slice_sum[at]) break;
        rest -= s.slice_sum[at];
      }
      at = i;
    }
    s.slice = at;
    s.rest = rest;
  }
  __syncthreads();
}
__device__ __forceinline__ void write_out(const RowDraw& d, const RowTotal& r, int32_t id, float y, int32_t* to_id, float* to_logprob) {
  *to_id = id;
  if (to_logprob)
    *to_logprob = id < 0 ? -__builtin_inff()
                         : (float)(((double)y - (double)r.top) / (double)d.temperature - (log(r.sum) + (r.E - octaves(r.top, d.per)) * 0.69314718055994530942));
}

// The row's bins from its slices' into s.bins and s.counts, relative to the octave E, and what lies in front of each (s.before_*;
// masses in 2^E).  All threads.
__device__ void row_bins(const Slot* slots, const u64* bins, int32_t n, double E, Shared& s) {
  const int32_t tid = (int32_t)threadIdx.x;
  __syncthreads();
  if (tid < kBins) {
    u64 mass = 0;
    uint32_t count = 0;
    for (int32_t i = 0; i < n; ++i) {
      if (!(take_in(&slots[i].top) > -__builtin_inff())) continue;
      const double d = (E - take_in(&slots[i].E)) * kBinsAnOctave;
      if (!(d <= (double)tid)) continue;
      const u64 x = take_in(bins + (size_t)i * kBins + (tid - (int32_t)d));
      mass += x & kMassMask;
      count += (uint32_t)(x >> kCountShift);
    }
    s.bins[tid] = mass;
    s.counts[tid] = count;
  }
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
__device__ __forceinline__ double bin_mass(const Shared& s, int32_t bin) { return ldexp((double)s.bins[bin], -kMassBits - bin / kBinsAnOctave); }
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
// the bin in which min_p of the largest weight lies, kBins if below all
__device__ int32_t bin_of_min(const RowDraw& d, float top, double E) {
  if (!(d.min_p > 0.0f)) return kBins;
  const double t = octaves(top, d.per) + log2((double)d.min_p);
  const int32_t b = Power(t).bin(t, E);
  return b < 0 ? 0 : b;
}

template <Elem E>
__global__ __launch_bounds__(kSliceThreads) void draw_slices_kernel(Logits in, LogitRules r, DrawRules dr, DrawMemory m, int32_t n_slices, int32_t* __restrict__ ids,
                                                                    float* __restrict__ logprobs) {
  extern __shared__ __align__(16) uint32_t tables[];
  __shared__ Shared s;
  const int32_t b = (int32_t)blockIdx.y, slice = (int32_t)blockIdx.x, tid = (int32_t)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Row<E> row(in, b);
  const RowDraw d(dr, b, in.V);
  Slot* const slots = m.slots + (size_t)b * m.slices;
  u64* const bins = m.bins + (size_t)b * m.slices * kBins;
  int32_t first = row.first_token(slice);
  float y[kGroups][8];
  load_slice<E>(row, r, b, first, tables, y);

  float top = -__builtin_inff();
  int32_t top_id = -1;
#pragma unroll
  for (int j = 0; j < kGroups; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (y[j][i] > top) { top = y[j][i]; top_id = token_of<E>(first, j, i); }
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
#pragma unroll
    for (int j = 0; j < kGroups; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (y[j][i] > -__builtin_inff()) {
          const double t = octaves(y[j][i], d.per);
          const Power w(t);
          sum += w.weight(slot.E);
          if (d.cut) {
            const int32_t bin = w.bin(t, slot.E);
            if (bin < kBins) atomicAdd(&s.bins[bin], w.mass() + (1ull << kCountShift));
          }
        }
    sum = wave_sum(sum);
    __syncthreads();
    if (lane == 0) s.sum[0][wave] = sum;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) slot.sum += s.sum[0][k];
  }
  if (tid == 0) put_out(slots + slice, slot);
  if (d.cut && tid < kBins) put_out(bins + (size_t)slice * kBins + tid, s.bins[tid]);
  if (!last_of(m.arrived + b, (uint32_t)n_slices, s)) return;

  const RowTotal total = row_total(slots, n_slices, s);
  if (total.top == -__builtin_inff() || d.greedy) {
    if (tid == 0) {
      write_out(d, total, total.top == -__builtin_inff() ? -1 : total.top_id, total.top, ids + b, logprobs ? logprobs + b : nullptr);
      m.plans[b].cut = 0;
    }
    return;
  }
  if (!d.cut) {
    find_slice(d.u, n_slices, s);
    const double rest = s.rest, Es = total.E;
    first = row.first_token(s.slice);
    load_slice<E>(row, r, b, first, tables, y);
    auto weight = [&](float v, int32_t) { return v > -__builtin_inff() ? Power(octaves(v, d.per)).weight(Es) : 0.0; };
    const int32_t id = find_token<E>(y, first, rest, s, weight);
#pragma unroll
    for (int j = 0; j < kGroups; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (token_of<E>(first, j, i) == id) write_out(d, total, id, y[j][i], ids + b, logprobs ? logprobs + b : nullptr);
    if (tid == 0 && id < 0) write_out(d, total, -1, 0.0f, ids + b, logprobs ? logprobs + b : nullptr);
    if (tid == 0) m.plans[b].cut = 0;
    return;
  }
  // the bins in which a cut can lie: that of the k-th token unless it ends there, those of p of what lies up to it, that of min_p
  row_bins(slots, bins, n_slices, total.E, s);
  if (tid == 0) {
    RowPlan plan{};
    plan.E = total.E;
    plan.top = total.top;
    plan.cut = 1;
    auto want = [&](int32_t bin) { plan.wanted[bin / 64] |= 1ull << (bin & 63); };
    double least = s.before_mass[kBins], most = least;
    int32_t last = kBins - 1;
    if (d.top_k && (uint32_t)d.top_k < s.before_count[kBins]) {
      last = bin_of_count(s, (uint32_t)d.top_k);
      most = s.before_mass[last + 1];
      least = most;
      if ((uint32_t)d.top_k != s.before_count[last + 1]) {
        want(last);
        least = s.before_mass[last];
      }
    }
    if (d.top_p < 1.0f) {
      const int32_t from = bin_of_mass(s, (double)d.top_p * least * (1.0 - 1e-9)), to = min(last, bin_of_mass(s, fmin((double)d.top_p * most * (1.0 + 1e-9), s.before_mass[kBins])));
      for (int32_t k = min(from, to); k <= to; ++k) want(k);
    }
    const int32_t low = bin_of_min(d, total.top, total.E);
    if (low < kBins) want(low);
    m.plans[b] = plan;
  }
}

// Goes through the tokens of the wanted bins: f(key, bin, id).  All threads; `listed` of them, or more than the list holds.
template <Elem E, class F>
__device__ __forceinline__ void for_candidates(const Row<E>& row, const LogitRules& r, const RowDraw& d, const RowPlan& plan, int32_t b, int32_t n_slices, const u64* list,
                                               uint32_t listed, uint32_t* tables, F&& f) {
  if (listed <= kMostCandidates) {
    for (uint32_t i = threadIdx.x; i < listed; i += kSliceThreads) {
      const u64 x = take_in(list + i);
      f((uint32_t)(x >> 32), (int32_t)(x >> 24 & 255u), (int32_t)(x & 0xffffffu));
    }
    return;
  }
  for (int32_t slice = 0; slice < n_slices; ++slice) {
    const int32_t first = row.first_token(slice);
    float y[kGroups][8];
    __syncthreads();  // (the tables of the last slice have been read)
    load_slice<E>(row, r, b, first, tables, y);
    for (int j = 0; j < kGroups; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (!(y[j][i] > -__builtin_inff())) continue;
        const double t = octaves(y[j][i], d.per);
        const int32_t bin = Power(t).bin(t, plan.E);
        if (bin < kBins && (plan.wanted[bin / 64] >> (bin & 63) & 1u)) f(key_of(y[j][i]), bin, token_of<E>(first, j, i));
      }
  }
}

// The end of a beginning of the row's order: tokens of heavier bins, and of `bin` those with a larger key and of those with `key`
// the ones up to `id`.
struct Cut {
  int32_t bin;
  uint32_t key;
  int32_t id;
  __device__ __forceinline__ bool keeps(int32_t in, uint32_t k, int32_t i) const { return in < bin || (in == bin && (k > key || (k == key && i <= id))); }
};

// Narrows the tokens of a bin that `within` keeps down to the one at which `need` (tokens, or mass in the bin's whole numbers) is reached.
// each(f) goes through the candidates.  Returns the mass up to there.
template <class Each> __device__ u64 select(Each&& each, Cut within, int32_t bin, bool by_count, u64 need, double per, int32_t V, Cut* out, Shared& s) {
  const int32_t tid = (int32_t)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t lo = ~0u, hi = 0;
  each([&](uint32_t key, int32_t in, int32_t id) {
    if (in == bin && within.keeps(in, key, id)) { lo = min(lo, key); hi = max(hi, key); }
  });
  __syncthreads();
  if (tid == 0) { s.flag[0] = ~0u; s.flag[1] = 0; }
  __syncthreads();
  atomicMin(&s.flag[0], lo);
  atomicMax(&s.flag[1], hi);
  __syncthreads();
  lo = s.flag[0];
  hi = s.flag[1];
  if (lo > hi) {
    *out = within;
    return 0;
  }
  u64 up_to = 0, tied_mass = 0;
  uint32_t tied = 0;
  // a pass: which of 1024 stretches of [from, to], in falling order of what, has the token
  auto narrow = [&](auto&& what, bool weighed) {
    for (int i = tid; i < 1024; i += kSliceThreads) { s.bins[i] = 0; s.counts[i] = 0; }
    __syncthreads();
    each([&](uint32_t key, int32_t in, int32_t id) {
      if (in != bin || !within.keeps(in, key, id)) return;
      const int32_t at = what(key, id);
      if (at < 0) return;
      atomicAdd(&s.counts[at], 1u);
      if (weighed) atomicAdd(&s.bins[at], Power(octaves(value_of(key), per)).mass());
    });
    __syncthreads();
    // two neighbours a thread
    const bool counted = by_count || !weighed;
    const u64 m0 = s.bins[2 * tid], m1 = s.bins[2 * tid + 1];
    const uint32_t c0 = s.counts[2 * tid], c1 = s.counts[2 * tid + 1];
    u64 all_mass = m0 + m1, all = counted ? (u64)c0 + c1 : m0 + m1;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) {
      const u64 other = __shfl_up(all, e), other_mass = __shfl_up(all_mass, e);
      if (lane >= e) { all += other; all_mass += other_mass; }
    }
    if (lane == 63) { s.part[wave] = all; s.sum[0][wave] = __longlong_as_double((long long)all_mass); }
    if (tid == 0) s.found[0] = 1023;
    __syncthreads();
    u64 in_front = 0, mass_in_front = 0;
    for (int k = 0; k < wave; ++k) { in_front += s.part[k]; mass_in_front += (u64)__double_as_longlong(s.sum[0][k]); }
    all += in_front;
    all_mass += mass_in_front;
    const u64 v0 = counted ? (u64)c0 : m0, v1 = counted ? (u64)c1 : m1, begin = all - v0 - v1;
    const bool here = begin < need && need <= all;
    const int which = need <= begin + v0 ? 0 : 1;
    __syncthreads();
    if (here) {
      s.found[0] = 2 * tid + which;
      s.part[0] = begin + (which ? v0 : 0);                     // in front of the stretch
      s.part[1] = all_mass - m0 - m1 + (which ? m0 : 0);
      s.part[2] = which ? m1 : m0;
      s.counts[0] = which ? c1 : c0;
    }
    __syncthreads();
    need -= s.part[0];
    if (weighed) { up_to += s.part[1]; tied_mass = s.part[2]; }
    tied = s.counts[0];
    const int32_t at = s.found[0];
    __syncthreads();
    return at;
  };
  // rounding can leave a need above what there is: the last token then
  {
    u64 all = 0;
    each([&](uint32_t key, int32_t in, int32_t id) {
      if (in == bin && within.keeps(in, key, id)) all += by_count ? 1 : Power(octaves(value_of(key), per)).mass();
    });
#pragma unroll
    for (int e = 32; e; e >>= 1) all += __shfl_xor(all, e);
    if (lane == 0) s.part[wave] = all;
    __syncthreads();
    all = 0;
    for (int k = 0; k < kWaves; ++k) all += s.part[k];
    __syncthreads();
    if (need > all) need = all;
    if (need == 0) need = 1;
  }
  for (int pass = 0; pass < 5; ++pass) {  // (10 bits each)
    const uint32_t width = hi - lo;
    const int shift = width < 1024 ? 0 : 22 - __clz((int)width);
    const uint32_t from = hi, floor_key = lo;
    const int32_t at = narrow([&](uint32_t key, int32_t) { return key <= from && key >= floor_key ? (int32_t)((from - key) >> shift) : -1; }, true);
    hi = from - ((uint32_t)at << shift);
    lo = shift == 0 ? hi : max(floor_key, hi - ((1u << shift) - 1u));
    if (hi == lo) break;
  }
  // of the tokens with this key the first so many
  const u64 each_mass = tied_mass / max(tied, 1u);
  const u64 mass_in_front = up_to;
  u64 wanted = by_count ? need : (need + each_mass - 1) / max(each_mass, (u64)1);
  if (wanted >= tied) {
    *out = Cut{bin, hi, within.bin == bin && within.key == hi ? within.id : INT32_MAX};
    return mass_in_front + tied_mass;
  }
  need = wanted;
  int32_t first = 0, last = V - 1;
  const uint32_t only = hi;
  for (int pass = 0; pass < 4 && first != last; ++pass) {
    const uint32_t width = (uint32_t)(last - first);
    const int shift = width < 1024 ? 0 : 22 - __clz((int)width);
    const int32_t from = first, to = last;
    const int32_t at = narrow([&](uint32_t key, int32_t id) { return key == only && id >= from && id <= to ? (int32_t)((uint32_t)(id - from) >> shift) : -1; }, false);
    first = from + (at << shift);
    last = min(to, first + (1 << shift) - 1);
  }
  *out = Cut{bin, only, first};
  return mass_in_front + wanted * each_mass;
}

template <Elem E>
__global__ __launch_bounds__(kSliceThreads) void draw_cut_kernel(Logits in, LogitRules r, DrawRules dr, DrawMemory m, int32_t n_slices, int32_t* __restrict__ ids,
                                                                 float* __restrict__ logprobs) {
  extern __shared__ __align__(16) uint32_t tables[];
  __shared__ Shared s;
  const int32_t b = (int32_t)blockIdx.y, slice = (int32_t)blockIdx.x, tid = (int32_t)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const RowPlan plan = m.plans[b];
  if (!plan.cut) return;
  const Row<E> row(in, b);
  const RowDraw d(dr, b, in.V);
  const Slot* const slots = m.slots + (size_t)b * m.slices;
  const u64* const bins = m.bins + (size_t)b * m.slices * kBins;
  u64* const list = m.candidates + (size_t)b * kMostCandidates;
  float y[kGroups][8];

  // the tokens of the wanted bins, if the slice has any
  if (tid == 0) s.flag[1] = 0;
  __syncthreads();
  const Slot slot = slots[slice];
  if (slot.top > -__builtin_inff() && tid < kBins && (plan.wanted[tid / 64] >> (tid & 63) & 1u)) {
    const double at = (double)tid - (plan.E - slot.E) * kBinsAnOctave;
    if (at >= 0.0 && bins[(size_t)slice * kBins + (int32_t)at] >> kCountShift) s.flag[1] = 1;
  }
  __syncthreads();
  if (s.flag[1]) {
    const int32_t first = row.first_token(slice);
    load_slice<E>(row, r, b, first, tables, y);
#pragma unroll
    for (int j = 0; j < kGroups; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double t = octaves(y[j][i], d.per);
        const int32_t bin = y[j][i] > -__builtin_inff() ? Power(t).bin(t, plan.E) : kBins;
        const bool mine = bin < kBins && (plan.wanted[bin / 64] >> (bin & 63) & 1u);
        const u64 who = __ballot(mine);
        if (!who) continue;
        uint32_t at = 0;
        if (lane == 0) at = __hip_atomic_fetch_add(m.n_candidates + b, (uint32_t)__popcll(who), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        at = __builtin_amdgcn_readfirstlane(at) + (uint32_t)__popcll(who & ((1ull << lane) - 1ull));
        if (mine && at < kMostCandidates) put_out(list + at, (u64)key_of(y[j][i]) << 32 | (u64)bin << 24 | (u64)(uint32_t)token_of<E>(first, j, i));
      }
  }
  if (!last_of(m.arrived + m.rows + b, (uint32_t)n_slices, s)) return;

  const uint32_t listed = take_in(m.n_candidates + b);
  __syncthreads();
  if (tid == 0) put_out(m.n_candidates + b, 0u);
  auto each = [&](auto&& f) { for_candidates<E>(row, r, d, plan, b, n_slices, list, listed, tables, f); };
  const RowTotal total = row_total(slots, n_slices, s);
  row_bins(slots, bins, n_slices, total.E, s);
  // what the selections below need of the bins, before they use the same memory
  const bool by_k = d.top_k && (uint32_t)d.top_k < s.before_count[kBins];
  Cut cut{kBins, 0, INT32_MAX};
  int32_t k_bin = kBins - 1;
  u64 k_need = 0;
  bool k_inside = false;
  double up_to = s.before_mass[kBins], k_before = 0.0;
  if (by_k) {
    k_bin = bin_of_count(s, (uint32_t)d.top_k);
    k_before = s.before_mass[k_bin];
    k_need = (uint32_t)d.top_k - s.before_count[k_bin];
    k_inside = (uint32_t)d.top_k != s.before_count[k_bin + 1];
    up_to = s.before_mass[k_bin + 1];
    cut = Cut{k_bin, 0, INT32_MAX};
  }
  if (k_inside) {
    const u64 mass = select(each, cut, k_bin, true, k_need, d.per, in.V, &cut, s);
    up_to = k_before + ldexp((double)mass, -kMassBits - k_bin / kBinsAnOctave);
    row_bins(slots, bins, n_slices, total.E, s);
  }
  if (d.top_p < 1.0f) {
    const double target = (double)d.top_p * up_to;
    const int32_t p_bin = min(k_bin, bin_of_mass(s, target));
    const double need = ldexp(target - s.before_mass[p_bin], kMassBits + p_bin / kBinsAnOctave);
    if (plan.wanted[p_bin / 64] >> (p_bin & 63) & 1u) {
      const Cut within = cut;
      select(each, within, p_bin, false, need >= 1.0 ? (u64)ceil(need) : 1u, d.per, in.V, &cut, s);
    }
  }
  const int32_t low = bin_of_min(d, total.top, total.E), edge = min(cut.bin, low);
  // kept: what the cut keeps and min_p does not drop; always the largest
  auto kept = [&](uint32_t key, int32_t bin, int32_t id) {
    if (!cut.keeps(bin, key, id) || bin > low) return false;
    return bin < low || exp(((double)value_of(key) - (double)total.top) / (double)d.temperature) >= (double)d.min_p;
  };
  // the slices' sums: bins in front of the edge as they are, those of its tokens one by one if it is divided
  const bool divided = edge < kBins && (edge == low || cut.key != 0 || cut.id != INT32_MAX);
  for (int32_t i = tid; i < n_slices; i += kSliceThreads) s.slice_more[i] = 0;
  __syncthreads();
  if (divided) {
    const int32_t first = row.first_token(0);
    each([&](uint32_t key, int32_t in_bin, int32_t id) {
      if (in_bin != edge) return;
      const Power w(octaves(value_of(key), d.per));
      if (kept(key, in_bin, id)) atomicAdd(&s.slice_more[(uint32_t)(id - first) / kSliceTokens], w.mass());
    });
  }
  __syncthreads();
  for (int32_t i = wave; i < n_slices; i += kWaves) {
    const Slot one = slots[i];
    double sum = 0.0;
    if (one.top > -__builtin_inff()) {
      const double off = (total.E - one.E) * kBinsAnOctave;  // of the slice's bins in the row's
#pragma unroll
      for (int k = 0; k < kBins / 64; ++k) {
        const int32_t bin = lane * (kBins / 64) + k;  // of the slice
        const double at = off + (double)bin;
        if (at < (double)(divided ? edge : min(edge + 1, kBins))) sum += ldexp((double)(bins[(size_t)i * kBins + bin] & kMassMask), -kMassBits - (int32_t)at / kBinsAnOctave);
      }
    }
    sum = wave_sum(sum);
    if (lane == 0) s.slice_sum[i] = sum + (divided ? ldexp((double)s.slice_more[i], -kMassBits - edge / kBinsAnOctave) : 0.0);
  }
  __syncthreads();
  find_slice(d.u, n_slices, s);
  const double rest = s.rest;
  const int32_t first = row.first_token(s.slice);
  load_slice<E>(row, r, b, first, tables, y);
  const int32_t id = find_token<E>(y, first, rest, s, [&](float v, int32_t token) {
    if (!(v > -__builtin_inff())) return 0.0;
    const double t = octaves(v, d.per);
    const Power w(t);
    const int32_t bin = w.bin(t, total.E);
    return bin < kBins && kept(key_of(v), bin, token) ? w.weight(total.E) : 0.0;
  });
#pragma unroll
  for (int j = 0; j < kGroups; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (token_of<E>(first, j, i) == id) write_out(d, total, id, y[j][i], ids + b, logprobs ? logprobs + b : nullptr);
  if (tid == 0 && id < 0) write_out(d, total, -1, 0.0f, ids + b, logprobs ? logprobs + b : nullptr);
}

template <template <Elem> class Launch, class... Args>
void by_type(Elem e, const Args&... args) {
  if (e == Elem::kF32) Launch<Elem::kF32>::run(args...);
  else if (e == Elem::kBF16) Launch<Elem::kBF16>::run(args...);
  else Launch<Elem::kF16>::run(args...);
}
template <Elem E> struct Process {
  static void run(const Logits& in, const int32_t& B, const LogitRules& r, void* const& out, const int64_t& out_stride, const hipStream_t& stream) {
    hipLaunchKernelGGL(process_logits_kernel<E>, dim3(slices_of<E>(in), B), dim3(kSliceThreads), rule_table_bytes(r), stream, in, r,
                       static_cast<typename Type<E>::bits*>(out), out_stride);
  }
};
template <class K> void more_lds(K kernel) {
  (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kSliceTokens * 4);
}
template <Elem E> struct Draw {
  static void run(const Logits& in, const int32_t& B, const LogitRules& r, const DrawRules& d, const DrawMemory& m, int32_t* const& ids, float* const& logprobs,
                  const hipStream_t& stream) {
    static const bool prepared = (more_lds(&draw_slices_kernel<E>), more_lds(&draw_cut_kernel<E>), true);
    (void)prepared;
    const int32_t n = slices_of<E>(in);
    hipLaunchKernelGGL(draw_slices_kernel<E>, dim3(n, B), dim3(kSliceThreads), rule_table_bytes(r), stream, in, r, d, m, n, ids, logprobs);
    if (d.uniform && (d.top_k || d.top_p || d.min_p))
      hipLaunchKernelGGL(draw_cut_kernel<E>, dim3(n, B), dim3(kSliceThreads), rule_table_bytes(r), stream, in, r, d, m, n, ids, logprobs);
  }
};

}  // namespace

void launch_process_logits(const Logits& in, Elem type, int32_t B, const LogitRules& rules, void* out, int64_t out_stride, hipStream_t stream) {
  by_type<Process>(type, in, B, rules, out, out_stride, stream);
}

size_t sampler_bytes(int32_t max_rows, int32_t V) {
  size_t bytes = 0;
  memory_at(nullptr, max_rows, V, &bytes);
  return bytes;
}

void launch_sample(const Logits& in, Elem type, int32_t B, const LogitRules& rules, const DrawRules& draw, void* memory, int32_t max_rows, int32_t max_V, int32_t* ids,
                   float* logprobs, hipStream_t stream) {
  size_t bytes = 0;
  by_type<Draw>(type, in, B, rules, draw, memory_at(memory, max_rows, max_V, &bytes), ids, logprobs, stream);
}

}  // namespace xgm
