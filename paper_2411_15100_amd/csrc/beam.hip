// Several beams a request: which continuations go on, and what the rows that go on keep.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "elements.hpp"
#include "logits.hpp"
#include "slices.hpp"

namespace xgm {

namespace {

// ------------------------------------------------------------- continuations of beams
// A continuation of row b is worth logit + base, base = score - log(sum of exp of the row's logits), in 64 bits: two continuations of
// different rows may be as near to each other as two numbers get, and the order of a sum in 32 bits would decide between them.
// First kernel, a workgroup per slice of a row: it reads the logits once, under the rules, and leaves the slice's sum of weights and its
// n_out best tokens in order (a key: the logit as a whole number, then the id's complement, so that no two are alike).  Second
// kernel, a workgroup per request: it knows every row's base and takes the n_out best of all lists.  (As one kernel whose last workgroup of a
// request goes on, what the second needs of registers and LDS keeps waves of the first from running: 128 rows of 151936 took 70 us.)
// A list begins with a bound that n tokens reach (bounds_of): no more has to be looked at.  The tokens above it are compared each with each.
// 128 rows of 151936 (bf16, 5 rows of 13 open, n = 8): 30 and 12 us; of the first 8 are loads, 5 the bound, 10 weights in 64 bits, the rest the list: instruction
// issue and barriers, 2.4 rounds of workgroups; the second is a chain of loads, sums, a logarithm and lists on 16 compute units.  4 rows of 32000: 8 and 6 us.
// One request of 64 beams of 128256 tokens, 128 continuations: 41 and 34 us.
constexpr int kMostFound = 1024;   // tokens of a slice above its bound that are kept in LDS
constexpr int kMostJoined = 2048;  // continuations of a request, likewise
constexpr int kMostSlices = (1 << 20) / kSliceTokens + 1;

struct BeamSlot {  // what a slice leaves beside its list
  double E, sum;
  float top;  // -inf: it has no list
};
struct BeamMemory {
  BeamSlot* slots;  // [rows][slices]
  u64* lists;       // [rows][slices][n_out], 0 behind the last
  int32_t slices;
};
size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }
int32_t most_slices(int32_t V) { return (V + 7 + kSliceTokens - 1) / kSliceTokens; }
BeamMemory memory_at(void* at, int32_t rows, int32_t V, size_t* bytes) {
  BeamMemory m{};
  m.slices = most_slices(V);
  char* p = static_cast<char*>(at);
  auto take = [&](size_t n) { char* q = p; p += rounded(n); return q; };
  m.slots = reinterpret_cast<BeamSlot*>(take((size_t)rows * m.slices * sizeof(BeamSlot)));
  m.lists = reinterpret_cast<u64*>(take((size_t)rows * m.slices * kMaxContinuations * 8));
  *bytes = (size_t)(p - static_cast<char*>(at));
  return m;
}

// A token in the order of its row: the larger logit first, then the lower id.  0 is none.
__device__ __forceinline__ u64 token_key(float y, int32_t id) { return (u64)key_of(y) << 32 | (uint32_t)~id; }
__device__ __forceinline__ int32_t id_of(u64 key) { return (int32_t)~(uint32_t)key; }
__device__ __forceinline__ float logit_of(u64 key) { return value_of((uint32_t)(key >> 32)); }

// A continuation in the order of its request: the larger sum first, then `place` falling: the lower row, the larger logit, the lower id.
__device__ __forceinline__ u64 order_of(double x) {
  const u64 u = (u64)__double_as_longlong(x == 0.0 ? 0.0 : x);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double sum_of(u64 order) { return __longlong_as_double((long long)(order >> 63 ? order & ~(1ull << 63) : ~order)); }
constexpr int kIdBits = 20;
static_assert(kMaxBeams <= 64, "six bits of a place");
__device__ __forceinline__ u64 place_in(int32_t beam, u64 key) {
  return (u64)(kMaxBeams - 1 - beam) << (32 + kIdBits) | (key >> 32) << kIdBits | ((uint32_t)key & ((1u << kIdBits) - 1u));
}
__device__ __forceinline__ int32_t beam_of(u64 place) { return kMaxBeams - 1 - (int32_t)(place >> (32 + kIdBits)); }
__device__ __forceinline__ int32_t id_at(u64 place) { return (int32_t)(~(uint32_t)place & ((1u << kIdBits) - 1u)); }

template <class T> struct Maxima {  // of threads; of groups of them
  T of[kSliceThreads], least[kWaves], top[kWaves];
};
struct BeamShared {
  Maxima<float> most;
  double sum[kWaves];
  uint32_t n_found, counts[kWaves];
  u64 found[kMostFound], better[kMostFound];
};
struct JoinShared {
  double base[kMaxBeams];
  Maxima<double> most;
  int32_t is_ended[kMaxBeams];
  uint32_t n_joined, counts[kWaves];
  u64 order[kMostJoined], place[kMostJoined];
  int32_t rows[kMaxContinuations], ids[kMaxContinuations];
  float scores[kMaxContinuations];
};

__device__ __forceinline__ bool is_live(const BeamSearch& s, int32_t b) { return s.scores[b] > -__builtin_inff() && s.scores[b] < __builtin_inff(); }
__device__ __forceinline__ bool is_ended(const BeamSearch& s, int32_t b) { return s.ended && s.ended[b] != 0; }

__device__ __forceinline__ uint32_t count_all(uint32_t mine, uint32_t (&counts)[kWaves]) {
#pragma unroll
  for (int d = 32; d; d >>= 1) mine += __shfl_xor(mine, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = mine;
  __syncthreads();
  uint32_t all = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) all += counts[k];
  return all;
}

// A bound that n numbers of the workgroup reach, or -inf, by the largest number of every thread.  Up to kWaves of them: threads form as many groups (a power of
// two), and the bound is the least of the groups' largest.  More: of kWaves groups the bound is the least of the ceil(n / kWaves)-th largest ones, which
// few others reach (of 8192 tokens 150 to 200 for n = 128; with n groups and their largest it was 600).  A group's threads lie evenly over all: where a
// row ends in the slice every group still has some of its tokens.
static_assert(kMaxContinuations <= kSliceThreads, "a thread each");
template <class T> struct Bounds {
  T least, top;  // the bound, and the largest number of all
};
template <class T> __device__ __forceinline__ Bounds<T> bounds_of(T mine, int n, Maxima<T>& m) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  __syncthreads();
  m.of[threadIdx.x] = mine;
  __syncthreads();
  if (n <= kWaves) {  // (every wave finds all of it: no barrier more)
    int groups = 1;
    while (groups < n) groups *= 2;
    T r = m.of[lane];  // lanes that lie `groups` apart are of one
#pragma unroll
    for (int k = 1; k < kWaves; ++k) r = max(r, m.of[k * 64 + lane]);
    for (int d = 32; d >= groups; d >>= 1) r = max(r, (T)__shfl_xor(r, d));
    Bounds<T> b{r, r};
    for (int d = groups / 2; d; d >>= 1) {
      b.least = min(b.least, (T)__shfl_xor(b.least, d));
      b.top = max(b.top, (T)__shfl_xor(b.top, d));
    }
    return b;
  }
  T x = m.of[lane * kWaves + wave];
#pragma unroll
  for (int size = 2; size <= 64; size *= 2)  // in falling order
#pragma unroll
    for (int d = size / 2; d; d >>= 1) {
      const T other = (T)__shfl_xor(x, d);
      x = ((lane & size) == 0) == ((lane & d) == 0) ? max(x, other) : min(x, other);
    }
  if (lane == (n + kWaves - 1) / kWaves - 1) m.least[wave] = x;
  if (lane == 0) m.top[wave] = x;
  __syncthreads();
  Bounds<T> b{m.least[0], m.top[0]};
#pragma unroll
  for (int k = 1; k < kWaves; ++k) {
    b.least = min(b.least, m.least[k]);
    b.top = max(b.top, m.top[k]);
  }
  return b;
}
// y[k], by the steps of a tree
__device__ __forceinline__ float token_at(const Tokens& y, int k) {
  float x[kTokens];
#pragma unroll
  for (int i = 0; i < kTokens; ++i) x[i] = y[i];
#pragma unroll
  for (int n = kTokens / 2; n; n >>= 1)
#pragma unroll
    for (int i = 0; i < n; ++i) {
      float upper = x[i + n];
      asm("" : "+v"(upper));  // (else the compiler makes it one access by a number that differs between lanes, in a loop over them: 13 us of 47)
      x[i] = k & n ? upper : x[i];
    }
  return x[0];
}

template <Elem E>
__global__ __launch_bounds__(kSliceThreads, 6) void beam_slices_kernel(Logits in, LogitRules r, BeamSearch s, BeamMemory m) {
  extern __shared__ __align__(16) char lds[];
  RuleTable& table = *reinterpret_cast<RuleTable*>(lds);
  BeamShared& sh = *reinterpret_cast<BeamShared*>(lds);
  __shared__ double roots[16];
  const int32_t slice = (int32_t)blockIdx.x, b = (int32_t)blockIdx.y, tid = (int32_t)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t n = s.n_out;
  if (!is_live(s, b) || is_ended(s, b)) return;
  fill_roots(roots);
  {
    const Row<E> row(in, b);
    const int32_t first = row.first_token(slice);
    Tokens y;
    load_slice<E>(row, r, b, first, table, y);
    float mine = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < kTokens; ++k) mine = fmaxf(mine, y[k]);
    if (tid == 0) sh.n_found = 0;  // (read behind the next barriers)
    const Bounds<float> bounds = bounds_of(mine, n, sh.most);
    const float top = bounds.top;
    BeamSlot slot{0.0, 0.0, top};
    u64* const list = m.lists + ((size_t)b * m.slices + slice) * n;
    if (top > -__builtin_inff()) {
      constexpr double per = 1.4426950408889634074;
      slot.E = floor(octaves(top, per));
      double sum = 0.0;
      auto add = [&](float v) {
        if (v > -__builtin_inff()) sum += Power(octaves(v, per), slot.E, roots).weight();
      };
#pragma unroll 1
      for (int k = 0; k < kTokens / 4; ++k) {  // (instructions that are fetched once cost as much as carrying them out)
        add(y[0]); add(y[1]); add(y[2]); add(y[3]);
        y = __builtin_shufflevector(y, y, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 0, 1, 2, 3);
      }
      sum = wave_sum(sum);
      if (lane == 0) sh.sum[wave] = sum;
      uint32_t good = 0;
#pragma unroll
      for (int k = 0; k < kTokens; ++k) good |= (y[k] > -__builtin_inff() && y[k] >= bounds.least ? 1u : 0u) << k;
      auto collect = [&] {
        if (!good) return;
        uint32_t at = atomicAdd(&sh.n_found, (uint32_t)__builtin_popcount(good));
#pragma unroll 1
        for (uint32_t left = good; left; left &= left - 1, ++at) {
          const int k = __builtin_ctz(left);
          if (at < kMostFound) sh.found[at] = token_key(token_at(y, k), first + place_of(k));
        }
      };
      collect();
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kWaves; ++k) slot.sum += sh.sum[k];
      uint32_t all = sh.n_found;
      if (all > kMostFound) {  // many equal ones: the key of the n-th best, bit by bit
        auto above = [&](u64 least) {
          uint32_t bits = 0;
#pragma unroll 1
          for (int k = 0; k < kTokens; ++k) {
            const float v = token_at(y, k);
            bits |= (v > -__builtin_inff() && token_key(v, first + place_of(k)) >= least ? 1u : 0u) << k;
          }
          return bits;
        };
        u64 edge = 0;
#pragma unroll 1
        for (int bit = 63; bit >= 0; --bit) {
          const u64 at = edge | 1ull << bit;
          if (count_all((uint32_t)__builtin_popcount(above(at)), sh.counts) >= (uint32_t)n) edge = at;
        }
        good = above(edge);
        if (tid == 0) sh.n_found = 0;
        __syncthreads();
        collect();
        __syncthreads();
        all = (uint32_t)n;
      }
      const u64* found = sh.found;
      // Where masks leave tokens in a few places a bound says little; another one among what was found, which lies in no order, says more.
      if (all > (uint32_t)(2 * n + 80)) {
        static_assert(kMostFound == 2 * kSliceThreads, "two tokens a thread");
        const u64 none = 0;
        const u64 one = (uint32_t)tid < all ? sh.found[tid] : none, two = (uint32_t)tid + kSliceThreads < all ? sh.found[tid + kSliceThreads] : none;
        const float next = bounds_of(max(one, two) ? logit_of(max(one, two)) : -__builtin_inff(), n, sh.most).least;
        if (tid == 0) sh.n_found = 0;  // (all have read it: they have met behind that)
        __syncthreads();
        if (one && logit_of(one) >= next) sh.better[atomicAdd(&sh.n_found, 1u)] = one;
        if (two && logit_of(two) >= next) sh.better[atomicAdd(&sh.n_found, 1u)] = two;
        __syncthreads();
        all = sh.n_found;
        found = sh.better;
      }
      for (uint32_t i = (uint32_t)tid; i < all; i += kSliceThreads) {
        const u64 key = found[i];
        uint32_t rank = 0;
        for (uint32_t k = 0; k < all; ++k) rank += found[k] > key;
        if (rank < (uint32_t)n) list[rank] = key;
      }
      if ((uint32_t)tid >= all && tid < n) list[tid] = 0;
    } else if (tid < n) {
      list[tid] = 0;
    }
    if (tid == 0) m.slots[(size_t)b * m.slices + slice] = slot;
  }
}

__global__ __launch_bounds__(kSliceThreads) void beam_join_kernel(BeamSearch s, BeamMemory m, int32_t n_slices) {
  __shared__ JoinShared join;
  __shared__ double roots[16];
  const int32_t request = (int32_t)blockIdx.x, tid = (int32_t)threadIdx.x, lane = tid & 63, wave = tid >> 6, n = s.n_out;
  fill_roots(roots);
  // What is needed first is read at once: the thread's first entries of the lists, and what the slices left.
  const int32_t b0 = request * s.beams;
  // (the lists' first entries come first, then the second ones: the bound below is taken from them)
  const int32_t n_lists = s.beams * n_slices, entries = n_lists * n;
  constexpr int kHeld = 4;  // entries of a thread
  const u64* const lists = m.lists + (size_t)b0 * m.slices * n;
  u64 held[kHeld];
  auto key_at = [&](int32_t e) -> u64 {
    const int32_t rank = e / n_lists, list = e - rank * n_lists, beam = list / n_slices;
    return lists[((size_t)beam * m.slices + (list - beam * n_slices)) * n + rank];
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int32_t e = k * kSliceThreads + tid;
    held[k] = e < entries ? key_at(e) : 0;
  }
  __syncthreads();
  // A row's slices lie with 16, 32 or 64 lanes, as many as it has.
  const int part = n_slices <= 16 ? 16 : n_slices <= 32 ? 32 : 64;
  for (int32_t i0 = wave * (64 / part); i0 < s.beams; i0 += kWaves * (64 / part)) {
    const int32_t i = i0 + lane / part, b = b0 + min(i, s.beams - 1);
    const BeamSlot* const slots = m.slots + (size_t)b * m.slices;
    const bool ended = is_ended(s, b), live = is_live(s, b), open = live && !ended;
    constexpr int kEach = (kMostSlices + 63) / 64;
    float top = -__builtin_inff();
    double most = -__builtin_inf(), octave[kEach], x[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int32_t k = lane % part + part * j;
      const bool there = open && k < n_slices;
      const float t = there ? slots[k].top : -__builtin_inff();
      octave[j] = there ? slots[k].E : 0.0;
      x[j] = there ? slots[k].sum : 0.0;
      if (!(t > -__builtin_inff())) octave[j] = -__builtin_inf();
      top = fmaxf(top, t);
      most = fmax(most, octave[j]);
    }
    for (int d = part / 2; d; d >>= 1) {
      top = fmaxf(top, __shfl_xor(top, d));
      most = fmax(most, __shfl_xor(most, d));
    }
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (octave[j] - most > -1100.0) sum += ldexp(x[j], (int)(octave[j] - most));
    for (int d = part / 2; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane % part == 0 && i < s.beams) {
      const double score = (double)s.scores[b];
      double base = live && ended ? score : -__builtin_inf();
      // (relative to the largest logit's own weight: a token that is alone costs nothing)
      constexpr double per = 1.4426950408889634074;
      if (top > -__builtin_inff()) base = score - ((double)top + log(sum / Power(octaves(top, per), most, roots).weight()));
      join.base[i] = base;
      join.is_ended[i] = ended;
    }
  }
  if (tid == 0) join.n_joined = 0;
  __syncthreads();
  // f(entry's sum, its place) for the thread's entries.  (A row that is not live has what an earlier call left there.)
  auto with = [&](int32_t e, u64 key, auto&& f) {
    const int32_t list = e % n_lists, beam = list / n_slices;
    const double base = join.base[beam];
    if (!(base > -__builtin_inf())) return;
    if (join.is_ended[beam]) {
      if (e == beam * n_slices) f(base, place_in(beam, (u64)key_of(0.0f) << 32));
    } else if (key) {
      f((double)logit_of(key) + base, place_in(beam, key));
    }
  };
  auto for_held = [&](auto&& f) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (k * kSliceThreads + tid < entries) with(k * kSliceThreads + tid, held[k], f);
  };
  // All entries, beam after beam as they lie in memory: what a request needs only where its bounds say too little.
  auto for_all = [&](auto&& f) {
    for (int32_t beam = 0; beam < s.beams; ++beam) {
      if (!(join.base[beam] > -__builtin_inf())) continue;
      const u64* const own = lists + (size_t)beam * m.slices * n;
      const int32_t all = join.is_ended[beam] ? 1 : n_slices * n;
      for (int32_t i = tid; i < all; i += kSliceThreads) with(i % n * n_lists + beam * n_slices + i / n, own[i], f);
    }
  };
  auto join_in = [&](u64 order, u64 place) {
    const uint32_t at = atomicAdd(&join.n_joined, 1u);
    if (at < kMostJoined) {
      join.order[at] = order;
      join.place[at] = place;
    }
  };
  auto joined = [&] {
    __syncthreads();
    return join.n_joined;
  };
  auto again = [&] {  // (all have read how many there are)
    __syncthreads();
    if (tid == 0) join.n_joined = 0;
    __syncthreads();
  };
  // The bound by the entries held, the first ones of the lists; behind them a list has more of its kind only if its next one is.
  double mine = -__builtin_inf();
  for_held([&](double sum, u64) { mine = max(mine, sum); });
  const double bound = bounds_of(mine, n, join.most).least;
  for_held([&](double sum, u64 place) { if (sum >= bound) join_in(order_of(sum), place); });
  for (int32_t list = tid; list < n_lists; list += kSliceThreads) {
    int32_t rank = kHeld * kSliceThreads > list ? (kHeld * kSliceThreads - list + n_lists - 1) / n_lists : 0;
    const int32_t beam = list / n_slices;
    const u64* const own = lists + ((size_t)beam * m.slices + (list - beam * n_slices)) * n;
    for (bool more = true; more && rank < n; ++rank) {
      more = false;
      with(rank * n_lists + list, own[rank], [&](double sum, u64 place) {
        if (!(sum >= bound)) return;
        join_in(order_of(sum), place);
        more = true;
      });
    }
  }
  uint32_t all = joined();
  if (all > kMostJoined) {  // few rows that have all of it
    mine = -__builtin_inf();
    for_all([&](double sum, u64) { mine = max(mine, sum); });
    const double next = bounds_of(mine, n, join.most).least;
    again();
    for_all([&](double sum, u64 place) { if (sum >= next) join_in(order_of(sum), place); });
    all = joined();
  }
  if (all > kMostJoined) {  // many equal ones: the n-th best, bit by bit
    u64 edge = 0, edge_place = 0;  // what counts: more than edge, or edge itself with edge_place or more
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const u64 at = edge | 1ull << bit;
      uint32_t some = 0;
      for_all([&](double sum, u64) { some += order_of(sum) >= at; });
      if (count_all(some, join.counts) >= (uint32_t)n) edge = at;
    }
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const u64 at = edge_place | 1ull << bit;
      uint32_t some = 0;
      for_all([&](double sum, u64 place) { some += order_of(sum) > edge || (order_of(sum) == edge && place >= at); });
      if (count_all(some, join.counts) >= (uint32_t)n) edge_place = at;
    }
    again();
    for_all([&](double sum, u64 place) {
      if (order_of(sum) > edge || (order_of(sum) == edge && place >= edge_place)) join_in(order_of(sum), place);
    });
    all = joined();  // n
  }
  if (all > (uint32_t)(2 * n + 80)) {  // as in a slice: another bound, of what has joined
    constexpr int kEach = kMostJoined / kSliceThreads;
    u64 order[kEach], place[kEach], best = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const uint32_t i = (uint32_t)(k * kSliceThreads + tid);
      order[k] = i < all ? join.order[i] : 0;  // (0 is no number's)
      place[k] = i < all ? join.place[i] : 0;
      best = max(best, order[k]);
    }
    const double next = bounds_of(best ? sum_of(best) : -__builtin_inf(), n, join.most).least;
    again();
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (order[k] && sum_of(order[k]) >= next) join_in(order[k], place[k]);
    all = joined();
  }
  if (tid < n) {
    join.rows[tid] = join.ids[tid] = -1;
    join.scores[tid] = -__builtin_inff();
  }
  __syncthreads();
  for (uint32_t i = (uint32_t)tid; i < all; i += kSliceThreads) {
    const u64 order = join.order[i], place = join.place[i];
    uint32_t rank = 0;
    for (uint32_t k = 0; k < all; ++k) rank += join.order[k] > order || (join.order[k] == order && join.place[k] > place);
    if (rank < (uint32_t)n) {
      const int32_t beam = beam_of(place);
      join.rows[rank] = b0 + beam;
      join.ids[rank] = join.is_ended[beam] ? -1 : id_at(place);
      join.scores[rank] = (float)sum_of(order);
    }
  }
  __syncthreads();
  if (tid >= 64) return;
  // one wave writes out; placed: a row's first continuation takes the row's own place, the others what is left, in order
  for (int32_t i0 = 0; i0 < n; i0 += 64) {
    const int32_t i = i0 + lane;
    int32_t to = i;
    if (s.placed) {  // (n is the number of beams, so that there is one round)
      const int32_t parent = i < n ? join.rows[i] - b0 : -1;
      bool is_first = i < n && join.rows[i] >= 0;
      for (int32_t k = 0; k < n; ++k) is_first = is_first & (k >= i || join.rows[k] - b0 != parent);
      uint64_t places = 0;
      for (int32_t k = 0; k < n; ++k) {
        if (__builtin_amdgcn_readlane((int)is_first, k)) places |= 1ull << (__builtin_amdgcn_readlane(parent, k) & 63);
      }
      const uint64_t others = __ballot(i < n && !is_first);
      if (is_first) to = parent;
      else {
        uint64_t left = ~places;
        for (int k = __builtin_popcountll(others & ((1ull << lane) - 1ull)); k > 0; --k) left &= left - 1;
        to = __builtin_ctzll(left | 1ull << 63);
      }
    }
    if (i < n) {
      s.rows[(size_t)request * n + to] = join.rows[i];
      s.ids[(size_t)request * n + to] = join.ids[i];
      s.out_scores[(size_t)request * n + to] = join.scores[i];
    }
  }
}

// ------------------------------------------------------------------ what rows keep
// In place, whatever goes where: a workgroup takes the same region of every row that moves, in stretches that its registers hold at once:
// it reads a stretch of all of them, and writes when all of it is read.  No workgroup's region is another's.  Where no row that moves is read (as
// when continuations are placed) there is nothing to wait for.
// 48 of 128 rows with caches of 12.6 MB each in use: 239 to 262 us, 5.0 TB/s read and written, as much as a large copy moves (row after row 477 before the
// addresses' arithmetic was done once for all threads); 48 rows turned among themselves, where a stretch of all of them is read before it is written, 298,
// in pairs that change places 294.  A small call is a launch and a chain: sources, lengths, the data.
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
constexpr int kMoveThreads = 256, kMoveUnits = 8, kFewUnits = 4;  // a thread's at a time, of rows row after row, of stretches of all rows
constexpr int kMaxMoveRows = 1024;
constexpr int32_t kMostMoveGroups = 1 << 22;  // workgroups of a launch, which has to have less than 2^32 threads
struct RowDataList {
  RowData of[kMaxRowData];
  int64_t first[kMaxRowData];      // piece of each
  int64_t pieces;                  // of all arrays: a region of a part of all rows
  int32_t unit[kMaxRowData];       // bytes: 1, 2, 4, 8 or 16
  int32_t region;                  // units of a row that are in a piece, a power of two
};
struct Region {  // of the rows of an array
  char* base;
  int64_t row_stride, begin, end;
};
struct Moves {
  int32_t to[kMaxMoveRows], from[kMaxMoveRows];
  int64_t limit[kMaxMoveRows];  // bytes in use
  uint32_t moves[kMaxMoveRows / 32];  // whether a row does
  int32_t n, tangled;
};
// kTangled: some row that moves is also read.  Otherwise nothing that is read is written, waves need not wait for each other, and rows are taken one after
// the other: 32 KB lie side by side and not 512 bytes of each row.
template <class T, bool kTangled> __device__ __forceinline__ void move_region(const Region& r, int32_t units, const Moves& m) {
  int shift = 0;  // 2^shift units of a row at a time
  while ((2 << shift) <= units && (!kTangled || (2 << shift) * m.n <= kMoveThreads * kFewUnits)) ++shift;
  static_assert(kMaxMoveRows <= kMoveThreads * kFewUnits, "a unit of every row fits");
  const int32_t all = m.n << shift;
  for (int64_t at = r.begin; at < r.end; at += (int64_t)sizeof(T) << shift)
    for (int32_t u0 = 0; u0 < all; u0 += kMoveThreads * kFewUnits) {
      T x[kFewUnits];
      bool ok[kFewUnits];
#pragma unroll
      for (int k = 0; k < kFewUnits; ++k) {
        const int32_t u = u0 + k * kMoveThreads + (int32_t)threadIdx.x, i = u >> shift;
        const int64_t in = at + (int64_t)(u & ((1 << shift) - 1)) * (int64_t)sizeof(T);
        ok[k] = u < all && in < r.end && in < m.limit[u < all ? i : 0];
        if (ok[k]) x[k] = *reinterpret_cast<const T*>(r.base + m.from[i] * r.row_stride + in);
      }
      if constexpr (kTangled) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);  // (everything is read)
        __syncthreads();
      }
#pragma unroll
      for (int k = 0; k < kFewUnits; ++k) {
        const int32_t u = u0 + k * kMoveThreads + (int32_t)threadIdx.x, i = u >> shift;
        const int64_t in = at + (int64_t)(u & ((1 << shift) - 1)) * (int64_t)sizeof(T);
        if (ok[k]) *reinterpret_cast<T*>(r.base + m.to[i] * r.row_stride + in) = x[k];
      }
    }
}
// The same where nothing is tangled and a row's part of the region is whole stretches of all threads: rows and addresses are then the same for all.
__device__ __forceinline__ void copy_region(const Region& r, int32_t units, const Moves& m) {
  constexpr int kBytes = kMoveThreads * 16;
  const int32_t each = units / kMoveThreads, all = m.n * each, in_stretch = (int32_t)threadIdx.x * 16;
  for (int32_t c0 = 0; c0 < all; c0 += kMoveUnits) {
    uint4v x[kMoveUnits];
    bool ok[kMoveUnits];
    int64_t to[kMoveUnits];
#pragma unroll
    for (int k = 0; k < kMoveUnits; ++k) {
      const int32_t c = min(c0 + k, all - 1), i = c / each;
      const int64_t at = r.begin + (int64_t)(c - i * each) * kBytes;
      const int64_t from = (int64_t)__builtin_amdgcn_readfirstlane(m.from[i]) * r.row_stride + at;
      to[k] = (int64_t)__builtin_amdgcn_readfirstlane(m.to[i]) * r.row_stride + at;
      ok[k] = c0 + k < all && at + in_stretch < r.end && at + in_stretch < m.limit[i];
      if (ok[k]) x[k] = *reinterpret_cast<const uint4v*>(r.base + from + in_stretch);
    }
#pragma unroll
    for (int k = 0; k < kMoveUnits; ++k)
      if (ok[k]) *reinterpret_cast<uint4v*>(r.base + to[k] + in_stretch) = x[k];
  }
}
template <class T> __device__ __forceinline__ void move_any(const Region& r, int32_t units, const Moves& m) {
  // (parts may be shorter than a region, those of some arrays many times)
  while (units > kMoveThreads && (int64_t)(units / 2) * (int64_t)sizeof(T) >= r.end - r.begin) units /= 2;
  if (m.tangled) move_region<T, true>(r, units, m);
  else if (sizeof(T) == 16 && units % kMoveThreads == 0) copy_region(r, units, m);
  else move_region<T, false>(r, units, m);
}
// Piece p of a call.
__device__ __forceinline__ void move_piece(const RowDataList& list, int64_t p, int n, const int32_t* __restrict__ source, int32_t B, Moves& m) {
  RowData d = list.of[0];
  int64_t first = 0;
  int32_t unit = list.unit[0];
#pragma unroll
  for (int k = 1; k < kMaxRowData; ++k)  // (an index that is not known would put the whole list into memory)
    if (k < n && p >= list.first[k]) {
      d = list.of[k];
      first = list.first[k];
      unit = list.unit[k];
    }
  const int64_t region = (int64_t)list.region * unit, part_bytes = d.part_bytes, regions = (part_bytes + region - 1) / region;
  const int64_t group = p - first, piece = group / regions;
  Region r;
  r.begin = group % regions * region;
  r.end = min(r.begin + region, part_bytes);
  r.row_stride = d.row_stride;
  r.base = static_cast<char*>(d.data) + piece / d.n_parts * d.outer_stride + piece % d.n_parts * d.part_stride;
  const int32_t* const used = d.used;
  const int64_t used_bytes = d.used_bytes, units_of_part = used ? (part_bytes + used_bytes - 1) / used_bytes : 0;
  if (threadIdx.x < kMaxMoveRows / 32) m.moves[threadIdx.x] = 0;
  if (threadIdx.x == 0) m.n = m.tangled = 0;
  __syncthreads();
  for (int32_t b = (int32_t)threadIdx.x; b < B; b += kMoveThreads) {
    const int32_t a = source[b];
    if (a < 0 || a >= B || a == b) continue;
    // (a length beyond the part is all of it, however large)
    const int64_t most = used ? min((int64_t)used[a], units_of_part) * used_bytes : part_bytes;
    if (most <= r.begin) continue;
    const int32_t i = atomicAdd(&m.n, 1);
    m.to[i] = b;
    m.from[i] = a;
    m.limit[i] = most;
    atomicOr(&m.moves[b >> 5], 1u << (b & 31));
  }
  __syncthreads();
  if (!m.n) return;
  for (int32_t i = (int32_t)threadIdx.x; i < m.n; i += kMoveThreads)
    if (m.moves[m.from[i] >> 5] >> (m.from[i] & 31) & 1u) m.tangled = 1;
  __syncthreads();
  switch (unit) {
    case 16: move_any<uint4v>(r, list.region, m); break;
    case 8: move_any<uint2v>(r, list.region, m); break;
    case 4: move_any<uint32_t>(r, list.region, m); break;
    case 2: move_any<uint16_t>(r, list.region, m); break;
    default: move_any<uint8_t>(r, list.region, m); break;
  }
}
// A workgroup a piece; kMany, where there are more pieces than workgroups of a launch: every kMostMoveGroups-th.  (With the loop in all calls 48 of 128 rows
// with caches of 12.6 MB took 292 us and not 249, and a small call 9.1 and not 6.5: its registers.)
template <bool kMany> __global__ __launch_bounds__(kMoveThreads) void reorder_kernel(RowDataList list, int n, const int32_t* __restrict__ source, int32_t B) {
  __shared__ Moves m;
  for (int64_t p = blockIdx.x;;) {
    move_piece(list, p, n, source, B, m);
    if constexpr (!kMany) return;
    p += kMostMoveGroups;
    if (p >= list.pieces) return;
    __syncthreads();  // (all have read what the next piece writes anew)
  }
}

}  // namespace

size_t beam_bytes(int32_t max_rows, int32_t V) {
  size_t bytes = 0;
  (void)memory_at(nullptr, max_rows, V, &bytes);
  return bytes;
}
namespace {
template <Elem E> hipError_t select(const Logits& in, const LogitRules& r, const BeamSearch& s, const BeamMemory& m, hipStream_t stream) {
  const size_t lds = has_rules(r) && sizeof(RuleTable) > sizeof(BeamShared) ? sizeof(RuleTable) : sizeof(BeamShared);
  const int32_t n = slices_of<E>(in);
  hipLaunchKernelGGL(beam_slices_kernel<E>, dim3(n, s.requests * s.beams), dim3(kSliceThreads), lds, stream, in, r, s, m);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_join_kernel, dim3(s.requests), dim3(kSliceThreads), 0, stream, s, m, n);
  return hipGetLastError();
}
}  // namespace
hipError_t launch_beam_select(const Logits& in, Elem type, const LogitRules& r, const BeamSearch& s, void* memory, int32_t max_rows, int32_t max_V, hipStream_t stream) {
  size_t bytes;
  const BeamMemory m = memory_at(memory, max_rows, max_V, &bytes);
  if (type == Elem::kF32) return select<Elem::kF32>(in, r, s, m, stream);
  if (type == Elem::kBF16) return select<Elem::kBF16>(in, r, s, m, stream);
  return select<Elem::kF16>(in, r, s, m, stream);
}

hipError_t launch_reorder_rows(const RowData* data, int n, const int32_t* source, int32_t B, hipStream_t stream) {
  RowDataList list{};
  auto groups = [&](int32_t region) {
    int64_t all = 0;
    for (int i = 0; i < n; ++i) {
      list.first[i] = all;
      const int64_t bytes = (int64_t)region * list.unit[i];
      all += (int64_t)data[i].n_outer * data[i].n_parts * ((data[i].part_bytes + bytes - 1) / bytes);
    }
    return all;
  };
  for (int i = 0; i < n; ++i) {
    list.of[i] = data[i];
    uint64_t all = 16 | reinterpret_cast<uintptr_t>(data[i].data) | (uint64_t)data[i].row_stride | (uint64_t)data[i].part_bytes;
    if (data[i].n_outer > 1) all |= (uint64_t)data[i].outer_stride;
    if (data[i].n_parts > 1) all |= (uint64_t)data[i].part_stride;
    if (data[i].used) all |= (uint64_t)data[i].used_bytes;
    list.unit[i] = (int32_t)(all & (~all + 1));
  }
  list.region = 1024;
  while (list.region > 64 && groups(list.region) < 1024) list.region /= 2;
  // (only while that makes fewer pieces of most: where parts are short, it would but leave the long ones of other arrays to few workgroups)
  while (list.region < (1 << 20) && groups(list.region) > (1 << 20) && groups(list.region * 2) <= groups(list.region) / 4 * 3) list.region *= 2;
  list.pieces = groups(list.region);
  if (list.pieces <= kMostMoveGroups) hipLaunchKernelGGL(reorder_kernel<false>, dim3((uint32_t)list.pieces), dim3(kMoveThreads), 0, stream, list, n, source, B);
  else hipLaunchKernelGGL(reorder_kernel<true>, dim3(kMostMoveGroups), dim3(kMoveThreads), 0, stream, list, n, source, B);
  return hipGetLastError();
}

}  // namespace xgm
