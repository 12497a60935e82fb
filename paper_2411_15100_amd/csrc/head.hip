// The output projection with a matrix in 4 bits, under the masks (section 2.1: a masked token's logit is -inf whatever
// its value, so its row of the matrix need not be read).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "elements.hpp"
#include "logits.hpp"

namespace xgm {

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <Elem H> __device__ __forceinline__ float4v mfma(uint4v a, uint4v b, float4v c) {
  if constexpr (H == Elem::kBF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A code n becomes the number 16 + n by one AND-OR: the code's bits are the top of the mantissa of 16.  Codes i and i + 4 of
// a word end up next to each other, so columns are taken in the order 0 4 1 5 2 6 3 7 on both sides.  What the 16 and the
// zero point add is (16 + zero) times the sum of the hidden states, exact in its products as the rest is.
// (The two constants are kept from the compiler, which else spends an AND and an OR with a literal each: an instruction takes one
// of them from a scalar register and the other from a vector register.)
template <Elem H> struct Numbers {
  uint32_t mask = H == Elem::kBF16 ? 0x00780078u : 0x03c003c0u, sixteen = H == Elem::kBF16 ? 0x41804180u : 0x4c004c00u;
  __device__ __forceinline__ Numbers() { asm("" : "+s"(mask), "+v"(sixteen)); }
  __device__ __forceinline__ uint4v operator()(uint32_t w) const {
    if constexpr (H == Elem::kBF16)
      return uint4v{(w << 3 & mask) | sixteen, (w >> 1 & mask) | sixteen, (w >> 5 & mask) | sixteen, (w >> 9 & mask) | sixteen};
    else
      return uint4v{(w << 6 & mask) | sixteen, (w << 2 & mask) | sixteen, (w >> 2 & mask) | sixteen, (w >> 6 & mask) | sixteen};
  }
};
template <Elem H> constexpr uint32_t kOnes = H == Elem::kBF16 ? 0x3f803f80u : 0x3c003c00u;

// 8 hidden states in that order
__device__ __forceinline__ uint4v in_order(uint4v x) {
  return uint4v{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}

// word j of the quarter q of a wave <-> word q of quarter j
__device__ __forceinline__ uint4v exchanged(uint4v d) {
  auto a = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
  auto e = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto f = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  return uint4v{e[0], e[1], f[0], f[1]};
}

__device__ __forceinline__ void store_logit(const Head& h, Elem type, int64_t at, float y) {
  if (type == Elem::kF32) static_cast<uint32_t*>(h.logits)[at] = narrowed<Elem::kF32>(y);
  else if (type == Elem::kBF16) static_cast<uint16_t*>(h.logits)[at] = narrowed<Elem::kBF16>(y);
  else static_cast<uint16_t*>(h.logits)[at] = narrowed<Elem::kF16>(y);
}

// ---------------------------------------------------------------- few rows in the batch
// Shares of 16 NB rows, whose hidden states and their sums fit LDS.  A wave takes 16 rows of the matrix (a tile) and all columns, so
// that waves need nothing of each other: it reads the codes a step of 512 columns (4 chunks of 128) at a time, the next ones while
// it multiplies the last, 64 bytes of each row and chunk.  Hidden states lie in LDS in the order in which the products take them,
// zeros behind the last column (what is read of the matrix there is some earlier part of the row); rows of the batch that are not
// there are read from the last one and their sums dropped.
// Under masks the workgroup lists the rows of its share that some request allows, and its waves take 16 of those at a time.
// Where a workgroup has fewer tiles than waves, several waves take the steps of one in turn and their sums meet in LDS.
// One row of the batch is bound by the bytes of the matrix: 128256 rows of 4096 columns take 55 us, 4.9 TB/s, as much as a large copy
// moves.  24 rows (50001 x 2080, groups of 32, zero points: 51 us, 1.3 TB/s) are bound by what is done for each 32 columns of a tile
// besides two products: unpacking, scale, zero point, and 4 KB out of LDS.
// P: parts of a step that have a scale of their own: 4 (groups of 128 or a multiple), 8 (64) or 16 (32, or other multiples of it).
constexpr int kFewMaxThreads = 1024;  // of NB = 1; two rows of products need the registers of half as many waves
template <int NB> constexpr int kFewThreads = kFewMaxThreads / NB;
constexpr int kFewRows = 1024;  // of the matrix at a time (a list of them lies in LDS)
constexpr int kChunks = 4;      // of a step
constexpr uint32_t kFewMaxLds = 160 * 1024;

struct FewLayout {  // of dynamic LDS, bytes
  uint32_t sums, partial, list, end;
};
__host__ __device__ inline int32_t few_steps(int32_t K) { return (K + 128 * kChunks - 1) / (128 * kChunks); }
__host__ __device__ inline FewLayout few_layout(int32_t K, int32_t rows, int parts, int nb) {
  const uint32_t steps = (uint32_t)few_steps(K);
  FewLayout l;
  l.sums = steps * kChunks * 256 * (uint32_t)rows;
  l.partial = l.sums + steps * (uint32_t)(parts * nb * 64);
  l.list = l.partial + kFewMaxThreads * 16;
  l.end = l.list + kFewRows * 4 + kFewRows / 32 * 4 + 16;
  return l;
}

// the scales and zero points of a row over a step, as they lie in memory
template <int P, bool Z> struct StepGroups {
  uint32_t scales[P / 2];
  uint32_t zeros[P / 4];
};
// per_row groups of the row begin `row` behind the two addresses; columns_each: of a group, in units of 512 / P
template <int P, bool Z>
__device__ __forceinline__ void load_groups(StepGroups<P, Z>& g, const uint16_t* scales, const uint8_t* zeros, uint32_t row, int32_t step, int32_t per_row, int32_t units) {
  if (units == 1 && (step + 1) * P <= per_row) {
    __builtin_memcpy(g.scales, scales + row + step * P, 2 * P);
    if constexpr (Z) __builtin_memcpy(g.zeros, zeros + row + step * P, P);
    return;
  }
  for (int p = 0; p < P / 2; ++p) g.scales[p] = 0;
  for (int p = 0; p < P / 4; ++p) g.zeros[p] = 0;
  for (int p = 0; p < P; ++p) {
    const int32_t at = min((step * P + p) / units, per_row - 1);
    g.scales[p / 2] |= (uint32_t)scales[row + at] << (16 * (p & 1));
    if constexpr (Z) g.zeros[p / 4] |= (uint32_t)zeros[row + at] << (8 * (p & 3));
  }
}

// Lists the rows of the matrix among the `here` <= kFewRows from `base` (a multiple of 16) on that some of the `rows` rows of the batch
// from first_b on allows, as numbers behind base, and masks the logits of the others.  Returns how many.
__device__ int32_t list_rows(const Head& h, Elem out_type, int32_t first_b, int32_t rows, int64_t base, int32_t here, int32_t* list, uint32_t* any, int32_t* n_listed) {
  const int32_t tid = (int32_t)threadIdx.x, threads = (int32_t)blockDim.x;
  __syncthreads();
  if (tid < kFewRows / 32) any[tid] = 0;
  if (tid == 0) *n_listed = 0;
  __syncthreads();
  const int32_t w0 = (int32_t)(base >> 5), shift = (int32_t)(base & 31), words = (here + shift + 31) / 32;
  for (int32_t i = tid; i < words * rows; i += threads) {
    const int32_t b = i / words, w = i % words;
    uint32_t m = w0 + w < h.W_mask ? h.mask[(size_t)(first_b + b) * h.W_mask + w0 + w] : 0u;
    if (w0 + w == h.V_mask >> 5) m &= (1u << (h.V_mask & 31)) - 1u;  // (what lies behind the masks' vocabulary is not listed)
    if (m && shift) {
      if (w > 0) atomicOr(&any[w - 1], m << 16);
      if (w < kFewRows / 32) atomicOr(&any[w], m >> 16);
    } else if (m) {
      atomicOr(&any[w], m);
    }
  }
  __syncthreads();
  for (int32_t r = tid; r < here; r += threads) {
    if (any[r >> 5] >> (r & 31) & 1u) {
      int32_t place = __builtin_popcount(any[r >> 5] & ((1u << (r & 31)) - 1u));
      for (int32_t w = 0; w < r >> 5; ++w) place += __builtin_popcount(any[w]);
      list[place] = r;
      atomicAdd(n_listed, 1);
    } else {
      for (int32_t b = 0; b < rows; ++b) store_logit(h, out_type, (int64_t)(first_b + b) * h.logits_stride + base + r, -__builtin_inff());
    }
  }
  __syncthreads();
  return *n_listed;
}

template <Elem H, int NB, int P, bool Z>
__global__ __launch_bounds__(kFewThreads<NB>) void q4_few_kernel(Head h, Elem out_type, int32_t tiles_each) {
  extern __shared__ __align__(16) char lds[];
  constexpr int kParts = P / kChunks, kProducts = 4 / kParts;  // of a chunk, of a part
  constexpr bool kAsTheyLie = kParts == 1;
  const int32_t tid = (int32_t)threadIdx.x, threads = (int32_t)blockDim.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = threads >> 6;
  const int32_t n = lane & 15, q = lane >> 4;  // row of the tile (and of the batch, on the other side), quarter of the wave
  const int32_t first_b = (int32_t)blockIdx.y * 16 * NB, rows = min(h.B - first_b, 16 * NB);
  const int32_t n_steps = few_steps(h.K);
  const FewLayout at = few_layout(h.K, min(h.B, 16 * NB), P, NB);
  uint4v* const hidden = reinterpret_cast<uint4v*>(lds);  // [chunk][product][quarter][row]
  float4v* const hidden_sums = reinterpret_cast<float4v*>(lds + at.sums);  // [step][part][NB][quarter]
  float4v* const partial = reinterpret_cast<float4v*>(lds + at.partial);  // [wave][lane]
  int32_t* const list = reinterpret_cast<int32_t*>(lds + at.list);
  uint32_t* const any = reinterpret_cast<uint32_t*>(list + kFewRows);
  int32_t* const n_listed = reinterpret_cast<int32_t*>(any + kFewRows / 32);

  // product i of a chunk takes columns 32 i + 8 q .. of it, or 32 q + 8 i, as the codes lie in memory, where the chunk has one scale
  for (int32_t b = 0; b < rows; ++b) {
    const uint16_t* row = static_cast<const uint16_t*>(h.hidden) + (int64_t)(first_b + b) * h.hidden_stride;
    for (int32_t k8 = tid; k8 < n_steps * kChunks * 16; k8 += threads) {
      uint4v v = {0, 0, 0, 0};
      if (k8 * 8 < h.K) v = *reinterpret_cast<const uint4v*>(row + k8 * 8);
      const int32_t in = k8 & 15, place = kAsTheyLie ? (in & 3) * 4 + (in >> 2) : in;
      hidden[((k8 >> 4) * 16 + place) * rows + b] = in_order(v);
    }
  }
  const uint4v* mine[NB];
  for (int nb = 0; nb < NB; ++nb) mine[nb] = hidden + q * rows + min(nb * 16 + n, rows - 1);
  auto state = [&](int32_t product, int nb) { return mine[nb][product * 4 * rows]; };  // (4 products to a chunk)
  bool summed = false;
  const Numbers<H> numbers;

  const int32_t per_row = h.K / h.group, units = h.group / (512 / P);
  const uint32_t last_codes = (uint32_t)(h.K / 2 - 16);
  const int64_t row0 = (int64_t)blockIdx.x * tiles_each * 16, row1 = min((int64_t)h.V, row0 + (int64_t)tiles_each * 16);
  for (int64_t base = row0; base < row1; base += kFewRows) {
    const int32_t here = (int32_t)min((int64_t)kFewRows, row1 - base);
    int32_t count = here;
    if (h.mask) {
      count = list_rows(h, out_type, first_b, rows, base, here, list, any, n_listed);
    }
    const int32_t tiles = (count + 15) / 16;
    int32_t sharing = 1;  // waves to a tile, no more than there are where masks leave no tile
    while (sharing * 2 <= n_steps && sharing * 2 * max(tiles, 1) <= waves) sharing *= 2;
    const int32_t sub = wave & (sharing - 1), abreast = waves / sharing, rounds = (tiles + abreast - 1) / abreast;
    const uint8_t* const base_codes = h.codes + base * (h.K / 2);
    const uint16_t* const base_scales = static_cast<const uint16_t*>(h.scales) + base * per_row;
    const uint8_t* const base_zeros = Z ? h.zeros + base * per_row : nullptr;
    uint4v codes[kChunks], next_codes[kChunks];
    StepGroups<P, Z> groups, next_groups;
    auto row_of = [&](int32_t t) -> uint32_t {
      const int32_t i = min(t * 16 + n, count - 1);
      return (uint32_t)(h.mask ? list[i] : i);
    };
    auto load = [&](uint32_t v, int32_t step, uint4v (&c)[kChunks], StepGroups<P, Z>& g) {
      const uint32_t row = v * (uint32_t)(h.K / 2);
#pragma unroll
      for (int j = 0; j < kChunks; ++j)
        c[j] = *reinterpret_cast<const uint4v*>(base_codes + (row + min((uint32_t)((step * kChunks + j) * 64 + q * 16), last_codes)));
      load_groups<P, Z>(g, base_scales, base_zeros, v * (uint32_t)per_row, step, per_row, units);
    };
    int32_t t = wave / sharing;
    uint32_t v = 0, next_v = 0;
    if (t < tiles) {
      v = next_v = row_of(t);
      load(v, sub, codes, groups);
    }
    if (!summed) {  // (the first codes are on their way meanwhile)
      summed = true;
      __syncthreads();
      for (int32_t u = wave; u < n_steps * P; u += waves) {
        const uint4v ones = {kOnes<H>, kOnes<H>, kOnes<H>, kOnes<H>};
        for (int nb = 0; nb < NB; ++nb) {
          float4v s = {0, 0, 0, 0};
          for (int i = 0; i < kProducts; ++i) s = mfma<H>(state(u * kProducts + i, nb), ones, s);
          if (n == 0) hidden_sums[(u * NB + nb) * 4 + q] = Z ? s : s * -24.0f;
        }
      }
      __syncthreads();
    }
    for (int32_t round = 0; round < rounds; ++round) {
      float4v acc[NB];
      for (int nb = 0; nb < NB; ++nb) acc[nb] = float4v{0, 0, 0, 0};
      if (t < tiles) {
        for (int32_t step = sub; step < n_steps; step += sharing) {
          int32_t next_t = t, next_step = step + sharing;
          if (next_step >= n_steps) {
            next_step = sub;
            next_t += abreast;
            if (next_t < tiles) next_v = row_of(next_t);
          }
          if (next_t < tiles) load(next_v, next_step, next_codes, next_groups);
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            if ((step * kChunks + j) * 128 >= h.K) break;
            const uint4v c = kAsTheyLie ? codes[j] : exchanged(codes[j]);
#pragma unroll
            for (int r = 0; r < kParts; ++r) {
              const int p = j * kParts + r;
              const float scale = widened<H>((uint16_t)(groups.scales[p / 2] >> (16 * (p & 1))));
              const float shift = Z ? -16.0f - (float)(groups.zeros[p / 4] >> (8 * (p & 3)) & 255u) : 0.0f;
              float4v part[NB];
              for (int nb = 0; nb < NB; ++nb) {
                part[nb] = hidden_sums[((step * P + p) * NB + nb) * 4 + q];
                if constexpr (Z) part[nb] *= shift;
              }
#pragma unroll
              for (int i = r * kProducts; i < (r + 1) * kProducts; ++i) {
                const uint4v w = numbers(c[i]);
                for (int nb = 0; nb < NB; ++nb) part[nb] = mfma<H>(state((step * kChunks + j) * 4 + i, nb), w, part[nb]);
              }
              for (int nb = 0; nb < NB; ++nb) acc[nb] += part[nb] * scale;
            }
            __builtin_amdgcn_sched_barrier(0);  // (else hidden states of all chunks are read at once, and registers spill)
          }
          for (int j = 0; j < kChunks; ++j) codes[j] = next_codes[j];
          groups = next_groups;
        }
      }
      for (int nb = 0; nb < NB; ++nb) {
        if (sharing > 1) {
          partial[tid] = acc[nb];
          __syncthreads();
          if (sub == 0)
            for (int32_t w = 1; w < sharing; ++w) acc[nb] += partial[tid + w * 64];
          __syncthreads();
        }
        if (sub == 0 && t * 16 + n < count) {
          for (int i = 0; i < 4; ++i) {
            const int32_t b = nb * 16 + q * 4 + i;
            if (b >= rows) continue;
            const int64_t token = base + v;
            const bool ok = !h.mask || (h.mask[(size_t)(first_b + b) * h.W_mask + (token >> 5)] >> (token & 31) & 1u);
            store_logit(h, out_type, (int64_t)(first_b + b) * h.logits_stride + token, ok ? acc[nb][i] : -__builtin_inff());
          }
        }
      }
      t += abreast;
      v = next_v;
    }
  }
}

// --------------------------------------------------------------- many rows in the batch
// Up to 16 MW WM rows and any number of columns.  The eight waves of a workgroup form WM groups that share the rows of the batch, and
// in each 8 / WM waves that share the matrix, up to four tiles each: 64 x 64 logits a wave for MW = 4, for which it reads 4 KB of
// hidden states and 1 KB of codes out of LDS per 16 products.  Columns go by chunks of 128.  The codes of a chunk are read from
// memory three chunks before they are needed, by all waves in equal parts, and go through two buffers in LDS, hidden states
// through three; one barrier a chunk.
// A workgroup's share is cut into passes of the tiles that its waves hold.
// 128 rows (151936 x 4096, groups of 128) take 302 us, 0.53 PFLOP/s: the waves of a SIMD spend as long on unpacking codes, scaling sums and
// on LDS as on products, and the barrier of a chunk leaves little of one under the other.  With eight waves for 64 x 64 logits each
// instead of 32 x 32 it went from 565 to 441 us, with workgroups on different chunks to 303.
constexpr int kManyThreads = 512, kManyTiles = 4;  // tiles of a wave

// How the parts of a chunk find their scales: one for the chunk, looked up by its number; halves; quarters; quarters that are looked up.
enum Sharing : int { kWhole = 0, kHalves = 1, kQuarters = 2, kLookedUp = 3 };
template <int S> constexpr int kPartsOf = S == kWhole ? 1 : S == kHalves ? 2 : 4;
struct GroupIndex {
  int32_t per_row;     // groups of a row
  uint32_t reciprocal;  // of the parts in a group, in 2^-32 (0: one)
};
__device__ __forceinline__ int32_t group_of(GroupIndex g, int32_t part) {
  return min(g.reciprocal ? (int32_t)__umulhi((uint32_t)part, g.reciprocal) : part, g.per_row - 1);
}
template <int S, bool Z> struct ChunkGroups {  // scales and zero points of a row over a chunk
  uint32_t scales[S >= kQuarters ? 2 : 1];
  uint32_t zeros;
};
// The row begins `row` groups behind the two addresses.  Parts behind the last column get some scale of the row (kLookedUp), or 0.
template <int S, bool Z>
__device__ __forceinline__ void load_chunk_groups(ChunkGroups<S, Z>& g, const uint16_t* scales, const uint8_t* zeros, uint32_t row, int32_t chunk, GroupIndex index) {
  if constexpr (S == kWhole) {
    const uint32_t at = row + (uint32_t)group_of(index, chunk);
    g.scales[0] = scales[at];
    if constexpr (Z) g.zeros = zeros[at];
  } else if constexpr (S == kLookedUp) {
    g.scales[0] = g.scales[1] = g.zeros = 0;
    for (int p = 0; p < 4; ++p) {
      const uint32_t at = row + (uint32_t)group_of(index, chunk * 4 + p);
      g.scales[p / 2] |= (uint32_t)scales[at] << (16 * (p & 1));
      if constexpr (Z) g.zeros |= (uint32_t)zeros[at] << (8 * p);
    }
  } else {
    constexpr int P = kPartsOf<S>;
    const int32_t first = min(chunk * P, index.per_row - P), behind = chunk * P - first;
    if constexpr (S == kHalves) {
      uint32_t x;
      __builtin_memcpy(&x, scales + row + first, 4);
      g.scales[0] = x >> (16 * behind);
      if constexpr (Z) {
        uint16_t z;
        __builtin_memcpy(&z, zeros + row + first, 2);
        g.zeros = (uint32_t)z >> (8 * behind);
      }
    } else {
      uint64_t x;
      __builtin_memcpy(&x, scales + row + first, 8);
      x >>= 16 * behind;
      g.scales[0] = (uint32_t)x;
      g.scales[1] = (uint32_t)(x >> 32);
      if constexpr (Z) {
        uint32_t z;
        __builtin_memcpy(&z, zeros + row + first, 4);
        g.zeros = z >> (8 * behind);
      }
    }
  }
}

template <Elem H, int MW, int WM, int S, bool Z>
__global__ __launch_bounds__(kManyThreads, 2) void q4_many_kernel(Head h, Elem out_type, int32_t tiles_each, uint32_t reciprocal) {
  constexpr int PC = kPartsOf<S>, kRows = 16 * MW * WM, kWaves = kManyThreads / 64, kWide = kWaves / WM;  // waves that share the matrix
  constexpr int kPass = kWide * kManyTiles, kBring = kPass / kWaves;  // tiles of a pass; those of which a wave brings the codes
  constexpr int kUnits = (kRows * 16 + kManyThreads - 1) / kManyThreads;  // 8 hidden states each, that a thread brings a chunk
  constexpr int kProducts = 4 / PC;
  // [product and quarter][row], rows exchanged by the number of the first index: 16 rows of one, and one row of 16, lie in different banks
  __shared__ uint4v hidden[3][16 * kRows];
  __shared__ float4v sums[2][PC][kRows / 4];      // of the hidden states of a part
  __shared__ uint4v codes[2][kPass][64];
  __shared__ ChunkGroups<S, Z> groups[2][kPass][16];
  __shared__ int32_t list[kFewRows];
  __shared__ uint32_t any[kFewRows / 32];
  __shared__ int32_t n_listed;
  const int32_t tid = (int32_t)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t n = lane & 15, q = lane >> 4, wm = wave % WM, wn = wave / WM;
  const int32_t first_b = (int32_t)blockIdx.y * kRows, rows = min(h.B - first_b, kRows);
  const int32_t n_chunks = (h.K + 127) / 128;
  const GroupIndex index{h.K / h.group, reciprocal};
  const uint32_t last_codes = (uint32_t)(h.K / 2 - 16);
  const Numbers<H> numbers;
  const uint16_t* const all_states = static_cast<const uint16_t*>(h.hidden) + (int64_t)first_b * h.hidden_stride;

  // Rows of the matrix and of the hidden states lie a power of two apart as a rule, so that the same columns of all of them are on few
  // channels of the L2: the workgroups of an XCD begin with different chunks.
  const int32_t begin = (int32_t)(blockIdx.x >> 3) % n_chunks;
  auto turned = [&](int32_t chunk) { return chunk + begin < n_chunks ? chunk + begin : chunk + begin - n_chunks; };
  int64_t state_at[kUnits];  // where the thread's hidden states of a chunk begin, and where in a buffer they go
  int32_t state_to[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int32_t at = u * kManyThreads + tid, b = at >> 4, in = at & 15, place = PC == 1 ? (in & 3) * 4 + (in >> 2) : in;
    state_at[u] = (int64_t)min(b, rows - 1) * h.hidden_stride + in * 8;
    state_to[u] = place * kRows + (b ^ place);
  }
  const int32_t states_left = h.K - (tid & 15) * 8;  // columns from the thread's place on
  auto load_states = [&](int32_t turn, uint4v (&x)[kUnits]) {
    const int32_t chunk = turned(turn);
    const bool there = chunk * 128 < states_left;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      x[u] = uint4v{0, 0, 0, 0};
      if (there) x[u] = *reinterpret_cast<const uint4v*>(all_states + chunk * 128 + state_at[u]);
    }
  };
  auto put_states = [&](const uint4v (&x)[kUnits], int buffer) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
      if (kUnits * kManyThreads == kRows * 16 || u * kManyThreads + tid < kRows * 16) hidden[buffer][state_to[u]] = in_order(x[u]);
  };

  const int64_t row0 = (int64_t)blockIdx.x * tiles_each * 16, row1 = min((int64_t)h.V, row0 + (int64_t)tiles_each * 16);
  for (int64_t base = row0; base < row1; base += kFewRows) {
    const int32_t here = (int32_t)min((int64_t)kFewRows, row1 - base);
    int32_t count = here;
    if (h.mask) count = list_rows(h, out_type, first_b, rows, base, here, list, any, &n_listed);
    const int32_t tiles = (count + 15) / 16;
    const uint8_t* const base_codes = h.codes + base * (h.K / 2);
    const uint16_t* const base_scales = static_cast<const uint16_t*>(h.scales) + base * index.per_row;
    const uint8_t* const base_zeros = Z ? h.zeros + base * index.per_row : nullptr;
    auto row_of = [&](int32_t tile) -> uint32_t {
      const int32_t i = min(tile * 16 + n, count - 1);
      return (uint32_t)(h.mask ? list[i] : i);
    };
    for (int32_t pass = 0; pass < tiles; pass += kPass) {
      const int32_t pass_tiles = min(kPass, tiles - pass), each = (pass_tiles + kWide - 1) / kWide;
      const int32_t first = wn * each, mine = max(0, min(each, pass_tiles - first));
      const int32_t bring = max(0, min(kBring, pass_tiles - wave * kBring));
      uint32_t code_at[kBring], group_at[kBring];
#pragma unroll
      for (int c = 0; c < kBring; ++c) {
        const uint32_t v = row_of(pass + wave * kBring + c);
        code_at[c] = v * (uint32_t)(h.K / 2);
        group_at[c] = v * (uint32_t)index.per_row;
      }
      struct Brought {
        uint4v codes[kBring];
        ChunkGroups<S, Z> groups[kBring];
      };
      auto load = [&](int32_t turn, Brought& to) {
        const int32_t chunk = turned(turn);
        const uint32_t in_row = min((uint32_t)(chunk * 64 + q * 16), last_codes);
#pragma unroll
        for (int c = 0; c < kBring; ++c) {
          if (c >= bring) break;
          to.codes[c] = *reinterpret_cast<const uint4v*>(base_codes + (code_at[c] + in_row));
          load_chunk_groups<S, Z>(to.groups[c], base_scales, base_zeros, group_at[c], chunk, index);
        }
      };
      auto put = [&](const Brought& from, int buffer) {
#pragma unroll
        for (int c = 0; c < kBring; ++c) {
          if (c >= bring) break;
          codes[buffer][wave * kBring + c][lane] = PC == 1 ? from.codes[c] : exchanged(from.codes[c]);
          if (q == 0) groups[buffer][wave * kBring + c][n] = from.groups[c];
        }
      };
      float4v acc[kManyTiles][MW];
#pragma unroll
      for (int c = 0; c < kManyTiles; ++c)
        for (int m = 0; m < MW; ++m) acc[c][m] = float4v{0, 0, 0, 0};
      // the sums over the parts of a chunk, 16 rows to a wave
      auto add_up = [&](int at, int buffer) {
        if (wave >= kRows / 16) return;
        const uint4v ones = {kOnes<H>, kOnes<H>, kOnes<H>, kOnes<H>};
#pragma unroll
        for (int r = 0; r < PC; ++r) {
          float4v s = {0, 0, 0, 0};
          for (int i = r * kProducts; i < (r + 1) * kProducts; ++i) s = mfma<H>(hidden[at][(i * 4 + q) * kRows + wave * 16 + (n ^ (i * 4 + q))], ones, s);
          if (n == 0) sums[buffer][r][wave * 4 + q] = Z ? s : s * -24.0f;
        }
      };
      const int refill_at = wave < kWaves / 2 ? 0 : 2;  // (the two waves of a SIMD at different times: one multiplies while the other waits)
      auto multiply = [&](int at, int buffer, auto&& refill) {
#pragma unroll
        for (int r = 0; r < PC; ++r) {
          uint4v a[kProducts][MW];
#pragma unroll
          for (int i = 0; i < kProducts; ++i)
            for (int m = 0; m < MW; ++m) {
              const int32_t place = (r * kProducts + i) * 4 + q;
              a[i][m] = hidden[at][place * kRows + (wm * MW + m) * 16 + (n ^ place)];
            }
          // the sums of a tile are scaled while the next one's products are made
          float4v part[2][MW];
          float scale[2] = {0.0f, 0.0f};
#pragma unroll
          for (int c = 0; c <= kManyTiles; ++c) {
            if (r == 0 && (c == 0 || c == 2) && c == refill_at) refill();
            if (c < mine && c < kManyTiles) {
              const ChunkGroups<S, Z> g = groups[buffer][first + c][n];
              const uint4v four = codes[buffer][first + c][lane];
              scale[c & 1] = widened<H>((uint16_t)(g.scales[r / 2] >> (16 * (r & 1))));
              const float shift = Z ? -16.0f - (float)(g.zeros >> (8 * r) & 255u) : 1.0f;
              for (int m = 0; m < MW; ++m) {
                part[c & 1][m] = sums[buffer][r][(wm * MW + m) * 4 + q];
                if constexpr (Z) part[c & 1][m] *= shift;
              }
#pragma unroll
              for (int i = 0; i < kProducts; ++i) {
                const uint4v w = numbers(four[r * kProducts + i]);
                for (int m = 0; m < MW; ++m) part[c & 1][m] = mfma<H>(a[i][m], w, part[c & 1][m]);
              }
            }
            if (c > 0 && c <= mine)
              for (int m = 0; m < MW; ++m) acc[c - 1][m] += part[(c - 1) & 1][m] * scale[(c - 1) & 1];
            __builtin_amdgcn_sched_barrier(0);  // (what belongs to all tiles at once would not fit the registers)
          }
        }
      };
      uint4v x[kUnits];
      Brought next_codes;
      load_states(0, x);
      load(0, next_codes);
      __syncthreads();  // (the last pass has read its last chunk)
      put_states(x, 0);
      if (n_chunks > 1) {
        load_states(1, x);
        put_states(x, 1);
      }
      put(next_codes, 0);
      if (n_chunks > 2) load_states(2, x);
      if (n_chunks > 1) load(1, next_codes);
      __syncthreads();
      add_up(0, 0);
      __syncthreads();
      // multiplies a chunk, adds up the next one and puts into LDS what comes then: hidden states of the one after, in a ring
      // of three buffers, and codes of the next
      int ring = 0;
#pragma unroll 1
      for (int32_t chunk = 0; chunk < n_chunks; ++chunk) {
        const int buffer = chunk & 1, next = ring == 2 ? 0 : ring + 1, last = next == 2 ? 0 : next + 1;
        multiply(ring, buffer, [&] {
          if (chunk + 2 < n_chunks) {
            put_states(x, last);
            if (chunk + 3 < n_chunks) load_states(chunk + 3, x);
          }
          if (chunk + 1 < n_chunks) {
            put(next_codes, buffer ^ 1);
            if (chunk + 2 < n_chunks) load(chunk + 2, next_codes);
            add_up(next, buffer ^ 1);
          }
        });
        ring = next;
        __syncthreads();
      }
      auto store = [&](auto type) {
        constexpr Elem O = decltype(type)::value;
        int32_t row = wm * MW * 16 + q * 4;
        asm volatile("" : "+v"(row));  // (else the addresses of all rows are computed ahead of the loops and fill the registers)
        typename Type<O>::bits* const out = static_cast<typename Type<O>::bits*>(h.logits) + (int64_t)(first_b + row) * h.logits_stride + base;
        for (int c = 0; c < kManyTiles; ++c) {
          if (c >= mine || (pass + first + c) * 16 + n >= count) continue;
          const uint32_t v = row_of(pass + first + c);
          const int64_t token = base + v;
#pragma unroll
          for (int m = 0; m < MW; ++m)
            for (int i = 0; i < 4; ++i) {
              const int32_t b = row + m * 16 + i;
              if (b >= rows) continue;
              const bool ok = !h.mask || (h.mask[(size_t)(first_b + b) * h.W_mask + (token >> 5)] >> (token & 31) & 1u);
              float y = 0.0f;
#pragma unroll
              for (int e = 0; e < kManyTiles; ++e)
                if (e == c) y = acc[e][m][i];
              out[(int64_t)(m * 16 + i) * h.logits_stride + v] = narrowed<O>(ok ? y : -__builtin_inff());
            }
        }
      };
      if (out_type == Elem::kF32) store(std::integral_constant<Elem, Elem::kF32>());
      else if (out_type == Elem::kBF16) store(std::integral_constant<Elem, Elem::kBF16>());
      else store(std::integral_constant<Elem, Elem::kF16>());
    }
  }
}

constexpr int kComputeUnits = 256;

template <Elem H, int NB, int P, bool Z> hipError_t launch_few(const Head& h, Elem out_type, hipStream_t stream) {
  static LdsRoom room;
  if (const hipError_t e = room(reinterpret_cast<const void*>(&q4_few_kernel<H, NB, P, Z>), kFewMaxLds); e != hipSuccess) return e;
  const int32_t tiles = (int32_t)(((int64_t)h.V + 15) / 16), each = (tiles + kComputeUnits - 1) / kComputeUnits, steps = few_steps(h.K);
  int32_t threads = 64;  // waves for its tiles, or for the steps of the few that masks leave
  while (threads < kFewThreads<NB> && threads < 64 * (h.mask && steps > each ? steps : each * (each < 16 ? steps : 1))) threads *= 2;
  const dim3 grid((tiles + each - 1) / each, (h.B + 16 * NB - 1) / (16 * NB));
  hipLaunchKernelGGL((q4_few_kernel<H, NB, P, Z>), grid, dim3(threads), few_layout(h.K, h.B < 16 * NB ? h.B : 16 * NB, P, NB).end, stream, h, out_type, each);
  return hipGetLastError();
}
template <Elem H, int NB, int P> hipError_t launch_few_zeros(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.zeros) return launch_few<H, NB, P, true>(h, out_type, stream);
  return launch_few<H, NB, P, false>(h, out_type, stream);
}
int few_parts(int32_t group) { return group % 128 == 0 ? 4 : group == 64 ? 8 : 16; }
bool few_fits(const Head& h, int32_t rows, int nb) { return few_layout(h.K, rows, few_parts(h.group), nb).end <= kFewMaxLds; }
template <Elem H, int NB> hipError_t launch_few_groups(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.group % 128 == 0) return launch_few_zeros<H, NB, 4>(h, out_type, stream);
  if (h.group == 64) return launch_few_zeros<H, NB, 8>(h, out_type, stream);
  return launch_few_zeros<H, NB, 16>(h, out_type, stream);
}
template <Elem H, int MW, int WM, int S, bool Z> hipError_t launch_many(const Head& h, Elem out_type, hipStream_t stream) {
  const int32_t tiles = (int32_t)(((int64_t)h.V + 15) / 16), each = (tiles + kComputeUnits - 1) / kComputeUnits;
  const dim3 grid((tiles + each - 1) / each, (h.B + 16 * MW * WM - 1) / (16 * MW * WM));
  const uint32_t parts = (uint32_t)(h.group / (128 / kPartsOf<S>));
  hipLaunchKernelGGL((q4_many_kernel<H, MW, WM, S, Z>), grid, dim3(kManyThreads), 0, stream, h, out_type, each, parts > 1 ? (uint32_t)(((1ull << 32) + parts - 1) / parts) : 0u);
  return hipGetLastError();
}
template <Elem H, int MW, int WM, int S> hipError_t launch_many_zeros(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.zeros) return launch_many<H, MW, WM, S, true>(h, out_type, stream);
  return launch_many<H, MW, WM, S, false>(h, out_type, stream);
}
template <Elem H, int MW, int WM> hipError_t launch_many_groups(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.group % 128 == 0) return launch_many_zeros<H, MW, WM, kWhole>(h, out_type, stream);
  if (h.group == 64 && h.K >= 128) return launch_many_zeros<H, MW, WM, kHalves>(h, out_type, stream);
  if (h.group == 32 && h.K >= 128) return launch_many_zeros<H, MW, WM, kQuarters>(h, out_type, stream);
  return launch_many_zeros<H, MW, WM, kLookedUp>(h, out_type, stream);
}
// Up to 32 rows go through LDS as a whole where they fit: 24 rows of 50001 x 2080 in groups of 32 take 51 us that way and 63 as many
// rows, 17 of 151936 x 2048 73 and 115.  Where 17 to 32 rows do not fit but 16 do, the matrix is read twice: 24 rows of 50001 x 4096 in
// groups of 128 57 us, 70 as many rows; 32 of 151936 x 4096 150 and 158; under masks that leave 100 tokens a row 23 and 42.
template <Elem H> hipError_t launch_head(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.B <= 16 && few_fits(h, h.B, 1)) return launch_few_groups<H, 1>(h, out_type, stream);
  if (h.B <= 32 && few_fits(h, h.B, 2)) return launch_few_groups<H, 2>(h, out_type, stream);
  if (h.B <= 32 && few_fits(h, 16, 1)) return launch_few_groups<H, 1>(h, out_type, stream);
  if (h.B <= 32) return launch_many_groups<H, 2, 1>(h, out_type, stream);
  if (h.B <= 64) return launch_many_groups<H, 4, 1>(h, out_type, stream);
  return launch_many_groups<H, 4, 2>(h, out_type, stream);
}

}  // namespace

hipError_t launch_q4_logits(const Head& h, Elem hidden_type, Elem logits_type, hipStream_t stream) {
  if (hidden_type == Elem::kF16) return launch_head<Elem::kF16>(h, logits_type, stream);
  return launch_head<Elem::kBF16>(h, logits_type, stream);
}

}  // namespace xgm
