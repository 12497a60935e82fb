// The output projection with a matrix in 4 bits, under the masks (section 2.1: a masked token's logit is -inf whatever
// its value, so its row of the matrix need not be read).
#include <hip/hip_runtime.h>

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
template <Elem H> __device__ __forceinline__ uint4v numbers(uint32_t w) {
  if constexpr (H == Elem::kBF16)
    return uint4v{(w << 3 & 0x00780078u) | 0x41804180u, (w >> 1 & 0x00780078u) | 0x41804180u, (w >> 5 & 0x00780078u) | 0x41804180u,
                  (w >> 9 & 0x00780078u) | 0x41804180u};
  else
    return uint4v{(w << 6 & 0x03c003c0u) | 0x4c004c00u, (w << 2 & 0x03c003c0u) | 0x4c004c00u, (w >> 2 & 0x03c003c0u) | 0x4c004c00u,
                  (w >> 6 & 0x03c003c0u) | 0x4c004c00u};
}
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
// Up to 16 NB rows, whose hidden states fit LDS.  A wave takes 16 rows of the matrix (a tile) and all columns, so that waves need
// nothing of each other: it reads the codes a step of 512 columns (4 chunks of 128) at a time, the next ones while it multiplies
// the last, 64 bytes of each row and chunk.  Hidden states lie in LDS in the order in which the products take them, zeros behind
// the last column (what is read of the matrix there is some earlier part of the row); rows of the batch that are not there are read
// from the last one and their sums dropped.
// Under masks the workgroup lists the rows of its share that some request allows, and its waves take 16 of those at a time.
// Where a workgroup has fewer tiles than waves, several waves take the steps of one in turn and their sums meet in LDS.
// P: parts of a step that have a scale of their own: 4 (groups of 128 or a multiple), 8 (64) or 16 (32, or other multiples of it).
constexpr int kFewMaxThreads = 1024;
constexpr int kFewRows = 1024;  // of the matrix at a time (a list of them lies in LDS)
constexpr int kChunks = 4;      // of a step
constexpr size_t kFewHiddenBytes = 128 * 1024;  // at most, of hidden states in LDS

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

template <Elem H, int NB, int P, bool Z>
__global__ __launch_bounds__(kFewMaxThreads) void q4_few_kernel(Head h, Elem out_type, int32_t tiles_each) {
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

  const int32_t per_row = h.K / h.group, units = h.group / (512 / P);
  const uint32_t last_codes = (uint32_t)(h.K / 2 - 16);
  const int64_t row0 = (int64_t)blockIdx.x * tiles_each * 16, row1 = min((int64_t)h.V, row0 + (int64_t)tiles_each * 16);
  for (int64_t base = row0; base < row1; base += kFewRows) {
    const int32_t here = (int32_t)min((int64_t)kFewRows, row1 - base);
    int32_t count = here;
    if (h.mask) {
      __syncthreads();
      if (tid < kFewRows / 32) any[tid] = 0;
      if (tid == 0) *n_listed = 0;
      __syncthreads();
      const int32_t w0 = (int32_t)(base >> 5), shift = (int32_t)(base & 31), words = (here + shift + 31) / 32;  // (shares begin on 16)
      for (int32_t i = tid; i < words * rows; i += threads) {
        const int32_t b = i / words, w = i % words;
        const uint32_t m = h.mask[(size_t)(first_b + b) * h.W_mask + w0 + w];
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
      count = *n_listed;
    }
    const int32_t tiles = (count + 15) / 16;
    int32_t sharing = 1;  // waves to a tile
    while (sharing * 2 <= n_steps && sharing * 2 * tiles <= waves) sharing *= 2;
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
                const uint4v w = numbers<H>(c[i]);
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

// ------------------------------------------------------------------ any number of columns
constexpr int kAnyThreads = 256;

// A wave takes one row of the matrix and one of the batch; its lanes take the columns 8 at a time.
template <Elem H>
__global__ __launch_bounds__(kAnyThreads) void q4_any_kernel(Head h, Elem out_type) {
  const int32_t v = (int32_t)(blockIdx.x * (kAnyThreads / 64) + (threadIdx.x >> 6)), b = (int32_t)blockIdx.y, lane = (int32_t)(threadIdx.x & 63u);
  if (v >= h.V) return;
  const int64_t out = (int64_t)b * h.logits_stride + v;
  if (h.mask && !(h.mask[(size_t)b * h.W_mask + (v >> 5)] >> (v & 31) & 1u)) {
    if (lane == 0) store_logit(h, out_type, out, -__builtin_inff());
    return;
  }
  const uint16_t* x = static_cast<const uint16_t*>(h.hidden) + (int64_t)b * h.hidden_stride;
  const uint16_t* scales = static_cast<const uint16_t*>(h.scales) + (size_t)v * (h.K / h.group);
  const uint8_t* zeros = h.zeros ? h.zeros + (size_t)v * (h.K / h.group) : nullptr;
  const uint8_t* codes = h.codes + (size_t)v * (h.K / 2);
  float sum = 0.0f;
  for (int32_t k = lane * 8; k < h.K; k += 512) {
    const uint32_t n = *reinterpret_cast<const uint32_t*>(codes + k / 2);
    const int32_t g = k / h.group;
    const float z = zeros ? (float)zeros[g] : 8.0f;
    float part = 0.0f;
    for (int j = 0; j < 8; ++j) part += widened<H>(x[k + j]) * ((float)(n >> (4 * j) & 15u) - z);
    sum += part * widened<H>(scales[g]);
  }
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) store_logit(h, out_type, out, sum);
}

constexpr int kComputeUnits = 256;

template <Elem H, int NB, int P, bool Z> void launch_few(const Head& h, Elem out_type, hipStream_t stream) {
  static const bool prepared = hipFuncSetAttribute(reinterpret_cast<const void*>(&q4_few_kernel<H, NB, P, Z>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess;
  (void)prepared;
  const int32_t tiles = (int32_t)(((int64_t)h.V + 15) / 16), each = (tiles + kComputeUnits - 1) / kComputeUnits, steps = few_steps(h.K);
  int32_t threads = 64;  // waves for its tiles, or for the steps of the few that masks leave
  while (threads < kFewMaxThreads && threads < 64 * (h.mask && steps > each ? steps : each * (each < 16 ? steps : 1))) threads *= 2;
  const dim3 grid((tiles + each - 1) / each, (h.B + 16 * NB - 1) / (16 * NB));
  hipLaunchKernelGGL((q4_few_kernel<H, NB, P, Z>), grid, dim3(threads), few_layout(h.K, h.B < 16 * NB ? h.B : 16 * NB, P, NB).end, stream, h, out_type, each);
}
template <Elem H, int NB, int P> void launch_few_zeros(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.zeros) launch_few<H, NB, P, true>(h, out_type, stream);
  else launch_few<H, NB, P, false>(h, out_type, stream);
}
template <Elem H, int NB> void launch_few_groups(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.group % 128 == 0) launch_few_zeros<H, NB, 4>(h, out_type, stream);
  else if (h.group == 64) launch_few_zeros<H, NB, 8>(h, out_type, stream);
  else launch_few_zeros<H, NB, 16>(h, out_type, stream);
}
template <Elem H> void launch_head(const Head& h, Elem out_type, hipStream_t stream) {
  const size_t row = (size_t)few_steps(h.K) * kChunks * 256;  // bytes of LDS for a row of hidden states
  if (h.B > 16 && row * (h.B < 32 ? h.B : 32) <= kFewHiddenBytes) return launch_few_groups<H, 2>(h, out_type, stream);
  if (row * (h.B < 16 ? h.B : 16) <= kFewHiddenBytes) return launch_few_groups<H, 1>(h, out_type, stream);
  const dim3 grid((h.V + kAnyThreads / 64 - 1) / (kAnyThreads / 64), h.B);
  hipLaunchKernelGGL(q4_any_kernel<H>, grid, dim3(kAnyThreads), 0, stream, h, out_type);
}

}  // namespace

void launch_q4_logits(const Head& h, Elem hidden_type, Elem logits_type, hipStream_t stream) {
  if (hidden_type == Elem::kF16) launch_head<Elem::kF16>(h, logits_type, stream);
  else launch_head<Elem::kBF16>(h, logits_type, stream);
}

}  // namespace xgm
