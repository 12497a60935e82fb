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

// How the columns of a chunk of 128 share scales: all of them (groups of 128 or a multiple), halves (64), quarters (32), or
// quarters whose group has to be looked up (other multiples of 32).
enum Sharing : int { kWhole = 0, kHalves = 1, kQuarters = 2, kLookedUp = 3 };
template <int S> constexpr int kParts = S == kWhole ? 1 : S == kHalves ? 2 : 4;

// the scales and zero points of one row of the matrix over one chunk
template <int S, Elem H> struct GroupValues {
  float scale[kParts<S>], zero[kParts<S>];
};
template <int S, Elem H> struct RawGroups {  // as they lie in memory
  uint64_t scales;
  uint32_t zeros;
};
template <int S, Elem H> __device__ __forceinline__ RawGroups<S, H> load_groups(const Head& h, int64_t row, int32_t chunk) {
  RawGroups<S, H> r{0, 0x08080808u};
  const int32_t per_row = h.K / h.group;
  const uint16_t* scales = static_cast<const uint16_t*>(h.scales) + row * per_row;
  const uint8_t* zeros = h.zeros ? h.zeros + row * per_row : nullptr;
  if constexpr (S == kWhole) {
    const int32_t g = chunk / (h.group / 128);
    r.scales = scales[g];
    if (zeros) r.zeros = zeros[g];
  } else {
    const int32_t parts = h.K / (128 / kParts<S>) - chunk * kParts<S>;  // that are left in the row
    if (S != kLookedUp && parts >= kParts<S>) {
      const int32_t g = chunk * kParts<S>;
      if constexpr (S == kHalves) {
        uint32_t s;
        uint16_t z;
        __builtin_memcpy(&s, scales + g, 4);
        r.scales = s;
        if (zeros) {
          __builtin_memcpy(&z, zeros + g, 2);
          r.zeros = z;
        }
      } else {
        __builtin_memcpy(&r.scales, scales + g, 8);
        if (zeros) __builtin_memcpy(&r.zeros, zeros + g, 4);
      }
    } else {
      if (zeros) r.zeros = 0;
      for (int p = 0; p < kParts<S>; ++p) {
        if (p >= parts) break;
        const int32_t g = (chunk * kParts<S> + p) * (128 / kParts<S>) / h.group;
        r.scales |= (uint64_t)scales[g] << (16 * p);
        if (zeros) r.zeros |= (uint32_t)zeros[g] << (8 * p);
      }
    }
  }
  return r;
}
template <int S, Elem H> __device__ __forceinline__ GroupValues<S, H> group_values(RawGroups<S, H> r) {
  GroupValues<S, H> v;
  for (int p = 0; p < kParts<S>; ++p) {
    v.scale[p] = widened<H>((uint16_t)(r.scales >> (16 * p)));
    v.zero[p] = (float)(r.zeros >> (8 * p) & 255u);
  }
  return v;
}

// ---------------------------------------------------------------- few rows in the batch
// Up to 16 NB rows.  A workgroup goes through its share of the matrix 16 rows (a tile) at a time; its eight waves share the columns,
// CW chunks of 128 each, and hold the hidden states of theirs in registers, so that nothing but the matrix moves: a wave
// reads whole stretches of 64 CW bytes of 16 rows, one tile ahead of the products.  The waves' sums meet in LDS, two buffers
// in turn, one barrier a tile; another wave each time adds them up and writes the logits.
// Under masks the workgroup lists the rows of its share that some request allows, and takes 16 of those at a time.
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves;
constexpr int kFewRows = 1024;  // of the matrix at a time (a list of them lies in LDS)

template <int S, int NB> constexpr size_t few_lds(int32_t K) {
  return (size_t)((K + 127) / 128) * kParts<S> * NB * 16 * 4;
}

template <Elem H, int NB, int CW, int S>
__global__ __launch_bounds__(kFewThreads, 2) void q4_few_kernel(Head h, Elem out_type, int32_t tiles_each) {
  extern __shared__ float4v hidden_sums[];  // [chunk][part][16 NB rows]
  __shared__ float4v sums[2][kFewWaves][NB][64];
  __shared__ int32_t list[kFewRows];
  __shared__ uint32_t any[kFewRows / 32];
  __shared__ int32_t n_listed;
  const int32_t tid = (int32_t)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t n = lane & 15, q = lane >> 4;  // row of the tile (and of the batch, on the other side), quarter of the wave
  const int32_t first_b = (int32_t)blockIdx.y * 16 * NB, rows = min(h.B - first_b, 16 * NB);
  const int32_t n_chunks = (h.K + 127) / 128, blocks = h.K / 32;

  // hidden states: product i of a chunk takes columns 32 i + 8 q .. of it (kWhole: 32 q + 8 i, as the codes lie in memory)
  uint4v x[NB][CW][4];
  for (int j = 0; j < CW; ++j) {
    const int32_t chunk = wave * CW + j;
    for (int nb = 0; nb < NB; ++nb) {
      const int32_t b = nb * 16 + n;
      const uint16_t* row = static_cast<const uint16_t*>(h.hidden) + (int64_t)(first_b + b) * h.hidden_stride;
      for (int i = 0; i < 4; ++i) {
        const int32_t k = chunk * 128 + (S == kWhole ? 32 * q + 8 * i : 32 * i + 8 * q);
        uint4v v = {0, 0, 0, 0};
        if (b < rows && k < h.K) v = *reinterpret_cast<const uint4v*>(row + k);
        x[nb][j][i] = in_order(v);
      }
      const uint4v ones = {kOnes<H>, kOnes<H>, kOnes<H>, kOnes<H>};
      for (int p = 0; p < kParts<S>; ++p) {
        float4v s = {0, 0, 0, 0};
        for (int i = p * 4 / kParts<S>; i < (p + 1) * 4 / kParts<S>; ++i) s = mfma<H>(x[nb][j][i], ones, s);
        if (n == 0 && chunk < n_chunks) hidden_sums[((chunk * kParts<S> + p) * NB + nb) * 4 + q] = s;
      }
    }
  }

  const int64_t row0 = (int64_t)blockIdx.x * tiles_each * 16, row1 = min((int64_t)h.V, row0 + (int64_t)tiles_each * 16);
  for (int64_t base = row0; base < row1; base += kFewRows) {
    const int32_t here = (int32_t)min((int64_t)kFewRows, row1 - base);
    int32_t count = here;
    __syncthreads();  // (what the last rows left in LDS has been read)
    if (h.mask) {
      if (tid < kFewRows / 32) any[tid] = 0;
      if (tid == 0) n_listed = 0;
      __syncthreads();
      const int32_t w0 = (int32_t)(base >> 5), shift = (int32_t)(base & 31), words = (here + shift + 31) / 32;  // (shares begin on 16)
      for (int32_t i = tid; i < words * rows; i += kFewThreads) {
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
      for (int32_t r0 = 0; r0 < here; r0 += kFewThreads) {
        const int32_t r = r0 + tid;
        const bool wanted = r < here && (any[r >> 5] >> (r & 31) & 1u);
        if (wanted) {
          int32_t at = __builtin_popcount(any[r >> 5] & ((1u << (r & 31)) - 1u));
          for (int32_t w = 0; w < r >> 5; ++w) at += __builtin_popcount(any[w]);
          list[at] = r;
          atomicAdd(&n_listed, 1);
        } else if (r < here) {
          for (int32_t b = 0; b < rows; ++b) store_logit(h, out_type, (int64_t)(first_b + b) * h.logits_stride + base + r, -__builtin_inff());
        }
      }
      __syncthreads();
      count = n_listed;
    }
    const int32_t tiles = (count + 15) / 16;
    uint4v codes[CW], next_codes[CW];
    RawGroups<S, H> groups[CW], next_groups[CW];
    auto row_of = [&](int32_t t) -> int64_t {
      const int32_t at = min(t * 16 + n, count - 1);
      return base + (h.mask ? list[at] : at);
    };
    auto load = [&](int32_t t, uint4v (&c)[CW], RawGroups<S, H> (&g)[CW]) {
      const int64_t v = row_of(t);
      const uint8_t* row = h.codes + v * (h.K / 2);
      for (int j = 0; j < CW; ++j) {
        const int32_t chunk = wave * CW + j;
        c[j] = uint4v{0, 0, 0, 0};
        if (chunk < n_chunks) {
          if (chunk * 4 + q < blocks) c[j] = *reinterpret_cast<const uint4v*>(row + chunk * 64 + q * 16);
          g[j] = load_groups<S, H>(h, v, chunk);
        }
      }
    };
    if (tiles > 0) load(0, codes, groups);
    for (int32_t t = 0; t < tiles; ++t) {
      if (t + 1 < tiles) load(t + 1, next_codes, next_groups);
      float4v acc[NB];
      for (int nb = 0; nb < NB; ++nb) acc[nb] = float4v{0, 0, 0, 0};
      for (int j = 0; j < CW; ++j) {
        const int32_t chunk = wave * CW + j;
        if (chunk >= n_chunks) break;
        const uint4v c = S == kWhole ? codes[j] : exchanged(codes[j]);
        const GroupValues<S, H> g = group_values<S, H>(groups[j]);
        for (int p = 0; p < kParts<S>; ++p) {
          float4v part[NB];
          for (int nb = 0; nb < NB; ++nb) part[nb] = hidden_sums[((chunk * kParts<S> + p) * NB + nb) * 4 + q] * -(16.0f + g.zero[p]);
          for (int i = p * 4 / kParts<S>; i < (p + 1) * 4 / kParts<S>; ++i) {
            const uint4v w = numbers<H>(c[i]);
            for (int nb = 0; nb < NB; ++nb) part[nb] = mfma<H>(x[nb][j][i], w, part[nb]);
          }
          for (int nb = 0; nb < NB; ++nb) acc[nb] += part[nb] * g.scale[p];
        }
      }
      for (int nb = 0; nb < NB; ++nb) sums[t & 1][wave][nb][lane] = acc[nb];
      __syncthreads();
      if (wave == (t & (kFewWaves - 1))) {
        const bool there = t * 16 + n < count;
        const int64_t v = row_of(t);
        for (int nb = 0; nb < NB; ++nb) {
          float4v y = sums[t & 1][0][nb][lane];
          for (int w = 1; w < kFewWaves; ++w) y += sums[t & 1][w][nb][lane];
          for (int i = 0; i < 4; ++i) {
            const int32_t b = nb * 16 + q * 4 + i;
            if (!there || b >= rows) continue;
            const bool ok = !h.mask || (h.mask[(size_t)(first_b + b) * h.W_mask + (v >> 5)] >> (v & 31) & 1u);
            store_logit(h, out_type, (int64_t)(first_b + b) * h.logits_stride + v, ok ? y[i] : -__builtin_inff());
          }
        }
      }
      for (int j = 0; j < CW; ++j) {
        codes[j] = next_codes[j];
        groups[j] = next_groups[j];
      }
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

constexpr int kFewGroups = 512;  // workgroups of a launch: two a compute unit

template <Elem H, int NB, int CW, int S> void launch_few(const Head& h, Elem out_type, hipStream_t stream) {
  const int32_t tiles = (int32_t)(((int64_t)h.V + 15) / 16), each = (tiles + kFewGroups - 1) / kFewGroups;
  const dim3 grid((tiles + each - 1) / each, (h.B + 16 * NB - 1) / (16 * NB));
  hipLaunchKernelGGL((q4_few_kernel<H, NB, CW, S>), grid, dim3(kFewThreads), (few_lds<S, NB>(h.K)), stream, h, out_type, each);
}
template <Elem H, int NB, int S> void launch_few_columns(const Head& h, Elem out_type, hipStream_t stream) {
  const int32_t chunks = (h.K + 127) / 128;
  if (chunks <= kFewWaves) launch_few<H, NB, 1, S>(h, out_type, stream);
  else if (chunks <= 2 * kFewWaves) launch_few<H, NB, 2, S>(h, out_type, stream);
  else if (NB == 2 || chunks <= 4 * kFewWaves) launch_few<H, NB, 4, S>(h, out_type, stream);
  else if constexpr (NB == 1) launch_few<H, 1, 8, S>(h, out_type, stream);
}
template <Elem H, int NB> void launch_few_groups(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.group % 128 == 0) launch_few_columns<H, NB, kWhole>(h, out_type, stream);
  else if (h.group == 64) launch_few_columns<H, NB, kHalves>(h, out_type, stream);
  else if (h.group == 32) launch_few_columns<H, NB, kQuarters>(h, out_type, stream);
  else launch_few_columns<H, NB, kLookedUp>(h, out_type, stream);
}
template <Elem H> void launch_head(const Head& h, Elem out_type, hipStream_t stream) {
  if (h.K <= 128 * 8 * kFewWaves) {
    if (h.B > 16 && h.K <= 128 * 4 * kFewWaves) launch_few_groups<H, 2>(h, out_type, stream);
    else launch_few_groups<H, 1>(h, out_type, stream);
    return;
  }
  const dim3 grid((h.V + kAnyThreads / 64 - 1) / (kAnyThreads / 64), h.B);
  hipLaunchKernelGGL(q4_any_kernel<H>, grid, dim3(kAnyThreads), 0, stream, h, out_type);
}

}  // namespace

void launch_q4_logits(const Head& h, Elem hidden_type, Elem logits_type, hipStream_t stream) {
  if (hidden_type == Elem::kF16) launch_head<Elem::kF16>(h, logits_type, stream);
  else launch_head<Elem::kBF16>(h, logits_type, stream);
}

}  // namespace xgm
