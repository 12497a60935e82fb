// The output projection with a matrix in 8-bit floating point (e4m3), a scale for each block of 128 x 128, under the masks; hidden
// states brought to 8 bits with a scale for each 128 columns; rows of the matrix, in 4 or 8 bits, as hidden states.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <type_traits>

#include "elements.hpp"
#include "logits.hpp"

namespace xgm {

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Codes go through the matrix instructions as f16, which holds every e4m3 number, or as they are: the instructions for 8 bits take half the time, but of
// each 8 neighbouring products they cut off what lies below 2^-13 of the largest one's power of two (measured: 2^16 + 2^3 is exact, 2^16 + 2^2 is 2^16, unless
// they lie in different eights; between eights nothing is lost down to 2^-23).  The largest loses nothing, the 7 others less than 2^-13 of it each: less
// than 2^-10.2 of the sum of the eights' largest products, and so of the sum of all |products| (up to 2^-11.4 of that was seen in numbers at random, and 2^-10.4
// in those made for it).  That is less than half a step of bf16, 2^-9, of a sum that does not cancel, and more than f16's, 2^-12 to 2^-11: the second way is
// for logits in bf16 of more than 64 rows alone; all others have sums with the 24 bits of a float.
__device__ __forceinline__ f16x8 halves(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
struct Halves {  // 32 numbers of a row
  f16x8 of[4];
  __device__ __forceinline__ Halves(uint4v lo, uint4v hi) : of{halves(lo[0], lo[1]), halves(lo[2], lo[3]), halves(hi[0], hi[1]), halves(hi[2], hi[3])} {}
};
struct Eights {
  int8v of;
  __device__ __forceinline__ Eights(uint4v lo, uint4v hi) : of{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]} {}
};
__device__ __forceinline__ float4v products(const Eights& a, const Eights& b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.of, b.of, float4v{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}
// 16 x 16 sums over 128 columns, of which a lane holds 32 of its row: the same ones on both sides, whichever they are.
__device__ __forceinline__ float4v products(const Halves& a, const Halves& b) {
  float4v c = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.of[i], b.of[i], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ void store_logit(const F8Head& h, Elem type, int64_t at, float y) {
  if (type == Elem::kF32) static_cast<uint32_t*>(h.logits)[at] = narrowed<Elem::kF32>(y);
  else if (type == Elem::kBF16) static_cast<uint16_t*>(h.logits)[at] = narrowed<Elem::kBF16>(y);
  else static_cast<uint16_t*>(h.logits)[at] = narrowed<Elem::kF16>(y);
}
// of four neighbouring tokens, the first of which lies at a multiple of four elements
template <Elem E> __device__ __forceinline__ void store_four(const F8Head& h, int64_t at, const float (&y)[4]) {
  typedef typename Type<E>::bits bits;
  typedef bits bits4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bits4*>(static_cast<bits*>(h.logits) + at) = bits4{narrowed<E>(y[0]), narrowed<E>(y[1]), narrowed<E>(y[2]), narrowed<E>(y[3])};
}
__device__ __forceinline__ void store_logits(const F8Head& h, Elem type, int64_t at, const float (&y)[4]) {
  if (type == Elem::kF32) store_four<Elem::kF32>(h, at, y);
  else if (type == Elem::kBF16) store_four<Elem::kBF16>(h, at, y);
  else store_four<Elem::kF16>(h, at, y);
}
// whether rows of logits begin at such a multiple
bool in_fours(const F8Head& h, Elem type) {
  const uintptr_t size = type == Elem::kF32 ? 4 : 2;
  return reinterpret_cast<uintptr_t>(h.logits) % (4 * size) == 0 && h.logits_stride % 4 == 0;
}

// ---------------------------------------------------------- hidden states to 8 bits
// A power of two as the scale of a block: no value loses bits in the division, so that the only rounding is that to e4m3, and the range that a
// scale in between would gain is less than one of its 17 octaves.
__device__ __forceinline__ uint32_t exponent_of(float most) {  // of the scale, as it stands in a float
  const uint32_t u = __float_as_uint(most);
  const int32_t e = (int32_t)(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u);  // (448 is 1.75 * 2^8)
  return (uint32_t)(min(max(e, -126), 120) + 127);
}
template <Elem E> struct Eight {
  float x[8];
  __device__ __forceinline__ void load(const void* at) {
    typedef typename Type<E>::bits bits;
    uint4v w[sizeof(bits) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(bits) / 2; ++i) w[i] = static_cast<const uint4v*>(at)[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(bits) == 4) x[i] = widened<E>(w[i / 4][i % 4]);
      else x[i] = widened<E>((uint16_t)(w[0][i / 2] >> (16 * (i & 1))));
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  }
  __device__ __forceinline__ float most() const {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));  // (a NaN is no maximum)
    return m;
  }
  // `most`: the block's largest number, which is infinite where one of the eight may be
  __device__ __forceinline__ uint2 codes(float inverse, float most) const {
    float t[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) t[k] = x[k] * inverse;
    if (most > FLT_MAX) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (!(fabsf(t[k]) <= FLT_MAX)) t[k] = __builtin_nanf("");  // (e4m3 has no infinity)
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int word = __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * i], t[4 * i + 1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[4 * i + 2], t[4 * i + 3], word, true);
    }
    return uint2{w[0], w[1]};
  }
};
// the largest of 16 neighbouring lanes: they turn by 8, 4, 2 and 1
template <int kBy> __device__ __forceinline__ float turned_in_16(float m) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0x120 + kBy, 15, 15, true));
}
__device__ __forceinline__ float most_of_16(float m) {
  m = fmaxf(m, turned_in_16<8>(m));
  m = fmaxf(m, turned_in_16<4>(m));
  m = fmaxf(m, turned_in_16<2>(m));
  return fmaxf(m, turned_in_16<1>(m));
}
// 16 lanes to a block.  Columns behind K, up to `width`, become zeros.
template <Elem E>
__global__ __launch_bounds__(256) void f8_quantize_kernel(const void* x, int64_t stride, int32_t B, int32_t K, int32_t width, uint8_t* codes, int64_t codes_stride, float* scales, int64_t scales_row, int64_t scales_block) {
  const int32_t blocks = f8_blocks(K);
  const int64_t block = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 16;
  if (block >= (int64_t)B * blocks) return;  // (16 lanes together)
  const int32_t b = (int32_t)(block / blocks), kb = (int32_t)(block % blocks), k = kb * 128 + ((int32_t)threadIdx.x & 15) * 8;
  Eight<E> v;
  if (k < K) v.load(static_cast<const typename Type<E>::bits*>(x) + b * stride + k);
  else v.clear();
  const float most = most_of_16(v.most());
  const uint32_t e = exponent_of(most);
  if (k < width) *reinterpret_cast<uint2*>(codes + b * codes_stride + k) = v.codes(__uint_as_float((254u - e) << 23), most);
  if (((int32_t)threadIdx.x & 15) == 0) scales[b * scales_row + kb * scales_block] = __uint_as_float(e << 23);
}

// ------------------------------------------------------------------- the projection
// Lists the rows of the matrix among the `here` <= kListed from `base` (a multiple of 16) on that some of the `rows` rows of the batch
// from first_b on allows, as numbers behind base, and masks the logits of the others.  Returns how many.
constexpr int kListed = 1024;
struct List {
  int32_t row[kListed];
  uint32_t any[kListed / 32];
  int32_t n;
};
// (a load whatever the token is: many of them are on their way at once)
__device__ __forceinline__ uint32_t allowed(const F8Head& h, int32_t b, int64_t token) {
  return h.mask[(size_t)b * h.W_mask + (min(token, (int64_t)h.V_mask - 1) >> 5)] >> (token & 31) & (uint32_t)(token < h.V_mask);
}
__device__ int32_t list_rows(const F8Head& h, Elem out_type, int32_t first_b, int32_t rows, int64_t base, int32_t here, bool wide, List& list) {
  int32_t tid = (int32_t)threadIdx.x;
  const int32_t threads = (int32_t)blockDim.x;
  asm volatile("" : "+v"(tid));  // (else places in the list are kept in registers while the matrix goes by)
  __syncthreads();
  if (tid < kListed / 32) list.any[tid] = 0;
  if (tid == 0) list.n = 0;
  __syncthreads();
  const int32_t w0 = (int32_t)(base >> 5), shift = (int32_t)(base & 31), words = (here + shift + 31) / 32;
  for (int32_t i = tid; i < words * rows; i += threads) {
    const int32_t b = i / words, w = i % words;
    uint32_t m = w0 + w < h.W_mask ? h.mask[(size_t)(first_b + b) * h.W_mask + w0 + w] : 0u;
    if (w0 + w == h.V_mask >> 5) m &= (1u << (h.V_mask & 31)) - 1u;  // (what lies behind the masks' vocabulary is not listed)
    if (m && shift) {
      if (w > 0) atomicOr(&list.any[w - 1], m << 16);
      if (w < kListed / 32) atomicOr(&list.any[w], m >> 16);
    } else if (m) {
      atomicOr(&list.any[w], m);
    }
  }
  __syncthreads();
  for (int32_t r = tid; r < here; r += threads) {
    if (list.any[r >> 5] >> (r & 31) & 1u) {
      int32_t place = __builtin_popcount(list.any[r >> 5] & ((1u << (r & 31)) - 1u));
      for (int32_t w = 0; w < r >> 5; ++w) place += __builtin_popcount(list.any[w]);
      list.row[place] = r;
      atomicAdd(&list.n, 1);
    }
  }
  // four rows at a time, of as many rows of the batch as there are threads
  int32_t fours = (here + 3) / 4;
  asm volatile("" : "+v"(fours));  // (as tid above)
  const int32_t abreast = max(threads / fours, 1), b0 = tid / fours;
  if (b0 < abreast)
    for (int32_t i = tid - b0 * fours; i < fours; i += threads) {
      const int32_t r = i * 4;
      const uint32_t any = list.any[r >> 5] >> (r & 31) & 15u;
      if (any == 15u) continue;
      const float none[4] = {-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
#pragma unroll 1
      for (int32_t b = b0; b < rows; b += abreast) {
        const int64_t at = (int64_t)(first_b + b) * h.logits_stride + base + r;
        if (wide && any == 0 && r + 4 <= here) {
          store_logits(h, out_type, at, none);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (!(any >> k & 1u) && r + k < here) store_logit(h, out_type, at + k, none[k]);
        }
      }
    }
  __syncthreads();
  return list.n;
}

// ---------------------------------------------------------------- few rows in the batch
// Shares of 16 NB rows, whose hidden states fit LDS in 8 bits; a workgroup brings them there itself.  A wave takes 16 rows of the matrix (a
// tile) and all columns, so that waves need nothing of each other: it reads the codes a step of kStep blocks of 128 columns at a
// time, the next ones while it multiplies the last.  Under masks the workgroup lists the rows of its share that some request
// allows, and its waves take 16 of those at a time.  Where a workgroup has fewer tiles than waves, several waves take the steps of one
// in turn and their sums meet in LDS.
// One row of 32000 x 2048 takes 15 us, 4.4 TB/s, 16 rows 18: conversions (58 VALU instructions a block and 16 rows beside 4 matrix instructions) and hidden
// states, which every workgroup brings to 8 bits by itself: 11 us of the 20 that 32 rows of 4096 x 4096 take.  Sums go out four at a time: one by one
// 32 rows of 151936 x 1024 took 46 us, and 41.
constexpr int kFewThreads = 1024;
constexpr int kStep = 2;
constexpr uint32_t kMaxLds = 160 * 1024;
struct FewLayout {  // of dynamic LDS, bytes
  uint32_t scales, partial, list, end;
};
// 16 columns of all rows lie side by side, an odd number of them, so that a row's lie in different banks.
__host__ __device__ inline int32_t few_pitch(int32_t rows) { return rows | 1; }
__host__ __device__ inline FewLayout few_layout(int32_t K, int32_t rows) {
  const uint32_t blocks = (uint32_t)f8_blocks(K);
  FewLayout l;
  l.scales = blocks * 128 * (uint32_t)few_pitch(rows);
  l.partial = l.scales + (blocks * (uint32_t)rows * 4 + 15) / 16 * 16;
  l.list = l.partial + kFewThreads * 16;
  l.end = l.list + (uint32_t)sizeof(List);
  return l;
}
enum class States : int { kF8, kBF16, kF16 };

template <States T, int NB, bool kMasked>
__global__ __launch_bounds__(kFewThreads) void f8_few_kernel(F8Head h, Elem out_type, int32_t tiles_each, bool wide) {
  extern __shared__ __align__(16) char lds[];
  const int32_t tid = (int32_t)threadIdx.x, threads = (int32_t)blockDim.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = threads >> 6;
  const int32_t n = lane & 15, q = lane >> 4;
  const int32_t first_b = (int32_t)blockIdx.y * 16 * NB, rows = min(h.B - first_b, 16 * NB), blocks = f8_blocks(h.K);
  const FewLayout at = few_layout(h.K, min(h.B, 16 * NB));
  const int32_t pitch = few_pitch(min(h.B, 16 * NB));
  uint4v* const hidden = reinterpret_cast<uint4v*>(lds);  // [block][16 columns][row]
  float* const hidden_scales = reinterpret_cast<float*>(lds + at.scales);  // [block][row]
  float4v* const partial = reinterpret_cast<float4v*>(lds + at.partial);
  List& list = *reinterpret_cast<List*>(lds + at.list);

  const int32_t n_steps = (blocks + kStep - 1) / kStep;
  const int64_t row0 = (int64_t)blockIdx.x * tiles_each * 16, row1 = min((int64_t)h.V, row0 + (int64_t)tiles_each * 16);
  struct Codes {
    uint4v of[kStep][2];
    float scale[kStep];
  };
  auto load = [&](const uint8_t* row, const float* scales, int32_t step, Codes& c) {
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      const int32_t block = min(step * kStep + j, blocks - 1);
      // (behind the last column some earlier part of the row: hidden states are 0 there)
#pragma unroll
      for (int i = 0; i < 2; ++i) c.of[j][i] = *reinterpret_cast<const uint4v*>(row + min(block * 128 + i * 64 + q * 16, h.K - 16));
      c.scale[j] = scales[block];
    }
  };

  bool brought = false;
  for (int64_t base = row0; base < row1; base += kListed) {
    const int32_t here = (int32_t)min((int64_t)kListed, row1 - base);
    int32_t count = here;
    if constexpr (kMasked) count = list_rows(h, out_type, first_b, rows, base, here, wide, list);
    const int32_t tiles = (count + 15) / 16;
    int32_t sharing = 1;  // waves to a tile, no more than there are where masks leave no tile
    while (sharing * 2 <= n_steps && sharing * 2 * max(tiles, 1) <= waves) sharing *= 2;
    const int32_t sub = wave & (sharing - 1), abreast = waves / sharing, rounds = (tiles + abreast - 1) / abreast;
    auto row_of = [&](int32_t t, int32_t i) -> int32_t {  // the i-th of a tile
      const int32_t k = min(t * 16 + i, count - 1);
      return kMasked ? list.row[k] : k;
    };
    Codes codes, next_codes;
    int32_t t = wave / sharing;
    const uint8_t *row = nullptr, *next_row = nullptr;
    const float *scales = nullptr, *next_scales = nullptr;
    auto point = [&](int32_t tile, const uint8_t*& r, const float*& s) {
      const int64_t v = base + row_of(tile, n);
      r = h.codes + v * h.K;
      s = h.scales + (v >> 7) * blocks;
    };
    if (t < tiles) {
      point(t, row, scales);
      load(row, scales, sub, codes);
      next_row = row;
      next_scales = scales;
    }
    if (!brought) {  // (the first codes are on their way meanwhile)
      brought = true;
      const int32_t units = blocks * rows * 16;  // 8 columns each, 16 neighbouring threads to a block
      constexpr int kAtOnce = 4;                 // of a thread
      const uint32_t inverse = (uint32_t)(0x100000000ull / (uint32_t)rows) + 1u;  // (quotients of less than 2^26 by it are exact)
      auto block_of = [&](int32_t u) { return rows == 1 ? u >> 4 : (int32_t)__umulhi((uint32_t)u >> 4, inverse); };
      int32_t begin = tid;
      asm volatile("" : "+v"(begin));  // (as in list_rows)
      for (int32_t u0 = begin; u0 < units; u0 += threads * kAtOnce) {
        Eight<T == States::kF16 ? Elem::kF16 : Elem::kBF16> x[kAtOnce];
        uint2 w[kAtOnce];
        float scale[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int32_t u = u0 + i * threads, block = block_of(u), b = (u >> 4) - block * rows, k = block * 128 + (u & 15) * 8;
          const bool there = u < units && k < h.K;
          if constexpr (T == States::kF8) {
            w[i] = uint2{0, 0};
            if (there) w[i] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(h.hidden.at) + (first_b + b) * h.hidden.stride + k);
            if (u < units) scale[i] = h.hidden.scales[(int64_t)(first_b + b) * blocks + block];
          } else {
            x[i].clear();
            if (there) x[i].load(static_cast<const uint16_t*>(h.hidden.at) + (first_b + b) * h.hidden.stride + k);
          }
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int32_t u = u0 + i * threads, block = block_of(u), b = (u >> 4) - block * rows, k8 = u & 15;
          if constexpr (T != States::kF8) {
            const float most = most_of_16(x[i].most());
            const uint32_t e = exponent_of(most);
            w[i] = x[i].codes(__uint_as_float((254u - e) << 23), most);
            scale[i] = __uint_as_float(e << 23);
          }
          if (u >= units) break;
          reinterpret_cast<uint2*>(hidden)[((block * 8 + (k8 >> 1)) * pitch + b) * 2 + (k8 & 1)] = w[i];
          if (k8 == 0) hidden_scales[block * rows + b] = scale[i];
        }
      }
      __syncthreads();
    }
    for (int32_t round = 0; round < rounds; ++round) {
      float4v acc[NB];
      for (int nb = 0; nb < NB; ++nb) acc[nb] = float4v{0, 0, 0, 0};
      if (t < tiles) {
        for (int32_t step = sub; step < n_steps; step += sharing) {
          int32_t next_step = step + sharing;
          bool more = true;
          if (next_step >= n_steps) {
            next_step = sub;
            more = t + abreast < tiles;
            if (more) point(t + abreast, next_row, next_scales);
          }
          if (more) load(next_row, next_scales, next_step, next_codes);
#pragma unroll
          for (int j = 0; j < kStep; ++j) {
            const int32_t block = step * kStep + j;
            if (block >= blocks) break;
            const Halves a(codes.of[j][0], codes.of[j][1]);
            // the scale of a row lies with the lane that holds its codes; the sums of rows 4 q .. lie elsewhere
            float4v scale;
            if constexpr (kMasked) {
#pragma unroll
              for (int i = 0; i < 4; ++i) scale[i] = __shfl(codes.scale[j], q * 4 + i);
            } else {
              scale[0] = codes.scale[j];  // (16 rows lie in one block of the matrix)
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const int32_t b = min(nb * 16 + n, rows - 1);
              const Halves x(hidden[(block * 8 + q) * pitch + b], hidden[(block * 8 + 4 + q) * pitch + b]);
              const float4v sum = products(a, x);
              const float state_scale = hidden_scales[block * rows + b];
              if constexpr (kMasked) acc[nb] += sum * (scale * state_scale);
              else acc[nb] += sum * (scale[0] * state_scale);
            }
          }
          codes = next_codes;
        }
      }
      int32_t in = n, i0 = q * 4, me = tid;
      asm volatile("" : "+v"(in), "+v"(i0), "+v"(me));  // (as in list_rows)
      if (sharing > 1) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          partial[me] = acc[nb];
          __syncthreads();
          if (sub == 0) {
#pragma unroll 3
            for (int32_t w = 1; w < sharing; ++w) acc[nb] += partial[me + w * 64];
          }
          __syncthreads();
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (sub != 0 || t >= tiles || nb * 16 + in >= rows) continue;
        const int32_t b = first_b + nb * 16 + in;
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = !kMasked || allowed(h, b, base + row_of(t, i0 + i)) ? acc[nb][i] : -__builtin_inff();
        const int64_t at = b * h.logits_stride + base;
        const int32_t r0 = row_of(t, i0);
        if (wide && t * 16 + i0 + 4 <= count && (!kMasked || (r0 % 4 == 0 && row_of(t, i0 + 3) == r0 + 3))) {
          store_logits(h, out_type, at + r0, y);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (t * 16 + i0 + i < count) store_logit(h, out_type, at + row_of(t, i0 + i), y[i]);
        }
      }
      t += abreast;
      row = next_row;
      scales = next_scales;
    }
  }
}

// --------------------------------------------------------------- many rows in the batch
// Up to 16 MW WM rows and any number of columns, both sides in 8 bits through LDS, a block of 128 columns at a time.  The eight waves of a
// workgroup form WM groups that share the rows of the batch, and in each 8 / WM waves that share the matrix, up to TW tiles each.
// What a block needs goes from memory to LDS without passing a register, into a ring of kStages buffers: while a block is multiplied the
// next kStages - 1 are on their way; one barrier a block.  16 bytes of a row lie in LDS at their place in the row with the row's last three bits
// exchanged into it: eight rows of one place, as a wave reads them, lie in different banks.
// One row of 128256 x 4096 takes 95 us, 5.5 TB/s, 32 rows 101: the bytes of the matrix.  (Of 32 rows and less a block without them takes 0.5 to 0.6 us, for
// conversions and the barrier: four buffers instead of three take 1 us more a call.)
// 128 rows of 151936 x 4096 take 153 us, 4.3 TB/s: memory, of which two blocks are on their way to each compute unit; through registers, a block ahead, it
// took 264.  1024 rows of 128256 x 4096 take 624 us, 1.72 PFLOP/s (605 to 631 from card to card, and up to 770 for the first passes, until clocks have settled; pairs of
// figures below are of one card each); without its loads 456, at which clock and power hold the matrix instructions
// (8192 x 8192 x 8192 in a library reach 2.67 PFLOP/s, and this product without scales of blocks 544 us).
// With f16 instructions (logits in f16 and in 32 bits) 128 rows take 216 and 219 us, 1024 rows 1052 and 1070, of which the instructions alone are 889.
constexpr int kManyThreads = 512, kManyWaves = kManyThreads / 64;
template <int MW, int WM, int TW> struct ManyShape {
  static constexpr int kRows = 16 * MW * WM, kWide = kManyWaves / WM, kPass = kWide * TW, kMatrix = 16 * kPass;
  static constexpr int kBrought = kRows < 64 ? 64 : kRows;  // (fewer rows come with copies of the last one)
  static constexpr int kStateLoads = kBrought / 8 / kManyWaves, kCodeLoads = kMatrix / 8 / kManyWaves;  // of a wave, 64 x 16 bytes each
  static constexpr int kStages = kBrought + kMatrix <= 384 ? 3 : 2;
  static_assert(kBrought % 64 == 0 && kCodeLoads > 0 && kRows + kMatrix <= kManyThreads, "equal parts for all waves, and a scale a thread");
};
template <int MW, int WM, int TW> struct Stage {
  typedef ManyShape<MW, WM, TW> Shape;
  uint4v states[Shape::kBrought * 8];
  uint4v codes[Shape::kMatrix * 8];
  float scales[kManyThreads];  // of the rows of the batch, then of those of the matrix
};
struct StateScales {  // where the scale of a row and a block lies
  int64_t row, block;
};
__device__ const uint4v kZeros = {0, 0, 0, 0};
// 16 or 4 bytes a lane; `to` is the place of the wave's first lane.  (Written out because the compiler would let every read of LDS wait for all
// of these; they have no result in a register, and who reads what they bring waits for them behind barrier_behind_loads.  Nor does it see to wait
// states in such a text: a load to LDS comes one of them behind the instruction that sets its m0, and one with a scalar address five behind a vector
// instruction that writes it, as those do that bring spilled ones back.)
__device__ __forceinline__ uint32_t lds_place(const void* to) {
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)to);
}
__device__ __forceinline__ void bring16(const void* from, const void* to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(lds_place(to)), "v"(from) : "memory");
}
// the same from an address that all lanes share and an offset each
__device__ __forceinline__ void bring16(const void* from, uint32_t offset, const void* to) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(lds_place(to)), "v"(offset), "s"(from) : "memory");
}
__device__ __forceinline__ void bring4(const void* from, const void* to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" : : "{m0}"(lds_place(to)), "v"(from) : "memory");
}
// A barrier for which a wave waits until no more than n of its loads are on their way, and none of its reads of LDS.
template <int n> __device__ __forceinline__ void barrier_behind_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 7 << 4);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
struct Nothing {};
template <int MW, int WM, int TW, bool kMasked, class Operand>
__global__ __launch_bounds__(kManyThreads, 2) void f8_many_kernel(F8Head h, StateScales strides, Elem out_type, int32_t batch_tiles, int32_t shares, int32_t tiles_each, bool wide) {
  typedef ManyShape<MW, WM, TW> Shape;
  constexpr int kLoads = Shape::kStateLoads + Shape::kCodeLoads + 1;
  typedef Stage<MW, WM, TW> Buffer;
  __shared__ Buffer stage0, stage1;  // (of their own names: a read of one does not wait for loads to another)
  __shared__ std::conditional_t<Shape::kStages == 3, Buffer, Nothing> stage2;
  __shared__ std::conditional_t<kMasked, List, Nothing> list;
  const int32_t tid = (int32_t)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t n = lane & 15, q = lane >> 4, wm = wave % WM, wn = wave / WM;
  // workgroups that share a part of the matrix follow each other on one XCD
  int32_t share, batch_tile;
  {
    const int32_t id = (int32_t)blockIdx.x, whole = shares / 8 * 8 * batch_tiles;
    if (id < whole) {
      share = id / 8 / batch_tiles * 8 + id % 8;
      batch_tile = id / 8 % batch_tiles;
    } else {
      share = shares / 8 * 8 + (id - whole) / batch_tiles;
      batch_tile = (id - whole) % batch_tiles;
    }
  }
  const int32_t first_b = batch_tile * Shape::kRows, rows = min(h.B - first_b, Shape::kRows), blocks = f8_blocks(h.K);

  // Rows of the matrix and of the hidden states lie a power of two apart as a rule, so that the same columns of all of them are on few
  // channels of the L2: the workgroups of an XCD begin with different blocks.
  const int32_t begin = share / 8 % blocks;
  auto turned = [&](int32_t block) { return block + begin < blocks ? block + begin : block + begin - blocks; };
  const uint8_t* const all_states = static_cast<const uint8_t*>(h.hidden.at) + first_b * h.hidden.stride;
  const uint32_t in_row = (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);  // what a lane brings of 8 rows
  // Addresses of all that a wave brings lie in registers, where there are enough.  kLean: the sums need them; 8 rows come from one address and an
  // offset that stays the same, and those past the last one, or columns around the last one, from an address each that is computed anew every time
  // (which the asm below sees to).
  constexpr bool kLean = Shape::kStages == 2;
  static_assert(!kLean || !kMasked, "rows of a list do not follow each other");
  const bool near = h.hidden.stride < 1 << 28;  // (offsets within 8 rows fit 32 bits)
  [[maybe_unused]] const uint32_t code_offset = (uint32_t)(lane >> 3) * (uint32_t)h.K + in_row, state_offset = (uint32_t)(lane >> 3) * (uint32_t)h.hidden.stride + in_row;
  [[maybe_unused]] const uint8_t* state_at[Shape::kStateLoads];
  if constexpr (!kLean) {
#pragma unroll
    for (int u = 0; u < Shape::kStateLoads; ++u)
      state_at[u] = all_states + min((wave * Shape::kStateLoads + u) * 8 + (lane >> 3), rows - 1) * h.hidden.stride + in_row;
  }
  const int64_t row0 = (int64_t)share * tiles_each * 16, row1 = min((int64_t)h.V, row0 + (int64_t)tiles_each * 16);
  constexpr int64_t kTogether = kMasked ? kListed : 32768;  // (rows of the matrix, whose codes begin within 32 bits of each other)
  for (int64_t base = row0; base < row1; base += kTogether) {
    const int32_t here = (int32_t)min(kTogether, row1 - base);
    int32_t count = here;
    if constexpr (kMasked) count = list_rows(h, out_type, first_b, rows, base, here, wide, list);
    const int32_t tiles = (count + 15) / 16;
    auto row_of = [&](int32_t i) -> int32_t {
      const int32_t k = min(i, count - 1);
      if constexpr (kMasked) return list.row[k];
      else return k;
    };
    const uint8_t* const base_codes = h.codes + base * h.K;
    const int32_t passes = (tiles + Shape::kPass - 1) / Shape::kPass, even = passes ? (tiles + passes - 1) / passes : 0;
    if (tiles == 0) continue;
    // What a wave brings of a pass, from_row .. last_row of the rows here, 8 rows at a time.
    int32_t from_row = 0, last_row = 0;
    [[maybe_unused]] uint32_t code_at[Shape::kCodeLoads];
    const float* scale_at = nullptr;
    auto point = [&](int32_t pass) {
      from_row = pass * 16;
      last_row = min(from_row + even * 16, count) - 1;
      if constexpr (!kLean) {
#pragma unroll
        for (int u = 0; u < Shape::kCodeLoads; ++u)
          code_at[u] = (uint32_t)row_of(min(from_row + (wave * Shape::kCodeLoads + u) * 8 + (lane >> 3), last_row)) * (uint32_t)h.K;
      }
      if (tid < Shape::kRows) scale_at = h.hidden.scales + (first_b + min(tid, rows - 1)) * strides.row;
      else scale_at = h.scales + ((base + row_of(min(from_row + tid - Shape::kRows, last_row))) >> 7) * blocks;
    };
    // the i-th of a wave's kLoads loads of a block
    auto load = [&](int i, int32_t turn, Buffer& to) {
      const int32_t block = turned(turn);
      const bool whole = (block + 1) * 128 <= h.K;
      int32_t thread = tid;
      if (i < Shape::kCodeLoads) {  // (behind the last column some earlier part of the row: hidden states are 0 there)
        const int32_t first = (wave * Shape::kCodeLoads + i) * 8;
        uint4v* const place = &to.codes[first * 8];
        if constexpr (!kLean) {
          bring16(base_codes + (code_at[i] + (uint32_t)min(block * 128 + (int32_t)in_row, h.K - 16)), place);
        } else if (whole && from_row + first + 7 <= last_row) {
          bring16(base_codes + ((int64_t)(from_row + first) * h.K + block * 128), code_offset, place);
        } else {
          asm volatile("" : "+v"(thread));
          const int32_t in = thread >> 3 & 7, k = block * 128 + ((thread & 7) ^ in) * 16;
          bring16(base_codes + ((uint32_t)min(from_row + first + in, last_row) * (uint32_t)h.K + (uint32_t)min(k, h.K - 16)), place);
        }
      } else if (i < Shape::kCodeLoads + Shape::kStateLoads) {
        const int u = i - Shape::kCodeLoads;
        const int32_t first = (wave * Shape::kStateLoads + u) * 8;
        uint4v* const place = &to.states[first * 8];
        const auto or_zeros = [&](const uint8_t* at, int32_t k) {
          return reinterpret_cast<const void*>(k < h.K ? reinterpret_cast<uintptr_t>(at) : reinterpret_cast<uintptr_t>(&kZeros));
        };
        if constexpr (!kLean) {
          bring16(or_zeros(state_at[u] + block * 128, block * 128 + (int32_t)in_row), place);
        } else if (whole && near && first + 8 <= rows) {
          bring16(all_states + (first * h.hidden.stride + block * 128), state_offset, place);
        } else {
          asm volatile("" : "+v"(thread));
          const int32_t in = thread >> 3 & 7, k = block * 128 + ((thread & 7) ^ in) * 16;
          bring16(or_zeros(all_states + min(first + in, rows - 1) * h.hidden.stride + k, k), place);
        }
      } else {
        asm volatile("" : "+v"(thread));
        bring4(scale_at + block * (thread < Shape::kRows ? (int32_t)strides.block : 1), &to.scales[wave * 64]);
      }
    };
    // all of a block, or its codes, or the rest
    auto load_codes = [&](int32_t turn, Buffer& to) {
#pragma unroll
      for (int i = 0; i < Shape::kCodeLoads; ++i) load(i, turn, to);
    };
    auto load_others = [&](int32_t turn, Buffer& to) {
#pragma unroll
      for (int i = Shape::kCodeLoads; i < kLoads; ++i) load(i, turn, to);
    };
    auto begin_pass = [&](int32_t pass) {
      point(pass);
      load_others(0, stage0);
      load_codes(0, stage0);
      if (blocks > 1) {
        if (Shape::kStages == 3) load_others(1, stage1);
        load_codes(1, stage1);
      }
    };
    barrier_behind_loads<0>();  // (what was there before has been read)
    begin_pass(0);
    for (int32_t pass = 0; pass < tiles; pass += even) {
      const int32_t pass_tiles = min(even, tiles - pass), each = (pass_tiles + Shape::kWide - 1) / Shape::kWide;
      const int32_t first = wn * each, mine = max(0, min(each, pass_tiles - first));
      float4v acc[TW][MW];
#pragma unroll
      for (int c = 0; c < TW; ++c)
        for (int m = 0; m < MW; ++m) acc[c][m] = float4v{0, 0, 0, 0};
      // Multiplies a block.  The loads of another one are seen to when the first reads of LDS are on their way: between the products, where they
      // keep nobody waiting, they come too late for the next barrier (1024 rows of 128256 x 4096: 642 us, and 676).
      auto multiply = [&](auto tiles_of_wave, const Buffer& s, auto&& load_other) {
        constexpr int N = decltype(tiles_of_wave)::value;
        // (registers: scales of rows are read where they are used, and a tile is scaled right behind the next: 85 rows of 50102 x 2048, most rows listed,
        // 62 us and not 56, but 267 rows of 14681 x 2048 with few 29 and not 48, as waves without a tile have nothing to multiply)
        constexpr bool kTight = kMasked && sizeof(Operand) > 32 && N * MW > 8;
        const int place = q ^ (n & 7);
        auto operand = [&](const uint4v* row) { return Operand(row[place], row[place ^ 4]); };
        const uint4v* const my_codes = &s.codes[(first * 16 + n) * 8];
        const uint4v* const my_states = &s.states[(wm * MW * 16 + n) * 8];
        uint4v lo = my_states[place], hi = my_states[place ^ 4];
        float state_scale = s.scales[wm * MW * 16 + n];
        float4v scale[N];
#pragma unroll
        for (int c = 0; c < N; ++c) {
          if constexpr (kMasked && !kTight) scale[c] = *reinterpret_cast<const float4v*>(&s.scales[Shape::kRows + (first + c) * 16 + q * 4]);
          else if constexpr (!kMasked) scale[c][0] = s.scales[Shape::kRows + (first + c) * 16];
        }
        const Operand a[4] = {operand(my_codes), operand(my_codes + (N > 1) * 128), operand(my_codes + (N > 2) * 256), operand(my_codes + (N > 3) * 384)};
        // the sums of a tile are scaled while the next ones' products are made
        // (1024 rows of 128256 x 4096: one behind 643 us, two 639, four 617)
        constexpr int kBehind = kMasked && sizeof(Operand) > 32 ? N == 1 || kTight ? 1 : 2 : 4;  // (registers)
        constexpr int kRoundsBehind = (kBehind + N - 1) / N;
        float4v sum[kBehind + 1];
        float scale_of[kRoundsBehind + 1];
        load_other();
#pragma unroll
        for (int m = 0; m < MW + kRoundsBehind; ++m) {
          const Operand x(lo, hi);
          scale_of[m % (kRoundsBehind + 1)] = state_scale;
          if (m + 1 < MW) {
            lo = my_states[(m + 1) * 128 + place];
            hi = my_states[(m + 1) * 128 + (place ^ 4)];
            state_scale = s.scales[(wm * MW + m + 1) * 16 + n];
          }
#pragma unroll
          for (int c = 0; c < N; ++c) {
            const int t = m * N + c, was = t - kBehind;
            if (m < MW) sum[t % (kBehind + 1)] = products(a[c], x);
            if (was >= 0 && was < MW * N) {
              float4v& to = acc[was % N][was / N];
              const float state = scale_of[was / N % (kRoundsBehind + 1)];
              if constexpr (kTight) {
                int at = q * 4;
                asm volatile("" : "+v"(at));
                to += sum[was % (kBehind + 1)] * (*reinterpret_cast<const float4v*>(&s.scales[Shape::kRows + (first + was % N) * 16 + at]) * state);
              } else if constexpr (kMasked) to += sum[was % (kBehind + 1)] * (scale[was % N] * state);
              else to += sum[was % (kBehind + 1)] * (scale[was % N][0] * state);
              asm volatile("" : "+v"(to));  // (here, and not when all products are made: they would not fit the registers)
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      // A block is there when all waves have waited for their parts of it.  Of three buffers the one of the block before it is free then.  Of two,
      // codes are in registers before the first product: behind a barrier more, those of the block after the next come to the same place, and are
      // on their way for two blocks, as memory asks; hidden states, which come from the L2, for one (1024 rows of 128256 x 4096: 611 us, and 627
      // where all of the next block comes at once).
      auto turn = [&](int32_t block, Buffer& now, Buffer& other) {
        if constexpr (Shape::kStages == 3) {
          if (block + 1 < blocks) barrier_behind_loads<kLoads>();
          else barrier_behind_loads<0>();
          auto load_next = [&] {
            if (block + 2 >= blocks) return;
            load_others(block + 2, other);
            load_codes(block + 2, other);
          };
          // Few tiles: waves without one have nothing to multiply (128 rows of 10000 x 4096 take 26.5 us, and 37 where all of them multiply TW).
          if (mine > 1) multiply(std::integral_constant<int, TW>(), now, load_next);
          else if (mine == 1) multiply(std::integral_constant<int, 1>(), now, load_next);
          else load_next();
        } else {
          if (block + 1 < blocks) barrier_behind_loads<Shape::kCodeLoads>();
          else barrier_behind_loads<0>();
          multiply(std::integral_constant<int, TW>(), now, [&] {
            barrier_behind_loads<63>();  // (for reads of LDS alone)
            if (block + 1 < blocks) load_others(block + 1, other);
            if (block + 2 < blocks) load_codes(block + 2, now);
          });
        }
      };
#pragma unroll 1
      for (int32_t block = 0; block < blocks; block += Shape::kStages) {
        if constexpr (Shape::kStages == 3) {
          turn(block, stage0, stage2);
          if (block + 1 < blocks) turn(block + 1, stage1, stage0);
          if (block + 2 < blocks) turn(block + 2, stage2, stage1);
        } else {
          turn(block, stage0, stage1);
          if (block + 1 < blocks) turn(block + 1, stage1, stage0);
        }
      }
      if (pass + even < tiles) {  // the next pass's first blocks come while this one's logits go
        barrier_behind_loads<0>();
        begin_pass(pass + even);
      }
      auto store = [&](auto type) {
        constexpr Elem O = decltype(type)::value;
        typedef typename Type<O>::bits bits;
        int32_t in0 = wm * MW * 16 + n;
        asm volatile("" : "+v"(in0));  // (else the addresses of all rows are computed ahead of the loops and fill the registers)
#pragma unroll
        for (int c = 0; c < TW; ++c) {
          if (c >= mine) continue;
          const int32_t i0 = (pass + first + c) * 16 + q * 4;
          int32_t r[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) r[i] = row_of(i0 + i);
          [[maybe_unused]] uint32_t open = 0;  // bit 4 m + i
          if constexpr (kMasked) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int m = 0; m < MW; ++m) open |= allowed(h, first_b + min(in0 + m * 16, rows - 1), base + r[i]) << (4 * m + i);
          }
          const bool in_one = wide && i0 + 4 <= count && (!kMasked || (r[0] % 4 == 0 && r[3] == r[0] + 3));
#pragma unroll
          for (int m = 0; m < MW; ++m) {
            const int32_t in = in0 + m * 16, b = first_b + in;
            if (in >= rows) continue;
            const int64_t at = b * h.logits_stride + base;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = !kMasked || (open >> (4 * m + i) & 1u) ? acc[c][m][i] : -__builtin_inff();
            if (in_one) {
              store_four<O>(h, at + r[0], y);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (i0 + i < count) static_cast<bits*>(h.logits)[at + r[i]] = narrowed<O>(y[i]);
            }
          }
        }
      };
      if (std::is_same_v<Operand, Eights> || out_type == Elem::kBF16) store(std::integral_constant<Elem, Elem::kBF16>());
      else if constexpr (!std::is_same_v<Operand, Eights>) {
        if (out_type == Elem::kF32) store(std::integral_constant<Elem, Elem::kF32>());
        else store(std::integral_constant<Elem, Elem::kF16>());
      }
    }
  }
}

// scales of hidden states, [row][block] to [block][row]
__global__ __launch_bounds__(256) void f8_turn_scales_kernel(const float* from, int32_t B, int32_t blocks, float* to) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (int64_t)B * blocks) to[i] = from[i % B * blocks + i / B];
}

constexpr int kComputeUnits = 256;

int64_t padded(int32_t K) { return (int64_t)f8_blocks(K) * 128; }

// ------------------------------------------------------ rows of the matrix as hidden states
// A thread takes 16 columns at a time, of 32 bits four of each 16 bytes side by side with its neighbours' (16384 rows of 4096 columns in 32 bits: 62 us, and 90
// as 64 bytes a thread; 16 bits are no faster so, 45 us and 44), 2^shift threads a row.  value * (scale * factor) in 64 bits, where both products are exact, rounded once.
// 16384 rows of 4096 columns (8 bits to bf16) take 44 us, 4.4 TB/s: memory, as products in 32 bits would; 128 rows 3.4 us and a launch.
constexpr int kEmbedThreads = 256;
constexpr int32_t kMostEmbedGroups = 1 << 23;  // workgroups of a launch, which has to have less than 2^32 threads
template <Elem S, Elem O, bool Q4> __device__ __forceinline__ void embed_row(const Embed& e, int32_t i, int32_t t, int shift, bool wide) {
  typedef typename Type<O>::bits bits;
  const int32_t id = e.ids[i];
  const bool there = id >= 0 && id < e.V;
  const int64_t v = there ? id : 0;
  const double factor = (double)e.factor;
  bits* const out = static_cast<bits*>(e.out) + (int64_t)i * e.out_stride;
  constexpr int kUnit = sizeof(bits) == 4 ? 4 : 16, kUnits = 16 / kUnit;  // columns
  typedef std::conditional_t<Q4, std::conditional_t<kUnit == 4, uint16_t, uint2>, std::conditional_t<kUnit == 4, uint32_t, uint4v>> Codes;
  for (int32_t k0 = 0; k0 < e.K; k0 += 16 << shift) {
    Codes w[kUnits];
    double scale[kUnits];
    [[maybe_unused]] int zero[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int32_t k = min(k0 + ((u << shift) + t) * kUnit, e.K - kUnit);
      if constexpr (Q4) {
        const int64_t g = v * (e.K / e.group) + k / e.group;  // (a group is a multiple of 32)
        w[u] = *reinterpret_cast<const Codes*>(e.codes + (v * e.K + k) / 2);
        zero[u] = e.zeros ? e.zeros[g] : 8;
        scale[u] = (double)widened<S>(static_cast<const typename Type<S>::bits*>(e.scales)[g]);
      } else {
        w[u] = *reinterpret_cast<const Codes*>(e.codes + v * e.K + k);
        scale[u] = (double)static_cast<const float*>(e.scales)[(v >> 7) * f8_blocks(e.K) + (k >> 7)];
      }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int32_t k = k0 + ((u << shift) + t) * kUnit;
      if (k >= e.K) break;
      const double by = scale[u] * factor;
      float x[kUnit];
      if constexpr (Q4) {
#pragma unroll
        for (int j = 0; j < kUnit; ++j) {
          uint32_t word;
          if constexpr (kUnit == 4) word = w[u];
          else word = j < 8 ? w[u].x : w[u].y;
          x[j] = (float)((int)(word >> (4 * (j & 7)) & 15u) - zero[u]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kUnit / 4; ++j) {
          int word;
          if constexpr (kUnit == 4) word = (int)w[u];
          else word = (int)w[u][j];
          x[4 * j] = __builtin_amdgcn_cvt_f32_fp8(word, 0);
          x[4 * j + 1] = __builtin_amdgcn_cvt_f32_fp8(word, 1);
          x[4 * j + 2] = __builtin_amdgcn_cvt_f32_fp8(word, 2);
          x[4 * j + 3] = __builtin_amdgcn_cvt_f32_fp8(word, 3);
        }
      }
      constexpr int kWords = kUnit * (int)sizeof(bits) / 4;
      uint32_t y[kWords] = {};  // as it goes to memory
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const uint32_t one = there ? (uint32_t)narrowed<O>((double)x[j] * by) : 0u;
        if constexpr (sizeof(bits) == 4) y[j] = one;
        else y[j / 2] |= one << (16 * (j & 1));
      }
      if (wide) {
#pragma unroll
        for (int j = 0; j < kWords; j += 4) *reinterpret_cast<uint4v*>(out + k + j * 4 / (int)sizeof(bits)) = uint4v{y[j], y[j + 1], y[j + 2], y[j + 3]};
      } else {
#pragma unroll
        for (int j = 0; j < kUnit; ++j) out[k + j] = (bits)(sizeof(bits) == 4 ? y[j] : y[j / 2] >> (16 * (j & 1)));
      }
    }
  }
}
// A row's threads take another one where there are more rows than a launch has room for.
template <Elem S, Elem O, bool Q4> __global__ __launch_bounds__(kEmbedThreads) void embed_kernel(Embed e, int shift, bool wide) {
  const int32_t t = (int32_t)threadIdx.x & ((1 << shift) - 1), rows = kEmbedThreads >> shift;
  for (uint32_t i = blockIdx.x * (uint32_t)rows + (threadIdx.x >> shift); i < (uint32_t)e.n; i += (uint32_t)kMostEmbedGroups * (uint32_t)rows)
    embed_row<S, O, Q4>(e, (int32_t)i, t, shift, wide);
}
template <Elem S, bool Q4> hipError_t launch_embed(const Embed& e, Elem out_type, hipStream_t stream) {
  int shift = 0;
  while (shift < 8 && (16 << shift) < e.K) ++shift;
  const int32_t rows = kEmbedThreads >> shift;
  const int size = out_type == Elem::kF32 ? 4 : 2;
  const bool wide = reinterpret_cast<uintptr_t>(e.out) % 16 == 0 && e.out_stride * size % 16 == 0;
  const int32_t groups = (e.n + rows - 1) / rows;
  const dim3 grid((uint32_t)(groups < kMostEmbedGroups ? groups : kMostEmbedGroups));
  if (out_type == Elem::kF32) hipLaunchKernelGGL((embed_kernel<S, Elem::kF32, Q4>), grid, dim3(kEmbedThreads), 0, stream, e, shift, wide);
  else if (out_type == Elem::kBF16) hipLaunchKernelGGL((embed_kernel<S, Elem::kBF16, Q4>), grid, dim3(kEmbedThreads), 0, stream, e, shift, wide);
  else hipLaunchKernelGGL((embed_kernel<S, Elem::kF16, Q4>), grid, dim3(kEmbedThreads), 0, stream, e, shift, wide);
  return hipGetLastError();
}

struct Quantized {
  uint8_t* codes;
  int64_t stride;
  int32_t width;  // columns of it
  float* scales;
  StateScales strides;
};
template <Elem E> hipError_t quantize(const void* x, int32_t B, int32_t K, int64_t stride, const Quantized& to, hipStream_t stream) {
  const int64_t groups = ((int64_t)B * f8_blocks(K) + 15) / 16;
  hipLaunchKernelGGL(f8_quantize_kernel<E>, dim3((uint32_t)groups), dim3(256), 0, stream, x, stride, B, K, to.width, to.codes, to.stride, to.scales, to.strides.row,
                     to.strides.block);
  return hipGetLastError();
}
hipError_t quantize_any(const void* x, Elem type, int32_t B, int32_t K, int64_t stride, const Quantized& to, hipStream_t stream) {
  if (type == Elem::kF32) return quantize<Elem::kF32>(x, B, K, stride, to, stream);
  if (type == Elem::kBF16) return quantize<Elem::kBF16>(x, B, K, stride, to, stream);
  return quantize<Elem::kF16>(x, B, K, stride, to, stream);
}

// tiles of a workgroup where the batch goes in shares of `rows`: so many that all workgroups run at once
int32_t few_tiles(const F8Head& h, int32_t rows) {
  const int32_t tiles = (int32_t)(((int64_t)h.V + 15) / 16), shares = (h.B + rows - 1) / rows, most = shares < kComputeUnits ? kComputeUnits / shares : 1;
  return (tiles + most - 1) / most;
}
template <States T, int NB, bool kMasked> hipError_t launch_few(const F8Head& h, Elem out_type, hipStream_t stream) {
  static LdsRoom room;
  if (const hipError_t e = room(reinterpret_cast<const void*>(&f8_few_kernel<T, NB, kMasked>), kMaxLds); e != hipSuccess) return e;
  const int32_t tiles = (int32_t)(((int64_t)h.V + 15) / 16), each = few_tiles(h, 16 * NB), steps = (f8_blocks(h.K) + kStep - 1) / kStep;
  int32_t threads = 64;  // waves for its tiles, or for the steps of the few that masks leave
  while (threads < kFewThreads && threads < 64 * (kMasked && steps > each ? steps : each * (each < 16 ? steps : 1))) threads *= 2;
  const dim3 grid((tiles + each - 1) / each, (h.B + 16 * NB - 1) / (16 * NB));
  hipLaunchKernelGGL((f8_few_kernel<T, NB, kMasked>), grid, dim3(threads), few_layout(h.K, h.B < 16 * NB ? h.B : 16 * NB).end, stream, h, out_type, each, in_fours(h, out_type));
  return hipGetLastError();
}
template <States T, int NB> hipError_t launch_few_masked(const F8Head& h, Elem out_type, hipStream_t stream) {
  return h.mask ? launch_few<T, NB, true>(h, out_type, stream) : launch_few<T, NB, false>(h, out_type, stream);
}
template <int NB> hipError_t launch_few_states(const F8Head& h, Elem hidden_type, Elem out_type, hipStream_t stream) {
  if (h.hidden.scales) return launch_few_masked<States::kF8, NB>(h, out_type, stream);
  if (hidden_type == Elem::kF16) return launch_few_masked<States::kF16, NB>(h, out_type, stream);
  return launch_few_masked<States::kBF16, NB>(h, out_type, stream);
}
bool few_fits(const F8Head& h, int32_t rows) { return few_layout(h.K, rows).end <= kMaxLds; }

template <int MW, int WM, int TW, bool kMasked, class Operand> hipError_t launch_many(const F8Head& h, const StateScales& strides, Elem out_type, hipStream_t stream) {
  typedef ManyShape<MW, WM, TW> Shape;
  const int32_t tiles = (int32_t)(((int64_t)h.V + 15) / 16), batch_tiles = (h.B + Shape::kRows - 1) / Shape::kRows;
  const int32_t most = batch_tiles < kComputeUnits ? kComputeUnits / batch_tiles : 1, each = (tiles + most - 1) / most, shares = (tiles + each - 1) / each;
  hipLaunchKernelGGL((f8_many_kernel<MW, WM, TW, kMasked, Operand>), dim3((uint32_t)(shares * batch_tiles)), dim3(kManyThreads), 0, stream, h, strides, out_type,
                     batch_tiles, shares, each, in_fours(h, out_type));
  return hipGetLastError();
}
template <int MW, int WM, int TW, class Operand> hipError_t launch_many_masked(const F8Head& h, const StateScales& strides, Elem out_type, hipStream_t stream) {
  return h.mask ? launch_many<MW, WM, TW, true, Operand>(h, strides, out_type, stream) : launch_many<MW, WM, TW, false, Operand>(h, strides, out_type, stream);
}

}  // namespace

size_t f8_work_bytes(int32_t B, int32_t K) { return (size_t)B * (size_t)(padded(K) + f8_blocks(K) * 4); }

hipError_t launch_f8_quantize(const void* x, Elem type, int32_t B, int32_t K, int64_t stride, uint8_t* codes, int64_t codes_stride, float* scales, hipStream_t stream) {
  return quantize_any(x, type, B, K, stride, Quantized{codes, codes_stride, K, scales, StateScales{f8_blocks(K), 1}}, stream);
}

namespace {
// Which kernel takes a batch, by what a call takes them in us: a workgroup of few rows a start, its hidden states and its tiles (of one to four, loads come
// back meanwhile); one of many rows (which waits for a launch that brings hidden states to 8 bits) a time for each block of columns of each of its passes,
// which is that of a barrier and of loads that come back, less where no wave has more than a tile, or where that is more the bytes of its tiles.
// For bf16, few and many, us:
//   4096 x 4096: 1 row 7 and 19, 16 rows 13 and 19, 32 rows 20 and 20, 64 rows 20.5 and 24.5, 128 rows 24.4 and 21.7
//   10000 x 4096: 16 rows 16.3 and 19.1, 32 rows 23.1 and 21.0, 64 rows 29.5 and 26.4
//   50001 x 2080: 1 row 25.5 and 26.3, 16 rows 29.5 and 27.6, 32 rows 36.5 and 31.6
//   128256 x 4096: 1 row 103 and 95, 16 rows 115 and 96, 32 rows 128 and 101; 151936 x 1024: 31 and 33, 36 and 37, 41 and 41
// of many 500 rows of 2048 x 4096 24 in tiles of 128 rows and 64 in those of 256, 1024 of 128256 x 4096 700 and 628, 384 of them 270 and 349.
// Logits in 32 bits or f16, 128 rows of 4096 x 4096: few 24.3, many 25.7, of 10000 x 4096 40.8 and 36.9.
// What masks leave is not known on the host: the choice is that for whole matrices.  bf16, few and many, us, with 5 rows of 13 open / with 400 tokens a row:
//   10000 x 4096: 1 row 12.9 and 22.6 / 8.1 and 20.4, 16 rows 18.1 and 22.8 / 15.1 and 22.2, 32 rows 26.3 and 22.3 / 25.9 and 22.9, 64 rows 33.2 and 28.8 / 33.6 and 30.1,
//     128 rows 44.5 and 30.5 / 44.5 and 32.7
//   50001 x 2080: 1 row 23.1 and 21.7 / 7.8 and 14.5, 16 rows 26.1 and 23.2 / 12.0 and 15.5, 32 rows 33.6 and 26.9 / 20.2 and 18.5, 64 rows 52.2 and 38.0 / 28.8 and 31.2,
//     128 rows 72.5 and 46.5 / 38.3 and 47.4
//   128256 x 4096: 1 row 96.6 and 113 / 8.8 and 20.5, 16 rows 110 and 122 / 19.5 and 25.8, 32 rows 122 and 126 / 35.6 and 33.6, 64 rows 174 and 140 / 49.5 and 54.4,
//     128 rows 309 and 162 / 80.1 and 85.7
enum class Many { kFew, k16, k32, k64, k128, k128Whole, k256 };
int32_t few_rows(const F8Head& h) { return h.B <= 16 ? 16 : 32; }
double few_time(const F8Head& h) {
  const int32_t each = few_tiles(h, few_rows(h)), rows = h.B < 32 ? h.B : 32;
  return 5.0 + f8_blocks(h.K) * ((each < 4 ? 0.05 * each : 0.1 * each - 0.15) + rows * (0.0125 + 0.0005 * each));
}
// one, block: of a block of a pass in which no wave has more than a tile, and of others
double many_time(const F8Head& h, int32_t rows, int32_t waves, double start, double one, double block, double tile) {
  const int32_t each = few_tiles(h, rows), passes = (each + 15) / 16;  // (a pass is 16 tiles in all of them)
  const double latency = each <= waves ? one : passes * block, bytes = each * tile;
  return start + f8_blocks(h.K) * (latency > bytes ? latency : bytes);
}
Many kernel_of(const F8Head& h, Elem logits_type) {
  const bool whole = logits_type != Elem::kBF16;  // (sums of 24 bits)
  Many best = Many::k16;
  double time = 0.0;
  auto offer = [&](Many kernel, double t) {
    if (time == 0.0 || t < time) best = kernel, time = t;
  };
  const double start = h.hidden.scales ? 6.0 : 10.0;
  if (h.B <= 16) offer(Many::k16, many_time(h, 16, 8, start, 0.28, 0.46, 0.083));
  else if (h.B <= 32) offer(Many::k32, many_time(h, 32, 8, start, 0.32, 0.63, 0.09));
  else if (h.B <= 64) offer(Many::k64, many_time(h, 64, 8, start, 0.43, 0.95, 0.09));
  else if (whole) offer(Many::k128Whole, many_time(h, 128, 4, 10.0, 0.5, 1.85, 0.0));
  else offer(Many::k128, many_time(h, 128, 4, 10.0, 0.48, 1.1, 0.0));
  if (!whole && !h.mask && h.B > 128) offer(Many::k256, many_time(h, 256, 0, 10.0, 0.0, 1.95, 0.0));  // (with lists of rows its registers would not do)
  if (few_fits(h, h.B < 32 ? h.B : 32)) offer(Many::kFew, few_time(h));
  return best;
}
}  // namespace
hipError_t launch_f8_logits(const F8Head& head, Elem hidden_type, Elem logits_type, void* work, hipStream_t stream) {
  F8Head h = head;
  const Many kernel = kernel_of(h, logits_type);
  if (kernel == Many::kFew) return few_rows(h) == 16 ? launch_few_states<1>(h, hidden_type, logits_type, stream) : launch_few_states<2>(h, hidden_type, logits_type, stream);
  StateScales strides{f8_blocks(h.K), 1};
  // A block's scales side by side: as they are, 256 rows take as many requests as 16 KB of codes.  (Of 64 rows and less, as they are: 64 rows of
  // 128256 x 4096 take 105 us and 106 with the launch for it, 32 of 50001 x 2080 29.2 and 30.8.)
  if (h.hidden.scales && work && h.B > 64) {
    float* const scales = static_cast<float*>(work);
    strides = StateScales{1, h.B};
    const int64_t n = (int64_t)h.B * f8_blocks(h.K);
    hipLaunchKernelGGL(f8_turn_scales_kernel, dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, stream, h.hidden.scales, h.B, f8_blocks(h.K), scales);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    h.hidden.scales = scales;
  }
  if (!h.hidden.scales) {
    uint8_t* const codes = static_cast<uint8_t*>(work);
    float* const scales = reinterpret_cast<float*>(codes + h.B * padded(h.K));
    strides = StateScales{1, h.B};
    if (const hipError_t e = quantize_any(h.hidden.at, hidden_type, h.B, h.K, h.hidden.stride, Quantized{codes, padded(h.K), (int32_t)padded(h.K), scales, strides}, stream);
        e != hipSuccess)
      return e;
    h.hidden = F8States{codes, padded(h.K), scales};
  }
  switch (kernel) {
    case Many::k16: return launch_many_masked<1, 1, 2, Halves>(h, strides, logits_type, stream);
    case Many::k32: return launch_many_masked<2, 1, 2, Halves>(h, strides, logits_type, stream);
    case Many::k64: return launch_many_masked<4, 1, 2, Halves>(h, strides, logits_type, stream);
    case Many::k128Whole: return launch_many_masked<4, 2, 4, Halves>(h, strides, logits_type, stream);
    case Many::k256: return launch_many<8, 2, 4, false, Eights>(h, strides, logits_type, stream);
    default: return launch_many_masked<4, 2, 4, Eights>(h, strides, logits_type, stream);
  }
}

hipError_t launch_q4_embed(const Embed& e, Elem scales_type, Elem out_type, hipStream_t stream) {
  if (scales_type == Elem::kF16) return launch_embed<Elem::kF16, true>(e, out_type, stream);
  return launch_embed<Elem::kBF16, true>(e, out_type, stream);
}
hipError_t launch_f8_embed(const Embed& e, Elem out_type, hipStream_t stream) { return launch_embed<Elem::kF32, false>(e, out_type, stream); }

}  // namespace xgm
