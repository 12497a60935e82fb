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
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Codes go through the matrix instructions as f16, which holds every e4m3 number: the instructions for 8 bits add up neighbouring products
// with 14 bits of the largest of them, and sums of logits are to have the 24 of a float.
__device__ __forceinline__ f16x8 halves(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// 16 x 16 sums over 128 columns, of which a lane holds 32 of its row: the same ones on both sides, whichever they are.
__device__ __forceinline__ float4v products(uint4v a0, uint4v a1, uint4v b0, uint4v b1) {
  float4v c = {0, 0, 0, 0};
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(a0[0], a0[1]), halves(b0[0], b0[1]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(a0[2], a0[3]), halves(b0[2], b0[3]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(a1[0], a1[1]), halves(b1[0], b1[1]), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(a1[2], a1[3]), halves(b1[2], b1[3]), c, 0, 0, 0);
}

__device__ __forceinline__ void store_logit(const F8Head& h, Elem type, int64_t at, float y) {
  if (type == Elem::kF32) static_cast<uint32_t*>(h.logits)[at] = narrowed<Elem::kF32>(y);
  else if (type == Elem::kBF16) static_cast<uint16_t*>(h.logits)[at] = narrowed<Elem::kBF16>(y);
  else static_cast<uint16_t*>(h.logits)[at] = narrowed<Elem::kF16>(y);
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
  __device__ __forceinline__ uint2 codes(float inverse) const {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float t[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        t[k] = x[4 * i + k] * inverse;
        if (!(fabsf(t[k]) <= FLT_MAX)) t[k] = __builtin_nanf("");  // (an infinity becomes NaN, which e4m3 has)
      }
      int word = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], word, true);
    }
    return uint2{w[0], w[1]};
  }
};
// the largest of 16 neighbouring lanes
__device__ __forceinline__ float most_of_16(float m) {
#pragma unroll
  for (int d = 8; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  return m;
}
// 16 lanes to a block.  Columns behind K, up to `width`, become zeros.
template <Elem E>
__global__ __launch_bounds__(256) void f8_quantize_kernel(const void* x, int64_t stride, int32_t B, int32_t K, int32_t width, uint8_t* codes, int64_t codes_stride, float* scales) {
  const int32_t blocks = f8_blocks(K);
  const int64_t block = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 16;
  if (block >= (int64_t)B * blocks) return;  // (16 lanes together)
  const int32_t b = (int32_t)(block / blocks), kb = (int32_t)(block % blocks), k = kb * 128 + ((int32_t)threadIdx.x & 15) * 8;
  Eight<E> v;
  if (k < K) v.load(static_cast<const typename Type<E>::bits*>(x) + b * stride + k);
  else v.clear();
  const uint32_t e = exponent_of(most_of_16(v.most()));
  if (k < width) *reinterpret_cast<uint2*>(codes + b * codes_stride + k) = v.codes(__uint_as_float((254u - e) << 23));
  if (((int32_t)threadIdx.x & 15) == 0) scales[block] = __uint_as_float(e << 23);
}

// ------------------------------------------------------------------- the projection
// A wave takes 16 rows of the matrix and 16 of the batch.
__global__ __launch_bounds__(256) void f8_logits_kernel(F8Head h, Elem out_type) {
  const int32_t lane = (int32_t)threadIdx.x & 63, n = lane & 15, q = lane >> 4;
  const int64_t v0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 16;
  const int32_t b0 = (int32_t)blockIdx.y * 16;
  if (v0 >= h.V) return;
  const int64_t v = min(v0 + n, (int64_t)h.V - 1);
  const int32_t b = min(b0 + n, h.B - 1), blocks = f8_blocks(h.K);
  const uint8_t* const row = h.codes + v * h.K;
  const uint8_t* const state = static_cast<const uint8_t*>(h.hidden.at) + b * h.hidden.stride;
  const float* const row_scales = h.scales + (v0 >> 7) * blocks;  // (16 rows lie in one block)
  const float* const state_scales = h.hidden.scales + (int64_t)b * blocks;
  float4v acc = {0, 0, 0, 0};
  for (int32_t kb = 0; kb < blocks; ++kb) {
    const int32_t k0 = kb * 128 + q * 16, k1 = k0 + 64;
    const uint4v none = {0, 0, 0, 0};
    uint4v a0 = none, a1 = none, x0 = none, x1 = none;
    if (k0 < h.K) {
      a0 = *reinterpret_cast<const uint4v*>(row + k0);
      x0 = *reinterpret_cast<const uint4v*>(state + k0);
    }
    if (k1 < h.K) {
      a1 = *reinterpret_cast<const uint4v*>(row + k1);
      x1 = *reinterpret_cast<const uint4v*>(state + k1);
    }
    acc += products(a0, a1, x0, x1) * (row_scales[kb] * state_scales[kb]);
  }
  for (int i = 0; i < 4; ++i) {
    const int64_t token = v0 + q * 4 + i;
    if (token >= h.V || b0 + n >= h.B) continue;
    const bool ok = !h.mask || (token < h.V_mask && (h.mask[(size_t)b * h.W_mask + (token >> 5)] >> (token & 31) & 1u));
    store_logit(h, out_type, b * h.logits_stride + token, ok ? acc[i] : -__builtin_inff());
  }
}

int64_t padded(int32_t K) { return (int64_t)f8_blocks(K) * 128; }

// ------------------------------------------------------ rows of the matrix as hidden states
// value * scale * factor in 64 bits, rounded once.
template <Elem S, Elem O, bool Q4> __global__ __launch_bounds__(256) void embed_kernel(Embed e) {
  typedef typename Type<O>::bits bits;
  const int32_t units = e.K / 8;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < (int64_t)e.n * units; u += (int64_t)gridDim.x * 256) {
    const int32_t i = (int32_t)(u / units), k = (int32_t)(u % units) * 8, id = e.ids[i];
    const bool there = id >= 0 && id < e.V;
    float x[8];
    double scale = 0.0;
    if constexpr (Q4) {
      const int64_t g = (int64_t)(there ? id : 0) * (e.K / e.group) + k / e.group;
      const uint32_t w = there ? *reinterpret_cast<const uint32_t*>(e.codes + ((int64_t)id * e.K + k) / 2) : 0u;
      const int zero = e.zeros ? e.zeros[g] : 8;
      scale = (double)widened<S>(static_cast<const typename Type<S>::bits*>(e.scales)[g]);
      for (int j = 0; j < 8; ++j) x[j] = (float)((int)(w >> (4 * j) & 15u) - zero);
    } else {
      const uint2 w = there ? *reinterpret_cast<const uint2*>(e.codes + (int64_t)id * e.K + k) : uint2{0, 0};
      scale = (double)static_cast<const float*>(e.scales)[(int64_t)((there ? id : 0) >> 7) * f8_blocks(e.K) + (k >> 7)];
      x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w.x, 0); x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w.x, 1);
      x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w.x, 2); x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w.x, 3);
      x[4] = __builtin_amdgcn_cvt_f32_fp8((int)w.y, 0); x[5] = __builtin_amdgcn_cvt_f32_fp8((int)w.y, 1);
      x[6] = __builtin_amdgcn_cvt_f32_fp8((int)w.y, 2); x[7] = __builtin_amdgcn_cvt_f32_fp8((int)w.y, 3);
    }
    bits* const out = static_cast<bits*>(e.out) + (int64_t)i * e.out_stride + k;
    for (int j = 0; j < 8; ++j) out[j] = there ? narrowed<O>((double)x[j] * scale * (double)e.factor) : narrowed<O>(0.0f);
  }
}
template <Elem S, bool Q4> hipError_t launch_embed(const Embed& e, Elem out_type, hipStream_t stream) {
  const int64_t units = (int64_t)e.n * (e.K / 8), groups = (units + 255) / 256;
  const dim3 grid((uint32_t)(groups < (1 << 30) ? groups : 1 << 30));
  if (out_type == Elem::kF32) hipLaunchKernelGGL((embed_kernel<S, Elem::kF32, Q4>), grid, dim3(256), 0, stream, e);
  else if (out_type == Elem::kBF16) hipLaunchKernelGGL((embed_kernel<S, Elem::kBF16, Q4>), grid, dim3(256), 0, stream, e);
  else hipLaunchKernelGGL((embed_kernel<S, Elem::kF16, Q4>), grid, dim3(256), 0, stream, e);
  return hipGetLastError();
}

template <Elem E> hipError_t quantize(const void* x, int32_t B, int32_t K, int64_t stride, int32_t width, uint8_t* codes, int64_t codes_stride, float* scales, hipStream_t stream) {
  const int64_t groups = ((int64_t)B * f8_blocks(K) + 15) / 16;
  hipLaunchKernelGGL(f8_quantize_kernel<E>, dim3((uint32_t)groups), dim3(256), 0, stream, x, stride, B, K, width, codes, codes_stride, scales);
  return hipGetLastError();
}
hipError_t quantize_any(const void* x, Elem type, int32_t B, int32_t K, int64_t stride, int32_t width, uint8_t* codes, int64_t codes_stride, float* scales, hipStream_t stream) {
  if (type == Elem::kF32) return quantize<Elem::kF32>(x, B, K, stride, width, codes, codes_stride, scales, stream);
  if (type == Elem::kBF16) return quantize<Elem::kBF16>(x, B, K, stride, width, codes, codes_stride, scales, stream);
  return quantize<Elem::kF16>(x, B, K, stride, width, codes, codes_stride, scales, stream);
}

}  // namespace

size_t f8_work_bytes(int32_t B, int32_t K) { return (size_t)B * (size_t)(padded(K) + f8_blocks(K) * 4); }

hipError_t launch_f8_quantize(const void* x, Elem type, int32_t B, int32_t K, int64_t stride, uint8_t* codes, int64_t codes_stride, float* scales, hipStream_t stream) {
  return quantize_any(x, type, B, K, stride, K, codes, codes_stride, scales, stream);
}

hipError_t launch_f8_logits(const F8Head& head, Elem hidden_type, Elem logits_type, void* work, hipStream_t stream) {
  F8Head h = head;
  if (!h.hidden.scales) {
    uint8_t* const codes = static_cast<uint8_t*>(work);
    float* const scales = reinterpret_cast<float*>(codes + h.B * padded(h.K));
    if (const hipError_t e = quantize_any(h.hidden.at, hidden_type, h.B, h.K, h.hidden.stride, (int32_t)padded(h.K), codes, padded(h.K), scales, stream); e != hipSuccess) return e;
    h.hidden = F8States{codes, padded(h.K), scales};
  }
  const dim3 grid((uint32_t)(((int64_t)h.V + 63) / 64), (uint32_t)((h.B + 15) / 16));
  hipLaunchKernelGGL(f8_logits_kernel, grid, dim3(256), 0, stream, h, logits_type);
  return hipGetLastError();
}

hipError_t launch_q4_embed(const Embed& e, Elem scales_type, Elem out_type, hipStream_t stream) {
  if (scales_type == Elem::kF16) return launch_embed<Elem::kF16, true>(e, out_type, stream);
  return launch_embed<Elem::kBF16, true>(e, out_type, stream);
}
hipError_t launch_f8_embed(const Embed& e, Elem out_type, hipStream_t stream) { return launch_embed<Elem::kF32, false>(e, out_type, stream); }

}  // namespace xgm
