// 8-bit activation checkpoints (include/falqon_train.h): E4M3 codes with one power-of-two scale per 32 values of a row.
// Powers of two make the scaling exact, so a value is rounded once, and the 64-bit definition gives the same codes.
#pragma once

#include <cstdint>

#include "chain_math.cuh"
#include "ptx.cuh"

namespace falqon {

constexpr int kMx8Block = 32;

// The scale byte of a block whose largest |value| has this fp32 bit pattern.  448 = 1.75 * 2^8: the exponent less 8, plus one
// if the mantissa is above 1.75 (adding 0x1FFFFF to the bits carries into the exponent exactly then); 255 for inf and NaN.
__device__ __forceinline__ uint32_t mx8_exponent(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 255u;
  return static_cast<uint32_t>(max(static_cast<int>((amax_bits + 0x1FFFFFu) >> 23) - 8, 0));
}
// 2^(127 - e): e is at most 247 here, so this is a normal number; NaN for a block marked 255.
__device__ __forceinline__ float mx8_encode_factor(uint32_t e) {
  return __uint_as_float(e == 255u ? 0x7FC00000u : (254u - e) << 23);
}
// 2^(e - 127), of which e = 0 is subnormal.
__device__ __forceinline__ float mx8_decode_factor(uint32_t e) {
  return __uint_as_float(e == 255u ? 0x7FC00000u : e == 0u ? 0x00400000u : e << 23);
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <typename T>
struct Vec8;   // eight values as they lie in memory

struct bf16_t { uint16_t bits; };

template <>
struct Vec8<bf16_t> {
  uint4 q;
  __device__ __forceinline__ void load(const bf16_t* p) { q = ld_stream(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void zero() { q = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void unpack(float (&x)[8]) const { unpack8(q, x); }
  __device__ __forceinline__ void pack(const float (&x)[8]) { q = pack8(x); }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<uint4*>(p) = q; }
  // fp32 bit pattern of the largest |value|
  __device__ __forceinline__ uint32_t max_abs() const { return max_abs_bf16(q, 0u) << 16; }
};
template <>
struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = ld_stream(reinterpret_cast<const float4*>(p));
    b = ld_stream(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
  __device__ __forceinline__ void pack(const float (&x)[8]) {
    a = make_float4(x[0], x[1], x[2], x[3]);
    b = make_float4(x[4], x[5], x[6], x[7]);
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
  __device__ __forceinline__ uint32_t max_abs() const {
    return max(max(max(abs_bits(a.x), abs_bits(a.y)), max(abs_bits(a.z), abs_bits(a.w))),
               max(max(abs_bits(b.x), abs_bits(b.y)), max(abs_bits(b.z), abs_bits(b.w))));
  }
};

__device__ __forceinline__ float load1(const bf16_t* p) {
  return bf16_bits_to_float(ld_stream(reinterpret_cast<const uint16_t*>(p)));
}
__device__ __forceinline__ float load1(const float* p) { return ld_stream(p); }
// Stores one value and returns the fp32 bit pattern of what was stored, without its sign.
__device__ __forceinline__ uint32_t store1(bf16_t* p, float v) {
  const uint32_t b = pack2(v, 0.0f) & 0xFFFFu;
  p->bits = static_cast<uint16_t>(b);
  return (b & 0x7FFFu) << 16;
}
__device__ __forceinline__ uint32_t store1(float* p, float v) {
  *p = v;
  return abs_bits(v);
}

// The codes of eight values under an encode factor; each product is exact.
__device__ __forceinline__ uint2 mx8_encode8(const float (&x)[8], float f) {
  return make_uint2(cvt_fp8x4<0>(x[0] * f, x[1] * f, x[2] * f, x[3] * f), cvt_fp8x4<0>(x[4] * f, x[5] * f, x[6] * f, x[7] * f));
}
__device__ __forceinline__ uint8_t mx8_encode1(float x, float f) { return static_cast<uint8_t>(cvt_fp8x2<0>(x * f, 0.0f) & 0xFFu); }
__device__ __forceinline__ void mx8_decode8(const uint2& q, float f, float (&x)[8]) {
  const uint32_t w[2] = {q.x, q.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 lo = e4m3x2_to_float2(w[i] & 0xFFFFu), hi = e4m3x2_to_float2(w[i] >> 16);
    x[4 * i] = lo.x * f, x[4 * i + 1] = lo.y * f, x[4 * i + 2] = hi.x * f, x[4 * i + 3] = hi.y * f;
  }
}
__device__ __forceinline__ float mx8_decode1(uint8_t c, float f) { return e4m3x2_to_float2(c).x * f; }

// Block maxima across lanes: four lanes of eight values, or a warp of one value each.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
  return max(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
}

// Raises *amax to the CTA's largest |value| (m: fp32 bit patterns without the sign) with one atomic; all threads call it.
__device__ __forceinline__ void raise_amax(uint32_t m, float* amax) {
  __shared__ uint32_t s_amax;
  if (threadIdx.x == 0) s_amax = 0u;
  __syncthreads();
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0 && m != 0u) atomicMax(&s_amax, m);
  __syncthreads();
  if (threadIdx.x == 0 && s_amax != 0u) atomicMax(reinterpret_cast<unsigned int*>(amax), s_amax);
}

}  // namespace falqon
