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

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
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
  __device__ __forceinline__ void pairs(uint64_t (&x)[4]) const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = pack_f32x2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u));
  }
  __device__ __forceinline__ void pack(const float (&x)[8]) { q = pack8(x); }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<uint4*>(p) = q; }
  // fp32 bit pattern of the largest |value| (a NaN if there is one)
  __device__ __forceinline__ uint32_t max_abs() const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t m = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) asm("{\n\t.reg .b32 t;\n\tabs.bf16x2 t, %1;\n\tmax.NaN.bf16x2 %0, %0, t;\n\t}" : "+r"(m) : "r"(w[k]));
    return max(m << 16, m & 0xFFFF0000u);
  }
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
  __device__ __forceinline__ void pairs(uint64_t (&x)[4]) const {
    x[0] = pack_f32x2(a.x, a.y), x[1] = pack_f32x2(a.z, a.w), x[2] = pack_f32x2(b.x, b.y), x[3] = pack_f32x2(b.z, b.w);
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
    return abs_bits(max_nan(max_nan(max_nan(fabsf(a.x), fabsf(a.y)), max_nan(fabsf(a.z), fabsf(a.w))),
                            max_nan(max_nan(fabsf(b.x), fabsf(b.y)), max_nan(fabsf(b.z), fabsf(b.w)))));
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

__device__ __forceinline__ uint8_t mx8_encode1(float x, float f) { return static_cast<uint8_t>(cvt_fp8x2<0>(x * f, 0.0f) & 0xFFu); }
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


// ---- arithmetic on two fp32 values per instruction (each half an ordinary rounded operation)
using f2 = uint64_t;                                    // two fp32 values
__device__ __forceinline__ f2 twice(float x) { return pack_f32x2(x, x); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float halves(f2 a) {         // the sum of the two
  float lo, hi;
  unpack_f32x2(a, lo, hi);
  return lo + hi;
}

// Four E4M3 codes as two pairs of fp32, exact.
__device__ __forceinline__ void decode4(uint32_t w, f2& lo, f2& hi) {
  float v[4];
  asm("{\n\t.reg .b16 a, b, h0, h1, h2, h3;\n\t.reg .b32 p, q;\n\t"
      "mov.b32 {a, b}, %4;\n\t"
      "cvt.rn.f16x2.e4m3x2 p, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 q, b;\n\t"
      "mov.b32 {h0, h1}, p;\n\tmov.b32 {h2, h3}, q;\n\t"
      "cvt.f32.f16 %0, h0;\n\tcvt.f32.f16 %1, h1;\n\tcvt.f32.f16 %2, h2;\n\tcvt.f32.f16 %3, h3;\n\t}"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
      : "r"(w));
  lo = pack_f32x2(v[0], v[1]);
  hi = pack_f32x2(v[2], v[3]);
}
// 2^(e - 127) for codes as checkpoints hold them: a block marked 255 has NaN codes, whatever they are multiplied by.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(max(e << 23, 0x00400000u)); }

// The largest |value| a thread has stored (NaN if there was one).
template <typename T>
struct Largest;
template <>
struct Largest<float> {
  float m = 0.0f;
  __device__ __forceinline__ void see(const Vec8<float>& v) {
    const float x[8] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(x[e]));
  }
  __device__ __forceinline__ uint32_t bits() const { return abs_bits(m); }
};
template <>
struct Largest<bf16_t> {
  uint32_t m = 0u;      // two values
  __device__ __forceinline__ void see(const Vec8<bf16_t>& v) {
    const uint32_t w[4] = {v.q.x, v.q.y, v.q.z, v.q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      asm("{\n\t.reg .b32 t;\n\tabs.bf16x2 t, %1;\n\tmax.NaN.bf16x2 %0, %0, t;\n\t}" : "+r"(m) : "r"(w[k]));
  }
  __device__ __forceinline__ uint32_t bits() const { return max(m << 16, m & 0xFFFF0000u); }
};

// Eight results, rounded once.
template <typename T>
__device__ __forceinline__ Vec8<T> write8(T* p, const f2 (&x)[4]) {
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(x[k], v[2 * k], v[2 * k + 1]);
  Vec8<T> o;
  o.pack(v);
  o.store(p);
  return o;
}
// The codes of eight values under an encode factor; each product is exact.
__device__ __forceinline__ uint2 mx8_encode8(const f2 (&x)[4], float f) {
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(mul2(x[k], twice(f)), v[2 * k], v[2 * k + 1]);
  return make_uint2(cvt_fp8x4<0>(v[0], v[1], v[2], v[3]), cvt_fp8x4<0>(v[4], v[5], v[6], v[7]));
}
// Eight codes times f.
__device__ __forceinline__ void mx8_decode8(const uint2& q, float f, f2 (&x)[4]) {
  decode4(q.x, x[0], x[1]);
  decode4(q.y, x[2], x[3]);
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = mul2(x[k], twice(f));
}

}  // namespace falqon
