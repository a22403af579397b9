// 8-bit codes by blocks of 128 (include/falqon_dense.h): quantizer and its inverse.
//   e = the smallest e >= 0 with amax * 2^(127 - e) <= the type's largest value;  code = round(v * 2^(127 - e))
// HBM-bound: a value is read once, whatever is made of it.  A CTA takes one 128 x 128 tile into registers (64 values a thread, all
// loads in flight at once), so that the maxima of its rows, of its columns or of the whole tile cost shuffles and 4 KB of shared
// memory, and the codes of both directions come from one read.
#include "../../include/falqon_dense.h"
#include "chain_math.cuh"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kB = FALQON_BLOCK;
constexpr int kThreads = 256, kWarps = kThreads / 32;

// The scale byte for a block whose largest |value| has this fp32 bit pattern: kFmt 0 as in a checkpoint; 57344 = 1.75 * 2^15.
template <int kFmt>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  if (kFmt == 0) return mx8_exponent(amax_bits);
  if (amax_bits >= 0x7F800000u) return 255u;
  return static_cast<uint32_t>(max(static_cast<int>((amax_bits + 0x1FFFFFu) >> 23) - 15, 0));
}

struct QuantArgs {
  int64_t rows, cols, ld;
  int64_t col_tiles;
  uint8_t *row_codes, *row_scales;   // along rows (or, kTile, by tiles)
  uint8_t *col_codes, *col_scales;   // along columns
};

// Maxima of eight columns: of bf16 as pairs in the type itself, of fp32 as bit patterns without the sign.
template <typename T>
struct ColMax;
template <>
struct ColMax<bf16_t> {
  uint32_t m[4] = {0u, 0u, 0u, 0u};
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ __forceinline__ void see(const Vec8<bf16_t>& v) {
    const uint32_t w[4] = {v.q.x, v.q.y, v.q.z, v.q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = larger(m[k], w[k] & 0x7FFF7FFFu);
  }
  __device__ __forceinline__ void across(int s) {
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = larger(m[k], __shfl_xor_sync(0xFFFFFFFFu, m[k], s));
  }
  __device__ __forceinline__ uint32_t bits(int j) const { return j & 1 ? m[j >> 1] & 0xFFFF0000u : m[j >> 1] << 16; }
};
template <>
struct ColMax<float> {
  uint32_t m[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
  __device__ __forceinline__ void see(const Vec8<float>& v) {
    const float x[8] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = max(m[k], abs_bits(x[k]));
  }
  __device__ __forceinline__ void across(int s) {
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = max(m[k], __shfl_xor_sync(0xFFFFFFFFu, m[k], s));
  }
  __device__ __forceinline__ uint32_t bits(int j) const { return m[j]; }
};

// Codes of eight values times four pairs of factors (powers of two: exact).
template <int kFmt, typename T>
__device__ __forceinline__ uint2 codes8(const Vec8<T>& v, const f2 (&f)[4]) {
  f2 x[4];
  v.pairs(x);
  float y[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(mul2(x[k], f[k]), y[2 * k], y[2 * k + 1]);
  return make_uint2(cvt_fp8x4<kFmt>(y[0], y[1], y[2], y[3]), cvt_fp8x4<kFmt>(y[4], y[5], y[6], y[7]));
}

// The largest |value| of two rows over the 16 lanes that hold them, as fp32 bit patterns: bf16 rows side by side in one register.
__device__ __forceinline__ void row_maxima(const Vec8<bf16_t>& a, const Vec8<bf16_t>& b, uint32_t& ma, uint32_t& mb) {
  auto of = [](const Vec8<bf16_t>& v) {
    const uint32_t w[4] = {v.q.x, v.q.y, v.q.z, v.q.w};
    uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int k = 1; k < 4; ++k) m = ColMax<bf16_t>::larger(m, w[k] & 0x7FFF7FFFu);
    return m;
  };
  const uint32_t x = of(a), y = of(b);
  uint32_t m = ColMax<bf16_t>::larger(__byte_perm(x, y, 0x5410), __byte_perm(x, y, 0x7632));
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) m = ColMax<bf16_t>::larger(m, __shfl_xor_sync(0xFFFFFFFFu, m, s));
  ma = m << 16, mb = m & 0xFFFF0000u;
}
__device__ __forceinline__ void row_maxima(const Vec8<float>& a, const Vec8<float>& b, uint32_t& ma, uint32_t& mb) {
  ma = a.max_abs(), mb = b.max_abs();
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) {
    ma = max(ma, __shfl_xor_sync(0xFFFFFFFFu, ma, s));
    mb = max(mb, __shfl_xor_sync(0xFFFFFFFFu, mb, s));
  }
}

// Rows of whole 16-byte vectors.  A warp lies on 16 rows of the tile, two at a time, 16 lanes x 8 values to a row; values stay as they
// came (bf16: half the registers).
template <typename T, int kFmt, bool kRow, bool kCol, bool kTile>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? (kRow && kCol ? 3 : 4) : 2)
block_quant_kernel(const T* x, const QuantArgs a) {
  constexpr int kPasses = 8;
  __shared__ __align__(16) uint32_t s_max[kWarps][kB];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t tile_r = blockIdx.x / static_cast<uint32_t>(a.col_tiles), tile_c = blockIdx.x - tile_r * a.col_tiles;
  const int64_t row0 = tile_r * kB + warp * 16 + (lane >> 4), col = tile_c * kB + (lane & 15) * 8;
  // passes with a row of this lane; none behind the right edge (a vector is inside or outside as a whole)
  const int passes = col < a.cols && row0 < a.rows ? static_cast<int>(min(static_cast<int64_t>(kPasses), (a.rows - row0 + 1) / 2)) : 0;

  Vec8<T> v[kPasses];
  {
    const T* src = x + row0 * a.ld + col;
#pragma unroll
    for (int p = 0; p < kPasses; ++p, src += 2 * a.ld) {
      if (p < passes) v[p].load(src); else v[p].zero();
    }
  }
  const int64_t first = row0 * a.cols + col, step = 2 * a.cols;
  auto same = [](f2 (&f)[4], uint32_t e) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = twice(mx8_encode_factor(e));
  };

  ColMax<T> m;
  if constexpr (kCol || kTile) {
#pragma unroll
    for (int p = 0; p < kPasses; ++p) m.see(v[p]);
    m.across(16);
  }
  if constexpr (kCol) {
    if (lane < 16) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<uint4*>(&s_max[warp][lane * 8 + 4 * h]) = make_uint4(m.bits(4 * h), m.bits(4 * h + 1), m.bits(4 * h + 2), m.bits(4 * h + 3));
    }
  }
  if constexpr (kTile) {
    uint32_t all = m.bits(0);
#pragma unroll
    for (int j = 1; j < 8; ++j) all = max(all, m.bits(j));
    all = __reduce_max_sync(0xFFFFFFFFu, all);
    if (lane == 0) s_max[warp][0] = all;
  }
  if constexpr (kRow) {
    uint8_t* dst = a.row_codes + first;
    uint8_t* scale = a.row_scales + row0 * a.col_tiles + tile_c;
#pragma unroll
    for (int p = 0; p < kPasses; p += 2) {
      uint32_t r[2];
      row_maxima(v[p], v[p + 1], r[0], r[1]);
#pragma unroll
      for (int k = 0; k < 2; ++k, dst += step, scale += 2 * a.col_tiles) {
        const uint32_t e = scale_byte<kFmt>(r[k]);
        f2 f[4];
        same(f, e);
        const uint2 c = codes8<kFmt>(v[p + k], f);
        if (p + k < passes) {
          *reinterpret_cast<uint2*>(dst) = c;
          if ((lane & 15) == 0) *scale = static_cast<uint8_t>(e);
        }
      }
    }
  }
  if constexpr (kTile) {
    __syncthreads();
    uint32_t all = 0u;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all = max(all, s_max[w][0]);
    const uint32_t e = scale_byte<kFmt>(all);
    if (threadIdx.x == 0) a.row_scales[tile_r * a.col_tiles + tile_c] = static_cast<uint8_t>(e);
    f2 f[4];
    same(f, e);
    uint8_t* dst = a.row_codes + first;
#pragma unroll
    for (int p = 0; p < kPasses; ++p, dst += step)
      if (p < passes) *reinterpret_cast<uint2*>(dst) = codes8<kFmt>(v[p], f);
  }
  if constexpr (kCol) {
    __syncthreads();
    // a column's maximum is taken by one thread and handed to the 16 that need it
    if (threadIdx.x < kB) {
      uint32_t c = 0u;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) c = max(c, s_max[w][threadIdx.x]);
      const uint32_t e = scale_byte<kFmt>(c);
      s_max[0][threadIdx.x] = __float_as_uint(mx8_encode_factor(e));
      if (tile_c * kB + threadIdx.x < a.cols) a.col_scales[tile_r * a.cols + tile_c * kB + threadIdx.x] = static_cast<uint8_t>(e);
    }
    __syncthreads();
    f2 f[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 q = *reinterpret_cast<const float4*>(&s_max[0][(lane & 15) * 8 + 4 * h]);
      f[2 * h] = pack_f32x2(q.x, q.y), f[2 * h + 1] = pack_f32x2(q.z, q.w);
    }
    uint8_t* dst = a.col_codes + first;
#pragma unroll
    for (int p = 0; p < kPasses; ++p, dst += step)
      if (p < passes) *reinterpret_cast<uint2*>(dst) = codes8<kFmt>(v[p], f);
  }
}

// Any other width, pitch or alignment: 32 lanes to a row, values 32 apart, a row at a time, four values a lane.
template <typename T, int kFmt, bool kRow, bool kCol, bool kTile>
__global__ void __launch_bounds__(kThreads, 2)
block_quant_ragged_kernel(const T* x, const QuantArgs a) {
  constexpr int kPasses = 16, kValues = 4;
  __shared__ __align__(16) uint32_t s_max[kWarps][kB];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t tile_r = blockIdx.x / a.col_tiles, tile_c = blockIdx.x - tile_r * a.col_tiles;
  const int64_t row0 = tile_r * kB + warp * 16, col0 = tile_c * kB + lane;
  const int rows = row0 < a.rows ? static_cast<int>(min(static_cast<int64_t>(kPasses), a.rows - row0)) : 0;
  bool in[kValues];
#pragma unroll
  for (int j = 0; j < kValues; ++j) in[j] = col0 + 32 * j < a.cols;
  float v[kPasses][kValues];
  {
    const T* src = x + row0 * a.ld + col0;
#pragma unroll
    for (int p = 0; p < kPasses; ++p, src += a.ld)
#pragma unroll
      for (int j = 0; j < kValues; ++j) v[p][j] = p < rows && in[j] ? load1(src + 32 * j) : 0.0f;
  }
  const int64_t first = row0 * a.cols + col0;
  auto store = [&](uint8_t* dst, int p, const float (&f)[kValues]) {
    const uint32_t c = cvt_fp8x4<kFmt>(v[p][0] * f[0], v[p][1] * f[1], v[p][2] * f[2], v[p][3] * f[3]);
#pragma unroll
    for (int j = 0; j < kValues; ++j)
      if (p < rows && in[j]) dst[32 * j] = static_cast<uint8_t>(c >> (8 * j));
  };
  if constexpr (kRow) {
    uint8_t* dst = a.row_codes + first;
    uint8_t* scale = a.row_scales + row0 * a.col_tiles + tile_c;
#pragma unroll
    for (int p = 0; p < kPasses; ++p, dst += a.cols, scale += a.col_tiles) {
      uint32_t r = 0u;
#pragma unroll
      for (int j = 0; j < kValues; ++j) r = max(r, abs_bits(v[p][j]));
      const uint32_t e = scale_byte<kFmt>(__reduce_max_sync(0xFFFFFFFFu, r));
      const float y = mx8_encode_factor(e), f[kValues] = {y, y, y, y};
      store(dst, p, f);
      if (lane == 0 && p < rows) *scale = static_cast<uint8_t>(e);
    }
  }
  if constexpr (kCol || kTile) {
    uint32_t m[kValues];
#pragma unroll
    for (int j = 0; j < kValues; ++j) {
      m[j] = 0u;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) m[j] = max(m[j], abs_bits(v[p][j]));
      s_max[warp][32 * j + lane] = m[j];
    }
    __syncthreads();
    float f[kValues];
    uint32_t c[kValues];
#pragma unroll
    for (int j = 0; j < kValues; ++j) {
      c[j] = 0u;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) c[j] = max(c[j], s_max[w][32 * j + lane]);
    }
    if constexpr (kTile) {
      const uint32_t e = scale_byte<kFmt>(__reduce_max_sync(0xFFFFFFFFu, max(max(c[0], c[1]), max(c[2], c[3]))));
      if (threadIdx.x == 0) a.row_scales[tile_r * a.col_tiles + tile_c] = static_cast<uint8_t>(e);
#pragma unroll
      for (int j = 0; j < kValues; ++j) f[j] = mx8_encode_factor(e);
    } else {
#pragma unroll
      for (int j = 0; j < kValues; ++j) {
        const uint32_t e = scale_byte<kFmt>(c[j]);
        f[j] = mx8_encode_factor(e);
        if (warp == 0 && in[j]) a.col_scales[tile_r * a.cols + col0 + 32 * j] = static_cast<uint8_t>(e);
      }
    }
    uint8_t* dst = (kTile ? a.row_codes : a.col_codes) + first;
#pragma unroll
    for (int p = 0; p < kPasses; ++p, dst += a.cols) store(dst, p, f);
  }
}

// ---------------------------------------------------------------- the inverse
__device__ __forceinline__ float decode1(uint8_t code, int fmt) {
  if (fmt == 0) return e4m3x2_to_float2(code).x;
  uint32_t h2;
  asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h2) : "h"(static_cast<uint16_t>(code)));
  float r;
  asm("{\n\t.reg .f16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.f32.f16 %0, lo;\n\t}" : "=f"(r) : "r"(h2));
  return r;
}

// A value a thread, in rows of 256: read and written once; for looking at weights and for export, not for a step.
template <typename T>
__global__ void __launch_bounds__(kThreads)
block_dequant_kernel(const uint8_t* codes, const uint8_t* scales, int fmt, int along, int64_t rows, int64_t cols, T* y) {
  pdl_trigger();
  pdl_wait();
  const int64_t blocks = (cols + kB - 1) / kB, spans = (cols + kThreads - 1) / kThreads;
  for (int64_t u = blockIdx.x; u < rows * spans; u += gridDim.x) {
    const int64_t r = u / spans, c = (u - r * spans) * kThreads + threadIdx.x;
    if (c >= cols) continue;
    const int64_t at = along == FALQON_ALONG_ROW ? r * blocks + c / kB : along == FALQON_ALONG_COL ? (r / kB) * cols + c : (r / kB) * blocks + c / kB;
    store1(y + r * cols + c, decode1(ld_stream(codes + r * cols + c), fmt) * mx8_decode_factor(ld_stream(scales + at)));
  }
}

bool sizes_ok(int64_t rows, int64_t cols) {
  constexpr int64_t kMost = int64_t{1} << 30;
  return rows >= 1 && cols >= 1 && rows <= kMost && cols <= kMost && rows <= (int64_t{1} << 42) / cols;
}
bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int finish(cudaError_t e) { return e == cudaSuccess ? FALQON_OK : FALQON_ERR_CUDA; }

constexpr int kBoth = 3;

template <typename T, int kFmt, bool kRow, bool kCol, bool kTile>
cudaError_t launch_one(const T* x, const QuantArgs& a, int64_t tiles, bool vec, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(tiles)), block(kThreads);
  return vec ? launch_pdl(block_quant_kernel<T, kFmt, kRow, kCol, kTile>, grid, block, 0, st, 1, x, a)
             : launch_pdl(block_quant_ragged_kernel<T, kFmt, kRow, kCol, kTile>, grid, block, 0, st, 1, x, a);
}
template <typename T, int kFmt>
cudaError_t launch_of(int what, const T* x, const QuantArgs& a, int64_t tiles, bool vec, cudaStream_t st) {
  switch (what) {
    case FALQON_ALONG_ROW: return launch_one<T, kFmt, true, false, false>(x, a, tiles, vec, st);
    case FALQON_ALONG_COL: return launch_one<T, kFmt, false, true, false>(x, a, tiles, vec, st);
    case FALQON_TILE: return launch_one<T, kFmt, false, false, true>(x, a, tiles, vec, st);
    default: return launch_one<T, kFmt, true, true, false>(x, a, tiles, vec, st);
  }
}

template <typename T>
int quantize(int what, const void* x, int64_t rows, int64_t cols, int64_t ld, int fmt, uint8_t* row_codes, uint8_t* row_scales,
             uint8_t* col_codes, uint8_t* col_scales, cudaStream_t st) {
  const int64_t tiles = ((rows + kB - 1) / kB) * ((cols + kB - 1) / kB);
  const QuantArgs a{rows, cols, ld, (cols + kB - 1) / kB, row_codes, row_scales, col_codes, col_scales};
  const bool vec = cols % 8 == 0 && (ld * sizeof(T)) % 16 == 0 && aligned_to(x, 16) && aligned_to(row_codes, 8) && aligned_to(col_codes, 8);
  const T* src = static_cast<const T*>(x);
  return finish(fmt == FALQON_E4M3 ? launch_of<T, 0>(what, src, a, tiles, vec, st) : launch_of<T, 1>(what, src, a, tiles, vec, st));
}

int quantize_checked(int what, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int fmt, uint8_t* row_codes,
                     uint8_t* row_scales, uint8_t* col_codes, uint8_t* col_scales, cudaStream_t st) {
  if (x == nullptr || x == row_codes || x == col_codes || !sizes_ok(rows, cols) || ld < cols || ld > (int64_t{1} << 44) / rows || (dtype != FALQON_BF16 && dtype != FALQON_F32) ||
      (fmt != FALQON_E4M3 && fmt != FALQON_E5M2) || !aligned_to(x, dtype == FALQON_BF16 ? 2 : 4))
    return FALQON_ERR_INVALID_ARG;
  return dtype == FALQON_BF16 ? quantize<bf16_t>(what, x, rows, cols, ld, fmt, row_codes, row_scales, col_codes, col_scales, st)
                              : quantize<float>(what, x, rows, cols, ld, fmt, row_codes, row_scales, col_codes, col_scales, st);
}

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

int falqon_block_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, falqon_fp8 fmt, falqon_blocking along,
                          uint8_t* codes, uint8_t* scales, falqon_stream stream) {
  if (codes == nullptr || scales == nullptr || (along != FALQON_ALONG_ROW && along != FALQON_ALONG_COL && along != FALQON_TILE))
    return FALQON_ERR_INVALID_ARG;
  const bool col = along == FALQON_ALONG_COL;
  return quantize_checked(along, x, dtype, rows, cols, ld, fmt, col ? nullptr : codes, col ? nullptr : scales, col ? codes : nullptr,
                          col ? scales : nullptr, static_cast<cudaStream_t>(stream));
}

int falqon_block_quantize_both(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, falqon_fp8 fmt, uint8_t* row_codes,
                               uint8_t* row_scales, uint8_t* col_codes, uint8_t* col_scales, falqon_stream stream) {
  if (row_codes == nullptr || row_scales == nullptr || col_codes == nullptr || col_scales == nullptr || row_codes == col_codes)
    return FALQON_ERR_INVALID_ARG;
  return quantize_checked(kBoth, x, dtype, rows, cols, ld, fmt, row_codes, row_scales, col_codes, col_scales, static_cast<cudaStream_t>(stream));
}

int falqon_block_dequantize(const uint8_t* codes, const uint8_t* scales, falqon_fp8 fmt, falqon_blocking along, int64_t rows, int64_t cols,
                            void* y, int dtype, falqon_stream stream) {
  if (codes == nullptr || scales == nullptr || y == nullptr || !sizes_ok(rows, cols) || (fmt != FALQON_E4M3 && fmt != FALQON_E5M2) ||
      (along != FALQON_ALONG_ROW && along != FALQON_ALONG_COL && along != FALQON_TILE) || (dtype != FALQON_BF16 && dtype != FALQON_F32) ||
      !aligned_to(y, dtype == FALQON_BF16 ? 2 : 4))
    return FALQON_ERR_INVALID_ARG;
  const int64_t units = rows * ((cols + kThreads - 1) / kThreads), cap = static_cast<int64_t>(sm_count()) * 8;
  const dim3 grid(static_cast<unsigned>(units < cap ? units : cap));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return finish(dtype == FALQON_BF16
                    ? launch_pdl(block_dequant_kernel<bf16_t>, grid, dim3(kThreads), 0, st, 1, codes, scales, static_cast<int>(fmt),
                                 static_cast<int>(along), rows, cols, static_cast<bf16_t*>(y))
                    : launch_pdl(block_dequant_kernel<float>, grid, dim3(kThreads), 0, st, 1, codes, scales, static_cast<int>(fmt),
                                 static_cast<int>(along), rows, cols, static_cast<float*>(y)));
}

}  // extern "C"
