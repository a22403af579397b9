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

// How a warp lies on its 16 rows of the tile.  Vectors: 16 lanes x 8 values a row, two rows at a time (16-byte loads, 8-byte stores).
// Singles (rows that are not 16-byte aligned, or a width that is no multiple of eight): 32 lanes, values 32 apart, a row at a time.
template <bool kVec>
struct Lay {
  static constexpr int kValues = kVec ? 8 : 4;           // of a lane in a row
  static constexpr int kPasses = 64 / kValues;
  static __device__ __forceinline__ int row(int lane, int pass) { return kVec ? 2 * pass + (lane >> 4) : pass; }
  static __device__ __forceinline__ int col(int lane, int j) { return kVec ? (lane & 15) * 8 + j : lane + 32 * j; }
};

template <typename T, int kFmt, bool kVec, bool kRow, bool kCol, bool kTile>
__global__ void __launch_bounds__(kThreads)
block_quant_kernel(const T* x, const QuantArgs a) {
  using L = Lay<kVec>;
  __shared__ uint32_t s_max[kWarps][kB];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t tile_r = blockIdx.x / a.col_tiles, tile_c = blockIdx.x - tile_r * a.col_tiles;
  const int64_t row0 = tile_r * kB + warp * 16, col0 = tile_c * kB;
  const bool col_in = col0 + L::col(lane, 0) < a.cols;   // vectors are inside or outside as a whole

  float v[L::kPasses][L::kValues];
#pragma unroll
  for (int p = 0; p < L::kPasses; ++p) {
    const int64_t r = row0 + L::row(lane, p);
    const T* src = x + r * a.ld + col0;
    if constexpr (kVec) {
      Vec8<T> q;
      if (r < a.rows && col_in) q.load(src + L::col(lane, 0)); else q.zero();
      q.unpack(v[p]);
    } else {
#pragma unroll
      for (int j = 0; j < L::kValues; ++j)
        v[p][j] = r < a.rows && col0 + L::col(lane, j) < a.cols ? load1(src + L::col(lane, j)) : 0.0f;
    }
  }

  auto store = [&](uint8_t* codes, int p, const float (&f)[L::kValues]) {
    const int64_t r = row0 + L::row(lane, p);
    if (r >= a.rows) return;
    uint8_t* dst = codes + r * a.cols + col0;
    if constexpr (kVec) {
      if (col_in)
        *reinterpret_cast<uint2*>(dst + L::col(lane, 0)) =
            make_uint2(cvt_fp8x4<kFmt>(v[p][0] * f[0], v[p][1] * f[1], v[p][2] * f[2], v[p][3] * f[3]),
                       cvt_fp8x4<kFmt>(v[p][4] * f[4], v[p][5] * f[5], v[p][6] * f[6], v[p][7] * f[7]));
    } else {
#pragma unroll
      for (int j = 0; j < L::kValues; ++j)
        if (col0 + L::col(lane, j) < a.cols) dst[L::col(lane, j)] = static_cast<uint8_t>(cvt_fp8x2<kFmt>(v[p][j] * f[j], 0.0f) & 0xFFu);
    }
  };

  if constexpr (kRow) {
    const int64_t blocks = a.col_tiles;
#pragma unroll
    for (int p = 0; p < L::kPasses; ++p) {
      uint32_t m = 0u;
#pragma unroll
      for (int j = 0; j < L::kValues; ++j) m = max(m, abs_bits(v[p][j]));
#pragma unroll
      for (int s = 1; s < (kVec ? 16 : 32); s <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, s));
      const uint32_t e = scale_byte<kFmt>(m);
      float f[L::kValues];
#pragma unroll
      for (int j = 0; j < L::kValues; ++j) f[j] = mx8_encode_factor(e);
      store(a.row_codes, p, f);
      const int64_t r = row0 + L::row(lane, p);
      if ((lane & (kVec ? 15 : 31)) == 0 && r < a.rows) a.row_scales[r * blocks + tile_c] = static_cast<uint8_t>(e);
    }
  }
  if constexpr (kCol || kTile) {
    uint32_t m[L::kValues];
#pragma unroll
    for (int j = 0; j < L::kValues; ++j) {
      m[j] = 0u;
#pragma unroll
      for (int p = 0; p < L::kPasses; ++p) m[j] = max(m[j], abs_bits(v[p][j]));
      if (kVec) m[j] = max(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 16));
    }
    if constexpr (kTile) {
      uint32_t all = m[0];
#pragma unroll
      for (int j = 1; j < L::kValues; ++j) all = max(all, m[j]);
      all = __reduce_max_sync(0xFFFFFFFFu, all);
      if (lane == 0) s_max[warp][0] = all;
      __syncthreads();
      all = 0u;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) all = max(all, s_max[w][0]);
      const uint32_t e = scale_byte<kFmt>(all);
      if (threadIdx.x == 0) a.row_scales[tile_r * a.col_tiles + tile_c] = static_cast<uint8_t>(e);
      float f[L::kValues];
#pragma unroll
      for (int j = 0; j < L::kValues; ++j) f[j] = mx8_encode_factor(e);
#pragma unroll
      for (int p = 0; p < L::kPasses; ++p) store(a.row_codes, p, f);
    } else {
      if (!kVec || lane < 16) {
#pragma unroll
        for (int j = 0; j < L::kValues; ++j) s_max[warp][L::col(lane, j)] = m[j];
      }
      __syncthreads();
      float f[L::kValues];
#pragma unroll
      for (int j = 0; j < L::kValues; ++j) {
        uint32_t c = 0u;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) c = max(c, s_max[w][L::col(lane, j)]);
        const uint32_t e = scale_byte<kFmt>(c);
        f[j] = mx8_encode_factor(e);
        if (warp == 0 && (!kVec || lane < 16) && col0 + L::col(lane, j) < a.cols)
          a.col_scales[tile_r * a.cols + col0 + L::col(lane, j)] = static_cast<uint8_t>(e);
      }
#pragma unroll
      for (int p = 0; p < L::kPasses; ++p) store(a.col_codes, p, f);
    }
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

template <typename T, int kFmt, bool kVec>
cudaError_t launch_of(int what, const T* x, const QuantArgs& a, int64_t tiles, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(tiles)), block(kThreads);
  switch (what) {
    case FALQON_ALONG_ROW: return launch_pdl(block_quant_kernel<T, kFmt, kVec, true, false, false>, grid, block, 0, st, 1, x, a);
    case FALQON_ALONG_COL: return launch_pdl(block_quant_kernel<T, kFmt, kVec, false, true, false>, grid, block, 0, st, 1, x, a);
    case FALQON_TILE: return launch_pdl(block_quant_kernel<T, kFmt, kVec, false, false, true>, grid, block, 0, st, 1, x, a);
    default: return launch_pdl(block_quant_kernel<T, kFmt, kVec, true, true, false>, grid, block, 0, st, 1, x, a);
  }
}
constexpr int kBoth = 3;

template <typename T>
int quantize(int what, const void* x, int64_t rows, int64_t cols, int64_t ld, int fmt, uint8_t* row_codes, uint8_t* row_scales,
             uint8_t* col_codes, uint8_t* col_scales, cudaStream_t st) {
  const int64_t tiles = ((rows + kB - 1) / kB) * ((cols + kB - 1) / kB);
  const QuantArgs a{rows, cols, ld, (cols + kB - 1) / kB, row_codes, row_scales, col_codes, col_scales};
  const bool vec = cols % 8 == 0 && (ld * sizeof(T)) % 16 == 0 && aligned_to(x, 16) && aligned_to(row_codes, 8) && aligned_to(col_codes, 8);
  const T* src = static_cast<const T*>(x);
  if (fmt == FALQON_E4M3) return finish(vec ? launch_of<T, 0, true>(what, src, a, tiles, st) : launch_of<T, 0, false>(what, src, a, tiles, st));
  return finish(vec ? launch_of<T, 1, true>(what, src, a, tiles, st) : launch_of<T, 1, false>(what, src, a, tiles, st));
}

int quantize_checked(int what, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int fmt, uint8_t* row_codes,
                     uint8_t* row_scales, uint8_t* col_codes, uint8_t* col_scales, cudaStream_t st) {
  if (x == nullptr || x == row_codes || x == col_codes || !sizes_ok(rows, cols) || ld < cols || ld > (int64_t{1} << 40) || (dtype != FALQON_BF16 && dtype != FALQON_F32) ||
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
