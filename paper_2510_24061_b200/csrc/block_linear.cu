// A few tokens through a layer held in 8 bits by blocks of 128 (include/falqon_dense.h: falqon_block_linear, and the other
// products' forward of few rows):   y[t][i] = sum over kb of 2^(ex[t][kb] + ew[i / 128][kb] - 254) * sum over k in kb of x[t][k] w[i][k]
// Bound by the bytes of w, which are read once, straight into registers: no stage in shared memory, no tile of 256 rows of which a
// few are used.  A CTA takes 16 rows of w; its eight warps share the blocks of K and are added up in order at the end.  A warp
// multiplies a block with mma.sync m16n8k16: codes are exact in fp16 (their scales stay outside), so products are exact and sums
// fp32.  The order of k inside a block is free as long as both operands have the same: a lane's fragments are 16 consecutive
// bytes of a row of w and of a token.
// With up to kMostPlain tokens the CTA quantizes x itself, which saves a launch; every CTA does that work again, so with more
// tokens a quantizer runs first.
#include <type_traits>

#include "../../include/falqon_dense.h"
#include "block_linear.h"
#include "chain_math.cuh"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kRows = 16;                  // of w, a CTA's
constexpr int kAhead = 2;                  // blocks of K whose loads a warp has in flight

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two codes (the low or the high half of a word) as two fp16, exact.
template <int kFmt>
__device__ __forceinline__ uint32_t halves_of(uint32_t w, bool high) {
  uint32_t r;
  const uint16_t c = static_cast<uint16_t>(high ? w >> 16 : w);
  if (kFmt == 0) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(c));
  else           asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(r) : "h"(c));
  return r;
}
// v * 2^(ea + eb - 254), NaN if a byte is 255.  The exponents' sum may leave the range of fp32 where the result does not.
__device__ __forceinline__ float scaled(float v, uint32_t ea, uint32_t eb) {
  const int s = static_cast<int>(ea + eb) - 254, lo = max(min(s, 127), -126), rest = s - lo;
  // rest is -128 .. 127: as a product of two normal powers of two
  const int r0 = rest / 2, r1 = rest - r0;
  auto two_to = [](int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); };
  const float r = rest == 0 ? v * two_to(lo) : v * two_to(lo) * two_to(r0) * two_to(r1);
  return ea == 255u || eb == 255u ? __uint_as_float(0x7FC00000u) : r;
}

struct LinearArgs {
  const uint8_t *w, *w_scales, *x_codes, *x_scales;
  const void* x;
  int T, n, m, blocks;
  void* y;
  bool bf16;
};

// A lane's part of a block of w: 16 bytes of rows g and g + 8 in each half of the block; and of the tokens' codes.
template <int kTiles>
struct Part {
  uint4 w[2][2];       // [half][row g, row g + 8]
  uint4 x[kTiles][2];  // [tile of eight tokens][half]
  uint32_t ew, ex[kTiles][2];
};

template <int kTiles, int kWFmt, int kXFmt, typename X>   // X: uint8_t for codes, else the type of x
__global__ void __launch_bounds__(kThreads)
block_linear_kernel(const LinearArgs p) {
  constexpr bool kPlain = !std::is_same<X, uint8_t>::value;
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int row0 = blockIdx.x * kRows;
  pdl_trigger();
  pdl_wait();

  const int mine = (p.blocks - warp + kWarps - 1) / kWarps;      // blocks warp, warp + 8, ..
  // kPlain: this warp's codes [mine][T][128] and their scale bytes
  const int most = (p.blocks + kWarps - 1) / kWarps;
  uint8_t* codes = smem + static_cast<size_t>(warp) * most * p.T * (FALQON_BLOCK + 16);
  uint8_t* bytes = codes + static_cast<size_t>(most) * p.T * FALQON_BLOCK;

  const uint8_t* w0 = p.w + static_cast<int64_t>(row0 + g) * p.n + 16 * t;
  const uint8_t* w1 = w0 + static_cast<int64_t>(8) * p.n;
  const uint8_t* ws = p.w_scales + static_cast<int64_t>(row0 >> 7) * p.blocks;

  Part<kTiles> part[kAhead];
  auto fetch = [&](Part<kTiles>& q, int i) {
    const int kb = warp + i * kWarps, k0 = kb * FALQON_BLOCK;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + 64 * h + 16 * t;
      const bool in = k < p.n;                 // n is a multiple of 16: all inside or all outside
      q.w[h][0] = in ? ld_stream(reinterpret_cast<const uint4*>(w0 + k0 + 64 * h)) : make_uint4(0u, 0u, 0u, 0u);
      q.w[h][1] = in ? ld_stream(reinterpret_cast<const uint4*>(w1 + k0 + 64 * h)) : make_uint4(0u, 0u, 0u, 0u);
      if constexpr (!kPlain) {
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          const int tok = 8 * j + g;
          q.x[j][h] = in && tok < p.T ? ld_stream(reinterpret_cast<const uint4*>(p.x_codes + static_cast<int64_t>(tok) * p.n + k)) : make_uint4(0u, 0u, 0u, 0u);
        }
      }
    }
    q.ew = ld_stream(ws + kb);
    if constexpr (!kPlain) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int tok = 8 * j + 2 * t + c;   // the tokens of this lane's sums
          q.ex[j][c] = tok < p.T ? ld_stream(p.x_scales + static_cast<int64_t>(tok) * p.blocks + kb) : 0u;
        }
    }
  };
#pragma unroll
  for (int a = 0; a < kAhead; ++a)
    if (a < mine) fetch(part[a], a);

  if constexpr (kPlain) {       // while those are on their way
    for (int u = 0; u < mine * p.T; ++u) {
      const int i = u / p.T, tok = u - i * p.T, k = (warp + i * kWarps) * FALQON_BLOCK + 4 * lane;
      float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (k < p.n) {
        const X* src = static_cast<const X*>(p.x) + static_cast<int64_t>(tok) * p.n + k;
        if constexpr (std::is_same<X, float>::value) {
          const float4 f = ld_stream(reinterpret_cast<const float4*>(src));
          v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
        } else {
          const uint2 b = ld_stream(reinterpret_cast<const uint2*>(src));
          v[0] = __uint_as_float(b.x << 16), v[1] = __uint_as_float(b.x & 0xFFFF0000u);
          v[2] = __uint_as_float(b.y << 16), v[3] = __uint_as_float(b.y & 0xFFFF0000u);
        }
      }
      const uint32_t e = mx8_exponent(__reduce_max_sync(0xFFFFFFFFu, max(max(abs_bits(v[0]), abs_bits(v[1])), max(abs_bits(v[2]), abs_bits(v[3])))));
      const float f = mx8_encode_factor(e);
      *reinterpret_cast<uint32_t*>(codes + static_cast<size_t>(u) * FALQON_BLOCK + 4 * lane) = cvt_fp8x4<0>(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
      if (lane == 0) bytes[u] = static_cast<uint8_t>(e);
    }
    __syncwarp();
  }

  float sum[kTiles][4] = {};
  auto multiply = [&](Part<kTiles>& q, int i) {
    if constexpr (kPlain) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        q.x[0][h] = g < p.T ? *reinterpret_cast<const uint4*>(codes + static_cast<size_t>(i * p.T + g) * FALQON_BLOCK + 64 * h + 16 * t) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int c = 0; c < 2; ++c) q.ex[0][c] = 2 * t + c < p.T ? bytes[i * p.T + 2 * t + c] : 0u;
    }
    float acc[kTiles][4] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t r0[4] = {q.w[h][0].x, q.w[h][0].y, q.w[h][0].z, q.w[h][0].w};
      const uint32_t r1[4] = {q.w[h][1].x, q.w[h][1].y, q.w[h][1].z, q.w[h][1].w};
#pragma unroll
      for (int s = 0; s < 4; ++s) {     // four codes of each row and token a step
        const uint32_t a0 = halves_of<kWFmt>(r0[s], false), a2 = halves_of<kWFmt>(r0[s], true);
        const uint32_t a1 = halves_of<kWFmt>(r1[s], false), a3 = halves_of<kWFmt>(r1[s], true);
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          const uint32_t xw = s == 0 ? q.x[j][h].x : s == 1 ? q.x[j][h].y : s == 2 ? q.x[j][h].z : q.x[j][h].w;
          mma_f16(acc[j], a0, a1, a2, a3, halves_of<kXFmt>(xw, false), halves_of<kXFmt>(xw, true));
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) sum[j][c] += scaled(acc[j][c], q.ew, q.ex[j][c & 1]);
  };
  for (int i0 = 0; i0 < mine; i0 += kAhead) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int i = i0 + a;
      if (i < mine) {
        multiply(part[a], i);
        if (i + kAhead < mine) fetch(part[a], i + kAhead);
      }
    }
  }

  // the warps' sums, in order; row g (+ 8), tokens 2 t, 2 t + 1 of each tile
  __syncthreads();       // the codes have been read
  constexpr int kPitch = kRows + 1;
  float* red = reinterpret_cast<float*>(smem) + static_cast<size_t>(warp) * kTiles * 8 * kPitch;
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    red[(8 * j + 2 * t) * kPitch + g] = sum[j][0];
    red[(8 * j + 2 * t + 1) * kPitch + g] = sum[j][1];
    red[(8 * j + 2 * t) * kPitch + g + 8] = sum[j][2];
    red[(8 * j + 2 * t + 1) * kPitch + g + 8] = sum[j][3];
  }
  __syncthreads();
  for (int o = threadIdx.x; o < p.T * kRows; o += kThreads) {
    const int tok = o / kRows, r = o - tok * kRows;
    const float* all = reinterpret_cast<const float*>(smem) + tok * kPitch + r;
    float v = all[0];
#pragma unroll
    for (int wi = 1; wi < kWarps; ++wi) v += all[static_cast<size_t>(wi) * kTiles * 8 * kPitch];
    const int64_t at = static_cast<int64_t>(tok) * p.m + row0 + r;
    if (p.bf16) store1(static_cast<bf16_t*>(p.y) + at, v);
    else store1(static_cast<float*>(p.y) + at, v);
  }
}

template <int kTiles, int kWFmt, int kXFmt, typename X>
cudaError_t launch_of(const LinearArgs& a, cudaStream_t st) {
  const size_t sums = static_cast<size_t>(kWarps) * kTiles * 8 * (kRows + 1) * 4;
  size_t smem = sums;
  if (!std::is_same<X, uint8_t>::value) {
    const size_t codes = static_cast<size_t>(kWarps) * ((a.blocks + kWarps - 1) / kWarps) * a.T * (FALQON_BLOCK + 16);
    if (codes > smem) smem = codes;
  }
  static DeviceMask configured{0};
  const cudaError_t e = set_max_dynamic_smem(block_linear_kernel<kTiles, kWFmt, kXFmt, X>, 200 * 1024, configured);
  if (e != cudaSuccess) return e;
  return launch_pdl(block_linear_kernel<kTiles, kWFmt, kXFmt, X>, dim3(static_cast<unsigned>(a.m / kRows)), dim3(kThreads), smem, st, 1, a);
}
template <int kTiles, int kWFmt>
cudaError_t launch_codes(const LinearArgs& a, int x_fmt, cudaStream_t st) {
  return x_fmt == FALQON_E4M3 ? launch_of<kTiles, kWFmt, 0, uint8_t>(a, st) : launch_of<kTiles, kWFmt, 1, uint8_t>(a, st);
}
template <int kWFmt>
cudaError_t launch_tiles(const LinearArgs& a, int x_fmt, cudaStream_t st) {
  return a.T <= 8 ? launch_codes<1, kWFmt>(a, x_fmt, st) : a.T <= 16 ? launch_codes<2, kWFmt>(a, x_fmt, st) : launch_codes<4, kWFmt>(a, x_fmt, st);
}

}  // namespace

bool block_linear_plain(int64_t T, int64_t n) { return T <= kMostPlain && T * ((n + 127) / 128 + kWarps) * (FALQON_BLOCK + 16) <= 200 * 1024; }

cudaError_t launch_block_linear_codes(const uint8_t* x, const uint8_t* xs, int x_fmt, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T,
                                      int64_t n, int64_t m, void* y, bool bf16, cudaStream_t st) {
  const LinearArgs a{w, ws, x, xs, nullptr, static_cast<int>(T), static_cast<int>(n), static_cast<int>(m), static_cast<int>((n + 127) / 128), y, bf16};
  return w_fmt == FALQON_E4M3 ? launch_tiles<0>(a, x_fmt, st) : launch_tiles<1>(a, x_fmt, st);
}
cudaError_t launch_block_linear_plain(const void* x, bool x_bf16, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T, int64_t n, int64_t m,
                                      void* y, bool bf16, cudaStream_t st) {
  const LinearArgs a{w, ws, nullptr, nullptr, x, static_cast<int>(T), static_cast<int>(n), static_cast<int>(m), static_cast<int>((n + 127) / 128), y, bf16};
  if (w_fmt == FALQON_E4M3) return x_bf16 ? launch_of<1, 0, 0, bf16_t>(a, st) : launch_of<1, 0, 0, float>(a, st);
  return x_bf16 ? launch_of<1, 1, 0, bf16_t>(a, st) : launch_of<1, 1, 0, float>(a, st);
}

}  // namespace falqon
