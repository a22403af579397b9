// One or two tokens, and up to kMostFew where w has at most 2^25 weights, through a layer held in 8 bits by blocks of 128
// (include/falqon_dense.h: falqon_block_linear, and falqon_block_forward of so few rows):
//   y[t][i] = sum over blocks kb of 2^(ex[t][kb] + ew[i / 128][kb] - 254) * sum over k in kb of x[t][k] w[i][k]
// Bound by the bytes of w, which are read once, straight into registers: no stage in shared memory, no tile of 256 rows of which a few are
// used.  A warp reads 512 codes of a row at a time (whole lines), a lane 16 of them, all of one block; codes are multiplied as fp16
// (products exact) into fp32 sums, the scales stay outside of a lane's 16.  Some warps of a CTA share the contraction, each with its own part of x;
// CTAs walk over the rows, two units of kRows x 512 codes on their way.  x is quantized by every warp for its own part, which is
// read once per CTA.  4096 -> 11008, bf16: one token 11.4 us (4.0 TB/s; the loads alone 8.9), two 15.0; the tensor cores' tiles with a
// quantizer before them 18.6 to 20 us from three tokens up to 130.  4096 -> 4096: one token 5.5, two 7.4, four 10.9 us (bound by the
// multiplications), theirs 13 to 15.  (By mma.sync m16n8k16, whose rate is low here, with 16 rows and all of x to a CTA: one token 15.8, four 27.7.)
#include <type_traits>

#include "../../include/falqon_dense.h"
#include "block_linear.h"
#include "chain_math.cuh"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kChunk = 512;                // codes of a row that a warp reads at once
constexpr int kMostWarps = 8;

struct LinearArgs {
  const uint8_t *w, *w_scales, *x_codes, *x_scales;
  const void* x;
  int T, n, m, blocks;
  void* y;
  bool bf16;
  // kw warps share the contraction, `rounds` chunks each; rw groups of them take rows of their own; the CTA walks `turns` times
  int kw, rw, rounds, turns;
};

// 16 codes as fp16, exact.
template <int kFmt>
__device__ __forceinline__ void decode16(const uint4& q, uint32_t (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (kFmt == 0)
      asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(v[2 * i]), "=r"(v[2 * i + 1]) : "r"(w[i]));
    else
      asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e5m2x2 %0, a;\n\tcvt.rn.f16x2.e5m2x2 %1, b;\n\t}" : "=r"(v[2 * i]), "=r"(v[2 * i + 1]) : "r"(w[i]));
  }
}
// acc + a.lo * b.lo, acc2 + a.hi * b.hi: fp16 factors, their product exact, fp32 sums
__device__ __forceinline__ void fma_halves(float& acc, float& acc2, uint32_t a, uint32_t b) {
  asm("{\n\t.reg .f16 al, ah, bl, bh;\n\tmov.b32 {al, ah}, %2;\n\tmov.b32 {bl, bh}, %3;\n\t"
      "fma.rn.f32.f16 %0, al, bl, %0;\n\tfma.rn.f32.f16 %1, ah, bh, %1;\n\t}" : "+f"(acc), "+f"(acc2) : "r"(a), "r"(b));
}

// 2^(ea + eb - 254) as a product of two: the sum of the exponents may leave the range of fp32 where the result does not.  NaN if a byte is 255.
__device__ __forceinline__ void factors(uint32_t ea, uint32_t eb, float& f, float& g) {
  const int s = static_cast<int>(ea + eb) - 254, half = s / 2, rest = s - half;       // -127 .. 127 each
  auto two_to = [](int e) { return __uint_as_float(e <= -127 ? 0x00400000u : static_cast<uint32_t>(e + 127) << 23); };
  f = ea == 255u || eb == 255u ? __uint_as_float(0x7FC00000u) : two_to(half);
  g = two_to(rest);
}

template <typename X>
__device__ __forceinline__ void load16(const X* p, bool in, float (&v)[16]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    Vec8<X> q;
    if (in) q.load(p + 8 * h); else q.zero();
    float u[8];
    q.unpack(u);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[8 * h + j] = u[j];
  }
}

// kT: tokens, filled up with zeros.  X: uint8_t where x comes as codes, else its type.
template <int kT, int kWFmt, int kXFmt, typename X>
__global__ void __launch_bounds__(32 * kMostWarps, 2)
block_linear_kernel(const LinearArgs p) {
  constexpr int kRows = kT <= 2 ? 8 : 4;         // of a unit
  constexpr int kAhead = 2;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float s_sum[2][kMostWarps][kRows * kT];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kwi = warp % p.kw, rwi = warp / p.kw;
  const int row_units = p.m / kRows;

  // unit u of this warp: turn u / rounds, round u % rounds
  struct Unit { uint4 w[kRows]; uint32_t ew; };
  auto fetch = [&](Unit& q, int turn, int round) {
    const int at = (turn * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x)) * p.rw + rwi;
    const int k = (kwi + round * p.kw) * kChunk + 16 * lane;
    const bool in = at < row_units && k < p.n;   // n is a multiple of 16
    const int64_t row = static_cast<int64_t>(at) * kRows;
    const uint8_t* src = p.w + row * p.n + k;
#pragma unroll
    for (int r = 0; r < kRows; ++r) q.w[r] = in ? ld_stream(reinterpret_cast<const uint4*>(src + static_cast<int64_t>(r) * p.n)) : make_uint4(0u, 0u, 0u, 0u);
    q.ew = in ? ld_stream(p.w_scales + (row >> 7) * p.blocks + (k >> 7)) : 0u;
  };
  const int units = p.turns * p.rounds;
  Unit unit[kAhead];
  int f_turn = 0, f_round = 0;
  auto fetch_next = [&](Unit& q) {
    if (f_turn >= p.turns) return;
    fetch(q, f_turn, f_round);
    if (++f_round == p.rounds) f_round = 0, ++f_turn;
  };
#pragma unroll
  for (int a = 0; a < kAhead; ++a) fetch_next(unit[a]);

  // this warp's part of x, while those are on their way: codes [rounds][kT][512], and a scale byte per lane [rounds][kT][32]
  uint8_t* codes = smem + static_cast<size_t>(warp) * p.rounds * kT * (kChunk + 32);
  uint8_t* bytes = codes + static_cast<size_t>(p.rounds) * kT * kChunk;
  for (int round = 0; round < p.rounds; ++round) {
    const int k = (kwi + round * p.kw) * kChunk + 16 * lane;
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      const bool in = t < p.T && k < p.n;
      uint4 c = make_uint4(0u, 0u, 0u, 0u);
      uint32_t e = 0u;
      if constexpr (std::is_same<X, uint8_t>::value) {
        if (in) {
          c = ld_stream(reinterpret_cast<const uint4*>(p.x_codes + static_cast<int64_t>(t) * p.n + k));
          e = ld_stream(p.x_scales + static_cast<int64_t>(t) * p.blocks + (k >> 7));
        }
      } else {
        float v[16];
        load16(static_cast<const X*>(p.x) + static_cast<int64_t>(t) * p.n + k, in, v);
        uint32_t m = 0u;
#pragma unroll
        for (int j = 0; j < 16; ++j) m = max(m, abs_bits(v[j]));
#pragma unroll
        for (int s = 1; s < 8; s <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, s));     // eight lanes to a block
        e = mx8_exponent(m);
        const float f = mx8_encode_factor(e);
        c = make_uint4(cvt_fp8x4<0>(v[0] * f, v[1] * f, v[2] * f, v[3] * f), cvt_fp8x4<0>(v[4] * f, v[5] * f, v[6] * f, v[7] * f),
                       cvt_fp8x4<0>(v[8] * f, v[9] * f, v[10] * f, v[11] * f), cvt_fp8x4<0>(v[12] * f, v[13] * f, v[14] * f, v[15] * f));
      }
      reinterpret_cast<uint4*>(codes + static_cast<size_t>(round * kT + t) * kChunk)[lane] = c;
      bytes[(round * kT + t) * 32 + lane] = static_cast<uint8_t>(e);
    }
  }
  __syncwarp();

  float part[kT][kRows];
  auto multiply = [&](const Unit& q, int round) {
    uint32_t x[kT][8];
    float f[kT], g[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      decode16<kXFmt>(reinterpret_cast<const uint4*>(codes + static_cast<size_t>(round * kT + t) * kChunk)[lane], x[t]);
      factors(q.ew, bytes[(round * kT + t) * 32 + lane], f[t], g[t]);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      uint32_t w[8];
      decode16<kWFmt>(q.w[r], w);
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) fma_halves(a, b, w[j], x[t][j]);
        const float d = (a + b) * f[t];
        part[t][r] = round == 0 ? d * g[t] : fmaf(d, g[t], part[t][r]);
      }
    }
  };
  // The rows' sums over the lanes, by halves: a lane ends up with row (lane / (32 / kRows)); then over the warps, in order.
  auto finish = [&](int turn) {
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      float v[kRows];
#pragma unroll
      for (int r = 0; r < kRows; ++r) v[r] = part[t][r];
#pragma unroll
      for (int s = 16, left = kRows; s > 0; s >>= 1) {
        if (left > 1) {
          left >>= 1;
#pragma unroll
          for (int r = 0; r < left; ++r) {
            const bool up = (lane & s) != 0;
            const float send = up ? v[r] : v[r + left], keep = up ? v[r + left] : v[r];
            v[r] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, s);
          }
        } else {
          v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], s);
        }
      }
      if ((lane & (32 / kRows - 1)) == 0) s_sum[turn & 1][warp][t * kRows + lane / (32 / kRows)] = v[0];
    }
    __syncthreads();       // (the buffer of the turn before last has been read by everybody: they have passed the last turn's)
    const int o = threadIdx.x, rg = o / (kRows * kT), in = o - rg * kRows * kT, t = in / kRows, r = in - t * kRows;
    const int at = (turn * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x)) * p.rw + rg;
    if (rg < p.rw && t < p.T && at < row_units) {
      float v = s_sum[turn & 1][rg * p.kw][in];
      for (int w = 1; w < p.kw; ++w) v += s_sum[turn & 1][rg * p.kw + w][in];
      const int64_t to = static_cast<int64_t>(t) * p.m + static_cast<int64_t>(at) * kRows + r;
      if (p.bf16) store1(static_cast<bf16_t*>(p.y) + to, v);
      else store1(static_cast<float*>(p.y) + to, v);
    }
  };
  int turn = 0, round = 0;
  for (int u0 = 0; u0 < units; u0 += kAhead) {
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      if (u0 + a >= units) break;
      multiply(unit[a], round);
      fetch_next(unit[a]);
      if (++round == p.rounds) {
        finish(turn);
        round = 0, ++turn;
      }
    }
  }
}

struct Split { int kw, rw, rounds; };
// Warps of a CTA: where they share the contraction, so many that the last round is as full as possible.
Split split_of(int64_t n) {
  const int chunks = static_cast<int>((n + kChunk - 1) / kChunk);
  if (chunks <= 4) return {chunks, kMostWarps / chunks, 1};
  int best = kMostWarps;
  for (int kw = kMostWarps - 1; kw >= 5; --kw)
    if ((chunks + kw - 1) / kw * kw < (chunks + best - 1) / best * best) best = kw;
  return {best, 1, (chunks + best - 1) / best};
}
int tokens_of(int64_t T) { return T <= 1 ? 1 : T <= 2 ? 2 : 4; }
size_t smem_of(const Split& s, int tokens) { return static_cast<size_t>(s.kw * s.rw) * s.rounds * tokens * (kChunk + 32); }
constexpr size_t kMostSmem = 100 * 1024;     // two CTAs to an SM

template <int kT, int kWFmt, int kXFmt, typename X>
cudaError_t launch_of(LinearArgs a, cudaStream_t st) {
  const Split s = split_of(a.n);
  const int warps = s.kw * s.rw, groups = (a.m / (kT <= 2 ? 8 : 4) + s.rw - 1) / s.rw, most = sm_count() * (2 * kMostWarps / warps);
  a.kw = s.kw, a.rw = s.rw, a.rounds = s.rounds;
  const int grid0 = groups < most ? groups : most;
  a.turns = (groups + grid0 - 1) / grid0;
  const int grid = (groups + a.turns - 1) / a.turns;     // as even as turns allow
  static DeviceMask configured{0};
  const cudaError_t e = set_max_dynamic_smem(block_linear_kernel<kT, kWFmt, kXFmt, X>, static_cast<int>(kMostSmem), configured);
  if (e != cudaSuccess) return e;
  return launch_pdl(block_linear_kernel<kT, kWFmt, kXFmt, X>, dim3(static_cast<unsigned>(grid)), dim3(static_cast<unsigned>(32 * warps)),
                    smem_of(s, kT), st, 1, a);
}
template <int kWFmt, int kXFmt, typename X>
cudaError_t launch_tokens(const LinearArgs& a, cudaStream_t st) {
  switch (tokens_of(a.T)) {
    case 1: return launch_of<1, kWFmt, kXFmt, X>(a, st);
    case 2: return launch_of<2, kWFmt, kXFmt, X>(a, st);
    default: return launch_of<4, kWFmt, kXFmt, X>(a, st);
  }
}

}  // namespace

bool block_linear_takes(int64_t T, int64_t n, int64_t m) {
  // Three and four tokens: as long as the multiplications, which go with n m, are hidden by what the other way takes anyway (16.8 million
  // weights 10.9 us here, 13 to 15 there; 45 million 23.2 and 18.6).
  return T <= (n * m <= (int64_t{1} << 25) ? kMostFew : 2) && smem_of(split_of(n), tokens_of(T)) <= kMostSmem;
}

cudaError_t launch_block_linear_codes(const uint8_t* x, const uint8_t* xs, int x_fmt, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T,
                                      int64_t n, int64_t m, void* y, bool bf16, cudaStream_t st) {
  const LinearArgs a{w, ws, x, xs, nullptr, static_cast<int>(T), static_cast<int>(n), static_cast<int>(m), static_cast<int>((n + 127) / 128), y, bf16, 0, 0, 0, 0};
  if (w_fmt == FALQON_E4M3) return x_fmt == FALQON_E4M3 ? launch_tokens<0, 0, uint8_t>(a, st) : launch_tokens<0, 1, uint8_t>(a, st);
  return x_fmt == FALQON_E4M3 ? launch_tokens<1, 0, uint8_t>(a, st) : launch_tokens<1, 1, uint8_t>(a, st);
}
cudaError_t launch_block_linear_plain(const void* x, bool x_bf16, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T, int64_t n, int64_t m,
                                      void* y, bool bf16, cudaStream_t st) {
  const LinearArgs a{w, ws, nullptr, nullptr, x, static_cast<int>(T), static_cast<int>(n), static_cast<int>(m), static_cast<int>((n + 127) / 128), y, bf16, 0, 0, 0, 0};
  if (w_fmt == FALQON_E4M3) return x_bf16 ? launch_tokens<0, 0, bf16_t>(a, st) : launch_tokens<0, 0, float>(a, st);
  return x_bf16 ? launch_tokens<1, 0, bf16_t>(a, st) : launch_tokens<1, 0, float>(a, st);
}

}  // namespace falqon
