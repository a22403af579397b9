// An update orthogonalised by Newton-Schulz products (include/falqon_dense.h):
//   X = g / (|g|_F + eps);  steps times:  G = X X^T,  B = b G + c G G,  X <- a X + B X     (from the short side, s x s)
// Bound by the tensor cores: per step s^2 l (G, of which half is computed: it is symmetric) + s^3 (G G, half) + 2 s^2 l operations.
//
// Numbers.  The singular values of X start as small as they like beside its norm and grow by a = 3.4 a step, noise in X with them: held in
// bf16, results are 1 to 30 % off.  So X, and with it the term a X, is two fp16 numbers hi + lo (22 bits).  The products' operands are
// the hi parts alone where results are bf16 (errors of 2^-12 of G and B; results 1.7e-3 to 2.4e-3 off, of which 1.66e-3 are their own
// rounding; short sides up to 96 have the last of a step's products in full), and three products hi hi + hi lo + lo hi where they are
// fp32.  All stored values are 2^13 times what they stand for: the host has made sure that none passes 7.98, and small ones keep their
// digits above fp16's smallest.  Where |g| is below eps / 2, X is small
// altogether and only grows by the first coefficient a step: X and B are then held 2^x and 2^b times as large, by exponents of each matrix and step
// that ortho_scale_kernel derives from |g| / (|g| + eps) (1024 x 1024 at 1e-7 of eps: results 2 % off without them).
//
// One kernel does the three products: 256 x block_n tiles by CTA pairs (tcgen05.mma kind::f16, cta_group::2), operands K-major or MN-major
// by TMA, so that tall matrices need no transposed copy; its epilogue is out = alpha D + beta C, written as hi and lo, as the result, or
// (few tiles, a long contraction: split over CTAs) as fp32 parts that a small kernel adds up in order.
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "../../include/falqon_dense.h"
#include "gemm_common.cuh"
#include "internal.h"
#include "mx8.cuh"
#include "ortho_thin.h"
#include "ptx.cuh"
#include "tile_walk.cuh"

namespace falqon {
namespace {

constexpr float kScale = 8192.0f;            // 2^13
constexpr int kKBlock = 64;                  // fp16 values of K in a stage: 128 bytes
constexpr uint32_t kHalfChunk = 64 * 128;    // 64 rows of 64 values: an MN-major chunk
// A stage: 128 rows of A and block_n / 2 of B; with kPrecise the lo parts of both, too, and tiles half as wide at the most.
constexpr int kMostStages = 6;
template <bool kPrecise>
struct Stage {
  static constexpr int kCount = kPrecise ? 4 : kMostStages;
  static constexpr uint32_t kBytes = (kPrecise ? 48 : 32) * 1024;
  static constexpr uint32_t kB = (kPrecise ? 2 : 1) * kATileBytes;      // B hi; A hi at 0, A lo behind it
  static constexpr uint32_t kBLo = kB + kATileBytes / 2;
};
constexpr uint32_t kStagingOff = 6 * 32 * 1024;
constexpr uint32_t kBarsOff = kStagingOff + kStagingBytes;
constexpr uint32_t kSmem = kBarsOff + 256 + 1024;

enum Mode { kHiLo, kFinal, kPart };
enum Product { kGram, kSquare, kApply };     // G = X X^T, B = b G + c G G, X <- a X + B X

// Powers of two that a matrix's X before a step (x) and B of the step (b) are held with, beside kScale: [batch][steps].
struct Exponents { int x, b; };
constexpr int kMostX = 126, kMostB = 2 * kMostX;

struct ProductArgs {
  int M, N, batch;
  int kblocks;                 // blocks of K
  int splits, per_split;       // CTAs that share the blocks of a tile
  int m_tiles, tiles;          // tiles of a matrix
  TileWalk walk;               // over all tiles of all matrices and splits
  bool symmetric;              // only tiles that touch the upper triangle; the lower one is their mirror
  bool a_mn, b_mn;
  uint32_t idesc;              // without N
  Product product;
  float alpha, beta;           // before exponents
  int post;                    // kFinal: the scale's power of two, which is taken last, so that a small scale costs alpha no digits
  const Exponents* exps;       // of this step, matrices `steps` apart
  int steps;
  const __half *c_hi, *c_lo;   // [batch][M][ld_c]; c_lo nullable, both null: no such term
  int64_t ld_c, stride_c;
  Mode mode;
  __half *o_hi, *o_lo;         // kHiLo, o_lo nullable
  int64_t ld_o, stride_o;
  void* out;                   // kFinal: [batch][M][N]
  bool out_bf16, out_vec;
  float* parts;                // kPart: [batch][splits][M][ld_o]
  int* status;
};

struct Maps { CUtensorMap a_hi, a_lo, b_hi, b_lo; };

// Tile `t` of a symmetric product: columns by columns, the row tiles that do not lie wholly below the diagonal.
__device__ __forceinline__ void locate(const ProductArgs& p, int t, int& m_idx, int& n_idx) {
  if (!p.symmetric) {
    n_idx = t / p.m_tiles;
    m_idx = t - n_idx * p.m_tiles;
    return;
  }
  n_idx = 0;
  for (;; ++n_idx) {
    const int rows = min(p.m_tiles, ((n_idx + 1) * p.walk.block_n + 255) / 256);
    if (t < rows) break;
    t -= rows;
  }
  m_idx = t;
}

struct Item {       // a piece of work: columns of a tile of a matrix (none: behind the right edge), and the part of its contraction
  int b, split, row0, n0, width, k_begin, k_end;
  __device__ __forceinline__ Item(const ProductArgs& p, int item) {
    int first;
    const int t = walk_tile(p.walk, item, &first, &width), per_matrix = p.tiles * p.splits;
    b = t / per_matrix;
    const int rest = t - b * per_matrix;
    split = rest / p.tiles;
    int m_idx, n_idx;
    locate(p, rest - split * p.tiles, m_idx, n_idx);
    row0 = m_idx * 256;
    n0 = n_idx * p.walk.block_n + first;
    width = n0 < p.N ? min(width, (p.N - n0 + 31) / 32 * 32) : 0;
    k_begin = split * p.per_split;
    k_end = min(p.kblocks, k_begin + p.per_split);
  }
};

__device__ __forceinline__ Exponents exponents_at(const Exponents* p) {
  const int2 v = ld_stream(reinterpret_cast<const int2*>(p));
  return Exponents{v.x, v.y};
}
// What D, C and a final result of matrix b are multiplied by.
struct Factors { float alpha, beta, post; };
__device__ __forceinline__ Factors factors_of(const ProductArgs& p, int b) {
  Factors f{p.alpha, p.beta, 1.0f};
  if (p.product == kGram) return f;
  const Exponents* at = p.exps + static_cast<int64_t>(b) * p.steps;
  const Exponents e = exponents_at(at);
  if (p.product == kSquare) {
    if ((e.x | e.b) != 0) f.alpha = ldexpf(f.alpha, e.b - 4 * e.x), f.beta = ldexpf(f.beta, e.b - 2 * e.x);
    return f;
  }
  const int up = p.mode == kFinal ? 0 : exponents_at(at + 1).x - e.x;
  if ((up | e.b) != 0) f.alpha = ldexpf(f.alpha, up - e.b), f.beta = ldexpf(f.beta, up);
  if (p.mode == kFinal) f.post = ldexpf(1.0f, p.post - e.x);
  return f;
}

__device__ __forceinline__ void store_hi_lo(__half* hi, __half* lo, const float (&v)[4]) {      // lo: nullable
  __half2 h0 = __floats2half2_rn(v[0], v[1]), h1 = __floats2half2_rn(v[2], v[3]);
  uint2 u;
  u.x = *reinterpret_cast<uint32_t*>(&h0), u.y = *reinterpret_cast<uint32_t*>(&h1);
  *reinterpret_cast<uint2*>(hi) = u;
  if (lo != nullptr) {
    const float2 f0 = __half22float2(h0), f1 = __half22float2(h1);
    h0 = __floats2half2_rn(v[0] - f0.x, v[1] - f0.y), h1 = __floats2half2_rn(v[2] - f1.x, v[3] - f1.y);
    u.x = *reinterpret_cast<uint32_t*>(&h0), u.y = *reinterpret_cast<uint32_t*>(&h1);
    *reinterpret_cast<uint2*>(lo) = u;
  }
}
__device__ __forceinline__ void add_halves(float (&v)[4], const uint2& u, float f) {
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&u.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&u.y));
  v[0] = fmaf(a.x, f, v[0]), v[1] = fmaf(a.y, f, v[1]), v[2] = fmaf(b.x, f, v[2]), v[3] = fmaf(b.y, f, v[3]);
}

// A warp's staging buffer: 32 rows of 32 fp32, 16-byte pieces swizzled so that neither rows, nor four rows by eight pieces, nor
// columns (eight groups of four rows) meet in a bank.
__device__ __forceinline__ int staged(int row, int col) { return row * 32 + ((((col >> 2) ^ row ^ (row >> 2)) & 7) << 2) + (col & 3); }

// 32 x 32 values of D at (row0, col0), one row a lane, through the staging buffer to where they belong: a lane then holds four columns of a
// row, eight lanes a row, so that C is read and results are written in whole sectors.
__device__ __forceinline__ void finish_chunk(const ProductArgs& p, const Item& it, const Factors& f, int row0, int col0, const float (&d)[32], float* stage) {
  if (row0 >= p.M || col0 >= p.N) return;
  if (p.symmetric && col0 < row0) return;           // the mirror of what another chunk writes
  const int lane = threadIdx.x & 31, sub = lane >> 3, col = (lane & 7) * 4;
  const bool diagonal = p.symmetric && row0 == col0, mirror = p.symmetric && !diagonal && p.mode == kHiLo;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *reinterpret_cast<float4*>(stage + staged(lane, 4 * j)) = make_float4(d[4 * j], d[4 * j + 1], d[4 * j + 2], d[4 * j + 3]);
  // rows 4 i + sub that there are, of this lane's columns
  const int rows = col0 + col < p.N ? min(32, p.M - row0) - sub : 0;
  uint2 ch[8], cl[8];
  const bool with_c = p.c_hi != nullptr, with_lo = p.c_lo != nullptr;
  {
    const int64_t at = it.b * p.stride_c + (row0 + sub) * p.ld_c + col0 + col, step = 4 * p.ld_c;
    const __half *hi = p.c_hi + at, *lo = p.c_lo + at;
    const int hi_rows = with_c ? rows : 0, lo_rows = with_lo ? rows : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i, hi += step, lo += step) {
      ch[i] = 4 * i < hi_rows ? ld_stream(reinterpret_cast<const uint2*>(hi)) : make_uint2(0u, 0u);
      cl[i] = 4 * i < lo_rows ? ld_stream(reinterpret_cast<const uint2*>(lo)) : make_uint2(0u, 0u);
    }
  }
  __syncwarp();
  // alpha D + beta C of this lane's four columns of row 4 i + sub
  auto value = [&](int i, float (&v)[4]) {
    const int rl = 4 * i + sub;
    if (diagonal) {     // the upper triangle's value on both sides
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = stage[staged(min(rl, col + k), max(rl, col + k))];
    } else {
      const float4 q = *reinterpret_cast<const float4*>(stage + staged(rl, col));
      v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] *= f.alpha;
    if (with_lo) add_halves(v, cl[i], f.beta);
    if (with_c) add_halves(v, ch[i], f.beta);
    if (mirror) *reinterpret_cast<float4*>(stage + staged(rl, col)) = make_float4(v[0], v[1], v[2], v[3]);
  };
  float v[4];
  if (p.mode == kHiLo) {
    const int64_t at = it.b * p.stride_o + (row0 + sub) * p.ld_o + col0 + col, step = 4 * p.ld_o;
    __half *hi = p.o_hi + at, *lo = p.o_lo != nullptr ? p.o_lo + at : nullptr;
#pragma unroll
    for (int i = 0; i < 8; ++i, hi += step) {
      value(i, v);
      if (4 * i < rows) store_hi_lo(hi, lo, v);
      if (lo != nullptr) lo += step;
    }
  } else if (p.mode == kPart) {
    float* to = p.parts + ((static_cast<int64_t>(it.b) * p.splits + it.split) * p.M + row0 + sub) * p.ld_o + col0 + col;
    const int64_t step = 4 * p.ld_o;
#pragma unroll
    for (int i = 0; i < 8; ++i, to += step) {
      value(i, v);
      if (4 * i < rows) *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
    }
  } else if (p.out_vec) {
    const int64_t at = (static_cast<int64_t>(it.b) * p.M + row0 + sub) * p.N + col0 + col, step = 4 * static_cast<int64_t>(p.N);
    uint16_t* half = static_cast<uint16_t*>(p.out) + at;
    float* full = static_cast<float*>(p.out) + at;
#pragma unroll
    for (int i = 0; i < 8; ++i, half += step, full += step) {
      value(i, v);
      if (4 * i < rows) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] *= f.post;
        if (p.out_bf16) *reinterpret_cast<uint2*>(half) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        else *reinterpret_cast<float4*>(full) = make_float4(v[0], v[1], v[2], v[3]);
      }
    }
  } else {
#pragma unroll 1
    for (int i = 0; 4 * i < rows; ++i) {
      // (the arrays of C's values are indexed by constants elsewhere; here a select does it)
      uint2 h = ch[0], l = cl[0];
#pragma unroll
      for (int j = 1; j < 8; ++j)
        if (j == i) h = ch[j], l = cl[j];
      const float4 q = *reinterpret_cast<const float4*>(stage + staged(4 * i + sub, col));
      v[0] = q.x * f.alpha, v[1] = q.y * f.alpha, v[2] = q.z * f.alpha, v[3] = q.w * f.alpha;
      if (with_lo) add_halves(v, l, f.beta);
      if (with_c) add_halves(v, h, f.beta);
      const int64_t at = (static_cast<int64_t>(it.b) * p.M + row0 + 4 * i + sub) * p.N + col0 + col;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (col0 + col + k < p.N) {
          if (p.out_bf16) store1(static_cast<bf16_t*>(p.out) + at + k, v[k] * f.post);
          else static_cast<float*>(p.out)[at + k] = v[k] * f.post;
        }
    }
  }
  __syncwarp();
  if (mirror) {       // a column of the chunk is a row of its mirror
    const int64_t at = it.b * p.stride_o + (col0 + sub) * p.ld_o + row0 + col, step = 4 * p.ld_o;
    __half *hi = p.o_hi + at, *lo = p.o_lo != nullptr ? p.o_lo + at : nullptr;
    const int mirrored = row0 + col < p.M ? min(32, p.N - col0) - sub : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i, hi += step) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = stage[staged(col + k, 4 * i + sub)];
      if (4 * i < mirrored) store_hi_lo(hi, lo, v);
      if (lo != nullptr) lo += step;
    }
    __syncwarp();
  }
}

// kPrecise: both operands as hi + lo, which a stage holds together: hi hi in one accumulator, hi lo + lo hi in a second, whose sums are
// 2^11 times smaller.  The tensor core's additions cut off instead of rounding, which over a long sum of squares (G's diagonal) is a
// bias; so the first is added up in registers every block or two of K (1000 x 1531: results 1.5e-5 off without, 7.9e-6 every 8
// blocks, 3.9e-6 every 4, 2.0e-6 every 2 in 3 % more time; plain fp32 products 3.0e-6).  Columns 0..255 are two accumulators of hi hi, a chunk each in turn, 256..511 two of
// the others, a tile each in turn: by the time a tile's first chunk may be written, the tile before the last has been read.
// Short sides up to 512 every block: where all singular values are of a size the last steps multiply the bias tenfold (143 x 977 2.9e-6 -> 1.7e-6, plain
// fp32 products 1.3e-6; 403 x 6139 3.1e-6, plain 2.2e-6), for 3 to 4 % of the time; 4096 x 4096 would take 13 % more and be no more exact than it needs to be.
constexpr int64_t kShortChunks = 512;

// kChunk: blocks of K between these additions; 0: not kPrecise.  (At run time it cost 4 %.)
template <int kChunk>
__global__ void __launch_bounds__(kGemmThreads, 1)
ortho_product_kernel(const __grid_constant__ Maps maps, const ProductArgs p) {
  constexpr bool kPrecise = kChunk > 0;
  using St = Stage<kPrecise>;
  constexpr int kStages = St::kCount;
  constexpr uint32_t kStageBytes = St::kBytes;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t bars = base + kBarsOff;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kStages + s); };
  auto acc_full_bar = [&](int a) { return bars + 8u * (2 * kStages + a); };
  auto acc_empty_bar = [&](int a) { return bars + 8u * (2 * kStages + 2 + a); };
  const uint32_t slot = bars + 8u * (2 * kStages + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    prefetch_tensor_map(&maps.a_hi);
    prefetch_tensor_map(&maps.b_hi);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full_bar(a), 1);
      mbar_init(acc_empty_bar(a), 2 * kEpilogueWarps);
    }
    mbar_fence_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(slot, kTmemCols);
    tmem_relinquish_pair();
  }
  pdl_trigger();
  tc_fence_before_sync();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after_sync();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(gen + (slot - base));
  pdl_wait();

  const int pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;
  const int items = p.walk.items;
  bool aborted = false;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    int stage = 0;
    uint32_t phase = 0;
    for (int item = pair; item < items && !aborted; item += pairs) {
      const Item it(p, item);
      if (it.width == 0) continue;
      const int b_chunks = (it.width / 2 + 63) / 64;
      const uint32_t bytes = (kPrecise ? 2 : 1) * (kATileBytes + (p.b_mn ? b_chunks * kHalfChunk : static_cast<uint32_t>(p.walk.block_n / 2) * 128u));
      const int row0 = it.row0 + static_cast<int>(rank) * kBlockM, bn0 = it.n0 + static_cast<int>(rank) * (it.width >> 1);
      for (int kb = it.k_begin; kb < it.k_end; ++kb) {
        if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, p.status)) { aborted = true; break; }
        if (elect_one()) {
          const int k0 = kb * kKBlock;
          if (leader) mbar_expect_tx(full_bar(stage), 2 * bytes);
          const uint32_t fb = map_to_cta(full_bar(stage), 0);
          const uint32_t dst = base + static_cast<uint32_t>(stage) * kStageBytes;
          auto load_a = [&](const CUtensorMap* m, uint32_t to) {
            if (p.a_mn) {
              tma_load_3d_pair(to, m, fb, row0, k0, it.b);
              tma_load_3d_pair(to + kHalfChunk, m, fb, row0 + 64, k0, it.b);
            } else {
              tma_load_3d_pair(to, m, fb, k0, row0, it.b);
            }
          };
          auto load_b = [&](const CUtensorMap* m, uint32_t to) {
            if (p.b_mn) {
              for (int c = 0; c < b_chunks; ++c) tma_load_3d_pair(to + c * kHalfChunk, m, fb, bn0 + 64 * c, k0, it.b);
            } else {
              tma_load_3d_pair(to, m, fb, k0, bn0, it.b);
            }
          };
          load_a(&maps.a_hi, dst);
          load_b(&maps.b_hi, dst + St::kB);
          if constexpr (kPrecise) {
            load_a(&maps.a_lo, dst + kATileBytes);
            load_b(&maps.b_lo, dst + St::kBLo);
          }
        }
        __syncwarp();
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
    }
    for (int i = 0; i < kStages && !aborted; ++i) {
      if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, p.status)) aborted = true;
      if (++stage == kStages) { stage = 0; phase ^= 1u; }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (leader) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0, parity = 0;
      const uint64_t a_desc0 = p.a_mn ? make_smem_desc(base, kHalfChunk, 1024) : make_smem_desc(base, 16, 1024);
      const uint64_t b_desc0 = p.b_mn ? make_smem_desc(base + St::kB, kHalfChunk, 1024) : make_smem_desc(base + St::kB, 16, 1024);
      const uint32_t a_step = (p.a_mn ? 16 * 128 : 32) >> 4, b_step = (p.b_mn ? 16 * 128 : 32) >> 4;    // 16 values of K
      for (int item = pair; item < items && !aborted; item += pairs) {
        const Item it(p, item);
        if (it.width == 0) continue;
        const uint32_t idesc = p.idesc | (static_cast<uint32_t>(it.width >> 3) << 17);
        const int chunk = kPrecise ? kChunk : it.k_end - it.k_begin;
        for (int k0 = it.k_begin; k0 < it.k_end && !aborted; k0 += chunk) {
          if (!mbar_wait_warp(acc_empty_bar(acc), acc_phase ^ 1u, p.status)) { aborted = true; break; }
          tc_fence_after_sync();
          const uint32_t d = tmem + static_cast<uint32_t>(acc) * (kPrecise ? kAccCols / 2 : kAccCols);
          const uint32_t d2 = tmem + kAccCols + parity * (kAccCols / 2);
          const int end = min(it.k_end, k0 + chunk);
          for (int kb = k0; kb < end; ++kb) {
            if (!mbar_wait_warp(full_bar(stage), phase, p.status)) { aborted = true; break; }
            tc_fence_after_sync();
            const uint32_t off = (static_cast<uint32_t>(stage) * kStageBytes) >> 4;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint64_t ad = a_desc0 + off + k * a_step, bd = b_desc0 + off + k * b_step;
                const uint32_t more = (kb > k0 || k > 0) ? 1u : 0u;
                umma_f16_pair(d, ad, bd, idesc, more);
                if constexpr (kPrecise) {
                  umma_f16_pair(d2, ad + (kATileBytes >> 4), bd, idesc, (kb > it.k_begin || k > 0) ? 1u : 0u);
                  umma_f16_pair(d2, ad, bd + ((St::kBLo - St::kB) >> 4), idesc, 1u);
                }
              }
              umma_commit_pair(empty_bar(stage), 3);
            }
            __syncwarp();
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
          if (aborted) break;
          if (elect_one()) umma_commit_pair(acc_full_bar(acc), 3);
          __syncwarp();
          acc ^= 1;
          if (acc == 0) acc_phase ^= 1u;
        }
        parity ^= 1u;
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue
    const int quad = warp & 3, half = (warp - 2) >> 2;
    float* stage_out = reinterpret_cast<float*>(gen + kStagingOff + (warp - 2) * kStageOutBytes);
    const uint32_t lane_base = static_cast<uint32_t>(quad * 32) << 16;
    int acc = 0;
    uint32_t acc_phase = 0, parity = 0;
    auto next_acc = [&]() {       // this accumulator has been read
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(map_to_cta(acc_empty_bar(acc), 0));
      acc ^= 1;
      if (acc == 0) acc_phase ^= 1u;
    };
    for (int item = pair; item < items && !aborted; item += pairs) {
      const Item it(p, item);
      if (it.width == 0) continue;
      const int chunks = it.width / 32, first = half == 0 ? 0 : (chunks + 1) / 2, count = half == 0 ? (chunks + 1) / 2 : chunks / 2;
      const int row0 = it.row0 + static_cast<int>(rank) * kBlockM + quad * 32;
      const Factors f = factors_of(p, it.b);
      if constexpr (kPrecise) {
        float sum[2][32];
        for (int k0 = it.k_begin; k0 < it.k_end; k0 += kChunk) {
          if (!mbar_wait_warp(acc_full_bar(acc), acc_phase, p.status)) { aborted = true; break; }
          tc_fence_after_sync();
          const uint32_t t = tmem + lane_base + static_cast<uint32_t>(acc) * (kAccCols / 2) + 32 * first;
          const uint32_t t2 = tmem + lane_base + kAccCols + parity * (kAccCols / 2) + 32 * first;
          auto add = [&](uint32_t from, bool set) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              if (c < count) {
                uint32_t v[32];
                __syncwarp();
                tmem_ld_32x32b_x32(from + 32 * c, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[c][j] = set ? __uint_as_float(v[j]) : sum[c][j] + __uint_as_float(v[j]);
              }
            }
          };
          add(t, k0 == it.k_begin);
          if (k0 + kChunk >= it.k_end) add(t2, false);
          next_acc();
        }
        if (aborted) break;
#pragma unroll
        for (int c = 0; c < 2; ++c)
          if (c < count) finish_chunk(p, it, f, row0, it.n0 + 32 * (first + c), sum[c], stage_out);
        parity ^= 1u;
      } else {
        if (!mbar_wait_warp(acc_full_bar(acc), acc_phase, p.status)) { aborted = true; break; }
        tc_fence_after_sync();
        const uint32_t t = tmem + lane_base + static_cast<uint32_t>(acc) * kAccCols + 32 * first;
        for (int c = 0; c < count; ++c) {
          uint32_t v[32];
          __syncwarp();
          tmem_ld_32x32b_x32(t + 32 * c, v);
          tmem_ld_wait();
          float d[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) d[j] = __uint_as_float(v[j]);
          finish_chunk(p, it, f, row0, it.n0 + 32 * (first + c), d, stage_out);
        }
        next_acc();
      }
    }
  }

  // ------------------------------------------------------------ common exit
  if (aborted) {
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 200000ull) { }
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

// ---------------------------------------------------------------- the parts of G added up in order, mirrored
// out = the parts' sum + beta C: parts [batch][splits][s][ld], of which chunks of 32 x 32 on and above the diagonal are filled; a CTA takes
// one of these.  C (nullable): laid out like the result; beta is then b of B = b G + c G G, exps this step's exponents, `steps` apart.
__global__ void __launch_bounds__(1024)
ortho_add_parts_kernel(const float* parts, int splits, int s, int64_t ld, float beta, const Exponents* exps, int steps, const __half* c_hi,
                       const __half* c_lo, __half* hi, __half* lo, int64_t ld_o, int64_t stride_o) {
  __shared__ float tile[32][33];
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.z, r0 = blockIdx.y * 32, c0 = blockIdx.x * 32;
  if (c0 < r0) return;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, r = r0 + y, c = c0 + x;
  float v = 0.0f;
  if (r < s && c < s) {
    const float* q = parts + (static_cast<int64_t>(b) * splits * s + r) * ld + c;
    // in order, the loads of eight parts on their way at once (a value a thread: 256 threads with four each took 10 us for 18 parts of 300 x 300)
    for (int k = 0; k < splits; k += 8) {
      float part[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) part[i] = k + i < splits ? ld_stream(q + static_cast<int64_t>(k + i) * s * ld) : 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) v += part[i];
    }
    auto term = [&](const __half* m) {
      return __half2float(__ushort_as_half(ld_stream(reinterpret_cast<const unsigned short*>(m) + b * stride_o + r * ld_o + c)));
    };
    if (c_hi != nullptr) {
      const Exponents e = exponents_at(exps + static_cast<int64_t>(b) * steps);
      if ((e.x | e.b) != 0) beta = ldexpf(beta, e.b - 2 * e.x);
      if (c_lo != nullptr) v = fmaf(term(c_lo), beta, v);
      v = fmaf(term(c_hi), beta, v);
    }
  }
  tile[y][x] = v;
  __syncthreads();
  auto put = [&](int row, int col, float w) {
    if (row >= s || col >= s) return;
    const int64_t at = b * stride_o + row * ld_o + col;
    const __half h = __float2half_rn(w);
    hi[at] = h;
    if (lo != nullptr) lo[at] = __float2half_rn(w - __half2float(h));
  };
  const bool diagonal = r0 == c0;
  put(r, c, diagonal ? tile[min(y, x)][max(y, x)] : v);
  if (!diagonal) put(c0 + y, r0 + x, tile[x][y]);
}

// ---------------------------------------------------------------- the norm, and X from g
constexpr int kThreads = 256;

// Sums of squares of a matrix's parts, fp64: no square overflows or is lost.
template <typename T, bool kVec>
__global__ void __launch_bounds__(kThreads)
ortho_norm_kernel(const T* g, int64_t count, double* parts) {
  __shared__ double s_sum[kThreads / 32];
  pdl_trigger();
  pdl_wait();
  const T* x = g + blockIdx.y * count;
  double sum = 0.0;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kThreads;
  if constexpr (kVec) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < count / 8; i += stride) {
      Vec8<T> v;
      v.load(x + 8 * i);
      float f[8];
      v.unpack(f);
#pragma unroll
      for (int k = 0; k < 8; ++k) sum = fma(static_cast<double>(f[k]), static_cast<double>(f[k]), sum);
    }
  } else {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < count; i += stride) {
      const double f = load1(x + i);
      sum = fma(f, f, sum);
    }
  }
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) sum += s_sum[w];
    parts[static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x] = sum;
  }
}

// How often v can be doubled and stays below 1, at most `most` times.
__device__ __forceinline__ int doublings(double v, int most) {
  int e;
  frexp(v, &e);          // v = m * 2^e with m < 1; zero: 0
  return min(max(-e, 0), most);
}

struct Steps {
  int count;
  float abc[3 * FALQON_ORTHO_MAX_STEPS];
  float bound[FALQON_ORTHO_MAX_STEPS];       // of the singular values of X before each step, where |g| is far above eps
};

// The exponents of a matrix whose X has the 2-norm `ratio`, from bounds of its singular values s before each step: s is at most the norm, then
// at most |a| s + |b| s^3 + |c| s^5 and what it is for any matrix; b s^2 + c s^4 bounds B.  None for norms that are held well as they are.
__device__ __forceinline__ void write_exponents(const Steps& p, double ratio, Exponents* e) {
  const bool small = ratio <= 0.5;
  double s = ratio;
  for (int k = 0; k < p.count; ++k) {
    s = fmin(1.001 * s, static_cast<double>(p.bound[k]));      // (what rounding may add)
    const double a = fabs(p.abc[3 * k]), x = s * s, q = x * (fabs(p.abc[3 * k + 1]) + x * fabs(p.abc[3 * k + 2]));
    e[k] = small ? Exponents{doublings(s, kMostX), doublings(1.001 * q, kMostB)} : Exponents{0, 0};
    s *= a + q;
  }
}

// X = g * 2^(13 + x) / (|g| + eps) as hi and lo; a lane takes eight columns of a row.  Its exponents, x of which is the first.
template <typename T, bool kVec>
__global__ void __launch_bounds__(kThreads)
ortho_scale_kernel(const T* g, int64_t rows, int64_t cols, const double* parts, int nparts, double eps, const __grid_constant__ Steps steps,
                   Exponents* exps, __half* hi, __half* lo, int64_t ld, int64_t stride_o) {
  __shared__ double s_sum[kThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.y;
  double sum = 0.0;      // every CTA adds the same numbers in the same order
  for (int i = threadIdx.x; i < nparts; i += kThreads) sum += ld_stream(parts + static_cast<int64_t>(b) * nparts + i);
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < kThreads / 32; ++w) sum += s_sum[w];
  const double norm = sqrt(sum) + eps;
  const double ratio = norm > 0.0 ? sqrt(sum) / norm : 0.0;
  if (blockIdx.x == 0 && threadIdx.x == 0) write_exponents(steps, ratio, exps + static_cast<int64_t>(b) * steps.count);
  // an infinity or a NaN anywhere: NaN everywhere; nothing but zeros: zeros
  double f = !(sum <= 1.7976931348623157e308) ? nan("") : norm > 0.0 ? static_cast<double>(kScale) / norm : 0.0;
  if (ratio <= 0.5) f = ldexp(f, doublings(1.001 * ratio, kMostX));
  const int64_t groups = (cols + 7) / 8, total = rows * groups;
  const T* x = g + b * rows * cols;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; u < total; u += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t r = u / groups, c = (u - r * groups) * 8;
    float v[8];
    if constexpr (kVec) {
      Vec8<T> q;
      q.load(x + r * cols + c);
      q.unpack(v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = c + k < cols ? load1(x + r * cols + c + k) : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = static_cast<float>(static_cast<double>(v[k]) * f);
    const int64_t at = b * stride_o + r * ld + c;
    const float v0[4] = {v[0], v[1], v[2], v[3]}, v1[4] = {v[4], v[5], v[6], v[7]};
    store_hi_lo(hi + at, lo + at, v0);
    store_hi_lo(hi + at + 4, lo + at + 4, v1);
  }
}

// ---------------------------------------------------------------- host side
constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};
constexpr double kMostStored = 7.9;      // times 2^13 it stays below fp16's largest, 65504
// B may come nearer to it: its bound is that of b x + c x^2 at what G is held as, and what rounding adds is fp32's.  (Published schedules
// for small singular values begin with polynomials that reach 7.97.)
constexpr double kMostOfB = 7.98;

// Whether no value that is stored on the way can pass its limit: bounds of the singular values, step by step, which are left in
// `bounds` (nullable).
bool range_ok(const float* abc, int steps, float* bounds) {
  double bound = 1.0;
  for (int i = 0; i < steps; ++i) {
    const double a = abc ? abc[3 * i] : kQuintic[0], b = abc ? abc[3 * i + 1] : kQuintic[1], c = abc ? abc[3 * i + 2] : kQuintic[2];
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
    bound *= 1.001;                       // what rounding may add
    if (bounds != nullptr) bounds[i] = std::nextafter(static_cast<float>(bound), 1e30f);
    double p = 0.0, q = 0.0;
    auto at = [&](double x) {             // x = s^2
      const double v = std::fabs(b * x + c * x * x), s = std::sqrt(x), w = std::fabs(s * (a + b * x + c * x * x));
      if (v > q) q = v;
      if (w > p) p = w;
    };
    const double most = bound * bound;
    auto inside = [&](double x) { if (x > 0.0 && x < most) at(x); };
    at(most);
    if (c != 0.0) {
      inside(-b / (2.0 * c));                                   // of b x + c x^2
      const double disc = 9.0 * b * b - 20.0 * a * c;           // of s p(s): a + 3 b x + 5 c x^2 = 0
      if (disc >= 0.0) inside((-3.0 * b + std::sqrt(disc)) / (10.0 * c)), inside((-3.0 * b - std::sqrt(disc)) / (10.0 * c));
    } else if (b != 0.0) {
      inside(-a / (3.0 * b));
    }
    if (!(most <= kMostStored) || !(q <= kMostOfB) || !(p <= kMostStored)) return false;
    bound = p;
  }
  return true;
}

// The coefficients of all steps.
void coefficients_of(const falqon_ortho* p, float* abc) {
  for (int i = 0; i < p->steps; ++i)
    for (int k = 0; k < 3; ++k) abc[3 * i + k] = p->coefficients != nullptr ? p->coefficients[3 * i + k] : kQuintic[k];
}

// How a product is run: its tiles' width and walk, and over how many CTAs a tile's contraction is split.
struct Way {
  TileWalk walk;
  int tiles, splits;
};
// The way that should take the least time.  A block of K takes an instruction of 256 rows about as long at 64 columns as at 128 (measured:
// 0.22 us at 64 columns, 0.39 at 256; three products at once 0.73 and 0.78 at 64 and 128), so wide tiles whose contraction is split beat
// narrow ones, where the adding up (a launch, 4 us, and its bytes) is worth it.
Way pick_way(int64_t M, int64_t N, int64_t K, int64_t batch, bool symmetric, bool precise) {
  const int64_t pairs = sm_count() / 2, blocks = (K + kKBlock - 1) / kKBlock;
  const int constant = precise ? 850 : 178;
  const double per_unit = precise ? 0.0008 : 0.0009;
  double best = 0.0;
  Way way{};
  for (int w = precise ? 128 : 256; w >= 64; w -= 32) {
    int64_t tiles = 0;
    const int64_t mt = (M + 255) / 256, nt = (N + w - 1) / w;
    if (!symmetric) tiles = mt * nt;
    else for (int64_t n = 0; n < nt; ++n) tiles += std::min(mt, ((n + 1) * w + 255) / 256);
    const int64_t most = symmetric ? std::max<int64_t>(1, std::min(pairs / (tiles * batch), blocks / 4)) : 1;
    for (int64_t s = 1; s <= most; ++s) {
      const int64_t per = (blocks + s - 1) / s, splits = (blocks + per - 1) / per;      // none without a block
      int64_t cost;
      const TileWalk walk = plan_walk(tiles * batch * splits, pairs, w, constant, &cost);
      double us = static_cast<double>(cost) * per_unit * static_cast<double>(per);
      if (splits > 1) us += 4.0 + static_cast<double>(batch * splits * M * N) * 4e-6;   // half of M N written, then read: 4 bytes at 2 TB/s
      if (best == 0.0 || us < best) best = us, way = Way{walk, static_cast<int>(tiles), static_cast<int>(splits)};
    }
  }
  return way;
}

// bf16 results: up to this short side the product B X is three, too.  The roundings of B and X average out over the short side, and over few
// values they leave as much as the results' own rounding: 69 x 759 2.56e-3 off, so 1.93e-3, where rounding the exact results leaves 1.66e-3 (96 x 14336
// 2.2e-3 and 1.8e-3, 512 x 4096 2.15e-3 and 1.8e-3).  It costs a seventh to a quarter of the time (69 x 759 96 -> 109 us, 16 of 14336 x 80 516 -> 651, 512 x
// 4096 159 -> 191), which longer sides are spared.
constexpr int64_t kPreciseApply = 96;

struct Layout {
  int64_t s, l, ld, ld_s;        // short and long side; pitches of X and of the square matrices
  bool tall, precise, apply_precise;      // precise: three products for one
  Way gram, square;
  int norm_parts;
  size_t x_bytes, sq_bytes;
  size_t x[4], sq[4], parts, norm, exps, total;    // offsets: X hi, lo of two turns; G hi, lo, B hi, lo
};

bool plan_ok(const falqon_ortho* p) {
  return p != nullptr && p->batch >= 1 && p->batch <= 65535 && p->rows >= 1 && p->cols >= 1 && p->rows <= 32768 && p->cols <= 32768 &&
         p->batch <= (int64_t{1} << 36) / (p->rows * p->cols) && (p->dtype == FALQON_BF16 || p->dtype == FALQON_F32) &&
         (p->out_dtype == FALQON_BF16 || p->out_dtype == FALQON_F32) && p->steps >= 1 && p->steps <= FALQON_ORTHO_MAX_STEPS;
}

Layout layout_of(const falqon_ortho* p) {
  Layout y{};
  y.tall = p->rows > p->cols;
  y.s = y.tall ? p->cols : p->rows;
  y.l = y.tall ? p->rows : p->cols;
  y.precise = p->out_dtype == FALQON_F32;
  y.apply_precise = y.precise || y.s <= kPreciseApply;
  y.ld = round_up(p->cols, 64);
  y.ld_s = round_up(y.s, 64);
  y.x_bytes = static_cast<size_t>(p->batch * p->rows * y.ld) * 2;
  y.sq_bytes = static_cast<size_t>(p->batch * y.s * y.ld_s) * 2;
  y.gram = pick_way(y.s, y.s, y.l, p->batch, true, y.precise);
  y.square = pick_way(y.s, y.s, y.s, p->batch, true, y.precise);
  const int splits = std::max(y.gram.splits, y.square.splits);
  const int64_t count = p->rows * p->cols;
  int64_t np = (count + 16383) / 16384;
  const int64_t cap = std::max<int64_t>(1, 8 * static_cast<int64_t>(sm_count()) / p->batch);
  y.norm_parts = static_cast<int>(np < cap ? np : cap);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 1023) / 1024 * 1024; return o; };
  for (int i = 0; i < 4; ++i) y.x[i] = take(y.x_bytes);
  for (int i = 0; i < 4; ++i) y.sq[i] = take((i & 1) == 0 || y.precise || (i == 3 && y.apply_precise) ? y.sq_bytes : 0);
  y.parts = take(splits > 1 ? static_cast<size_t>(p->batch) * splits * y.s * y.ld_s * 4 : 0);
  y.norm = take(static_cast<size_t>(p->batch) * y.norm_parts * 8);
  y.exps = take(static_cast<size_t>(p->batch) * p->steps * sizeof(Exponents));
  y.total = at;
  return y;
}

struct Matrix {          // [batch][rows][cols] as hi and lo; mn: contracted along its rows
  const __half *hi, *lo;
  int64_t rows, cols, ld;
  bool mn;
};

cudaError_t launch_product(ProductArgs g, const Way& way, const Matrix& a, const Matrix& b, int64_t batch, int64_t M, int64_t N, int64_t K, bool precise,
                           cudaStream_t st) {
  g.M = static_cast<int>(M), g.N = static_cast<int>(N), g.batch = static_cast<int>(batch);
  g.kblocks = static_cast<int>((K + kKBlock - 1) / kKBlock);
  g.walk = way.walk, g.tiles = way.tiles, g.splits = way.splits;
  g.m_tiles = static_cast<int>((M + 255) / 256);
  g.per_split = (g.kblocks + g.splits - 1) / g.splits;
  g.a_mn = a.mn, g.b_mn = b.mn;
  // fp32 accumulate, fp16 operands (0), majors at 15 and 16, M / 16 at 24
  g.idesc = (1u << 4) | ((a.mn ? 1u : 0u) << 15) | ((b.mn ? 1u : 0u) << 16) | (static_cast<uint32_t>(256 >> 4) << 24);
  g.status = device_status_ptr();
  if (g.status == nullptr) return cudaErrorInvalidValue;
  Maps maps;
  auto map = [&](CUtensorMap* m, const Matrix& x, const __half* p, uint32_t box_rows) {
    return make_tensor_map_batch16(m, p, batch, x.rows, x.cols, x.ld, x.rows * x.ld, 64, box_rows);
  };
  const uint32_t a_box = a.mn ? 64 : 128, b_box = b.mn ? 64 : static_cast<uint32_t>(g.walk.block_n / 2);
  if (!map(&maps.a_hi, a, a.hi, a_box) || !map(&maps.b_hi, b, b.hi, b_box)) return cudaErrorInvalidValue;
  if (!precise) maps.a_lo = maps.a_hi, maps.b_lo = maps.b_hi;
  else if (!map(&maps.a_lo, a, a.lo, a_box) || !map(&maps.b_lo, b, b.lo, b_box)) return cudaErrorInvalidValue;
  const int64_t all = sm_count() / 2, pairs = g.walk.items < all ? g.walk.items : all;
  const dim3 grid(static_cast<unsigned>(2 * pairs)), block(kGemmThreads);
  auto launch = [&](auto kernel, DeviceMask& done) {
    const cudaError_t e = set_max_dynamic_smem(kernel, static_cast<int>(kSmem), done);
    return e != cudaSuccess ? e : launch_pdl(kernel, grid, block, kSmem, st, 2, maps, g);
  };
  static DeviceMask done0{0}, done1{0}, done2{0};
  if (!precise) return launch(ortho_product_kernel<0>, done0);
  return std::min(a.rows, a.cols) <= kShortChunks && std::min(b.rows, b.cols) <= kShortChunks ? launch(ortho_product_kernel<1>, done1)
                                                                                           : launch(ortho_product_kernel<2>, done2);
}

template <typename T>
cudaError_t launch_start(const falqon_ortho* p, const Layout& y, const void* g, double* norm, Exponents* exps, __half* hi, __half* lo, cudaStream_t st) {
  const T* x = static_cast<const T*>(g);
  const int64_t count = p->rows * p->cols;
  const bool vec = count % 8 == 0 && (reinterpret_cast<uintptr_t>(g) & 15) == 0, rows_vec = vec && p->cols % 8 == 0;
  const dim3 block(kThreads), grid(static_cast<unsigned>(y.norm_parts), static_cast<unsigned>(p->batch));
  cudaError_t e = vec ? launch_pdl(ortho_norm_kernel<T, true>, grid, block, 0, st, 1, x, count, norm)
                      : launch_pdl(ortho_norm_kernel<T, false>, grid, block, 0, st, 1, x, count, norm);
  if (e != cudaSuccess) return e;
  const int64_t units = p->rows * ((p->cols + 7) / 8), want = (units + kThreads - 1) / kThreads;
  const int64_t cap = std::max<int64_t>(1, 8 * static_cast<int64_t>(sm_count()) / p->batch);
  const dim3 grid2(static_cast<unsigned>(want < cap ? want : cap), static_cast<unsigned>(p->batch));
  const int64_t stride = p->rows * y.ld;
  Steps steps{};
  steps.count = p->steps;
  coefficients_of(p, steps.abc);
  if (!range_ok(p->coefficients, p->steps, steps.bound)) return cudaErrorInvalidValue;
  return rows_vec ? launch_pdl(ortho_scale_kernel<T, true>, grid2, block, 0, st, 1, x, p->rows, p->cols, norm, y.norm_parts,
                               static_cast<double>(p->eps), steps, exps, hi, lo, y.ld, stride)
                  : launch_pdl(ortho_scale_kernel<T, false>, grid2, block, 0, st, 1, x, p->rows, p->cols, norm, y.norm_parts,
                               static_cast<double>(p->eps), steps, exps, hi, lo, y.ld, stride);
}

int run(const falqon_ortho* p, const Layout& y, const void* g, void* out, uint8_t* scratch, cudaStream_t st) {
  auto halves = [&](size_t off) { return reinterpret_cast<__half*>(scratch + off); };
  double* norm = reinterpret_cast<double*>(scratch + y.norm);
  Exponents* exps = reinterpret_cast<Exponents*>(scratch + y.exps);
  cudaError_t e = p->dtype == FALQON_BF16 ? launch_start<bf16_t>(p, y, g, norm, exps, halves(y.x[0]), halves(y.x[1]), st)
                                          : launch_start<float>(p, y, g, norm, exps, halves(y.x[0]), halves(y.x[1]), st);
  if (e != cudaSuccess) return FALQON_ERR_CUDA;
  __half *g_hi = halves(y.sq[0]), *g_lo = y.precise ? halves(y.sq[1]) : nullptr, *b_hi = halves(y.sq[2]), *b_lo = y.apply_precise ? halves(y.sq[3]) : nullptr;
  const int64_t sq_stride = y.s * y.ld_s, x_stride = p->rows * y.ld;
  const Way apply = pick_way(p->rows, p->cols, y.s, p->batch, false, y.apply_precise);
  // a symmetric product: to `hi`, `lo` at once, or in parts that are added up there
  auto symmetric = [&](ProductArgs a, const Way& way, const Matrix& x, int64_t K, __half* hi, __half* lo) {
    a.symmetric = true;
    a.mode = way.splits > 1 ? kPart : kHiLo;
    a.parts = reinterpret_cast<float*>(scratch + y.parts);
    a.o_hi = hi, a.o_lo = lo, a.ld_o = y.ld_s, a.stride_o = sq_stride;
    const __half *c_hi = a.c_hi, *c_lo = a.c_lo;
    if (way.splits > 1) a.c_hi = a.c_lo = nullptr;
    cudaError_t r = launch_product(a, way, x, x, p->batch, y.s, y.s, K, y.precise, st);
    if (r != cudaSuccess || way.splits == 1) return r;
    const unsigned n = static_cast<unsigned>((y.s + 31) / 32);
    return launch_pdl(ortho_add_parts_kernel, dim3(n, n, static_cast<unsigned>(p->batch)), dim3(1024), 0, st, 1, a.parts, way.splits, static_cast<int>(y.s),
                      y.ld_s, a.beta, a.exps, a.steps, c_hi, c_lo, hi, lo, y.ld_s, sq_stride);
  };
  for (int i = 0; i < p->steps; ++i) {
    const float* abc = p->coefficients != nullptr ? p->coefficients + 3 * i : kQuintic;
    const int now = 2 * (i & 1), then = 2 - now;
    __half *x_hi = halves(y.x[now]), *x_lo = halves(y.x[now + 1]);
    auto of_step = [&](Product product) {
      ProductArgs a{};
      a.product = product, a.exps = exps + i, a.steps = p->steps;
      return a;
    };
    // G = X X^T (X^T X where tall)
    {
      ProductArgs a = of_step(kGram);
      a.alpha = 1.0f / kScale;
      if (symmetric(a, y.gram, Matrix{x_hi, x_lo, p->rows, p->cols, y.ld, y.tall}, y.l, g_hi, g_lo) != cudaSuccess) return FALQON_ERR_CUDA;
    }
    // B = b G + c G G
    {
      ProductArgs a = of_step(kSquare);
      a.alpha = abc[2] / kScale, a.beta = abc[1];
      a.c_hi = g_hi, a.c_lo = g_lo, a.ld_c = y.ld_s, a.stride_c = sq_stride;
      if (symmetric(a, y.square, Matrix{g_hi, g_lo, y.s, y.s, y.ld_s, false}, y.s, b_hi, b_lo) != cudaSuccess) return FALQON_ERR_CUDA;
    }
    // X <- a X + B X (a X + X B where tall)
    {
      const bool last = i + 1 == p->steps;
      const Matrix m{b_hi, b_lo, y.s, y.s, y.ld_s, false}, x{x_hi, x_lo, p->rows, p->cols, y.ld, !y.tall};
      ProductArgs a = of_step(kApply);
      int power = 0;
      const float f = last ? 2.0f * std::frexp(p->scale, &power) / kScale : 1.0f;       // 1 <= |m| < 2, or 0
      a.post = power - 1;
      a.alpha = f / kScale, a.beta = abc[0] * f;
      a.c_hi = x_hi, a.c_lo = x_lo, a.ld_c = y.ld, a.stride_c = x_stride;
      a.mode = last ? kFinal : kHiLo;
      a.o_hi = halves(y.x[then]), a.o_lo = halves(y.x[then + 1]), a.ld_o = y.ld, a.stride_o = x_stride;
      a.out = out, a.out_bf16 = p->out_dtype == FALQON_BF16;
      a.out_vec = p->cols % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & (a.out_bf16 ? 7 : 15)) == 0;
      e = y.tall ? launch_product(a, apply, x, m, p->batch, p->rows, p->cols, y.s, y.apply_precise, st)
                 : launch_product(a, apply, m, x, p->batch, p->rows, p->cols, y.s, y.apply_precise, st);
      if (e != cudaSuccess) return FALQON_ERR_CUDA;
    }
  }
  return FALQON_OK;
}

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

size_t falqon_orthogonalize_scratch_bytes(const falqon_ortho* p) {
  if (!plan_ok(p)) return 0;
  float abc[3 * FALQON_ORTHO_MAX_STEPS];
  coefficients_of(p, abc);
  return ortho_thin_takes(p->rows, p->cols, p->out_dtype == FALQON_BF16, abc, p->steps) ? ortho_thin_scratch_bytes(p->batch, p->rows, p->cols) : layout_of(p).total;
}

int falqon_orthogonalize(const falqon_ortho* p, const void* g, void* out, void* scratch, size_t scratch_bytes, falqon_stream stream) {
  if (!plan_ok(p) || g == nullptr || out == nullptr || !(p->eps >= 0.0f) || !std::isfinite(p->eps) || !std::isfinite(p->scale) ||
      !range_ok(p->coefficients, p->steps, nullptr) || (reinterpret_cast<uintptr_t>(g) & (p->dtype == FALQON_BF16 ? 1 : 3)) != 0 ||
      (reinterpret_cast<uintptr_t>(out) & (p->out_dtype == FALQON_BF16 ? 1 : 3)) != 0 || (g == out && p->dtype != p->out_dtype))
    return FALQON_ERR_INVALID_ARG;
  if (scratch == nullptr || (reinterpret_cast<uintptr_t>(scratch) & 15) != 0) return FALQON_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ThinPlan thin{p->batch, p->rows, p->cols, p->dtype == FALQON_BF16, p->out_dtype == FALQON_BF16, p->steps, p->eps, p->scale, {}};
  coefficients_of(p, thin.abc);
  if (ortho_thin_takes(p->rows, p->cols, thin.out_bf16, thin.abc, p->steps)) {
    if (scratch_bytes < ortho_thin_scratch_bytes(p->batch, p->rows, p->cols)) return FALQON_ERR_WORKSPACE;
    return launch_ortho_thin(thin, g, out, scratch, st) == cudaSuccess ? FALQON_OK : FALQON_ERR_CUDA;
  }
  const Layout y = layout_of(p);
  return scratch_bytes < y.total ? FALQON_ERR_WORKSPACE : run(p, y, g, out, static_cast<uint8_t*>(scratch), st);
}

}  // extern "C"
