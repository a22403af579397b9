// 8-bit activation checkpoints and the gated MLP that keeps and reads them (include/falqon_train.h).
//   z = silu(g) * u, s = 1 / (1 + exp(-g));  du = dz * g * s;  dg = dz * u * (s + g * s * (1 - s))
// HBM-bound: every tensor is read or written once, 16 bytes per lane and access, two vectors of each tensor in flight per lane.
// A block of 32 values is four neighbouring lanes of eight values, its largest value two shuffles away.  bf16 at 4096 x 11008 with
// both checkpoints: forward 62 us (5.9 TB/s), backward 61 us (6.0 TB/s); 8192 x 13824 backward 144 us (6.3 TB/s).
#include <type_traits>

#include "../../include/falqon_train.h"
#include "chain_math.cuh"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kThreads = 256;

// How a tensor is cut into vectors of eight values:
//   kFlat   rows are whole blocks of 32: vectors and blocks run in step over the whole tensor, four lanes to a block (forward, bf16
//           4096 x 11008: 62 us, by kVector's places 66; fp32 101, by kVector's 112)
//   kVector rows are multiples of eight: four lanes to a block, a row's last block may be short (bf16 30000 x 1000 forward: 48 us,
//           by kRagged's kernels 137)
//   kRagged any other width: vectors run over the whole tensor regardless of rows, so that all but its last are aligned, and
//           blocks begin anywhere in them (kernels of their own below; single values per lane took five times as long)
enum Cut { kFlat, kVector, kRagged };

// Where a lane's vector lies (kFlat, kVector).  `slot` counts vectors, four to a block, the blocks of all rows laid end to end.
template <Cut kCut>
struct Place {
  int64_t block, at;   // scale byte, first value
  bool valid;
  __device__ __forceinline__ Place(int64_t slot, int64_t slots, int64_t cols, int64_t blocks_per_row) {
    valid = slot < slots;
    block = slot >> 2;
    if (kCut == kFlat) {
      at = slot * 8;
    } else {
      const int64_t row = (slots >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(block) / static_cast<uint32_t>(blocks_per_row))
                                             : block / blocks_per_row;
      const int64_t col = (block - row * blocks_per_row) * kMx8Block + (slot & 3) * 8;
      valid = valid && col < cols;
      at = row * cols + col;
    }
  }
};

template <typename T>
__device__ __forceinline__ Vec8<T> load_if(const T* p, bool valid) {
  Vec8<T> v;
  if (valid) v.load(p); else v.zero();
  return v;
}

// Encodes the lanes' values of one block; all lanes of the warp call it.  m: the bit pattern of the lane's largest |value|.
template <Cut kCut>
__device__ __forceinline__ void encode(const f2 (&x)[4], uint32_t m, const Place<kCut>& pl, uint8_t* codes, uint8_t* scales) {
  const uint32_t e = mx8_exponent(quad_max(m));
  if (!pl.valid) return;
  *reinterpret_cast<uint2*>(codes + pl.at) = mx8_encode8(x, mx8_encode_factor(e));
  if ((threadIdx.x & 3) == 0) scales[pl.block] = static_cast<uint8_t>(e);
}

// A lane's vector of a checkpoint, as it lies in memory.
template <Cut kCut>
struct Coded {
  uint2 q;
  uint32_t e;
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, const Place<kCut>& pl) {
    e = ld_stream(scales + pl.block);
    q = ld_stream(reinterpret_cast<const uint2*>(codes + pl.at));
  }
};

// 1 / (1 + exp(-x)) of two values.  As it stands exp(-x) overflows at x = -88.8 and the reciprocal is subnormal, and flushed, from -87.4 on,
// where x times it is still a normal number; so it is taken in forms that stay in range:
//   fp32 results   t = exp(-|x|): 1 / (1 + t) or t / (1 + t), with expf and the reciprocal instruction, 4 units of 2^-23 at most
//   bf16 results   2^-24 / (2^-24 + exp(-x) * 2^-24), the last product formed in the exponent, from the special-function unit: |x| * 2^-23
//                  from the exponent's rounding and 8 * 2^-23 from the rest (the results' rounding is 2^-8)
__device__ __forceinline__ f2 sigmoid2(f2 x, bf16_t) {
  constexpr float kShift = 24.0f, kScale = 0x1p-24f;
  float a, b, r, q;
  unpack_f32x2(fma2(x, twice(-1.4426950408889634f), twice(-kShift)), a, b);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
  unpack_f32x2(add2(pack_f32x2(a, b), twice(kScale)), a, b);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q) : "f"(b));
  return mul2(pack_f32x2(r, q), twice(kScale));
}
__device__ __forceinline__ float sigmoid1(float x) {
  const float t = expf(-fabsf(x));
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + t));
  return x < 0.0f ? t * r : r;
}
__device__ __forceinline__ f2 sigmoid2(f2 x, float) {
  float lo, hi;
  unpack_f32x2(x, lo, hi);
  return pack_f32x2(sigmoid1(lo), sigmoid1(hi));
}

template <typename T>
__device__ __forceinline__ void gate8(const f2 (&g)[4], const f2 (&u)[4], f2 (&z)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) z[k] = mul2(mul2(g[k], sigmoid2(g[k], T{})), u[k]);
}
template <typename T>
__device__ __forceinline__ void gate_grad8(const f2 (&g)[4], const f2 (&u)[4], const f2 (&dz)[4], f2 (&dg)[4], f2 (&du)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f2 s = sigmoid2(g[k], T{}), gs = mul2(g[k], s);
    du[k] = mul2(dz[k], gs);
    // s * (1 + g * (1 - s)) = s + g * s * (1 - s)
    dg[k] = mul2(mul2(dz[k], u[k]), fma2(gs, fma2(s, twice(-1.0f), twice(1.0f)), s));
  }
}

// The lanes' loop: a CTA takes kUnroll neighbouring runs of kThreads slots at a time, with all their loads in flight before the
// first is used; whole warps stay together.
template <int kUnroll, class Body>
__device__ __forceinline__ void for_slots(int64_t slots, Body body) {
  const int lane = threadIdx.x & 31;
  for (int64_t s = static_cast<int64_t>(blockIdx.x) * (kUnroll * kThreads) + threadIdx.x; s - lane < slots;
       s += static_cast<int64_t>(gridDim.x) * (kUnroll * kThreads))
    body(s);
}

template <typename T, Cut kCut>
__global__ void __launch_bounds__(kThreads) save_kernel(const T* x, int64_t slots, int64_t cols, int64_t blocks_per_row, uint8_t* codes,
                                                        uint8_t* scales) {
  pdl_trigger();
  pdl_wait();
  for_slots<1>(slots, [&](int64_t s) {
    const Place<kCut> pl(s, slots, cols, blocks_per_row);
    const Vec8<T> v = load_if(x + pl.at, pl.valid);
    f2 p[4];
    v.pairs(p);
    encode<kCut>(p, v.max_abs(), pl, codes, scales);
  });
}

template <typename T, Cut kCut>
__global__ void __launch_bounds__(kThreads) load_kernel(T* x, int64_t slots, int64_t cols, int64_t blocks_per_row, const uint8_t* codes,
                                                        const uint8_t* scales) {
  pdl_trigger();
  pdl_wait();
  for_slots<1>(slots, [&](int64_t s) {
    const Place<kCut> pl(s, slots, cols, blocks_per_row);
    if (!pl.valid) return;
    Coded<kCut> c;
    c.load(codes, scales, pl);
    f2 p[4];
    mx8_decode8(c.q, mx8_decode_factor(c.e), p);
    write8(x + pl.at, p);
  });
}

constexpr int kGateUnroll = 2;

template <typename T, Cut kCut>
__global__ void __launch_bounds__(kThreads) gate_forward_kernel(const T* g, const T* u, T* z, int64_t slots, int64_t cols,
                                                                int64_t blocks_per_row, uint8_t* g_codes, uint8_t* g_scales,
                                                                uint8_t* u_codes, uint8_t* u_scales, float* amax) {
  pdl_trigger();
  pdl_wait();
  Largest<T> largest;
  for_slots<kGateUnroll>(slots, [&](int64_t s) {
    Vec8<T> a[kGateUnroll], b[kGateUnroll];
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * kThreads, slots, cols, blocks_per_row);
      a[j] = load_if(g + pl.at, pl.valid);
      b[j] = load_if(u + pl.at, pl.valid);
    }
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * kThreads, slots, cols, blocks_per_row);
      f2 x[4], y[4], o[4];
      a[j].pairs(x);
      b[j].pairs(y);
      gate8<T>(x, y, o);
      if (pl.valid) {
        const Vec8<T> w = write8(z + pl.at, o);
        if (amax != nullptr) largest.see(w);
      }
      if (g_codes != nullptr) {
        encode<kCut>(x, a[j].max_abs(), pl, g_codes, g_scales);
        encode<kCut>(y, b[j].max_abs(), pl, u_codes, u_scales);
      }
    }
  });
  if (amax != nullptr) raise_amax(largest.bits(), amax);
}

// CTAs per SM, that is registers: bf16 four (8192 x 13824: 144 us, three 153), fp32 three (4096 x 11008: 108 us, four 121).
template <typename T, Cut kCut>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) gate_backward_kernel(const uint8_t* g_codes, const uint8_t* g_scales, const uint8_t* u_codes,
                                                                 const uint8_t* u_scales, const T* dz, T* dg, T* du, int64_t slots,
                                                                 int64_t cols, int64_t blocks_per_row, float* amax_dg, float* amax_du) {
  pdl_trigger();
  pdl_wait();
  Largest<T> lg, lu;
  for_slots<kGateUnroll>(slots, [&](int64_t s) {
    Coded<kCut> a[kGateUnroll], b[kGateUnroll];
    Vec8<T> t[kGateUnroll];
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * kThreads, slots, cols, blocks_per_row);
      if (!pl.valid) continue;
      a[j].load(g_codes, g_scales, pl);
      b[j].load(u_codes, u_scales, pl);
      t[j].load(dz + pl.at);
    }
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * kThreads, slots, cols, blocks_per_row);
      if (!pl.valid) continue;
      f2 x[4], y[4], d[4], og[4], ou[4];
      mx8_decode8(a[j].q, scale_of(a[j].e), x);
      mx8_decode8(b[j].q, scale_of(b[j].e), y);
      t[j].pairs(d);
      gate_grad8<T>(x, y, d, og, ou);
      const Vec8<T> wg = write8(dg + pl.at, og), wu = write8(du + pl.at, ou);
      if (amax_dg != nullptr) lg.see(wg);
      if (amax_du != nullptr) lu.see(wu);
    }
  });
  if (amax_dg != nullptr) raise_amax(lg.bits(), amax_dg);
  if (amax_du != nullptr) {
    __syncthreads();   // raise_amax's shared word
    raise_amax(lu.bits(), amax_du);
  }
}

// ---- any width: aligned vectors over the tensor as one run of values
// Rows of any width: their length, the blocks they have, and a multiplier for division by the length (exact below 2^32: the
// 64-bit reciprocal's error times the number stays below one quotient's step).
struct Rows {
  int64_t cols, blocks_per_row, total, blocks;
  uint64_t reciprocal;
  __device__ __forceinline__ int64_t row_of(int64_t at) const {
    if (cols == 1) return at;                                  // its reciprocal is 2^64
    return (total >> 32) == 0 ? static_cast<int64_t>(__umul64hi(static_cast<uint64_t>(at), reciprocal)) : at / cols;
  }
};
// Where eight values from `at` on lie: the first `split` in block `block`, the rest in the next one; `more`: not all of them (blocks
// are numbered through, so every boundary, within a row or at its end, is one on; only short rows and row ends have two within
// eight values).
struct Spread {
  int64_t block;
  int col, split;
  bool more;
  __device__ __forceinline__ Spread(int64_t at, const Rows& r) {
    const int64_t row = r.row_of(at);
    const int cols = static_cast<int>(r.cols);
    col = static_cast<int>(at - row * r.cols);
    block = row * r.blocks_per_row + (col >> 5);
    split = min(kMx8Block - (col & (kMx8Block - 1)), cols - col);
    const int rest = cols - col - split;                       // of the row
    more = split + min(kMx8Block, rest == 0 ? cols : rest) < 8;
  }
};
// The block of each single value, one after the other.
struct Walk {
  int col, cols;
  __device__ __forceinline__ Walk(const Spread& p, const Rows& r) : col(p.col), cols(static_cast<int>(r.cols)) {}
  __device__ __forceinline__ bool step() {                     // to the next value; whether a new block begins there
    ++col;
    const bool end = col == cols;
    if (end) col = 0;
    return end || (col & (kMx8Block - 1)) == 0;
  }
};
// The vector at value `at`, of which `total` may leave only a part (the tensor's last): then single values, zeros after them.
template <typename T>
__device__ __forceinline__ void load_part(const T* p, int64_t at, int64_t total, f2 (&x)[4]) {
  if (at + 8 <= total) {
    Vec8<T> v;
    v.load(p + at);
    v.pairs(x);
    return;
  }
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = at + e < total ? load1(p + at + e) : 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = pack_f32x2(v[2 * k], v[2 * k + 1]);
}
template <typename T>
__device__ __forceinline__ void store_part(T* p, int64_t at, int64_t total, const f2 (&x)[4], Largest<T>& largest) {
  if (at + 8 <= total) {
    largest.see(write8(p + at, x));
    return;
  }
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(x[k], v[2 * k], v[2 * k + 1]);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (at + e >= total) v[e] = 0.0f; else store1(p + at + e, v[e]);
  }
  Vec8<T> w;
  w.pack(v);
  largest.see(w);
}
__device__ __forceinline__ uint2 load_codes_part(const uint8_t* p, int64_t at, int64_t total) {
  if (at + 8 <= total) return ld_stream(reinterpret_cast<const uint2*>(p + at));
  uint32_t w[2] = {0u, 0u};
  for (int e = 0; e < 8 && at + e < total; ++e) w[e >> 2] |= static_cast<uint32_t>(ld_stream(p + at + e)) << (8 * (e & 3));
  return make_uint2(w[0], w[1]);
}

// Saves one tensor (kGate false), or two and their gated product.  A CTA takes a tile of values; the largest |value| of every block
// that touches it is collected in shared memory (a thread's eight values lie in one or two blocks: as many shared-memory
// maxima), with up to 31 values to both sides read again so that the blocks at its ends are complete.
constexpr int kTileVecs = 2 * kThreads, kTileBlocks = kTileVecs * 8 + 64;   // rows of one value: a block each

// The largest |value| of each block, from eight values of one tensor.
__device__ __forceinline__ void collect(const f2 (&x)[4], const Spread& p, const Rows& r, int64_t block0, int blocks, uint32_t* top) {
  const int b = static_cast<int>(p.block - block0);
  uint32_t v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float lo, hi;
    unpack_f32x2(x[k], lo, hi);
    v[2 * k] = abs_bits(lo);
    v[2 * k + 1] = abs_bits(hi);
  }
  if (!p.more) {
    uint32_t m = 0u, n = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m = max(m, e < p.split ? v[e] : 0u);
      n = max(n, e < p.split ? 0u : v[e]);
    }
    if (m != 0u) atomicMax(top + b, m);
    if (n != 0u) atomicMax(top + b + 1, n);                    // a value beyond the tensor's end is 0
    return;
  }
  Walk w(p, r);
  int at = b;
#pragma unroll 1
  for (int e = 0; e < 8; ++e) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = i == e ? v[i] : m;
    if (m != 0u) atomicMax(top + at, m);
    if (w.step()) at = min(at + 1, blocks - 1);
  }
}
// The factor of each of eight values: factor(b) is that of block b.
template <class Factor>
__device__ __forceinline__ void spread_factors(const Spread& p, const Rows& r, float f0, float f1, Factor factor, f2 (&f)[4]) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < p.split ? f0 : f1;
  if (p.more) {
    Walk w(p, r);
    int64_t b = p.block;
    float now = f0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = now;
      if (e < 7 && w.step()) {
        b = min(b + 1, r.blocks - 1);
        now = factor(b);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) f[k] = pack_f32x2(v[2 * k], v[2 * k + 1]);
}

// Bound by instructions: finding and spreading the blocks' scales is most of them.  Four CTAs per SM cost a few spilled words and hide
// the barriers and the shared-memory maxima: bf16 4096 x 11007 with both checkpoints 168 us, with three 208 (2.2 TB/s; 62 us at 11008).
template <typename T, bool kGate>
__global__ void __launch_bounds__(kThreads, 4) ragged_encode_kernel(const T* g, const T* u, T* z, const Rows r, uint8_t* g_codes, uint8_t* g_scales,
                                                                 uint8_t* u_codes, uint8_t* u_scales, float* amax) {
  __shared__ uint32_t top[kGate ? 2 : 1][kTileBlocks];
  pdl_trigger();
  pdl_wait();
  Largest<T> largest;
  const bool coded = g_codes != nullptr;
  const int64_t total = r.total, vecs = (total + 7) / 8;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * kTileVecs; first < vecs; first += static_cast<int64_t>(gridDim.x) * kTileVecs) {
    const int64_t end = min(first + kTileVecs, vecs), lo = max(first - 4, static_cast<int64_t>(0)), hi = min(end + 4, vecs);
    f2 x[2][4], y[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t v = first + j * kThreads + threadIdx.x;
      if (v >= end) continue;
      load_part(g, v * 8, total, x[j]);
      if (kGate) load_part(u, v * 8, total, y[j]);
    }
    const int64_t block0 = Spread(lo * 8, r).block;
    const int blocks = static_cast<int>(Spread(min(hi * 8, total) - 1, r).block - block0) + 1;
    if (coded) {
      for (int i = threadIdx.x; i < blocks; i += kThreads) {
        top[0][i] = 0u;
        if (kGate) top[1][i] = 0u;
      }
      __syncthreads();
      if (threadIdx.x < 8) {                                   // the neighbours' values
        const int64_t v = threadIdx.x < 4 ? first - 4 + threadIdx.x : end + threadIdx.x - 4;
        if (v >= lo && v < hi) {
          const Spread p(v * 8, r);
          f2 n[4];
          load_part(g, v * 8, total, n);
          collect(n, p, r, block0, blocks, top[0]);
          if (kGate) {
            load_part(u, v * 8, total, n);
            collect(n, p, r, block0, blocks, top[1]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t v = first + j * kThreads + threadIdx.x;
        if (v >= end) continue;
        const Spread p(v * 8, r);
        collect(x[j], p, r, block0, blocks, top[0]);
        if (kGate) collect(y[j], p, r, block0, blocks, top[1]);
      }
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t v = first + j * kThreads + threadIdx.x, at = v * 8;
      if (v >= end) continue;
      if (kGate) {
        f2 o[4];
        gate8<T>(x[j], y[j], o);
        store_part(z, at, total, o, largest);
      }
      if (!coded) continue;
      const Spread p(at, r);
      const int b = static_cast<int>(p.block - block0), next = min(b + 1, blocks - 1);
      const auto put = [&](const f2 (&v8)[4], const uint32_t* tops, uint8_t* codes) {
        const auto of = [&](uint32_t m) { return mx8_encode_factor(mx8_exponent(m)); };
        f2 f[4];
        spread_factors(p, r, of(tops[b]), of(tops[next]), [&](int64_t i) { return of(tops[min(static_cast<int>(i - block0), blocks - 1)]); }, f);
        float c[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) unpack_f32x2(mul2(v8[k], f[k]), c[2 * k], c[2 * k + 1]);
        const uint2 q = make_uint2(cvt_fp8x4<0>(c[0], c[1], c[2], c[3]), cvt_fp8x4<0>(c[4], c[5], c[6], c[7]));
        if (at + 8 <= total) {
          *reinterpret_cast<uint2*>(codes + at) = q;
        } else {
          for (int e = 0; at + e < total; ++e) codes[at + e] = static_cast<uint8_t>((e < 4 ? q.x : q.y) >> (8 * (e & 3)));
        }
      };
      put(x[j], top[0], g_codes);
      if (kGate) put(y[j], top[1], u_codes);
    }
    if (coded) {
      for (int i = threadIdx.x; i < blocks; i += kThreads) {   // the scales of the blocks that begin in this tile
        const int64_t b = block0 + i, row = b / r.blocks_per_row, at = row * r.cols + (b - row * r.blocks_per_row) * kMx8Block;
        if (at < first * 8 || at >= end * 8) continue;
        g_scales[b] = static_cast<uint8_t>(mx8_exponent(top[0][i]));
        if (kGate) u_scales[b] = static_cast<uint8_t>(mx8_exponent(top[1][i]));
      }
      __syncthreads();                                         // before the next tile's maxima
    }
  }
  if (amax != nullptr) raise_amax(largest.bits(), amax);
}

// Eight codes from value `at` on, as they lie in memory, with the scales of the two blocks they lie in as a rule.
struct RaggedCodes {
  uint2 q;
  uint32_t e0, e1;
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int64_t at, const Spread& p, const Rows& r) {
    q = load_codes_part(codes, at, r.total);
    e0 = ld_stream(scales + p.block);
    e1 = ld_stream(scales + min(p.block + 1, r.blocks - 1));
  }
  template <class Factor>
  __device__ __forceinline__ void decode(const uint8_t* scales, const Spread& p, const Rows& r, Factor factor, f2 (&x)[4]) const {
    f2 f[4];
    spread_factors(p, r, factor(e0), factor(e1), [&](int64_t b) { return factor(ld_stream(scales + b)); }, f);
    decode4(q.x, x[0], x[1]);
    decode4(q.y, x[2], x[3]);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = mul2(x[k], f[k]);
  }
};

template <typename T>
__global__ void __launch_bounds__(kThreads) ragged_load_kernel(T* x, const Rows r, const uint8_t* codes, const uint8_t* scales) {
  pdl_trigger();
  pdl_wait();
  Largest<T> unused;
  const int64_t vecs = (r.total + 7) / 8;
  for (int64_t v = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; v < vecs; v += static_cast<int64_t>(gridDim.x) * kThreads) {
    const Spread p(v * 8, r);
    RaggedCodes c;
    c.load(codes, scales, v * 8, p, r);
    f2 o[4];
    c.decode(scales, p, r, [](uint32_t e) { return mx8_decode_factor(e); }, o);
    store_part(x, v * 8, r.total, o, unused);
  }
}

// bf16 4096 x 11007: 89 us with four CTAs per SM (4.1 TB/s), 98 with three.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) ragged_gate_backward_kernel(const uint8_t* g_codes, const uint8_t* g_scales, const uint8_t* u_codes,
                                                                        const uint8_t* u_scales, const T* dz, T* dg, T* du, const Rows r,
                                                                        float* amax_dg, float* amax_du) {
  pdl_trigger();
  pdl_wait();
  Largest<T> lg, lu;
  const int64_t vecs = (r.total + 7) / 8, step = static_cast<int64_t>(gridDim.x) * (2 * kThreads);
  for (int64_t v0 = static_cast<int64_t>(blockIdx.x) * (2 * kThreads) + threadIdx.x; v0 < vecs; v0 += step) {
    RaggedCodes a[2], b[2];
    f2 d[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t at = (v0 + j * kThreads) * 8;
      if (at >= r.total) continue;
      const Spread p(at, r);
      a[j].load(g_codes, g_scales, at, p, r);
      b[j].load(u_codes, u_scales, at, p, r);
      load_part(dz, at, r.total, d[j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t at = (v0 + j * kThreads) * 8;
      if (at >= r.total) continue;
      const Spread p(at, r);
      f2 x[4], y[4], og[4], ou[4];
      const auto factor = [](uint32_t e) { return scale_of(e); };
      a[j].decode(g_scales, p, r, factor, x);
      b[j].decode(u_scales, p, r, factor, y);
      gate_grad8<T>(x, y, d[j], og, ou);
      store_part(dg, at, r.total, og, lg);
      store_part(du, at, r.total, ou, lu);
    }
  }
  if (amax_dg != nullptr) raise_amax(lg.bits(), amax_dg);
  if (amax_du != nullptr) {
    __syncthreads();   // raise_amax's shared word
    raise_amax(lu.bits(), amax_du);
  }
}

inline bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The extent of a call, checked.
struct Extent {
  int64_t blocks_per_row, slots;   // slots: kFlat, kVector
  Rows rows_;                      // kRagged
  Cut cut;
  bool set(int64_t rows, int64_t cols, int dtype) {
    if (rows < 1 || cols < 1 || rows > (1ll << 31) || cols > (1ll << 31) || rows > (1ll << 42) / cols) return false;
    if (dtype != FALQON_BF16 && dtype != FALQON_F32) return false;
    cut = cols % kMx8Block == 0 ? kFlat : cols % 8 == 0 ? kVector : kRagged;
    blocks_per_row = (cols + kMx8Block - 1) / kMx8Block;
    slots = rows * blocks_per_row * 4;
    rows_ = Rows{cols, blocks_per_row, rows * cols, rows * blocks_per_row, ~0ull / static_cast<uint64_t>(cols) + 1};
    return true;
  }
  // CTAs for runs of `per_cta` vectors, eight to an SM at the most.
  dim3 grid(int64_t per_cta) const {
    const int64_t vecs = cut == kRagged ? (rows_.total + 7) / 8 : slots, ctas = (vecs + per_cta - 1) / per_cta, cap = static_cast<int64_t>(sm_count()) * 8;
    return dim3(static_cast<unsigned>(ctas < cap ? ctas : cap));
  }
};
// Calls go(value type, cut) for the kernel of this extent and type, cut being kFlat or kVector; ragged(value type) for kRagged.
template <Cut kCut>
using CutIs = std::integral_constant<Cut, kCut>;
template <typename F, typename G>
int with_kernel(const Extent& e, int dtype, F go, G ragged) {
  if (e.cut == kRagged) return dtype == FALQON_BF16 ? ragged(bf16_t{}) : ragged(0.0f);
  if (dtype == FALQON_BF16) return e.cut == kFlat ? go(bf16_t{}, CutIs<kFlat>{}) : go(bf16_t{}, CutIs<kVector>{});
  return e.cut == kFlat ? go(0.0f, CutIs<kFlat>{}) : go(0.0f, CutIs<kVector>{});
}

int finish(cudaError_t e) { return e == cudaSuccess ? FALQON_OK : FALQON_ERR_CUDA; }

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

int falqon_checkpoint_save(const void* x, int dtype, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales,
                           falqon_stream stream) {
  Extent e;
  if (x == nullptr || codes == nullptr || scales == nullptr || !ok16(x) || !ok16(codes) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_kernel(
      e, dtype,
      [&](auto type, auto cut) {
        using T = decltype(type);
        return finish(launch_pdl(save_kernel<T, cut.value>, e.grid(kThreads), dim3(kThreads), 0, st, 1, static_cast<const T*>(x), e.slots, cols,
                                 e.blocks_per_row, codes, scales));
      },
      [&](auto type) {
        using T = decltype(type);
        return finish(launch_pdl(ragged_encode_kernel<T, false>, e.grid(kTileVecs), dim3(kThreads), 0, st, 1, static_cast<const T*>(x),
                                 static_cast<const T*>(nullptr), static_cast<T*>(nullptr), e.rows_, codes, scales,
                                 static_cast<uint8_t*>(nullptr), static_cast<uint8_t*>(nullptr), static_cast<float*>(nullptr)));
      });
}

int falqon_checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* x, int dtype,
                           falqon_stream stream) {
  Extent e;
  if (x == nullptr || codes == nullptr || scales == nullptr || !ok16(x) || !ok16(codes) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_kernel(
      e, dtype,
      [&](auto type, auto cut) {
        using T = decltype(type);
        return finish(launch_pdl(load_kernel<T, cut.value>, e.grid(kThreads), dim3(kThreads), 0, st, 1, static_cast<T*>(x), e.slots, cols,
                                 e.blocks_per_row, codes, scales));
      },
      [&](auto type) {
        using T = decltype(type);
        return finish(launch_pdl(ragged_load_kernel<T>, e.grid(kThreads), dim3(kThreads), 0, st, 1, static_cast<T*>(x), e.rows_,
                                 codes, scales));
      });
}

int falqon_gate_forward(const void* g, const void* u, int dtype, int64_t rows, int64_t cols, void* z, uint8_t* g_codes,
                        uint8_t* g_scales, uint8_t* u_codes, uint8_t* u_scales, float* amax_out, falqon_stream stream) {
  Extent e;
  const int kept = (g_codes != nullptr) + (g_scales != nullptr) + (u_codes != nullptr) + (u_scales != nullptr);
  if (g == nullptr || u == nullptr || z == nullptr || !ok16(g) || !ok16(u) || !ok16(z) || !ok16(g_codes) || !ok16(u_codes) ||
      z == g || z == u || (kept != 0 && kept != 4) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_kernel(
      e, dtype,
      [&](auto type, auto cut) {
        using T = decltype(type);
        return finish(launch_pdl(gate_forward_kernel<T, cut.value>, e.grid(kGateUnroll * kThreads), dim3(kThreads), 0, st, 1,
                                 static_cast<const T*>(g), static_cast<const T*>(u), static_cast<T*>(z), e.slots, cols, e.blocks_per_row, g_codes,
                                 g_scales, u_codes, u_scales, amax_out));
      },
      [&](auto type) {
        using T = decltype(type);
        return finish(launch_pdl(ragged_encode_kernel<T, true>, e.grid(kTileVecs), dim3(kThreads), 0, st, 1, static_cast<const T*>(g),
                                 static_cast<const T*>(u), static_cast<T*>(z), e.rows_, g_codes, g_scales, u_codes,
                                 u_scales, amax_out));
      });
}

int falqon_gate_backward(const uint8_t* g_codes, const uint8_t* g_scales, const uint8_t* u_codes, const uint8_t* u_scales,
                         const void* dz, int dtype, int64_t rows, int64_t cols, void* dg, void* du, float* amax_dg, float* amax_du,
                         falqon_stream stream) {
  Extent e;
  if (g_codes == nullptr || g_scales == nullptr || u_codes == nullptr || u_scales == nullptr || dz == nullptr || dg == nullptr ||
      du == nullptr || dg == du || !ok16(g_codes) || !ok16(u_codes) || !ok16(dz) || !ok16(dg) || !ok16(du) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_kernel(
      e, dtype,
      [&](auto type, auto cut) {
        using T = decltype(type);
        return finish(launch_pdl(gate_backward_kernel<T, cut.value>, e.grid(kGateUnroll * kThreads), dim3(kThreads), 0, st, 1, g_codes, g_scales,
                                 u_codes, u_scales, static_cast<const T*>(dz), static_cast<T*>(dg), static_cast<T*>(du), e.slots, cols,
                                 e.blocks_per_row, amax_dg, amax_du));
      },
      [&](auto type) {
        using T = decltype(type);
        return finish(launch_pdl(ragged_gate_backward_kernel<T>, e.grid(2 * kThreads), dim3(kThreads), 0, st, 1, g_codes, g_scales, u_codes, u_scales,
                                 static_cast<const T*>(dz), static_cast<T*>(dg), static_cast<T*>(du), e.rows_, amax_dg, amax_du));
      });
}

}  // extern "C"
