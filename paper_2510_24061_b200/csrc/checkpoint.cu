// 8-bit activation checkpoints and the gated MLP that keeps and reads them (include/falqon_train.h).  HBM-bound: every tensor
// is read or written once.  A block of 32 values is four neighbouring lanes of eight values (rows of a multiple of eight
// values) or one warp of single values (any other width).
#include <type_traits>

#include "../../include/falqon_train.h"
#include "chain_math.cuh"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kThreads = 256;

// How rows are cut into lanes' shares ("slots").
//   kFlat   rows are whole blocks of 32: eight values per lane, slots and values run in step over the whole tensor
//   kVector rows are multiples of eight: eight values per lane, four lanes to a block, a row's last block may be short
//   kSingle any other width: one value per lane, a warp to a block
enum Cut { kFlat, kVector, kSingle };
template <Cut kCut>
constexpr int kShare = kCut == kSingle ? 1 : 8;

// Where a lane's values lie.
template <Cut kCut>
struct Place {
  static constexpr int kLanes = kMx8Block / kShare<kCut>;
  int64_t block, at;   // scale byte, first value
  bool valid;
  __device__ __forceinline__ Place(int64_t slot, int64_t slots, int64_t cols, int64_t blocks_per_row) {
    valid = slot < slots;
    block = slot / kLanes;
    if (kCut == kFlat) {
      at = slot * 8;
    } else {
      const int64_t row = (slots >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(block) / static_cast<uint32_t>(blocks_per_row))
                                             : block / blocks_per_row;
      const int64_t col = (block - row * blocks_per_row) * kMx8Block + (slot % kLanes) * kShare<kCut>;
      valid = valid && col < cols;
      at = row * cols + col;
    }
  }
};

// A lane's share of a tensor: eight values or one (then only the first pair's first half is used).
template <typename T, Cut kCut>
struct Share {
  Vec8<T> v;
  float x;
  __device__ __forceinline__ void load(const T* p, bool valid) {
    if constexpr (kCut == kSingle) {
      x = valid ? load1(p) : 0.0f;
    } else {
      if (valid) v.load(p); else v.zero();
    }
  }
  __device__ __forceinline__ uint32_t max_abs() const {
    if constexpr (kCut == kSingle) return abs_bits(x); else return v.max_abs();
  }
  __device__ __forceinline__ void pairs(f2 (&p)[4]) const {
    if constexpr (kCut == kSingle) p[0] = pack_f32x2(x, 0.0f); else v.pairs(p);
  }
};
template <Cut kCut>
constexpr int kPairs = kCut == kSingle ? 1 : 4;

template <typename T, Cut kCut>
__device__ __forceinline__ uint32_t write(T* p, const f2 (&x)[4], bool want_max) {   // the bit pattern of the largest |value| stored
  if constexpr (kCut == kSingle) {
    float lo, hi;
    unpack_f32x2(x[0], lo, hi);
    return store1(p, lo);
  } else {
    const Vec8<T> o = write8(p, x);
    return want_max ? o.max_abs() : 0u;
  }
}

// Encodes the lanes' values of one block; all lanes of the warp call it.  m: the bit pattern of the lane's largest |value|.
template <Cut kCut>
__device__ __forceinline__ void encode(const f2 (&x)[4], uint32_t m, const Place<kCut>& pl, uint8_t* codes, uint8_t* scales) {
  const uint32_t e = mx8_exponent(kCut == kSingle ? __reduce_max_sync(0xFFFFFFFFu, m) : quad_max(m));
  if (!pl.valid) return;
  const float f = mx8_encode_factor(e);
  if constexpr (kCut == kSingle) {
    float lo, hi;
    unpack_f32x2(x[0], lo, hi);
    codes[pl.at] = mx8_encode1(lo, f);
  } else {
    *reinterpret_cast<uint2*>(codes + pl.at) = mx8_encode8(x, f);
  }
  if (threadIdx.x % Place<kCut>::kLanes == 0) scales[pl.block] = static_cast<uint8_t>(e);
}

// A lane's share of a checkpoint, as it lies in memory.
template <Cut kCut>
struct Coded {
  uint2 q;
  uint32_t e;
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, const Place<kCut>& pl) {
    e = ld_stream(scales + pl.block);
    if constexpr (kCut == kSingle) q.x = ld_stream(codes + pl.at); else q = ld_stream(reinterpret_cast<const uint2*>(codes + pl.at));
  }
  __device__ __forceinline__ void pairs(f2 (&x)[4], float f) const {
    if constexpr (kCut == kSingle) x[0] = pack_f32x2(mx8_decode1(static_cast<uint8_t>(q.x), f), 0.0f); else mx8_decode8(q, f, x);
  }
};

// 1 / (1 + exp(-x)).  For bf16 results two special-function instructions (a few 2^-22, the results' rounding is 2^-8); fp32 results
// take expf and the reciprocal, within 2 units in the last place.
template <typename T>
__device__ __forceinline__ float sigmoid_of(float x) {
  float e, r;
  if constexpr (sizeof(T) == 2) {
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * -1.4426950408889634f));
  } else {
    e = expf(-x);
  }
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return r;
}
template <typename T>
__device__ __forceinline__ f2 sigmoid2(f2 x) {
  float lo, hi;
  unpack_f32x2(x, lo, hi);
  return pack_f32x2(sigmoid_of<T>(lo), sigmoid_of<T>(hi));
}

// The lanes' loop: kUnroll slots at a time with all their loads in flight before the first is used; whole warps stay together.
template <int kUnroll, class Body>
__device__ __forceinline__ void for_slots(int64_t slots, Body body) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  const int lane = threadIdx.x & 31;
  for (int64_t s = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; s - lane < slots; s += kUnroll * step) body(s, step);
}

template <typename T, Cut kCut>
__global__ void __launch_bounds__(kThreads) save_kernel(const T* x, int64_t slots, int64_t cols, int64_t blocks_per_row, uint8_t* codes,
                                                        uint8_t* scales) {
  pdl_trigger();
  pdl_wait();
  for_slots<1>(slots, [&](int64_t s, int64_t) {
    const Place<kCut> pl(s, slots, cols, blocks_per_row);
    Share<T, kCut> v;
    v.load(x + pl.at, pl.valid);
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
  for_slots<1>(slots, [&](int64_t s, int64_t) {
    const Place<kCut> pl(s, slots, cols, blocks_per_row);
    if (!pl.valid) return;
    Coded<kCut> c;
    c.load(codes, scales, pl);
    f2 p[4];
    c.pairs(p, mx8_decode_factor(c.e));
    write<T, kCut>(x + pl.at, p, false);
  });
}

constexpr int kGateUnroll = 2;

template <typename T, Cut kCut>
__global__ void __launch_bounds__(kThreads) gate_forward_kernel(const T* g, const T* u, T* z, int64_t slots, int64_t cols,
                                                                int64_t blocks_per_row, uint8_t* g_codes, uint8_t* g_scales,
                                                                uint8_t* u_codes, uint8_t* u_scales, float* amax) {
  pdl_trigger();
  pdl_wait();
  uint32_t mx = 0;
  for_slots<kGateUnroll>(slots, [&](int64_t s, int64_t step) {
    Share<T, kCut> a[kGateUnroll], b[kGateUnroll];
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * step, slots, cols, blocks_per_row);
      a[j].load(g + pl.at, pl.valid);
      b[j].load(u + pl.at, pl.valid);
    }
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * step, slots, cols, blocks_per_row);
      f2 x[4], y[4], o[4];
      a[j].pairs(x);
      b[j].pairs(y);
#pragma unroll
      for (int k = 0; k < kPairs<kCut>; ++k) o[k] = mul2(mul2(x[k], sigmoid2<T>(x[k])), y[k]);
      if (pl.valid) mx = max(mx, write<T, kCut>(z + pl.at, o, amax != nullptr));
      if (g_codes != nullptr) {
        encode<kCut>(x, a[j].max_abs(), pl, g_codes, g_scales);
        encode<kCut>(y, b[j].max_abs(), pl, u_codes, u_scales);
      }
    }
  });
  if (amax != nullptr) raise_amax(mx, amax);
}

template <typename T, Cut kCut>
__global__ void __launch_bounds__(kThreads) gate_backward_kernel(const uint8_t* g_codes, const uint8_t* g_scales, const uint8_t* u_codes,
                                                                 const uint8_t* u_scales, const T* dz, T* dg, T* du, int64_t slots,
                                                                 int64_t cols, int64_t blocks_per_row, float* amax_dg, float* amax_du) {
  pdl_trigger();
  pdl_wait();
  uint32_t mg = 0, mu = 0;
  for_slots<kGateUnroll>(slots, [&](int64_t s, int64_t step) {
    Coded<kCut> a[kGateUnroll], b[kGateUnroll];
    Share<T, kCut> t[kGateUnroll];
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * step, slots, cols, blocks_per_row);
      if (!pl.valid) continue;
      a[j].load(g_codes, g_scales, pl);
      b[j].load(u_codes, u_scales, pl);
      t[j].load(dz + pl.at, true);
    }
#pragma unroll
    for (int j = 0; j < kGateUnroll; ++j) {
      const Place<kCut> pl(s + j * step, slots, cols, blocks_per_row);
      if (!pl.valid) continue;
      f2 x[4], y[4], d[4], og[4], ou[4];
      a[j].pairs(x, scale_of(a[j].e));
      b[j].pairs(y, scale_of(b[j].e));
      t[j].pairs(d);
#pragma unroll
      for (int k = 0; k < kPairs<kCut>; ++k) {
        const f2 sg = sigmoid2<T>(x[k]), gs = mul2(x[k], sg);
        ou[k] = mul2(d[k], gs);
        // s * (1 + g * (1 - s)) = s + g * s * (1 - s)
        const f2 slope = fma2(gs, fma2(sg, twice(-1.0f), twice(1.0f)), sg);
        og[k] = mul2(mul2(d[k], y[k]), slope);
      }
      mg = max(mg, write<T, kCut>(dg + pl.at, og, amax_dg != nullptr));
      mu = max(mu, write<T, kCut>(du + pl.at, ou, amax_du != nullptr));
    }
  });
  if (amax_dg != nullptr) raise_amax(mg, amax_dg);
  if (amax_du != nullptr) {
    __syncthreads();   // raise_amax's shared word
    raise_amax(mu, amax_du);
  }
}

inline bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The extent of a call, checked.
struct Extent {
  int64_t slots, blocks_per_row;
  Cut cut;
  unsigned grid;
  bool set(int64_t rows, int64_t cols, int dtype) {
    if (rows < 1 || cols < 1 || rows > (1ll << 31) || cols > (1ll << 31) || rows > (1ll << 42) / cols) return false;
    if (dtype != FALQON_BF16 && dtype != FALQON_F32) return false;
    cut = cols % kMx8Block == 0 ? kFlat : cols % 8 == 0 ? kVector : kSingle;
    blocks_per_row = (cols + kMx8Block - 1) / kMx8Block;
    slots = rows * blocks_per_row * (cut == kSingle ? 32 : 4);
    const int64_t ctas = (slots + kThreads - 1) / kThreads, cap = static_cast<int64_t>(sm_count()) * 8;
    grid = static_cast<unsigned>(ctas < cap ? ctas : cap);
    return true;
  }
};
// Calls go(value type, cut) for the kernel of this extent and type.
template <Cut kCut>
using CutIs = std::integral_constant<Cut, kCut>;
template <typename F>
int with_kernel(const Extent& e, int dtype, F go) {
  if (dtype == FALQON_BF16)
    return e.cut == kFlat ? go(bf16_t{}, CutIs<kFlat>{}) : e.cut == kVector ? go(bf16_t{}, CutIs<kVector>{}) : go(bf16_t{}, CutIs<kSingle>{});
  return e.cut == kFlat ? go(0.0f, CutIs<kFlat>{}) : e.cut == kVector ? go(0.0f, CutIs<kVector>{}) : go(0.0f, CutIs<kSingle>{});
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
  return with_kernel(e, dtype, [&](auto type, auto cut) {
    using T = decltype(type);
    return finish(launch_pdl(save_kernel<T, cut.value>, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1,
                             static_cast<const T*>(x), e.slots, cols, e.blocks_per_row, codes, scales));
  });
}

int falqon_checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* x, int dtype,
                           falqon_stream stream) {
  Extent e;
  if (x == nullptr || codes == nullptr || scales == nullptr || !ok16(x) || !ok16(codes) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  return with_kernel(e, dtype, [&](auto type, auto cut) {
    using T = decltype(type);
    return finish(launch_pdl(load_kernel<T, cut.value>, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1,
                             static_cast<T*>(x), e.slots, cols, e.blocks_per_row, codes, scales));
  });
}

int falqon_gate_forward(const void* g, const void* u, int dtype, int64_t rows, int64_t cols, void* z, uint8_t* g_codes,
                        uint8_t* g_scales, uint8_t* u_codes, uint8_t* u_scales, float* amax_out, falqon_stream stream) {
  Extent e;
  const int kept = (g_codes != nullptr) + (g_scales != nullptr) + (u_codes != nullptr) + (u_scales != nullptr);
  if (g == nullptr || u == nullptr || z == nullptr || !ok16(g) || !ok16(u) || !ok16(z) || !ok16(g_codes) || !ok16(u_codes) ||
      (kept != 0 && kept != 4) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  return with_kernel(e, dtype, [&](auto type, auto cut) {
    using T = decltype(type);
    return finish(launch_pdl(gate_forward_kernel<T, cut.value>, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1,
                             static_cast<const T*>(g), static_cast<const T*>(u), static_cast<T*>(z), e.slots, cols, e.blocks_per_row,
                             g_codes, g_scales, u_codes, u_scales, amax_out));
  });
}

int falqon_gate_backward(const uint8_t* g_codes, const uint8_t* g_scales, const uint8_t* u_codes, const uint8_t* u_scales,
                         const void* dz, int dtype, int64_t rows, int64_t cols, void* dg, void* du, float* amax_dg, float* amax_du,
                         falqon_stream stream) {
  Extent e;
  if (g_codes == nullptr || g_scales == nullptr || u_codes == nullptr || u_scales == nullptr || dz == nullptr || dg == nullptr ||
      du == nullptr || dg == du || !ok16(g_codes) || !ok16(u_codes) || !ok16(dz) || !ok16(dg) || !ok16(du) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  return with_kernel(e, dtype, [&](auto type, auto cut) {
    using T = decltype(type);
    return finish(launch_pdl(gate_backward_kernel<T, cut.value>, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1,
                             g_codes, g_scales, u_codes, u_scales, static_cast<const T*>(dz), static_cast<T*>(dg), static_cast<T*>(du),
                             e.slots, cols, e.blocks_per_row, amax_dg, amax_du));
  });
}

}  // extern "C"
