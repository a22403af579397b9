// 8-bit activation checkpoints and the gated MLP that keeps and reads them (include/falqon_train.h).  HBM-bound: every tensor
// is read or written once.  A block of 32 values is four neighbouring lanes of eight values (rows of a multiple of eight
// values) or one warp of single values (any other width).
#include "../../include/falqon_train.h"
#include "chain_math.cuh"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kThreads = 256;

// Where a lane's values lie: `slot` counts lanes' shares (eight values or one), kLanes of them to a block of 32, the blocks of
// all rows laid end to end.  A row's last block may be short.
template <int kVec>
struct Place {
  static constexpr int kLanes = kMx8Block / kVec;
  int64_t block, at;   // scale byte, first value
  bool valid;
  __device__ __forceinline__ Place(int64_t slot, int64_t slots, int64_t cols, int64_t blocks_per_row, bool whole) {
    valid = slot < slots;
    block = slot / kLanes;
    if (whole) {       // rows are whole blocks: values and slots run in step
      at = slot * kVec;
    } else {
      const int64_t row = (slots >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(block) / static_cast<uint32_t>(blocks_per_row))
                                             : block / blocks_per_row;
      const int64_t col = (block - row * blocks_per_row) * kMx8Block + (slot % kLanes) * kVec;
      valid = valid && col < cols;
      at = row * cols + col;
    }
  }
};

template <int kVec>
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
  return kVec == 8 ? quad_max(m) : __reduce_max_sync(0xFFFFFFFFu, m);
}

// Encodes the lanes' values of one block (all lanes of the warp call it; m: the fp32 bit pattern of the lane's largest |value|).
template <int kVec>
__device__ __forceinline__ void encode(const float (&x)[kVec], uint32_t m, const Place<kVec>& pl, uint8_t* codes, uint8_t* scales) {
  const uint32_t e = mx8_exponent(block_max<kVec>(m));
  if (!pl.valid) return;
  const float f = mx8_encode_factor(e);
  if constexpr (kVec == 8) {
    *reinterpret_cast<uint2*>(codes + pl.at) = mx8_encode8(x, f);
  } else {
    codes[pl.at] = mx8_encode1(x[0], f);
  }
  if (threadIdx.x % Place<kVec>::kLanes == 0) scales[pl.block] = static_cast<uint8_t>(e);
}

// kVec values at p (zeros when there are none) and the bit pattern of the largest |value|.
template <typename T, int kVec>
__device__ __forceinline__ uint32_t read(const T* p, bool valid, float (&x)[kVec]) {
  if constexpr (kVec == 8) {
    Vec8<T> v;
    if (valid) v.load(p); else v.zero();
    v.unpack(x);
    return v.max_abs();
  } else {
    x[0] = valid ? load1(p) : 0.0f;
    return abs_bits(x[0]);
  }
}
template <typename T, int kVec>
__device__ __forceinline__ uint32_t write(T* p, const float (&x)[kVec]) {
  if constexpr (kVec == 8) {
    Vec8<T> v;
    v.pack(x);
    v.store(p);
    return v.max_abs();
  } else {
    return store1(p, x[0]);
  }
}
template <int kVec>
__device__ __forceinline__ void read_codes(const uint8_t* codes, const uint8_t* scales, const Place<kVec>& pl, float (&x)[kVec]) {
  const float f = mx8_decode_factor(ld_stream(scales + pl.block));
  if constexpr (kVec == 8) {
    mx8_decode8(ld_stream(reinterpret_cast<const uint2*>(codes + pl.at)), f, x);
  } else {
    x[0] = mx8_decode1(ld_stream(codes + pl.at), f);
  }
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kThreads) save_kernel(const T* x, int64_t slots, int64_t cols, int64_t blocks_per_row, bool whole,
                                                        uint8_t* codes, uint8_t* scales) {
  pdl_trigger();
  pdl_wait();
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  const int lane = threadIdx.x & 31;
  for (int64_t s = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; s - lane < slots; s += step) {
    const Place<kVec> pl(s, slots, cols, blocks_per_row, whole);
    float v[kVec];
    const uint32_t m = read<T, kVec>(x + pl.at, pl.valid, v);
    encode<kVec>(v, m, pl, codes, scales);
  }
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kThreads) load_kernel(T* x, int64_t slots, int64_t cols, int64_t blocks_per_row, bool whole,
                                                        const uint8_t* codes, const uint8_t* scales) {
  pdl_trigger();
  pdl_wait();
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t s = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; s < slots; s += step) {
    const Place<kVec> pl(s, slots, cols, blocks_per_row, whole);
    if (!pl.valid) continue;
    float v[kVec];
    read_codes<kVec>(codes, scales, pl, v);
    write<T, kVec>(x + pl.at, v);
  }
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kThreads) gate_forward_kernel(const T* g, const T* u, T* z, int64_t slots, int64_t cols,
                                                                int64_t blocks_per_row, bool whole, uint8_t* g_codes,
                                                                uint8_t* g_scales, uint8_t* u_codes, uint8_t* u_scales, float* amax) {
  pdl_trigger();
  pdl_wait();
  uint32_t mx = 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  const int lane = threadIdx.x & 31;
  for (int64_t s = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; s - lane < slots; s += step) {
    const Place<kVec> pl(s, slots, cols, blocks_per_row, whole);
    float a[kVec], b[kVec], o[kVec];
    const uint32_t ma = read<T, kVec>(g + pl.at, pl.valid, a), mb = read<T, kVec>(u + pl.at, pl.valid, b);
#pragma unroll
    for (int i = 0; i < kVec; ++i) o[i] = a[i] * sigmoidf(a[i]) * b[i];
    if (pl.valid) mx = max(mx, write<T, kVec>(z + pl.at, o));
    if (g_codes != nullptr) {
      encode<kVec>(a, ma, pl, g_codes, g_scales);
      encode<kVec>(b, mb, pl, u_codes, u_scales);
    }
  }
  if (amax != nullptr) raise_amax(mx, amax);
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kThreads) gate_backward_kernel(const uint8_t* g_codes, const uint8_t* g_scales, const uint8_t* u_codes,
                                                                 const uint8_t* u_scales, const T* dz, T* dg, T* du, int64_t slots,
                                                                 int64_t cols, int64_t blocks_per_row, bool whole, float* amax_dg,
                                                                 float* amax_du) {
  pdl_trigger();
  pdl_wait();
  uint32_t mg = 0, mu = 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t s = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; s < slots; s += step) {
    const Place<kVec> pl(s, slots, cols, blocks_per_row, whole);
    if (!pl.valid) continue;
    float a[kVec], b[kVec], t[kVec], og[kVec], ou[kVec];
    read_codes<kVec>(g_codes, g_scales, pl, a);
    read_codes<kVec>(u_codes, u_scales, pl, b);
    read<T, kVec>(dz + pl.at, true, t);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const float sg = sigmoidf(a[i]);
      ou[i] = t[i] * a[i] * sg;
      og[i] = t[i] * b[i] * sg * (1.0f + a[i] * (1.0f - sg));
    }
    mg = max(mg, write<T, kVec>(dg + pl.at, og));
    mu = max(mu, write<T, kVec>(du + pl.at, ou));
  }
  if (amax_dg != nullptr) raise_amax(mg, amax_dg);
  if (amax_du != nullptr) {
    __syncthreads();   // raise_amax's shared word
    raise_amax(mu, amax_du);
  }
}

inline bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The extent of a call, checked; vec: whether rows are whole vectors of eight.
struct Extent {
  int64_t slots, blocks_per_row;
  bool vec, whole;
  unsigned grid;
  bool set(int64_t rows, int64_t cols, int dtype) {
    if (rows < 1 || cols < 1 || rows > (1ll << 31) || cols > (1ll << 31) || rows > (1ll << 42) / cols) return false;
    if (dtype != FALQON_BF16 && dtype != FALQON_F32) return false;
    vec = cols % 8 == 0;
    whole = cols % kMx8Block == 0;
    blocks_per_row = (cols + kMx8Block - 1) / kMx8Block;
    slots = rows * blocks_per_row * (vec ? 4 : 32);
    const int64_t ctas = (slots + kThreads - 1) / kThreads, cap = static_cast<int64_t>(sm_count()) * 8;
    grid = static_cast<unsigned>(ctas < cap ? ctas : cap);
    return true;
  }
};

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
  const auto go = [&](auto kernel, auto* typed) {
    return finish(launch_pdl(kernel, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1, typed, e.slots, cols,
                             e.blocks_per_row, e.whole, codes, scales));
  };
  if (dtype == FALQON_BF16) {
    const bf16_t* t = static_cast<const bf16_t*>(x);
    return e.vec ? go(save_kernel<bf16_t, 8>, t) : go(save_kernel<bf16_t, 1>, t);
  }
  const float* t = static_cast<const float*>(x);
  return e.vec ? go(save_kernel<float, 8>, t) : go(save_kernel<float, 1>, t);
}

int falqon_checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* x, int dtype,
                           falqon_stream stream) {
  Extent e;
  if (x == nullptr || codes == nullptr || scales == nullptr || !ok16(x) || !ok16(codes) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  const auto go = [&](auto kernel, auto* typed) {
    return finish(launch_pdl(kernel, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1, typed, e.slots, cols,
                             e.blocks_per_row, e.whole, codes, scales));
  };
  if (dtype == FALQON_BF16) {
    bf16_t* t = static_cast<bf16_t*>(x);
    return e.vec ? go(load_kernel<bf16_t, 8>, t) : go(load_kernel<bf16_t, 1>, t);
  }
  float* t = static_cast<float*>(x);
  return e.vec ? go(load_kernel<float, 8>, t) : go(load_kernel<float, 1>, t);
}

int falqon_gate_forward(const void* g, const void* u, int dtype, int64_t rows, int64_t cols, void* z, uint8_t* g_codes,
                        uint8_t* g_scales, uint8_t* u_codes, uint8_t* u_scales, float* amax_out, falqon_stream stream) {
  Extent e;
  const int kept = (g_codes != nullptr) + (g_scales != nullptr) + (u_codes != nullptr) + (u_scales != nullptr);
  if (g == nullptr || u == nullptr || z == nullptr || !ok16(g) || !ok16(u) || !ok16(z) || !ok16(g_codes) || !ok16(u_codes) ||
      (kept != 0 && kept != 4) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  const auto go = [&](auto kernel, auto* typed) {
    using T = std::remove_pointer_t<decltype(typed)>;
    return finish(launch_pdl(kernel, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1, static_cast<const T*>(g),
                             static_cast<const T*>(u), typed, e.slots, cols, e.blocks_per_row, e.whole, g_codes, g_scales, u_codes,
                             u_scales, amax_out));
  };
  if (dtype == FALQON_BF16) {
    bf16_t* t = static_cast<bf16_t*>(z);
    return e.vec ? go(gate_forward_kernel<bf16_t, 8>, t) : go(gate_forward_kernel<bf16_t, 1>, t);
  }
  float* t = static_cast<float*>(z);
  return e.vec ? go(gate_forward_kernel<float, 8>, t) : go(gate_forward_kernel<float, 1>, t);
}

int falqon_gate_backward(const uint8_t* g_codes, const uint8_t* g_scales, const uint8_t* u_codes, const uint8_t* u_scales,
                         const void* dz, int dtype, int64_t rows, int64_t cols, void* dg, void* du, float* amax_dg, float* amax_du,
                         falqon_stream stream) {
  Extent e;
  if (g_codes == nullptr || g_scales == nullptr || u_codes == nullptr || u_scales == nullptr || dz == nullptr || dg == nullptr ||
      du == nullptr || dg == du || !ok16(g_codes) || !ok16(u_codes) || !ok16(dz) || !ok16(dg) || !ok16(du) || !e.set(rows, cols, dtype))
    return FALQON_ERR_INVALID_ARG;
  const auto go = [&](auto kernel, auto* typed) {
    using T = std::remove_pointer_t<decltype(typed)>;
    return finish(launch_pdl(kernel, dim3(e.grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 1, g_codes, g_scales, u_codes,
                             u_scales, static_cast<const T*>(dz), typed, static_cast<T*>(du), e.slots, cols, e.blocks_per_row,
                             e.whole, amax_dg, amax_du));
  };
  if (dtype == FALQON_BF16) {
    bf16_t* t = static_cast<bf16_t*>(dg);
    return e.vec ? go(gate_backward_kernel<bf16_t, 8>, t) : go(gate_backward_kernel<bf16_t, 1>, t);
  }
  float* t = static_cast<float*>(dg);
  return e.vec ? go(gate_backward_kernel<float, 8>, t) : go(gate_backward_kernel<float, 1>, t);
}

}  // extern "C"
