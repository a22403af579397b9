// The norms after and before a block, fused with the block's gate and the residual scale (include/falqon_train.h).
//   forward    n = y * ip * wpost;  H = s * h + gate * n;  x = H * iq * wpre
//   backward   xh = H * iq;  a = dx * wpre;  d = dh_out + iq * (a - xh * mean(a * xh));  dh = s * d
//              yh = y * ip;  b = q * d with q = gate * wpost;  dy = ip * (b - yh * mean(b * yh))
//              dwpre = sum_t dx * xh;  S_g = sum_{t in g} d * yh;  dgate_g = wpost * S_g;  dwpost = sum_g gate_g * S_g
// The two means of a row's backward come out of ONE reduction, because the second is linear in the first:
//   sum b * yh = sum q * yh * (dh_out + iq * a) - iq * mean(a * xh) * sum q * yh * xh.
// Column sums: a CTA owns consecutive rows of one gate group and keeps its columns' sums in registers; the partial sums are
// added in a fixed order by a second kernel, so every run gives the same bits.
#include "../../include/falqon_train.h"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kNormUnits = 148;    // a CTA per SM

struct NormArgs {
  const void *h, *y, *post_gain, *pre_gain, *gate;
  const uint8_t *h_codes_in, *h_scales_in, *y_codes_in, *y_scales_in;   // backward
  uint8_t *h_codes, *h_scales, *y_codes, *y_scales;                     // forward
  const void *dx, *dh_out;
  void *h_out, *x, *dh, *dy;
  float *inv_post, *inv_pre;                 // written by the forward, read by the backward
  float *amax;
  float *part_s, *part_p;                    // [units][cols] each, nullable: column sums S and dwpre
  int64_t rows, cols, rows_per_gate, pieces, rows_per_piece;
  float res_scale, gain_offset, eps, inv_cols;
  int post, pre, gain_f32;
};

__device__ __forceinline__ float gain_at(const void* p, int64_t i, int f32) {
  return f32 ? ld_stream(static_cast<const float*>(p) + i) : load1(static_cast<const bf16_t*>(p) + i);
}
__device__ __forceinline__ float weight_at(const void* p, int64_t i, const NormArgs& a) {
  return p == nullptr ? 1.0f : a.gain_offset + gain_at(p, i, a.gain_f32);
}

// Sums over the CTA (whole warps); every thread gets them.  `red`: 32 * kN floats; `phase` alternates so that one barrier per
// call is enough (2 buffers).
template <int kN>
__device__ __forceinline__ void cta_sums(float (&v)[kN], float* red, int& phase) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  float* buf = red + phase * 32 * kN;
  phase ^= 1;
#pragma unroll
  for (int k = 0; k < kN; ++k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if (lane == 0) buf[k * 32 + warp] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    float t = lane < warps ? buf[k * 32 + lane] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    v[k] = t;
  }
}

// ---- any width: a thread holds kItems single columns tid, tid + threads, ...; a checkpoint's block is a warp
// Squares are divided by the width before they are added, so that only a mean beyond fp32's range overflows.
template <typename T, int kItems>
__global__ void __launch_bounds__(1024) norm_forward_kernel(const NormArgs a) {
  __shared__ float red[2 * 32];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  uint32_t mx = 0;
  const int64_t blocks_per_row = (a.cols + kMx8Block - 1) / kMx8Block;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t base = row * a.cols;
    const int64_t gbase = a.gate != nullptr ? row / a.rows_per_gate * a.cols : 0;
    float y[kItems], H[kItems];
    float ss[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int64_t c = threadIdx.x + static_cast<int64_t>(i) * blockDim.x;
      const bool in = c < a.cols;
      y[i] = in ? load1(static_cast<const T*>(a.y) + base + c) : 0.0f;
      H[i] = in && a.h != nullptr ? load1(static_cast<const T*>(a.h) + base + c) : 0.0f;
      ss[0] = __fmaf_rn(y[i] * a.inv_cols, y[i], ss[0]);
      const int64_t at = row * blocks_per_row + (c >> 5);
      if (a.h_codes != nullptr) {
        const uint32_t e = mx8_exponent(__reduce_max_sync(0xFFFFFFFFu, abs_bits(H[i])));
        if (in) a.h_codes[base + c] = mx8_encode1(H[i], mx8_encode_factor(e));
        if (in && (threadIdx.x & 31) == 0) a.h_scales[at] = static_cast<uint8_t>(e);
      }
      if (a.y_codes != nullptr) {
        const uint32_t e = mx8_exponent(__reduce_max_sync(0xFFFFFFFFu, abs_bits(y[i])));
        if (in) a.y_codes[base + c] = mx8_encode1(y[i], mx8_encode_factor(e));
        if (in && (threadIdx.x & 31) == 0) a.y_scales[at] = static_cast<uint8_t>(e);
      }
    }
    float ip = 1.0f;
    if (a.post) {
      cta_sums<1>(ss, red, phase);
      ip = rsqrtf(ss[0] + a.eps);
      if (threadIdx.x == 0) a.inv_post[row] = ip;
    }
    ss[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int64_t c = threadIdx.x + static_cast<int64_t>(i) * blockDim.x;
      if (c < a.cols) {
        float n = a.post ? y[i] * ip * weight_at(a.post_gain, c, a) : y[i];
        if (a.gate != nullptr) n *= gain_at(a.gate, gbase + c, a.gain_f32);
        H[i] = a.h != nullptr ? __fmaf_rn(a.res_scale, H[i], n) : n;
        if (a.h_out != nullptr) store1(static_cast<T*>(a.h_out) + base + c, H[i]);
        ss[0] = __fmaf_rn(H[i] * a.inv_cols, H[i], ss[0]);
      }
    }
    if (a.pre) {
      cta_sums<1>(ss, red, phase);
      const float iq = rsqrtf(ss[0] + a.eps);
      if (threadIdx.x == 0) a.inv_pre[row] = iq;
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int64_t c = threadIdx.x + static_cast<int64_t>(i) * blockDim.x;
        if (c < a.cols) mx = max(mx, store1(static_cast<T*>(a.x) + base + c, H[i] * iq * weight_at(a.pre_gain, c, a)));
      }
    }
  }
  if (a.amax != nullptr) raise_amax(mx, a.amax);
}

template <typename T>
__device__ __forceinline__ float saved_at(const void* plain, const uint8_t* codes, const uint8_t* scales, int64_t base, int64_t c,
                                          int64_t scale_base) {
  if (plain != nullptr) return load1(static_cast<const T*>(plain) + base + c);
  if (codes == nullptr) return 0.0f;
  return mx8_decode1(ld_stream(codes + base + c), mx8_decode_factor(ld_stream(scales + scale_base + (c >> 5))));
}

template <typename T, int kItems>
__global__ void __launch_bounds__(1024) norm_backward_kernel(const NormArgs a) {
  __shared__ float red[2 * 3 * 32];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  uint32_t mx = 0;
  const int64_t blocks_per_row = (a.cols + kMx8Block - 1) / kMx8Block;
  const int64_t groups = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate;
  float P[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) P[i] = 0.0f;
  for (int64_t unit = blockIdx.x; unit < groups * a.pieces; unit += gridDim.x) {
    const int64_t group = unit / a.pieces;
    const int64_t first = group * a.rows_per_gate + (unit - group * a.pieces) * a.rows_per_piece;
    const int64_t last = min(min(first + a.rows_per_piece, (group + 1) * a.rows_per_gate), a.rows);
    float S[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) S[i] = 0.0f;
    for (int64_t row = first; row < last; ++row) {
      const int64_t base = row * a.cols, sbase = row * blocks_per_row;
      const float ip = a.post ? ld_stream(a.inv_post + row) : 1.0f, iq = a.pre ? ld_stream(a.inv_pre + row) : 0.0f;
      float dx[kItems], g[kItems], xh[kItems], yh[kItems], q[kItems], w[kItems];
      float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int64_t c = threadIdx.x + static_cast<int64_t>(i) * blockDim.x;
        dx[i] = g[i] = xh[i] = yh[i] = q[i] = w[i] = 0.0f;
        if (c >= a.cols) continue;
        q[i] = (a.post ? weight_at(a.post_gain, c, a) : 1.0f) * (a.gate != nullptr ? gain_at(a.gate, group * a.cols + c, a.gain_f32) : 1.0f);
        yh[i] = saved_at<T>(a.y, a.y_codes_in, a.y_scales_in, base, c, sbase) * ip;
        const float h = saved_at<T>(a.h, a.h_codes_in, a.h_scales_in, base, c, sbase);
        xh[i] = __fmaf_rn(q[i], yh[i], a.res_scale * h) * iq;
        if (a.dh_out != nullptr) g[i] = load1(static_cast<const T*>(a.dh_out) + base + c);
        if (a.pre) {
          w[i] = weight_at(a.pre_gain, c, a);
          dx[i] = load1(static_cast<const T*>(a.dx) + base + c);
          const float t = dx[i] * w[i];
          g[i] = __fmaf_rn(iq, t, g[i]);
          sum[0] = __fmaf_rn(t, xh[i], sum[0]);
        }
        sum[1] = __fmaf_rn(q[i] * yh[i], g[i], sum[1]);
        sum[2] = __fmaf_rn(q[i] * yh[i], xh[i], sum[2]);
      }
      cta_sums<3>(sum, red, phase);
      const float k1 = iq * (sum[0] * a.inv_cols);                        // d = g - xh * k1
      const float k2 = a.post ? (sum[1] - k1 * sum[2]) * a.inv_cols : 0.0f;
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int64_t c = threadIdx.x + static_cast<int64_t>(i) * blockDim.x;
        if (c >= a.cols) continue;
        const float d = __fmaf_rn(-xh[i], k1, g[i]);
        if (a.dh != nullptr) store1(static_cast<T*>(a.dh) + base + c, a.res_scale * d);
        if (a.dy != nullptr) mx = max(mx, store1(static_cast<T*>(a.dy) + base + c, ip * __fmaf_rn(-yh[i], k2, q[i] * d)));
        S[i] = __fmaf_rn(d, yh[i], S[i]);
        P[i] = __fmaf_rn(dx[i], xh[i], P[i]);
      }
    }
    if (a.part_s != nullptr) {
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        const int64_t c = threadIdx.x + static_cast<int64_t>(i) * blockDim.x;
        if (c < a.cols) a.part_s[unit * a.cols + c] = S[i];
      }
    }
  }
  if (a.part_p != nullptr) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int64_t c = threadIdx.x + static_cast<int64_t>(i) * blockDim.x;
      if (c < a.cols) a.part_p[blockIdx.x * a.cols + c] = P[i];
    }
  }
  if (a.amax != nullptr) raise_amax(mx, a.amax);
}

// ---- widths that are multiples of 16: rows stream through shared memory
// A row belongs to a group of whole warps; a warp has kNv neighbouring spans of 256 columns, a lane eight columns of each.
// Every warp copies its own spans of the next rows with 16-byte asynchronous copies into a ring of `depth` stages that only
// it reads, so the copies in flight cost no registers and no barrier.  Two rows at a time (two groups of 256 threads at 4096
// columns): while one group waits for its row's sums, the other computes.  Arithmetic is two values per instruction (f32x2,
// each half an ordinary rounded operation), since a row's instructions, not its bytes, were the limit without it.
struct Shape {
  int cols, group_threads, groups, depth, warp_stage;   // groups: rows a CTA works on at a time; warp_stage: bytes of a warp's stage
  int weights_in_smem;
};
constexpr int kMaxDepth = 4;

template <typename T>
__device__ __forceinline__ void copy_span(uint32_t dst, const T* src, int col0, int cols, int lane) {   // 256 columns of one tensor
  constexpr int n = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < 256 / n / 32; ++j) {
    const int ch = j * 32 + lane;
    if (col0 + ch * n < cols) cp_async16(dst + ch * 16, src + ch * n);
  }
}
template <typename T>
__device__ __forceinline__ void read_span(const uint8_t* src, int lane, f2 (&x)[4]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 q = *reinterpret_cast<const uint4*>(src + lane * 16);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = pack_f32x2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u));
  } else {
    const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(src + lane * 32), b = *reinterpret_cast<const ulonglong2*>(src + lane * 32 + 16);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  }
}
// f: the scale, or its product with a factor of the row (a power of two times a factor is exact).
__device__ __forceinline__ void read_codes(const uint8_t* src, int lane, float f, f2 (&x)[4]) {
  mx8_decode8(*reinterpret_cast<const uint2*>(src + lane * 8), f, x);
}
// cp.async.wait_group takes a constant: at most depth - 1 younger groups may be open.
__device__ __forceinline__ void wait_stage(int depth) {
  switch (depth) {
    case 1: cp_async_wait<0>(); break;
    case 2: cp_async_wait<1>(); break;
    case 3: cp_async_wait<2>(); break;
    default: cp_async_wait<3>(); break;
  }
}

// Sums over a row group of up to 16 warps; every thread gets them.  `red`: the group's kSumFloats<kN>, two halves used in turn so that
// one barrier per call is enough.  Within a warp two sums share their shuffles (after one exchange, even lanes add up the
// first and odd lanes the second); across warps one lane takes one warp's part of one sum.
template <int kN>
constexpr int kSumFloats = 2 * 16 * kN;
template <int kN>
__device__ __forceinline__ void group_sums(float (&v)[kN], float* red, int& phase, int warp, int lane, int warps, int barrier) {
  static_assert(kN == 1 || kN == 3, "");
  constexpr uint32_t all = 0xFFFFFFFFu;
  float* buf = red + phase * 16 * kN;
  if constexpr (kN == 3) {
    const bool odd = (lane & 1) != 0;
    const float other = __shfl_xor_sync(all, odd ? v[0] : v[1], 1);
    float ab = (odd ? v[1] : v[0]) + other, c = v[2] + __shfl_xor_sync(all, v[2], 1);
#pragma unroll
    for (int o = 16; o > 1; o >>= 1) {
      ab += __shfl_xor_sync(all, ab, o);
      c += __shfl_xor_sync(all, c, o);
    }
    if (warps == 1) {
      v[0] = __shfl_sync(all, ab, 0);
      v[1] = __shfl_sync(all, ab, 1);
      v[2] = c;
      return;
    }
    if (lane < 2) buf[lane * 16 + warp] = ab;
    if (lane == 2) buf[32 + warp] = c;
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[0] += __shfl_xor_sync(all, v[0], o);
    if (warps == 1) return;
    if (lane == 0) buf[warp] = v[0];
  }
  phase ^= 1;
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(warps * 32) : "memory");
  const int k = lane >> 3, w = lane & 7;                       // eight lanes to a sum
  float t = 0.0f;
  if (k < kN) {
    if (w < warps) t = buf[k * 16 + w];
    if (w + 8 < warps) t += buf[k * 16 + w + 8];
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) t += __shfl_xor_sync(all, t, o);
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = __shfl_sync(all, t, i * 8);
}

// Eight weights of columns c .. c + 7.
__device__ __forceinline__ void gains8(const void* p, int64_t i, const NormArgs& a, float offset, float (&w)[8]) {
  if (p == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    return;
  }
  if (a.gain_f32) {
    Vec8<float> v;
    v.load(static_cast<const float*>(p) + i);
    v.unpack(w);
  } else {
    Vec8<bf16_t> v;
    v.load(static_cast<const bf16_t*>(p) + i);
    v.unpack(w);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] += offset;
}
// q = gate * wpost and w = wpre of eight columns.
__device__ __forceinline__ void weights8(const NormArgs& a, int64_t group, int c, float (&q)[8], float (&w)[8]) {
  float g[8];
  gains8(a.post ? a.post_gain : nullptr, c, a, a.gain_offset, q);
  gains8(a.gate, group * a.cols + c, a, 0.0f, g);
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] *= g[e];
  gains8(a.pre ? a.pre_gain : nullptr, c, a, a.gain_offset, w);
}
// All columns' q and w, kept in shared memory for the rows of one gate group (or, where they do not fit beside the ring, fetched
// again, from L2, for every row).
__device__ __forceinline__ void fill_weights(const NormArgs& a, int64_t group, float* wsm, int cols) {
  __syncthreads();
  for (int c = threadIdx.x * 8; c < cols; c += blockDim.x * 8) {
    float q[8], w[8];
    weights8(a, group, c, q, w);
    Vec8<float> v;
    v.pack(q);
    v.store(wsm + c);
    v.pack(w);
    v.store(wsm + cols + c);
  }
  __syncthreads();
}
__device__ __forceinline__ void weights_of(const float* wsm, int at, f2 (&x)[4]) {
  const ulonglong2* p = reinterpret_cast<const ulonglong2*>(wsm + at);
  const ulonglong2 lo = p[0], hi = p[1];
  x[0] = lo.x, x[1] = lo.y, x[2] = hi.x, x[3] = hi.y;
}
struct Weights {
  const NormArgs& a;
  const float* wsm;
  int64_t group;
  int cols, in_smem;
  __device__ __forceinline__ void get(int which, int c, f2 (&x)[4]) const {      // 0: q, 1: w
    if (in_smem) {
      weights_of(wsm, which * cols + c, x);
    } else {
      float q[8], w[8];
      weights8(a, group, c, q, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = which == 0 ? pack_f32x2(q[2 * k], q[2 * k + 1]) : pack_f32x2(w[2 * k], w[2 * k + 1]);
    }
  }
};

__device__ __forceinline__ void put_codes8(const f2 (&x)[4], uint8_t* codes, uint8_t* scale, bool in, int lane) {
  float v[8], m = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(x[k], v[2 * k], v[2 * k + 1]);
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(v[e]));
  const uint32_t e8 = mx8_exponent(quad_max(abs_bits(m)));
  if (!in) return;
  *reinterpret_cast<uint2*>(codes) = mx8_encode8(x, mx8_encode_factor(e8));
  if ((lane & 3) == 0) *scale = static_cast<uint8_t>(e8);
}

// What a thread knows of its place, and the rows of a unit: unit = (gate group, run of its rows).
struct Seat {
  int lane, group, warp, warps;
  __device__ __forceinline__ explicit Seat(const Shape& sh) {
    const int tid = threadIdx.x;
    lane = tid & 31;
    group = tid / sh.group_threads;
    warp = (tid - group * sh.group_threads) >> 5;
    warps = sh.group_threads >> 5;
  }
  template <int kNv>
  __device__ __forceinline__ int column() const { return warp * kNv * 256 + lane * 8; }   // its first; span i is 256 * i further
};
struct Unit {
  int gate, first, last;                                       // rows < 2^31
  __device__ __forceinline__ Unit(const NormArgs& a, int64_t unit) {
    gate = static_cast<int>(unit / a.pieces);
    const int64_t begin = gate * a.rows_per_gate + (unit - gate * a.pieces) * a.rows_per_piece;
    first = static_cast<int>(min(begin, a.rows));
    last = static_cast<int>(min(min(begin + a.rows_per_piece, (gate + 1) * a.rows_per_gate), a.rows));
  }
};

template <typename T, int kNv>
__global__ void __launch_bounds__(512, kNv == 2 ? 2 : 1) norm_forward_rows_kernel(const NormArgs a, const Shape sh) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_trigger();
  pdl_wait();
  const bool has_h = a.h != nullptr, post = a.post, pre = a.pre, has_out = a.h_out != nullptr;
  const bool coded_h = a.h_codes != nullptr, coded_y = a.y_codes != nullptr;
  const Seat me(sh);
  const int cols = sh.cols, lane = me.lane, c0 = me.column<kNv>();
  const int64_t blocks_per_row = (cols + kMx8Block - 1) / kMx8Block;
  uint8_t* ring = smem + static_cast<size_t>(threadIdx.x >> 5) * sh.depth * sh.warp_stage;
  float* const tail = reinterpret_cast<float*>(smem + static_cast<size_t>(blockDim.x >> 5) * sh.depth * sh.warp_stage);
  float* red = tail + me.group * kSumFloats<1>;
  float* wsm = tail + sh.groups * kSumFloats<1>;
  constexpr int kSpan = 256 * sizeof(T);                       // bytes of a span; a stage holds [span][y, h]
  const int64_t units = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate * a.pieces;
  const f2 inv_cols = twice(a.inv_cols), res_scale = twice(a.res_scale);
  int phase = 0;
  Largest<T> largest;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u(a, unit);
    const auto issue = [&](int row, int stage) {
      if (row < u.last) {
        const uint32_t dst = smem_u32(ring) + stage * sh.warp_stage;
        const int64_t at = static_cast<int64_t>(row) * cols + me.warp * kNv * 256;
        const T *y = static_cast<const T*>(a.y) + at, *h = static_cast<const T*>(a.h) + at;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          const int col0 = (me.warp * kNv + i) * 256;
          copy_span<T>(dst + i * 2 * kSpan, y + i * 256, col0, cols, lane);
          if (has_h) copy_span<T>(dst + (i * 2 + 1) * kSpan, h + i * 256, col0, cols, lane);
        }
      }
      cp_async_commit();
    };
    for (int s = 0; s < sh.depth; ++s) issue(u.first + me.group + s * sh.groups, s);
    if (sh.weights_in_smem) fill_weights(a, u.gate, wsm, cols);
    const Weights weights{a, wsm, u.gate, cols, sh.weights_in_smem};
    int stage = 0;
    for (int row = u.first + me.group; row < u.last; row += sh.groups) {
      const int64_t at = static_cast<int64_t>(row) * cols + c0;
      wait_stage(sh.depth);
      __syncwarp();
      const uint8_t* src = ring + stage * sh.warp_stage;
      f2 y[kNv][4], H[kNv][4], ss = 0;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        const bool in = c0 + i * 256 < cols;
#pragma unroll
        for (int k = 0; k < 4; ++k) y[i][k] = H[i][k] = 0;
        if (in) {
          read_span<T>(src + i * 2 * kSpan, lane, y[i]);
          if (has_h) read_span<T>(src + (i * 2 + 1) * kSpan, lane, H[i]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) ss = fma2(mul2(y[i][k], inv_cols), y[i][k], ss);
        const int64_t block = row * blocks_per_row + ((c0 + i * 256) >> 5);
        if (coded_h) put_codes8(H[i], a.h_codes + at + i * 256, a.h_scales + block, in, lane);
        if (coded_y) put_codes8(y[i], a.y_codes + at + i * 256, a.y_scales + block, in, lane);
      }
      __syncwarp();                                            // the warp has read its stage
      issue(row + sh.depth * sh.groups, stage);
      stage = stage + 1 == sh.depth ? 0 : stage + 1;
      float sum[1], ip = 1.0f;
      if (post) {
        sum[0] = halves(ss);
        group_sums<1>(sum, red, phase, me.warp, lane, me.warps, me.group + 1);
        ip = rsqrtf(sum[0] + a.eps);
        if (me.warp == 0 && lane == 0) a.inv_post[row] = ip;
      }
      ss = 0;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        if (c0 + i * 256 >= cols) continue;
        f2 q[4];
        weights.get(0, c0 + i * 256, q);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f2 n = mul2(mul2(y[i][k], twice(ip)), q[k]);
          H[i][k] = has_h ? fma2(res_scale, H[i][k], n) : n;
          ss = fma2(mul2(H[i][k], inv_cols), H[i][k], ss);
        }
        if (has_out) write8(static_cast<T*>(a.h_out) + at + i * 256, H[i]);
      }
      if (pre) {
        sum[0] = halves(ss);
        group_sums<1>(sum, red, phase, me.warp, lane, me.warps, me.group + 1);
        const float iq = rsqrtf(sum[0] + a.eps);
        if (me.warp == 0 && lane == 0) a.inv_pre[row] = iq;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          if (c0 + i * 256 >= cols) continue;
          f2 w[4];
          weights.get(1, c0 + i * 256, w);
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = mul2(mul2(H[i][k], twice(iq)), w[k]);
          largest.see(write8(static_cast<T*>(a.x) + at + i * 256, w));
        }
      }
    }
  }
  if (a.amax != nullptr) raise_amax(largest.bits(), a.amax);
}

// The row groups' column sums, added in group order through shared memory (over the ring, which is idle then), to out[cols].
template <int kNv>
__device__ __forceinline__ void sum_groups(const f2 (&v)[kNv][4], float* out, uint8_t* smem, const Shape& sh, const Seat& me) {
  float* all = reinterpret_cast<float*>(smem) + me.group * sh.cols;            // [groups][cols]
  if (sh.groups > 1) __syncthreads();
#pragma unroll
  for (int i = 0; i < kNv; ++i) {
    const int c = me.column<kNv>() + i * 256;
    if (c >= sh.cols) continue;
    ulonglong2* to = reinterpret_cast<ulonglong2*>((sh.groups > 1 ? all : out) + c);
    to[0] = make_ulonglong2(v[i][0], v[i][1]);
    to[1] = make_ulonglong2(v[i][2], v[i][3]);
  }
  if (sh.groups == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < sh.cols; c += blockDim.x) {
    float t = 0.0f;
    for (int g = 0; g < sh.groups; ++g) t += reinterpret_cast<const float*>(smem)[g * sh.cols + c];
    out[c] = t;
  }
  __syncthreads();
}

// In the terms of the file's head, with H in the place of xh = H * iq:  t = iq * dx * w;  g = dh_out + t;  b = q * yh;
//   A = mean(t * H), B = sum b * g, C = sum b * H:  d = g - k1 * H with k1 = iq^2 * A;  dy = ip * (q * d - yh * k2), k2 = (B - k1 * C) / cols.
// kNv = 2 keeps g and H of the row in registers between the sums and the results (yh is read again); kNv = 4 computes all again.
template <typename T, bool kCoded, int kNv>
__global__ void __launch_bounds__(512) norm_backward_rows_kernel(const NormArgs a, const Shape sh) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_trigger();
  pdl_wait();
  const bool has_h = (kCoded ? a.h_codes_in != nullptr : a.h != nullptr), has_dx = a.dx != nullptr, has_g = a.dh_out != nullptr;
  const bool post = a.post, pre = a.pre, want_dh = a.dh != nullptr, want_dy = a.dy != nullptr;
  const Seat me(sh);
  const int cols = sh.cols, lane = me.lane, c0 = me.column<kNv>();
  const int64_t blocks_per_row = (cols + kMx8Block - 1) / kMx8Block;
  uint8_t* ring = smem + static_cast<size_t>(threadIdx.x >> 5) * sh.depth * sh.warp_stage;
  float* const tail = reinterpret_cast<float*>(smem + static_cast<size_t>(blockDim.x >> 5) * sh.depth * sh.warp_stage);
  float* red = tail + me.group * kSumFloats<3>;
  float* wsm = tail + sh.groups * kSumFloats<3>;               // [2][cols]: q and w
  constexpr int kSpan = 256 * sizeof(T), kSaved = kCoded ? 256 : kSpan;         // a stage holds [span][dx, dh_out, h, y]
  constexpr int kSet = 2 * kSpan + 2 * kSaved;
  constexpr bool kKeep = kNv <= 2;
  constexpr int kKept = kKeep ? kNv : 1;
  const int64_t units = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate * a.pieces;
  const f2 res_scale = twice(a.res_scale);
  Largest<T> largest;
  int phase = 0;
  f2 P[kNv][4];
#pragma unroll
  for (int i = 0; i < kNv; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) P[i][k] = 0;

  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u(a, unit);
    const auto issue = [&](int row, int stage) {
      if (row < u.last) {
        const uint32_t dst = smem_u32(ring) + stage * sh.warp_stage;
        const int64_t at = static_cast<int64_t>(row) * cols + me.warp * kNv * 256;
        const T *dx = static_cast<const T*>(a.dx) + at, *g = static_cast<const T*>(a.dh_out) + at;
        const T *h = static_cast<const T*>(a.h) + at, *y = static_cast<const T*>(a.y) + at;
        const uint8_t* half = lane < 16 ? a.h_codes_in : a.y_codes_in;          // lanes 0..15 copy h's codes, 16..31 y's
        const uint8_t* codes = half + at + (lane & 15) * 16;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          const int col0 = (me.warp * kNv + i) * 256;
          if (has_dx) copy_span<T>(dst + i * kSet, dx + i * 256, col0, cols, lane);
          if (has_g) copy_span<T>(dst + i * kSet + kSpan, g + i * 256, col0, cols, lane);
          if (kCoded) {
            if ((half != nullptr && col0 + (lane & 15) * 16 < cols)) cp_async16(dst + i * kSet + 2 * kSpan + lane * 16, codes + i * 256);
          } else {
            if (has_h) copy_span<T>(dst + i * kSet + 2 * kSpan, h + i * 256, col0, cols, lane);
            copy_span<T>(dst + i * kSet + 2 * kSpan + kSaved, y + i * 256, col0, cols, lane);
          }
        }
      }
      cp_async_commit();
    };
    for (int s = 0; s < sh.depth; ++s) issue(u.first + me.group + s * sh.groups, s);
    f2 S[kNv][4];
#pragma unroll
    for (int i = 0; i < kNv; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) S[i][k] = 0;
    // what else a row needs, fetched one row ahead (scales as bytes: nothing waits for them before their row)
    float ip_next = 1.0f, iq_next = 0.0f;
    uint32_t eh_next[kNv], ey_next[kNv];
    const auto fetch = [&](int next) {
      const int64_t row = min(next, u.last - 1);               // no branch: the values would have to be waited for where it joins
      if (post) ip_next = ld_stream(a.inv_post + row);
      if (pre) iq_next = ld_stream(a.inv_pre + row);
      if (kCoded) {
        const int64_t block = row * blocks_per_row + (c0 >> 5);
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          if (c0 + i * 256 >= cols) continue;
          ey_next[i] = ld_stream(a.y_scales_in + block + i * 8);
          if (has_h) eh_next[i] = ld_stream(a.h_scales_in + block + i * 8);
        }
      }
    };
    if (u.first < u.last) fetch(u.first + me.group);
    if (sh.weights_in_smem) fill_weights(a, u.gate, wsm, cols);
    const Weights weights{a, wsm, u.gate, cols, sh.weights_in_smem};
    int stage = 0;
    for (int row = u.first + me.group; row < u.last; row += sh.groups) {
      const int64_t at = static_cast<int64_t>(row) * cols + c0;
      const float ip = ip_next, iq = iq_next;
      float fh[kNv], fy[kNv];
#pragma unroll
      for (int i = 0; i < kNv; ++i) fh[i] = scale_of(eh_next[i]), fy[i] = scale_of(ey_next[i]) * ip;
      wait_stage(sh.depth);
      __syncwarp();
      fetch(row + sh.groups);
      const uint8_t* src = ring + stage * sh.warp_stage;
      const auto read_yh = [&](int i, f2 (&yh)[4]) {
        const uint8_t* set = src + i * kSet + 2 * kSpan + kSaved;
        if constexpr (kCoded) {
          read_codes(set, lane, fy[i], yh);
        } else {
          read_span<T>(set, lane, yh);
#pragma unroll
          for (int k = 0; k < 4; ++k) yh[k] = mul2(yh[k], twice(ip));
        }
      };
      // dxi = iq * dx, t = dxi * w, g, H and b of one span
      const auto values = [&](int i, f2 (&dxi)[4], f2 (&t)[4], f2 (&g)[4], f2 (&H)[4], f2 (&b)[4]) {
        const uint8_t* set = src + i * kSet;
        const int c = c0 + i * 256;
        f2 yh[4];
        read_yh(i, yh);
        weights.get(0, c, b);
        if (has_h) {
          if constexpr (kCoded) read_codes(set + 2 * kSpan, lane, fh[i], H);
          else read_span<T>(set + 2 * kSpan, lane, H);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          b[k] = mul2(b[k], yh[k]);
          H[k] = has_h ? fma2(H[k], res_scale, b[k]) : b[k];
          g[k] = dxi[k] = t[k] = 0;
        }
        if (has_g) read_span<T>(set + kSpan, lane, g);
        if (has_dx) {
          read_span<T>(set, lane, dxi);
          weights.get(1, c, t);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            dxi[k] = mul2(dxi[k], twice(iq));
            t[k] = mul2(dxi[k], t[k]);
            g[k] = add2(g[k], t[k]);
          }
        }
      };
      f2 sums[3] = {0, 0, 0}, dxi[4], t[4], b[4], g[kKept][4], H[kKept][4];
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        const int j = kKeep ? i : 0;
        if (c0 + i * 256 >= cols) continue;
        values(i, dxi, t, g[j], H[j], b);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          sums[0] = fma2(t[k], H[j][k], sums[0]);
          sums[1] = fma2(b[k], g[j][k], sums[1]);
          sums[2] = fma2(b[k], H[j][k], sums[2]);
          P[i][k] = fma2(dxi[k], H[j][k], P[i][k]);
        }
      }
      float sum[3] = {halves(sums[0]), halves(sums[1]), halves(sums[2])};
      group_sums<3>(sum, red, phase, me.warp, lane, me.warps, me.group + 1);
      const float k1 = iq * iq * (sum[0] * a.inv_cols);
      const float k2 = post ? (sum[1] - k1 * sum[2]) * a.inv_cols : 0.0f;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        const int j = kKeep ? i : 0;
        if (c0 + i * 256 >= cols) continue;
        if (!kKeep) values(i, dxi, t, g[j], H[j], b);
        f2 q[4], yh[4];
        weights.get(0, c0 + i * 256, q);
        read_yh(i, yh);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f2 d = fma2(H[j][k], twice(-k1), g[j][k]);
          S[i][k] = fma2(d, yh[k], S[i][k]);
          q[k] = mul2(fma2(yh[k], twice(-k2), mul2(q[k], d)), twice(ip));
          yh[k] = mul2(d, res_scale);
        }
        if (want_dh) write8(static_cast<T*>(a.dh) + at + i * 256, yh);
        if (want_dy) largest.see(write8(static_cast<T*>(a.dy) + at + i * 256, q));
      }
      __syncwarp();                                            // the warp has read its stage
      issue(row + sh.depth * sh.groups, stage);
      stage = stage + 1 == sh.depth ? 0 : stage + 1;
    }
    if (a.part_s != nullptr) sum_groups<kNv>(S, a.part_s + unit * cols, smem, sh, me);
  }
  if (a.part_p != nullptr) sum_groups<kNv>(P, a.part_p + static_cast<int64_t>(blockIdx.x) * cols, smem, sh, me);
  if (a.amax != nullptr) raise_amax(largest.bits(), a.amax);
}

// ---- the usual call: both norms, a residual, every result, rows of 512 columns per warp (512, 1024, .. 8192)
// The same work as the two kernels above with nothing left to test in the row loop and offsets that advance by a row: they are
// bound by the instructions a row takes, and tests and address arithmetic were half of them.
constexpr int kFullDepth = 2;                                  // two rows ahead per group cover the latency

template <typename T>
__device__ __forceinline__ void copy_lane(uint32_t dst, const T* src, int lane) {   // 512 columns; src: the lane's first value
  if constexpr (sizeof(T) == 2) {
    cp_async16(dst, src);
    cp_async16(dst + 512, src + 256);
  } else {                                                     // 128 columns per instruction: src is 4 * lane values from the first
#pragma unroll
    for (int j = 0; j < 4; ++j) cp_async16(dst + 512 * j, src + 128 * j);
  }
}

template <typename T, bool kCodes>
__global__ void __launch_bounds__(512, 2) norm_forward_full_kernel(const NormArgs a, const Shape sh) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_trigger();
  pdl_wait();
  constexpr int kSpan = 256 * sizeof(T), kStage = 4 * kSpan;   // a stage holds [y, h][span]
  const Seat me(sh);
  const int cols = sh.cols, lane = me.lane, c0 = me.column<2>(), groups = sh.groups;
  const uint8_t* ring = smem + (threadIdx.x >> 5) * (kFullDepth * kStage);
  const uint32_t ring_lane = smem_u32(ring) + lane * 16;
  float* const tail = reinterpret_cast<float*>(smem + (blockDim.x >> 5) * (kFullDepth * kStage));
  float* red = tail + me.group * kSumFloats<1>;
  float* wsm = tail + groups * kSumFloats<1>;
  const int64_t units = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate * a.pieces;
  const int64_t step = static_cast<int64_t>(groups) * cols;
  const int lane_shift = sizeof(T) == 2 ? 0 : -4 * lane;       // from a lane's first column to what it copies
  int phase = 0;
  Largest<T> largest;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u(a, unit);
    int row = u.first + me.group;
    int64_t at = static_cast<int64_t>(row) * cols + c0;
    const auto copy = [&](int64_t from, uint32_t dst) {
      copy_lane<T>(dst, static_cast<const T*>(a.y) + from + lane_shift, lane);
      copy_lane<T>(dst + 2 * kSpan, static_cast<const T*>(a.h) + from + lane_shift, lane);
    };
    if (row < u.last) copy(at, ring_lane);
    cp_async_commit();
    if (row + groups < u.last) copy(at + step, ring_lane + kStage);
    cp_async_commit();
    fill_weights(a, u.gate, wsm, cols);
    int stage = 0;
    for (; row < u.last; row += groups, at += step, stage ^= kStage) {
      cp_async_wait<kFullDepth - 1>();
      __syncwarp();
      const uint8_t* src = ring + stage;
      f2 y[2][4], H[2][4], ss = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        read_span<T>(src + i * kSpan, lane, y[i]);
        read_span<T>(src + (2 + i) * kSpan, lane, H[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) ss = fma2(mul2(y[i][k], twice(a.inv_cols)), y[i][k], ss);
      }
      __syncwarp();                                            // the warp has read its stage
      if (row + kFullDepth * groups < u.last) copy(at + kFullDepth * step, ring_lane + stage);
      cp_async_commit();
      if (kCodes) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          put_codes8(H[i], a.h_codes + at + i * 256, a.h_scales + (at >> 5) + i * 8, true, lane);
          put_codes8(y[i], a.y_codes + at + i * 256, a.y_scales + (at >> 5) + i * 8, true, lane);
        }
      }
      float sum[1] = {halves(ss)};
      group_sums<1>(sum, red, phase, me.warp, lane, me.warps, me.group + 1);
      const float ip = rsqrtf(sum[0] + a.eps);
      ss = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f2 q[4];
        weights_of(wsm, c0 + i * 256, q);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          H[i][k] = fma2(twice(a.res_scale), H[i][k], mul2(mul2(y[i][k], twice(ip)), q[k]));
          ss = fma2(mul2(H[i][k], twice(a.inv_cols)), H[i][k], ss);
        }
        write8(static_cast<T*>(a.h_out) + at + i * 256, H[i]);
      }
      sum[0] = halves(ss);
      group_sums<1>(sum, red, phase, me.warp, lane, me.warps, me.group + 1);
      const float iq = rsqrtf(sum[0] + a.eps);
      if (c0 == 0) {
        a.inv_post[row] = ip;
        a.inv_pre[row] = iq;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f2 w[4];
        weights_of(wsm, cols + c0 + i * 256, w);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = mul2(mul2(H[i][k], twice(iq)), w[k]);
        largest.see(write8(static_cast<T*>(a.x) + at + i * 256, w));
      }
    }
  }
  if (a.amax != nullptr) raise_amax(largest.bits(), a.amax);
}

template <typename T, bool kCoded>
__global__ void __launch_bounds__(512) norm_backward_full_kernel(const NormArgs a, const Shape sh) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_trigger();
  pdl_wait();
  constexpr int kSpan = 256 * sizeof(T), kSaved = kCoded ? 256 : kSpan;
  constexpr int kStage = 4 * kSpan + 4 * kSaved;               // a stage holds [dx, dh_out][span] and [span][h, y] codes or [h, y][span]
  constexpr int kH = 4 * kSpan, kY = kH + (kCoded ? 256 : 2 * kSpan), kNext = kCoded ? 512 : kSpan;   // from a span's saved values to the next's
  const Seat me(sh);
  const int cols = sh.cols, lane = me.lane, c0 = me.column<2>(), groups = sh.groups;
  const uint8_t* ring = smem + (threadIdx.x >> 5) * (kFullDepth * kStage);
  const uint32_t ring_lane = smem_u32(ring) + lane * 16;
  float* const tail = reinterpret_cast<float*>(smem + (blockDim.x >> 5) * (kFullDepth * kStage));
  float* red = tail + me.group * kSumFloats<3>;
  float* wsm = tail + groups * kSumFloats<3>;                  // [2][cols]: q and w
  const int64_t units = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate * a.pieces;
  const int64_t step = static_cast<int64_t>(groups) * cols;
  const int lane_shift = sizeof(T) == 2 ? 0 : -4 * lane;       // from a lane's first column to what it copies
  const uint8_t* codes = (lane < 16 ? a.h_codes_in : a.y_codes_in) + (lane & 15) * 16 - lane * 8;   // lanes 0..15 copy h's codes, 16..31 y's
  Largest<T> largest;
  int phase = 0;
  f2 P[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) P[i][k] = 0;

  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u(a, unit);
    int row = u.first + me.group;
    int64_t at = static_cast<int64_t>(row) * cols + c0;
    const auto copy = [&](int64_t from, uint32_t dst) {
      copy_lane<T>(dst, static_cast<const T*>(a.dx) + from + lane_shift, lane);
      copy_lane<T>(dst + 2 * kSpan, static_cast<const T*>(a.dh_out) + from + lane_shift, lane);
      if constexpr (kCoded) {
        cp_async16(dst + kH, codes + from);
        cp_async16(dst + kH + kNext, codes + from + 256);
      } else {
        copy_lane<T>(dst + kH, static_cast<const T*>(a.h) + from + lane_shift, lane);
        copy_lane<T>(dst + kY, static_cast<const T*>(a.y) + from + lane_shift, lane);
      }
    };
    if (row < u.last) copy(at, ring_lane);
    cp_async_commit();
    if (row + groups < u.last) copy(at + step, ring_lane + kStage);
    cp_async_commit();
    f2 S[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) S[i][k] = 0;
    // what else a row needs, fetched one row ahead without a branch (where branches join, the values would be waited for)
    float ip_next, iq_next;
    uint32_t eh_next[2], ey_next[2];
    const auto fetch = [&](int64_t r, int64_t first) {
      ip_next = ld_stream(a.inv_post + r);
      iq_next = ld_stream(a.inv_pre + r);
      if (kCoded) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ey_next[i] = ld_stream(a.y_scales_in + (first >> 5) + i * 8);
          eh_next[i] = ld_stream(a.h_scales_in + (first >> 5) + i * 8);
        }
      }
    };
    if (row < u.last) fetch(row, at);
    fill_weights(a, u.gate, wsm, cols);
    int stage = 0;
    for (; row < u.last; row += groups, at += step, stage ^= kStage) {
      const float ip = ip_next, iq = iq_next;
      float fh[2], fy[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) fh[i] = kCoded ? scale_of(eh_next[i]) * a.res_scale : a.res_scale, fy[i] = kCoded ? scale_of(ey_next[i]) * ip : ip;
      cp_async_wait<kFullDepth - 1>();
      __syncwarp();
      const bool more = row + groups < u.last;
      fetch(more ? row + groups : row, more ? at + step : at);
      const uint8_t* src = ring + stage;
      const auto saved = [&](const uint8_t* p, f2 (&x)[4]) {   // not yet multiplied by its factor
        if constexpr (kCoded) {
          const uint2 q = *reinterpret_cast<const uint2*>(p + lane * 8);
          decode4(q.x, x[0], x[1]);
          decode4(q.y, x[2], x[3]);
        } else {
          read_span<T>(p, lane, x);
        }
      };
      f2 sums[3] = {0, 0, 0}, g[2][4], H[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f2 b[4], t[4], dxi[4];
        saved(src + kY + i * kNext, b);
        weights_of(wsm, c0 + i * 256, t);
        saved(src + kH + i * kNext, H[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          b[k] = mul2(mul2(b[k], twice(fy[i])), t[k]);
          H[i][k] = fma2(H[i][k], twice(fh[i]), b[k]);
        }
        read_span<T>(src + i * kSpan, lane, dxi);
        read_span<T>(src + (2 + i) * kSpan, lane, g[i]);
        weights_of(wsm, cols + c0 + i * 256, t);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          dxi[k] = mul2(dxi[k], twice(iq));
          t[k] = mul2(dxi[k], t[k]);
          g[i][k] = add2(g[i][k], t[k]);
          sums[0] = fma2(t[k], H[i][k], sums[0]);
          sums[1] = fma2(b[k], g[i][k], sums[1]);
          sums[2] = fma2(b[k], H[i][k], sums[2]);
          P[i][k] = fma2(dxi[k], H[i][k], P[i][k]);
        }
      }
      float sum[3] = {halves(sums[0]), halves(sums[1]), halves(sums[2])};
      group_sums<3>(sum, red, phase, me.warp, lane, me.warps, me.group + 1);
      const float k1 = iq * iq * (sum[0] * a.inv_cols);
      const float k2 = (sum[1] - k1 * sum[2]) * a.inv_cols;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f2 q[4], yh[4];
        weights_of(wsm, c0 + i * 256, q);
        saved(src + kY + i * kNext, yh);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f2 d = fma2(H[i][k], twice(-k1), g[i][k]);
          yh[k] = mul2(yh[k], twice(fy[i]));
          S[i][k] = fma2(d, yh[k], S[i][k]);
          q[k] = mul2(fma2(yh[k], twice(-k2), mul2(q[k], d)), twice(ip));
          yh[k] = mul2(d, twice(a.res_scale));
        }
        write8(static_cast<T*>(a.dh) + at + i * 256, yh);
        largest.see(write8(static_cast<T*>(a.dy) + at + i * 256, q));
      }
      __syncwarp();                                            // the warp has read its stage
      if (row + kFullDepth * groups < u.last) copy(at + kFullDepth * step, ring_lane + stage);
      cp_async_commit();
    }
    if (a.part_s != nullptr) sum_groups<2>(S, a.part_s + unit * cols, smem, sh, me);
  }
  if (a.part_p != nullptr) sum_groups<2>(P, a.part_p + static_cast<int64_t>(blockIdx.x) * cols, smem, sh, me);
  if (a.amax != nullptr) raise_amax(largest.bits(), a.amax);
}

// The gradients of gains and gate from the partial column sums.  A CTA takes 32 columns (a row of them is eight lanes of four), a warp
// four partial rows at a time; a team of warps shares a gate group's rows, so that few groups use all warps too.  All loads of a
// sum are in flight at once and every addition has its place: the order never changes.
constexpr int kFinishWarps = 16;
struct FinishArgs {
  const float *part_s, *part_p;
  const void *post_gain, *gate;
  float *dpost_gain, *dpre_gain, *dgate;
  int64_t cols, groups, pieces, ctas;
  float gain_offset;
  int post, gain_f32, team;      // team: warps to a group, a power of two
};
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 shfl4(float4 a, int o) {
  constexpr uint32_t all = 0xFFFFFFFFu;
  return make_float4(__shfl_xor_sync(all, a.x, o), __shfl_xor_sync(all, a.y, o), __shfl_xor_sync(all, a.z, o), __shfl_xor_sync(all, a.w, o));
}
// Rows from, from + 4 * team, .. of n (a lane's row is from + lane / 8), four columns; kVec: columns are a multiple of four.
template <bool kVec>
__device__ __forceinline__ float4 partial_sum(const float* p, int64_t from, int64_t n, int64_t stride, int64_t cols, int64_t c) {
  constexpr int kAhead = 4;
  float4 t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int64_t r = from; r < n; r += kAhead * stride) {
    float4 v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      v[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const int64_t row = r + j * stride;
      if (row >= n || c >= cols) continue;
      const float* q = p + row * cols + c;
      if (kVec) {
        v[j] = ld_stream(reinterpret_cast<const float4*>(q));
      } else {
        v[j].x = ld_stream(q);
        if (c + 1 < cols) v[j].y = ld_stream(q + 1);
        if (c + 2 < cols) v[j].z = ld_stream(q + 2);
        if (c + 3 < cols) v[j].w = ld_stream(q + 3);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) t = add4(t, v[j]);
  }
  t = add4(t, shfl4(t, 8));
  return add4(t, shfl4(t, 16));
}
template <bool kVec>
__global__ void __launch_bounds__(32 * kFinishWarps) norm_finish_kernel(const FinishArgs a) {
  __shared__ float4 red_s[kFinishWarps][8], red_p[kFinishWarps][8];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, column = threadIdx.x & 31;
  const int64_t c4 = static_cast<int64_t>(blockIdx.x) * 32 + (lane & 7) * 4, c = static_cast<int64_t>(blockIdx.x) * 32 + column;
  const int teams = kFinishWarps / a.team, team = warp / a.team, member = warp % a.team;
  if (a.part_p != nullptr) {
    const float4 t = partial_sum<kVec>(a.part_p, warp * 4 + (lane >> 3), a.ctas, 4 * kFinishWarps, a.cols, c4);
    if (lane < 8) red_p[warp][lane] = t;
  }
  const bool in = c < a.cols;
  const float wpost = in && a.post && a.post_gain != nullptr ? a.gain_offset + gain_at(a.post_gain, c, a.gain_f32) : 1.0f;
  float dpost = 0.0f;                                          // of the warp's groups: warp w adds up groups w, w + teams, ..
  const int64_t batches = a.part_s != nullptr ? (a.groups + teams - 1) / teams : 0;
  for (int64_t batch = 0; batch < batches; ++batch) {
    const int64_t g = batch * teams + team;
    if (g < a.groups) {
      const float4 t = partial_sum<kVec>(a.part_s + g * a.pieces * a.cols, member * 4 + (lane >> 3), a.pieces, 4 * a.team, a.cols, c4);
      if (lane < 8) red_s[warp][lane] = t;
    }
    if (a.team > 1) __syncthreads(); else __syncwarp();
    const int64_t mine = batch * teams + warp;                 // warp w < teams finishes team w's group
    if (warp < teams && mine < a.groups && in) {
      float s = 0.0f;
      for (int m = 0; m < a.team; ++m) s += reinterpret_cast<const float*>(red_s[warp * a.team + m])[column];
      if (a.dgate != nullptr) a.dgate[mine * a.cols + c] = wpost * s;
      dpost = __fmaf_rn(a.gate != nullptr ? gain_at(a.gate, mine * a.cols + c, a.gain_f32) : 1.0f, s, dpost);
    }
    if (a.team > 1) __syncthreads(); else __syncwarp();
  }
  __syncthreads();
  if (warp == 0 && in && a.dpre_gain != nullptr) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kFinishWarps; ++w) s += reinterpret_cast<const float*>(red_p[w])[column];
    a.dpre_gain[c] = s;
  }
  if (a.dpost_gain == nullptr) return;
  reinterpret_cast<float*>(red_s[warp])[column] = dpost;
  __syncthreads();
  if (warp == 0 && in) {
    float s = 0.0f;
    for (int w = 0; w < teams; ++w) s += reinterpret_cast<const float*>(red_s[w])[column];
    a.dpost_gain[c] = s;
  }
}

inline bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int finish(cudaError_t e) { return e == cudaSuccess ? FALQON_OK : FALQON_ERR_CUDA; }

bool plan_ok(const falqon_block_norm* p) {
  return p != nullptr && p->rows >= 1 && p->rows < (1ll << 31) && p->cols >= 1 && p->cols <= FALQON_NORM_MAX_COLS &&
         p->rows_per_gate >= 1 && (p->dtype == FALQON_BF16 || p->dtype == FALQON_F32) &&
         (p->gain_dtype == FALQON_BF16 || p->gain_dtype == FALQON_F32) && (p->flags & ~(FALQON_NORM_POST | FALQON_NORM_PRE)) == 0 &&
         p->eps >= 0.0f && p->res_scale == p->res_scale && p->gain_offset == p->gain_offset && ok16(p->post_gain) &&
         ok16(p->pre_gain) && ok16(p->gate);
}

// How rows are dealt out: every gate group in `pieces` runs of rows, a unit each; one gate row for all makes one group.
struct Split {
  int64_t rows_per_gate, groups, pieces, rows_per_piece, units, ctas;
  Split(const falqon_block_norm* p, int64_t target) {
    rows_per_gate = p->gate == nullptr || p->rows_per_gate > p->rows ? p->rows : p->rows_per_gate;
    groups = (p->rows + rows_per_gate - 1) / rows_per_gate;
    pieces = groups >= target ? 1 : target / groups;
    rows_per_piece = (rows_per_gate + pieces - 1) / pieces;
    pieces = (rows_per_gate + rows_per_piece - 1) / rows_per_piece;
    units = groups * pieces;
    ctas = units < target ? units : target;
  }
  void put(NormArgs* a) const {
    a->rows_per_gate = rows_per_gate;
    a->pieces = pieces;
    a->rows_per_piece = rows_per_piece;
  }
};

bool staged(int64_t cols) { return cols % 16 == 0; }
// CTAs that share a backward's rows: one per SM where rows stream through its shared memory; four where every row is fetched when it
// is due and only other CTAs' rows cover the wait (613 x 1011 fp32: 41 us with one, 20 with four).
int64_t backward_units(int64_t cols) { return staged(cols) ? kNormUnits : 4 * kNormUnits; }

NormArgs common(const falqon_block_norm* p) {
  NormArgs a{};
  a.post_gain = p->post_gain;
  a.pre_gain = p->pre_gain;
  a.gate = p->gate;
  a.rows = p->rows;
  a.cols = p->cols;
  a.rows_per_gate = p->rows_per_gate;
  a.res_scale = p->res_scale;
  a.gain_offset = p->gain_offset;
  a.eps = p->eps;
  a.inv_cols = 1.0f / static_cast<float>(p->cols);
  a.post = (p->flags & FALQON_NORM_POST) != 0;
  a.pre = (p->flags & FALQON_NORM_PRE) != 0;
  a.gain_f32 = p->gain_dtype == FALQON_F32;
  return a;
}

// The smallest number of columns per thread that keeps a row within 256 threads, or 16 with up to 1024 threads.
int items_for(int64_t cols) {
  int items = 1;
  while (items < 16 && cols > items * 256) items *= 2;
  return items;
}
template <typename F>
int with_items(int items, F go) {
  switch (items) {
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 4: return go(std::integral_constant<int, 4>{});
    case 8: return go(std::integral_constant<int, 8>{});
    default: return go(std::integral_constant<int, 16>{});
  }
}

// The staged kernels' shape.  set_bytes: of a span of 256 columns of every tensor; red: floats of reduction space per row group.
constexpr int kSmemLimit = 226 * 1024;    // dynamic; the kernels have a few bytes of their own besides
int spans_for(int64_t cols) { return cols <= 2 * 512 * 8 ? 2 : 4; }
// set_bytes: of a span of 256 columns of every tensor; red: floats of reduction space per row group.
bool make_shape(int64_t cols, int64_t rows_per_cta, int set_bytes, int red, int smem_limit, Shape* sh, size_t* smem) {
  const int nv = spans_for(cols), vec = static_cast<int>(cols / 8);
  sh->cols = static_cast<int>(cols);
  sh->group_threads = (vec + 32 * nv - 1) / (32 * nv) * 32;
  sh->groups = 512 / sh->group_threads;
  if (sh->groups > rows_per_cta) sh->groups = static_cast<int>(rows_per_cta < 1 ? 1 : rows_per_cta);
  sh->warp_stage = nv * set_bytes;
  const int warps = sh->groups * sh->group_threads / 32, fixed = sh->groups * red * 4;
  const int weights = static_cast<int>(cols) * 8, stage = warps * sh->warp_stage;
  sh->weights_in_smem = fixed + weights + stage <= smem_limit;
  const int room = smem_limit - fixed - (sh->weights_in_smem ? weights : 0);
  sh->depth = room / stage < kMaxDepth ? room / stage : kMaxDepth;
  *smem = static_cast<size_t>(fixed) + (sh->weights_in_smem ? weights : 0) + static_cast<size_t>(sh->depth) * stage;
  return sh->depth >= 1;
}

bool whole_spans(int64_t cols) { return cols % 512 == 0 && cols <= 8192; }
// Shape of the usual call's kernels: a fixed depth and the weights in shared memory, or false.
bool make_full_shape(int64_t cols, int64_t rows_per_cta, int stage_bytes, int red, Shape* sh, size_t* smem) {
  sh->cols = static_cast<int>(cols);
  sh->group_threads = static_cast<int>(cols / 16);
  sh->groups = 512 / sh->group_threads;
  if (sh->groups > rows_per_cta) sh->groups = static_cast<int>(rows_per_cta < 1 ? 1 : rows_per_cta);
  *smem = static_cast<size_t>(sh->groups * sh->group_threads / 32) * kFullDepth * stage_bytes + sh->groups * red * 4 + static_cast<size_t>(cols) * 8;
  return *smem <= static_cast<size_t>(kSmemLimit);
}
template <typename K>
int start_rows(K kernel, DeviceMask& done, const NormArgs& a, const Shape& sh, size_t smem, int64_t ctas, cudaStream_t stream) {
  if (set_max_dynamic_smem(kernel, kSmemLimit, done) != cudaSuccess) return FALQON_ERR_CUDA;
  return finish(launch_pdl(kernel, dim3(static_cast<unsigned>(ctas)), dim3(static_cast<unsigned>(sh.groups * sh.group_threads)), smem, stream, 1, a, sh));
}
template <typename T, int kNv>
int launch_forward_rows(const NormArgs& a, int64_t ctas, cudaStream_t stream) {
  static DeviceMask done[3];
  Shape sh;
  size_t smem;
  if (kNv == 2 && whole_spans(a.cols) && a.h != nullptr && a.h_out != nullptr && a.post && a.pre && (a.h_codes != nullptr) == (a.y_codes != nullptr) &&
      make_full_shape(a.cols, a.rows_per_piece, 4 * 256 * sizeof(T), kSumFloats<1>, &sh, &smem))
    return a.h_codes != nullptr ? start_rows(norm_forward_full_kernel<T, true>, done[0], a, sh, smem, ctas, stream)
                                : start_rows(norm_forward_full_kernel<T, false>, done[1], a, sh, smem, ctas, stream);
  const int limit = kNv == 2 ? kSmemLimit / 2 - 1024 : kSmemLimit;       // two CTAs per SM
  if (!make_shape(a.cols, a.rows_per_piece, 2 * 256 * sizeof(T), kSumFloats<1>, limit, &sh, &smem) &&
      !make_shape(a.cols, a.rows_per_piece, 2 * 256 * sizeof(T), kSumFloats<1>, kSmemLimit, &sh, &smem))
    return FALQON_ERR_UNSUPPORTED;
  return start_rows(norm_forward_rows_kernel<T, kNv>, done[2], a, sh, smem, ctas, stream);
}
template <typename T, bool kCoded, int kNv>
int launch_backward_rows(const NormArgs& a, int64_t ctas, cudaStream_t stream) {
  static DeviceMask done[2];
  Shape sh;
  size_t smem;
  const int set = 2 * 256 * sizeof(T) + 2 * 256 * (kCoded ? 1 : sizeof(T));
  if (kNv == 2 && whole_spans(a.cols) && (kCoded ? a.h_codes_in != nullptr : a.h != nullptr) && a.dx != nullptr && a.dh_out != nullptr && a.post && a.pre &&
      a.dh != nullptr && a.dy != nullptr && make_full_shape(a.cols, a.rows_per_piece, 2 * set, kSumFloats<3>, &sh, &smem))
    return start_rows(norm_backward_full_kernel<T, kCoded>, done[0], a, sh, smem, ctas, stream);
  if (!make_shape(a.cols, a.rows_per_piece, set, kSumFloats<3>, kSmemLimit, &sh, &smem)) return FALQON_ERR_UNSUPPORTED;
  return start_rows(norm_backward_rows_kernel<T, kCoded, kNv>, done[1], a, sh, smem, ctas, stream);
}
template <typename F>
int with_spans(int64_t cols, F go) {
  return spans_for(cols) == 2 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{});
}

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

int falqon_block_norm_forward(const falqon_block_norm* p, const void* h, const void* y, void* h_out, void* x, float* inv_post,
                              float* inv_pre, uint8_t* h_codes, uint8_t* h_scales, uint8_t* y_codes, uint8_t* y_scales,
                              float* amax_x, falqon_stream stream) {
  if (!plan_ok(p)) return FALQON_ERR_INVALID_ARG;
  NormArgs a = common(p);
  if (y == nullptr || !ok16(h) || !ok16(y) || !ok16(h_out) || !ok16(x) || !ok16(h_codes) || !ok16(y_codes) ||
      (h_codes != nullptr) != (h_scales != nullptr) || (y_codes != nullptr) != (y_scales != nullptr) ||
      (h_codes != nullptr && h == nullptr) || (a.post && inv_post == nullptr) || (a.pre && (x == nullptr || inv_pre == nullptr)) ||
      (!a.pre && h_out == nullptr))
    return FALQON_ERR_INVALID_ARG;
  a.h = h;
  a.y = y;
  a.h_out = h_out;
  a.x = a.pre ? x : nullptr;
  a.inv_post = inv_post;
  a.inv_pre = inv_pre;
  a.h_codes = h_codes;
  a.h_scales = h_scales;
  a.y_codes = y_codes;
  a.y_scales = y_scales;
  a.amax = a.pre ? amax_x : nullptr;
  if (staged(a.cols)) {
    const Split s(p, spans_for(a.cols) == 2 ? 2 * kNormUnits : kNormUnits);
    NormArgs b = a;
    s.put(&b);
    const int rc = with_spans(a.cols, [&](auto n) {
      return p->dtype == FALQON_BF16 ? launch_forward_rows<bf16_t, n.value>(b, s.ctas, static_cast<cudaStream_t>(stream))
                                     : launch_forward_rows<float, n.value>(b, s.ctas, static_cast<cudaStream_t>(stream));
    });
    if (rc != FALQON_ERR_UNSUPPORTED) return rc;
  }
  const int items = items_for(a.cols);
  const unsigned threads = static_cast<unsigned>(((a.cols + items - 1) / items + 31) / 32 * 32);
  const int64_t cap = static_cast<int64_t>(sm_count()) * 16;
  const unsigned grid = static_cast<unsigned>(a.rows < cap ? a.rows : cap);
  return with_items(items, [&](auto n) {
    return finish(p->dtype == FALQON_BF16 ? launch_pdl(norm_forward_kernel<bf16_t, n.value>, dim3(grid), dim3(threads), 0,
                                                       static_cast<cudaStream_t>(stream), 1, a)
                                          : launch_pdl(norm_forward_kernel<float, n.value>, dim3(grid), dim3(threads), 0,
                                                       static_cast<cudaStream_t>(stream), 1, a));
  });
}

size_t falqon_block_norm_scratch_bytes(const falqon_block_norm* p) {
  if (!plan_ok(p)) return 0;
  const Split s(p, backward_units(p->cols));
  return static_cast<size_t>(s.units + s.ctas) * static_cast<size_t>(p->cols) * sizeof(float);
}

int falqon_block_norm_backward(const falqon_block_norm* p, const void* dx, const void* dh_out, const void* h, const uint8_t* h_codes,
                               const uint8_t* h_scales, const void* y, const uint8_t* y_codes, const uint8_t* y_scales,
                               const float* inv_post, const float* inv_pre, void* dh, void* dy, float* dpost_gain, float* dpre_gain,
                               float* dgate, float* amax_dy, void* scratch, size_t scratch_bytes, falqon_stream stream) {
  if (!plan_ok(p)) return FALQON_ERR_INVALID_ARG;
  NormArgs a = common(p);
  const bool coded = y == nullptr;
  const bool residual = coded ? h_codes != nullptr : h != nullptr;
  if ((coded && (y_codes == nullptr || y_scales == nullptr || h != nullptr)) || (!coded && (y_codes != nullptr || h_codes != nullptr)) ||
      (h_codes != nullptr && h_scales == nullptr) || (a.pre && (dx == nullptr || inv_pre == nullptr)) || (!a.pre && dh_out == nullptr) ||
      (a.post && inv_post == nullptr) || (dh != nullptr && !residual) || (dh == nullptr && dy == nullptr && !dpost_gain && !dpre_gain && !dgate) ||
      (dh != nullptr && dh == dy) || (dpost_gain != nullptr && (!a.post || p->post_gain == nullptr)) ||
      (dpre_gain != nullptr && (!a.pre || p->pre_gain == nullptr)) || (dgate != nullptr && p->gate == nullptr) || !ok16(dx) ||
      !ok16(dh_out) || !ok16(h) || !ok16(h_codes) || !ok16(y) || !ok16(y_codes) || !ok16(dh) || !ok16(dy) || !ok16(dpost_gain) ||
      !ok16(dpre_gain) || !ok16(dgate) || (amax_dy != nullptr && dy == nullptr))
    return FALQON_ERR_INVALID_ARG;
  const Split s(p, backward_units(p->cols));
  const bool sums_s = dpost_gain != nullptr || dgate != nullptr, sums_p = dpre_gain != nullptr;
  if ((sums_s || sums_p) && (scratch == nullptr || !ok16(scratch) || scratch_bytes < falqon_block_norm_scratch_bytes(p)))
    return FALQON_ERR_WORKSPACE;
  a.dx = a.pre ? dx : nullptr;
  a.dh_out = dh_out;
  a.h = h;
  a.y = y;
  a.h_codes_in = h_codes;
  a.h_scales_in = h_scales;
  a.y_codes_in = y_codes;
  a.y_scales_in = y_scales;
  a.inv_post = const_cast<float*>(inv_post);
  a.inv_pre = const_cast<float*>(inv_pre);
  a.dh = dh;
  a.dy = dy;
  a.amax = amax_dy;
  s.put(&a);
  a.part_s = sums_s ? static_cast<float*>(scratch) : nullptr;
  a.part_p = sums_p ? static_cast<float*>(scratch) + s.units * a.cols : nullptr;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int rc = FALQON_ERR_UNSUPPORTED;
  if (staged(a.cols))
    rc = with_spans(a.cols, [&](auto n) {
      if (p->dtype == FALQON_BF16)
        return coded ? launch_backward_rows<bf16_t, true, n.value>(a, s.ctas, st) : launch_backward_rows<bf16_t, false, n.value>(a, s.ctas, st);
      return coded ? launch_backward_rows<float, true, n.value>(a, s.ctas, st) : launch_backward_rows<float, false, n.value>(a, s.ctas, st);
    });
  if (rc == FALQON_ERR_UNSUPPORTED) {                          // any other width, or rows that do not fit the ring
    const int items = items_for(a.cols);
    const dim3 grid(static_cast<unsigned>(s.ctas)), block(static_cast<unsigned>(((a.cols + items - 1) / items + 31) / 32 * 32));
    rc = with_items(items, [&](auto n) {
      return finish(p->dtype == FALQON_BF16 ? launch_pdl(norm_backward_kernel<bf16_t, n.value>, grid, block, 0, st, 1, a)
                                            : launch_pdl(norm_backward_kernel<float, n.value>, grid, block, 0, st, 1, a));
    });
  }
  if (rc != FALQON_OK || (!sums_s && !sums_p)) return rc;
  FinishArgs f{};
  f.part_s = a.part_s;
  f.part_p = a.part_p;
  f.post_gain = p->post_gain;
  f.gate = p->gate;
  f.dpost_gain = dpost_gain;
  f.dpre_gain = dpre_gain;
  f.dgate = dgate;
  f.cols = a.cols;
  f.groups = s.groups;
  f.pieces = s.pieces;
  f.ctas = s.ctas;
  f.gain_offset = a.gain_offset;
  f.post = a.post;
  f.gain_f32 = a.gain_f32;
  for (f.team = kFinishWarps; f.team > 1 && f.team * s.groups > kFinishWarps;) f.team /= 2;
  return finish(launch_pdl(a.cols % 4 == 0 ? norm_finish_kernel<true> : norm_finish_kernel<false>, dim3(static_cast<unsigned>((a.cols + 31) / 32)),
                           dim3(32 * kFinishWarps), 0, st, 1, f));
}

}  // extern "C"
