// The norms after and before a block, fused with the block's gate and the residual scale (include/falqon_train.h).
//   forward    n = y * ip * wpost;  H = s * h + gate * n;  x = H * iq * wpre
//   backward   xh = H * iq;  a = dx * wpre;  d = dh_out + iq * (a - xh * mean(a * xh));  dh = s * d
//              yh = y * ip;  b = q * d with q = gate * wpost;  dy = ip * (b - yh * mean(b * yh))
//              dwpre = sum_t dx * xh;  S_g = sum_{t in g} d * yh;  dgate_g = wpost * S_g;  dwpost = sum_g gate_g * S_g
// The two means of a row's backward come out of ONE reduction, because the second is linear in the first:
//   sum b * yh = sum q * yh * (dh_out + iq * a) - iq * mean(a * xh) * sum q * yh * xh.
// Both forms are off by roundings of sum |q * yh * (dh_out + iq * a)|; so a row whose d nearly cancels, because dx is nearly along x and dh_out
// is small, has a mean(b * yh) right to those terms' size and not to its own, as its d is itself.
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
  int64_t rows, cols, rows_per_gate, rows_per_piece;
  int units, pieces;                         // all units; those of a gate group
  float res_scale, gain_offset, eps, inv_cols;
  int post, pre, gain_f32;
};

__device__ __forceinline__ float gain_at(const void* p, int64_t i, int f32) {
  return f32 ? ld_stream(static_cast<const float*>(p) + i) : load1(static_cast<const bf16_t*>(p) + i);
}
__device__ __forceinline__ float weight_at(const void* p, int64_t i, const NormArgs& a) {
  return p == nullptr ? 1.0f : a.gain_offset + gain_at(p, i, a.gain_f32);
}

// The rows of a unit, which is a run of the rows of one gate group (32-bit division: a 64-bit one is a hundred instructions).
struct Unit {
  int gate, first, last;                                       // at most FALQON_NORM_MAX_ROWS, so that a row number plus what is looked ahead (64) fits
  __device__ __forceinline__ Unit(const NormArgs& a, int unit) {
    gate = unit / a.pieces;
    const int64_t begin = gate * a.rows_per_gate + (unit - gate * a.pieces) * a.rows_per_piece;
    first = static_cast<int>(min(begin, a.rows));
    last = static_cast<int>(min(min(begin + a.rows_per_piece, (gate + 1) * a.rows_per_gate), a.rows));
  }
};

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

// ---- rows that do not fit in shared memory: a CTA takes a row at a time, a thread kItems single columns tid, tid + threads, .. in registers,
// and a checkpoint's block is a warp.  Nothing is fetched ahead: bf16 4096 x 4096 would take 357 us forward and 1300 backward from
// checkpoints, where the staged kernels take 37 and 54.  The widest rows that are staged, of multiples of 16 / of other widths:
//   forward   bf16 all / all;  fp32 all / 14335
//   backward  bf16 from checkpoints all / 16350, from bf16 all / 14431;  fp32 from checkpoints all / 12742, from fp32 14432 / 9624
constexpr int kItems = 16;   // of up to 1024 threads: FALQON_NORM_MAX_COLS
// Squares are divided by the width before they are added, so that only a mean beyond fp32's range overflows.
__global__ void __launch_bounds__(1024, 1) norm_forward_f32_kernel(const NormArgs a) {
  using T = float;                                             // bf16 rows always fit
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

template <typename T>
__global__ void __launch_bounds__(1024, 1) norm_backward_kernel(const NormArgs a) {
  __shared__ float red[2 * 3 * 32];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  uint32_t mx = 0;
  const int64_t blocks_per_row = (a.cols + kMx8Block - 1) / kMx8Block;
  float P[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) P[i] = 0.0f;
  for (int64_t unit = blockIdx.x; unit < a.units; unit += gridDim.x) {
    const Unit u(a, static_cast<int>(unit));
    const int64_t group = u.gate, first = u.first, last = u.last;
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

// ---- forward, widths that are multiples of 16: rows stream through shared memory
// A row belongs to a group of whole warps; a warp has kNv neighbouring spans of 256 columns, a lane eight columns of each.
// Every warp copies its own spans of the next rows with 16-byte asynchronous copies into a ring of `depth` stages that only
// it reads, so the copies in flight cost no registers and no barrier.  Several rows at a time: while one group waits for its
// row's sums, the others compute.  Arithmetic is two values per instruction (f32x2, each half an ordinary rounded operation),
// since a row's instructions, not its bytes, were the limit without it.
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
// cp.async.wait_group takes a constant: at most depth - 1 younger groups may be open.
__device__ __forceinline__ void wait_stage(int depth) {
  switch (depth) {
    case 1: cp_async_wait<0>(); break;
    case 2: cp_async_wait<1>(); break;
    case 3: cp_async_wait<2>(); break;
    default: cp_async_wait<3>(); break;
  }
}

// The sum over a row group of up to 16 warps; every thread gets it.  `red`: the group's kSumFloats, zero before the first call (a warp
// that is not there adds 0): two halves used in turn, so that one barrier per call is enough.
constexpr int kSumFloats = 2 * 16;
__device__ __forceinline__ float group_sum(float v, float* red, int& phase, int warp, int lane, int warps, int barrier) {
  constexpr uint32_t all = 0xFFFFFFFFu;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(all, v, o);
  if (warps == 1) return v;
  float* buf = red + phase;
  phase ^= 16;
  if (lane == 0) buf[warp] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(warps * 32) : "memory");
  const bool many = warps > 8;
  v = buf[lane & (many ? 15 : 7)];
  if (many) v += __shfl_xor_sync(all, v, 8);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(all, v, o);
  return v;
}
// Clears a CTA's reduction space.
__device__ __forceinline__ void clear_sums(float* red, int floats) {
  for (int i = threadIdx.x; i < floats; i += blockDim.x) red[i] = 0.0f;
  __syncthreads();
}

// A load that leaves the value as it is where there is nothing to fetch: no branch, so nothing waits for it before its use.
__device__ __forceinline__ void fetch_if(bool there, float& v, const float* p) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q ld.global.cg.f32 %0, [%1];\n\t}" : "+f"(v) : "l"(p), "r"(static_cast<int>(there)));
}
__device__ __forceinline__ void fetch_if(bool there, uint32_t& v, const uint8_t* p) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q ld.global.cg.u8 %0, [%1];\n\t}" : "+r"(v) : "l"(p), "r"(static_cast<int>(there)));
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

// What a thread knows of its place.
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
  clear_sums(tail, sh.groups * kSumFloats);
  float* red = tail + me.group * kSumFloats;
  float* wsm = tail + sh.groups * kSumFloats;
  constexpr int kSpan = 256 * sizeof(T);                       // bytes of a span; a stage holds [span][y, h]
  const int units = a.units;
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
      float ip = 1.0f;
      if (post) {
        ip = rsqrtf(group_sum(halves(ss), red, phase, me.warp, lane, me.warps, me.group + 1) + a.eps);
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
        const float iq = rsqrtf(group_sum(halves(ss), red, phase, me.warp, lane, me.warps, me.group + 1) + a.eps);
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

// ---- forward, the full call: both norms, a residual, every result, rows of 1024 columns per warp (1024, 2048, .. 8192)
// The same work with nothing left to test in the row loop and offsets that advance by a row; four spans a lane (a row of 4096 columns
// is 128 threads, four rows a CTA), so that a row's two reductions are shared by 1024 columns a warp.  HBM-bound as far as
// instructions allow: 4096 x 4096 bf16 with both checkpoints 36.5 us (4.6 TB/s of what it must move; two spans a lane and two CTAs per
// SM 42; the kernel above, for any call, 52), 8192 x 8192 without 98 us (5.5 TB/s; the kernel above 149).
constexpr int kFullDepth = 2;                                  // two rows ahead per group cover the latency
constexpr int kFullSpans = 4;

template <typename T, int kNv>
__device__ __forceinline__ void copy_lane(uint32_t dst, const T* src) {   // kNv spans of 256 columns; src: the lane's first value
  constexpr int n = 16 / sizeof(T) * 32;                       // columns per instruction
#pragma unroll
  for (int j = 0; j < kNv * 256 / n; ++j) cp_async16(dst + 512 * j, src + n * j);
}

template <typename T, bool kCodes>
__global__ void __launch_bounds__(512, 1) norm_forward_full_kernel(const NormArgs a, const Shape sh) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_trigger();
  pdl_wait();
  constexpr int kNv = kFullSpans;
  constexpr int kSpan = 256 * sizeof(T), kStage = 2 * kNv * kSpan;   // a stage holds [y, h][span]
  const Seat me(sh);
  const int cols = sh.cols, lane = me.lane, c0 = me.column<kNv>(), groups = sh.groups;
  const uint8_t* ring = smem + (threadIdx.x >> 5) * (kFullDepth * kStage);
  const uint32_t ring_lane = smem_u32(ring) + lane * 16;
  float* const tail = reinterpret_cast<float*>(smem + (blockDim.x >> 5) * (kFullDepth * kStage));
  clear_sums(tail, sh.groups * kSumFloats);
  float* red = tail + me.group * kSumFloats;
  float* wsm = tail + groups * kSumFloats;
  const int units = a.units;
  const int64_t step = static_cast<int64_t>(groups) * cols;
  const int lane_shift = sizeof(T) == 2 ? 0 : -4 * lane;       // from a lane's first column to what it copies
  int phase = 0;
  Largest<T> largest;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u(a, unit);
    int row = u.first + me.group;
    int64_t at = static_cast<int64_t>(row) * cols + c0;
    const auto copy = [&](int64_t from, uint32_t dst) {
      copy_lane<T, kNv>(dst, static_cast<const T*>(a.y) + from + lane_shift);
      copy_lane<T, kNv>(dst + kNv * kSpan, static_cast<const T*>(a.h) + from + lane_shift);
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
      f2 y[kNv][4], H[kNv][4], ss = 0;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        read_span<T>(src + i * kSpan, lane, y[i]);
        read_span<T>(src + (kNv + i) * kSpan, lane, H[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) ss = fma2(mul2(y[i][k], twice(a.inv_cols)), y[i][k], ss);
      }
      __syncwarp();                                            // the warp has read its stage
      if (row + kFullDepth * groups < u.last) copy(at + kFullDepth * step, ring_lane + stage);
      cp_async_commit();
      if (kCodes) {
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          put_codes8(H[i], a.h_codes + at + i * 256, a.h_scales + (at >> 5) + i * 8, true, lane);
          put_codes8(y[i], a.y_codes + at + i * 256, a.y_scales + (at >> 5) + i * 8, true, lane);
        }
      }
      const float ip = rsqrtf(group_sum(halves(ss), red, phase, me.warp, lane, me.warps, me.group + 1) + a.eps);
      ss = 0;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        f2 q[4];
        weights_of(wsm, c0 + i * 256, q);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          H[i][k] = fma2(twice(a.res_scale), H[i][k], mul2(mul2(y[i][k], twice(ip)), q[k]));
          ss = fma2(mul2(H[i][k], twice(a.inv_cols)), H[i][k], ss);
        }
        write8(static_cast<T*>(a.h_out) + at + i * 256, H[i]);
      }
      const float iq = rsqrtf(group_sum(halves(ss), red, phase, me.warp, lane, me.warps, me.group + 1) + a.eps);
      if (c0 == 0) {
        a.inv_post[row] = ip;
        a.inv_pre[row] = iq;
      }
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        f2 w[4];
        weights_of(wsm, cols + c0 + i * 256, w);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = mul2(mul2(H[i][k], twice(iq)), w[k]);
        const Vec8<T> o = write8(static_cast<T*>(a.x) + at + i * 256, w);
        if (a.amax != nullptr) largest.see(o);
      }
    }
  }
  if (a.amax != nullptr) raise_amax(largest.bits(), a.amax);
}

// ---- any width: the same rings and runs with single values
// Rows begin anywhere, so a copy takes the 16-byte pieces that cover its values (of the neighbouring rows' values a few come along and
// are not looked at), and in shared memory lanes read single values: value e of a lane in a span is column 32 * e + lane, so that
// neighbouring lanes read and write neighbouring values, and every e is one block of a checkpoint.  Bound by instructions, single values
// taking eight times the accesses: bf16 4096 x 4095 with checkpoints 78 us forward and 108 backward, where 4096 x 4096 takes 37 and 54
// (and by these kernels about as long as 4095).
__device__ __forceinline__ float single_at(uint32_t at, bf16_t) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
  return bf16_bits_to_float(v);
}
__device__ __forceinline__ float single_at(uint32_t at, float) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
  return v;
}
__device__ __forceinline__ uint32_t byte_at(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}
// A lane's eight values of a span whose first lies at `at`; `left`: columns from it to the row's end.
template <typename T>
__device__ __forceinline__ void read_singles(uint32_t at, int left, int lane, f2 (&x)[4]) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e * 32 + lane < left ? single_at(at + (e * 32 + lane) * static_cast<int>(sizeof(T)), T{}) : 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = pack_f32x2(v[2 * k], v[2 * k + 1]);
}
// The same of eight codes: not yet multiplied by their scales.
__device__ __forceinline__ void read_single_codes(uint32_t at, int left, int lane, f2 (&x)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t lo = 64 * k + lane < left ? byte_at(at + 64 * k + lane) : 0u, hi = 64 * k + 32 + lane < left ? byte_at(at + 64 * k + 32 + lane) : 0u;
    const float2 f = e4m3x2_to_float2(lo | hi << 8);
    x[k] = pack_f32x2(f.x, f.y);
  }
}
__device__ __forceinline__ void read_single_weights(const float* w, int left, int lane, f2 (&x)[4]) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e * 32 + lane < left ? w[e * 32 + lane] : 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = pack_f32x2(v[2 * k], v[2 * k + 1]);
}
template <typename T>
__device__ __forceinline__ uint32_t write_singles(T* p, int left, int lane, const f2 (&x)[4]) {   // the largest |value| stored, as bits
  uint32_t m = 0u;
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(x[k], v[2 * k], v[2 * k + 1]);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e * 32 + lane < left) m = max(m, store1(p + e * 32 + lane, v[e]));
  return m;
}
__device__ __forceinline__ void put_single_codes(const f2 (&x)[4], int left, int lane, uint8_t* codes, uint8_t* scales) {
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(x[k], v[2 * k], v[2 * k + 1]);
  uint32_t top = 0u;                                           // of block `lane`: lane e works out the scale of block e for all
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, abs_bits(v[e]));
    if (lane == e) top = m;
  }
  const uint32_t e8 = mx8_exponent(top);
  const float factor = mx8_encode_factor(e8);
  if (lane < 8 && lane * 32 < left) scales[lane] = static_cast<uint8_t>(e8);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float f = __shfl_sync(0xFFFFFFFFu, factor, e);
    if (e * 32 + lane < left) codes[e * 32 + lane] = mx8_encode1(v[e], f);
  }
}
// Copies the 16-byte pieces that cover the 256 values from `at` on, of a tensor of `total` values: the first value lies offset_of(at)
// bytes behind dst then.
template <typename T>
__device__ __forceinline__ uint32_t offset_of(int64_t at) {
  return static_cast<uint32_t>(at * static_cast<int64_t>(sizeof(T))) & 15u;
}
template <typename T>
__device__ __forceinline__ void copy_loose(uint32_t dst, const T* base, int64_t at, int64_t total, int lane) {
  const int64_t from = at * static_cast<int64_t>(sizeof(T)) & ~static_cast<int64_t>(15), end = total * static_cast<int64_t>(sizeof(T));
#pragma unroll
  for (int ch = lane; ch < 256 * static_cast<int>(sizeof(T)) / 16 + 1; ch += 32) {
    const int64_t left = end - (from + ch * 16);
    if (left <= 0) break;
    const int bytes = left < 16 ? static_cast<int>(left) : 16;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + ch * 16), "l"(reinterpret_cast<const uint8_t*>(base) + from + ch * 16), "r"(bytes)
                 : "memory");
  }
}
__device__ __forceinline__ void fill_weights_singly(const NormArgs& a, int64_t group, float* wsm, int cols) {
  __syncthreads();
  for (int c = threadIdx.x; c < cols; c += blockDim.x) {
    const float q = a.post ? weight_at(a.post_gain, c, a) : 1.0f;
    wsm[c] = a.gate != nullptr ? q * gain_at(a.gate, group * cols + c, a.gain_f32) : q;
    wsm[cols + c] = a.pre ? weight_at(a.pre_gain, c, a) : 1.0f;
  }
  __syncthreads();
}

template <typename T, int kNv>
__global__ void __launch_bounds__(512) norm_forward_loose_kernel(const NormArgs a, const Shape sh) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_trigger();
  pdl_wait();
  const bool has_h = a.h != nullptr;
  const Seat me(sh);
  const int cols = sh.cols, lane = me.lane, c0 = me.warp * kNv * 256;
  const int64_t blocks_per_row = (cols + kMx8Block - 1) / kMx8Block, total = a.rows * cols;
  const uint32_t ring = smem_u32(smem) + (threadIdx.x >> 5) * sh.depth * sh.warp_stage;
  float* const tail = reinterpret_cast<float*>(smem + static_cast<size_t>(blockDim.x >> 5) * sh.depth * sh.warp_stage);
  clear_sums(tail, sh.groups * kSumFloats);
  float* red = tail + me.group * kSumFloats;
  float* wsm = tail + sh.groups * kSumFloats;
  constexpr int kSpan = 256 * sizeof(T) + 16;                  // bytes of a span and what comes along; a stage holds [span][y, h]
  const int units = a.units;
  const f2 inv_cols = twice(a.inv_cols);
  int phase = 0;
  uint32_t mx = 0;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u(a, unit);
    const auto issue = [&](int row, int stage) {
      if (row < u.last) {
        const uint32_t dst = ring + stage * sh.warp_stage;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          if (c0 + i * 256 >= cols) continue;
          const int64_t at = static_cast<int64_t>(row) * cols + c0 + i * 256;
          copy_loose(dst + i * 2 * kSpan, static_cast<const T*>(a.y), at, total, lane);
          if (has_h) copy_loose(dst + (i * 2 + 1) * kSpan, static_cast<const T*>(a.h), at, total, lane);
        }
      }
      cp_async_commit();
    };
    for (int s = 0; s < sh.depth; ++s) issue(u.first + me.group + s * sh.groups, s);
    fill_weights_singly(a, u.gate, wsm, cols);
    int stage = 0;
    for (int row = u.first + me.group; row < u.last; row += sh.groups) {
      const int64_t at = static_cast<int64_t>(row) * cols + c0;
      wait_stage(sh.depth);
      __syncwarp();
      const uint32_t src = ring + stage * sh.warp_stage;
      f2 y[kNv][4], H[kNv][4], ss = 0;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        const int left = cols - c0 - i * 256;                  // of a span beyond the row: none
        const uint32_t off = offset_of<T>(at + i * 256);
        read_singles<T>(src + i * 2 * kSpan + off, left, lane, y[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) H[i][k] = 0;
        if (has_h) read_singles<T>(src + (i * 2 + 1) * kSpan + off, left, lane, H[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) ss = fma2(mul2(y[i][k], inv_cols), y[i][k], ss);
      }
      __syncwarp();                                            // the warp has read its stage
      issue(row + sh.depth * sh.groups, stage);
      stage = stage + 1 == sh.depth ? 0 : stage + 1;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        const int left = cols - c0 - i * 256;
        if (left <= 0) continue;
        const int64_t block = row * blocks_per_row + (c0 + i * 256) / kMx8Block;
        if (a.h_codes != nullptr) put_single_codes(H[i], left, lane, a.h_codes + at + i * 256, a.h_scales + block);
        if (a.y_codes != nullptr) put_single_codes(y[i], left, lane, a.y_codes + at + i * 256, a.y_scales + block);
      }
      float ip = 1.0f;
      if (a.post) {
        ip = rsqrtf(group_sum(halves(ss), red, phase, me.warp, lane, me.warps, me.group + 1) + a.eps);
        if (me.warp == 0 && lane == 0) a.inv_post[row] = ip;
      }
      ss = 0;
#pragma unroll
      for (int i = 0; i < kNv; ++i) {
        const int left = cols - c0 - i * 256;
        if (left <= 0) continue;
        f2 q[4];
        read_single_weights(wsm + c0 + i * 256, left, lane, q);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f2 n = mul2(mul2(y[i][k], twice(ip)), q[k]);
          H[i][k] = has_h ? fma2(twice(a.res_scale), H[i][k], n) : n;
          ss = fma2(mul2(H[i][k], inv_cols), H[i][k], ss);
        }
        if (a.h_out != nullptr) write_singles(static_cast<T*>(a.h_out) + at + i * 256, left, lane, H[i]);
      }
      if (a.pre) {
        const float iq = rsqrtf(group_sum(halves(ss), red, phase, me.warp, lane, me.warps, me.group + 1) + a.eps);
        if (me.warp == 0 && lane == 0) a.inv_pre[row] = iq;
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          const int left = cols - c0 - i * 256;
          if (left <= 0) continue;
          f2 w[4];
          read_single_weights(wsm + cols + c0 + i * 256, left, lane, w);
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = mul2(mul2(H[i][k], twice(iq)), w[k]);
          mx = max(mx, write_singles(static_cast<T*>(a.x) + at + i * 256, left, lane, w));
        }
      }
    }
  }
  if (a.amax != nullptr) raise_amax(mx, a.amax);
}

// ---- backward, widths that are multiples of 16: runs of rows through shared memory
// A CTA brings R neighbouring rows of all four tensors into shared memory by bulk copies (a run of rows is one run of bytes), two runs
// in turn.  First its warps share the rows, for the three sums of each; then they share the columns ("stripes" of 256, eight to a
// lane), every warp going through all rows of the run with its columns' weights and sums in registers.  So a row's reduction is
// a part of a warp's, there are two barriers per run instead of one per row, and no thread holds a row's values while it waits.  The
// values are formed twice, from shared memory.  In the terms of the file's head, with H in the place of xh = H * iq:
//   t = dx * w;  g = dh_out + iq * t;  b = q * yh;  A = sum t * H, B = sum b * g, C = sum b * H
//   d = g - k1 * H with k1 = iq^3 * A / cols;  dy = ip * (q * d - yh * k2) with k2 = (B - k1 * C) / cols
// Bound by instructions, since every value is decoded and formed twice, and by warps that the shares leave without work (issued on 48 % of
// cycles by 16 warps, the most whose registers and shared memory fit: of 4096 columns from checkpoints a run is 3 rows, whose sums 12 warps share;
// of 5120 columns, two stripes to a warp, 10 write the results): 4096 x 4096 from checkpoints 54 us with the finish below (3.1 TB/s of what it
// must move), 8192 x 5120 from bf16 121 us (4.2 TB/s).  Rows in registers from the sums to the results, a barrier per row: 57 and 150 us.
constexpr int kMaxRun = 32;                                    // a lane per row
constexpr int kScaleBytes = 4;                                 // of a run, per thread
struct Run {
  int cols, stripes, warps, run, parts, part_spans, split, stripe_warps, buffers, weights_in_smem, blocks_per_row;
  int area, saved_area, buffer;                                // bytes: of a run of dx, of h or y, of a buffer
  int scale_bytes;                                             // of all scales; 0 where h and y are saved as they are
};
// Shared memory behind the buffers.
struct RunTail {
  float* wsm;                                                  // [2][cols]
  float4* red;                                                 // [run][parts]
  uint8_t* scales;                                             // [2][h, y][run * blocks_per_row]
  uint32_t full;                                               // mbarriers, one per buffer
};
__device__ __host__ __forceinline__ size_t run_tail_bytes(const Run& r) {
  return 16 + static_cast<size_t>(r.run) * r.parts * 16 + r.scale_bytes + (r.weights_in_smem ? static_cast<size_t>(r.cols) * 8 : 0);
}

// Eight values of a run in shared memory.
template <typename T>
__device__ __forceinline__ void read8(uint32_t at, f2 (&x)[4]) {
  if constexpr (sizeof(T) == 2) {
    uint32_t w[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = pack_f32x2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u));
  } else {
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(x[0]), "=l"(x[1]) : "r"(at));
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(x[2]), "=l"(x[3]) : "r"(at + 16));
  }
}
// The same of a saved tensor, not yet multiplied by its scale.
template <typename T, bool kCoded>
__device__ __forceinline__ void read_saved(uint32_t at, f2 (&x)[4]) {
  if constexpr (kCoded) {
    uint32_t w[2];
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    decode4(w[0], x[0], x[1]);
    decode4(w[1], x[2], x[3]);
  } else {
    read8<T>(at, x);
  }
}
// Where a lane's eight columns of a row lie in shared memory: dx (dh_out is `area` further), h (y `saved_area` further), the scale of h
// (y's `half` further).
struct Spot {
  uint32_t dx, h, scale;
};

// kLoose: the 16-byte pieces that cover n rows from `row` on, into a run's buffer, as bulk copies by one lane; values in a last piece
// that the tensor does not fill are copied singly by the warp (they are read after a barrier or more).
template <typename V>
__device__ __forceinline__ uint32_t loose_bytes(int64_t at, int64_t count, int64_t total) {   // of the whole pieces
  const int64_t from = at * static_cast<int64_t>(sizeof(V)) & ~static_cast<int64_t>(15), whole = total * static_cast<int64_t>(sizeof(V)) & ~static_cast<int64_t>(15);
  const int64_t end = ((at + count) * static_cast<int64_t>(sizeof(V)) + 15) & ~static_cast<int64_t>(15);
  return static_cast<uint32_t>(max(min(end, whole) - from, static_cast<int64_t>(0)));
}
template <typename V>
__device__ __forceinline__ void loose_copy(uint8_t* dst, const V* base, int64_t at, int64_t count, int64_t total, uint32_t bar, int lane) {
  const uint8_t* src = reinterpret_cast<const uint8_t*>(base);
  const int64_t from = at * static_cast<int64_t>(sizeof(V)) & ~static_cast<int64_t>(15);
  const uint32_t bytes = loose_bytes<V>(at, count, total);
  if (lane == 0 && bytes > 0) bulk_load_1d(smem_u32(dst), src + from, bytes, bar);
  const int64_t rest = (at + count) * static_cast<int64_t>(sizeof(V)) - (from + bytes);       // bytes, less than 16
  if (lane < rest / static_cast<int64_t>(sizeof(V)))
    reinterpret_cast<V*>(dst + bytes)[lane] = ld_stream(reinterpret_cast<const V*>(src + from + bytes) + lane);
}
template <typename T, bool kCoded>
__device__ __forceinline__ void bring_loose(const NormArgs& a, const Run& sh, int row, int n, bool has_h, bool has_dx, bool has_g, uint8_t* buf, uint32_t bar) {
  using V = std::conditional_t<sizeof(T) == 2, uint16_t, float>;
  using S = std::conditional_t<kCoded, uint8_t, V>;
  const int lane = threadIdx.x & 31;
  const int64_t at = static_cast<int64_t>(row) * sh.cols, count = static_cast<int64_t>(n) * sh.cols, total = a.rows * sh.cols;
  const S* h = static_cast<const S*>(kCoded ? static_cast<const void*>(a.h_codes_in) : a.h);
  const S* y = static_cast<const S*>(kCoded ? static_cast<const void*>(a.y_codes_in) : a.y);
  if (lane == 0)
    mbar_expect_tx(bar, (has_dx + has_g) * loose_bytes<V>(at, count, total) + (1 + has_h) * loose_bytes<S>(at, count, total));
  __syncwarp();
  if (has_dx) loose_copy(buf, static_cast<const V*>(a.dx), at, count, total, bar, lane);
  if (has_g) loose_copy(buf + sh.area, static_cast<const V*>(a.dh_out), at, count, total, bar, lane);
  if (has_h) loose_copy(buf + 2 * sh.area, h, at, count, total, bar, lane);
  loose_copy(buf + 2 * sh.area + sh.saved_area, y, at, count, total, bar, lane);
}

// The sums of one stripe's columns over the warps that shared its rows, added in their order through shared memory, to out[cols].
template <int kNv, bool kLoose>
__device__ __forceinline__ void store_stripes(const f2 (&v)[kNv][4], float* out, float* space, const Run& sh, int stripe, int member) {
  const int lane = threadIdx.x & 31;
  if (sh.split > 1) __syncthreads();
#pragma unroll
  for (int i = 0; i < kNv; ++i) {
    if (kLoose) {
      const int c = (stripe + i) * 256;
      if (member < sh.split && c < sh.cols) write_singles((sh.split > 1 ? space + member * sh.cols : out) + c, sh.cols - c, lane, v[i]);
      continue;
    }
    const int c = (stripe + i) * 256 + lane * 8;
    if (member >= sh.split || c >= sh.cols) continue;
    ulonglong2* to = reinterpret_cast<ulonglong2*>((sh.split > 1 ? space + member * sh.cols : out) + c);
    to[0] = make_ulonglong2(v[i][0], v[i][1]);
    to[1] = make_ulonglong2(v[i][2], v[i][3]);
  }
  if (sh.split == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < sh.cols; c += blockDim.x) {
    float t = 0.0f;
    for (int m = 0; m < sh.split; ++m) t += space[m * sh.cols + c];
    out[c] = t;
  }
  fence_proxy_async_smem();                                    // bulk copies write here next
  __syncthreads();
}

template <typename T, bool kCoded, int kNv, bool kFull, bool kLoose>
__global__ void __launch_bounds__(512) norm_backward_run_kernel(const NormArgs a, const Run sh, int* status) {
  extern __shared__ __align__(128) uint8_t smem[];
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cols = sh.cols;
  RunTail tail;
  {
    uint8_t* p = smem + static_cast<size_t>(sh.buffers) * sh.buffer;
    tail.full = smem_u32(p);
    tail.red = reinterpret_cast<float4*>(p + 16);
    tail.scales = p + 16 + static_cast<size_t>(sh.run) * sh.parts * 16;
    tail.wsm = reinterpret_cast<float*>(tail.scales + sh.scale_bytes);
  }
  if (tid == 0) {
    for (int b = 0; b < sh.buffers; ++b) mbar_init(tail.full + 8 * b, 1);
    mbar_fence_init();
  }
  __syncthreads();
  pdl_wait();
  const bool post = kFull || a.post, pre = kFull || a.pre, want_dh = kFull || a.dh != nullptr, want_dy = kFull || a.dy != nullptr;
  const bool has_h = kFull || (kCoded ? a.h_codes_in != nullptr : a.h != nullptr), has_dx = kFull || a.dx != nullptr, has_g = kFull || a.dh_out != nullptr;
  const int stripe = (warp % sh.stripe_warps) * kNv, member = warp / sh.stripe_warps;
  const int units = a.units;
  const int half = sh.run * sh.blocks_per_row;                 // scale bytes of one tensor's run
  const int lane_col = kLoose ? 0 : lane * 8;                  // of a span: the lane's first column, or where all lanes begin
  uint32_t mx = 0;
  Largest<T> largest;
  uint32_t parity = 0;                                         // of each buffer's next wait, a bit
  f2 P[kNv][4];
#pragma unroll
  for (int i = 0; i < kNv; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) P[i][k] = 0;

  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const Unit u(a, unit);
    const int runs = (u.last - u.first + sh.run - 1) / sh.run;
    const auto bring = [&](int c, int b) {                     // one thread (kLoose: one warp): the c-th run into buffer b
      if (c >= runs) return;
      if constexpr (kLoose) return bring_loose<T, kCoded>(a, sh, u.first + c * sh.run, min(sh.run, u.last - (u.first + c * sh.run)), has_h, has_dx, has_g,
                                                          smem + b * sh.buffer, tail.full + 8 * b);
      const int row = u.first + c * sh.run, n = min(sh.run, u.last - row);
      const int64_t at = static_cast<int64_t>(row) * cols;
      const uint32_t dst = smem_u32(smem) + b * sh.buffer, bar = tail.full + 8 * b, bytes = n * cols * static_cast<int>(sizeof(T));
      const uint32_t saved = kCoded ? n * cols : bytes;
      mbar_expect_tx(bar, (has_dx ? bytes : 0) + (has_g ? bytes : 0) + (has_h ? saved : 0) + saved);
      if (has_dx) bulk_load_1d(dst, static_cast<const T*>(a.dx) + at, bytes, bar);
      if (has_g) bulk_load_1d(dst + sh.area, static_cast<const T*>(a.dh_out) + at, bytes, bar);
      const uint8_t *h = kCoded ? a.h_codes_in : static_cast<const uint8_t*>(a.h), *y = kCoded ? a.y_codes_in : static_cast<const uint8_t*>(a.y);
      constexpr int kBytes = kCoded ? 1 : sizeof(T);
      if (has_h) bulk_load_1d(dst + 2 * sh.area, h + at * kBytes, saved, bar);
      bulk_load_1d(dst + 2 * sh.area + sh.saved_area, y + at * kBytes, saved, bar);
    };
    const bool courier = kLoose ? warp == 0 : tid == 0;
    if (courier)
      for (int b = 0; b < sh.buffers; ++b) bring(b, b);
    // what else a run needs, fetched one run ahead: a lane's row's factors, and the scales
    float ip_next = 1.0f, iq_next = 0.0f;
    uint32_t scale_next[kScaleBytes] = {0u, 0u, 0u, 0u};
    const auto fetch = [&](int c) {
      const int row = u.first + c * sh.run, n = min(sh.run, u.last - row);
      if (post) fetch_if(lane < n, ip_next, a.inv_post + row + lane);
      if (pre) fetch_if(lane < n, iq_next, a.inv_pre + row + lane);
      if (kCoded) {
        const int count = n * sh.blocks_per_row;
        const int64_t at = static_cast<int64_t>(row) * sh.blocks_per_row;
#pragma unroll
        for (int j = 0; j < kScaleBytes; ++j) {
          const int i = tid + j * blockDim.x;                  // h's bytes of the run, then y's
          const bool of_y = i >= half;
          const int k = of_y ? i - half : i;
          fetch_if(i < 2 * half && k < count && (of_y || has_h), scale_next[j], (of_y ? a.y_scales_in : a.h_scales_in) + at + k);
        }
      }
    };
    const auto keep = [&](int b) {
      if (!kCoded) return;
#pragma unroll
      for (int j = 0; j < kScaleBytes; ++j)
        if (tid + j * static_cast<int>(blockDim.x) < 2 * half) tail.scales[b * 2 * half + tid + j * blockDim.x] = static_cast<uint8_t>(scale_next[j]);
    };
    fetch(0);
    keep(0);
    if (kLoose) fill_weights_singly(a, u.gate, tail.wsm, cols);
    else if (kFull || sh.weights_in_smem) fill_weights(a, u.gate, tail.wsm, cols);
    else __syncthreads();
    const Weights weights{a, tail.wsm, u.gate, cols, sh.weights_in_smem};
    const auto get = [&](int col, f2 (&q)[4], f2 (&w)[4]) {
      if (kLoose) {
        read_single_weights(tail.wsm + col, cols - col, lane, q);
        read_single_weights(tail.wsm + cols + col, cols - col, lane, w);
      } else if (kFull) {                                      // then they are in shared memory
        weights_of(tail.wsm, col, q);
        weights_of(tail.wsm, cols + col, w);
      } else {
        weights.get(0, col, q);
        weights.get(1, col, w);
      }
    };
    f2 S[kNv][4], q[4], w[4];
#pragma unroll
    for (int i = 0; i < kNv; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) S[i][k] = 0;

    for (int c = 0, b = 0; c < runs; ++c, b = b + 1 == sh.buffers ? 0 : b + 1) {
      const int row0 = u.first + c * sh.run, n = min(sh.run, u.last - row0);
      const float ip_lane = ip_next, iq_lane = iq_next;
      if (c + 1 < runs) fetch(c + 1);
      mbar_wait(tail.full + 8 * b, parity >> b & 1, status);
      parity ^= 1u << b;
      constexpr int kBytes = kCoded ? 1 : sizeof(T);
      const int64_t run_at = static_cast<int64_t>(row0) * cols;
      const uint32_t off_v = kLoose ? offset_of<T>(run_at) : 0u, off_s = kLoose ? (kCoded ? offset_of<uint8_t>(run_at) : off_v) : 0u;
      const auto spot = [&](int r, int col) {
        const int at = r * cols + col;
        const uint32_t buf = smem_u32(smem) + b * sh.buffer;
        return Spot{buf + off_v + at * static_cast<int>(sizeof(T)), buf + off_s + 2 * sh.area + at * kBytes,
                    smem_u32(tail.scales) + (c & 1) * 2 * half + r * sh.blocks_per_row + (col >> 5)};
      };
      // of a lane's columns: yh (y times its scale and ip), b = q * yh, H, and t = dx * w with g = dh_out + iq * t
      // (kLoose: of a span's columns, of which `left` lie in the row)
      const auto form = [&](const Spot& p, int left, float ip, float iq, f2 (&yh)[4], f2 (&b4)[4], f2 (&H)[4], f2 (&dx)[4], f2 (&t)[4], f2 (&g)[4]) {
        if constexpr (kLoose) {
          f2 fy[4], fh[4];
          if (kCoded) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const bool one = 64 * k < left, two = 64 * k + 32 < left;
              fy[k] = pack_f32x2(one ? scale_of(byte_at(p.scale + half + 2 * k)) * ip : 0.0f, two ? scale_of(byte_at(p.scale + half + 2 * k + 1)) * ip : 0.0f);
              fh[k] = has_h ? pack_f32x2(one ? scale_of(byte_at(p.scale + 2 * k)) * a.res_scale : 0.0f,
                                         two ? scale_of(byte_at(p.scale + 2 * k + 1)) * a.res_scale : 0.0f) : 0;
            }
            read_single_codes(p.h + sh.saved_area, left, lane, yh);
            if (has_h) read_single_codes(p.h, left, lane, H);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) fy[k] = twice(ip), fh[k] = twice(a.res_scale);
            read_singles<T>(p.h + sh.saved_area, left, lane, yh);
            if (has_h) read_singles<T>(p.h, left, lane, H);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            yh[k] = mul2(yh[k], fy[k]);
            b4[k] = mul2(q[k], yh[k]);
            H[k] = has_h ? fma2(H[k], fh[k], b4[k]) : b4[k];
            g[k] = dx[k] = t[k] = 0;
          }
          if (has_g) read_singles<T>(p.dx + sh.area, left, lane, g);
          if (has_dx) {
            read_singles<T>(p.dx, left, lane, dx);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              t[k] = mul2(dx[k], w[k]);
              g[k] = fma2(t[k], twice(iq), g[k]);
            }
          }
          return;
        }
        const float fy = kCoded ? scale_of(byte_at(p.scale + half)) * ip : ip, fh = kCoded ? scale_of(byte_at(p.scale)) * a.res_scale : a.res_scale;
        read_saved<T, kCoded>(p.h + sh.saved_area, yh);
        if (has_h) read_saved<T, kCoded>(p.h, H);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          yh[k] = mul2(yh[k], twice(fy));
          b4[k] = mul2(q[k], yh[k]);
          H[k] = has_h ? fma2(H[k], twice(fh), b4[k]) : b4[k];
        }
        if (has_g) {
          read8<T>(p.dx + sh.area, g);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) g[k] = 0;
        }
        if (has_dx) {
          read8<T>(p.dx, dx);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            t[k] = mul2(dx[k], w[k]);
            g[k] = fma2(t[k], twice(iq), g[k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) dx[k] = t[k] = 0;
        }
      };
      // the rows' sums, `parts` warps to a row
      for (int task = warp; task < n * sh.parts; task += sh.warps) {
        const int r = task / sh.parts, part = task - r * sh.parts;
        const float ip = __shfl_sync(0xFFFFFFFFu, ip_lane, r), iq = __shfl_sync(0xFFFFFFFFu, iq_lane, r);
        f2 sums[3] = {0, 0, 0};
        int col = part * sh.part_spans * 256 + lane_col;
        const int end = kFull || kLoose ? min((part + 1) * sh.part_spans * 256, cols) : min((part + 1) * sh.part_spans * 256 + lane * 8, cols);
        Spot p = spot(r, col);
#pragma unroll 1
        for (; col < end; col += 256) {
          f2 yh[4], b4[4], H[4], dx[4], t[4], g[4];
          get(col, q, w);
          form(p, cols - col, ip, iq, yh, b4, H, dx, t, g);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            sums[0] = fma2(t[k], H[k], sums[0]);
            sums[1] = fma2(b4[k], g[k], sums[1]);
            sums[2] = fma2(b4[k], H[k], sums[2]);
          }
          p.dx += 256 * sizeof(T);
          p.h += 256 * kBytes;
          p.scale += 8;
        }
        __syncwarp();
        float s[3] = {halves(sums[0]), halves(sums[1]), halves(sums[2])};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
          for (int k = 0; k < 3; ++k) s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], o);
        }
        if (lane == 0) tail.red[task] = make_float4(s[0], s[1], s[2], 0.0f);
      }
      __syncthreads();
      float k1_lane = 0.0f, k2_lane = 0.0f;                    // of the lane's row
      if (lane < n) {
        float s[3] = {0.0f, 0.0f, 0.0f};
        for (int p = 0; p < sh.parts; ++p) {
          const float4 x = tail.red[lane * sh.parts + p];
          s[0] += x.x, s[1] += x.y, s[2] += x.z;
        }
        k1_lane = iq_lane * iq_lane * (iq_lane * s[0] * a.inv_cols);
        k2_lane = post ? (s[1] - k1_lane * s[2]) * a.inv_cols : 0.0f;
      }
      // the results, a stripe of columns to a warp
      const int col0 = stripe * 256 + lane_col;
      if (kNv == 1 && (kFull || col0 < cols)) {
        get(col0, q, w);
      }
      int r = member < sh.split ? member : n;
      Spot p = spot(r, col0);
      int64_t at = static_cast<int64_t>(row0 + r) * cols + col0;
      const int64_t ahead = static_cast<int64_t>(sh.split) * cols;
      for (; r < n; r += sh.split, at += ahead) {
        const float ip = __shfl_sync(0xFFFFFFFFu, ip_lane, r), iq = __shfl_sync(0xFFFFFFFFu, iq_lane, r);
        const float k1 = __shfl_sync(0xFFFFFFFFu, k1_lane, r), k2 = __shfl_sync(0xFFFFFFFFu, k2_lane, r);
#pragma unroll
        for (int i = 0; i < kNv; ++i) {
          const int col = col0 + i * 256;
          if (kNv == 1 ? !kFull && col >= cols : col >= cols) continue;
          if (kNv > 1) {
            get(col, q, w);
          }
          f2 yh[4], b4[4], H[4], dx[4], t[4], g[4];
          form(Spot{p.dx + i * 256 * static_cast<int>(sizeof(T)), p.h + i * 256 * kBytes, p.scale + i * 8}, cols - col, ip, iq, yh, b4, H, dx, t, g);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            P[i][k] = fma2(mul2(dx[k], twice(iq)), H[k], P[i][k]);
            const f2 d = fma2(H[k], twice(-k1), g[k]);
            S[i][k] = fma2(d, yh[k], S[i][k]);
            g[k] = mul2(d, twice(a.res_scale));
            t[k] = mul2(fma2(yh[k], twice(-k2), mul2(q[k], d)), twice(ip));
          }
          if constexpr (kLoose) {
            if (want_dh) write_singles(static_cast<T*>(a.dh) + at + i * 256, cols - col, lane, g);
            if (want_dy) mx = max(mx, write_singles(static_cast<T*>(a.dy) + at + i * 256, cols - col, lane, t));
            continue;
          }
          if (want_dh) write8(static_cast<T*>(a.dh) + at + i * 256, g);
          if (want_dy) {
            const Vec8<T> o = write8(static_cast<T*>(a.dy) + at + i * 256, t);
            if (a.amax != nullptr) largest.see(o);
          }
        }
        p.dx += sh.split * cols * static_cast<int>(sizeof(T));
        p.h += sh.split * cols * kBytes;
        p.scale += sh.split * sh.blocks_per_row;
      }
      if (c + 1 < runs) keep((c + 1) & 1);
      __syncthreads();                                         // the buffer is read, the next run's scales are there
      if (courier) bring(c + sh.buffers, b);
      if (kLoose && sh.buffers == 1) __syncthreads();          // single values among what was brought
    }
    if (a.part_s != nullptr) store_stripes<kNv, kLoose>(S, a.part_s + unit * cols, reinterpret_cast<float*>(smem), sh, stripe, member);
    else __syncthreads();
  }
  if (a.part_p != nullptr) store_stripes<kNv, kLoose>(P, a.part_p + static_cast<int64_t>(blockIdx.x) * cols, reinterpret_cast<float*>(smem), sh, stripe, member);
  if (a.amax != nullptr) raise_amax(kLoose ? mx : largest.bits(), a.amax);
}

// The gradients of gains and gate from the partial column sums.  A CTA takes 32 columns (a row of them is eight lanes of four), a warp
// four partial rows at a time; a team of warps shares a gate group's rows, so that few groups use all warps too.  The loads of both
// sums, and of the next groups', are in flight before the first addition, and every addition has its place: the order never changes.
// 7 us behind a backward of 4096 columns, of which the partial sums' bytes are one; the rest is the launch and three dependent loads.
constexpr int kFinishWarps = 16;
struct FinishArgs {
  const float *part_s, *part_p;
  const void *post_gain, *gate;
  float *dpost_gain, *dpre_gain, *dgate;
  int64_t cols;
  int groups, pieces, ctas;      // of part_s: groups * pieces rows; of part_p: a row per CTA
  float gain_offset;
  int post, gain_f32, team, batches;   // team: warps to a group, a power of two; batches: of as many groups as there are teams
};
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 shfl4(float4 a, int o) {
  constexpr uint32_t all = 0xFFFFFFFFu;
  return make_float4(__shfl_xor_sync(all, a.x, o), __shfl_xor_sync(all, a.y, o), __shfl_xor_sync(all, a.z, o), __shfl_xor_sync(all, a.w, o));
}
// The sum of rows from, from + stride, .. of n (a lane's row is that of its eighth of the warp), of four columns from c on.
// kVec: the columns are a multiple of four (8192 x 5120 in 16 gate groups: the whole backward 121 us, 123 by single values).
template <bool kVec>
struct PartialSum {
  static constexpr int kAhead = 4;
  const float* p;
  int row, n, stride;
  float4 v[kAhead];
  __device__ __forceinline__ void fetch(int64_t cols, int64_t c) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      v[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const int at = row + j * stride;
      if (at >= n || c >= cols) continue;
      const float* q = p + at * cols + c;
      if (kVec) {
        v[j] = ld_stream(reinterpret_cast<const float4*>(q));
      } else {
        v[j].x = ld_stream(q);
        if (c + 1 < cols) v[j].y = ld_stream(q + 1);
        if (c + 2 < cols) v[j].z = ld_stream(q + 2);
        if (c + 3 < cols) v[j].w = ld_stream(q + 3);
      }
    }
  }
  __device__ __forceinline__ void start(const float* from, int first, int rows, int step, int64_t cols, int64_t c) {
    p = from;
    row = first;
    n = rows;
    stride = step;
    fetch(cols, c);
  }
  __device__ __forceinline__ float4 finish(int64_t cols, int64_t c) {
    float4 t = add4(add4(v[0], v[1]), add4(v[2], v[3]));
    for (row += kAhead * stride; row < n; row += kAhead * stride) {
      fetch(cols, c);
      t = add4(t, add4(add4(v[0], v[1]), add4(v[2], v[3])));
    }
    t = add4(t, shfl4(t, 8));
    return add4(t, shfl4(t, 16));
  }
};
template <bool kVec>
__global__ void __launch_bounds__(32 * kFinishWarps) norm_finish_kernel(const FinishArgs a) {
  __shared__ float4 red_s[kFinishWarps][8], red_p[kFinishWarps][8];
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t c4 = static_cast<int64_t>(blockIdx.x) * 32 + (lane & 7) * 4, c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  const int teams = kFinishWarps / a.team, team = warp / a.team, member = warp % a.team;
  pdl_wait();
  PartialSum<kVec> sp, ss;
  if (a.part_p != nullptr) sp.start(a.part_p, warp * 4 + (lane >> 3), a.ctas, 4 * kFinishWarps, a.cols, c4);
  const auto start_group = [&](int g) {
    if (g < a.groups)
      ss.start(a.part_s + static_cast<int64_t>(g) * a.pieces * a.cols, member * 4 + (lane >> 3), a.pieces, 4 * a.team, a.cols, c4);
  };
  if (a.batches > 0) start_group(team);
  const bool in = c < a.cols;
  const float wpost = in && a.post && a.post_gain != nullptr ? a.gain_offset + gain_at(a.post_gain, c, a.gain_f32) : 1.0f;
  float dpost = 0.0f;                                          // of the warp's groups: warp w adds up groups w, w + teams, ..
  if (a.part_p != nullptr) {
    const float4 t = sp.finish(a.cols, c4);
    if (lane < 8) red_p[warp][lane] = t;
  }
  for (int batch = 0; batch < a.batches; ++batch) {
    const int g = batch * teams + team, mine = batch * teams + warp;   // warp w < teams finishes team w's group
    const bool ends = warp < teams && mine < a.groups && in;
    const float gate = ends && a.gate != nullptr ? gain_at(a.gate, mine * a.cols + c, a.gain_f32) : 1.0f;
    if (g < a.groups) {
      const float4 t = ss.finish(a.cols, c4);
      if (lane < 8) red_s[warp][lane] = t;
      start_group(g + teams);
    }
    if (a.team > 1) __syncthreads(); else __syncwarp();
    if (ends) {
      float s = 0.0f;
      for (int m = 0; m < a.team; ++m) s += reinterpret_cast<const float*>(red_s[warp * a.team + m])[lane];
      if (a.dgate != nullptr) a.dgate[mine * a.cols + c] = wpost * s;
      dpost = __fmaf_rn(gate, s, dpost);
    }
    if (a.team > 1) __syncthreads(); else __syncwarp();
  }
  reinterpret_cast<float*>(red_s[warp])[lane] = dpost;         // the warp's own place in every batch, or that of a member it has read
  __syncthreads();
  if (warp == 0 && in && a.dpost_gain != nullptr) {
    float s = 0.0f;
    for (int w = 0; w < teams; ++w) s += reinterpret_cast<const float*>(red_s[w])[lane];
    a.dpost_gain[c] = s;
  }
  if (warp == 1 && in && a.dpre_gain != nullptr) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kFinishWarps; ++w) s += reinterpret_cast<const float*>(red_p[w])[lane];
    a.dpre_gain[c] = s;
  }
}

inline bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int finish(cudaError_t e) { return e == cudaSuccess ? FALQON_OK : FALQON_ERR_CUDA; }

bool plan_ok(const falqon_block_norm* p) {
  return p != nullptr && p->rows >= 1 && p->rows <= FALQON_NORM_MAX_ROWS && p->cols >= 1 && p->cols <= FALQON_NORM_MAX_COLS &&
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
    a->units = static_cast<int>(units);
    a->pieces = static_cast<int>(pieces);
    a->rows_per_piece = rows_per_piece;
  }
};

bool staged(int64_t cols) { return cols % 16 == 0; }
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

unsigned item_threads(int64_t cols) { return static_cast<unsigned>(((cols + kItems - 1) / kItems + 31) / 32 * 32); }

constexpr int kSmemLimit = 226 * 1024;    // dynamic; the kernels have a few bytes of their own besides
int spans_for(int64_t cols) { return cols <= 2 * 512 * 8 ? 2 : 4; }
int group_warps(int64_t cols, int nv) { return static_cast<int>((cols + 256 * nv - 1) / (256 * nv)); }
// Of the any-width forward, which has one CTA per SM: four spans to a warp where more of its 16 warps are at work then, since a group is
// whole (4096 x 5001 bf16 with both checkpoints: three groups of five warps 99 us, one of ten 129).
int loose_spans(int64_t cols, int64_t rows_per_cta) {
  const auto at_work = [&](int nv) {
    const int64_t warps = group_warps(cols, nv), groups = 16 / warps;
    return warps * (groups < rows_per_cta ? groups : rows_per_cta);
  };
  return at_work(4) > at_work(2) ? 4 : 2;
}
// set_bytes: of a span of 256 columns of every tensor; red: floats of reduction space per row group.
bool make_shape(int64_t cols, int nv, int64_t rows_per_cta, int set_bytes, int red, int smem_limit, Shape* sh, size_t* smem) {
  sh->cols = static_cast<int>(cols);
  sh->group_threads = 32 * group_warps(cols, nv);
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

bool whole_spans(int64_t cols) { return cols % (256 * kFullSpans) == 0 && cols <= 8192; }
// Shape of the full call's kernels: a fixed depth and the weights in shared memory, or false.
bool make_full_shape(int64_t cols, int nv, int64_t rows_per_cta, int stage_bytes, int red, Shape* sh, size_t* smem) {
  sh->cols = static_cast<int>(cols);
  sh->group_threads = static_cast<int>(cols / (8 * nv));
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
// Each kernel with as many CTAs as are resident: one per SM, or two of norm_forward_rows_kernel with two spans a lane (4096 x 5120 bf16 with the
// norm before the next block only: 52 us, one per SM 73; fp32 with both norms: 73 and 84; fp32 4096 x 1024 and norms after the block only at
// 4096 are the other way, by 5 to 7 %).
template <typename T, int kNv>
int launch_forward_rows(const falqon_block_norm* p, NormArgs a, cudaStream_t stream) {
  static DeviceMask done[3];
  Shape sh;
  size_t smem;
  if (kNv == 2 && whole_spans(a.cols) && a.h != nullptr && a.h_out != nullptr && a.post && a.pre && (a.h_codes != nullptr) == (a.y_codes != nullptr)) {
    const Split s(p, kNormUnits);
    s.put(&a);
    if (make_full_shape(a.cols, kFullSpans, a.rows_per_piece, 2 * kFullSpans * 256 * sizeof(T), kSumFloats, &sh, &smem))
      return a.h_codes != nullptr ? start_rows(norm_forward_full_kernel<T, true>, done[0], a, sh, smem, s.ctas, stream)
                                  : start_rows(norm_forward_full_kernel<T, false>, done[1], a, sh, smem, s.ctas, stream);
  }
  const Split s(p, kNv == 2 ? 2 * kNormUnits : kNormUnits);
  s.put(&a);
  const int limit = kNv == 2 ? kSmemLimit / 2 - 1024 : kSmemLimit;       // two CTAs per SM
  if (!make_shape(a.cols, kNv, a.rows_per_piece, 2 * 256 * sizeof(T), kSumFloats, limit, &sh, &smem)) return FALQON_ERR_UNSUPPORTED;   // of no width
  return start_rows(norm_forward_rows_kernel<T, kNv>, done[2], a, sh, smem, s.ctas, stream);
}
// How a backward's runs are cut: stripes per warp, rows per run, and the shared memory it takes; false where not even one row fits.
bool make_run(int64_t cols, int64_t rows_per_piece, int value_bytes, bool coded, bool loose, int* spans, Run* r, size_t* smem) {
  const int saved_bytes = coded ? 1 : value_bytes;
  r->cols = static_cast<int>(cols);
  r->stripes = static_cast<int>((cols + 255) / 256);
  r->blocks_per_row = static_cast<int>((cols + kMx8Block - 1) / kMx8Block);
  // As few stripes to a warp as 16 warps can take: their weights and sums are registers, and more warps than 16 have too few of them.
  // From checkpoints, bf16: 4096 x 4096 with one 54 us, with two 59; 8192 x 6144 with two 139, with one and 24 warps 195; 4096 x 11008 with
  // three 218, with four 262.
  *spans = (r->stripes + 15) / 16;
  r->stripe_warps = (r->stripes + *spans - 1) / *spans;
  r->warps = 16;
  const int row = static_cast<int>(cols) * (2 * value_bytes + 2 * saved_bytes);
  for (int attempt = 0; attempt < 3; ++attempt) {              // two buffers and the weights; without the weights; one buffer
    if (loose && attempt == 1) continue;
    r->weights_in_smem = loose || attempt == 0;
    r->buffers = attempt < 2 ? 2 : 1;
    int run = (kSmemLimit - (r->weights_in_smem ? r->cols * 8 : 0)) / (r->buffers * row);
    if (run > kMaxRun) run = kMaxRun;
    if (run > rows_per_piece) run = static_cast<int>(rows_per_piece);
    for (; run >= 1; --run) {
      r->run = run;
      r->split = r->warps / r->stripe_warps;                   // a row of the run each; so their sums, 4 bytes a column, fit over the buffers
      if (r->split > run) r->split = run;
      r->parts = r->warps / run;
      if (r->parts > r->stripes) r->parts = r->stripes;
      if (r->parts < 1) r->parts = 1;
      r->part_spans = (r->stripes + r->parts - 1) / r->parts;
      r->area = loose ? (run * r->cols * value_bytes + 47) / 16 * 16 : run * r->cols * value_bytes;
      r->saved_area = loose ? (run * r->cols * saved_bytes + 47) / 16 * 16 : run * r->cols * saved_bytes;
      r->buffer = (2 * r->area + 2 * r->saved_area + 127) / 128 * 128;
      r->scale_bytes = coded ? (4 * run * r->blocks_per_row + 15) / 16 * 16 : 0;
      *smem = static_cast<size_t>(r->buffers) * r->buffer + run_tail_bytes(*r);
      if (*smem <= static_cast<size_t>(kSmemLimit) && (!coded || 2 * run * r->blocks_per_row <= kScaleBytes * 32 * r->warps))
        return true;
    }
  }
  return false;
}
template <typename T, bool kCoded, int kNv, bool kFull, bool kLoose>
int start_run(const NormArgs& a, const Run& r, size_t smem, int64_t ctas, int* status, cudaStream_t stream) {
  static DeviceMask done{0};
  const auto kernel = norm_backward_run_kernel<T, kCoded, kNv, kFull, kLoose>;
  if (set_max_dynamic_smem(kernel, kSmemLimit, done) != cudaSuccess) return FALQON_ERR_CUDA;
  return finish(launch_pdl(kernel, dim3(static_cast<unsigned>(ctas)), dim3(32u * r.warps), smem, stream, 1, a, r, status));
}
template <typename T, bool kCoded>
int launch_backward_runs(const NormArgs& a, int64_t ctas, int* status, cudaStream_t stream) {
  Run r;
  size_t smem;
  int spans;
  const bool loose = !staged(a.cols);
  if (!make_run(a.cols, a.rows_per_piece, sizeof(T), kCoded, loose, &spans, &r, &smem)) return FALQON_ERR_UNSUPPORTED;
  // the full call: both norms, both gradients in and out, a residual, whole stripes (4096 x 4096 from checkpoints 57 us, as any call 74, side by side)
  const bool full = a.cols % 256 == 0 && r.weights_in_smem && (kCoded ? a.h_codes_in != nullptr : a.h != nullptr) && a.dx != nullptr && a.dh_out != nullptr &&
                    a.post && a.pre && a.dh != nullptr && a.dy != nullptr;
  const auto go = [&](auto kind) {                             // 0: any call, 1: the full call, 2: any width
    constexpr bool kFull = decltype(kind)::value == 1, kLoose = decltype(kind)::value == 2;
    if (spans == 1) return start_run<T, kCoded, 1, kFull, kLoose>(a, r, smem, ctas, status, stream);
    if (spans == 2) return start_run<T, kCoded, 2, kFull, kLoose>(a, r, smem, ctas, status, stream);
    if (spans == 3) return start_run<T, kCoded, 3, false, kLoose>(a, r, smem, ctas, status, stream);
    return start_run<T, kCoded, 4, false, kLoose>(a, r, smem, ctas, status, stream);
  };
  if (loose) return go(std::integral_constant<int, 2>{});
  return full ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 0>{});
}
template <typename T, int kNv>
int launch_forward_loose(const NormArgs& a, int64_t ctas, cudaStream_t stream) {
  static DeviceMask done{0};
  Shape sh;
  size_t smem;
  if (!make_shape(a.cols, kNv, a.rows_per_piece, 2 * (256 * sizeof(T) + 16), kSumFloats, kSmemLimit, &sh, &smem) || !sh.weights_in_smem) return FALQON_ERR_UNSUPPORTED;
  return start_rows(norm_forward_loose_kernel<T, kNv>, done, a, sh, smem, ctas, stream);
}
template <typename F>
int with_spans(int spans, F go) {
  return spans == 2 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{});
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
      (!a.pre && h_out == nullptr) || (a.pre && x == h_out))
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
  if (staged(a.cols))
    return with_spans(spans_for(a.cols), [&](auto n) {
      return p->dtype == FALQON_BF16 ? launch_forward_rows<bf16_t, n.value>(p, a, static_cast<cudaStream_t>(stream))
                                     : launch_forward_rows<float, n.value>(p, a, static_cast<cudaStream_t>(stream));
    });
  const Split s(p, kNormUnits);
  NormArgs b = a;
  s.put(&b);
  const int rc = with_spans(loose_spans(a.cols, s.rows_per_piece), [&](auto n) {
    return p->dtype == FALQON_BF16 ? launch_forward_loose<bf16_t, n.value>(b, s.ctas, static_cast<cudaStream_t>(stream))
                                   : launch_forward_loose<float, n.value>(b, s.ctas, static_cast<cudaStream_t>(stream));
  });
  if (rc != FALQON_ERR_UNSUPPORTED || p->dtype == FALQON_BF16) return rc;
  const int64_t cap = static_cast<int64_t>(sm_count()) * 2;
  const dim3 grid(static_cast<unsigned>(a.rows < cap ? a.rows : cap)), block(item_threads(a.cols));
  return finish(launch_pdl(norm_forward_f32_kernel, grid, block, 0, static_cast<cudaStream_t>(stream), 1, a));
}

size_t falqon_block_norm_scratch_bytes(const falqon_block_norm* p) {
  if (!plan_ok(p)) return 0;
  const Split s(p, kNormUnits);
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
  const Split s(p, kNormUnits);
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
  {
    int* status = device_status_ptr();
    if (status == nullptr) return FALQON_ERR_CUDA;
    if (p->dtype == FALQON_BF16)
      rc = coded ? launch_backward_runs<bf16_t, true>(a, s.ctas, status, st) : launch_backward_runs<bf16_t, false>(a, s.ctas, status, st);
    else
      rc = coded ? launch_backward_runs<float, true>(a, s.ctas, status, st) : launch_backward_runs<float, false>(a, s.ctas, status, st);
  }
  if (rc == FALQON_ERR_UNSUPPORTED)
    rc = finish(launch_pdl(p->dtype == FALQON_BF16 ? norm_backward_kernel<bf16_t> : norm_backward_kernel<float>, dim3(static_cast<unsigned>(s.ctas)),
                           dim3(item_threads(a.cols)), 0, st, 1, a));
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
  f.groups = static_cast<int>(s.groups);
  f.pieces = static_cast<int>(s.pieces);
  f.ctas = static_cast<int>(s.ctas);
  f.gain_offset = a.gain_offset;
  f.post = a.post;
  f.gain_f32 = a.gain_f32;
  for (f.team = kFinishWarps; f.team > 1 && f.team * s.groups > kFinishWarps;) f.team /= 2;
  f.batches = sums_s ? (f.groups + kFinishWarps / f.team - 1) / (kFinishWarps / f.team) : 0;
  return finish(launch_pdl(a.cols % 4 == 0 ? norm_finish_kernel<true> : norm_finish_kernel<false>, dim3(static_cast<unsigned>((a.cols + 31) / 32)),
                           dim3(32 * kFinishWarps), 0, st, 1, f));
}

}  // extern "C"
