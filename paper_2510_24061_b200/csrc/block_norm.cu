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

constexpr int kNormUnits = 148;    // CTAs that share the rows of a backward

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

// The gradients of gains and gate from the partial column sums: a CTA takes 32 columns, its eight warps share the partials of a
// column (every eighth each, in order) and are added in warp order.
constexpr int kFinishWarps = 8;
struct FinishArgs {
  const float *part_s, *part_p;
  const void *post_gain, *gate;
  float *dpost_gain, *dpre_gain, *dgate;
  int64_t cols, groups, pieces, ctas;
  float gain_offset;
  int post, gain_f32;
};
__global__ void __launch_bounds__(32 * kFinishWarps) norm_finish_kernel(const FinishArgs a) {
  __shared__ float red[kFinishWarps][32];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  const bool in = c < a.cols;
  const auto column_sum = [&](const float* p, int64_t n) {
    float t = 0.0f;
    if (in)
      for (int64_t i = warp; i < n; i += kFinishWarps) t += ld_stream(p + i * a.cols + c);
    __syncthreads();
    red[warp][lane] = t;
    __syncthreads();
    t = 0.0f;
#pragma unroll
    for (int w = 0; w < kFinishWarps; ++w) t += red[w][lane];
    return t;
  };
  if (a.part_s != nullptr) {
    const float wpost = in && a.post && a.post_gain != nullptr ? a.gain_offset + gain_at(a.post_gain, c, a.gain_f32) : 1.0f;
    float dpost = 0.0f;
    for (int64_t g = 0; g < a.groups; ++g) {
      const float s = column_sum(a.part_s + g * a.pieces * a.cols, a.pieces);
      if (in && warp == 0) {
        if (a.dgate != nullptr) a.dgate[g * a.cols + c] = wpost * s;
        dpost = __fmaf_rn(a.gate != nullptr ? gain_at(a.gate, g * a.cols + c, a.gain_f32) : 1.0f, s, dpost);
      }
    }
    if (a.dpost_gain != nullptr && in && warp == 0) a.dpost_gain[c] = dpost;
  }
  if (a.dpre_gain != nullptr) {
    const float s = column_sum(a.part_p, a.ctas);
    if (in && warp == 0) a.dpre_gain[c] = s;
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

// How a backward's rows are dealt out: every gate group in `pieces` runs of rows, a unit each; one gate row for all makes one group.
struct Split {
  int64_t rows_per_gate, groups, pieces, rows_per_piece, units, ctas;
  explicit Split(const falqon_block_norm* p) {
    rows_per_gate = p->gate == nullptr || p->rows_per_gate > p->rows ? p->rows : p->rows_per_gate;
    groups = (p->rows + rows_per_gate - 1) / rows_per_gate;
    pieces = groups >= kNormUnits ? 1 : kNormUnits / groups;
    rows_per_piece = (rows_per_gate + pieces - 1) / pieces;
    pieces = (rows_per_gate + rows_per_piece - 1) / rows_per_piece;
    units = groups * pieces;
    ctas = units < kNormUnits ? units : kNormUnits;
  }
};

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
  const Split s(p);
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
  const Split s(p);
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
  a.rows_per_gate = s.rows_per_gate;
  a.pieces = s.pieces;
  a.rows_per_piece = s.rows_per_piece;
  a.part_s = sums_s ? static_cast<float*>(scratch) : nullptr;
  a.part_p = sums_p ? static_cast<float*>(scratch) + s.units * a.cols : nullptr;
  const int items = items_for(a.cols);
  const unsigned threads = static_cast<unsigned>(((a.cols + items - 1) / items + 31) / 32 * 32);
  const unsigned grid = static_cast<unsigned>(s.ctas);
  const int rc = with_items(items, [&](auto n) {
    return finish(p->dtype == FALQON_BF16 ? launch_pdl(norm_backward_kernel<bf16_t, n.value>, dim3(grid), dim3(threads), 0,
                                                       static_cast<cudaStream_t>(stream), 1, a)
                                          : launch_pdl(norm_backward_kernel<float, n.value>, dim3(grid), dim3(threads), 0,
                                                       static_cast<cudaStream_t>(stream), 1, a));
  });
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
  return finish(launch_pdl(norm_finish_kernel, dim3(static_cast<unsigned>((a.cols + 31) / 32)), dim3(32 * kFinishWarps), 0,
                           static_cast<cudaStream_t>(stream), 1, f));
}

}  // extern "C"
