// Orthogonalised updates of thin matrices, as adapters have them (include/falqon_dense.h): the short side s is at most 128.
// Every iterate is X_k = X P_k with P_k a polynomial in G = X^T X (s x s), so the long side need only be read twice:
//   G = X^T X,  f = 1 / (sqrt(trace G) + eps);   per step  Q = a + b G + c G G,  P <- P Q,  G <- (G Q) Q;   out = scale f X P
// instead of twice a step, and the steps are products of s x s matrices.  What this costs is digits: an error d of G in the direction of a
// singular value that is small beside the norm grows by a^2 a step (11.9 for Muon's polynomial) and P with it, so all of it runs in fp64
// (mma.sync m8n8k4, whose rate is that of plain fp64): d is about 2^-50, and matrices whose steps would grow it past 2^-24 go the other
// way.  Results then carry their own rounding alone.
// Bound: G and the last product by the fp64 tensor rate (2 s^2 l operations each; the first only on and above the diagonal), the steps
// by latency: four products each, three of them in turn, and two exchanges; which a cluster of up to eight CTAs shares.
#include <algorithm>
#include <cmath>

#include "../../include/falqon_dense.h"
#include "internal.h"
#include "mx8.cuh"
#include "ortho_thin.h"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kThreads = 256, kWarps = 8;

// Made for 4, 8 or 16 tiles of eight along the short side, which is filled up with zeros: every bound a constant.
template <int kTiles>
struct Shape {
  static constexpr int kSide = 8 * kTiles;
  // four more than a multiple of 16 doubles, so that four rows by four columns lie in different banks
  static constexpr int kPitch = (kSide + 15) / 16 * 16 + 4;
  static constexpr int kRowsK = kTiles <= 8 ? 64 : 32;             // long-side rows in a tile of shared memory
  static constexpr int kSize = kSide * kSide;
  static constexpr int kCluster = kTiles < 8 ? kTiles : 8;         // CTAs that share a matrix's steps
};

__device__ __forceinline__ void dmma(double (&c)[2], double a, double b) {
  asm volatile("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};" : "+d"(c[0]), "+d"(c[1]) : "d"(a), "d"(b));
}

// kRowsK rows of the long side from k0, as they come, into registers; and from there as doubles [kRowsK][kPitch], zero where there is
// nothing.
template <typename T, bool kTall, int kTiles>
struct Slab {
  using S = Shape<kTiles>;
  static constexpr int kEach = S::kRowsK * S::kSide / kThreads;
  float v[kEach];
  static __device__ __forceinline__ void place(int u, int& k, int& i) {
    const int idx = threadIdx.x + u * kThreads;
    k = kTall ? idx / S::kSide : idx % S::kRowsK, i = kTall ? idx % S::kSide : idx / S::kRowsK;
  }
  __device__ __forceinline__ void load(const T* x, int64_t l, int64_t end, int s, int64_t k0) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      int k, i;
      place(u, k, i);
      v[u] = k0 + k < end && i < s ? load1(x + (kTall ? (k0 + k) * s + i : i * l + k0 + k)) : 0.0f;
    }
  }
  __device__ __forceinline__ void put(double* t) const {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      int k, i;
      place(u, k, i);
      t[k * S::kPitch + i] = v[u];
    }
  }
};

// Parts of G: parts [batch][gridDim.x][side][side], the 8 x 8 tiles on and above the diagonal.  A warp takes tile rows r1 = q and r2 =
// tiles - 1 - q, which together are tiles + 1 tiles whatever q is; where there are fewer such pairs than warps, groups of warps share the
// long side and are added up in order.
template <typename T, bool kTall, int kTiles>
__global__ void __launch_bounds__(kThreads, kTiles <= 8 ? 2 : 1)
thin_gram_kernel(const T* g, int64_t l, int s, int64_t rows_per_part, double* parts) {
  using S = Shape<kTiles>;
  constexpr int kPairs = kTiles / 2, kGroups = kWarps / kPairs;
  __shared__ __align__(16) double tile[S::kRowsK * S::kPitch];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int q = warp % kPairs, group = warp / kPairs, r1 = q, r2 = kTiles - 1 - q;
  const T* x = g + blockIdx.y * l * s;
  const int64_t begin = blockIdx.x * rows_per_part, end = min(l, begin + rows_per_part);
  double acc1[kTiles][2] = {}, acc2[kPairs][2] = {};
  Slab<T, kTall, kTiles> slab;
  slab.load(x, l, end, s, begin);
  for (int64_t k0 = begin; k0 < end; k0 += S::kRowsK) {
    __syncthreads();
    slab.put(tile);
    __syncthreads();
    if (k0 + S::kRowsK < end) slab.load(x, l, end, s, k0 + S::kRowsK);
    const double* at = tile + (4 * group + (lane & 3)) * S::kPitch + (lane >> 2);
#pragma unroll 2
    for (int k = 0; k < S::kRowsK / 4 / kGroups; ++k, at += 4 * kGroups * S::kPitch) {
      const double a1 = at[8 * r1], a2 = at[8 * r2];
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {          // tile column kTiles - 1 - j
        if (j >= kPairs && j >= kTiles - r1) continue;
        const double b = at[8 * (kTiles - 1 - j)];
        dmma(acc1[j], a1, b);
        if (j < kPairs && j <= q) dmma(acc2[j < kPairs ? j : 0], a2, b);
      }
    }
  }
  // the groups, in order
  double* out = parts + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * S::kSize;
  const int at = (lane >> 2) * S::kSide + 2 * (lane & 3);
  for (int turn = 0; turn < kGroups; ++turn) {
    __syncthreads();
    if (group != turn) continue;
    auto add = [&](int r, int c, const double (&v)[2]) {
      double2* p = reinterpret_cast<double2*>(out + 8 * r * S::kSide + 8 * c + at);
      double2 d = turn == 0 ? make_double2(0.0, 0.0) : __ldcg(p);
      d.x += v[0], d.y += v[1];
      __stcg(p, d);
    };
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      if (j < kTiles - r1) add(r1, kTiles - 1 - j, acc1[j]);
      if (j < kPairs && j <= q) add(r2, kTiles - 1 - j, acc2[j < kPairs ? j : 0]);
    }
  }
}

struct ChainArgs {
  const double* parts;
  int nparts, steps;
  double eps, scale;
  double* out;                   // [batch][side][side]: P times scale and f
  int* status;
  float abc[3 * kThinMostSteps];
};

// The steps.  A cluster to a matrix: a CTA owns tile rows cta, cta + cluster, .. (their rows of G and P in its shared memory), a warp tile
// columns w, w + 8, ..  The right operand of a product (G and Q in turn) lies whole in every CTA: a CTA copies its rows of it
// to all of them (bulk copies that count on the receiver's barrier), by two buffers in turn where two fit.  The matrices are symmetric and commute, so both operands are read by rows.
template <int kTiles>
__global__ void __launch_bounds__(kThreads)
thin_chain_kernel(const __grid_constant__ ChainArgs p) {
  using S = Shape<kTiles>;
  constexpr int kC = S::kCluster, kOwnRows = kTiles / kC, kOwnCols = (kTiles + kWarps - 1) / kWarps;
  constexpr int kBuffers = kTiles <= 8 ? 2 : 1, kFull = S::kSide * S::kPitch, kOwn = 8 * kOwnRows * S::kPitch;
  extern __shared__ __align__(16) double smem[];
  __shared__ double s_f;
  __shared__ __align__(8) uint64_t s_bar[kBuffers];
  double *g_rows = smem + kBuffers * kFull, *p_rows = g_rows + kOwn;       // tile row cta + kC t at 8 t
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = static_cast<int>(cluster_ctarank()), b = blockIdx.x / kC;
  const int fi = lane >> 2, fj = 2 * (lane & 3);                 // this lane's two results in a tile
  int now = 0;                                                   // the buffer of the right operand
  uint32_t phase[kBuffers] = {};
  bool lost = false;             // a copy that has not come in time: go on without waiting, the status says so
  if (threadIdx.x == 0) {
    for (int i = 0; i < kBuffers; ++i) mbar_init(smem_u32(&s_bar[i]), 1);
    mbar_fence_init();
  }

  double d1[kOwnRows][kOwnCols][2], d2[kOwnRows][kOwnCols][2];
  auto each = [&](auto f) {
#pragma unroll
    for (int t = 0; t < kOwnRows; ++t)
#pragma unroll
      for (int u = 0; u < kOwnCols; ++u)
        if (warp + kWarps * u < kTiles) f(t, u, cta + kC * t, warp + kWarps * u);
  };
  auto product = [&](const double* rows, int c, double (&d)[2]) {     // rows: eight rows of the left operand
    const double* pa = rows + (lane >> 2) * S::kPitch + (lane & 3);
    const double* pb = smem + now * kFull + (8 * c + (lane >> 2)) * S::kPitch + (lane & 3);
    double even[2] = {0.0, 0.0}, odd[2] = {0.0, 0.0};
#pragma unroll
    for (int k = 0; k < S::kSide; k += 8) {
      dmma(even, pa[k], pb[k]);
      dmma(odd, pa[k + 4], pb[k + 4]);
    }
    d[0] = even[0] + odd[0], d[1] = even[1] + odd[1];
  };
  auto keep = [&](double* rows, int t, int c, const double (&d)[2]) {
    *reinterpret_cast<double2*>(rows + (8 * t + fi) * S::kPitch + 8 * c + fj) = make_double2(d[0], d[1]);
  };
  // d becomes the right operand, everywhere
  auto publish = [&](const double (&d)[kOwnRows][kOwnCols][2]) {
    if (kBuffers == 1) {          // everybody has read what it replaces
      cluster_arrive();
      cluster_wait();
    }
    const int next = kBuffers == 1 ? 0 : now ^ 1;
    each([&](int t, int u, int r, int c) {
      *reinterpret_cast<double2*>(smem + next * kFull + (8 * r + fi) * S::kPitch + 8 * c + fj) = make_double2(d[t][u][0], d[t][u][1]);
    });
    fence_proxy_async_smem();
    __syncthreads();
    constexpr uint32_t kRowBytes = 8 * S::kPitch * 8;
    const uint32_t bar = smem_u32(&s_bar[next]);
    if (threadIdx.x == 0) mbar_expect_tx(bar, (kC - 1) * kOwnRows * kRowBytes);
    if (threadIdx.x < kC * kOwnRows) {          // a copy per thread
      const int peer = threadIdx.x % kC, r = cta + kC * (threadIdx.x / kC);
      const uint32_t rows = smem_u32(smem + next * kFull + 8 * r * S::kPitch);
      if (peer != cta) bulk_copy_to_cta(map_to_cta(rows, static_cast<uint32_t>(peer)), rows, kRowBytes, map_to_cta(bar, static_cast<uint32_t>(peer)));
    }
    if (!lost) lost = !mbar_wait_warp(bar, phase[next], p.status);
    phase[next] ^= 1u;
    now = next;
  };

  const double* parts = p.parts + static_cast<int64_t>(b) * p.nparts * S::kSize;
  each([&](int t, int u, int r, int c) {       // G from its parts, below the diagonal from above it
    double x = 0.0, y = 0.0;
    const int i = 8 * r + fi, j = 8 * c + fj;
    const double* q = parts + (r <= c ? i * S::kSide + j : j * S::kSide + i);
#pragma unroll 8
    for (int k = 0; k < p.nparts; ++k, q += S::kSize) {
      if (r <= c) {
        const double2 v = __ldcg(reinterpret_cast<const double2*>(q));
        x += v.x, y += v.y;
      } else {
        x += __ldcg(q), y += __ldcg(q + S::kSide);
      }
    }
    d1[t][u][0] = x, d1[t][u][1] = y;
    keep(g_rows, t, c, d1[t][u]);
  });
  cluster_arrive();               // the peers have started: their barriers are there, their shared memory may be written
  cluster_wait();
  publish(d1);
  if (warp == 0) {
    double t = 0.0;
    for (int i = lane; i < S::kSide; i += 32) t += smem[now * kFull + i * S::kPitch + i];
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, s);
    const double norm = sqrt(t) + p.eps;
    // an infinity or a NaN anywhere: NaN everywhere; nothing but zeros: zeros
    if (lane == 0) s_f = !(t <= 1.7976931348623157e308) ? nan("") : norm > 0.0 ? 1.0 / norm : 0.0;
  }
  __syncthreads();
  const double f = s_f;
  double gs = f * f;              // what G still has to be multiplied by
  for (int step = 0;; ++step) {
    const double ca = p.abc[3 * step], cb = p.abc[3 * step + 1] * gs, cc = p.abc[3 * step + 2] * gs * gs;
    const bool last = step + 1 == p.steps;
    each([&](int t, int u, int r, int c) {     // Q = a + b G + c G G
      product(g_rows + 8 * t * S::kPitch, c, d1[t][u]);
      const double2 g = *reinterpret_cast<const double2*>(g_rows + (8 * t + fi) * S::kPitch + 8 * c + fj);
      const int i = 8 * r + fi, j = 8 * c + fj;
      d1[t][u][0] = cb * g.x + cc * d1[t][u][0] + (i == j ? ca : 0.0);
      d1[t][u][1] = cb * g.y + cc * d1[t][u][1] + (i == j + 1 ? ca : 0.0);
      if (step == 0) keep(p_rows, t, c, d1[t][u]);
    });
    if (step == 0 && last) break;              // d1 is P
    publish(d1);
    each([&](int t, int u, int, int c) {       // P <- P Q, and G Q
      if (step > 0) product(p_rows + 8 * t * S::kPitch, c, d1[t][u]);
      if (!last) product(g_rows + 8 * t * S::kPitch, c, d2[t][u]);
    });
    if (last) break;
    __syncthreads();                           // the rows of P and G have been read
    each([&](int t, int u, int, int c) {
      if (step > 0) keep(p_rows, t, c, d1[t][u]);
      keep(g_rows, t, c, d2[t][u]);
    });
    __syncthreads();
    each([&](int t, int u, int, int c) {       // G <- (G Q) Q: by the CTA's own rows, so that only Q and G are handed round
      product(g_rows + 8 * t * S::kPitch, c, d1[t][u]);
      d1[t][u][0] *= gs, d1[t][u][1] *= gs;
    });
    gs = 1.0;
    __syncthreads();
    each([&](int t, int u, int, int c) { keep(g_rows, t, c, d1[t][u]); });
    publish(d1);
  }
  each([&](int t, int u, int r, int c) {
    __stcg(reinterpret_cast<double2*>(p.out + static_cast<int64_t>(b) * S::kSize + (8 * r + fi) * S::kSide + 8 * c + fj),
           make_double2(p.scale * f * d1[t][u][0], p.scale * f * d1[t][u][1]));
  });
  cluster_arrive();               // nobody leaves while its shared memory may still be written
  cluster_wait();
}

// out = X P by the long side's rows; a warp keeps its tile columns of P (w, w + 8) in registers.
template <typename T, bool kTall, int kTiles>
__global__ void __launch_bounds__(kThreads, kTiles <= 8 ? 2 : 1)
thin_apply_kernel(const T* g, int64_t l, int s, const double* pm, void* out, bool out_bf16, bool out_pairs) {
  using S = Shape<kTiles>;
  // tile columns of a warp; with fewer columns than warps, groups of warps share the rows
  constexpr int kCols = kTiles > kWarps ? kTiles / kWarps : 1, kGroups = kTiles < kWarps ? kWarps / kTiles : 1;
  __shared__ __align__(16) double tile[S::kRowsK * S::kPitch];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = warp % kTiles, group = warp / kTiles;
  const T* x = g + blockIdx.y * l * s;
  Slab<T, kTall, kTiles> slab;
  const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRowsK;
  slab.load(x, l, l, s, static_cast<int64_t>(blockIdx.x) * S::kRowsK);
  double w[kCols][2 * kTiles];
#pragma unroll
  for (int h = 0; h < kCols; ++h)
#pragma unroll
    for (int k = 0; k < 2 * kTiles; ++k)
      w[h][k] = __ldcg(pm + blockIdx.y * static_cast<int64_t>(S::kSize) + (8 * (col + kWarps * h) + (lane >> 2)) * S::kSide + 4 * k + (lane & 3));
  for (int64_t k0 = static_cast<int64_t>(blockIdx.x) * S::kRowsK; k0 < l; k0 += step) {
    __syncthreads();
    slab.put(tile);
    __syncthreads();
    if (k0 + step < l) slab.load(x, l, l, s, k0 + step);
#pragma unroll 1
    for (int rt = 2 * group; rt < S::kRowsK / 8; rt += 2 * kGroups) {     // two tile rows at a time: chains that do not wait for one another
      double acc[2][kCols][2] = {};
      const double* at = tile + (8 * rt + (lane >> 2)) * S::kPitch + (lane & 3);
#pragma unroll
      for (int k = 0; k < 2 * kTiles; ++k) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const double v = at[8 * y * S::kPitch + 4 * k];
#pragma unroll
          for (int h = 0; h < kCols; ++h) {
            if (kTall) dmma(acc[y][h], v, w[h][k]); else dmma(acc[y][h], w[h][k], v);
          }
        }
      }
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int h = 0; h < kCols; ++h) {
          // tall: row of the long side, two columns of the short one; wide: the other way round
          const int64_t long_at = k0 + 8 * (rt + y) + (kTall ? (lane >> 2) : 2 * (lane & 3));
          const int short_at = 8 * (col + kWarps * h) + (kTall ? 2 * (lane & 3) : (lane >> 2));
          const int64_t o = static_cast<int64_t>(blockIdx.y) * l * s + (kTall ? long_at * s + short_at : short_at * l + long_at);
          const bool in0 = long_at < l && short_at < s, in1 = kTall ? in0 && short_at + 1 < s : in0 && long_at + 1 < l;
          const float v0 = static_cast<float>(acc[y][h][0]), v1 = static_cast<float>(acc[y][h][1]);
          if (out_pairs && in1) {
            if (out_bf16) *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(out) + o) = pack2(v0, v1);
            else *reinterpret_cast<float2*>(static_cast<float*>(out) + o) = make_float2(v0, v1);
          } else {
            if (out_bf16) {
              if (in0) store1(static_cast<bf16_t*>(out) + o, v0);
              if (in1) store1(static_cast<bf16_t*>(out) + o + 1, v1);
            } else {
              if (in0) static_cast<float*>(out)[o] = v0;
              if (in1) static_cast<float*>(out)[o + 1] = v1;
            }
          }
        }
    }
  }
}

// ---------------------------------------------------------------- host side
int64_t side_of(int64_t s) { return s <= 32 ? 32 : s <= 64 ? 64 : 128; }
int64_t parts_of(int64_t batch, int64_t l) {      // of the long side, at least 64 rows each: a CTA to an SM
  return std::max<int64_t>(1, std::min((l + 63) / 64, sm_count() / batch));
}

template <typename T, bool kTall, int kTiles>
cudaError_t launch_of(const ThinPlan& p, int64_t l, int s, const void* g, void* out, void* scratch, cudaStream_t st) {
  using S = Shape<kTiles>;
  const T* x = static_cast<const T*>(g);
  double* pm = static_cast<double*>(scratch);
  double* parts = pm + p.batch * S::kSize;
  int64_t nparts = parts_of(p.batch, l);
  const int64_t per = round_up((l + nparts - 1) / nparts, S::kRowsK);
  nparts = (l + per - 1) / per;
  const unsigned batch = static_cast<unsigned>(p.batch);
  cudaError_t e = launch_pdl(thin_gram_kernel<T, kTall, kTiles>, dim3(static_cast<unsigned>(nparts), batch), dim3(kThreads), 0, st, 1, x, l, s, per, parts);
  if (e != cudaSuccess) return e;
  ChainArgs c{};
  c.parts = parts, c.nparts = static_cast<int>(nparts), c.steps = p.steps, c.eps = p.eps, c.scale = p.scale, c.out = pm, c.status = device_status_ptr();
  if (c.status == nullptr) return cudaErrorInvalidValue;
  for (int i = 0; i < 3 * p.steps; ++i) c.abc[i] = p.abc[i];
  constexpr int kChainBytes = ((kTiles <= 8 ? 2 : 1) * S::kSide + 2 * 8 * (kTiles / S::kCluster)) * S::kPitch * 8;
  static DeviceMask done{0};
  if ((e = set_max_dynamic_smem(thin_chain_kernel<kTiles>, kChainBytes, done)) != cudaSuccess) return e;
  e = launch_pdl(thin_chain_kernel<kTiles>, dim3(S::kCluster * batch), dim3(kThreads), kChainBytes, st, S::kCluster, c);
  if (e != cudaSuccess) return e;
  const int64_t chunks = (l + S::kRowsK - 1) / S::kRowsK, cap = std::max<int64_t>(1, (kTiles <= 8 ? 2 : 1) * sm_count() / p.batch);
  const bool pairs = (kTall ? s : l) % 2 == 0 && (reinterpret_cast<uintptr_t>(out) & (p.out_bf16 ? 3 : 7)) == 0;
  return launch_pdl(thin_apply_kernel<T, kTall, kTiles>, dim3(static_cast<unsigned>(chunks < cap ? chunks : cap), batch), dim3(kThreads), 0, st, 1, x, l,
                    s, static_cast<const double*>(pm), out, p.out_bf16, pairs);
}
template <typename T, bool kTall>
cudaError_t launch_side(const ThinPlan& p, int64_t l, int s, const void* g, void* out, void* scratch, cudaStream_t st) {
  return s <= 32 ? launch_of<T, kTall, 4>(p, l, s, g, out, scratch, st)
                 : s <= 64 ? launch_of<T, kTall, 8>(p, l, s, g, out, scratch, st) : launch_of<T, kTall, 16>(p, l, s, g, out, scratch, st);
}

}  // namespace

bool ortho_thin_takes(int64_t rows, int64_t cols, bool out_bf16, const float* abc, int steps) {
  const int64_t s = rows < cols ? rows : cols;
  // The other way takes 17 to 22 launches, whatever the size, but works at the fp16 rate, and at a third of it for fp32 results.  bf16, 7 of
  // 4096 x 64: 65 us here, 124 there; 64 of 14336 x 64: 1040 and 1270; 7 of 4096 x 128: 202 and 168; 16: 400 and 260.  fp32, 7 of 4096 x
  // 128: 181 and 223; 16 of 128 x 14336: 674 and 1131; 64 of 4096 x 128: 1076 and 912 -- there the rule, which looks at the short side alone,
  // costs a sixth of the time, and buys results that carry their own rounding only.
  if (s > (out_bf16 ? kThinMost / 2 : kThinMost)) return false;
  // how far an error of G may grow before the last step's polynomial is taken: 2^-50 to 2^-24
  double growth = 1.0;
  for (int i = 0; i + 1 < steps; ++i) growth *= std::max(1.0, static_cast<double>(abc[3 * i]) * abc[3 * i]);
  return growth <= 67108864.0;
}

size_t ortho_thin_scratch_bytes(int64_t batch, int64_t rows, int64_t cols) {
  const int64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows, side = side_of(s);
  return static_cast<size_t>(batch) * (1 + parts_of(batch, l)) * side * side * 8;
}

cudaError_t launch_ortho_thin(const ThinPlan& p, const void* g, void* out, void* scratch, cudaStream_t st) {
  const bool tall = p.rows > p.cols;
  const int64_t l = tall ? p.rows : p.cols;
  const int s = static_cast<int>(tall ? p.cols : p.rows);
  if (p.in_bf16) return tall ? launch_side<bf16_t, true>(p, l, s, g, out, scratch, st) : launch_side<bf16_t, false>(p, l, s, g, out, scratch, st);
  return tall ? launch_side<float, true>(p, l, s, g, out, scratch, st) : launch_side<float, false>(p, l, s, g, out, scratch, st);
}

}  // namespace falqon
