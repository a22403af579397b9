// Orthogonalised updates of thin matrices, as adapters have them (include/falqon_dense.h): the short side s is at most 128.
// Every iterate is X_k = X P_k with P_k a polynomial in G = X^T X (s x s), so the long side need only be read twice:
//   G = X^T X,  f = 1 / (sqrt(trace G) + eps);   per step  Q = a + b G + c G G,  P <- P Q,  G <- G Q Q;   out = scale f X P
// instead of twice a step, and the steps are products of s x s matrices.  What this costs is digits: an error d of G in the direction of a
// singular value that is small beside the norm grows by a^2 a step (11.9 for Muon's polynomial) and P with it, so all of it runs in fp64
// (mma.sync m8n8k4, whose rate is that of plain fp64): d is about 2^-50, and matrices whose steps would grow it past 2^-24 go the other
// way.  Results then carry their own rounding alone.
// Bound: G and the last product by the fp64 tensor rate (2 s^2 l operations each; the first only on and above the diagonal), the steps
// by latency: 3 products each, which a cluster of eight CTAs shares through L2 (its matrices are a few dozen KB).
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
constexpr int kRowsK = 32;                 // long-side rows in a tile of shared memory
constexpr int kMostTiles = 16;             // 8 x 8 tiles along the short side
constexpr int kCluster = 8;

__device__ __forceinline__ void dmma(double (&c)[2], double a, double b) {
  asm volatile("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};" : "+d"(c[0]), "+d"(c[1]) : "d"(a), "d"(b));
}
// Pitch of a tile of doubles: 4 (mod 16), so that four rows by four columns lie in different banks.
__host__ __device__ __forceinline__ int pitch_of(int s8) { return (s8 + 15) / 16 * 16 + 4; }

// 32 rows of the long side from k0, as they come, into registers; and from there as doubles [32][pitch], zero where there is nothing.
template <typename T, bool kTall>
struct Slab {
  float v[kRowsK * 8 * kMostTiles / kThreads];
  __device__ __forceinline__ void load(const T* x, int64_t l, int64_t end, int s, int s8, int64_t k0) {
#pragma unroll
    for (int u = 0; u < kRowsK * 8 * kMostTiles / kThreads; ++u) {
      const int idx = threadIdx.x + u * kThreads;
      if (idx >= kRowsK * s8) break;
      const int k = kTall ? idx / s8 : idx % kRowsK, i = kTall ? idx - k * s8 : idx / kRowsK;
      v[u] = k0 + k < end && i < s ? load1(x + (kTall ? (k0 + k) * s + i : i * l + k0 + k)) : 0.0f;
    }
  }
  __device__ __forceinline__ void put(double* t, int s8, int pitch) const {
#pragma unroll
    for (int u = 0; u < kRowsK * 8 * kMostTiles / kThreads; ++u) {
      const int idx = threadIdx.x + u * kThreads;
      if (idx >= kRowsK * s8) break;
      const int k = kTall ? idx / s8 : idx % kRowsK, i = kTall ? idx - k * s8 : idx / kRowsK;
      t[k * pitch + i] = v[u];
    }
  }
};

// Parts of G: parts [batch][gridDim.x][s8][s8], the 8 x 8 tiles on and above the diagonal.  A warp takes tile rows r1 = q and r2 =
// tiles - 1 - q, which together are tiles + 1 tiles whatever q is; where there are fewer such pairs than warps, groups of warps share the
// long side and are added up in order.
template <typename T, bool kTall>
__global__ void __launch_bounds__(kThreads)
thin_gram_kernel(const T* g, int64_t l, int s, int64_t rows_per_part, double* parts) {
  extern __shared__ __align__(16) double tile[];
  pdl_trigger();
  pdl_wait();
  const int s8 = (s + 7) / 8 * 8, tiles = s8 / 8, pitch = pitch_of(s8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pairs = (tiles + 1) / 2, groups = kWarps / pairs, q = warp % pairs, group = warp / pairs;
  const bool works = group < groups;
  const int r1 = q, r2 = tiles - 1 - q;
  const T* x = g + blockIdx.y * l * s;
  const int64_t begin = blockIdx.x * rows_per_part, end = min(l, begin + rows_per_part);
  double acc1[kMostTiles][2] = {}, acc2[kMostTiles / 2][2] = {};
  Slab<T, kTall> slab;
  slab.load(x, l, end, s, s8, begin);
  for (int64_t k0 = begin; k0 < end; k0 += kRowsK) {
    __syncthreads();
    slab.put(tile, s8, pitch);
    __syncthreads();
    if (k0 + kRowsK < end) slab.load(x, l, end, s, s8, k0 + kRowsK);
    if (works) {
      for (int k4 = 4 * group; k4 < kRowsK; k4 += 4 * groups) {
        const double* at = tile + (k4 + (lane & 3)) * pitch + (lane >> 2);
        const double a1 = at[8 * r1], a2 = at[8 * r2];
#pragma unroll
        for (int j = 0; j < kMostTiles; ++j) {          // tile column tiles - 1 - j
          if (j < tiles - r1) {
            const double b = at[8 * (tiles - 1 - j)];
            dmma(acc1[j], a1, b);
            if (j < kMostTiles / 2 && j < tiles - r2 && r2 != r1) dmma(acc2[j < kMostTiles / 2 ? j : 0], a2, b);
          }
        }
      }
    }
  }
  // the groups, in order
  double* out = parts + (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * s8 * s8;
  const int at = (lane >> 2) * s8 + 2 * (lane & 3);
  for (int turn = 0; turn < groups; ++turn) {
    __syncthreads();
    if (!works || group != turn) continue;
    auto add = [&](int r, int c, const double (&v)[2]) {
      double2* p = reinterpret_cast<double2*>(out + 8 * r * s8 + 8 * c + at);
      double2 d = turn == 0 ? make_double2(0.0, 0.0) : __ldcg(p);
      d.x += v[0], d.y += v[1];
      __stcg(p, d);
    };
#pragma unroll
    for (int j = 0; j < kMostTiles; ++j) {
      if (j < tiles - r1) add(r1, tiles - 1 - j, acc1[j]);
      if (j < kMostTiles / 2 && j < tiles - r2 && r2 != r1) add(r2, tiles - 1 - j, acc2[j < kMostTiles / 2 ? j : 0]);
    }
  }
}

struct ChainArgs {
  const double* parts;
  int nparts, s, steps;
  double eps, scale;
  double* work;                  // [batch][6][s8][s8]; the last P, times scale and f, ends up in the first
  float abc[3 * kThinMostSteps];
};

// Tile (r, c) of A B for symmetric s8 x s8 matrices that commute: rows of A against rows of B.  A lane's k are 16 k0 + 4 (lane % 4) .. + 3.
__device__ __forceinline__ void tile_product(const double* a, const double* b, int r, int c, int s8, double (&d)[2]) {
  const int lane = threadIdx.x & 31;
  const double* pa = a + (8 * r + (lane >> 2)) * s8 + 4 * (lane & 3);
  const double* pb = b + (8 * c + (lane >> 2)) * s8 + 4 * (lane & 3);
  double even[2] = {0.0, 0.0}, odd[2] = {0.0, 0.0};
  const bool upper_in = 4 * (lane & 3) < 8;       // s8 is a multiple of 8: the last 16 may be half
#pragma unroll 4
  for (int k = 0; k < s8; k += 16) {
    double2 a0 = make_double2(0.0, 0.0), a1 = a0, b0 = a0, b1 = a0;
    if (k + 16 <= s8 || upper_in) {
      a0 = __ldcg(reinterpret_cast<const double2*>(pa + k)), a1 = __ldcg(reinterpret_cast<const double2*>(pa + k) + 1);
      b0 = __ldcg(reinterpret_cast<const double2*>(pb + k)), b1 = __ldcg(reinterpret_cast<const double2*>(pb + k) + 1);
    }
    dmma(even, a0.x, b0.x);
    dmma(odd, a0.y, b0.y);
    dmma(even, a1.x, b1.x);
    dmma(odd, a1.y, b1.y);
  }
  d[0] = even[0] + odd[0], d[1] = even[1] + odd[1];
}

// The steps.  A cluster of eight CTAs to a matrix: CTA c owns tile rows c and c + 8, its warp w tile columns w and w + 8.
__global__ void __launch_bounds__(kThreads)
thin_chain_kernel(const __grid_constant__ ChainArgs p) {
  __shared__ double s_norm;
  pdl_trigger();
  pdl_wait();
  const int s8 = (p.s + 7) / 8 * 8, tiles = s8 / 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cta = static_cast<int>(cluster_ctarank()), b = blockIdx.x / kCluster;
  const int64_t size = static_cast<int64_t>(s8) * s8;
  double* work = p.work + b * 6 * size;
  double *pa = work, *pb = work + size, *ga = work + 2 * size, *gb = work + 3 * size, *qm = work + 4 * size, *rm = work + 5 * size;
  auto each_tile = [&](auto f) {
    for (int r = cta; r < tiles; r += kCluster)
      for (int c = warp; c < tiles; c += kWarps) f(r, c, static_cast<int64_t>(8 * r + (lane >> 2)) * s8 + 8 * c + 2 * (lane & 3));
  };
  auto put = [](double* m, int64_t at, double x, double y) { __stcg(reinterpret_cast<double2*>(m + at), make_double2(x, y)); };
  auto meet = [] { cluster_arrive(); cluster_wait(); };

  const double* parts = p.parts + static_cast<int64_t>(b) * p.nparts * size;
  each_tile([&](int r, int c, int64_t at) {       // G from its parts, below the diagonal from above it
    double x = 0.0, y = 0.0;
    const int i = 8 * r + (lane >> 2), j = 8 * c + 2 * (lane & 3);
    for (int k = 0; k < p.nparts; ++k) {
      const double* q = parts + k * size;
      if (r <= c) {
        const double2 d = __ldcg(reinterpret_cast<const double2*>(q + at));
        x += d.x, y += d.y;
      } else {
        x += __ldcg(q + static_cast<int64_t>(j) * s8 + i), y += __ldcg(q + static_cast<int64_t>(j + 1) * s8 + i);
      }
    }
    put(ga, at, x, y);
  });
  meet();
  if (warp == 0) {
    double t = 0.0;
    for (int i = lane; i < s8; i += 32) t += __ldcg(ga + static_cast<int64_t>(i) * s8 + i);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, s);
    const double norm = sqrt(t) + p.eps;
    // an infinity or a NaN anywhere: NaN everywhere; nothing but zeros: zeros
    if (lane == 0) s_norm = !(t <= 1.7976931348623157e308) ? nan("") : norm > 0.0 ? 1.0 / norm : 0.0;
  }
  __syncthreads();
  const double f = s_norm;
  double gs = f * f;              // what G still has to be multiplied by
  for (int step = 0; step < p.steps; ++step) {
    const double ca = p.abc[3 * step], cb = p.abc[3 * step + 1], cc = p.abc[3 * step + 2];
    const bool last = step + 1 == p.steps;
    each_tile([&](int r, int c, int64_t at) {     // Q = a + b G + c G G
      double d[2];
      tile_product(ga, ga, r, c, s8, d);
      const double2 g = __ldcg(reinterpret_cast<const double2*>(ga + at));
      const int i = 8 * r + (lane >> 2), j = 8 * c + 2 * (lane & 3);
      double x = cb * gs * g.x + cc * gs * gs * d[0] + (i == j ? ca : 0.0), y = cb * gs * g.y + cc * gs * gs * d[1] + (i == j + 1 ? ca : 0.0);
      put(qm, at, x, y);
      if (step == 0) put(pb, at, x, y);
    });
    meet();
    each_tile([&](int r, int c, int64_t at) {     // P <- P Q (rows of P: this CTA's own), R = Q Q
      double d[2];
      if (step > 0) {
        tile_product(pa, qm, r, c, s8, d);
        put(pb, at, d[0], d[1]);
      }
      if (!last) {
        tile_product(qm, qm, r, c, s8, d);
        put(rm, at, d[0], d[1]);
      }
    });
    double* swap = pa;
    pa = pb, pb = swap;
    if (last) break;
    meet();
    each_tile([&](int r, int c, int64_t at) {     // G <- G Q Q
      double d[2];
      tile_product(ga, rm, r, c, s8, d);
      put(gb, at, gs * d[0], gs * d[1]);
    });
    gs = 1.0;
    swap = ga;
    ga = gb, gb = swap;
    meet();
  }
  __syncthreads();      // the rows that the last step read may be where the result goes
  // each tile by the warp that has just written it
  each_tile([&](int, int, int64_t at) {
    const double2 d = __ldcg(reinterpret_cast<const double2*>(pa + at));
    put(work, at, p.scale * f * d.x, p.scale * f * d.y);
  });
}

// out = X P by the long side's rows, 32 at a time; a warp keeps its tile columns of P (w, w + 8) in registers.
template <typename T, bool kTall>
__global__ void __launch_bounds__(kThreads)
thin_apply_kernel(const T* g, int64_t l, int s, const double* work, void* out, bool out_bf16, bool out_pairs) {
  extern __shared__ __align__(16) double tile[];
  pdl_trigger();
  pdl_wait();
  const int s8 = (s + 7) / 8 * 8, tiles = s8 / 8, pitch = pitch_of(s8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const T* x = g + blockIdx.y * l * s;
  const double* pm = work + blockIdx.y * 6 * static_cast<int64_t>(s8) * s8;
  double w[2][2 * kMostTiles];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int k = 0; k < 2 * kMostTiles; ++k)
      w[h][k] = warp + 8 * h < tiles && k < 2 * tiles ? __ldcg(pm + static_cast<int64_t>(8 * (warp + 8 * h) + (lane >> 2)) * s8 + 4 * k + (lane & 3)) : 0.0;
  Slab<T, kTall> slab;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRowsK;
  slab.load(x, l, l, s, s8, static_cast<int64_t>(blockIdx.x) * kRowsK);
  for (int64_t k0 = static_cast<int64_t>(blockIdx.x) * kRowsK; k0 < l; k0 += step) {
    __syncthreads();
    slab.put(tile, s8, pitch);
    __syncthreads();
    if (k0 + step < l) slab.load(x, l, l, s, s8, k0 + step);
    for (int rt = 0; rt < kRowsK / 8; ++rt) {
      double acc[2][2] = {};
      const double* at = tile + (8 * rt + (lane >> 2)) * pitch + (lane & 3);
#pragma unroll
      for (int k = 0; k < 2 * kMostTiles; ++k) {
        if (k < 2 * tiles) {
          const double v = at[4 * k];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (warp + 8 * h < tiles) {
              if (kTall) dmma(acc[h], v, w[h][k]); else dmma(acc[h], w[h][k], v);
            }
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (warp + 8 * h >= tiles) continue;
        // tall: row of the long side, two columns of the short one; wide: the other way round
        const int64_t long_at = k0 + 8 * rt + (kTall ? (lane >> 2) : 2 * (lane & 3));
        const int short_at = 8 * (warp + 8 * h) + (kTall ? 2 * (lane & 3) : (lane >> 2));
        const int64_t o = static_cast<int64_t>(blockIdx.y) * l * s + (kTall ? long_at * s + short_at : short_at * l + long_at);
        const bool in0 = long_at < l && short_at < s, in1 = kTall ? in0 && short_at + 1 < s : in0 && long_at + 1 < l;
        const float v0 = static_cast<float>(acc[h][0]), v1 = static_cast<float>(acc[h][1]);
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
int64_t parts_of(int64_t batch, int64_t l) {
  const int64_t most = (l + 2 * kRowsK - 1) / (2 * kRowsK), want = (sm_count() + batch - 1) / batch;
  return std::max<int64_t>(1, std::min(most, want));
}

template <typename T, bool kTall>
cudaError_t launch_of(const ThinPlan& p, int64_t l, int s, const void* g, void* out, void* scratch, cudaStream_t st) {
  const T* x = static_cast<const T*>(g);
  const int s8 = (s + 7) / 8 * 8;
  const size_t size = static_cast<size_t>(s8) * s8;
  double* work = static_cast<double*>(scratch);
  double* parts = work + p.batch * 6 * size;
  int64_t nparts = parts_of(p.batch, l);
  const int64_t per = round_up((l + nparts - 1) / nparts, kRowsK);
  nparts = (l + per - 1) / per;
  const size_t smem = static_cast<size_t>(kRowsK) * pitch_of(s8) * 8;
  const unsigned batch = static_cast<unsigned>(p.batch);
  cudaError_t e = launch_pdl(thin_gram_kernel<T, kTall>, dim3(static_cast<unsigned>(nparts), batch), dim3(kThreads), smem, st, 1, x, l, s, per, parts);
  if (e != cudaSuccess) return e;
  ChainArgs c{};
  c.parts = parts, c.nparts = static_cast<int>(nparts), c.s = s, c.steps = p.steps, c.eps = p.eps, c.scale = p.scale, c.work = work;
  for (int i = 0; i < 3 * p.steps; ++i) c.abc[i] = p.abc[i];
  e = launch_pdl(thin_chain_kernel, dim3(kCluster * batch), dim3(kThreads), 0, st, kCluster, c);
  if (e != cudaSuccess) return e;
  const int64_t chunks = (l + kRowsK - 1) / kRowsK, cap = std::max<int64_t>(1, 2 * sm_count() / p.batch);
  const bool pairs = (kTall ? s : l) % 2 == 0 && (reinterpret_cast<uintptr_t>(out) & (p.out_bf16 ? 3 : 7)) == 0;
  return launch_pdl(thin_apply_kernel<T, kTall>, dim3(static_cast<unsigned>(chunks < cap ? chunks : cap), batch), dim3(kThreads), smem, st, 1, x, l, s,
                    static_cast<const double*>(work), out, p.out_bf16, pairs);
}

}  // namespace

bool ortho_thin_takes(int64_t batch, int64_t rows, int64_t cols, const float* abc, int steps) {
  const int64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
  if (s > kThinMost) return false;
  // how far an error of G may grow before the last step's polynomial is taken: 2^-50 to 2^-24
  double growth = 1.0;
  for (int i = 0; i + 1 < steps; ++i) growth *= std::max(1.0, static_cast<double>(abc[3 * i]) * abc[3 * i]);
  if (!(growth <= 67108864.0)) return false;
  return s * s * l <= (int64_t{1} << 31) / batch;
}

size_t ortho_thin_scratch_bytes(int64_t batch, int64_t rows, int64_t cols) {
  const int64_t s = rows < cols ? rows : cols, l = rows < cols ? cols : rows, s8 = round_up(s, 8);
  return static_cast<size_t>(batch) * (6 + parts_of(batch, l)) * s8 * s8 * 8;
}

cudaError_t launch_ortho_thin(const ThinPlan& p, const void* g, void* out, void* scratch, cudaStream_t st) {
  const bool tall = p.rows > p.cols;
  const int64_t l = tall ? p.rows : p.cols;
  const int s = static_cast<int>(tall ? p.cols : p.rows);
  if (p.in_bf16) return tall ? launch_of<bf16_t, true>(p, l, s, g, out, scratch, st) : launch_of<bf16_t, false>(p, l, s, g, out, scratch, st);
  return tall ? launch_of<float, true>(p, l, s, g, out, scratch, st) : launch_of<float, false>(p, l, s, g, out, scratch, st);
}

}  // namespace falqon
