// The preference loss of paired sequences and its gradient (include/falqon_train.h).
//   row_stats_kernel   one pass over the counted rows' logits with a running maximum m and sum of exp(x - m)
//   sequence_kernel    joins a row's parts, takes log-probabilities, sums them per sequence, the pair's loss, d loss / d logp per row
//   logit_grad_kernel  dlogits = dlogp * ([v == target] - exp(x - m) / sum)
// exp(x - m) is taken as 2^((x - m) * log2 e) with the difference formed first: exact near the maximum whatever its size, and
// a row of the type's lowest values (a mask over the whole vocabulary) does not overflow on the way.  Its relative error, fp32 logits
// included: |x - m| * 2^-24 from the rounding of the difference, which any 32-bit form has, as much again from the product, a quarter of it
// from the constant, and 2^-22 from the instruction.  In a row's sum the values far below the maximum weigh nothing; of the gradient's
// values it is the error they are stored with (2^-17 of a value 55 below the maximum, whose own weight is 10^-24).
// HBM-bound: the forward reads each counted row once, the backward reads it again and writes every row once.  A row is a CTA's, so that
// all its vectors are in flight together and one row's reduction passes under the others' loads: 4096 x 32000 bf16, of which 3080 rows
// are counted, 38 us (5.2 TB/s; two special-function instructions and eight others per pair of values are issued on 54 % of cycles, and
// deeper prefetching, 2 or 8 vectors a turn, or a turn ahead, did not help).  The gradient of 16384 x 32000 runs at 6.6 TB/s.  The
// sequences' kernel is a chain of dependent loads, 5 us at any size.
#include <cfloat>
#include <type_traits>

#include "../../include/falqon_train.h"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kRowThreads = 256;
constexpr int kSeqThreads = 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxParts = 64;              // parts of one row
constexpr float kNotCounted = -1.0f;       // in the place of a row's (first part's) sum, which is never negative
constexpr size_t kCounterBytes = 256;      // the last-CTA counter at the head of the scratch

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

template <typename T>
struct Row {                               // vectors of 16 bytes
  static constexpr int kN = 16 / sizeof(T), kPairs = kN / 2;
};
__device__ __forceinline__ void expand(const uint4& q, f2 (&x)[4], bf16_t) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = pack_f32x2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u));
}
__device__ __forceinline__ void expand(const uint4& q, f2 (&x)[2], float) {
  x[0] = pack_f32x2(__uint_as_float(q.x), __uint_as_float(q.y));
  x[1] = pack_f32x2(__uint_as_float(q.z), __uint_as_float(q.w));
}
__device__ __forceinline__ uint4 shrink(const f2 (&x)[4], bf16_t) {
  float v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) unpack_f32x2(x[k], v[2 * k], v[2 * k + 1]);
  return pack8(v);
}
__device__ __forceinline__ uint4 shrink(const f2 (&x)[2], float) {
  float v[4];
  unpack_f32x2(x[0], v[0], v[1]);
  unpack_f32x2(x[1], v[2], v[3]);
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
// The largest of a vector's values (a NaN may be passed over: its exponential is one all the same).
__device__ __forceinline__ float largest_of(const uint4* q, int n, bf16_t) {
  uint32_t m = 0xFF80FF80u;                // two times -inf
#pragma unroll
  for (int j = 0; j < n; ++j) {
    const uint32_t w[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[k]));
  }
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
}
__device__ __forceinline__ float largest_of(const uint4* q, int n, float) {
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < n; ++j)
    m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(q[j].x), __uint_as_float(q[j].y)), fmaxf(__uint_as_float(q[j].z), __uint_as_float(q[j].w))));
  return m;
}
// exp(x - m) of two values.
__device__ __forceinline__ f2 exp_of2(f2 x, f2 minus_m) {
  float lo, hi;
  unpack_f32x2(mul2(add2(x, minus_m), twice(kLog2e)), lo, hi);
  return pack_f32x2(ex2(lo), ex2(hi));
}

// A row that may start anywhere: `head` single values up to a 16-byte boundary, `body` vectors, and the rest.
struct Span {
  int head;
  int64_t body, tail;                      // vectors; first value of the tail
};
template <typename T>
__device__ __forceinline__ Span span_of(const T* p, int64_t vocab) {
  constexpr int n = Row<T>::kN;
  const int off = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
  Span s;
  s.head = off == 0 ? 0 : n - off;
  if (s.head > vocab) s.head = static_cast<int>(vocab);
  s.body = (vocab - s.head) / n;
  s.tail = s.head + s.body * n;
  return s;
}

__device__ __forceinline__ float exp_of(float d) { return ex2(d * kLog2e); }

// A running maximum and the sum of exp(x - m) of the values seen.
struct Running {
  float m = -INFINITY, s = 0.0f;
  __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.0f : m; }   // all -inf so far: their powers are 0
  __device__ __forceinline__ void raise(float top) {
    if (top > m) {
      s *= exp_of(m - top);
      m = top;
    }
  }
  __device__ __forceinline__ void add(float x) {
    raise(x);
    s += exp_of(x - base());
  }
  __device__ __forceinline__ void join(float om, float os) {
    raise(om);
    s += os * exp_of(om - base());
  }
  // Those of a warp's lanes together: every sum brought to the largest maximum once, then added.
  __device__ __forceinline__ void join_warp() {
    float top;
    asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(top) : "f"(m));
    const float own = m;
    m = top;
    s *= exp_of(own - base());
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  }
};

// The vectors of a part, blockIdx.y: `chunk` of them, the last part's to the row's end.
struct Part {
  int64_t begin, end;
  __device__ __forceinline__ Part(const Span& sp, int64_t chunk) {
    begin = static_cast<int64_t>(blockIdx.y) * chunk;
    end = blockIdx.y == gridDim.y - 1 ? sp.body : min(begin + chunk, sp.body);
  }
};

// kTeam threads to a row or a part of one: a CTA, or a warp where rows are short (then parts == 1).
template <typename T, int kTeam>
__global__ void __launch_bounds__(kRowThreads) row_stats_kernel(int64_t rows, const T* logits, int64_t vocab, int64_t ld, const int64_t* targets,
                                                                int64_t chunk, float2* out, float* target_logit, unsigned int* counter, int* status) {
  __shared__ float red_m[kRowThreads / 32], red_s[kRowThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int part = blockIdx.y, parts = gridDim.y, tid = threadIdx.x % kTeam;
  if (blockIdx.x == 0 && part == 0 && threadIdx.x == 0) *counter = 0u;   // for the kernel after this one
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kRowThreads / kTeam) + threadIdx.x / kTeam;
  if (kTeam < kRowThreads && row >= rows) return;
  const int64_t target = ld_stream(targets + row);
  if (target < 0 || target >= vocab) {
    if (part == 0 && tid == 0) {
      out[row * parts] = make_float2(0.0f, kNotCounted);
      if (target >= vocab) atomicExch(status, FALQON_ERR_INVALID_ARG);
    }
    return;
  }
  const T* p = logits + row * ld;
  float at_target = 0.0f;                  // fetched here, beside the stream, and not in a gather of the next kernel
  if (part == 0 && tid == 0) at_target = load1(p + target);
  const Span sp = span_of(p, vocab);
  Running r;
  const uint4* body = reinterpret_cast<const uint4*>(p + sp.head);
  const auto [begin, end] = Part(sp, chunk);
  f2 sum = 0;                              // the running sum, two halves of it
  constexpr int kUnroll = 4;
  constexpr uint32_t kNone = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;   // -inf: adds nothing
  for (int64_t v = begin + tid; v < end; v += kUnroll * kTeam) {
    uint4 q[kUnroll];
    if (v + (kUnroll - 1) * kTeam < end) {
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) q[j] = ld_stream(body + v + j * kTeam);
    } else {
#pragma unroll
      for (int j = 0; j < kUnroll; ++j)
        q[j] = v + j * kTeam < end ? ld_stream(body + v + j * kTeam) : make_uint4(kNone, kNone, kNone, kNone);
    }
    const float top = largest_of(q, kUnroll, T{});
    if (top > r.m) {                       // seldom after the first vectors
      sum = mul2(sum, twice(exp_of(r.m - top)));
      r.m = top;
    }
    const f2 minus = twice(-r.base());
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      f2 x[Row<T>::kPairs];
      expand(q[j], x, T{});
#pragma unroll
      for (int k = 0; k < Row<T>::kPairs; ++k) sum = add2(sum, exp_of2(x[k], minus));
    }
  }
  r.s = halves(sum);
  if (part == 0) {
    if (tid < sp.head) r.add(load1(p + tid));
    if (tid < vocab - sp.tail) r.add(load1(p + sp.tail + tid));
  }
  r.join_warp();
  if (kTeam > 32) {
    if ((tid & 31) == 0) {
      red_m[tid >> 5] = r.m;
      red_s[tid >> 5] = r.s;
    }
    __syncthreads();
    if (tid >= 32) return;
    const bool one = tid < kTeam / 32;
    r.m = one ? red_m[tid] : -INFINITY;
    r.s = one ? red_s[tid] : 0.0f;
    r.join_warp();
  }
  if (tid == 0) {
    out[row * parts + part] = make_float2(r.m, r.s);
    if (part == 0) target_logit[row] = at_target;
  }
}

struct SeqArgs {
  const int64_t* cu;
  int64_t rows;
  const float2* part;                      // [rows][parts]
  const float* target_logit;               // [rows]
  int parts;
  float2* stats;                           // [rows], nullable (may be `part` when parts == 1)
  float *logp, *seq_logp;                  // logp nullable
  // pairs only
  const float* ref;
  float *loss, *pair_loss, *dlogp;
  unsigned int* counter;
  int kind, average;
  float beta, margin, smoothing, nll_weight;
};

// Sums over the CTA in a fixed order, for its first warp.  64-bit additions are slow here (a warp's takes many cycles), so sums are
// taken in 64 bits once per row and then by shuffles, counts as integers, and one warp does the rest for all.
struct Sums {
  double first, second;                    // of the chosen (or only) and the rejected sequence
  unsigned n_first, n_second;
};
__device__ __forceinline__ Sums warp_sums(Sums v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.first += __shfl_xor_sync(0xFFFFFFFFu, v.first, o);
    v.second += __shfl_xor_sync(0xFFFFFFFFu, v.second, o);
  }
  v.n_first = __reduce_add_sync(0xFFFFFFFFu, v.n_first);
  v.n_second = __reduce_add_sync(0xFFFFFFFFu, v.n_second);
  return v;
}
__device__ __forceinline__ Sums cta_sums(Sums v, Sums* red) {
  v = warp_sums(v);
  const int warps = static_cast<int>(blockDim.x >> 5);
  if (warps == 1) return v;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  if (threadIdx.x >= 32) return v;
  return warp_sums(static_cast<int>(threadIdx.x) < warps ? red[threadIdx.x] : Sums{0.0, 0.0, 0u, 0u});
}

// The log-probability of one row (0 and false: not counted) from its target's logit, its first part and the others.
__device__ __forceinline__ bool row_logp(const SeqArgs& a, int64_t row, float x, const float2& head, float& lp) {
  lp = 0.0f;
  if (head.y == kNotCounted) return false;           // the other parts were not written
  Running r{head.x, head.y};
  const float2* part = a.part + row * a.parts;
  constexpr int kAhead = 4;
  for (int i = 1; i < a.parts; i += kAhead) {
    float2 q[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) q[j] = i + j < a.parts ? ld_stream(part + i + j) : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) r.join(q[j].x, q[j].y);
  }
  if (a.stats != nullptr) a.stats[row] = make_float2(r.m, r.s);
  lp = (x - r.m) - logf(r.s);
  return true;
}

__device__ __forceinline__ int64_t bound_at(const SeqArgs& a, int64_t i) {   // cu_rows[i], brought into [0, rows]
  const int64_t v = ld_stream(a.cu + i);
  return v < 0 ? 0 : v > a.rows ? a.rows : v;
}

// Rows outside every sequence: not counted.
__device__ __forceinline__ void clear_rows(const SeqArgs& a, int64_t begin, int64_t end) {
  for (int64_t row = begin + threadIdx.x; row < end; row += blockDim.x) {
    if (a.logp != nullptr) a.logp[row] = 0.0f;
    if (a.dlogp != nullptr) a.dlogp[row] = 0.0f;
  }
}

// log sigmoid and sigmoid of d and of -d.  q = exp(-|d|) is taken in 32 bits, its argument's rounding made good to the first order, so that
// every value has a few units of 2^-23 of its own size; what is added to large numbers is added in 64 bits.  (The 64-bit functions would
// be hundreds of instructions in a kernel that is one dependent chain.)
struct Sigmoids {
  double log_of, log_of_minus;
  float of, of_minus;
  __device__ __forceinline__ explicit Sigmoids(double d) {
    const double size = fabs(d) > 256.0 ? 256.0 : fabs(d);   // exp(-256) is 0 in 32 bits; a NaN stays one
    const float near = static_cast<float>(size);
    const float e = expf(-near), q = __fmaf_rn(-e, static_cast<float>(size - static_cast<double>(near)), e);
    const double tail = static_cast<double>(log1pf(q));
    log_of = (d < 0.0 ? d : 0.0) - tail;
    log_of_minus = (d > 0.0 ? -d : 0.0) - tail;
    const float large = 1.0f / (1.0f + q), small = q * large;
    of = d < 0.0 ? small : large;
    of_minus = d < 0.0 ? large : small;
  }
};

template <bool kPairs>
__global__ void __launch_bounds__(kSeqThreads) sequence_kernel(const SeqArgs a) {
  __shared__ Sums red[kSeqThreads / 32];
  __shared__ float s_coef[2];
  __shared__ bool s_last;
  pdl_trigger();
  pdl_wait();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kPairs ? 2 : 1);
  const int64_t begin = bound_at(a, first), mid = max(begin, bound_at(a, first + 1)), end = kPairs ? max(mid, bound_at(a, first + 2)) : mid;
  float ref[2] = {0.0f, 0.0f};
  if (kPairs && a.ref != nullptr) {
    ref[0] = ld_stream(a.ref + first);
    ref[1] = ld_stream(a.ref + first + 1);
  }
  if (blockIdx.x == 0) clear_rows(a, 0, begin);
  if (blockIdx.x == gridDim.x - 1) clear_rows(a, end, a.rows);
  uint64_t seen = 0;                       // which of the thread's first 64 rows are counted
  int turn = 0;
  Sums t{0.0, 0.0, 0u, 0u};
  constexpr int kRows = 4;                 // a thread's rows in flight
  for (int64_t row0 = begin + threadIdx.x; row0 < end; row0 += kRows * blockDim.x) {
    float x[kRows];
    float2 head[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int64_t row = row0 + j * blockDim.x;
      if (row >= end) break;
      x[j] = ld_stream(a.target_logit + row);        // anything where the row is not counted
      head[j] = ld_stream(a.part + row * a.parts);
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j, ++turn) {
      const int64_t row = row0 + j * blockDim.x;
      if (row >= end) break;
      float lp;
      const bool counted = row_logp(a, row, x[j], head[j], lp);
      if (a.logp != nullptr) a.logp[row] = lp;
      if (!counted) continue;
      if (turn < 64) seen |= 1ull << turn;
      if (kPairs && row >= mid) {
        t.second += static_cast<double>(lp);
        ++t.n_second;
      } else {
        t.first += static_cast<double>(lp);
        ++t.n_first;
      }
    }
  }
  t = cta_sums(t, red);
  if (threadIdx.x < 32) {
    const double n1 = max(t.n_first, 1u), n2 = max(t.n_second, 1u);
    const double chosen = a.average ? t.first / n1 : t.first;
    if constexpr (!kPairs) {
      if (threadIdx.x == 0) a.seq_logp[first] = static_cast<float>(chosen);
    } else {
      // 64 bits up to the results: u, d and the squared loss are differences of numbers much larger than themselves
      const double rejected = a.average ? t.second / n2 : t.second;
      const double u = (chosen - static_cast<double>(ref[0])) - (rejected - static_cast<double>(ref[1]));
      const double beta = a.beta, d = beta * u - a.margin;
      double l, du;
      if (a.kind == FALQON_PREFERENCE_SIGMOID) {
        const double eps = a.smoothing;    // a term of weight 0 is left out: its logarithm may be infinite
        const Sigmoids s(d);
        l = (eps < 1.0 ? -(1.0 - eps) * s.log_of : 0.0) - (eps > 0.0 ? eps * s.log_of_minus : 0.0);
        du = beta * (eps * s.of - (1.0 - eps) * s.of_minus);
      } else if (a.kind == FALQON_PREFERENCE_HINGE) {
        l = d < 1.0 ? 1.0 - d : d >= 1.0 ? 0.0 : d;     // a NaN stays one
        du = d < 1.0 ? -beta : d >= 1.0 ? 0.0 : d;
      } else {
        const double v = u - a.margin - 0.5 / beta;
        l = v * v;
        du = 2.0 * v;
      }
      const double pairs = gridDim.x, nll = a.nll_weight == 0.0f ? 0.0 : static_cast<double>(a.nll_weight) / n1;
      if (nll != 0.0) l -= nll * t.first;
      if (threadIdx.x == 0) {
        const float out = static_cast<float>(l);
        a.seq_logp[first] = static_cast<float>(chosen);
        a.seq_logp[first + 1] = static_cast<float>(rejected);
        a.pair_loss[blockIdx.x] = out;
        if (gridDim.x == 1) *a.loss = out;
        s_coef[0] = static_cast<float>(((a.average ? du / n1 : du) - nll) / pairs);
        s_coef[1] = static_cast<float>(-(a.average ? du / n2 : du) / pairs);
      }
    }
  }
  if constexpr (kPairs) {
    // the CTA that finishes last takes the mean of all pairs' losses, in an order of its own that never changes
    if (threadIdx.x == 0) {
      s_last = false;
      if (gridDim.x > 1) {
        __threadfence();
        s_last = atomicAdd(a.counter, 1u) == gridDim.x - 1;
      }
    }
    __syncthreads();
    if (a.dlogp != nullptr) {
      const float c = s_coef[0], r = s_coef[1];
      turn = 0;
      for (int64_t row = begin + threadIdx.x; row < end; row += blockDim.x, ++turn) {
        const bool counted = turn < 64 ? (seen >> turn & 1) != 0 : ld_stream(&a.part[row * a.parts].y) != kNotCounted;
        a.dlogp[row] = !counted ? 0.0f : row < mid ? c : r;
      }
    }
    if (s_last) {
      __threadfence();
      Sums all{0.0, 0.0, 0u, 0u};
      for (int64_t i = threadIdx.x; i < gridDim.x; i += blockDim.x) all.first += static_cast<double>(ld_stream(a.pair_loss + i));
      all = cta_sums(all, red);
      if (threadIdx.x == 0) *a.loss = static_cast<float>(all.first / static_cast<double>(gridDim.x));
    }
  }
}

// kSame: logits and dlogits rows have the same offset from a 16-byte boundary, so vectors can be stored; else single values are (the
// whole step of 16384 x 32000 bf16: 410 us with vectors, 1456 with single values).
template <typename T, bool kSame, int kTeam>
__global__ void __launch_bounds__(kRowThreads) logit_grad_kernel(int64_t rows, const T* logits, int64_t vocab, int64_t ld, const int64_t* targets,
                                                                 int64_t chunk, const float2* stats, const float* dlogp, const float* dloss,
                                                                 T* out, int64_t ld_out, float* amax) {
  pdl_trigger();
  pdl_wait();
  constexpr int n = Row<T>::kN;
  // the last rows first: of what the forward has read, they are still in L2
  const int64_t row = rows - 1 - (static_cast<int64_t>(blockIdx.x) * (kRowThreads / kTeam) + threadIdx.x / kTeam);
  const int tid = threadIdx.x % kTeam;
  uint32_t mx = 0;
  if (row >= 0) {
    const float own = ld_stream(dlogp + row), c = own * (dloss != nullptr ? ld_stream(dloss) : 1.0f);
    const T* p = logits + row * ld;
    T* o = out + row * ld_out;
    const Span sp = span_of(p, vocab);
    const auto [begin, end] = Part(sp, chunk);
    const uint4* body = reinterpret_cast<const uint4*>(p + sp.head);
    const bool zero = own == 0.0f || c == 0.0f;                // a row that is not counted stays so under an infinite or NaN dloss
    const float2 st = zero ? make_float2(0.0f, 1.0f) : ld_stream(stats + row);
    const int64_t target = zero ? -1 : ld_stream(targets + row);
    const float f = -c / st.y;
    const auto one = [&](int64_t i) {
      const float g = zero ? 0.0f : __fmaf_rn(f, exp_of(load1(p + i) - st.x), i == target ? c : 0.0f);
      mx = max(mx, store1(o + i, g));
    };
    // one vector: its values' gradients
    const auto put = [&](int64_t v, const uint4& q) {
      const int64_t at = sp.head + v * n;
      f2 x[Row<T>::kPairs];
      if (zero) {
#pragma unroll
        for (int k = 0; k < Row<T>::kPairs; ++k) x[k] = 0;
      } else {
        expand(q, x, T{});
#pragma unroll
        for (int k = 0; k < Row<T>::kPairs; ++k) x[k] = mul2(twice(f), exp_of2(x[k], twice(-st.x)));
        if (target >= at && target < at + n) {
#pragma unroll
          for (int k = 0; k < Row<T>::kPairs; ++k) {
            if (at + 2 * k == target) x[k] = add2(x[k], pack_f32x2(c, 0.0f));
            if (at + 2 * k + 1 == target) x[k] = add2(x[k], pack_f32x2(0.0f, c));
          }
        }
      }
      const uint4 w = shrink(x, T{});
      if (kSame) {
        *reinterpret_cast<uint4*>(o + at) = w;
        if (amax != nullptr) {
          expand(w, x, T{});
#pragma unroll
          for (int k = 0; k < Row<T>::kPairs; ++k) {
            float lo, hi;
            unpack_f32x2(x[k], lo, hi);
            mx = max(mx, max(abs_bits(lo), abs_bits(hi)));
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < Row<T>::kPairs; ++k) {
          float lo, hi;
          unpack_f32x2(x[k], lo, hi);
          mx = max(mx, max(store1(o + at + 2 * k, lo), store1(o + at + 2 * k + 1, hi)));
        }
      }
    };
    constexpr int kUnroll = 4;
    int64_t v = begin + tid;
    for (; v + (kUnroll - 1) * kTeam < end; v += kUnroll * kTeam) {
      uint4 q[kUnroll];
      if (!zero) {
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) q[j] = ld_stream(body + v + j * kTeam);
      }
#pragma unroll
      for (int j = 0; j < kUnroll; ++j) put(v + j * kTeam, q[j]);
    }
    for (; v < end; v += kTeam) put(v, zero ? make_uint4(0u, 0u, 0u, 0u) : ld_stream(body + v));
    if (blockIdx.y == 0) {
      if (tid < sp.head) one(tid);
      if (tid < vocab - sp.tail) one(sp.tail + tid);
    }
  }
  if (amax != nullptr) raise_amax(mx, amax);
}

// Logits may start at any value of their type: a row's vectors begin at the next 16-byte boundary.
inline bool ok_values(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == FALQON_BF16 ? 1 : 3)) == 0; }
inline bool ok16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int finish(cudaError_t e) { return e == cudaSuccess ? FALQON_OK : FALQON_ERR_CUDA; }

bool sizes_ok(int64_t rows, int64_t vocab, int dtype) {
  return rows >= 1 && rows < (1ll << 31) / kMaxParts && vocab >= 1 && vocab < (1ll << 31) &&
         (dtype == FALQON_BF16 || dtype == FALQON_F32);
}

// Into how many parts a row is cut: none where the rows alone fill the GPU, and no part below two vectors per thread.  Loss and gradient
// of 300 x 128000 bf16: 43 us by four parts, 58 by whole rows.
int parts_for(int64_t rows, int64_t vocab, int dtype) {
  const int64_t want = (148 * 8 + rows - 1) / rows;
  const int64_t most = vocab / (dtype == FALQON_BF16 ? 8 : 4) / (2 * kRowThreads);
  int64_t parts = want < most ? want : most;
  if (parts > kMaxParts) parts = kMaxParts;
  return static_cast<int>(parts < 1 ? 1 : parts);
}

// Vectors of a part, of a row that begins on a 16-byte boundary; the others' have one less at the most.
int64_t chunk_for(int64_t vocab, int dtype, int parts) { return (vocab / (dtype == FALQON_BF16 ? 8 : 4) + parts - 1) / parts; }

// A thread per row of the average sequence (or pair): 1500 x 8000 bf16, four pairs, loss and gradient 26.7 us, with 1024 threads 28.0.  Four warps
// at least, since sequences differ and a thread takes several rows of a long one: 699 pairs of 2 rows and one of 8000, 1000 columns, 46 us, from
// one warp on 135, from eight on 40, which 4096 pairs of 10 rows pay with 81 us, against 69 and 68.
unsigned sequence_threads(int64_t rows, int64_t ctas) {
  const int64_t t = (rows / ctas + 31) / 32 * 32;
  return static_cast<unsigned>(t < 128 ? 128 : t > kSeqThreads ? kSeqThreads : t);
}

// A warp to a row where rows are short and enough of them, a CTA otherwise; by the 16-byte vectors of a row.  A CTA takes 5 us per 1000 rows
// whatever their length; a warp, which has a few loads in flight only, needs ten or more beside it on its SM.  Loss and gradient, bf16, by
// warps / by CTAs:
//               1000 columns   2000        4000        6000        8000        12000
//   300 rows     12.4 / 11.8   14.5 / 12.4 16.5 / 12.4 18.6 / 12.4 20.6 / 14.4
//   1000 rows    12.4 / 14.4   14.2 / 15.1 16.5 / 16.5 23.5 / 17.3 28.7 / 20.8
//   2400 rows    14.4 / 19.3   16.5 / 21.4 24.7 / 25.4 30.3 / 28.8 35.9 / 33.5 47.8 / 41.3
//   4000 rows    16.5 / 24.7   20.7 / 30.8 29.0 / 34.9 37.3 / 41.3 45.8 / 49.4
//   12000 rows   30.7 / 63.5   40.6 / 72.4 67.2 / 92.5 92.2 / 112  118 / 126
//   16000 rows   36.5 / 81.2   50.5 / 96.8 84.2 / 124  115 / 149   147 / 164   208 / 221
bool by_warps(int64_t rows, int64_t vocab, int dtype) {
  const int64_t vecs = vocab / (dtype == FALQON_BF16 ? 8 : 4);
  return vecs < 1024 && (rows >= 4000 || (vecs < 512 && 2 * vecs <= rows));            // then a row has one part
}

template <typename T>
cudaError_t launch_row_stats(const void* logits, int64_t rows, int64_t vocab, int64_t ld, const int64_t* targets, int parts, bool warps, float2* out,
                             float* target_logit, unsigned int* counter, int* status, cudaStream_t stream) {
  const int64_t per = warps ? kRowThreads / 32 : 1, chunk = chunk_for(vocab, sizeof(T) == 2 ? FALQON_BF16 : FALQON_F32, parts);
  return launch_pdl(warps ? row_stats_kernel<T, 32> : row_stats_kernel<T, kRowThreads>, dim3(static_cast<unsigned>((rows + per - 1) / per), parts),
                    dim3(kRowThreads), 0, stream, 1, rows, static_cast<const T*>(logits), vocab, ld, targets, chunk, out, target_logit, counter, status);
}
cudaError_t launch_row_stats(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const int64_t* targets, int parts,
                             float2* out, float* target_logit, unsigned int* counter, int* status, cudaStream_t stream) {
  const bool warps = by_warps(rows, vocab, dtype);
  return dtype == FALQON_BF16 ? launch_row_stats<bf16_t>(logits, rows, vocab, ld, targets, parts, warps, out, target_logit, counter, status, stream)
                              : launch_row_stats<float>(logits, rows, vocab, ld, targets, parts, warps, out, target_logit, counter, status, stream);
}

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

size_t falqon_preference_scratch_bytes(int64_t rows, int64_t vocab, int dtype) {
  if (!sizes_ok(rows, vocab, dtype)) return 0;
  return kCounterBytes + static_cast<size_t>(rows) * (parts_for(rows, vocab, dtype) * sizeof(float2) + sizeof(float));
}

int falqon_sequence_logprob(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const int64_t* targets,
                            const int64_t* cu_rows, int64_t n_seq, int average, float* logp, float* seq_logp, void* scratch,
                            size_t scratch_bytes, falqon_stream stream) {
  if (logits == nullptr || targets == nullptr || cu_rows == nullptr || seq_logp == nullptr || !ok_values(logits, dtype) ||
      !sizes_ok(rows, vocab, dtype) || ld < vocab || n_seq < 1 || n_seq > (1ll << 30))
    return FALQON_ERR_INVALID_ARG;
  if (scratch == nullptr || !ok16(scratch) || scratch_bytes < falqon_preference_scratch_bytes(rows, vocab, dtype)) return FALQON_ERR_WORKSPACE;
  int* status = device_status_ptr();
  if (status == nullptr) return FALQON_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int parts = parts_for(rows, vocab, dtype);
  SeqArgs a{};
  float2* part = reinterpret_cast<float2*>(static_cast<uint8_t*>(scratch) + kCounterBytes);
  a.cu = cu_rows;
  a.rows = rows;
  float* target_logit = reinterpret_cast<float*>(part + rows * parts);
  a.part = part;
  a.parts = parts;
  a.target_logit = target_logit;
  a.logp = logp;
  a.seq_logp = seq_logp;
  a.average = average != 0;
  const cudaError_t e = launch_row_stats(logits, dtype, rows, vocab, ld, targets, parts, part, target_logit, static_cast<unsigned int*>(scratch), status, st);
  if (e != cudaSuccess) return FALQON_ERR_CUDA;
  return finish(launch_pdl(sequence_kernel<false>, dim3(static_cast<unsigned>(n_seq)), dim3(sequence_threads(rows, n_seq)), 0, st, 1, a));
}

static bool preference_ok(const falqon_preference* p) {
  return p != nullptr && sizes_ok(p->rows, p->vocab, p->dtype) && p->ld >= p->vocab && p->pairs >= 1 && p->pairs < (1ll << 30) &&
         p->kind >= FALQON_PREFERENCE_SIGMOID && p->kind <= FALQON_PREFERENCE_IPO && (p->flags & ~FALQON_PREFERENCE_AVERAGE) == 0 &&
         p->beta > 0.0f && p->beta <= FLT_MAX && p->margin >= -FLT_MAX && p->margin <= FLT_MAX && p->label_smoothing >= 0.0f &&
         p->label_smoothing <= 1.0f && (p->label_smoothing == 0.0f || p->kind == FALQON_PREFERENCE_SIGMOID) &&
         p->nll_weight >= 0.0f && p->nll_weight <= FLT_MAX;
}

int falqon_preference_forward(const falqon_preference* p, const void* logits, const int64_t* targets, const int64_t* cu_rows,
                              const float* ref_logp, float* loss, float* pair_loss, float* seq_logp, float* logp, float* row_stats,
                              float* dlogp, void* scratch, size_t scratch_bytes, falqon_stream stream) {
  if (!preference_ok(p) || logits == nullptr || targets == nullptr || cu_rows == nullptr || loss == nullptr || pair_loss == nullptr ||
      seq_logp == nullptr || logp == nullptr || !ok_values(logits, p->dtype) || (row_stats != nullptr) != (dlogp != nullptr) ||
      (reinterpret_cast<uintptr_t>(row_stats) & 7) != 0)
    return FALQON_ERR_INVALID_ARG;
  if (scratch == nullptr || !ok16(scratch) || scratch_bytes < falqon_preference_scratch_bytes(p->rows, p->vocab, p->dtype))
    return FALQON_ERR_WORKSPACE;
  int* status = device_status_ptr();
  if (status == nullptr) return FALQON_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int parts = parts_for(p->rows, p->vocab, p->dtype);
  float2* stats = reinterpret_cast<float2*>(row_stats);
  float2* const own = reinterpret_cast<float2*>(static_cast<uint8_t*>(scratch) + kCounterBytes);
  float2* part = parts == 1 && stats != nullptr ? stats : own;
  float* target_logit = reinterpret_cast<float*>(own + p->rows * parts);
  SeqArgs a{};
  a.cu = cu_rows;
  a.rows = p->rows;
  a.part = part;
  a.parts = parts;
  a.target_logit = target_logit;
  a.stats = part == stats ? nullptr : stats;
  a.logp = logp;
  a.seq_logp = seq_logp;
  a.ref = ref_logp;
  a.loss = loss;
  a.pair_loss = pair_loss;
  a.dlogp = dlogp;
  a.counter = static_cast<unsigned int*>(scratch);
  a.kind = p->kind;
  a.average = (p->flags & FALQON_PREFERENCE_AVERAGE) != 0;
  a.beta = p->beta;
  a.margin = p->margin;
  a.smoothing = p->label_smoothing;
  a.nll_weight = p->nll_weight;
  const cudaError_t e = launch_row_stats(logits, p->dtype, p->rows, p->vocab, p->ld, targets, parts, part, target_logit, a.counter, status, st);
  if (e != cudaSuccess) return FALQON_ERR_CUDA;
  return finish(launch_pdl(sequence_kernel<true>, dim3(static_cast<unsigned>(p->pairs)), dim3(sequence_threads(p->rows, p->pairs)), 0, st, 1, a));
}

int falqon_preference_backward(const falqon_preference* p, const void* logits, const int64_t* targets, const float* row_stats,
                               const float* dlogp, const float* dloss, void* dlogits, int64_t ld_out, float* amax_out,
                               falqon_stream stream) {
  if (!preference_ok(p) || logits == nullptr || targets == nullptr || row_stats == nullptr || dlogp == nullptr || dlogits == nullptr ||
      ld_out < p->vocab || !ok_values(logits, p->dtype) || !ok_values(dlogits, p->dtype) || (reinterpret_cast<uintptr_t>(row_stats) & 7) != 0 ||
      (logits == dlogits && ld_out != p->ld))
    return FALQON_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int parts = parts_for(p->rows, p->vocab, p->dtype);
  const bool same = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits)) & 15) == 0 &&
                    (ld_out - p->ld) % (p->dtype == FALQON_BF16 ? 8 : 4) == 0;
  const bool warps = by_warps(p->rows, p->vocab, p->dtype);
  const int64_t per = warps ? kRowThreads / 32 : 1, chunk = chunk_for(p->vocab, p->dtype, parts);
  const float2* stats = reinterpret_cast<const float2*>(row_stats);
  const auto go = [&](auto kernel, auto* typed) {
    using T = std::remove_pointer_t<decltype(typed)>;
    return finish(launch_pdl(kernel, dim3(static_cast<unsigned>((p->rows + per - 1) / per), parts), dim3(kRowThreads), 0, st, 1, p->rows,
                             static_cast<const T*>(logits), p->vocab, p->ld, targets, chunk, stats, dlogp, dloss, typed, ld_out, amax_out));
  };
  const auto pick = [&](auto* typed) {
    using T = std::remove_pointer_t<decltype(typed)>;
    if (warps) return same ? go(logit_grad_kernel<T, true, 32>, typed) : go(logit_grad_kernel<T, false, 32>, typed);
    return same ? go(logit_grad_kernel<T, true, kRowThreads>, typed) : go(logit_grad_kernel<T, false, kRowThreads>, typed);
  };
  return p->dtype == FALQON_BF16 ? pick(static_cast<bf16_t*>(dlogits)) : pick(static_cast<float*>(dlogits));
}

}  // extern "C"
