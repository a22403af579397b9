// The preference loss of paired sequences and its gradient (include/falqon_train.h).
//   row_stats_kernel   one pass over the counted rows' logits with a running maximum m and sum of exp(x - m)
//   sequence_kernel    joins a row's parts, takes log-probabilities, sums them per sequence, the pair's loss, d loss / d logp per row
//   logit_grad_kernel  dlogits = dlogp * ([v == target] - exp(x - m) / sum)
// exp(x - m) is taken as 2^((x - m) * log2 e) with the difference formed first: exact near the maximum whatever its size, and
// a row of the type's lowest values (a mask over the whole vocabulary) does not overflow on the way.
// HBM-bound: the forward reads each counted row once, the backward reads it again and writes every row once.
#include <cfloat>

#include "../../include/falqon_train.h"
#include "internal.h"
#include "mx8.cuh"
#include "ptx.cuh"

namespace falqon {
namespace {

constexpr int kRowThreads = 256;
constexpr int kSeqThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxParts = 64;              // parts of one row
constexpr size_t kCounterBytes = 256;      // the last-CTA counter at the head of the scratch

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

template <typename T>
struct Row {                               // vectors of 16 bytes
  static constexpr int kN = 16 / sizeof(T);
};
__device__ __forceinline__ void expand(const uint4& q, float (&x)[8], bf16_t) { unpack8(q, x); }
__device__ __forceinline__ void expand(const uint4& q, float (&x)[4], float) {
  x[0] = __uint_as_float(q.x), x[1] = __uint_as_float(q.y), x[2] = __uint_as_float(q.z), x[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ uint4 shrink(const float (&x)[8], bf16_t) { return pack8(x); }
__device__ __forceinline__ uint4 shrink(const float (&x)[4], float) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
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
};

template <typename T>
__global__ void __launch_bounds__(kRowThreads) row_stats_kernel(const T* logits, int64_t vocab, int64_t ld, const int64_t* targets,
                                                                int parts, float2* out, unsigned int* counter, int* status) {
  __shared__ float red_m[kRowThreads / 32], red_s[kRowThreads / 32];
  pdl_trigger();
  pdl_wait();
  constexpr int n = Row<T>::kN;
  if (blockIdx.x == 0 && threadIdx.x == 0) *counter = 0u;   // for the kernel after this one
  const int64_t row = blockIdx.x / parts;
  const int part = static_cast<int>(blockIdx.x - row * parts);
  const int64_t target = ld_stream(targets + row);
  if (target < 0) return;
  if (target >= vocab) {
    if (part == 0 && threadIdx.x == 0) atomicExch(status, FALQON_ERR_INVALID_ARG);
    return;
  }
  const T* p = logits + row * ld;
  const Span sp = span_of(p, vocab);
  Running r;
  const uint4* body = reinterpret_cast<const uint4*>(p + sp.head);
  const int64_t begin = sp.body * part / parts, end = sp.body * (part + 1) / parts;
  constexpr int kUnroll = 4;
  for (int64_t v = begin + threadIdx.x; v < end; v += kRowThreads * kUnroll) {
    uint4 q[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j)
      if (v + j * kRowThreads < end) q[j] = ld_stream(body + v + j * kRowThreads);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      if (v + j * kRowThreads >= end) break;
      float x[n];
      expand(q[j], x, T{});
      float top = x[0];
#pragma unroll
      for (int i = 1; i < n; ++i) top = fmaxf(top, x[i]);
      r.raise(top);
      const float b = r.base();
#pragma unroll
      for (int i = 0; i < n; ++i) r.s += exp_of(x[i] - b);
    }
  }
  if (part == 0) {
    if (static_cast<int>(threadIdx.x) < sp.head) r.add(load1(p + threadIdx.x));
    if (threadIdx.x < vocab - sp.tail) r.add(load1(p + sp.tail + threadIdx.x));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float om = __shfl_xor_sync(0xFFFFFFFFu, r.m, o), os = __shfl_xor_sync(0xFFFFFFFFu, r.s, o);
    r.join(om, os);
  }
  if ((threadIdx.x & 31) == 0) {
    red_m[threadIdx.x >> 5] = r.m;
    red_s[threadIdx.x >> 5] = r.s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kRowThreads / 32; ++w) r.join(red_m[w], red_s[w]);
    out[row * parts + part] = make_float2(r.m, r.s);
  }
}

struct SeqArgs {
  const int64_t *targets, *cu;
  int64_t rows, vocab, ld, seqs;
  const float2* part;                      // [rows][parts]
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

__device__ __forceinline__ double block_sum(double v, double* red) {   // fixed order; every thread gets it
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kSeqThreads / 32; ++w) t += red[w];
  return t;
}

// The log-probability of one row (0, not counted: false).
template <typename T>
__device__ __forceinline__ bool row_logp(const SeqArgs& a, const T* logits, int64_t row, float& lp) {
  const int64_t target = ld_stream(a.targets + row);
  lp = 0.0f;
  if (target < 0 || target >= a.vocab) return false;
  const float x = load1(logits + row * a.ld + target);
  Running r;
  for (int i = 0; i < a.parts; ++i) {
    const float2 q = ld_stream(a.part + row * a.parts + i);
    r.join(q.x, q.y);
  }
  if (a.stats != nullptr) a.stats[row] = make_float2(r.m, r.s);
  lp = (x - r.m) - logf(r.s);
  return true;
}

// Rows [begin, end) of one sequence: the sum of their log-probabilities and how many are counted; logp per row is stored.
template <typename T>
__device__ __forceinline__ void sequence_sum(const SeqArgs& a, const T* logits, int64_t begin, int64_t end, double* red, double& sum,
                                             double& count) {
  double s = 0.0, n = 0.0;
  for (int64_t row = begin + threadIdx.x; row < end; row += kSeqThreads) {
    float lp;
    if (row_logp(a, logits, row, lp)) {
      s += static_cast<double>(lp);
      n += 1.0;
    }
    if (a.logp != nullptr) a.logp[row] = lp;
  }
  sum = block_sum(s, red);
  count = block_sum(n, red);
}

__device__ __forceinline__ int64_t bound_at(const SeqArgs& a, int64_t i) {   // cu_rows[i], brought into [0, rows]
  const int64_t v = ld_stream(a.cu + i);
  return v < 0 ? 0 : v > a.rows ? a.rows : v;
}

// Rows outside every sequence: not counted.
__device__ __forceinline__ void clear_rows(const SeqArgs& a, int64_t begin, int64_t end) {
  for (int64_t row = begin + threadIdx.x; row < end; row += kSeqThreads) {
    if (a.logp != nullptr) a.logp[row] = 0.0f;
    if (a.dlogp != nullptr) a.dlogp[row] = 0.0f;
  }
}

__device__ __forceinline__ double log_sigmoid(double d) { return (d < 0.0 ? d : 0.0) - log1p(exp(-fabs(d))); }

template <typename T, bool kPairs>
__global__ void __launch_bounds__(kSeqThreads) sequence_kernel(const SeqArgs a, const T* logits) {
  __shared__ double red[kSeqThreads / 32];
  __shared__ bool s_last;
  pdl_trigger();
  pdl_wait();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kPairs ? 2 : 1);
  const int64_t begin = bound_at(a, first), mid = max(begin, bound_at(a, first + 1));
  double sum, count;
  if (blockIdx.x == 0) clear_rows(a, 0, begin);
  sequence_sum(a, logits, begin, mid, red, sum, count);
  const double per = a.average ? 1.0 / max(count, 1.0) : 1.0;
  if constexpr (!kPairs) {
    if (blockIdx.x == gridDim.x - 1) clear_rows(a, mid, a.rows);
    if (threadIdx.x == 0) a.seq_logp[first] = static_cast<float>(sum * per);
  } else {
    const int64_t end = max(mid, bound_at(a, first + 2));
    double sum2, count2;
    sequence_sum(a, logits, mid, end, red, sum2, count2);
    if (blockIdx.x == gridDim.x - 1) clear_rows(a, end, a.rows);
    const double per2 = a.average ? 1.0 / max(count2, 1.0) : 1.0;
    const double chosen = sum * per, rejected = sum2 * per2;
    const double u = a.ref != nullptr ? (chosen - static_cast<double>(ld_stream(a.ref + first))) -
                                            (rejected - static_cast<double>(ld_stream(a.ref + first + 1)))
                                      : chosen - rejected;
    const double beta = a.beta, d = beta * u - a.margin;
    double l, du;
    if (a.kind == FALQON_PREFERENCE_SIGMOID) {
      const double eps = a.smoothing;      // a term of weight 0 is left out: its logarithm may be infinite
      l = (eps < 1.0 ? -(1.0 - eps) * log_sigmoid(d) : 0.0) - (eps > 0.0 ? eps * log_sigmoid(-d) : 0.0);
      du = beta * (-(1.0 - eps) / (1.0 + exp(d)) + eps / (1.0 + exp(-d)));
    } else if (a.kind == FALQON_PREFERENCE_HINGE) {
      l = d < 1.0 ? 1.0 - d : d >= 1.0 ? 0.0 : d;     // a NaN stays one
      du = d < 1.0 ? -beta : d >= 1.0 ? 0.0 : d;
    } else {
      const double t = u - a.margin - 1.0 / (2.0 * beta);
      l = t * t;
      du = 2.0 * t;
    }
    const double pairs = static_cast<double>(gridDim.x);
    const double nll = static_cast<double>(a.nll_weight) / max(count, 1.0);
    if (nll != 0.0) l -= nll * sum;
    if (threadIdx.x == 0) {
      a.seq_logp[first] = static_cast<float>(chosen);
      a.seq_logp[first + 1] = static_cast<float>(rejected);
      a.pair_loss[blockIdx.x] = static_cast<float>(l);
    }
    if (a.dlogp != nullptr) {
      const float c = static_cast<float>((du * per - nll) / pairs), r = static_cast<float>(-du * per2 / pairs);
      for (int64_t row = begin + threadIdx.x; row < end; row += kSeqThreads) {
        const int64_t target = ld_stream(a.targets + row);
        a.dlogp[row] = target < 0 || target >= a.vocab ? 0.0f : row < mid ? c : r;
      }
    }
    // the CTA that finishes last takes the mean of all pairs' losses, in an order of its own that never changes
    if (threadIdx.x == 0) {
      __threadfence();
      s_last = atomicAdd(a.counter, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (s_last) {
      __threadfence();
      double t = 0.0;
      for (int64_t i = threadIdx.x; i < gridDim.x; i += kSeqThreads) t += static_cast<double>(ld_stream(a.pair_loss + i));
      t = block_sum(t, red);
      if (threadIdx.x == 0) *a.loss = static_cast<float>(t / pairs);
    }
  }
}

// kSame: logits and dlogits rows have the same offset from a 16-byte boundary, so vectors can be stored; else single values are.
template <typename T, bool kSame>
__global__ void __launch_bounds__(kRowThreads) logit_grad_kernel(const T* logits, int64_t vocab, int64_t ld, const int64_t* targets,
                                                                 int parts, const float2* stats, const float* dlogp, const float* dloss,
                                                                 T* out, int64_t ld_out, float* amax) {
  pdl_trigger();
  pdl_wait();
  constexpr int n = Row<T>::kN;
  const int64_t row = blockIdx.x / parts;
  const int part = static_cast<int>(blockIdx.x - row * parts);
  const float c = ld_stream(dlogp + row) * (dloss != nullptr ? ld_stream(dloss) : 1.0f);
  const T* p = logits + row * ld;
  T* o = out + row * ld_out;
  const Span sp = span_of(p, vocab);
  const int64_t begin = sp.body * part / parts, end = sp.body * (part + 1) / parts;
  const uint4* body = reinterpret_cast<const uint4*>(p + sp.head);
  const bool zero = c == 0.0f;
  const float2 st = zero ? make_float2(0.0f, 1.0f) : ld_stream(stats + row);
  const int64_t target = zero ? -1 : ld_stream(targets + row);
  const float f = -c / st.y;
  uint32_t mx = 0;
  const auto one = [&](int64_t i) {
    const float g = zero ? 0.0f : __fmaf_rn(f, exp_of(load1(p + i) - st.x), i == target ? c : 0.0f);
    mx = max(mx, store1(o + i, g));
  };
  constexpr int kUnroll = 4;
  for (int64_t v = begin + threadIdx.x; v < end; v += kRowThreads * kUnroll) {
    uint4 q[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j)
      if (!zero && v + j * kRowThreads < end) q[j] = ld_stream(body + v + j * kRowThreads);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      if (v + j * kRowThreads >= end) break;
      const int64_t at = sp.head + (v + j * kRowThreads) * n;
      float x[n];
      if (zero) {
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = 0.0f;
      } else {
        expand(q[j], x, T{});
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = f * exp_of(x[i] - st.x);
        if (target >= at && target < at + n) {
#pragma unroll
          for (int i = 0; i < n; ++i)
            if (at + i == target) x[i] += c;
        }
      }
      if (kSame) {
        const uint4 w = shrink(x, T{});
        *reinterpret_cast<uint4*>(o + at) = w;
        if (amax != nullptr) {
          float s[n];
          expand(w, s, T{});
#pragma unroll
          for (int i = 0; i < n; ++i) mx = max(mx, abs_bits(s[i]));
        }
      } else {
#pragma unroll
        for (int i = 0; i < n; ++i) mx = max(mx, store1(o + at + i, x[i]));
      }
    }
  }
  if (part == 0) {
    if (static_cast<int>(threadIdx.x) < sp.head) one(threadIdx.x);
    if (threadIdx.x < vocab - sp.tail) one(sp.tail + threadIdx.x);
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

// Into how many parts a row is cut: none where the rows alone fill the GPU, and no part below two vectors per thread.
int parts_for(int64_t rows, int64_t vocab, int dtype) {
  const int64_t want = (148 * 8 + rows - 1) / rows;
  const int64_t most = vocab / (dtype == FALQON_BF16 ? 8 : 4) / (2 * kRowThreads);
  int64_t parts = want < most ? want : most;
  if (parts > kMaxParts) parts = kMaxParts;
  return static_cast<int>(parts < 1 ? 1 : parts);
}

cudaError_t launch_row_stats(const void* logits, int dtype, int64_t rows, int64_t vocab, int64_t ld, const int64_t* targets, int parts,
                             float2* out, unsigned int* counter, int* status, cudaStream_t stream) {
  const dim3 grid(static_cast<unsigned>(rows * parts)), block(kRowThreads);
  return dtype == FALQON_BF16 ? launch_pdl(row_stats_kernel<bf16_t>, grid, block, 0, stream, 1, static_cast<const bf16_t*>(logits), vocab,
                                           ld, targets, parts, out, counter, status)
                              : launch_pdl(row_stats_kernel<float>, grid, block, 0, stream, 1, static_cast<const float*>(logits), vocab,
                                           ld, targets, parts, out, counter, status);
}

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

size_t falqon_preference_scratch_bytes(int64_t rows, int64_t vocab, int dtype) {
  if (!sizes_ok(rows, vocab, dtype)) return 0;
  return kCounterBytes + static_cast<size_t>(rows) * parts_for(rows, vocab, dtype) * sizeof(float2);
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
  a.targets = targets;
  a.cu = cu_rows;
  a.rows = rows;
  a.vocab = vocab;
  a.ld = ld;
  a.seqs = n_seq;
  a.part = part;
  a.parts = parts;
  a.logp = logp;
  a.seq_logp = seq_logp;
  a.average = average != 0;
  const cudaError_t e = launch_row_stats(logits, dtype, rows, vocab, ld, targets, parts, part, static_cast<unsigned int*>(scratch), status, st);
  if (e != cudaSuccess) return FALQON_ERR_CUDA;
  const dim3 grid(static_cast<unsigned>(n_seq)), block(kSeqThreads);
  return finish(dtype == FALQON_BF16
                    ? launch_pdl(sequence_kernel<bf16_t, false>, grid, block, 0, st, 1, a, static_cast<const bf16_t*>(logits))
                    : launch_pdl(sequence_kernel<float, false>, grid, block, 0, st, 1, a, static_cast<const float*>(logits)));
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
  float2* part = parts == 1 && stats != nullptr ? stats : reinterpret_cast<float2*>(static_cast<uint8_t*>(scratch) + kCounterBytes);
  SeqArgs a{};
  a.targets = targets;
  a.cu = cu_rows;
  a.rows = p->rows;
  a.vocab = p->vocab;
  a.ld = p->ld;
  a.seqs = 2 * p->pairs;
  a.part = part;
  a.parts = parts;
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
  const cudaError_t e = launch_row_stats(logits, p->dtype, p->rows, p->vocab, p->ld, targets, parts, part, a.counter, status, st);
  if (e != cudaSuccess) return FALQON_ERR_CUDA;
  const dim3 grid(static_cast<unsigned>(p->pairs)), block(kSeqThreads);
  return finish(p->dtype == FALQON_BF16
                    ? launch_pdl(sequence_kernel<bf16_t, true>, grid, block, 0, st, 1, a, static_cast<const bf16_t*>(logits))
                    : launch_pdl(sequence_kernel<float, true>, grid, block, 0, st, 1, a, static_cast<const float*>(logits)));
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
  const dim3 grid(static_cast<unsigned>(p->rows * parts)), block(kRowThreads);
  const float2* stats = reinterpret_cast<const float2*>(row_stats);
  const auto go = [&](auto kernel, auto* typed) {
    using T = std::remove_pointer_t<decltype(typed)>;
    return finish(launch_pdl(kernel, grid, block, 0, st, 1, static_cast<const T*>(logits), p->vocab, p->ld, targets, parts, stats, dlogp,
                             dloss, typed, ld_out, amax_out));
  };
  const bool same = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits)) & 15) == 0 &&
                    (ld_out - p->ld) % (p->dtype == FALQON_BF16 ? 8 : 4) == 0;
  if (p->dtype == FALQON_BF16) {
    bf16_t* t = static_cast<bf16_t*>(dlogits);
    return same ? go(logit_grad_kernel<bf16_t, true>, t) : go(logit_grad_kernel<bf16_t, false>, t);
  }
  float* t = static_cast<float*>(dlogits);
  return same ? go(logit_grad_kernel<float, true>, t) : go(logit_grad_kernel<float, false>, t);
}

}  // extern "C"
