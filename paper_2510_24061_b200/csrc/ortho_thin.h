// Host side of ortho_thin.cu: matrices with a short side of at most 128, orthogonalised from their Gram matrix in fp64 (not part of
// the public ABI).
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

namespace falqon {

constexpr int64_t kThinMost = 128;          // short side
constexpr int kThinMostSteps = 32;

struct ThinPlan {
  int64_t batch, rows, cols;
  bool in_bf16, out_bf16;
  int steps;
  float eps, scale;
  float abc[3 * kThinMostSteps];
};

// Whether matrices of this shape, with results of this type and these steps, are taken.
bool ortho_thin_takes(int64_t rows, int64_t cols, bool out_bf16, const float* abc, int steps);
size_t ortho_thin_scratch_bytes(int64_t batch, int64_t rows, int64_t cols);
cudaError_t launch_ortho_thin(const ThinPlan& p, const void* g, void* out, void* scratch, cudaStream_t st);

}  // namespace falqon
