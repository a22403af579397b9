// Host side of block_linear.cu: products of few tokens with a layer held in 8 bits by blocks (not part of the public ABI).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace falqon {

constexpr int64_t kMostFew = 32;        // tokens that the kernel for few rows takes
constexpr int64_t kMostPlain = 4;       // tokens that it quantizes itself

// Whether T tokens of n values may come unquantized (their codes fit in shared memory).
bool block_linear_plain(int64_t T, int64_t n);
// T <= kMostFew; n, m multiples of 16.
cudaError_t launch_block_linear_codes(const uint8_t* x, const uint8_t* xs, int x_fmt, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T,
                                      int64_t n, int64_t m, void* y, bool bf16, cudaStream_t st);
// block_linear_plain(T, n)
cudaError_t launch_block_linear_plain(const void* x, bool x_bf16, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T, int64_t n, int64_t m,
                                      void* y, bool bf16, cudaStream_t st);

}  // namespace falqon
