// Host side of block_linear.cu: products of few tokens with a layer held in 8 bits by blocks (not part of the public ABI).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace falqon {

constexpr int64_t kMostFew = 4;

// Whether the kernel takes T tokens of n values for m results: one or two, and up to kMostFew where w has at most 2^25 weights, if their
// codes fit in shared memory.
bool block_linear_takes(int64_t T, int64_t n, int64_t m);
// block_linear_takes(T, n, m); n, m multiples of 16; x as codes, or plain (quantized on the way).
cudaError_t launch_block_linear_codes(const uint8_t* x, const uint8_t* xs, int x_fmt, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T,
                                      int64_t n, int64_t m, void* y, bool bf16, cudaStream_t st);
cudaError_t launch_block_linear_plain(const void* x, bool x_bf16, const uint8_t* w, const uint8_t* ws, int w_fmt, int64_t T, int64_t n, int64_t m,
                                      void* y, bool bf16, cudaStream_t st);

}  // namespace falqon
