// The 4-bit products and the quantisation behind them, for the entry points built from both.
#pragma once
#include <cuda_runtime.h>

#include "refadapt.h"

namespace ra {

// Columns that share a scale.
constexpr int block_of(int format) { return format == RA_Q4_E8M0 ? 32 : 16; }

namespace gemm4 {
ra_status run(const char* who, const ra_gemm4_args& a, cudaStream_t st);
}  // namespace gemm4

}  // namespace ra
