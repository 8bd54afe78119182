// The 4-bit products and the quantisation behind them, for the entry points built from both.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "refadapt.h"

namespace ra {

// Columns that share a scale.
constexpr int block_of(int format) { return format == RA_Q4_E8M0 ? 32 : 16; }

namespace gemm4 {
// GELU of x below this is taken as at it, 1e-17 or less from zero (NaN stays NaN): the tanh form has infinity times
// zero at minus infinity.
constexpr float GELU_END = -7.5f;
// Calls of one row a segment have a kernel of their own (gemm4_row.cu) where it is the faster one: as long
// as one tile of 64 columns to an SM covers the weights' rows; K up to MAX_ROW_K. The arguments are checked.
constexpr int MAX_ROW_K = 32768;
ra_status run_row(const char* who, const ra_gemm4_args& a, cudaStream_t st);
// The checks, and the launch. `who` names the entry point in errors. made: the weights' codes come from the launch
// before (asking for them early is no use then). `then`: a second product of one segment in the launch (B = 1,
// STORE, same format, K no longer than a's); outputs and inputs of both are checked together.
ra_status run(const char* who, const ra_gemm4_args& a, cudaStream_t st, bool made, const ra_gemm4_args* then = nullptr);
ra_status run_two(const char* who, const ra_gemm4_args& a, const ra_gemm4_args& b, cudaStream_t st, bool made);
}  // namespace gemm4

}  // namespace ra
