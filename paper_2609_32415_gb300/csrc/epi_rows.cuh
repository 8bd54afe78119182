// Rows of a GEMM epilogue between global memory and a warp's registers: a thread
// has a row (its TMEM lane) of 32 columns, global accesses take 64 contiguous
// bytes of eight rows per instruction, and a 2 KB staging buffer per warp turns
// one into the other. ncol: columns of the 32 that exist (a multiple of 8).
#pragma once
#include <cstdint>

#include "tc_ptx.cuh"

namespace ra {

// The 64-byte row slots of a warp's staging buffer: 16-byte piece q of row r.
// The permutation keeps both access patterns free of bank conflicts (every
// lane its own row; eight rows, four lanes a row).
__device__ __forceinline__ uint4* stage_slot(uint8_t* stage, int r, int q) {
  return reinterpret_cast<uint4*>(stage + r * 64 + ((q ^ ((r >> 1) & 3)) << 4));
}
// Four 16-byte loads per lane of up to 32 rows of 64 bytes at `src` (row
// stride in bytes): load i is piece lane % 4 of row 8 i + lane / 4.
__device__ __forceinline__ void rows_fetch(const char* src, int64_t stride, int nrow, uint4 (&v)[4], int ncol = 32) {
  const int lane = threadIdx.x & 31, r0 = lane >> 2;
  const char* ptr = src + r0 * stride + (lane & 3) * 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = (r0 + 8 * i < nrow && 8 * (lane & 3) < ncol) ? *reinterpret_cast<const uint4*>(ptr + 8 * i * stride)
                                                         : make_uint4(0, 0, 0, 0);
}
// rows_fetch's registers -> the lane's own row (64 bytes), through the staging buffer.
__device__ __forceinline__ void rows_turn(uint8_t* stage, const uint4 (&v)[4], uint4 (&own)[4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 4; ++i) *stage_slot(stage, 8 * i + (lane >> 2), lane & 3) = v[i];
  __syncwarp();
#pragma unroll
  for (int q = 0; q < 4; ++q) own[q] = *stage_slot(stage, lane, q);
  __syncwarp();
}
// Every lane's row of 32 bf16 -> up to 32 rows of 64 bytes at `dst`.
__device__ __forceinline__ void rows_put(uint8_t* stage, const uint4 (&own)[4], char* dst, int64_t stride, int nrow,
                                         int ncol = 32) {
  const int lane = threadIdx.x & 31, r0 = lane >> 2;
#pragma unroll
  for (int q = 0; q < 4; ++q) *stage_slot(stage, lane, q) = own[q];
  __syncwarp();
  char* ptr = dst + r0 * stride + (lane & 3) * 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = *stage_slot(stage, r0 + 8 * i, lane & 3);
    if (r0 + 8 * i < nrow && 8 * (lane & 3) < ncol) *reinterpret_cast<uint4*>(ptr + 8 * i * stride) = v;
  }
  __syncwarp();
}
// 32 fp32 of every lane's row -> bf16 -> up to 32 rows of 64 bytes at `dst`.
__device__ __forceinline__ void rows_store(uint8_t* stage, const float (&x)[32], char* dst, int64_t stride, int nrow,
                                           int ncol = 32) {
  uint4 own[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    own[q] = make_uint4(pack_bf16x2(x[8 * q], x[8 * q + 1]), pack_bf16x2(x[8 * q + 2], x[8 * q + 3]),
                        pack_bf16x2(x[8 * q + 4], x[8 * q + 5]), pack_bf16x2(x[8 * q + 6], x[8 * q + 7]));
  rows_put(stage, own, dst, stride, nrow, ncol);
}

// The same for rows of 64 columns (128 bytes): whole lines of four rows per
// instruction, a staging buffer of 4 KB; ncol of the 64 columns exist.
__device__ __forceinline__ void rows_put128(uint8_t* stage, const uint4 (&own)[8], char* dst, int64_t stride, int nrow,
                                            int ncol) {
  const int lane = threadIdx.x & 31, r0 = lane >> 3;
  auto slot = [&](int r, int q) { return reinterpret_cast<uint4*>(stage + r * 128 + ((q ^ (r & 7)) << 4)); };
#pragma unroll
  for (int q = 0; q < 8; ++q) *slot(lane, q) = own[q];
  __syncwarp();
  char* ptr = dst + r0 * stride + (lane & 7) * 16;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 v = *slot(r0 + 4 * i, lane & 7);
    if (r0 + 4 * i < nrow && 8 * (lane & 7) < ncol) *reinterpret_cast<uint4*>(ptr + 4 * i * stride) = v;
  }
  __syncwarp();
}

}  // namespace ra
