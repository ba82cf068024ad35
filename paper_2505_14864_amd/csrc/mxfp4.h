// Microscaled 4-bit floating point (MXFP4): blocks of 32 values along a row, E2M1 codes and one power-of-two scale (E8M0) per block.
//
// Packed form of a matrix [rows, K]: tiles of 16 rows x 128 values, 1 KB each, then the scales.
//   code of (r, k):  byte ((r / 16) * Kb + k / 128) * 1024 + (k % 128) / 32 * 256 + r % 16 * 16 + k % 32 / 2, even k in the low half
//   scale of the block: byte Rb * Kb * 1024 + ((r / 16) * Kq + k / 512) * 256 + (k % 128) / 32 * 64 + r % 16 * 4 + k % 512 / 128
// with Rb = ceil(rows / 16), Kb = ceil(K / 128), Kq = ceil(K / 512); what lies behind the matrix's edges is zero.
// A tile is an operand of v_mfma_scale_f32_16x16x128_f8f6f4 lane by lane: lane l takes its 16 bytes l (row l % 16, block l / 16), and
// its 32-bit word l of the scales holds that block's scales of four consecutive tiles, from which the instruction picks a byte.  So a
// tile is one contiguous kilobyte for a wavefront's load, whether into registers or into LDS, and is read from LDS without conflicts.
#pragma once

#include "common.h"

namespace dynmo {

constexpr int kMxTile = 1024, kMxScales = 256;  // bytes of a tile, and of the scales of four

inline __host__ __device__ int mx_row_blocks(int rows) { return (rows + 15) / 16; }
inline __host__ __device__ int mx_k_blocks(int K) { return (K + 127) / 128; }
inline __host__ __device__ int mx_k_quads(int K) { return (K + 511) / 512; }
inline __host__ __device__ size_t mx_code_bytes(int row_blocks, int K) { return (size_t)row_blocks * mx_k_blocks(K) * kMxTile; }
inline __host__ __device__ size_t mx_scale_bytes(int row_blocks, int K) { return (size_t)row_blocks * mx_k_quads(K) * kMxScales; }
inline __host__ __device__ size_t mx_bytes(int rows, int K) {
  return mx_code_bytes(mx_row_blocks(rows), K) + mx_scale_bytes(mx_row_blocks(rows), K);
}

// A block's scale from the bits of its largest magnitude: 2^(floor(log2(amax)) - 2), so that the largest value lands in [4, 8) and
// what is over 6 saturates; as a byte exponent + 127, at least 0, and 255 (not a number) for a block with an infinity or a NaN.
__device__ __forceinline__ uint32_t mx_scale_of(uint32_t amax_bits) {
  const uint32_t field = amax_bits >> 23;
  return field == 255 ? 255u : field < 2 ? 0u : field - 2;
}
// 2^(byte - 127); 0 is the subnormal 2^-127
__device__ __forceinline__ float mx_scale_value(uint32_t byte) { return __uint_as_float(byte == 0 ? 0x00400000u : byte << 23); }

// mxfp4.hip.  Quantises the rows of the expert segments for the grouped products: row block b of the result holds sixteen rows of one
// expert (an expert's last block fewer), the experts' blocks one after another; `gather`: row p is x[gather[p] / gather_div], or nullptr.
int32_t mx_quantize_segments(const dynmo_desc* d, const void* x, const int32_t* gather, const int32_t* seg, int K, void* codes, void* scales,
                             hipStream_t st);
// The reverse, for rows that are read next: row p of `dst` [T*k, K] becomes the values that its codes stand for; rows behind the last segment are
// left as they are.
int32_t mx_dequantize_segments(const dynmo_desc* d, const void* codes, const void* scales, const int32_t* seg, int K, bf16_t* dst, hipStream_t st);

constexpr int64_t kMaxBlocks = 1 << 24;  // workgroups of 256 threads: a launch has fewer than 2^32
// The most row blocks that the segments can have; the callers of the two above refuse kMaxBlocks and more
inline int64_t mx_max_row_blocks(const dynmo_desc* d) {
  const int64_t rows = (int64_t)d->T * d->k;
  return rows / 16 + (rows < d->E ? rows : d->E);
}

}  // namespace dynmo
