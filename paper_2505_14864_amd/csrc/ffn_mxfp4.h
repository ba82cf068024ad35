// What the kernels of the grouped FFN on MXFP4 weights share (ffn_mxfp4.hip: output tiles, ffn_mxfp4_few.hip: the down product of few rows): a product's
// parameters, the matrix instruction and the stores of its results.
#pragma once

#include "ffn_gemm.h"
#include "mxfp4.h"
#include "tile_list.h"

namespace dynmo {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));

struct MxProduct {
  const int32_t* seg;
  int E;
  int N;            // columns of the result: F for gate/up, H for down
  int K;
  const char* X;    // the rows: codes, in row blocks of one expert each
  const char* Xs;   // and their scales
  const char* W1;   // gate, or down
  const char* W2;   // up
  size_t w_bytes;   // of one expert's matrix
  char* A;          // gate/up: the quantised result (K of the down product = N)
  char* As;
  bf16_t* C0;       // down: Y; gate/up: G to save, or nullptr
  bf16_t* C1;       // U to save, or nullptr
  TileList list;
};

// Operand A (16 x 128 4-bit values) is the weights and operand B the rows, so that a lane of the result holds four consecutive columns, 4 (lane /
// 16) .. + 3, of row lane % 16.  J: which byte of the scale words.
template <int J>
__device__ __forceinline__ f32x4_t mx_mfma(v4i a, v4i b, f32x4_t c, int sa, int sb) {
  const v8i a8 = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, b8 = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, J, sa, J, sb);
}

__device__ __forceinline__ uint2 pack_bf16x4(f32x4_t v) { return {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }

// 32 columns from n on, a block of the down product's k, of row block rb: silu(G) U quantised and stored.  The block lies in two results (16 columns each) and four lanes, so its largest value takes two lane exchanges.
// The logistic function uses the hardware's reciprocal (1 ulp): what follows is a grid of eight steps.
__device__ __forceinline__ void mx_store_swiglu(const MxProduct& p, const f32x4_t (&g)[2], const f32x4_t (&u)[2], int rb, int n) {
  const int lane = threadIdx.x & 63, quad = lane >> 4, row = lane & 15;
  const int Fb = mx_k_blocks(p.N), Fq = mx_k_quads(p.N);
  if (n >= Fb * 128) return;
  float h[2][4];
  uint32_t amax = 0;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      h[c][r] = silu_mul(g[c][r], u[c][r]);
      amax = max(amax, __float_as_uint(h[c][r]) & 0x7fffffffu);
    }
  }
  // a swap of two copies leaves both quads of a pair, and both pairs, in every lane
  auto r = __builtin_amdgcn_permlane16_swap(amax, amax, false, false);
  amax = max(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(amax, amax, false, false);
  amax = max(r[0], r[1]);
  const uint32_t byte = mx_scale_of(amax);
  const float scale = mx_scale_value(byte);
  uint32_t code = 0;  // four codes of each half
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, h[0][0], h[0][1], scale, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, h[0][2], h[0][3], scale, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, h[1][0], h[1][1], scale, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, h[1][2], h[1][3], scale, 3);
  code = byte == 255 ? 0u : code;
  // a pair of quads has eight codes of each half: its first quad stores those of the first half, its second those of the other
  r = __builtin_amdgcn_permlane16_swap(code, code, false, false);
  const uint32_t word = quad & 1 ? r[0] >> 16 | (r[1] & 0xffff0000u) : (r[0] & 0xffffu) | r[1] << 16;
  *(uint32_t*)(p.A + ((size_t)rb * Fb + n / 128) * kMxTile + n % 128 / 32 * 256 + row * 16 + (quad & 1) * 8 + (quad >> 1) * 4) = word;
  if (quad == 0) p.As[((size_t)rb * Fq + n / 512) * kMxScales + (n % 128 / 32 * 16 + row) * 4 + n % 512 / 128] = (char)byte;
}

// NB results side by side (get(0) .. get(NB - 1), 16 columns each from col0 on) of the sixteen rows from m on, as bfloat16.  They pass through
// the wavefront's own LDS `patch`, so that a store covers 16 NB columns of a row: from the lanes that have them, 32 bytes of a row each, the stores
// of 32768 x 4096 results of a sum over 688 took three times what the memory needs (kPatch bytes, 16-byte aligned).
template <int NB>
constexpr int kPatch = 16 * (NB * 32 + 16);
template <int NB, typename Get>
__device__ __forceinline__ void mx_store_rows(char* patch, bf16_t* C, int N, int m, int m_end, int col0, Get&& get) {
  constexpr int kPitch = NB * 32 + 16, kLanes = NB * 2, kRows = 64 / kLanes;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int a = 0; a < NB; ++a) *(uint2*)(patch + (lane & 15) * kPitch + a * 32 + (lane >> 4) * 8) = pack_bf16x4(get(a));
  wave_lds_order();
#pragma unroll
  for (int r0 = 0; r0 < 16; r0 += kRows) {
    const int r = r0 + lane / kLanes, col = col0 + lane % kLanes * 8;
    if (m + r < m_end && col < N) *(u32x4*)(C + (size_t)(m + r) * N + col) = *(const u32x4*)(patch + r * kPitch + lane % kLanes * 16);
  }
  wave_lds_order();
}

// Which expert's row block (of 16) or row tile: lane e counts those of expert e, `upto` of the experts up to and with e.  Six additions of
// neighbouring lanes: the shifts within a row of sixteen, then the rows' last lanes to the rows behind them.
__device__ __forceinline__ int experts_upto(int count) {
  count += __builtin_amdgcn_update_dpp(0, count, 0x111, 0xf, 0xf, true);  // row_shr:1, :2, :4, :8
  count += __builtin_amdgcn_update_dpp(0, count, 0x112, 0xf, 0xf, true);
  count += __builtin_amdgcn_update_dpp(0, count, 0x114, 0xf, 0xf, true);
  count += __builtin_amdgcn_update_dpp(0, count, 0x118, 0xf, 0xf, true);
  count += __builtin_amdgcn_update_dpp(0, count, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  count += __builtin_amdgcn_update_dpp(0, count, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return count;
}

// ffn_mxfp4_few.hip: the down product; at most `max_experts` experts have rows, which are few (right for any number)
int32_t mx_few_rows(const MxProduct& p, int max_experts, KernelId id, hipStream_t st);

}  // namespace dynmo
