// Grouped SwiGLU FFN on MXFP4 weights: the down product of few rows per expert, whose output tiles are too few to read the weights at the
// rate of the memory.
//
// Bound: reading the weights once.  They do not pass through LDS: a wavefront loads the tiles of 16 weight rows x 128 values from global memory
// straight into the operands of the matrix instructions, a contiguous kilobyte each, some steps ahead, and needs no barrier inside its k loop.  A
// workgroup takes 32 weight rows of one expert; its four wavefronts take the tiles of a row block in turn, so that together they
// stream it from end to end, and add their fp32 sums in LDS, in a fixed order: k is long, and is split over wavefronts instead of
// workgroups, without a second pass.
//
// Measured, us, against tiles of 128 x 128: 4096 x 14336, one row on each of two experts 40 -> 14 (4.5 TB/s), 64 rows over eight 49 -> 44 (5.7 TB/s);
// 1024 x 4096, 16 rows 9.7 -> 5.4.  16 weight rows per workgroup 15 / 52 / 5.8, 64 19 / 47 / 6.2, eight wavefronts 15 / 53 / 6.0.  Gate/up has
// twice the weights and a short k, tiles enough for the 128 x 128 kernel to read them at 5.3 to 6 TB/s (one row 24 us against 29, eight experts
// 84 against 82), and the same kernel with the rows quantised on the way in was slower than with a launch for that (one row 42 against 24 + 5).
#include "ffn_mxfp4.h"

namespace dynmo {

constexpr int kFewWaves = 4, kFewBlocks = 2;  // wavefronts, and blocks of 16 weight rows

__global__ __launch_bounds__(64 * kFewWaves, 2) void ffn_mx_few_kernel(const MxProduct p) {
  __shared__ f32x4_t part[kFewWaves][kFewBlocks][64];
  const int n0 = blockIdx.x * 16 * kFewBlocks, nb0 = n0 / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // grid y counts the experts that have rows, so that the workgroups with work are the first ones
  const int lane_begin = p.seg[min(lane, p.E)], lane_end = p.seg[min(lane + 1, p.E)];
  const int blocks = mx_row_blocks(lane_end - lane_begin), blocks_upto = experts_upto(blocks);
  const unsigned long long used = __ballot(blocks > 0);
  const unsigned long long mine = __ballot(blocks > 0 && __popcll(used & ((1ull << lane) - 1ull)) == (int)blockIdx.y);
  if (mine == 0) return;
  const int e = __builtin_ctzll(mine);
  const int begin = __builtin_amdgcn_readlane(lane_begin, e), end = __builtin_amdgcn_readlane(lane_end, e);
  const int rb_first = __builtin_amdgcn_readlane(blocks_upto, e) - __builtin_amdgcn_readlane(blocks, e);

  const int Kb = mx_k_blocks(p.K), Kq = mx_k_quads(p.K), Wb = mx_row_blocks(p.N);
  // a row block of an operand is a scalar offset further on, which the bounds check does not see
  auto rsrc = [](const char* q) { return __builtin_amdgcn_make_buffer_rsrc((void*)q, 0, 0x7ffffffe, 0x00020000); };
  const char* const w_codes = p.W1 + e * p.w_bytes + (size_t)nb0 * Kb * kMxTile;
  const char* const w_scales = p.W1 + e * p.w_bytes + (size_t)Wb * Kb * kMxTile + (size_t)nb0 * Kq * kMxScales;
  // a wavefront's tiles are wave, wave + 4, ..: byte `wave` of the scale words, which is moved to the bottom
  static_assert(kFewWaves == 4, "scale words hold four tiles");
  const int steps = (Kb + kFewWaves - 1) / kFewWaves, byte_at = 8 * wave;
  // Workgroups start at different places of the k range (and go round): started together at k = 0, with weight rows
  // a power of two apart, they would all ask the same few memory channels.
  const int first_step = (blockIdx.x + blockIdx.y) % steps;

  auto pass = [&](int row0, auto RB_C) {
    constexpr int RB = decltype(RB_C)::value;
    constexpr int D = RB <= 2 ? 4 : 3;  // steps in registers
    const int rb0 = rb_first + row0 / 16, t_blocks = (end - begin - row0 + 15) / 16;
    const char* const x_codes = p.X + (size_t)rb0 * Kb * kMxTile;
    const char* const x_scales = p.Xs + (size_t)rb0 * Kq * kMxScales;
    v4i w[D][kFewBlocks], x[D][RB];
    int sw[D][kFewBlocks], sx[D][RB];
    auto load = [&](int d, int step) {
      const int turn = step + first_step;
      const int t = (step >= steps ? steps : turn < steps ? turn : turn - steps) * kFewWaves + wave;  // past the last step: beyond K
      auto get = [&](const char* codes, const char* scales, int r, bool ok, v4i* c, int* s) {
        ok = ok && t < Kb;
        *c = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rsrc(codes), ok ? lane * 16 : kOob, (r * Kb + t) * kMxTile, 0));
        *s = __builtin_amdgcn_raw_buffer_load_b32(rsrc(scales), ok ? lane * 4 : kOob, (r * Kq + t / 4) * kMxScales, 0);
      };
#pragma unroll
      for (int j = 0; j < kFewBlocks; ++j) get(w_codes, w_scales, j, nb0 + j < Wb, &w[d][j], &sw[d][j]);
#pragma unroll
      for (int i = 0; i < RB; ++i) get(x_codes, x_scales, i, i < t_blocks, &x[d][i], &sx[d][i]);
      __builtin_amdgcn_sched_barrier(0);
    };
    f32x4_t acc[RB][kFewBlocks] = {};
#pragma unroll
    for (int d = 0; d + 1 < D; ++d) load(d, d);
    for (int step = 0; step < steps; step += D) {
#pragma unroll
      for (int d = 0; d < D; ++d) {
        load((d + D - 1) % D, step + d + D - 1);
#pragma unroll
        for (int j = 0; j < kFewBlocks; ++j)
#pragma unroll
          for (int i = 0; i < RB; ++i)
            acc[i][j] = mx_mfma<0>(w[d][j], x[d][i], acc[i][j], (uint32_t)sw[d][j] >> byte_at, (uint32_t)sx[d][i] >> byte_at);
      }
    }
    // ---- the wavefronts' sums, added in their order; a wavefront stores a column block
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kFewBlocks; ++j) part[wave][j][lane] = acc[i][j];
      __syncthreads();
      if (wave >= kFewBlocks) continue;
      f32x4_t v = part[0][wave][lane];
#pragma unroll
      for (int k = 1; k < kFewWaves; ++k) v += part[k][wave][lane];
      const int m = begin + row0 + i * 16 + (lane & 15), col = n0 + wave * 16 + (lane >> 4) * 4;
      if (m < end && col < p.N) *(uint2*)(p.C0 + (size_t)m * p.N + col) = pack_bf16x4(v);
    }
  };
  for (int row0 = 0; row0 < end - begin; row0 += 64) {
    const int left = end - begin - row0;
    if (left <= 16) pass(row0, std::integral_constant<int, 1>{});
    else if (left <= 32) pass(row0, std::integral_constant<int, 2>{});
    else pass(row0, std::integral_constant<int, 4>{});
  }
}

int32_t mx_few_rows(const MxProduct& p, int max_experts, KernelId id, hipStream_t st) {
  const dim3 grid((p.N + 16 * kFewBlocks - 1) / (16 * kFewBlocks), max_experts);
  DYNMO_TIMED_LAUNCH(id, st, ffn_mx_few_kernel<<<grid, dim3(64 * kFewWaves), 0, st>>>(p));
  return DYNMO_OK;
}

}  // namespace dynmo
