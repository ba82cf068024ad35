// Grouped SwiGLU FFN, forward, on MXFP4 weights (mxfp4.h): the rows are quantised block by block, and both products run on the scaled
// matrix instructions (v_mfma_scale_f32_16x16x128_f8f6f4, 4-bit operands, fp32 accumulation).
//
//   G = Q(X) Wg^T, U = Q(X) Wu^T, A = Q(silu(G) U), Y = A Wd^T
//
// G, U and A are fp32 values up to A's quantisation: rounding them to bf16 in between would move values over the borders of a
// four-bit grid that has eight steps.  Saved G and U, and Y, are rounded to bf16 once.
//
// One workgroup of four wavefronts (2 x 2) per output tile of 128 or 256 weight rows x 128 rows; the hardware deals them, and three (two) of them share a
// compute unit, so that one's prologue, waits and epilogue run under the others' matrix instructions.  k goes in steps of 128 through a ring of three
// LDS stages: a step's tiles of 1 KB are loaded into LDS as they lie in memory and read from there without bank conflicts (counted: none); the
// scales of four steps come with every fourth.  A load has a descriptor that stays and a scalar offset that moves: with addresses worked
// out per load the scalar instructions took 15 % (gate/up of 8192 rows 686 -> 600 us).
//
// Bound, 8192 rows over 8 experts, 4096 x 14336: gate/up 3.6 PFLOP/s (534 us), down 3.4 (282), of 6.5 to 7 that the instruction alone reaches on random
// operands from registers.  Counted: the matrix pipes are busy 50 % (down 46 %) of 0.92 M (0.50 M) cycles, at 1.9 GHz.  So a step of a 256 x 128 tile
// takes some 965 (1050) clocks of a compute unit, its share of the epilogue included, where its matrix instructions need 512 and its LDS traffic, 4 x
// 12 KB read and 24 KB written at 128 bytes a clock, 576: neither is full, LDS is the fuller one, and the rest is where the two do not overlap.  For a
// 128 x 128 tile it is 256 against 384.  The clock is lowered by the chip's power: on operands of zeros the same launches took 443 and 233 us
// when they took 590 and 291.  447 and 202 us without the loads, 355 and 234 without the matrix instructions and the reads.
// Measured and no faster: tiles of 256 x 256 by eight wavefronts (603, 324) or by four of 128 x 128 (667, 330), 128 x 256 (595, 293), the next step's
// operands read from LDS during the present one (609, 304), row tiles walked in chunks of 8, 12 or 16.  Two stages instead of three: down of 256
// rows 51 -> 83 us; four: a workgroup less per compute unit, gate/up of 64 ragged experts 67 -> 75, of 2000 rows 165 -> 215.
// Few rows: bound by reading the weights once (64 rows over 8 experts, gate/up 84 us, 6 TB/s).
#include "ffn_mxfp4.h"

namespace dynmo {

typedef __attribute__((address_space(3))) v4i lds_v4i;
typedef __attribute__((address_space(3))) int lds_int;

// load_to_lds() of ffn_gemm.h with a scalar offset, which the bounds check does not see
template <int LDS_CONST>
__device__ __forceinline__ void load_to_lds_at(desc_t d, uint32_t lds_base, uint32_t lane_offset, uint32_t offset) {
  asm volatile("s_add_i32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds_base), "v"(lane_offset), "s"(d), "s"(offset), "n"(LDS_CONST)
               : "memory", "scc");
}

// BW x BT blocks of 16 x 16 per wavefront, WW x WT wavefronts
template <int BW_, int BT_, int WW_, int WT_>
struct MxShape {
  static constexpr int BW = BW_, BT = BT_, WW = WW_, WT = WT_;
  static constexpr int kWaves = WW * WT, kThreads = 64 * kWaves;
  static constexpr int kWBlocks = BW * WW, kTBlocks = BT * WT, kBlocks = kWBlocks + kTBlocks;  // of the tile
  static constexpr int kStages = 3, kAhead = kStages - 1;
  static constexpr int kLoads = kBlocks / kWaves;                                // tiles that a wavefront loads per step
  static constexpr int kScaleLoads = (kBlocks / 4 + kWaves - 1) / kWaves;  // loads of the scales of four steps, 1 KB each
  static constexpr int kStage = kBlocks * kMxTile, kScaleAt = kStages * kStage, kLds = kScaleAt + kScaleLoads * kWaves * 1024;
  static_assert(kBlocks % kWaves == 0 && kWBlocks % 8 == 0 && kTBlocks % 4 == 0, "the scales of four blocks are loaded together");
  static_assert(kAhead <= 3, "one buffer for the scales: those of the next four steps are loaded after the present ones have been read");
};

template <bool GATEUP, class S>
__global__ __launch_bounds__(S::kThreads, 2) void ffn_mx_kernel(const MxProduct p) {
  constexpr int BW = S::BW, BT = S::BT, WW = S::WW, WT = S::WT;
  __shared__ __attribute__((aligned(1024))) char smem[S::kLds];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ww = wave / WT, wt = wave % WT;
  constexpr int TN = S::kWBlocks * 16 / (GATEUP ? 2 : 1), TM = S::kTBlocks * 16;

  // ---- which tile: lane e of every wavefront counts the row tiles and the row blocks of expert e
  const int nt = GATEUP ? (mx_k_blocks(p.N) * 128 + TN - 1) / TN : (p.N + TN - 1) / TN;  // gate/up writes whole tiles of the next k
  const int begin = lane < p.E ? p.seg[lane] : 0, end = lane < p.E ? p.seg[lane + 1] : 0;
  const int mt = (end - begin + TM - 1) / TM, blocks = mx_row_blocks(end - begin);
  const int upto = experts_upto(mt), blocks_upto = experts_upto(blocks);
  const int total = __builtin_amdgcn_readlane(upto, 63) * nt;
  const int pos = list_position(p.list, blockIdx.x, total, TM, S::kWBlocks * 16, p.E, __ballot(mt > 1) == 0);
  const unsigned long long owners = __ballot(upto * nt > pos);
  if (owners == 0) return;  // past the last tile
  const int e = __builtin_ctzll(owners);
  const int mt_e = __builtin_amdgcn_readlane(mt, e);
  int mi, ni;
  tile_of(pos - (__builtin_amdgcn_readlane(upto, e) - mt_e) * nt, mt_e, nt, &mi, &ni);
  const int m0 = __builtin_amdgcn_readlane(begin, e) + mi * TM, m_end = __builtin_amdgcn_readlane(end, e);
  const int n0 = ni * TN;
  const int rb0 = __builtin_amdgcn_readlane(blocks_upto, e) - __builtin_amdgcn_readlane(blocks, e) + mi * S::kTBlocks;
  const int t_blocks = min(S::kTBlocks, (m_end - m0 + 15) / 16);

  // ---- operands: block b of a step is weight block b (gate/up: the first half gate, the second half the matching up rows) or row block
  // b - kWBlocks.  A wavefront's loads have a descriptor each, which stays; what changes from step to step is the scalar offset.
  const int Kb = mx_k_blocks(p.K), Kq = mx_k_quads(p.K), Wb = mx_row_blocks(p.N);
  const char* const w1 = p.W1 + e * p.w_bytes;
  const char* const w2 = GATEUP ? p.W2 + e * p.w_bytes : w1;
  const size_t scales_at = (size_t)Wb * Kb * kMxTile;
  constexpr int kHalf = GATEUP ? S::kWBlocks / 2 : S::kWBlocks;
  const int nb0 = n0 / 16;
  const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
  desc_t from[S::kLoads], scales_from[S::kScaleLoads];
  uint32_t scales_off[S::kScaleLoads];
  static_for<S::kLoads>([&](auto J) {
    constexpr int j = decltype(J)::value;
    const int b = wave * S::kLoads + j, t = b - S::kWBlocks, r = GATEUP && b >= kHalf ? b - kHalf : b;
    const char* w = (GATEUP && b >= kHalf ? w2 : w1) + (size_t)(nb0 + r) * Kb * kMxTile;
    const char* x = p.X + (size_t)(rb0 + t) * Kb * kMxTile;
    from[j] = make_desc((const bf16_t*)(t >= 0 ? x : w), (t >= 0 ? t < t_blocks : nb0 + r < Wb) ? 0x7ffffffeu : 0u);
  });
  static_for<S::kScaleLoads>([&](auto J) {
    constexpr int j = decltype(J)::value;
    const int b = (wave * S::kScaleLoads + j) * 4, t = b - S::kWBlocks, r = GATEUP && b >= kHalf ? b - kHalf : b;  // four blocks of one matrix
    const char* w = (GATEUP && b >= kHalf ? w2 : w1) + scales_at + (size_t)(nb0 + r) * Kq * kMxScales;
    const char* x = p.Xs + (size_t)(rb0 + t) * Kq * kMxScales;
    scales_from[j] = make_desc((const bf16_t*)(t >= 0 ? x : w), 0x7ffffffeu);
    const int q = lane >> 4;
    scales_off[j] = (t >= 0 ? t + q < t_blocks : nb0 + r + q < Wb) ? (uint32_t)q * (uint32_t)Kq * kMxScales + (lane & 15) * 16 : kOob;
  });
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + wave * S::kLoads * kMxTile);
  const uint32_t scales_to = __builtin_amdgcn_readfirstlane(lds0 + S::kScaleAt + wave * S::kScaleLoads * 1024);
  auto issue = [&](int step, uint32_t stage, auto SCALES) {  // past the last step the loads fetch nothing
    const uint32_t off = step < Kb ? lane * 16 : kOob;
    static_for<S::kLoads>([&](auto J) {
      constexpr int j = decltype(J)::value;
      load_to_lds_at<j * kMxTile>(from[j], to + stage, off, (uint32_t)step * kMxTile);
    });
    if constexpr (decltype(SCALES)::value) {
      static_for<S::kScaleLoads>([&](auto J) {
        constexpr int j = decltype(J)::value;
        load_to_lds_at<j * 1024>(scales_from[j], scales_to, step < Kb ? scales_off[j] : kOob, (uint32_t)(step / 4) * kMxScales);
      });
    }
  };

  const int my_blocks = max(0, min(BT, (t_blocks - wt + WT - 1) / WT));  // row blocks wt, wt + WT, .. of the tile
  // the first of this wavefront's weight blocks (gate/up: gate blocks, then the up blocks kHalf further on), and of its row blocks
  const int w_first = GATEUP ? ww * (BW / 2) : ww * BW, t_first = S::kWBlocks + wt;
  constexpr auto w_place = [](int i) { return GATEUP && i >= BW / 2 ? kHalf + i - BW / 2 : i; };
  const uint32_t w_at = lds0 + w_first * kMxTile + lane * 16, t_at = lds0 + t_first * kMxTile + lane * 16;
  const uint32_t sw_at = lds0 + S::kScaleAt + w_first * kMxScales + lane * 4, st_at = lds0 + S::kScaleAt + t_first * kMxScales + lane * 4;

  f32x4_t acc[BW][BT] = {};
  static_for<S::kAhead>([&](auto J) {
    constexpr int j = decltype(J)::value;
    issue(j, j * S::kStage, std::integral_constant<bool, j % 4 == 0>{});
  });
  auto loop = [&](auto ROWS_C) {
    constexpr int ROWS = decltype(ROWS_C)::value;
    int sw[BW], sx[BT];
    uint32_t stage = 0, freed = S::kAhead * S::kStage;  // the stage read, the stage filled
    for (int kt = 0; kt < Kb; kt += 4) {
      static_for<4>([&](auto J) {
        constexpr int j = decltype(J)::value;
        if (kt + j < Kb) {
          // this wavefront's share of the stage has landed and its reads of the previous stage are done; behind the barrier
          // that holds for all.  Loads of the steps j + 1 .. j + kAhead - 1 may still be on their way.
          constexpr int scales = ((j + 1) % 4 == 0 && S::kAhead > 1) + ((j + 2) % 4 == 0 && S::kAhead > 2);
          wait_stage<(S::kAhead - 1) * S::kLoads + scales * S::kScaleLoads>();
          __builtin_amdgcn_s_barrier();
          issue(kt + j + S::kAhead, freed, std::integral_constant<bool, (j + S::kAhead) % 4 == 0>{});
          if constexpr (ROWS > 0) {
            if constexpr (j == 0) {
#pragma unroll
              for (int i = 0; i < BW; ++i) sw[i] = *(const lds_int*)(uintptr_t)(sw_at + w_place(i) * kMxScales);
#pragma unroll
              for (int i = 0; i < ROWS; ++i) sx[i] = *(const lds_int*)(uintptr_t)(st_at + WT * i * kMxScales);
            }
            v4i w[BW], x[BT];
#pragma unroll
            for (int i = 0; i < BW; ++i) w[i] = *(const lds_v4i*)(uintptr_t)(w_at + stage + w_place(i) * kMxTile);
#pragma unroll
            for (int i = 0; i < ROWS; ++i) x[i] = *(const lds_v4i*)(uintptr_t)(t_at + stage + WT * i * kMxTile);
#pragma unroll
            for (int b = 0; b < ROWS; ++b)
#pragma unroll
              for (int a = 0; a < BW; ++a) acc[a][b] = mx_mfma<j>(w[a], x[b], acc[a][b], sw[a], sx[b]);
          }
          freed = stage;
          stage = stage + S::kStage == S::kScaleAt ? 0 : stage + S::kStage;
        }
      });
    }
  };
  if (my_blocks == 0) loop(std::integral_constant<int, 0>{});
  else if (my_blocks <= BT / 4) loop(std::integral_constant<int, BT / 4>{});
  else if (my_blocks <= BT / 2) loop(std::integral_constant<int, BT / 2>{});
  else if (my_blocks <= BT * 3 / 4) loop(std::integral_constant<int, BT * 3 / 4>{});
  else loop(std::integral_constant<int, BT>{});
  wait_stage<0>();  // every load (masked ones included) has landed

  __builtin_amdgcn_s_barrier();

  // ---- epilogue
  char* const patch = smem + wave * kPatch<GATEUP ? BW / 2 : BW>;
  static_assert(S::kWaves * kPatch<BW> <= S::kLds, "");
#pragma unroll
  for (int b = 0; b < BT; ++b) {
    if (b >= my_blocks) break;
    const int tb = wt + WT * b, m = m0 + tb * 16;
    if constexpr (GATEUP) {
      const int n = n0 + ww * (BW / 2) * 16;
      if (p.C0) {
        mx_store_rows<BW / 2>(patch, p.C0, p.N, m, m_end, n, [&](int a) { return acc[a][b]; });
        mx_store_rows<BW / 2>(patch, p.C1, p.N, m, m_end, n, [&](int a) { return acc[BW / 2 + a][b]; });
      }
#pragma unroll
      for (int a = 0; a < BW / 2; a += 2) {
        const f32x4_t g2[2] = {acc[a][b], acc[a + 1][b]}, u2[2] = {acc[BW / 2 + a][b], acc[BW / 2 + a + 1][b]};
        mx_store_swiglu(p, g2, u2, rb0 + tb, n + a * 16);
      }
    } else {
      mx_store_rows<BW>(patch, p.C0, p.N, m, m_end, n0 + ww * BW * 16, [&](int a) { return acc[a][b]; });
    }
  }
}

// The most output tiles that a product can have
template <bool GATEUP, class S>
static int64_t mx_tile_count(const dynmo_desc* d) {
  constexpr int TN = S::kWBlocks * 16 / (GATEUP ? 2 : 1), TM = S::kTBlocks * 16;
  const int64_t rows = (int64_t)d->T * d->k, row_tiles = rows / TM + (rows < d->E ? rows : d->E);
  return row_tiles * (((GATEUP ? (int64_t)mx_k_blocks(d->F) * 128 : d->H) + TN - 1) / TN);
}
// A launch has fewer than 2^32 threads; the list is rounded up to whole runs
constexpr int64_t kMaxTiles = (1 << 24) - (1 << 12);

template <bool GATEUP, class S>
static int32_t launch_mx(MxProduct p, const dynmo_desc* d, KernelId id, hipStream_t st) {
  const int64_t tiles = mx_tile_count<GATEUP, S>(d);
  if (tiles == 0) return DYNMO_OK;
  p.list = tile_list((int)tiles);
  DYNMO_TIMED_LAUNCH(id, st, ffn_mx_kernel<GATEUP, S><<<dim3(p.list.blocks), dim3(S::kThreads), 0, st>>>(p));
  return DYNMO_OK;
}

// Tiles of 256 weight rows where they fill the chip four times over (two workgroups on each of 256 compute units), of 128 (three) else.  A
// larger tile moves a quarter less through LDS and has a longer prologue and epilogue, so it also wins where few of them have a long k to go, and
// not where many have a short one.  Both, us (tiles of 256):
//   gate/up  8192 rows, 8 experts, 4096 x 14336 (8064) 602 / 636; 12000, 32, 3968 x 2816 (2816) 172 / 185; 6000, 8, 4096 x 8192 (3456) 223 / 233; 32768, 64,
//            2048 x 1024 (2560) 97 / 98; 16384, 16, 1024 x 4096 (4608) 115 / 113; but 16384, 8, 512 x 2048 (2176) 45 / 41, 32768, 16, 4096 x 688 (1664) 130 / 127
//   down     32768, 64, 1024 -> 2048 (2560) 66 / 69; 12000, 32, 2816 -> 3968 (2048) 101 / 107
//            long sums: 8192, 1, 8192 -> 2048 (576) 65 / 79; 4000, 4, 14336 -> 4096 (576) 121 / 143; 6000, 8, 8192 -> 2048 (432) 66 / 76; 6000, 8, 8192 -> 4096
//            (936) 129 / 135; but 4096, 4, 4096 -> 4096 (576) 57 / 48, 16384, 16, 4096 -> 1024 (576) 55 / 50, 2000, 8, 14336 -> 4096 (400) 116 / 112
using Wide = MxShape<8, 4, 2, 2>;
using Narrow = MxShape<4, 4, 2, 2>;
template <bool GATEUP>
static bool takes_wide(const dynmo_desc* d) {
  const int64_t tiles = mx_tile_count<GATEUP, Wide>(d);
  const int steps = mx_k_blocks(GATEUP ? d->H : d->F);
  return GATEUP ? tiles >= 4 * 512 && steps >= 8 : tiles >= 4 * 512 || (tiles >= 416 && steps >= 64);
}
template <bool GATEUP>
static int32_t mx_tiles(const MxProduct& p, const dynmo_desc* d, KernelId id, hipStream_t st) {
  return takes_wide<GATEUP>(d) ? launch_mx<GATEUP, Wide>(p, d, id, st) : launch_mx<GATEUP, Narrow>(p, d, id, st);
}
template <bool GATEUP>
static bool too_many_tiles(const dynmo_desc* d) {
  return (takes_wide<GATEUP>(d) ? mx_tile_count<GATEUP, Wide>(d) : mx_tile_count<GATEUP, Narrow>(d)) > kMaxTiles;
}
// Up to 64 tokens and as many tiles as compute units the down product reads the weights faster without tiles (figures in ffn_mxfp4_few.hip; more
// tokens: 8 experts, 256 rows, 4096 x 14336 57 against 52).  From 512 tiles on it depends on the length of the sum and little is at stake; the whole call, us,
// tiles / without: 16 experts, 4096 x 14336, 16 rows 180 / 177, 128 rows 259 / 258; 16, 4096 x 2048, 16 rows 31.8 / 32.2, 256 rows 39.5 / 40.7; 8, 8192 x 8192, 64 rows
// 147 / 150; 32, 4096 x 4096, 128 rows, 1024 tiles 153 / 150; 64, 2048 x 1408, 384 rows, 1024 tiles 59.8 / 65.4.
// 0: tiles; else the experts that can have rows.
static int few_rows_experts(const dynmo_desc* d) {
  const int64_t rows = (int64_t)d->T * d->k, experts = rows < d->E ? rows : d->E;
  return d->T <= 64 && experts * ((d->H + 127) / 128) <= 256 ? (int)experts : 0;
}
// Whether the row blocks and both products' tiles fit launches: asked before the first one is made
static bool mx_fits(const dynmo_desc* d) {
  return mx_max_row_blocks(d) < kMaxBlocks && !too_many_tiles<true>(d) && (few_rows_experts(d) || !too_many_tiles<false>(d));
}

struct MxWorkspace {
  size_t x, xs, a, as, bytes;  // offsets from a 256-byte boundary
};
static MxWorkspace mx_workspace(const dynmo_desc* d) {
  const size_t blocks = (size_t)mx_max_row_blocks(d);
  MxWorkspace w;
  w.x = 0;
  w.xs = w.x + blocks * mx_k_blocks(d->H) * kMxTile;
  w.a = w.xs + blocks * mx_k_quads(d->H) * kMxScales;
  w.as = w.a + blocks * mx_k_blocks(d->F) * kMxTile;
  w.bytes = w.as + blocks * mx_k_quads(d->F) * kMxScales + 256;
  return w;
}
static size_t mx_rows_bytes(const dynmo_desc* d) { return align_up((size_t)d->T * d->k * d->H * elem_bytes(d->dtype), 256); }

}  // namespace dynmo

using namespace dynmo;

extern "C" size_t dynmo_grouped_ffn_mxfp4_workspace_bytes(const dynmo_desc* d) {
  if (check_desc(d) || d->dtype != DYNMO_BF16) return 0;
  return mx_workspace(d).bytes;
}

extern "C" int32_t dynmo_grouped_ffn_mxfp4(const dynmo_desc* d, const void* x, const int32_t* src_slot, const int32_t* seg_offsets,
                                           const void* Wg, const void* Wu, const void* Wd, void* y_p, void* G_save, void* U_save,
                                           void* workspace, size_t workspace_bytes, void* stream) {
  const int32_t rc = check_desc(d);
  if (rc) return rc;
  if (d->dtype != DYNMO_BF16) return DYNMO_EUNSUPPORTED;
  if (d->H > 1 << 22 || d->F > 1 << 22 || !mx_fits(d)) return DYNMO_EUNSUPPORTED;  // a tile's row blocks are addressed with 32-bit byte offsets
  if (!x || !seg_offsets || !Wg || !Wu || !Wd || !y_p || !workspace || !G_save != !U_save) return DYNMO_EINVAL;
  if (misaligned16(x, Wg, Wu, Wd, y_p, G_save, U_save)) return DYNMO_EINVAL;
  const MxWorkspace w = mx_workspace(d);
  if (workspace_bytes < w.bytes) return DYNMO_EWORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  char* base = (char*)align_up((size_t)workspace, 256);
  int32_t r = mx_quantize_segments(d, x, src_slot, seg_offsets, d->H, base + w.x, base + w.xs, st);
  if (r) return r;
  MxProduct p = {};
  p.seg = seg_offsets;
  p.E = d->E;
  p.N = d->F;
  p.K = d->H;
  p.X = base + w.x;
  p.Xs = base + w.xs;
  p.W1 = (const char*)Wg;
  p.W2 = (const char*)Wu;
  p.w_bytes = mx_bytes(d->F, d->H);
  p.A = base + w.a;
  p.As = base + w.as;
  p.C0 = (bf16_t*)G_save;
  p.C1 = (bf16_t*)U_save;
  r = mx_tiles<true>(p, d, K_FFN_GATEUP, st);
  if (r) return r;
  p.N = d->H;
  p.K = d->F;
  p.X = base + w.a;
  p.Xs = base + w.as;
  p.W1 = (const char*)Wd;
  p.w_bytes = mx_bytes(d->H, d->F);
  p.C0 = (bf16_t*)y_p;
  if (const int experts = few_rows_experts(d)) return mx_few_rows(p, experts, K_FFN_DOWN, st);
  return mx_tiles<false>(p, d, K_FFN_DOWN, st);
}

extern "C" size_t dynmo_grouped_ffn_mxfp4_bwd_workspace_bytes(const dynmo_desc* d) {
  if (check_desc(d) || d->dtype != DYNMO_BF16) return 0;
  return mx_rows_bytes(d) + dynmo_grouped_ffn_bwd_workspace_bytes(d);  // Q(X), and what the bf16 products need
}

extern "C" int32_t dynmo_grouped_ffn_mxfp4_bwd(const dynmo_desc* d, const void* dy_p, const void* fwd_workspace, size_t fwd_workspace_bytes,
                                               const void* G_save, const void* U_save, const int32_t* seg_offsets, const void* Wg,
                                               const void* Wu, const void* Wd, void* dx_p, void* dWg, void* dWu, void* dWd,
                                               void* workspace, size_t workspace_bytes, void* stream) {
  const int32_t rc = check_desc(d);
  if (rc) return rc;
  if (d->dtype != DYNMO_BF16 || d->H > 1 << 22 || d->F > 1 << 22 || !mx_fits(d)) return DYNMO_EUNSUPPORTED;
  if (!fwd_workspace || !workspace) return DYNMO_EINVAL;
  const MxWorkspace w = mx_workspace(d);
  if (fwd_workspace_bytes < w.bytes || workspace_bytes < dynmo_grouped_ffn_mxfp4_bwd_workspace_bytes(d)) return DYNMO_EWORKSPACE;
  const char* saved = (const char*)align_up((size_t)fwd_workspace, 256);
  const MxSaved mx = {saved + w.x, saved + w.xs, saved + w.a, saved + w.as, (void*)align_up((size_t)workspace, 256)};
  return ffn_bwd_entry(d, dy_p, mx.rows, G_save, U_save, seg_offsets, Wg, Wu, Wd, dx_p, dWg, dWu, dWd, (char*)workspace + mx_rows_bytes(d),
                       workspace_bytes - mx_rows_bytes(d), nullptr, &mx, stream);
}
