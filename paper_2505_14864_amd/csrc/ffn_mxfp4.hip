// Grouped SwiGLU FFN, forward, on MXFP4 weights (mxfp4.h): the rows are quantised block by block, and both products run on the scaled
// matrix instructions (v_mfma_scale_f32_16x16x128_f8f6f4, 4-bit operands, fp32 accumulation).
//
//   G = Q(X) Wg^T, U = Q(X) Wu^T, A = Q(silu(G) U), Y = A Wd^T
//
// G, U and A are fp32 values up to A's quantisation: rounding them to bf16 in between would move values over the borders of a
// four-bit grid that has eight steps.  Operand A of an MFMA is the weights and operand B the rows, so that a lane of the result holds four consecutive columns
// of one row, and a block of 32 columns lies in two results and four lanes: its largest value takes two lane exchanges.
//
// One workgroup of four wavefronts (2 x 2) per output tile of 128 weight rows x 128 rows, k in steps of 128 through a ring of three LDS
// stages; a step's tiles of 1 KB are loaded into LDS as they lie in memory.
#include "ffn_gemm.h"
#include "mxfp4.h"
#include "tile_list.h"

namespace dynmo {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4i lds_v4i;
typedef __attribute__((address_space(3))) int lds_int;

struct MxProduct {
  const int32_t* seg;
  int E;
  int N;               // columns of the result: F for gate/up, H for down
  int K;
  const char* X;       // the rows: codes, in row blocks of one expert each
  const char* Xs;      // and their scales
  const char* W1;      // gate, or down
  const char* W2;      // up
  size_t w_bytes;      // of one expert's matrix
  char* A;             // gate/up: the quantised result (K of the down product = N)
  char* As;
  bf16_t* C0;          // down: Y; gate/up: G to save, or nullptr
  bf16_t* C1;          // U to save, or nullptr
  TileList list;
};

__device__ __forceinline__ desc_t bytes_desc(const char* p) { return make_desc((const bf16_t*)p, 0x7ffffffeu); }

template <int J>
__device__ __forceinline__ f32x4_t mx_mfma(v4i a, v4i b, f32x4_t c, int sa, int sb) {
  const v8i a8 = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, b8 = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, J, sa, J, sb);
}

// BW x BT blocks of 16 x 16 per wavefront, WW x WT wavefronts
template <int BW_, int BT_, int WW_, int WT_>
struct MxShape {
  static constexpr int BW = BW_, BT = BT_, WW = WW_, WT = WT_;
  static constexpr int kWaves = WW * WT, kThreads = 64 * kWaves;
  static constexpr int kWBlocks = BW * WW, kTBlocks = BT * WT, kBlocks = kWBlocks + kTBlocks;  // of the tile
  static constexpr int kStages = 3, kAhead = kStages - 1;
  static constexpr int kStage = kBlocks * kMxTile, kScaleAt = kStages * kStage, kLds = kScaleAt + kBlocks * kMxScales;
  static constexpr int kLoads = kBlocks / kWaves;               // tiles that a wavefront loads per step
  static constexpr int kScaleLoads = kBlocks / 4 / kWaves;      // loads of the scales of four steps, 1 KB each
  static_assert(kBlocks % kWaves == 0 && kBlocks % (4 * kWaves) == 0, "");
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
  int upto = mt, blocks_upto = blocks;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(upto, d, 64), ob = __shfl_up(blocks_upto, d, 64);
    if (lane >= d) upto += o, blocks_upto += ob;
  }
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
  const int Kb = mx_k_blocks(p.K), Kq = mx_k_quads(p.K), Wb = mx_row_blocks(p.N);
  const char* const w1 = p.W1 + e * p.w_bytes;
  const char* const w2 = GATEUP ? p.W2 + e * p.w_bytes : w1;
  const size_t scales_at = (size_t)Wb * Kb * kMxTile;
  constexpr int kHalf = GATEUP ? S::kWBlocks / 2 : S::kWBlocks;
  const int nb0 = n0 / 16;
  const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
  const uint32_t tile_ld = (uint32_t)Kb * kMxTile, scale_ld = (uint32_t)Kq * kMxScales;
  // where block b of the step lies: its matrix, and its row block there, or -1 where there is none
  auto place = [&](int b, int* which) {
    if (b >= S::kWBlocks) {
      *which = 2;
      return b - S::kWBlocks < t_blocks ? b - S::kWBlocks : -1;
    }
    *which = b >= kHalf ? 1 : 0;
    const int r = b >= kHalf ? b - kHalf : b;
    return nb0 + r < Wb ? r : -1;
  };
  auto issue = [&](int step, uint32_t stage, auto SCALES) {
    const bool any = step < Kb;
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds0 + stage + wave * S::kLoads * kMxTile);
    static_for<S::kLoads>([&](auto J) {
      constexpr int j = decltype(J)::value;
      int which;
      const int r = place(wave * S::kLoads + j, &which);
      const char* base = which == 2 ? p.X + ((size_t)rb0 * Kb + step) * kMxTile : (which == 1 ? w2 : w1) + ((size_t)nb0 * Kb + step) * kMxTile;
      load_to_lds<j * kMxTile>(bytes_desc(base), lds, any && r >= 0 ? (uint32_t)r * tile_ld + lane * 16 : kOob);
    });
    if constexpr (decltype(SCALES)::value) {
      const int kq = step / 4;
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + S::kScaleAt + wave * S::kScaleLoads * 1024);
      static_for<S::kScaleLoads>([&](auto J) {
        constexpr int j = decltype(J)::value;
        int which;  // the four blocks of a load lie in one matrix
        const int b = (wave * S::kScaleLoads + j) * 4;
        place(b, &which);
        int unused;
        const int r = place(b + (lane >> 4), &unused);
        const char* base = which == 2 ? p.Xs + ((size_t)rb0 * Kq + kq) * kMxScales : (which == 1 ? w2 : w1) + scales_at + ((size_t)nb0 * Kq + kq) * kMxScales;
        load_to_lds<j * 1024>(bytes_desc(base), to, any && r >= 0 ? (uint32_t)r * scale_ld + (lane & 15) * 16 : kOob);
      });
    }
  };

  const int my_blocks = max(0, min(BT, (t_blocks - wt + WT - 1) / WT));  // row blocks wt, wt + WT, .. of the tile
  auto w_block = [&](int i) { return GATEUP ? (i < BW / 2 ? ww * (BW / 2) + i : kHalf + ww * (BW / 2) + i - BW / 2) : ww * BW + i; };
  auto t_block = [&](int i) { return S::kWBlocks + wt + WT * i; };

  f32x4_t acc[BW][BT] = {};
  static_for<S::kAhead>([&](auto J) {
    constexpr int j = decltype(J)::value;
    issue(j, j * S::kStage, std::integral_constant<bool, j % 4 == 0>{});
  });
  int sw[BW], sx[BT];
  uint32_t stage = 0, freed = S::kAhead * S::kStage;
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
        if (j == 0) {
#pragma unroll
          for (int i = 0; i < BW; ++i) sw[i] = *(const lds_int*)(uintptr_t)(lds0 + S::kScaleAt + w_block(i) * kMxScales + lane * 4);
#pragma unroll
          for (int i = 0; i < BT; ++i) sx[i] = *(const lds_int*)(uintptr_t)(lds0 + S::kScaleAt + t_block(i) * kMxScales + lane * 4);
        }
        if (my_blocks > 0) {
          v4i w[BW], x[BT];
#pragma unroll
          for (int i = 0; i < BW; ++i) w[i] = *(const lds_v4i*)(uintptr_t)(lds0 + stage + w_block(i) * kMxTile + lane * 16);
#pragma unroll
          for (int i = 0; i < BT; ++i) x[i] = *(const lds_v4i*)(uintptr_t)(lds0 + stage + t_block(i) * kMxTile + lane * 16);
#pragma unroll
          for (int b = 0; b < BT; ++b)
#pragma unroll
            for (int a = 0; a < BW; ++a) acc[a][b] = mx_mfma<j>(w[a], x[b], acc[a][b], sw[a], sx[b]);
        }
        freed = stage;
        stage = stage + S::kStage == S::kScaleAt ? 0 : stage + S::kStage;
      }
    });
  }
  wait_stage<0>();  // every load (masked ones included) has landed

  // ---- epilogue.  Element r of block (a, b): column 16 a + 4 (lane / 16) + r, row lane % 16 of row block b.
  const int g = lane >> 4, row = lane & 15;
#pragma unroll
  for (int b = 0; b < BT; ++b) {
    if (b >= my_blocks) break;
    const int tb = wt + WT * b, m = m0 + tb * 16 + row;
    if constexpr (GATEUP) {
      const int Fb = mx_k_blocks(p.N), Fq = mx_k_quads(p.N);
#pragma unroll
      for (int a = 0; a < BW / 2; a += 2) {  // two blocks are 32 columns: a block of the next product's k
        const int n = n0 + (ww * (BW / 2) + a) * 16;
        float h[2][4];
        uint32_t amax = 0;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int col = n + c * 16 + g * 4;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float gv = acc[a + c][b][r], uv = acc[BW / 2 + a + c][b][r];
            h[c][r] = gv / (1.f + __expf(-gv)) * uv;
            amax = max(amax, __float_as_uint(h[c][r]) & 0x7fffffffu);
          }
          if (p.C0 && m < m_end && col < p.N) {
            const uint2 gs = {pack_bf16x2(acc[a + c][b][0], acc[a + c][b][1]), pack_bf16x2(acc[a + c][b][2], acc[a + c][b][3])};
            const f32x4_t u4 = acc[BW / 2 + a + c][b];
            const uint2 us = {pack_bf16x2(u4[0], u4[1]), pack_bf16x2(u4[2], u4[3])};
            *(uint2*)(p.C0 + (size_t)m * p.N + col) = gs;
            *(uint2*)(p.C1 + (size_t)m * p.N + col) = us;
          }
        }
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 16, 64));
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32, 64));
        const uint32_t byte = mx_scale_of(amax);
        const float scale = mx_scale_value(byte);
        if (n >= Fb * 128) continue;
        char* block = p.A + ((size_t)(rb0 + tb) * Fb + n / 128) * kMxTile + n % 128 / 32 * 256 + row * 16;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t code = 0;
          code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, h[c][0], h[c][1], scale, 0);
          code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, h[c][2], h[c][3], scale, 1);
          *(uint16_t*)(block + c * 8 + g * 2) = byte == 255 ? (uint16_t)0 : (uint16_t)code;
        }
        if (g == 0) p.As[((size_t)(rb0 + tb) * Fq + n / 512) * kMxScales + (n % 128 / 32 * 16 + row) * 4 + n % 512 / 128] = (char)byte;
      }
    } else {
#pragma unroll
      for (int a = 0; a < BW; ++a) {
        const int col = n0 + (ww * BW + a) * 16 + g * 4;
        if (m >= m_end || col >= p.N) continue;
        const uint2 y = {pack_bf16x2(acc[a][b][0], acc[a][b][1]), pack_bf16x2(acc[a][b][2], acc[a][b][3])};
        *(uint2*)(p.C0 + (size_t)m * p.N + col) = y;
      }
    }
  }
}

template <bool GATEUP, class S>
static int32_t launch_mx(MxProduct p, const dynmo_desc* d, KernelId id, hipStream_t st) {
  constexpr int TN = S::kWBlocks * 16 / (GATEUP ? 2 : 1), TM = S::kTBlocks * 16;
  const int64_t rows = (int64_t)d->T * d->k, row_tiles = rows / TM + (rows < d->E ? rows : d->E);
  const int64_t tiles = row_tiles * (((GATEUP ? (int64_t)mx_k_blocks(p.N) * 128 : p.N) + TN - 1) / TN);
  if (tiles == 0) return DYNMO_OK;
  if (tiles > (1 << 30)) return DYNMO_EUNSUPPORTED;
  p.list = tile_list((int)tiles);
  DYNMO_TIMED_LAUNCH(id, st, ffn_mx_kernel<GATEUP, S><<<dim3(p.list.blocks), dim3(S::kThreads), 0, st>>>(p));
  return DYNMO_OK;
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
  if (d->H > 1 << 22 || d->F > 1 << 22) return DYNMO_EUNSUPPORTED;  // a tile's row blocks are addressed with 32-bit byte offsets
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
  r = launch_mx<true, MxShape<4, 4, 2, 2>>(p, d, K_FFN_GATEUP, st);
  if (r) return r;
  p.N = d->H;
  p.K = d->F;
  p.X = base + w.a;
  p.Xs = base + w.as;
  p.W1 = (const char*)Wd;
  p.w_bytes = mx_bytes(d->H, d->F);
  p.C0 = (bf16_t*)y_p;
  return launch_mx<false, MxShape<4, 4, 2, 2>>(p, d, K_FFN_DOWN, st);
}
