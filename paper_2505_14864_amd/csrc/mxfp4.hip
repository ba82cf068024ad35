// MXFP4 quantisation and its reverse.  Bound by memory: a value is read once and 17/32 byte written (or the other way round).
#include "ffn_mxfp4.h"

namespace dynmo {

// A wavefront takes tiles of 16 rows x 128 values, one after another along a row block, and asks for the next one before it works on the
// present one.  Four lanes hold a block of 32 (eight values each), sixteen lanes a row, so that a load of the wavefront covers 256 (fp32: 512)
// contiguous bytes of four rows, and a store 64 bytes of each block column.  The four wavefronts of a workgroup share a row block.
constexpr int kQuantThreads = 256, kQuantWaves = 4;

// ONCE: past the caches.  A tensor that is quantised is read once, and what it would push out of them is its packed form, which is used next; rows
// that are gathered are read as often as they have experts.  (8 x 14336 x 4096 in fp32 and back, us: loads and stores past the caches 427 + 404,
// the stores only 406 + 495, neither 439 + 492; gathered rows, 8 times each: 22 past the caches, 16.)
template <bool ONCE, typename T>
__device__ __forceinline__ void load8(const T* p, int left, u32x4* v) {
  constexpr int kVec = Elem<T>::kVec;
#pragma unroll
  for (int i = 0; i < 8 / kVec; ++i) {
    v[i] = u32x4{0u, 0u, 0u, 0u};
    if (i * kVec < left) v[i] = ONCE ? __builtin_nontemporal_load((const u32x4*)(p + i * kVec)) : *(const u32x4*)(p + i * kVec);
  }
}

// the value of lane ^ 1, lane ^ 2
__device__ __forceinline__ uint32_t quad_xor1(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t quad_xor2(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true); }

// Eight values of each lane -> their codes, and the block's scale byte (the same in the four lanes of a block).  Of bfloat16 values the largest
// magnitude is found on pairs, and the conversion takes them as they are.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ uint32_t quantize_block(const u32x4* piece, uint32_t* scale) {
  uint32_t amax = 0;
  if constexpr (sizeof(T) == 2) {
    u16x2 two = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) two = __builtin_elementwise_max(two, __builtin_bit_cast(u16x2, piece[0][i] & 0x7fff7fffu));
    amax = (uint32_t)max(two.x, two.y) << 16;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, piece[i / 4][i % 4] & 0x7fffffffu);
  }
  amax = max(amax, quad_xor1(amax));
  amax = max(amax, quad_xor2(amax));
  *scale = mx_scale_of(amax);
  const float unit = mx_scale_value(*scale);
  uint32_t c = 0;
  if constexpr (sizeof(T) == 2) {
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)piece[0].x), unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)piece[0].y), unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)piece[0].z), unit, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, (uint32_t)piece[0].w), unit, 3);
  } else {
    float v[8];
    unpack16<float>(piece[0], v);
    unpack16<float>(piece[1], v + 4);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], unit, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], unit, 3);
  }
  return *scale == 255 ? 0u : c;
}

// Tiles first, first + stride, .. of a row block.  src[i]: this lane's row 4 i + lane / 16 of it, or nullptr.
template <bool ONCE, typename T>
__device__ __forceinline__ void quantize_rows(const T* const (&src)[4], int K, int first, int stride, char* codes, char* scales) {
  constexpr int kPieces = 8 / Elem<T>::kVec;
  const int lane = threadIdx.x & 63, g = (lane & 15) >> 2, Kb = mx_k_blocks(K), tiles = mx_k_quads(K) * 4;
  u32x4 next[4][kPieces];
  auto load = [&](int kb) {
    const int k = kb * 128 + (lane & 15) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) load8<ONCE>(src[i] + k, src[i] ? K - k : 0, next[i]);
  };
  load(first);
  for (int kb = first; kb < tiles; kb += stride) {  // tiles from Kb on have scales (zero) only
    u32x4 now[4][kPieces];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < kPieces; ++c) now[i][c] = next[i][c];
    if (kb + stride < Kb) load(kb + stride);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * i + (lane >> 4);
      uint32_t scale = 0;
      if (kb < Kb) {
        *(uint32_t*)(codes + (size_t)kb * kMxTile + g * 256 + r * 16 + (lane & 3) * 4) = quantize_block<T>(now[i], &scale);
      }
      if ((lane & 3) == 0) scales[(size_t)(kb / 4) * kMxScales + (g * 16 + r) * 4 + kb % 4] = (char)scale;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx_quantize_kernel(const T* __restrict__ src, char* __restrict__ packed, int rows, int K, int parts) {
  const int Kb = mx_k_blocks(K), Kq = mx_k_quads(K), Rb = mx_row_blocks(rows);
  const unsigned part = blockIdx.x % parts, at = blockIdx.x / parts;
  const int rb = at % Rb, lane = threadIdx.x & 63;
  const long m = at / Rb;
  char* matrix = packed + m * mx_bytes(rows, K);
  const T* row[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = rb * 16 + 4 * i + (lane >> 4);
    row[i] = r < rows ? src + (m * rows + r) * (long)K : nullptr;
  }
  quantize_rows<true>(row, K, part * kQuantWaves + (threadIdx.x >> 6), parts * kQuantWaves, matrix + (size_t)rb * Kb * kMxTile,
                   matrix + mx_code_bytes(Rb, K) + (size_t)rb * Kq * kMxScales);
}

// A wavefront takes a tile, values four at a time: a store of the wavefront covers the 128 values of two rows (fp32: 512 contiguous bytes each).
// `codes`, `scales`: of the row block; row(r): where row r of the sixteen goes, or nullptr behind the last one.  ONCE: the stores go past the caches
// (figures at load8); of 1003 x 1032 bf16 values 4.2 us either way.
template <bool ONCE, typename T, typename Row>
__device__ __forceinline__ void dequantize_tile(const char* codes, const char* scales, int kb, int K, Row&& row) {
  const int lane = threadIdx.x & 63, c0 = (lane & 31) * 4, k = kb * 128 + c0, g = c0 / 32;
  if (k >= K) return;
  codes += (size_t)kb * kMxTile + g * 256 + c0 % 32 / 2;
  scales += (size_t)(kb / 4) * kMxScales + g * 64 + kb % 4;
  uint32_t code[8], byte[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // behind the last row there are zeros
    code[i] = *(const uint16_t*)(codes + (2 * i + (lane >> 5)) * 16);
    byte[i] = *(const uint8_t*)(scales + (2 * i + (lane >> 5)) * 4);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    T* to = row(2 * i + (lane >> 5));
    if (!to) break;
    to += k;
    const float scale = mx_scale_value(byte[i]);
    f32x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], scale, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[i], scale, 1);
    if (byte[i] == 255) lo.x = lo.y = hi.x = hi.y = __uint_as_float(0x7fc00000u);
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    auto store = [](auto v, auto* p) {
      if constexpr (ONCE) __builtin_nontemporal_store(v, p);
      else *p = v;
    };
    if constexpr (sizeof(T) == 2) store(u32x2{pack_bf16x2(lo.x, lo.y), pack_bf16x2(hi.x, hi.y)}, (u32x2*)to);
    else store(u32x4{__float_as_uint(lo.x), __float_as_uint(lo.y), __float_as_uint(hi.x), __float_as_uint(hi.y)}, (u32x4*)to);
  }
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx_dequantize_kernel(const char* __restrict__ packed, T* __restrict__ dst, int rows, int K) {
  const int Kb = mx_k_blocks(K), Kq = mx_k_quads(K), Rb = mx_row_blocks(rows);
  const unsigned kq = blockIdx.x % Kq, at = blockIdx.x / Kq;
  const int rb = at % Rb;
  const long m = at / Rb;
  const char* matrix = packed + m * mx_bytes(rows, K);
  dequantize_tile<true, T>(matrix + (size_t)rb * Kb * kMxTile, matrix + mx_code_bytes(Rb, K) + (size_t)rb * Kq * kMxScales,
                           kq * 4 + (threadIdx.x >> 6), K, [&](int r) -> T* {
                             return rb * 16 + r < rows ? dst + (m * rows + rb * 16 + r) * (long)K : nullptr;
                           });
}

// Row block rb of the segments: its rows are first .. last - 1, up to sixteen of them counted from first.  false: there is no such block.
__device__ __forceinline__ bool segment_block(const int32_t* __restrict__ seg, int E, int rb, int* first, int* last) {
  // lane e counts the row blocks of expert e; a prefix sum and a ballot find the owner of block rb
  const int lane = threadIdx.x & 63;
  const int begin = lane < E ? seg[lane] : 0, end = lane < E ? seg[lane + 1] : 0;
  const int blocks = mx_row_blocks(end - begin), upto = experts_upto(blocks);
  const unsigned long long owners = __ballot(upto > rb);
  if (owners == 0) return false;
  const int e = __builtin_ctzll(owners);
  *first = __builtin_amdgcn_readlane(begin, e) + (rb - (__builtin_amdgcn_readlane(upto, e) - __builtin_amdgcn_readlane(blocks, e))) * 16;
  *last = __builtin_amdgcn_readlane(end, e);
  return true;
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx_quantize_segments_kernel(const T* __restrict__ x, const int32_t* __restrict__ gather,
                                                                             int gather_div, const int32_t* __restrict__ seg, int E, int K, int parts,
                                                                             char* __restrict__ codes, char* __restrict__ scales) {
  const int Kb = mx_k_blocks(K), Kq = mx_k_quads(K);
  const int part = blockIdx.x % (unsigned)parts, rb = blockIdx.x / (unsigned)parts, lane = threadIdx.x & 63;
  int first, last;
  if (!segment_block(seg, E, rb, &first, &last)) return;
  const T* row[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = first + 4 * i + (lane >> 4);
    row[i] = p < last ? x + (size_t)(gather ? gather[p] / gather_div : p) * K : nullptr;
  }
  quantize_rows<false>(row, K, part * kQuantWaves + (threadIdx.x >> 6), parts * kQuantWaves, codes + (size_t)rb * Kb * kMxTile,
                   scales + (size_t)rb * Kq * kMxScales);
}

// Bound by memory; 8192 rows of 4096 and 14336 values 28 and 90 us (3 to 3.3 TB/s), beside weight gradients of 850 us each.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx_dequantize_segments_kernel(const char* __restrict__ codes, const char* __restrict__ scales,
                                                                               const int32_t* __restrict__ seg, int E, int K, int parts,
                                                                               T* __restrict__ dst) {
  const int Kb = mx_k_blocks(K), Kq = mx_k_quads(K);
  const int part = blockIdx.x % (unsigned)parts, rb = blockIdx.x / (unsigned)parts;
  int first, last;
  if (!segment_block(seg, E, rb, &first, &last)) return;
  for (int kq = part; kq < Kq; kq += parts)
    dequantize_tile<false, T>(codes + (size_t)rb * Kb * kMxTile, scales + (size_t)rb * Kq * kMxScales, kq * 4 + (threadIdx.x >> 6), K,
                              [&](int r) -> T* { return first + r < last ? dst + (size_t)(first + r) * K : nullptr; });
}

// Workgroups per row block: as many as the block has tiles for, but no more than some eight per compute unit in all.
static int parts_of(int64_t row_blocks, int K) {
  const int64_t most = mx_k_quads(K), some = (2048 + row_blocks - 1) / (row_blocks > 0 ? row_blocks : 1);
  return (int)(some < most ? some : most);
}

int32_t mx_quantize_segments(const dynmo_desc* d, const void* x, const int32_t* gather, const int32_t* seg, int K, void* codes, void* scales,
                             hipStream_t st) {
  const int64_t row_blocks = mx_max_row_blocks(d);
  if (row_blocks == 0) return DYNMO_OK;
  const int parts = parts_of(row_blocks, K);
  DYNMO_TIMED_LAUNCH(K_MXFP4_QUANTIZE, st, mx_quantize_segments_kernel<bf16_t><<<dim3((unsigned)(row_blocks * parts)), dim3(kQuantThreads), 0, st>>>(
                                               (const bf16_t*)x, gather, d->k, seg, d->E, K, parts, (char*)codes, (char*)scales));
  return DYNMO_OK;
}

int32_t mx_dequantize_segments(const dynmo_desc* d, const void* codes, const void* scales, const int32_t* seg, int K, bf16_t* dst, hipStream_t st) {
  const int64_t row_blocks = mx_max_row_blocks(d);
  if (row_blocks == 0) return DYNMO_OK;
  const int parts = parts_of(row_blocks, K);
  DYNMO_TIMED_LAUNCH(K_MXFP4_DEQUANTIZE, st, mx_dequantize_segments_kernel<bf16_t><<<dim3((unsigned)(row_blocks * parts)), dim3(kQuantThreads), 0, st>>>(
                                                 (const char*)codes, (const char*)scales, seg, d->E, K, parts, dst));
  return DYNMO_OK;
}

static int32_t check_matrix(int32_t n, int32_t rows, int32_t K, int32_t dtype, const void* values, const void* packed, int64_t* blocks) {
  if (n < 0 || rows < 0 || K <= 0 || (dtype != DYNMO_F32 && dtype != DYNMO_BF16)) return DYNMO_EINVAL;
  if (K % (dtype == DYNMO_BF16 ? 8 : 4)) return DYNMO_EUNSUPPORTED;  // rows move in 16-byte pieces
  if (K > 0x7fffffff - 512 || rows > 0x7fffffff - 16) return DYNMO_EUNSUPPORTED;
  const __int128 all = (__int128)n * mx_row_blocks(rows) * mx_k_quads(K);
  if (all >= kMaxBlocks) return DYNMO_EUNSUPPORTED;
  *blocks = (int64_t)all;
  if (*blocks == 0) return DYNMO_OK;
  if (!values || !packed || misaligned16(values, packed)) return DYNMO_EINVAL;
  return DYNMO_OK;
}

}  // namespace dynmo

using namespace dynmo;

extern "C" size_t dynmo_mxfp4_bytes(int32_t rows, int32_t K) {
  if (rows < 0 || K <= 0 || K > 0x7fffffff - 512 || rows > 0x7fffffff - 16) return 0;
  return mx_bytes(rows, K);
}

extern "C" int32_t dynmo_mxfp4_quantize(int32_t n, int32_t rows, int32_t K, int32_t dtype, const void* src, void* packed, void* stream) {
  int64_t blocks;
  const int32_t rc = check_matrix(n, rows, K, dtype, src, packed, &blocks);
  if (rc || blocks == 0) return rc;
  hipStream_t st = (hipStream_t)stream;
  const int64_t row_blocks = (int64_t)n * mx_row_blocks(rows);
  const int parts = parts_of(row_blocks, K);
  const dim3 grid((unsigned)(row_blocks * parts)), threads(kQuantThreads);
  if (dtype == DYNMO_BF16) {
    DYNMO_TIMED_LAUNCH(K_MXFP4_QUANTIZE, st, mx_quantize_kernel<bf16_t><<<grid, threads, 0, st>>>((const bf16_t*)src, (char*)packed, rows, K, parts));
  } else {
    DYNMO_TIMED_LAUNCH(K_MXFP4_QUANTIZE, st, mx_quantize_kernel<float><<<grid, threads, 0, st>>>((const float*)src, (char*)packed, rows, K, parts));
  }
  return DYNMO_OK;
}

extern "C" int32_t dynmo_mxfp4_dequantize(int32_t n, int32_t rows, int32_t K, int32_t dtype, const void* packed, void* dst, void* stream) {
  int64_t blocks;
  const int32_t rc = check_matrix(n, rows, K, dtype, dst, packed, &blocks);
  if (rc || blocks == 0) return rc;
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)blocks), threads(kQuantThreads);
  if (dtype == DYNMO_BF16) {
    DYNMO_TIMED_LAUNCH(K_MXFP4_DEQUANTIZE, st, mx_dequantize_kernel<bf16_t><<<grid, threads, 0, st>>>((const char*)packed, (bf16_t*)dst, rows, K));
  } else {
    DYNMO_TIMED_LAUNCH(K_MXFP4_DEQUANTIZE, st, mx_dequantize_kernel<float><<<grid, threads, 0, st>>>((const char*)packed, (float*)dst, rows, K));
  }
  return DYNMO_OK;
}
