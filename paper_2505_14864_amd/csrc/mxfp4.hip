// MXFP4 quantisation and its reverse.  Bound by memory: a value is read once and 17/32 byte written (or the other way round).
#include "mxfp4.h"

#include "profile.h"

namespace dynmo {

// One workgroup: 16 rows x 512 values, a wavefront for each tile of 128.  Four lanes hold a block of 32 (eight values each), sixteen
// lanes a row, so that a wavefront reads 256 (fp32: 512) contiguous bytes of four rows at a time; the scales of the four tiles meet in LDS.
constexpr int kQuantThreads = 256;

template <typename T>
__device__ __forceinline__ void load8(const T* p, int left, float* v) {
  constexpr int kVec = Elem<T>::kVec;
#pragma unroll
  for (int i = 0; i < 8; i += kVec) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    unpack16<T>(i < left ? *(const u32x4*)(p + i) : zero, v + i);
  }
}

// Eight values of each lane -> their codes, and the block's scale byte (the same in the four lanes of a block)
__device__ __forceinline__ uint32_t quantize_block(const float* v, uint32_t* scale) {
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1, 64));
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2, 64));
  *scale = mx_scale_of(amax);
  return *scale == 255 ? 0u : mx_codes8(v, mx_scale_value(*scale));
}

// `row(r)`: the source row of row r (0 .. 15) of the block, or nullptr
template <typename T, typename Row>
__device__ __forceinline__ void quantize_rows(Row&& row, int K, int kq, int Kb, char* codes, char* scales) {
  __shared__ uint32_t quad[64];
  const int lane = threadIdx.x & 63, tile = threadIdx.x >> 6, kb = kq * 4 + tile;
  const int k = kb * 128 + (lane & 15) * 8, g = (lane & 15) >> 2;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + (lane >> 4);
    const T* src = row(r);
    float v[8];
    load8<T>(src + k, src ? K - k : 0, v);
    uint32_t scale;
    const uint32_t c = quantize_block(v, &scale);
    if (kb < Kb) *(uint32_t*)(codes + (size_t)kb * kMxTile + g * 256 + r * 16 + (lane & 3) * 4) = c;
    if ((lane & 3) == 0) ((uint8_t*)quad)[(g * 16 + r) * 4 + tile] = (uint8_t)scale;
  }
  __syncthreads();
  if (threadIdx.x < 64) *(uint32_t*)(scales + (size_t)kq * kMxScales + lane * 4) = quad[lane];
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx_quantize_kernel(const T* __restrict__ src, char* __restrict__ packed, int rows, int K) {
  const int Kb = mx_k_blocks(K), Kq = mx_k_quads(K), Rb = mx_row_blocks(rows);
  const unsigned kq = blockIdx.x % Kq, at = blockIdx.x / Kq;
  const int rb = at % Rb;
  const long m = at / Rb;
  char* matrix = packed + m * mx_bytes(rows, K);
  quantize_rows<T>([&](int r) { return rb * 16 + r < rows ? src + (m * rows + rb * 16 + r) * (long)K : nullptr; }, K, kq, Kb,
                   matrix + (size_t)rb * Kb * kMxTile, matrix + mx_code_bytes(Rb, K) + (size_t)rb * Kq * kMxScales);
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx_dequantize_kernel(const char* __restrict__ packed, T* __restrict__ dst, int rows, int K) {
  const int Kb = mx_k_blocks(K), Kq = mx_k_quads(K), Rb = mx_row_blocks(rows);
  const unsigned kq = blockIdx.x % Kq, at = blockIdx.x / Kq;
  const int rb = at % Rb;
  const long m = at / Rb;
  const char* matrix = packed + m * mx_bytes(rows, K);
  const char* codes = matrix + (size_t)rb * Kb * kMxTile;
  const char* scales = matrix + mx_code_bytes(Rb, K) + ((size_t)rb * Kq + kq) * kMxScales;
  const int lane = threadIdx.x & 63, tile = threadIdx.x >> 6, kb = kq * 4 + tile;
  const int k = kb * 128 + (lane & 15) * 8, g = (lane & 15) >> 2;
  if (k >= K) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + (lane >> 4);
    if (rb * 16 + r >= rows) break;
    const uint32_t c = *(const uint32_t*)(codes + (size_t)kb * kMxTile + g * 256 + r * 16 + (lane & 3) * 4);
    const uint32_t byte = ((const uint8_t*)scales)[(g * 16 + r) * 4 + tile];
    const float scale = mx_scale_value(byte);
    float v[8];
    f32x2_t two;
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), v[0] = two.x, v[1] = two.y;
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1), v[2] = two.x, v[3] = two.y;
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), v[4] = two.x, v[5] = two.y;
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3), v[6] = two.x, v[7] = two.y;
    if (byte == 255)
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = __uint_as_float(0x7fc00000u);
    T* to = dst + (m * rows + rb * 16 + r) * (long)K + k;
    constexpr int kVec = Elem<T>::kVec;
#pragma unroll
    for (int q = 0; q < 8; q += kVec)
      if (k + q < K) *(u32x4*)(to + q) = pack16<T>(v + q);
  }
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void mx_quantize_segments_kernel(const T* __restrict__ x, const int32_t* __restrict__ gather,
                                                                             int gather_div, const int32_t* __restrict__ seg, int E, int K,
                                                                             char* __restrict__ codes, char* __restrict__ scales) {
  const int Kb = mx_k_blocks(K), Kq = mx_k_quads(K);
  const int kq = blockIdx.x % (unsigned)Kq, rb = blockIdx.x / (unsigned)Kq;
  // lane e counts the row blocks of expert e; a prefix sum and a ballot find the owner of block rb
  const int lane = threadIdx.x & 63;
  const int begin = lane < E ? seg[lane] : 0, end = lane < E ? seg[lane + 1] : 0;
  const int blocks = mx_row_blocks(end - begin);
  int upto = blocks;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(upto, m, 64);
    if (lane >= m) upto += o;
  }
  const unsigned long long owners = __ballot(upto > rb);
  if (owners == 0) return;
  const int e = __builtin_ctzll(owners);
  const int first = __builtin_amdgcn_readlane(begin, e) + (rb - (__builtin_amdgcn_readlane(upto, e) - __builtin_amdgcn_readlane(blocks, e))) * 16;
  const int last = __builtin_amdgcn_readlane(end, e);
  quantize_rows<T>(
      [&](int r) -> const T* {
        if (first + r >= last) return nullptr;
        return x + (long)(gather ? gather[first + r] / gather_div : first + r) * K;
      },
      K, kq, Kb, codes + (size_t)rb * Kb * kMxTile, scales + (size_t)rb * Kq * kMxScales);
}

int32_t mx_quantize_segments(const dynmo_desc* d, const void* x, const int32_t* gather, const int32_t* seg, int K, void* codes, void* scales,
                             hipStream_t st) {
  const int64_t blocks = mx_max_row_blocks(d) * mx_k_quads(K);
  if (blocks == 0) return DYNMO_OK;
  if (blocks > 0x7fffffff) return DYNMO_EUNSUPPORTED;
  DYNMO_TIMED_LAUNCH(K_MXFP4_QUANTIZE, st, mx_quantize_segments_kernel<bf16_t><<<dim3((unsigned)blocks), dim3(kQuantThreads), 0, st>>>(
                                               (const bf16_t*)x, gather, d->k, seg, d->E, K, (char*)codes, (char*)scales));
  return DYNMO_OK;
}

static int32_t check_matrix(int32_t n, int32_t rows, int32_t K, int32_t dtype, const void* values, const void* packed, int64_t* blocks) {
  if (n < 0 || rows < 0 || K <= 0 || (dtype != DYNMO_F32 && dtype != DYNMO_BF16)) return DYNMO_EINVAL;
  if (K % (dtype == DYNMO_BF16 ? 8 : 4)) return DYNMO_EUNSUPPORTED;  // rows move in 16-byte pieces
  if (K > 0x7fffffff - 512 || rows > 0x7fffffff - 16) return DYNMO_EUNSUPPORTED;
  const __int128 all = (__int128)n * mx_row_blocks(rows) * mx_k_quads(K);
  if (all > 0x7fffffff) return DYNMO_EUNSUPPORTED;
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
  const dim3 grid((unsigned)blocks), threads(kQuantThreads);
  if (dtype == DYNMO_BF16) {
    DYNMO_TIMED_LAUNCH(K_MXFP4_QUANTIZE, st, mx_quantize_kernel<bf16_t><<<grid, threads, 0, st>>>((const bf16_t*)src, (char*)packed, rows, K));
  } else {
    DYNMO_TIMED_LAUNCH(K_MXFP4_QUANTIZE, st, mx_quantize_kernel<float><<<grid, threads, 0, st>>>((const float*)src, (char*)packed, rows, K));
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
