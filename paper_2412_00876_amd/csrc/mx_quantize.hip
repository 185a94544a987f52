// dllava_mx_quantize, dllava_mx_dequantize: rows to microscaled 4-bit floating point and back.
//
// Pure streams.  A block of four waves takes the 16 x 512 piece whose scales lie together: a wave a row at a time, a lane eight columns
// (16 bytes of bfloat16), four lanes the 32 elements of a scale; the codes of a row's piece leave as 256 consecutive bytes, the
// piece's 256 scale bytes through LDS as one line.
#include "mx.h"

namespace dllava {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kRowsPerWave = kMxTile / kWaves;

// where the scale byte of row r (of 16) and block c (of 16) lies in the piece's 256
__device__ __forceinline__ int scale_slot(int r, int c) { return (c % 4) * 64 + r * 4 + c / 4; }

template <typename T>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const T* __restrict__ x, int64_t ldx, int64_t M, int64_t K, int windows,
                                                               uint32_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  __shared__ __align__(16) uint8_t sm[kMxTile * kMxWindow / kMxBlock];
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  const int64_t tile = blockIdx.x / windows;
  const int win = static_cast<int>(blockIdx.x % windows);
  const int64_t col = static_cast<int64_t>(win) * kMxWindow + 8 * lane;
  float v[kRowsPerWave][8];
#pragma unroll
  for (int i = 0; i < kRowsPerWave; ++i) {
    const int64_t row = tile * kMxTile + i * kWaves + w;
    if (row < M && col < K) {
      mx_load8(x + row * ldx + col, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsPerWave; ++i) {
    const int r = i * kWaves + w;
    const int64_t row = tile * kMxTile + r;
    const uint32_t s = row < M && col < K ? mx_scale_byte(mx_block_amax(v[i])) : 127u;  // (a block's four lanes are inside or outside together)
    if (lane % 4 == 0) sm[scale_slot(r, lane / 4)] = static_cast<uint8_t>(s);
    if (row < M) codes[(row * windows + win) * (kMxWindow / 8) + lane] = mx_encode8(v[i], s);
  }
  __syncthreads();
  if (tid < kWave) reinterpret_cast<uint32_t*>(scales)[static_cast<int64_t>(blockIdx.x) * kWave + tid] = reinterpret_cast<const uint32_t*>(sm)[tid];
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t M,
                                                                 int64_t K, int windows, T* __restrict__ y, int64_t ldy) {
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  const int64_t tile = blockIdx.x / windows;
  const int win = static_cast<int>(blockIdx.x % windows);
  const int64_t col = static_cast<int64_t>(win) * kMxWindow + 8 * lane;
  if (col >= K) return;
  uint32_t c[kRowsPerWave], s[kRowsPerWave];
#pragma unroll
  for (int i = 0; i < kRowsPerWave; ++i) {
    const int r = i * kWaves + w;
    const int64_t row = tile * kMxTile + r;
    c[i] = row < M ? codes[(row * windows + win) * (kMxWindow / 8) + lane] : 0u;
    s[i] = scales[static_cast<int64_t>(blockIdx.x) * 256 + scale_slot(r, lane / 4)];
  }
#pragma unroll
  for (int i = 0; i < kRowsPerWave; ++i) {
    const int64_t row = tile * kMxTile + i * kWaves + w;
    if (row < M) mx_store8(y + row * ldy + col, mx_decode8(c[i], s[i] << 23));
  }
}

int check(const char* who, const void* x, int64_t ldx, int64_t M, int64_t K, const void* packed, size_t packed_bytes, int dtype) {
  DLLAVA_REQUIRE(dtype == DLLAVA_F32 || dtype == DLLAVA_BF16, DLLAVA_EDTYPE, "%s: unknown dtype %d", who, dtype);
  DLLAVA_REQUIRE(M >= 0 && M <= 0x7fffffffLL, DLLAVA_EINVAL, "%s: M = %lld", who, (long long)M);
  DLLAVA_REQUIRE(K > 0 && K % kMxBlock == 0 && K <= 0x7fffffffLL, DLLAVA_ESHAPE, "%s: K must be a positive multiple of 32 (got %lld)", who, (long long)K);
  DLLAVA_REQUIRE(ldx >= K && ldx * static_cast<int64_t>(dtype_size(dtype)) % 16 == 0, DLLAVA_EINVAL,
                 "%s: the row stride %lld must be at least K and a multiple of 16 bytes", who, (long long)ldx);
  if (M == 0) return DLLAVA_OK;
  DLLAVA_REQUIRE(x && packed, DLLAVA_ENULL, "%s: the rows and the packed buffer are required", who);
  DLLAVA_REQUIRE(aligned(x, 16) && aligned(packed, 256), DLLAVA_EINVAL, "%s: rows must be 16-byte, the packed buffer 256-byte aligned", who);
  DLLAVA_REQUIRE(packed_bytes >= dllava_mx_bytes(M, K), DLLAVA_ECAPACITY, "%s: the packed buffer needs %zu bytes (got %zu)", who,
                 dllava_mx_bytes(M, K), packed_bytes);
  DLLAVA_REQUIRE(ceil_div(M, kMxTile) * (mx_padded(K) / kMxWindow) < (1 << 24), DLLAVA_ESHAPE,
                 "%s: ceil(M / 16) * ceil(K / 512) must be below 2^24", who);
  return DLLAVA_OK;
}

}  // namespace
}  // namespace dllava

using namespace dllava;

extern "C" size_t dllava_mx_bytes(int64_t M, int64_t K) {
  if (M < 0 || K <= 0 || K % kMxBlock != 0 || M > 0x7fffffffLL || K > 0x7fffffffLL) return 0;
  return round_up(mx_code_bytes(M, K) + mx_scale_bytes(M, K), 256);
}

extern "C" int dllava_mx_quantize(const void* x, int64_t ldx, int64_t M, int64_t K, void* packed, size_t packed_bytes, int dtype, void* stream) {
  if (int rc = check("mx_quantize", x, ldx, M, K, packed, packed_bytes, dtype)) return rc;
  if (M == 0) return DLLAVA_OK;
  const int windows = static_cast<int>(mx_padded(K) / kMxWindow);
  const dim3 grid(static_cast<unsigned>(ceil_div(M, kMxTile) * windows));
  uint32_t* codes = static_cast<uint32_t*>(packed);
  uint8_t* scales = static_cast<uint8_t*>(packed) + mx_code_bytes(M, K);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == DLLAVA_BF16)
    hipLaunchKernelGGL(mx_quantize_kernel<bf16_t>, grid, dim3(kThreads), 0, st, static_cast<const bf16_t*>(x), ldx, M, K, windows, codes, scales);
  else
    hipLaunchKernelGGL(mx_quantize_kernel<float>, grid, dim3(kThreads), 0, st, static_cast<const float*>(x), ldx, M, K, windows, codes, scales);
  DLLAVA_CHECK_LAUNCH("mx_quantize_kernel");
  return DLLAVA_OK;
}

extern "C" int dllava_mx_dequantize(const void* packed, size_t packed_bytes, int64_t M, int64_t K, void* y, int64_t ldy, int dtype, void* stream) {
  if (int rc = check("mx_dequantize", y, ldy, M, K, packed, packed_bytes, dtype)) return rc;
  if (M == 0) return DLLAVA_OK;
  const int windows = static_cast<int>(mx_padded(K) / kMxWindow);
  const dim3 grid(static_cast<unsigned>(ceil_div(M, kMxTile) * windows));
  const uint32_t* codes = static_cast<const uint32_t*>(packed);
  const uint8_t* scales = static_cast<const uint8_t*>(packed) + mx_code_bytes(M, K);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == DLLAVA_BF16)
    hipLaunchKernelGGL(mx_dequantize_kernel<bf16_t>, grid, dim3(kThreads), 0, st, codes, scales, M, K, windows, static_cast<bf16_t*>(y), ldy);
  else
    hipLaunchKernelGGL(mx_dequantize_kernel<float>, grid, dim3(kThreads), 0, st, codes, scales, M, K, windows, static_cast<float*>(y), ldy);
  DLLAVA_CHECK_LAUNCH("mx_dequantize_kernel");
  return DLLAVA_OK;
}
