// dllava_mx_linear: y = act(x W^T + bias) (+ | *) residual, rows and weights in 4 bits, on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// A lane's operand is the 32 elements of one scale (16 bytes), and its scale one byte of a register: four consecutive products of a
// wave take the four bytes of the scales that lie together (see the packed form in dllava_mx.h).
#include "mx_linear.h"

namespace dllava {

int mx_linear_check(const char* who, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N, int act, const void* residual,
                    const void* y, int64_t ldy, int dtype);  // mx_few.hip
MxLinearArgs mx_linear_args(int64_t M, int64_t K, const void* Wq, const float* bias, int64_t N, int act, const void* residual, void* y, int64_t ldy);

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 operand(const uint4& c) {
  return i32x8{static_cast<int>(c.x), static_cast<int>(c.y), static_cast<int>(c.z), static_cast<int>(c.w), 0, 0, 0, 0};
}

// A block of four waves: 64 features x 64 rows, a wave 32 x 32, operands straight from memory.
__global__ __launch_bounds__(256) void mx_linear_kernel(MxLinearArgs a, int n_ft) {
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, g = lane / 16, r16 = lane % 16;
  const int n0 = static_cast<int>(blockIdx.x % n_ft) * 64 + 32 * (w / 2);
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / n_ft) * 64 + 32 * (w % 2);
  if (n0 >= a.N || m0 >= a.M) return;
  const int64_t row_bytes = static_cast<int64_t>(a.windows) * (kMxWindow / 2);
  const uint8_t *wr[2], *ws[2], *xr[2], *xs[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int n = n0 + 16 * i + r16 < a.N ? n0 + 16 * i + r16 : a.N - 1;
    const int nt = n0 + 16 * i < a.N ? n0 / 16 + i : (a.N - 1) / 16;
    const int64_t m = m0 + 16 * i + r16 < a.M ? m0 + 16 * i + r16 : a.M - 1;
    const int64_t mt = m0 + 16 * i < a.M ? m0 / 16 + i : (a.M - 1) / 16;
    wr[i] = a.Wc + n * row_bytes + 16 * g;
    xr[i] = a.Xc + m * row_bytes + 16 * g;
    ws[i] = a.Ws + static_cast<int64_t>(nt) * a.windows * 256 + 4 * lane;
    xs[i] = a.Xs + mt * a.windows * 256 + 4 * lane;
  }
  f32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int64_t win = 0; win < a.windows; ++win) {
    uint4 wc[2][4], xc[2][4];
    int sw[2], sx[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sw[i] = *reinterpret_cast<const int*>(ws[i] + win * 256);
      sx[i] = *reinterpret_cast<const int*>(xs[i] + win * 256);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        wc[i][s] = *reinterpret_cast<const uint4*>(wr[i] + win * 256 + 64 * s);
        xc[i][s] = *reinterpret_cast<const uint4*>(xr[i] + win * 256 + 64 * s);
      }
    }
#define DLLAVA_STEP(s)                                                                                                                          \
  for (int i = 0; i < 2; ++i)                                                                                                                   \
    for (int j = 0; j < 2; ++j)                                                                                                                 \
      acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(wc[i][s]), operand(xc[j][s]), acc[i][j], 4, 4, s, sw[i], s, sx[j]);
    _Pragma("unroll") DLLAVA_STEP(0) _Pragma("unroll") DLLAVA_STEP(1) _Pragma("unroll") DLLAVA_STEP(2) _Pragma("unroll") DLLAVA_STEP(3)
#undef DLLAVA_STEP
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = n0 + 16 * i + 4 * g;
      const int64_t m = m0 + 16 * j + r16;
      if (n < a.N && m < a.M) mx_store_results(a, m, n, make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]));
    }
}

}  // namespace
}  // namespace dllava

using namespace dllava;

extern "C" int dllava_mx_linear(const void* xq, size_t xq_bytes, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N,
                                int act, const void* residual, void* y, int64_t ldy, int dtype, void* stream) {
  if (int rc = mx_linear_check("mx_linear", M, K, Wq, Wq_bytes, bias, N, act, residual, y, ldy, dtype)) return rc;
  if (M == 0 || N == 0) return DLLAVA_OK;
  DLLAVA_REQUIRE(xq, DLLAVA_ENULL, "mx_linear: xq is required");
  DLLAVA_REQUIRE(aligned(xq, 256), DLLAVA_EINVAL, "mx_linear: xq must be 256-byte aligned");
  DLLAVA_REQUIRE(xq_bytes >= dllava_mx_bytes(M, K), DLLAVA_ECAPACITY, "mx_linear: the packed rows are %zu bytes (got %zu)", dllava_mx_bytes(M, K), xq_bytes);
  MxLinearArgs a = mx_linear_args(M, K, Wq, bias, N, act, residual, y, ldy);
  a.Xc = static_cast<const uint8_t*>(xq);
  a.Xs = a.Xc + mx_code_bytes(M, K);
  const int64_t n_ft = ceil_div(N, 64), blocks = n_ft * ceil_div(M, 64);
  DLLAVA_REQUIRE(blocks <= 0x7fffffffLL, DLLAVA_ESHAPE, "mx_linear: too many results");
  hipLaunchKernelGGL(mx_linear_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, static_cast<hipStream_t>(stream), a, static_cast<int>(n_ft));
  DLLAVA_CHECK_LAUNCH("mx_linear_kernel");
  return DLLAVA_OK;
}
