// dllava_mx_linear_few: y = act(x W^T + bias) (+ | *) residual for the few rows of a decode step, weights in 4 bits.
//
// The weights' 17/32 byte an element are the traffic.  A block of eight waves takes 16 * FT features and all rows; its waves
// take windows of 512 columns in turn, add up their parts in registers and join them in LDS at the end, in the order of the
// waves: no block waits for another, and no workspace is needed.  A lane reads 16 bytes of codes, 32 elements of one feature; they
// become bfloat16 (exact: two significant bits times a power of two) in registers, four operands of v_mfma_f32_16x16x32_bf16, whose
// columns are the rows of x.  The order in which a product runs over K is free: step s of a piece takes elements 8s .. 8s + 7 of each
// lane's 32, and x is read to match.
#include "mx_linear.h"

namespace dllava {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;

template <int FT>
struct Weights {  // of one window: this lane's 32 elements of each of its four pieces, and their scales
  uint4 c[FT][4];
  uint32_t s[FT];
};

template <int FT, int MT>
__global__ __launch_bounds__(kWaves* kWave) void mx_few_kernel(MxLinearArgs a) {
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, g = lane / 16, r16 = lane % 16;
  const int n0 = blockIdx.x * 16 * FT;
  const int64_t row_bytes = static_cast<int64_t>(a.windows) * (kMxWindow / 2);
  const uint8_t* wrow[FT];
  const uint8_t* srow[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) {
    const int n = n0 + 16 * f + r16 < a.N ? n0 + 16 * f + r16 : a.N - 1;  // features past N are computed and dropped
    const int tile = n0 + 16 * f < a.N ? n0 / 16 + f : (a.N - 1) / 16;
    wrow[f] = a.Wc + n * row_bytes + 16 * g;
    srow[f] = a.Ws + static_cast<int64_t>(tile) * a.windows * 256 + 4 * lane;
  }
  const bf16_t* xrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = 16 * t + r16 < a.M ? 16 * t + r16 : a.M - 1;
    xrow[t] = a.X + m * a.ldx + 32 * g;
  }
  auto load = [&](Weights<FT>& p, int win) {
#pragma unroll
    for (int f = 0; f < FT; ++f) {
#pragma unroll
      for (int j = 0; j < 4; ++j) p.c[f][j] = *reinterpret_cast<const uint4*>(wrow[f] + static_cast<int64_t>(win) * 256 + 64 * j);
      p.s[f] = *reinterpret_cast<const uint32_t*>(srow[f] + static_cast<int64_t>(win) * 256);
    }
  };
  f32x4 acc[FT][MT];
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  Weights<FT> p, next;
  if (w < a.windows) load(p, w);
  for (int win = w; win < a.windows; win += kWaves) {
    if (win + kWaves < a.windows) load(next, win + kWaves);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = win * kMxWindow + 128 * j;
      const bool in = col + 32 * g < a.K;  // behind K the weights' codes are zeros; x is not there
      uint4 x[MT][4];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int s = 0; s < 4; ++s) x[t][s] = in ? *reinterpret_cast<const uint4*>(xrow[t] + col + 8 * s) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const uint32_t sb = p.s[f] >> (8 * j) << 23;
        const uint32_t c[4] = {p.c[f][j].x, p.c[f][j].y, p.c[f][j].z, p.c[f][j].w};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const bf16x8 wv = __builtin_bit_cast(bf16x8, mx_decode8(c[s], sb));
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, __builtin_bit_cast(bf16x8, x[t][s]), acc[f][t], 0, 0, 0);
        }
      }
    }
    p = next;
  }
  // register e of acc[f][t]: feature n0 + 16 f + 4 g + e, row 16 t + r16
  __shared__ float4 sm[kWaves][FT * MT][kWave];
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < MT; ++t) sm[w][f * MT + t][lane] = make_float4(acc[f][t][0], acc[f][t][1], acc[f][t][2], acc[f][t][3]);
  __syncthreads();
  for (int i = w; i < FT * MT; i += kWaves) {
    float4 v = sm[0][i][lane];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) {
      const float4 u = sm[k][i][lane];
      v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
    }
    const int n = n0 + 16 * (i / MT) + 4 * g;
    const int64_t m = 16 * (i % MT) + r16;
    if (n < a.N && m < a.M) mx_store_results(a, m, n, v);
  }
}

template <int FT>
int launch_rows(const MxLinearArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(ceil_div(a.N, 16 * FT))), block(kWaves * kWave);
  const int64_t tiles = ceil_div(a.M, 16);
  if (tiles == 1) hipLaunchKernelGGL((mx_few_kernel<FT, 1>), grid, block, 0, st, a);
  else if (tiles == 2) hipLaunchKernelGGL((mx_few_kernel<FT, 2>), grid, block, 0, st, a);
  else if (tiles == 3) hipLaunchKernelGGL((mx_few_kernel<FT, 3>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((mx_few_kernel<FT, 4>), grid, block, 0, st, a);
  DLLAVA_CHECK_LAUNCH("mx_few_kernel");
  return DLLAVA_OK;
}

}  // namespace

int mx_linear_check(const char* who, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N, int act, const void* residual,
                    const void* y, int64_t ldy, int dtype) {
  DLLAVA_REQUIRE(dtype == DLLAVA_BF16, DLLAVA_EDTYPE, "%s: only DLLAVA_BF16 is supported (got dtype %d)", who, dtype);
  DLLAVA_REQUIRE(M >= 0 && M <= 0x7fffffffLL, DLLAVA_EINVAL, "%s: M = %lld", who, (long long)M);
  DLLAVA_REQUIRE(K > 0 && K % kMxBlock == 0 && K < (1 << 23), DLLAVA_ESHAPE, "%s: K must be a positive multiple of 32 below 2^23 (got %lld)", who,
                 (long long)K);
  DLLAVA_REQUIRE(N >= 0 && N % 8 == 0 && N <= 0x7fffffffLL - 512, DLLAVA_ESHAPE, "%s: N must be a multiple of 8 (got %lld)", who, (long long)N);
  DLLAVA_REQUIRE(act >= 0 && act <= 2, DLLAVA_EINVAL, "%s: act = %d", who, act);
  DLLAVA_REQUIRE(ldy >= N && ldy % 8 == 0, DLLAVA_EINVAL, "%s: ldy = %lld must be at least N and a multiple of 8", who, (long long)ldy);
  if (M == 0 || N == 0) return DLLAVA_OK;
  DLLAVA_REQUIRE(Wq && y, DLLAVA_ENULL, "%s: weights and y are required", who);
  DLLAVA_REQUIRE(act != 2 || residual, DLLAVA_ENULL, "%s: act 2 needs the gate", who);
  DLLAVA_REQUIRE(aligned(Wq, 256) && aligned(y, 16) && aligned(residual, 16) && aligned(bias, 16), DLLAVA_EINVAL,
                 "%s: weights must be 256-byte, y, residual and bias 16-byte aligned", who);
  DLLAVA_REQUIRE(Wq_bytes >= dllava_mx_bytes(N, K), DLLAVA_ECAPACITY, "%s: the packed weights are %zu bytes (got %zu)", who, dllava_mx_bytes(N, K),
                 Wq_bytes);
  return DLLAVA_OK;
}

MxLinearArgs mx_linear_args(int64_t M, int64_t K, const void* Wq, const float* bias, int64_t N, int act, const void* residual, void* y, int64_t ldy) {
  MxLinearArgs a{};
  a.Wc = static_cast<const uint8_t*>(Wq);
  a.Ws = a.Wc + mx_code_bytes(N, K);
  a.M = M, a.N = static_cast<int32_t>(N), a.K = static_cast<int32_t>(K);
  a.windows = static_cast<int32_t>(mx_padded(K) / kMxWindow);
  a.bias = bias, a.R = static_cast<const bf16_t*>(residual), a.Y = static_cast<bf16_t*>(y), a.ldy = ldy, a.act = act;
  return a;
}

}  // namespace dllava

using namespace dllava;

extern "C" int dllava_mx_linear_few(const void* x, int64_t ldx, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N,
                                    int act, const void* residual, void* y, int64_t ldy, int dtype, void* stream) {
  if (int rc = mx_linear_check("mx_linear_few", M, K, Wq, Wq_bytes, bias, N, act, residual, y, ldy, dtype)) return rc;
  DLLAVA_REQUIRE(M <= 64, DLLAVA_ESHAPE, "mx_linear_few: at most 64 rows (got %lld); dllava_mx_linear takes more", (long long)M);
  DLLAVA_REQUIRE(ldx >= K && ldx % 8 == 0, DLLAVA_EINVAL, "mx_linear_few: ldx = %lld must be at least K and a multiple of 8", (long long)ldx);
  if (M == 0 || N == 0) return DLLAVA_OK;
  DLLAVA_REQUIRE(x, DLLAVA_ENULL, "mx_linear_few: x is required");
  DLLAVA_REQUIRE(aligned(x, 16), DLLAVA_EINVAL, "mx_linear_few: x must be 16-byte aligned");
  MxLinearArgs a = mx_linear_args(M, K, Wq, bias, N, act, residual, y, ldy);
  a.X = static_cast<const bf16_t*>(x), a.ldx = ldx;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (N <= 16 * 512) return launch_rows<1>(a, st);
  return launch_rows<2>(a, st);
}
