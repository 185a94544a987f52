// dllava_mx_linear: y = act(x W^T + bias) (+ | *) residual, rows and weights in 4 bits, on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// A lane's operand is the 32 elements of one scale (16 bytes), and its scale one byte of a register: four consecutive products of a
// wave take the four bytes of the scales that lie together (see the packed form in dllava_mx.h).
#include "mx_linear.h"
#include "mx_ring.h"

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

// A tile of 32*FI features x 32*JT rows on the ring of mx_ring.h, PER_CU blocks per compute unit.
template <int FI, int JT, int PER_CU>
__global__ __launch_bounds__(kRingThreads, PER_CU) void mx_ring_kernel(MxLinearArgs a, int n_ft, int n_rt, int per_xcd) {
  constexpr int kTok = 32 * JT, kFeat = 32 * FI, kChunks = kFeat / 8;
  __shared__ __align__(1024) char smem_raw[5 * kFeat * kRingRowBytes];
  static_assert(kTok * kFeat * 2 <= 5 * kFeat * kRingRowBytes, "the output tile takes the ring's place");
  DLLAVA_LDS char* smem = (DLLAVA_LDS char*)smem_raw;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  int ft, rt;
  if (!ring_tile(n_ft, n_rt, per_xcd, ft, rt)) return;
  const int N = a.N;
  const int64_t M = a.M, row_bytes = static_cast<int64_t>(a.windows) * (kMxWindow / 2), tile_bytes = static_cast<int64_t>(a.windows) * 256;
  uint32_t ga[FI], gb[JT], sa[FI], sb[JT];
  // features and rows past the end are computed from the last one, and dropped
#pragma unroll
  for (int j = 0; j < FI; ++j) {
    const int row = ring_load_row(w, j, lane), u = ft * kFeat + row < N ? row : N - 1 - ft * kFeat;
    ga[j] = static_cast<uint32_t>(u) * static_cast<uint32_t>(row_bytes) + ring_load_chunk_bytes(row, lane);
    const int last = (N - 1) / 16 - ft * (kFeat / 16), t = FI * (w >> 1) + j;
    sa[j] = static_cast<uint32_t>(t < last ? t : last) * static_cast<uint32_t>(tile_bytes);
  }
#pragma unroll
  for (int j = 0; j < JT; ++j) {
    const int64_t left = M - 1 - static_cast<int64_t>(rt) * kTok;
    const int row = ring_load_row(w, j, lane), u = row < left ? row : static_cast<int>(left);
    gb[j] = static_cast<uint32_t>(u) * static_cast<uint32_t>(row_bytes) + ring_load_chunk_bytes(row, lane);
    const int64_t last = (M - 1) / 16 - static_cast<int64_t>(rt) * (kTok / 16);
    const int t = JT * (w & 1) + j;
    sb[j] = static_cast<uint32_t>(t < last ? t : static_cast<int>(last)) * static_cast<uint32_t>(tile_bytes);
  }
  ring_f32x4 acc[FI][JT];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < JT; ++j) acc[i][j] = ring_f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t n0 = static_cast<int64_t>(ft) * kFeat, m0 = static_cast<int64_t>(rt) * kTok;
  const int64_t n_tiles = (N + 15) / 16 - n0 / 16, m_tiles = (M + 15) / 16 - m0 / 16;
  mx_ring_halves<FI, JT>(mx_make_buffer(a.Wc + n0 * row_bytes, (N - n0) * row_bytes), ga, mx_make_buffer(a.Xc + m0 * row_bytes, (M - m0) * row_bytes), gb,
                         mx_make_buffer(a.Ws + n0 / 16 * tile_bytes, n_tiles * tile_bytes), sa,
                         mx_make_buffer(a.Xs + m0 / 16 * tile_bytes, m_tiles * tile_bytes), sb, a.windows, smem, w, acc);
  __syncthreads();  // the ring memory becomes the transposed output tile

  // lane: row 16*JT*(w%2) + 16*j + lane%16; register r of acc[i]: feature 16*FI*(w/2) + 16*i + 4*(lane/16) + r
  constexpr int kMask = kChunks < 16 ? kChunks - 1 : 15;
  const int g = lane >> 4;
  bf16_t* sO = reinterpret_cast<bf16_t*>(smem_raw);  // [kTok rows][chunks of 8 features], chunk c of row t at c ^ (t & kMask)
  const int f_lane = ft * kFeat + 16 * FI * (w >> 1) + 4 * g;
  float4 bs[FI];
#pragma unroll
  for (int i = 0; i < FI; ++i)
    bs[i] = a.bias && f_lane + 16 * i < N ? *reinterpret_cast<const float4*>(a.bias + f_lane + 16 * i) : make_float4(0.f, 0.f, 0.f, 0.f);
  uint2 rr[JT][FI];
  if (a.R) {  // all requested at once, into the registers that the fragments have left
#pragma unroll
    for (int j = 0; j < JT; ++j) {
      int64_t m = static_cast<int64_t>(rt) * kTok + 16 * JT * (w & 1) + 16 * j + (lane & 15);
      if (m >= M) m = M - 1;
      const bf16_t* rrow = a.R + m * a.ldy;
#pragma unroll
      for (int i = 0; i < FI; ++i) rr[j][i] = *reinterpret_cast<const uint2*>(rrow + (f_lane + 16 * i < N ? f_lane + 16 * i : ft * kFeat));
    }
  }
#pragma unroll
  for (int j = 0; j < JT; ++j) {
    const int t = 16 * JT * (w & 1) + 16 * j + (lane & 15);
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      float4 v = make_float4(acc[i][j][0] + bs[i].x, acc[i][j][1] + bs[i].y, acc[i][j][2] + bs[i].z, acc[i][j][3] + bs[i].w);
      const uint2 o = mx_result(a, v, rr[j][i]);
      const int c = 2 * FI * (w >> 1) + 2 * i + (g >> 1);  // chunk of 8 features; this lane's half of it: g % 2
      *reinterpret_cast<uint2*>(sO + t * kFeat + ((c ^ (t & kMask)) * 8) + (g & 1) * 4) = o;
    }
    __builtin_amdgcn_sched_barrier(0);  // one column at a time: the accumulators leave no registers for more
  }
  __syncthreads();
  constexpr int kStep = kRingThreads / kChunks;  // thread: one chunk of every kStep-th row
  const int c = tid % kChunks, f = ft * kFeat + c * 8;
  if (f >= N) return;
#pragma unroll 4
  for (int k = 0; k < kTok / kStep; ++k) {
    const int t = tid / kChunks + kStep * k;
    const int64_t m = static_cast<int64_t>(rt) * kTok + t;
    const uint4 piece = *reinterpret_cast<const uint4*>(sO + t * kFeat + ((c ^ (t & kMask)) * 8));
    if (m < M) *reinterpret_cast<uint4*>(a.Y + m * a.ldy + f) = piece;
  }
}

template <int FI, int JT, int PER_CU>
int launch_ring(const MxLinearArgs& a, hipStream_t st) {
  const int64_t n_ft = ceil_div(a.N, 32 * FI), n_rt = ceil_div(a.M, 32 * JT), per_xcd = ceil_div(n_ft * n_rt, kRingXcds);
  DLLAVA_REQUIRE(per_xcd * kRingXcds <= 0x7fffffffLL, DLLAVA_ESHAPE, "mx_linear: too many results");
  hipLaunchKernelGGL((mx_ring_kernel<FI, JT, PER_CU>), dim3(static_cast<unsigned>(per_xcd * kRingXcds)), dim3(kRingThreads), 0, st, a,
                     static_cast<int>(n_ft), static_cast<int>(n_rt), static_cast<int>(per_xcd));
  DLLAVA_CHECK_LAUNCH("mx_ring_kernel");
  return DLLAVA_OK;
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
  switch (launch_override(DLLAVA_LAUNCH_LINEAR_TILE)) {
    case 8: return launch_ring<8, 8, 1>(a, static_cast<hipStream_t>(stream));
    case 7: return launch_ring<8, 7, 1>(a, static_cast<hipStream_t>(stream));
    case 6: return launch_ring<8, 6, 1>(a, static_cast<hipStream_t>(stream));
    case 4: return launch_ring<8, 4, 1>(a, static_cast<hipStream_t>(stream));
    case 12: return launch_ring<4, 4, 2>(a, static_cast<hipStream_t>(stream));
    default: break;
  }
  const int64_t n_ft = ceil_div(N, 64), blocks = n_ft * ceil_div(M, 64);
  DLLAVA_REQUIRE(blocks <= 0x7fffffffLL, DLLAVA_ESHAPE, "mx_linear: too many results");
  hipLaunchKernelGGL(mx_linear_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, static_cast<hipStream_t>(stream), a, static_cast<int>(n_ft));
  DLLAVA_CHECK_LAUNCH("mx_linear_kernel");
  return DLLAVA_OK;
}
