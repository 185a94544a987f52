// dllava_mx_linear: y = act(x W^T + bias) (+ | *) residual, rows and weights in 4 bits, on v_mfma_scale_f32_16x16x128_f8f6f4.
//
// A lane's operand is the 32 elements of one scale (16 bytes), and its scale one byte of a register: four consecutive products of a
// wave take the four bytes of the scales that lie together (see the packed form in dllava_mx.h).  The products' rate is four times that
// of bfloat16, so nearly everything else bounds them: 16384 x 8192 x 8192 takes 487 us (4.5 PFLOP/s), where a stage of 256 x 256 x 256 takes 1.43 us
// with random values, 1.12 with zeros (the clock gives way to the power) and 0.85 by the products' own rate; at 4096 columns a
// tile's ends and the last round of tiles count, and what the results take to memory: 5003 x 11008 x 4096 115 us (3.9 PFLOP/s), 135 with a gate that is
// read (110 MB, as many as are written), 136 with GELU.
#include "mx_linear.h"
#include "mx_ring.h"

namespace dllava {

int mx_linear_check(const char* who, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N, int act, const void* residual,
                    const void* y, int64_t ldy, int dtype);  // mx_few.hip
MxLinearArgs mx_linear_args(int64_t M, int64_t K, const void* Wq, const float* bias, int64_t N, int act, const void* residual, void* y, int64_t ldy);

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x8 operand(const uint4& c) {
  return i32x8{static_cast<int>(c.x), static_cast<int>(c.y), static_cast<int>(c.z), static_cast<int>(c.w), 0, 0, 0, 0};
}

// Where tile number `local` of an XCD lies: tiles are numbered in groups of kRingGroup row tiles, inside a group feature tile by
// feature tile, and an XCD takes an eighth of that order (see ring_tile).  False: there is none.
struct MxTiles {
  int n_ft, n_rt, per_xcd;
};
__device__ __forceinline__ bool find_tile(const MxTiles& t, int local, int& ft, int& rt) {
  const int64_t idx = static_cast<int64_t>(blockIdx.x % kRingXcds) * t.per_xcd + local;
  if (local >= t.per_xcd || idx >= static_cast<int64_t>(t.n_ft) * t.n_rt) return false;
  const int per_group = kRingGroup * t.n_ft;
  const int group = static_cast<int>(idx / per_group), in_group = static_cast<int>(idx % per_group);
  const int left = t.n_rt - group * kRingGroup, here = left < kRingGroup ? left : kRingGroup;
  ft = in_group / here;
  rt = group * kRingGroup + in_group % here;
  return true;
}

// What becomes of the sums (their bias is in them from the start).
enum Epilogue { kPlain, kAdd, kGelu, kGate };

__device__ __forceinline__ float silu_fast(float x) { return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * x)); }

// Tiles of 32*FI features x 32*JT rows, PER_CU blocks per compute unit, each several tiles (mx_ring.h).
template <int FI, int JT, int PER_CU, Epilogue E>
__global__ __launch_bounds__(kRingThreads, PER_CU) void mx_ring_kernel(MxLinearArgs a, MxTiles tiles) {
  constexpr int kTok = 32 * JT, kFeat = 32 * FI;
  __shared__ __align__(1024) char smem_raw[5 * kFeat * kRingRowBytes];
  DLLAVA_LDS char* smem = (DLLAVA_LDS char*)smem_raw;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), g = lane >> 4, r16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int step = static_cast<int>(gridDim.x) / kRingXcds;
  int local = static_cast<int>(blockIdx.x) / kRingXcds, ft, rt;
  if (!find_tile(tiles, local, ft, rt)) return;
  const int64_t row_bytes = static_cast<int64_t>(a.windows) * (kMxWindow / 2), tile_bytes = static_cast<int64_t>(a.windows) * 256;
  uint32_t ga[FI], gb[JT];
#pragma unroll
  for (int j = 0; j < FI; ++j) {
    const int row = ring_load_row(w, j, lane);
    ga[j] = static_cast<uint32_t>(row) * static_cast<uint32_t>(row_bytes) + ring_load_chunk_bytes(row, lane);
  }
#pragma unroll
  for (int j = 0; j < JT; ++j) {
    const int row = ring_load_row(w, j, lane);
    gb[j] = static_cast<uint32_t>(row) * static_cast<uint32_t>(row_bytes) + ring_load_chunk_bytes(row, lane);
  }
  auto buffers = [&](int f, int r) DLLAVA_INLINE {
    const int64_t n0 = static_cast<int64_t>(f) * kFeat, m0 = static_cast<int64_t>(r) * kTok;
    return MxTileBuffers{mx_make_buffer(a.Wc + n0 * row_bytes, (a.N - n0) * row_bytes), mx_make_buffer(a.Xc + m0 * row_bytes, (a.M - m0) * row_bytes),
                         mx_make_buffer(a.Ws + n0 / 16 * tile_bytes, ((a.N + 15) / 16 - n0 / 16) * tile_bytes),
                         mx_make_buffer(a.Xs + m0 / 16 * tile_bytes, ((a.M + 15) / 16 - m0 / 16) * tile_bytes)};
  };
  ring_f32x4 acc[FI][JT];
  int ft_next = ft, rt_next = rt;
  bool more = false;
  const bool has_r = E == kAdd || E == kGate || (E == kGelu && a.R != nullptr);
  // Register e of acc[i][j]: feature 16 i + 4 g + e of the wave's, row 16 j + r16.  For accesses of 16 bytes fragments 2p and 2p + 1 trade
  // rows of lanes: a lane then has eight consecutive features of one of them (n_out + 32 p of the tile), four lanes 64 bytes of a row.
  const int n_lane = 16 * FI * (w >> 1) + 4 * g, n_out = 16 * FI * (w >> 1) + 16 * (g & 1) + 8 * (g >> 1);
  const uint32_t ld = static_cast<uint32_t>(a.ldy) * 2, lane_at = static_cast<uint32_t>(16 * JT * (w & 1) + r16) * ld + 2 * static_cast<uint32_t>(n_out);
  // R's lines of a tile are asked for while its last products run, a line a lane every other stage, so that they are in the caches at its end:
  // all tiles end at about the same time.  5003 rows x 4096 features x 4096 columns with a residual 60.2 -> 57.1 us, 16384 x 11008 x 4096 444 -> 435;
  // with a gate 5003 x 11008 x 4096 140.3 -> 138.5.  (Every stage of the last ones: slower than without.  Tiles of 128 rows lose 1 %.)
  constexpr bool kAhead = (E == kAdd || E == kGate) && JT >= 6;
  constexpr int kLines = FI / 2, kTouches = (kTok * kLines + kRingThreads - 1) / kRingThreads;
  const uint32_t touch_at = static_cast<uint32_t>(tid / kLines) * ld + 128 * (tid % kLines);
  uint32_t touched = 0, touch = 0;
  mx_buffer R = mx_make_buffer(a.R, 0);
  mx_ring_stream<FI, JT>(
      buffers(ft, rt), ga, gb, a.windows, smem, w, acc,
      [&]() DLLAVA_INLINE {
        ft = ft_next, rt = rt_next;
        local += step;
        more = find_tile(tiles, local, ft_next, rt_next);
        if constexpr (kAhead) {
          const int64_t m0 = static_cast<int64_t>(rt) * kTok, c0 = static_cast<int64_t>(ft) * kFeat, rows = a.M - m0 < kTok ? a.M - m0 : kTok;
          R = mx_make_buffer(a.R + m0 * a.ldy + c0, (rows - 1) * static_cast<int64_t>(ld) + 2 * (a.N - c0));
          touch = c0 + 64 * (tid % kLines) < a.N ? touch_at : 0x80000000u;
        }
        const int64_t n0 = static_cast<int64_t>(ft) * kFeat + n_lane;
        static_for<FI>([&](auto I) DLLAVA_INLINE {
          if (a.bias) {
            const float4 b = n0 + 16 * I.value < a.N ? *reinterpret_cast<const float4*>(a.bias + n0 + 16 * I.value) : make_float4(0.f, 0.f, 0.f, 0.f);
            static_for<JT>([&](auto J) DLLAVA_INLINE { mx_start(acc[I.value][J.value], b); });
          } else {
            static_for<JT>([&](auto J) DLLAVA_INLINE { mx_start(acc[I.value][J.value]); });
          }
        });
        return buffers(ft_next, rt_next);  // (the tile's own where there is no other: find_tile then leaves the numbers alone)
      },
      [&](int left) DLLAVA_INLINE {
        if constexpr (kAhead) {
          if (left <= kTouches) {
            asm volatile("" ::"v"(touched));
            touched = __builtin_amdgcn_raw_buffer_load_b32(R, touch, static_cast<uint32_t>(kTouches - left) * (kRingThreads / kLines) * ld, 0);
          }
        }
      },
      [&]() DLLAVA_INLINE {
        const int64_t n0 = static_cast<int64_t>(ft) * kFeat, m0 = static_cast<int64_t>(rt) * kTok, rows = a.M - m0 < kTok ? a.M - m0 : kTok;
        const int64_t bytes = (rows - 1) * static_cast<int64_t>(ld) + 2 * (a.N - n0);  // behind the last row's end nothing is read or written
        const mx_buffer Y = mx_make_buffer(a.Y + m0 * a.ldy + n0, bytes);
        if constexpr (!kAhead) R = mx_make_buffer(a.R + m0 * a.ldy + n0, bytes);
        uint32_t off[FI / 2];
#pragma unroll
        for (int p = 0; p < FI / 2; ++p) off[p] = n0 + n_out + 32 * p < a.N ? lane_at + 64 * p : 0x80000000u;  // features past N: out of range
        constexpr int kDeep = FI == 8 ? 3 : 2;  // columns whose R is on its way
        u32x4 r[kDeep][FI / 2];
        auto load_r = [&](auto J) DLLAVA_INLINE {
          constexpr int j = decltype(J)::value;
#pragma unroll
          for (int p = 0; p < FI / 2; ++p) r[j % kDeep][p] = __builtin_amdgcn_raw_buffer_load_b128(R, off[p], 16 * j * ld, 0);
        };
        if (has_r) static_for<(kDeep < JT ? kDeep : JT)>(load_r);
        if constexpr (kAhead) asm volatile("" ::"v"(touched));
        static_for<JT>([&](auto J) DLLAVA_INLINE {
          constexpr int j = decltype(J)::value;
          u32x4 out[FI / 2];
          static_for<FI / 2>([&](auto Pi) DLLAVA_INLINE {
            constexpr int p = decltype(Pi)::value;
            float x[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = acc[2 * p][j][e], x[4 + e] = acc[2 * p + 1][j][e];
            if constexpr (E == kGelu) {
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = gelu_erf_fast(x[e]);
            }
            if (has_r) {
              const u32x4 q = r[j % kDeep][p];
              const auto s0 = __builtin_amdgcn_permlane16_swap(q[0], q[2], false, false), s1 = __builtin_amdgcn_permlane16_swap(q[1], q[3], false, false);
              const float v[8] = {bf16lo_to_f32(s0[0]), bf16hi_to_f32(s0[0]), bf16lo_to_f32(s1[0]), bf16hi_to_f32(s1[0]),
                                  bf16lo_to_f32(s0[1]), bf16hi_to_f32(s0[1]), bf16lo_to_f32(s1[1]), bf16hi_to_f32(s1[1])};
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = E == kGate ? x[e] * silu_fast(v[e]) : x[e] + v[e];
            }
            const auto s0 = __builtin_amdgcn_permlane16_swap(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[4], x[5]), false, false);
            const auto s1 = __builtin_amdgcn_permlane16_swap(pack_bf16x2(x[2], x[3]), pack_bf16x2(x[6], x[7]), false, false);
            out[p] = u32x4{s0[0], s1[0], s0[1], s1[1]};
          });
          if constexpr (j + kDeep < JT)
            if (has_r) load_r(std::integral_constant<int, (j + kDeep < JT ? j + kDeep : j)>{});
#pragma unroll
          for (int p = 0; p < FI / 2; ++p) __builtin_amdgcn_raw_buffer_store_b128(out[p], Y, off[p], 16 * j * ld, 0);
          __builtin_amdgcn_sched_barrier(0);  // one column at a time: the accumulators leave no registers for more
        });
        return more;
      });
}

template <int FI, int JT, int PER_CU, Epilogue E>
int launch_ring_as(const MxLinearArgs& a, hipStream_t st) {
  const int64_t n_ft = ceil_div(a.N, 32 * FI), n_rt = ceil_div(a.M, 32 * JT), per_xcd = ceil_div(n_ft * n_rt, kRingXcds);
  DLLAVA_REQUIRE(per_xcd <= 0x7fffffffLL - 64 && n_rt <= 0x7fffffffLL, DLLAVA_ESHAPE, "mx_linear: too many results");
  const int64_t at_once = 32 * PER_CU, blocks = per_xcd < at_once ? per_xcd : at_once;
  hipLaunchKernelGGL((mx_ring_kernel<FI, JT, PER_CU, E>), dim3(static_cast<unsigned>(blocks * kRingXcds)), dim3(kRingThreads), 0, st, a,
                     MxTiles{static_cast<int>(n_ft), static_cast<int>(n_rt), static_cast<int>(per_xcd)});
  DLLAVA_CHECK_LAUNCH("mx_ring_kernel");
  return DLLAVA_OK;
}
template <int FI, int JT, int PER_CU>
int launch_ring(const MxLinearArgs& a, hipStream_t st) {
  if (a.act == 1) return launch_ring_as<FI, JT, PER_CU, kGelu>(a, st);
  if (a.act == 2) return launch_ring_as<FI, JT, PER_CU, kGate>(a, st);
  return a.R ? launch_ring_as<FI, JT, PER_CU, kAdd>(a, st) : launch_ring_as<FI, JT, PER_CU, kPlain>(a, st);
}

// Tiles of 16*FT features x 16*RT rows for launches whose large tiles would leave most of the chip idle: a block of eight waves shares out
// the pieces of 256 columns, every wave the whole tile, operands straight from memory (no two waves read the same bytes), and the waves'
// sums are joined in LDS, in their order.
constexpr int kSplitWaves = 8;
template <int FT, int RT>
__global__ __launch_bounds__(kSplitWaves* kWave) void mx_split_kernel(MxLinearArgs a, int n_ft) {
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, g = lane / 16, r16 = lane % 16;
  const int n0 = static_cast<int>(blockIdx.x % n_ft) * 16 * FT;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / n_ft) * 16 * RT;
  const int64_t row_bytes = static_cast<int64_t>(a.windows) * (kMxWindow / 2);
  const uint8_t *code[FT + RT], *scale[FT + RT];  // features and rows past the end are computed from the last one, and dropped
#pragma unroll
  for (int i = 0; i < FT; ++i) {
    const int n = n0 + 16 * i + r16 < a.N ? n0 + 16 * i + r16 : a.N - 1, t = n0 + 16 * i < a.N ? n0 / 16 + i : (a.N - 1) / 16;
    code[i] = a.Wc + n * row_bytes + 16 * g;
    scale[i] = a.Ws + static_cast<int64_t>(t) * a.windows * 256 + 4 * lane;
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t m = m0 + 16 * i + r16 < a.M ? m0 + 16 * i + r16 : a.M - 1, t = m0 + 16 * i < a.M ? m0 / 16 + i : (a.M - 1) / 16;
    code[FT + i] = a.Xc + m * row_bytes + 16 * g;
    scale[FT + i] = a.Xs + t * a.windows * 256 + 4 * lane;
  }
  struct Piece {  // 256 columns: a memory line of every row
    uint4 c[FT + RT][2];
    uint32_t s[FT + RT];
  };
  auto load = [&](Piece& p, int piece) {
#pragma unroll
    for (int i = 0; i < FT + RT; ++i) {
      p.c[i][0] = *reinterpret_cast<const uint4*>(code[i] + static_cast<int64_t>(piece) * 128);
      p.c[i][1] = *reinterpret_cast<const uint4*>(code[i] + static_cast<int64_t>(piece) * 128 + 64);
      p.s[i] = *reinterpret_cast<const uint16_t*>(scale[i] + static_cast<int64_t>(piece / 2) * 256 + piece % 2 * 2);
    }
  };
  f32x4 acc[FT][RT];
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int pieces = (a.K + 255) / 256;
  Piece p, next;
  if (w < pieces) load(p, w);
  for (int piece = w; piece < pieces; piece += kSplitWaves) {
    if (piece + kSplitWaves < pieces) load(next, piece + kSplitWaves);
#pragma unroll
    for (int i = 0; i < FT; ++i)
#pragma unroll
      for (int j = 0; j < RT; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(p.c[i][0]), operand(p.c[FT + j][0]), acc[i][j], 4, 4, 0,
                                                                     static_cast<int>(p.s[i]), 0, static_cast<int>(p.s[FT + j]));
#pragma unroll
    for (int i = 0; i < FT; ++i)
#pragma unroll
      for (int j = 0; j < RT; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(p.c[i][1]), operand(p.c[FT + j][1]), acc[i][j], 4, 4, 1,
                                                                     static_cast<int>(p.s[i]), 1, static_cast<int>(p.s[FT + j]));
    p = next;
  }
  __shared__ float4 sm[kSplitWaves][FT * RT][kWave];
#pragma unroll
  for (int i = 0; i < FT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) sm[w][i * RT + j][lane] = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
  __syncthreads();
#pragma unroll
  for (int i = w; i < FT * RT; i += kSplitWaves) {
    float4 v = sm[0][i][lane];
#pragma unroll
    for (int k = 1; k < kSplitWaves; ++k) {
      const float4 u = sm[k][i][lane];
      v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
    }
    const int n = n0 + 16 * (i / RT) + 4 * g;
    const int64_t m = m0 + 16 * (i % RT) + r16;
    if (n < a.N && m < a.M) mx_store_results(a, m, n, v);
  }
}

template <int FT, int RT>
int launch_split(const MxLinearArgs& a, hipStream_t st) {
  const int64_t n_ft = ceil_div(a.N, 16 * FT), blocks = n_ft * ceil_div(a.M, 16 * RT);
  DLLAVA_REQUIRE(blocks < (1 << 23), DLLAVA_ESHAPE, "mx_linear: too many results for rows of y that far apart");
  hipLaunchKernelGGL((mx_split_kernel<FT, RT>), dim3(static_cast<unsigned>(blocks)), dim3(kSplitWaves * kWave), 0, st, a, static_cast<int>(n_ft));
  DLLAVA_CHECK_LAUNCH("mx_split_kernel");
  return DLLAVA_OK;
}

// The tiles of the ring, in nanoseconds: a stage when every compute unit works (and the clock gives way to the power) and when few do, and
// what a tile takes beside its stages.  Measured with random values at 4096 and 8192 columns, 8 rounds of tiles on every compute unit.
// Of the 128 x 128 tile two blocks share a compute unit: busy is a round of both.
struct MxRingTile {
  int id;  // what the launch override takes
  int fi, jt, per_cu;
  int64_t busy, alone, ends;
};
constexpr MxRingTile kMxTiles[] = {{8, 8, 8, 1, 1430, 1120, 9000}, {7, 8, 7, 1, 1350, 1060, 5000}, {6, 8, 6, 1, 1200, 920, 4000},
                                   {4, 8, 4, 1, 900, 710, 3000},   {12, 4, 4, 2, 1010, 410, 2000}};
constexpr int kMxSplit = 2;  // the override's value for mx_split_kernel

// The tile that takes least: whole rounds of tiles on all compute units, then the rest, whose stages are shorter the fewer there are; a GELU
// is 20 ns for each of a lane's results.  Predicted / measured in us: 5003 rows x 11008 features x 4096 columns, 256 x 224 111 / 116,
// 256 x 192 119 / 120, 256 x 256 130 / 125, 256 x 128 126 / 128, 128 x 128 136 / 129; 5003 x 4096 x 11008 126 / 122, 115 / 111, 136 / 135, 129 / 124,
// 121 / 120; 2000 x 4096 x 4096 26.9 / 28.5, 23.7 / 26.1, 31.9 / 31.9, 22.4 / 22.6, 23.2 / 22.8.
int pick_tile(const MxLinearArgs& a) {
  const int64_t nk = 2 * a.windows;
  int best = 0;
  int64_t best_cost = 0;
  for (const MxRingTile& t : kMxTiles) {
    const int64_t tiles = ceil_div(a.N, 32 * t.fi) * ceil_div(a.M, 32 * t.jt), at_once = 256 * t.per_cu, full = tiles / at_once, rest = tiles % at_once;
    const int64_t ends = t.ends + (a.act == 1 ? 20 * 4 * t.fi * t.jt : 0);
    int64_t cost = full * (nk * t.busy + ends);
    if (rest) cost += nk * (t.alone + (t.busy - t.alone) * rest / at_once) + ends;
    if (!best || cost < best_cost) best = t.id, best_cost = cost;
  }
  return best;
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
  hipStream_t st = static_cast<hipStream_t>(stream);
  // Few results: 64 x 32 tiles, as long as each compute unit has one at most (203 rows x 520 features x 1376 columns 5.5 us, 128 x 128 tiles
  // 8.9; 70 x 1024 x 4096 9.0 / 10.5; 100 x 4096 x 4096 9.2 / 10.8; 66 x 4096 x 11008 19.2 / 21.7; past that line, 200 x 4096 x 4096, 17.3 / 11.1).
  // They also take rows of y so far apart that a tile's would not fit the 31 bits of a buffer's offsets.
  int tile = launch_override(DLLAVA_LAUNCH_LINEAR_TILE);
  const bool known = tile == 8 || tile == 7 || tile == 6 || tile == 4 || tile == 12 || tile == kMxSplit;
  if (!known) tile = ceil_div(N, 64) * ceil_div(M, 32) <= 256 ? kMxSplit : pick_tile(a);
  if (ldy >= (int64_t{1} << 21)) tile = kMxSplit;
  switch (tile) {
    case kMxSplit: return launch_split<4, 2>(a, st);
    case 12: return launch_ring<4, 4, 2>(a, st);
    case 4: return launch_ring<8, 4, 1>(a, st);
    case 6: return launch_ring<8, 6, 1>(a, st);
    case 7: return launch_ring<8, 7, 1>(a, st);
    default: return launch_ring<8, 8, 1>(a, st);
  }
}
