// dllava_mx_linear_few: y = act(x W^T + bias) (+ | *) residual for the few rows of a decode step, weights in 4 bits.
//
// The weights' 17/32 byte an element are the traffic from memory, but every block reads all of x: beside the 98 KB of weights that a compute
// unit has of 4096 x 11008, 37 rows of x are 814 KB, from L2.  A block of eight waves takes 16 * FT features and all rows; its waves take
// windows of 512 columns in turn, add up their parts in registers and join them in LDS at the end, in the order of the waves: no block
// waits for another, and no workspace is needed.
//  * x goes to LDS by asynchronous loads of whole 128-byte lines, tiles of 64 columns, a ring of D of them for each wave alone (no
//    barriers).  (Straight to registers, in the layout of the products, the same bytes took twice as long: a load then touches parts of 32
//    lines; 37 rows x 4096 features x 11008 columns 32 us instead of 18.5.)
//  * A lane reads 16 bytes of codes, 32 elements of one feature, which become bfloat16 in registers (exact: two significant bits times a
//    power of two), operands of v_mfma_f32_16x16x32_bf16, whose columns are the rows of x.  A product takes eight columns of each of its
//    four lane groups, consecutive ones in LDS; the codes are exchanged between the groups to match, four swaps for 16 features x 128.
#include "gemm_ring.h"
#include "mx_linear.h"

namespace dllava {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;
constexpr int kTileCols = 64;  // of x in LDS: a memory line of each row

// A tile's operands from LDS: two of each 16 rows, 2 KB apart.  In asm since the compiler would wait for every asynchronous load first; the wait
// is part of it, so that no register is taken as read before it is.
template <int MT>
__device__ __forceinline__ void lds_read_tile(ring_u32x4 (&x)[MT][2], uint32_t at0, uint32_t at1) {
  if constexpr (MT == 1)
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x[0][0]), "=&v"(x[0][1]) : "v"(at0), "v"(at1) : "memory");
  if constexpr (MT == 2)
    asm volatile(
        "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:2048\n\tds_read_b128 %3, %5 offset:2048\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1])
        : "v"(at0), "v"(at1)
        : "memory");
  if constexpr (MT == 3)
    asm volatile(
        "ds_read_b128 %0, %6\n\tds_read_b128 %1, %7\n\tds_read_b128 %2, %6 offset:2048\n\tds_read_b128 %3, %7 offset:2048\n\t"
        "ds_read_b128 %4, %6 offset:4096\n\tds_read_b128 %5, %7 offset:4096\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1])
        : "v"(at0), "v"(at1)
        : "memory");
  if constexpr (MT == 4)
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %8 offset:2048\n\tds_read_b128 %3, %9 offset:2048\n\t"
        "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %9 offset:4096\n\tds_read_b128 %6, %8 offset:6144\n\t"
        "ds_read_b128 %7, %9 offset:6144\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[3][0]), "=&v"(x[3][1])
        : "v"(at0), "v"(at1)
        : "memory");
}

// FT tiles of 16 features, RG groups of eight rows (what a load of x covers).
template <int FT, int RG>
__global__ __launch_bounds__(kWaves* kWave) void mx_few_kernel(MxLinearArgs a) {
  constexpr int MT = (RG + 1) / 2;  // tiles of 16 rows (of an odd RG's last one the upper rows are whatever LDS holds: not used)
  constexpr int D = MT <= 2 ? 4 : (MT == 3 ? 3 : 2);
  constexpr bool kSlots = 8 % D == 0;  // a tile's slot follows from its number
  constexpr int kTileBytes = MT * 16 * kTileCols * 2, kWaveBytes = D * kTileBytes;
  constexpr int kSumBytes = kWaves * FT * MT * kWave * 16, kLds = kWaves * kWaveBytes > kSumBytes ? kWaves * kWaveBytes : kSumBytes;
  __shared__ __align__(1024) char smem_raw[kLds];
  DLLAVA_LDS char* smem = (DLLAVA_LDS char*)smem_raw;
  const int tid = threadIdx.x, lane = tid % kWave, g = lane / 16, r16 = lane % 16;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n0 = blockIdx.x * 16 * FT;
  const int64_t row_bytes = static_cast<int64_t>(a.windows) * (kMxWindow / 2);
  const uint8_t* wrow[FT];
  const uint8_t* srow[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) {
    const int n = n0 + 16 * f + r16 < a.N ? n0 + 16 * f + r16 : a.N - 1;  // features past N are computed and dropped
    const int tile = n0 + 16 * f < a.N ? n0 / 16 + f : (a.N - 1) / 16;
    wrow[f] = a.Wc + n * row_bytes + 16 * g;
    srow[f] = a.Ws + static_cast<int64_t>(tile) * a.windows * 256 + 4 * r16;
  }
  // x as a buffer: what is behind it -- rows past M, and by a lane's choice columns past K -- reads as zeros.  A load covers eight rows of a
  // tile; chunk c (of 8 columns) of row r lies at place c ^ ((r / 2) % 8) of the row.
  const uint32_t ldx = static_cast<uint32_t>(a.ldx) * 2;
  const auto X = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(a.X), 0, static_cast<uint32_t>(a.M - 1) * ldx + static_cast<uint32_t>(a.K) * 2, 0x00020000);
  const int dma_row = lane >> 3;
  uint32_t dma_at[RG];
  int dma_col[2];  // of rows 0..7 and 8..15 of every 16
#pragma unroll
  for (int i = 0; i < RG; ++i) {
    const int row = 8 * i + dma_row, chunk = (lane & 7) ^ ((row >> 1) & 7);
    dma_at[i] = row < a.M ? static_cast<uint32_t>(row) * ldx + 16 * chunk : 0x80000000u;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) dma_col[i] = 8 * ((lane & 7) ^ (((8 * i + dma_row) >> 1) & 7));
  const uint32_t ring = static_cast<uint32_t>(w) * kWaveBytes;
  auto request_x = [&](int col, int slot) __attribute__((always_inline)) {  // columns col .. col + 63
    const bool ragged = col + kTileCols > a.K;
#pragma unroll
    for (int i = 0; i < RG; ++i) {
      const uint32_t at = ragged && col + dma_col[i % 2] >= a.K ? 0x80000000u : dma_at[i];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(X, (DLLAVA_LDS void*)(smem + ring + slot * kTileBytes + i * 1024), 16, at, col < a.K ? 2 * col : 0, 0, 0);
    }
  };
  const uint32_t frag = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem)) + ring + r16 * 128;
  const uint32_t swizzle = (r16 >> 1) & 7;

  f32x4 acc[FT][MT];
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  // A window is four pieces of 128 columns, two tiles each; blocks begin at different pieces.  On their way: the codes of the next four
  // pieces, D - 1 tiles of x.
  const int turn = static_cast<int>(blockIdx.x);
  auto col_of = [&](int win, int tile) __attribute__((always_inline)) { return win * kMxWindow + 128 * ((tile / 2 + turn) % 4) + kTileCols * (tile % 2); };
  uint4 c[4][FT];
  uint32_t sc[FT][4], sc_next[FT][4];  // [i]: a byte for block i of each piece
  auto load_w = [&](int win, int j) __attribute__((always_inline)) {
#pragma unroll
    for (int f = 0; f < FT; ++f) c[j][f] = *reinterpret_cast<const uint4*>(wrow[f] + static_cast<int64_t>(win) * 256 + 64 * ((j + turn) % 4));
  };
  auto load_s = [&](int win) __attribute__((always_inline)) {
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc_next[f][i] = *reinterpret_cast<const uint32_t*>(srow[f] + static_cast<int64_t>(win) * 256 + 64 * i);
  };
  if (w < a.windows) {
    load_s(w);
#pragma unroll
    for (int j = 0; j < 4; ++j) load_w(w, j);
#pragma unroll
    for (int t = 0; t < D - 1; ++t) request_x(col_of(w, t), t);
  }
  int slot_now = 0;  // of the tile at hand, where it does not follow from the tile's number
  // One window; LAST: the wave's last one, behind which nothing is asked for.
  auto window = [&](int win, auto LAST) __attribute__((always_inline)) {
    constexpr bool kLast = decltype(LAST)::value;
    const int next = win + kWaves;
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[f][i] = sc_next[f][i];
    if constexpr (!kLast) load_s(next);
    uint32_t words[FT][4];
    static_for<8>([&](auto Tile) __attribute__((always_inline)) {
      constexpr int tile = decltype(Tile)::value, j = tile / 2, ahead = tile + D - 1;
      const int slot = kSlots ? tile % D : slot_now;
      if constexpr (!kLast || ahead < 8) request_x(col_of(ahead < 8 ? win : next, ahead % 8), slot == 0 ? D - 1 : slot - 1);
      if constexpr (tile % 2 == 0) {
#pragma unroll
        for (int f = 0; f < FT; ++f) {
          // word i of lane group g: columns 8i of block g -> word i: columns 8g of block i
          const auto p02 = __builtin_amdgcn_permlane32_swap(c[j][f].x, c[j][f].z, false, false);
          const auto p13 = __builtin_amdgcn_permlane32_swap(c[j][f].y, c[j][f].w, false, false);
          const auto p01 = __builtin_amdgcn_permlane16_swap(p02[0], p13[0], false, false);
          const auto p23 = __builtin_amdgcn_permlane16_swap(p02[1], p13[1], false, false);
          words[f][0] = p01[0], words[f][1] = p01[1], words[f][2] = p23[0], words[f][3] = p23[1];
        }
      }
      // this wave's loads of the tile have landed: RG loads of each of the tiles asked for behind it may be on their way (and whatever else was
      // requested since, which only makes the wait longer)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kLast && ahead >= 8 ? 7 - tile : D - 1) * RG) : "memory");
      ring_u32x4 x[MT][2];
      lds_read_tile<MT>(x, frag + slot * kTileBytes + (g ^ swizzle) * 16, frag + slot * kTileBytes + ((4 + g) ^ swizzle) * 16);
#pragma unroll
      for (int f = 0; f < FT; ++f) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t sb = sc[f][2 * (tile % 2) + i] >> (8 * ((j + turn) % 4)) << 23;
          const bf16x8 wv = __builtin_bit_cast(bf16x8, mx_decode8(words[f][2 * (tile % 2) + i], sb));
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, __builtin_bit_cast(bf16x8, x[t][i]), acc[f][t], 0, 0, 0);
        }
      }
      if constexpr (!kLast && tile % 2 == 1) load_w(next, j);
      if constexpr (!kSlots) slot_now = slot_now + 1 < D ? slot_now + 1 : 0;
    });
  };
  if (w < a.windows) {
    int win = w;
    for (; win + kWaves < a.windows; win += kWaves) window(win, std::false_type{});
    window(win, std::true_type{});
  }
  __syncthreads();  // the rings' memory takes the sums
  // register e of acc[f][t]: feature n0 + 16 f + 4 g + e, row 16 t + r16
  float4* const sm = reinterpret_cast<float4*>(smem_raw);  // [kWaves][FT * MT][kWave]
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int t = 0; t < MT; ++t) sm[(w * FT * MT + f * MT + t) * kWave + lane] = make_float4(acc[f][t][0], acc[f][t][1], acc[f][t][2], acc[f][t][3]);
  __syncthreads();
  for (int i = w; i < FT * MT; i += kWaves) {
    float4 v = sm[i * kWave + lane];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) {
      const float4 u = sm[(k * FT * MT + i) * kWave + lane];
      v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
    }
    const int n = n0 + 16 * (i / MT) + 4 * g;
    const int64_t m = 16 * (i % MT) + r16;
    if (n < a.N && m < a.M) mx_store_results(a, m, n, v);
  }
}

template <int FT, int RG>
int launch_few(const MxLinearArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((mx_few_kernel<FT, RG>), dim3(static_cast<unsigned>(ceil_div(a.N, 16 * FT))), dim3(kWaves * kWave), 0, st, a);
  DLLAVA_CHECK_LAUNCH("mx_few_kernel");
  return DLLAVA_OK;
}
template <int RG>
int launch_rows(const MxLinearArgs& a, int ft, hipStream_t st) {
  if (ft == 1) return launch_few<1, RG>(a, st);
  if (ft == 2) return launch_few<2, RG>(a, st);
  return launch_few<3, RG == 3 || RG == 4 ? 5 : RG>(a, st);  // (three and four groups: the registers do not suffice; rows past M cost nothing)
}

// Tiles of features per block: whole rounds of a block on each compute unit; a round takes, for every 512 columns of a wave, 0.7 us for eight rows
// and 1.7 for 16 features, and its start 0.8, of which little is seen where two blocks share a unit.  Measured, one tile / two / three, in us: rows x
// features x columns 1 x 11008 x 4096 9.4 / 9.9 / 9.1, 64 24.0 / 21.4 / 15.0; 1 x 13824 x 5120 13.8 / 13.4 / 19.1, 64 39.0 / 28.1 / 33.0; 1 x 4096 x 4096 4.7 /
// 5.8 / 7.2; 37 x 4096 x 11008 18.5 / 22.3 / 26.6; 1 x 32000 x 4096 20.9 / 18.1 / 22.9, 64 60.7 / 42.1 / 40.0.
int pick_features(const MxLinearArgs& a, int rg) {
  int best = 1;
  int64_t best_cost = 0;
  for (int ft = 1; ft <= 3; ++ft) {
    const int64_t rounds = ceil_div(ceil_div(a.N, 16 * ft), 256), start = ft <= 2 && rg <= 2 ? 800 : 6400;
    const int64_t cost = rounds * (start + a.windows * (700 * rg + 1700 * ft));
    if (ft == 1 || cost < best_cost) best = ft, best_cost = cost;
  }
  return best;
}

}  // namespace

int mx_linear_check(const char* who, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N, int act, const void* residual,
                    const void* y, int64_t ldy, int dtype) {
  DLLAVA_REQUIRE(dtype == DLLAVA_BF16, DLLAVA_EDTYPE, "%s: only DLLAVA_BF16 is supported (got dtype %d)", who, dtype);
  DLLAVA_REQUIRE(M >= 0 && M <= 0x7fffffffLL, DLLAVA_EINVAL, "%s: M = %lld", who, (long long)M);
  DLLAVA_REQUIRE(K > 0 && K % kMxBlock == 0 && K < (1 << 23), DLLAVA_ESHAPE, "%s: K must be a positive multiple of 32 below 2^23 (got %lld)", who,
                 (long long)K);
  DLLAVA_REQUIRE(N >= 0 && N % 8 == 0 && N < (1 << 27), DLLAVA_ESHAPE, "%s: N must be a multiple of 8 below 2^27 (got %lld)", who, (long long)N);
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
  // (64 rows of x are addressed by 31-bit offsets)
  DLLAVA_REQUIRE(ldx < (int64_t{1} << 24), DLLAVA_ESHAPE, "mx_linear_few: ldx = %lld must be below 2^24", (long long)ldx);
  if (M == 0 || N == 0) return DLLAVA_OK;
  DLLAVA_REQUIRE(x, DLLAVA_ENULL, "mx_linear_few: x is required");
  DLLAVA_REQUIRE(aligned(x, 16), DLLAVA_EINVAL, "mx_linear_few: x must be 16-byte aligned");
  MxLinearArgs a = mx_linear_args(M, K, Wq, bias, N, act, residual, y, ldy);
  a.X = static_cast<const bf16_t*>(x), a.ldx = ldx;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int rg = static_cast<int>(ceil_div(M, 8)), forced = launch_override(DLLAVA_LAUNCH_LINEAR_TILE);
  const int ft = forced >= 1 && forced <= 3 ? forced : pick_features(a, rg);
  switch (rg) {
    case 1: return launch_rows<1>(a, ft, st);
    case 2: return launch_rows<2>(a, ft, st);
    case 3: return launch_rows<3>(a, ft, st);
    case 4: return launch_rows<4>(a, ft, st);
    case 5: return launch_rows<5>(a, ft, st);
    case 6: return launch_rows<6>(a, ft, st);
    case 7: return launch_rows<7>(a, ft, st);
    default: return launch_rows<8>(a, ft, st);
  }
}
