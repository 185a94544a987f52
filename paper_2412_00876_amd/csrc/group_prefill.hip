// dllava_group_prefill_attn: causal attention of packed prompts (Eq. 1 of the paper), several query heads to a head of K and V, rows
// of any stride.
//
// bfloat16: the matrix-core kernel of attn_tiles.h.  What it takes per item (one query head, NWQ * 32 query rows) does not depend on
// whose keys it reads; the query heads of a group run on one die at about the same time (where eight divides their number), so that
// their K/V tiles come from its cache.  The probabilities are rounded to bfloat16 (nearest) for the second product, as those of the decode steps over the cache in
// 4 bits are; their sum is taken before.  Bound by the matrix cores: 4 x 3000 rows, 32 query heads of 128 over 8, 314 us, 940 TFLOP/s.
// float32: the wave-level streaming attention of attend.h, one wave per row and query head.
#include "attend.h"
#include "attn_tiles.h"

namespace dllava {
namespace {

template <int DH, int NWQ>
__global__ __launch_bounds__(NWQ * kWave, NWQ < 4 ? 1 : 2) void group_tiles_kernel(PrefillArgs args) {
  attend_items<DH, NWQ, Mode::Group>(args);
}

template <int DH, int NWQ>
int launch(const PrefillArgs& a, int64_t rows, hipStream_t st) {
  static std::atomic<int64_t> blocks{0};
  if (a.B > kWave && (ceil_div(rows, NWQ * 32) + a.B) * a.H * (NWQ * kWave) > 0xffffffffLL) return 1;  // (a block to an item: threads of a launch)
  return launch_items(group_tiles_kernel<DH, NWQ>, NWQ, blocks, "group_tiles_kernel", a, rows, st);
}

// Waves of an item, 32 query rows each: four, but two for short sequences as long as there are not many, whose items then start sooner and
// spread further.  Two / four waves in us, 32 heads of 128 over 8: 4 x 128 rows 8.2 / 8.9, 8 x 128 9.1 / 9.8, 4 x 256 11.5 / 11.7, 1 x 500 15.7 / 16.3, 2 x 500 16.6 / 16.4,
// 16 x 300 of 32 heads 50.5 / 42.3; 14 heads of 64 over 2, 9 x 0..260 8.8 / 9.4, 1 x 2000 35.5 / 34.6; 8 heads of 128, 1 x 1000 24.5 / 24.3.
template <int DH>
int launch_waves(const PrefillArgs& a, int64_t rows, hipStream_t st) {
  const int64_t work = rows * a.H;
  int nwq = work > 32 * 1024 || rows > 400 * static_cast<int64_t>(a.B) ? 4 : (work >= 1024 ? 2 : 1);
  if (const ForcedForm forced = forced_form(launch_override(DLLAVA_LAUNCH_PREFILL_WAVES)); forced.waves) nwq = forced.waves;
  if (nwq == 4) return launch<DH, 4>(a, rows, st);
  if (nwq == 2) return launch<DH, 2>(a, rows, st);
  return launch<DH, 1>(a, rows, st);
}

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void group_generic_kernel(PrefillArgs a) {
  using C = AttendCfg<T, DH>;
  const int j = blockIdx.x;
  const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
  const int h = blockIdx.y * kWaves + w;
  if (j >= a.off[a.B] || h >= a.H) return;
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.off[mid] <= j) lo = mid; else hi = mid;
  }
  const int r0 = a.off[lo], nkeys = j - r0 + 1;
  const size_t stride = a.kv_row_bytes / sizeof(T), first = static_cast<size_t>(r0) * stride + static_cast<size_t>(h / a.group) * DH;
  float qs[C::E];
  load_query<T, DH>(static_cast<const T*>(a.Q) + static_cast<size_t>(j) * (a.q_row_bytes / sizeof(T)) + static_cast<size_t>(h) * DH, a.scale_log2, qs);
  AttnState<C::E> st;
  st.clear();
  for (int c0 = 0; c0 < nkeys; c0 += kPage) {
    const T* kb = static_cast<const T*>(a.K) + first + static_cast<size_t>(c0) * stride;
    const T* vb = static_cast<const T*>(a.V) + first + static_cast<size_t>(c0) * stride;
    if (nkeys - c0 >= kPage)
      attend_chunk<T, DH, false>(kb, vb, stride, kPage, qs, st);
    else
      attend_chunk<T, DH, true>(kb, vb, stride, nkeys - c0, qs, st);
  }
  merge_groups<T, DH>(st);
  if (lane < C::G) {
    T* orow = static_cast<T*>(a.O) + (static_cast<size_t>(j) * a.H + h) * DH + lane * C::E;
    const float inv = 1.f / st.l;
#pragma unroll
    for (int e = 0; e < C::E; ++e) Elem<T>::store(orow + e, st.acc[e] * inv);
  }
}

template <int DH>
int launch_f32(const PrefillArgs& a, int64_t rows, hipStream_t st) {
  hipLaunchKernelGGL((group_generic_kernel<float, DH>), dim3(static_cast<unsigned>(rows), static_cast<unsigned>(ceil_div(a.H, kWaves))), dim3(kThreads), 0, st, a);
  DLLAVA_CHECK_LAUNCH("group_generic_kernel");
  return DLLAVA_OK;
}

}  // namespace
}  // namespace dllava

using namespace dllava;

extern "C" int dllava_group_prefill_attn(const void* Q, int64_t ldq, const void* K, const void* V, int64_t ldkv, int32_t B, const int32_t* off,
                                         int64_t rows, int32_t Hq, int32_t Hkv, int32_t Dh, float scale, void* O, int dtype, void* stream) {
  DLLAVA_REQUIRE(B >= 0 && rows >= 0, DLLAVA_EINVAL, "group_prefill: B = %d, rows = %lld", B, (long long)rows);
  DLLAVA_REQUIRE(rows <= 0x7fffffffLL, DLLAVA_ESHAPE, "group_prefill: rows must fit in int32");
  DLLAVA_REQUIRE(dtype == DLLAVA_F32 || dtype == DLLAVA_BF16, DLLAVA_EDTYPE, "group_prefill: unknown dtype %d", dtype);
  DLLAVA_REQUIRE(Dh == 64 || Dh == 128, DLLAVA_ESHAPE, "group_prefill: Dh must be 64 or 128 (got %d)", Dh);
  DLLAVA_REQUIRE(Hkv > 0 && Hq > 0 && Hq <= 65535 && Hq % Hkv == 0, DLLAVA_ESHAPE, "group_prefill: Hq = %d must be a multiple of Hkv = %d, at most 65535", Hq, Hkv);
  DLLAVA_REQUIRE(scale == scale && scale > 0.f && scale < INFINITY, DLLAVA_EINVAL, "group_prefill: bad scale");
  const int64_t es = static_cast<int64_t>(dtype_size(dtype)), most = int64_t{1} << 27;
  DLLAVA_REQUIRE(ldq >= static_cast<int64_t>(Hq) * Dh && ldkv >= static_cast<int64_t>(Hkv) * Dh && ldq % (16 / es) == 0 && ldkv % (16 / es) == 0,
                 DLLAVA_EINVAL, "group_prefill: row strides %lld and %lld must hold the heads and be multiples of 16 bytes", (long long)ldq, (long long)ldkv);
  DLLAVA_REQUIRE(ldq <= most / es && ldkv <= most / es, DLLAVA_ESHAPE, "group_prefill: a row may take 2^27 bytes at most");
  if (B == 0 || rows == 0) return DLLAVA_OK;
  DLLAVA_REQUIRE(Q && K && V && O && off, DLLAVA_ENULL, "group_prefill: Q, K, V, O and off are required");
  DLLAVA_REQUIRE(aligned(Q, 16) && aligned(O, 16) && aligned(K, 16) && aligned(V, 16), DLLAVA_EINVAL, "group_prefill: Q, K, V, O must be 16-byte aligned");
  PrefillArgs a{};
  a.Q = Q, a.K = K, a.V = V, a.O = O, a.off = off, a.B = B, a.H = Hq, a.group = Hq / Hkv;
  a.q_row_bytes = static_cast<uint32_t>(ldq * es), a.kv_row_bytes = static_cast<uint32_t>(ldkv * es);
  a.scale_log2 = scale * 1.44269504088896340736f;
  hipStream_t st = static_cast<hipStream_t>(stream);
  DLLAVA_REQUIRE(dtype == DLLAVA_BF16 || rows < (1 << 24), DLLAVA_ESHAPE, "group_prefill: DLLAVA_F32 takes fewer than 2^24 rows");
  if (dtype == DLLAVA_F32) return Dh == 128 ? launch_f32<128>(a, rows, st) : launch_f32<64>(a, rows, st);
  const int rc = Dh == 128 ? launch_waves<128>(a, rows, st) : launch_waves<64>(a, rows, st);
  DLLAVA_REQUIRE(rc <= 0, DLLAVA_ESHAPE, "group_prefill: too many rows or sequences");
  return rc;
}
