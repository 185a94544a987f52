// dllava_mx_cache_store, dllava_mx_cache_load: keys and values into and out of a paged cache in 4 bits.
//
// Pure streams.  A wave takes one head of one page's piece of a sequence: 16 tokens at most, a lane eight elements of a token (four
// lanes a block of 32).  Keys keep their order.  A byte of the values holds columns c and c + 16 of a block, which lie in lanes two
// apart: the two exchange their codes and write half of the bytes each.  No byte is shared between tokens, so tokens of other calls in the
// same page are left alone.
#include "mx.h"

namespace dllava {

int check_mx_cache(const dllava_kv_cache* c, const char* who) {
  DLLAVA_REQUIRE(c, DLLAVA_ENULL, "%s: cache is NULL", who);
  DLLAVA_REQUIRE(c->dtype == DLLAVA_MX, DLLAVA_EDTYPE, "%s: the cache must be in 4 bits (DLLAVA_MX; got dtype %d)", who, c->dtype);
  DLLAVA_REQUIRE(c->pages && c->block_table && c->cache_len, DLLAVA_ENULL, "%s: cache pages, block_table and cache_len are required", who);
  DLLAVA_REQUIRE(c->page_size == kPage, DLLAVA_ESHAPE, "%s: page_size must be 16 (got %d)", who, c->page_size);
  DLLAVA_REQUIRE(c->Dh == 64 || c->Dh == 128, DLLAVA_ESHAPE, "%s: Dh must be 64 or 128 (got %d)", who, c->Dh);
  DLLAVA_REQUIRE(c->H > 0 && c->n_pages > 0 && c->max_pages_per_seq > 0, DLLAVA_ESHAPE, "%s: cache H, n_pages and max_pages_per_seq must be positive", who);
  DLLAVA_REQUIRE(c->H <= 65535 && c->max_pages_per_seq <= 0x7fffffff / kPage, DLLAVA_ESHAPE, "%s: cache H or max_pages_per_seq too large", who);
  DLLAVA_REQUIRE(aligned(c->pages, 16), DLLAVA_EINVAL, "%s: cache pages must be 16-byte aligned", who);
  return DLLAVA_OK;
}

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

struct CacheArgs {
  const void* K;
  const void* V;
  int64_t ldkv;
  int32_t B;
  const int32_t* off;
  const int32_t* start;
  const int32_t* src_off;
  const int32_t* src_idx;
  int32_t rows;
  uint8_t* pages;
  const int32_t* block_table;
  int32_t* cache_len;
  int32_t max_pages, H;
  int32_t* err_flag;
};

// What a block works on: up to 16 rows of a sequence, the ones that lie in one page.
struct Piece {
  int b, row, n;  // sequence, its first row here (counted from off[b]), rows
  int64_t pos;    // that row's position
  bool inside;    // the page is one of the sequence's
};
// Pieces are numbered in slots: those of sequence b from off[b] / 16 + 2b on (a sequence of n rows touches at most n / 16 + 2 pages).
// n == 0: none.
__device__ __forceinline__ Piece find_piece(const CacheArgs& a, int slot) {
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.off[mid] / kPage + 2 * mid <= slot) lo = mid; else hi = mid;
  }
  Piece p{lo, 0, 0, 0, false};
  const int r0 = a.off[lo], end = a.off[lo + 1] < a.rows ? a.off[lo + 1] : a.rows, i = slot - (r0 / kPage + 2 * lo);
  const int n = end - r0, s = a.start ? (a.start[lo] > 0 ? a.start[lo] : 0) : 0;
  if (i < 0 || n <= 0) return p;
  const int64_t page = s / kPage + static_cast<int64_t>(i), end_pos = static_cast<int64_t>(s) + n;
  const int64_t first = page * kPage > s ? page * kPage : s, last = (page + 1) * kPage < end_pos ? (page + 1) * kPage : end_pos;
  if (first >= last) return p;
  p.row = static_cast<int>(first - s), p.n = static_cast<int>(last - first), p.pos = first, p.inside = page < a.max_pages;
  return p;
}
__device__ __forceinline__ uint8_t* head_of(const CacheArgs& a, const Piece& p, int h, int DH) {
  const int page = a.block_table[static_cast<size_t>(p.b) * a.max_pages + static_cast<size_t>(p.pos / kPage)];
  return a.pages + (static_cast<size_t>(page) * a.H + h) * mx_page_bytes(DH);
}

template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void mx_cache_store_kernel(CacheArgs a) {
  constexpr int kLanes = DH / 8, kTokens = kWave / kLanes, kSteps = kPage / kTokens, kBlocks = DH / kMxBlock;
  if (blockIdx.x == 0 && blockIdx.y == 0)  // the lengths, which nothing here reads
    for (int b = threadIdx.x; b < a.B; b += kThreads) {
      const int64_t end = a.off[b + 1] < a.rows ? a.off[b + 1] : a.rows, n = end - a.off[b];
      const int64_t len = (a.start && a.start[b] > 0 ? a.start[b] : 0) + (n > 0 ? n : 0), cap = static_cast<int64_t>(a.max_pages) * kPage;
      a.cache_len[b] = static_cast<int32_t>(len < cap ? len : cap);
      if (len > cap && a.err_flag) *a.err_flag = 1;
    }
  const Piece p = find_piece(a, blockIdx.x);
  const int lane = threadIdx.x % kWave, h = blockIdx.y * kWaves + threadIdx.x / kWave;
  if (p.n == 0 || !p.inside || h >= a.H) return;
  const int i8 = lane % kLanes, t_in = lane / kLanes;
  uint8_t* const page = head_of(a, p, h, DH);
  const int32_t r0 = a.off[p.b];
  float k[kSteps][8], v[kSteps][8];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = s * kTokens + t_in;
    if (i < p.n) {
      const int row = r0 + p.row + i;
      const int64_t src = (a.src_idx ? static_cast<int64_t>(a.src_off[p.b]) + a.src_idx[row] : row) * a.ldkv + static_cast<int64_t>(h) * DH + 8 * i8;
      mx_load8(static_cast<const T*>(a.K) + src, k[s]);
      mx_load8(static_cast<const T*>(a.V) + src, v[s]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) k[s][e] = v[s][e] = 0.f;
    }
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = s * kTokens + t_in, t = static_cast<int>(p.pos % kPage) + i;  // slot in the page
    const uint32_t ks = mx_scale_byte(mx_block_amax(k[s])), vs = mx_scale_byte(mx_block_amax(v[s]));
    const uint32_t kc = mx_encode8(k[s], ks), mine = mx_encode8(v[s], vs);
    const uint32_t other = __shfl_xor(mine, 2, kWave);
    if (i >= p.n) continue;
    *reinterpret_cast<uint32_t*>(page + t * (DH / 2) + 4 * i8) = kc;
    // lane i8: block i8 / 4, columns 8 (i8 % 4) ..: the lower half of the block's bytes where i8 % 4 < 2
    const bool low = (i8 & 2) == 0;
    const uint32_t lo = low ? mine : other, hi = low ? other : mine;
    const int c0 = 8 * (i8 & 1) + (low ? 0 : 4);
    uint8_t* const dst = page + 8 * DH + ((t / 4 * 16 + c0) * 4 + t % 4) * kBlocks + i8 / 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int sh = 4 * e + (low ? 0 : 16);
      dst[e * 4 * kBlocks] = static_cast<uint8_t>(((lo >> sh) & 15u) | (((hi >> sh) & 15u) << 4));
    }
    if (i8 % 4 == 0) {
      page[16 * DH + t * kBlocks + i8 / 4] = static_cast<uint8_t>(ks);
      page[16 * DH + DH / 2 + t * kBlocks + i8 / 4] = static_cast<uint8_t>(vs);
    }
  }
}

template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void mx_cache_load_kernel(CacheArgs a) {
  constexpr int kLanes = DH / 8, kTokens = kWave / kLanes, kSteps = kPage / kTokens, kBlocks = DH / kMxBlock;
  const Piece p = find_piece(a, blockIdx.x);
  const int lane = threadIdx.x % kWave, h = blockIdx.y * kWaves + threadIdx.x / kWave;
  if (p.n == 0 || h >= a.H) return;
  const int i8 = lane % kLanes, t_in = lane / kLanes;
  const uint8_t* const page = p.inside ? head_of(a, p, h, DH) : nullptr;  // (positions behind the capacity have no page)
  const int len = p.inside ? a.cache_len[p.b] : 0;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = s * kTokens + t_in, t = static_cast<int>(p.pos % kPage) + i;
    if (i >= p.n) continue;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (p.pos + i < len) {
      k = mx_decode8(*reinterpret_cast<const uint32_t*>(page + t * (DH / 2) + 4 * i8), static_cast<uint32_t>(page[16 * DH + t * kBlocks + i8 / 4]) << 23);
      const uint8_t* src = page + 8 * DH + ((t / 4 * 16 + 8 * (i8 & 1)) * 4 + t % 4) * kBlocks + i8 / 4;
      uint32_t c = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) c |= ((src[e * 4 * kBlocks] >> ((i8 & 2) ? 4 : 0)) & 15u) << (4 * e);
      v = mx_decode8(c, static_cast<uint32_t>(page[16 * DH + DH / 2 + t * kBlocks + i8 / 4]) << 23);
    }
    const int64_t dst = (static_cast<int64_t>(a.off[p.b]) + p.row + i) * a.ldkv + static_cast<int64_t>(h) * DH + 8 * i8;
    mx_store8(const_cast<T*>(static_cast<const T*>(a.K)) + dst, k);
    mx_store8(const_cast<T*>(static_cast<const T*>(a.V)) + dst, v);
  }
}
int prepare(const char* who, const void* K, const void* V, int64_t ldkv, int32_t B, const int32_t* off, const int32_t* start, int64_t rows,
            const dllava_kv_cache* cache, int dtype, CacheArgs& a, dim3& grid) {
  DLLAVA_REQUIRE(dtype == DLLAVA_F32 || dtype == DLLAVA_BF16, DLLAVA_EDTYPE, "%s: unknown dtype %d", who, dtype);
  if (int rc = check_mx_cache(cache, who)) return rc;
  DLLAVA_REQUIRE(B >= 0 && rows >= 0, DLLAVA_EINVAL, "%s: B = %d, rows = %lld", who, B, (long long)rows);
  DLLAVA_REQUIRE(ldkv >= static_cast<int64_t>(cache->H) * cache->Dh && ldkv * static_cast<int64_t>(dtype_size(dtype)) % 16 == 0, DLLAVA_EINVAL,
                 "%s: ldkv = %lld must be at least H * Dh and a multiple of 16 bytes", who, (long long)ldkv);
  if (B == 0) return DLLAVA_OK;
  const int64_t pieces = rows / kPage + 2 * static_cast<int64_t>(B) + 1;
  DLLAVA_REQUIRE(rows <= 0x7fffffffLL && pieces <= 0x7fffffffLL, DLLAVA_ESHAPE, "%s: rows and B must fit in int32", who);
  DLLAVA_REQUIRE(off && (rows == 0 || (K && V)), DLLAVA_ENULL, "%s: off, K and V are required", who);
  DLLAVA_REQUIRE(aligned(K, 16) && aligned(V, 16), DLLAVA_EINVAL, "%s: K and V must be 16-byte aligned", who);
  a.K = K, a.V = V, a.ldkv = ldkv, a.B = B, a.off = off, a.start = start, a.rows = static_cast<int32_t>(rows);
  a.pages = static_cast<uint8_t*>(cache->pages), a.block_table = cache->block_table, a.cache_len = cache->cache_len;
  a.max_pages = cache->max_pages_per_seq, a.H = cache->H;
  grid = dim3(static_cast<unsigned>(pieces), static_cast<unsigned>(ceil_div(cache->H, kWaves)));
  return DLLAVA_OK;
}

}  // namespace
}  // namespace dllava

using namespace dllava;

extern "C" int dllava_mx_cache_store(const void* K, const void* V, int64_t ldkv, int32_t B, const int32_t* off, const int32_t* start, int64_t rows,
                                     const int32_t* src_off, const int32_t* src_idx, const dllava_kv_cache* cache, int32_t* err_flag, int dtype,
                                     void* stream) {
  CacheArgs a{};
  dim3 grid;
  if (int rc = prepare("mx_cache_store", K, V, ldkv, B, off, start, rows, cache, dtype, a, grid)) return rc;
  DLLAVA_REQUIRE((src_off == nullptr) == (src_idx == nullptr), DLLAVA_ENULL, "mx_cache_store: src_off and src_idx go together");
  DLLAVA_REQUIRE(!start || start + B <= cache->cache_len || cache->cache_len + B <= start, DLLAVA_EINVAL,
                 "mx_cache_store: start must not overlap cache_len, which the call writes");
  if (B == 0) return DLLAVA_OK;
  a.src_off = src_off, a.src_idx = src_idx, a.err_flag = err_flag;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (cache->Dh == 128) {
    if (dtype == DLLAVA_BF16) hipLaunchKernelGGL((mx_cache_store_kernel<bf16_t, 128>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((mx_cache_store_kernel<float, 128>), grid, dim3(kThreads), 0, st, a);
  } else {
    if (dtype == DLLAVA_BF16) hipLaunchKernelGGL((mx_cache_store_kernel<bf16_t, 64>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((mx_cache_store_kernel<float, 64>), grid, dim3(kThreads), 0, st, a);
  }
  DLLAVA_CHECK_LAUNCH("mx_cache_store_kernel");
  return DLLAVA_OK;
}

extern "C" int dllava_mx_cache_load(const dllava_kv_cache* cache, int32_t B, const int32_t* off, const int32_t* start, int64_t rows, void* K, void* V,
                                    int64_t ldkv, int dtype, void* stream) {
  CacheArgs a{};
  dim3 grid;
  if (int rc = prepare("mx_cache_load", K, V, ldkv, B, off, start, rows, cache, dtype, a, grid)) return rc;
  if (B == 0 || rows == 0) return DLLAVA_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (cache->Dh == 128) {
    if (dtype == DLLAVA_BF16) hipLaunchKernelGGL((mx_cache_load_kernel<bf16_t, 128>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((mx_cache_load_kernel<float, 128>), grid, dim3(kThreads), 0, st, a);
  } else {
    if (dtype == DLLAVA_BF16) hipLaunchKernelGGL((mx_cache_load_kernel<bf16_t, 64>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((mx_cache_load_kernel<float, 64>), grid, dim3(kThreads), 0, st, a);
  }
  DLLAVA_CHECK_LAUNCH("mx_cache_load_kernel");
  return DLLAVA_OK;
}
