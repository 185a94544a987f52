// dllava_mx_cache_store, dllava_mx_cache_load: keys and values into and out of a paged cache in 4 bits.
//
// Pure streams.  A wave takes one head of one page's piece of a sequence: 16 tokens at most, a lane eight elements of a token (four
// lanes a block of 32).  Keys keep their order.  A byte of the values holds columns c and c + 16 of a block, which lie in lanes two
// apart, and the bytes of a token's blocks at equal columns lie together: the lanes exchange their codes (two apart, then the blocks'
// lanes, four and eight apart) and each writes a word of whole bytes.  No byte is shared between tokens, so tokens of other calls in the same page
// are left alone.  Measured, 16 sequences of 352 of 704 rows, 32 heads of 128, bfloat16 (117 MB, 24 us at the rate of a copy): 29.6 us in,
// 30.4 us out; 36.1 and 41.3 with the values' bytes one by one.
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
  int lo = 0;
  for (int n = a.B; n > 1;) {  // 64 sequences in question at a time
    const int step = (n + kWave - 1) / kWave, i = static_cast<int>(threadIdx.x % kWave) * step, mid = lo + i;
    const uint64_t at = __ballot(i < n && a.off[i < n ? mid : lo] / kPage + 2 * (i < n ? mid : lo) <= slot);
    const int last = at ? 63 - __clzll(at) : 0;
    lo += last * step, n = n - last * step < step ? n - last * step : step;
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

template <int CTRL>
__device__ __forceinline__ uint32_t lanes(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t lane_xor2(uint32_t v) { return lanes<0x4E>(v); }                // quad_perm [2,3,0,1]
__device__ __forceinline__ uint32_t lane_xor4(uint32_t v) { return lanes<0x141>(lanes<0x1B>(v)); }  // quad_perm [3,2,1,0], row_half_mirror
__device__ __forceinline__ uint32_t lane_xor8(uint32_t v) { return lanes<0x128>(v); }               // row_ror:8
// Byte e of lane m's word to byte m of lane e's, m the lane's block: of four (Dh = 128, lanes 4 apart), or of two (the words' halves: bytes
// 0 and 1 of lane e hold what both have in byte e, bytes 2 and 3 what they have in byte e + 2).  Twice is once undone.
template <int BLOCKS>
__device__ __forceinline__ uint32_t transpose_blocks(uint32_t w, int m) {
  const uint32_t o = lane_xor4(w);
  w = __builtin_amdgcn_perm(o, w, m & 1 ? 0x03070105u : 0x06020400u);  // bytes 0..3: w's, 4..7: o's
  if (BLOCKS == 4) {
    const uint32_t far = lane_xor8(w);
    w = __builtin_amdgcn_perm(far, w, m & 2 ? 0x03020706u : 0x05040100u);
  }
  return w;
}
__device__ __forceinline__ uint32_t nibbles_to_bytes(uint32_t x) {  // of the lower half
  x = (x | x << 8) & 0x00ff00ffu;
  return (x | x << 4) & 0x0f0f0f0fu;
}
__device__ __forceinline__ uint32_t bytes_to_nibbles(uint32_t x) {  // their lower four bits
  x &= 0x0f0f0f0fu;
  x = (x | x >> 4) & 0x00ff00ffu;
  return (x | x >> 8) & 0xffffu;
}
// A lane's words of a token's values: bytes of all blocks at column c0 + m (and, of two blocks, at c0 + m + 2 in the upper half).
template <int DH>
struct ValueBytes {
  static constexpr int kBlocks = DH / kMxBlock;
  static __device__ __forceinline__ int at(int t, int c) { return 8 * DH + ((t / 4 * 16 + c) * 4 + t % 4) * kBlocks; }
  static __device__ __forceinline__ void store(uint8_t* page, int t, int c0, int m, uint32_t w) {
    if constexpr (kBlocks == 4) {
      *reinterpret_cast<uint32_t*>(page + at(t, c0 + m)) = w;
    } else {
      *reinterpret_cast<uint16_t*>(page + at(t, c0 + m)) = static_cast<uint16_t>(w);
      *reinterpret_cast<uint16_t*>(page + at(t, c0 + m + 2)) = static_cast<uint16_t>(w >> 16);
    }
  }
  static __device__ __forceinline__ uint32_t load(const uint8_t* page, int t, int c0, int m) {
    if constexpr (kBlocks == 4) return *reinterpret_cast<const uint32_t*>(page + at(t, c0 + m));
    return *reinterpret_cast<const uint16_t*>(page + at(t, c0 + m)) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(page + at(t, c0 + m + 2))) << 16;
  }
};

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
  const int i8 = lane % kLanes, t_in = lane / kLanes, m = i8 / 4;
  uint8_t* const page = head_of(a, p, h, DH);
  const int32_t r0 = a.off[p.b];
  float k[kSteps][8], v[kSteps][8];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = s * kTokens + t_in, row = r0 + p.row + (i < p.n ? i : 0);  // (past the piece: its first token, not stored)
    const int64_t src = (a.src_idx ? static_cast<int64_t>(a.src_off[p.b]) + a.src_idx[row] : row) * a.ldkv + static_cast<int64_t>(h) * DH + 8 * i8;
    mx_load8(static_cast<const T*>(a.K) + src, k[s]);
    mx_load8(static_cast<const T*>(a.V) + src, v[s]);
  }
  // lane i8: block m, columns 8 (i8 % 4) ..: with the lane two apart, the lower half of the block's bytes where i8 % 4 < 2
  const bool low = (i8 & 2) == 0;
  const int c0 = 8 * (i8 & 1) + (low ? 0 : 4);
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = s * kTokens + t_in, t = static_cast<int>(p.pos % kPage) + i;  // slot in the page
    const uint32_t ks = mx_scale_byte(mx_block_amax(k[s])), vs = mx_scale_byte(mx_block_amax(v[s]));
    const uint32_t kc = mx_encode8(k[s], ks), mine = mx_encode8(v[s], vs), other = lane_xor2(mine);
    const uint32_t lower = low ? mine & 0xffffu : other >> 16, upper = low ? other & 0xffffu : mine >> 16;
    const uint32_t bytes = transpose_blocks<kBlocks>(nibbles_to_bytes(lower) | nibbles_to_bytes(upper) << 4, m);
    const uint32_t scales = transpose_blocks<kBlocks>(ks | vs << 8, m);  // lane m = 0: of the keys' blocks, 1: of the values'
    if (i >= p.n) continue;
    *reinterpret_cast<uint32_t*>(page + t * (DH / 2) + 4 * i8) = kc;
    ValueBytes<DH>::store(page, t, c0, m, bytes);
    if (i8 == 0 || i8 == 4) {
      uint8_t* const dst = page + 16 * DH + m * (DH / 2) + t * kBlocks;
      if constexpr (kBlocks == 4) *reinterpret_cast<uint32_t*>(dst) = scales;
      else *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(scales);
    }
  }
}

template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void mx_cache_load_kernel(CacheArgs a) {
  constexpr int kLanes = DH / 8, kTokens = kWave / kLanes, kSteps = kPage / kTokens, kBlocks = DH / kMxBlock;
  const Piece p = find_piece(a, blockIdx.x);
  const int lane = threadIdx.x % kWave, h = blockIdx.y * kWaves + threadIdx.x / kWave;
  if (p.n == 0 || h >= a.H) return;
  const int i8 = lane % kLanes, t_in = lane / kLanes, m = i8 / 4;
  const uint8_t* const page = p.inside ? head_of(a, p, h, DH) : a.pages;  // (positions behind the capacity have no page; not used)
  const int len = p.inside ? a.cache_len[p.b] : 0;
  const bool low = (i8 & 2) == 0;
  const int c0 = 8 * (i8 & 1) + (low ? 0 : 4);
  uint32_t kc[kSteps], w[kSteps], ks[kSteps], vs[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int t = (static_cast<int>(p.pos % kPage) + s * kTokens + t_in) % kPage;  // (past the piece: another slot, not used)
    kc[s] = *reinterpret_cast<const uint32_t*>(page + t * (DH / 2) + 4 * i8);
    w[s] = ValueBytes<DH>::load(page, t, c0, m);
    ks[s] = page[16 * DH + t * kBlocks + m], vs[s] = page[16 * DH + DH / 2 + t * kBlocks + m];
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = s * kTokens + t_in;
    const uint32_t mine = transpose_blocks<kBlocks>(w[s], m);       // block m's bytes at columns c0 .. c0 + 3
    const uint32_t other = lane_xor2(mine);                         // at the other four of 8 (i8 % 2) ..
    const uint32_t codes = low ? bytes_to_nibbles(mine) | bytes_to_nibbles(other) << 16 : bytes_to_nibbles(other >> 4) | bytes_to_nibbles(mine >> 4) << 16;
    if (i >= p.n) continue;
    const bool held = p.pos + i < len;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const int64_t dst = (static_cast<int64_t>(a.off[p.b]) + p.row + i) * a.ldkv + static_cast<int64_t>(h) * DH + 8 * i8;
    mx_store8(const_cast<T*>(static_cast<const T*>(a.K)) + dst, held ? mx_decode8(kc[s], ks[s] << 23) : zero);
    mx_store8(const_cast<T*>(static_cast<const T*>(a.V)) + dst, held ? mx_decode8(codes, vs[s] << 23) : zero);
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
  DLLAVA_REQUIRE(rows <= 0x7fffffffLL && pieces < (1 << 24), DLLAVA_ESHAPE, "%s: rows / 16 + 2 B must be below 2^24", who);
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
