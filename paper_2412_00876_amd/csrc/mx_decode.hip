// dllava_mx_decode_attn_append: one decode step over a paged cache in 4 bits, grouped heads, conditional append (Eq. 6 of the paper).
//
// The cache is the traffic: 17/32 byte an element, read once for the query heads of a group together.  A wave walks steps of 32
// tokens (two pages) of one K/V head:
//     S^T = K Q^T     v_mfma_f32_16x16x32_bf16, 16 tokens x 16 query heads; a lane's 16 bytes of keys (8 at head size 64) are a fourth
//                     of a token, and the products take its elements in the order in which they lie
//     O^T = V^T P^T   columns x query heads; S^T leaves a lane with tokens 4g .. 4g + 3 of one query head, and the cache keeps the
//                     values so that a lane finds the same tokens of "its" column of every block in one piece: the probabilities
//                     never leave their lane
// Codes become bfloat16 in registers (exact), keys and values with their scales.  The softmax keeps a running reference per query head
// that moves only when a score passes it by more than kSlack powers of two.  Sums and statistics are float32; the probabilities are
// rounded to bfloat16 for the product (half a step is 2^-9 of each, which the sum over tokens averages out below the output's own
// rounding) and added up before that.
//
// How the work is dealt.  The steps of all units -- a unit is (sequence, K/V head, up to 16 of its query heads) -- are numbered one behind the
// other, in the order of the sequences, and cut into equal shares: one for each block, a fourth of it for each wave, whatever the lengths
// are (split by sequence and head, the longest sequence decided: 32 of 2000 to 8000 tokens took 66 us at best).  A wave therefore has one unit
// whose start is not its own, units of its own and one that it does not end.  Own units are written at once; the others' parts are joined in
// LDS, once per block, and the at most two units that reach into other blocks through the workspace: the last of their blocks to
// arrive adds the parts up in the order of the blocks.
// A wave's loads are one stream through its units: two steps' pages are on their way while a third is worked on.
//
// cache_len moves when all blocks have read it; the new token goes to a slot that no block of this launch looks at (tokens behind the
// length are masked by position, and their scales are replaced, whatever they hold).
#include "mx.h"

namespace dllava {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kHeads = 16;       // query heads of a unit, at most
constexpr int kStep = 2 * kPage;
constexpr int kBlocksPerUnit = 64;  // blocks that a unit may reach into, less one
constexpr int kBlocksMax = 512;  // two for each compute unit
constexpr int kMinShare = 8;     // steps of a block, at least
constexpr int kCut = 16, kLeastCut = 32;  // steps: see the shares
constexpr int kCnt = 64;         // int32 slots per counter: a memory line each
constexpr int kReadCounters = 16;
constexpr float kSlack = 8.f;

struct MxDecodeArgs {
  const bf16_t* q;
  const bf16_t* k_new;
  const bf16_t* v_new;
  const float* logits;
  const uint8_t* keep_override;
  float threshold, scale_log2;
  uint8_t* pages;
  const int32_t* block_table;
  int32_t* cache_len;
  int32_t max_pages, B, H, group, tiles;  // query heads per K/V head; tiles of 16 of them
  int32_t* cnt_read;  // [kReadCounters + 1] blocks that have read cache_len; the last one counts full counters
  int32_t* cnt_done;  // [blocks] parts that are there of the unit that starts in block i and ends in another
  float* part;        // [blocks][2][part_heads][DH + 2]
  int32_t part_heads; // query heads of a unit, at most
  bf16_t* o;
  uint8_t* keep_out;
  int32_t* err_flag;
};

// What a step reads: this lane's pieces of two pages.
template <int DH>
struct Step {
  static constexpr int kWords = DH / 32;  // words of codes in a piece, K and V alike
  uint32_t k[2][kWords], v[2][kWords];
  uint32_t ks[2];          // scale byte of the keys' piece
  uint32_t vs[2][4];       // scale bytes of the blocks of tokens 4g .. 4g + 3, a word a token (head size 64: half a word)
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&d)[N], const uint8_t* p) {
  if constexpr (N == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    d[0] = v.x, d[1] = v.y, d[2] = v.z, d[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    d[0] = v.x, d[1] = v.y;
  }
}

// Where a lane's pieces lie in a page of one head.
struct LaneAt {
  uint32_t k, v, ks, vs;
};
template <int DH>
__device__ __forceinline__ LaneAt lane_at(int lane) {
  constexpr int kBlocks = DH / 32;
  const uint32_t g = lane / 16, r16 = lane % 16;
  return {r16 * (DH / 2) + g * (DH / 8), 8u * DH + lane * (DH / 8), 16u * DH + r16 * kBlocks + g * kBlocks / 4, 16u * DH + DH / 2 + g * 4 * kBlocks};
}
template <int DH>
__device__ __forceinline__ void load_page(Step<DH>& s, int i, const uint8_t* page, const LaneAt& at) {  // page: wave-uniform
  load_words(s.k[i], page + at.k);
  load_words(s.v[i], page + at.v);
  s.ks[i] = page[at.ks];
  if constexpr (DH == 128) {
    load_words(s.vs[i], page + at.vs);
  } else {
    uint32_t two[2];
    load_words(two, page + at.vs);
    s.vs[i][0] = two[0], s.vs[i][1] = two[1];
  }
}

template <int DH>
struct Wave {
  uint4 q[DH / 32];       // queries, the operand of product i
  f32x4 o[DH / 16];       // columns 16 i + 4 g + e of query head r16
  float m, l;             // reference (powers of two), sum of this lane's probabilities

  // Scores of 32 tokens into probabilities; x: scaled, -inf where there is no token.
  __device__ __forceinline__ uint4 softmax(float (&x)[8]) {
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    if (__any(top > m + kSlack)) {  // (the first step: from -inf)
      top = fmaxf(top, __shfl_xor(top, 16, kWave));
      top = fmaxf(top, __shfl_xor(top, 32, kWave));
      const float to = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) o[i] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = __builtin_amdgcn_exp2f(x[e] - ref);
      s += x[e];
    }
    l += s;
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
  __device__ __forceinline__ f32x4 product(const uint4& a, const uint4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }

  // One step; there > 0: tokens that exist from its first one on (32 or more: all of its).
  __device__ __forceinline__ void attend(Step<DH>& s, int there, float scale_log2, int lane) {
    const int g = lane / 16;
    float x[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < DH / 32; ++w) c = product(mx_decode8(s.k[i][w], s.ks[i] << 23), q[w], c);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = c[e] * scale_log2;
    }
    if (there < kStep) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (kPage * i + 4 * g + e >= there) {
            x[4 * i + e] = -INFINITY;
            // a finite scale, whatever the slot holds: the codes are finite, and the probability is zero
            if constexpr (DH == 128) s.vs[i][e] = 0x7f7f7f7fu;
            else s.vs[i][e / 2] = e % 2 ? (s.vs[i][e / 2] & 0xffffu) | 0x7f7f0000u : (s.vs[i][e / 2] & 0xffff0000u) | 0x7f7fu;
          }
    }
    const uint4 p = softmax(x);
    // block m, half h: columns 32 m + 16 h + r16.  Byte m of token j's word (head size 64: byte 2 (j % 2) + m of word j / 2) holds both
    // halves, which are sorted by tokens; its scale is the same byte of the scales' word.
#pragma unroll
    for (int m_ = 0; m_ < DH / 32; ++m_) {
      uint32_t both[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int byte = DH == 128 ? m_ : 2 * (j % 2) + m_, word = DH == 128 ? j : j / 2;
          const uint32_t z = s.vs[i][word], c = s.v[i][word];
          const uint32_t sb = byte == 0 ? mx_scale_bits<0>(z) : byte == 1 ? mx_scale_bits<1>(z) : byte == 2 ? mx_scale_bits<2>(z) : mx_scale_bits<3>(z);
          both[i][j] = byte == 0 ? mx_decode2<0>(c, sb) : byte == 1 ? mx_decode2<1>(c, sb) : byte == 2 ? mx_decode2<2>(c, sb) : mx_decode2<3>(c, sb);
        }
      const uint4 low = make_uint4(__builtin_amdgcn_perm(both[0][1], both[0][0], 0x05040100u), __builtin_amdgcn_perm(both[0][3], both[0][2], 0x05040100u),
                                   __builtin_amdgcn_perm(both[1][1], both[1][0], 0x05040100u), __builtin_amdgcn_perm(both[1][3], both[1][2], 0x05040100u));
      const uint4 high = make_uint4(__builtin_amdgcn_perm(both[0][1], both[0][0], 0x07060302u), __builtin_amdgcn_perm(both[0][3], both[0][2], 0x07060302u),
                                    __builtin_amdgcn_perm(both[1][1], both[1][0], 0x07060302u), __builtin_amdgcn_perm(both[1][3], both[1][2], 0x07060302u));
      o[2 * m_] = product(low, p, o[2 * m_]);
      o[2 * m_ + 1] = product(high, p, o[2 * m_ + 1]);
    }
  }

  // The current token, as it was given: token 0 of a step whose others do not exist.
  struct New {
    uint4 k[DH / 32];
    uint32_t v[DH / 16];
  };
  __device__ __forceinline__ void load_new(New& t, const bf16_t* k, const bf16_t* v, int lane) {
#pragma unroll
    for (int w = 0; w < DH / 32; ++w) t.k[w] = *reinterpret_cast<const uint4*>(k + lane / 16 * (DH / 4) + 8 * w);
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) t.v[i] = v[16 * i + lane % 16];
  }
  __device__ __forceinline__ void attend_new(const New& t, float scale_log2, int lane) {
    const int g = lane / 16, r16 = lane % 16;
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < DH / 32; ++w) c = product(r16 == 0 ? t.k[w] : make_uint4(0, 0, 0, 0), q[w], c);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = -INFINITY;
    if (g == 0) x[0] = c[0] * scale_log2;
    const uint4 p = softmax(x);
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) o[i] = product(make_uint4(g == 0 ? t.v[i] : 0u, 0, 0, 0), p, o[i]);
  }
};

// Stores the new token of (b, h) in slot `at` of its page: lanes 0 .. DH/8 - 1 of a wave, the whole wave calls.
template <int DH>
__device__ __forceinline__ void append(const MxDecodeArgs& a, int b, int h, int at, int lane) {
  constexpr int kLanes = DH / 8, kBlocks = DH / 32;
  const int i8 = lane % kLanes, t = at % kPage;
  const size_t src = (static_cast<size_t>(b) * a.H + h) * DH + 8 * i8;
  float k[8], v[8];
  mx_load8(a.k_new + src, k);
  mx_load8(a.v_new + src, v);
  const uint32_t ks = mx_scale_byte(mx_block_amax(k)), vs = mx_scale_byte(mx_block_amax(v));
  const uint32_t kc = mx_encode8(k, ks), mine = mx_encode8(v, vs), other = __shfl_xor(mine, 2, kWave);
  if (lane >= kLanes) return;
  uint8_t* const page = a.pages + (static_cast<size_t>(a.block_table[static_cast<size_t>(b) * a.max_pages + at / kPage]) * a.H + h) * mx_page_bytes(DH);
  *reinterpret_cast<uint32_t*>(page + t * (DH / 2) + 4 * i8) = kc;
  const bool low = (i8 & 2) == 0;
  const uint32_t lo = low ? mine : other, hi = low ? other : mine;
  uint8_t* const dst = page + 8 * DH + ((t / 4 * 16 + 8 * (i8 & 1) + (low ? 0 : 4)) * 4 + t % 4) * kBlocks + i8 / 4;
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

// The lengths' last reader moves them.
__device__ __forceinline__ void commit(const MxDecodeArgs& a) {
  const int cap = a.max_pages * kPage;
  for (int b = threadIdx.x; b < a.B; b += kThreads) {
    const bool keep = a.keep_override ? a.keep_override[b] != 0 : keep_from_logits(a.logits, b, a.threshold);
    if (a.keep_out) a.keep_out[b] = keep ? 1 : 0;
    if (!keep) continue;
    const int L = a.cache_len[b];
    if (L >= 0 && L < cap) a.cache_len[b] = L + 1;
    else if (a.err_flag) *a.err_flag = 1;
  }
}
// This block has read what it needs of cache_len: its number among those of its counter (thread 0 calls; the value is used later) ...
__device__ __forceinline__ int reader_ticket(const MxDecodeArgs& a) { return add_agent(&a.cnt_read[blockIdx.x % kReadCounters * kCnt], 1); }
// ... and whether every other block has, too.
__device__ __forceinline__ bool last_reader(const MxDecodeArgs& a, int ticket) {
  const int G = static_cast<int>(gridDim.x), k = static_cast<int>(blockIdx.x) % kReadCounters;
  const int of_k = (G - k + kReadCounters - 1) / kReadCounters, used = G < kReadCounters ? G : kReadCounters;
  if (ticket != of_k - 1) return false;
  zero_agent(&a.cnt_read[k * kCnt]);
  if (add_agent(&a.cnt_read[kReadCounters * kCnt], 1) != used - 1) return false;
  zero_agent(&a.cnt_read[kReadCounters * kCnt]);
  return true;
}

// Inclusive sum over the lanes up to this one, and the maximum of all (in lane 63), on the DPP data path.
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int v, int otherwise) {
  return __builtin_amdgcn_update_dpp(otherwise, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int scan_sum(int v) {
  v += from_lane<0x111, 0xf>(v, 0);  // row_shr by 1, 2, 4, 8
  v += from_lane<0x112, 0xf>(v, 0);
  v += from_lane<0x114, 0xf>(v, 0);
  v += from_lane<0x118, 0xf>(v, 0);
  v += from_lane<0x142, 0xa>(v, 0);  // the last lane of rows 0 and 2 to the rows behind them
  v += from_lane<0x143, 0xc>(v, 0);  // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ int scan_max(int v) {  // (of values >= 0)
  int o;
  o = from_lane<0x111, 0xf>(v, 0), v = o > v ? o : v;
  o = from_lane<0x112, 0xf>(v, 0), v = o > v ? o : v;
  o = from_lane<0x114, 0xf>(v, 0), v = o > v ? o : v;
  o = from_lane<0x118, 0xf>(v, 0), v = o > v ? o : v;
  o = from_lane<0x142, 0xa>(v, 0), v = o > v ? o : v;
  o = from_lane<0x143, 0xc>(v, 0), v = o > v ? o : v;
  return v;
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

template <int DH>
__global__ __launch_bounds__(kThreads, 2) void mx_decode_kernel(MxDecodeArgs a) {
  const int tid = threadIdx.x, lane = tid % kWave, w = uniform(tid / kWave), g = lane / 16, r16 = lane % 16;
  const int HT = a.H * a.tiles, cap = a.max_pages * kPage;
  constexpr int kPart = DH + 2;
  __shared__ float sm_o[kWaves][2][kHeads][DH];
  __shared__ float sm_m[kWaves][2][kHeads], sm_l[kWaves][2][kHeads];
  __shared__ int sm_unit[kWaves][2], sm_start[kWaves][2], sm_steps[kWaves][2];  // of a wave's parts: the unit (-1: none), its first step, its steps,
  __shared__ int sm_q0[kWaves][2], sm_heads[kWaves][2];                         // its first query head (of all sequences') and their number
  __shared__ float sm_f[(kBlocksPerUnit + 1) * kHeads], sm_total[kHeads];
  __shared__ int sm_commit, sm_flag[2];
  if (tid < kWaves * 2) (&sm_unit[0][0])[tid] = -1;

  // Lengths.  At most 64 sequences: one lane each, read once.  (An atomic load is performed where it stands.)
  auto read_len = [&](int b) __attribute__((always_inline)) {
    const int L = __hip_atomic_load(&a.cache_len[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    return L < 0 ? 0 : (L > cap ? cap : L);
  };
  auto steps_of = [](int L) __attribute__((always_inline)) { return L > kStep ? (L + kStep - 1) / kStep : 1; };
  const bool by_lane = a.B <= kWave;
  int len_l = 0, total = 0, upto_l = 0, longest = 0;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    len_l = b0 + lane < a.B ? read_len(b0 + lane) : 0;
    upto_l = scan_sum(b0 + lane < a.B ? steps_of(len_l) * HT : 0);
    total += __builtin_amdgcn_readlane(upto_l, kWave - 1);
    longest = len_l > longest ? len_l : longest;
  }
  longest = __builtin_amdgcn_readlane(scan_max(longest), kWave - 1);
  auto len_of = [&](int b) __attribute__((always_inline)) { return by_lane ? __builtin_amdgcn_readlane(len_l, b) : uniform(read_len(b)); };
  __syncthreads();
  int ticket = 0;
  if (by_lane && tid == 0) ticket = reader_ticket(a);
  // The blocks' shares.  Equal ones, not too small, and so that a unit reaches into kBlocksPerUnit + 1 blocks at most; or, where that makes the
  // longest share kCut steps longer at most, each unit by itself in `parts` shares of its own (a cut costs two blocks a trip to memory and
  // one of them two more, about as long as kCut steps take a block).  Units are then numbered `pad` steps apart.
  const int G = static_cast<int>(gridDim.x), even = (total + G - 1) / G, n_max = steps_of(longest), units_all = a.B * HT;
  const int least = (n_max + kBlocksPerUnit - 1) / kBlocksPerUnit, parts = G / units_all < n_max / kLeastCut ? G / units_all : n_max / kLeastCut;
  const int alone = (n_max + (parts > 1 ? parts : 1) - 1) / (parts > 1 ? parts : 1);
  const bool apart = units_all <= G && alone <= even + kCut && alone >= least;
  const int pad = uniform(apart ? (n_max + alone - 1) / alone * alone : 0);
  const int share = uniform(apart ? alone : (even > least ? (even > kMinShare ? even : kMinShare) : (least > kMinShare ? least : kMinShare)));
  if (apart) total = uniform(units_all * pad);
  const int64_t lo64 = static_cast<int64_t>(blockIdx.x) * share;
  const int lo = lo64 < total ? static_cast<int>(lo64) : total;
  int hi = total - lo < share ? total : lo + share;

  // A place in the numbered steps: step s of n of unit (b, h, tile), whose first step is number `start`.  (All of it is wave-uniform, which the
  // compiler has to be told where it cannot see it.)
  struct Place {
    int b, h, tile, s, n, L, start;
  };
  auto find = [&](int pos) __attribute__((always_inline)) {
    Place p{0, 0, 0, 0, 1, 0, 0};
    if (apart) {
      const int unit = uniform(pos / pad), b = uniform(unit / HT), rel = unit - b * HT;
      p.b = b, p.h = uniform(rel / a.tiles), p.tile = rel - p.h * a.tiles, p.s = pos - unit * pad, p.L = len_of(b), p.n = steps_of(p.L), p.start = unit * pad;
      return p;
    }
    int below = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
      int len = len_l, upto = upto_l;
      if (!by_lane) {
        len = b0 + lane < a.B ? read_len(b0 + lane) : 0;
        upto = scan_sum(b0 + lane < a.B ? steps_of(len) * HT : 0);
      }
      const unsigned long long past = __ballot(below + upto > pos);
      if (past) {
        const int l = __builtin_ctzll(past), L = __builtin_amdgcn_readlane(len, l), n = steps_of(L);
        const int in = pos - (below + __builtin_amdgcn_readlane(upto, l) - n * HT), rel = uniform(in / n), h = uniform(rel / a.tiles);
        p = Place{uniform(b0 + l), h, rel - h * a.tiles, in - rel * n, n, L, pos - in + rel * n};
        break;
      }
      below += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return p;
  };
  auto next_unit = [&](Place& p) __attribute__((always_inline)) {  // there is one
    p.start += p.n;
    p.s = 0;
    if (++p.tile < a.tiles) return;
    p.tile = 0;
    if (++p.h < a.H) return;
    p.h = 0;
    p.L = len_of(++p.b);
    p.n = steps_of(p.L);
  };
  auto settle = [&](Place& p) __attribute__((always_inline)) {
    p.b = uniform(p.b), p.h = uniform(p.h), p.tile = uniform(p.tile), p.s = uniform(p.s), p.n = uniform(p.n), p.L = uniform(p.L), p.start = uniform(p.start);
  };

  Place here{0, 0, 0, 0, 1, 0, 0};
  if (apart && lo < hi) {  // of the unit's steps those that there are
    here = find(lo);
    const int end = uniform(here.start + here.n);
    if (hi > end) hi = end > lo ? end : lo;
  }
  const int wlo = uniform(lo + static_cast<int>(static_cast<int64_t>(hi - lo) * w / kWaves));
  const int whi = uniform(lo + static_cast<int>(static_cast<int64_t>(hi - lo) * (w + 1) / kWaves));

  // The new tokens' appends, a wave each in turn (to slots that no one looks at in this launch).
  auto append_some = [&]() __attribute__((always_inline)) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWaves + w; i < static_cast<int64_t>(a.B) * a.H; i += static_cast<int64_t>(G) * kWaves) {
      const int b = uniform(static_cast<int>(i / a.H)), h = uniform(static_cast<int>(i % a.H));
      const bool keep = a.keep_override ? a.keep_override[b] != 0 : keep_from_logits(a.logits, b, a.threshold);
      const int L = len_of(b);
      if (keep && L < cap) append<DH>(a, b, h, L, lane);
    }
  };
  if (wlo >= whi) append_some();
  if (wlo < whi) {
    // The stream of loads: F is the next step to request, page[] its pages' numbers, scalar loads made one step before (the table does not change
    // while this kernel runs; as vector loads they would be waited for with everything that is in flight).
    if (apart) here.s += wlo - lo;
    else here = find(wlo);
    Place F = here;
    settle(F);
    Place C = F;                        // the step to work on
    int left = whi - wlo, to_load = left;
    typedef const int32_t __attribute__((address_space(4)))* ConstI32;
    const LaneAt at = lane_at<DH>(lane);
    int page[2];
    auto load_ids = [&]() __attribute__((always_inline)) {
      const ConstI32 table = (ConstI32)a.block_table + static_cast<size_t>(F.b) * a.max_pages;
      const int last = F.L > 0 ? (F.L - 1) / kPage : 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) page[i] = table[2 * F.s + i < last ? 2 * F.s + i : last];  // past the end: the last page again (masked)
    };
    load_ids();
    // (A request past the wave's end asks for the last step again, so that as many loads are in flight whichever way the loop was taken, and
    // the compiler's waits leave the later ones alone.)
    auto fetch = [&](Step<DH>& st) __attribute__((always_inline)) {
      settle(F);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        load_page<DH>(st, i, a.pages + (static_cast<size_t>(static_cast<uint32_t>(uniform(page[i]))) * a.H + F.h) * mx_page_bytes(DH), at);
      to_load = uniform(to_load) - 1;
      if (to_load > 0) {
        if (++F.s == F.n) next_unit(F);
      }
      load_ids();
    };
    Wave<DH> T;
    uint4 q_next[DH / 32];
    auto load_q = [&](const Place& p) __attribute__((always_inline)) {
      const int heads = a.group - kHeads * p.tile;
      const bf16_t* q = a.q + ((static_cast<size_t>(p.b) * a.H + p.h) * a.group + kHeads * p.tile + r16) * DH + g * (DH / 4);
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) q_next[i] = r16 < heads ? *reinterpret_cast<const uint4*>(q + 8 * i) : make_uint4(0, 0, 0, 0);
    };
    load_q(C);
    bool first = true;                  // C's unit is the wave's first
    auto begin_unit = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < DH / 32; ++i) T.q[i] = q_next[i];
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) T.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      T.m = -INFINITY, T.l = 0.f;
      if (left > C.n - C.s) {           // the wave's next unit
        Place n = C;
        next_unit(n);
        load_q(n);
      }
    };
    int from = C.s;                     // the unit's steps here start at this one
    auto consume = [&](Step<DH>& st) __attribute__((always_inline)) {
      settle(C);
      left = uniform(left), from = uniform(from);
      const int there = C.L - C.s * kStep, tile = C.tile;
      const size_t bh = static_cast<size_t>(C.b) * a.H + C.h;
      typename Wave<DH>::New fresh;
      const bool ends = C.s + 1 == C.n;
      if (ends) T.load_new(fresh, a.k_new + bh * DH, a.v_new + bh * DH, lane);
      if (there > 0) T.attend(st, there, a.scale_log2, lane);
      if (ends) T.attend_new(fresh, a.scale_log2, lane);
      --left;
      if (++C.s < C.n && left > 0) return;
      T.l += __shfl_xor(T.l, 16, kWave);
      T.l += __shfl_xor(T.l, 32, kWave);
      if (C.s == C.n && from == 0) {    // all of the unit
        const float inv = 1.f / T.l;
        bf16_t* o = a.o + (bh * a.group + kHeads * tile + r16) * DH + 4 * g;
        if (r16 < a.group - kHeads * tile) {
#pragma unroll
          for (int i = 0; i < DH / 16; ++i)
            *reinterpret_cast<uint2*>(o + 16 * i) = make_uint2(pack_bf16x2(T.o[i][0] * inv, T.o[i][1] * inv), pack_bf16x2(T.o[i][2] * inv, T.o[i][3] * inv));
        }
      } else {
        const int slot = first ? 0 : 1;
#pragma unroll
        for (int i = 0; i < DH / 16; ++i)
          *reinterpret_cast<float4*>(&sm_o[w][slot][r16][16 * i + 4 * g]) = make_float4(T.o[i][0], T.o[i][1], T.o[i][2], T.o[i][3]);
        if (g == 0) {
          sm_m[w][slot][r16] = T.m;
          sm_l[w][slot][r16] = T.l;
        }
        if (lane == 0) {
          sm_unit[w][slot] = C.b * HT + C.h * a.tiles + tile;
          sm_start[w][slot] = C.start;
          sm_steps[w][slot] = C.n;
          sm_q0[w][slot] = static_cast<int>(bh) * a.group + kHeads * tile;
          sm_heads[w][slot] = a.group - kHeads * tile < kHeads ? a.group - kHeads * tile : kHeads;
        }
      }
      if (left > 0) {
        next_unit(C);
        first = false;
        from = 0;
        begin_unit();
      }
    };
    Step<DH> s0, s1, s2;
    fetch(s0);
    fetch(s1);
    append_some();
    begin_unit();
    for (;;) {
      fetch(s2);
      consume(s0);
      if (left <= 0) break;
      fetch(s0);
      consume(s1);
      if (left <= 0) break;
      fetch(s1);
      consume(s2);
      if (left <= 0) break;
    }
  }
  __syncthreads();
  if (!by_lane && tid == 0) ticket = reader_ticket(a);

  // The waves' parts, in the order of their steps: those of one unit are joined, to its output or to a part of it -- the block's first unit and
  // its last may reach into other blocks.
  constexpr int kParts = 2 * kWaves;
  int reach[2] = {-1, -1};
  // (Read by lanes, one each, and taken from there: as loads one behind the other they took longer than the sums.)
  const int in8 = lane % kParts;
  const int unit_l = (&sm_unit[0][0])[in8], start_l = (&sm_start[0][0])[in8], steps_l = (&sm_steps[0][0])[in8], q0_l = (&sm_q0[0][0])[in8], heads_l = (&sm_heads[0][0])[in8];
  bool known_l = unit_l < 0;
#pragma unroll
  for (int j = 0; j < kParts - 1; ++j) known_l = known_l || (j < in8 && __builtin_amdgcn_readlane(unit_l, j) == unit_l);
  const unsigned firsts = static_cast<unsigned>(__ballot(!known_l)) & ((1u << kParts) - 1);
  for (unsigned todo = firsts; todo; todo &= todo - 1) {
    const int k = __builtin_ctz(todo), unit = __builtin_amdgcn_readlane(unit_l, k);
    const int start = __builtin_amdgcn_readlane(start_l, k), end = start + __builtin_amdgcn_readlane(steps_l, k);
    const unsigned mine = static_cast<unsigned>(__ballot(unit_l == unit)) & ((1u << kParts) - 1);
    const bool whole = start >= lo && end <= hi;
    const int side = start <= lo ? 0 : 1;
    if (!whole) {
      if (side == 0) reach[0] = k;
      else reach[1] = k;
    }
    const int heads = __builtin_amdgcn_readlane(heads_l, k);
    const size_t q0 = static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(q0_l, k)));
    float* const part = a.part + (static_cast<size_t>(blockIdx.x) * 2 + side) * a.part_heads * kPart;
    for (int i = tid; i < heads * (DH / 4); i += kThreads) {
      const int q = i / (DH / 4), c = i % (DH / 4) * 4;
      float m[kParts], M = -INFINITY, l = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < kParts; ++j) {
        m[j] = mine >> j & 1 ? (&sm_m[0][0][0])[j * kHeads + q] : -INFINITY;
        M = fmaxf(M, m[j]);
      }
#pragma unroll
      for (int j = 0; j < kParts; ++j) {
        if (!(mine >> j & 1)) continue;
        const float f = m[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[j] - M);
        const float4 v = *reinterpret_cast<const float4*>(&sm_o[0][0][0][0] + (j * kHeads + q) * DH + c);
        l += f * (&sm_l[0][0][0])[j * kHeads + q];
        o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      }
      if (whole) {
        const float inv = 1.f / l;
        *reinterpret_cast<uint2*>(a.o + (q0 + q) * DH + c) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
      } else {
        st_agent(part + q * kPart + c, o.x);
        st_agent(part + q * kPart + c + 1, o.y);
        st_agent(part + q * kPart + c + 2, o.z);
        st_agent(part + q * kPart + c + 3, o.w);
        if (c == 0) {
          st_agent(part + q * kPart + DH, M);
          st_agent(part + q * kPart + DH + 1, l);
        }
      }
    }
  }
  if (reach[0] >= 0 || reach[1] >= 0) {  // (the same in all threads)
    block_publish();
    auto first_block_of = [&](int k) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(start_l, k) / share; };
    auto blocks_of = [&](int k) __attribute__((always_inline)) {
      return (__builtin_amdgcn_readlane(start_l, k) + __builtin_amdgcn_readlane(steps_l, k) - 1) / share - first_block_of(k) + 1;
    };
    const int k_w = w == 0 ? reach[0] : reach[1], count_at = k_w >= 0 ? first_block_of(k_w) : 0, count_to = k_w >= 0 ? blocks_of(k_w) : 0;
    if (lane == 0 && w < 2) {  // a wave for each of the two
      int last = 0;
      if (k_w >= 0) {
        int32_t* const count = &a.cnt_done[static_cast<size_t>(count_at) * kCnt];
        last = add_agent(count, 1) == count_to - 1;
        if (last) zero_agent(count);
      }
      sm_flag[w] = last;
    }
    __syncthreads();
    for (int side = 0; side < 2; ++side) {
      if (!sm_flag[side]) continue;
      const int k = side == 0 ? reach[0] : reach[1], start = __builtin_amdgcn_readlane(start_l, k), first_block = first_block_of(k), blocks = blocks_of(k);
      const int heads = __builtin_amdgcn_readlane(heads_l, k);
      const size_t q0 = static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(q0_l, k)));
      auto part_of = [&](int j) __attribute__((always_inline)) {  // of block first_block + j: its first unit's, where the unit starts before it or with it
        const int64_t block = first_block + j;
        return a.part + (static_cast<size_t>(block) * 2 + (start <= block * share ? 0 : 1)) * a.part_heads * kPart;
      };
      constexpr int kFew = 6;
      if (blocks <= kFew) {  // all on their way at once
        for (int i = tid; i < heads * (DH / 2); i += kThreads) {
          const int q = i / (DH / 2), c = i % (DH / 2) * 2;
          float m[kFew], l[kFew], v[kFew][2], M = -INFINITY, sum = 0.f, x = 0.f, y = 0.f;
#pragma unroll
          for (int j = 0; j < kFew; ++j) {
            const float* const p = part_of(j < blocks ? j : 0) + q * kPart;
            m[j] = ld_agent(p + DH), l[j] = ld_agent(p + DH + 1), v[j][0] = ld_agent(p + c), v[j][1] = ld_agent(p + c + 1);
          }
#pragma unroll
          for (int j = 0; j < kFew; ++j) {
            if (j >= blocks) m[j] = -INFINITY;
            M = fmaxf(M, m[j]);
          }
#pragma unroll
          for (int j = 0; j < kFew; ++j) {
            if (j >= blocks) continue;
            const float f = m[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[j] - M);
            sum += f * l[j], x += f * v[j][0], y += f * v[j][1];
          }
          const float inv = 1.f / sum;
          *reinterpret_cast<uint32_t*>(a.o + (q0 + q) * DH + c) = pack_bf16x2(x * inv, y * inv);
        }
        continue;
      }
      // the parts' references and sums, a thread each, then their factors
      float* const sm_w = &sm_o[0][0][0][0];  // (the waves' parts have been used)
      for (int i = tid; i < blocks * heads; i += kThreads) {
        const float* const p = part_of(i / heads) + (i % heads) * kPart + DH;
        sm_f[i] = ld_agent(p);
        sm_w[i] = ld_agent(p + 1);
      }
      __syncthreads();
      for (int q = w; q < heads; q += kWaves) {  // a wave a head, a lane a part (and lane 0 the 65th, if there is one)
        const float m0 = lane < blocks ? sm_f[lane * heads + q] : -INFINITY, m1 = lane + kWave < blocks ? sm_f[(lane + kWave) * heads + q] : -INFINITY;
        float M = fmaxf(m0, m1);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, kWave));
        const float f0 = m0 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m0 - M), f1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - M);
        float l = 0.f;
        if (lane < blocks) {
          l = f0 * sm_w[lane * heads + q];
          sm_f[lane * heads + q] = f0;
        }
        if (lane + kWave < blocks) {
          l += f1 * sm_w[(lane + kWave) * heads + q];
          sm_f[(lane + kWave) * heads + q] = f1;
        }
        l = wave_sum(l);
        if (lane == 0) sm_total[q] = l;
      }
      __syncthreads();
      for (int i = tid; i < heads * (DH / 2); i += kThreads) {
        const int q = i / (DH / 2), c = i % (DH / 2) * 2;
        float x = 0.f, y = 0.f;
        int j = 0;
        for (; j + 8 <= blocks; j += 8) {  // eight parts on their way at a time
          float v[8][2];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float* const p = part_of(j + e) + q * kPart + c;
            v[e][0] = ld_agent(p), v[e][1] = ld_agent(p + 1);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float f = sm_f[(j + e) * heads + q];
            x += f * v[e][0], y += f * v[e][1];
          }
        }
        for (; j < blocks; ++j) {
          const float f = sm_f[j * heads + q];
          const float* const p = part_of(j) + q * kPart + c;
          x += f * ld_agent(p), y += f * ld_agent(p + 1);
        }
        const float inv = 1.f / sm_total[q];
        *reinterpret_cast<uint32_t*>(a.o + (q0 + q) * DH + c) = pack_bf16x2(x * inv, y * inv);
      }
      __syncthreads();
    }
  }
  if (tid == 0) sm_commit = last_reader(a, ticket);
  __syncthreads();
  if (sm_commit) commit(a);
}

int tiles_of(int group) { return (group + kHeads - 1) / kHeads; }

// Blocks of a launch: two per compute unit, fewer where there cannot be that many shares.
int64_t blocks_of(int64_t units, int64_t max_pages) {
  const int64_t g = ceil_div(units * (max_pages / 2 + 1), kMinShare);
  return g > kBlocksMax ? kBlocksMax : g;
}
// Counters lie where no other call, of whatever sizes, has parts: a workspace serves calls of different sizes in turn.
constexpr size_t kCounterBytes = static_cast<size_t>(kBlocksMax + kReadCounters + 1) * kCnt * sizeof(int32_t);

}  // namespace
}  // namespace dllava

using namespace dllava;

extern "C" size_t dllava_mx_decode_workspace(int32_t B, int32_t Hq, int32_t H, int32_t Dh, int32_t max_pages_per_seq) {
  if (B <= 0 || H <= 0 || Hq <= 0 || Hq % H != 0 || Dh <= 0 || max_pages_per_seq <= 0) return 256;
  const int group = Hq / H;
  const int64_t blocks = blocks_of(static_cast<int64_t>(B) * H * tiles_of(group), max_pages_per_seq);
  return round_up(kCounterBytes + static_cast<size_t>(blocks) * 2 * (group < kHeads ? group : kHeads) * (Dh + 2) * sizeof(float), 256);
}

extern "C" int dllava_mx_decode_attn_append(const void* q, const void* k_new, const void* v_new, int32_t B, int32_t Hq, const float* logits,
                                            float threshold, const uint8_t* keep_override, const dllava_kv_cache* cache, float scale, void* o,
                                            uint8_t* keep_out, int32_t* err_flag, void* workspace, size_t workspace_bytes, void* stream) {
  DLLAVA_REQUIRE(B >= 0, DLLAVA_EINVAL, "mx_decode: B = %d < 0", B);
  if (int rc = check_mx_cache(cache, "mx_decode")) return rc;
  DLLAVA_REQUIRE(Hq > 0 && Hq % cache->H == 0, DLLAVA_ESHAPE, "mx_decode: Hq = %d must be a positive multiple of the cache's %d heads", Hq, cache->H);
  DLLAVA_REQUIRE(threshold == threshold, DLLAVA_EINVAL, "mx_decode: threshold is NaN");
  DLLAVA_REQUIRE(scale == scale && scale > 0.f && scale < INFINITY, DLLAVA_EINVAL, "mx_decode: bad scale");
  if (B == 0) return DLLAVA_OK;
  DLLAVA_REQUIRE(logits || keep_override, DLLAVA_ENULL, "mx_decode: need logits or keep_override");
  DLLAVA_REQUIRE(q && k_new && v_new && o, DLLAVA_ENULL, "mx_decode: q, k_new, v_new and o are required");
  DLLAVA_REQUIRE(aligned(q, 16) && aligned(k_new, 16) && aligned(v_new, 16) && aligned(o, 16), DLLAVA_EINVAL,
                 "mx_decode: q, k_new, v_new, o must be 16-byte aligned");
  const int tiles = tiles_of(Hq / cache->H);
  const int64_t units = static_cast<int64_t>(B) * cache->H * tiles;
  DLLAVA_REQUIRE(B <= 65535 && static_cast<int64_t>(cache->H) * tiles <= 65535 && units * (cache->max_pages_per_seq / 2 + 1) <= 0x7fffffffLL - 4096 &&
                     static_cast<int64_t>(B) * Hq <= 0x7fffffffLL,
                 DLLAVA_ESHAPE, "mx_decode: B, the number of heads or the cache is too large");
  const size_t need = dllava_mx_decode_workspace(B, Hq, cache->H, cache->Dh, cache->max_pages_per_seq);
  DLLAVA_REQUIRE(workspace && aligned(workspace, 256) && workspace_bytes >= need, DLLAVA_EWORKSPACE,
                 "mx_decode: workspace needs %zu bytes, 256-byte aligned (got %zu)", need, workspace_bytes);
  MxDecodeArgs a{};
  a.q = static_cast<const bf16_t*>(q), a.k_new = static_cast<const bf16_t*>(k_new), a.v_new = static_cast<const bf16_t*>(v_new);
  a.logits = logits, a.keep_override = keep_override, a.threshold = threshold, a.scale_log2 = scale * 1.44269504088896340736f;
  a.pages = static_cast<uint8_t*>(cache->pages), a.block_table = cache->block_table, a.cache_len = cache->cache_len;
  a.max_pages = cache->max_pages_per_seq, a.B = B, a.H = cache->H, a.group = Hq / cache->H, a.tiles = tiles;
  a.part_heads = a.group < kHeads ? a.group : kHeads;
  const int64_t most = blocks_of(units, cache->max_pages_per_seq);
  int64_t blocks = most;
  if (const int v = launch_override(DLLAVA_LAUNCH_DECODE_SPLITS)) blocks = v < most ? v : most;  // tests: fewer blocks, larger shares
  a.cnt_read = static_cast<int32_t*>(workspace);
  a.cnt_done = a.cnt_read + (kReadCounters + 1) * kCnt;
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
  a.o = static_cast<bf16_t*>(o), a.keep_out = keep_out, a.err_flag = err_flag;
  const dim3 grid(static_cast<unsigned>(blocks));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (cache->Dh == 128) hipLaunchKernelGGL(mx_decode_kernel<128>, grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(mx_decode_kernel<64>, grid, dim3(kThreads), 0, st, a);
  DLLAVA_CHECK_LAUNCH("mx_decode_kernel");
  return DLLAVA_OK;
}
