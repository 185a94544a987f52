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
// The S * kWaves waves of (sequence, K/V head) take the steps in turn.  Blocks of one (sequence, head) hand their parts over through the
// workspace, the last to arrive adds them up in the order of their numbers.  cache_len[b] moves when the last block of the sequence
// has read it; the new token goes to a slot that no block of this launch looks at (tokens behind the length are masked by position,
// and their scales are replaced, whatever they hold).
#include "mx.h"

namespace dllava {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kHeads = 16;      // query heads of a block, at most
constexpr int kStep = 2 * kPage;
constexpr int kMaxSplit = 64;
constexpr int kCnt = 64;        // int32 slots per counter: a memory line each
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
  int32_t n_split;
  int32_t* cnt_done;  // [B * H * tiles] blocks whose part is published (n_split > 1)
  int32_t* cnt_b;     // [B] (head, tile)s whose blocks have all read cache_len
  float* part;        // [B * H * tiles][n_split][part_heads][DH + 2]
  int32_t part_heads; // query heads of a block, at most
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
  uint32_t vs[2][4];       // scale bytes of the blocks of tokens 4g .. 4g + 3, a word a token (head size 64: its lower half)
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

template <int DH>
__device__ __forceinline__ void load_page(Step<DH>& s, int i, const uint8_t* page, int lane) {
  constexpr int kBlocks = DH / 32;
  const int g = lane / 16, r16 = lane % 16;
  load_words(s.k[i], page + r16 * (DH / 2) + g * (DH / 8));
  load_words(s.v[i], page + 8 * DH + lane * (DH / 8));
  s.ks[i] = page[16 * DH + r16 * kBlocks + g * kBlocks / 4];
  const uint8_t* vs = page + 16 * DH + DH / 2 + g * 4 * kBlocks;
  if constexpr (DH == 128) {
    load_words(s.vs[i], vs);
  } else {
    uint32_t two[2];
    load_words(two, vs);
    s.vs[i][0] = two[0], s.vs[i][1] = two[0] >> 16, s.vs[i][2] = two[1], s.vs[i][3] = two[1] >> 16;
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

  // One step; there: tokens of it that exist (32: all).
  template <bool MASKED>
  __device__ __forceinline__ void attend(Step<DH>& s, int there, float scale_log2, int lane) {
    const int g = lane / 16;
    float x[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < DH / 32; ++w) c = product(mx_decode8(s.k[i][w], s.ks[i] << 23), q[w], c);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[4 * i + e] = c[e] * scale_log2;
        if (MASKED && kPage * i + 4 * g + e >= there) {
          x[4 * i + e] = -INFINITY;
          s.vs[i][e] = 0x7f7f7f7fu;  // a finite scale, whatever the slot holds: the codes are finite, and the probability is zero
        }
      }
    }
    const uint4 p = softmax(x);
    // block m, half h: columns 32 m + 16 h + r16.  Byte m of token j's word (DH 128; head size 64: bytes 2 (j % 2) + m of word j / 2)
    // holds both halves, which the two pages' tokens are sorted into.
#pragma unroll
    for (int m_ = 0; m_ < DH / 32; ++m_) {
      uint32_t both[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t sb = m_ == 0 ? mx_scale_bits<0>(s.vs[i][j]) : m_ == 1 ? mx_scale_bits<1>(s.vs[i][j]) : m_ == 2 ? mx_scale_bits<2>(s.vs[i][j]) : mx_scale_bits<3>(s.vs[i][j]);
          const int byte = DH == 128 ? m_ : 2 * (j % 2) + m_;
          const uint32_t c = s.v[i][DH == 128 ? j : j / 2];
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
  __device__ __forceinline__ void attend_new(const bf16_t* k, const bf16_t* v, float scale_log2, int lane) {
    const int g = lane / 16, r16 = lane % 16;
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < DH / 32; ++w) {
      const uint4 piece = *reinterpret_cast<const uint4*>(k + g * (DH / 4) + 8 * w);
      c = product(r16 == 0 ? piece : make_uint4(0, 0, 0, 0), q[w], c);
    }
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = -INFINITY;
    if (g == 0) x[0] = c[0] * scale_log2;
    const uint4 p = softmax(x);
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) o[i] = product(make_uint4(g == 0 ? v[16 * i + r16] : 0u, 0, 0, 0), p, o[i]);
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

template <int DH>
__global__ __launch_bounds__(kThreads) void mx_decode_kernel(MxDecodeArgs a) {
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave, g = lane / 16, r16 = lane % 16;
  const int split = blockIdx.x, h = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles, b = blockIdx.z;
  const int S = a.n_split;
  const size_t unit = (static_cast<size_t>(b) * a.H + h) * a.tiles + tile;
  const int heads = a.group - kHeads * tile < kHeads ? a.group - kHeads * tile : kHeads;  // of this block
  const size_t q0 = (static_cast<size_t>(b) * a.H + h) * a.group + kHeads * tile;       // the first of them in q and o

  // (an atomic load: read once, though cache_len is written at the launch's end)
  const int L0 = __hip_atomic_load(&a.cache_len[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  const int cap = a.max_pages * kPage, L = L0 < 0 ? 0 : (L0 > cap ? cap : L0);
  const int steps = (L + kStep - 1) / kStep, last_page = L > 0 ? (L - 1) / kPage : 0;
  const int32_t* table = a.block_table + static_cast<size_t>(b) * a.max_pages;

  Wave<DH> T;
#pragma unroll
  for (int i = 0; i < DH / 32; ++i)
    T.q[i] = r16 < heads ? *reinterpret_cast<const uint4*>(a.q + (q0 + r16) * DH + g * (DH / 4) + 8 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < DH / 16; ++i) T.o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  T.m = -INFINITY, T.l = 0.f;

  const int stride = S * kWaves;
  auto load = [&](Step<DH>& s, int step) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = 2 * step + i < last_page ? 2 * step + i : last_page;  // past the end: the last page again (masked)
      load_page<DH>(s, i, a.pages + (static_cast<size_t>(table[p]) * a.H + h) * mx_page_bytes(DH), lane);
    }
  };
  Step<DH> cur, next;
  int step = split * kWaves + w;
  if (step < steps) load(cur, step);
  if (split == 0 && w == 0) T.attend_new(a.k_new + (static_cast<size_t>(b) * a.H + h) * DH, a.v_new + (static_cast<size_t>(b) * a.H + h) * DH, a.scale_log2, lane);
  const bool keep = a.keep_override ? a.keep_override[b] != 0 : keep_from_logits(a.logits, b, a.threshold);
  if (split == 0 && tile == 0 && w == kWaves - 1 && keep && L0 >= 0 && L0 < cap) append<DH>(a, b, h, L0, lane);
  while (step < steps) {
    const int to = step + stride;
    if (to < steps) load(next, to);
    const int there = L - step * kStep;
    if (there >= kStep)
      T.template attend<false>(cur, kStep, a.scale_log2, lane);
    else
      T.template attend<true>(cur, there, a.scale_log2, lane);
    cur = next;
    step = to;
  }

  // the waves of the block
  __shared__ float sm_o[kWaves][kHeads][DH];
  __shared__ float sm_m[kWaves][kHeads], sm_l[kWaves][kHeads];
  __shared__ int sm_flag;
  T.l += __shfl_xor(T.l, 16, kWave);
  T.l += __shfl_xor(T.l, 32, kWave);
  if (r16 < heads) {
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) *reinterpret_cast<float4*>(&sm_o[w][r16][16 * i + 4 * g]) = make_float4(T.o[i][0], T.o[i][1], T.o[i][2], T.o[i][3]);
    if (g == 0) {
      sm_m[w][r16] = T.m;
      sm_l[w][r16] = T.l;
    }
  }
  __syncthreads();  // every wave has read cache_len, too
  constexpr int kPart = DH + 2;
  const size_t part_size = static_cast<size_t>(a.part_heads) * kPart;
  float* const parts = a.part + unit * S * part_size;
  for (int i = tid; i < heads * DH; i += kThreads) {
    const int q = i / DH, c = i % DH;
    float M = sm_m[0][q], l = 0.f, o = 0.f;
#pragma unroll
    for (int k = 1; k < kWaves; ++k) M = fmaxf(M, sm_m[k][q]);
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float f = sm_m[k][q] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm_m[k][q] - M);
      l += f * sm_l[k][q];
      o += f * sm_o[k][q][c];
    }
    if (S == 1) {
      a.o[(q0 + q) * DH + c] = f32_to_bf16(o / l);
    } else {
      float* const part = parts + split * part_size + q * kPart;
      st_agent(part + c, o);
      if (c == 0) {
        st_agent(part + DH, M);
        st_agent(part + DH + 1, l);
      }
    }
  }
  bool done = S == 1;  // this block's (head, tile) is complete, and every block of it has read cache_len
  if (S > 1) {
    block_publish();
    if (tid == 0) {
      sm_flag = add_agent(&a.cnt_done[unit * kCnt], 1) == S - 1;
      if (sm_flag) zero_agent(&a.cnt_done[unit * kCnt]);
    }
    __syncthreads();
    done = sm_flag != 0;
    if (done) {
      for (int i = tid; i < heads * DH; i += kThreads) {
        const int q = i / DH, c = i % DH;
        float M = -INFINITY;
        for (int s = 0; s < S; ++s) M = fmaxf(M, ld_agent(parts + s * part_size + q * kPart + DH));
        float l = 0.f, o = 0.f;
        for (int s = 0; s < S; ++s) {
          const float* const part = parts + s * part_size + q * kPart;
          const float m = ld_agent(part + DH), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
          l += f * ld_agent(part + DH + 1);
          o += f * ld_agent(part + c);
        }
        a.o[(q0 + q) * DH + c] = f32_to_bf16(o / l);
      }
    }
  }
  if (done && tid == 0 && add_agent(&a.cnt_b[b * kCnt], 1) == a.H * a.tiles - 1) {
    zero_agent(&a.cnt_b[b * kCnt]);
    if (a.keep_out) a.keep_out[b] = keep ? 1 : 0;
    if (keep) {
      if (L0 >= 0 && L0 < cap) a.cache_len[b] = L0 + 1;
      else if (a.err_flag) *a.err_flag = 1;
    }
  }
}

int tiles_of(int group) { return (group + kHeads - 1) / kHeads; }

// Blocks per (sequence, K/V head, tile) that the workspace has room for.
int split_room(int64_t units) {
  const int64_t s = 2048 / units;
  return s < 1 ? 1 : (s > kMaxSplit ? kMaxSplit : static_cast<int>(s));
}
// Those of a launch: enough for the chip, each wave with a step to take.
int pick_split(int64_t units, int max_pages) {
  int64_t s = 1024 / units;
  const int64_t useful = ceil_div(max_pages, 2 * kWaves), room = split_room(units);
  if (s > useful) s = useful;
  if (const int v = launch_override(DLLAVA_LAUNCH_DECODE_SPLITS)) s = v;
  if (s > room) s = room;
  return s < 1 ? 1 : static_cast<int>(s);
}

size_t counter_bytes(int64_t B, int64_t units) { return static_cast<size_t>(B + units) * kCnt * sizeof(int32_t); }
size_t part_bytes(int64_t units, int group, int Dh) {
  const int room = split_room(units);
  return room == 1 ? 0 : static_cast<size_t>(units) * room * (group < kHeads ? group : kHeads) * (Dh + 2) * sizeof(float);
}

}  // namespace
}  // namespace dllava

using namespace dllava;

extern "C" size_t dllava_mx_decode_workspace(int32_t B, int32_t Hq, int32_t H, int32_t Dh, int32_t max_pages_per_seq) {
  if (B <= 0 || H <= 0 || Hq <= 0 || Hq % H != 0 || Dh <= 0) return 256;
  (void)max_pages_per_seq;
  const int64_t units = static_cast<int64_t>(B) * H * tiles_of(Hq / H);
  return round_up(counter_bytes(B, units) + part_bytes(units, Hq / H, Dh), 256);
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
  DLLAVA_REQUIRE(B <= 65535 && static_cast<int64_t>(cache->H) * tiles <= 65535, DLLAVA_ESHAPE, "mx_decode: B or the number of heads is too large");
  const size_t need = dllava_mx_decode_workspace(B, Hq, cache->H, cache->Dh, cache->max_pages_per_seq);
  DLLAVA_REQUIRE(workspace && aligned(workspace, 256) && workspace_bytes >= need, DLLAVA_EWORKSPACE,
                 "mx_decode: workspace needs %zu bytes, 256-byte aligned (got %zu)", need, workspace_bytes);
  MxDecodeArgs a{};
  a.q = static_cast<const bf16_t*>(q), a.k_new = static_cast<const bf16_t*>(k_new), a.v_new = static_cast<const bf16_t*>(v_new);
  a.logits = logits, a.keep_override = keep_override, a.threshold = threshold, a.scale_log2 = scale * 1.44269504088896340736f;
  a.pages = static_cast<uint8_t*>(cache->pages), a.block_table = cache->block_table, a.cache_len = cache->cache_len;
  a.max_pages = cache->max_pages_per_seq, a.B = B, a.H = cache->H, a.group = Hq / cache->H, a.tiles = tiles;
  a.part_heads = a.group < kHeads ? a.group : kHeads;
  const int64_t units = static_cast<int64_t>(B) * cache->H * tiles;
  a.n_split = pick_split(units, cache->max_pages_per_seq);
  a.cnt_b = static_cast<int32_t*>(workspace);
  a.cnt_done = a.cnt_b + static_cast<size_t>(B) * kCnt;
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + counter_bytes(B, units));
  a.o = static_cast<bf16_t*>(o), a.keep_out = keep_out, a.err_flag = err_flag;
  const dim3 grid(static_cast<unsigned>(a.n_split), static_cast<unsigned>(cache->H * tiles), static_cast<unsigned>(B));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (cache->Dh == 128) hipLaunchKernelGGL(mx_decode_kernel<128>, grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(mx_decode_kernel<64>, grid, dim3(kThreads), 0, st, a);
  DLLAVA_CHECK_LAUNCH("mx_decode_kernel");
  return DLLAVA_OK;
}
