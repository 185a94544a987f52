// Tile products of two packed 4-bit matrices on the matrix cores: the ring of five half-stage slots of gemm_ring.h (see there for its
// waits, its LDS layout and what shaped it), with v_mfma_scale_f32_16x16x128_f8f6f4, as ONE stream of stages over all tiles of a block.
//
// A 16 x 16 product over 128 columns of 4-bit elements takes as many bytes (16 per lane and operand) and, by its rate, as many
// clocks as one over 32 columns of bfloat16, so a stage is the same 128 bytes of a row: 256 columns, two k-steps.  What is different:
//  * Scales, one byte per operand's lane and product.  They come straight into registers: a word per lane and fragment holds the
//    bytes of the four k-steps of a window of 512 columns (two stages), which the products pick by op_sel.  The words of the next
//    window are requested behind the A tile of the stage after next, so the wait for that tile is theirs, too.
//  * Tiles are buffers: a load takes a scalar offset (the stage) and a lane's own, which is the same in every tile, and what lies
//    behind a tile's last row reads as zeros.  (As global loads the same requests took two 64-bit additions each, and beside them the
//    compiler waited for ALL outstanding loads before it used a scale.)
//  * A tile of 4096 columns is 16 stages, 20 us, and its ends (first loads, last stores) were another 8 to 18.  A block therefore
//    takes several tiles, and the first two stages of the next one are requested, and the first fragments read, while the last
//    products of this one run: at a tile's end nothing but its results is left to do, straight from the registers.
#pragma once

#include "gemm_ring.h"
#include "mx.h"

namespace dllava {

// product with the scale bytes number S of sa and sb
template <int S>
__device__ __forceinline__ void mx_mfma(ring_f32x4& c, const ring_u32x4& a, const ring_u32x4& b, uint32_t sa, uint32_t sb) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%5,0] op_sel_hi:[%6,%6,0] cbsz:4 blgp:4"
               : "+a"(c)
               : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(S & 1), "n"(S >> 1));
}

typedef __amdgpu_buffer_rsrc_t mx_buffer;
__device__ __forceinline__ mx_buffer mx_make_buffer(const void* base, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, static_cast<uint32_t>(bytes < 0xffffffffLL ? bytes : 0xffffffffLL), 0x00020000);
}
// The operands of a tile, from its first rows on: codes, and scale bytes.
struct MxTileBuffers {
  mx_buffer a, b, as, bs;
};

__device__ __forceinline__ void mx_move(uint32_t& to, uint32_t from) {
  to = from;
  asm volatile("" : "+v"(to));
}
// accumulators' first values, written where they belong
__device__ __forceinline__ void mx_start(ring_f32x4& c) {
  static_for<4>([&](auto I) DLLAVA_INLINE {
    float z;
    asm volatile("v_accvgpr_write_b32 %0, 0" : "=a"(z));
    c[I.value] = z;
  });
  ring_tie_acc(c);
}
__device__ __forceinline__ void mx_start(ring_f32x4& c, const float4& v) {
  const float f[4] = {v.x, v.y, v.z, v.w};
  static_for<4>([&](auto I) DLLAVA_INLINE {
    float z;
    asm volatile("v_accvgpr_write_b32 %0, %1" : "=a"(z) : "v"(f[I.value]));
    c[I.value] = z;
  });
  ring_tie_acc(c);
}

// All tiles of a block.  ga[j] / gb[j]: this lane's byte offsets (row * row bytes + ring_load_chunk_bytes) for its tile loads; windows = Kp / 512 >= 1; w = wave index (wave-uniform).
//   first: the buffers of the first tile;  begin(): a tile begins: sets acc, returns the buffers of the tile after it (or its own again)
//   on_the_way(left): left windows of the tile are left, the one at hand included; loads made here have the time of a stage
//   done(): the tile is complete in acc (its layout: gemm_ring_halves); returns whether there is another
template <int FI, int JT, typename Begin, typename OnTheWay, typename Done>
__device__ __forceinline__ void mx_ring_stream(const MxTileBuffers& first, const uint32_t (&ga)[FI], const uint32_t (&gb)[JT], int windows,
                                               DLLAVA_LDS char* smem, int w, ring_f32x4 (&acc)[FI][JT], Begin&& begin, OnTheWay&& on_the_way, Done&& done) {
  static_assert(JT >= 4 && JT <= FI, "a slot holds the rows of either tile");
  constexpr int kMF = FI * JT, kNR = FI + JT;
  constexpr uint32_t kStage = kRingRowBytes;  // bytes of a row
  const int lane = threadIdx.x & (kWave - 1);
  const uint32_t row_bytes = 2 * kStage * static_cast<uint32_t>(windows), scale_bytes = 256u * static_cast<uint32_t>(windows);
  const uint32_t s0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const uint32_t fo = (lane & 15) * kRingRowBytes + (((lane >> 4) ^ ((lane & 15) >> 1)) * 16);
  const uint32_t a_at = s0 + (w >> 1) * (16 * FI) * kRingRowBytes + fo, b_at = s0 + (w & 1) * (16 * JT) * kRingRowBytes + fo;
  ring_u32x4 ua[FI], ub[JT], va[FI], vb[JT];
  uint32_t xa[FI], xb[JT], na[FI], nb[JT];  // scales of this window and of the next

  // the streams of requests: codes (tile and stage), scales (tile and window)
  MxTileBuffers N = begin();  // (the tile after the one whose products run; the requests are two stages ahead of those)
  mx_buffer A = first.a, B = first.b, As = first.as, Bs = first.bs;
  uint32_t ahead = 0, window = 0;  // byte offsets of the stage and of the window that are requested next
  auto next_stage = [&]() DLLAVA_INLINE {
    ahead += kStage;
    if (ahead == row_bytes) {
      ahead = 0;
      A = N.a, B = N.b;
    }
  };
  auto next_window = [&]() DLLAVA_INLINE {
    window += 256;
    if (window == scale_bytes) {
      window = 0;
      As = N.as, Bs = N.bs;
    }
  };

  auto dma = [&](const mx_buffer& src, uint32_t lane_offset, uint32_t k, uint32_t slot, int j) DLLAVA_INLINE {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (DLLAVA_LDS void*)(smem + slot + (w + 4 * j) * 1024), 16, lane_offset, k, 0, 0);
  };
  auto read1 = [&](ring_u32x4 (&fa)[FI], ring_u32x4 (&fb)[JT], uint32_t ab, uint32_t bb, auto I) DLLAVA_INLINE {
    constexpr int i = decltype(I)::value;
    if constexpr (i < FI)
      fa[i] = ring_lds_read16<i * 16 * kRingRowBytes>(ab);
    else
      fb[i - FI] = ring_lds_read16<(i - FI) * 16 * kRingRowBytes>(bb);
  };
  auto wait = [&](ring_u32x4 (&fa)[FI], ring_u32x4 (&fb)[JT]) DLLAVA_INLINE {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    ring_tie(fa);
    ring_tie(fb);
  };
  uint32_t at = 0;
  auto scale1 = [&](auto I) DLLAVA_INLINE {  // one of the words of the window that is requested next, in turn
    constexpr int i = decltype(I)::value;
    if constexpr (i == 0) at = window + static_cast<uint32_t>(FI * (w >> 1)) * scale_bytes;
    if constexpr (i == FI) at = window + static_cast<uint32_t>(JT * (w & 1)) * scale_bytes;
    if constexpr (i < FI)
      na[i] = __builtin_amdgcn_raw_buffer_load_b32(As, 4 * lane, at, 0);
    else
      nb[i - FI] = __builtin_amdgcn_raw_buffer_load_b32(Bs, 4 * lane, at, 0);
    at += scale_bytes;
  };
  auto take_scales = [&]() DLLAVA_INLINE {
    static_for<FI>([&](auto I) DLLAVA_INLINE { mx_move(xa[I.value], na[I.value]); });
    static_for<JT>([&](auto I) DLLAVA_INLINE { mx_move(xb[I.value], nb[I.value]); });
    asm volatile("s_nop 3" ::: "memory");  // plain writes before a product
  };
  auto kstep = [&](ring_u32x4 (&fa)[FI], ring_u32x4 (&fb)[JT], ring_u32x4 (&ra)[FI], ring_u32x4 (&rb)[JT], uint32_t ab, uint32_t bb,
                   auto S, auto IS_A, uint32_t slot, auto&& hook) DLLAVA_INLINE {
    constexpr int NL = decltype(IS_A)::value ? FI : JT;
    constexpr int kGap = kMF / NL;
    static_for<kMF>([&](auto Mi) DLLAVA_INLINE {
      constexpr int m = decltype(Mi)::value;
      mx_mfma<decltype(S)::value>(acc[m / JT][m % JT], fa[m / JT], fb[m % JT], xa[m / JT], xb[m % JT]);
      if constexpr (m % 2 == 0 && m / 2 < kNR) read1(ra, rb, ab, bb, std::integral_constant<int, m / 2>{});
      if constexpr (m % kGap == kGap - 1 && m / kGap < NL) {
        if constexpr (decltype(IS_A)::value)
          dma(A, ga[m / kGap], ahead, slot, m / kGap);
        else
          dma(B, gb[m / kGap], ahead, slot, m / kGap);
      }
      hook(std::integral_constant<int, kMF - 1 - m>{});
      if constexpr (m % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    });
  };
  static_assert(kMF / 2 >= kNR, "a k-step has room for the reads of the next one");

  // Half-stages in ring order, as in gemm_ring_halves: B(0), A(0), B(1), A(1), ...; iteration k multiplies stage k, requests B(k+2)
  // behind its first k-step and A(k+2) behind its second, which its barrier precedes.
  constexpr uint32_t kS = 32 * FI * kRingRowBytes;
  static_for<kNR>([&](auto I) DLLAVA_INLINE { scale1(I); });
  next_window();
  static_for<JT>([&](auto J) DLLAVA_INLINE { dma(B, gb[J.value], ahead, 0 * kS, J.value); });
  static_for<FI>([&](auto J) DLLAVA_INLINE { dma(A, ga[J.value], ahead, 1 * kS, J.value); });
  next_stage();
  static_for<JT>([&](auto J) DLLAVA_INLINE { dma(B, gb[J.value], ahead, 2 * kS, J.value); });
  static_for<FI>([&](auto J) DLLAVA_INLINE { dma(A, ga[J.value], ahead, 3 * kS, J.value); });
  next_stage();
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(JT + FI) : "memory");
  __builtin_amdgcn_s_barrier();
  take_scales();
  asm volatile("s_nop 7" ::: "memory");
  static_for<kNR>([&](auto I) DLLAVA_INLINE { read1(ua, ub, a_at + kS, b_at, I); });

  uint32_t o0 = 0, o1 = kS, o2 = 2 * kS, o3 = 3 * kS, o4 = 4 * kS;  // byte offsets of the slots of B(k), A(k), B(k+1), A(k+1), B(k+2)
  uint32_t ab = (a_at ^ 64u) + o1, bb = (b_at ^ 64u) + o0;
  int left = windows;
  // one stage; P: its number in the window
  auto stage = [&](auto P) DLLAVA_INLINE {
    constexpr int p = decltype(P)::value;
    wait(ua, ub);
    kstep(ua, ub, va, vb, ab, bb, std::integral_constant<int, 2 * p>{}, std::false_type{}, o4, [&](auto E) DLLAVA_INLINE {
      if constexpr (decltype(E)::value == 4) {
        ab = a_at + o3;
        bb = b_at + o2;
      }
    });
    // the fragments of the last k-step are in registers: this wave is done with the stage's slots
    wait(va, vb);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(JT) : "memory");
    __builtin_amdgcn_s_barrier();
    kstep(va, vb, ua, ub, ab, bb, std::integral_constant<int, 2 * p + 1>{}, std::true_type{}, o0, [&](auto E) DLLAVA_INLINE {
      constexpr int m = kMF - 1 - decltype(E)::value;  // (behind product m)
      if constexpr (p == 0 && m < kNR) scale1(std::integral_constant<int, m>{});
      if constexpr (p == 0 && m == kNR) on_the_way(left);
      if constexpr (decltype(E)::value == 4) {
        const uint32_t t0 = o0, t1 = o1;
        o0 = o2, o1 = o3, o2 = o4, o3 = t0, o4 = t1;
      }
      if constexpr (decltype(E)::value == 2) {
        ab = (a_at ^ 64u) + o1;
        bb = (b_at ^ 64u) + o0;
      }
      if constexpr (decltype(E)::value == 0) {
        next_stage();
        if constexpr (p == 0) next_window();
      }
    });
  };
  for (;;) {
    left = windows;
    do {
      stage(std::integral_constant<int, 0>{});
      stage(std::integral_constant<int, 1>{});
      take_scales();
    } while (--left > 0);
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");  // the last products, whose latency the compiler does not know, are written
    static_for<FI>([&](auto I) DLLAVA_INLINE { static_for<JT>([&](auto J) DLLAVA_INLINE { ring_tie_acc(acc[I.value][J.value]); }); });
    if (!done()) break;
    N = begin();
    if (windows == 1) A = N.a, B = N.b, As = N.as, Bs = N.bs;  // tiles so short that the requests are a tile ahead
    asm volatile("s_nop 7" ::: "memory");  // acc before the first product
  }
  // what was requested and read past the end is drained
  wait(ua, ub);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

}  // namespace dllava
