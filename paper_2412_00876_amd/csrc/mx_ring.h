// 32*FI x 32*JT x Kp tile product of two packed 4-bit matrices on the matrix cores: the ring of five half-stage slots of
// gemm_ring.h (see there for its waits, its LDS layout and what shaped it), with v_mfma_scale_f32_16x16x128_f8f6f4.
//
// A 16 x 16 product over 128 columns of 4-bit elements takes as many bytes (16 per lane and operand) and, by its rate, as many
// clocks as one over 32 columns of bfloat16, so a stage is the same 128 bytes of a row: 256 columns, two k-steps.  What is new are
// the scales, one byte per operand's lane and product.  They come straight into registers: a word per lane and fragment holds the
// bytes of the four k-steps of a window of 512 columns (two stages), which the products pick by op_sel.  The words of the next window
// are requested behind the A tile of the stage after next, so the wait for that tile is theirs, too.
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

// A tile's bytes as a buffer: loads take a scalar offset (the stage) and a lane's own, and what lies behind the end reads as zeros.
typedef __amdgpu_buffer_rsrc_t mx_buffer;
__device__ __forceinline__ mx_buffer mx_make_buffer(const void* base, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, static_cast<uint32_t>(bytes < 0xffffffffLL ? bytes : 0xffffffffLL), 0x00020000);
}

__device__ __forceinline__ void mx_move(uint32_t& to, uint32_t from) {
  to = from;
  asm volatile("" : "+v"(to));
}

// ga / gb, w and acc as for gemm_ring_halves; A / B: the codes from the tiles' first rows on; As / Bs: the scales of the tiles' first 16
// rows, first window, and what follows; sa[i] / sb[j]: wave-uniform byte offsets of the scales of the wave's fragments in them;
// windows = Kp / 512 >= 1.
template <int FI, int JT>
__device__ __forceinline__ void mx_ring_halves(mx_buffer A, const uint32_t (&ga)[FI], mx_buffer B, const uint32_t (&gb)[JT], mx_buffer As,
                                               const uint32_t (&sa)[FI], mx_buffer Bs, const uint32_t (&sb)[JT], int windows, DLLAVA_LDS char* smem, int w, ring_f32x4 (&acc)[FI][JT]) {
  static_assert(JT >= 4 && JT <= FI, "a slot holds the rows of either tile");
  constexpr int kMF = FI * JT, kNR = FI + JT;
  constexpr int kStage = kRingRowBytes;  // bytes of a row
  const int lane = threadIdx.x & (kWave - 1);
  const int nk = 2 * windows;
  const uint32_t s0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const uint32_t fo = (lane & 15) * kRingRowBytes + (((lane >> 4) ^ ((lane & 15) >> 1)) * 16);
  const uint32_t a_at = s0 + (w >> 1) * (16 * FI) * kRingRowBytes + fo, b_at = s0 + (w & 1) * (16 * JT) * kRingRowBytes + fo;
  ring_u32x4 ua[FI], ub[JT], va[FI], vb[JT];
  uint32_t xa[FI], xb[JT], na[FI], nb[JT];  // scales of this window and of the next

  // stages past the end re-read the last one (in bounds, unused)
  auto koff = [&](int kt) DLLAVA_INLINE { return static_cast<uint32_t>(kt < nk ? kt : nk - 1) * kStage; };
  auto dma = [&](mx_buffer src, uint32_t lane_offset, uint32_t k, uint32_t slot, int j) DLLAVA_INLINE {
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
  auto scale1 = [&](uint32_t window, auto I) DLLAVA_INLINE {  // one of a window's words
    constexpr int i = decltype(I)::value;
    if constexpr (i < FI)
      na[i] = __builtin_amdgcn_raw_buffer_load_b32(As, 4 * lane, sa[i < FI ? i : 0] + window, 0);
    else
      nb[i - FI] = __builtin_amdgcn_raw_buffer_load_b32(Bs, 4 * lane, sb[i < FI ? 0 : i - FI] + window, 0);
  };
  auto next_scales = [&]() DLLAVA_INLINE {
    static_for<FI>([&](auto I) DLLAVA_INLINE { mx_move(xa[I.value], na[I.value]); });
    static_for<JT>([&](auto I) DLLAVA_INLINE { mx_move(xb[I.value], nb[I.value]); });
    asm volatile("s_nop 3" ::: "memory");  // plain writes before a product
  };
  uint32_t window = 0;  // byte offset of the window whose words are loaded next
  auto kstep = [&](ring_u32x4 (&fa)[FI], ring_u32x4 (&fb)[JT], ring_u32x4 (&ra)[FI], ring_u32x4 (&rb)[JT], uint32_t ab, uint32_t bb,
                   auto S, auto IS_A, uint32_t k, uint32_t slot, auto&& hook) DLLAVA_INLINE {
    constexpr int NL = decltype(IS_A)::value ? FI : JT;
    constexpr int kGap = kMF / NL;
    static_for<kMF>([&](auto Mi) DLLAVA_INLINE {
      constexpr int m = decltype(Mi)::value;
      mx_mfma<decltype(S)::value>(acc[m / JT][m % JT], fa[m / JT], fb[m % JT], xa[m / JT], xb[m % JT]);
      if constexpr (m % 2 == 0 && m / 2 < kNR) read1(ra, rb, ab, bb, std::integral_constant<int, m / 2>{});
      if constexpr (m % kGap == kGap - 1 && m / kGap < NL) {
        if constexpr (decltype(IS_A)::value)
          dma(A, ga[m / kGap], k, slot, m / kGap);
        else
          dma(B, gb[m / kGap], k, slot, m / kGap);
      }
      hook(std::integral_constant<int, kMF - 1 - m>{});
      if constexpr (m % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    });
  };
  static_assert(kMF / 2 >= kNR, "a k-step has room for the reads of the next one");

  constexpr uint32_t kS = 32 * FI * kRingRowBytes;
  static_for<kNR>([&](auto I) DLLAVA_INLINE { scale1(0, I); });
  static_for<JT>([&](auto J) DLLAVA_INLINE { dma(B, gb[J.value], koff(0), 0 * kS, J.value); });
  static_for<FI>([&](auto J) DLLAVA_INLINE { dma(A, ga[J.value], koff(0), 1 * kS, J.value); });
  static_for<JT>([&](auto J) DLLAVA_INLINE { dma(B, gb[J.value], koff(1), 2 * kS, J.value); });
  static_for<FI>([&](auto J) DLLAVA_INLINE { dma(A, ga[J.value], koff(1), 3 * kS, J.value); });
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(JT + FI) : "memory");
  __builtin_amdgcn_s_barrier();
  next_scales();
  asm volatile("s_nop 15" ::: "memory");  // the accumulators' first values, written by plain instructions, before the first product
  static_for<kNR>([&](auto I) DLLAVA_INLINE { read1(ua, ub, a_at + kS, b_at, I); });

  uint32_t ahead = koff(2);  // stage kt + 2 of either matrix
  uint32_t o0 = 0, o1 = kS, o2 = 2 * kS, o3 = 3 * kS, o4 = 4 * kS;  // byte offsets of the slots of B(k), A(k), B(k+1), A(k+1), B(k+2)
  uint32_t ab = (a_at ^ 64u) + o1, bb = (b_at ^ 64u) + o0;
  int left = nk;  // stages still to multiply
  // one stage; P: its number in the window
  auto stage = [&](auto P) DLLAVA_INLINE {
    constexpr int p = decltype(P)::value;
    wait(ua, ub);
    kstep(ua, ub, va, vb, ab, bb, std::integral_constant<int, 2 * p>{}, std::false_type{}, ahead, o4, [&](auto E) DLLAVA_INLINE {
      if constexpr (decltype(E)::value == 4) {
        ab = a_at + o3;
        bb = b_at + o2;
      }
      if constexpr (p == 0 && decltype(E)::value == 2) {  // the next window's scales; past the end the last one's again
        if (left > 2) window += 256;
      }
    });
    // the fragments of the last k-step are in registers: this wave is done with the stage's slots
    wait(va, vb);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(JT) : "memory");
    __builtin_amdgcn_s_barrier();
    kstep(va, vb, ua, ub, ab, bb, std::integral_constant<int, 2 * p + 1>{}, std::true_type{}, ahead, o0, [&](auto E) DLLAVA_INLINE {
      if constexpr (decltype(E)::value == 6) {
        if (left > 3) ahead += kStage;
      }
      if constexpr (decltype(E)::value == 4) {
        const uint32_t t0 = o0, t1 = o1;
        o0 = o2, o1 = o3, o2 = o4, o3 = t0, o4 = t1;
      }
      if constexpr (decltype(E)::value == 2) {
        ab = (a_at ^ 64u) + o1;
        bb = (b_at ^ 64u) + o0;
      }
      if constexpr (p == 0) {  // scale words behind products 0 .. kNR - 1 (counted from the k-step's start: E counts down)
        constexpr int m = kMF - 1 - decltype(E)::value;
        if constexpr (m < kNR) scale1(window, std::integral_constant<int, m>{});
      }
    });
    --left;
  };
  do {
    stage(std::integral_constant<int, 0>{});
    stage(std::integral_constant<int, 1>{});
    next_scales();
  } while (left > 0);
  // the reads and loads issued for stages past the end are drained, and the last products have been written
  wait(ua, ub);
  asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
  static_for<FI>([&](auto I) DLLAVA_INLINE { static_for<JT>([&](auto J) DLLAVA_INLINE { ring_tie_acc(acc[I.value][J.value]); }); });
}

}  // namespace dllava
