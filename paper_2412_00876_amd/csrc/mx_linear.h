// What the linear layers with 4-bit weights share: their arguments and what becomes of a sum.
#pragma once

#include "mx.h"

namespace dllava {

struct MxLinearArgs {
  const uint8_t* Wc;   // codes [N][Kp / 2]
  const uint8_t* Ws;   // scale bytes
  const uint8_t* Xc;   // rows: codes and scale bytes, or
  const uint8_t* Xs;
  const bf16_t* X;     // bfloat16 values
  int64_t ldx;
  int64_t M;
  int32_t N, K;
  int32_t windows;     // Kp / 512
  const float* bias;
  const bf16_t* R;     // residual or gate, laid out as Y (may be Y), or null
  bf16_t* Y;
  int64_t ldy;
  int32_t act;         // 1: GELU; 2: times SiLU(R) instead of plus R
};

// Four results, with the bias in them, to what is stored; r: the residual's or the gate's four values, where there are any.
__device__ __forceinline__ uint2 mx_result(const MxLinearArgs& a, float4 v, const uint2& p) {
  if (a.act == 1) v = make_float4(gelu_erf_fast(v.x), gelu_erf_fast(v.y), gelu_erf_fast(v.z), gelu_erf_fast(v.w));
  if (a.R) {
    const float r[4] = {bf16lo_to_f32(p.x), bf16hi_to_f32(p.x), bf16lo_to_f32(p.y), bf16hi_to_f32(p.y)};
    if (a.act == 2) {
      auto silu = [](float x) { return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * x)); };
      v.x *= silu(r[0]), v.y *= silu(r[1]), v.z *= silu(r[2]), v.w *= silu(r[3]);
    } else {
      v.x += r[0], v.y += r[1], v.z += r[2], v.w += r[3];
    }
  }
  return make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}
// The results of features n .. n + 3 of row m, each rounded once.
__device__ __forceinline__ void mx_store_results(const MxLinearArgs& a, int64_t m, int n, float4 v) {
  if (a.bias) {
    const float4 b = *reinterpret_cast<const float4*>(a.bias + n);
    v.x += b.x, v.y += b.y, v.z += b.z, v.w += b.w;
  }
  const int64_t at = m * a.ldy + n;
  *reinterpret_cast<uint2*>(a.Y + at) = mx_result(a, v, a.R ? *reinterpret_cast<const uint2*>(a.R + at) : make_uint2(0u, 0u));
}

}  // namespace dllava
