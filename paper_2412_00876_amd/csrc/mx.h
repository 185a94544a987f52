// Microscaled 4-bit floating point (include/dllava_mx.h has the format): rounding, reading, and where things lie.
#pragma once

#include "common.h"
#include "dllava_mx.h"

namespace dllava {

constexpr int kMxBlock = 32;    // elements that share a scale
constexpr int kMxWindow = 512;  // columns of a packed matrix whose scales lie together: 16 blocks, four in each fourth of a wave
constexpr int kMxTile = 16;     // rows of a packed matrix whose scales lie together

inline int64_t mx_padded(int64_t K) { return (K + kMxWindow - 1) / kMxWindow * kMxWindow; }
inline size_t mx_code_bytes(int64_t M, int64_t K) { return static_cast<size_t>(M) * static_cast<size_t>(mx_padded(K) / 2); }
inline size_t mx_scale_bytes(int64_t M, int64_t K) {
  return static_cast<size_t>(ceil_div(M, kMxTile)) * kMxTile * static_cast<size_t>(mx_padded(K) / kMxBlock);
}

// The scale byte of a block from the bits of its largest magnitude (an infinity's or NaN's where it holds one).  Adding 0x1fffff
// carries into the exponent where the fraction is above 0x600000, that is 1.75.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
  const int s = static_cast<int>((amax_bits + 0x1fffffu) >> 23) - 2;
  return amax_bits >= 0x7f800000u ? 255u : static_cast<uint32_t>(s < 1 ? 1 : (s > 252 ? 252 : s));
}
__device__ __forceinline__ uint32_t mx_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// Eight values to eight codes, the first in the lowest four bits.  The conversion divides by the power of two in `scale`'s exponent,
// rounds to nearest even and saturates (its results were compared with the format's definition for all bfloat16 values at four scales and
// four million float32 values at others).
__device__ __forceinline__ uint32_t mx_encode8(const float* v, uint32_t scale_byte) {
  const float s = __uint_as_float(scale_byte << 23);
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
}
// The two codes of byte SEL of c as bfloat16, the lower one in the lower half.  Of `scale` the conversion takes the eight exponent
// bits alone (sign and fraction may be anything: a scale byte is shifted into place and what is beside it stays); all ones give NaN.
template <int SEL>
__device__ __forceinline__ uint32_t mx_decode2(uint32_t c, uint32_t scale_bits) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, __uint_as_float(scale_bits), SEL));
}
// byte I of w where a float's exponent stands (other bits: whatever is beside it)
template <int I>
__device__ __forceinline__ uint32_t mx_scale_bits(uint32_t w) {
  return I == 3 ? w >> 1 : w << (23 - 8 * I);
}
// eight codes to eight bfloat16 values
__device__ __forceinline__ uint4 mx_decode8(uint32_t c, uint32_t scale_bits) {
  return make_uint4(mx_decode2<0>(c, scale_bits), mx_decode2<1>(c, scale_bits), mx_decode2<2>(c, scale_bits), mx_decode2<3>(c, scale_bits));
}

// Eight consecutive elements of a row as float32.
__device__ __forceinline__ void mx_load8(const float* p, float* f) {
  const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
  Elem<float>::unpack(a, f);
  Elem<float>::unpack(b, f + 4);
}
__device__ __forceinline__ void mx_load8(const bf16_t* p, float* f) { Elem<bf16_t>::unpack(*reinterpret_cast<const uint4*>(p), f); }
// bfloat16 values of two-a-word pairs, stored in either type (exact)
__device__ __forceinline__ void mx_store8(bf16_t* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }
__device__ __forceinline__ void mx_store8(float* p, const uint4& v) {
  float f[8];
  Elem<bf16_t>::unpack(v, f);
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
// The largest magnitude's bits over the four lanes that hold a block (lanes 4i .. 4i + 3).
__device__ __forceinline__ uint32_t mx_block_amax(const float* v) {
  uint32_t m = mx_magnitude(v[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    const uint32_t x = mx_magnitude(v[e]);
    m = x > m ? x : m;
  }
  uint32_t o = __builtin_amdgcn_update_dpp(0, m, 0xB1, 0xf, 0xf, true);  // quad_perm [1,0,3,2]
  m = o > m ? o : m;
  o = __builtin_amdgcn_update_dpp(0, m, 0x4E, 0xf, 0xf, true);  // quad_perm [2,3,0,1]
  return o > m ? o : m;
}

int check_mx_cache(const dllava_kv_cache* c, const char* who);  // host validation of a cache in 4 bits (mx_cache.hip)
__host__ __device__ constexpr int mx_page_bytes(int Dh) { return 17 * Dh; }  // of one head

}  // namespace dllava
