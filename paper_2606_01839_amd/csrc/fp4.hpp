// Blocks of a pool that holds K and V in 4 bits (the MX element e2m1 with power-of-two scales), shared by
// the kernels that write and read them.
//
// A block of (layer, page, kv head) is 17 D bytes (D = 128: 2176 against 8192 in bf16), read by a wave with
// lane = 16 qd + c, NW = D / 32 words (of eight 4-bit codes) a lane and part:
//   K    [qd 4][key c 16][NW words]: dims (D/4) qd .. (D/4) qd + D/4 - 1 of key c
//   V    [qd 4][c 16][NW words]: for dim tile t = 0 .. D/16 - 1 the keys 4 qd .. 4 qd + 3 of dim 16 t + c
//        (tile t in half t % 2 of word t / 2)
//   scales [D bytes]: K [group of 32 dims][key], V [key], then zeros. Byte e stands for 2^(e - 127).
// So one 16- (D = 64: 8-) byte load a lane reads a page's K, one its V, each 1 KiB (512 bytes) of
// consecutive bytes; both are matrix-core operands after conversion alone: 8 dims of a key (K), 4 keys of
// a dim (V). K has a scale for every 32 dims of a token, which the conversion instruction applies; V one for
// every token, since a lane's V values are of different tokens: a scale the softmax weight can take, where one
// for every 32 dims would take D / 32 scaled copies of the weights. (Rounding error of V, 2-norm, with
// normal / Laplace values: 0.113 / 0.134 of the values with one scale for 128 dims, 0.115 / 0.127 for 32.)
// The padding to 17 D keeps blocks on 64-byte boundaries; without it they would be 4% (D = 64: 1.5%) smaller.
#pragma once

#include "device_common.hpp"

namespace cs {

template <int D>
struct Fp4Block {
  static constexpr int kWords = D / 32;                 // words of codes a lane holds of K, and of V
  static constexpr int kK = 0, kV = 8 * D;              // byte offsets
  static constexpr int kKScale = 16 * D, kVScale = kKScale + D / 2, kPad = kVScale + kPageTokens;
  static constexpr int kBytes = 17 * D;
  // byte offset of the codes of dims 8 ch .. 8 ch + 7 of token t (K part, one word)
  static __device__ __forceinline__ int k_word(int t, int ch) {
    return kK + ((ch / kWords) * kPageTokens + t) * (4 * kWords) + (ch % kWords) * 4;
  }
  // K scale of the group of 32 dims that lane 16 qd + c holds dims of
  static __device__ __forceinline__ int k_scale(int qd, int c) {
    return kKScale + (D == 128 ? qd : qd >> 1) * kPageTokens + c;
  }
  static __device__ __forceinline__ size_t at(int layer, int page, int head, int64_t n_pages, int n_kv_heads) {
    return ((static_cast<size_t>(layer) * static_cast<size_t>(n_pages) + static_cast<size_t>(page)) *
                static_cast<size_t>(n_kv_heads) + static_cast<size_t>(head)) * static_cast<size_t>(kBytes);
  }
};

// The scale byte of a group whose largest magnitude has the given fp32 bits (sign cleared): the power of
// two floor(log2 a) - 2, so that a / scale lies in [4, 8) and e2m1's largest value, 6, is reached; at
// least 2^-126. A group with an infinity or NaN gets 255, which reads back as NaN.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t abs_bits) {
  const int e = static_cast<int>(abs_bits >> 23);
  return e == 255 ? 255u : static_cast<uint32_t>(max(e - 2, 1));
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
// 2^(byte - 127) (0 for the zero byte of an unwritten slot, infinity for 255)
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// byte b of w as such a scale
__device__ __forceinline__ float fp4_scale_of(uint32_t w, int b) {
  return __uint_as_float(b == 0 ? (w << 23) & 0x7F800000u : (w >> (8 * b)) << 23 & 0x7F800000u);
}

// Two codes (byte B of w) as bf16 values times a power of two (v_cvt_scalef32_pk_bf16_fp4; it uses the
// scale's exponent only). Exact.
template <int B>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
// The eight codes of w.
__device__ __forceinline__ uint4 fp4_word(uint32_t w, float scale) {
  return make_uint4(fp4_pair<0>(w, scale), fp4_pair<1>(w, scale), fp4_pair<2>(w, scale), fp4_pair<3>(w, scale));
}
// Four codes (half H of w) that belong to four tokens of scales s[0 .. 3].
template <int H>
__device__ __forceinline__ uint2 fp4_quad(uint32_t w, const float (&s)[4]) {
  const uint32_t a = (fp4_pair<2 * H>(w, s[0]) & 0xFFFFu) | (fp4_pair<2 * H>(w, s[1]) & 0xFFFF0000u);
  const uint32_t b = (fp4_pair<2 * H + 1>(w, s[2]) & 0xFFFFu) | (fp4_pair<2 * H + 1>(w, s[3]) & 0xFFFF0000u);
  return make_uint2(a, b);
}

// Eight fp32 values to codes (round to nearest even, saturating: v_cvt_scalef32_pk_fp4_f32).
__device__ __forceinline__ uint32_t fp4_encode8(const float (&x)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return w;
}

// The bits of a V word that belong to keys [lo, hi) of the page's 16, for lane row qd (keys 4 qd ..).
__device__ __forceinline__ uint32_t fp4_key_bits(int qd, int lo, int hi) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) m |= (4 * qd + k >= lo && 4 * qd + k < hi ? 0xFu : 0u) << (4 * k);
  return m * 0x10001u;
}

}  // namespace cs
