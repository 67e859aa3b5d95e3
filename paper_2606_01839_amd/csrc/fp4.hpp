// Blocks of a pool that holds K and V in 4 bits (the MX element e2m1 with power-of-two scales), shared by
// the kernels that write and read them.
//
// A block of (layer, page, kv head) is 17 D bytes (D = 128: 2176 against 8192 in bf16), two codes a byte:
//   K    [D/32 groups][16 tokens][32 dims]
//   V    [qd 4][c 16][D/16 tiles t][4 tokens]: dim 16 t + c of tokens 4 qd .. 4 qd + 3
//   scales [D bytes]: K [16 tokens][D/32 groups], V [16 tokens], then zeros. Byte e stands for 2^(e - 127).
// Lane 16 qd + c of a wave holds D/32 words (of eight codes) of each, one 16- (D = 64: 8-) byte load a page, 1 KiB
// (512 bytes) of consecutive bytes: of K the dims (D/4) qd .. of token c, of V four tokens of the dims 16 t + c.
// Both are matrix-core operands as they are or after conversion alone. K has a scale for every 32 dims of a
// token, which the MX matrix instructions apply; V one for every token, since a lane's V values are of different
// tokens: a scale the softmax weight can take, where one for every 32 dims would take D / 32 scaled copies
// of the weights. (Rounding error of V, 2-norm, with normal / Laplace values: 0.113 / 0.134 of the values with
// one scale for 128 dims, 0.115 / 0.127 for 32.)
// The padding to 17 D keeps blocks on 64-byte boundaries; without it they would be 2% (D = 64: 1.5%) smaller.
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
  static __device__ __forceinline__ int k_word(int t, int ch) { return kK + ((ch >> 2) * kPageTokens + t) * 16 + (ch & 3) * 4; }
  // ... and of the scale of 32 dims of it
  static __device__ __forceinline__ int k_scale(int t, int group) { return kKScale + t * (D / 32) + group; }
  // K codes and scale of lane 16 qd + c
  static __device__ __forceinline__ int k_lane(int lane) {
    const int c = lane & 15, qd = lane >> 4;
    return D == 128 ? kK + 16 * lane : kK + (qd >> 1) * 256 + c * 16 + (qd & 1) * 8;
  }
  static __device__ __forceinline__ int k_scale_lane(int lane) { return k_scale(lane & 15, D == 128 ? lane >> 4 : lane >> 5); }
  static __device__ __forceinline__ size_t at(int layer, int page, int head, int64_t n_pages, int n_kv_heads) {
    return ((static_cast<size_t>(layer) * static_cast<size_t>(n_pages) + static_cast<size_t>(page)) *
                static_cast<size_t>(n_kv_heads) + static_cast<size_t>(head)) * static_cast<size_t>(kBytes);
  }
};

// The scale byte of a group whose largest magnitude has the given fp32 bits (sign cleared): the power of
// two floor(log2 a) - 2, so that a / scale lies in [4, 8) and e2m1's largest value, 6, is reached; at
// least 2^-126. A group with an infinity or NaN gets 255, which reads back as NaN; of V its codes are zeros,
// so that the decode's weight times that scale, an infinity, gives NaN with them too.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t abs_bits) {
  const int e = static_cast<int>(abs_bits >> 23);
  return e == 255 ? 255u : static_cast<uint32_t>(max(e - 2, 1));
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
// 2^(byte - 127) (0 for the zero byte of an unwritten slot, infinity for 255)
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// byte b of w as such a scale
__device__ __forceinline__ float fp4_scale_of(uint32_t w, int b) {
  return __uint_as_float(((w >> (8 * b)) & 0xFFu) << 23);
}

// the same for the conversion instructions, which look at a scale's exponent bits only
__device__ __forceinline__ float fp4_exponent_of(uint32_t w, int b) {
  return __uint_as_float(b == 0 ? w << 23 : b == 1 ? w << 15 : b == 2 ? w << 7 : w >> 1);
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

// ------------------------------------------------------------------------------------------------
// The score product. K's codes and scales are operands of the MX matrix instructions as they lie in the page,
// at four times the rate of bf16 if the other operand has 6 bits or fewer (measured: a 32x32x64 product of
// 4 by 6 bits takes the 39 cycles of a 32x32x16 one in bf16, of 4 by 8 bits 73). So a query enters as the sum of three
// e3m2 numbers, of 3 significant bits each and scales 2^0, 2^-4, 2^-8 of the first's: with the largest
// magnitude of a block of 32 dims scaled to [8, 16) each takes what the one before left (at most 1 of the
// first's units, 16 of its own; the format ends at 28), and the sum is a bf16 query's 8 bits exactly for values
// down to 2^-8 of the largest, and within 2^-16 of the largest for all. Three products cost 3/4 of the bf16 one
// and no conversion of K. (Two e4m3 numbers are exact over a wider range but cost as much as bf16; two of
// e2m3 are within 2^-10 of the largest only: as much as the softmax weights' rounding.)
// ------------------------------------------------------------------------------------------------
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

// 32 consecutive dims of a query (a lane's share of the operand); bytes 0, 1, 2 of `scale` go with p[0 .. 2]
struct Bf6Query {
  u32x6 p[3];
  uint32_t scale;
};

// 32 fp32 values / scale as e3m2 (the instruction interleaves its two sources), and back. Written as asm for
// the early clobber: both instructions take several passes, and with a result register among its sources,
// as the compiler allocates them for the builtins, the conversion reads values that it has already overwritten.
__device__ __forceinline__ u32x6 to_bf6(const f32x16& even, const f32x16& odd, float scale) {
  u32x6 r;
  asm("v_cvt_scalef32_2xpk16_bf6_f32 %0, %1, %2, %3\n\ts_nop 4" : "=&v"(r) : "v"(even), "v"(odd), "v"(scale));
  return r;
}
__device__ __forceinline__ f32x32 from_bf6(u32x6 x, float scale) {
  f32x32 r;
  asm("v_cvt_scalef32_pk32_f32_bf6 %0, %1, %2\n\ts_nop 4" : "=&v"(r) : "v"(x), "v"(scale));
  return r;
}

__device__ __forceinline__ Bf6Query split_query(const uint4 (&x)[4]) {
  f32x16 even, odd;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      even[4 * i + j] = bf16_lo(w[j]);
      odd[4 * i + j] = bf16_hi(w[j]);
      m = max(m, max(abs_bits(bf16_lo(w[j])), abs_bits(bf16_hi(w[j]))));
    }
  }
  const uint32_t top = max(m >> 23, 12u);   // at least 2^-115: smaller queries lose bits of scores below 2^-100
  Bf6Query q;
  // (e3m2 has no infinity or NaN: a block with one gets the scale that makes its scores NaN)
  q.scale = top == 255 ? 0xFFFFFFu : (top - 3) | (top - 7) << 8 | (top - 11) << 16;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const float s = fp4_scale(top - 3 - 4 * k);
    q.p[k] = to_bf6(even, odd, s);
    if (k == 2) break;
    const f32x32 back = from_bf6(q.p[k], s);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] -= back[2 * i];
      odd[i] -= back[2 * i + 1];
    }
  }
  return q;
}

__device__ __forceinline__ i32x8 mx_operand(uint4 w) {
  return i32x8{static_cast<int>(w.x), static_cast<int>(w.y), static_cast<int>(w.z), static_cast<int>(w.w), 0, 0, 0, 0};
}
__device__ __forceinline__ i32x8 mx_operand(u32x6 w) {
  return i32x8{static_cast<int>(w[0]), static_cast<int>(w[1]), static_cast<int>(w[2]), static_cast<int>(w[3]),
               static_cast<int>(w[4]), static_cast<int>(w[5]), 0, 0};
}
// acc + K . part P of the query: 32 keys x 64 dims x 32 queries (lane = 32 (dims / 32) + key, query), or 16 x 128 x
// 16. K's scale is byte S of `ks`. Operand formats: 4 = e2m1, 3 = e3m2.
template <int P, int S>
__device__ __forceinline__ f32x16 mx_score(uint4 k, uint32_t ks, const Bf6Query& q, f32x16 acc) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand(k), mx_operand(q.p[P]), acc, 4, 3, S, ks, P, q.scale);
}
template <int P, int S>
__device__ __forceinline__ f32x4 mx_score(uint4 k, uint32_t ks, const Bf6Query& q, f32x4 acc) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand(k), mx_operand(q.p[P]), acc, 4, 3, S, ks, P, q.scale);
}

}  // namespace cs
