// Rotary positions on the device: angles, and the rotation of rows of heads.
//
// Pair i of a row at position p turns by p f_i radians. f_i / 2 pi is kept as a 64-bit fraction of a turn,
// so p times it, modulo 2^64, is the angle's fraction of a turn to 2^-34 at any p < 2^31 (in fp32
// the angle of position 10^5 would be off by 4e-3 radians). Its upper 32 bits, signed, are within half a turn of zero;
// rounded to fp32 they are off by up to 2^-26 turns (9.4e-8 radians) and 2^-32, and v_sin_f32 and v_cos_f32, which
// take turns, by 1.9e-7 (measured over 4 million angles). With the fp32 arithmetic a rotated value is within
// 2^-21 = 4.8e-7 of |a| + |b| before it is rounded (measured where the terms cancel: 2.0e-7).
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"

namespace cs {

// cos and sin of a pair's angle, times the amplitude
__device__ __forceinline__ f32x2 rope_turn(uint64_t frac, uint32_t pos, float amplitude) {
  const int32_t turn = static_cast<int32_t>((frac * pos) >> 32);
  const float t = static_cast<float>(turn) * 0x1p-32f;
  return f32x2{amplitude * __builtin_amdgcn_cosf(t), amplitude * __builtin_amdgcn_sinf(t)};
}

// Rotation of dims 8 ch .. 8 ch + 7 of a row held by this lane (x, fp32); the row's D / 8 lanes are
// consecutive. `cs_row`: the row's (cos, sin) of each pair. All lanes of the wave take part (shuffles).
template <int D>
__device__ __forceinline__ void rope_rotate(float (&x)[8], int ch, const RopeArgs& r, const f32x2* cs_row) {
  if (r.interleaved) {
    if (8 * ch < 2 * r.pairs) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 t = cs_row[4 * ch + i];
        const float a = x[2 * i], b = x[2 * i + 1];
        x[2 * i] = a * t.x - b * t.y;
        x[2 * i + 1] = a * t.y + b * t.x;
      }
    }
    return;
  }
  // halves: dim i and dim i + pairs; pairs is a multiple of 8, so a lane's dims lie in one half
  const int off = r.pairs / 8;
  const bool first = ch < off, turns = ch < 2 * off;
  const int lane = __lane_id();
  const int partner = turns ? (first ? lane + off : lane - off) : lane;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __int_as_float(__builtin_amdgcn_ds_bpermute(partner << 2, __float_as_int(x[i])));
  if (turns) {
    const f32x2* t = cs_row + 8 * (first ? ch : ch - off);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * t[i].x + (first ? -y[i] : y[i]) * t[i].y;
  }
}

__device__ __forceinline__ void unpack8(uint4 v, float (&x)[8]) {
  x[0] = bf16_lo(v.x), x[1] = bf16_hi(v.x), x[2] = bf16_lo(v.y), x[3] = bf16_hi(v.y);
  x[4] = bf16_lo(v.z), x[5] = bf16_hi(v.z), x[6] = bf16_lo(v.w), x[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

}  // namespace cs
