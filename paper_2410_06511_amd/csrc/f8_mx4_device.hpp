// Blocks of 32 in registers: scale, codes and back.
#pragma once
#include "f8_device.hpp"
#include "f8_mx4.hpp"

namespace f8 {

// Byte of the scale of row `row`, block `b` among those of rows padded to `srows`.
__device__ inline int64_t mx4_scale_at(int64_t srows, int row, int b)
{
    return ((int64_t)(b / 16) * srows + row) * 16 + 4 * (b % 4) + b % 16 / 4;
}

// E8M0 code of a block of 32 bf16 from the largest magnitude's exponent field: that less 2.  (Subnormal magnitudes have the field 0
// and fall to the least scale, 2^-127, with all others below 2^-124.)  Infinity or NaN: 255, NaN.
__device__ inline uint32_t mx4_scale_of_field(uint32_t e) { return e == 255 ? 255 : e > 2 ? e - 2 : 0; }
__device__ inline uint32_t mx4_scale_of(const uint4 (&v)[4])
{
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) m = absmax_acc(m, v[k]);
    return mx4_scale_of_field(pk_collapse(m) >> 7);
}
// The same of a block that four neighbouring lanes hold, in each of them (exchanges within a quad: lanes 1, 0, 3, 2 and 2, 3, 0, 1).
__device__ inline uint32_t mx4_scale_of_quad(const uint4& v)
{
    uint32_t m = pk_collapse(absmax_acc(0, v));
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true);
    m = o > m ? o : m;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true);
    return mx4_scale_of_field((o > m ? o : m) >> 7);
}

// Codes of eight values: the chip's conversion divides by the scale and rounds to nearest even, saturating.  Its scale is an fp32
// number; the least, 2^-127, is subnormal there, so such a block and its scale are taken 2^64 up (exact: the values are below 2^-124).
__device__ inline uint32_t mx4_encode8(uint4 v, uint32_t code)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    uint32_t field = code == 255 ? 127u : code;
    if (code == 0) {  // (a branch that few waves take: as a selection it would be half of the work)
        const auto up = [](uint32_t x) { return pack_bf16(bf16_lo(x) * 0x1p64f, bf16_hi(x) * 0x1p64f); };
        v = make_uint4(up(v.x), up(v.y), up(v.z), up(v.w)), field = 64;
        asm volatile("");
    }
    const float scale = __uint_as_float(field << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v.x), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v.y), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v.z), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v.w), scale, 3);
}
__device__ inline uint4 mx4_encode(const uint4 (&v)[4], uint32_t code)
{
    return make_uint4(mx4_encode8(v[0], code), mx4_encode8(v[1], code), mx4_encode8(v[2], code), mx4_encode8(v[3], code));
}

// Eight codes with the scale code e, in bf16 (exact: the least value is 2^-128; scales above 2^125 may overflow to infinity).
__device__ inline uint4 mx4_decode8(uint32_t w, uint32_t e)
{
    float f[8];
    const float s = e == 255 ? __builtin_nanf("") : e == 0 ? 0x1p-127f : __uint_as_float(e << 23);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t c = w >> (4 * j) & 15u, x = c >> 1 & 3u, m = c & 1u;
        const float v = x ? __uint_as_float(((x + 126u) << 23) | (m << 22)) : 0.5f * (float)m;
        f[j] = (c & 8u ? -v : v) * s;
    }
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

}  // namespace f8
