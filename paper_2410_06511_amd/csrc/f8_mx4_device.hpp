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

// E8M0 code of a block of 32 bf16: the exponent field of the largest magnitude less 2.  (Subnormal magnitudes have the field 0
// and fall to the least scale, 2^-127, with all others below 2^-124.)  Infinity or NaN: 255, NaN.
__device__ inline uint32_t mx4_scale_of(const uint4 (&v)[4])
{
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) m = absmax_acc(m, v[k]);
    const uint32_t e = pk_collapse(m) >> 7;
    return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}

// The codes: the chip's conversion divides by the scale and rounds to nearest even, saturating.  Its scale is an fp32 number; the
// least, 2^-127, is subnormal there, so such a block and its scale are taken 2^64 up (exact: the values are below 2^-124).
__device__ inline uint4 mx4_encode(const uint4 (&v)[4], uint32_t code)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    uint32_t o[4];
    const bool low = code == 0;
    const float scale = __uint_as_float((low ? 64u : code == 255 ? 127u : code) << 23);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
        uint32_t r = 0;
        const auto up = [&](uint32_t x) { return low ? pack_bf16(bf16_lo(x) * 0x1p64f, bf16_hi(x) * 0x1p64f) : x; };
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, up(w[0])), scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, up(w[1])), scale, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, up(w[2])), scale, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, up(w[3])), scale, 3);
        o[k] = r;
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
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
