// MXFP4 (OCP microscaling format, E2M1 elements): 32 consecutive values of a row share a scale 2^(byte - 127); an element is a sign and one of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6.  With m the block's largest magnitude
//     scale = 2^clamp(floor(log2 m) - 2, -127, 127),    element = round to nearest even of value / scale, at most 6 in magnitude.
// floor(log2 m) is the exponent field of m as fp32, which takes every 16-bit type exactly; a block of zeros (or with m below 2^-124) has the byte 0.
// A NaN or an infinity in a block makes its byte 0xFF, a NaN for all 32 (the format's elements have neither).  Values divide by a power of two
// exactly, so that the result is the same wherever it is computed.
#ifndef SS_MX4_H_
#define SS_MX4_H_
#include "ss_rows.h"
#include "ss_pw_choice.h"

namespace ss {

inline size_t mx4_packed_size(const Mx4Dims &t) { return (size_t)kHeaderBytes + (size_t)t.Mt * t.Ks * 1024 + (size_t)t.Mt * t.Kq * 256; }

// Largest magnitude pattern of 8 values (as an integer it orders finite values by size, and infinities and NaN above them).
__device__ __forceinline__ uint32_t magnitude8(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) m = max(m, as_bits(v[e]) & 0x7FFFFFFFu);
    return m;
}

// The same of a run as it lies in memory, as an fp32 pattern: 16-bit patterns are compared in pairs.
template <int DT>
__device__ __forceinline__ uint32_t magnitude(const Run<DT> &r)
{
    if constexpr (DT == SS_F32) {
        float v[8];
        widen_run<DT>(r, v);
        return magnitude8(v);
    } else {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 m = {0, 0};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t word = r.v[0][e] & 0x7FFF7FFFu;
            m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, word));
        }
        const uint16_t low = m[0], high = m[1];
        return as_bits(widen<DT>(low > high ? low : high));
    }
}

// The maximum over the four lanes of a quad, which hold a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1 /* quad_perm 1 0 3 2 */, 0xF, 0xF, true));
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E /* quad_perm 2 3 0 1 */, 0xF, 0xF, true));
}

// The scale byte for a block whose largest magnitude pattern is m.
__device__ __forceinline__ uint32_t mx4_scale(uint32_t m)
{
    return m >= 0x7F800000u ? 0xFFu : (uint32_t)max((int)(m >> 23) - 2, 0);
}

// Eight elements as 4-bit codes, the first in the lowest bits.  V_CVT_SCALEF32_PK_FP4_F32 divides by the scale, rounds to nearest even and
// saturates (all 65536 results of 12 scales from 2^-127 to 2^127 checked against the definition).
__device__ __forceinline__ uint32_t mx4_codes8(const float (&v)[8], uint32_t byte)
{
    if (byte == 0xFFu) return 0;
    const float scale = as_float(byte == 0 ? 0x00400000u : byte << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
}

// The same for a run as it lies in memory; 16-bit values are converted as they are.
template <int DT>
__device__ __forceinline__ uint32_t mx4_codes(const Run<DT> &r, uint32_t byte)
{
    if constexpr (DT == SS_F32) {
        float v[8];
        widen_run<DT>(r, v);
        return mx4_codes8(v, byte);
    } else {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        if (byte == 0xFFu) return 0;
        const float scale = as_float(byte == 0 ? 0x00400000u : byte << 23);
        const uint32_t w0 = r.v[0][0], w1 = r.v[0][1], w2 = r.v[0][2], w3 = r.v[0][3];
        uint32_t c = 0;
        if constexpr (DT == SS_F16) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w0), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w1), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w2), scale, 2);
            return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w3), scale, 3);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w0), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w1), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w2), scale, 2);
            return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w3), scale, 3);
        }
    }
}

// What eight codes stand for.
__device__ __forceinline__ void mx4_values8(uint32_t c, uint32_t byte, float (&v)[8])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 t[4];
    t[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 0);
    t[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 1);
    t[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 2);
    t[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 3);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float f = __builtin_amdgcn_ldexpf(t[e >> 1][e & 1], (int)byte - 127);
        v[e] = byte == 0xFFu ? __builtin_nanf("") : f;
    }
}

// A device call on the current device's stream failed or not.
inline int launched() { return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_HIP; }

int mx4_quantize(const void *x, int64_t rows, int cols, int64_t ldx, int dtype, uint8_t *codes, uint8_t *scales, hipStream_t s);

}  // namespace ss

#endif
