// FP8 E4M3 with a scale for each block of 128 consecutive values of a row.  With m the block's largest magnitude
//     scale = 2^clamp(ceil(log2(m / 448)), -127, 127),    element = round to nearest even of value / scale, at most 448 in magnitude:
// the least power of two that leaves nothing to saturate, so that an element has the type's four significant bits wherever the block does not reach
// over more than 2^15.  A power of two, and not m / 448 itself: values divide by it exactly, the result is the same wherever it is computed, and the
// matrix instruction multiplies by it without a vector instruction (a scale in 32 bits is a multiply-add for each sum and block).  A block of zeros
// has the byte 0.  A NaN or an infinity in a block makes its byte 0xFF, a NaN for all 128.
#ifndef SS_F8_H_
#define SS_F8_H_
#include "ss_mx4.h"
#include "ss_f8_choice.h"

namespace ss {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// The scale byte for a block whose largest magnitude has the fp32 pattern m: its exponent less 8, one more if its fraction is above 448's.
__device__ __forceinline__ uint32_t f8_scale(uint32_t m)
{
    return m >= 0x7F800000u ? 0xFFu : (uint32_t)max((int)((m + 0x1FFFFFu) >> 23) - 8, 0);
}

__device__ __forceinline__ float f8_unit(uint32_t byte) { return as_float(byte == 0 ? 0x00400000u : byte << 23); }

// The maximum over the 16 lanes of a row of the wave, which hold a block.
__device__ __forceinline__ uint32_t row16_max(uint32_t m)
{
    m = quad_max(m);
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141 /* the mirror image in 8 lanes */, 0xF, 0xF, true));
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140 /* the mirror image in 16 */, 0xF, 0xF, true));
}

typedef short i16x2 __attribute__((ext_vector_type(2)));

// Four values as elements, the first in the lowest byte.  V_CVT_SCALEF32_PK_FP8_F32 divides by the scale and rounds to nearest even.
__device__ __forceinline__ uint32_t f8_codes4(float a, float b, float c, float d, float unit)
{
    i16x2 t = {0, 0};
    t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(t, a, b, unit, false);
    t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(t, c, d, unit, true);
    return __builtin_bit_cast(uint32_t, t);
}

__device__ __forceinline__ u32x2 f8_codes8(const float (&v)[8], uint32_t byte)
{
    const float unit = f8_unit(byte);
    const u32x2 c = {f8_codes4(v[0], v[1], v[2], v[3], unit), f8_codes4(v[4], v[5], v[6], v[7], unit)};
    return byte == 0xFFu ? u32x2{0, 0} : c;
}

// The same for a run as it lies in memory; 16-bit values are converted as they are.
template <int DT>
__device__ __forceinline__ u32x2 f8_codes(const Run<DT> &r, uint32_t byte)
{
    if constexpr (DT == SS_F32) {
        float v[8];
        widen_run<DT>(r, v);
        return f8_codes8(v, byte);
    } else {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        if (byte == 0xFFu) return u32x2{0, 0};
        const float unit = f8_unit(byte);
        u32x2 c;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t w0 = r.v[0][2 * h], w1 = r.v[0][2 * h + 1];
            i16x2 t = {0, 0};
            if constexpr (DT == SS_F16) {
                t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(t, __builtin_bit_cast(f16x2, w0), unit, false);
                t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(t, __builtin_bit_cast(f16x2, w1), unit, true);
            } else {
                t = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(t, __builtin_bit_cast(bf16x2, w0), unit, false);
                t = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(t, __builtin_bit_cast(bf16x2, w1), unit, true);
            }
            c[h] = __builtin_bit_cast(uint32_t, t);
        }
        return c;
    }
}

// What eight elements stand for.
__device__ __forceinline__ void f8_values8(const u32x2 &c, uint32_t byte, float (&v)[8])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const uint32_t w = c[h];
        const f32x2 low = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        v[4 * h] = low[0];
        v[4 * h + 1] = low[1];
        v[4 * h + 2] = high[0];
        v[4 * h + 3] = high[1];
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float f = __builtin_amdgcn_ldexpf(v[e], (int)byte - 127);
        v[e] = byte == 0xFFu ? __builtin_nanf("") : f;
    }
}

int f8_quantize(const void *x, int64_t rows, int cols, int64_t ldx, int dtype, uint8_t *codes, uint8_t *scales, hipStream_t s);

}  // namespace ss

#endif
