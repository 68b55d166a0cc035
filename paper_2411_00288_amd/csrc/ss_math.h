// Device helpers that the library's kernels share: register types, stores, barriers, roundings and activations.
#ifndef SS_MATH_H_
#define SS_MATH_H_
#include "ss_internal.h"

namespace ss {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x16 __attribute__((ext_vector_type(16)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// A 16-byte buffer store at a lane's offset plus a uniform one.  The sum is the lane's operand and not the instruction's scalar offset: without a scalar
// offset the compiler keeps the store's data registers unwritten for two wait states behind it, with one it takes none to be needed, and a vector
// instruction that followed at once has changed the stored words (a pixel's first dword was that instruction's result, now and then).
template <int POLICY = 0>
__device__ __forceinline__ void store_b128(const u32x4 &v, const __amdgpu_buffer_rsrc_t &r, int lane_off, int off)
{
    __builtin_amdgcn_raw_buffer_store_b128(v, r, lane_off + off, 0, POLICY);
}

// Workgroup barrier that orders LDS traffic only: the waves' outstanding global loads (weight ring, staging loads)
// and stores (output tile) stay in flight across it.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Two fp32 values to one dword of 16-bit floats, round to nearest even, in one instruction (V_CVT_PK_F16_F32 /
// V_CVT_PK_BF16_F32).
template <int DT>
__device__ __forceinline__ uint32_t cvt_pack2(float a, float b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const f32x2 v = {a, b};
    if constexpr (DT == SS_F16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// max(v, floor) that hands a NaN through (the IEEE 754-2019 maximum, one V_MAXIMUM3_F32): ReLU with floor = 0, the
// identity with floor = -inf.  (A sum of exactly -0 comes out as +0.)
__device__ __forceinline__ float floor_at(float v, float floor)
{
    return __builtin_elementwise_maximum(v, floor);
}

// Exact value of a 16-bit pattern as fp32.
template <int DT>
__device__ __forceinline__ float widen(uint16_t bits)
{
    if constexpr (DT == SS_F16)
        return (float)__builtin_bit_cast(_Float16, bits);
    else
        return __builtin_bit_cast(float, (uint32_t)bits << 16);
}

// GELU z * Phi(z) with the exact standard normal CDF.  With a = |z| and h = Phi(-a):
//     z >= 0:  z (1 - h) = z - a h        z < 0:  z h = -a h        i.e.  gelu(z) = max(z, 0) - a h,
// which needs no select.  log2 Phi(-a) is smooth and close to a parabola: a polynomial and one exp2.  Two fits, each as long as
// the values of its output type ODT ask for (a negative leading coefficient takes either to 0 behind its range):
//   binary16   a h rounds to 0 from a = 5.5 on: degree 8, fitted on [0, 6].  Eleven full-rate instructions and one half-rate one
//              (52 clocks per wave: measured, a fused multiply-add takes 4 and exp2 8).
//   bfloat16   holds the whole lower tail: degree 10, fitted on [0, 12.95], where Phi reaches 2^-126, the least value exp2 gives
//              (60 clocks).
// Fitted for the smallest largest error of Phi (|error| < 1e-7 in fp32 arithmetic), and in the tail for relative errors: 6e-7 at
// a = 1, 2e-5 at 3, 3e-4 at 5; from there degree 8 loses the tail (6e-3 at 6.3, 8e-2 at 7, nothing is left at 10), degree 10 has
// 1e-3 at 6, 3e-3 at 8, 2.3e-2 at 10 and 3.5e-2 at 12.9.  The rational form 7.1.26 of Abramowitz & Stegun takes twelve and two
// instructions for 2e-7 absolute and 9e-4 at 4, 5e-3 at 6, 1.2e-2 at 8, 2.2e-2 at 10, 3.6e-2 at 12.5.  A NaN stays a NaN.
// At an infinity a h is infinity times 0 and the difference a NaN, which the minimum (of a NaN and a number, the number) replaces by max(z, 0): +infinity, and at -infinity
// 0, the limits.  Elsewhere the difference is the smaller one and keeps its bits.  (One register less than a bounded a, which made the kernels with short MXFP4 reductions
// spill: 64 -> 64 on 99284 rows 9.7 -> 11.2 us.)
template <int ODT>
__device__ __forceinline__ float log2_upper_tail(float a)
{
    float q;
    if constexpr (ODT == SS_F16) {
        q = -8.120558493747162e-07f;
        q = __builtin_fmaf(q, a, 1.4290432782061204e-05f);
        q = __builtin_fmaf(q, a, -6.487764435589362e-05f);
        q = __builtin_fmaf(q, a, -0.0004287622419436152f);
        q = __builtin_fmaf(q, a, 0.007434012361791795f);
        q = __builtin_fmaf(q, a, -0.05273924310954606f);
        q = __builtin_fmaf(q, a, -0.4591337784121185f);
        q = __builtin_fmaf(q, a, -1.1511134917708818f);
        q = __builtin_fmaf(q, a, -0.9999998474115108f);
    } else {
        q = -3.325034692025497e-09f;
        q = __builtin_fmaf(q, a, 1.58049019205464e-07f);
        q = __builtin_fmaf(q, a, -3.0015255561011145e-06f);
        q = __builtin_fmaf(q, a, 2.81424345303094e-05f);
        q = __builtin_fmaf(q, a, -0.00011069921310991049f);
        q = __builtin_fmaf(q, a, -0.00034601808874867857f);
        q = __builtin_fmaf(q, a, 0.007352784276008606f);
        q = __builtin_fmaf(q, a, -0.052697665989398956f);
        q = __builtin_fmaf(q, a, -0.45914411544799805f);
        q = __builtin_fmaf(q, a, -1.1511123180389404f);
        q = __builtin_fmaf(q, a, -0.9999998807907104f);
    }
    return q;
}

template <int ODT>
__device__ __forceinline__ float gelu_cdf(float z)
{
    const float a = fabsf(z), q = log2_upper_tail<ODT>(a);
    // (the IEEE 754-2019 maximum: fmaxf takes a second instruction, which quiets a signalling NaN first)
    const float positive = floor_at(z, 0.f);
    return __builtin_fminf(__builtin_fmaf(-a, __builtin_amdgcn_exp2f(q), positive), positive);
}

}  // namespace ss

#endif
