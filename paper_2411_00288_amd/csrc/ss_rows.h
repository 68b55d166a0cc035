// Rows of channels-last activations in registers: runs of 8 channels of a row, 16- or 32-bit, at any address that is a multiple of
// an element.  (Not a multiple of 16 bytes: an odd number of channels, or a view of a wider tensor.  gfx950 takes such 16-byte accesses as they
// are, so there is one path for all of them.)
#ifndef SS_ROWS_H_
#define SS_ROWS_H_
#include "ss_math.h"

namespace ss {

// (By value: __builtin_bit_cast of an element of a vector variable takes the vector's first one.)
__device__ __forceinline__ float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

template <int DT> constexpr int item_bytes() { return DT == SS_F32 ? 4 : 2; }

typedef u32x4 At2 __attribute__((aligned(2)));
typedef u32x4 At4 __attribute__((aligned(4)));
struct Vec16 { At2 v; };
struct Vec32 { At4 v; };
static_assert(sizeof(Vec16) == 16 && alignof(Vec16) == 2 && alignof(Vec32) == 4, "16 bytes on an element's boundary");

// One value of type DT at p.
template <int DT>
__device__ __forceinline__ float load1(const void *p)
{
    if constexpr (DT == SS_F32)
        return *static_cast<const float *>(p);
    else
        return widen<DT>(*static_cast<const uint16_t *>(p));
}

template <int DT>
__device__ __forceinline__ void store1(void *p, float v)
{
    if constexpr (DT == SS_F32)
        *static_cast<float *>(p) = v;
    else
        *static_cast<uint16_t *>(p) = (uint16_t)cvt_pack2<DT>(v, 0.f);
}

// A run as it lies in memory (32-bit: two vectors).
template <int DT> struct Run { u32x4 v[DT == SS_F32 ? 2 : 1]; };

// p[0..n), the others zero; n <= 0: nothing is read.
template <int DT>
__device__ __forceinline__ Run<DT> load_run(const void *p, int n)
{
    Run<DT> r = {};
    if (n >= 8) {
        if constexpr (DT == SS_F32) {
            r.v[0] = static_cast<const Vec32 *>(p)[0].v;
            r.v[1] = static_cast<const Vec32 *>(p)[1].v;
        } else {
            r.v[0] = static_cast<const Vec16 *>(p)->v;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 7; e++)
            if (e < n) {
                if constexpr (DT == SS_F32)
                    r.v[e / 4][e % 4] = static_cast<const uint32_t *>(p)[e];
                else
                    r.v[0][e / 2] |= (uint32_t) static_cast<const uint16_t *>(p)[e] << (16 * (e % 2));
            }
    }
    return r;
}

// Channels c .. c + 7 of a row of at least 8: one load from inside the row whatever the lane, so that loads follow each other without a branch between them.
// place_wide then moves what a lane at the row's end got into place.  LAST: nobody reads the row again soon, and its lines need not stay in the caches.
template <int DT, bool LAST>
__device__ __forceinline__ Run<DT> load_wide(const void *row, int c, int cols)
{
    const char *const p = static_cast<const char *>(row) + (long long)min(c, cols - 8) * item_bytes<DT>();
    Run<DT> r;
    if constexpr (DT == SS_F32) {
        const Vec32 *const v = reinterpret_cast<const Vec32 *>(p);
        r.v[0] = LAST ? __builtin_nontemporal_load(&v[0].v) : v[0].v;
        r.v[1] = LAST ? __builtin_nontemporal_load(&v[1].v) : v[1].v;
    } else {
        const Vec16 *const v = reinterpret_cast<const Vec16 *>(p);
        r.v[0] = LAST ? __builtin_nontemporal_load(&v->v) : v->v;
    }
    return r;
}

// What load_wide read, with zeros past the row's end, and everywhere where the row is not `active`.
template <int DT>
__device__ __forceinline__ void place_wide(Run<DT> &r, int c, int cols, bool active)
{
    constexpr int N = DT == SS_F32 ? 2 : 1;
    if (c + 8 <= cols && active) return;
    const int by = c + 8 - cols;                           // (8 and more: nothing is left)
    uint32_t w[4 * N + 4];
#pragma unroll
    for (int e = 0; e < 4 * N; e++) w[e] = r.v[e / 4][e % 4];
#pragma unroll
    for (int e = 4 * N; e < 4 * N + 4; e++) w[e] = 0;
    constexpr int UNIT = DT == SS_F32 ? 1 : 2;             // elements of a word
#pragma unroll
    for (int step = 4; step >= UNIT; step /= 2)
        if (by & step) {
#pragma unroll
            for (int e = 0; e < 4 * N; e++) w[e] = w[e + step / UNIT];
        }
    if (UNIT == 2 && (by & 1)) {
#pragma unroll
        for (int e = 0; e < 4 * N; e++) w[e] = (w[e] >> 16) | (w[e + 1] << 16);
    }
#pragma unroll
    for (int e = 0; e < 4 * N; e++) r.v[e / 4][e % 4] = active && by < 8 ? w[e] : 0u;
}

template <int DT>
__device__ __forceinline__ void widen_run(const Run<DT> &r, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if constexpr (DT == SS_F32)
            v[e] = as_float(r.v[e / 4][e % 4]);
        else if constexpr (DT == SS_BF16)
            v[e] = as_float(e % 2 ? r.v[0][e / 2] & 0xFFFF0000u : r.v[0][e / 2] << 16);
        else
            v[e] = widen<DT>((uint16_t)(r.v[0][e / 2] >> (16 * (e % 2))));
    }
}

// v[0..n) = p[0..n), the others zero; n <= 0: nothing is read.
template <int DT>
__device__ __forceinline__ void load8(const void *p, int n, float (&v)[8])
{
    widen_run<DT>(load_run<DT>(p, n), v);
}

// p[0..n) = v[0..n), rounded to nearest even.
template <int DT>
__device__ __forceinline__ void store8(void *p, int n, const float (&v)[8])
{
    if (n >= 8) {
        if constexpr (DT == SS_F32) {
            u32x4 a, b;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                a[e] = as_bits(v[e]);
                b[e] = as_bits(v[4 + e]);
            }
            static_cast<Vec32 *>(p)[0].v = a;
            static_cast<Vec32 *>(p)[1].v = b;
        } else {
            u32x4 a;
#pragma unroll
            for (int e = 0; e < 4; e++) a[e] = cvt_pack2<DT>(v[2 * e], v[2 * e + 1]);
            static_cast<Vec16 *>(p)->v = a;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (e < n) store1<DT>(static_cast<char *>(p) + e * item_bytes<DT>(), v[e]);
    }
}

}  // namespace ss

#endif
