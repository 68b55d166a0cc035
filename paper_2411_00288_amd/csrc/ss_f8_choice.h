// Sizes of FP8 operands with a scale for each block of 128, and which kernel a pointwise layer on them takes (host code, no device calls;
// kernels: ss_pw_f8.hip).
#ifndef SS_F8_CHOICE_H_
#define SS_F8_CHOICE_H_
#include "ss_pw_choice.h"

namespace ss {

struct F8Dims {
    int KB;        // blocks of a row
    int S;         // scale bytes of a row: KB rounded up to 4, the surplus zero
    int P;         // code bytes of a row: its channels rounded up to 64, the surplus zero
    int Mt, Ks;    // 32-row tiles, reduction steps of 64
    int Kq;        // scale words of a tile and row: 4 blocks each
};

inline F8Dims f8_dims(int rows, int K)
{
    F8Dims t;
    t.KB = (K + 127) / 128;
    t.S = (t.KB + 3) / 4 * 4;
    t.Ks = (K + 63) / 64;
    t.P = t.Ks * 64;
    t.Mt = (rows + 31) / 32;
    t.Kq = t.S / 4;
    return t;
}

// A reduction's limit: 256 rows of it are a buffer of less than 2^31 bytes.
constexpr int kF8MostK = 1 << 22;

constexpr size_t f8_scales_at(const F8Dims &t) { return (size_t)kHeaderBytes + (size_t)t.Mt * t.Ks * 2048; }
inline size_t f8_packed_size(const F8Dims &t) { return f8_scales_at(t) + (size_t)t.Mt * t.Kq * 128; }

// The kernels, by the ids of the test hook.
enum F8Kernel { F8_TILE_64 = 80, F8_TILE_128, F8_TILE_256, F8_FEW_32, F8_FEW_64 };

inline F8Kernel choose_f8_codes(const F8Dims &t, long long rows, long long cus)
{
    if (rows <= 32 || (rows + 31) / 32 * t.Mt <= cus * 5 / 4) return F8_FEW_32;
    const long long tiles256 = ((rows + 255) / 256) * ((t.Mt + 7) / 8), tiles128 = ((rows + 127) / 128) * ((t.Mt + 3) / 4);
    if (tiles256 >= cus && t.Ks >= 16) return F8_TILE_256;
    return tiles128 >= cus ? F8_TILE_128 : F8_TILE_64;
}

// LDS of the few-row kernel: the waves' sums.
inline size_t f8_few_lds(int waves) { return (size_t)waves * 16 * 65 * 4; }

}  // namespace ss

#endif
