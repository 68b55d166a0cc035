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
enum F8Kernel { F8_TILE_64 = 80, F8_TILE_128, F8_TILE_256, F8_FEW_32, F8_FEW_64, F816_FEW, F816_ROWS, F816_ROWS_128, F816_CODES };

// Estimated time of the tiled kernels in us: what a compute unit's tiles cost besides their steps, and a step.  Of 256 x 256 a compute unit holds one, of 128 x 128 two and of 64 x 64
// several, which hide each other's beginnings and ends.  From 20 layers of 64 -> 64 to 8192 -> 8192 channels and 1 to 401408 rows, among them (estimates /
// measurements of 64 x 64, 128 x 128 and 256 x 256):
//     64 -> 256 on 200704 rows   33 / 31   29 / 27   45 / 56        1024 -> 1024 on 65536      152 / 138   81 / 76   88 / 83
//     8192 -> 1024 on 12544     188 / 200 126 / 127 103 / 99        8192 -> 8192 on 8192              493 / 542 411 / 417
inline double f8_tile_us(const F8Dims &t, long long rows, int m, long long cus)
{
    const double tiles = (double)((t.Mt * 32ll + m - 1) / m) * (double)((rows + m - 1) / m) / (double)cus;
    const double whole = (double)(long long)(tiles + 0.999999);
    if (m == 256) return whole * (10.5 + 0.72 * t.Ks);
    if (m == 128) return (tiles <= 1 ? 4.2 + 0.2 * t.Ks : 3.0 + (tiles < 4 ? whole : tiles) * (1.9 + 0.225 * t.Ks));
    return 2.5 + (tiles < 4 ? whole : tiles) * (0.5 + 0.115 * t.Ks);
}

inline F8Kernel best_f8_tile(const F8Dims &t, long long rows, long long cus)
{
    const double small = f8_tile_us(t, rows, 64, cus), middle = f8_tile_us(t, rows, 128, cus), large = f8_tile_us(t, rows, 256, cus);
    return large < small && large < middle ? F8_TILE_256 : middle < small ? F8_TILE_128 : F8_TILE_64;
}

inline double f8_tiles_us(const F8Dims &t, long long rows, long long cus)
{
    const F8Kernel k = best_f8_tile(t, rows, cus);
    return f8_tile_us(t, rows, k == F8_TILE_256 ? 256 : k == F8_TILE_128 ? 128 : 64, cus);
}

// On codes.  Up to 32 rows, and of short reductions until their workgroups of 32 channels and 32 rows fill the chip, the kernel whose waves share the reduction (8192 -> 8192 on 16
// rows 15 us, in tiles 26; 2048 -> 1000 on one 4.7 and 5.4; 768 -> 2304 on 100 4.7 and 4.7, but 4096 -> 4096 on 100 17 and 9); of wide layers with long
// reductions up to 48 rows, two tiles of them to the workgroup.
inline F8Kernel choose_f8_codes(const F8Dims &t, long long rows, long long cus)
{
    if (rows <= 32 || (t.KB <= 16 && (rows + 31) / 32 * t.Mt <= cus)) return F8_FEW_32;
    if (rows <= 48 && t.KB > 32) return F8_FEW_64;
    return best_f8_tile(t, rows, cus);
}

// LDS of the few-row kernel: its quantised rows, later the waves' sums.
inline size_t f8_few_lds(const F8Dims &t, int waves, int quantised_rows)
{
    const size_t pad = (size_t)(quantised_rows | 1), rows = quantised_rows ? (size_t)4 * t.Ks * pad * 16 + (size_t)t.Kq * pad * 4 : 0;
    return std::max(rows, (size_t)waves * 16 * 65 * 4);
}

// LDS of the kernel for reductions that fit it: quantised rows, their scales, the bias.
inline size_t f8_rows_lds(const F8Dims &t, int px) { return (size_t)4 * t.Ks * (px + 1) * 16 + ((size_t)t.Kq * (px + 1) * 4 + 15) / 16 * 16 + (size_t)t.Mt * 128; }

// How many workgroups share the output channels of 32 rows of the kernel for reductions that fit LDS: until there is one to a compute unit, and at least a
// unit of 64 channels for each of their four waves.
inline int f8_rows_splits(const F8Dims &t, long long rows, long long cus)
{
    const long long blocks = (rows + 31) / 32, units = (t.Mt + 1) / 2;
    return (int)std::max(1ll, std::min((units + 3) / 4, cus / blocks));
}

// Waves of the few-row kernel on 16-bit input: as many as there are blocks, or as the quantisation keeps busy.
inline int f8_few16_waves(const F8Dims &t, long long rows, int K)
{
    const long long elements = rows * K;
    return t.KB > 8 || elements > 16384 ? 16 : t.KB > 4 || elements > 8192 ? 8 : 4;
}

// Waves of the kernel with 32 rows in LDS: four where LDS holds four such workgroups and there are many rows, else eight.
inline int f8_rows_waves(const F8Dims &t, long long rows, long long cus) { return t.KB == 1 || (rows >= 128 * cus && 4 * f8_rows_lds(t, 32) <= kPwLds) ? 4 : 8; }

// Does the kernel take such a layer at all?
inline bool f8_fits16(const F8Dims &t, long long rows, F8Kernel k)
{
    switch (k) {
        case F816_FEW: return rows <= 32 && f8_few_lds(t, 16, (int)rows) <= kPwLds;
        case F816_ROWS: return f8_rows_lds(t, 32) <= kPwLds;
        case F816_ROWS_128: return t.KB == 1 && f8_rows_lds(t, 128) <= kPwLds;
        default: return true;
    }
}

// On 16-bit input.  Few rows while every workgroup's own quantisation of them is short (1024 -> 4096 on 16 rows 4.8 us, and with a quantisation of its own 3.6 + 4.6; 4096 -> 4096 on
// 32 14.3 and 12.8).  Otherwise the shorter estimate: of the kernel that quantises in LDS, whose waves walk down the channels (a workgroup's 4 us, 2.5 for each
// 1000 channels of the reduction and 0.15 a step and 32 channels; what follows the first two of a compute unit overlaps, with 4.2 TB/s for what is moved, and the weights, which
// every 32 rows read again, at 17 TB/s), or of a quantisation at 6 TB/s and the product on its codes.  Measured, the former and the latter: 384 -> 96 on 401408 rows 84 and 121 us,
// 256 -> 512 on 50176 24 and 28, 1024 -> 256 on 12544 13 and 14, 2048 -> 512 on 3136 15 and 14, 2048 -> 2048 on 20000 154 and 102, 1024 -> 1024 on 65536 127 and 106.
// 128 rows to the workgroup with reductions of one block and many rows (64 -> 256 on 200704 rows 53 -> 32 us).
inline F8Kernel choose_f8_16(const F8Dims &t, long long rows, long long cus)
{
    if (rows * t.P <= 49152 && f8_fits16(t, rows, F816_FEW)) return F816_FEW;
    if (!f8_fits16(t, rows, F816_ROWS)) return F816_CODES;
    const double K = t.P, out = rows * t.Mt * 64.0;
    const long long blocks = (rows + 31) / 32, splits = f8_rows_splits(t, rows, cus), units = (t.Mt + splits * 8 - 1) / (splits * 8);
    const double one = 4.0 + 0.0025 * K + 0.15 * units * t.Ks, rounds = (double)(blocks * splits) / (2.0 * cus);
    const bool wide = rows >= 128 * cus && f8_fits16(t, rows, F816_ROWS_128);
    double lds = one + std::max((rounds - 1.0) * (wide ? 0.25 : 0.7) * one, (rows * K * 2 + out) / 4.2e6);
    if (!wide) lds = std::max(lds, (double)blocks * t.Mt * t.Ks * 2112 / 17e6);
    const double codes = 6.0 + rows * K * 3 / 6e6 + (choose_f8_codes(t, rows, cus) >= F8_FEW_32 ? 4.0 + 0.05 * t.Ks : f8_tiles_us(t, rows, cus));
    if (codes < lds) return F816_CODES;
    return wide ? F816_ROWS_128 : F816_ROWS;
}

}  // namespace ss

#endif
