// Which kernel a pointwise MXFP4 layer takes (host code, no device calls; kernels: ss_pw_mx4.hip).
#ifndef SS_PW_CHOICE_H_
#define SS_PW_CHOICE_H_
#include "ss_internal.h"
#include <algorithm>

namespace ss {

// Row sizes of a quantised activation and tile counts of quantised weights.
struct Mx4Dims {
    int KB;        // blocks of a row
    int S;         // scale bytes of a row: KB rounded up to 4, the surplus zero
    int Mt, Ks;    // 32-row tiles, reduction steps of 64
    int Kq;        // scale words of a tile and lane: 4 steps each
};

inline Mx4Dims mx4_dims(int rows, int K)
{
    Mx4Dims t;
    t.KB = (K + 31) / 32;
    t.S = (t.KB + 3) / 4 * 4;
    t.Mt = (rows + 31) / 32;
    t.Ks = (t.KB + 1) / 2;
    t.Kq = (t.Ks + 3) / 4;
    return t;
}

// Rows of one launch, of `threads` threads to the row, in whole tiles of up to 256 rows: a launch has fewer than 2^32 threads (the
// runtime cuts a larger one without an error: of 1140850765 rows 1073741773 were not written), so that 2^30 rows and more go in pieces.
inline long long piece_rows(long long threads) { return std::max(256ll, (1ll << 31) / threads / 256 * 256); }

// The kernels, by the ids of the test hook.  On codes: tiles of 64 x 64, 128 x 128 and 256 x 256, few rows 32 and 64 at a time.  On 16-bit input: few rows,
// reductions that fit LDS with 32 rows to the workgroup and (one chunk) with 128, and a quantisation of its own with the product on its codes.
enum PwKernel { PW_TILE_64 = 70, PW_TILE_128, PW_TILE_256, PW_FEW_32, PW_FEW_64, PW16_FEW, PW16_ROWS, PW16_ROWS_128, PW16_CODES };

constexpr size_t kPwLds = 160 * 1024;

// LDS of the few-row kernel: its quantised rows, later the waves' sums.
inline size_t few_lds(const Mx4Dims &t, int waves, int quantised_rows)
{
    const size_t pad = (size_t)(quantised_rows | 1), rows = quantised_rows ? (size_t)2 * t.Ks * pad * 16 + (size_t)t.Kq * 2 * pad * 4 : 0;
    return std::max(rows, (size_t)waves * 16 * 65 * 4);
}

// LDS of the kernel for reductions that fit it: quantised rows, their scales, the bias.
inline size_t rows_lds(const Mx4Dims &t, int px)
{
    return (size_t)2 * t.Ks * (px + 1) * 16 + ((size_t)t.Kq * 2 * (px + 1) * 4 + 15) / 16 * 16 + (size_t)t.Mt * 128;
}

// Estimated time of the tiled kernels in us: what a compute unit's tiles cost besides their steps, and a step; small tiles of one unit run beside each other, which hides
// their beginnings and ends, and, of 128 x 128, short reductions behind their stores.  From 19 layers of 64 -> 256 to 8192 -> 8192 channels and 100 to 401408 rows, among
// them (estimates / measurements of 64 x 64, 128 x 128 and 256 x 256):
//     64 -> 256 on 200704 rows   39 / 40   27 / 29   87 / 40        1024 -> 256 on 12544          9 / 9      7 / 7    16 / 13
//     8192 -> 1024 on 12544     125 / 118  64 / 76   58 / 56        8192 -> 8192 on 3136        250 / 218  126 / 127 116 / 110
inline double tile_us(const Mx4Dims &t, long long rows, int m, long long cus)
{
    const double tiles = (double)((t.Mt * 32ll + m - 1) / m) * (double)((rows + m - 1) / m) / (double)cus;
    const double whole = (double)(long long)(tiles + 0.999999);
    if (m == 256) return whole * (10.5 + 0.37 * t.Ks);
    if (m == 128) return 3.8 + (tiles < 2 ? whole : tiles) * std::max(1.9, 0.8 + 0.146 * t.Ks);
    return 3.2 + 0.65 * (tiles < 4 ? whole : tiles) + 0.073 * t.Ks * std::max(tiles < 4 ? whole : tiles, 1.4);
}

inline PwKernel best_tile(const Mx4Dims &t, long long rows, long long cus)
{
    const double small = tile_us(t, rows, 64, cus), middle = tile_us(t, rows, 128, cus), large = tile_us(t, rows, 256, cus);
    return large < small && large < middle ? PW_TILE_256 : middle < small ? PW_TILE_128 : PW_TILE_64;
}

// On codes.  Few rows until their workgroups of 32 channels and 32 rows fill the chip (768 -> 2304 on 100 rows, 288 of them: 4.6 us, in tiles 4.7; 4096 -> 4096 on 100, 512
// of them: 13.2 and 8.2), and of wide layers with long reductions up to 48 rows, two tiles of them to the workgroup (8192 -> 8192 on 33 rows 14 us, in tiles 17; on 64
// 19 and 17).
inline PwKernel choose_codes(const Mx4Dims &t, long long rows, long long cus)
{
    if (rows <= 32 || (rows + 31) / 32 * t.Mt <= cus * 5 / 4) return PW_FEW_32;
    if (rows <= 48 && t.Kq > 8) return PW_FEW_64;
    return best_tile(t, rows, cus);
}

inline double tiles_us(const Mx4Dims &t, long long rows, long long cus)
{
    const PwKernel k = best_tile(t, rows, cus);
    return tile_us(t, rows, k == PW_TILE_256 ? 256 : k == PW_TILE_128 ? 128 : 64, cus);
}

// How many workgroups share the output channels of 32 rows of the kernel for reductions that fit LDS: until there is one to a compute unit, and at least a
// unit of 64 channels for each of their four waves.
inline int rows_splits(const Mx4Dims &t, long long rows, long long cus)
{
    const long long blocks = (rows + 31) / 32, units = (t.Mt + 1) / 2;
    return (int)std::max(1ll, std::min((units + 3) / 4, cus / blocks));
}

// Waves of the few-row kernel on 16-bit input: as many as there are scale words, or as the quantisation keeps busy.
inline int few16_waves(const Mx4Dims &t, long long rows, int K)
{
    const long long elements = rows * K;
    return t.Kq > 8 || elements > 16384 ? 16 : t.Kq > 4 || elements > 8192 ? 8 : 4;
}

// Waves of that kernel's workgroups with 32 rows.  Of many rows with longer reductions four, where LDS holds four such workgroups: they hide each other's loads and quantisation
// (384 -> 96 on 401408 rows 109 -> 77 us).  Fewer of them leave the compute unit idle (4096 -> 4096 on 32768 rows, one workgroup, 905 us, with eight waves 544; 4096 -> 1024, two,
// 181 and 164).
inline int rows_waves(const Mx4Dims &t, long long rows, long long cus)
{
    return t.Kq == 1 || (rows >= 128 * cus && 4 * rows_lds(t, 32) <= kPwLds) ? 4 : 8;
}

// Does an output of the kernel with rows in LDS pass the caches by?  The lines of an output larger than the last-level cache are gone from it before anyone reads them, and leave in the order of
// their rows only if they are not kept: 96 -> 384 on 401408 rows (308 MB) 126 -> 96 us, and 66 in whole lines; of 154 MB, on 200704 rows, 46 -> 52.  (Tiles of codes: 104 -> 88, and 38 -> 44.)
// Beside a residual, which is read 16 bytes of a pixel at a time, also a small one with a reduction of one chunk, by itself and with a layer behind it that reads it (us kept and past the caches:
// 64 -> 64 on 200704 rows 22 and 16, on 401408 38 and 28; 64 -> 256 on 12544 7.8 and 6.0, on 200704 58 and 42; 256 -> 1024 on 12544 17 and 16; GELU, 96 -> 384 on 100352 46 and 42).
inline bool rows_past_caches(const Mx4Dims &t, long long rows, int cout, bool residual) { return rows * cout * 2 > 256ll << 20 || (residual && t.Kq == 1); }

// Does the kernel take such a layer at all?
inline bool fits16(const Mx4Dims &t, long long rows, PwKernel k)
{
    switch (k) {
        case PW16_FEW: return rows <= 32 && few_lds(t, 16, (int)rows) <= kPwLds;
        case PW16_ROWS: return rows_lds(t, 32) <= kPwLds;
        case PW16_ROWS_128: return t.Kq == 1 && rows_lds(t, 128) <= kPwLds;
        default: return true;
    }
}

// On 16-bit input.  Few rows while every workgroup's own quantisation of them is short (1024 -> 4096: 16 rows 4.6 us, and with a quantisation of its own 3.3 + 2.9; 4096 ->
// 4096: 24 rows 9.1 and 6.3 + 3.0).  Otherwise the shorter estimate: of the kernel that quantises in LDS, whose waves walk down the channels (a workgroup's 4 us, 2.6 for each
// 1024 channels of the reduction and 0.11 a step and 32 channels; what follows the first two of a compute unit overlaps, with 4.2 TB/s for what is moved; where LDS holds one
// workgroup of them, nothing overlaps, and there are whole rounds; and the weights, which every 32 rows read again, come at 11 TB/s), or of a quantisation at
// 4 TB/s and the tiled product (measured, the former and the latter: 2048 -> 512 on 3136 rows 13 and 14 us, 512 -> 2048 on 12544 28 and 29, 4096 -> 4096 on 2048 47 and 33, 1024 ->
// 8192 on 12544 135 and 103; many rows and two workgroups of LDS, 2048 -> 2048 on 20000 rows 100 and 76, on 65536 291 and 241, 1024 -> 1024 on 65536 93 and 94; one workgroup,
// 4096 -> 4096 on 20000 rows 378 and 226, on 32768 544 and 340).  128 rows to the workgroup, one tile of them to the wave, with short reductions and many rows (64 -> 256 on
// 200704 rows 47 -> 31 us, on 12544 7.4 and 8.2).
inline PwKernel choose16(const Mx4Dims &t, long long rows, long long cus)
{
    if (rows * t.KB <= 1536 && fits16(t, rows, PW16_FEW)) return PW16_FEW;
    if (!fits16(t, rows, PW16_ROWS)) return PW16_CODES;
    const double K = t.KB * 32.0, out = rows * t.Mt * 64.0;
    const long long blocks = (rows + 31) / 32, splits = rows_splits(t, rows, cus), units = (t.Mt + splits * 8 - 1) / (splits * 8);
    const double one = 4.0 + 0.0025 * K + 0.11 * units * t.Ks, rounds = (double)(blocks * splits) / (2.0 * cus);
    const bool wide = rows >= 128 * cus && fits16(t, rows, PW16_ROWS_128);
    double lds = one + std::max((rounds - 1.0) * (wide ? 0.35 : 0.7) * one, (rows * K * 2 + out) / 4.2e6);
    if (2 * rows_lds(t, 32) > kPwLds) lds = std::max(lds, (double)((blocks * splits + cus - 1) / cus) * one);
    if (!wide) lds = std::max(lds, (double)blocks * t.Mt * t.Ks * 1088 / 11e6);
    const double codes = 3.2 + rows * K * 2.53 / 4e6 + (choose_codes(t, rows, cus) >= PW_FEW_32 ? 4.0 + 0.05 * t.Ks : tiles_us(t, rows, cus));
    if (codes < lds) return PW16_CODES;
    return wide ? PW16_ROWS_128 : PW16_ROWS;
}

}  // namespace ss

#endif
