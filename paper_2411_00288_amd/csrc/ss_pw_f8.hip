// Pointwise layer on FP8 operands with a scale for each block of 128: y = act(Wq xq + bias + residual).
#include "ss_f8.h"
#include "ss_pw_tail.h"
#include "ss_conv_params.h"

namespace ss {

// One product of 32 output channels and 32 pixels over 64 reduction indices: lane l gives the values 32*(l/32) to 31 more of weight row l%32 and of pixel l%32, and, in byte
// SEL of a word, the scale of their block; it gets the channels 8*(v/4) + 4*(l/32) + v%4, v = 0..15, of pixel l%32.  Sums are fp32, but for the products of eight neighbouring indices, which
// are added first and of which the instruction drops what lies below 2^-13 of the largest: an error of 2e-5 to 6e-5 of the sum where half a step of the output is 5e-4 or 4e-3.  (Exact sums
// take the bfloat16 instruction, at half the rate.)
template <int SEL>
__device__ __forceinline__ f32x16 mma_f8(const u32x4 (&a)[2], const u32x4 (&b)[2], const f32x16 &c, uint32_t scale_a, uint32_t scale_b)
{
    const i32x8 wide_a = {(int)a[0][0], (int)a[0][1], (int)a[0][2], (int)a[0][3], (int)a[1][0], (int)a[1][1], (int)a[1][2], (int)a[1][3]};
    const i32x8 wide_b = {(int)b[0][0], (int)b[0][1], (int)b[0][2], (int)b[0][3], (int)b[1][0], (int)b[1][1], (int)b[1][2], (int)b[1][3]};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide_a, wide_b, c, 0, 0, SEL, (int)scale_a, SEL, (int)scale_b);
}

// A step's products with NJ tiles of pixels, from tile J0 on.
template <int SEL, int J0, int MI, int NJ, int NI>
__device__ __forceinline__ void step_f8(const u32x4 (&a)[MI][2], const u32x4 (&b)[NJ][2], f32x16 (&acc)[MI][NI], const uint32_t (&sa)[MI], const uint32_t (&sb)[NI])
{
#pragma unroll
    for (int j = 0; j < NJ; j++)
#pragma unroll
        for (int i = 0; i < MI; i++) acc[i][J0 + j] = mma_f8<SEL>(a[i], b[j], acc[i][J0 + j], sa[i], sb[J0 + j]);
}

// Large products: four waves of MI x NI tiles of 32 x 32, WM of them across the output channels, over chunks of 128 reduction indices: a block, two steps of the instruction.
//   weights     straight from memory into registers, in the instruction's own order, three steps ahead
//   activation  a chunk at a time, straight from memory into one of two LDS buffers, a chunk ahead; 16-byte pieces trade places within their row so that
//               a wave's read of 32 rows does not meet a bank twice
// Four chunks share a scale word, whose byte the instruction picks.  A chunk of which the rows have only half is worked on by half.
// 8192^3 in tiles of 256 x 256 417 to 460 us from card to card (2.4 to 2.6 PFLOP/s of the 4.2 that the instruction sustains alone; 13 registers are spilled behind the loop), in 128 x 128 542; 8192 -> 1024 on 12544
// rows 99 and 127; 1024 -> 1024 on 65536 83 and 76.
template <int DT, int MI, int NI, int WM, int OUT>
__global__ __launch_bounds__(256, MI * NI >= 16 ? 1 : 2) void pw_f8_tile_kernel(PwArgs p, int tiles_m, int tiles_n)
{
    constexpr int WN = 4 / WM, BN = 32 * WN * NI, PIECES = BN / 32;
    // (two variables: reads of one do not wait for loads to the other)
    __shared__ __attribute__((aligned(16))) uint8_t even_s[BN * 128], odd_s[BN * 128];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), half = lane / 32;
    const int Ks = (p.K + 63) / 64, KB = (p.K + 127) / 128, S = (KB + 3) / 4 * 4, Kq = S / 4, Mt = (p.cout + 31) / 32;
    // An XCD (workgroups b, b + 8, ...) works on neighbouring tiles, in bands of eight tiles of channels: 32 of them in flight read 8 + 4 panels.
    const int total = tiles_m * tiles_n, xcd = blockIdx.x % 8;
    const int id = xcd * (total / 8) + min(xcd, total % 8) + blockIdx.x / 8;
    const int band = id / (8 * tiles_n), band_m = min(8, tiles_m - band * 8), in_band = id - band * 8 * tiles_n;
    const int tm = band * 8 + in_band % band_m, tn = in_band / band_m;
    const int mt0 = (tm * WM + wave / WN) * MI;
    const long long row0 = (long long)tn * BN;
    const unsigned pitch = (unsigned)Ks * 64u;
    const int rows = (int)min((long long)BN, p.P - row0);
    const int whole = Ks / 2;
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.codes) + row0 * pitch, 0, (int)(rows * pitch), 0x00020000);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.scales) + row0 * S, 0, rows * S, 0x00020000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w), 0, (int)((unsigned)Mt * Ks * 2048u), 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w_scales), 0, Mt * Kq * 128, 0x00020000);
    // (place l%8 of row l/8 of eight holds piece l%8 ^ l/8, in every other eight rows with the lowest bit turned)
    const unsigned from = (unsigned)(wave * 8 + lane / 8) * pitch + (unsigned)(lane % 8 ^ lane / 8 ^ wave % 2) * 16u;
    auto stage = [&](int q, uint8_t *to) {                  // chunk q, to LDS; past the last, nothing from memory
        const unsigned at = 2 * q < Ks ? from + (unsigned)q * 128u : 0x80000000u;
#pragma unroll
        for (int i = 0; i < PIECES; i++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void *)(to + (i * 4 + wave) * 1024), 16, (int)(at + (unsigned)i * 32u * pitch), 0, 0, 0);
    };
    const int px0 = (wave % WN) * NI * 32;
    auto scale_words = [&](int word, uint32_t (&sa)[MI], uint32_t (&sb)[NI]) {
#pragma unroll
        for (int i = 0; i < MI; i++)
            sa[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ra, (lane % 32) * 4, (min(mt0 + i, Mt - 1) * Kq + min(word, Kq - 1)) * 128, 0);
#pragma unroll
        for (int j = 0; j < NI; j++)                       // (past a row's scales: past the buffer's end, which reads zero)
            sb[j] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, word < Kq ? (px0 + j * 32 + lane % 32) * S + word * 4 : -4, 0, 0);
    };
    // (a step in groups of at most four tiles of pixels: all eight at once, twice, are more registers than there are)
    constexpr int NJ = NI < 4 ? NI : 4, NG = NI / NJ;
    u32x4 wa[4][MI][2], xb[2][NJ][2];
    uint32_t sa[MI], sb[NI], na[MI], nb[NI];
    auto weights = [&](int step, u32x4 (&to)[MI][2]) {
        const int k = min(step, Ks - 1);          // (a step past the last has zeros, a tile past the last is not stored)
        const int at = step < Ks ? lane * 16 : -16;
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int h = 0; h < 2; h++)
                to[i][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, at, ((min(mt0 + i, Mt - 1) * Ks + k) * 2 + h) * 1024, 0));
    };
    auto pixels = [&](const uint8_t *codes_s, int s, int g, u32x4 (&to)[NJ][2]) {
#pragma unroll
        for (int j = 0; j < NJ; j++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int row = px0 + (g * NJ + j) * 32 + lane % 32, b = 4 * s + 2 * half + h;
                to[j][h] = *reinterpret_cast<const u32x4 *>(codes_s + row * 128 + ((b ^ (row & 7) ^ ((row >> 3) & 1)) * 16));
            }
    };
    if constexpr (MI * NI >= 16) {                          // (multiplied by zero weights behind the last chunk: no NaN may stand there)
#pragma unroll
        for (int i = 0; i < BN * 8 / 256; i++) reinterpret_cast<u32x4 *>(even_s)[i * 256 + tid] = reinterpret_cast<u32x4 *>(odd_s)[i * 256 + tid] = u32x4{};
        __syncthreads();
    }
    f32x16 acc[MI][NI] = {};
    scale_words(0, sa, sb);
    __builtin_amdgcn_sched_barrier(0);
    stage(0, even_s);
    __builtin_amdgcn_sched_barrier(0);
    weights(0, wa[0]);
    weights(1, wa[1]);
    __builtin_amdgcn_sched_barrier(0);
    wait_loads<4 * MI>();                                   // chunk 0 is there
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
    stage(1, odd_s);
    __builtin_amdgcn_sched_barrier(0);
    weights(2, wa[2]);
    pixels(even_s, 0, 0, xb[0]);
    // Chunk q, its number modulo four known: while a group's products are made, the next group's pixels and the weights of the third step from it come; the
    // barrier stands before the last group, in front of the next chunk's first read and behind the last of the current one's, whose buffer is then filled with the
    // chunk after the next.  No branches: the compiler moves matrix instructions behind one, away from their loads; what is loaded behind the last chunk is not used.
    // LOOP: within the loop, where every load has a reader.  Of the chunks behind it some have none, which the compiler removes: a count of them there would let pieces of the next chunk
    // be on their way when other waves read them, so all is waited for.  (96 -> 384 on 401408 rows 84 us, 80 with the count; a last chunk without the barrier and what it asks for takes the
    // tiles of 128 x 128 registers: 85, and 65536 x 448 -> 1024 50 -> 51.)
    auto chunk = [&](int q, auto number, auto loop) {
        constexpr int N = decltype(number)::value;
        constexpr bool LOOP = decltype(loop)::value;
        uint8_t *const mine = N % 2 ? odd_s : even_s, *const other = N % 2 ? even_s : odd_s;
        const auto group = [&](auto which) {
            constexpr int W = decltype(which)::value, s = W / NG, g = W % NG, next = (W + 1) % (2 * NG);
            __builtin_amdgcn_sched_barrier(0);
            if (next == 0) {
                wait_loads<LOOP ? 4 * MI + (N == 1 ? MI + NI : 0) : 0>();           // the next chunk is there: what came behind it may be under way
                lds_barrier();
                __builtin_amdgcn_sched_barrier(0);
                stage(q + 2, mine);
                __builtin_amdgcn_sched_barrier(0);          // (the count above is of the loads behind it)
            }
            pixels(next == 0 ? other : mine, next / NG, next % NG, xb[(W + 1) % 2]);
            if (g == 0) weights(2 * q + s + 3, wa[(2 * N + s + 3) % 4]);
            if (N == 1 && W == 0) scale_words(q / 4 + 1, na, nb);
            step_f8<N, g * NJ>(wa[(2 * N + s) % 4], xb[W % 2], acc, sa, sb);
#pragma unroll
            for (int i = 0; i < MI * NJ; i++) {             // between two matrix instructions each, some of the others
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x320, 2, 0);
            }
        };
        group(Int<0>{});
        group(Int<1>{});
        if constexpr (NG == 2) {
            group(Int<2>{});
            group(Int<3>{});
        }
        if constexpr (N == 3) {
#pragma unroll
            for (int i = 0; i < MI; i++) sa[i] = na[i];
#pragma unroll
            for (int j = 0; j < NI; j++) sb[j] = nb[j];
        }
    };
    int q = 0;
    // The largest tiles have no registers for a way out of the middle: they go on to a scale word's end, with zero weights.
    const int end = MI * NI >= 16 ? (Ks + 1) / 2 : whole - 3;
    for (; q < end; q += 4) {
        chunk(q, Int<0>{}, std::true_type{});
        chunk(q + 1, Int<1>{}, std::true_type{});
        chunk(q + 2, Int<2>{}, std::true_type{});
        chunk(q + 3, Int<3>{}, std::true_type{});
    }
    if constexpr (MI * NI < 16) {
        const int left = whole - q;
        if (left > 0) chunk(q, Int<0>{}, std::false_type{});
        if (left > 1) chunk(q + 1, Int<1>{}, std::false_type{});
        if (left > 2) chunk(q + 2, Int<2>{}, std::false_type{});
        if (Ks % 2) {
            if (left == 0) step_f8<0, 0>(wa[0], xb[0], acc, sa, sb);
            if (left == 1) step_f8<1, 0>(wa[2], xb[0], acc, sa, sb);
            if (left == 2) step_f8<2, 0>(wa[0], xb[0], acc, sa, sb);
            if (left == 3) step_f8<3, 0>(wa[2], xb[0], acc, sa, sb);
        }
    }
    wait_loads<0>();                                        // (no load to LDS outlives its workgroup)
    if ((mt0 + MI) * 32 <= p.cout && row0 + px0 + NI * 32 <= p.P)              // uniform
        pw_store<DT, MI, NI, true, true, OUT>(p, acc, mt0, row0 + px0, lane);
    else
        pw_store<DT, MI, NI, false, true, KEPT>(p, acc, mt0, row0 + px0, lane);
}

// 16-bit input rows of a workgroup, quantised into LDS.  Piece b (16 channels) of row r stands at ((b * pad + r) * 16): the lanes of a fragment read consecutive
// pieces.  WIDE: K is at least 8.  The scale of block k is byte k % 4 of word (k / 4) * pad + r.  Pieces 0 .. 4 Ks - 1, rows 0 .. count - 1; what is past the
// matrix is zero.
template <int DT, int THREADS, int U, bool WIDE>
__device__ __forceinline__ void quantise_rows(const PwRowsArgs &r, long long row0, int rows, int count, int K, int Ks, int pad, uint8_t *codes_s, uint8_t *scales_s)
{
    const int runs = (Ks + 1) / 2 * 16, total = count * runs;
    const uint16_t *const x = r.x + row0 * r.ldx;
    int row = (int)(((unsigned long long)threadIdx.x * r.mul) >> r.sh), run = (int)threadIdx.x - row * runs;
    for (int base = 0; base < total; base += THREADS * U) {
        Run<DT> raw[U];
        int rw[U], rn[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            rw[u] = row;
            rn[u] = run;
            if (base + u * THREADS < total) {              // uniform
                if constexpr (WIDE)
                    raw[u] = load_wide<DT, false>(x + (long long)min(row, rows - 1) * (int)r.ldx, run * 8, K);
                else
                    raw[u] = load_run<DT>(x + (long long)row * (int)r.ldx + run * 8, row < rows ? K - run * 8 : 0);
            }
            row += r.step_row;
            run += r.step_run;
            if (run >= runs) {
                run -= runs;
                row++;
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (base + u * THREADS >= total) break;        // uniform
            const int b = rn[u] / 2, k = rn[u] / 16;
            if constexpr (WIDE) place_wide<DT>(raw[u], rn[u] * 8, K, rw[u] < rows);
            const uint32_t byte = f8_scale(row16_max(magnitude<DT>(raw[u])));
            const u32x2 c = f8_codes<DT>(raw[u], byte);
            if (rw[u] >= count) continue;
            if (b < 4 * Ks) *reinterpret_cast<u32x2 *>(codes_s + (__umul24(b, pad) + rw[u]) * 16 + rn[u] % 2 * 8) = c;
            if (rn[u] % 16 == 0) scales_s[(__umul24(k / 4, pad) + rw[u]) * 4 + k % 4] = (uint8_t)byte;
        }
    }
}

// Layers on 16-bit input whose reduction fits LDS: a workgroup quantises its 32 NT rows once, and its waves take units of output channels and 32 rows in turn (the
// units of the same channels side by side, so that their weights are in the L1).  The input is read once, whatever the number of channels, unless there are few
// rows: then several workgroups share the channels of one's rows.  The next weights are on their way from the L2 while the current ones are multiplied or, with a
// reduction of one block (SHORT), while the sums are finished.  One block: units of 64 channels; longer: units of 32.
// Bound by memory: 96 -> 384 on 401408 rows 76 us (5.1 TB/s), 64 -> 256 on 200704 32, 384 -> 96 on 401408 84; with a residual, 64 -> 256 on 200704 58 (4.0 TB/s).
template <int DT, int NT, bool SHORT, bool WIDE, int THREADS>
__global__ __launch_bounds__(THREADS, SHORT && NT == 1 ? 3 : 4) void pw_f8_rows_kernel(PwArgs p, PwRowsArgs r)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    constexpr int PX = 32 * NT, PAD = PX + 1, WAVES = THREADS / 64, MI = SHORT ? 2 : 1;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const int Ks = (p.K + 63) / 64, KB = SHORT ? 1 : (p.K + 127) / 128, Kq = (KB + 3) / 4, Mt = (p.cout + 31) / 32;
    const unsigned part = blockIdx.x / r.blocks;
    const int first = (int)part * r.units * NT, units = min((Mt + MI - 1) / MI, ((int)part + 1) * r.units) * NT;
    const long long row0 = (long long)(blockIdx.x - part * r.blocks) * PX;
    uint8_t *const codes_s = smem, *const scales_s = smem + 4 * Ks * PAD * 16;
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w), 0, (int)((unsigned)Mt * Ks * 2048u), 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w_scales), 0, Mt * Kq * 128, 0x00020000);
    u32x4 wa[2][MI][2], wn[2][MI][2];
    uint32_t sa[MI], sn[MI];
    auto fetch = [&](int mt, int q, u32x4 (&w)[2][MI][2], uint32_t (&sc)[MI]) {
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = min(mt + i, Mt - 1);
            sc[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ra, (lane % 32) * 4, (m * Kq + q / 4) * 128, 0) >> (8 * (q % 4));
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int h = 0; h < 2; h++)
                    w[s][i][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, lane * 16, ((m * Ks + min(q * 2 + s, Ks - 1)) * 2 + h) * 1024, 0));
        }
    };
    auto multiply = [&](int at, int q, f32x16 (&acc)[MI][1]) {
        const uint32_t sb[1] = {*reinterpret_cast<const uint32_t *>(scales_s + ((q / 4) * PAD + at + lane % 32) * 4) >> (8 * (q % 4))};
#pragma unroll
        for (int s = 0; s < 2; s++) {
            if (q * 2 + s < Ks) {
                u32x4 xb[1][2];
#pragma unroll
                for (int h = 0; h < 2; h++) xb[0][h] = *reinterpret_cast<const u32x4 *>(codes_s + ((8 * q + 4 * s + 2 * half + h) * PAD + at + lane % 32) * 16);
                step_f8<0, 0>(wa[s], xb, acc, sa, sb);
            }
        }
    };
    // The sums start from the bias, which waits in LDS: a load behind the last unit's stores would wait for those, too.
    float *const bias_s = reinterpret_cast<float *>(scales_s + (Kq * PAD * 4 + 15) / 16 * 16);
    auto start = [&](int mt, f32x16 (&acc)[MI][1]) {
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const f32x4 b = *reinterpret_cast<const f32x4 *>(bias_s + min(mt + i, Mt - 1) * 32 + 8 * g + 4 * half);
#pragma unroll
                for (int e = 0; e < 4; e++) acc[i][0][4 * g + e] = b[e];
            }
    };
    for (int o = threadIdx.x; o < Mt * 32; o += THREADS) bias_s[o] = p.bias != nullptr && o < p.cout ? p.bias[o] : 0.f;
    if constexpr (SHORT)
        fetch(min((first + wave) / NT * MI, Mt - 1), 0, wa, sa);
    else
        fetch(min((first + wave) / NT * MI, Mt - 1), 0, wn, sn);
    quantise_rows<DT, THREADS, SHORT ? 4 : 8, WIDE>(r, row0, (int)min((long long)PX, p.P - row0), PX, p.K, Ks, PAD, codes_s, scales_s);
    __syncthreads();
    // Whole tiles have a loop of their own: a load is waited for by the number of memory instructions behind it, and the compiler takes the least of any way
    // through the loop for it, so that tiles with fewer stores would have every wave wait for the stores of the others.
    __builtin_amdgcn_s_waitcnt(0x0F70);                    // (vmcnt 0, the first weights: so that the loop is entered with none on their way)
    const auto walk = [&](auto whole, auto out, auto with) {
        constexpr bool ALL = decltype(whole)::value;
        constexpr int OUT = decltype(out)::value, WITH = decltype(with)::value;
        f32x16 acc[MI][1];
        int unit = first + wave, q = 0;
        start(unit / NT * MI, acc);
        while (unit < units) {
            const int mt = unit / NT * MI, at = unit % NT * 32;
            if constexpr (SHORT) {
                multiply(at, 0, acc);
                unit += WAVES;
                fetch(min(unit / NT * MI, Mt - 1), 0, wa, sa);
                pw_store<DT, MI, 1, ALL, false, OUT, WITH>(p, acc, mt, row0 + at, lane);
                __builtin_amdgcn_sched_barrier(0);
                start(unit / NT * MI, acc);
            } else {
#pragma unroll
                for (int i = 0; i < MI; i++) {
                    sa[i] = sn[i];
#pragma unroll
                    for (int s = 0; s < 2; s++)
#pragma unroll
                        for (int h = 0; h < 2; h++) wa[s][i][h] = wn[s][i][h];
                }
                const bool done = q + 1 == KB;
                const int next = done ? unit + WAVES : unit, nq = done ? 0 : q + 1;
                fetch(min(next / NT * MI, Mt - 1), nq, wn, sn);
                multiply(at, q, acc);
                if (done) {
                    pw_store<DT, MI, 1, ALL, false, OUT, WITH>(p, acc, mt, row0 + at, lane);
                    start(next / NT * MI, acc);
                }
                unit = next;
                q = nq;
            }
        }
    };
    // (a residual takes registers: in a loop that looks for one the others' sums are spilled, 401408 x 96 -> 384 in 4 bits 78 -> 86 us)
    const auto ways = [&](auto with) {
        if (p.cout % 64 != 0 || row0 + PX > p.P)
            walk(std::false_type{}, Int<KEPT>{}, with);
        else if (!p.stream)
            walk(std::true_type{}, Int<KEPT>{}, with);
        else if (!SHORT || p.act == SS_ACT_GELU)
            walk(std::true_type{}, Int<PAST>{}, with);
        else if constexpr (SHORT)
            walk(std::true_type{}, Int<LINES>{}, with);
    };
    if (p.residual == nullptr)
        ways(Int<NO_RES>{});
    else
        ways(Int<RES>{});
}

// Few rows: bound by reading the weights once, or by a memory latency or two.  A workgroup makes 32 output channels of 32 NI rows; its NW waves share
// the reduction, a block of 128 each in turn, and join their sums in LDS.  QUANT: the rows are quantised into LDS first, by all threads, while the first
// weights are on their way.  2048 -> 1000 on one row 4.3 us, 8192 -> 8192 on 16 rows on codes 15 us (67 MB of weights at 4.5 TB/s).
template <int DT, int NW, int NI, bool QUANT, bool WIDE>
__global__ __launch_bounds__(NW * 64) void pw_f8_few_kernel(PwArgs p, PwRowsArgs r)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    static_assert(!QUANT || NI == 1, "rows in LDS");
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const int Ks = (p.K + 63) / 64, KB = (p.K + 127) / 128, S = (KB + 3) / 4 * 4, Kq = S / 4, Mt = (p.cout + 31) / 32;
    const int mt = blockIdx.x % Mt;
    const long long row0 = (long long)(blockIdx.x / Mt) * (32 * NI);
    const int rows = (int)min((long long)(32 * NI), p.P - row0), pad = rows | 1;
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w) + (size_t)mt * Ks * 2048, 0, Ks * 2048, 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w_scales) + (size_t)mt * Kq * 128, 0, Kq * 128, 0x00020000);
    // (the offsets are the lanes' own: only those are held against the buffer's end, which a step past the last reads zeros behind)
    auto weights = [&](int q, u32x4 (&wa)[2][1][2], uint32_t &word) {
        word = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ra, (q / 4) * 128 + (lane % 32) * 4, 0, 0);
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int h = 0; h < 2; h++) wa[s][0][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, (q * 4 + s * 2 + h) * 1024 + lane * 16, 0, 0));
    };
    u32x4 wa[2][1][2], wn[2][1][2];
    uint32_t word_a, word_n;
    weights(wave, wa, word_a);
    weights(wave + NW, wn, word_n);
    uint8_t *const scales_s = smem + 4 * Ks * pad * 16;
    if constexpr (QUANT) {
        quantise_rows<DT, NW * 64, 8, WIDE>(r, row0, rows, rows, p.K, Ks, pad, smem, scales_s);
        __syncthreads();
    }
    f32x16 acc[1][NI] = {};
    const uint8_t *px[NI], *ps[NI];
#pragma unroll
    for (int j = 0; j < NI; j++) {
        const int row = min(j * 32 + lane % 32, rows - 1);                     // (lanes past the last row repeat it)
        px[j] = QUANT ? smem + (2 * half * pad + row) * 16 : p.codes + (row0 + row) * (Ks * 64) + half * 32;
        ps[j] = QUANT ? scales_s + row * 4 : p.scales + (row0 + row) * S;
    }
    const int step_at = QUANT ? 4 * pad * 16 : 64, piece_at = QUANT ? pad * 16 : 16, word_at = QUANT ? pad * 4 : 4;
    for (int q = wave; q < KB; q += NW) {
        u32x4 xb[2][NI][2];
        uint32_t sa[1], sb[NI];
        const int turn = 8 * (q % 4);
        sa[0] = word_a >> turn;
#pragma unroll
        for (int j = 0; j < NI; j++) {
            sb[j] = *reinterpret_cast<const uint32_t *>(ps[j] + q / 4 * word_at) >> turn;
#pragma unroll
            for (int s = 0; s < 2; s++)
#pragma unroll
                for (int h = 0; h < 2; h++) xb[s][j][h] = *reinterpret_cast<const u32x4 *>(px[j] + min(2 * q + s, Ks - 1) * step_at + h * piece_at);
        }
        // (a step past the last has zero weights, and the last step's pixels again)
        step_f8<0, 0>(wa[0], xb[0], acc, sa, sb);
        if (2 * q + 1 < Ks) step_f8<0, 0>(wa[1], xb[1], acc, sa, sb);
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int h = 0; h < 2; h++) wa[s][0][h] = wn[s][0][h];
        word_a = word_n;
        weights(q + 2 * NW, wn, word_n);
    }
    // the waves' sums, 32 rows at a time: register v of lane l at (wave * 16 + v) * 65 + l, so that 32 channels of a row are 32 banks
    float *const sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int j = 0; j < NI; j++) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < 16; v++) sums[(wave * 16 + v) * 65 + lane] = acc[0][j][v];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16 / NW; i++) {
            const int at = i * NW * 64 + threadIdx.x, c = at % 32, row = j * 32 + at / 32, o = mt * 32 + c;
            if (row >= rows || o >= p.cout) continue;
            const int v = c / 8 * 4 + c % 4, l = c / 4 % 2 * 32 + at / 32;
            float z = p.bias != nullptr ? p.bias[o] : 0.f;
            if (p.residual != nullptr) z += widen<DT>(p.residual[(row0 + row) * p.ldr + o]);
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < NW; w++) s += sums[(w * 16 + v) * 65 + l];
            z += s;
            if (p.act == SS_ACT_RELU) z = floor_at(z, 0.f);
            if (p.act == SS_ACT_GELU) z = gelu_cdf<DT>(z);
            store1<DT>(p.y + (row0 + row) * p.ldy + o, z);
        }
    }
}

namespace {

int check_f8(const ss_weight_desc *d)
{
    size_t bytes;
    return ss_f8_packed_bytes(d, &bytes);
}

int check_pw_f8(const ss_weight_desc *d, int64_t rows, const void *packed, const float *bias, const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy)
{
    const int st = check_f8(d);
    if (st != SS_OK) return st;
    if (act != SS_ACT_NONE && act != SS_ACT_RELU && act != SS_ACT_GELU) return SS_ERR_INVALID_ARG;
    if (rows < 0 || ldy < d->cout || (residual && ldr < d->cout)) return SS_ERR_INVALID_ARG;
    if (rows > INT32_MAX || ldy > INT32_MAX || (residual && ldr > INT32_MAX)) return SS_ERR_UNSUPPORTED;
    if (rows == 0) return SS_OK;
    if (!packed || !y || !aligned(packed, 16) || !aligned(y, 2) || !aligned(bias, 4) || !aligned(residual, 2)) return SS_ERR_INVALID_ARG;
    return SS_OK;
}

size_t to256(size_t bytes) { return (bytes + 255) / 256 * 256; }

PwArgs pw_args(const ss_weight_desc *d, int64_t rows, const void *packed, const float *bias, const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy)
{
    const F8Dims t = f8_dims(d->cout, d->cin);
    PwArgs a{};
    a.w = static_cast<const uint8_t *>(packed) + kHeaderBytes;
    a.w_scales = static_cast<const uint8_t *>(packed) + f8_scales_at(t);
    a.bias = bias;
    a.residual = static_cast<const uint16_t *>(residual);
    a.y = static_cast<uint16_t *>(y);
    a.ldr = ldr;
    a.ldy = ldy;
    a.P = (int)rows;
    a.cout = d->cout;
    a.K = d->cin;
    a.act = act;
    a.stream = rows * d->cout * 2ll > 256ll << 20;        // (an output that the last-level cache does not hold)
    return a;
}

// The test hook's kernel, or the library's choice.
F8Kernel codes_kernel(const F8Dims &t, long long rows)
{
    const int forced = forced_tile();
    if (forced >= F8_TILE_64 && forced <= F8_FEW_64) return (F8Kernel)forced;
    return choose_f8_codes(t, rows, std::max(compute_units(), 1));
}

F8Kernel kernel16(const F8Dims &t, long long rows)
{
    const int forced = forced_tile();
    if (forced >= F816_FEW && forced <= F816_CODES && f8_fits16(t, rows, (F8Kernel)forced)) return (F8Kernel)forced;
    return choose_f8_16(t, rows, std::max(compute_units(), 1));
}

template <int DT, int MI, int NI, int WM, int OUT>
int launch_tile(const PwArgs &a, const F8Dims &t, hipStream_t s)
{
    constexpr int BN = 32 * NI * (4 / WM);
    const long long tm = (t.Mt + MI * WM - 1) / (MI * WM), tn = ((long long)a.P + BN - 1) / BN;
    if (tm * tn > 0xFFFFFFll) return SS_ERR_UNSUPPORTED;
    pw_f8_tile_kernel<DT, MI, NI, WM, OUT><<<dim3((unsigned)(tm * tn)), dim3(256), 0, s>>>(a, (int)tm, (int)tn);
    return launched();
}

template <int DT>
int product_codes(const PwArgs &a, const F8Dims &t, F8Kernel kernel, hipStream_t s)
{
    const auto tile = [&](auto mi, auto ni, auto wm) -> int {
        constexpr int MI = decltype(mi)::value, NI = decltype(ni)::value, WM = decltype(wm)::value;
        return a.stream ? launch_tile<DT, MI, NI, WM, LINES>(a, t, s) : launch_tile<DT, MI, NI, WM, KEPT>(a, t, s);
    };
    const auto few = [&](auto ni) -> int {
        constexpr int NI = decltype(ni)::value;
        const long long blocks = ((long long)a.P + 32 * NI - 1) / (32 * NI) * t.Mt;
        if (blocks > 0x3FFFFFll) return SS_ERR_UNSUPPORTED;
        if (NI == 2 || t.KB > 8) return launch_lds<pw_f8_few_kernel<DT, 16, NI, false, false>>(blocks, 1024, f8_few_lds(t, 16, 0), s, a, PwRowsArgs{});
        if constexpr (NI == 1)              // (two tiles of rows are for long reductions)
            return t.KB > 4 ? launch_lds<pw_f8_few_kernel<DT, 8, NI, false, false>>(blocks, 512, f8_few_lds(t, 8, 0), s, a, PwRowsArgs{})
                            : launch_lds<pw_f8_few_kernel<DT, 4, NI, false, false>>(blocks, 256, f8_few_lds(t, 4, 0), s, a, PwRowsArgs{});
    };
    switch (kernel) {
        case F8_TILE_64: return tile(Int<1>{}, Int<1>{}, Int<2>{});
        case F8_TILE_128: return tile(Int<1>{}, Int<4>{}, Int<4>{});
        case F8_TILE_256: return tile(Int<2>{}, Int<8>{}, Int<4>{});
        case F8_FEW_32: return few(Int<1>{});
        default: return few(Int<2>{});
    }
}

template <int DT>
int product16(const PwArgs &a, const F8Dims &t, F8Kernel kernel, const void *x, int64_t ldx, hipStream_t s)
{
    PwRowsArgs r{};
    r.x = static_cast<const uint16_t *>(x);
    r.ldx = ldx;
    const int runs = t.KB * 16;
    fast_div_setup((unsigned)runs, &r.mul, &r.sh);
    const auto go = [&](auto wide) -> int {
        constexpr bool WIDE = decltype(wide)::value;
        const auto few = [&](auto nw) -> int {
            constexpr int NW = decltype(nw)::value;
            r.step_row = NW * 64 / runs;
            r.step_run = NW * 64 % runs;
            return launch_lds<pw_f8_few_kernel<DT, NW, 1, true, WIDE>>(t.Mt, NW * 64, f8_few_lds(t, NW, a.P), s, a, r);
        };
        const auto rows = [&](auto nt, auto brief, auto threads) -> int {
            constexpr int NT = decltype(nt)::value, THREADS = decltype(threads)::value;
            // Where a call moves more than most of the last-level cache, half lines of its output are gone from there before their other halves come: 64 -> 256 with a residual on 200704 rows,
            // 231 MB, wrote 1.35 times its output and took 69 us, and 1.14 times and 58 in whole lines past the caches.  (Tiles of codes, the same layer: 57 by the caches, 62 past them.)
            PwArgs b = a;
            b.stream = a.stream || a.P * (2ll * a.cout * (a.residual != nullptr ? 2 : 1) + 2ll * a.K) > 192ll << 20;
            r.step_row = THREADS / runs;
            r.step_run = THREADS % runs;
            const long long blocks = ((long long)a.P + 32 * NT - 1) / (32 * NT);
            const int splits = NT == 1 ? f8_rows_splits(t, a.P, std::max(compute_units(), 1)) : 1;
            r.blocks = (unsigned)blocks;
            r.units = ((decltype(brief)::value ? (t.Mt + 1) / 2 : t.Mt) + splits - 1) / splits;
            return launch_lds<pw_f8_rows_kernel<DT, NT, decltype(brief)::value, WIDE, THREADS>>(blocks * splits, THREADS, f8_rows_lds(t, 32 * NT), s, b, r);
        };
        if (kernel == F816_FEW) {
            const int waves = f8_few16_waves(t, a.P, a.K);
            return waves == 16 ? few(Int<16>{}) : waves == 8 ? few(Int<8>{}) : few(Int<4>{});
        }
        if (kernel == F816_ROWS_128) return rows(Int<4>{}, std::true_type{}, Int<256>{});
        if (t.KB == 1) return rows(Int<1>{}, std::true_type{}, Int<256>{});
        return f8_rows_waves(t, a.P, std::max(compute_units(), 1)) == 4 ? rows(Int<1>{}, std::false_type{}, Int<256>{}) : rows(Int<1>{}, std::false_type{}, Int<512>{});
    };
    return a.K >= 8 ? go(std::true_type{}) : go(std::false_type{});
}

// The layer in pieces of `piece` rows, so that no launch has 2^32 threads: launch(arguments, first row).
template <typename F>
int in_pieces(const PwArgs &all, long long piece, F &&launch)
{
    for (long long at = 0; at < all.P; at += piece) {
        PwArgs a = all;
        a.P = (int)std::min(piece, all.P - at);
        a.y += at * a.ldy;
        if (a.residual != nullptr) a.residual += at * a.ldr;
        const int st = launch(a, at);
        if (st != SS_OK) return st;
    }
    return SS_OK;
}

int product(const ss_weight_desc *d, const PwArgs &all, const uint8_t *codes, const uint8_t *scales, hipStream_t s)
{
    const F8Dims t = f8_dims(d->cout, d->cin);
    return in_pieces(all, piece_rows(4ll * ((t.Mt + 1) / 2)), [&](PwArgs &a, long long at) {       // (tiles of 64 x 64 have the most threads)
        a.codes = codes + at * t.P;
        a.scales = scales + at * t.S;
        const F8Kernel kernel = codes_kernel(t, a.P);
        return d->dtype == SS_F16 ? product_codes<SS_F16>(a, t, kernel, s) : product_codes<SS_BF16>(a, t, kernel, s);
    });
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_pw_f8_q_fwd(const ss_weight_desc *desc, const void *codes, const void *scales, int64_t rows, const void *packed, const float *bias,
                              const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy, void *stream)
{
    const int st = check_pw_f8(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (st != SS_OK) return st;
    if (rows == 0) return SS_OK;
    if (!codes || !scales || !aligned(codes, 16) || !aligned(scales, 4)) return SS_ERR_INVALID_ARG;
    return product(desc, pw_args(desc, rows, packed, bias, residual, ldr, act, y, ldy), static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales),
                   static_cast<hipStream_t>(stream));
}

extern "C" int ss_pw_f8_workspace_bytes(const ss_weight_desc *desc, int64_t rows, size_t *bytes)
{
    const int st = check_f8(desc);
    if (st != SS_OK) return st;
    if (!bytes || rows < 0) return SS_ERR_INVALID_ARG;
    if (rows > INT32_MAX) return SS_ERR_UNSUPPORTED;
    const F8Dims t = f8_dims(desc->cout, desc->cin);
    *bytes = rows > 0 && kernel16(t, rows) == F816_CODES ? to256((size_t)rows * t.P) + (size_t)rows * t.S : 0;
    return SS_OK;
}

extern "C" int ss_pw_f8_fwd(const ss_weight_desc *desc, const void *x, int64_t rows, int64_t ldx, const void *packed, const float *bias, const void *residual,
                            int64_t ldr, int32_t act, void *y, int64_t ldy, void *workspace, size_t ws_bytes, void *stream)
{
    int st = check_pw_f8(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (st != SS_OK) return st;
    if (ldx < desc->cin) return SS_ERR_INVALID_ARG;
    if (ldx > INT32_MAX) return SS_ERR_UNSUPPORTED;
    if (rows == 0) return SS_OK;
    if (!x || !aligned(x, 2)) return SS_ERR_INVALID_ARG;
    const F8Dims t = f8_dims(desc->cout, desc->cin);
    const F8Kernel kernel = kernel16(t, rows);
    const size_t codes_bytes = to256((size_t)rows * t.P);
    if (kernel == F816_CODES && (!workspace || !aligned(workspace, 16) || ws_bytes < codes_bytes + (size_t)rows * t.S)) return SS_ERR_WORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const PwArgs a = pw_args(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (kernel != F816_CODES)
        return in_pieces(a, piece_rows(16), [&](const PwArgs &part, long long at) {                // (eight waves to 32 rows)
            const void *const first = static_cast<const uint16_t *>(x) + at * ldx;
            return desc->dtype == SS_F16 ? product16<SS_F16>(part, t, kernel, first, ldx, s) : product16<SS_BF16>(part, t, kernel, first, ldx, s);
        });
    uint8_t *codes = static_cast<uint8_t *>(workspace), *scales = codes + codes_bytes;
    st = f8_quantize(x, rows, desc->cin, ldx, desc->dtype, codes, scales, s);
    if (st != SS_OK) return st;
    return product(desc, a, codes, scales, s);
}
