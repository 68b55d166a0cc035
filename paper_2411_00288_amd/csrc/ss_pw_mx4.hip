// Pointwise layer on MXFP4 operands: y = act(Wq xq + bias + residual).
#include "ss_mx4.h"
#include "ss_pw_tail.h"
#include "ss_conv_params.h"

namespace ss {

// One product of 32 output channels and 32 pixels over 64 reduction indices: lane l gives the 32 values of block l/32 of weight row l%32 and of
// pixel l%32, and the byte of their scales; it gets the channels 8*(v/4) + 4*(l/32) + v%4, v = 0..15, of pixel l%32.
template <int SEL>
__device__ __forceinline__ f32x16 mma_mx4(const u32x4 &a, const u32x4 &b, const f32x16 &c, uint32_t scale_a, uint32_t scale_b)
{
    const i32x8 wide_a = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, wide_b = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide_a, wide_b, c, 4, 4, SEL, (int)scale_a, SEL, (int)scale_b);
}

constexpr int kChunk = 8;                                  // blocks of a reduction chunk: 256 channels, four steps, one scale word

// The product of step s of a scale word.
template <int MI, int NI>
__device__ __forceinline__ void step_mx4(int s, const u32x4 (&a)[MI], const u32x4 (&b)[NI], f32x16 (&acc)[MI][NI], const uint32_t (&sa)[MI], const uint32_t (&sb)[NI])
{
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NI; j++) {
            if (s == 0) acc[i][j] = mma_mx4<0>(a[i], b[j], acc[i][j], sa[i], sb[j]);
            if (s == 1) acc[i][j] = mma_mx4<1>(a[i], b[j], acc[i][j], sa[i], sb[j]);
            if (s == 2) acc[i][j] = mma_mx4<2>(a[i], b[j], acc[i][j], sa[i], sb[j]);
            if (s == 3) acc[i][j] = mma_mx4<3>(a[i], b[j], acc[i][j], sa[i], sb[j]);
        }
}

// Large products: four waves of MI x NI tiles of 32 x 32, WM of them across the output channels.
//   weights     straight from memory into registers, in the instruction's own order, three steps (of 64 reduction indices) ahead
//   activation  256 channels at a time, straight from memory into one of two LDS buffers, a chunk ahead; 16-byte pieces trade places within their row so that
//               a wave's read of 32 rows does not meet a bank twice
// What goes through registers to LDS, or is loaded by two waves, costs: with the activation in registers on its way and 2 x 2 waves of 4 x 4 tiles 8192^3 took 287 us, with loads to
// LDS 257, with four waves across the channels, 2 x 8 tiles each, none of whose weights another loads, 255; in 128 x 128 tiles 1 x 4 instead of 2 x 2 376 -> 345, and 315 with
// the pixels' scales, of which a load finds 64 lines, brought for two chunks at a time.
// A reduction past the last block meets zero scales on both sides; rows past the last are not stored.
template <int DT, int MI, int NI, int WM, int OUT>
__global__ __launch_bounds__(256, MI * NI >= 16 ? 1 : 2) void pw_mx4_tile_kernel(PwArgs p, int tiles_m, int tiles_n)
{
    constexpr int WN = 4 / WM, BN = 32 * WN * NI, PIECES = BN / 32;
    // (two variables: reads of one do not wait for loads to the other)
    __shared__ __attribute__((aligned(16))) uint8_t even_s[BN * kChunk * 16], odd_s[BN * kChunk * 16];
    constexpr int NW = NI < 4 ? NI : 4;                    // scale words of a read
    using Words = std::conditional_t<NW == 1, uint32_t, uint32_t __attribute__((ext_vector_type(NW)))>;
    __shared__ Words scales_s[2][4][BN / NW];              // [pair of chunks][word: two to the chunk][wave and lane]: each of the lane's pixels
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int KB = (p.K + 31) / 32, S = (KB + 3) / 4 * 4, Ks = (KB + 1) / 2, Kq = (Ks + 3) / 4, Mt = (p.cout + 31) / 32;
    // An XCD (workgroups b, b + 8, ...) works on neighbouring tiles, in bands of eight tiles of channels: 32 of them in flight read 8 + 4 panels.
    const int total = tiles_m * tiles_n, xcd = blockIdx.x % 8;
    const int id = xcd * (total / 8) + min(xcd, total % 8) + blockIdx.x / 8;
    const int band = id / (8 * tiles_n), band_m = min(8, tiles_m - band * 8), in_band = id - band * 8 * tiles_n;
    const int tm = band * 8 + in_band % band_m, tn = in_band / band_m;
    const int mt0 = (tm * WM + wave / WN) * MI;
    const long long row0 = (long long)tn * BN;
    const unsigned pitch = (unsigned)KB * 16u;
    const int rows = (int)min((long long)BN, p.P - row0);
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.codes) + row0 * pitch, 0, (int)(rows * pitch), 0x00020000);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.scales) + row0 * S, 0, rows * S, 0x00020000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w), 0, Mt * Ks * 1024, 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w_scales), 0, Mt * Kq * 256, 0x00020000);
    constexpr int WORDS = BN / 64;                         // scale words that a thread brings of a pair of chunks
    const int px = tid % BN, word0 = tid / BN * WORDS;
    uint32_t ps[WORDS];
    // (place l%8 of row l/8 of eight holds block l%8 ^ l/8, in every other eight rows with the lowest bit turned)
    const unsigned from = (unsigned)(wave * 8 + lane / 8) * pitch + (unsigned)(lane % 8 ^ lane / 8 ^ wave % 2) * 16u;
    auto stage = [&](int q, uint8_t *to) {                  // chunk q of the activation, to LDS; past the last, nothing from memory
        const unsigned at = q < Kq ? from + (unsigned)q * (kChunk * 16) : 0x80000000u;
#pragma unroll
        for (int i = 0; i < PIECES; i++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void *)(to + (i * 4 + wave) * 1024), 16, (int)(at + (unsigned)i * 32u * pitch), 0, 0, 0);
    };
    // The scales of a pair of chunks, to registers and on to LDS: a line of them is not loaded twice for two chunks.
    auto fetch = [&](int pair, int first, int last) {
#pragma unroll
        for (int d = first; d < last; d++) {
            const int b = (pair * 4 + word0 + d) * 4;      // (past a row's scales: past the buffer's end, which reads zero)
            ps[d] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, b < S ? px * S + b : -4, 0, 0);
        }
    };
    auto fill = [&](int pair) {
#pragma unroll
        for (int d = 0; d < WORDS; d++)
            reinterpret_cast<uint32_t *>(scales_s[pair & 1][word0 + d])[(px / (32 * NI) * 32 + px % 32) * NI + px / 32 % NI] = ps[d];
    };
    u32x4 wa[4][MI];
    uint32_t sa[MI], na[MI];
    auto weights = [&](int ks, u32x4 (&to)[MI]) {
        const int k = min(ks, Ks - 1);                     // (a step past the last has zero scales, a tile past the last is not stored)
#pragma unroll
        for (int i = 0; i < MI; i++)
            to[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, lane * 16, (min(mt0 + i, Mt - 1) * Ks + k) * 1024, 0));
    };
    auto weight_scales = [&](int q, uint32_t (&to)[MI]) {
#pragma unroll
        for (int i = 0; i < MI; i++)
            to[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ra, lane * 4, (min(mt0 + i, Mt - 1) * Kq + min(q, Kq - 1)) * 256, 0);
    };
    const int px0 = (wave % WN) * NI * 32, half = lane / 32;
    u32x4 xb[2][NI];
    uint32_t sb[NI];
    auto pixels = [&](const uint8_t *codes_s, int s, u32x4 (&to)[NI]) {
#pragma unroll
        for (int j = 0; j < NI; j++) {
            const int row = px0 + j * 32 + lane % 32, b = 2 * s + half;
            to[j] = *reinterpret_cast<const u32x4 *>(codes_s + row * 128 + ((b ^ (row & 7) ^ ((row >> 3) & 1)) * 16));
        }
    };
    f32x16 acc[MI][NI] = {};
    // (what the loop waits for first comes first: it is compiled to wait for as few younger loads as either way into it has)
    fetch(0, 0, WORDS);
    weight_scales(0, sa);
    __builtin_amdgcn_sched_barrier(0);
    stage(0, even_s);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < 3; s++) weights(s, wa[s]);
    fill(0);
    __builtin_amdgcn_sched_barrier(0);
    wait_loads<3 * MI>();                                   // chunk 0 is there
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
    stage(1, odd_s);
    pixels(even_s, 0, xb[0]);
    // One wave to the SIMD has nothing to hide a wait behind but its own matrix instructions, so everything a step needs is asked for a step or more before: the
    // pixels' next step while the current one is multiplied, the weights three steps ahead, and the barrier stands between step 2 and step 3, in front of the next
    // chunk's first read and behind the last of the current one's, whose buffer is then filled with the chunk after the next.  No branches: the compiler moves matrix
    // instructions behind one, away from their loads; what is loaded behind the last chunk is not used.
    const uint32_t mine_of = half ? 0x07050301u : 0x06040200u;         // the bytes of the lane's blocks
    auto chunk = [&](int q, auto odd) {
        constexpr int parity = decltype(odd)::value;
        uint8_t *const mine = parity ? odd_s : even_s, *const other = parity ? even_s : odd_s;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < NI; j += NW) {
            const int at = ((wave % WN * 32 + lane % 32) * NI + j) / NW;
            const Words low = scales_s[q / 2 & 1][2 * parity][at], high = scales_s[q / 2 & 1][2 * parity + 1][at];
#pragma unroll
            for (int k = 0; k < NW; k++) {
                if constexpr (NW == 1)
                    sb[j] = __builtin_amdgcn_perm(high, low, mine_of);
                else
                    sb[j + k] = __builtin_amdgcn_perm(high[k], low[k], mine_of);
            }
        }
#pragma unroll
        for (int s = 0; s < 4; s++) {
            __builtin_amdgcn_sched_barrier(0);              // (loads stay in their step: moved ahead they take more registers than there are)
            if (s == 3) {
                wait_loads<4 * MI + (parity ? 0 : WORDS)>();                   // the next chunk is there: what steps 0 to 2 asked for may be under way
                lds_barrier();
                __builtin_amdgcn_sched_barrier(0);
                stage(q + 2, mine);
            }
            pixels(s == 3 ? other : mine, (s + 1) % 4, xb[(s + 1) % 2]);
            weights(q * 4 + s + 3, wa[(s + 3) % 4]);
            if (s == 0) weight_scales(q + 1, na);
            if (s == 1 && parity == 1) fill(q / 2 + 1);
            if (s == 1 && parity == 0) fetch(q / 2 + 1, 0, WORDS / 2);
            if (s == 2 && parity == 0) fetch(q / 2 + 1, WORDS / 2, WORDS);
            step_mx4<MI, NI>(s, wa[s], xb[s % 2], acc, sa, sb);
#pragma unroll
            for (int i = 0; i < MI * NI / 2; i++) {         // between two matrix instructions each, one of the others
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x320, 2, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < MI; i++) sa[i] = na[i];
    };
    int q = 0;
    for (; q + 1 < Kq; q += 2) {
        chunk(q, Int<0>{});
        chunk(q + 1, Int<1>{});
    }
    if (q < Kq) chunk(q, Int<0>{});
    wait_loads<0>();                                        // (no load to LDS outlives its workgroup)
    if ((mt0 + MI) * 32 <= p.cout && row0 + px0 + NI * 32 <= p.P)              // uniform
        pw_store<DT, MI, NI, true, true, OUT>(p, acc, mt0, row0 + px0, lane);
    else
        pw_store<DT, MI, NI, false, true, KEPT>(p, acc, mt0, row0 + px0, lane);
}

// 16-bit input rows of a workgroup, quantised into LDS.  Block b of row r stands at ((b * pad + r) * 16): the lanes of a fragment read consecutive
// pieces, and with an odd `pad` the quads of a row's neighbouring blocks write to different banks.  WIDE: K is at least 8.  The scale of b = 8 q + 2 s + half is byte s of word
// (q * 2 + half) * pad + r, the four steps of a lane.  Blocks 0 .. 2 Ks - 1, rows 0 .. count - 1; what is past the matrix is zero.
//
// A thread's runs are THREADS apart: `step_row` rows and `step_run` runs, or one row more and a row's runs less, so that only the first takes a division.
template <int DT, int THREADS, int U, bool WIDE>
__device__ __forceinline__ void quantise_rows(const PwRowsArgs &r, long long row0, int rows, int count, int K, int Ks, int pad, uint8_t *codes_s, uint8_t *scales_s)
{
    const int runs = 8 * Ks, total = count * runs;
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
            const int b = rn[u] / 4;
            if constexpr (WIDE) place_wide<DT>(raw[u], rn[u] * 8, K, rw[u] < rows);
            const uint32_t byte = mx4_scale(quad_max(magnitude<DT>(raw[u])));
            const uint32_t c = mx4_codes<DT>(raw[u], byte);
            if (rw[u] >= count) continue;
            *reinterpret_cast<uint32_t *>(codes_s + (__umul24(b, pad) + rw[u]) * 16 + rn[u] % 4 * 4) = c;
            if (rn[u] % 4 == 0) scales_s[(__umul24(b / 8 * 2 + b % 2, pad) + rw[u]) * 4 + b % 8 / 2] = (uint8_t)byte;
        }
    }
}

// Layers on 16-bit input whose reduction fits LDS: a workgroup quantises its 32 NT rows once, and its waves take units of output channels and 32 rows in turn (the
// units of the same channels side by side, so that their weights are in the L1).  The input is read once, whatever the number of channels, unless there are few
// rows: then several workgroups share the channels of one's rows.  The next weights are on their way from the L2 while the current ones are multiplied or, with a
// reduction of one chunk (SHORT), while the sums are finished: that is what such a layer's time goes to, a GELU foremost, so its registers go to waves instead.
// One chunk: four waves, units of 64 channels; longer: units of 32, and eight waves, so that the rows are loaded and quantised by twice as many threads (1024 -> 256 on 12544 rows
// 13.9 -> 12.2 us), or, of many rows, four (384 -> 96 on 401408 rows 109 -> 77 us, 512 -> 256 on 50176 23 -> 22; of few, 1024 -> 128 on 3136, 7.6 and 9.2).
// Bound by memory: 96 -> 384 on 401408 rows 66 us (5.8 TB/s), 96 -> 96 34 us (4.5 TB/s); by the vector ALU with a GELU, the former 104 to 114.
template <int DT, int NT, bool SHORT, bool WIDE, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void pw_mx4_rows_kernel(PwArgs p, PwRowsArgs r)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    constexpr int PX = 32 * NT, PAD = PX + 1, WAVES = THREADS / 64, MI = SHORT ? 2 : 1;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const int KB = (p.K + 31) / 32, Ks = (KB + 1) / 2, Kq = SHORT ? 1 : (Ks + 3) / 4, Mt = (p.cout + 31) / 32;
    const unsigned part = blockIdx.x / r.blocks;
    const int first = (int)part * r.units * NT, units = min((Mt + MI - 1) / MI, ((int)part + 1) * r.units) * NT;
    const long long row0 = (long long)(blockIdx.x - part * r.blocks) * PX;
    uint8_t *const codes_s = smem, *const scales_s = smem + 2 * Ks * PAD * 16;
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w), 0, Mt * Ks * 1024, 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w_scales), 0, Mt * Kq * 256, 0x00020000);
    u32x4 wa[4][MI], wn[4][MI];
    uint32_t sa[MI], sn[MI];
    auto fetch = [&](int mt, int q, u32x4 (&w)[4][MI], uint32_t (&sc)[MI]) {
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const int m = min(mt + i, Mt - 1);
            sc[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ra, lane * 4, (m * Kq + q) * 256, 0);
#pragma unroll
            for (int s = 0; s < 4; s++)
                w[s][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, lane * 16, (m * Ks + min(q * 4 + s, Ks - 1)) * 1024, 0));
        }
    };
    auto multiply = [&](int at, int q, f32x16 (&acc)[MI][1]) {
        const uint32_t sb[1] = {*reinterpret_cast<const uint32_t *>(scales_s + ((q * 2 + half) * PAD + at + lane % 32) * 4)};
#pragma unroll
        for (int s = 0; s < 4; s++) {
            if (q * 4 + s < Ks) {
                const u32x4 xb[1] = {*reinterpret_cast<const u32x4 *>(codes_s + ((8 * q + 2 * s + half) * PAD + at + lane % 32) * 16)};
                step_mx4<MI, 1>(s, wa[s], xb, acc, sa, sb);
            }
        }
    };
    // The sums start from the bias, which waits in LDS: a load behind the last unit's stores would wait for those, too.
    float *const bias_s = reinterpret_cast<float *>(scales_s + (Kq * 2 * PAD * 4 + 15) / 16 * 16);
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
    // through the loop for it, so that tiles with fewer stores had every wave wait for the stores of the others (401408 x 96 -> 384: 126 -> 95 us, then).
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
                    for (int s = 0; s < 4; s++) wa[s][i] = wn[s][i];
                }
                const bool done = q + 1 == Kq;
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
// the reduction, a chunk each in turn, and join their sums in LDS.  QUANT: the rows are quantised into LDS first, by all threads, while the first
// weights are on their way.  2048 -> 1000 on one row 3.6 us, 8192 -> 8192 on 16 rows on codes 10 us (36 MB of weights and scales at 3.5 TB/s).
template <int DT, int NW, int NI, bool QUANT, bool WIDE>
__global__ __launch_bounds__(NW * 64) void pw_mx4_few_kernel(PwArgs p, PwRowsArgs r)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    static_assert(!QUANT || NI == 1, "rows in LDS");
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const int KB = (p.K + 31) / 32, S = (KB + 3) / 4 * 4, Ks = (KB + 1) / 2, Kq = (Ks + 3) / 4, Mt = (p.cout + 31) / 32;
    const int mt = blockIdx.x % Mt;
    const long long row0 = (long long)(blockIdx.x / Mt) * (32 * NI);
    const int rows = (int)min((long long)(32 * NI), p.P - row0), pad = rows | 1;
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w) + (size_t)mt * Ks * 1024, 0, Ks * 1024, 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w_scales) + (size_t)mt * Kq * 256, 0, Kq * 256, 0x00020000);
    // (the offsets are the lanes' own: only those are held against the buffer's end, which a step past the last reads zeros behind)
    auto weights = [&](int q, u32x4 (&wa)[4][1], uint32_t (&sa)[1]) {
        sa[0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ra, q * 256 + lane * 4, 0, 0);
#pragma unroll
        for (int s = 0; s < 4; s++) wa[s][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, (q * 4 + s) * 1024 + lane * 16, 0, 0));
    };
    u32x4 wa[4][1], wn[4][1];
    uint32_t sa[1], sn[1];
    weights(wave, wa, sa);
    weights(wave + NW, wn, sn);
    uint8_t *const scales_s = smem + 2 * Ks * pad * 16;
    if constexpr (QUANT) {
        quantise_rows<DT, NW * 64, 8, WIDE>(r, row0, rows, rows, p.K, Ks, pad, smem, scales_s);
        __syncthreads();
    }
    f32x16 acc[1][NI] = {};
    int px[NI];
#pragma unroll
    for (int j = 0; j < NI; j++) px[j] = min(j * 32 + lane % 32, rows - 1);     // (lanes past the last row repeat it)
    for (int q = wave; q < Kq; q += NW) {
        u32x4 xb[4][NI];
        uint32_t sb[NI];
#pragma unroll
        for (int j = 0; j < NI; j++) {
            if constexpr (QUANT) {
                sb[j] = *reinterpret_cast<const uint32_t *>(scales_s + ((q * 2 + half) * pad + px[j]) * 4);
            } else {
                const uint32_t *const s = reinterpret_cast<const uint32_t *>(p.scales + (row0 + px[j]) * S) + 2 * q;
                sb[j] = __builtin_amdgcn_perm(8 * q + 4 < S ? s[1] : 0u, s[0], half ? 0x07050301u : 0x06040200u);
            }
#pragma unroll
            for (int s = 0; s < 4; s++) {
                const int b = 8 * q + 2 * s + half;
                if constexpr (QUANT)
                    xb[s][j] = *reinterpret_cast<const u32x4 *>(smem + (min(b, 2 * Ks - 1) * pad + px[j]) * 16);
                else
                    xb[s][j] = *reinterpret_cast<const u32x4 *>(p.codes + ((row0 + px[j]) * KB + min(b, KB - 1)) * 16);
            }
        }
        // (steps past the last: zero weights and zero scales; of QUANT's rows the scales of such steps were never written)
#pragma unroll
        for (int s = 0; s < 4; s++)
            if (q * 4 + s < Ks) step_mx4<1, NI>(s, wa[s], xb[s], acc, sa, sb);
#pragma unroll
        for (int s = 0; s < 4; s++) wa[s][0] = wn[s][0];
        sa[0] = sn[0];
        weights(q + 2 * NW, wn, sn);
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

int check_pw(const ss_weight_desc *d, int64_t rows, const void *packed, const float *bias, const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy)
{
    const int st = check_desc(d, false);
    if (st != SS_OK) return st;
    if (d->kh != 1 || d->kw != 1 || is_byte_type(d->dtype)) return SS_ERR_UNSUPPORTED;
    if (act != SS_ACT_NONE && act != SS_ACT_RELU && act != SS_ACT_GELU) return SS_ERR_INVALID_ARG;
    if (rows < 0 || ldy < d->cout || (residual && ldr < d->cout)) return SS_ERR_INVALID_ARG;
    if (rows > INT32_MAX || ldy > INT32_MAX || (residual && ldr > INT32_MAX)) return SS_ERR_UNSUPPORTED;
    if (rows == 0) return SS_OK;
    if (!packed || !y || !aligned(packed, 16) || !aligned(y, 2) || !aligned(bias, 4) || !aligned(residual, 2)) return SS_ERR_INVALID_ARG;
    return SS_OK;
}

size_t codes_bytes(const Mx4Dims &t, int64_t rows) { return ((size_t)rows * t.KB * 16 + 255) / 256 * 256; }

PwArgs pw_args(const ss_weight_desc *d, int64_t rows, const void *packed, const float *bias, const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy)
{
    const Mx4Dims t = mx4_dims(d->cout, d->cin);
    PwArgs a{};
    a.w = static_cast<const uint8_t *>(packed) + kHeaderBytes;
    a.w_scales = a.w + (size_t)t.Mt * t.Ks * 1024;
    a.bias = bias;
    a.residual = static_cast<const uint16_t *>(residual);
    a.y = static_cast<uint16_t *>(y);
    a.ldr = ldr;
    a.ldy = ldy;
    a.P = (int)rows;
    a.cout = d->cout;
    a.K = d->cin;
    a.act = act;
    a.stream = rows_past_caches(t, rows, d->cout, false);   // (the kernel with rows in LDS looks again, at the residual)
    return a;
}

// The test hook's kernel where it is one that takes the layer, or the library's choice.
PwKernel codes_kernel(const Mx4Dims &t, long long rows)
{
    const int forced = forced_tile();
    if (forced >= PW_TILE_64 && forced <= PW_FEW_64) return (PwKernel)forced;
    return choose_codes(t, rows, std::max(compute_units(), 1));
}

PwKernel kernel16(const Mx4Dims &t, long long rows)
{
    const int forced = forced_tile();
    if (forced >= PW16_FEW && forced <= PW16_CODES && fits16(t, rows, (PwKernel)forced)) return (PwKernel)forced;
    return choose16(t, rows, std::max(compute_units(), 1));
}

template <int DT>
int product_codes(const PwArgs &a, const Mx4Dims &t, hipStream_t s)
{
    const auto tile = [&](auto mi, auto ni, auto wm) -> int {
        constexpr int MI = decltype(mi)::value, NI = decltype(ni)::value, WM = decltype(wm)::value, BN = 32 * NI * (4 / WM);
        const long long tm = (t.Mt + MI * WM - 1) / (MI * WM), tn = ((long long)a.P + BN - 1) / BN;
        if (tm * tn > 0x7FFFFFFFll) return SS_ERR_UNSUPPORTED;
        if (a.stream)
            pw_mx4_tile_kernel<DT, MI, NI, WM, LINES><<<dim3((unsigned)(tm * tn)), dim3(256), 0, s>>>(a, (int)tm, (int)tn);
        else
            pw_mx4_tile_kernel<DT, MI, NI, WM, KEPT><<<dim3((unsigned)(tm * tn)), dim3(256), 0, s>>>(a, (int)tm, (int)tn);
        return launched();
    };
    const auto few = [&](auto ni) -> int {
        constexpr int NI = decltype(ni)::value;
        const long long blocks = ((long long)a.P + 32 * NI - 1) / (32 * NI) * t.Mt;
        if (NI == 2 || t.Kq > 8) return launch_lds<pw_mx4_few_kernel<DT, 16, NI, false, false>>(blocks, 1024, few_lds(t, 16, 0), s, a, PwRowsArgs{});
        if constexpr (NI == 1)              // (two tiles of rows are for long reductions)
            return t.Kq > 4 ? launch_lds<pw_mx4_few_kernel<DT, 8, NI, false, false>>(blocks, 512, few_lds(t, 8, 0), s, a, PwRowsArgs{})
                            : launch_lds<pw_mx4_few_kernel<DT, 4, NI, false, false>>(blocks, 256, few_lds(t, 4, 0), s, a, PwRowsArgs{});
    };
    switch (codes_kernel(t, a.P)) {
        case PW_TILE_64: return tile(Int<1>{}, Int<1>{}, Int<2>{});
        case PW_TILE_128: return tile(Int<1>{}, Int<4>{}, Int<4>{});
        case PW_TILE_256: return tile(Int<2>{}, Int<8>{}, Int<4>{});
        case PW_FEW_32: return few(Int<1>{});
        default: return few(Int<2>{});
    }
}

template <int DT>
int product16(const PwArgs &a, const Mx4Dims &t, PwKernel kernel, const void *x, int64_t ldx, hipStream_t s)
{
    PwRowsArgs r{};
    r.x = static_cast<const uint16_t *>(x);
    r.ldx = ldx;
    const int runs = t.Ks * 8;
    fast_div_setup((unsigned)runs, &r.mul, &r.sh);
    const auto go = [&](auto wide) -> int {
        constexpr bool WIDE = decltype(wide)::value;
        const auto few = [&](auto nw) -> int {
            constexpr int NW = decltype(nw)::value;
            r.step_row = NW * 64 / runs;
            r.step_run = NW * 64 % runs;
            return launch_lds<pw_mx4_few_kernel<DT, NW, 1, true, WIDE>>(t.Mt, NW * 64, few_lds(t, NW, a.P), s, a, r);
        };
        const auto rows = [&](auto nt, auto brief, auto threads) -> int {
            constexpr int NT = decltype(nt)::value, THREADS = decltype(threads)::value;
            r.step_row = THREADS / runs;
            r.step_run = THREADS % runs;
            const long long blocks = ((long long)a.P + 32 * NT - 1) / (32 * NT);
            const int splits = NT == 1 ? rows_splits(t, a.P, std::max(compute_units(), 1)) : 1;
            r.blocks = (unsigned)blocks;
            r.units = (decltype(brief)::value ? (t.Mt + 1) / 2 : t.Mt) + splits - 1;
            r.units /= splits;
            PwArgs b = a;
            b.stream = a.stream || rows_past_caches(t, a.P, a.cout, a.residual != nullptr);
            return launch_lds<pw_mx4_rows_kernel<DT, NT, decltype(brief)::value, WIDE, THREADS>>(blocks * splits, THREADS, rows_lds(t, 32 * NT), s, b, r);
        };
        if (kernel == PW16_FEW) {
            const int waves = few16_waves(t, a.P, a.K);
            return waves == 16 ? few(Int<16>{}) : waves == 8 ? few(Int<8>{}) : few(Int<4>{});
        }
        if (kernel == PW16_ROWS_128) return rows(Int<4>{}, std::true_type{}, Int<256>{});
        if (t.Kq == 1) return rows(Int<1>{}, std::true_type{}, Int<256>{});
        return rows_waves(t, a.P, std::max(compute_units(), 1)) == 4 ? rows(Int<1>{}, std::false_type{}, Int<256>{}) : rows(Int<1>{}, std::false_type{}, Int<512>{});
    };
    return a.K >= 8 ? go(std::true_type{}) : go(std::false_type{});
}

// The layer in pieces of `piece` rows: launch(arguments, first row).
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
    const Mx4Dims t = mx4_dims(d->cout, d->cin);
    return in_pieces(all, piece_rows(4ll * ((t.Mt + 1) / 2)), [&](PwArgs &a, long long at) {       // (tiles of 64 x 64 have the most threads)
        a.codes = codes + at * t.KB * 16;
        a.scales = scales + at * t.S;
        return d->dtype == SS_F16 ? product_codes<SS_F16>(a, t, s) : product_codes<SS_BF16>(a, t, s);
    });
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_pw_mx4_q_fwd(const ss_weight_desc *desc, const void *codes, const void *scales, int64_t rows, const void *packed, const float *bias,
                               const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy, void *stream)
{
    const int st = check_pw(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (st != SS_OK) return st;
    if (rows == 0) return SS_OK;
    if (!codes || !scales || !aligned(codes, 16) || !aligned(scales, 4)) return SS_ERR_INVALID_ARG;
    return product(desc, pw_args(desc, rows, packed, bias, residual, ldr, act, y, ldy), static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales),
                   static_cast<hipStream_t>(stream));
}

extern "C" int ss_pw_mx4_workspace_bytes(const ss_weight_desc *desc, int64_t rows, size_t *bytes)
{
    const int st = check_desc(desc, false);
    if (st != SS_OK) return st;
    if (desc->kh != 1 || desc->kw != 1 || is_byte_type(desc->dtype)) return SS_ERR_UNSUPPORTED;
    if (!bytes || rows < 0) return SS_ERR_INVALID_ARG;
    if (rows > INT32_MAX) return SS_ERR_UNSUPPORTED;
    const Mx4Dims t = mx4_dims(desc->cout, desc->cin);
    *bytes = rows > 0 && kernel16(t, rows) == PW16_CODES ? codes_bytes(t, rows) + (size_t)rows * t.S : 0;
    return SS_OK;
}

extern "C" int ss_pw_mx4_fwd(const ss_weight_desc *desc, const void *x, int64_t rows, int64_t ldx, const void *packed, const float *bias, const void *residual,
                             int64_t ldr, int32_t act, void *y, int64_t ldy, void *workspace, size_t ws_bytes, void *stream)
{
    int st = check_pw(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (st != SS_OK) return st;
    if (ldx < desc->cin) return SS_ERR_INVALID_ARG;
    if (ldx > INT32_MAX) return SS_ERR_UNSUPPORTED;
    if (rows == 0) return SS_OK;
    if (!x || !aligned(x, 2)) return SS_ERR_INVALID_ARG;
    const Mx4Dims t = mx4_dims(desc->cout, desc->cin);
    const PwKernel kernel = kernel16(t, rows);
    if (kernel == PW16_CODES && (!workspace || !aligned(workspace, 16) || ws_bytes < codes_bytes(t, rows) + (size_t)rows * t.S)) return SS_ERR_WORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const PwArgs a = pw_args(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (kernel != PW16_CODES)
        return in_pieces(a, piece_rows(16), [&](const PwArgs &part, long long at) {                // (eight waves to 32 rows)
            const void *const first = static_cast<const uint16_t *>(x) + at * ldx;
            return desc->dtype == SS_F16 ? product16<SS_F16>(part, t, kernel, first, ldx, s) : product16<SS_BF16>(part, t, kernel, first, ldx, s);
        });
    uint8_t *codes = static_cast<uint8_t *>(workspace), *scales = codes + codes_bytes(t, rows);
    st = mx4_quantize(x, rows, desc->cin, ldx, desc->dtype, codes, scales, s);
    if (st != SS_OK) return st;
    return product(desc, a, codes, scales, s);
}
