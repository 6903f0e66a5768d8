// Products of rows in 4 bits with a power of two for each 32 columns of both sides:
//
//   out[m][n] = sum over blocks b of 2^(xs[m][b] + ws[n][b] - 254) * (sum in b of x[m][c] * w[n][c])
//
// Products and scales are exact; sums are held in fp32 and rounded once to the output's type.
#include <cmath>
#include <type_traits>

#include "sp_rows.h"

namespace sp {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int KT = 128;        // bytes of a row in one step: 256 columns, 8 scales
constexpr int CHUNK = 16;      // bytes of one access: 32 columns, one scale
constexpr int CPR = KT / CHUNK;  // chunks per row and step
constexpr int SETS = CPR / 2;  // of factors in a step: 64 columns each
constexpr int64_t CUS = 256, LDS_BYTES = 160 * 1024;
constexpr int FP4 = 4;         // the matrix instruction's number of the format
constexpr uint32_t GROUP = 8;  // columns of tiles that an XCD works through together

// 16 bytes a lane, straight to LDS, at `at` in a buffer; zeros past its end.  The whole place is the
// lane's: the hardware leaves an offset that all lanes share out of its comparison with the buffer's size.
__device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t rows, uint32_t at, uint8_t *dst)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (__attribute__((address_space(3))) void *)dst, CHUNK, at, 0, 0, 0);
}

// Scales of one side as the product reads them: eight bytes of a row for each step, in the caller's
// rows (a step is 8 bytes on, a row its stride) or packed step by step (k_pack_scales).
struct Scales4 {
    const uint8_t *p;
    int64_t row, step;
};

// ---------------------------------------------------------------- tiles
//
// A block computes tiles of BM x BN outputs, each wave WM x WN of them in 32 x 32 pieces, over steps of
// 128 bytes of a row: a whole line, which comes from L2 once (in steps of 64 bytes a tile's lines
// were gone from L1 before their second half was asked for).  LDS holds STAGES steps.  A step is four
// sets of factors, each read from LDS while the set before is multiplied.  Before its last set a
// step's buffer has been read by all: behind the barrier there the loads of the step STAGES
// ahead go straight into it, one by one between the matrix instructions.  The steps of a block's tiles
// follow each other without a gap: while a tile is stored, the next one's first steps are on their way.
// A row's eight chunks are rotated among themselves by its number (chunk c of row r sits at
// c ^ (r >> 1 & 7)), so that the 16 lanes that LDS serves at a time fall on different banks.  A
// lane's scales, eight bytes of its row, come to registers a step ahead, and one byte permutation leaves
// those of its half, a byte for each set.  w is the left factor of the matrix instruction: its four
// consecutive rows per lane are four consecutive outputs.
//
// 8192^3 270 us, 4.1 PFLOP/s, 8192 x 16384 x 4096 302; matrix instructions alone, on registers of random
// codes, reach 6.1 PFLOP/s at the clock that power leaves (8.7 on zeros).  Left out, the scales' loads are 10 and
// 16 us of that, the outputs 16 and 32, the rows' loads 104 and 79, all three 121 and 134.  256 x 256 in four waves of
// 128 x 128 and not eight of 128 x 64: with those LDS was read for as long as the matrix cores were
// busy (8192^3 513 us with steps of 64 bytes and the scales through LDS; without scales 326, without loads 328).
template <int BM, int BN, int WM, int WN, int STAGES, typename TO, bool PARTIAL>
__global__ void __launch_bounds__(BM / WM *BN / WN *WAVE)
    k_product4(Product4Args a, Scales4 sx, Scales4 sw, int32_t tiles_n, uint32_t tiles_m, int32_t per_split)
{
    constexpr int NW = (BM / WM) * (BN / WN), NT = NW * WAVE;
    constexpr int TM = WM / 32, TN = WN / 32, TF = TM + TN;
    constexpr int RPL = WAVE / CPR;              // rows per load of a wave
    constexpr int LOADS = (BM + BN) * CPR / NT;  // of a wave and step
    static_assert(LOADS * NT == (BM + BN) * CPR && BM % (NW * RPL) == 0 && NW % 2 == 0, "whole loads");
    constexpr int BUF = (BM + BN) * KT;
    __shared__ __attribute__((aligned(16))) uint8_t sm[STAGES * BUF];
    const int wave = wave_id(), lane = lane_id();
    const uint32_t tiles = (uint32_t)tiles_n * tiles_m;
    const auto tile_at = [&](uint32_t i, int64_t &m0, int64_t &n0) {
        uint32_t tile_m = 0, tile_n = i;
        if (tiles_m > 1) {
            const uint32_t tile = (uint32_t)xcd_block(i, tiles);
            const uint32_t group = tile / (GROUP * tiles_m), in = tile - group * GROUP * tiles_m;
            const uint32_t wide = (uint32_t)tiles_n - group * GROUP < GROUP ? (uint32_t)tiles_n - group * GROUP : GROUP;
            tile_m = in / wide;
            tile_n = group * GROUP + in % wide;
        }
        m0 = (int64_t)tile_m * BM;
        n0 = (int64_t)tile_n * BN;
    };
    const int32_t first = (int32_t)blockIdx.y * per_split;
    const int32_t all = (a.blocks + CPR - 1) / CPR, end = first + per_split < all ? first + per_split : all;
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    const auto row_at = [](int64_t row, int64_t last) { return (uint32_t)(row < last ? row : last); };

    // What is loaded next: rows of a tile, a step.  The rows are buffers from the tile's first one on, whose
    // bounds the hardware checks (strides are below 2^23, so places in 256 rows are below 2^31): rows past the
    // last are zeros, and so is everything once nothing is left to load.  Bytes behind a row's last chunk are its
    // neighbour's; their scales are zeros, so they count nothing (2^-254 times a finite value is below
    // anything that fp32 holds).
    uint32_t load_tile = blockIdx.x;
    int32_t load_step = first;
    __amdgpu_buffer_rsrc_t x_rows, w_rows;
    const int my_row = wave * RPL + lane / CPR;
    const int my_chunk = (lane % CPR) ^ (my_row >> 1 & (CPR - 1));  // (NW * RPL rows keep the rotation)
    static_assert(NW * RPL % 16 == 0, "a load's rows rotate as the first one's");
    const uint32_t x_at = (uint32_t)(my_row * (int)a.x_ld + my_chunk * CHUNK), w_at = (uint32_t)(my_row * (int)a.w_ld + my_chunk * CHUNK);
    const auto rows_of = [&](const uint8_t *p, int64_t ld, int64_t rows, int most) {
        if (rows > most) rows = most;
        return buffer(p, rows > 0 ? (uint32_t)((rows - 1) * ld + a.blocks * CHUNK) : 0);
    };
    const auto aim = [&]() {
        int64_t m0 = 0, n0 = 0;
        const bool more = load_tile < tiles;
        if (more) tile_at(load_tile, m0, n0);
        x_rows = rows_of(a.x + m0 * a.x_ld, a.x_ld, more ? a.m - m0 : 0, BM);
        w_rows = rows_of(a.w + n0 * a.w_ld, a.w_ld, more ? a.n - n0 : 0, BN);
    };
    const auto fetch = [&](int32_t stage, int i) {  // load i, into a stage
        const bool is_x = i * NW * RPL < BM;
        const int rows = i * NW * RPL - (is_x ? 0 : BM);
        const uint32_t from = (uint32_t)(rows * (int)(is_x ? a.x_ld : a.w_ld) + load_step * KT);
        to_lds(is_x ? x_rows : w_rows, (is_x ? x_at : w_at) + from, sm + stage * BUF + (i * NW + wave) * RPL * KT);
    };
    const auto fetched = [&]() {  // on to the next step, or tile
        if (++load_step < end) return;
        load_step = first;
        load_tile += gridDim.x;
        aim();
    };
    // Scales: x's pieces, then w's.
    const uint8_t *xs, *ws;
    uint32_t scale_place[TF];
    const auto aim_scales = [&](int64_t m0, int64_t n0) {
        int l = lane % 32;
        asm volatile("" : "+v"(l));
        xs = sx.p + m0 * sx.row;
        ws = sw.p + n0 * sw.row;
#pragma unroll
        for (int i = 0; i < TF; ++i)
            scale_place[i] = i < TM ? row_at(wm + i * 32 + l, a.m - 1 - m0) * (uint32_t)sx.row
                                    : row_at(wn + (i - TM) * 32 + l, a.n - 1 - n0) * (uint32_t)sw.row;
    };
    uint2 coming[TF];
    uint32_t now[TF];
    const auto fetch_scale = [&](int32_t step, int i) {
        coming[i] = *(const uint2 *)((i < TM ? xs + step * sx.step : ws + step * sw.step) + scale_place[i]);
    };
    const uint32_t half = lane / 32 ? 0x07050301u : 0x06040200u;
    const auto take_scales = [&](int32_t step) {
#pragma unroll
        for (int i = 0; i < TF; ++i) now[i] = __builtin_amdgcn_perm(coming[i].y, coming[i].x, half);
        if (step + 1 == all) {  // none past the rows' end
            const int left = a.blocks - step * CPR - lane / 32;
            const uint32_t mask = left > 6 ? ~0u : left > 4 ? 0xFFFFFFu : left > 2 ? 0xFFFFu : left > 0 ? 0xFFu : 0u;
#pragma unroll
            for (int i = 0; i < TF; ++i) now[i] &= mask;
        }
    };
    // All but the last OPEN of this wave's loads and stores are done, and every wave is done with the
    // buffer that is filled next.
    const auto landed = [](auto open) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(open)::value) : "memory");
    };

    v16f acc[TM][TN];
    const auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
    };

    v4i f[2][TF];  // x's, then w's
    const uint8_t *xb = sm + (wm + lane % 32) * KT, *wb = sm + (BM + wn + lane % 32) * KT;
    const auto read = [&](int32_t stage, int set, int i) {
        const int at = stage * BUF + ((set * 2 + lane / 32) ^ (lane >> 1 & (CPR - 1))) * CHUNK;
        f[set & 1][i] = i < TM ? *(const v4i *)(xb + i * 32 * KT + at) : *(const v4i *)(wb + (i - TM) * 32 * KT + at);
    };
    // A set multiplied.  Between the matrix instructions: the next set's reads (READS: from `stage`), the
    // scales of step `step` (SCALES), and the loads of the step that is loaded next (FETCHES: into `into`).
    const auto multiply = [&](auto which, auto reads, int32_t stage, auto scales, int32_t step, auto fetches, int32_t into) {
        constexpr int set = decltype(which)::value;
        constexpr bool READS = decltype(reads)::value, SCALES = decltype(scales)::value, FETCHES = decltype(fetches)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < TM * TN; ++p) {
            const v4i &u = f[set & 1][TM + p % TN], &v = f[set & 1][p / TN];
            acc[p / TN][p % TN] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                v8i{u.x, u.y, u.z, u.w, 0, 0, 0, 0}, v8i{v.x, v.y, v.z, v.w, 0, 0, 0, 0}, acc[p / TN][p % TN], FP4, FP4,
                set, (int)now[TM + p % TN], set, (int)now[p / TN]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TF; ++i)
                if (i * (TM * TN) / TF == p) {
                    if constexpr (READS) read(stage, (set + 1) % SETS, i);
                    if constexpr (SCALES) fetch_scale(step, i);
                }
            if constexpr (FETCHES) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (i * (TM * TN) / LOADS == p) fetch(into, i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // (else the compiler takes the multiplications of all four sets behind the step's branches)
#pragma unroll
        for (int p = 0; p < TM * TN; ++p) asm volatile("" : "+a"(acc[p / TN][p % TN]));
    };
    // A tile's outputs, straight from the registers: two lanes' halves of eight columns are exchanged where
    // they are 16 bits wide, so that each store is 16 bytes a lane.  32 rows are a buffer (strides are below
    // 2^23), and a store that is not wholly inside the output is aimed past its end, so that there are as
    // many stores everywhere; where a row's last one is not whole (`ragged`) they go column by column.
    // Sums are taken out of their registers one by one: left to the compiler they were all moved at once,
    // and what the next tile needs went to memory for them.
    const auto sum = [](float x) {
        float v;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(x));
        return v;
    };
    constexpr int EP = 16 / (int)sizeof(TO), STORES = TM * TN * 16 / EP;  // outputs of a lane and store; stores of a tile
    const auto store = [&](int64_t m0, int64_t n0) {
        constexpr uint32_t NOWHERE = 0xFFFFFF00u;
        TO *base = (PARTIAL ? (TO *)a.work + (int64_t)blockIdx.y * a.m * a.n : (TO *)a.out) + n0 + wn;
        const int64_t right = a.n - n0 - wn, down = a.m - m0 - wm;
        int l = lane;
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");  // (the last matrix instruction's result, which `sum` reads)
        asm volatile("" : "+v"(l));  // (else every store's place is worked out before the first tile and kept)
        const int32_t columns = (int32_t)(right < WN ? right : WN), col = l / 32 * EP;
        const uint32_t ld = (uint32_t)a.out_ld * (uint32_t)sizeof(TO), at = (uint32_t)(l % 32) * ld + (uint32_t)(col * (int)sizeof(TO));
        const bool ragged = right < WN && right % EP != 0;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int32_t rows = (int32_t)(down - i * 32 < 32 ? down - i * 32 : 32);
            const __amdgpu_buffer_rsrc_t to = buffer(base + (m0 + wm + i * 32) * a.out_ld, rows > 0 && columns > 0 ? (uint32_t)(rows - 1) * ld + (uint32_t)(columns * (int)sizeof(TO)) : 0);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; q += EP / 4) {
                    __builtin_amdgcn_sched_barrier(0);
                    Pack<TO, EP> o;
                    if constexpr (EP == 4) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) o.v[c] = from_float<TO>(sum(acc[i][j][q * 4 + c]));
                    } else {
                        Pack<TO, 4> lo, hi;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            lo.v[c] = from_float<TO>(sum(acc[i][j][q * 4 + c]));
                            hi.v[c] = from_float<TO>(sum(acc[i][j][q * 4 + 4 + c]));
                        }
                        uint32_t x[2], y[2];
                        __builtin_memcpy(x, &lo, 8);
                        __builtin_memcpy(y, &hi, 8);
                        const auto s0 = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false);
                        const auto s1 = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
                        const uint32_t w[4] = {s0[0], s1[0], s0[1], s1[1]};
                        __builtin_memcpy(&o, w, 16);
                    }
                    const int32_t left = columns - col - (j * 32 + q * 8);
                    constexpr uint32_t SIZE = (uint32_t)sizeof(TO);
                    const uint32_t here = at + (uint32_t)(j * 32 + q * 8) * SIZE;
                    if (!ragged) {
                        unit w;
                        __builtin_memcpy(&w, &o, 16);
                        __builtin_amdgcn_raw_buffer_store_b128(w, to, left >= EP ? here : NOWHERE, 0, 0);
                    } else {
#pragma unroll
                        for (int c = 0; c < EP; ++c) {
                            const uint32_t to_column = c < left ? here + (uint32_t)c * SIZE : NOWHERE;
                            if constexpr (SIZE == 4) {
                                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint((float)o.v[c]), to, to_column, 0, 0);
                            } else {
                                uint16_t h;
                                __builtin_memcpy(&h, &o.v[c], 2);
                                __builtin_amdgcn_raw_buffer_store_b16(h, to, to_column, 0, 0);
                            }
                        }
                    }
                }
        }
    };

    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    constexpr std::integral_constant<int, 0> set0{};
    constexpr std::integral_constant<int, 1> set1{};
    constexpr std::integral_constant<int, 2> set2{};
    constexpr std::integral_constant<int, 3> set3{};
    static_assert(SETS == 4, "four sets");
    // (At least as many came after the next step's: later steps' rows, this one's scales, a tile's stores.)
    constexpr int OPEN = (STAGES - 2) * LOADS + TF;
    constexpr std::integral_constant<int, (STAGES - 1) * LOADS> but_first{};
    constexpr std::integral_constant<int, OPEN> but_next{};
    constexpr std::integral_constant<int, OPEN + STORES < 63 ? OPEN + STORES : 63> but_stores{};

    uint32_t tile = blockIdx.x;
    int64_t m0, n0;
    tile_at(tile, m0, n0);
    aim();
    aim_scales(m0, n0);
#pragma unroll
    for (int i = 0; i < TF; ++i) fetch_scale(first, i);
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) fetch(s, i);
        fetched();
    }
    landed(but_first);
#pragma unroll
    for (int i = 0; i < TF; ++i) read(0, 0, i);
    int32_t stage = 0;
    bool stored = false;  // a tile, just before
    for (;;) {
        const int64_t m = m0, n = n0;
        const bool more = tile + gridDim.x < tiles;
        int32_t step = first;
        clear();
        do {
            const int32_t after = stage + 1 < STAGES ? stage + 1 : 0;
            take_scales(step);
            if (step + 1 == end && more) {  // the next step's scales are another tile's
                tile += gridDim.x;
                tile_at(tile, m0, n0);
                aim_scales(m0, n0);
            }
            multiply(set0, yes, stage, yes, step + 1 < end ? step + 1 : first, no, 0);
            multiply(set1, yes, stage, no, 0, no, 0);
            multiply(set2, yes, stage, no, 0, no, 0);
            if (stored) landed(but_stores);
            else landed(but_next);
            stored = false;
            multiply(set3, yes, after, no, 0, yes, stage);
            fetched();
            stage = after;
        } while (++step < end);
        store(m, n);
        stored = true;
        if (!more) break;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing may come to LDS once it is another block's)
}

// The parts of a split sum added up in their order and rounded: four outputs per thread.
template <typename TO>
__global__ void __launch_bounds__(BLOCK) k_product4_join(Product4Args a, int32_t splits)
{
    const int64_t total = a.m * a.n, i0 = ((int64_t)blockIdx.x * BLOCK + threadIdx.x) * 4;
    if (i0 >= total) return;
    const float *part = (const float *)a.work + i0;
    float v[4] = {0, 0, 0, 0};
    const int valid = total - i0 < 4 ? (int)(total - i0) : 4;
    if (valid == 4) {
#pragma unroll 4
        for (int32_t s = 0; s < splits; ++s) {
            Pack<float, 4> p;
            __builtin_memcpy(&p, part + s * total, sizeof p);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] += p.v[c];
        }
    } else {
        for (int32_t s = 0; s < splits; ++s)
            for (int c = 0; c < valid; ++c) v[c] += part[s * total + c];
    }
    int64_t m = i0 / a.n, n = i0 - m * a.n;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        if (c < valid) ((TO *)a.out)[m * a.out_ld + n] = from_float<TO>(v[c]);
        if (++n == a.n) n = 0, ++m;
    }
}

// Scales step by step: out[step][row] is the eight bytes of a row's step, zeros past its end.  A tile
// then reads its rows' scales of a step in whole lines; in the caller's rows they are 8 bytes of a
// line each, and as many lines as the factors themselves.
__global__ void __launch_bounds__(BLOCK) k_pack_scales(const uint8_t *scales, int64_t ld, int64_t rows, int32_t blocks, uint2 *out)
{
    constexpr int ROWS = 64, STEPS = 16;  // of a block; 16 threads read a row's 128 bytes
    __shared__ uint2 words[STEPS][ROWS + 1];
    const int64_t row0 = (int64_t)blockIdx.x * ROWS;
    const int32_t step0 = (int32_t)blockIdx.y * STEPS, steps = (blocks + CPR - 1) / CPR;
    for (int i = (int)threadIdx.x; i < ROWS * STEPS; i += BLOCK) {
        const int64_t row = row0 + i / STEPS;
        const int32_t step = step0 + i % STEPS;
        if (row >= rows || step >= steps) continue;
        uint2 w = *(const uint2 *)(scales + row * ld + step * CPR);
        const int left = blocks - step * CPR;
        if (left < 8) {
            w.y = left <= 4 ? 0u : w.y & ((1u << (8 * (left - 4))) - 1);
            w.x = left >= 4 ? w.x : w.x & ((1u << (8 * left)) - 1);
        }
        words[i % STEPS][i / STEPS] = w;
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < ROWS * STEPS; i += BLOCK) {
        const int64_t row = row0 + i % ROWS;
        const int32_t step = step0 + i / ROWS;
        if (row < rows && step < steps) out[step * rows + row] = words[i / ROWS][i % ROWS];
    }
}

// ---------------------------------------------------------------- host

static int64_t steps_of(int32_t blocks) { return (blocks + CPR - 1) / CPR; }

// How a product is cut: into tiles, and parts of k where the tiles are few.  The estimate, in us, for
// what a CU has to do one after the other: rounds of as many blocks as run at a time, each a fixed time
// (first loads, outputs) and its steps of k, with a block on a CU or as many as fit; for tiles of 256
// the packing of the scales; for parts a second launch and their traffic.  Measured on both sides
// of the lines that it draws (us of the kernels among others, in graphs; a call outside of one takes the host 9,
// of two launches 13; bf16; * what is taken).  Where bytes bind (1, 16 and 64 rows against 131072) the times are
// up to twice the estimate, in the small tiles alike:
//                          256x256  128x128  64x128  64x64  32x64   in parts
//   8192 x 16384 x 4096       300*     451
//   8192 x 8192 x 512          50       48*     62     74     91
//   4000 x 4000 x 4000         44*      55      75     95    110
//   4000 x 4000 x 1000         23       17*     21     29     34
//   777 x 10001 x 1000         33       18      18*    20     21
//   2048 x 2048 x 2048         26       11*     12     15     18    26 (2 of 128x128)
//   256 x 8192 x 8192          57       29      23*    28     36    26 (2 of 128x128)
//   128 x 8192 x 8192          55       29      23     18*    19    19 (2 of 64x128)
//   64 x 8192 x 8192           55       25      23     18     16*   15 (2 of 64x64, 4 of 64x128)
//   64 x 131072 x 4096         86       76      74*    90    106
//   16 x 131072 x 4096         80       65      62     71     61*
//   64 x 4096 x 4096           33       14      12     10      9*   10 (2 of 64x64 or 32x64)
//   1 x 131072 x 2048          51       31      29     29     28*
//   1 x 4096 x 8192            54       23      20     16     15    10* (8 of 32x64; 4 of 32x64 9, of 64x64 10)
struct Cut {
    int32_t tile, splits;
};
static Cut cut_product4(int64_t m, int64_t n, int32_t blocks)
{
    constexpr struct {
        int bm, bn, at_once;
        double alone, beside, fixed, once;
    } T[] = {{256, 256, 256, 2.05, 2.15, 6.0, 8.0}, {128, 128, 512, 0.85, 1.6, 2.6, 0.0}, {64, 128, 512, 0.65, 1.05, 1.5, 0.0},
             {64, 64, 512, 0.5, 0.75, 1.4, 0.0}, {32, 64, 768, 0.42, 0.57, 0.6, 0.0}};
    const int64_t steps = steps_of(blocks);
    Cut best{1, 1};
    double least = 1e300;
    for (int t = 0; t < 5; ++t) {
        const double tiles = (double)((m + T[t].bm - 1) / T[t].bm) * (double)((n + T[t].bn - 1) / T[t].bn);
        for (int sp = 1; sp <= 16; sp *= 2) {
            if (sp > 1 && (t == 0 || steps < 4 * sp || tiles * sp > 1024)) break;
            const double all = tiles * sp, step = all <= (double)CUS ? T[t].alone : T[t].beside;
            double us = T[t].once + std::ceil(all / T[t].at_once) * (T[t].fixed + step * (double)((steps + sp - 1) / sp));
            if (sp > 1) us += 4.5 + (double)m * (double)n * 4.0 * (2 * sp) / 4e6;
            if (us < least) least = us, best = Cut{t, sp};
        }
    }
    return best;
}

// The scales of tiles of 256 are packed: what each reads of them in the caller's rows is as many lines as
// the factors' (8192^3: 324 us with both in the caller's rows, 272 packed, when it was brought in; the packing of
// 8192 and 16384 rows of 4096 columns takes 4 and 6).
// (In one launch: of fewer than 2^30 rows.)
static bool packs(int64_t m, int64_t n, const Cut &c) { return c.tile == 0 && m < 1 << 30 && n < 1 << 30; }

int64_t product4_workspace(int64_t m, int64_t n, int32_t blocks)
{
    if (m == 0 || n == 0) return 0;
    const Cut c = cut_product4(m, n, blocks);
    return c.splits > 1 ? m * n * 4 * c.splits : packs(m, n, c) ? steps_of(blocks) * 8 * (m + n) : 0;
}

template <int BM, int BN, int WM, int WN, int STAGES, typename TO, bool PARTIAL>
static hipError_t run_tiles(const Product4Args &a, const Scales4 &sx, const Scales4 &sw, int32_t splits, hipStream_t s)
{
    const int64_t tm = (a.m + BM - 1) / BM, tn = (a.n + BN - 1) / BN;
    if (tm * tn > LAUNCH_BLOCKS / 2) {  // (up to 512 threads each; never in parts of k)
        Product4Args lo = a, hi = a;
        Scales4 hx = sx, hw = sw;
        if (tm >= tn) {
            lo.m = tm / 2 * BM;
            hi.m = a.m - lo.m;
            hi.x += lo.m * a.x_ld;
            hx.p += lo.m * sx.row;
            hi.out = (TO *)a.out + lo.m * a.out_ld;
        } else {
            lo.n = tn / 2 * BN;
            hi.n = a.n - lo.n;
            hi.w += lo.n * a.w_ld;
            hw.p += lo.n * sw.row;
            hi.out = (TO *)a.out + lo.n;
        }
        const hipError_t r = run_tiles<BM, BN, WM, WN, STAGES, TO, PARTIAL>(lo, sx, sw, splits, s);
        return r != hipSuccess ? r : run_tiles<BM, BN, WM, WN, STAGES, TO, PARTIAL>(hi, hx, hw, splits, s);
    }
    const int32_t steps = (int32_t)steps_of(a.blocks), per = (steps + splits - 1) / splits;
    // As many blocks as run at a time, where each has several tiles.
    constexpr int64_t AT_ONCE = CUS * (LDS_BYTES / (STAGES * (BM + BN) * KT));
    const int64_t blocks = splits > 1 || tm * tn < AT_ONCE ? tm * tn : AT_ONCE;
    const dim3 grid((unsigned)blocks, (unsigned)((steps + per - 1) / per)), block(BM / WM * (BN / WN) * WAVE);
    return launch(k_product4<BM, BN, WM, WN, STAGES, TO, PARTIAL>, grid, block, s, a, sx, sw, (int32_t)tn, (uint32_t)tm, per);
}

template <typename TO, bool PARTIAL>
static hipError_t run_cut(const Product4Args &a, const Scales4 &sx, const Scales4 &sw, const Cut &c, hipStream_t s)
{
    return c.tile == 0   ? run_tiles<256, 256, 128, 128, 2, TO, PARTIAL>(a, sx, sw, c.splits, s)
           : c.tile == 1 ? run_tiles<128, 128, 64, 64, 2, TO, PARTIAL>(a, sx, sw, c.splits, s)
           : c.tile == 2 ? run_tiles<64, 128, 32, 64, 3, TO, PARTIAL>(a, sx, sw, c.splits, s)
           : c.tile == 3 ? run_tiles<64, 64, 32, 32, 4, TO, PARTIAL>(a, sx, sw, c.splits, s)
                         : run_tiles<32, 64, 32, 32, 4, TO, PARTIAL>(a, sx, sw, c.splits, s);
}

hipError_t run_product4(const Product4Args &given, hipStream_t s)
{
    Product4Args a = given;
    if (a.m == 1) a.x_ld = a.xs_ld = a.out_ld = 0;  // the stride of a single row is never used
    if (a.n == 1) a.w_ld = a.ws_ld = 0;
    const Cut c = cut_product4(a.m, a.n, a.blocks);
    Scales4 sx{a.xs, a.xs_ld, CPR}, sw{a.ws, a.ws_ld, CPR};
    if (packs(a.m, a.n, c)) {
        const auto pack = [&](Scales4 &side, int64_t rows, uint2 *to) {
            const dim3 grid((unsigned)((rows + 63) / 64), (unsigned)((steps_of(a.blocks) + 15) / 16));
            const hipError_t e = launch(k_pack_scales, grid, dim3(BLOCK), s, side.p, side.row, rows, a.blocks, to);
            side = Scales4{(const uint8_t *)to, 8, rows * 8};
            return e;
        };
        uint2 *to = (uint2 *)a.work;
        hipError_t e = pack(sx, a.m, to);
        if (e == hipSuccess) e = pack(sw, a.n, to + steps_of(a.blocks) * a.m);
        if (e != hipSuccess) return e;
    }
    return with_type(a.out_type, [&](auto to) {
        using TO = decltype(to);
        if (c.splits == 1) return run_cut<TO, false>(a, sx, sw, c, s);
        Product4Args p = a;
        p.out_ld = a.n;
        hipError_t r = run_cut<float, true>(p, sx, sw, c, s);
        if (r != hipSuccess) return r;
        const int32_t steps = (int32_t)steps_of(a.blocks), per = (steps + c.splits - 1) / c.splits;
        const int64_t blocks = (a.m * a.n + 4 * BLOCK - 1) / (4 * BLOCK);
        if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
        return launch(k_product4_join<TO>, dim3((unsigned)blocks), dim3(BLOCK), s, a, (steps + per - 1) / per);
    });
}

}  // namespace sp
