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
constexpr int FP4 = 4;         // the matrix instruction's number of the format
constexpr uint32_t GROUP = 8;  // columns of tiles that an XCD works through together

__device__ __forceinline__ void to_lds(const uint8_t *src, uint8_t *dst)
{
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void *)src,
        (__attribute__((address_space(3))) void *)dst, CHUNK, 0, 0);
}

// Scales of one side as the product reads them: eight bytes of a row for each step, in the caller's
// rows (a step is 8 bytes on, a row its stride) or packed step by step (k_pack_scales).
struct Scales4 {
    const uint8_t *p;
    int64_t row, step;
};

// ---------------------------------------------------------------- tiles
//
// A block computes BM x BN outputs, each wave WM x WN of them in 32 x 32 pieces, over steps of
// 128 bytes of a row: a whole line, which comes from L2 once (in steps of 64 bytes a tile's lines
// were gone from L1 before their second half was asked for).  LDS holds STAGES steps.  A step is four
// sets of factors, each read from LDS while the set before is multiplied.  Before its last set a
// step's buffer has been read by all: behind the barrier there the loads of the step STAGES
// ahead go straight into it, one by one between the matrix instructions.  A row's eight
// chunks are rotated among themselves by its number (chunk c of row r sits at c ^ (r >> 1 & 7)), so that
// the 16 lanes that LDS serves at a time fall on different banks.  A lane's scales, eight bytes of
// its row, come to registers a step ahead, and one byte permutation leaves those of its
// half, a byte for each set.  w is the left factor of the matrix instruction: its four
// consecutive rows per lane are four consecutive outputs.
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
    uint32_t tile_m = 0, tile_n = blockIdx.x;
    if (tiles_m > 1) {
        const uint32_t tile = (uint32_t)xcd_block(blockIdx.x, gridDim.x);
        const uint32_t group = tile / (GROUP * tiles_m), in = tile - group * GROUP * tiles_m;
        const uint32_t wide = (uint32_t)tiles_n - group * GROUP < GROUP ? (uint32_t)tiles_n - group * GROUP : GROUP;
        tile_m = in / wide;
        tile_n = group * GROUP + in % wide;
    }
    const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BN;
    const int32_t first = (int32_t)blockIdx.y * per_split;
    const int32_t all = (a.blocks + CPR - 1) / CPR, steps = first + per_split < all ? first + per_split : all;
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;

    // This lane's chunk of each load: a place relative to the tile's first row (strides are below
    // 2^23, so it fits 32 bits); rows past the last take that one.
    const auto clamped = [&](bool is_x, int64_t row) {
        const int64_t last = is_x ? a.m - 1 - m0 : a.n - 1 - n0;
        return row < last ? row : last;
    };
    uint32_t place[LOADS];
    const int my_row = wave * RPL + lane / CPR;
    const int my_chunk = (lane % CPR) ^ (my_row >> 1 & (CPR - 1));  // (NW * RPL rows keep the rotation)
    static_assert(NW * RPL % 16 == 0, "a load's rows rotate as the first one's");
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const bool is_x = i * NW * RPL < BM;
        const int64_t at = clamped(is_x, i * NW * RPL + my_row - (is_x ? 0 : BM));
        place[i] = (uint32_t)at * (uint32_t)(is_x ? a.x_ld : a.w_ld) + (uint32_t)(my_chunk * CHUNK);
    }
    const uint8_t *xt = a.x + m0 * a.x_ld, *wt = a.w + n0 * a.w_ld;
    // Load i of a step; chunks past the rows' last one take that one.
    const auto fetch = [&](int32_t step, int i) {
        const bool is_x = i * NW * RPL < BM;
        const int32_t chunk = step * CPR + my_chunk, back = chunk >= a.blocks ? chunk - (a.blocks - 1) : 0;
        to_lds((is_x ? xt : wt) + step * KT + (place[i] - (uint32_t)(back * CHUNK)),
               sm + step % STAGES * BUF + (i * NW + wave) * RPL * KT);
    };
    // Scales: x's pieces, then w's.
    const uint8_t *scale_row[TF];
#pragma unroll
    for (int i = 0; i < TF; ++i)
        scale_row[i] = i < TM ? sx.p + (m0 + clamped(true, wm + i * 32 + lane % 32)) * sx.row
                              : sw.p + (n0 + clamped(false, wn + (i - TM) * 32 + lane % 32)) * sw.row;
    uint2 coming[TF];
    uint32_t now[TF];
    const auto fetch_scales = [&](int32_t step) {
#pragma unroll
        for (int i = 0; i < TF; ++i) coming[i] = *(const uint2 *)(scale_row[i] + step * (i < TM ? sx.step : sw.step));
    };
    const uint32_t half = lane / 32 ? 0x07050301u : 0x06040200u;
    const auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < TF; ++i) now[i] = __builtin_amdgcn_perm(coming[i].y, coming[i].x, half);
    };
    // All but the last OPEN of this wave's loads have arrived, and every wave is done with the buffer
    // that is filled next.
    const auto landed = [](auto open) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(open)::value) : "memory");
    };

    v16f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

    v4i f[2][TF];  // x's, then w's
    const uint8_t *xb = sm + (wm + lane % 32) * KT, *wb = sm + (BM + wn + lane % 32) * KT;
    const auto read = [&](int32_t step, int set, int i) {
        const int at = step % STAGES * BUF + ((set * 2 + lane / 32) ^ (lane >> 1 & (CPR - 1))) * CHUNK;
        f[set & 1][i] = i < TM ? *(const v4i *)(xb + i * 32 * KT + at) : *(const v4i *)(wb + (i - TM) * 32 * KT + at);
    };
    // A set multiplied.  Between the matrix instructions: the next set's reads (READS: of step `next`),
    // and the loads of step `ahead` (FETCHES).
    const auto multiply = [&](auto which, auto reads, int32_t next, auto fetches, int32_t ahead) {
        constexpr int set = decltype(which)::value;
        constexpr bool READS = decltype(reads)::value, FETCHES = decltype(fetches)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < TM * TN; ++p) {
            const v4i &u = f[set & 1][TM + p % TN], &v = f[set & 1][p / TN];
            acc[p / TN][p % TN] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                v8i{u.x, u.y, u.z, u.w, 0, 0, 0, 0}, v8i{v.x, v.y, v.z, v.w, 0, 0, 0, 0}, acc[p / TN][p % TN], FP4, FP4,
                set, (int)now[TM + p % TN], set, (int)now[p / TN]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (READS) {
#pragma unroll
                for (int i = 0; i < TF; ++i)
                    if (i * (TM * TN) / TF == p) read(next, (set + 1) % SETS, i);
            }
            if constexpr (FETCHES) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (i * (TM * TN) / LOADS == p) fetch(ahead, i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    constexpr std::integral_constant<int, 0> set0{};
    constexpr std::integral_constant<int, 1> set1{};
    constexpr std::integral_constant<int, 2> set2{};
    constexpr std::integral_constant<int, 3> set3{};
    static_assert(SETS == 4, "four sets");
    constexpr std::integral_constant<int, (STAGES - 1) * LOADS> but_first{};
    // (at least as many came after the next step's: later steps' rows and this one's scales)
    constexpr std::integral_constant<int, (STAGES - 2) * LOADS + TF> but_next{};

    fetch_scales(first);
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (first + s < steps) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) fetch(first + s, i);
        }
    if (steps - first >= STAGES) landed(but_first);
    else landed(set0);
#pragma unroll
    for (int i = 0; i < TF; ++i) read(first, 0, i);
    int32_t s = first;
    for (; s + STAGES < steps; ++s) {
        take_scales();
        fetch_scales(s + 1);
        multiply(set0, yes, s, no, 0);
        multiply(set1, yes, s, no, 0);
        multiply(set2, yes, s, no, 0);
        landed(but_next);
        multiply(set3, yes, s + 1, yes, s + STAGES);
    }
    for (; s + 1 < steps; ++s) {
        take_scales();
        fetch_scales(s + 1);
        multiply(set0, yes, s, no, 0);
        multiply(set1, yes, s, no, 0);
        multiply(set2, yes, s, no, 0);
        landed(set0);
        multiply(set3, yes, s + 1, no, 0);
    }
    // The last step: what lies past the rows' end counts nothing, its scales neither.
    take_scales();
    const int left = a.blocks - s * CPR - lane / 32, have = (a.blocks - s * CPR + 1) / 2;  // chunks of this lane's half; sets
    const uint32_t mask = left > 6 ? ~0u : left > 4 ? 0xFFFFFFu : left > 2 ? 0xFFFFu : left > 0 ? 0xFFu : 0u;
#pragma unroll
    for (int i = 0; i < TF; ++i) now[i] &= mask;
    const auto last_set = [&](auto which) {
        constexpr int set = decltype(which)::value;
        if (set >= have) return;  // the same for all
        if (set > 0) {
#pragma unroll
            for (int i = 0; i < TF; ++i) read(s, set, i);
        }
        if (left <= 2 * set) {
#pragma unroll
            for (int i = 0; i < TF; ++i) f[set & 1][i] = v4i{0, 0, 0, 0};
        }
        multiply(which, no, 0, no, 0);
    };
    last_set(set0);
    last_set(set1);
    last_set(set2);
    last_set(set3);
    __syncthreads();

    // Out through LDS, 32 rows at a time: a lane then has consecutive outputs of a row, 16
    // bytes of them, and a wave's store whole rows of its tile.
    constexpr int EP = 16 / (int)sizeof(TO);  // outputs per lane and store
    constexpr int LPR = WN / EP;              // lanes per row and store
    constexpr int STRIDE = WN * 4 + 16;
    static_assert(NW * 32 * STRIDE <= (int)sizeof sm && WAVE % LPR == 0, "staging fits the buffers");
    uint8_t *stage = sm + wave * 32 * STRIDE;
    const int64_t n = n0 + wn + lane % LPR * EP;
    TO *out = (PARTIAL ? (TO *)a.work + (int64_t)blockIdx.y * a.m * a.n : (TO *)a.out) + (m0 + wm + lane / LPR) * a.out_ld + n;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                Pack<float, 4> v;
#pragma unroll
                for (int c = 0; c < 4; ++c) v.v[c] = acc[i][j][q * 4 + c];
                __builtin_memcpy(
                    __builtin_assume_aligned(
                        stage + lane % 32 * STRIDE + (j * 32 + q * 8 + lane / 32 * 4) * 4, 16),
                    &v, sizeof v);
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += WAVE / LPR) {
            Pack<float, EP> v;
            __builtin_memcpy(&v, __builtin_assume_aligned(stage + (r0 + lane / LPR) * STRIDE +
                                                              lane % LPR * EP * 4, 16),
                             sizeof v);
            Pack<TO, EP> o;
#pragma unroll
            for (int c = 0; c < EP; ++c) o.v[c] = from_float<TO>(v.v[c]);
            TO *p = out + (int64_t)(i * 32 + r0) * a.out_ld;
            if (m0 + wm + i * 32 + r0 + lane / LPR >= a.m) continue;
            if (n + EP <= a.n) {
                put_bytes<false, sizeof o>(p, &o);
            } else {
#pragma unroll
                for (int c = 0; c < EP; ++c)
                    if (n + c < a.n) p[c] = o.v[c];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
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

// Packed scales pay for themselves where many tiles read them.
static bool packs(int64_t m, int64_t n, const Cut &c) { return c.tile == 0 && c.splits == 1; }

int64_t product4_workspace(int64_t m, int64_t n, int32_t blocks)
{
    if (m == 0 || n == 0) return 0;
    const Cut c = cut_product(m, n, (int64_t)blocks * CHUNK);
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
    const dim3 grid((unsigned)(tm * tn), (unsigned)((steps + per - 1) / per)), block(BM / WM * (BN / WN) * WAVE);
    return launch(k_product4<BM, BN, WM, WN, STAGES, TO, PARTIAL>, grid, block, s, a, sx, sw, (int32_t)tn, (uint32_t)tm, per);
}

template <typename TO, bool PARTIAL>
static hipError_t run_cut(const Product4Args &a, const Scales4 &sx, const Scales4 &sw, const Cut &c, hipStream_t s)
{
    return c.tile == 0   ? run_tiles<256, 256, 128, 128, 2, TO, PARTIAL>(a, sx, sw, c.splits, s)
           : c.tile == 1 ? run_tiles<128, 128, 64, 64, 4, TO, PARTIAL>(a, sx, sw, c.splits, s)
           : c.tile == 2 ? run_tiles<64, 128, 32, 64, 3, TO, PARTIAL>(a, sx, sw, c.splits, s)
           : c.tile == 3 ? run_tiles<64, 64, 32, 32, 4, TO, PARTIAL>(a, sx, sw, c.splits, s)
                         : run_tiles<32, 64, 32, 32, 4, TO, PARTIAL>(a, sx, sw, c.splits, s);
}

hipError_t run_product4(const Product4Args &given, hipStream_t s)
{
    Product4Args a = given;
    if (a.m == 1) a.x_ld = a.xs_ld = 0;  // the stride of a single row is never used
    if (a.n == 1) a.w_ld = a.ws_ld = 0;
    const Cut c = cut_product(a.m, a.n, (int64_t)a.blocks * CHUNK);
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
