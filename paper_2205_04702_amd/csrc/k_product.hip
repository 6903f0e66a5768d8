// Products of 8-bit integer rows with a scale for each row of both sides:
//
//   out[m][n] = xs[m] * ws[n] * sum over k of x[m][k] * w[n][k]
//
// The sums are exact in 32 bits (k <= 131071); each is rounded to fp32 once, scaled in
// fp32 and rounded once to the output's type.
#include <cmath>
#include <type_traits>

#include "sp_rows.h"

namespace sp {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

constexpr int KT = 64;      // bytes of a row in one step
constexpr int STAGES = 4;   // steps that LDS holds
constexpr int CHUNK = 16;   // bytes of one access
constexpr uint32_t GROUP = 8;  // columns of tiles that an XCD works through together

__device__ __forceinline__ void to_lds(const int8_t *src, int8_t *dst)
{
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void *)src,
        (__attribute__((address_space(3))) void *)dst, CHUNK, 0, 0);
}

// Rows whose start or stride is no multiple of 16 bytes go through registers: a chunk is
// 16 bytes at any address.  The chunks past a row's last whole one are loaded as the
// row's last 16 bytes and moved down by `over` bytes (16 and more: all of them).
__device__ __forceinline__ v4i moved_down(v4i v, int over)
{
    uint32_t w[4] = {(uint32_t)v.x, (uint32_t)v.y, (uint32_t)v.z, (uint32_t)v.w};
#pragma unroll
    for (int by = 4; by <= 16; by *= 2) {
        const bool move = by == 16 ? over >= 16 : (over & by) != 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = move ? (i + by / 4 < 4 ? w[i + by / 4] : 0u) : w[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = __builtin_amdgcn_alignbyte(i < 3 ? w[i + 1] : 0u, w[i], over & 3);
    return v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}
// The same of a row shorter than a chunk, byte by byte.
__device__ __forceinline__ v4i short_row(const int8_t *row, int32_t at, int32_t k)
{
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < CHUNK; ++i)
        if (at + i < k) w[i / 4] |= (uint32_t)(uint8_t)row[at + i] << (8 * (i % 4));
    return v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

// ---------------------------------------------------------------- tiles
//
// A block computes BM x BN outputs, each wave WM x WN of them in 32 x 32 pieces, over
// steps of 64 bytes of k.  LDS holds four steps: the rows of the step three ahead are on
// their way straight to LDS while one is multiplied, their loads issued one by one
// between the matrix instructions (issued together they kept a wave from those for as long as the
// multiplication takes).  A row's four chunks of a step are rotated among themselves by
// its number (chunk c of row r sits at c ^ (r >> 2 & 3)), so that the 16 lanes that LDS
// serves at a time, 16 rows of one chunk, fall on different banks.  w is the left
// factor of the matrix instruction: its four consecutive rows per lane are four
// consecutive outputs of a row.
//
// 8192^3 in tiles of 256: 480 to 500 us, 2.2 to 2.3 POP/s, at the clock that power leaves (1.65 GHz
// by the counters; matrix instructions alone took 368 us), the matrix cores busy 65 % of the time,
// 89 % of the reads served by L2.  Smaller tiles are bound by what a CU loads.
template <int BM, int BN, int WM, int WN, typename TO, bool ALIGNED>
__global__ void __launch_bounds__(BM / WM *BN / WN *WAVE) k_product(ProductArgs a, int32_t tiles_n, uint32_t tiles_m, int32_t per_split)
{
    constexpr int NW = (BM / WM) * (BN / WN), NT = NW * WAVE;
    constexpr int TM = WM / 32, TN = WN / 32;
    constexpr int CPR = KT / CHUNK, RPL = WAVE / CPR;  // chunks per row, rows per load of a wave
    constexpr int LOADS = (BM + BN) * CPR / NT;        // of a wave and step
    static_assert(LOADS * NT == (BM + BN) * CPR && BM % (NW * RPL) == 0, "whole loads");
    constexpr int BUF = (BM + BN) * KT;
    __shared__ __attribute__((aligned(16))) int8_t sm[STAGES * BUF];
    const int wave = wave_id(), lane = lane_id();
    // Which tile: each XCD takes a stretch of the tiles, in groups of eight columns of tiles, so
    // that what runs on it at a time (4 x 8 tiles, say, of 12 tiles' rows) shares its L2 and
    // rows of w are read by one XCD.  Tile after tile along a row of tiles and XCD after XCD,
    // groups of four columns, of eight, of sixteen (us, rows past the caches):
    //   8192 x 16384 x 512      125  134  126  135       5000 x 5000 x 5000    150  141  147  144
    //   8192 x 16384 x 4096     518  524  521  528       16384 x 2048 x 8192   266  250  250  250
    //   10000 x 30000 x 1000    444  418  398  429       1000 x 60000 x 4096   286  260  263  264
    //   6000 x 12000 x 3000     249  234  233  239       3000 x 20000 x 300     60   57   54   53
    // and within 2 % of the best of them in 17 more shapes, in 5000 x 5000 x 2500 within 4 %.  One row
    // of tiles has nothing to share, and the divisions' time to lose: 64 x 4096 x 4096 13.3 in
    // groups, 12.5 without.
    uint32_t tile_m = 0, tile_n = blockIdx.x;
    if (tiles_m > 1) {
        const uint32_t tile = (uint32_t)xcd_block(blockIdx.x, gridDim.x);
        const uint32_t group = tile / (GROUP * tiles_m), in = tile - group * GROUP * tiles_m;
        const uint32_t wide = (uint32_t)tiles_n - group * GROUP < GROUP ? (uint32_t)tiles_n - group * GROUP : GROUP;
        tile_m = in / wide;
        tile_n = group * GROUP + in % wide;
    }
    const int64_t m0 = (int64_t)tile_m * BM, n0 = (int64_t)tile_n * BN;
    constexpr bool PARTIAL = std::is_same<TO, int32_t>::value;  // sums of a part of k
    const int32_t first = (int32_t)blockIdx.y * per_split;
    const int32_t all = (a.k + KT - 1) / KT, steps = first + per_split < all ? first + per_split : all;

    // The scales this lane will need, now: at the end their latency, and the wait for earlier
    // stores that comes with any load, took as long as the stores themselves.
    constexpr int EP = 16 / (int)sizeof(TO);  // outputs per lane and store
    constexpr int LPR = WN / EP;              // lanes per row
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    const int64_t n = n0 + wn + lane % LPR * EP;
    float xs[TM], ws[EP];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm + i * 32 + lane % 32;
        xs[i] = PARTIAL ? 1.f : a.xs[m < a.m ? m : a.m - 1];
    }
#pragma unroll
    for (int c = 0; c < EP; ++c) ws[c] = PARTIAL ? 1.f : a.ws[n + c < a.n ? n + c : a.n - 1];

    // This lane's chunk of each load: a place relative to the tile's first row, which with
    // whole chunks fits 32 bits (ALIGNED: strides below 2^23).
    uint32_t place[LOADS];
    const int my_row = wave * RPL + lane / CPR;
    const int my_chunk = (lane % CPR) ^ (my_row >> 2 & (CPR - 1));  // (RPL rows keep the rotation)
    static_assert(NW * RPL % 16 == 0, "a load's rows rotate as the first one's");
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const bool is_x = i * NW * RPL < BM;
        const int64_t last = is_x ? a.m - 1 - m0 : a.n - 1 - n0;
        const int64_t at = i * NW * RPL + my_row - (is_x ? 0 : BM);
        place[i] = (uint32_t)(at < last ? at : last) * (uint32_t)(is_x ? a.x_ld : a.w_ld) +
                   (uint32_t)(my_chunk * CHUNK);
    }
    const int8_t *xt = a.x + m0 * a.x_ld, *wt = a.w + n0 * a.w_ld;
    // Load i of a step; chunks past the rows' last one take that one.  Unaligned, the load goes
    // to registers, and the one that they held, of the step before, to LDS: three
    // steps' loads are in LDS or on their way as well.
    v4i held[ALIGNED ? 1 : LOADS];
    const auto row_of = [&](int i) {
        const bool is_x = i * NW * RPL < BM;
        const int64_t last = is_x ? a.m - 1 - m0 : a.n - 1 - n0;
        const int64_t at = i * NW * RPL + my_row - (is_x ? 0 : BM);
        return (is_x ? xt : wt) + (at < last ? at : last) * (is_x ? a.x_ld : a.w_ld);
    };
    const auto buffer = [&](int32_t step, int i) {
        return sm + step % STAGES * BUF + (i * NW + wave) * RPL * KT;
    };
    const auto hold = [&](int32_t step, int i) {
        const int32_t kb = step * KT + my_chunk * CHUNK, last = a.k - CHUNK;
        __builtin_memcpy(&held[ALIGNED ? 0 : i], row_of(i) + (kb < last ? kb : last), CHUNK);
    };
    const auto put = [&](int32_t step, int i) {
        v4i v = held[ALIGNED ? 0 : i];
        if (step + 1 == all) {
            const int32_t over = step * KT + my_chunk * CHUNK - (a.k - CHUNK);
            v = moved_down(v, over > 0 ? over : 0);
        }
        *(v4i *)(buffer(step, i) + lane * CHUNK) = v;
    };
    const auto fetch = [&](int32_t step, int i) {
        if (ALIGNED) {
            const bool is_x = i * NW * RPL < BM;
            const int32_t kb = step * KT + my_chunk * CHUNK;
            const int32_t last = (a.k - 1) / CHUNK * CHUNK;
            const int32_t back = kb > last ? kb - last : 0;
            to_lds((is_x ? xt : wt) + step * KT + (place[i] - (uint32_t)back), buffer(step, i));
        } else {
            put(step - 1, i);
            hold(step, i);
        }
    };
    // Every wave's loads but its last `open` are in LDS, and every wave is done with the
    // buffer that is filled next.
    const auto landed = [](int open) {
        if (open >= 2 * LOADS) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * LOADS) : "memory");
        else if (open >= LOADS) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };

    v16i acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;

    // Two sets of factors in registers: while one is multiplied the next arrives from LDS,
    // also over the edge of a step.
    constexpr int KS = KT / 32;
    static_assert(KS == 2, "two sets");
    v4i x[2][TM], w[2][TN];
    const int8_t *xb = sm + (wm + lane % 32) * KT, *wb = sm + (BM + wn + lane % 32) * KT;
    const auto read = [&](int32_t step, int ks, int i) {  // factor i of a set: x's, then w's
        const int at = step % STAGES * BUF + ((ks * 2 + lane / 32) ^ (lane >> 2 & (CPR - 1))) * CHUNK;
        if (i < TM) x[ks][i] = *(const v4i *)(xb + i * 32 * KT + at);
        else w[ks][i - TM] = *(const v4i *)(wb + (i - TM) * 32 * KT + at);
    };
    // Set ks multiplied.  Between the matrix instructions: the other set's reads (of step
    // `next`), and the loads of step `ahead`; -1: none.
    const auto multiply = [&](int ks, int32_t next, int32_t ahead) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < TM * TN; ++t) {
            acc[t / TN][t % TN] = __builtin_amdgcn_mfma_i32_32x32x32_i8(
                w[ks][t % TN], x[ks][t / TN], acc[t / TN][t % TN], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (next >= 0) {
#pragma unroll
                for (int i = 0; i < TM + TN; ++i)
                    if (i * (TM * TN) / (TM + TN) == t) read(next, ks ^ 1, i);
            }
            if (ahead >= 0) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (i * (TM * TN) / LOADS == t) fetch(ahead, i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (ALIGNED) {
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (first + s < steps) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) fetch(first + s, i);
            }
    } else if (a.k < CHUNK) {  // one step
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            *(v4i *)(buffer(first, i) + lane * CHUNK) = short_row(row_of(i), my_chunk * CHUNK, a.k);
    } else {  // two steps in LDS, the third held
        for (int s = 0; s < STAGES - 1; ++s)
            if (first + s < steps) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) hold(first + s, i);
                if (s < STAGES - 2) {
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) put(first + s, i);
                }
            }
    }
    landed((steps - first < STAGES - 1 ? steps - first - 1 : STAGES - 2) * LOADS);
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) read(first, 0, i);
    int32_t s = first;
    for (; s + STAGES - 1 < steps; ++s) {
        multiply(0, s, s + STAGES - 1);
        landed(2 * LOADS);
        multiply(1, s + 1, -1);
    }
    for (; s + 1 < steps; ++s) {
        if (!ALIGNED && s + 2 < steps) {  // (once: the step still held)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) put(s + 2, i);
        }
        multiply(0, s, -1);
        landed(s + 2 < steps ? LOADS : 0);
        multiply(1, s + 1, -1);
    }
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) read(s, 1, i);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {  // the last step: what lies past the rows' end counts nothing
        const int32_t left = a.k - s * KT - (ks * 2 + lane / 32) * CHUNK;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int32_t b = left - 4 * q;
            const int mask = b >= 4 ? -1 : b <= 0 ? 0 : (int)((1u << (8 * b)) - 1);
#pragma unroll
            for (int i = 0; i < TM; ++i) x[ks][i][q] &= mask;
        }
        multiply(ks, -1, -1);
    }
    __syncthreads();

    // Out through LDS, 32 rows at a time: a lane then has consecutive outputs of a row, 16
    // bytes of them, and a wave's store whole rows of its tile.
    constexpr int STRIDE = WN * 4 + 16;
    static_assert(NW * 32 * STRIDE <= (int)sizeof sm && WAVE % LPR == 0, "staging fits the buffers");
    int8_t *stage = sm + wave * 32 * STRIDE;
    using Held = typename std::conditional<PARTIAL, int32_t, float>::type;
    TO *out = (PARTIAL ? (TO *)a.work + (int64_t)blockIdx.y * a.m * a.n : (TO *)a.out) + (m0 + wm + lane / LPR) * a.out_ld + n;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                Pack<Held, 4> v;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    v.v[c] = PARTIAL ? (Held)acc[i][j][q * 4 + c] : (Held)((float)acc[i][j][q * 4 + c] * xs[i]);
                __builtin_memcpy(
                    __builtin_assume_aligned(
                        stage + lane % 32 * STRIDE + (j * 32 + q * 8 + lane / 32 * 4) * 4, 16),
                    &v, sizeof v);
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += WAVE / LPR) {
            Pack<Held, EP> v;
            __builtin_memcpy(&v, __builtin_assume_aligned(stage + (r0 + lane / LPR) * STRIDE +
                                                              lane % LPR * EP * 4, 16),
                             sizeof v);
            Pack<TO, EP> o;
#pragma unroll
            for (int c = 0; c < EP; ++c) o.v[c] = PARTIAL ? (TO)v.v[c] : from_float<TO>(v.v[c] * ws[c]);
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

// The parts of a split sum added up, scaled and rounded: four outputs per thread.
template <typename TO>
__global__ void __launch_bounds__(BLOCK) k_product_join(ProductArgs a, int32_t splits)
{
    const int64_t total = a.m * a.n, i0 = ((int64_t)blockIdx.x * BLOCK + threadIdx.x) * 4;
    if (i0 >= total) return;
    const int32_t *part = (const int32_t *)a.work + i0;
    int v[4] = {0, 0, 0, 0};
    const int valid = total - i0 < 4 ? (int)(total - i0) : 4;
    if (valid == 4) {
#pragma unroll 4
        for (int32_t s = 0; s < splits; ++s) {
            Pack<int, 4> p;
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
        if (c < valid) ((TO *)a.out)[m * a.out_ld + n] = from_float<TO>((float)v[c] * a.xs[m] * a.ws[n]);
        if (++n == a.n) n = 0, ++m;
    }
}

// ---------------------------------------------------------------- host

// How a product is cut: into tiles, and parts of k where the tiles are few.  The estimate,
// in us, for what each CU has to do one after the other: a tile's fixed time (first loads,
// outputs) and its steps of k, with the card mostly idle or busy, and for parts a second
// launch and their traffic.  Measured on both sides of the lines that it draws (us):
//                        256x256  128x128  64x128  64x64  32x64   in parts
//   8192 x 8192 x 8192       471      662
//   777 x 10001 x 1000        22       27      32     34     50
//   2048 x 2048 x 2048        28       18      19     22     27
//   1500 x 700 x 3000         35       21      15     17     19   19 (2 of 128x128)
//   256 x 4096 x 4096         42       25      19     15     15   19 (2 of 64x64)
//   128 x 8192 x 8192         84       50      44     36     41   27 (4 of 128x128)
//   64 x 4096 x 4096                   25      18     14     13   11 (4 of 64x64)
//   33 x 2000 x 512                     7       6      5      5    7 (2 of 32x64)
//   424 x 222 x 3424          40       23      16     12     12    9 (4 of 32x64)
struct Cut {
    int32_t tile, splits;
};
static Cut cut_product(int64_t m, int64_t n, int64_t k)
{
    constexpr struct {
        int bm, bn;
        double idle, busy, fixed;
    } T[] = {{256, 256, 0.56, 0.86, 7.3}, {128, 128, 0.33, 0.31, 1.8}, {64, 128, 0.22, 0.24, 1.0},
             {64, 64, 0.165, 0.19, 0.6}, {32, 64, 0.155, 0.16, 0.5}};
    const int64_t steps = (k + KT - 1) / KT;
    Cut best{1, 1};
    double least = 1e300;
    for (int t = 0; t < 5; ++t) {
        const double tiles = (double)((m + T[t].bm - 1) / T[t].bm) * (double)((n + T[t].bn - 1) / T[t].bn);
        for (int sp = 1; sp <= 16; sp *= 2) {
            if (sp > 1 && (steps < 4 * sp || tiles * sp > 1024)) break;
            const double blocks = tiles * sp, step = blocks <= 192 ? T[t].idle : T[t].busy;
            double us = std::ceil(blocks / 256) * (T[t].fixed + step * (double)((steps + sp - 1) / sp));
            if (sp > 1) us += 3.0 + (double)m * (double)n * 4.0 * (2 * sp) / 4e6;
            if (us < least) least = us, best = Cut{t, sp};
        }
    }
    return best;
}

int64_t product_workspace(int64_t m, int64_t n, int64_t k)
{
    if (m == 0 || n == 0) return 0;
    const Cut c = cut_product(m, n, k);
    return c.splits > 1 ? m * n * 4 * c.splits : 0;
}

template <int BM, int BN, int WM, int WN, typename TO>
static hipError_t run_tiles(const ProductArgs &a, int32_t splits, hipStream_t s)
{
    const bool aligned =
        ((uintptr_t)a.x | (uintptr_t)a.w | (uint64_t)a.x_ld | (uint64_t)a.w_ld) % CHUNK == 0 &&
        a.x_ld < 1 << 23 && a.w_ld < 1 << 23;
    const int64_t tm = (a.m + BM - 1) / BM, tn = (a.n + BN - 1) / BN;
    if (tm * tn > LAUNCH_BLOCKS / 2) {  // (up to 512 threads each; never in parts of k)
        ProductArgs lo = a, hi = a;
        if (tm >= tn) {
            lo.m = tm / 2 * BM;
            hi.m = a.m - lo.m;
            hi.x += lo.m * a.x_ld;
            hi.xs += lo.m;
            hi.out = (TO *)a.out + lo.m * a.out_ld;
        } else {
            lo.n = tn / 2 * BN;
            hi.n = a.n - lo.n;
            hi.w += lo.n * a.w_ld;
            hi.ws += lo.n;
            hi.out = (TO *)a.out + lo.n;
        }
        const hipError_t r = run_tiles<BM, BN, WM, WN, TO>(lo, splits, s);
        return r != hipSuccess ? r : run_tiles<BM, BN, WM, WN, TO>(hi, splits, s);
    }
    const int32_t steps = (a.k + KT - 1) / KT, per = (steps + splits - 1) / splits;
    const dim3 grid((unsigned)(tm * tn), (unsigned)((steps + per - 1) / per)), block(BM / WM * (BN / WN) * WAVE);
    return aligned ? launch(k_product<BM, BN, WM, WN, TO, true>, grid, block, s, a, (int32_t)tn, (uint32_t)tm, per)
                   : launch(k_product<BM, BN, WM, WN, TO, false>, grid, block, s, a, (int32_t)tn, (uint32_t)tm, per);
}

template <typename TO>
static hipError_t run_cut(const ProductArgs &a, const Cut &c, hipStream_t s)
{
    return c.tile == 0   ? run_tiles<256, 256, 128, 64, TO>(a, c.splits, s)
           : c.tile == 1 ? run_tiles<128, 128, 64, 64, TO>(a, c.splits, s)
           : c.tile == 2 ? run_tiles<64, 128, 32, 64, TO>(a, c.splits, s)
           : c.tile == 3 ? run_tiles<64, 64, 32, 32, TO>(a, c.splits, s)
                         : run_tiles<32, 64, 32, 32, TO>(a, c.splits, s);
}

hipError_t run_product(const ProductArgs &given, hipStream_t s)
{
    ProductArgs a = given;
    if (a.m == 1) a.x_ld = 0;  // the stride of a single row aligns, and misaligns, nothing
    if (a.n == 1) a.w_ld = 0;
    const Cut c = cut_product(a.m, a.n, a.k);
    return with_type(a.out_type, [&](auto to) {
        using TO = decltype(to);
        if (c.splits == 1) return run_cut<TO>(a, c, s);
        ProductArgs p = a;
        p.out_ld = a.n;
        hipError_t r = run_cut<int32_t>(p, c, s);
        if (r != hipSuccess) return r;
        const int32_t steps = (a.k + KT - 1) / KT, per = (steps + c.splits - 1) / c.splits;
        const int64_t blocks = (a.m * a.n + 4 * BLOCK - 1) / (4 * BLOCK);
        if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
        return launch(k_product_join<TO>, dim3((unsigned)blocks), dim3(BLOCK), s, a, (steps + per - 1) / per);
    });
}

}  // namespace sp
