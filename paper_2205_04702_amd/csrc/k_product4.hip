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

constexpr int KT = 64;         // bytes of a row in one step: 128 columns, 4 scales
constexpr int STAGES = 4;      // steps that LDS holds
constexpr int CHUNK = 16;      // bytes of one access: 32 columns, one scale
constexpr int FP4 = 4;         // the matrix instruction's number of the format
constexpr int SCALE_STEPS = 4; // steps whose scales are one chunk
constexpr uint32_t GROUP = 8;  // columns of tiles that an XCD works through together

__device__ __forceinline__ void to_lds(const uint8_t *src, uint8_t *dst)
{
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void *)src,
        (__attribute__((address_space(3))) void *)dst, CHUNK, 0, 0);
}

// ---------------------------------------------------------------- tiles
//
// A block computes BM x BN outputs, each wave WM x WN of them in 32 x 32 pieces, over steps of
// 64 bytes of a row.  LDS holds four steps: the rows of the step three ahead are on their way
// straight to LDS while one is multiplied, their loads issued one by one between the matrix
// instructions.  A row's four chunks of a step are rotated among themselves by its number (chunk
// c of row r sits at c ^ (r >> 2 & 3)), so that the 16 lanes that LDS serves at a time fall on
// different banks.  The scales of four steps are one chunk of a row's scales: thread t loads
// that of the tile's row t, with every fourth step, into one of two buffers.  w is the left factor
// of the matrix instruction: its four consecutive rows per lane are four consecutive outputs.
template <int BM, int BN, int WM, int WN, typename TO, bool PARTIAL>
__global__ void __launch_bounds__(BM / WM *BN / WN *WAVE) k_product4(Product4Args a, int32_t tiles_n, uint32_t tiles_m, int32_t per_split)
{
    constexpr int NW = (BM / WM) * (BN / WN), NT = NW * WAVE;
    constexpr int TM = WM / 32, TN = WN / 32;
    constexpr int CPR = KT / CHUNK, RPL = WAVE / CPR;  // chunks per row, rows per load of a wave
    constexpr int LOADS = (BM + BN) * CPR / NT;        // of a wave and step
    static_assert(LOADS * NT == (BM + BN) * CPR && BM % (NW * RPL) == 0 && NT >= BM + BN, "whole loads");
    constexpr int BUF = (BM + BN) * KT;
    __shared__ __attribute__((aligned(16))) uint8_t sm[STAGES * BUF];
    __shared__ __attribute__((aligned(16))) uint8_t sc[2 * NT * CHUNK];
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
    const int my_chunk = (lane % CPR) ^ (my_row >> 2 & (CPR - 1));  // (RPL rows keep the rotation)
    static_assert(NW * RPL % 16 == 0, "a load's rows rotate as the first one's");
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const bool is_x = i * NW * RPL < BM;
        const int64_t at = clamped(is_x, i * NW * RPL + my_row - (is_x ? 0 : BM));
        place[i] = (uint32_t)at * (uint32_t)(is_x ? a.x_ld : a.w_ld) + (uint32_t)(my_chunk * CHUNK);
    }
    const uint8_t *xt = a.x + m0 * a.x_ld, *wt = a.w + n0 * a.w_ld;
    const int t = (int)threadIdx.x;
    const uint8_t *scale_row = t < BM ? a.xs + (m0 + clamped(true, t)) * a.xs_ld
                                      : a.ws + (n0 + clamped(false, t - BM)) * a.ws_ld;
    const auto fetch_scales = [&](int32_t step) {
        to_lds(scale_row + step / SCALE_STEPS * CHUNK, sc + (step / SCALE_STEPS % 2 * NT + wave * WAVE) * CHUNK);
    };
    // Load i of a step; chunks past the rows' last one take that one.
    const auto fetch = [&](int32_t step, int i) {
        if (i == 0 && (step % SCALE_STEPS == 0 || step == first)) fetch_scales(step);
        const bool is_x = i * NW * RPL < BM;
        const int32_t chunk = step * CPR + my_chunk, back = chunk >= a.blocks ? chunk - (a.blocks - 1) : 0;
        to_lds((is_x ? xt : wt) + step * KT + (place[i] - (uint32_t)(back * CHUNK)),
               sm + step % STAGES * BUF + (i * NW + wave) * RPL * KT);
    };
    // Every wave's loads but its last `open` are in LDS (a step's scales come before its rows), and
    // every wave is done with the buffer that is filled next.
    const auto landed = [](int open) {
        if (open >= 2 * LOADS) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * LOADS) : "memory");
        else if (open >= LOADS) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };

    v16f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

    // Two sets of factors in registers: while one is multiplied the next arrives from LDS, also
    // over the edge of a step.  A step's four scales of a row are one word, whose bytes 0 and 2
    // are those of the step's two sets once it is shifted by the lane's half.
    constexpr int KS = KT / 32;
    static_assert(KS == 2, "two sets");
    v4i f[2][TM + TN];  // x's, then w's
    uint32_t now[TM + TN], next_scales[TM + TN];
    const uint8_t *xb = sm + (wm + lane % 32) * KT, *wb = sm + (BM + wn + lane % 32) * KT;
    const uint8_t *xsb = sc + (wm + lane % 32) * CHUNK, *wsb = sc + (BM + wn + lane % 32) * CHUNK;
    const auto read = [&](int32_t step, int ks, int i) {
        const int at = step % STAGES * BUF + ((ks * 2 + lane / 32) ^ (lane >> 2 & (CPR - 1))) * CHUNK;
        f[ks][i] = i < TM ? *(const v4i *)(xb + i * 32 * KT + at) : *(const v4i *)(wb + (i - TM) * 32 * KT + at);
        if (ks == 0) {
            const int s = step / SCALE_STEPS % 2 * NT * CHUNK + step % SCALE_STEPS * CPR;
            next_scales[i] = i < TM ? *(const uint32_t *)(xsb + i * 32 * CHUNK + s)
                                    : *(const uint32_t *)(wsb + (i - TM) * 32 * CHUNK + s);
        }
    };
    const auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < TM + TN; ++i) now[i] = next_scales[i] >> (lane / 32 * 8);
    };
    // Set ks multiplied.  Between the matrix instructions: the other set's reads (of step
    // `next`), and the loads of step `ahead`; -1: none.
    const auto multiply = [&](auto set, int32_t next, int32_t ahead) {
        constexpr int ks = decltype(set)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < TM * TN; ++p) {
            const v4i &u = f[ks][TM + p % TN], &v = f[ks][p / TN];
            acc[p / TN][p % TN] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                v8i{u.x, u.y, u.z, u.w, 0, 0, 0, 0}, v8i{v.x, v.y, v.z, v.w, 0, 0, 0, 0}, acc[p / TN][p % TN], FP4, FP4,
                2 * ks, (int)now[TM + p % TN], 2 * ks, (int)now[p / TN]);
            __builtin_amdgcn_sched_barrier(0);
            if (next >= 0) {
#pragma unroll
                for (int i = 0; i < TM + TN; ++i)
                    if (i * (TM * TN) / (TM + TN) == p) read(next, ks ^ 1, i);
            }
            if (ahead >= 0) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if (i * (TM * TN) / LOADS == p) fetch(ahead, i);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr std::integral_constant<int, 0> set0{};
    constexpr std::integral_constant<int, 1> set1{};
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if (first + s < steps) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) fetch(first + s, i);
        }
    landed((steps - first < STAGES - 1 ? steps - first - 1 : STAGES - 2) * LOADS);
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) read(first, 0, i);
    int32_t s = first;
    for (; s + STAGES - 1 < steps; ++s) {
        take_scales();
        multiply(set0, s, s + STAGES - 1);
        landed(2 * LOADS);
        multiply(set1, s + 1, -1);
    }
    for (; s + 1 < steps; ++s) {
        take_scales();
        multiply(set0, s, -1);
        landed(s + 2 < steps ? LOADS : 0);
        multiply(set1, s + 1, -1);
    }
    take_scales();
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) read(s, 1, i);
    // The last step: what lies past the rows' end counts nothing, its scales neither.
    const int left = a.blocks - s * CPR - lane / 32;
    const uint32_t mask = left > 2 ? 0xFF00FFu : left > 0 ? 0xFFu : 0u;
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) {
        now[i] &= mask;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (left <= 0) f[0][i][q] = 0;
            if (left <= 2) f[1][i][q] = 0;
        }
    }
    multiply(set0, -1, -1);
    multiply(set1, -1, -1);
    __syncthreads();

    // Out through LDS, 32 rows at a time: a lane then has consecutive outputs of a row, 16
    // bytes of them, and a wave's store whole rows of its tile.
    constexpr int EP = 16 / (int)sizeof(TO);  // outputs per lane and store
    constexpr int LPR = WN / EP;              // lanes per row
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

// ---------------------------------------------------------------- host

int64_t product4_workspace(int64_t m, int64_t n, int32_t blocks)
{
    if (m == 0 || n == 0) return 0;
    const Cut c = cut_product(m, n, (int64_t)blocks * CHUNK);
    return c.splits > 1 ? m * n * 4 * c.splits : 0;
}

template <int BM, int BN, int WM, int WN, typename TO, bool PARTIAL>
static hipError_t run_tiles(const Product4Args &a, int32_t splits, hipStream_t s)
{
    const int64_t tm = (a.m + BM - 1) / BM, tn = (a.n + BN - 1) / BN;
    if (tm * tn > LAUNCH_BLOCKS / 2) {  // (up to 512 threads each; never in parts of k)
        Product4Args lo = a, hi = a;
        if (tm >= tn) {
            lo.m = tm / 2 * BM;
            hi.m = a.m - lo.m;
            hi.x += lo.m * a.x_ld;
            hi.xs += lo.m * a.xs_ld;
            hi.out = (TO *)a.out + lo.m * a.out_ld;
        } else {
            lo.n = tn / 2 * BN;
            hi.n = a.n - lo.n;
            hi.w += lo.n * a.w_ld;
            hi.ws += lo.n * a.ws_ld;
            hi.out = (TO *)a.out + lo.n;
        }
        const hipError_t r = run_tiles<BM, BN, WM, WN, TO, PARTIAL>(lo, splits, s);
        return r != hipSuccess ? r : run_tiles<BM, BN, WM, WN, TO, PARTIAL>(hi, splits, s);
    }
    const int32_t steps = (a.blocks + KT / CHUNK - 1) / (KT / CHUNK), per = (steps + splits - 1) / splits;
    const dim3 grid((unsigned)(tm * tn), (unsigned)((steps + per - 1) / per)), block(BM / WM * (BN / WN) * WAVE);
    return launch(k_product4<BM, BN, WM, WN, TO, PARTIAL>, grid, block, s, a, (int32_t)tn, (uint32_t)tm, per);
}

template <typename TO, bool PARTIAL>
static hipError_t run_cut(const Product4Args &a, const Cut &c, hipStream_t s)
{
    return c.tile == 0   ? run_tiles<256, 256, 128, 64, TO, PARTIAL>(a, c.splits, s)
           : c.tile == 1 ? run_tiles<128, 128, 64, 64, TO, PARTIAL>(a, c.splits, s)
           : c.tile == 2 ? run_tiles<64, 128, 32, 64, TO, PARTIAL>(a, c.splits, s)
           : c.tile == 3 ? run_tiles<64, 64, 32, 32, TO, PARTIAL>(a, c.splits, s)
                         : run_tiles<32, 64, 32, 32, TO, PARTIAL>(a, c.splits, s);
}

hipError_t run_product4(const Product4Args &given, hipStream_t s)
{
    Product4Args a = given;
    if (a.m == 1) a.x_ld = a.xs_ld = 0;  // the stride of a single row is never used
    if (a.n == 1) a.w_ld = a.ws_ld = 0;
    const Cut c = cut_product(a.m, a.n, (int64_t)a.blocks * CHUNK);
    return with_type(a.out_type, [&](auto to) {
        using TO = decltype(to);
        if (c.splits == 1) return run_cut<TO, false>(a, c, s);
        Product4Args p = a;
        p.out_ld = a.n;
        hipError_t r = run_cut<float, true>(p, c, s);
        if (r != hipSuccess) return r;
        const int32_t steps = (a.blocks + KT / CHUNK - 1) / (KT / CHUNK), per = (steps + c.splits - 1) / c.splits;
        const int64_t blocks = (a.m * a.n + 4 * BLOCK - 1) / (4 * BLOCK);
        if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
        return launch(k_product4_join<TO>, dim3((unsigned)blocks), dim3(BLOCK), s, a, (steps + per - 1) / per);
    });
}

}  // namespace sp
