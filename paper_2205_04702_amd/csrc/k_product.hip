// Products of 8-bit integer rows with a scale for each row of both sides:
//
//   out[m][n] = xs[m] * ws[n] * sum over k of x[m][k] * w[n][k]
//
// The sums are exact in 32 bits (k <= 131071); each is rounded to fp32 once, scaled in
// fp32 and rounded once to the output's type.
#include "sp_rows.h"

namespace sp {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

constexpr int KT = 128;     // bytes of a row in one step
constexpr int CHUNK = 16;   // bytes of one access

__device__ __forceinline__ void to_lds(const int8_t *src, int8_t *dst)
{
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void *)src,
        (__attribute__((address_space(3))) void *)dst, CHUNK, 0, 0);
}

// A chunk of a row whose start or stride is no multiple of 16 bytes; bytes past the end
// are zeros.
__device__ __forceinline__ v4i guarded_chunk(const int8_t *row, int32_t at, int32_t k)
{
    v4i v = {0, 0, 0, 0};
    if (at + CHUNK <= k) {
        __builtin_memcpy(&v, row + at, CHUNK);
    } else {
#pragma unroll
        for (int i = 0; i < CHUNK; ++i)
            if (at + i < k) v[i / 4] |= (int)((uint32_t)(uint8_t)row[at + i] << (8 * (i % 4)));
    }
    return v;
}

// ---------------------------------------------------------------- tiles
//
// A block computes BM x BN outputs, each wave WM x WN of them in 32 x 32 pieces, over
// steps of 128 bytes of k, with two buffers in LDS: the rows of the next step arrive
// straight in LDS while this one is multiplied.  A row's eight chunks of a step are
// rotated among themselves by its number (chunk c of row r sits at c ^ (r >> 1 & 7)),
// so that the 16 lanes that LDS serves at a time, 16 rows of one chunk, fall on
// different banks.  w is the left factor of the matrix instruction: its four
// consecutive rows per lane are four consecutive outputs of a row.
template <int BM, int BN, int WM, int WN, typename TO, bool ALIGNED>
__global__ void __launch_bounds__(BM / WM *BN / WN *WAVE) k_product(ProductArgs a, int32_t tiles_n)
{
    constexpr int NW = (BM / WM) * (BN / WN), NT = NW * WAVE;
    constexpr int TM = WM / 32, TN = WN / 32;
    constexpr int LOADS = (BM + BN) * (KT / CHUNK) / NT;
    static_assert(LOADS * NT == (BM + BN) * (KT / CHUNK) && BM % (NW * 8) == 0, "whole loads");
    __shared__ __attribute__((aligned(16))) int8_t sm[2][(BM + BN) * KT];
    const int wave = wave_id(), lane = lane_id();
    const int64_t m0 = (int64_t)(blockIdx.x / (uint32_t)tiles_n) * BM;
    const int64_t n0 = (int64_t)(blockIdx.x % (uint32_t)tiles_n) * BN;
    const int32_t steps = (a.k + KT - 1) / KT;
    const int32_t last_chunk = (a.k - 1) / CHUNK * CHUNK;

    const auto fetch = [&](int buf, int32_t step) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = (i * NW + wave) * 8 + lane / 8;  // of the x rows, then the w rows
            const bool is_x = i * NW * 8 < BM;
            const int64_t last = is_x ? a.m - 1 : a.n - 1;
            const int64_t at = is_x ? m0 + r : n0 + (r - BM);
            const int8_t *row = is_x ? a.x + (at < last ? at : last) * a.x_ld
                                     : a.w + (at < last ? at : last) * a.w_ld;
            int32_t kb = step * KT + ((lane % 8) ^ (r >> 1 & 7)) * CHUNK;
            int8_t *dst = &sm[buf][(i * NW + wave) * 8 * KT];
            if (ALIGNED) {
                kb = kb < last_chunk ? kb : last_chunk;
                to_lds(row + kb, dst);
            } else {
                *(v4i *)(dst + lane * CHUNK) = guarded_chunk(row, kb, a.k);
            }
        }
    };

    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    v16i acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;

    // the loads of a step are in LDS: every wave waits for its own, then for the others
    const auto landed = [&] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    fetch(0, 0);
    landed();
    for (int32_t s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch((s + 1) & 1, s + 1);
        const int8_t *xb = &sm[s & 1][(wm + lane % 32) * KT];
        const int8_t *wb = &sm[s & 1][(BM + wn + lane % 32) * KT];
#pragma unroll
        for (int ks = 0; ks < KT / 32; ++ks) {
            const int at = ((ks * 2 + lane / 32) ^ (lane >> 1 & 7)) * CHUNK;
            v4i x[TM], w[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) x[i] = *(const v4i *)(xb + i * 32 * KT + at);
#pragma unroll
            for (int j = 0; j < TN; ++j) w[j] = *(const v4i *)(wb + j * 32 * KT + at);
            const int32_t left = a.k - s * KT - (ks * 2 + lane / 32) * CHUNK;
            if (left < CHUNK) {  // what lies past the rows' end counts nothing
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int32_t b = left - 4 * q;
                    const int mask = b >= 4 ? -1 : b <= 0 ? 0 : (int)((1u << (8 * b)) - 1);
#pragma unroll
                    for (int i = 0; i < TM; ++i) x[i][q] &= mask;
                }
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[j], x[i], acc[i][j], 0, 0, 0);
        }
        landed();
    }

    // Out through LDS, 32 rows at a time: a lane then has consecutive outputs of a row, 16
    // bytes of them, and a wave's store whole rows of its tile.
    constexpr int EP = 16 / (int)sizeof(TO);   // outputs per lane and store
    constexpr int LPR = WN / EP;               // lanes per row
    constexpr int STRIDE = WN * 4 + 16;
    static_assert(NW * 32 * STRIDE <= (int)sizeof sm && WAVE % LPR == 0, "staging fits the buffers");
    int8_t *stage = &sm[0][0] + wave * 32 * STRIDE;
    TO *out = (TO *)a.out;
    const int64_t n = n0 + wn + lane % LPR * EP;
    float ws[EP];
#pragma unroll
    for (int c = 0; c < EP; ++c) ws[c] = a.ws[n + c < a.n ? n + c : a.n - 1];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v4i v = {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2],
                               acc[i][j][q * 4 + 3]};
                *(v4i *)(stage + lane % 32 * STRIDE + (j * 32 + q * 8 + lane / 32 * 4) * 4) = v;
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += WAVE / LPR) {
            const int r = r0 + lane / LPR;
            const int64_t m = m0 + wm + i * 32 + r;
            int v[EP];
            __builtin_memcpy(v, __builtin_assume_aligned(stage + r * STRIDE + lane % LPR * EP * 4, 16),
                             sizeof v);
            if (m >= a.m || n >= a.n) continue;
            const float xs = a.xs[m];
            Pack<TO, EP> o;
#pragma unroll
            for (int c = 0; c < EP; ++c) o.v[c] = from_float<TO>((float)v[c] * xs * ws[c]);
            TO *p = out + m * a.out_ld + n;
            if (n + EP <= a.n) {
                __builtin_memcpy(p, &o, sizeof o);
            } else {
#pragma unroll
                for (int c = 0; c < EP; ++c)
                    if (n + c < a.n) p[c] = o.v[c];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

int64_t product_workspace(int64_t, int64_t, int64_t) { return 0; }

template <typename TO>
static hipError_t product_as(const ProductArgs &a, hipStream_t s)
{
    const bool aligned = ((uintptr_t)a.x | (uintptr_t)a.w | (uint64_t)a.x_ld | (uint64_t)a.w_ld) % CHUNK == 0;
    constexpr int BM = 128, BN = 128;
    const int64_t tm = (a.m + BM - 1) / BM, tn = (a.n + BN - 1) / BN;
    if (tm * tn > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)(tm * tn)), block(4 * WAVE);
    return aligned ? launch(k_product<BM, BN, 64, 64, TO, true>, grid, block, s, a, (int32_t)tn)
                   : launch(k_product<BM, BN, 64, 64, TO, false>, grid, block, s, a, (int32_t)tn);
}

hipError_t run_product(const ProductArgs &a, hipStream_t s)
{
    return with_type(a.out_type, [&](auto to) { return product_as<decltype(to)>(a, s); });
}

}  // namespace sp
