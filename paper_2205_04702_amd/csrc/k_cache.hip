// Rows in 8 bits: a cache that is quantised as it is written, and read back.
//
// A row of `dim` columns is held as dim bytes and one fp32 scale for each group
// of `group` columns: scale = amax / top, byte = x / scale rounded to nearest
// (ties to even), with top the largest magnitude of the kind: 127 for integers,
// 448 for 8-bit floats with 4 exponent and 3 mantissa bits.
#include "sp_rows.h"

namespace sp {

constexpr int KIND_INT = 5, KIND_FLOAT = 6;  // SP_I8, SP_F8
constexpr uint32_t INF_BITS = 0x7F800000u;
constexpr float SMALLEST_SCALE = 1.17549435e-38f;  // below it 1 / scale would overflow

template <int KIND>
__device__ __forceinline__ uint2 pack_oct(const float (&v)[OCT])
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (KIND == KIND_INT) {
            uint32_t x = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float r = fminf(fmaxf(rintf(v[4 * h + k]), -127.f), 127.f);
                x |= ((uint32_t)(int32_t)r & 0xFFu) << (8 * k);
            }
            w[h] = x;
        } else {
            int x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
            w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], x, true);
        }
    }
    return make_uint2(w[0], w[1]);
}

template <int KIND>
__device__ __forceinline__ void unpack_oct(const uint32_t (&x)[2], float (&v)[OCT])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (KIND == KIND_INT) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[4 * h + k] = (float)(int8_t)(x[h] >> (8 * k));
        } else {
            v[4 * h] = __builtin_amdgcn_cvt_f32_fp8((int)x[h], 0);
            v[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8((int)x[h], 1);
            v[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8((int)x[h], 2);
            v[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8((int)x[h], 3);
        }
    }
}

__device__ __forceinline__ void store_bytes(uint8_t *p, int valid, uint2 w)
{
    if (valid >= OCT) {
        __builtin_memcpy(p, &w, 8);
    } else {
#pragma unroll
        for (int k = 0; k < OCT; ++k)
            if (k < valid) p[k] = (uint8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3)));
    }
}
// ---------------------------------------------------------------- write
//
// A team of TEAM lanes holds one group, OPL octets in each lane (team-strided,
// so neighbouring lanes read neighbouring bytes), or walks over it a second time
// where it does not fit into registers (LOOP).  The maximum is taken over the
// magnitudes' bits: their order is that of the values, and infinity and NaN come
// out above everything.  A group that holds one of these gets a NaN scale and
// zero bytes (it reads back as NaN); one whose scale would be subnormal is held
// as zeros.
template <typename T, typename IX, int KIND, int TEAM, int OPL, bool LOOP>
__global__ void __launch_bounds__(BLOCK) k_cache_write(CacheArgs a, Split s, int32_t octs)
{
    constexpr float top = KIND == KIND_INT ? 127.f : 448.f;
    const int unit = (int)threadIdx.x / TEAM, lane = (int)threadIdx.x % TEAM;
    int64_t row;
    int32_t grp;
    bool on = split_at(s, blockIdx.x, unit, row, grp);
    int64_t slot = row;
    if (on && a.index) slot = (int64_t)((const IX *)a.index)[row];
    on = on && slot >= 0 && slot < a.slots;
    if (!on) return;  // whole teams
    const int32_t col0 = grp * a.group;
    const T *x = (const T *)a.x + row * a.x_ld + col0;
    uint8_t *q = (uint8_t *)a.q + slot * a.q_ld + col0;
    float v[OPL][OCT];
    uint32_t top_bits = 0;
    for (int32_t o0 = 0; o0 < (LOOP ? octs : 1); o0 += TEAM * OPL) {
#pragma unroll
        for (int i = 0; i < OPL; ++i) {
            const int32_t o = o0 + i * TEAM + lane;
            if (o < octs) load_oct<true, (TEAM > 4)>(x, o, cols_of(a.group), v[i]);
        }
#pragma unroll
        for (int i = 0; i < OPL; ++i) {
            if (o0 + i * TEAM + lane < octs) {
#pragma unroll
                for (int k = 0; k < OCT; ++k) {
                    const uint32_t b = __float_as_uint(v[i][k]) & 0x7FFFFFFFu;
                    const bool in = (o0 + i * TEAM + lane) * OCT + k < a.group;
                    top_bits = in && b > top_bits ? b : top_bits;
                }
            }
        }
    }
#pragma unroll
    for (int o = TEAM / 2; o > 0; o >>= 1) {
        const uint32_t b = (uint32_t)__shfl_xor((int)top_bits, o, WAVE);
        top_bits = b > top_bits ? b : top_bits;
    }
    const bool finite = top_bits < INF_BITS;
    float scale = __uint_as_float(top_bits) * (1.f / top);
    if (!(scale >= SMALLEST_SCALE)) scale = 0.f;
    const float inverse = finite && scale > 0.f ? 1.f / scale : 0.f;
    if (!finite) scale = __uint_as_float(0x7FC00000u);
    if (lane == 0) a.scales[slot * a.scales_ld + grp] = scale;
    for (int32_t o0 = 0; o0 < (LOOP ? octs : 1); o0 += TEAM * OPL) {
#pragma unroll
        for (int i = 0; i < OPL; ++i) {
            const int32_t o = o0 + i * TEAM + lane;
            if (o < octs) {
                const int valid = oct_valid(a.group, o);
                if (LOOP) load_oct<false, (TEAM > 4)>(x, o, cols_of(a.group), v[i]);
#pragma unroll
                for (int k = 0; k < OCT; ++k) v[i][k] = finite ? v[i][k] * inverse : 0.f;
                store_bytes(q + o * OCT, valid, pack_oct<KIND>(v[i]));
            }
        }
    }
}

template <typename T, typename IX, int KIND>
static hipError_t write_teams(const CacheArgs &a, hipStream_t st)
{
    const int32_t octs = (a.group + OCT - 1) / OCT, groups = a.dim / a.group;
    const auto go = [&](auto kern, int team) {
        const Split s = split_rows(a.n, groups, BLOCK / team);
        const int64_t blocks = split_blocks(s);
        if (blocks <= 0) return hipSuccess;
        if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
        return launch(kern, dim3((unsigned)blocks), dim3(BLOCK), st, a, s, octs);
    };
    if (octs <= 4) return go(k_cache_write<T, IX, KIND, 4, 1, false>, 4);
    if (octs <= 8) return go(k_cache_write<T, IX, KIND, 8, 1, false>, 8);
    if (octs <= 16) return go(k_cache_write<T, IX, KIND, 16, 1, false>, 16);
    if (octs <= 32) return go(k_cache_write<T, IX, KIND, 32, 1, false>, 32);
    if (octs <= 64) return go(k_cache_write<T, IX, KIND, 64, 1, false>, 64);
    if (octs <= 128) return go(k_cache_write<T, IX, KIND, 64, 2, false>, 64);
    if (octs <= 256) return go(k_cache_write<T, IX, KIND, 64, 4, false>, 64);
    if (octs <= 512) return go(k_cache_write<T, IX, KIND, 64, 8, false>, 64);
    return go(k_cache_write<T, IX, KIND, 64, 8, true>, 64);
}

hipError_t run_cache_write(const CacheArgs &a, hipStream_t s)
{
    return with_index(a.index_type, [&](auto ix) {
        return with_type(a.type, [&](auto t) {
            using IX = decltype(ix);
            using T = decltype(t);
            return a.kind == KIND_INT ? write_teams<T, IX, KIND_INT>(a, s)
                                      : write_teams<T, IX, KIND_FLOAT>(a, s);
        });
    });
}

// ---------------------------------------------------------------- read

// x[i] = bytes of slot index[i] times their groups' scales; zeros where index[i]
// is no slot.
template <typename T, typename IX, int KIND>
struct CacheRead {
    CacheArgs a;
    float per_group;  // octets of a group, inverted; 0: one group
    struct Regs {
        Raw<uint8_t> w;
        float scale;
        int64_t slot;
        bool live;
    };
    __device__ __forceinline__ void first(int64_t row, Regs &g) const
    {
        g.slot = a.index ? (int64_t)((const IX *)a.index)[row] : row;
    }
    template <bool STREAM>
    __device__ __forceinline__ void load(int64_t, int32_t oct, Regs &g) const
    {
        g.live = g.slot >= 0 && g.slot < a.slots;
        if (a.slots <= 0) return;  // the same for all
        const int64_t slot = g.live ? g.slot : 0;
        const int32_t grp = (int32_t)(((float)oct + 0.5f) * per_group);
        g.scale = a.scales[slot * a.scales_ld + grp];
        load_raw<false, STREAM>((const uint8_t *)a.q + slot * a.q_ld, oct, cols_of(a.dim), g.w);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(int64_t row, int32_t oct, bool fours, Regs &g) const
    {
        float v[OCT];
        settle(g.w, oct, cols_of(a.dim));
        unpack_oct<KIND>(g.w.w, v);
#pragma unroll
        for (int k = 0; k < OCT; ++k) v[k] = g.live ? v[k] * g.scale : 0.f;
        put_row_oct<STREAM>((T *)a.x + row * a.x_ld, oct, a.dim, fours, v);
    }
};

hipError_t run_cache_read(const CacheArgs &a, hipStream_t s)
{
    return with_index(a.index_type, [&](auto ix) {
        return with_type(a.type, [&](auto t) {
            using IX = decltype(ix);
            using T = decltype(t);
            const float per = a.group == a.dim ? 0.f : (float)OCT / (float)a.group;
            return a.kind == KIND_INT
                       ? run_octets(CacheRead<T, IX, KIND_INT>{a, per}, a.n, a.dim, s)
                       : run_octets(CacheRead<T, IX, KIND_FLOAT>{a, per}, a.n, a.dim, s);
        });
    });
}

}  // namespace sp
