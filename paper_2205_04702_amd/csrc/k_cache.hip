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

// An octet times `inverse` in bytes.  Integers: 1.5 * 2^23 added to a magnitude of at most
// 127 leaves it, rounded to the nearest integer (ties to even), in the low byte.  The
// product is rounded before that, as everywhere (no fused multiply-add).  inverse is
// 1 / (amax * (1 / top)), three roundings: nothing gets past top + 1/4.
template <int KIND>
__device__ __forceinline__ uint2 pack_oct(const float (&v)[OCT], float inverse)
{
#pragma clang fp contract(off)
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = v[4 * h + k] * inverse;
        if constexpr (KIND == KIND_INT) {
            uint32_t b[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) b[k] = __float_as_uint(y[k] + 12582912.f);
            // the low bytes of two words into the low half of one, then the halves together
            const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400);
            const uint32_t hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0c);
            w[h] = lo | hi;
        } else {
            const int x = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], x, true);
        }
    }
    return make_uint2(w[0], w[1]);
}

typedef float float_2 __attribute__((ext_vector_type(2)));
template <int KIND>
__device__ __forceinline__ void unpack_oct(const uint32_t (&x)[2], float (&v)[OCT])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (KIND == KIND_INT) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[4 * h + k] = (float)(int8_t)(x[h] >> (8 * k));
        } else {
            const float_2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[h], false);
            const float_2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[h], true);
            v[4 * h] = lo.x;
            v[4 * h + 1] = lo.y;
            v[4 * h + 2] = hi.x;
            v[4 * h + 3] = hi.y;
        }
    }
}

// The largest magnitude's bits in an octet as loaded, of its first `valid` columns: for
// 16-bit types the larger of two at a time, in the high or low half.
typedef uint16_t half_2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ uint32_t top_of(const Raw<T> &r, int valid)
{
    uint32_t m = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < OCT; ++k) {
            const uint32_t b = r.w[k] & 0x7FFFFFFFu;
            m = k < valid && b > m ? b : m;
        }
    } else {
        half_2 t = {0, 0};
#pragma unroll
        for (int i = 0; i < OCT / 2; ++i) {
            const int left = valid - 2 * i;
            uint32_t b = r.w[i] & (left >= 2 ? 0x7FFF7FFFu : left == 1 ? 0x7FFFu : 0u);
            half_2 h;
            __builtin_memcpy(&h, &b, 4);
            t = __builtin_elementwise_max(t, h);
        }
        m = t.x > t.y ? t.x : t.y;
    }
    return m;
}
// ... as the bits of a float.
template <typename T>
__device__ __forceinline__ uint32_t float_bits(uint32_t m)
{
    if constexpr (sizeof(T) == 4) return m;
    Raw<T> r;
    r.w[0] = m;
    return __float_as_uint(raw_float(r, 0));
}

// The maximum over each TEAM lanes, in all of them: exchanges inside rows of 16 lanes, then
// between them.
template <int TEAM>
__device__ __forceinline__ uint32_t team_max(uint32_t m)
{
    const auto with = [&](uint32_t o) { m = o > m ? o : m; };
    if constexpr (TEAM >= 2) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    if constexpr (TEAM >= 4) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));   // lane ^ 2
    if constexpr (TEAM >= 8) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));  // the other four of eight
    if constexpr (TEAM >= 16) with((uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xF, 0xF, true)); // the other eight
    if constexpr (TEAM >= 32) with((uint32_t)__shfl_xor((int)m, 16, WAVE));
    if constexpr (TEAM >= 64) with((uint32_t)__shfl_xor((int)m, 32, WAVE));
    return m;
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
// A team of TEAM lanes holds one group, OPL octets in each lane (team-strided, so
// neighbouring lanes read neighbouring bytes), or walks over it a second time where it
// does not fit into registers (LOOP); and U groups one after the other, whose rows and slots
// are all loaded first (with one group per team and its slot before its row, 65536 rows
// of 1024 were written at 3.9 TB/s).  The maximum is taken over the magnitudes' bits: their
// order is that of the values, and infinity and NaN come out above everything.  A group
// that holds one of these gets a NaN scale and zero bytes (it reads back as NaN); one
// whose scale would be subnormal is held as zeros.  65536 rows of 1024 bf16 into random
// slots, a scale per 128, 46 us (4.2 TB/s; 55 while the arithmetic on single values bounded it);
// 8192 rows of 4096 with a scale each 19 us (5.2 TB/s).
template <typename T, typename IX, int KIND, int TEAM, int OPL, int U, bool LOOP>
__global__ void __launch_bounds__(BLOCK) k_cache_write(CacheArgs a, Split s, int32_t octs)
{
    constexpr float top = KIND == KIND_INT ? 127.f : 448.f;
    constexpr bool WIDE = TEAM > 4;
    const int lane = (int)threadIdx.x % TEAM;
    const Cols cols = cols_of(a.group);
    Raw<T> v[U][OPL];
    int64_t slot[U], row[U];
    int32_t grp[U];
    bool on[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        on[u] = split_at(s, blockIdx.x, u * (BLOCK / TEAM) + (int)threadIdx.x / TEAM, row[u], grp[u]);
        if (!on[u]) split_at(s, blockIdx.x, 0, row[u], grp[u]);
        slot[u] = a.index ? (int64_t)((const IX *)a.index)[row[u]] : row[u];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < OPL; ++i) {
            const int32_t o = i * TEAM + lane;
            load_raw<true, WIDE>((const T *)a.x + row[u] * a.x_ld + grp[u] * a.group, o < octs ? o : 0,
                                 cols, v[u][i]);
        }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        on[u] = on[u] && slot[u] >= 0 && slot[u] < a.slots;
        if (!on[u]) continue;  // whole teams
        const T *x = (const T *)a.x + row[u] * a.x_ld + grp[u] * a.group;
        uint8_t *q = (uint8_t *)a.q + slot[u] * a.q_ld + grp[u] * a.group;
        uint32_t top_bits = 0;
        for (int32_t o0 = 0; o0 < (LOOP ? octs : 1); o0 += TEAM * OPL) {
#pragma unroll
            for (int i = 0; i < OPL; ++i) {
                const int32_t o = o0 + i * TEAM + lane;
                if (o >= octs) continue;
                if (LOOP && o0 > 0) load_raw<true, WIDE>(x, o, cols, v[u][i]);
                settle(v[u][i], o, cols);
                const uint32_t b = top_of(v[u][i], cols.over ? oct_valid(a.group, o) : OCT);
                top_bits = b > top_bits ? b : top_bits;
            }
        }
        top_bits = float_bits<T>(team_max<TEAM>(top_bits));
        const bool finite = top_bits < INF_BITS;
        float scale = __uint_as_float(top_bits) * (1.f / top);
        if (!(scale >= SMALLEST_SCALE)) scale = 0.f;
        const float inverse = finite && scale > 0.f ? 1.f / scale : 0.f;
        if (!finite) scale = __uint_as_float(0x7FC00000u);
        if (lane == 0) a.scales[slot[u] * a.scales_ld + grp[u]] = scale;
        for (int32_t o0 = 0; o0 < (LOOP ? octs : 1); o0 += TEAM * OPL) {
#pragma unroll
            for (int i = 0; i < OPL; ++i) {
                const int32_t o = o0 + i * TEAM + lane;
                if (o >= octs) continue;
                if (LOOP) {
                    load_raw<false, WIDE>(x, o, cols, v[u][i]);
                    settle(v[u][i], o, cols);
                }
                float f[OCT];
                raw_floats(v[u][i], f);
                uint2 w = pack_oct<KIND>(f, inverse);
                if (!finite) w = make_uint2(0, 0);
                store_bytes(q + o * OCT, oct_valid(a.group, o), w);
            }
        }
    }
}

// Four groups per team where that leaves blocks enough for the card, one otherwise: with 512
// blocks of four 6.6 us and 5.5 with one each (4096 rows of 1024 bf16, a scale per 128, random
// slots), with 1024 9.0 either way, 2048 13.5 and 15.1, 16384 78 and 93; groups of 64, 256 and 512
// the same within 3 %.
template <typename T, typename IX, int KIND>
static hipError_t write_teams(const CacheArgs &a, hipStream_t st)
{
    const int32_t octs = (a.group + OCT - 1) / OCT, groups = a.dim / a.group;
    const auto go = [&](auto kern, int units) {
        return launch_split(split_rows(a.n, groups, units), [&](const Split &s, dim3 grid) {
            return launch(kern, grid, dim3(BLOCK), st, a, s, octs);
        });
    };
    const auto one = [&](auto few, auto many, int team) {
        const int teams = BLOCK / team;
        return a.n * groups >= 4ll * teams * 2048 ? go(many, 4 * teams) : go(few, teams);
    };
    if (octs <= 4) return go(k_cache_write<T, IX, KIND, 4, 1, 1, false>, BLOCK / 4);
    if (octs <= 8) return one(k_cache_write<T, IX, KIND, 8, 1, 1, false>, k_cache_write<T, IX, KIND, 8, 1, 4, false>, 8);
    if (octs <= 16) return one(k_cache_write<T, IX, KIND, 16, 1, 1, false>, k_cache_write<T, IX, KIND, 16, 1, 4, false>, 16);
    if (octs <= 32) return one(k_cache_write<T, IX, KIND, 32, 1, 1, false>, k_cache_write<T, IX, KIND, 32, 1, 4, false>, 32);
    if (octs <= 64) return one(k_cache_write<T, IX, KIND, 64, 1, 1, false>, k_cache_write<T, IX, KIND, 64, 1, 4, false>, 64);
    if (octs <= 128) return go(k_cache_write<T, IX, KIND, 64, 2, 1, false>, BLOCK / 64);
    if (octs <= 256) return go(k_cache_write<T, IX, KIND, 64, 4, 1, false>, BLOCK / 64);
    if (octs <= 512) return go(k_cache_write<T, IX, KIND, 64, 8, 1, false>, BLOCK / 64);
    return go(k_cache_write<T, IX, KIND, 64, 8, 1, true>, BLOCK / 64);
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
// is no slot.  A lookup whose rows are bytes; bound by the bytes: 65536 random rows of 1024
// into bf16 39 us (5.2 TB/s).
template <typename T, typename IX, int KIND>
struct CacheRead {
    static constexpr bool DEEP = true;
    bool deep_pays() const { return whole_pieces((const T *)a.x, a.x_ld); }
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
        if (!g.live) g.w.w[0] = g.w.w[1] = 0, g.scale = 0.f;
        unpack_oct<KIND>(g.w.w, v);
#pragma unroll
        for (int k = 0; k < OCT; ++k) v[k] *= g.scale;
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
