// Rows in 4 bits: a cache that is quantised as it is written, and read back.
//
// Blocks of 32 columns share a scale, a power of two 2^(b - 127) held as the byte b.  A value
// is 4 bits, a sign and a magnitude of 0, .5, 1, 1.5, 2, 3, 4 or 6 (the OCP Microscaling
// formats' MXFP4), two to a byte, the even column low.  The scale puts the block's largest
// magnitude between 4 and 8, b = its fp32 exponent - 2: no product, no reciprocal, and every step
// but the one rounding to 4 bits is exact.  A row is whole blocks, zeros behind its last column.
#include "sp_rows.h"

namespace sp {

typedef float float_2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16_2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16_2 __attribute__((ext_vector_type(2)));

constexpr uint32_t NAN_SCALE = 255;

// An octet over the scale in 4 bits, to the nearest, ties to even codes, past 6 to 6.
template <typename T>
__device__ __forceinline__ uint32_t pack4(const Raw<T> &r, float scale)
{
    uint32_t w = 0;
    const auto pair = [&](int k, auto sel) {
        constexpr int S = decltype(sel)::value;
        if constexpr (sizeof(T) == 4) {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(r.w[2 * k]), __uint_as_float(r.w[2 * k + 1]),
                                                         scale, S);
        } else if constexpr (std::is_same<T, __bf16>::value) {
            bf16_2 h;
            __builtin_memcpy(&h, &r.w[k], 4);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, h, scale, S);
        } else {
            f16_2 h;
            __builtin_memcpy(&h, &r.w[k], 4);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, h, scale, S);
        }
    };
    pair(0, std::integral_constant<int, 0>());
    pair(1, std::integral_constant<int, 1>());
    pair(2, std::integral_constant<int, 2>());
    pair(3, std::integral_constant<int, 3>());
    return w;
}

__device__ __forceinline__ void unpack4(uint32_t w, float scale, float (&v)[OCT])
{
    const float_2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
    const float_2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const float_2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
    const float_2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}

// ---------------------------------------------------------------- write
//
// Four lanes hold a block, an octet each, and exchange their largest magnitudes; the grid's
// rows are as wide as whole blocks, so octets past the last column have lanes too.  Bound by the
// bytes: 65536 rows of 1024 bf16 into random slots 33 us (5.2 TB/s), of 1001 fp32 58.  fp32 takes an
// octet per thread at any size (four: 63).
template <typename T, typename IX>
struct Cache4Write {
    static constexpr bool DEEP = sizeof(T) < 4;
    bool deep_pays() const { return a.dim >= OCT; }
    Cache4Args a;
    struct Regs {
        Raw<T> r;
        int64_t slot;
    };
    __device__ __forceinline__ void first(int64_t row, Regs &g) const
    {
        g.slot = a.index ? (int64_t)((const IX *)a.index)[row] : row;
    }
    template <bool STREAM>
    __device__ __forceinline__ void load(int64_t row, int32_t oct, Regs &g) const
    {
        load_raw<STREAM, STREAM>((const T *)a.x + row * a.x_ld, oct, cols_of(a.dim), g.r);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(int64_t, int32_t oct, bool, Regs &g) const
    {
        if (g.slot < 0 || g.slot >= a.slots) return;  // whole blocks
        settle(g.r, oct, cols_of(a.dim));
        const int valid = oct_valid(a.dim, oct);
        if (valid < OCT) {
            const int bits = valid > 0 ? valid * (int)sizeof(T) * 8 : 0;
#pragma unroll
            for (int i = 0; i < Raw<T>::WORDS; ++i) {
                const int left = bits - 32 * i;
                g.r.w[i] &= left >= 32 ? ~0u : left <= 0 ? 0u : (1u << left) - 1;
            }
        }
        const uint32_t top = float_bits<T>(team_max<4>(top_of(g.r, OCT)));
        const uint32_t e = top >> 23, b = e == 255 ? NAN_SCALE : e > 2 ? e - 2 : 0;
        const uint32_t w = e == 255 ? 0u : pack4(g.r, __uint_as_float(b << 23));
        __builtin_memcpy(a.q + g.slot * a.q_ld + oct * 4, &w, 4);
        if ((oct & 3) == 0) a.scales[g.slot * a.scales_ld + oct / 4] = (uint8_t)b;
    }
};

hipError_t run_cache4_write(const Cache4Args &a, hipStream_t s)
{
    return with_index(a.index_type, [&](auto ix) {
        return with_type(a.type, [&](auto t) {
            return run_octets(Cache4Write<decltype(t), decltype(ix)>{a}, a.n, (a.dim + 31) / 32 * 32, s);
        });
    });
}

// ---------------------------------------------------------------- read

// x[i] = the values of slot index[i]; zeros where index[i] is no slot.  Bound by the bytes: 65536 random
// rows of 1024 into bf16 27 us (6.2 TB/s).
template <typename T, typename IX>
struct Cache4Read {
    static constexpr bool DEEP = true;
    bool deep_pays() const { return whole_pieces((const T *)a.x, a.x_ld); }
    Cache4Args a;
    struct Regs {
        uint32_t w, scale;
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
        g.scale = a.scales[slot * a.scales_ld + oct / 4];
        __builtin_memcpy(&g.w, a.q + slot * a.q_ld + oct * 4, 4);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(int64_t row, int32_t oct, bool fours, Regs &g) const
    {
        float v[OCT];
        if (!g.live) g.w = g.scale = 0;
        unpack4(g.w, __uint_as_float(g.scale << 23), v);
        put_row_oct<STREAM>((T *)a.x + row * a.x_ld, oct, a.dim, fours, v);
    }
};

// The same into fp32 rows, four columns a thread and store: by octets every other 16 bytes of a line went
// in a store of their own (65536 random rows of 1024 74 us, so 43).  A thread's columns end where 16
// aligned bytes of the output do, and each four threads' where 64 do, wherever the row starts, which lets stores go past the caches (LEAD:
// columns that its first threads lack): parts of 64 bytes that two waves write past them cost a read each
// (rows of 1001 85 us through the caches, 47 so, and 60 to 71 right behind a write of as many rows).
template <typename IX, bool LEAD>
struct Cache4ReadQuads {
    Cache4Args a;
    struct Regs {
        uint32_t w, low, high;
        int32_t col, shift;
        int64_t slot;
        bool live;
    };
    __device__ __forceinline__ void first(int64_t row, Regs &g) const
    {
        g.slot = a.index ? (int64_t)((const IX *)a.index)[row] : row;
    }
    template <bool STREAM>
    __device__ __forceinline__ void load(int64_t row, int32_t quad, Regs &g) const
    {
        g.live = g.slot >= 0 && g.slot < a.slots;
        g.col = quad * 4 - (LEAD ? (int32_t)((uintptr_t)((const float *)a.x + row * a.x_ld) / 4 % 16) : 0);
        if (a.slots <= 0) return;  // the same for all
        const int64_t slot = g.live ? g.slot : 0;
        const int32_t blocks = (a.dim + 31) / 32, last = blocks * 16 - 4, from = g.col >> 1;
        const int32_t byte = from < 0 ? 0 : from > last ? last : from;
        __builtin_memcpy(&g.w, a.q + slot * a.q_ld + byte, 4);
        g.shift = 4 * (g.col - 2 * byte);
        const auto block = [&](int32_t col) { return col < 0 ? 0 : col / 32 < blocks ? col / 32 : blocks - 1; };
        g.low = a.scales[slot * a.scales_ld + block(g.col)];
        g.high = LEAD ? a.scales[slot * a.scales_ld + block(g.col + 3)] : g.low;
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(int64_t row, int32_t, bool, Regs &g) const
    {
        const auto factor = [](uint32_t b) { return __uint_as_float(b == NAN_SCALE ? 0x7FC00000u : b ? b << 23 : 0x00400000u); };
        const float low = g.live ? factor(g.low) : 0.f, high = g.live ? factor(g.high) : 0.f;
        float v[OCT];
        unpack4(!g.live ? 0u : g.shift < 0 ? g.w << (-g.shift & 31) : g.w >> (g.shift & 31), 1.f, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] *= (g.col + k) >> 5 == g.col >> 5 ? low : high;
        float *p = (float *)a.x + row * a.x_ld + g.col;
        if (g.col >= 0 && g.col + 4 <= a.dim) {
            put_bytes<true, 16>(p, v);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (g.col + k >= 0 && g.col + k < a.dim) p[k] = v[k];
        }
    }
};
template <typename IX, bool LEAD>
static hipError_t read_quads(const Cache4Args &a, hipStream_t st)
{
    constexpr int QUADS = 4;  // of a thread
    const int64_t width = LEAD ? (a.dim + 15 + 15) / 16 * 4 : (a.dim + 3) / 4;
    return launch_split(split_rows(a.n, width, QUADS * BLOCK), [&](const Split &s, dim3 grid) {
        return launch(k_octets<Cache4ReadQuads<IX, LEAD>, QUADS>, grid, dim3(BLOCK), st, Cache4ReadQuads<IX, LEAD>{a}, s);
    });
}

hipError_t run_cache4_read(const Cache4Args &a, hipStream_t s)
{
    return with_index(a.index_type, [&](auto ix) {
        return with_type(a.type, [&](auto t) {
            const int64_t octets = a.n * ((a.dim + OCT - 1) / OCT);
            if (sizeof(t) == 4 && octets >= OCTETS_DEEP)
                return ((uintptr_t)a.x | (uint64_t)a.x_ld * 4) % 64 == 0 ? read_quads<decltype(ix), false>(a, s) : read_quads<decltype(ix), true>(a, s);
            return run_octets(Cache4Read<decltype(t), decltype(ix)>{a}, a.n, a.dim, s);
        });
    });
}

}  // namespace sp
