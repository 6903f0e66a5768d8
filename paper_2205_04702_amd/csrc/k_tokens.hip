// Token tables: lookup with scaling and dropout, and dropout by itself.
#include "sp_rows.h"

namespace sp {

// ---------------------------------------------------------------- lookup
//
// out[i] = factor * keep(i) * table[token[i]], rows of zeros where the token is
// no row of the table (padding).  A thread has its octet of one row: its token, then its
// columns, of four rows at a time where there are many.  Bound by the bytes: 16384 rows of
// 2048 in bf16 with dropout 20 us (67 MB written, 27 MB of distinct rows read; 17.5 a call with
// the rows in the caches from the call before, 23.6 with other tables in between; 131072 random
// rows of 2048 without 245 us, 4.4 TB/s).  Outputs go past the caches there, the table does not:
// tokens repeat.
template <typename TI, typename TO, typename IX, bool DROP>
struct Lookup {
    static constexpr bool DEEP = true;
    bool deep_pays() const { return whole_pieces(out, out_ld); }
    const IX *tokens;
    const TI *table;
    TO *out;
    int64_t rows, table_ld, out_ld;
    int32_t dim;
    float factor;
    Drop drop;
    struct Regs {
        Raw<TI> r;
        int64_t t;
        bool live;
    };
    __device__ __forceinline__ void first(int64_t row, Regs &g) const { g.t = (int64_t)tokens[row]; }
    template <bool STREAM>
    __device__ __forceinline__ void load(int64_t, int32_t oct, Regs &g) const
    {
        g.live = g.t >= 0 && g.t < rows;
        if (rows > 0) load_raw<false, STREAM>(table + (g.live ? g.t : 0) * table_ld, oct, cols_of(dim), g.r);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(int64_t row, int32_t oct, bool fours, Regs &g) const
    {
        Kept keep;
        if (DROP) keep = keep_oct(drop, (uint32_t)oct, (uint32_t)row);
        float v[OCT];
        settle(g.r, oct, cols_of(dim));
        raw_floats(g.r, v);
#pragma unroll
        for (int k = 0; k < OCT; ++k)
            v[k] = g.live && (!DROP || keep(drop, k)) ? v[k] * factor : 0.f;
        put_row_oct<STREAM>(out + row * out_ld, oct, dim, fours, v);
    }
};

hipError_t run_lookup(const LookupArgs &a, hipStream_t s)
{
    return with_index(a.token_type, [&](auto ix) {
        return with_type(a.table_type, [&](auto ti) {
            return with_type(a.out_type, [&](auto to) {
                using IX = decltype(ix);
                using TI = decltype(ti);
                using TO = decltype(to);
                const auto go = [&](auto op) {
                    op.tokens = (const IX *)a.tokens;
                    op.table = (const TI *)a.table;
                    op.out = (TO *)a.out;
                    op.rows = a.rows;
                    op.table_ld = a.table_ld;
                    op.out_ld = a.out_ld;
                    op.dim = a.dim;
                    op.factor = a.factor;
                    op.drop = a.drop;
                    return run_octets(op, a.n, a.dim, s);
                };
                return a.drop.drop ? go(Lookup<TI, TO, IX, true>{})
                                   : go(Lookup<TI, TO, IX, false>{});
            });
        });
    });
}

// ---------------------------------------------------------------- dropout
//
// out = [residual +] factor * keep * x.  The backward pass is the same call on
// the gradient: the mask is drawn again from seed, offset and place.  Bound by the bytes,
// each moved once: 16384 x 4096 in bf16 with a residual 65 us, 6.2 TB/s past the caches
// (78 us through them).  fp32 takes an octet per thread, near the caches, at any size: 8192 x 4096 49
// us, 54 deep; of 250 columns, 2^22 octets, 54 and 70.
template <typename T, bool RES>
struct Dropout {
    static constexpr bool DEEP = sizeof(T) < 4;
    bool deep_pays() const { return true; }
    const T *x, *residual;
    T *out;
    int64_t x_ld, residual_ld, out_ld;
    int32_t dim;
    float factor;
    Drop drop;
    struct Regs {
        Raw<T> x, r;
    };
    __device__ __forceinline__ void first(int64_t, Regs &) const {}
    template <bool STREAM>
    __device__ __forceinline__ void load(int64_t row, int32_t oct, Regs &g) const
    {
        load_raw<STREAM, STREAM>(x + row * x_ld, oct, cols_of(dim), g.x);
        if (RES) load_raw<STREAM, STREAM>(residual + row * residual_ld, oct, cols_of(dim), g.r);
    }
    template <bool STREAM>
    __device__ __forceinline__ void store(int64_t row, int32_t oct, bool fours, Regs &g) const
    {
        const Kept keep = keep_oct(drop, (uint32_t)oct, (uint32_t)row);
        float v[OCT], r[OCT];
        settle(g.x, oct, cols_of(dim));
        raw_floats(g.x, v);
        if (RES) {
            settle(g.r, oct, cols_of(dim));
            raw_floats(g.r, r);
        }
#pragma unroll
        for (int k = 0; k < OCT; ++k) {
            v[k] = keep(drop, k) ? v[k] * factor : 0.f;
            if (RES) v[k] += r[k];
        }
        put_row_oct<STREAM>(out + row * out_ld, oct, dim, fours, v);
    }
};

hipError_t run_dropout(const DropoutArgs &a, hipStream_t s)
{
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        const auto go = [&](auto op) {
            op.x = (const T *)a.x;
            op.residual = (const T *)a.residual;
            op.out = (T *)a.out;
            op.x_ld = a.x_ld;
            op.residual_ld = a.residual_ld;
            op.out_ld = a.out_ld;
            op.dim = a.dim;
            op.factor = a.factor;
            op.drop = a.drop;
            return run_octets(op, a.n, a.dim, s);
        };
        return a.residual ? go(Dropout<T, true>{}) : go(Dropout<T, false>{});
    });
}

}  // namespace sp
