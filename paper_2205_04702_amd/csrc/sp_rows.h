// Shared pieces of the operators on token tables and 8-bit rows: element types,
// eight-column accesses, the dropout generator, the split of rows over a grid.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sp_device.h"

namespace sp {

// ---------------------------------------------------------------- launches

// A launch whose status is its own: hipGetLastError would also report what an
// earlier call of the caller's program left behind.
template <typename... P, typename... A>
inline hipError_t launch(void (*k)(P...), dim3 grid, dim3 block, hipStream_t s, A... a)
{
    static_assert(sizeof...(P) == sizeof...(A), "one value per kernel argument");
    return [&](P... p) {
        void *args[] = {(void *)&p...};
        const hipError_t e =
            hipLaunchKernel(reinterpret_cast<const void *>(k), grid, block, args, 0, s);
        if (e != hipSuccess) (void)hipGetLastError();
        return e;
    }(static_cast<P>(a)...);
}

// ---------------------------------------------------------------- octets
//
// Rows are worked on in octets, eight columns of one row.  gfx950 takes global
// accesses of 16 bytes at any byte address, so an octet of 16-bit values is one
// access whatever the row's stride and width; only the last octet of a row
// whose width is no multiple of 8 goes value by value.

constexpr int OCT = 8;

template <typename T, int N>
struct Pack {
    T v[N];
};

template <typename T>
__device__ __forceinline__ float to_float(T x) { return (float)x; }
template <typename T>
__device__ __forceinline__ T from_float(float x) { return (T)x; }  // to nearest, ties to even

template <typename T>
__device__ __forceinline__ void load_oct(const T *p, int valid, float (&v)[OCT])
{
    if (valid >= OCT) {
        Pack<T, OCT> w;
        __builtin_memcpy(&w, p, sizeof w);
#pragma unroll
        for (int k = 0; k < OCT; ++k) v[k] = to_float(w.v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < OCT; ++k) v[k] = k < valid ? to_float(p[k]) : 0.f;
    }
}

template <typename T>
__device__ __forceinline__ void store_oct(T *p, int valid, const float (&v)[OCT])
{
    if (valid >= OCT) {
        Pack<T, OCT> w;
#pragma unroll
        for (int k = 0; k < OCT; ++k) w.v[k] = from_float<T>(v[k]);
        __builtin_memcpy(p, &w, sizeof w);
    } else {
#pragma unroll
        for (int k = 0; k < OCT; ++k)
            if (k < valid) p[k] = from_float<T>(v[k]);
    }
}

// ---------------------------------------------------------------- dropout
//
// Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011).  Counter (octet, row, offset low, offset
// high), key the seed; the four words are 16 bits for each of the octet's eight
// columns.  A column is kept where its bits are at least `drop` = 65536 p
// rounded, and what is kept is multiplied by 65536 / (65536 - drop), so the
// expectation is exact for the probability that 16 bits hold.  16 bits a column
// and not 32: ten rounds cost 20 multiplies of 32x32 bits at a quarter of the
// full rate, which for four columns would take as long as moving their bytes.
struct Drop {
    uint32_t k0, k1, o0, o1, drop;  // drop 0: keep everything
};

__device__ __forceinline__ uint32_t keep_oct(const Drop &d, uint32_t oct, uint32_t row)
{
    uint32_t a = oct, b = row, c = d.o0, e = d.o1, k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t x = (uint64_t)a * 0xD2511F53u, y = (uint64_t)c * 0xCD9E8D57u;
        a = (uint32_t)(y >> 32) ^ b ^ k0;
        b = (uint32_t)y;
        c = (uint32_t)(x >> 32) ^ e ^ k1;
        e = (uint32_t)x;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    uint32_t keep = 0;
    const uint32_t w[4] = {a, b, c, e};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        keep |= (uint32_t)((w[i] & 0xFFFFu) >= d.drop) << (2 * i);
        keep |= (uint32_t)((w[i] >> 16) >= d.drop) << (2 * i + 1);
    }
    return keep;
}

// ---------------------------------------------------------------- rows over a grid
//
// A block of 256 threads takes `units` consecutive units (octets, or groups of
// columns): whole rows where a row has fewer units than that, else a stretch of
// one row.  The place of a unit in its block is found in 32 bits (the division
// by multiplication is exact: unit <= 2^13 and width * row <= unit), the block's
// first row in 64.
struct Split {
    int64_t n;        // rows
    int32_t width;    // units per row
    int32_t span;     // units of one row that a block takes
    int32_t rows;     // rows that a block takes (1 where span < width)
    int32_t stretches;  // blocks per row of blocks
    float inv;        // 1 / span
};

inline Split split_rows(int64_t n, int64_t width, int units)
{
    Split s;
    s.n = n;
    s.width = (int32_t)width;
    s.span = (int32_t)(width < units ? width : units);
    s.rows = units / s.span;
    if (s.rows > n) s.rows = n > 0 ? (int32_t)n : 1;
    s.stretches = (int32_t)((width + s.span - 1) / s.span);
    s.inv = 1.0f / (float)s.span;
    return s;
}
inline int64_t split_blocks(const Split &s) { return (s.n + s.rows - 1) / s.rows * s.stretches; }

// Unit u of block b: its row and its place in the row; false where there is none.
__device__ __forceinline__ bool split_at(const Split &s, int64_t b, int u, int64_t &row,
                                         int32_t &at)
{
    int64_t rb = b;
    int32_t st = 0;
    if (s.stretches > 1) {
        rb = b / s.stretches;
        st = (int32_t)(b - rb * s.stretches);
    }
    const int r = (int)(((float)u + 0.5f) * s.inv);
    at = st * s.span + (u - r * s.span);
    row = rb * s.rows + r;
    return r < s.rows && row < s.n && at < s.width;
}

// Every octet of a split through op: the loads of a thread's U octets first.
template <class Op, int U>
__global__ void __launch_bounds__(BLOCK) k_octets(Op op, Split s)
{
    typename Op::Regs g[U];
    int64_t row[U];
    int32_t at[U];
    bool on[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
        on[k] = split_at(s, blockIdx.x, k * BLOCK + (int)threadIdx.x, row[k], at[k]);
        if (on[k]) op.load(row[k], at[k], g[k]);
    }
#pragma unroll
    for (int k = 0; k < U; ++k)
        if (on[k]) op.store(row[k], at[k], g[k]);
}

// With fewer octets than fill the card four times over, one octet per thread.
constexpr int64_t OCTETS_FILL = 4ll * 256 * 2048;
template <class Op>
inline hipError_t run_octets(const Op &op, int64_t n, int64_t dim, hipStream_t st)
{
    const int64_t width = (dim + OCT - 1) / OCT;
    const bool deep = n * width >= OCTETS_FILL;
    const Split s = split_rows(n, width, deep ? 4 * BLOCK : BLOCK);
    const int64_t blocks = split_blocks(s);
    if (blocks <= 0) return hipSuccess;
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    return deep ? launch(k_octets<Op, 4>, dim3((unsigned)blocks), dim3(BLOCK), st, op, s)
                : launch(k_octets<Op, 1>, dim3((unsigned)blocks), dim3(BLOCK), st, op, s);
}

__device__ __forceinline__ int oct_valid(int32_t dim, int32_t oct)
{
    const int v = dim - oct * OCT;
    return v < OCT ? v : OCT;
}

// ---------------------------------------------------------------- element types

// f(value of the type) for the floating types of the C interface.
template <class F>
inline hipError_t with_type(int32_t type, F f)
{
    switch (type) {
    case 0: return f(float());
    case 1: return f(__bf16());
    default: return f(_Float16());
    }
}
template <class F>
inline hipError_t with_index(int32_t type, F f)
{
    return type == 3 ? f(int32_t()) : f(int64_t());
}

// ---------------------------------------------------------------- host entry of each operator

struct LookupArgs {
    const void *tokens;
    int32_t token_type;
    int64_t n;
    const void *table;
    int32_t table_type;
    int64_t rows, table_ld;
    int32_t dim;
    float factor;
    Drop drop;
    void *out;
    int32_t out_type;
    int64_t out_ld;
};
hipError_t run_lookup(const LookupArgs &a, hipStream_t s);

struct DropoutArgs {
    const void *x, *residual;
    int32_t type;
    int64_t n;
    int32_t dim;
    int64_t x_ld, residual_ld;
    float factor;
    Drop drop;
    void *out;
    int64_t out_ld;
};
hipError_t run_dropout(const DropoutArgs &a, hipStream_t s);

struct GradArgs {
    const void *tokens;
    int32_t token_type;
    int64_t n;
    const void *grad;
    int32_t grad_type;
    int64_t grad_ld;
    int32_t dim;
    float factor;
    Drop drop;
    void *out;
    int32_t out_type;
    int64_t rows, out_ld;
    bool add;
    char *ws;
};
int64_t grad_workspace(int64_t n, int64_t rows, int32_t dim);
hipError_t run_grad(const GradArgs &a, hipStream_t s);

struct CacheArgs {
    const void *index;  // null: row i is slot i
    int32_t index_type;
    int64_t n;
    void *q;
    int32_t kind;
    int64_t slots, q_ld;
    float *scales;
    int64_t scales_ld;
    int32_t dim, group;
    void *x;  // the rows written, or read
    int32_t type;
    int64_t x_ld;
};
hipError_t run_cache_write(const CacheArgs &a, hipStream_t s);
hipError_t run_cache_read(const CacheArgs &a, hipStream_t s);

struct ProductArgs {
    const int8_t *x, *w;
    const float *xs, *ws;
    int64_t m, n;
    int32_t k;
    int64_t x_ld, w_ld;
    void *out;
    int32_t out_type;
    int64_t out_ld;
    char *work;
};
int64_t product_workspace(int64_t m, int64_t n, int64_t k);
hipError_t run_product(const ProductArgs &a, hipStream_t s);

}  // namespace sp
