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

// Moves of 16 bytes at any address.  STREAM: past the caches, for what is read or written
// once and is more than they hold; kept in them it would only displace what is read again.
typedef uint32_t word4 __attribute__((ext_vector_type(4)));
typedef uint32_t word4_any __attribute__((ext_vector_type(4), aligned(1)));
template <bool STREAM, int BYTES>
__device__ __forceinline__ void get_bytes(void *to, const void *from)
{
    if constexpr (STREAM && BYTES % 16 == 0) {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const word4 x = __builtin_nontemporal_load((const word4_any *)from + i);
            __builtin_memcpy((char *)to + 16 * i, &x, 16);
        }
    } else {
        __builtin_memcpy(to, from, BYTES);
    }
}
template <bool STREAM, int BYTES>
__device__ __forceinline__ void put_bytes(void *to, const void *from)
{
    if constexpr (STREAM && BYTES % 16 == 0) {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            word4 x;
            __builtin_memcpy(&x, (const char *)from + 16 * i, 16);
            __builtin_nontemporal_store((word4_any)x, (word4_any *)to + i);
        }
    } else {
        __builtin_memcpy(to, from, BYTES);
    }
}

template <typename T>
__device__ __forceinline__ float to_float(T x) { return (float)x; }
template <typename T>
__device__ __forceinline__ T from_float(float x) { return (T)x; }  // to nearest, ties to even

// An octet as it lies in memory.  Loads come without a branch around them, so that those
// of a thread are in flight together, and are turned into numbers when they are
// used: with the conversion beside the load, every load was waited for by itself.
template <typename T>
struct Raw {
    static constexpr int WORDS = (int)sizeof(T) * OCT / 4;
    uint32_t w[WORDS];
};

// The columns of a row, as octets.  The last octet of a row of 8 columns or more is loaded
// as the row's last eight columns and moved down (settle); a narrower row, value by value.
struct Cols {
    int32_t dim;
    int32_t over;  // columns that the last octet lacks, 0 .. 7
};
__device__ __forceinline__ Cols cols_of(int32_t dim) { return Cols{dim, -dim & (OCT - 1)}; }
__device__ __forceinline__ int oct_valid(int32_t dim, int32_t oct)
{
    const int v = dim - oct * OCT;
    return v < OCT ? v : OCT;
}

// WIDE: rows of 8 columns or more only.  (A branch per load, even one that all take alike,
// keeps the loads of a thread from being issued one after the other.)
template <bool STREAM, bool WIDE, typename T>
__device__ __forceinline__ void load_raw(const T *row, int32_t oct, const Cols &c, Raw<T> &r)
{
    if (WIDE || c.dim >= OCT) {
        const int32_t col = oct * OCT, last = c.dim - OCT;
        get_bytes<STREAM, sizeof r.w>(r.w, row + (col < last ? col : last));
    } else {  // last value first, each moving the later ones up (few registers, no speed)
        constexpr int N = Raw<T>::WORDS, UP = (4 - (int)sizeof(T)) & 3;
#pragma unroll
        for (int i = 0; i < N; ++i) r.w[i] = 0;
#pragma unroll 1
        for (int k = c.dim - 1; k >= 0; --k) {
            T x = row[k];
            uint32_t bits = 0;
            __builtin_memcpy(&bits, &x, sizeof x);
#pragma unroll
            for (int i = N - 1; i > 0; --i)
                r.w[i] = UP ? __builtin_amdgcn_alignbyte(r.w[i], r.w[i - 1], UP) : r.w[i - 1];
            r.w[0] = UP ? r.w[0] << (8 * (4 - UP)) | bits : bits;
        }
    }
}

// What was loaded for octet `oct`, its first columns first (beyond the row: anything).
template <typename T>
__device__ __forceinline__ void settle(Raw<T> &r, int32_t oct, const Cols &c)
{
    if (c.over == 0 || c.dim < OCT) return;  // the same for all
    const bool tail = oct * OCT > c.dim - OCT;
    const int bytes = c.over * (int)sizeof(T);
    constexpr int N = Raw<T>::WORDS;
#pragma unroll
    for (int by = 4; by < N * 4; by *= 2) {
        const bool move = tail && (bytes & by);
#pragma unroll
        for (int i = 0; i < N; ++i) r.w[i] = move ? (i + by / 4 < N ? r.w[i + by / 4] : 0u) : r.w[i];
    }
    if (sizeof(T) < 4) {
        const int sh = tail ? (bytes & 3) : 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            r.w[i] = __builtin_amdgcn_alignbyte(i + 1 < N ? r.w[i + 1] : 0u, r.w[i], sh);
    }
}

template <typename T>
__device__ __forceinline__ float raw_float(const Raw<T> &r, int k)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[k]);
    const uint16_t h = (uint16_t)(r.w[k / 2] >> (k % 2 * 16));
    T t;
    __builtin_memcpy(&t, &h, sizeof(T) < 4 ? sizeof t : 0);
    return to_float(t);
}
template <typename T>
__device__ __forceinline__ void raw_floats(const Raw<T> &r, float (&v)[OCT])
{
#pragma unroll
    for (int k = 0; k < OCT; ++k) v[k] = raw_float(r, k);
}

template <bool STREAM, bool WIDE, typename T>
__device__ __forceinline__ void load_oct(const T *row, int32_t oct, const Cols &c, float (&v)[OCT])
{
    Raw<T> r;
    load_raw<STREAM, WIDE>(row, oct, c, r);
    settle(r, oct, c);
    raw_floats(r, v);
}

template <bool STREAM = false, typename T>
__device__ __forceinline__ void store_oct(T *p, int valid, const float (&v)[OCT])
{
    if (valid >= OCT) {
        Pack<T, OCT> w;
#pragma unroll
        for (int k = 0; k < OCT; ++k) w.v[k] = from_float<T>(v[k]);
        put_bytes<STREAM, sizeof w>(p, &w);
    } else {
#pragma unroll
        for (int k = 0; k < OCT; ++k)
            if (k < valid) p[k] = from_float<T>(v[k]);
    }
}

// The value that lane CTRL's two bits for this lane name, among each four lanes.
template <int CTRL>
__device__ __forceinline__ float of_four(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}

// Stores octet `oct` of a row of dim columns.  fours: each four lanes (4i .. 4i + 3) that get
// here hold the octets 4j .. 4j + 3 of one row as far as it has them.  An octet of fp32
// is two 16-byte stores; the four lanes first exchange halves, so that each of the
// stores covers 64 consecutive bytes of four lanes and not every other 16.
template <bool STREAM = false, typename T>
__device__ __forceinline__ void put_row_oct(T *row, int32_t oct, int32_t dim, bool fours,
                                            const float (&v)[OCT])
{
    if constexpr (sizeof(T) == 4) {
        if (fours && (oct | 3) * OCT + OCT <= dim) {
            const bool odd = threadIdx.x & 1;
            Pack<T, 4> a, b;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float a0 = of_four<0x50>(v[k]), a1 = of_four<0x50>(v[4 + k]);  // lanes 0 0 1 1
                const float b0 = of_four<0xFA>(v[k]), b1 = of_four<0xFA>(v[4 + k]);  // lanes 2 2 3 3
                a.v[k] = odd ? a1 : a0;
                b.v[k] = odd ? b1 : b0;
            }
            T *p = row + (int64_t)(oct & ~3) * OCT + (threadIdx.x & 3) * 4;
            put_bytes<STREAM, sizeof a>(p, &a);
            put_bytes<STREAM, sizeof b>(p + 16, &b);
            return;
        }
    }
    const int left = dim - oct * OCT;
    store_oct<STREAM>(row + (int64_t)oct * OCT, left < OCT ? left : OCT, v);
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

struct Kept {
    uint32_t w[4];
    // whether column k (0 .. 7) of the octet is kept: the high halves compare as they lie
    __device__ __forceinline__ bool operator()(const Drop &d, int k) const
    {
        return (k & 1 ? w[k / 2] : w[k / 2] << 16) >= d.drop << 16;
    }
};

__device__ __forceinline__ uint32_t xor3(uint32_t x, uint32_t y, uint32_t z)
{
    return (uint32_t)__builtin_amdgcn_bitop3_b32((int)x, (int)y, (int)z, 0x96);
}

__device__ __forceinline__ Kept keep_oct(const Drop &d, uint32_t oct, uint32_t row)
{
    uint32_t a = oct, b = row, c = d.o0, e = d.o1, k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t x = (uint64_t)a * 0xD2511F53u, y = (uint64_t)c * 0xCD9E8D57u;
        a = xor3((uint32_t)(y >> 32), b, k0);
        b = (uint32_t)y;
        c = xor3((uint32_t)(x >> 32), e, k1);
        e = (uint32_t)x;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Kept{{a, b, c, e}};
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
    int64_t row0;     // the launch's first row
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
    s.row0 = 0;
    s.width = (int32_t)width;
    s.span = (int32_t)(width < units ? width : units);
    s.rows = units / s.span;
    if (s.rows > n) s.rows = n > 0 ? (int32_t)n : 1;
    s.stretches = (int32_t)((width + s.span - 1) / s.span);
    s.inv = 1.0f / (float)s.span;
    return s;
}
inline int64_t split_blocks(const Split &s) { return (s.n + s.rows - 1) / s.rows * s.stretches; }

// A launch has fewer than 2^32 threads along an axis.  go(split, blocks) launches one piece of
// a split, whole rows of blocks, of at most 2^23 blocks (of up to 511 threads).
constexpr int64_t LAUNCH_BLOCKS = 1 << 23;
template <class F>
inline hipError_t launch_split(Split s, F go)
{
    const int64_t row_blocks = (s.n + s.rows - 1) / s.rows, each = LAUNCH_BLOCKS / s.stretches;
    for (int64_t b = 0; b < row_blocks; b += each) {
        const int64_t k = row_blocks - b < each ? row_blocks - b : each;
        s.row0 = b * s.rows;
        const hipError_t e = go(s, dim3((unsigned)(k * s.stretches)));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

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
    row = s.row0 + rb * s.rows + r;
    return r < s.rows && row < s.n && at < s.width;
}

// Every octet of a split through op: the loads of a thread's U octets first (those of
// units that are none take the place of the block's first).
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
        if (!on[k]) split_at(s, blockIdx.x, 0, row[k], at[k]);
        op.first(row[k], g[k]);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) op.template load<(U > 1)>(row[k], at[k], g[k]);
#pragma unroll
    for (int k = 0; k < U; ++k)
        if (on[k]) op.template store<(U > 1)>(row[k], at[k], s.span % 4 == 0, g[k]);
}

// Four octets per thread, outputs (and inputs that are read once) past the caches, where
// there are octets for that and the operator allows it (DEEP) and says that it pays.  Below,
// one octet per thread, and the outputs stay near for the next kernel.  Deep and not (us,
// inputs past the caches, rows of 1024 bf16 columns): 2^19 octets lookup 4.4 and 5.5, dropout
// with a residual 6.9 and 6.8, cache read 4.6 and 4.8; 2^20 6.8 and 9.5, 11.5 and 12.0, 6.3 and
// 8.6; 2^22 21.8 and 27.0, 35.2 and 37.0, 15.6 and 23.5.  A lookup and two dropouts of what it
// gave, one after the other: 2^19 15.0 and 14.7, 2^20 22.0 and 23.1, 2^22 72 and 70.
constexpr int64_t OCTETS_DEEP = 1 << 20;
template <class Op>
inline hipError_t run_octets(const Op &op, int64_t n, int64_t dim, hipStream_t st)
{
    const int64_t width = (dim + OCT - 1) / OCT;
    if constexpr (Op::DEEP) {
        if (n * width >= OCTETS_DEEP && dim >= OCT && op.deep_pays())
            return launch_split(split_rows(n, width, 4 * BLOCK), [&](const Split &s, dim3 grid) {
                return launch(k_octets<Op, 4>, grid, dim3(BLOCK), st, op, s);
            });
    }
    return launch_split(split_rows(n, width, BLOCK), [&](const Split &s, dim3 grid) {
        return launch(k_octets<Op, 1>, grid, dim3(BLOCK), st, op, s);
    });
}

// For rows that are looked up deep pays but where they are fp32 and share 32-byte pieces, which
// past the caches are written in parts (us, deep and not, 2^22 octets: cached rows read into
// fp32 of 250 columns 55 and 41, 1001 60 and 47, 2048 34 and 40, 24 32 and 49; bf16 rows looked
// up into the same 55 and 43, 53 and 52, 44 and 41, 38 and 47).
template <typename TO>
inline bool whole_pieces(const TO *out, int64_t ld)
{
    return sizeof(TO) < 4 || ((uintptr_t)out | (uint64_t)ld * sizeof(TO)) % 32 == 0;
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
