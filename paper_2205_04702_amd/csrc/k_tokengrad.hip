// Gradient of a token lookup, summed by sorted tokens into a dense table gradient.
//
//   out[r] (+)= factor * sum over the positions i with token r of keep(i) * grad[i]
//
// in ascending order of position within fixed pieces, so a result never depends on the
// order in which blocks run, with fp32 sums rounded once when they are stored.  Rows
// without a token become zeros (or stay, where the sums are added).  Three ways to
// bring a token's positions together, by their number:
//   few (is_direct)    every position's block looks at all tokens itself: one launch
//   up to RANK_MAX     every position counts the entries before its own: its place
//   above              radix sort, stable, of (token, position)
// After the last two, k_grad_sum walks over the sorted entries in equal pieces,
// whatever the lengths of the runs, and k_grad_join adds up runs that were cut.
#include "sp_rows.h"

namespace sp {

constexpr int64_t DIRECT_MAX = 960;
constexpr int64_t DIRECT_BLOCKS = 2048;  // positions times slabs of columns
constexpr int64_t RANK_MAX = 8192;
constexpr int SLAB = WAVE * OCT;  // columns of one wave

// Measured on both sides of the lines (Zipf tokens, one launch or three): 960 tokens of 128
// columns 10 us and 14, of 1024 columns 20 and 23; 800 of 2048 columns 17 either way.
// Counting or sorting, tokens of 128 columns: 8000 counted 24 us, 9000 sorted 30; 16000
// counted 44, sorted 32.
static bool is_direct(int64_t n, int64_t dim)
{
    return n <= DIRECT_MAX && n * ((dim + SLAB - 1) / SLAB) <= DIRECT_BLOCKS;
}

// A sorted entry: token (rows for one that is no row) above its position.
__device__ __forceinline__ uint32_t key_of(uint64_t e) { return (uint32_t)(e >> 32); }

// A value that is the same for a whole wave, held once for it.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <typename IX>
__device__ __forceinline__ uint32_t key_at(const IX *tokens, int64_t i, int64_t rows)
{
    const int64_t t = (int64_t)tokens[i];
    return t >= 0 && t < rows ? (uint32_t)t : (uint32_t)rows;
}

__device__ __forceinline__ void zero_oct(float (&v)[OCT])
{
#pragma unroll
    for (int k = 0; k < OCT; ++k) v[k] = 0.f;
}

// An octet of one position as loaded, added to the sums where it counts and dropout lets
// it through.
template <typename TI>
__device__ __forceinline__ void add_oct(const GradArgs &a, Raw<TI> &r, int64_t pos, int32_t oct,
                                        bool counts, float (&acc)[OCT])
{
    settle(r, oct, cols_of(a.dim));
    if (a.drop.drop) {  // the same for all
        const Kept keep = keep_oct(a.drop, (uint32_t)oct, (uint32_t)pos);
#pragma unroll
        for (int k = 0; k < OCT; ++k) acc[k] += counts && keep(a.drop, k) ? raw_float(r, k) : 0.f;
    } else {
#pragma unroll
        for (int k = 0; k < OCT; ++k) acc[k] += counts ? raw_float(r, k) : 0.f;
    }
}

// A finished sum goes to its row of the table gradient (a team's lanes together).
template <typename TO>
__device__ __forceinline__ void put_oct(const GradArgs &a, int64_t row, int32_t oct,
                                        const float (&v)[OCT])
{
    TO *p = (TO *)a.out + row * a.out_ld;
    float w[OCT];
    if (a.add) {
        load_oct<false, false>(p, oct, cols_of(a.dim), w);
#pragma unroll
        for (int k = 0; k < OCT; ++k) w[k] += a.factor * v[k];
    } else {
#pragma unroll
        for (int k = 0; k < OCT; ++k) w[k] = a.factor * v[k];
    }
    put_row_oct(p, oct, a.dim, true, w);
}

// ---------------------------------------------------------------- few positions

constexpr int FILL_UNITS = 4096;  // 16-byte pieces of rows that one block of a fill looks after
template <typename TO>
constexpr int FILL_COLS = 16 / (int)sizeof(TO);

// Zeros to the pieces of block b's rows that `used` does not name.  Pieces of 16 bytes at
// multiples of 16, so that a wave's store is one aligned stretch (with octets, 32
// bytes of fp32 per lane in two stores, a fill of 1.07 GB ran at 4.3 TB/s).  Where
// rows start elsewhere, their first and last pieces are parts of one.
template <typename TO, int NT>
__device__ __forceinline__ void fill_zeros(const GradArgs &a, const Split &fill, int64_t b,
                                           int64_t row0, const uint8_t *used)
{
    constexpr int C = FILL_COLS<TO>;
    Pack<TO, C> z;
#pragma unroll
    for (int k = 0; k < C; ++k) z.v[k] = from_float<TO>(0.f);
#pragma unroll
    for (int k = 0; k < FILL_UNITS / NT; ++k) {
        int64_t row;
        int32_t at;
        if (!split_at(fill, b, k * NT + (int)threadIdx.x, row, at) || used[row - row0]) continue;
        TO *p = (TO *)a.out + row * a.out_ld;
        const int32_t col = at * C - (int32_t)((uintptr_t)p % 16 / sizeof(TO));
        if (col >= 0 && col + C <= a.dim) {
            __builtin_memcpy(__builtin_assume_aligned(p + col, 16), &z, sizeof z);
        } else {
            for (int q = 0; q < C; ++q)
                if (col + q >= 0 && col + q < a.dim) p[col + q] = z.v[0];
        }
    }
}
template <typename TO>
static int64_t fill_pieces(const GradArgs &a)
{
    constexpr int C = FILL_COLS<TO>;
    const bool aligned = ((uintptr_t)a.out | (uint64_t)a.out_ld * sizeof(TO)) % 16 == 0;
    return ((int64_t)a.dim + C - 1) / C + !aligned;
}

// Block b < sums: one position and slab of columns.  The block's waves look for the
// position's token among all tokens, 64 at a time, each in every eighth group of 64; at
// the token's first position they add up its rows, wave w those of the eight places from
// 8 w on in every group, and the first wave the waves' sums.  The other blocks write zeros to
// their rows without a token.  Bound by latency: 256 tokens of 512 columns into 8192 rows
// (17 MB) 6 us; a token that is all of 960 costs 35 us, its rows being one block's.
constexpr int DIRECT_NT = 512, DIRECT_WAVES = DIRECT_NT / WAVE;
constexpr int DIRECT_GROUPS = (int)(DIRECT_MAX / WAVE);
constexpr int DIRECT_AHEAD = 4;
static_assert(DIRECT_MAX % WAVE == 0 && DIRECT_WAVES == 8 && DIRECT_GROUPS <= WAVE, "whole groups");
template <typename TI, typename TO, typename IX, bool WIDE>
__global__ void __launch_bounds__(DIRECT_NT) k_grad_direct(GradArgs a, int32_t slabs, int64_t sums,
                                                           Split fill)
{
    __shared__ float part[DIRECT_WAVES - 1][SLAB];
    __shared__ uint64_t found[DIRECT_GROUPS];
    __shared__ uint8_t used[FILL_UNITS];
    const IX *tokens = (const IX *)a.tokens;
    const int n = (int)a.n;
    if ((int64_t)blockIdx.x < sums) {
        const int i = (int)(blockIdx.x / slabs), w = scalar(wave_id());
        const int32_t oct = (int32_t)(blockIdx.x % slabs) * WAVE + lane_id();
        const uint32_t key = key_at(tokens, i, a.rows);
        if (key == (uint32_t)a.rows) return;
        bool earlier = false;
#pragma unroll
        for (int g = w; g < DIRECT_GROUPS; g += DIRECT_WAVES) {
            const int p = g * WAVE + lane_id();
            const bool same = p < n && key_at(tokens, p < n ? p : 0, a.rows) == key;
            const uint64_t m = __ballot(same);
            if (lane_id() == 0) found[g] = m;
            earlier = earlier || (same && p < i);
        }
        if (__syncthreads_or(earlier)) return;
        const bool on = oct * OCT < a.dim;
        float acc[OCT];
        zero_oct(acc);
        const uint32_t places =
            lane_id() < DIRECT_GROUPS ? (uint32_t)(found[lane_id()] >> (8 * w)) & 0xFFu : 0u;
        uint64_t groups = __ballot(places != 0);
        uint32_t m = 0;
        int g = 0;
        while (groups || m) {
            Raw<TI> v[DIRECT_AHEAD];
            int p[DIRECT_AHEAD];
            bool any[DIRECT_AHEAD];
#pragma unroll
            for (int k = 0; k < DIRECT_AHEAD; ++k) {
                if (!m && groups) {
                    g = __ffsll((unsigned long long)groups) - 1;
                    m = (uint32_t)__builtin_amdgcn_readlane((int)places, g);
                    groups &= groups - 1;
                }
                any[k] = m != 0;
                p[k] = any[k] ? g * WAVE + w * 8 + __ffs(m) - 1 : i;
                m &= m - 1;
                load_raw<false, WIDE>((const TI *)a.grad + p[k] * a.grad_ld, on ? oct : 0, cols_of(a.dim), v[k]);
            }
#pragma unroll
            for (int k = 0; k < DIRECT_AHEAD; ++k) add_oct(a, v[k], p[k], oct, any[k], acc);
        }
        if (w > 0) {
#pragma unroll
            for (int c = 0; c < OCT; ++c) part[w - 1][c * WAVE + lane_id()] = acc[c];
        }
        __syncthreads();
        if (w == 0 && on) {
#pragma unroll
            for (int v = 0; v < DIRECT_WAVES - 1; ++v)
#pragma unroll
                for (int c = 0; c < OCT; ++c) acc[c] += part[v][c * WAVE + lane_id()];
            put_oct<TO>(a, key, oct, acc);
        }
        return;
    }
    const int64_t b = (int64_t)blockIdx.x - sums;
    const int64_t row0 = b / fill.stretches * fill.rows;
    for (int u = threadIdx.x; u < FILL_UNITS; u += DIRECT_NT) used[u] = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < n; p += DIRECT_NT) {
        const int64_t r = (int64_t)key_at(tokens, p, a.rows) - row0;
        if (r >= 0 && r < fill.rows) used[r] = 1;
    }
    __syncthreads();
    fill_zeros<TO, DIRECT_NT>(a, fill, b, row0, used);
}

// ---------------------------------------------------------------- places by counting

// RANK_POS positions per block; each of its 64 groups of RANK_POS lanes counts, for all of
// them, over a 64th of the keys, four at a time from LDS.  A key before the block's own
// positions counts where it is at most theirs, one after them where it is less; among
// the block's own positions equal keys are counted at the end.  Bound by its compares:
// 5003 tokens 7 us (19 with one position per lane of a whole wave, on a third of the CUs).
constexpr int RANK_NT = 1024;
constexpr int RANK_POS = 16;
constexpr int RANK_PARTS = RANK_NT / RANK_POS;
template <typename IX>
__global__ void __launch_bounds__(RANK_NT) k_grad_rank(const IX *tokens, int32_t n, int64_t rows,
                                                       uint64_t *out)
{
    __shared__ __attribute__((aligned(16))) uint32_t keys[RANK_MAX + RANK_POS];
    __shared__ uint32_t count[RANK_PARTS][RANK_POS];
    const int own = (int)blockIdx.x * RANK_POS;
    const int padded = (n + RANK_POS - 1) / RANK_POS * RANK_POS;
    for (int i = threadIdx.x; i < padded; i += RANK_NT)
        keys[i] = i < n ? key_at(tokens, i, rows) : 0xFFFFFFFFu;  // counts nowhere
    __syncthreads();
    const int pos = (int)threadIdx.x % RANK_POS, group = (int)threadIdx.x / RANK_POS;
    const uint32_t k = keys[own + pos];
    uint32_t c = 0;
#pragma unroll 4
    for (int j = group * 4; j < padded; j += RANK_PARTS * 4) {
        const uint4 x = *(const uint4 *)(keys + j);
        const uint32_t below = k + (j < own);
        c += (x.x < below) + (x.y < below) + (x.z < below) + (x.w < below);
    }
    if (group < pos) c += keys[own + group] == k;  // (RANK_PARTS >= RANK_POS)
    count[group][pos] = c;
    __syncthreads();
    if (threadIdx.x < RANK_POS && own + pos < n) {
        uint32_t at = 0;
#pragma unroll 8
        for (int w = 0; w < RANK_PARTS; ++w) at += count[w][pos];
        out[at] = (uint64_t)k << 32 | (uint32_t)(own + pos);
    }
}

// ---------------------------------------------------------------- radix sort

// Stable, least digit first, SORT_TILE entries per block.  Per pass the tiles count
// their digits (hist[tile][digit]); a tile of the scatter adds up what the digits below
// its own and the tiles before it hold, by itself while there are few tiles, after
// k_grad_prefix otherwise.  Its threads share the tiles in `parts`, as many as its threads
// hold digits (2 of nine bits, 16 of five), and the line lies where a part has SELF_TILES.
// By itself and after the prefix (whole gradients of 16 columns, us): two parts, 196 tiles 75
// and 81, 293 116 and 102; four, 489 99 and 110, 733 167 and 164; eight, 733 206 and 251, 1465
// 465 and 449; sixteen, 1465 193 and 274.  Tiles of 2048 in blocks of 16 waves: 16000
// tokens took 40 us with 4096 in 8 waves, 32 so; 400000 took 85 and 86.
constexpr int SORT_NT = 1024;
constexpr int SORT_ITEMS = 2;
constexpr int SORT_TILE = SORT_NT * SORT_ITEMS;
constexpr int DIGIT_MAX = 9;
constexpr int BINS_MAX = 1 << DIGIT_MAX;
constexpr int SELF_TILES = 128;
static_assert(BINS_MAX <= SORT_NT, "one thread per digit");

struct Digits {
    int32_t shift, bits;
};
__host__ __device__ constexpr int sort_parts(int bits) { return SORT_NT >> bits < 16 ? SORT_NT >> bits : 16; }

template <typename IX, bool FIRST>
__device__ __forceinline__ uint64_t sort_entry(const void *in, int64_t i, int64_t rows)
{
    if constexpr (FIRST)
        return (uint64_t)key_at((const IX *)in, i, rows) << 32 | (uint32_t)i;
    else
        return ((const uint64_t *)in)[i];
}

template <typename IX, bool FIRST>
__global__ void __launch_bounds__(SORT_NT) k_grad_hist(const void *in, int64_t n, int64_t rows,
                                                       Digits d, uint32_t *hist)
{
    __shared__ uint32_t bin[BINS_MAX];
    const int t = (int)threadIdx.x;
    if (t < BINS_MAX) bin[t] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * SORT_TILE;
#pragma unroll
    for (int k = 0; k < SORT_ITEMS; ++k) {
        const int64_t i = i0 + k * SORT_NT + t;
        if (i < n)
            atomicAdd(&bin[key_of(sort_entry<IX, FIRST>(in, i, rows)) >> d.shift & ((1u << d.bits) - 1)],
                      1u);
    }
    __syncthreads();
    if (t < 1 << d.bits) hist[(int64_t)blockIdx.x << d.bits | t] = bin[t];
}

// hist[tile][digit] becomes the entries of that digit in the tiles before; the digits'
// totals go behind the last tile.
__global__ void __launch_bounds__(SORT_NT) k_grad_prefix(uint32_t *hist, int64_t tiles, int32_t bits)
{
    const int t = (int)threadIdx.x;
    if (t >= 1 << bits) return;
    uint32_t sum = 0;
    int64_t k = 0;
    for (; k + 8 <= tiles; k += 8) {
        uint32_t x[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = hist[(k + q) << bits | t];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            hist[(k + q) << bits | t] = sum;
            sum += x[q];
        }
    }
    for (; k < tiles; ++k) {
        const uint32_t x = hist[k << bits | t];
        hist[k << bits | t] = sum;
        sum += x;
    }
    hist[tiles << bits | t] = sum;
}

template <typename IX, bool FIRST>
__global__ void __launch_bounds__(SORT_NT) k_grad_scatter(const void *in, int64_t n, int64_t rows,
                                                          Digits d, const uint32_t *hist,
                                                          int64_t tiles, bool prefixed,
                                                          uint64_t *out)
{
    constexpr int NW = SORT_NT / WAVE;
    __shared__ uint32_t cnt[NW][BINS_MAX];
    __shared__ uint32_t sums[2][SORT_NT];
    __shared__ uint32_t lds[NW];
    const int t = (int)threadIdx.x, w = wave_id(), lane = lane_id();
    const int bins = 1 << d.bits;
    for (int b = lane; b < bins; b += WAVE) cnt[w][b] = 0;
    // what lies before this tile's entries of digit t: the tiles in up to 16 parts (the chain
    // of loads over 64 tiles was most of this kernel's time: 131072 tokens 12 us, 10 so)
    uint32_t total = 0, before = 0;
    if (prefixed) {
        if (t < bins) {
            before = hist[(int64_t)blockIdx.x << d.bits | t];
            total = hist[tiles << d.bits | t];
        }
    } else {
        const int parts = sort_parts(d.bits), part = t >> d.bits;
        const int each = ((int)tiles + parts - 1) / parts, k1 = (part + 1) * each < (int)tiles ? (part + 1) * each : (int)tiles;
        if (part < parts) {
            const uint32_t *h = hist + (t & (bins - 1));
            for (int k = part * each; k < k1; k += 8) {
                uint32_t x[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) x[q] = h[(int64_t)(k + q < k1 ? k + q : k) << d.bits];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    if (k + q >= k1) x[q] = 0;
                    total += x[q];
                    before += k + q < (int)blockIdx.x ? x[q] : 0u;
                }
            }
            sums[0][t] = total;
            sums[1][t] = before;
        }
        __syncthreads();
        total = before = 0;
        if (t < bins)
            for (int q = 0; q < parts; ++q) {
                total += sums[0][q << d.bits | t];
                before += sums[1][q << d.bits | t];
            }
    }
    // entries, and the place of each among its wave's of the same digit: the waves
    // take consecutive stretches, the rounds of a wave follow one another
    const int64_t i0 = (int64_t)blockIdx.x * SORT_TILE + w * (SORT_ITEMS * WAVE);
    uint64_t e[SORT_ITEMS];
    uint32_t place[SORT_ITEMS];
#pragma unroll
    for (int k = 0; k < SORT_ITEMS; ++k) {
        const int64_t i = i0 + k * WAVE + lane;
        e[k] = i < n ? sort_entry<IX, FIRST>(in, i, rows) : 0;
    }
    __syncthreads();
    volatile uint32_t *mine = cnt[w];
#pragma unroll
    for (int k = 0; k < SORT_ITEMS; ++k) {
        const bool on = i0 + k * WAVE + lane < n;
        const uint32_t dig = key_of(e[k]) >> d.shift & (uint32_t)(bins - 1);
        uint64_t same = __ballot(on);
        for (int q = 0; q < d.bits; ++q) {
            const uint64_t has = __ballot(dig >> q & 1u);
            same &= dig >> q & 1u ? has : ~has;
        }
        const uint32_t base = mine[dig];
        place[k] = base + (uint32_t)__popcll(same & lanemask_lt());
        if (on && (same & lanemask_lt()) == 0) mine[dig] = base + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    uint32_t all;
    const uint32_t digits_below = block_excl_scan_n<SORT_NT>(total, lds, all);
    if (t < bins) {
        uint32_t run = digits_below + before;
#pragma unroll
        for (int q = 0; q < NW; ++q) {
            const uint32_t x = cnt[q][t];
            cnt[q][t] = run;
            run += x;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_ITEMS; ++k) {
        if (i0 + k * WAVE + lane < n) {
            const uint32_t dig = key_of(e[k]) >> d.shift & (uint32_t)(bins - 1);
            out[cnt[w][dig] + place[k]] = e[k];
        }
    }
}

// ---------------------------------------------------------------- sums

// A team of LPR lanes (an octet each) walks over `per` sorted entries and a slab of
// columns; a block's teams follow one another.  A run that lies within a team's piece
// is stored at once.  The others leave their parts in LDS, and the team (or, into the
// block, the first one) where the run begins adds them up in order; what crosses the
// block's edges goes to `part`: [block][0] what continues from the block before,
// [block][1] what begins here and continues.  Blocks after the sums write the zeros:
// they search for their rows' entries.  Bound by the bytes: 131072 rows of 2048 bf16 into
// 131072 fp32 rows 303 us (1.6 GB, 5.3 TB/s), 5003 into 50001 of 1001 32 us (6.2 TB/s).
constexpr int SUM_NT = 512;
// Entries whose rows a team has in flight: with a team smaller than a wave they are in vector
// registers, and eight leave too few waves (30000 rows of 250 fp32 columns 58 us, with
// four 47).
constexpr int sum_ahead(int lpr) { return lpr < WAVE ? 4 : 8; }

struct SumShape {
    int32_t per;      // entries per team
    int32_t slabs;    // of LPR octets
    int64_t chunks;   // blocks along the entries
    int64_t part_ld;  // floats of one row of part
};

// First index whose key is at least `key`, else n: every lane of the wave looks at the
// end of one of 64 pieces.
__device__ __forceinline__ int64_t wave_first_at_least(const uint64_t *e, int64_t n, uint32_t key)
{
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t step = (hi - lo + WAVE - 1) / WAVE, beg = lo + lane_id() * step;
        const int64_t end = beg + step < hi ? beg + step : hi;
        const bool less = beg < hi && key_of(e[beg < hi ? end - 1 : lo]) < key;
        lo += (int64_t)__popcll(__ballot(less)) * step;  // (pieces below the key come first)
        if (lo >= hi) return hi;
        if (step == 1) return lo;
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo;
}

// First index in [lo, hi) whose key is at least `key`, else hi.
__device__ __forceinline__ int64_t first_at_least(const uint64_t *e, int64_t lo, int64_t hi,
                                                  uint32_t key)
{
    while (lo < hi) {
        const int64_t mid = lo + (hi - lo) / 2;
        if (key_of(e[mid]) < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

template <typename TI, typename TO, int LPR>
__global__ void __launch_bounds__(SUM_NT) k_grad_sum(GradArgs a, const uint64_t *__restrict__ e,
                                                     SumShape sh, float *__restrict__ part,
                                                     Split fill)
{
    constexpr int TEAMS = SUM_NT / LPR, AHEAD = sum_ahead(LPR);
    __shared__ float head[OCT][SUM_NT], tail[OCT][SUM_NT];
    __shared__ uint8_t through[TEAMS];
    __shared__ uint8_t used[FILL_UNITS];
    const int64_t n = a.n, sums = sh.chunks * sh.slabs;
    if ((int64_t)blockIdx.x < sums) {
        const int64_t chunk = (int64_t)blockIdx.x / sh.slabs;
        // with a whole wave per team its entries, places and branches are the wave's
        const int team = LPR == WAVE ? scalar(wave_id()) : (int)threadIdx.x / LPR;
        const int32_t oct = (int32_t)(blockIdx.x % sh.slabs) * LPR + (int)threadIdx.x % LPR;
        const bool on = oct * OCT < a.dim;
        const int64_t c0 = chunk * sh.per * TEAMS;
        int64_t p0 = c0 + (int64_t)team * sh.per, p1 = p0 + sh.per;
        p0 = p0 < n ? p0 : n;
        p1 = p1 < n ? p1 : n;
        const uint32_t none = (uint32_t)a.rows;  // sorts behind every row
        const uint32_t before = p0 > 0 && p0 < n ? key_of(e[p0 - 1]) : none;
        const uint32_t after = p1 < n ? key_of(e[p1]) : none;
        uint32_t cur = p0 < p1 ? key_of(e[p0]) : none;
        bool is_first = true, has_head = false, has_tail = false;
        float acc[OCT];
        zero_oct(acc);
        const auto finish = [&](bool is_last) {
            if (cur == none) return;
            const bool h = is_first && before == cur, t = is_last && after == cur;
            if (h) {
                has_head = true;
#pragma unroll
                for (int c = 0; c < OCT; ++c) head[c][threadIdx.x] = acc[c];
            } else if (t) {
#pragma unroll
                for (int c = 0; c < OCT; ++c) tail[c][threadIdx.x] = acc[c];
            } else if (on) {
                put_oct<TO>(a, cur, oct, acc);
            }
            has_tail = t;
            if (is_last) through[team] = h && t;
        };
        through[team] = 0;
        for (int64_t p = p0; p < p1; p += AHEAD) {
            uint64_t x[AHEAD];
            Raw<TI> v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) x[k] = e[p + k < p1 ? p + k : p1 - 1];
            if (key_of(x[0]) == none) break;  // nothing but padding from here on
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                load_raw<true, (LPR > 4)>((const TI *)a.grad + (int64_t)(uint32_t)x[k] * a.grad_ld, on ? oct : 0,
                         cols_of(a.dim), v[k]);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (p + k < p1) {
                    if (key_of(x[k]) != cur) {
                        finish(false);
                        is_first = false;
                        cur = key_of(x[k]);
                        zero_oct(acc);
                    }
                    add_oct(a, v[k], (uint32_t)x[k], oct, true, acc);
                }
            }
        }
        if (p0 < p1) finish(true);
        __syncthreads();
        // runs that begin before the block, then runs that begin in this team's piece
        const int lane = (int)threadIdx.x % LPR;
        const auto chain = [&](uint32_t key, int from, bool more, int slot) {
            int j = from;
            while (more && j < TEAMS) {
#pragma unroll
                for (int c = 0; c < OCT; ++c) acc[c] += head[c][j * LPR + lane];
                more = through[j];
                ++j;
            }
            if (slot == 1 && !more) {
                if (on) put_oct<TO>(a, key, oct, acc);
            } else if (on) {  // [0]: the rest of a run from before; [1]: the start of a longer one
                float *p = part + (chunk * 2 + slot) * sh.part_ld + oct * OCT;
                Pack<float, OCT> w;
#pragma unroll
                for (int c = 0; c < OCT; ++c) w.v[c] = acc[c];
                __builtin_memcpy(p, &w, sizeof w);
            }
        };
        if (team == 0 && has_head) {
#pragma unroll
            for (int c = 0; c < OCT; ++c) acc[c] = head[c][threadIdx.x];
            chain(before, 1, through[0], 0);
        }
        if (has_tail && !through[team]) {
#pragma unroll
            for (int c = 0; c < OCT; ++c) acc[c] = tail[c][threadIdx.x];
            chain(after, team + 1, true, 1);
        }
        return;
    }
    const int64_t b = (int64_t)blockIdx.x - sums;
    const int64_t row0 = b / fill.stretches * fill.rows;
    const int64_t row1 = row0 + fill.rows < a.rows ? row0 + fill.rows : a.rows;
    // the entries of the block's rows, between two searches, say which rows have one
    __shared__ int64_t ends[2];
    if (wave_id() < 2) {
        const int64_t at = wave_first_at_least(e, n, (uint32_t)(wave_id() ? row1 : row0));
        if (lane_id() == 0) ends[wave_id()] = at;
    }
    for (int u = threadIdx.x; u < FILL_UNITS; u += SUM_NT) used[u] = 0;
    __syncthreads();
    const int64_t lo = ends[0], hi = ends[1];
    if (hi - lo <= 4 * SUM_NT) {
        for (int64_t i = lo + threadIdx.x; i < hi; i += SUM_NT) used[key_of(e[i]) - row0] = 1;
    } else {
        for (int64_t r = row0 + threadIdx.x; r < row1; r += SUM_NT) {
            const int64_t at = first_at_least(e, lo, hi, (uint32_t)r);
            used[r - row0] = at < hi && key_of(e[at]) == (uint32_t)r;
        }
    }
    __syncthreads();
    fill_zeros<TO, SUM_NT>(a, fill, b, row0, used);
}

// A run that goes over the edge of chunk c and begins in it: its parts, in order.
// Four waves take consecutive stretches of the parts.  A few dependent loads: 5 to 9 us.
template <typename TO>
__global__ void __launch_bounds__(BLOCK) k_grad_join(GradArgs a, const uint64_t *e, SumShape sh,
                                                     int64_t step, const float *part)
{
    __shared__ float sum[3][SLAB];
    const int32_t slabs = (int32_t)((a.dim + SLAB - 1) / SLAB);
    const int64_t c = (int64_t)blockIdx.x / slabs;
    const int32_t oct = (int32_t)(blockIdx.x % slabs) * WAVE + lane_id();
    const int64_t edge = (c + 1) * step;
    if (edge >= a.n) return;
    const uint32_t key = key_of(e[edge]);
    if (key == (uint32_t)a.rows || key_of(e[edge - 1]) != key) return;
    if (c > 0 && key_of(e[c * step]) == key && key_of(e[c * step - 1]) == key) return;  // began earlier
    int64_t parts = 0;  // chunks after c that the run reaches into
    for (int64_t j = c + 1;; j += BLOCK) {
        const int64_t at = (j + threadIdx.x) * step;
        const int got = __syncthreads_count(at < a.n && key_of(e[at < a.n ? at : 0]) == key);
        parts += got;
        if (got < BLOCK) break;
    }
    const int64_t per = (parts + 3) / 4;
    const int64_t j0 = c + 1 + wave_id() * per;
    const int64_t j1 = j0 + per < c + 1 + parts ? j0 + per : c + 1 + parts;
    const bool on = oct * OCT < a.dim;
    const Cols whole = cols_of((int32_t)sh.part_ld);  // rows of part are whole octets
    float acc[OCT];
    zero_oct(acc);
    if (on) {
        if (wave_id() == 0) load_oct<false, true>(part + (c * 2 + 1) * sh.part_ld, oct, whole, acc);
        for (int64_t j = j0; j < j1; j += 4) {
            Raw<float> v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                load_raw<false, true>(part + (j + k < j1 ? j + k : j) * 2 * sh.part_ld, oct, whole, v[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int q = 0; q < OCT; ++q) acc[q] += j + k < j1 ? raw_float(v[k], q) : 0.f;
        }
    }
    if (wave_id() > 0) {
#pragma unroll
        for (int q = 0; q < OCT; ++q) sum[wave_id() - 1][q * WAVE + lane_id()] = acc[q];
    }
    __syncthreads();
    if (wave_id() == 0 && on) {
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int q = 0; q < OCT; ++q) acc[q] += sum[w][q * WAVE + lane_id()];
        put_oct<TO>(a, key, oct, acc);
    }
}

// ---------------------------------------------------------------- host

static int team_lanes(int32_t dim)
{
    int l = 4;
    while (l < WAVE && l * OCT < dim) l *= 2;
    return l;
}

// Pieces of 4 to 32 entries per team: enough blocks for the card where there are few
// entries, few cut runs where there are many.  Narrow rows have many teams in a block and
// take 8 or 16 at least: a run goes from team to team in turn.  Whole gradients, us, with 256,
// 512, 1024, 2048 and 4096 blocks aimed at: 131072 x 512 107 107 104 104 121, 1000000 x 256 239 239
// 239 246 251, 20000 x 2048 98 91 91 93 93, narrow or few rows the same within 2 %; with 8, 16, 32,
// 64 and 128 entries at most: 131072 x 2048 355 346 339 342 343, 1000000 x 256 266 246 239 256 256.
static SumShape sum_shape(int64_t n, int32_t dim)
{
    const int lpr = team_lanes(dim), teams = SUM_NT / lpr;
    SumShape s;
    s.slabs = (dim + lpr * OCT - 1) / (lpr * OCT);
    const int64_t per = n * s.slabs / ((int64_t)teams * 1024), least = lpr < 16 ? 64 / lpr : 4;
    s.per = (int32_t)(per < least ? least : per > 32 ? 32 : per);
    s.chunks = (n + (int64_t)s.per * teams - 1) / ((int64_t)s.per * teams);
    s.part_ld = ((int64_t)dim + OCT - 1) / OCT * OCT;
    return s;
}

struct GradWs {
    int64_t e0, e1, hist, part, bytes;
    int64_t tiles;
};
static GradWs grad_layout(int64_t n, int32_t dim)
{
    GradWs w{};
    if (is_direct(n, dim)) return w;
    const auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
    w.tiles = (n + SORT_TILE - 1) / SORT_TILE;
    w.e0 = 0;
    w.e1 = up(n * 8);
    w.hist = w.e1 + (n > RANK_MAX ? up(n * 8) : 0);
    w.part = w.hist + (n > RANK_MAX ? up((w.tiles + 1) * BINS_MAX * 4) : 0);
    const SumShape s = sum_shape(n, dim);
    w.bytes = w.part + up(s.chunks * 2 * s.part_ld * 4);
    return w;
}

int64_t grad_workspace(int64_t n, int64_t, int32_t dim) { return grad_layout(n, dim).bytes; }

template <typename IX>
static hipError_t sort_tokens(const GradArgs &a, const GradWs &w, uint64_t **sorted, hipStream_t s)
{
    uint64_t *e0 = (uint64_t *)(a.ws + w.e0), *e1 = (uint64_t *)(a.ws + w.e1);
    if (a.n <= RANK_MAX) {
        *sorted = e0;
        return launch(k_grad_rank<IX>, dim3((unsigned)((a.n + RANK_POS - 1) / RANK_POS)), dim3(RANK_NT), s,
                      (const IX *)a.tokens, (int32_t)a.n, a.rows, e0);
    }
    int bits = 1;
    while (a.rows >> bits) ++bits;  // keys are 0 .. rows
    const int passes = (bits + DIGIT_MAX - 1) / DIGIT_MAX, width = (bits + passes - 1) / passes;
    uint32_t *hist = (uint32_t *)(a.ws + w.hist);
    const dim3 grid((unsigned)w.tiles), block(SORT_NT);
    const bool prefixed = w.tiles > (int64_t)SELF_TILES * sort_parts(width);
    const void *in = a.tokens;
    uint64_t *out = e0;
    for (int p = 0; p < passes; ++p) {
        const Digits d{p * width, width};
        hipError_t r = p == 0 ? launch(k_grad_hist<IX, true>, grid, block, s, in, a.n, a.rows, d, hist)
                              : launch(k_grad_hist<IX, false>, grid, block, s, in, a.n, a.rows, d, hist);
        if (r == hipSuccess && prefixed)
            r = launch(k_grad_prefix, dim3(1), block, s, hist, w.tiles, width);
        if (r == hipSuccess)
            r = p == 0 ? launch(k_grad_scatter<IX, true>, grid, block, s, in, a.n, a.rows, d,
                                (const uint32_t *)hist, w.tiles, prefixed, out)
                       : launch(k_grad_scatter<IX, false>, grid, block, s, in, a.n, a.rows, d,
                                (const uint32_t *)hist, w.tiles, prefixed, out);
        if (r != hipSuccess) return r;
        *sorted = out;
        in = out;
        out = out == e0 ? e1 : e0;
    }
    return hipSuccess;
}

template <typename TI, typename TO, typename IX>
static hipError_t run_grad_as(const GradArgs &a, hipStream_t s)
{
    const Split fill = split_rows(a.add ? 0 : a.rows, fill_pieces<TO>(a), FILL_UNITS);
    const int64_t fills = split_blocks(fill);
    if (is_direct(a.n, a.dim)) {
        const int32_t slabs = (int32_t)((a.dim + SLAB - 1) / SLAB);
        const int64_t sums = a.n * slabs;
        if (sums + fills == 0) return hipSuccess;
        if (sums + fills > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
        return launch(a.dim >= OCT ? k_grad_direct<TI, TO, IX, true> : k_grad_direct<TI, TO, IX, false>,
                      dim3((unsigned)(sums + fills)), dim3(DIRECT_NT), s, a, slabs, sums, fill);
    }
    const GradWs w = grad_layout(a.n, a.dim);
    const SumShape sh = sum_shape(a.n, a.dim);
    const int64_t sums = sh.chunks * sh.slabs;
    if (sums + fills > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    uint64_t *e = nullptr;
    hipError_t r = sort_tokens<IX>(a, w, &e, s);
    if (r != hipSuccess) return r;
    float *part = (float *)(a.ws + w.part);
    const int lpr = team_lanes(a.dim);
    const auto sum = [&](auto kern) {
        return launch(kern, dim3((unsigned)(sums + fills)), dim3(SUM_NT), s, a, (const uint64_t *)e, sh,
                      part, fill);
    };
    r = lpr == 4    ? sum(k_grad_sum<TI, TO, 4>)
        : lpr == 8  ? sum(k_grad_sum<TI, TO, 8>)
        : lpr == 16 ? sum(k_grad_sum<TI, TO, 16>)
        : lpr == 32 ? sum(k_grad_sum<TI, TO, 32>)
                    : sum(k_grad_sum<TI, TO, 64>);
    if (r != hipSuccess || sh.chunks == 1) return r;
    const int64_t slabs = (a.dim + SLAB - 1) / SLAB;
    return launch(k_grad_join<TO>, dim3((unsigned)((sh.chunks - 1) * slabs)), dim3(BLOCK), s, a,
                  (const uint64_t *)e, sh, (int64_t)sh.per * (SUM_NT / lpr), (const float *)part);
}

hipError_t run_grad(const GradArgs &a, hipStream_t s)
{
    return with_index(a.token_type, [&](auto ix) {
        return with_type(a.grad_type, [&](auto ti) {
            return with_type(a.out_type, [&](auto to) {
                using IX = decltype(ix);
                using TI = decltype(ti);
                using TO = decltype(to);
                return run_grad_as<TI, TO, IX>(a, s);
            });
        });
    });
}

}  // namespace sp
