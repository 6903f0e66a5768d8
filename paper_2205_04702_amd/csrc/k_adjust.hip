// Scores adjusted before a token is chosen from them: penalties for tokens that came before,
// biases, and a mask of the tokens that a grammar allows.
//
//   y = s;  c = how often v is among the row's previous tokens
//   c > 0:          y = (s > 0 ? s / repetition : s * repetition) - (presence + frequency * c)
//   v has a bias:   y += bias (of several entries for v the last)
//   v not allowed:  y = -infinity, whatever s holds
#include "sp_rows.h"

namespace sp {

// A column's word in LDS: how often it came before in the low 21 bits (at most 2^20 tokens), the last of
// its bias entries, counted from 1, above (at most 2047 of them).
constexpr int COUNT_BITS = 21;
constexpr uint32_t COUNT_MASK = (1u << COUNT_BITS) - 1;
typedef uint32_t word_4 __attribute__((ext_vector_type(4)));

// N tokens of a list of n for a thread, from `from` on, NT apart, all loaded at once (one at a time, the
// loads' latencies were most of the call: 64 rows of 131072 columns with 4096 tokens each 30 us).
template <int NT, int N>
struct Tokens {
    int64_t v[N];
    __device__ __forceinline__ void load(const void *list, int32_t type, int64_t at, int32_t n, int32_t from)
    {
        if (n == 0) return;
        if (type == 3) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = ((const int32_t *)list)[at + (from + k * NT < n ? from + k * NT : n - 1)];
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = ((const int64_t *)list)[at + (from + k * NT < n ? from + k * NT : n - 1)];
        }
    }
    // go(column, i) for those that fall on columns first .. first + width - 1
    template <class F>
    __device__ __forceinline__ void each(int32_t n, int32_t from, int32_t first, int32_t width, F go) const
    {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (from + k * NT < n && (uint64_t)(v[k] - first) < (uint64_t)width) go((int32_t)(v[k] - first), from + k * NT);
    }
};
template <int NT, int N, class F>
__device__ __forceinline__ void each_token(Tokens<NT, N> &tokens, const void *list, int32_t type, int64_t at, int32_t n, int32_t first,
                                           int32_t width, F go)
{
    for (int32_t from = (int32_t)threadIdx.x;;) {  // (the first of them are loaded)
        tokens.each(n, from, first, width, go);
        from += N * NT;
        if (from >= n) break;
        tokens.load(list, type, at, n, from);
    }
}

// A block takes a stretch of U * NT units of one row.  Its scores are loaded first; while they are on
// their way it notes the bias entries and counts the row's previous tokens that fall on the stretch, by
// integer atomics in LDS, whose order changes nothing; then it goes over the columns once.
template <typename T, int NT, int U, bool LISTS, bool STREAM>
__global__ void __launch_bounds__(NT) k_adjust(AdjustArgs a, int32_t stretches)
{
    constexpr int C = COLS<T>, WIDTH = U * NT * C;
    __shared__ __attribute__((aligned(16))) uint32_t words[LISTS ? WIDTH : 1];
    const int64_t b = xcd_block(blockIdx.x, gridDim.x);
    const int64_t row = b / stretches;
    const int32_t first = (int32_t)(b - row * stretches) * WIDTH;
    const int32_t width = a.vocab - first < WIDTH ? a.vocab - first : WIDTH;
    const int32_t units = width / C, rest = width - units * C;  // (a rest in the row's last stretch only)
    const int t = (int)threadIdx.x;
    const T *scores = (const T *)a.scores + row * a.ld + first;
    T *out = (T *)a.out + row * a.out_ld + first;
    const __amdgpu_buffer_rsrc_t from = buffer(scores, units * 16), to = buffer(out, units * 16);
    unit x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load_unit<STREAM>(from, t + u * NT);
    T last = from_float<T>(0.f);
    if (t < rest) last = scores[units * C + t];
    // The mask's bits of each unit (bit v % 8 of byte v / 8, as the words lie in memory).
    uint32_t bits[U], last_bit = 1;
    const uint8_t *allowed = a.allowed + row * a.allowed_ld;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        bits[u] = ~0u;
        const int32_t v = first + (t + u * NT) * C;
        if (a.allowed && t + u * NT < units) bits[u] = allowed[v / 8] >> (v % 8);
    }
    if (a.allowed && t < rest) last_bit = allowed[(first + units * C + t) / 8] >> ((first + units * C + t) % 8) & 1;
    Tokens<NT, 2> entries;
    Tokens<NT, 8> before;
    if (LISTS && a.bias_tokens) entries.load(a.bias_tokens, a.bias_type, row * a.bias_tokens_ld, a.biases, t);
    if (LISTS && a.previous) before.load(a.previous, a.previous_type, row * a.previous_ld, a.length, t);
    float repetition = a.repetition, presence = a.presence, frequency = a.frequency;
    if (LISTS) {
        if (a.penalties) {
            const float *p = a.penalties + row * a.penalties_ld;
            repetition = p[0], presence = p[1], frequency = p[2];
        }
        for (int i = t; i < WIDTH / 4; i += NT) *(word_4 *)&words[4 * i] = word_4{0, 0, 0, 0};
        __syncthreads();
        if (a.bias_tokens) {
            each_token(entries, a.bias_tokens, a.bias_type, row * a.bias_tokens_ld, a.biases, first, width,
                       [&](int32_t v, int32_t i) { atomicMax(&words[v], (uint32_t)(i + 1) << COUNT_BITS); });
            __syncthreads();
        }
        if (a.previous) {
            each_token(before, a.previous, a.previous_type, row * a.previous_ld, a.length, first, width,
                       [&](int32_t v, int32_t) { atomicAdd(&words[v], 1u); });
            __syncthreads();
        }
    }
    const float *bias = a.bias + row * a.bias_ld;
    const auto adjusted = [&](float v, uint32_t word) {
        const uint32_t count = word & COUNT_MASK, entry = word >> COUNT_BITS;
        if (count) {
            v = v > 0.f ? v / repetition : v * repetition;
            v -= presence + frequency * (float)count;
        }
        return entry ? v + bias[entry - 1] : v;
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t at = (t + u * NT) * C;
        float v[C];
#pragma unroll
        for (int k = 0; k < C; ++k) v[k] = column<T>(x[u], k);
        if (LISTS) {
            uint32_t w[C], any = 0;
#pragma unroll
            for (int k = 0; k < C; k += 4) __builtin_memcpy(&w[k], __builtin_assume_aligned(&words[at + k], 16), 16);
#pragma unroll
            for (int k = 0; k < C; ++k) any |= w[k];
            if (any) {
#pragma unroll
                for (int k = 0; k < C; ++k)
                    if (w[k]) v[k] = adjusted(v[k], w[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < C; ++k) v[k] = bits[u] >> k & 1 ? v[k] : -__builtin_inff();
        store_unit<STREAM, T>(to, t + u * NT, v);
    }
    if (t < rest) {
        const float v = to_float(last);
        out[units * C + t] = from_float<T>(!last_bit ? -__builtin_inff() : LISTS ? adjusted(v, words[units * C + t]) : v);
    }
}

hipError_t run_adjust(const AdjustArgs &a, hipStream_t s)
{
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        const auto go = [&](auto kern, int nt, int u) {
            const int64_t width = (int64_t)u * nt * COLS<T>, stretches = (a.vocab + width - 1) / width;
            const int64_t each = LAUNCH_BLOCKS / 4 / stretches;  // (of up to 1024 threads)
            for (int64_t i = 0; i < a.n; i += each) {
                AdjustArgs p = a;
                p.n = a.n - i < each ? a.n - i : each;
                p.scores = (const T *)a.scores + i * a.ld;
                p.out = (T *)a.out + i * a.out_ld;
                p.previous = index_past(a.previous, a.previous_type, i * a.previous_ld);
                p.penalties = a.penalties ? a.penalties + i * a.penalties_ld : nullptr;
                p.bias_tokens = index_past(a.bias_tokens, a.bias_type, i * a.bias_tokens_ld);
                p.bias = a.bias ? a.bias + i * a.bias_ld : nullptr;
                p.allowed = a.allowed ? a.allowed + i * a.allowed_ld : nullptr;
                const hipError_t e = launch(kern, dim3((unsigned)(p.n * stretches)), dim3(nt), s, p, (int32_t)stretches);
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        };
        // Long stretches read the lists less often, but zero and go over words that rows narrower than they are do
        // not have.  So a row that is one short stretch (4096 bytes) takes one, and else calls take long stretches
        // where all short ones together would read more than 2^22 tokens, or from 2^23 scores on, which then go
        // past the caches; texts of more than 8192 tokens the longest.  Measured (us of a kernel among others, in graphs:
        // 256 threads of 1 unit, 512 of 2, 1024 of 2, then 512 and 1024 of 2 past the caches; * what is taken):
        //   scores, tokens each
        //   8388 x 1000 bf16, 50                20.4*  40.7  82.9  40.5
        //   8388 x 1000 bf16, 16384              200*   196   190   195
        //   1677 x 5000 bf16, 1000              15.4   14.9  22.6  14.6   (just below 2^23: short ones)
        //   3355 x 2500 fp32, 1000              24.9   22.5  36.5  21.2
        //   8 x 131072 bf16, 4096                4.9*   5.9   7.3   5.9   7.3
        //   8 x 131072 bf16, 8192                6.0*   6.6   7.7   6.6   7.7
        //   8 x 131072 bf16, 16384               8.4    7.8*  8.7   7.8   8.6
        //   16 x 131072 bf16, 300                5.1*   5.3   6.1   5.3   6.1
        //   16 x 131072 bf16, 4096               6.4*   6.1   7.5   6.1   7.5
        //   32 x 131072 bf16, 300                7.7*   7.4   7.0   6.9   6.7
        //   32 x 131072 bf16, 4096               9.5    8.5*  8.4   7.7   7.8
        //   32 x 131072 bf16, 16384             21.0   11.9  10.3* 10.4   9.0
        //   31 x 262144 fp32, 300               16.4*  14.0  15.7  15.1  16.4
        //   31 x 262144 fp32, 4096              22.5   14.7* 16.3  16.2  17.2
        //   31 x 262144 fp32, 16384             62.8   24.6  19.8* 26.3  20.4
        //   64 x 131072 bf16, 300               11.4   11.2  11.3   9.0*  8.8
        //   64 x 131072 bf16, 4096              15.4   13.0  13.6  10.9* 11.0
        //   64 x 131072 bf16, 8192              21.6   15.4  14.3  12.8* 11.6
        //   64 x 131072 bf16, 16384             36.0   18.4  15.8  17.2  14.6*
        //   200 x 50001 fp32, 300               23.3   19.6  21.3  18.6* 20.6
        //   512 x 32768 bf16, 16384             81.4   38.0  34.8  31.1  28.5*
        // What reads the scores next finds those that went past the caches in memory only: with a maximum of each row
        // behind the call, 32 x 131072 of 300 tokens takes 34.2 through the caches and 44.6 past them, 64 x 131072
        // 38.0 and 48.0.
        // Without lists, a mask alone (256 threads of 1 unit through the caches and past them): 32 x 131072 bf16 4.6
        // and 4.1, 64 x 131072 6.9 and 6.9, 128 x 131072 11.2 and 12.0; 100 x 200000 fp32 26.2 past them.
        const bool large = a.n * a.vocab >= 1 << 23;
        if (!a.previous && !a.bias_tokens)
            return large ? go(k_adjust<T, 256, 1, false, true>, 256, 1) : go(k_adjust<T, 256, 1, false, false>, 256, 1);
        const int64_t tokens = (a.previous ? a.length : 0) + (a.bias_tokens ? a.biases : 0);
        const int64_t stretches = (a.vocab + 256 * COLS<T> - 1) / (256 * COLS<T>), reads = a.n * stretches * tokens;
        if (stretches == 1 || (!large && reads <= 1 << 22)) return go(k_adjust<T, 256, 1, true, false>, 256, 1);
        if (!large)
            return a.length > 8192 && reads >= 1 << 24 ? go(k_adjust<T, 1024, 2, true, false>, 1024, 2) : go(k_adjust<T, 512, 2, true, false>, 512, 2);
        return a.length > 8192 ? go(k_adjust<T, 1024, 2, true, true>, 1024, 2) : go(k_adjust<T, 512, 2, true, true>, 512, 2);
    });
}

}  // namespace sp
