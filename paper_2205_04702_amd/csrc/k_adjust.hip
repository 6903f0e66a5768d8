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
        // Large calls take longer stretches, and scores and outputs past the caches; long texts, which
        // every stretch of a row reads, the longest (us: 512 threads of 2 units, 1024 of 2, 256 of 4,
        // 256 of 1; then the first through the caches):
        //   64 x 131072 bf16, 4096 tokens, 300 biases, a mask    12.2  12.4  14.0  17.0  14.2
        //   333 x 50001 fp32, 1777 tokens                        27.8  30.7  28.6  35.7  30.9
        //   256 x 131072 bf16, 512 tokens, 50 biases             33.1  36.7  31.0  48.3  38.9
        //   512 x 32768 bf16, 8000 tokens                        22.5  22.6  27.3  37.0  22.6
        //   500 x 262144 bf16, 16000 tokens, 100 biases, a mask   206   158   219   541   227
        // Without lists, 100 x 200000 fp32 with a mask: 256 threads of 1 unit 26.2, of 4 28.8 (past the
        // caches), 34.4 (through them).
        const bool large = a.n * a.vocab >= 1 << 23;
        if (!a.previous && !a.bias_tokens)
            return large ? go(k_adjust<T, 256, 1, false, true>, 256, 1) : go(k_adjust<T, 256, 1, false, false>, 256, 1);
        if (!large) return go(k_adjust<T, 256, 1, true, false>, 256, 1);
        return a.length > 8192 ? go(k_adjust<T, 1024, 2, true, true>, 1024, 2) : go(k_adjust<T, 512, 2, true, true>, 512, 2);
    });
}

}  // namespace sp
