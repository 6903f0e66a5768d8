// Scores adjusted before a token is chosen from them: penalties for tokens that came before,
// biases, and a mask of the tokens that a grammar allows.
//
//   y = s;  c = how often v is among the row's previous tokens
//   c > 0:          y = (s > 0 ? s / repetition : s * repetition) - (presence + frequency * c)
//   v has a bias:   y += bias (of several entries for v the last)
//   v not allowed:  y = -infinity, whatever s holds
#include "sp_rows.h"

namespace sp {

// A block takes a stretch of U * 2048 columns of one row.  It counts the row's previous tokens that
// fall on the stretch, and notes the last bias entry of each column, in LDS by integer atomics
// (their order changes nothing), then goes over the columns once.
template <typename T, int U, bool PREV, bool BIAS>
__global__ void __launch_bounds__(BLOCK) k_adjust(AdjustArgs a, int32_t stretches)
{
    constexpr int COLS = U * BLOCK * OCT;
    __shared__ uint32_t count[PREV ? COLS : 1];
    __shared__ int32_t entry[BIAS ? COLS : 1];
    const int64_t b = xcd_block(blockIdx.x, gridDim.x);
    const int64_t row = b / stretches;
    const int32_t col0 = (int32_t)(b - row * stretches) * COLS;
    const int32_t width = a.vocab - col0 < COLS ? a.vocab - col0 : COLS;
    const int t = (int)threadIdx.x;
    const T *scores = (const T *)a.scores + row * a.ld;
    const Cols cols = cols_of(a.vocab);
    Raw<T> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t at = (u * BLOCK + t) * OCT;
        load_raw<false, (U > 1)>(scores, (col0 + (at < width ? at : 0)) / OCT, cols, r[u]);
    }
    if (PREV || BIAS) {
        for (int i = t; i < COLS; i += BLOCK) {
            if (PREV) count[i] = 0;
            if (BIAS) entry[i] = -1;
        }
        __syncthreads();
        if (PREV) {
            const int64_t at = row * a.previous_ld;
            for (int i = t; i < a.length; i += BLOCK) {
                const int64_t v = index_at(a.previous, a.previous_type, at + i) - col0;
                if (v >= 0 && v < width) atomicAdd(&count[v], 1u);
            }
        }
        if (BIAS) {
            const int64_t at = row * a.bias_tokens_ld;
            for (int i = t; i < a.biases; i += BLOCK) {
                const int64_t v = index_at(a.bias_tokens, a.bias_type, at + i) - col0;
                if (v >= 0 && v < width) atomicMax(&entry[v], i);
            }
        }
        __syncthreads();
    }
    float repetition = a.repetition, presence = a.presence, frequency = a.frequency;
    if (PREV && a.penalties) {
        const float *p = a.penalties + row * a.penalties_ld;
        repetition = p[0], presence = p[1], frequency = p[2];
    }
    T *out = (T *)a.out + row * a.out_ld;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t at = (u * BLOCK + t) * OCT, oct = (col0 + at) / OCT;
        if (at >= width) continue;
        float v[OCT];
        settle(r[u], oct, cols);
        raw_floats(r[u], v);
#pragma unroll
        for (int k = 0; k < OCT; ++k) {
            if (PREV) {
                const uint32_t c = count[at + k];
                if (c) {
                    v[k] = v[k] > 0.f ? v[k] / repetition : v[k] * repetition;
                    v[k] -= presence + frequency * (float)c;
                }
            }
            if (BIAS) {
                const int32_t e = entry[at + k];
                if (e >= 0) v[k] += a.bias[row * a.bias_ld + e];
            }
        }
        if (a.allowed) {
            const uint32_t bits = a.allowed[row * a.allowed_ld + oct];
#pragma unroll
            for (int k = 0; k < OCT; ++k)
                if (!(bits >> k & 1)) v[k] = -__builtin_inff();
        }
        put_row_oct(out, oct, a.vocab, false, v);
    }
}

hipError_t run_adjust(const AdjustArgs &a, hipStream_t s)
{
    return with_type(a.type, [&](auto t) {
        using T = decltype(t);
        const auto go = [&](auto kern, int u) {
            const int64_t stretches = (a.vocab + u * BLOCK * OCT - 1) / (u * BLOCK * OCT);
            const int64_t each = LAUNCH_BLOCKS / stretches;
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
                const hipError_t e = launch(kern, dim3((unsigned)(p.n * stretches)), dim3(BLOCK), s, p, (int32_t)stretches);
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        };
        const bool deep = a.n * a.vocab >= 1 << 23 && a.vocab >= 4 * BLOCK * OCT;
        const auto pick = [&](auto few, auto many) { return deep ? go(many, 4) : go(few, 1); };
        if (a.previous && a.bias_tokens) return pick(k_adjust<T, 1, true, true>, k_adjust<T, 4, true, true>);
        if (a.previous) return pick(k_adjust<T, 1, true, false>, k_adjust<T, 4, true, false>);
        if (a.bias_tokens) return pick(k_adjust<T, 1, false, true>, k_adjust<T, 4, false, true>);
        return pick(k_adjust<T, 1, false, false>, k_adjust<T, 4, false, false>);
    });
}

}  // namespace sp
