// Distillation of a row of scores from a teacher's top logits, and its gradient to the scores.
//
//   p_j = softmax over the row's entries j of teacher_j / T   (entries whose token is a column)
//   q_v = softmax over the columns of scores_v / T
//   loss = T^2 sum_j p_j (log p_j - log q_token(j))
//   d weight * loss / d scores_v = weight T (q_v - sum over j with token(j) = v of p_j)
//
// A row without an entry, or whose entries are all -infinity, has loss 0 and gradient 0,
// whatever its scores hold.
#include "sp_rows.h"

namespace sp {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NONE = -__builtin_inff();

// A softmax's largest value and the sum of exp2((value - largest) * c), of a part of the values.
// c is log2(e) / T: differences first, so that near the largest nothing is lost to c's rounding.
struct Soft {
    float top, sum;
};
__device__ __forceinline__ float part_of(float v, float top, float c) { return exp2f((v - top) * c); }
__device__ __forceinline__ void join(Soft &s, Soft o, float c)
{
    const float top = fmaxf(s.top, o.top);
    if (top > NONE) {  // (both empty: sums of 0, or of NaN, stay what they are)
        s.sum = s.sum * part_of(s.top, top, c) + o.sum * part_of(o.top, top, c);
        s.top = top;
    } else {
        s.sum += o.sum;
    }
}

// The same over the block, in all of its threads.  `lds` holds NT / WAVE entries; two barriers.
template <int NT>
__device__ __forceinline__ Soft block_soft(Soft s, Soft *lds, float c)
{
#pragma unroll
    for (int o = WAVE / 2; o > 0; o >>= 1) {
        const Soft other{__shfl_xor(s.top, o, WAVE), __shfl_xor(s.sum, o, WAVE)};
        join(s, other, c);
    }
    if (lane_id() == 0) lds[wave_id()] = s;
    __syncthreads();
    s = lds[0];
#pragma unroll
    for (int w = 1; w < NT / WAVE; ++w) join(s, lds[w], c);
    __syncthreads();
    return s;
}
template <int NT>
__device__ __forceinline__ float block_total(float v, float *lds)
{
    v = wave_sum(v);
    if (lane_id() == 0) lds[wave_id()] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < NT / WAVE; ++w) v += lds[w];
    __syncthreads();
    return v;
}

// An octet into a part of the softmax: one rescaling for its eight columns.
template <typename T>
__device__ __forceinline__ void add_oct(Soft &s, const float (&v)[OCT], int valid, float c)
{
    float top = s.top;
#pragma unroll
    for (int k = 0; k < OCT; ++k) top = fmaxf(top, k < valid ? v[k] : NONE);
    const float base = top > NONE ? top : 0.f;
    float sum = s.top > NONE ? s.sum * part_of(s.top, base, c) : s.sum;
#pragma unroll
    for (int k = 0; k < OCT; ++k) sum += k < valid ? part_of(v[k], base, c) : 0.f;
    s = Soft{top, sum};
}

// ---------------------------------------------------------------- the teacher's entries
//
// Entries in LDS, a thread at a time for each NT-th.  Tokens that are listed more than once
// are found with a hash of the tokens, in which each keeps the lowest entry that lists it.
constexpr int MAX_K = 1024, SLOTS = 2 * MAX_K;
struct Entries {
    int32_t token[MAX_K];  // -1: none
    float p[MAX_K], score[MAX_K];
    int32_t key[SLOTS], lowest[SLOTS];
    int32_t repeated;
};
constexpr int32_t FREE = -1;

__device__ __forceinline__ int slot_of(const Entries &e, int32_t token, int mask)
{
    int h = (int)((uint32_t)token * 0x9E3779B1u >> 16) & mask;
    while (e.key[h] != token) h = (h + 1) & mask;
    return h;
}

// One block per row, which is read once for the sums and, for the gradient, once more.
template <typename T, typename TO, int NT, bool GRAD>
__global__ void __launch_bounds__(NT) k_distill(DistillArgs a)
{
    __shared__ Soft soft[NT / WAVE];
    __shared__ float total[NT / WAVE];
    __shared__ Entries e;
    const int64_t row = blockIdx.x;
    const int t = (int)threadIdx.x;
    const float c = LOG2E / a.temperature;
    const T *scores = (const T *)a.scores + row * a.ld;
    const Cols cols = cols_of(a.vocab);
    const int32_t octs = (a.vocab + OCT - 1) / OCT;
    TO *grad = GRAD ? (TO *)a.grad + row * a.grad_ld : nullptr;

    int mask = 1;
    while (mask < 2 * a.k) mask *= 2;
    mask -= 1;
    if (GRAD) {
        for (int i = t; i <= mask; i += NT) e.key[i] = FREE, e.lowest[i] = MAX_K;
        if (t == 0) e.repeated = 0;
    }
    Soft teacher{NONE, 0.f};
    for (int j = t; j < a.k; j += NT) {
        const int64_t token = index_at(a.tokens, a.token_type, row * a.tokens_ld + j);
        const bool live = token >= 0 && token < a.vocab;
        const float v = live ? float_at(a.teacher, a.teacher_type, row * a.teacher_ld + j) : NONE;
        e.token[j] = live ? (int32_t)token : -1;
        e.p[j] = v;
        e.score[j] = live ? to_float(scores[token]) : 0.f;
        join(teacher, Soft{v, v > NONE ? 1.f : v != v ? v : 0.f}, c);
    }
    teacher = block_soft<NT>(teacher, soft, c);
    if (teacher.sum == 0.f) {  // the same for all
        if (t == 0) a.loss[row] = 0.f;
        if (GRAD) {
            const float zeros[OCT] = {};
            for (int32_t o = t; o < octs; o += NT) put_row_oct(grad, o, a.vocab, false, zeros);
        }
        return;
    }

    Soft s{NONE, 0.f};
    for (int32_t o = t; o < octs; o += NT) {
        float v[OCT];
        load_oct<false, false>(scores, o, cols, v);
        add_oct<T>(s, v, oct_valid(a.vocab, o), c);
    }
    s = block_soft<NT>(s, soft, c);
    const float log_sum = log2f(s.sum) * LN2, log_mass = log2f(teacher.sum) * LN2;
    const float per_t = 1.f / a.temperature, mass = 1.f / teacher.sum;

    float loss = 0.f;
    for (int j = t; j < a.k; j += NT) {
        const float v = e.p[j], p = part_of(v, teacher.top, c) * mass;
        const float log_p = (v - teacher.top) * per_t - log_mass;
        const float log_q = (e.score[j] - s.top) * per_t - log_sum;
        if (e.token[j] >= 0 && !(p == 0.f)) loss += p * (log_p - (s.sum == 0.f ? NONE : log_q));
        e.p[j] = e.token[j] >= 0 ? p : 0.f;
        if (GRAD && e.token[j] >= 0) {
            int h = (int)((uint32_t)e.token[j] * 0x9E3779B1u >> 16) & mask;
            for (;;) {  // (at most half of the slots are taken)
                const int32_t old = atomicCAS(&e.key[h], FREE, e.token[j]);
                if (old == FREE) break;
                if (old == e.token[j]) {
                    e.repeated = 1;
                    break;
                }
                h = (h + 1) & mask;
            }
            atomicMin(&e.lowest[h], j);
        }
    }
    loss = block_total<NT>(loss, total);
    if (t == 0) a.loss[row] = loss * a.temperature * a.temperature;
    if (!GRAD) return;

    const float g = (a.weights ? a.weights[row] : a.weight) * a.temperature;
    const float base = s.top > NONE ? s.top : 0.f, part = s.sum == 0.f ? 0.f : 1.f / s.sum;
    for (int32_t o = t; o < octs; o += NT) {
        float v[OCT];
        load_oct<false, false>(scores, o, cols, v);
#pragma unroll
        for (int k = 0; k < OCT; ++k) v[k] = part_of(v[k], base, c) * part * g;
        put_row_oct(grad, o, a.vocab, false, v);
    }
    __syncthreads();
    // The teacher's columns again, over what was stored: the lowest entry of each token.
    for (int j = t; j < a.k; j += NT) {
        const int32_t token = e.token[j];
        if (token < 0 || e.lowest[slot_of(e, token, mask)] != j) continue;
        float p = e.p[j];
        if (e.repeated)
            for (int i = j + 1; i < a.k; ++i) p += e.token[i] == token ? e.p[i] : 0.f;
        grad[token] = from_float<TO>((part_of(e.score[j], base, c) * part - p) * g);
    }
}

int64_t distill_workspace(int64_t, int32_t, int32_t, bool) { return 0; }

hipError_t run_distill(const DistillArgs &given, hipStream_t s)
{
    return with_type(given.type, [&](auto ti) {
        return with_type(given.grad ? given.grad_type : 0, [&](auto to) {
            using T = decltype(ti);
            using TO = decltype(to);
            for (int64_t i = 0; i < given.n; i += LAUNCH_BLOCKS) {
                DistillArgs a = given;
                a.n = given.n - i < LAUNCH_BLOCKS ? given.n - i : LAUNCH_BLOCKS;
                a.scores = (const T *)given.scores + i * given.ld;
                a.tokens = index_past(given.tokens, given.token_type, i * given.tokens_ld);
                a.teacher = (const char *)given.teacher + i * given.teacher_ld * (given.teacher_type == 0 ? 4 : 2);
                a.loss += i;
                if (a.weights) a.weights += i;
                if (a.grad) a.grad = (TO *)given.grad + i * given.grad_ld;
                const hipError_t e = a.grad ? launch(k_distill<T, TO, BLOCK, true>, dim3((unsigned)a.n), dim3(BLOCK), s, a)
                                            : launch(k_distill<T, float, BLOCK, false>, dim3((unsigned)a.n), dim3(BLOCK), s, a);
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        });
    });
}

}  // namespace sp
