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
constexpr int64_t CUS = 256, FEW_ROWS = 64;
constexpr int32_t LONG_ROW = 49152;

// A softmax's largest value and the sum of exp2((value - largest) * c), of a part of the values.
// c is log2(e) / T: differences first, so that nothing is lost to c's rounding near the largest, and
// scores of any size keep their order.  Exponentials below the smallest normal number are 0.
struct Soft {
    float top, sum;
};
__device__ __forceinline__ float part_of(float v, float top, float c)
{
    return __builtin_amdgcn_exp2f((v - top) * c);
}
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

// N units of a thread into a part of the softmax: one rescaling for all of their columns.
template <typename T, int N>
__device__ __forceinline__ void add_units(Soft &s, const unit *x, float c)
{
    float top = s.top;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int k = 0; k < COLS<T>; ++k) top = fmaxf(top, column<T>(x[i], k));
    const float base = top > NONE ? top : 0.f;
    float sum = s.top > NONE ? s.sum * part_of(s.top, base, c) : s.sum;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float part = 0.f;
#pragma unroll
        for (int k = 0; k < COLS<T>; ++k) part += part_of(column<T>(x[i], k), base, c);
        sum += part;
    }
    s = Soft{top, sum};
}

// ---------------------------------------------------------------- tokens that are listed twice
//
// A hash of a row's tokens, in which each keeps the first and the last entry that list it.
constexpr int32_t FREE = -1;

template <int K>
struct Hash {
    int32_t key[2 * K], first[2 * K], last[2 * K];
    float p[2 * K];    // of all entries that list the token
    int32_t repeated;  // some token is listed more than once
};
__device__ __forceinline__ int hash_of(int32_t token, int mask) { return (int)((uint32_t)token * 0x9E3779B1u >> 16) & mask; }
__device__ __forceinline__ int hash_mask(int k)  // at most half of the slots are taken
{
    int mask = 1;
    while (mask < 2 * k) mask *= 2;
    return mask - 1;
}
template <int K>
__device__ __forceinline__ void clear(Hash<K> &h, int mask)
{
    for (int i = (int)threadIdx.x; i <= mask; i += (int)blockDim.x) h.key[i] = FREE, h.first[i] = K, h.last[i] = -1;
    if (threadIdx.x == 0) h.repeated = 0;
}
template <int K>
__device__ __forceinline__ void note(Hash<K> &h, int mask, int32_t token, int j, float p)
{
    int at = hash_of(token, mask);
    for (;;) {
        const int32_t old = atomicCAS(&h.key[at], FREE, token);
        if (old == token) h.repeated = 1;
        if (old == FREE || old == token) break;
        at = (at + 1) & mask;
    }
    atomicMin(&h.first[at], j);
    atomicMax(&h.last[at], j);
    h.p[at] = p;  // (of repeated tokens add_repeated() takes care)
}
template <int K>
__device__ __forceinline__ int slot_of(const Hash<K> &h, int mask, int32_t token)  // of a token that is there
{
    int at = hash_of(token, mask);
    while (h.key[at] != token) at = (at + 1) & mask;
    return at;
}
template <int K>
__device__ __forceinline__ bool is_listed(const Hash<K> &h, int mask, int32_t token)
{
    int at = hash_of(token, mask);
    while (h.key[at] != token && h.key[at] != FREE) at = (at + 1) & mask;
    return h.key[at] == token;
}

// The sums of p of tokens that are listed more than once, as integers: p times the power of two that puts
// the token's largest p between 2^50 and 2^51, so that no order of the additions changes them.  (Added up
// entry after entry, each time from LDS, 8192 x 1500 with 512 random entries took 2.3 ms, 0.17 so.)
template <int K>
struct Repeats {
    uint32_t top[2 * K];  // the largest p's bits
    uint64_t sum[2 * K];
};
// Every thread of the block, if any token is repeated: entry threadIdx.x (token -1: none) and its p.
template <int K>
__device__ __forceinline__ void add_repeated(Repeats<K> &r, Hash<K> &h, int mask, int32_t token, float p)
{
    for (int i = (int)threadIdx.x; i <= mask; i += (int)blockDim.x) r.top[i] = 0, r.sum[i] = 0;
    __syncthreads();
    const int slot = token >= 0 ? slot_of(h, mask, token) : 0;
    const bool again = token >= 0 && h.first[slot] != h.last[slot];
    if (again) atomicMax(&r.top[slot], __float_as_uint(p));
    __syncthreads();
    const int e = again ? (int)(r.top[slot] >> 23) : 0;
    if (again) atomicAdd((unsigned long long *)&r.sum[slot], e < 255 ? (unsigned long long)ldexpf(p, 177 - e) : 0ull);
    __syncthreads();
    if (again && h.first[slot] == (int)threadIdx.x)  // (NaN comes out above every number, one with a sign above that)
        h.p[slot] = e >= 255 ? __uint_as_float(0x7FC00000u) : ldexpf((float)r.sum[slot], e - 177);
    __syncthreads();
}

// ---------------------------------------------------------------- entries
//
// Thread j has entry j of the teacher (k <= NT): its token (-1: none), logit and score.
struct Entry {
    int32_t token;
    float logit, score;
};
// An entry (and the row's weight) as loaded: taken apart only when it is needed, so that nothing waits for it.
struct RawEntry {
    uint32_t low, high, logit, score;
    float weight;
};
__device__ __forceinline__ void load_entry(const DistillArgs &a, int64_t row, RawEntry &r)
{
    r.weight = a.weights ? a.weights[row] : a.weight;
    if ((int)threadIdx.x >= a.k) return;
    const int64_t at = row * a.tokens_ld + threadIdx.x, from = row * a.teacher_ld + threadIdx.x;
    if (a.token_type == 3) {
        r.low = ((const uint32_t *)a.tokens)[at];
    } else {
        r.low = ((const uint32_t *)a.tokens)[2 * at];
        r.high = ((const uint32_t *)a.tokens)[2 * at + 1];
    }
    r.logit = a.teacher_type == 0 ? ((const uint32_t *)a.teacher)[from] : ((const uint16_t *)a.teacher)[from];
}
__device__ __forceinline__ Entry entry_of(const DistillArgs &a, const RawEntry &r)
{
    Entry e{-1, NONE, 0.f};
    if ((int)threadIdx.x >= a.k || r.low >= (uint32_t)a.vocab || (a.token_type != 3 && r.high != 0)) return e;
    e.token = (int32_t)r.low;
    const uint16_t h = (uint16_t)r.logit;
    __bf16 b;
    _Float16 f;
    __builtin_memcpy(&b, &h, 2);
    __builtin_memcpy(&f, &h, 2);
    e.logit = a.teacher_type == 0 ? __uint_as_float(r.logit) : a.teacher_type == 1 ? to_float(b) : to_float(f);
    return e;
}
template <typename T>
__device__ __forceinline__ void load_score(const Entry &e, const T *scores, RawEntry &r)
{
    if (e.token < 0) return;
    if (sizeof(T) == 4) r.score = ((const uint32_t *)scores)[e.token];
    else r.score = ((const uint16_t *)scores)[e.token];
}
template <typename T>
__device__ __forceinline__ float score_of(const Entry &e, const RawEntry &r)
{
    return e.token < 0 ? 0.f : column<T>(unit{r.score, 0, 0, 0}, 0);
}
__device__ __forceinline__ Soft soft_of(const Entry &e)
{
    return Soft{e.logit, e.logit > NONE ? 1.f : e.logit != e.logit ? e.logit : 0.f};
}
// An entry's p, and its part of the loss without T^2.
__device__ __forceinline__ float mass_of(const Entry &e, Soft teacher, float c)
{
    return e.token >= 0 ? part_of(e.logit, teacher.top, c) / teacher.sum : 0.f;
}
__device__ __forceinline__ float loss_of(const Entry &e, float p, Soft teacher, Soft s, float temperature)
{
    const float log_p = (e.logit - teacher.top) / temperature - __builtin_amdgcn_logf(teacher.sum) * LN2;
    const float log_q = s.sum == 0.f ? NONE : (e.score - s.top) / temperature - __builtin_amdgcn_logf(s.sum) * LN2;
    return p == 0.f ? 0.f : p * (log_p - log_q);
}
// The largest and the sum over a wave, in all of its lanes: exchanges inside rows of 16 lanes, then
// between them.
template <class F>
__device__ __forceinline__ float wave_all(float x, F with)
{
    const auto lane = [&](auto ctrl) {
        x = with(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, true)));
    };
    lane(std::integral_constant<int, 0xB1>());   // lane ^ 1
    lane(std::integral_constant<int, 0x4E>());   // lane ^ 2
    lane(std::integral_constant<int, 0x141>());  // the other four of eight
    lane(std::integral_constant<int, 0x140>());  // the other eight
    x = with(x, __shfl_xor(x, 16, WAVE));
    return with(x, __shfl_xor(x, 32, WAVE));
}
__device__ __forceinline__ float wave_total(float x)
{
    return wave_all(x, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ Soft wave_soft(Soft s, float c)
{
    const float top = wave_all(s.top, [](float a, float b) { return fmaxf(a, b); });
    return Soft{top, wave_total(top > NONE ? s.sum * part_of(s.top, top, c) : s.sum)};
}

// ---------------------------------------------------------------- a block for a row
//
// A row is read once: HELD units a thread stay in registers as they were loaded, between the sums and
// the gradient; what a longer row has beyond is read again.  A block goes from row to row, and loads
// the next one's units into the registers that the gradient's stores leave, so that loads, stores and
// exponentials of a block overlap although most often one block fills a CU.  Two barriers a row: after
// the sums, and after the teacher's entries were noted: a bit for each column of the held units, and a
// hash from token to entry, so that a unit is stored once, with its corrections (stored over
// the gradient afterwards, they cost 58 of 181 us at 20000 x 8192 in bf16 with 64 entries).
//
// Bound by the bytes: 4096 x 131072 in bf16 385 to 424 us (5.1 to 5.6 TB/s; 2 % less with an exponent of one
// operation, 7 % without exponentials), the loss alone of 2048 x 131072 87 us (6.2 TB/s).  Read
// again and not held, 4096 x 131072 took 596 us (of 507 at the time).  Four waves a SIMD leave 128 registers a
// thread: with 16 units held up to 6 of a thread's numbers that no row changes are in memory, and loaded once a
// row where they are needed (15 to 19 scalars lie in lanes of vector registers); the units stay.
//
// Units are counted from where 64 aligned bytes of the gradient's row start, and the columns before (head) and
// behind them (rest) go one by one, so that the gradient may go past the caches wherever rows start: parts
// of 64 bytes that two waves write there cost a read each, and through the caches 8192 x 50001 in
// bf16 took 385 us, 340 so.
template <typename T, typename TO, int NT, int HELD, bool GRAD>
__global__ void __launch_bounds__(NT, HELD > 4 || NT > 512 ? 4 : 5) k_distill(DistillArgs a)
{
    constexpr int N = 4, C = COLS<T>, NW = NT / WAVE;  // N units are added at once
    static_assert(HELD % N == 0, "whole steps");
    __shared__ Soft sums[NW], masses[NW];
    __shared__ float losses[NW];
    __shared__ int32_t alive[2][NW];
    __shared__ Hash<NT> hash[2];
    __shared__ Repeats<NT> repeats;
    __shared__ uint32_t columns[GRAD ? NT * HELD / 4 : 1];  // a byte for each held unit, a thread's together
    int t = (int)threadIdx.x;
    const int wave = wave_id(), entry_waves = (a.k + WAVE - 1) / WAVE, mask = hash_mask(a.k);
    const float c = LOG2E / a.temperature;
    constexpr int LINE = 64 / (int)sizeof(TO);
    struct Row {
        const T *scores;
        int32_t head, units, odd;  // columns before the units, units, columns that are in none
        __device__ __forceinline__ int32_t odd_column(int t) const { return t < head ? t : units * C + t; }
        __device__ __forceinline__ __amdgpu_buffer_rsrc_t from(bool on) const { return buffer(scores + head, on ? units * 16 : 0); }
    };
    const auto row_at = [&](int64_t row) {
        Row r;
        r.scores = (const T *)a.scores + row * a.ld;
        r.head = GRAD ? (int32_t)(-((uintptr_t)((const TO *)a.grad + row * a.grad_ld) / sizeof(TO)) % LINE) : 0;
        if (r.head > a.vocab) r.head = a.vocab;
        r.units = (a.vocab - r.head) / C;
        r.odd = a.vocab - r.units * C;
        return r;
    };
    static_assert(LINE + C <= WAVE, "a thread for each odd column");
    // Whether any entry of a row counts, from what each wave found; a barrier lies between.
    const auto note_alive = [&](int turn, const Entry &e) {
        const bool on = __any(!(e.logit == NONE));
        if (lane_id() == 0) alive[turn][wave] = on;
    };
    const auto is_alive = [&](int turn) {
        int32_t on = 0;
        for (int w = 0; w < entry_waves; ++w) on |= alive[turn][w];
        return on != 0;
    };

    unit r[HELD];
    T odd = from_float<T>(0.f);  // a column that is in no unit
    int64_t row = blockIdx.x;
    Row here = row_at(row);
    RawEntry raw{};
    load_entry(a, row, raw);
    Entry e = entry_of(a, raw);
    note_alive(1, e);
    if (GRAD) {
        clear(hash[0], mask);
#pragma unroll
        for (int i = 0; i < HELD / 4; ++i) columns[t * (HELD / 4) + i] = 0;
    }
    __syncthreads();
    bool on = is_alive(1);
    load_score(e, here.scores, raw);
    if (t < here.odd) odd = here.scores[here.odd_column(t)];
    {
        const __amdgpu_buffer_rsrc_t from = here.from(on);
#pragma unroll
        for (int i = 0; i < HELD; ++i) r[i] = load_unit<true>(from, t + i * NT);
    }
    for (int turn = 0;; turn ^= 1) {
        // (else every unit's place is worked out before the loop and kept)
        asm volatile("" : "+v"(t));
        const int32_t units = here.units;
        const bool more = row + gridDim.x < a.n;
        const int64_t next = more ? row + gridDim.x : row;
        RawEntry raw_next{};
        load_entry(a, next, raw_next);
        Soft s{NONE, 0.f};
        if (on) {
#pragma unroll
            for (int i = 0; i < HELD; i += N)
                if (i * NT < units) {
                    if ((i + N) * NT > units) {
#pragma unroll
                        for (int k = i; k < i + N; ++k)
                            if (t + k * NT >= units) r[k] = all_of<T>(NONE);
                    }
                    add_units<T, N>(s, r + i, c);
                    __builtin_amdgcn_sched_barrier(0);
                }
            const __amdgpu_buffer_rsrc_t from = here.from(true);
            for (int32_t u = HELD * NT + t; u < units; u += N * NT) {
                unit x[N];
#pragma unroll
                for (int k = 0; k < N; ++k) x[k] = load_unit<!GRAD>(from, u + k * NT);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (u + k * NT >= units) x[k] = all_of<T>(NONE);
                add_units<T, N>(s, x, c);
            }
            if (t < here.odd) {
                const float v = to_float(odd);
                join(s, Soft{v, v > NONE ? 1.f : v != v ? v : 0.f}, c);
            }
            s = wave_soft(s, c);
            if (lane_id() == 0) sums[wave] = s;
            if (wave < entry_waves) {
                const Soft m = wave_soft(soft_of(e), c);
                if (lane_id() == 0) masses[wave] = m;
            }
        }
        Entry f = entry_of(a, raw_next);
        note_alive(turn, f);
        __syncthreads();
        const bool next_on = more && is_alive(turn);
        const Row coming = row_at(next);
        const __amdgpu_buffer_rsrc_t from = coming.from(next_on);
        const T own = odd;
        if (next_on) {
            load_score(f, coming.scores, raw_next);
            if (t < coming.odd) odd = coming.scores[coming.odd_column(t)];
        }
        Soft m{NONE, 0.f};
        float p = 0.f;
        if (on) {
            s = sums[0];
#pragma unroll
            for (int w = 1; w < NW; ++w) join(s, sums[w], c);
            for (int w = 0; w < entry_waves; ++w) join(m, masses[w], c);
            if (wave < entry_waves) {
                e.score = score_of<T>(e, raw);
                p = mass_of(e, m, c);
                const float loss = wave_total(loss_of(e, p, m, s, a.temperature));
                if (lane_id() == 0) losses[wave] = loss;
                if (GRAD) {
                    if (e.token >= 0) {
                        note(hash[turn], mask, e.token, t, p);
                        const int32_t v = e.token - here.head, u = v / C, i = u / NT;
                        if (v >= 0 && u < units && i < HELD)
                            atomicOr(&columns[u % NT * (HELD / 4) + i / 4], 1u << (i % 4 * 8 + v % C));
                    }
                }
            }
        }
        if (GRAD) {
            clear(hash[turn ^ 1], mask);
            TO *grad = (TO *)a.grad + row * a.grad_ld;
            const __amdgpu_buffer_rsrc_t to = buffer(grad + here.head, units * C * (int)sizeof(TO));
            const float g = raw.weight * a.temperature;
            const float base = s.top > NONE ? s.top : 0.f, part = !on || s.sum == 0.f ? 0.f : 1.f / s.sum, by = part * g;
            __syncthreads();
            uint32_t mine[HELD / 4];
#pragma unroll
            for (int i = 0; i < HELD / 4; ++i) {
                mine[i] = columns[t * (HELD / 4) + i];
                columns[t * (HELD / 4) + i] = 0;
            }
            if (hash[turn].repeated)  // the same for all
                add_repeated(repeats, hash[turn], mask, e.token, p);
            const auto corrected = [&](int32_t token) { return hash[turn].p[slot_of(hash[turn], mask, token)] * g; };
            const auto store = [&](unit x, int32_t u, uint32_t bits) {
                float v[C];
                // (converted again: else the sums' fp32 values are kept in registers till here)
                asm("" : "+v"(x));
#pragma unroll
                for (int k = 0; k < C; ++k) v[k] = on ? part_of(column<T>(x, k), base, c) * by : 0.f;
                while (bits) {
                    const int at = __ffs(bits) - 1;
                    const float by_teacher = corrected(here.head + u * C + at);
#pragma unroll
                    for (int k = 0; k < C; ++k) v[k] -= k == at ? by_teacher : 0.f;
                    bits &= bits - 1;
                }
                store_unit<true, TO>(to, u, v);
            };
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                store(r[i], t + i * NT, mine[i / 4] >> (i % 4 * 8) & 0xFF);
                r[i] = load_unit<true>(from, t + i * NT);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (t < here.odd) {
                const int32_t at = here.odd_column(t);
                float v = on ? part_of(to_float(own), base, c) * by : 0.f;
                if (on && is_listed(hash[turn], mask, at)) v -= corrected(at);
                grad[at] = from_float<TO>(v);
            }
            if (units > HELD * NT) {  // the same for all: what was not held, corrected afterwards
                const __amdgpu_buffer_rsrc_t again = here.from(on);
                for (int32_t u = HELD * NT + t; u < units; u += NT) store(load_unit<true>(again, u), u, 0);
                __syncthreads();
                const int32_t v = e.token - here.head;
                if (on && e.token >= 0 && v / C >= HELD * NT && v < units * C && hash[turn].first[slot_of(hash[turn], mask, e.token)] == t)
                    grad[e.token] = from_float<TO>(part_of(e.score, base, c) * by - corrected(e.token));
            }
        } else {
#pragma unroll
            for (int i = 0; i < HELD; ++i) r[i] = load_unit<true>(from, t + i * NT);
            __syncthreads();
        }
        if (t == 0) {
            float loss = 0.f;
            if (on)
                for (int w = 0; w < entry_waves; ++w) loss += losses[w];
            a.loss[row] = loss * a.temperature * a.temperature;
        }
        if (!more) return;
        row = next;
        here = coming;
        e = f;
        raw = raw_next;
        on = next_on;
    }
}

// ---------------------------------------------------------------- few rows
//
// Rows too few to fill the card are cut into parts of whole units: sums of each part, then (a second
// launch) each block joins its row's and goes on with its part.  The entries' scores are kept by the
// first launch, for the second may store over them.
struct Parts {
    int32_t parts, columns;  // of a part, a multiple of 8
    Soft *sums;              // [n][parts]
    float *scores;           // [n][k]
};
// Parts so that there are two blocks a CU, of 4096 columns at least.  Whole rows and parts (us a call
// with gradient, of which the host takes 11 and, for two launches, 15): 131072 columns in bf16 1 row 18.9
// and 15.1, 64 rows 21.8 and 15.6, 128 rows 22.6 and 23.8; in fp32 64 rows 26.1 and 21.7, 128 rows 31.9
// and 42.0; 50001 columns in bf16 16 rows 15.3 and 15.3, 64 rows 16.1 and 15.3.
static Parts cut_rows(int64_t n, int32_t vocab, char *work)
{
    const int64_t most = (vocab + 4095) / 4096, want = n > 0 ? (2 * CUS + n - 1) / n : 1;
    const int64_t parts = n <= FEW_ROWS && vocab >= LONG_ROW ? (want < most ? want : most) : 1;
    const int32_t columns = (int32_t)(((vocab + parts - 1) / parts + 7) / 8 * 8);
    return Parts{(vocab + columns - 1) / columns, columns, (Soft *)work, nullptr};
}

template <typename T>
__global__ void __launch_bounds__(BLOCK) k_distill_part(DistillArgs a, Parts q)
{
    constexpr int N = 4, C = COLS<T>, NW = BLOCK / WAVE;
    __shared__ Soft sums[NW];
    const int64_t row = blockIdx.y;
    const int part = (int)blockIdx.x, t = (int)threadIdx.x;
    const float c = LOG2E / a.temperature;
    const T *scores = (const T *)a.scores + row * a.ld;
    const int32_t units = a.vocab / C, rest = a.vocab - units * C;
    const int32_t first = part * (q.columns / C);
    int32_t end = first + q.columns / C;
    if (end > units) end = units;
    const __amdgpu_buffer_rsrc_t from = buffer(scores, units * 16);
    Soft s{NONE, 0.f};
    for (int32_t u = first + t; u < end; u += N * BLOCK) {
        unit x[N];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = load_unit<false>(from, u + k * BLOCK);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (u + k * BLOCK >= end) x[k] = all_of<T>(NONE);
        add_units<T, N>(s, x, c);
    }
    if (part == q.parts - 1 && t < rest) {
        const float v = to_float(scores[units * C + t]);
        join(s, Soft{v, v > NONE ? 1.f : v != v ? v : 0.f}, c);
    }
    if (part == 0)
        for (int j = t; j < a.k; j += BLOCK) {
            const int64_t token = index_at(a.tokens, a.token_type, row * a.tokens_ld + j);
            q.scores[row * a.k + j] = token >= 0 && token < a.vocab ? to_float(scores[token]) : 0.f;
        }
    s = wave_soft(s, c);
    if (lane_id() == 0) sums[wave_id()] = s;
    __syncthreads();
    if (t == 0) {
#pragma unroll
        for (int w = 1; w < NW; ++w) join(s, sums[w], c);
        q.sums[row * q.parts + part] = s;
    }
}

template <typename T, typename TO, int NT, bool GRAD>
__global__ void __launch_bounds__(NT) k_distill_rest(DistillArgs a, Parts q)
{
    constexpr int N = 4, C = COLS<T>, NW = NT / WAVE;
    __shared__ Soft masses[NW];
    __shared__ float losses[NW];
    __shared__ Hash<NT> hash;
    __shared__ Repeats<NT> repeats;
    const int64_t row = blockIdx.y;
    const int part = (int)blockIdx.x, t = (int)threadIdx.x, wave = wave_id();
    const int entry_waves = (a.k + WAVE - 1) / WAVE, mask = hash_mask(a.k);
    const float c = LOG2E / a.temperature;
    const T *scores = (const T *)a.scores + row * a.ld;
    const int32_t units = a.vocab / C, rest = a.vocab - units * C;
    const int32_t first = part * (q.columns / C);
    int32_t end = first + q.columns / C;
    if (end > units) end = units;

    RawEntry raw{};
    load_entry(a, row, raw);
    Soft s{NONE, 0.f};
    for (int i = lane_id(); i < q.parts; i += WAVE) join(s, q.sums[row * q.parts + i], c);
    s = wave_soft(s, c);
    Entry e = entry_of(a, raw);
    if (e.token >= 0) e.score = q.scores[row * a.k + t];
    if (wave < entry_waves) {
        const Soft m = wave_soft(soft_of(e), c);
        if (lane_id() == 0) masses[wave] = m;
    }
    if (GRAD) clear(hash, mask);
    __syncthreads();
    Soft m{NONE, 0.f};
    for (int w = 0; w < entry_waves; ++w) join(m, masses[w], c);
    const bool on = !(m.sum == 0.f);
    float p = 0.f;
    if (on && wave < entry_waves) {
        p = mass_of(e, m, c);
        const float loss = wave_total(loss_of(e, p, m, s, a.temperature));
        if (lane_id() == 0) losses[wave] = loss;
        if (GRAD) {
            if (e.token >= 0) note(hash, mask, e.token, t, p);
        }
    }
    if (GRAD) {
        TO *grad = (TO *)a.grad + row * a.grad_ld;
        const __amdgpu_buffer_rsrc_t from = buffer(scores, on ? end * 16 : 0), to = buffer(grad, end * C * (int)sizeof(TO));
        const float g = raw.weight * a.temperature;
        const float base = s.top > NONE ? s.top : 0.f, by = !on || s.sum == 0.f ? 0.f : g / s.sum;
        for (int32_t u = first + t; u < end; u += N * NT) {
            unit x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = load_unit<false>(from, u + i * NT);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float v[C];
#pragma unroll
                for (int k = 0; k < C; ++k) v[k] = on ? part_of(column<T>(x[i], k), base, c) * by : 0.f;
                store_unit<false, TO>(to, u + i * NT, v);
            }
        }
        const bool own_rest = part == q.parts - 1;
        if (own_rest && t < rest)
            grad[units * C + t] = from_float<TO>(on ? part_of(to_float(scores[units * C + t]), base, c) * by : 0.f);
        __syncthreads();  // the teacher's columns again, over what was stored
        if (hash.repeated) add_repeated(repeats, hash, mask, on ? e.token : -1, p);  // the same for all
        if (on && e.token >= 0 && ((e.token >= first * C && e.token < end * C) || (own_rest && e.token >= units * C)) &&
            hash.first[slot_of(hash, mask, e.token)] == t)
            grad[e.token] = from_float<TO>(part_of(e.score, base, c) * by - hash.p[slot_of(hash, mask, e.token)] * g);
    } else {
        __syncthreads();
    }
    if (part == 0 && t == 0) {
        float loss = 0.f;
        if (on)
            for (int w = 0; w < entry_waves; ++w) loss += losses[w];
        a.loss[row] = loss * a.temperature * a.temperature;
    }
}

int64_t distill_workspace(int64_t n, int32_t vocab, int32_t k, bool)
{
    const Parts q = cut_rows(n, vocab, nullptr);
    return q.parts > 1 ? n * (q.parts * (int64_t)sizeof(Soft) + k * (int64_t)sizeof(float)) : 0;
}

hipError_t run_distill(const DistillArgs &given, hipStream_t s)
{
    return with_type(given.type, [&](auto ti) {
        return with_type(given.grad ? given.grad_type : 0, [&](auto to) {
            using T = decltype(ti);
            using TO = decltype(to);
            const int64_t units = given.vocab / COLS<T>;
            const auto go = [&](auto kern, int nt, int waves) {
                const int64_t blocks = waves ? CUS * waves * WAVE / nt : LAUNCH_BLOCKS / 4;  // (of up to 1024 threads)
                return launch(kern, dim3((unsigned)(given.n < blocks ? given.n : blocks)), dim3(nt), s, given);
            };
            Parts q = cut_rows(given.n, given.vocab, given.work);
            if (q.parts > 1) {
                q.scores = (float *)(q.sums + given.n * q.parts);
                const dim3 grid((unsigned)q.parts, (unsigned)given.n), one(1, (unsigned)given.n);
                const hipError_t e = launch(k_distill_part<T>, grid, dim3(BLOCK), s, given, q);
                if (e != hipSuccess) return e;
                if (!given.grad)
                    return given.k <= 256 ? launch(k_distill_rest<T, float, 256, false>, one, dim3(256), s, given, q)
                                          : launch(k_distill_rest<T, float, 1024, false>, one, dim3(1024), s, given, q);
                return given.k <= 256 ? launch(k_distill_rest<T, TO, 256, true>, grid, dim3(256), s, given, q)
                                      : launch(k_distill_rest<T, TO, 1024, true>, grid, dim3(1024), s, given, q);
            }
            if (!given.grad) {
                if (given.k <= 64 && units <= 64 * 8) return go(k_distill<T, float, 64, 4, false>, 64, 0);
                if (given.k <= 256 && (given.n > CUS || units <= 1024)) return go(k_distill<T, float, 256, 4, false>, 256, 0);
                return go(k_distill<T, float, 1024, 4, false>, 1024, 0);
            }
            if (given.k <= 64 && units <= 64 * 4) return go(k_distill<T, TO, 64, 4, true>, 64, 20);
            if (given.k <= 64 && units <= 64 * 16) return go(k_distill<T, TO, 64, 16, true>, 64, 16);
            if (given.k <= 256 && units <= 256 * 4) return go(k_distill<T, TO, 256, 4, true>, 256, 20);
            if (given.k <= 256 && units <= 256 * 16) return go(k_distill<T, TO, 256, 16, true>, 256, 16);
            if (given.k <= 512 && units <= 512 * 4) return go(k_distill<T, TO, 512, 4, true>, 512, 16);
            if (given.k <= 512 && units <= 512 * 16) return go(k_distill<T, TO, 512, 16, true>, 512, 16);
            return go(k_distill<T, TO, 1024, 16, true>, 1024, 16);
        });
    });
}

}  // namespace sp
