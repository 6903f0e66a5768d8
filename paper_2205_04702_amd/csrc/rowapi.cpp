// C entry points of the operators on token tables and 8-bit rows: checks of the
// arguments, then launches on the caller's stream.  They hold no state, allocate
// nothing and wait for nothing.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/scratchpipe.h"
#include "sp_internal.h"
#include "sp_rows.h"

using namespace sp;

namespace {

static_assert(SP_F32 == 0 && SP_BF16 == 1 && SP_F16 == 2 && SP_I32 == 3 && SP_I64 == 4 && SP_I8 == 5 && SP_F8 == 6,
              "the kernels' numbers of the element types");

constexpr int64_t MAX_N = 0x7FFFFFFF;      // rows of one call
constexpr int64_t MAX_DIM = 1 << 20;       // columns of a table, gradient or cache
constexpr int64_t MAX_WIDTH = 1 << 30;     // columns of dropout's rows
constexpr int64_t MAX_LD = 1ll << 40;
constexpr int64_t MAX_K = 131071;          // 128 * 128 * k stays within 32 bits

sp_status bad(const char *fmt, ...) __attribute__((format(printf, 1, 2)));
sp_status bad(const char *fmt, ...)
{
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return set_error(SP_ERR_INVALID_ARG, buf);
}

bool is_float(int32_t t) { return t == SP_F32 || t == SP_BF16 || t == SP_F16; }
bool is_index(int32_t t) { return t == SP_I32 || t == SP_I64; }
uint64_t size_of(int32_t t)
{
    return t == SP_F32 || t == SP_I32 ? 4 : t == SP_BF16 || t == SP_F16 ? 2 : t == SP_I64 ? 8 : 1;
}
bool misaligned(const void *p, int32_t type) { return (uintptr_t)p % size_of(type) != 0; }

// 65536 p, rounded; false where p is no probability below 1 or rounds to 1.
bool drop_bits(float p, uint32_t *out)
{
    if (!(p >= 0.f && p < 1.f)) return false;
    *out = (uint32_t)std::floor((double)p * 65536.0 + 0.5);
    return *out < 65536;
}
Drop drop_of(uint32_t bits, uint64_t seed, uint64_t offset)
{
    return Drop{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32),
                bits};
}
float factor_of(double scale, uint32_t bits) { return (float)(scale * (65536.0 / (65536.0 - bits))); }

sp_status done(hipError_t e, const char *what)
{
    if (e == hipSuccess) return SP_OK;
    char buf[256];
    snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
    return set_error(SP_ERR_HIP, buf);
}

// One matrix of a call: pointer, type, row stride.
sp_status check_rows(const char *what, const void *p, int32_t type, int64_t n, int64_t dim, int64_t ld)
{
    if (n > 0 && !p) return bad("null %s", what);
    if (misaligned(p, type)) return bad("%s is not aligned to its element type", what);
    if (ld < dim || ld > MAX_LD) return bad("row stride %lld of %s not in %lld..2^40", (long long)ld, what, (long long)dim);
    return SP_OK;
}

}  // namespace

#define TRY(x)                        \
    do {                              \
        const sp_status _s = (x);     \
        if (_s != SP_OK) return _s;   \
    } while (0)

extern "C" sp_status sp_lookup(const void *tokens, int32_t token_type, int64_t n, const void *table,
                               int32_t table_type, int64_t rows, int64_t dim, int64_t table_ld,
                               float scale, float p, uint64_t seed, uint64_t offset, void *out,
                               int32_t out_type, int64_t out_ld, void *stream)
{
    uint32_t bits;
    if (!is_index(token_type)) return bad("token type %d", token_type);
    if (!is_float(table_type) || !is_float(out_type)) return bad("element type of the table or the output");
    if (n < 0 || n > MAX_N) return bad("%lld tokens", (long long)n);
    if (rows < 0 || rows > MAX_N) return bad("%lld rows", (long long)rows);
    if (dim < 1 || dim > MAX_DIM) return bad("dim %lld not in 1..%lld", (long long)dim, (long long)MAX_DIM);
    if (!drop_bits(p, &bits)) return bad("p %g not in 0 .. 1 - 2^-17", (double)p);
    TRY(check_rows("tokens", tokens, token_type, n, 1, 1));
    TRY(check_rows("table", table, table_type, rows, dim, table_ld));
    TRY(check_rows("output", out, out_type, n, dim, out_ld));
    if (n == 0) return SP_OK;
    const LookupArgs a{tokens, token_type, n, table, table_type, rows, table_ld, (int32_t)dim,
                       factor_of(scale, bits), drop_of(bits, seed, offset), out, out_type, out_ld};
    return done(run_lookup(a, (hipStream_t)stream), "sp_lookup");
}

extern "C" sp_status sp_lookup_grad_workspace(int64_t n, int64_t rows, int64_t dim, int64_t *bytes)
{
    if (!bytes) return bad("null bytes");
    if (n < 0 || n > MAX_N) return bad("%lld tokens", (long long)n);
    if (rows < 0 || rows > MAX_N) return bad("%lld rows", (long long)rows);
    if (dim < 1 || dim > MAX_DIM) return bad("dim %lld not in 1..%lld", (long long)dim, (long long)MAX_DIM);
    *bytes = grad_workspace(n, rows, (int32_t)dim);
    return SP_OK;
}

extern "C" sp_status sp_lookup_grad(const void *tokens, int32_t token_type, int64_t n,
                                    const void *grad, int32_t grad_type, int64_t dim, int64_t grad_ld,
                                    float scale, float p, uint64_t seed, uint64_t offset, void *out,
                                    int32_t out_type, int64_t rows, int64_t out_ld,
                                    int32_t accumulate, void *workspace, int64_t workspace_bytes,
                                    void *stream)
{
    uint32_t bits;
    int64_t need = 0;
    if (!is_index(token_type)) return bad("token type %d", token_type);
    if (!is_float(grad_type) || !is_float(out_type)) return bad("element type of the gradient or the output");
    TRY(sp_lookup_grad_workspace(n, rows, dim, &need));
    if (!drop_bits(p, &bits)) return bad("p %g not in 0 .. 1 - 2^-17", (double)p);
    TRY(check_rows("tokens", tokens, token_type, n, 1, 1));
    TRY(check_rows("gradient", grad, grad_type, n, dim, grad_ld));
    TRY(check_rows("output", out, out_type, rows, dim, out_ld));
    if (rows == 0) return SP_OK;
    if (need > 0 && (!workspace || workspace_bytes < need))
        return bad("workspace of %lld bytes, %lld needed", (long long)(workspace ? workspace_bytes : 0),
                   (long long)need);
    if (need > 0 && (uintptr_t)workspace % 16 != 0) return bad("workspace is not aligned to 16 bytes");
    const GradArgs a{tokens, token_type, n, grad, grad_type, grad_ld, (int32_t)dim,
                     factor_of(scale, bits), drop_of(bits, seed, offset), out, out_type, rows, out_ld,
                     accumulate != 0, (char *)workspace};
    return done(run_grad(a, (hipStream_t)stream), "sp_lookup_grad");
}

extern "C" sp_status sp_dropout(const void *x, int32_t type, int64_t n, int64_t dim, int64_t x_ld,
                                const void *residual, int64_t residual_ld, float p, uint64_t seed,
                                uint64_t offset, void *out, int64_t out_ld, void *stream)
{
    uint32_t bits;
    if (!is_float(type)) return bad("element type %d", type);
    if (n < 0 || n > MAX_N) return bad("%lld rows", (long long)n);
    if (dim < 1 || dim > MAX_WIDTH) return bad("dim %lld not in 1..2^30", (long long)dim);
    if (!drop_bits(p, &bits)) return bad("p %g not in 0 .. 1 - 2^-17", (double)p);
    TRY(check_rows("input", x, type, n, dim, x_ld));
    if (residual) TRY(check_rows("residual", residual, type, n, dim, residual_ld));
    TRY(check_rows("output", out, type, n, dim, out_ld));
    if (n == 0) return SP_OK;
    const DropoutArgs a{x, residual, type, n, (int32_t)dim, x_ld, residual_ld, factor_of(1.0, bits),
                        drop_of(bits, seed, offset), out, out_ld};
    return done(run_dropout(a, (hipStream_t)stream), "sp_dropout");
}

static sp_status check_cache(const void *index, int32_t index_type, int64_t n, const void *q, int32_t kind,
                             int64_t slots, int64_t q_ld, const float *scales, int64_t scales_ld,
                             int64_t dim, int64_t group, const void *x, int32_t type, int64_t x_ld)
{
    if (index && !is_index(index_type)) return bad("index type %d", index_type);
    if (kind != SP_I8 && kind != SP_F8) return bad("cache type %d", kind);
    if (!is_float(type)) return bad("element type %d", type);
    if (n < 0 || n > MAX_N) return bad("%lld rows", (long long)n);
    if (slots < 0 || slots > MAX_N) return bad("%lld slots", (long long)slots);
    if (dim < 1 || dim > MAX_DIM) return bad("dim %lld not in 1..%lld", (long long)dim, (long long)MAX_DIM);
    if (group < 1 || group > dim || dim % group != 0 || (group != dim && group % 8 != 0))
        return bad("group %lld: a divisor of dim %lld that is dim itself or a multiple of 8",
                   (long long)group, (long long)dim);
    if (index) TRY(check_rows("index", index, index_type, n, 1, 1));
    TRY(check_rows("cache", q, kind, slots, dim, q_ld));
    TRY(check_rows("scales", scales, SP_F32, slots, dim / group, scales_ld));
    TRY(check_rows("rows", x, type, n, dim, x_ld));
    if (!index && n > slots) return bad("%lld rows without an index, %lld slots", (long long)n, (long long)slots);
    return SP_OK;
}

extern "C" sp_status sp_cache_write(const void *x, int32_t type, int64_t n, int64_t dim, int64_t x_ld,
                                    const void *index, int32_t index_type, int64_t group, void *q,
                                    int32_t kind, int64_t slots, int64_t q_ld, float *scales,
                                    int64_t scales_ld, void *stream)
{
    TRY(check_cache(index, index_type, n, q, kind, slots, q_ld, scales, scales_ld, dim, group, x, type, x_ld));
    if (n == 0) return SP_OK;
    const CacheArgs a{index, index ? index_type : SP_I32, n, q, kind, slots, q_ld, scales, scales_ld,
                      (int32_t)dim, (int32_t)group, const_cast<void *>(x), type, x_ld};
    return done(run_cache_write(a, (hipStream_t)stream), "sp_cache_write");
}

extern "C" sp_status sp_cache_read(const void *q, int32_t kind, int64_t slots, int64_t dim, int64_t q_ld,
                                   const float *scales, int64_t scales_ld, int64_t group,
                                   const void *index, int32_t index_type, int64_t n, void *out,
                                   int32_t out_type, int64_t out_ld, void *stream)
{
    TRY(check_cache(index, index_type, n, q, kind, slots, q_ld, scales, scales_ld, dim, group, out, out_type,
                    out_ld));
    if (n == 0) return SP_OK;
    const CacheArgs a{index, index ? index_type : SP_I32, n, const_cast<void *>(q), kind, slots, q_ld,
                      const_cast<float *>(scales), scales_ld, (int32_t)dim, (int32_t)group, out, out_type,
                      out_ld};
    return done(run_cache_read(a, (hipStream_t)stream), "sp_cache_read");
}

extern "C" sp_status sp_product_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes)
{
    if (!bytes) return bad("null bytes");
    if (m < 0 || m > MAX_N || n < 0 || n > MAX_N) return bad("%lld x %lld outputs", (long long)m, (long long)n);
    if (k < 1 || k > MAX_K) return bad("k %lld not in 1..%lld", (long long)k, (long long)MAX_K);
    *bytes = product_workspace(m, n, k);
    return SP_OK;
}

extern "C" sp_status sp_product(const int8_t *x, const float *x_scales, int64_t m, int64_t x_ld,
                                const int8_t *w, const float *w_scales, int64_t n, int64_t w_ld,
                                int64_t k, void *out, int32_t out_type, int64_t out_ld, void *workspace,
                                int64_t workspace_bytes, void *stream)
{
    int64_t need = 0;
    if (!is_float(out_type)) return bad("element type %d", out_type);
    TRY(sp_product_workspace(m, n, k, &need));
    if (m == 0 || n == 0) return SP_OK;
    TRY(check_rows("x", x, SP_I8, m, k, x_ld));
    TRY(check_rows("w", w, SP_I8, n, k, w_ld));
    TRY(check_rows("x's scales", x_scales, SP_F32, m, 1, 1));
    TRY(check_rows("w's scales", w_scales, SP_F32, n, 1, 1));
    TRY(check_rows("output", out, out_type, m, n, out_ld));
    if (need > 0 && (!workspace || workspace_bytes < need))
        return bad("workspace of %lld bytes, %lld needed", (long long)(workspace ? workspace_bytes : 0),
                   (long long)need);
    if (need > 0 && (uintptr_t)workspace % 16 != 0) return bad("workspace is not aligned to 16 bytes");
    const ProductArgs a{x, w, x_scales, w_scales, m, n, (int32_t)k, x_ld, w_ld, out, out_type, out_ld,
                        (char *)workspace};
    return done(run_product(a, (hipStream_t)stream), "sp_product");
}
