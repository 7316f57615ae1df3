// Host side of include/lora_experts.h: every argument is checked here, before the device is touched.
#include "../../include/lora_experts.h"
#include "lora_experts.h"
#include "lora_internal.h"

#include <cstdarg>
#include <cstdio>

static_assert(LORA_MAX_EXPERTS == lora::kMaxExperts, "the header states the kernels' limit");

static lora_status_t fail(lora_status_t st, const char *fmt, ...)
{
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    return (lora_status_t)lora::report(st, text);
}

static lora_status_t of_hip(hipError_t e, const char *what)
{
    return e == hipSuccess ? LORA_OK : fail(LORA_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

// (nothing below throws: no containers, no new)
#define TRY(call)                            \
    do {                                     \
        const lora_status_t st_ = (call);    \
        if (st_ != LORA_OK) return st_;      \
    } while (0)

static lora_status_t check_sizes(int32_t in, int32_t out)
{
    if (in <= 0 || in % 64 || out <= 0 || out % 128)
        return fail(LORA_ERR_SHAPE, "in_features (%d) must be a positive multiple of 64 and out_features (%d) of 128", in, out);
    // (bytes of a row then fit 32 bits, those of all experts 63)
    if (in > LORA_EXPERTS_MAX_FEATURES || out > LORA_EXPERTS_MAX_FEATURES)
        return fail(LORA_ERR_SHAPE, "in_features (%d) or out_features (%d) beyond %d", in, out, LORA_EXPERTS_MAX_FEATURES);
    return LORA_OK;
}

static lora_status_t check_rows(const void *p, int64_t ld, int64_t row, int64_t unit, const char *what)
{
    if (!p) return fail(LORA_ERR_INVALID_ARG, "%s is NULL", what);
    if (((uintptr_t)p) % 16) return fail(LORA_ERR_INVALID_ARG, "%s is not 16-byte aligned", what);
    if (ld < row || ld % unit || ld > INT64_MAX / 4 / INT32_MAX)
        return fail(LORA_ERR_INVALID_ARG, "row stride of %s (%lld) must be a multiple of %lld of at least %lld", what, (long long)ld, (long long)unit,
                    (long long)row);
    return LORA_OK;
}

static lora_status_t check_values(const void *p, const char *what)
{
    if (!p || ((uintptr_t)p) % 4) return fail(LORA_ERR_INVALID_ARG, "%s is NULL or not 4-byte aligned", what);
    return LORA_OK;
}

static lora_status_t check_scales(const float *p, int64_t ld, int32_t blocks)
{
    TRY(check_values(p, "scales"));
    if (ld < blocks || ld > INT64_MAX / 8 / INT32_MAX) return fail(LORA_ERR_INVALID_ARG, "row stride of scales (%lld) must be at least %d", (long long)ld, blocks);
    return LORA_OK;
}

static lora_status_t check_experts(int32_t n)
{
    if (n < 1 || n > LORA_MAX_EXPERTS) return fail(LORA_ERR_SHAPE, "n_experts (%d) outside 1..%d", n, LORA_MAX_EXPERTS);
    return LORA_OK;
}

static lora_status_t check_picks(int64_t tokens, int32_t picks)
{
    if (tokens < 0) return fail(LORA_ERR_INVALID_ARG, "tokens = %lld", (long long)tokens);
    if (picks < 1 || picks > LORA_MAX_PICKS) return fail(LORA_ERR_SHAPE, "picks (%d) outside 1..%d", picks, LORA_MAX_PICKS);
    if (tokens * picks > INT32_MAX) return fail(LORA_ERR_SHAPE, "%lld tokens x %d picks do not fit 32 bits", (long long)tokens, picks);
    return LORA_OK;
}

static lora_status_t check_packed(const void *p)
{
    if (!p || ((uintptr_t)p) % 256) return fail(LORA_ERR_INVALID_ARG, "the packed weights are NULL or not 256-byte aligned");
    return LORA_OK;
}

static inline int32_t blocks_of(int32_t in) { return (int32_t)(((int64_t)in + lora::kScaleBlock - 1) / lora::kScaleBlock); }

// pieces of 128 bytes of a row
static inline int32_t pieces_of(int32_t in, int bits) { return bits == 16 ? in / 64 : blocks_of(in); }

extern "C" lora_status_t lora_rows_quantize(const void *x, int64_t ldx, int64_t rows, int32_t in_features, void *q, int64_t ldq, float *scales,
                                            int64_t ld_scales, void *stream)
{
    if (rows < 0 || rows > INT32_MAX) return fail(LORA_ERR_INVALID_ARG, "rows = %lld", (long long)rows);
    TRY(check_sizes(in_features, 128));
    if (rows == 0) return LORA_OK;
    const int32_t blocks = blocks_of(in_features);
    TRY(check_rows(x, ldx, in_features, 8, "x"));
    TRY(check_rows(q, ldq, (int64_t)blocks * lora::kScaleBlock, 16, "q"));
    TRY(check_scales(scales, ld_scales, blocks));
    return of_hip(lora::launch_rows_quantize((const uint16_t *)x, ldx, rows, in_features, (uint8_t *)q, ldq, scales, ld_scales, (hipStream_t)stream),
                  "lora_rows_quantize");
}

static lora_status_t packed_bytes(int32_t n_experts, int32_t in, int32_t out, int32_t bits, size_t *bytes)
{
    TRY(check_experts(n_experts));
    TRY(check_sizes(in, out));
    if (bits != 16 && bits != 8) return fail(LORA_ERR_INVALID_ARG, "bits = %d: 16 (bf16) or 8 (E4M3)", bits);
    *bytes = (size_t)n_experts * out * pieces_of(in, bits) * lora::kPieceBytes;
    return LORA_OK;
}

extern "C" lora_status_t lora_experts_packed_bytes(int32_t n_experts, int32_t in_features, int32_t out_features, int32_t bits, size_t *bytes)
{
    if (!bytes) return fail(LORA_ERR_INVALID_ARG, "bytes is NULL");
    return packed_bytes(n_experts, in_features, out_features, bits, bytes);
}

extern "C" lora_status_t lora_experts_pack_weight(const void *w, int32_t n_experts, int32_t in_features, int32_t out_features, int32_t bits,
                                                  void *dev_packed, size_t packed, void *stream)
{
    size_t need = 0;
    TRY(packed_bytes(n_experts, in_features, out_features, bits, &need));
    TRY(check_rows(w, in_features, in_features, 1, "w"));
    TRY(check_packed(dev_packed));
    if (packed < need) return fail(LORA_ERR_OOM, "the packed weights need %zu bytes, %zu are there", need, packed);
    const int row_bytes = bits == 16 ? 2 * in_features : blocks_of(in_features) * lora::kScaleBlock;
    return of_hip(lora::launch_experts_pack((const char *)w, n_experts, row_bytes, bits == 16 ? row_bytes : in_features, out_features, bits == 8,
                                            (char *)dev_packed, (hipStream_t)stream),
                  "lora_experts_pack_weight");
}

// the product's arguments that its four entry points share; LORA_OK with a.n_rows == 0 where there is nothing to do
static lora_status_t check_product(lora::ExpertsArgs &a, int bits, const void *x, int64_t ldx, const float *scales, int64_t ld_scales, int32_t in,
                                   const void *w_packed, const float *w_scales, int32_t out, void *y, int64_t ldy)
{
    TRY(check_sizes(in, out));
    if (a.tokens < 0 || a.n_rows < 0) return fail(LORA_ERR_INVALID_ARG, "%d rows of x, %d of y", a.tokens, a.n_rows);
    if (a.n_rows == 0 || a.tokens == 0) {
        a.n_rows = 0;
        return LORA_OK;
    }
    a.pieces = pieces_of(in, bits);
    TRY(check_rows(x, ldx, bits == 16 ? in : (int64_t)a.pieces * lora::kPieceBytes, bits == 16 ? 8 : 16, bits == 16 ? "x" : "q"));
    if (bits == 8) {
        TRY(check_scales(scales, ld_scales, a.pieces));
        TRY(check_values(w_scales, "w_scales"));
    }
    // (the kernels take rows of x by 32-bit numbers of 16 bytes, and their scales by 32-bit indices)
    if ((a.tokens - 1) * (bits == 16 ? ldx / 8 : ldx / 16) > UINT32_MAX - 8 || (bits == 8 && (a.tokens - 1) * ld_scales > UINT32_MAX))
        return fail(LORA_ERR_SHAPE, "%d rows with a stride of %lld take more than 64 GiB, or their scales more than 16", a.tokens, (long long)ldx);
    TRY(check_packed(w_packed));
    TRY(check_rows(y, ldy, out, 8, "y"));
    a.x = (const char *)x;
    a.ldx_bytes = bits == 16 ? 2 * ldx : ldx;
    a.x_scales = scales;
    a.ld_scales = ld_scales;
    a.w = (const char *)w_packed;
    a.w_scales = w_scales;
    a.out = out;
    a.y = (uint16_t *)y;
    a.ldy = ldy;
    return LORA_OK;
}

static lora_status_t launch_product(const lora::ExpertsArgs &a, int bits, void *stream, const char *what)
{
    const hipError_t e = lora::launch_experts_linear(a, bits == 8, (hipStream_t)stream);
    if (e == hipErrorInvalidConfiguration)
        return fail(LORA_ERR_SHAPE, "%s: %d rows of %d experts x %d out_features are more tiles than a launch can have", what, a.n_rows, a.n_experts, a.out);
    return of_hip(e, what);
}

extern "C" lora_status_t lora_linear_scaled(const void *q, int64_t ldq, const float *scales, int64_t ld_scales, int32_t rows, int32_t in_features,
                                            const void *w_packed, const float *w_scales, int32_t out_features, void *y, int64_t ldy, void *stream)
{
    lora::ExpertsArgs a = {};
    a.tokens = a.n_rows = rows;
    a.n_experts = a.picks = 1;
    TRY(check_product(a, 8, q, ldq, scales, ld_scales, in_features, w_packed, w_scales, out_features, y, ldy));
    return a.n_rows == 0 ? LORA_OK : launch_product(a, 8, stream, "lora_linear_scaled");
}

static lora_status_t experts_linear(int bits, const void *x, int64_t ldx, const float *scales, int64_t ld_scales, int32_t tokens,
                                    const int32_t *starts, const int32_t *order, int32_t picks, int32_t n_rows, int32_t n_experts, int32_t in,
                                    const void *w_packed, const float *w_scales, int32_t out, void *y, int64_t ldy, void *stream, const char *what)
{
    TRY(check_experts(n_experts));
    if (order) {
        TRY(check_picks(tokens, picks));
        if (n_rows != tokens * picks) return fail(LORA_ERR_INVALID_ARG, "n_rows (%d) is not tokens (%d) x picks (%d)", n_rows, tokens, picks);
    } else if (n_rows != tokens)
        return fail(LORA_ERR_INVALID_ARG, "without an order n_rows (%d) is tokens (%d)", n_rows, tokens);
    lora::ExpertsArgs a = {};
    a.tokens = tokens;
    a.starts = starts;
    a.order = order;
    a.picks = order ? picks : 1;
    a.n_rows = n_rows;
    a.n_experts = n_experts;
    TRY(check_product(a, bits, x, ldx, scales, ld_scales, in, w_packed, w_scales, out, y, ldy));
    if (a.n_rows == 0) return LORA_OK;
    TRY(check_values(starts, "starts"));
    if (order) TRY(check_values(order, "order"));
    return launch_product(a, bits, stream, what);
}

extern "C" lora_status_t lora_experts_linear(const void *x, int64_t ldx, int32_t tokens, const int32_t *starts, const int32_t *order, int32_t picks,
                                             int32_t n_rows, int32_t n_experts, int32_t in_features, const void *w_packed, int32_t out_features,
                                             void *y, int64_t ldy, void *stream)
{
    return experts_linear(16, x, ldx, nullptr, 0, tokens, starts, order, picks, n_rows, n_experts, in_features, w_packed, nullptr, out_features, y, ldy,
                          stream, "lora_experts_linear");
}

extern "C" lora_status_t lora_experts_linear_scaled(const void *q, int64_t ldq, const float *scales, int64_t ld_scales, int32_t tokens,
                                                    const int32_t *starts, const int32_t *order, int32_t picks, int32_t n_rows, int32_t n_experts,
                                                    int32_t in_features, const void *w_packed, const float *w_scales, int32_t out_features, void *y,
                                                    int64_t ldy, void *stream)
{
    return experts_linear(8, q, ldq, scales, ld_scales, tokens, starts, order, picks, n_rows, n_experts, in_features, w_packed, w_scales, out_features, y,
                          ldy, stream, "lora_experts_linear_scaled");
}

extern "C" lora_status_t lora_experts_group_workspace_bytes(int64_t n_picks, int32_t n_experts, size_t *bytes)
{
    if (!bytes) return fail(LORA_ERR_INVALID_ARG, "bytes is NULL");
    if (n_picks < 0 || n_picks > INT32_MAX) return fail(LORA_ERR_INVALID_ARG, "n_picks = %lld", (long long)n_picks);
    TRY(check_experts(n_experts));
    *bytes = lora::group_counts(n_picks) ? (size_t)lora::group_most_chunks(n_picks) * n_experts * sizeof(int32_t) : 0;
    return LORA_OK;
}

extern "C" lora_status_t lora_experts_group(const int32_t *ids, int64_t ld_ids, int32_t tokens, int32_t picks, int32_t n_experts, int32_t *starts,
                                            int32_t *order, int32_t *place, void *workspace, size_t ws_bytes, void *stream)
{
    TRY(check_picks(tokens, picks));
    TRY(check_experts(n_experts));
    const int64_t n = (int64_t)tokens * picks;
    const size_t need = lora::group_counts(n) ? (size_t)lora::group_chunks(n) * n_experts * sizeof(int32_t) : 0;
    TRY(check_values(starts, "starts"));
    if (tokens > 0) {
        TRY(check_values(ids, "ids"));
        TRY(check_values(order, "order"));
        TRY(check_values(place, "place"));
        if (ld_ids < picks || ld_ids > INT64_MAX / 8 / INT32_MAX) return fail(LORA_ERR_INVALID_ARG, "row stride of ids (%lld) must be at least picks (%d)", (long long)ld_ids, picks);
    }
    if (need > 0 && (!workspace || ((uintptr_t)workspace) % 16 || ws_bytes < need))
        return fail(LORA_ERR_WORKSPACE, "a 16-byte aligned workspace of %zu bytes is needed, %zu are there", need, workspace ? ws_bytes : (size_t)0);
    return of_hip(lora::launch_experts_group(ids, ld_ids, tokens, picks, n_experts, starts, order, place, (int32_t *)workspace, (hipStream_t)stream),
                  "lora_experts_group");
}

extern "C" lora_status_t lora_experts_combine(const void *y, int64_t ldy, int32_t n_rows, const int32_t *place, const float *weights, int32_t tokens,
                                              int32_t picks, int32_t out_features, void *z, int64_t ldz, void *stream)
{
    TRY(check_picks(tokens, picks));
    TRY(check_sizes(64, out_features));
    if (n_rows < 0) return fail(LORA_ERR_INVALID_ARG, "n_rows = %d", n_rows);
    if (tokens == 0) return LORA_OK;
    if (n_rows > 0) TRY(check_rows(y, ldy, out_features, 8, "y"));
    TRY(check_values(place, "place"));
    TRY(check_values(weights, "weights"));
    TRY(check_rows(z, ldz, out_features, 8, "z"));
    return of_hip(lora::launch_experts_combine((const uint16_t *)y, ldy, n_rows, place, weights, tokens, picks, out_features, (uint16_t *)z, ldz,
                                               (hipStream_t)stream),
                  "lora_experts_combine");
}
