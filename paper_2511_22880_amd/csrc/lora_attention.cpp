// Host side of include/lora_attention.h: every argument is checked here, before the device is touched.
#include "../../include/lora_attention.h"
#include "lora_attention.h"
#include "lora_internal.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

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

// rows of heads: a token's and a head's stride
static lora_status_t check_heads(const void *p, int64_t token, int64_t head, int32_t heads, int32_t dim, const char *what)
{
    if (!p || ((uintptr_t)p) % 16) return fail(LORA_ERR_INVALID_ARG, "%s is NULL or not 16-byte aligned", what);
    constexpr int64_t kMost = INT64_MAX / 4 / INT32_MAX;
    if (token < 0 || token % 8 || token > kMost || (heads > 1 && (head < dim || head > kMost)) || head % 8 || head < 0)
        return fail(LORA_ERR_INVALID_ARG, "strides of %s (%lld a token, %lld a head) must be multiples of 8, a head's of at least %d", what,
                    (long long)token, (long long)head, dim);
    return LORA_OK;
}

// .. that are written: no two rows share elements, whether a token's heads stand side by side or a head's tokens do
static lora_status_t check_written(const void *p, int64_t token, int64_t head, int32_t tokens, int32_t heads, int32_t dim, const char *what)
{
    TRY(check_heads(p, token, head, heads, dim, what));
    const int64_t row = heads > 1 ? (int64_t)(heads - 1) * head + dim : dim, column = (int64_t)(tokens - 1) * token + dim;
    if (tokens > 1 && token < row && (token < dim || (heads > 1 && head < column)))
        return fail(LORA_ERR_INVALID_ARG, "rows of %s (%lld a token, %lld a head) overlap", what, (long long)token, (long long)head);
    return LORA_OK;
}

static lora_status_t check_ints(const void *p, const char *what)
{
    if (!p || ((uintptr_t)p) % 4) return fail(LORA_ERR_INVALID_ARG, "%s is NULL or not 4-byte aligned", what);
    return LORA_OK;
}

static lora_status_t check_count(int32_t tokens, int32_t heads)
{
    if (tokens < 0) return fail(LORA_ERR_INVALID_ARG, "tokens = %d", tokens);
    if (heads < 1 || heads > LORA_MAX_HEADS) return fail(LORA_ERR_SHAPE, "heads (%d) outside 1..%d", heads, LORA_MAX_HEADS);
    return LORA_OK;
}

static lora_status_t check_rotary(const lora_rotary_t *r, int32_t dim, const int32_t *positions)
{
    if (!r->turns || ((uintptr_t)r->turns) % 8) return fail(LORA_ERR_INVALID_ARG, "turns is NULL or not 8-byte aligned");
    if (r->dims < 16 || r->dims % 16 || r->dims > dim) return fail(LORA_ERR_SHAPE, "turned dims (%d) must be a multiple of 16, of 16 to %d", r->dims, dim);
    return check_ints(positions, "positions");
}

static lora_status_t check_cache(const lora_cache_t *c)
{
    if (!c) return fail(LORA_ERR_INVALID_ARG, "cache is NULL");
    if (c->bits != 16 && c->bits != 8) return fail(LORA_ERR_INVALID_ARG, "bits = %d: 16 (bf16) or 8 (E4M3)", c->bits);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(LORA_ERR_SHAPE, "head_dim of a cache (%d) is 64 or 128", c->head_dim);
    if (c->kv_heads < 1 || c->kv_heads > LORA_MAX_HEADS) return fail(LORA_ERR_SHAPE, "kv_heads (%d) outside 1..%d", c->kv_heads, LORA_MAX_HEADS);
    if (c->page_size < 16 || c->page_size > LORA_MAX_PAGE || (c->page_size & (c->page_size - 1)))
        return fail(LORA_ERR_SHAPE, "page_size (%d) must be a power of two, of 16 to %d", c->page_size, LORA_MAX_PAGE);
    if (c->pages < 1 || (int64_t)c->pages * c->page_size > INT32_MAX)
        return fail(LORA_ERR_SHAPE, "%d pages of %d slots: at least one, and slots that 32 bits count", c->pages, c->page_size);
    if (!c->k || ((uintptr_t)c->k) % 16 || !c->v || ((uintptr_t)c->v) % 16) return fail(LORA_ERR_INVALID_ARG, "the cache's k or v is NULL or not 16-byte aligned");
    if (c->bits == 8 && (!c->k_scales || ((uintptr_t)c->k_scales) % 16 || !c->v_scales || ((uintptr_t)c->v_scales) % 16))
        return fail(LORA_ERR_INVALID_ARG, "the cache's k_scales or v_scales is NULL or not 16-byte aligned");
    return LORA_OK;
}

static lora::PagedCache cache_of(const lora_cache_t *c)
{
    int shift = 4;
    while ((1 << shift) < c->page_size) ++shift;
    return lora::PagedCache{(char *)c->k, (char *)c->v, c->k_scales, c->v_scales, c->pages, shift, c->kv_heads, c->head_dim, c->bits == 8};
}

static void set_rotary(lora::TurnArgs &a, const lora_rotary_t *r)
{
    a.turns = r->turns;
    a.dims = r->dims;
    a.magnitude = r->magnitude;
    a.interleaved = r->interleaved != 0;
}

// 2^32 / n, rounded up: the kernels' divisor
static uint32_t reciprocal(int32_t n) { return n == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + n - 1) / n); }

extern "C" lora_status_t lora_rotary_turns(int32_t dims, double base, int32_t scaling, double factor, double low, double high, double length,
                                           uint64_t *turns, float *magnitude)
{
    if (!turns) return fail(LORA_ERR_INVALID_ARG, "turns is NULL");
    if (dims < 16 || dims % 16 || dims > LORA_MAX_HEAD_DIM) return fail(LORA_ERR_SHAPE, "turned dims (%d) must be a multiple of 16, of 16 to %d", dims, LORA_MAX_HEAD_DIM);
    if (!(base > 1.0) || !std::isfinite(base)) return fail(LORA_ERR_INVALID_ARG, "base = %g", base);
    if (scaling < LORA_ROTARY_PLAIN || scaling > LORA_ROTARY_DIMENSION) return fail(LORA_ERR_INVALID_ARG, "scaling = %d", scaling);
    const bool by_part = scaling == LORA_ROTARY_WAVELENGTH || scaling == LORA_ROTARY_DIMENSION;
    if (scaling != LORA_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return fail(LORA_ERR_INVALID_ARG, "factor = %g: 1 or more", factor);
    if (by_part && (!(low > 0.0) || !(high > low) || !std::isfinite(high) || !(length >= 1.0) || !std::isfinite(length)))
        return fail(LORA_ERR_INVALID_ARG, "low = %g, high = %g, length = %g: 0 < low < high, length 1 or more", low, high, length);
    const long double pi = 3.14159265358979323846264338327950288L, lb = logl((long double)base);
    auto held = [](long double v) { return v < 0 ? 0.0L : v > 1 ? 1.0L : v; };
    long double a = 0, b = 0;
    if (scaling == LORA_ROTARY_DIMENSION) {
        auto pair = [&](double n) { return dims * logl((long double)length / (2 * pi * n)) / (2 * lb); };
        a = floorl(pair(high));
        b = ceill(pair(low));
        if (a < 0) a = 0;
        if (b > dims - 1) b = dims - 1;
    }
    for (int32_t i = 0; i < dims / 2; ++i) {
        const long double f = expl(-2.0L * i / dims * lb);
        long double keep = 1;
        if (scaling == LORA_ROTARY_LINEAR)
            keep = 0;
        else if (scaling == LORA_ROTARY_WAVELENGTH)
            keep = held(((long double)length * f / (2 * pi) - low) / ((long double)high - low));
        else if (scaling == LORA_ROTARY_DIMENSION)
            keep = 1 - held((i - a) / (b - a > 0.001L ? b - a : 0.001L));
        // (f is at most 1 radian: less than a turn)
        turns[i] = (uint64_t)((keep * f + (1 - keep) * f / factor) / (2 * pi) * 18446744073709551616.0L);
    }
    if (magnitude) *magnitude = scaling == LORA_ROTARY_DIMENSION ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return LORA_OK;
}

static lora_status_t launch_turn(const lora::TurnArgs &a, void *stream, const char *what)
{
    const hipError_t e = lora::launch_turn(a, (hipStream_t)stream);
    if (e == hipErrorInvalidConfiguration) return fail(LORA_ERR_SHAPE, "%s: %d tokens x %d heads are more rows than a launch can have", what, a.tokens, a.heads);
    return of_hip(e, what);
}

extern "C" lora_status_t lora_rotary(const void *x, int64_t x_token, int64_t x_head, int32_t tokens, int32_t heads, int32_t head_dim,
                                     const int32_t *positions, const lora_rotary_t *rotary, int32_t inverse, void *y, int64_t y_token, int64_t y_head,
                                     void *stream)
{
    TRY(check_count(tokens, heads));
    if (head_dim < 16 || head_dim % 16 || head_dim > LORA_MAX_HEAD_DIM)
        return fail(LORA_ERR_SHAPE, "head_dim (%d) must be a multiple of 16, of 16 to %d", head_dim, LORA_MAX_HEAD_DIM);
    if ((int64_t)tokens * heads > INT32_MAX) return fail(LORA_ERR_SHAPE, "%d tokens x %d heads do not fit 32 bits", tokens, heads);
    if (!rotary) return fail(LORA_ERR_INVALID_ARG, "rotary is NULL");
    if (tokens == 0) return LORA_OK;
    TRY(check_heads(x, x_token, x_head, heads, head_dim, "x"));
    TRY(check_written(y, y_token, y_head, tokens, heads, head_dim, "y"));
    TRY(check_rotary(rotary, head_dim, positions));
    if (x == y && (x_token != y_token || x_head != y_head)) return fail(LORA_ERR_INVALID_ARG, "y is x with other strides");
    lora::TurnArgs a = {};
    a.q = {(uint16_t *)x, x_token, x_head};
    a.y = {(uint16_t *)y, y_token, y_head};
    a.q_heads = a.heads = heads;
    a.per_heads = reciprocal(heads);
    a.tokens = tokens;
    a.dim = head_dim;
    a.positions = positions;
    a.inverse = inverse != 0;
    set_rotary(a, rotary);
    return launch_turn(a, stream, "lora_rotary");
}

extern "C" lora_status_t lora_cache_append(const void *k, int64_t k_token, int64_t k_head, const void *v, int64_t v_token, int64_t v_head,
                                           int32_t tokens, const int32_t *slots, const int32_t *positions, const lora_rotary_t *rotary,
                                           const lora_cache_t *cache, const void *q, int64_t q_token, int64_t q_head, int32_t q_heads, void *y,
                                           int64_t y_token, int64_t y_head, void *stream)
{
    TRY(check_cache(cache));
    TRY(check_count(tokens, q ? q_heads : 1));
    const int32_t heads = (q ? q_heads : 0) + 2 * cache->kv_heads, dim = cache->head_dim;
    if ((int64_t)tokens * heads > INT32_MAX) return fail(LORA_ERR_SHAPE, "%d tokens x %d heads do not fit 32 bits", tokens, heads);
    if (q && !rotary) return fail(LORA_ERR_INVALID_ARG, "q is there to be turned, and rotary is NULL");
    if (tokens == 0) return LORA_OK;
    TRY(check_heads(k, k_token, k_head, cache->kv_heads, dim, "k"));
    TRY(check_heads(v, v_token, v_head, cache->kv_heads, dim, "v"));
    TRY(check_ints(slots, "slots"));
    if (rotary) TRY(check_rotary(rotary, dim, positions));
    if (positions) TRY(check_ints(positions, "positions"));
    lora::TurnArgs a = {};
    if (q) {
        TRY(check_heads(q, q_token, q_head, q_heads, dim, "q"));
        TRY(check_written(y, y_token, y_head, tokens, q_heads, dim, "y"));
        if (q == y && (q_token != y_token || q_head != y_head)) return fail(LORA_ERR_INVALID_ARG, "y is q with other strides");
        a.q = {(uint16_t *)q, q_token, q_head};
        a.y = {(uint16_t *)y, y_token, y_head};
        a.q_heads = q_heads;
    }
    a.k = {(uint16_t *)k, k_token, k_head};
    a.v = {(uint16_t *)v, v_token, v_head};
    a.heads = heads;
    a.per_heads = reciprocal(heads);
    a.tokens = tokens;
    a.dim = dim;
    a.positions = positions;
    a.slots = slots;
    if (rotary) set_rotary(a, rotary);
    a.cache = cache_of(cache);
    return launch_turn(a, stream, "lora_cache_append");
}

static lora_status_t check_attention(int32_t tokens, int32_t q_heads, int32_t requests, int32_t width, const lora_cache_t *cache)
{
    TRY(check_cache(cache));
    TRY(check_count(tokens, q_heads));
    if (q_heads % cache->kv_heads) return fail(LORA_ERR_SHAPE, "q_heads (%d) is no multiple of kv_heads (%d)", q_heads, cache->kv_heads);
    // (a tile's columns are counted past the last one, and requests in equal parts for a work group's threads)
    if ((int64_t)tokens * q_heads > INT32_MAX - 1024) return fail(LORA_ERR_SHAPE, "%d tokens x %d heads do not fit 32 bits", tokens, q_heads);
    if (requests > INT32_MAX - 1024) return fail(LORA_ERR_SHAPE, "requests = %d", requests);
    if (requests < 0 || width < 0) return fail(LORA_ERR_INVALID_ARG, "requests = %d, width = %d", requests, width);
    if ((int64_t)width * cache->page_size > INT32_MAX - 2 * LORA_MAX_PAGE)
        return fail(LORA_ERR_SHAPE, "%d pages of %d slots a request: more keys than 32 bits count", width, cache->page_size);
    // (steps of the tiles are counted in 32 bits)
    const int64_t keys = (int64_t)width * cache->page_size;
    if (lora::most_steps(tokens, q_heads / cache->kv_heads, requests, keys) >= INT32_MAX)
        return fail(LORA_ERR_SHAPE, "%d tokens x %d heads of %d requests over %lld keys are more work than 32 bits count", tokens, q_heads, requests, (long long)keys);
    return LORA_OK;
}

extern "C" lora_status_t lora_attention_workspace_bytes(int32_t tokens, int32_t q_heads, int32_t requests, int32_t width, const lora_cache_t *cache,
                                                        size_t *bytes)
{
    if (!bytes) return fail(LORA_ERR_INVALID_ARG, "bytes is NULL");
    TRY(check_attention(tokens, q_heads, requests, width, cache));
    *bytes = lora::attend_most_bytes(tokens, q_heads / cache->kv_heads, cache->kv_heads, requests, (int64_t)width * cache->page_size, cache->head_dim, cache->bits == 8);
    return LORA_OK;
}

extern "C" lora_status_t lora_attention(const void *q, int64_t q_token, int64_t q_head, int32_t tokens, int32_t q_heads, const int32_t *starts,
                                        const int32_t *lengths, int32_t requests, const int32_t *page_table, int64_t ld_table, int32_t width,
                                        const uint64_t *tree, int32_t most, const lora_cache_t *cache, float scale, void *y, int64_t y_token,
                                        int64_t y_head, void *workspace, size_t ws_bytes, void *stream)
{
    TRY(check_attention(tokens, q_heads, requests, width, cache));
    if (most < 0) return fail(LORA_ERR_INVALID_ARG, "most = %d", most);
    if (!std::isfinite(scale)) return fail(LORA_ERR_INVALID_ARG, "scale = %g", (double)scale);
    if (tokens == 0 || requests == 0) return LORA_OK;
    TRY(check_heads(q, q_token, q_head, q_heads, cache->head_dim, "q"));
    TRY(check_written(y, y_token, y_head, tokens, q_heads, cache->head_dim, "y"));
    if (q == y) return fail(LORA_ERR_INVALID_ARG, "y is q");
    TRY(check_ints(starts, "starts"));
    TRY(check_ints(lengths, "lengths"));
    if (width > 0) {
        TRY(check_ints(page_table, "page_table"));
        if (ld_table < width || ld_table > INT64_MAX / 8 / INT32_MAX)
            return fail(LORA_ERR_INVALID_ARG, "row stride of page_table (%lld) must be at least %d", (long long)ld_table, width);
    }
    if (tree && ((uintptr_t)tree) % 8) return fail(LORA_ERR_INVALID_ARG, "tree is not 8-byte aligned");
    lora::AttendArgs a = {};
    a.q = {(uint16_t *)q, q_token, q_head};
    a.y = {(uint16_t *)y, y_token, y_head};
    a.tokens = tokens;
    a.group = q_heads / cache->kv_heads;
    a.per_group = reciprocal(a.group);
    a.starts = starts;
    a.lengths = lengths;
    a.table = page_table;
    a.ld_table = ld_table;
    a.requests = requests;
    a.room = width * cache->page_size;
    a.tree = tree;
    a.cache = cache_of(cache);
    // (nought times the -infinity of a key that is not seen would be NaN; times 2^-126 scores do not matter either)
    a.scale = std::fmax(std::fabs(scale) * 1.44269504088896340736f, 0x1p-126f);
    if (!std::isfinite(a.scale)) return fail(LORA_ERR_INVALID_ARG, "scale = %g: too large for its multiple by log2 e", (double)scale);
    a.flip = scale < 0.f ? 0x80008000u : 0u;
    a.slack = std::fmin(8.f / a.scale, 1e38f);
    const lora::AttendForms forms = lora::attend_forms(tokens, a.group, cache->kv_heads, requests, (int64_t)width * cache->page_size, most, cache->head_dim, cache->bits == 8);
    size_t need = 0;
    for (int i = 0; i < forms.n; ++i) {
        const size_t n = lora::attend_parts_bytes(forms.f[i], cache->kv_heads, cache->head_dim);
        if (n > need) need = n;
    }
    if (need > 0 && (!workspace || ((uintptr_t)workspace) % 16 || ws_bytes < need))
        return fail(LORA_ERR_WORKSPACE, "a 16-byte aligned workspace of %zu bytes is needed, %zu are there", need, workspace ? ws_bytes : (size_t)0);
    a.parts = (float *)workspace;
    for (int i = 0; i < forms.n; ++i)
        if (const hipError_t e = lora::launch_attention(a, forms.f[i], (hipStream_t)stream); e != hipSuccess) return of_hip(e, "lora_attention");
    return LORA_OK;
}
