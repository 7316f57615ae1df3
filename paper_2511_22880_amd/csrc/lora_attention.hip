// gfx950 kernels between the adapted projections (include/lora_attention.h): rotary positions, the paged cache's append, attention over it.
#include "lora_attention.h"
#include "lora_device.h"
#include "lora_internal.h"

#include <type_traits>

namespace lora {

static __device__ __forceinline__ float value_lo(uint32_t u) { return __uint_as_float(u << 16); }
static __device__ __forceinline__ float value_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }

// ------------------------------------------------------------------------------------------------
// Rows turned by their positions.  A row is (token, head), heads counted over q, k and v; a thread has 16 elements of one, two pieces of 8: eight pairs that are turned
// (half layout: the pieces are dims / 2 apart), or elements that pass.  A work group has as many consecutive rows as its threads hold; it asks for all of them,
// computes the cosines and sines of its few tokens once into LDS (a pair's angle for all heads at once: 64 angles a token, not 64 a head), and turns.  The angle is the
// low 64 bits of position * turns, of which the upper 32 count: exact to 2^-31 turns at any position, without a division or a table of positions. Bound by memory where
// there is much: 19675 tokens x 32 heads of 128, 322 MB, 56 us (5.7 TB/s, a half written); the same tokens' q, k and v into a cache in 8 bits, 445 MB, 87 us (5.1 TB/s:
// the maxima, quotients and conversions of k and v do not all hide).  One token 3.4 us, 256 tokens 4.5.  Four rows of a thread one after the other: 62 and 105 us; two:
// 55 and 90; loads and stores past the caches 72 to 80 and level.
// ------------------------------------------------------------------------------------------------
constexpr int kTurnThreads = 256;

template <bool BITS8>
static __device__ __forceinline__ void store_held(char *row, float *scale_at, const float (&a)[8], const float (&b)[8], int d0, int d1, int units, bool first)
{
    if constexpr (!BITS8) {
        uint16_t *y = reinterpret_cast<uint16_t *>(row);
        *reinterpret_cast<uint4 *>(y + d0) = uint4{pack_bf16_rne(a[0], a[1]), pack_bf16_rne(a[2], a[3]), pack_bf16_rne(a[4], a[5]), pack_bf16_rne(a[6], a[7])};
        *reinterpret_cast<uint4 *>(y + d1) = uint4{pack_bf16_rne(b[0], b[1]), pack_bf16_rne(b[2], b[3]), pack_bf16_rne(b[4], b[5]), pack_bf16_rne(b[6], b[7])};
    } else {
        // x * 448 / d, d = m 2^(e - 127): the power of two is exact, the quotient by m is corrected once (see lora_rows_quantize, whose rounding this is)
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, max(__float_as_uint(a[i]) & 0x7FFFFFFFu, __float_as_uint(b[i]) & 0x7FFFFFFFu));
        for (int d = 1; d < units; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
        const float largest = __uint_as_float(top);
        float scale = largest;
        uint32_t o[4] = {0u, 0u, 0u, 0u};
        if (top < 0x7F800000u) {
            const float d = fmaxf(largest, 448.f * 0x1p-126f);
            scale = d / 448.f;
            const uint32_t bits = __float_as_uint(d), e = bits >> 23;
            const float m = __uint_as_float((bits & 0x007FFFFFu) | 0x3F800000u), f = 1.75f * __uint_as_float((262u - e) << 23), r = __builtin_amdgcn_rcpf(m);
            auto quotient = [&](float x) __attribute__((always_inline)) {
                const float n = x * f, t = n * r;
                return fmaf(fmaf(-t, m, n), r, t);
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *c = i < 2 ? a + 4 * i : b + 4 * (i - 2);
                const int p = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(c[0]), quotient(c[1]), 0, false);
                o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(quotient(c[2]), quotient(c[3]), p, true);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = i < 8 ? a[i] : b[i - 8];
                o[i >> 2] |= (top > 0x7F800000u || (__float_as_uint(x) & 0x7FFFFFFFu) >= 0x7F800000u ? 0x7Fu : 0u) << (8 * (i & 3));
            }
        }
        *reinterpret_cast<uint2 *>(row + d0) = uint2{o[0], o[1]};
        *reinterpret_cast<uint2 *>(row + d1) = uint2{o[2], o[3]};
        if (first) *scale_at = scale;
    }
}

// KIND 0: q alone; 1: with a cache in bf16; 2: in 8 bits.
template <int KIND>
__global__ __launch_bounds__(kTurnThreads) void k_turn(TurnArgs a)
{
    extern __shared__ float2 turned[];  // [tokens here][pairs]: cosine and sine, times the magnitude
    const int tid = threadIdx.x, units = a.dim >> 4, at_once = kTurnThreads / units;
    const int r0 = tid / units, u = tid - r0 * units;
    const uint32_t first = blockIdx.x * (uint32_t)at_once;
    const int t_first = (int)(first / (uint32_t)a.heads), h_first = (int)(first - (uint32_t)t_first * a.heads);
    auto over_heads = [&](int flat) __attribute__((always_inline)) { return a.per_heads ? (int)__umulhi((uint32_t)flat, a.per_heads) : flat; };

    const int t = over_heads(h_first + r0), head = h_first + r0 - t * a.heads, token = t_first + t;
    const bool is_q = head < a.q_heads, is_k = !is_q && (KIND == 0 || head < a.q_heads + a.cache.kv_heads);
    bool there = token < a.tokens && r0 < at_once;
    const int tok = there ? token : 0;
    int slot = 0;
    if constexpr (KIND > 0) {
        slot = a.slots[tok];
        there &= (uint32_t)slot < (uint32_t)a.cache.pages << a.cache.page_shift;
    }
    if (a.positions) there &= a.positions[tok] >= 0;
    const bool turns = a.turns && (KIND == 0 || is_q || is_k) && u < a.dims >> 4, apart = turns && !a.interleaved;
    const int d0 = apart ? 8 * u : 16 * u, d1 = apart ? 8 * u + (a.dims >> 1) : 16 * u + 8;
    uint4 lo, hi;
    if (there) {
        HeadRows from = a.q;
        int h = head;
        if constexpr (KIND > 0) {
            from = is_q ? a.q : is_k ? a.k : a.v;
            h = is_q ? h : is_k ? h - a.q_heads : h - a.q_heads - a.cache.kv_heads;
        }
        const uint16_t *row = from.p + tok * from.token + h * from.head;
        lo = ld16(row + d0);
        hi = ld16(row + d1);
    }
    if (a.turns) {
        const int pairs = a.dims >> 1, n = (over_heads(h_first + at_once - 1) + 1) * pairs;
        for (int e = tid; e < n; e += kTurnThreads) {
            const int te = e / pairs, p = e - te * pairs, at = t_first + te < a.tokens ? t_first + te : 0;
            const uint64_t all = (uint64_t)(uint32_t)a.positions[at] * a.turns[p];
            // quarters of a turn apart, what is left within an eighth either way: as a float it is off by 2^-28 turns at most
            const uint32_t turn = (uint32_t)(all >> 32), quarter = (turn + 0x20000000u) >> 30;
            float s, c;
            sincospif((float)(int32_t)(turn - (quarter << 30)) * 0x1p-31f, &s, &c);
            if (quarter & 1) {
                const float was = c;
                c = -s;
                s = was;
            }
            if (quarter & 2) {
                c = -c;
                s = -s;
            }
            turned[e] = float2{c * a.magnitude, (a.inverse ? -s : s) * a.magnitude};
        }
        __syncthreads();
    }
    if (!there) return;
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    float x[8], z[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = value_lo(w[j]);
        x[2 * j + 1] = value_hi(w[j]);
        z[2 * j] = value_lo(w[4 + j]);
        z[2 * j + 1] = value_hi(w[4 + j]);
    }
    if (turns) {
        const float2 *cs = turned + t * (a.dims >> 1) + 8 * u;
        if (a.interleaved) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = cs[j], g = cs[4 + j];
                const float x0 = x[2 * j], x1 = x[2 * j + 1], z0 = z[2 * j], z1 = z[2 * j + 1];
                x[2 * j] = x0 * f.x - x1 * f.y;
                x[2 * j + 1] = x0 * f.y + x1 * f.x;
                z[2 * j] = z0 * g.x - z1 * g.y;
                z[2 * j + 1] = z0 * g.y + z1 * g.x;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 f = cs[j];
                const float x0 = x[j], z0 = z[j];
                x[j] = x0 * f.x - z0 * f.y;
                z[j] = x0 * f.y + z0 * f.x;
            }
        }
    }
    if (KIND == 0 || is_q) {
        store_held<false>(reinterpret_cast<char *>(a.y.p + token * a.y.token + head * a.y.head), nullptr, x, z, d0, d1, units, false);
    } else if constexpr (KIND > 0) {
        const int kh = head - a.q_heads - (is_k ? 0 : a.cache.kv_heads), page = slot >> a.cache.page_shift;
        const int64_t at = (((int64_t)page * a.cache.kv_heads + kh) << a.cache.page_shift) + (slot & ((1 << a.cache.page_shift) - 1));
        store_held<KIND == 2>((is_k ? a.cache.k : a.cache.v) + at * a.dim * (KIND == 2 ? 1 : 2), (is_k ? a.cache.k_scales : a.cache.v_scales) + at, x, z, d0, d1, units,
                              u == 0);
    }
}

hipError_t launch_turn(const TurnArgs &a, hipStream_t stream)
{
    const int at_once = kTurnThreads / (a.dim >> 4);
    const int64_t grid = ((int64_t)a.tokens * a.heads + at_once - 1) / at_once;
    if (grid > (int64_t)UINT32_MAX / kTurnThreads) return hipErrorInvalidConfiguration;
    // tokens that a work group meets at most, and LDS for their pairs: 16 KB where there is one head, a little more where tokens begin in its middle
    const size_t lds = a.turns ? (size_t)((at_once - 2) / a.heads + 2) * (a.dims >> 1) * sizeof(float2) : 0;
    auto *kernel = !a.cache.k ? k_turn<0> : a.cache.bits8 ? k_turn<2> : k_turn<1>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kTurnThreads), lds, stream, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// How the work of an attention call is dealt out.  A request's columns (row by row, the query heads of a key head's group side by side) are cut into tiles of TC; a
// tile takes as many steps of KEYS keys as its last row sees, one at least.  The steps of all tiles of all requests, in that order, are one list for every key head,
// and a head's `shares` work groups take equal runs of it.  A run that has all of a tile's steps writes its rows; otherwise it leaves sums, which k_attend_join brings
// together.  Where no tile has many steps (see attend_form) none is cut, and every tile has a work group.  The list follows from starts and lengths on the device
// alone: every work group adds up the requests' steps and finds its place in it, so the host need not know any length, and a captured call follows them: one trip to
// memory before the first page number.
// ------------------------------------------------------------------------------------------------
struct Request {
    int first, n, keys;  // first row, rows, keys
};

static __device__ __forceinline__ Request request_at(const AttendArgs &a, int r)
{
    const int s0 = min(max(a.starts[r], 0), a.tokens), s1 = min(max(a.starts[r + 1], 0), a.tokens);
    return Request{s0, max(s1 - s0, 0), min(max(a.lengths[r], 0), a.room)};
}

// sum of floor((a i + b) / m) for i < n: the part that whole multiples of m give, then the same question with the axes exchanged
static __device__ __forceinline__ uint32_t sum_of_floors(uint32_t n, uint32_t m, uint32_t a, uint32_t b)
{
    uint32_t sum = 0;
    while (true) {
        if (a >= m) {
            const uint32_t f = a / m;
            sum += (n & 1 ? n * ((n - 1) >> 1) : (n >> 1) * (n - 1)) * f;
            a -= f * m;
        }
        if (b >= m) {
            const uint32_t f = b / m;
            sum += n * f;
            b -= f * m;
        }
        const uint32_t top = a * n + b;
        if (top < m) return sum;
        n = top / m;
        b = top - n * m;
        const uint32_t t = m;
        m = a;
        a = t;
    }
}

template <int TC, int KEYS>
struct Dealt {
    // of a request
    struct Tiles {
        int n;          // tiles
        uint32_t last;  // steps of the last one, and of all where rows do not see more and more
        bool level;
        uint32_t whole, part;  // steps before the request's own keys; (context mod KEYS) * group + TC
    };
    static __device__ __forceinline__ Tiles tiles(const AttendArgs &a, const Request &q)
    {
        const int columns = q.n * a.group;
        if (q.n == 0 || columns <= a.least || columns > a.most) return Tiles{0, 0, true, 0, 0};
        const int context = q.keys - q.n;
        const uint32_t last = max(1u, (uint32_t)(q.keys + KEYS - 1) / KEYS);
        return Tiles{(columns - 1) / TC + 1, last, a.tree != nullptr || context < 0, (uint32_t)context / KEYS, (uint32_t)(context & (KEYS - 1)) * a.group + TC};
    }
    // steps of the first t tiles, t < n
    static __device__ __forceinline__ uint32_t before(const AttendArgs &a, const Tiles &s, uint32_t t)
    {
        const uint32_t m = (uint32_t)a.group * KEYS;
        return s.level ? t * s.last : t * s.whole + sum_of_floors(t, m, TC, s.part + m - 1);
    }
    static __device__ __forceinline__ uint32_t steps(const AttendArgs &a, const Tiles &s, uint32_t t)
    {
        const uint32_t m = (uint32_t)a.group * KEYS;
        return s.level || (int)t == s.n - 1 ? s.last : s.whole + (s.part + t * TC + m - 1) / m;
    }
    // of a request: its steps, or its tiles where those are not cut
    static __device__ __forceinline__ uint32_t all(const AttendArgs &a, const Tiles &s)
    {
        return s.n == 0 || !a.cut ? (uint32_t)s.n : (s.n == 1 ? 0u : before(a, s, s.n - 1)) + s.last;
    }

    // a place in the list
    struct Place {
        int r, t;
        uint32_t at, of;  // step of the tile, its steps
        Request q;
        Tiles s;
    };
    struct Found {
        uint32_t sums[8];
        int r;
        uint32_t at;
        Request q;
    };

    // Rows that starts in order give are fewer steps; where requests share rows there can be more, and nothing is done.
    static constexpr uint32_t kTooMany = 0x7FFFFFFFu;

    // Every thread of a work group: which(total) says which step of the list is meant, given how many there are (none: `total`, and false is returned).
    template <int THREADS, class Which>
    static __device__ __forceinline__ bool find(const AttendArgs &a, Found &f, Which which, Place &p)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int each = (a.requests + THREADS - 1) / THREADS, r0 = tid * each, r1 = min(a.requests, r0 + each);
        Request q{0, 0, 0};
        uint32_t mine = 0, n = 0;  // (steps of this thread's requests; of the last of them)
        for (int r = r0; r < r1; ++r) {
            q = request_at(a, r);
            mine = min(mine + (n = all(a, tiles(a, q))), kTooMany);
        }
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = (uint32_t)__shfl_up((int)upto, d, 64);
            upto = min(upto + (lane >= d ? o : 0), kTooMany);
        }
        if (lane == 63) f.sums[wave] = upto;
        __syncthreads();
        uint32_t total = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w == wave) upto += total;
            total = min(total + f.sums[w], kTooMany);
        }
        total = __builtin_amdgcn_readfirstlane(total);
        const uint32_t want = which(total);
        if (want >= total || total == kTooMany) return false;
        if (want < upto && want >= upto - mine) {
            int r = r1 - 1;
            uint32_t from = upto - n;
            while (want < from) {  // (no further than r0)
                q = request_at(a, --r);
                from -= all(a, tiles(a, q));
            }
            f.r = r;
            f.at = want - from;
            f.q = q;
        }
        __syncthreads();
        p.r = __builtin_amdgcn_readfirstlane(f.r);
        const uint32_t at = __builtin_amdgcn_readfirstlane(f.at);
        p.q = Request{__builtin_amdgcn_readfirstlane(f.q.first), __builtin_amdgcn_readfirstlane(f.q.n), __builtin_amdgcn_readfirstlane(f.q.keys)};
        p.s = tiles(a, p.q);
        if (!a.cut) {
            p.t = (int)at;
            p.at = 0;
            p.of = steps(a, p.s, p.t);
            return true;
        }
        // the last tile that begins at or before it, 64 at a time
        int lo = 0, hi = p.s.n - 1;
        while (hi > lo) {
            const int step = (hi - lo + 63) >> 6, t = lo + (lane + 1) * step;
            const int k = (int)__popcll(__ballot(t <= hi && before(a, p.s, t) <= at));
            lo += k * step;
            hi = min(hi, lo + step - 1);
        }
        p.t = lo;
        p.at = lo > 0 ? __builtin_amdgcn_readfirstlane(at - before(a, p.s, lo)) : at;
        p.of = steps(a, p.s, p.t);
        return true;
    }
    // the tile behind it; false where there is none
    static __device__ __forceinline__ bool next(const AttendArgs &a, Place &p)
    {
        p.at = 0;
        if (++p.t >= p.s.n) {
            p.t = 0;
            while (true) {
                if (++p.r >= a.requests) return false;
                p.q = request_at(a, p.r);
                p.s = tiles(a, p.q);
                if (p.s.n > 0) break;
                // over those behind it that have none either, 64 at a time
                const int r = p.r + 1 + (int)(threadIdx.x & 63);
                const uint64_t some = __ballot(r < a.requests && tiles(a, request_at(a, r)).n > 0);
                p.r += some ? __builtin_ctzll(some) : 64;
            }
        }
        p.of = steps(a, p.s, p.t);
        return true;
    }
};

// first step of a share of `total` (the first ones have one more; with fewer steps than shares those have one each)
static __device__ __forceinline__ uint32_t share_at(uint32_t total, int share, int shares)
{
    const uint32_t each = total / (uint32_t)shares, more = total - each * shares;
    return each * share + min((uint32_t)share, more);
}

// What a share leaves for k_attend_join: the tile that it began and did not end, whose last steps are in the shares up to `last` (-1: there is none).
struct CutTile {
    int first, columns, c0, last;  // its request's first row and columns, its own first column
};
static __device__ __forceinline__ CutTile *cut_tiles(const AttendArgs &a, int columns, int dim)
{
    return reinterpret_cast<CutTile *>(a.parts + (int64_t)a.cache.kv_heads * a.shares * 2 * columns * (dim + 2));
}
// one thread: the share ended `behind` steps before its tile does (0: with it)
template <class Place>
static __device__ __forceinline__ void leave_cut(const AttendArgs &a, CutTile *to, uint32_t total, int share, const Place &p, int c0, uint32_t behind)
{
    CutTile t{p.q.first, p.q.n * a.group, c0, -1};
    if (behind > 0 && p.at == 0) {
        // (shares are alike but for one step)
        const uint32_t begin = share_at(total, share + 1, a.shares), end = begin + behind, some = min((uint32_t)a.shares, total);
        t.last = min((int)some - 1, share + 1 + (int)((behind - 1) / (total / some)));
        while (share_at(total, t.last, a.shares) >= end) --t.last;
    }
    *to = t;
}

// where a share leaves its sums: slot 1 of those of a tile that begins in it, slot 0 of one that began earlier
static __device__ __forceinline__ int64_t part_of(int head, int shares, int share, bool begins) { return ((int64_t)head * shares + share) * 2 + begins; }

// ------------------------------------------------------------------------------------------------
// Attention of few columns: tiles of 16 C.  A wavefront takes 32 keys (8 bits: twice) at a time, the work group's four as many times that, each with a running maximum
// and sum of its own; what they have is brought together in LDS at the tile's end.  Nothing goes through LDS on the way: with S^T = K Q^T (16 x 16 x 32 matrix
// instructions) a lane holds a column's scores of eight keys, and those are what O^T = V^T P^T takes as the operand of eight values of k from that lane, if row m of
// the score tile t is key 8 (m / 4) + 4 t + m mod 4 and lane (quad, n) brings the keys 8 quad .. 8 quad + 7.  It reads their dims [n D / 16, (n + 1) D / 16): sixteen
// lanes a whole row of v; the element c of each is the operand of tile c, whose row n is dim n D / 16 + c, put together by byte permutes.
//
// The maximum that weights are relative to follows only when a score passes it by more than 2^8 (`slack`): weights are up to 2^8 then, which bf16 and fp32 hold as well
// as 1, and the sums are not rescaled at every step.  A weight is rounded to bf16 for its product with v, half a step of its own value, and in bf16 caches the sum is
// of the rounded ones: y is then a mean by weights that add up to one exactly.  In 8 bits the value's scale goes into the weight before that rounding, so the sum is of
// those before.
//
// Bound by memory.  256 requests of 200 to 8000 keys in bf16, 2.29 GB: 388 to 398 us, 5.8 to 5.9 TB/s; five of 60,000 to 130,000 in 8 bits, 810 MB: 138 us, 5.9 TB/s.
// The loads alone, nothing computed: 403 against 410 then, and 140 against 157.  Loads of what is read once go past the caches (400 against 408).
// ------------------------------------------------------------------------------------------------
template <int BYTES>
struct Bytes;
template <>
struct Bytes<4> {
    uint32_t w[1];
};
template <>
struct Bytes<8> {
    uint32_t w[2];
};
template <>
struct Bytes<16> {
    uint32_t w[4];
};
template <int BYTES>
static __device__ __forceinline__ Bytes<BYTES> ld_bytes(const char *p)
{
    typedef __attribute__((ext_vector_type(BYTES / 4))) uint32_t vec;
    return __builtin_bit_cast(Bytes<BYTES>, *reinterpret_cast<const vec *>(p));
}
template <>
__device__ __forceinline__ Bytes<4> ld_bytes<4>(const char *p)
{
    return Bytes<4>{{*reinterpret_cast<const uint32_t *>(p)}};
}

// .. past the caches (see ld16_stream): what one launch reads once
template <int BYTES>
static __device__ __forceinline__ Bytes<BYTES> ld_bytes_once(const char *p)
{
    typedef __attribute__((ext_vector_type(BYTES / 4))) uint32_t vec;
    return __builtin_bit_cast(Bytes<BYTES>, __builtin_nontemporal_load(reinterpret_cast<const vec *>(p)));
}
template <>
__device__ __forceinline__ Bytes<4> ld_bytes_once<4>(const char *p)
{
    return Bytes<4>{{__builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(p))}};
}

// two E4M3 values, of the low or the high half, as bf16: exact
template <bool HIGH>
static __device__ __forceinline__ uint32_t two_of_e4m3(uint32_t u)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HIGH));
}

// eight bf16 values with their signs exchanged where `flip` says so
static __device__ __forceinline__ uint4 flipped(uint4 u, uint32_t flip) { return uint4{u.x ^ flip, u.y ^ flip, u.z ^ flip, u.w ^ flip}; }

// a column's row of its request: column / group
static __device__ __forceinline__ int row_of_column(const AttendArgs &a, int column)
{
    if (a.per_group == 0) return column;
    const uint32_t i = __umulhi((uint32_t)column, a.per_group);
    return (int)(i - (i * a.group > (uint32_t)column));
}

// Two bf16 or four E4M3 values with zero for each that is an infinity or NaN; `some` is set where one is.
template <bool F8>
static __device__ __forceinline__ uint32_t finite_of(uint32_t u, uint32_t &some)
{
    const uint32_t odd = F8 ? ((u & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u : ((u & 0x7F807F80u) + 0x00800080u) & 0x80008000u;  // their sign bits
    some |= odd;
    return u & ~((odd - (odd >> (F8 ? 7 : 15))) | odd);
}

// A matrix instruction multiplies every column's weight by every value, and nought times an infinity is NaN: among keys that not all columns see, infinities and NaN
// of v are taken as zero, and the steps that held some are remembered here.  Behind a tile's rows (or its sums), which are then written, such values are
// added to the columns that see them, element by element, every element by one thread.  (Done between the steps instead, it takes 40 registers more.)
struct OddSteps {
    uint32_t from[2], to[2];  // of this tile and the next one
    __device__ __forceinline__ void clear(int i)
    {
        from[i] = UINT32_MAX;
        to[i] = 0;
    }
    __device__ __forceinline__ void note(int i, uint32_t step)
    {
        atomicMin(&from[i], step);
        atomicMax(&to[i], step + 1);
    }
};

// keys [from, to) of p's request; `whole`: y's rows, else the sums at `sums` [columns][D]
template <int D, bool F8, int THREADS, class Place>
static __device__ __forceinline__ void add_odd(const AttendArgs &a, const Place &p, int kh, int from, int to, int c0, int tile, bool whole, float *sums)
{
    const int dim = threadIdx.x % D, context = p.q.keys - p.q.n, columns = min(tile, p.q.n * a.group - c0);
    for (int key = from; key < min(to, p.q.keys); ++key) {
        const int id = a.table[p.r * a.ld_table + (key >> a.cache.page_shift)];
        if ((unsigned)id >= (unsigned)a.cache.pages) continue;
        const int64_t row = (((int64_t)id * a.cache.kv_heads + kh) << a.cache.page_shift) + (key & ((1 << a.cache.page_shift) - 1));
        float v;
        if constexpr (F8) {
            if ((reinterpret_cast<const uint8_t *>(a.cache.v)[row * D + dim] & 0x7F) != 0x7F) continue;
            v = __builtin_nanf("");
        } else {
            const uint32_t bits = reinterpret_cast<const uint16_t *>(a.cache.v)[row * D + dim];
            if ((bits & 0x7F80u) != 0x7F80u) continue;
            v = __uint_as_float(bits << 16);
        }
        for (int in = threadIdx.x / D; in < columns; in += THREADS / D) {
            const int i = row_of_column(a, c0 + in), own = key - context;
            if (a.tree ? own >= 0 && (own >= 64 || !(a.tree[p.q.first + i] >> own & 1)) : own > i) continue;
            if (whole) {
                uint16_t *y = a.y.p + (p.q.first + i) * a.y.token + (kh * a.group + (c0 + in - i * a.group)) * a.y.head + dim;
                *y = (uint16_t)pack_bf16_rne(__uint_as_float((uint32_t)*y << 16) + v, 0.f);
            } else {
                sums[(int64_t)in * D + dim] += v;
            }
        }
    }
}

// The first n bits, n held to 0 .. 32.
static __device__ __forceinline__ uint32_t first_bits(int n) { return (uint32_t)((1ull << min(max(n, 0), 32)) - 1); }

// Which of 32 keys from key0 on a column sees (`own` = key0 - context), those that there are: up to key `sees` without a tree.
static __device__ __forceinline__ uint32_t seen_of(int key0, int keys, bool tree, int sees, uint64_t word, int own)
{
    if (!tree) return first_bits(min(keys, sees + 1) - key0);
    const uint64_t mine = own >= 64 || own <= -64 ? 0 : own >= 0 ? word >> own : word << -own;
    return first_bits(keys - key0) & ((uint32_t)mine | first_bits(-own));
}

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// over a lane and the one 32 away
static __device__ __forceinline__ float max_of_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
static __device__ __forceinline__ float sum_of_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// over the four lanes 16 apart
static __device__ __forceinline__ float max_of_quads(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return max_of_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
static __device__ __forceinline__ float sum_of_quads(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return sum_of_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

template <int D, bool F8>
struct FewShape {
    static constexpr int kRowBytes = D * (F8 ? 1 : 2);
    static constexpr int kLoadsK = kRowBytes / 64;   // of 16 bytes a lane, of a tile of 16 keys
    static constexpr int kBytesV = kRowBytes / 16;   // of a key, a lane's
    static constexpr int kSteps = D / 32;            // of k, of the scores
    static constexpr int kTiles = D / 16;            // of v
    static constexpr int kBlocks = F8 ? 2 : 1;       // of 32 keys a wavefront takes at a time: as many bytes either way
};

template <int D, bool F8, int C>
__global__ __launch_bounds__(64 * kFewWaves, C == 1 ? 2 : 1) void k_attend_few(AttendArgs a)
{
    using S = FewShape<D, F8>;
    constexpr int TC = 16 * C, WAVES = kFewWaves, KEYS = few_keys(F8);
    using W = Dealt<TC, KEYS>;
    __shared__ typename W::Found found;
    __shared__ float2 sums[WAVES][TC];
    __shared__ float part[WAVES][4 * S::kTiles][64];
    __shared__ OddSteps odd;
    if (threadIdx.x == 0) odd.clear(0);
    int turn = 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, quad = lane >> 4;
    const int kh = (int)(blockIdx.x % (unsigned)a.cache.kv_heads), share = (int)(blockIdx.x / (unsigned)a.cache.kv_heads);
    typename W::Place p;
    uint32_t left = 0, all_steps = 0;
    if (!W::template find<256>(a, found, [&](uint32_t total) {
            if (!a.cut) return (uint32_t)share;
            all_steps = total;
            const uint32_t from = share_at(total, share, a.shares);
            left = share_at(total, share + 1, a.shares) - from;
            return from;
        }, p)) {
        if (a.cut && a.shares > 1 && tid == 0) cut_tiles(a, TC, D)[kh * a.shares + share].last = -1;
        return;
    }
    if (!a.cut) left = p.of;

    const int page = 1 << a.cache.page_shift;
    // a lane's keys of a step, and where their bytes are in 16 of them
    const int k_in = ((8 * (n >> 2) + (n & 3)) & 15) * S::kRowBytes + quad * 16;
    const int v_in = 8 * (quad & 1) * S::kRowBytes + n * S::kBytesV;

    while (true) {
        const uint32_t to = min(p.of, p.at + left);
        const bool whole = p.at == 0 && to == p.of;
        const int context = p.q.keys - p.q.n, columns = p.q.n * a.group, c0 = p.t * TC;
        // queries: the scores' other operand
        bf16x8 q[C][S::kSteps];
        int sees[C];        // last key a column sees (no tree)
        uint64_t word[C];   // which of its request's own keys (tree)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            int col = c0 + 16 * c + n;
            if (col >= columns) col = c0;
            const int i = row_of_column(a, col), row = p.q.first + i, h = kh * a.group + (col - i * a.group);
            const uint16_t *at = a.q.p + row * a.q.token + h * a.q.head;
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) q[c][s] = as_bf16x8(flipped(ld16(at + (F8 ? 64 * (s >> 1) + 16 * quad + 8 * (s & 1) : 32 * s + 8 * quad)), a.flip));
            sees[c] = context + i;
            word[c] = a.tree ? a.tree[row] : 0;
        }
        const int rows = row_of_column(a, min(columns, c0 + TC) - 1) - row_of_column(a, c0) + 1;  // that the tile is of
        // keys up to here are seen by all
        const int open = min(p.q.keys, a.tree ? context : context + row_of_column(a, c0) + 1);

        f32x4 o[C][S::kTiles];
        float top[C], sum[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            top[c] = -INFINITY;
            sum[c] = 0.f;
#pragma unroll
            for (int i = 0; i < S::kTiles; ++i) o[c][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        constexpr int B = S::kBlocks;
        Bytes<16> k[B][2][S::kLoadsK];
        Bytes<S::kBytesV> v[B][8];
        float4 ks[B][2], vs[B][2];
        // the pages of a wavefront's keys at step j, 16 by 16; -1 where there is none
        struct Pages {
            int id[2 * B];
        };
        const int32_t *table = a.table + p.r * a.ld_table;
        auto pages_of = [&](uint32_t j) __attribute__((always_inline)) {
            Pages g;
            const int key = (int)j * KEYS + 32 * B * wave;
#pragma unroll
            for (int i = 0; i < 2 * B; ++i) {
                const int at = key + 16 * i;
                const int id = at < p.q.keys ? table[at >> a.cache.page_shift] : -1;
                g.id[i] = (unsigned)id < (unsigned)a.cache.pages ? id : -1;
            }
            return g;
        };
        auto base_of = [&](const Pages &g, uint32_t j, int i) __attribute__((always_inline)) {
            const int in = ((int)j * KEYS + 32 * B * wave + 16 * i) & (page - 1);
            return ((int64_t)max(g.id[i], 0) * a.cache.kv_heads + kh) * page + in;  // in rows
        };
        auto load_k = [&](const Pages &g, uint32_t j) __attribute__((always_inline)) {
#pragma unroll
            for (int y = 0; y < B; ++y) {
                const int64_t r0 = base_of(g, j, 2 * y), r1 = base_of(g, j, 2 * y + 1);
                const char *at = a.cache.k + (n < 8 ? r0 : r1) * S::kRowBytes + k_in;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int s = 0; s < S::kLoadsK; ++s) k[y][t][s] = ld_bytes_once<16>(at + t * 4 * S::kRowBytes + s * 64);
                if constexpr (F8) {
                    const float *sc = a.cache.k_scales + (quad < 2 ? r0 : r1) + 8 * (quad & 1);
                    ks[y][0] = *reinterpret_cast<const float4 *>(sc);
                    ks[y][1] = *reinterpret_cast<const float4 *>(sc + 4);
                }
            }
        };
        auto load_v = [&](const Pages &g, uint32_t j) __attribute__((always_inline)) {
#pragma unroll
            for (int y = 0; y < B; ++y) {
                const int64_t r0 = base_of(g, j, 2 * y), r1 = base_of(g, j, 2 * y + 1), r = quad < 2 ? r0 : r1;
                const char *at = a.cache.v + r * S::kRowBytes + v_in;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[y][i] = ld_bytes_once<S::kBytesV>(at + i * S::kRowBytes);
                if constexpr (F8) {
                    const float *sc = a.cache.v_scales + r + 8 * (quad & 1);
                    vs[y][0] = *reinterpret_cast<const float4 *>(sc);
                    vs[y][1] = *reinterpret_cast<const float4 *>(sc + 4);
                }
            }
        };
        auto four = [](const float4 &f, int i) __attribute__((always_inline)) { return i == 0 ? f.x : i == 1 ? f.y : i == 2 ? f.z : f.w; };

        if (p.q.keys > 0) {
            Pages now = pages_of(p.at), then = pages_of(p.at + 1 < to ? p.at + 1 : p.at);
            load_k(now, p.at);
            load_v(now, p.at);
            for (uint32_t j = p.at; j < to; ++j) {
                const uint32_t j1 = j + 1 < to ? j + 1 : j, j2 = j + 2 < to ? j + 2 : j1;
                const Pages after = pages_of(j2);
                const int key0 = (int)j * KEYS + 32 * B * wave, mine = key0 + 8 * quad;
                bool plain = key0 + 32 * B <= open;
#pragma unroll
                for (int i = 0; i < 2 * B; ++i) plain &= now.id[i] >= 0;
                // scores
                f32x4 sc[C][B][2];
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int y = 0; y < B; ++y) sc[c][y][0] = sc[c][y][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < S::kSteps; ++s)
#pragma unroll
                    for (int y = 0; y < B; ++y)
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            bf16x8 x;
                            if constexpr (F8) {
                                const uint32_t w0 = k[y][t][s >> 1].w[2 * (s & 1)], w1 = k[y][t][s >> 1].w[2 * (s & 1) + 1];
                                x = as_bf16x8(uint4{two_of_e4m3<false>(w0), two_of_e4m3<true>(w0), two_of_e4m3<false>(w1), two_of_e4m3<true>(w1)});
                            } else {
                                x = __builtin_bit_cast(bf16x8, k[y][t][s]);
                            }
#pragma unroll
                            for (int c = 0; c < C; ++c) sc[c][y][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[c][s], sc[c][y][t], 0, 0, 0);
                        }
                if constexpr (F8) {
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int y = 0; y < B; ++y)
#pragma unroll
                            for (int i = 0; i < 8; ++i) sc[c][y][i >> 2][i & 3] *= four(ks[y][i >> 2], i & 3);
                }
                load_k(then, j1);
                uint32_t seen[C][B];
                if (!plain) {
#pragma unroll
                    for (int y = 0; y < B; ++y) {
                        const bool held = (quad < 2 ? now.id[2 * y] : now.id[2 * y + 1]) >= 0;  // (an index by lane would put them into memory)
#pragma unroll
                        for (int c = 0; c < C; ++c) {
                            seen[c][y] = seen_of(mine + 32 * y, held ? p.q.keys : 0, a.tree, sees[c], word[c], mine + 32 * y - context);
#pragma unroll
                            for (int i = 0; i < 8; ++i) sc[c][y][i >> 2][i & 3] = seen[c][y] >> i & 1 ? sc[c][y][i >> 2][i & 3] : -INFINITY;
                        }
                        // values that no column sees are taken as zero: of one row's columns those that it does not see, of more the keys that there are none of, and
                        // (see OddSteps) infinities and NaN
                        const uint32_t there = rows > 1 ? first_bits(held ? p.q.keys - (mine + 32 * y) : 0) : seen[0][y];
                        uint32_t some = 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
#pragma unroll
                            for (int x = 0; x < S::kBytesV / 4; ++x) {
                                v[y][i].w[x] &= 0u - (there >> i & 1);
                                if (rows > 1) v[y][i].w[x] = finite_of<F8>(v[y][i].w[x], some);
                            }
                        if (some) odd.note(turn, j);
                    }
                }
                // weights
                uint4 w[C][B];
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float t = sc[c][0][0][0];
#pragma unroll
                    for (int i = 1; i < 8 * B; ++i) t = fmaxf(t, sc[c][i >> 3][i >> 2 & 1][i & 3]);
                    t = max_of_quads(t);
                    if (__any(t > top[c] + a.slack)) {
                        t = fmaxf(t, top[c]);
                        const float f = t == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((top[c] - t) * a.scale);
                        sum[c] *= f;
#pragma unroll
                        for (int i = 0; i < S::kTiles; ++i) o[c][i] *= f;
                        top[c] = t;
                    }
                    const float from = top[c] == -INFINITY ? 0.f : -top[c] * a.scale;
#pragma unroll
                    for (int y = 0; y < B; ++y) {
                        uint32_t pairs[4];
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            float e0 = __builtin_amdgcn_exp2f(fmaf(sc[c][y][i >> 2][i & 3], a.scale, from));
                            float e1 = __builtin_amdgcn_exp2f(fmaf(sc[c][y][i >> 2][(i & 3) + 1], a.scale, from));
                            if constexpr (F8) {
                                sum[c] += e0 + e1;
                                e0 *= four(vs[y][i >> 2], i & 3);
                                e1 *= four(vs[y][i >> 2], (i & 3) + 1);
                            }
                            pairs[i / 2] = pack_bf16_rne(e0, e1);
                            if constexpr (!F8) sum[c] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pairs[i / 2]), bf16x2{(__bf16)1.f, (__bf16)1.f}, sum[c], false);
                        }
                        if (F8 && !plain) {  // (nought times a scale that is none is none)
#pragma unroll
                            for (int i = 0; i < 8; i += 2) {
                                const uint32_t two = seen[c][y] >> i;
                                pairs[i / 2] &= ((0u - (two & 1)) & 0xFFFFu) | ((0u - (two >> 1 & 1)) & 0xFFFF0000u);
                            }
                        }
                        w[c][y] = uint4{pairs[0], pairs[1], pairs[2], pairs[3]};
                    }
                }
                // values
#pragma unroll
                for (int y = 0; y < B; ++y) {
                    auto add = [&](int i, uint4 vt) __attribute__((always_inline)) {
#pragma unroll
                        for (int c = 0; c < C; ++c) o[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vt), as_bf16x8(w[c][y]), o[c][i], 0, 0, 0);
                    };
                    if constexpr (F8) {
#pragma unroll
                        for (int x = 0; x < S::kBytesV / 4; ++x) {
                            uint32_t four_keys[2][4];
#pragma unroll
                            for (int z = 0; z < 2; ++z) {
                                const uint32_t v0 = v[y][4 * z].w[x], v1 = v[y][4 * z + 1].w[x], v2 = v[y][4 * z + 2].w[x], v3 = v[y][4 * z + 3].w[x];
                                const uint32_t l01 = __builtin_amdgcn_perm(v1, v0, 0x05010400u), l23 = __builtin_amdgcn_perm(v3, v2, 0x05010400u);
                                const uint32_t h01 = __builtin_amdgcn_perm(v1, v0, 0x07030602u), h23 = __builtin_amdgcn_perm(v3, v2, 0x07030602u);
                                four_keys[z][0] = __builtin_amdgcn_perm(l23, l01, 0x05040100u);
                                four_keys[z][1] = __builtin_amdgcn_perm(l23, l01, 0x07060302u);
                                four_keys[z][2] = __builtin_amdgcn_perm(h23, h01, 0x05040100u);
                                four_keys[z][3] = __builtin_amdgcn_perm(h23, h01, 0x07060302u);
                            }
#pragma unroll
                            for (int b = 0; b < 4; ++b)
                                add(4 * x + b, uint4{two_of_e4m3<false>(four_keys[0][b]), two_of_e4m3<true>(four_keys[0][b]), two_of_e4m3<false>(four_keys[1][b]),
                                                     two_of_e4m3<true>(four_keys[1][b])});
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < S::kTiles; ++i) {
                            uint32_t d[4];
#pragma unroll
                            for (int z = 0; z < 4; ++z) d[z] = __builtin_amdgcn_perm(v[y][2 * z + 1].w[i >> 1], v[y][2 * z].w[i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
                            add(i, uint4{d[0], d[1], d[2], d[3]});
                        }
                    }
                }
                load_v(then, j1);
                now = then;
                then = after;
            }
        }

        // the wavefronts' sums: each on the largest of their maxima, then a quarter of a column's dims a wavefront
#pragma unroll
        for (int c = 0; c < C; ++c) {
            sum[c] = sum_of_quads(sum[c]);
            top[c] *= a.scale;
            if (quad == 0) sums[wave][16 * c + n] = float2{top[c], sum[c]};
        }
        __syncthreads();
        const int64_t slot = part_of(kh, a.shares, share, p.at == 0);
        float *slots = a.parts + (int64_t)a.cache.kv_heads * a.shares * 2 * TC * D;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float most = -INFINITY, all = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) most = fmaxf(most, sums[i][16 * c + n].x);
            const float from = most == -INFINITY ? 0.f : most, f = __builtin_amdgcn_exp2f(top[c] - from);
#pragma unroll
            for (int i = 0; i < WAVES; ++i) all += sums[i][16 * c + n].y * __builtin_amdgcn_exp2f(sums[i][16 * c + n].x - from);
            if (c > 0) __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < S::kTiles; ++i) part[wave][e * S::kTiles + i][lane] = o[c][i][e] * f;
            __syncthreads();
            const int in = 16 * c + n, col = c0 + in;
            if (col < columns) {
                float z[S::kTiles];
                const int dim = S::kTiles * (4 * quad + wave);
#pragma unroll
                for (int i = 0; i < S::kTiles; ++i) {
                    const int at = wave * S::kTiles + i;
                    z[i] = part[0][at][lane] + part[1][at][lane] + part[2][at][lane] + part[3][at][lane];
                }
                if (whole) {
                    const float by = all == 0.f ? 0.f : __builtin_amdgcn_rcpf(all);
                    const int i = row_of_column(a, col), row = p.q.first + i, h = kh * a.group + (col - i * a.group);
                    uint32_t *y = reinterpret_cast<uint32_t *>(a.y.p + row * a.y.token + h * a.y.head + dim);
#pragma unroll
                    for (int x = 0; x < S::kTiles; x += 4) *reinterpret_cast<uint2 *>(y + x / 2) = uint2{pack_bf16_rne(z[x] * by, z[x + 1] * by), pack_bf16_rne(z[x + 2] * by, z[x + 3] * by)};
                } else {
                    float *y = a.parts + (slot * TC + in) * D + dim;
#pragma unroll
                    for (int x = 0; x < S::kTiles; x += 4) *reinterpret_cast<float4 *>(y + x) = float4{z[x], z[x + 1], z[x + 2], z[x + 3]};
                    if (wave == 0 && quad == 0) *reinterpret_cast<float2 *>(slots + (slot * TC + in) * 2) = float2{most, all};
                }
            }
        }
        if (tid == 0) odd.clear(turn ^ 1);
        __syncthreads();
        if (odd.to[turn]) add_odd<D, F8, 256>(a, p, kh, odd.from[turn] * KEYS, odd.to[turn] * KEYS, c0, TC, whole, a.parts + slot * TC * D);
        turn ^= 1;
        left -= to - p.at;
        if (left == 0) {
            if (a.cut && a.shares > 1 && tid == 0) leave_cut(a, cut_tiles(a, TC, D) + kh * a.shares + share, all_steps, share, p, c0, p.of - to);
            return;
        }
        if (!W::next(a, p)) return;  // (steps are left, so there is a tile)
    }
}

// ------------------------------------------------------------------------------------------------
// Attention of many columns: tiles of 32 a wavefront, whose four or eight wavefronts share the keys and values of a step in LDS: 64 keys of 128 dims, or 128 of 64.
// S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 matrix instructions, 32 keys at a time.  A lane (half h, column n) ends up with the scores of keys
// 8 i + 4 h + 0 .. 3 of those; as in k_attend_few they become an operand where they are, for V^T is laid out by the same order of keys: piece (2 ks + h) of a dim's row
// has the keys 16 ks + 4 h + {0 .. 3, 8 .. 11}.  Half of the wavefronts fetch V and half K, through registers, a step ahead of LDS: V is turned there (a thread has 8 keys x
// kDimsV dims), 8-bit values become bf16 there, once for all wavefronts.  In LDS 16-byte pieces of a row are exchanged by its number so that neither writes nor reads
// of eight lanes meet in a bank.  Maxima and roundings are k_attend_few's.
//
// Bound by one wavefront's chain of instructions and the two on a SIMD, which overlap products and the rest in part only: pieces of 2000 to 4096 rows behind 4000 to
// 16000 keys, 961 GFLOP, 990 to 1040 us, 0.92 to 0.97 PFLOP/s (a large library product 1.23).  Of an earlier 1035 us the exponentials were 65, putting keys and values
// into LDS 135 and asking for them 125, though they were near (the same keys over and over: level).  So addresses come from lanes that have them (by a few instructions
// on one lane's value: trees 75.7 to 72.8), and eight wavefronts wait for each other every second step (with that 1065 to 1035; 131 KB of LDS, which one work group a
// compute unit has to itself).  The order laid down in `take` took it from 1200.  Trees of 8 to 24 tokens, 289 MB: 63 to 66 us and 8 of join, on another card 83 in all
// (3.9 to 4.5 TB/s), by the 64 KB that a compute unit's two work groups have on the way.  Registers are full with heads of 128, and some are spilled: 2 and 8 in bf16 (eight
// and four wavefronts), 27 and 32 in 8 bits; with heads of 64 none.  In 8 bits with heads of 128 the trees take 81 us (bf16 72) for half the bytes, 8 prompts of 256 to
// 2048 tokens 75 (59), the pieces 1100 (1000).  64 columns a wavefront instead of 32, half as many reads of LDS a product: 2066 to
// 2700 against 1435 then, one wavefront a SIMD; loads past the caches 1202 against 1080.  32 keys at a time with the exponentials beside the next ones' products: 1033
// against 1023, trees 76 against 73.6; the wavefronts that bring K doing so behind their products, those that bring V before: 1046 against 1030.
// ------------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(16))) float f32x16;

template <int D, bool F8, int WAVES>
struct WideShape {
    static constexpr int kKeys = 8192 / D;               // of a step
    static constexpr int kRow = D * (F8 ? 1 : 2);        // bytes of a key or value in the cache
    static constexpr int kGroups = kKeys / 16;           // of keys that lie on one page
    static constexpr int kSteps = D / 16;                // of k, of the scores
    static constexpr int kDims = D / 32;                 // tiles of O^T
    static constexpr int kDimsV = 32 / WAVES;            // a thread's of V
    static constexpr int kWordsV = kDimsV * (F8 ? 1 : 2) / 4;  // .. of a key
    static constexpr int kLoadsK = (F8 ? 16 : 32) / WAVES;     // of 16 bytes, a thread's
    static constexpr int kAcross = kRow / 16;            // threads that have a row of K
    static constexpr int kHeld = 8 * kWordsV > 4 * kLoadsK ? 8 * kWordsV : 4 * kLoadsK;
    // by which a row's pieces are exchanged.  K [key][dim]; V^T [dim][key], which is also written across its rows: eight threads of one piece, kDimsV rows apart
    static __device__ __forceinline__ int mix_k(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int mix_v(int r)
    {
        return D == 128 ? ((r >> 1) & 3) ^ ((r >> 3) & 1) ^ ((r >> 4) & 1) << 2 ^ ((r >> 5) & 1) << 1
                        : (r & 7) ^ ((r >> 3) & 1) << 3 ^ ((r >> 4) & 1) << 1 ^ ((r >> 5) & 1) << 2;
    }
    static __device__ __forceinline__ int k_at(int r, int p) { return r * (2 * D) + 16 * (p ^ mix_k(r)); }
    static __device__ __forceinline__ int v_at(int r, int p) { return r * (2 * kKeys) + 16 * (p ^ mix_v(r)); }
};

template <int D, bool F8, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void k_attend_wide(AttendArgs a)
{
    using S = WideShape<D, F8, WAVES>;
    constexpr int TC = 32 * WAVES, KEYS = S::kKeys;
    using W = Dealt<TC, KEYS>;
    __shared__ typename W::Found found;
    constexpr int kBuffers = WAVES == 8 ? 4 : 2, kAhead = kBuffers / 2;  // steps that are in LDS; half of them are being read, and the wavefronts wait for each other once they were
    __shared__ __attribute__((aligned(16))) char ks[kBuffers][16384], vs[kBuffers][16384];
    __shared__ __attribute__((aligned(16))) float scales[F8 ? kBuffers : 1][2][F8 ? KEYS : 4];
    __shared__ OddSteps odd;
    if (threadIdx.x == 0) odd.clear(0);
    int turn = 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const int kh = (int)(blockIdx.x % (unsigned)a.cache.kv_heads), share = (int)(blockIdx.x / (unsigned)a.cache.kv_heads);
    typename W::Place p;
    uint32_t left = 0, all_steps = 0;
    if (!W::template find<64 * WAVES>(a, found, [&](uint32_t total) {
            if (!a.cut) return (uint32_t)share;
            all_steps = total;
            const uint32_t from = share_at(total, share, a.shares);
            left = share_at(total, share + 1, a.shares) - from;
            return from;
        }, p)) {
        if (a.cut && a.shares > 1 && tid == 0) cut_tiles(a, TC, D)[kh * a.shares + share].last = -1;
        return;
    }
    if (!a.cut) left = p.of;
    const int page = 1 << a.cache.page_shift;
    const bool loads_v = wave < WAVES / 2;
    // V: 8 keys and kDimsV dims of a thread.  K: its row and piece within a load
    constexpr int kWide = D / S::kDimsV;  // threads that have a row of V
    const int vt = tid & (32 * WAVES - 1), v_kg = vt / kWide, v_dims = (vt % kWide) * S::kDimsV;
    const int k_row = lane / S::kAcross, k_piece = lane % S::kAcross, k_first = (wave - WAVES / 2) * (2 * KEYS / WAVES);
    constexpr int kRows = 64 / S::kAcross;  // of K in a load: 16 at most
    // where a lane's operands are
    int k_off[S::kSteps], v_off[KEYS / 16];
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) k_off[x] = S::k_at(n, 2 * x + h);
#pragma unroll
    for (int z = 0; z < KEYS / 16; ++z) v_off[z] = S::v_at(n, 2 * z + h);

    while (true) {
        const uint32_t to = min(p.of, p.at + left);
        const bool whole = p.at == 0 && to == p.of;
        const int context = p.q.keys - p.q.n, columns = p.q.n * a.group, c0 = p.t * TC;
        const bool busy = c0 + wave * 32 < columns;
        bf16x8 q[S::kSteps];
        int sees;
        uint64_t word;
        {
            int col = c0 + wave * 32 + n;
            if (col >= columns) col = c0;
            const int i = row_of_column(a, col), row = p.q.first + i, hd = kh * a.group + (col - i * a.group);
            const uint16_t *at = a.q.p + row * a.q.token + hd * a.q.head;
#pragma unroll
            for (int s = 0; s < S::kSteps; ++s) q[s] = as_bf16x8(flipped(ld16(at + 16 * s + 8 * h), a.flip));
            sees = context + i;
            word = a.tree ? a.tree[row] : 0;
        }
        // keys up to here are seen by all columns of the tile
        const int open = min(p.q.keys, a.tree ? context : context + row_of_column(a, c0) + 1);

        f32x16 o[S::kDims];
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < S::kDims; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] = 0.f;

        const int32_t *table = a.table + p.r * a.ld_table;
        // a lane has the page of 16 keys, group lane mod kGroups; -1 where there is none
        auto page_of = [&](uint32_t j) __attribute__((always_inline)) {
            const int key = (int)j * KEYS + 16 * (lane & (S::kGroups - 1));
            const int id = key < p.q.keys ? table[key >> a.cache.page_shift] : -1;
            return (unsigned)id < (unsigned)a.cache.pages ? id : -1;
        };
        uint32_t held[S::kHeld];  // fetched for the next step: of K, or of V (a key's after the other's)
        float sr[2];
        // rows of the cache in front of a lane's 16 keys (as page_of); one wavefront's loads take a lane's value as theirs
        auto rows_of = [&](int id, uint32_t j) __attribute__((always_inline)) {
            const int in = ((int)j * KEYS + 16 * (lane & (S::kGroups - 1))) & (page - 1);
            return (((int64_t)max(id, 0) * a.cache.kv_heads + kh) << a.cache.page_shift) + in;
        };
        auto lane_of = [&](int64_t v, int of) __attribute__((always_inline)) {
            return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), of) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, of));
        };
        auto any_lane_of = [&](int64_t v, int of) __attribute__((always_inline)) {
            return (int64_t)((uint64_t)(uint32_t)__shfl((int)(v >> 32), of, 64) << 32 | (uint32_t)__shfl((int)v, of, 64));
        };
        auto fetch = [&](int ids, uint32_t j) __attribute__((always_inline)) {
            const int64_t rows = rows_of(ids, j);
            if (loads_v) {
                const uint32_t in = (4 * (v_kg & 1)) * S::kRow + v_dims * (F8 ? 1 : 2);
                const char *at;
                if constexpr (2 * kWide >= 64)
                    at = a.cache.v + lane_of(rows, wave * (64 / kWide) >> 1) * S::kRow + in;
                else
                    at = a.cache.v + any_lane_of(rows, v_kg >> 1) * S::kRow + in;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const auto got = ld_bytes<4 * S::kWordsV>(at + (i < 4 ? i : i + 4) * S::kRow);
#pragma unroll
                    for (int x = 0; x < S::kWordsV; ++x) held[S::kWordsV * i + x] = got.w[x];
                }
                asm volatile("; values");  // (the two ways end differently: the compiler would else join their loads, a register at a time)
            } else {
                const uint32_t in = k_row * S::kRow + 16 * k_piece;
#pragma unroll
                for (int i = 0; i < S::kLoadsK; ++i) {
                    const int first = k_first + i * kRows;
                    const auto got = ld_bytes<16>(a.cache.k + (lane_of(rows, first >> 4) + (first & 15)) * S::kRow + in);
#pragma unroll
                    for (int x = 0; x < 4; ++x) held[4 * i + x] = got.w[x];
                }
                asm volatile("; keys");
            }
            if constexpr (F8) {
                if (tid < KEYS) {
                    const int64_t row = any_lane_of(rows, tid >> 4) + (tid & 15);
                    sr[0] = a.cache.k_scales[row];
                    sr[1] = a.cache.v_scales[row];
                }
            }
        };
        // ids: of the step that was fetched
        auto stage = [&](int ids, uint32_t j, int b) __attribute__((always_inline)) {
            const int key0 = (int)j * KEYS;
            if (loads_v) {
                const bool plain = key0 + KEYS <= open && __ballot(ids < 0) == 0;
                const int group = v_kg >> 1, first = key0 + 16 * group + 4 * (v_kg & 1);
                if (!plain) {
                    const uint32_t there = first_bits(__shfl(ids, group, 64) >= 0 ? p.q.keys - first : 0);
                    uint32_t some = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int x = 0; x < S::kWordsV; ++x)
                            held[S::kWordsV * i + x] = finite_of<F8>(held[S::kWordsV * i + x] & (0u - (there >> (i < 4 ? i : i + 4) & 1)), some);
                    if (some) odd.note(turn, j);
                }
                uint4 turned[S::kDimsV];
                if constexpr (F8) {
#pragma unroll
                    for (int x = 0; x < S::kWordsV; ++x) {
                        uint32_t four_keys[2][4];
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            auto v = [&](int i) __attribute__((always_inline)) { return held[S::kWordsV * (4 * y + i) + x]; };
                            const uint32_t l01 = __builtin_amdgcn_perm(v(1), v(0), 0x05010400u), l23 = __builtin_amdgcn_perm(v(3), v(2), 0x05010400u);
                            const uint32_t h01 = __builtin_amdgcn_perm(v(1), v(0), 0x07030602u), h23 = __builtin_amdgcn_perm(v(3), v(2), 0x07030602u);
                            four_keys[y][0] = __builtin_amdgcn_perm(l23, l01, 0x05040100u);
                            four_keys[y][1] = __builtin_amdgcn_perm(l23, l01, 0x07060302u);
                            four_keys[y][2] = __builtin_amdgcn_perm(h23, h01, 0x05040100u);
                            four_keys[y][3] = __builtin_amdgcn_perm(h23, h01, 0x07060302u);
                        }
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            turned[4 * x + c] = uint4{two_of_e4m3<false>(four_keys[0][c]), two_of_e4m3<true>(four_keys[0][c]), two_of_e4m3<false>(four_keys[1][c]),
                                                      two_of_e4m3<true>(four_keys[1][c])};
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < S::kDimsV; ++c) {
                        uint32_t d[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            d[y] = __builtin_amdgcn_perm(held[S::kWordsV * (2 * y + 1) + (c >> 1)], held[S::kWordsV * 2 * y + (c >> 1)], c & 1 ? 0x07060302u : 0x05040100u);
                        turned[c] = uint4{d[0], d[1], d[2], d[3]};
                    }
                }
#pragma unroll
                for (int c = 0; c < S::kDimsV; ++c) *reinterpret_cast<uint4 *>(vs[b] + S::v_at(v_dims + c, v_kg)) = turned[c];
                asm volatile("; values");
            } else {
#pragma unroll
                for (int i = 0; i < S::kLoadsK; ++i) {
                    const int key = k_first + i * kRows + k_row;
                    const uint32_t *w = held + 4 * i;
                    if constexpr (F8) {
                        *reinterpret_cast<uint4 *>(ks[b] + S::k_at(key, 2 * k_piece)) =
                            uint4{two_of_e4m3<false>(w[0]), two_of_e4m3<true>(w[0]), two_of_e4m3<false>(w[1]), two_of_e4m3<true>(w[1])};
                        *reinterpret_cast<uint4 *>(ks[b] + S::k_at(key, 2 * k_piece + 1)) =
                            uint4{two_of_e4m3<false>(w[2]), two_of_e4m3<true>(w[2]), two_of_e4m3<false>(w[3]), two_of_e4m3<true>(w[3])};
                    } else {
                        *reinterpret_cast<uint4 *>(ks[b] + S::k_at(key, k_piece)) = uint4{w[0], w[1], w[2], w[3]};
                    }
                }
                asm volatile("; keys");
            }
            if constexpr (F8) {
                const bool there = __shfl(ids, (tid & (KEYS - 1)) >> 4, 64) >= 0 && key0 + (tid & (KEYS - 1)) < p.q.keys;
                if (tid < KEYS) {
                    scales[b][0][tid] = sr[0];
                    scales[b][1][tid] = there ? sr[1] : 0.f;
                }
            }
        };

        // A step's keys, 64 at a time.  The order of instructions is laid down: operands are read from LDS beside the matrix instructions in front of those that
        // need them, and the second half's exponentials beside the first half's product with v.
        auto take = [&](bool plain, int b, int key0, uint64_t none) __attribute__((always_inline)) {
            constexpr int kPv = 2 * S::kDims;  // matrix instructions of 32 keys with v
            constexpr bool kEarly = WAVES == 8;  // (with four wavefronts each holds twice as much of the next step: it would have to put registers by)
            const char *kb = ks[b], *vb = vs[b];
            auto four = [](const float4 &f, int i) __attribute__((always_inline)) { return i == 0 ? f.x : i == 1 ? f.y : i == 2 ? f.z : f.w; };
#pragma unroll
            for (int u = 0; u < KEYS / 64; ++u) {
                auto read_k = [&](int kt, int x) __attribute__((always_inline)) { return as_bf16x8(*reinterpret_cast<const uint4 *>(kb + k_off[x] + kt * 64 * D)); };
                auto read_v = [&](int kt, int i) __attribute__((always_inline)) {
                    const int z = (2 * kt + i / S::kDims) ^ (i % S::kDims & 1) << (D == 128 ? 0 : 1);  // (mix_v takes bit 5 of the row)
                    return as_bf16x8(*reinterpret_cast<const uint4 *>(vb + v_off[z] + i % S::kDims * 64 * KEYS));
                };
                bf16x8 k[S::kSteps], v[kPv];
                f32x16 s[2];
#pragma unroll
                for (int e = 0; e < 16; ++e) s[0][e] = s[1][e] = 0.f;
                constexpr int kHalf = S::kSteps / 2;
#pragma unroll
                for (int x = 0; x < S::kSteps; ++x) k[x] = read_k(2 * u + (x & 1), x >> 1);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);  // products before what else the SIMD's other wavefront has (pieces 1002 to 989 us, large trees 72.5 to 70.1)
                // (the two tiles' products in turn: the next one of a sum would wait for the one before; trees 73.6 to 72.2 us)
#pragma unroll
                for (int x = 0; x < S::kSteps; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        bf16x8 &at = k[2 * (x % kHalf) + y];
                        s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at, q[x], s[y], 0, 0, 0);
                        if (x < kHalf)
                            at = read_k(2 * u + y, x + kHalf);
                        else if (kEarly && 2 * (x - kHalf) + y < kPv)
                            v[2 * (x - kHalf) + y] = read_v(2 * u, 2 * (x - kHalf) + y);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                __builtin_amdgcn_s_setprio(0);
                [[maybe_unused]] float4 by_v[4];
                uint32_t seen[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    if constexpr (F8) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float4 by_k = *reinterpret_cast<const float4 *>(&scales[b][0][64 * u + 32 * y + 8 * i + 4 * h]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[y][4 * i + e] *= four(by_k, e);
                        }
                    }
                    if (!plain) {
                        const int kt = 2 * u + y, first = key0 + 32 * kt;
                        const uint32_t there = ((none >> (2 * kt) & 1 ? 0u : 0xFFFFu) | (none >> (2 * kt + 1) & 1 ? 0u : 0xFFFF0000u)) >> (4 * h);
                        seen[y] = seen_of(first, p.q.keys, a.tree, sees, word, first - context) >> (4 * h) & there;
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[y][e] = seen[y] >> (8 * (e >> 2) + (e & 3)) & 1 ? s[y][e] : -INFINITY;
                    }
                }
                float t = fmaxf(s[0][0], s[1][0]);
#pragma unroll
                for (int e = 1; e < 16; ++e) t = fmaxf(fmaxf(t, s[0][e]), s[1][e]);
                t = max_of_halves(t);
                if (__any(t > top + a.slack)) {
                    t = fmaxf(t, top);
                    const float f = t == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((top - t) * a.scale);
                    sum *= f;
#pragma unroll
                    for (int i = 0; i < S::kDims; ++i) o[i] *= f;
                    top = t;
                }
                const float from = top == -INFINITY ? 0.f : -top * a.scale;
                uint32_t w[2][8];
                // two weights
                auto weigh = [&](int y, int e) __attribute__((always_inline)) {
                    float e0 = __builtin_amdgcn_exp2f(fmaf(s[y][e], a.scale, from)), e1 = __builtin_amdgcn_exp2f(fmaf(s[y][e + 1], a.scale, from));
                    if constexpr (F8) {
                        sum += e0 + e1;
                        e0 *= four(by_v[e >> 2], e & 3);
                        e1 *= four(by_v[e >> 2], (e & 3) + 1);
                    }
                    w[y][e / 2] = pack_bf16_rne(e0, e1);
                    if constexpr (!F8) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[y][e / 2]), bf16x2{(__bf16)1.f, (__bf16)1.f}, sum, false);
                };
                // (nought times a scale that is none is none)
                auto only_seen = [&](int y) __attribute__((always_inline)) {
                    if (F8 && !plain) {
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            const uint32_t pair = seen[y] >> (8 * (e >> 2) + (e & 3));
                            w[y][e / 2] &= (0u - (pair & 1) & 0xFFFFu) | (0u - (pair >> 1 & 1) & 0xFFFF0000u);
                        }
                    }
                };
                auto product = [&](int y, int i) __attribute__((always_inline)) {
                    const uint32_t *x = w[y] + 4 * (i / S::kDims);
                    o[i % S::kDims] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[i], as_bf16x8(uint4{x[0], x[1], x[2], x[3]}), o[i % S::kDims], 0, 0, 0);
                };
                auto read_scales = [&](int y) __attribute__((always_inline)) {
                    if constexpr (F8) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) by_v[i] = *reinterpret_cast<const float4 *>(&scales[b][1][64 * u + 32 * y + 8 * i + 4 * h]);
                    }
                };
                read_scales(0);
#pragma unroll
                for (int e = 0; e < 16; e += 2) weigh(0, e);
                only_seen(0);
                if constexpr (!kEarly) {
#pragma unroll
                    for (int i = 0; i < kPv; ++i) v[i] = read_v(2 * u, i);
                }
                read_scales(1);
                __builtin_amdgcn_s_setprio(1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < kPv; ++i) {
                    product(0, i);
                    v[i] = read_v(2 * u + 1, i);
#pragma unroll
                    for (int e = 16 / kPv * i; e < 16 / kPv * (i + 1); e += 2) weigh(1, e);
                    __builtin_amdgcn_sched_barrier(0);
                }
                only_seen(1);
#pragma unroll
                for (int i = 0; i < kPv; ++i) product(1, i);
                __builtin_amdgcn_s_setprio(0);
            }
        };
        if (p.q.keys > 0) {
            int ids[kAhead + 1];  // pages of the steps from j on
#pragma unroll
            for (int i = 0; i <= kAhead; ++i) ids[i] = page_of(p.at + i < to ? p.at + i : to - 1);
#pragma unroll
            for (int i = 0; i <= kAhead; ++i)
                if (p.at + i < to) {
                    fetch(ids[i], p.at + i);
                    if (i < kAhead) stage(ids[i], p.at + i, i);
                }
            __syncthreads();
            for (uint32_t j = p.at; j < to; ++j) {
                const int b = (j - p.at) & (kBuffers - 1);
                const int after = page_of(j + kAhead + 1 < to ? j + kAhead + 1 : to - 1);
                const int key0 = (int)j * KEYS;
                const uint64_t none = __ballot(ids[0] < 0);
                const bool plain = none == 0 && key0 + KEYS <= open;
                if (j + kAhead < to) stage(ids[kAhead], j + kAhead, b ^ kAhead);
                if (j + kAhead + 1 < to) fetch(after, j + kAhead + 1);
                if (busy) take(plain, b, key0, none);
                if ((b & (kAhead - 1)) == kAhead - 1) __syncthreads();
#pragma unroll
                for (int i = 0; i < kAhead; ++i) ids[i] = ids[i + 1];
                ids[kAhead] = after;
            }
        } else {
            __syncthreads();  // (what the tile before noted in `odd` has been read by all, and is cleared below)
        }

        const int64_t slot = part_of(kh, a.shares, share, p.at == 0);
        const int in = wave * 32 + n, col = c0 + in;
        const float all = sum_of_halves(sum);
        if (col < columns) {
            if (whole) {
                const float by = all == 0.f ? 0.f : __builtin_amdgcn_rcpf(all);
                const int i = row_of_column(a, col), row = p.q.first + i, hd = kh * a.group + (col - i * a.group);
                uint16_t *y = a.y.p + row * a.y.token + hd * a.y.head + 4 * h;
#pragma unroll
                for (int x = 0; x < S::kDims; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *reinterpret_cast<uint2 *>(y + 32 * x + 8 * e) =
                            uint2{pack_bf16_rne(o[x][4 * e] * by, o[x][4 * e + 1] * by), pack_bf16_rne(o[x][4 * e + 2] * by, o[x][4 * e + 3] * by)};
            } else {
                float *slots = a.parts + (int64_t)a.cache.kv_heads * a.shares * 2 * TC * D;
                float *y = a.parts + (slot * TC + in) * D + 4 * h;
#pragma unroll
                for (int x = 0; x < S::kDims; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *reinterpret_cast<float4 *>(y + 32 * x + 8 * e) = float4{o[x][4 * e], o[x][4 * e + 1], o[x][4 * e + 2], o[x][4 * e + 3]};
                if (h == 0) *reinterpret_cast<float2 *>(slots + (slot * TC + in) * 2) = float2{top * a.scale, all};
            }
        }
        if (tid == 0) odd.clear(turn ^ 1);
        __syncthreads();
        if (odd.to[turn]) add_odd<D, F8, 64 * WAVES>(a, p, kh, odd.from[turn] * KEYS, odd.to[turn] * KEYS, c0, TC, whole, a.parts + slot * TC * D);
        turn ^= 1;
        left -= to - p.at;
        if (left == 0) {
            if (a.cut && a.shares > 1 && tid == 0) leave_cut(a, cut_tiles(a, TC, D) + kh * a.shares + share, all_steps, share, p, c0, p.of - to);
            return;
        }
        if (!W::next(a, p)) return;  // (steps are left, so there is a tile)
    }
}

// Tiles that several shares have a part of: a work group has CW columns of the one that a share began and did not end.  16 / CW groups of threads share the parts, four
// of which a thread asks for at a time.  Bound by its own start and three trips to memory: 2.6 to 5 us behind few columns, 6 to 15 behind many (256 columns of 128 dims
// are 133 KB a part; 28 MB of them behind the trees of k_attend_wide's comment, 8 us).  Done by the last share to end instead, it would need counters that someone has
// cleared.
template <int D, int TC, int CW>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a)
{
    constexpr int kEach = D / 16, kGroups = 16 / CW;
    __shared__ float tops[256 / CW][CW], sums[kGroups][CW], rows[kGroups][CW][D];
    const int tid = threadIdx.x, kh = (int)(blockIdx.x % (unsigned)a.cache.kv_heads), share = (int)(blockIdx.x / (unsigned)a.cache.kv_heads);
    const CutTile tile = cut_tiles(a, TC, D)[kh * a.shares + share];
    const int in0 = CW * blockIdx.y, columns = tile.columns - tile.c0, last = tile.last;
    if (last < 0 || in0 >= columns) return;
    const float *slots = a.parts + (int64_t)a.cache.kv_heads * a.shares * 2 * TC * D;
    auto slot_of = [&](int s) __attribute__((always_inline)) { return part_of(kh, a.shares, s, s == share) * TC + in0; };
    {
        const int c = tid % CW;
        float most = -INFINITY;
        for (int s = share + tid / CW; s <= last; s += 256 / CW) most = fmaxf(most, slots[(slot_of(s) + c) * 2]);
        tops[tid / CW][c] = most;
    }
    __syncthreads();
    const int c = tid / (16 * kGroups), grp = tid / 16 % kGroups, dim = (tid & 15) * kEach;
    float most = -INFINITY;
    for (int i = 0; i < min(256 / CW, last - share + 1); ++i) most = fmaxf(most, tops[i][c]);
    const float from = most == -INFINITY ? 0.f : most;
    float all = 0.f, z[kEach] = {};
    for (int s = share + grp; s <= last; s += 4 * kGroups) {
        float2 sum[4];
        float part[4][kEach];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t at = slot_of(min(s + i * kGroups, last)) + c;
            sum[i] = *reinterpret_cast<const float2 *>(slots + at * 2);
#pragma unroll
            for (int x = 0; x < kEach; x += 4) *reinterpret_cast<float4 *>(part[i] + x) = *reinterpret_cast<const float4 *>(a.parts + at * D + dim + x);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool there = s + i * kGroups <= last;
            const float f = __builtin_amdgcn_exp2f(sum[i].x - from);
            all += there ? sum[i].y * f : 0.f;
#pragma unroll
            for (int x = 0; x < kEach; ++x) z[x] += there ? part[i][x] * f : 0.f;
        }
    }
    if constexpr (kGroups > 1) {
        if ((tid & 15) == 0) sums[grp][c] = all;
#pragma unroll
        for (int x = 0; x < kEach; ++x) rows[grp][c][dim + x] = z[x];
        __syncthreads();
        if (grp > 0) return;
        for (int g = 1; g < kGroups; ++g) {
            all += sums[g][c];
#pragma unroll
            for (int x = 0; x < kEach; ++x) z[x] += rows[g][c][dim + x];
        }
    }
    if (in0 + c >= columns) return;
    const float by = all == 0.f ? 0.f : __builtin_amdgcn_rcpf(all);
    const int col = tile.c0 + in0 + c, i = row_of_column(a, col), row = tile.first + i, h = kh * a.group + (col - i * a.group);
    uint32_t *y = reinterpret_cast<uint32_t *>(a.y.p + row * a.y.token + h * a.y.head + dim);
#pragma unroll
    for (int x = 0; x < kEach; x += 4) *reinterpret_cast<uint2 *>(y + x / 2) = uint2{pack_bf16_rne(z[x] * by, z[x + 1] * by), pack_bf16_rne(z[x + 2] * by, z[x + 3] * by)};
}

template <int D, int TC>
static hipError_t launch_join(const AttendArgs &a, hipStream_t stream)
{
    const unsigned ends = (unsigned)(a.shares - 1) * a.cache.kv_heads;
    // Columns of a work group, 4 / 16, us a call.  Few requests among many shares, whose tiles have many parts: one token of 1500 keys 10.5 / 11.0, five long
    // requests 142.2 / 143.4; more requests: 42 trees of up to 7 tokens 35.8 / 34.4, 83 of 2 48.6 / 47.6; tiles of many columns: trees 79 / 76 and 79 / 74.
    if constexpr (TC <= 32) {
        if (4 * (int64_t)a.requests < a.shares) {
            hipLaunchKernelGGL((k_attend_join<D, TC, 4>), dim3(ends, TC / 4), dim3(256), 0, stream, a);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((k_attend_join<D, TC, 16>), dim3(ends, TC / 16), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <int D, bool F8, int C>
static hipError_t launch_few(const AttendArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((k_attend_few<D, F8, C>), dim3((unsigned)a.shares * a.cache.kv_heads), dim3(64 * kFewWaves), 0, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || !a.cut || a.shares == 1) return e;
    return launch_join<D, 16 * C>(a, stream);
}

template <int D, bool F8, int WAVES>
static hipError_t launch_wide(const AttendArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL((k_attend_wide<D, F8, WAVES>), dim3((unsigned)a.shares * a.cache.kv_heads), dim3(64 * WAVES), 0, stream, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || !a.cut || a.shares == 1) return e;
    return launch_join<D, 32 * WAVES>(a, stream);
}

hipError_t launch_attention(AttendArgs a, const AttendForm &f, hipStream_t stream)
{
    a.shares = f.shares;
    a.cut = f.cut;
    a.least = f.least;
    a.most = f.most;
    auto by_columns = [&](auto dim, auto f8) {
        constexpr int D = decltype(dim)::value;
        constexpr bool F8 = decltype(f8)::value;
        return f.columns == 16    ? launch_few<D, F8, 1>(a, stream)
               : f.columns == 32  ? launch_few<D, F8, 2>(a, stream)
               : f.columns == 128 ? launch_wide<D, F8, 4>(a, stream)
                                  : launch_wide<D, F8, 8>(a, stream);
    };
    auto by_bits = [&](auto dim) { return a.cache.bits8 ? by_columns(dim, std::true_type{}) : by_columns(dim, std::false_type{}); };
    return a.cache.dim == 64 ? by_bits(std::integral_constant<int, 64>{}) : by_bits(std::integral_constant<int, 128>{});
}

}  // namespace lora
