// gfx950 kernels of the frozen layers beside an adapter (include/lora_experts.h): rows to 8 bits, products in block-scaled 8 bits and in
// bf16 over rows grouped by expert, the grouping itself, and the weighted sum behind it.
//
// Both element types walk k in pieces of 128 bytes: 64 bf16 or 128 8-bit values.  A weight tile of 16 columns x one piece is, for either type,
// two operands of 16 bytes a lane (halves of the piece): two 16x16x32 bf16 MFMAs, or one 16x16x128 f8f6f4 MFMA that takes both.  So
// the weights are packed alike:
//   expert e, 128-column strip, piece P, half h, sub-block b of 8, lane slot (kq, n): 16 bytes
//     128 P + 64 h + 16 kq .. of column 128 strip + 64 (b / 4) + 4 n + b mod 4
//   at  ((e * strips + strip) * pieces + P) * 16384 + operand_at(h, b) + (16 kq + n) * 16
// A wavefront's load of an operand is 1 KB of consecutive bytes, and of four sub-blocks lane n ends up with four consecutive columns.
// Half of a piece of a strip is what a large tile multiplies by at a time: in bf16 the first half of k for all columns, in 8 bits all of k
// for the first 64 columns.  The token operand uses the same mapping of lanes to k.
#include "lora_device.h"
#include "lora_experts.h"
#include "lora_internal.h"

#include <type_traits>

namespace lora {

typedef __attribute__((ext_vector_type(8))) int i32x8;

static __device__ __forceinline__ uint4 ldb16(const char *p) { return *reinterpret_cast<const uint4 *>(p); }
// past the caches, where ONCE says that nobody else wants it
template <bool ONCE>
static __device__ __forceinline__ uint4 ldw16(const char *p)
{
    return ONCE ? ld16_stream(reinterpret_cast<const uint16_t *>(p)) : ldb16(p);
}

static __device__ __forceinline__ i32x8 as_i32x8(uint4 lo, uint4 hi)
{
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

template <bool F8>
static __device__ __forceinline__ constexpr int operand_at(int h, int b)
{
    return F8 ? (b >> 2) * 8192 + h * 4096 + (b & 3) * 1024 : h * 8192 + b * 1024;
}

// LDS operations of a wavefront complete in order; the compiler keeps them so
static __device__ __forceinline__ void in_order()
{
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// A weight's scale as 2^(power - 127), which the matrix instruction applies to its sum for nothing, times the factor left over: half to one, unless the
// scale is beyond 2^100 or 2^-100.  x's scale times the whole one can be far below 2^-126, where it would lose bits (x's alone goes down to that) though y does not: a
// sum of 128 products of up to 448^2 lies up to 2^25 above it.  x's scale times the factor loses none to speak of, and never overflows where x's scale does
// not; a sum times 2^-100 to 2^100 is still exact.  Zero, infinities and NaN stay in the factor.
struct WeightScale {
    float factor;
    int powers;  // of x's operand (127: times one) in the first byte, of W's in the second: one register for both
};
constexpr int kPowersOne = 127 | 127 << 8;
static __device__ __forceinline__ WeightScale weight_scale(float w)
{
    const int e = min(max((int)((__float_as_uint(w) >> 23) & 0xFFu) - 126, -100), 100);
    return WeightScale{w * __uint_as_float((uint32_t)(127 - e) << 23), kPowersOne + (e << 8)};
}

// 16 x 16 products over 128 8-bit values of k (both operands E4M3, b's times 2^(power - 127)).  The instruction drops what lies 2^-17 below the
// largest of an element's 128 products (all in all up to 2^-10 of that product was seen), and the ones for 32 values of k do the same: of those that take 8 bits there is
// none more exact.  (E4M3 is exact in bf16, whose instruction adds in fp32: that would take twice as long at the matrix units and a conversion of
// every operand.)  A block's sum is fp32 from there on.
static __device__ __forceinline__ f32x4 mfma_e4m3(i32x8 a, i32x8 b, int powers)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, powers, 1, powers);
}

// ------------------------------------------------------------------------------------------------
// Which expert, rows and columns a work group's tile has.  The tiles of a launch are numbered expert by expert, inside it column tile by column tile,
// inside that row tile by row tile, so that a run of them shares its weights; how many there are follows from `starts` on the device
// alone, and every wavefront finds its tile by itself (a prefix sum over the experts' row tiles, 64 experts at a time).
// ------------------------------------------------------------------------------------------------
struct Tile {
    int expert, ct;
    int row0, rows;  // first place, places
    bool only;       // of wide tiles: the expert has no other rows
    bool four;       // .. those of up to 128 rows have four strips of columns, not two
};

static __device__ __forceinline__ int wave_scan(int v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d, 64);
        v += lane >= d ? o : 0;
    }
    return v;
}

// an expert's first place and how many it has; starts that do not fit the rows give an expert fewer or none
static __device__ __forceinline__ int expert_rows(const int32_t *__restrict__ starts, int e, int n_rows, int &first)
{
    const int a = min(max(starts[e], 0), n_rows), b = min(max(starts[e + 1], 0), n_rows);
    first = a;
    return max(b - a, 0);
}

static __device__ __forceinline__ int wave_sum(int v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return __builtin_amdgcn_readfirstlane(v);
}

// Row tile q of all, experts in their order, tiles(rows) of them for an expert: its expert, which of the expert's it is, how many those are, and the
// expert's places.  q is one of them.
struct RowTile {
    int expert, m, of, first, rows;
};
template <class Tiles>
static __device__ __forceinline__ RowTile find_row_tile(const int32_t *__restrict__ starts, int n_experts, int n_rows, int lane, int q, Tiles tiles)
{
    int before = 0;
    for (int base = 0; base < n_experts; base += 64) {
        const int e = base + lane;
        int first = 0;
        const int rows = e < n_experts ? expert_rows(starts, e, n_rows, first) : 0;
        const int mt = tiles(rows), upto = before + wave_scan(mt, lane);
        const uint64_t hit = __ballot(q < upto);
        if (hit) {
            const int l = __builtin_ctzll(hit), e_mt = __shfl(mt, l, 64);
            return RowTile{__builtin_amdgcn_readfirstlane(base + l), __builtin_amdgcn_readfirstlane(q - (__shfl(upto, l, 64) - e_mt)),
                           __builtin_amdgcn_readfirstlane(e_mt), __builtin_amdgcn_readfirstlane(__shfl(first, l, 64)),
                           __builtin_amdgcn_readfirstlane(__shfl(rows, l, 64))};
        }
        before = __shfl(upto, 63, 64);
    }
    return RowTile{0, 0, 1, 0, 0};
}

// The tile of R rows that work group `blk` has, of all; false if none.  Work group b runs on XCD b mod 8: every XCD an eighth of the tiles, in one run.
template <int R>
static __device__ __forceinline__ bool find_tile(const int32_t *__restrict__ starts, int n_experts, int n_rows, int n_ct, int lane, int blk, Tile &t)
{
    auto tiles = [](int rows) { return (rows + R - 1) / R; };
    int mine = 0, first;
    if (starts)
        for (int e = lane; e < n_experts; e += 64) mine += tiles(expert_rows(starts, e, n_rows, first));
    const int total = (starts ? wave_sum(mine) : tiles(n_rows)) * n_ct, per_xcd = (total + 7) >> 3, idx = (blk & 7) * per_xcd + (blk >> 3);
    if ((blk >> 3) >= per_xcd || idx >= total) return false;
    const RowTile r = starts ? find_row_tile(starts, n_experts, n_rows, lane, idx / n_ct, tiles) : RowTile{0, 0, tiles(n_rows), 0, n_rows};
    // inside an expert column tile by column tile, so that neighbours share W: which it is
    const int in_e = starts ? idx - (idx / n_ct - r.m) * n_ct : idx;
    t.ct = in_e / r.of;
    const int row = (in_e - t.ct * r.of) * R;
    t.expert = r.expert;
    t.row0 = r.first + row;
    t.rows = min(R, r.rows - row);
    return true;
}

// A tile of up to 128 rows has two strips of 128 columns, or four.  With two it takes 5/8 as long as a whole one (8 bits, k 4096: 37 - 43 us and 65; its
// wavefronts have 64 x 64 of it and wait for LDS), with four, where they have 64 x 128, little longer than that (63 - 71).  So: four where all tiles
// are then through earlier, in eighths of a whole one, by the count of tiles; where the compute units that whole ones leave have room for all of two strips, two.
// us, always two / always four / so: 6000 rows of 64 experts 4096 -> 2048 in 8 bits 131 / - / 106, 32 experts' 6000 of uneven numbers 100 / - / 89;
// 2560 rows of 32 3456 -> 1664 40.6 / 55.1 / 41.8, 2688 of 32 4352 -> 6272 207 / 172 / 178; over 36 random sizes of experts 4 %, 3 % and 2 % from the
// better of the first two.
static __device__ __forceinline__ bool four_strips(int whole, int n_rest, int n_ct)
{
    const int rest = n_rest * n_ct, rest4 = n_rest * ((n_ct + 1) >> 1), rounds = whole / kComputeUnits, left = whole - rounds * kComputeUnits;
    const int room = kComputeUnits - left;
    if (rest <= room) return false;
    return 8 * ((whole + rest4 + kComputeUnits - 1) / kComputeUnits) < max(8 * rounds + 10, (8 * whole + 5 * rest) / kComputeUnits + 3);
}

// How many whole tiles, the last ones, are cut into two of 128 rows: those of the last round of compute units, where all of them and the tiles of up to 128
// rows are through in one round that way.  8 bits, us, whole / cut: 1665 rows 1088 -> 11520 (315 tiles) 42.6 / 37.1, 2500 rows 4096 -> 7680 (300) 110 / 97,
// 3000 rows of 15 experts 4096 -> 2048 (120) 62.4 / 46.
static __host__ __device__ __forceinline__ int cut_tiles(int whole, int rest)
{
    const int left = whole % kComputeUnits;
    return 2 * left + rest <= kComputeUnits ? left : 0;
}

// The same for tiles of 256 rows x 256 columns, an expert's last one of up to 128 rows apart: the whole ones come first, and the others, which take about
// half as long, fill the compute units that the last round of those leaves idle.  Inside an expert column tiles in groups of four, in a group row tile by row tile:
// of 32 tiles in a run, one on each of an XCD's compute units, 8 row tiles x 4 column tiles walk k together, and every chunk of x and W that
// one of them brings into the XCD's L2 serves four or eight of them (8192 tokens 8192 -> 8192 in 8 bits 567 us column by column, 502 so).
static __device__ __forceinline__ bool find_wide_tile(const int32_t *__restrict__ starts, int n_experts, int n_rows, int n_ct, int lane, int blk, Tile &t)
{
    auto whole = [](int rows) { return (rows + 127) >> 8; };
    auto rest = [](int rows) { return ((rows + 255) >> 8) - ((rows + 127) >> 8); };
    int n_whole = whole(n_rows), n_rest = rest(n_rows);
    if (starts) {
        int a = 0, b = 0, first;
        for (int e = lane; e < n_experts; e += 64) {
            const int rows = expert_rows(starts, e, n_rows, first);
            a += whole(rows);
            b += rest(rows);
        }
        n_whole = wave_sum(a);
        n_rest = wave_sum(b);
    }
    const int cut = cut_tiles(n_whole * n_ct, n_rest * n_ct), uncut = n_whole * n_ct - cut;
    t.four = cut == 0 && four_strips(n_whole * n_ct, n_rest, n_ct);
    const int xcd = blk & 7, per_uncut = (uncut + 7) >> 3, per_cut = (2 * cut + 7) >> 3;
    int j = blk >> 3, half = -1, idx;  // half of a tile cut in two
    bool is_rest = false;
    if (j < per_uncut) {
        idx = xcd * per_uncut + j;
        if (idx >= uncut) return false;
    } else if ((j -= per_uncut) < per_cut) {
        idx = xcd * per_cut + j;
        if (idx >= 2 * cut) return false;
        half = idx & 1;
        idx = uncut + (idx >> 1);
    } else {
        j -= per_cut;
        is_rest = true;
        if (t.four) n_ct = (n_ct + 1) >> 1;
        const int per_rest = (n_rest * n_ct + 7) >> 3;
        idx = xcd * per_rest + j;
        if (j >= per_rest || idx >= n_rest * n_ct) return false;
    }
    const int q = idx / n_ct;
    const RowTile r = !starts   ? RowTile{0, is_rest ? 0 : q, is_rest ? n_rest : n_whole, 0, n_rows}
                      : is_rest ? find_row_tile(starts, n_experts, n_rows, lane, q, rest)
                                : find_row_tile(starts, n_experts, n_rows, lane, q, whole);
    const int in_e = idx - (q - r.m) * n_ct, grp = in_e / (r.of * 4), left = in_e - grp * (r.of * 4), wide = min(4, n_ct - grp * 4);
    const int m = left / wide, row = (is_rest ? whole(r.rows) : m) * 256 + (half > 0 ? 128 : 0);
    t.expert = r.expert;
    t.ct = grp * 4 + left - m * wide;
    t.row0 = r.first + row;
    t.rows = min(half < 0 ? 256 : 128, r.rows - row);
    t.only = half < 0 && r.rows <= 256;
    return true;
}

// row of x at a place, -1 if the order names none
static __device__ __forceinline__ int token_at(const ExpertsArgs &a, int place)
{
    int t = place;
    if (a.order) {
        const int pick = a.order[place];
        t = pick < 0 ? -1 : (int)((unsigned)pick / (unsigned)a.picks);
    }
    return t < a.tokens ? t : -1;
}

// ------------------------------------------------------------------------------------------------
// Tiles of few rows.  A work group has 16 RB rows x 16 CB columns, its wavefronts split k: wavefront w takes the pieces w, w + WAVES, ..,
// weights straight from memory in operand order, x as full cache lines through a private LDS region, no barrier in the loop; the partial sums
// meet in LDS in wavefront order.  What bounds it is one trip to memory, all of a wavefront's weights requested as early as registers allow: one row
// 4096 -> 4096 in 8 bits takes 4.6 us on the device (16.8 MB), 57 rows 3008 -> 1920 5.7.
// ------------------------------------------------------------------------------------------------
template <bool F8, int RB, int WAVES>
constexpr int kThinSlab = WAVES * (16 * RB * 128 + (F8 ? 16 * RB * 4 : 0));
template <bool F8, int RB, int CB, int WAVES>
constexpr int kThinLds = kThinSlab<F8, RB, WAVES> > WAVES * RB * CB * 1024 ? kThinSlab<F8, RB, WAVES> : WAVES *RB *CB * 1024;

template <bool F8, int RB, int CB, int D, int WAVES, bool ONCE>
__global__ __launch_bounds__(64 * WAVES, 1) void k_experts_thin(ExpertsArgs a)
{
    constexpr int NX = 2 * RB;                        // x loads of a wavefront per piece: 8 rows each
    constexpr int kSlab = 16 * RB * 128;              // bytes of a wavefront's x region
    constexpr int kRegion = kSlab + (F8 ? 64 * RB : 0);  // .. and the rows' scales
    constexpr int kTiles = RB * CB, R = 16 * RB;
    static_assert(RB <= 4, "a lane for the scale of every row");
    static_assert(CB <= 4, "sub-blocks of one half of a strip");
    __shared__ __attribute__((aligned(16))) char lds[kThinLds<F8, RB, CB, WAVES>];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, kq = lane >> 4;
    Tile t;
    if (!find_tile<R>(a.starts, a.n_experts, a.n_rows, a.out / (16 * CB), lane, (int)blockIdx.x, t)) return;
    const int strip = t.ct / (8 / CB), b0 = t.ct % (8 / CB) * CB;

    f32x4 acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int b = 0; b < CB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int np = a.pieces;
    const int mine = wave < np ? (np - 1 - wave) / WAVES + 1 : 0;
    if (mine > 0) {
        char *slab = lds + wave * kRegion;
        const int lr = lane >> 3, lc = lane & 7;
        // x: lane -> row lane / 8 of the load's 8, 16 bytes lane mod 8; in the region chunk c of row r sits in slot c XOR (r mod 8), so that
        // neither the writes nor the operand reads meet in a bank.  Rows the tile does not have read those of its first place.
        const char *xrow[NX];
#pragma unroll
        for (int q = 0; q < NX; ++q) {
            const int r = 8 * q + lr;
            const int tok = token_at(a, t.row0 + (r < t.rows ? r : 0));
            xrow[q] = a.x + (int64_t)max(tok, 0) * a.ldx_bytes + kPieceBytes * wave + 16 * lc;
        }
        const char *wbase = a.w + ((int64_t)t.expert * (a.out >> 7) + strip) * np * 16384 + (int64_t)wave * 16384 + operand_at<F8>(0, b0) + lane * 16;
        const float *xs_at = nullptr, *ws_at = nullptr;
        if constexpr (F8) {
            const int tok = token_at(a, t.row0 + (lane < t.rows ? lane : 0));
            xs_at = a.x_scales + (int64_t)max(tok, 0) * a.ld_scales + wave;
            int zero = 0;
            asm("" : "+v"(zero));  // (a vector load, counted in order with the others)
            ws_at = a.w_scales + ((int64_t)t.expert * (a.out >> 7) + strip) * np + wave + zero;
        }
        uint4 xq[D][NX], wq[D][2][CB];
        [[maybe_unused]] float sx[D], sw[D];
        // Loads without branches (around one the compiler would wait for everything in flight): past the last piece, the last one again.
        auto load_x = [&](int i, int d) __attribute__((always_inline)) {
            const int64_t at = i < mine ? i : mine - 1;
#pragma unroll
            for (int q = 0; q < NX; ++q) xq[d][q] = ldb16(xrow[q] + at * (kPieceBytes * WAVES));
            if constexpr (F8) {
                sx[d] = xs_at[at * WAVES];
                sw[d] = ws_at[at * WAVES];
            }
        };
        auto load_w = [&](int i, int d) __attribute__((always_inline)) {
            const int64_t at = i < mine ? i : mine - 1;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int b = 0; b < CB; ++b) wq[d][h][b] = ldw16<ONCE>(wbase + at * (16384 * WAVES) + operand_at<F8>(h, b));
        };
        [[maybe_unused]] int powers = kPowersOne;  // of the staged piece's scale of W
        auto stage = [&](int d) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < NX; ++q) *reinterpret_cast<uint4 *>(slab + (8 * q + lr) * 128 + ((lc ^ lr) << 4)) = xq[d][q];
            if constexpr (F8) {
                const WeightScale s = weight_scale(sw[d]);
                powers = s.powers;
                if (lane < R) reinterpret_cast<float *>(slab + kSlab)[lane] = sx[d] * s.factor;
            }
        };
        auto compute = [&](int d) __attribute__((always_inline)) {
            uint4 xo[2][RB];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < RB; ++i)
                    xo[h][i] = *reinterpret_cast<const uint4 *>(slab + (16 * i + n) * 128 + (((4 * h + kq) ^ (n & 7)) << 4));
            if constexpr (F8) {
#pragma unroll
                for (int i = 0; i < RB; ++i) {
                    const f32x4 s = *reinterpret_cast<const f32x4 *>(slab + kSlab + (16 * i + 4 * kq) * 4);
#pragma unroll
                    for (int b = 0; b < CB; ++b)
                        acc[i][b] += s * mfma_e4m3(as_i32x8(xo[0][i], xo[1][i]), as_i32x8(wq[d][0][b], wq[d][1][b]), powers);
                }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < RB; ++i)
#pragma unroll
                        for (int b = 0; b < CB; ++b)
                            acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(xo[h][i]), as_bf16x8(wq[d][h][b]), acc[i][b], 0, 0, 0);
            }
        };
#pragma unroll
        for (int d = 0; d < D; ++d) {
            load_x(d, d);
            __builtin_amdgcn_sched_barrier(0);
            load_w(d, d);
            __builtin_amdgcn_sched_barrier(0);
        }
        for (int i0 = 0; i0 < mine; i0 += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                stage(d);
                load_x(i0 + d + D, d);
                in_order();  // (the region is private to this wavefront)
                if (i0 + d < mine) compute(d);
                load_w(i0 + d + D, d);
                in_order();  // (the region is private to this wavefront)
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    __syncthreads();  // everyone has left the x regions
    f32x4(*red)[kTiles][64] = reinterpret_cast<f32x4(*)[kTiles][64]>(lds);
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int b = 0; b < CB; ++b) red[wave][i * CB + b][lane] = acc[i][b];
    __syncthreads();
    for (int o = tid; o < RB * 256; o += 64 * WAVES) {
        // row 16 i + 4 kq + e of the tile, columns 64 (b0 / 4) + 4 n + b0 mod 4 .. + CB - 1 of the strip
        const int i = o >> 8, l = ((o >> 4) & 3) * 16 + (o & 15), e = (o >> 6) & 3;
        const int r = 16 * i + 4 * (l >> 4) + e;
        if (r >= t.rows || token_at(a, t.row0 + r) < 0) continue;
        float f[CB];
#pragma unroll
        for (int b = 0; b < CB; ++b) f[b] = reinterpret_cast<const float *>(&red[0][i * CB + b][l])[e];
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
#pragma unroll
            for (int b = 0; b < CB; ++b) f[b] += reinterpret_cast<const float *>(&red[w][i * CB + b][l])[e];
        uint16_t *const to = a.y + (int64_t)(t.row0 + r) * a.ldy + strip * 128 + (b0 >> 2) * 64 + 4 * (l & 15) + (b0 & 3);
        [[maybe_unused]] uint32_t *const dst = reinterpret_cast<uint32_t *>(to);
        if constexpr (CB == 4)
            *reinterpret_cast<uint2 *>(dst) = uint2{pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3])};
        else if constexpr (CB == 2)
            *dst = pack_bf16_rne(f[0], f[1]);
        else
            *to = (uint16_t)pack_bf16_rne(f[0], 0.f);
    }
}

template <bool F8, int RB, int CB, int D, int WAVES, bool ONCE = false>
static hipError_t launch_thin(const ExpertsArgs &a, hipStream_t stream)
{
    const int64_t row_tiles = ((int64_t)a.n_rows + 16 * RB - 1) / (16 * RB) + met_experts(a.starts ? a.n_experts : 0, a.n_rows);
    const int64_t grid = (row_tiles * (a.out / (16 * CB)) + 7) / 8 * 8;
    if (!can_launch(grid, 64 * WAVES)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_experts_thin<F8, RB, CB, D, WAVES, ONCE>), dim3((unsigned)grid), dim3(64 * WAVES), 0, stream, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// Tiles of many rows: 64 WR rows (256, or 128 where an expert's last tile has no more) x NS strips of 128 columns (2; 4 of few rows: see four_strips),
// 8 wavefronts.  Wavefronts 0 .. 3 have the first half of the strips, 4 .. 7 the second; a wavefront has 64 rows x 128 columns of one, or, where
// 128 rows x 2 strips leave it no more, 64 x 64.
//   * x and W come by loads that write LDS directly, x in slots of one piece (128 bytes of k), W in slots of a step: half a piece, the half that
//     the packed order says, or a piece (64 x 64).  Three slots each: a step requests W of the step after the next, and the first step of a
//     piece x of the piece after the next.  x is gathered by the copy itself, whole cache lines of 8 rows; inside a 1 KB block of 8 rows chunk p of row r
//     sits in slot 8 r + (p XOR r), so that the lanes that read one chunk of 8 rows meet 8 bank groups.
//   * A step is a phase that requests copies and reads the step's operands from LDS, and a phase that multiplies (512 cycles of the matrix unit), with a
//     barrier behind each and the second half's wavefronts one phase behind: of the two wavefronts of a SIMD one multiplies while the other reads.
//     No request passes through registers the compiler tracks, so the waits count exactly what is under way.
//   * In 8 bits a product spans a whole block of 128: its sum starts at zero, and 4 fp32 FMAs with x's scale times W's add it to the accumulators
//     while the next ones run (half as long as the matrix unit takes).  A wavefront copies the scales of its own 64 rows, of four pieces at a
//     time: every row's lie in cache lines of their own, and one copy a piece took as long as half of the others together (8192 tokens
//     8192 -> 8192: copies alone 418 us with one a piece, 304 without any).  Rows of x enter registers while the piece before is multiplied
//     (64 x 128): a piece's first reading phase had 20 of its 28 operands, and lasted longer than the products beside it.
//   * What bounds it is the chip's power: 8192 tokens 8192 -> 8192 in 8 bits take 476 us (2.31 PFLOP/s) at 2.0 of 2.4 GHz, and the parts add up like
//     energies, not like times: products and LDS reads alone 278 (products from registers alone run at 4.05 PFLOP/s, 271 us), copies 105 more, the fp32
//     sums 110 more, in phases or without, copies requested two steps ahead or four.  In bf16 8002 rows of 8 experts 4096 -> 14336 take 755 us
//     (1.25 PFLOP/s; a library's product of 8192 such rows 719 to 767, products from registers alone 1.90 PFLOP/s).
// ------------------------------------------------------------------------------------------------
constexpr int kWideThreads8 = 512;
constexpr int kRing = 3;
// Products between one and its sum.  A phase's last ones leave theirs to the reading phase behind it, where the other wavefront multiplies: us with all of them
// in the phase itself / 1, 2, 3, 4 behind it, 8192 tokens 8192 -> 8192 496 / 488, 491, 500, 488, 32 of 256 x 256 tiles 96.6 / 92.9, 95.8, 97, 94.
constexpr int kLag = 1;
constexpr int kWideLds = kRing * 49152 + 8 * 2048;  // (of whichever form, in 8 bits)

// One dword a lane straight to LDS: lane l's at `to` + 4 l.
static __device__ __forceinline__ void dma4_to_lds(const void *g, uint32_t to)
{
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0)
                 : "v"(g), "s"(to)
                 : "memory");
}

// 16 bytes a lane straight to LDS: lane l's at `to` + 16 l.
static __device__ __forceinline__ void dma16x1_to_lds(const void *g, uint32_t to)
{
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0)
                 : "v"(g), "s"(to)
                 : "memory");
}

// N KB (2 or 4) from consecutive addresses, base (of the wavefront) + 16 lane, to consecutive LDS addresses; ONCE: past the caches.
template <int N, bool ONCE>
static __device__ __forceinline__ void dma_kb_to_lds(const char *base, uint32_t lane16, uint32_t to)
{
    uint32_t saved_m0;
#define LORA_COPY(offset, how) "global_load_lds_dwordx4 %1, %2 offset:" #offset how "\n\t"
#define LORA_COPIES_2(how) LORA_COPY(0, how) LORA_COPY(1024, how)
#define LORA_COPIES_4(how) LORA_COPIES_2(how) LORA_COPY(2048, how) LORA_COPY(3072, how)
#define LORA_COPY_ASM(copies)                                                                                                               \
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\t" copies "s_mov_b32 m0, %0"                                          \
                 : "=&s"(saved_m0)                                                                                                          \
                 : "v"(lane16), "s"(base), "s"(to)                                                                                          \
                 : "memory")
    if constexpr (N == 4 && ONCE)
        LORA_COPY_ASM(LORA_COPIES_4(" nt"));
    else if constexpr (N == 4)
        LORA_COPY_ASM(LORA_COPIES_4(""));
    else if constexpr (ONCE)
        LORA_COPY_ASM(LORA_COPIES_2(" nt"));
    else
        LORA_COPY_ASM(LORA_COPIES_2(""));
#undef LORA_COPY_ASM
#undef LORA_COPIES_4
#undef LORA_COPIES_2
#undef LORA_COPY
}

// The tiles' values are computed by here: the compiler moves them neither up nor down.
template <int N>
static __device__ __forceinline__ void here(f32x4 (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}
template <bool F8, int WR, int NS, bool ONCE>
static __device__ __forceinline__ void wide_body(const ExpertsArgs &a, const Tile &t, char *lds)
{
    constexpr int WS = 8 / NS;                     // wavefronts of a strip
    constexpr bool FULL = WS == WR;                // .. which have all of its columns, or half of them
    constexpr int NB = FULL ? 8 : 4;               // sub-blocks of a wavefront
    constexpr int SP = FULL ? 2 : 1;               // steps of a piece
    constexpr int XBUF = 64 * WR * kPieceBytes, WPART = 16384 / SP, WBUF = NS * WPART;
    constexpr int XC = WR, WC = WPART / 1024 / WS; // copies of a wavefront: x of a piece, W of a step
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, kq = lane >> 4;
    const int rw = wave % WR;                      // rows 64 rw .. of the tile
    const int half = FULL ? 0 : (wave >> 1) & 1;
    const int strip = NS * t.ct + wave / WS;
    // The last tile of a row of y may hold one strip: the wavefronts without one copy strip 0's W for nothing.
    const bool has_strip = strip * 128 < a.out;
    const int np = a.pieces, steps = np * SP;

    char *const xring = lds, *const wring = lds + kRing * XBUF;
    // rows of x by 32-bit offsets in 16 bytes (the host sees to it that they fit), which take half of the registers of addresses
    uint32_t xoff[WR];
#pragma unroll
    for (int j = 0; j < WR; ++j) {
        const int r = lane >> 3, row = 8 * (WR * wave + j) + r;
        const int tok = token_at(a, t.row0 + (row < t.rows ? row : 0));
        xoff[j] = (uint32_t)((uint64_t)max(tok, 0) * (uint64_t)a.ldx_bytes >> 4) + ((lane & 7) ^ r);
    }
    const int my_row = 64 * rw + lane;
    const int my_tok = token_at(a, t.row0 + (my_row < t.rows ? my_row : 0));
    const uint64_t there = __ballot(my_row < t.rows && my_tok >= 0);  // rows of this wavefront that are written
    [[maybe_unused]] const uint32_t soff = F8 ? (uint32_t)((uint64_t)max(my_tok, 0) * (uint64_t)a.ld_scales) : 0u;
    const int64_t es = (int64_t)t.expert * (a.out >> 7) + (has_strip ? strip : 0);
    const char *wsrc = a.w + es * np * 16384 + (wave % WS) * (WC * 1024);
    const char *xp = a.x;            // the next piece of every row
    const uint32_t lane16 = lane * 16;
    // (the scalar cache's path: a vector load would be counted among the copies)
    const __attribute__((address_space(4))) float *wscale =
        (const __attribute__((address_space(4))) float *)(uintptr_t)(F8 ? a.w_scales + es * np : nullptr);

    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)lds);
    const uint32_t x_end = lds0 + kRing * XBUF, w_end = x_end + kRing * WBUF;
    uint32_t x_to = lds0 + WR * wave * 1024, w_to = x_end + wave / WS * WPART + wave % WS * (WC * 1024);
    auto issue_x = [&]() __attribute__((always_inline)) {
        auto at = [&](int j) { return xp + (uint64_t)xoff[j] * 16 - 1024 * j; };  // as the copies take it
        if constexpr (WR == 4)
            dma16x4_to_lds(at(0), at(1), at(2), at(3), x_to);
        else
            dma16x2_to_lds(at(0), at(1), x_to);
        xp += kPieceBytes;
        x_to = x_to + XBUF >= x_end ? x_to - (kRing - 1) * XBUF : x_to + XBUF;
    };
    // The scales of this wavefront's rows, [piece of four][row], in 2 KB of its own.  Where rows of scales are whole numbers of 16 bytes: one copy of four
    // pieces of every row into the second KB, put in order in the first one when its turn comes.  Else four copies, into one KB and the other in turn.
    [[maybe_unused]] char *const sbuf = lds + kRing * (XBUF + WBUF) + wave * 2048;
    [[maybe_unused]] const uint32_t s_to = w_end + wave * 2048;
    [[maybe_unused]] const bool by16 = ((uintptr_t)a.x_scales % 16 | a.ld_scales % 4 | np % 4) == 0;
    [[maybe_unused]] int fours = 0;  // of pieces requested
    auto issue_scales = [&]() __attribute__((always_inline)) {
        if (4 * fours >= np) return;
        const float *sp = a.x_scales + soff;
        if (by16)
            dma16x1_to_lds(sp + 4 * fours, s_to + 1024);
        else
#pragma unroll
            for (int c = 0; c < 4; ++c) dma4_to_lds(sp + min(4 * fours + c, np - 1), s_to + (fours & 1) * 1024 + 256 * c);
        ++fours;
    };
    auto order_scales = [&]() __attribute__((always_inline)) {
        if (!by16) return;
        const f32x4 v = *reinterpret_cast<const f32x4 *>(sbuf + 1024 + 16 * lane);
#pragma unroll
        for (int c = 0; c < 4; ++c) *reinterpret_cast<float *>(sbuf + 256 * c + 4 * lane) = v[c];
    };
    auto issue_w = [&]() __attribute__((always_inline)) {
        dma_kb_to_lds<WC, ONCE>(wsrc, lane16, w_to);
        wsrc += WPART;
        w_to = w_to + WBUF >= w_end ? w_to - (kRing - 1) * WBUF : w_to + WBUF;
    };

    f32x4 acc[NB / 4][16];  // of 64 columns: sub-block b, 16 rows i at 4 b + i
#pragma unroll
    for (int g = 0; g < NB / 4; ++g)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[g][k] = f32x4{0.f, 0.f, 0.f, 0.f};

    if constexpr (F8) {
        issue_scales();
        if (!by16) issue_scales();
    }
    issue_x();
    issue_w();
    if (steps > 1) issue_w();
    if (np > 1) issue_x();
    if (np > 1)
        wait_vm<XC + WC>();
    else if (steps > 1)
        wait_vm<WC>();
    else
        wait_vm<0>();

    // the end of a phase: every wavefront has come this far
    auto phase_end = [&]() __attribute__((always_inline)) {
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    };
    if constexpr (F8) {
        order_scales();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (by16) issue_scales();
    }
    phase_end();

    // The copies of step q of a piece behind which come two pieces or more (AFTER = 2), one or none, and the wait for W of the next step and, where that
    // begins a piece, x of it: behind them were requested W of the step after and x of the piece after.
    auto request = [&](auto qc, auto afterc) __attribute__((always_inline)) {
        constexpr int q = decltype(qc)::value, AFTER = decltype(afterc)::value;
        if constexpr (SP == 2 ? AFTER >= 1 : AFTER == 2) issue_w();
        if constexpr (q == 0 && AFTER == 2) issue_x();
    };
    auto await = [&](auto afterc) __attribute__((always_inline)) {
        constexpr int AFTER = decltype(afterc)::value;
        wait_vm<AFTER == 2 ? XC + WC : SP == 2 && AFTER == 1 ? WC : 0>();
    };
    auto pieces = [&](auto step) __attribute__((always_inline)) {
        auto piece = [&](int P, auto after) __attribute__((always_inline)) {
            step(P, std::integral_constant<int, 0>{}, after);
            if constexpr (SP == 2) step(P, std::integral_constant<int, 1>{}, after);
        };
        for (int P = 0; P + 2 < np; ++P) piece(P, std::integral_constant<int, 2>{});
        if (np > 1) piece(np - 2, std::integral_constant<int, 1>{});
        piece(np - 1, std::integral_constant<int, 0>{});
    };
    // a wavefront without rows or columns: its part of the copies, and the others' phases
    if (t.rows <= 64 * rw || !has_strip) {
        if (wave >= 4) phase_end();
        pieces([&](int, auto q, auto after) __attribute__((always_inline)) {
            request(q, after);
            await(after);
            phase_end();
            phase_end();
        });
        if (wave < 4) phase_end();
        return;
    }

    constexpr int XH = FULL && !F8 ? 1 : 2;  // halves of x's rows in registers at a time
    constexpr int WB = FULL && !F8 ? 8 : 4, WH = FULL && !F8 ? 1 : 2;  // .. sub-blocks and halves of W
    uint4 xo[XH][4], wo[WH][WB];
    [[maybe_unused]] f32x4 sc[4];
    int xget = 0, wget = 0;
    [[maybe_unused]] int sget = 0, powers = kPowersOne;
    const int xlane = (8 * rw + (n >> 3)) * 1024 + (n & 7) * 128;
    const int wlane = wave / WS * WPART + lane * 16;
    // row 16 i + n of this wavefront's: block 8 rw + 2 i + n / 8, row n mod 8 of it
    auto x_at = [&](int i, int h) __attribute__((always_inline)) {
        return *reinterpret_cast<const uint4 *>(xring + xget + xlane + 2048 * i + (((4 * h + kq) ^ (n & 7)) * 16));
    };
    constexpr bool kEarlyX = F8 && FULL;  // rows of x are read while the piece before is multiplied
    if constexpr (kEarlyX) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) xo[h][i] = x_at(i, h);
    }
    if (wave >= 4) phase_end();  // the second half's wavefronts run one phase behind the first's
    // 8 bits: product k of a step (rows k / 4, sub-block k mod 4 of it) and the sums kLag products behind it
    [[maybe_unused]] f32x4 part[kLag + 1];
    if constexpr (F8) {
#pragma unroll
        for (int k = 0; k <= kLag; ++k) part[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto add = [&](int q, int k) __attribute__((always_inline)) {
        f32x4 &to = acc[q][4 * (k & 3) + (k >> 2)];
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = fmaf(sc[k >> 2][e], part[k % (kLag + 1)][e], to[e]);
    };
    pieces([&](int P, auto qc, auto afterc) __attribute__((always_inline)) {
        constexpr int q = decltype(qc)::value, AFTER = decltype(afterc)::value;
        request(qc, afterc);
        if constexpr (!kEarlyX && (XH == 1 || q == 0))
#pragma unroll
            for (int h = 0; h < XH; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) xo[h][i] = x_at(i, XH == 1 ? q : h);
#pragma unroll
        for (int h = 0; h < WH; ++h)
#pragma unroll
            for (int b = 0; b < WB; ++b) {
                const int at = FULL ? (F8 ? h * 4096 : 0) + b * 1024 : operand_at<F8>(h, 4 * half + b);
                wo[h][b] = *reinterpret_cast<const uint4 *>(wring + wget + wlane + at);
            }
        if constexpr (F8) {  // the sums that the products before did not wait for
            __builtin_amdgcn_sched_barrier(0);
            constexpr int before = (q + SP - 1) % SP;
#pragma unroll
            for (int k = 16 - kLag; k < 16; ++k) add(before, k);
            here(acc[before]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (F8 && q == 0) {
            const WeightScale w = weight_scale(wscale[P]);
            powers = w.powers;
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[i] = *reinterpret_cast<const f32x4 *>(sbuf + sget + (16 * i + 4 * kq) * 4) * w.factor;
            sget = (sget + 256) & (by16 ? 1023 : 2047);
        }
        if constexpr (F8 && q == SP - 1)
            if ((P & 3) == 3 && P + 1 < np) order_scales();
        __builtin_amdgcn_sched_barrier(0);
        await(afterc);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what was read is in registers: the slots may be written
        // (requested four pieces before their use: long landed by the time that the waits above let a wavefront come there)
        if constexpr (F8 && q == SP - 1)
            if ((P & 3) == 3) issue_scales();
        phase_end();
        if constexpr (q == SP - 1) xget = xget == (kRing - 1) * XBUF ? 0 : xget + XBUF;
        if constexpr (F8) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                part[k % (kLag + 1)] = mfma_e4m3(as_i32x8(xo[0][k >> 2], xo[XH - 1][k >> 2]), as_i32x8(wo[0][k & 3], wo[WH - 1][k & 3]), powers);
                __builtin_amdgcn_sched_barrier(0);
                if (k >= kLag) add(q, k - kLag);
                // these rows of x have been multiplied: the next piece's.  All of it has landed: W of this step, requested behind it, has been waited
                // for by every wavefront.
                if constexpr (kEarlyX && q == SP - 1 && AFTER >= 1)
                    if ((k & 3) == 3)
#pragma unroll
                        for (int h = 0; h < 2; ++h) xo[h][k >> 2] = x_at(k >> 2, h);
                __builtin_amdgcn_sched_barrier(0);
            }
            here(part);
            here(acc[q]);
        } else {
#pragma unroll
            for (int h = 0; h < XH; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        acc[b >> 2][4 * (b & 3) + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(xo[h][i]), as_bf16x8(wo[h][b]), acc[b >> 2][4 * (b & 3) + i], 0, 0, 0);
#pragma unroll
            for (int g = 0; g < NB / 4; ++g) here(acc[g]);
        }
        phase_end();
        wget = wget == (kRing - 1) * WBUF ? 0 : wget + WBUF;
    });
    if constexpr (F8)
#pragma unroll
        for (int k = 16 - kLag; k < 16; ++k) add(SP - 1, k);
    if (wave < 4) phase_end();

    uint16_t *const y0 = a.y + (int64_t)(t.row0 + 64 * rw) * a.ldy + strip * 128 + 64 * half + 4 * n;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 16 * i + 4 * kq + e;
            if ((there >> r) & 1)
#pragma unroll
                for (int g = 0; g < NB / 4; ++g)
                    *reinterpret_cast<uint2 *>(y0 + (int64_t)r * a.ldy + 64 * g) =
                        uint2{pack_bf16_rne(acc[g][i][e], acc[g][4 + i][e]), pack_bf16_rne(acc[g][8 + i][e], acc[g][12 + i][e])};
        }
}

template <bool F8>
__global__ __launch_bounds__(kWideThreads8, 1) void k_experts_wide(ExpertsArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[F8 ? kWideLds : kWideLds - 8 * 2048];
    const int n_ct = (a.out + 255) >> 8;
    Tile t;
    if (!find_wide_tile(a.starts, a.n_experts, a.n_rows, n_ct, threadIdx.x & 63, (int)blockIdx.x, t)) return;
    // W past the caches where an expert has this one tile of rows and the weights are many (see large_weights): us, 64 experts of 64 rows each,
    // 2048 -> 1536, in bf16 90 / 83, in 8 bits 54.6 / 50.5
    if (t.rows > 128)
        t.only && a.large ? wide_body<F8, 4, 2, true>(a, t, lds) : wide_body<F8, 4, 2, false>(a, t, lds);
    else if (t.four)
        t.only && a.large ? wide_body<F8, 2, 4, true>(a, t, lds) : wide_body<F8, 2, 4, false>(a, t, lds);
    else
        t.only && a.large ? wide_body<F8, 2, 2, true>(a, t, lds) : wide_body<F8, 2, 2, false>(a, t, lds);
}

template <bool F8>
static hipError_t launch_wide(const ExpertsArgs &a, hipStream_t stream)
{
    const int64_t row_tiles = ((int64_t)a.n_rows + 255) / 256 + met_experts(a.starts ? a.n_experts : 0, a.n_rows), n_ct = (a.out + 255) / 256;
    // an eighth of each kind is rounded up, and up to half a round of tiles cut in two
    int64_t grid = (row_tiles * n_ct + 7) / 8 * 8 + 16 + kComputeUnits / 2;
    if (!can_launch(grid, kWideThreads8)) return hipErrorInvalidConfiguration;
    if (!a.starts) {  // known here (150 work groups without a tile take about 1 us)
        const int whole = (int)(((int64_t)a.n_rows + 127) / 256 * n_ct), rest = (int)(row_tiles * n_ct) - whole;
        grid = (int64_t)(whole + 7) / 8 * 8 + (cut_tiles(whole, rest) + 7) / 8 * 8 + (rest + 7) / 8 * 8;
    }
    hipLaunchKernelGGL(k_experts_wide<F8>, dim3((unsigned)grid), dim3(kWideThreads8), 0, stream, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// Tiles of up to 64 rows whose columns the wavefronts share out: 16 RB rows x 64 CB columns, four wavefronts of 16 CB columns each.  A wavefront's
// weights come straight from memory in operand order, D pieces ahead, and no other wavefront wants them; x, which all four want, passes through
// LDS, two slots of a piece, a barrier per piece.  A compute unit with one such tile has a wavefront per SIMD, whose loads, LDS reads, products and sums
// wait for each other, deeper prefetch or not; there KS = 2 such groups of wavefronts take the pieces in turn, and their sums meet in LDS.
// ------------------------------------------------------------------------------------------------
constexpr int kMidWaves = 4;

template <bool F8, int RB, int CB, int D, int KS>
constexpr int kMidLoopLds = KS * (2 * 16 * RB * kPieceBytes + (F8 ? kMidWaves * 16 * RB * 4 : 0));
template <bool F8, int RB, int CB, int D, int KS>
constexpr int kMidLds = KS == 2 && RB * CB * kMidWaves * 1024 > kMidLoopLds<F8, RB, CB, D, KS> ? RB *CB *kMidWaves * 1024 : kMidLoopLds<F8, RB, CB, D, KS>;

template <bool F8, int RB, int CB, int D, int KS, bool ONCE>
__global__ __launch_bounds__(64 * kMidWaves * KS, 1) void k_experts_mid(ExpertsArgs a)
{
    constexpr int R = 16 * RB, XBUF = R * kPieceBytes;
    constexpr int NX = RB / 2;  // x loads of a wavefront per piece
    static_assert(RB % 2 == 0 && R <= 64, "whole loads of x, and a lane for the scale of every row");
    static_assert(CB == 2 || CB == 4, "what a lane stores of a row");
    static_assert(D % 2 == 0, "slots of x by the place in the unrolled loop");
    __shared__ __attribute__((aligned(16))) char all_lds[kMidLds<F8, RB, CB, D, KS>];
    const int tid = threadIdx.x % (64 * kMidWaves), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ks = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / (64 * kMidWaves));  // pieces ks, ks + KS, ..
    char *const lds = all_lds + ks * (kMidLoopLds<F8, RB, CB, D, KS> / KS);
    const int n = lane & 15, kq = lane >> 4;
    Tile t;
    if (!find_tile<R>(a.starts, a.n_experts, a.n_rows, a.out / (64 * CB), lane, (int)blockIdx.x, t)) return;
    // this wavefront's sub-blocks, of all in the row
    const int b_all = (t.ct * kMidWaves + wave) * CB, strip = b_all >> 3, b0 = b_all & 7;
    const int np = a.pieces;

    f32x4 acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int b = 0; b < CB; ++b) acc[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};

    // x: 16 bytes a lane, 8 lanes a row, the tile's rows in order over the wavefronts; chunk c of row r goes to slot c XOR (r mod 8)
    const char *xrow[NX];
    int xput[NX];
#pragma unroll
    for (int q = 0; q < NX; ++q) {
        const int l = q * 64 * kMidWaves + tid, r = l >> 3, c = l & 7;
        const int tok = token_at(a, t.row0 + (r < t.rows ? r : 0));
        xrow[q] = a.x + (int64_t)max(tok, 0) * a.ldx_bytes + 16 * c;
        xput[q] = r * kPieceBytes + ((c ^ (r & 7)) << 4);
    }
    const char *wbase = a.w + ((int64_t)t.expert * (a.out >> 7) + strip) * np * 16384 + operand_at<F8>(0, b0);
    const unsigned lane16 = lane * 16;
    [[maybe_unused]] const float *xs_at = nullptr, *ws_at = nullptr;
    [[maybe_unused]] float *const sc = reinterpret_cast<float *>(lds + 2 * XBUF) + wave * R;
    if constexpr (F8) {
        const int tok = token_at(a, t.row0 + (lane < t.rows ? lane : 0));
        xs_at = a.x_scales + (int64_t)max(tok, 0) * a.ld_scales;
        int zero = 0;
        asm("" : "+v"(zero));  // (a vector load, counted in order with the others)
        ws_at = a.w_scales + ((int64_t)t.expert * (a.out >> 7) + strip) * np + zero;
    }
    uint4 xq[D][NX], wq[D][2][CB];
    [[maybe_unused]] float sx[D], sw[D];
    // Loads without branches (around one the compiler would wait for everything in flight): past the last piece, the last one again.
    auto load_x = [&](int s, int d) __attribute__((always_inline)) {
        const int at = min(s * KS + ks, np - 1);
#pragma unroll
        for (int q = 0; q < NX; ++q) xq[d][q] = ldb16(xrow[q] + (int64_t)at * kPieceBytes);
        if constexpr (F8) {
            sx[d] = xs_at[at];
            sw[d] = ws_at[at];
        }
    };
    auto load_w = [&](int s, int d) __attribute__((always_inline)) {
        const char *p = wbase + (int64_t)min(s * KS + ks, np - 1) * 16384;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < CB; ++b) wq[d][h][b] = ldw16<ONCE>(p + operand_at<F8>(h, b) + lane16);
    };
    auto put_x = [&](int d, int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < NX; ++q) *reinterpret_cast<uint4 *>(lds + slot * XBUF + xput[q]) = xq[d][q];
    };
    auto barrier = [&]() __attribute__((always_inline)) {
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    };
#pragma unroll
    for (int d = 0; d < D; ++d) {
        load_x(d, d);
        __builtin_amdgcn_sched_barrier(0);
        load_w(d, d);
        __builtin_amdgcn_sched_barrier(0);
    }
    for (int s0 = 0; s0 * KS < np; s0 += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int slot = d & 1;
            put_x(d, slot);
            [[maybe_unused]] int powers = kPowersOne;
            if constexpr (F8) {
                const WeightScale s = weight_scale(sw[d]);
                powers = s.powers;
                if (lane < R) sc[lane] = sx[d] * s.factor;
            }
            load_x(s0 + d + D, d);
            // what a slot held two pieces ago has been read by everyone: each came to the barrier of the piece between behind its reads
            barrier();
            if ((s0 + d) * KS + ks < np) {
                const char *xs = lds + slot * XBUF;
                uint4 xo[2][RB];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < RB; ++i)
                        xo[h][i] = *reinterpret_cast<const uint4 *>(xs + (16 * i + n) * kPieceBytes + (((4 * h + kq) ^ (n & 7)) << 4));
                if constexpr (F8) {
#pragma unroll
                    for (int i = 0; i < RB; ++i) {
                        const f32x4 f = *reinterpret_cast<const f32x4 *>(sc + 16 * i + 4 * kq);
#pragma unroll
                        for (int b = 0; b < CB; ++b)
                            acc[i][b] += f * mfma_e4m3(as_i32x8(xo[0][i], xo[1][i]), as_i32x8(wq[d][0][b], wq[d][1][b]), powers);
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < RB; ++i)
#pragma unroll
                            for (int b = 0; b < CB; ++b)
                                acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(xo[h][i]), as_bf16x8(wq[d][h][b]), acc[i][b], 0, 0, 0);
                }
            }
            load_w(s0 + d + D, d);
            in_order();  // (the scales' region is this wavefront's own)
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    if constexpr (KS == 2) {
        __syncthreads();  // everyone has left the slots
        f32x4(*const other)[64 * kMidWaves] = reinterpret_cast<f32x4(*)[64 * kMidWaves]>(all_lds);
        if (ks == 1)
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
                for (int b = 0; b < CB; ++b) other[i * CB + b][tid] = acc[i][b];
        __syncthreads();
        if (ks == 1) return;
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int b = 0; b < CB; ++b) acc[i][b] += other[i * CB + b][tid];
    }

    uint16_t *const y0 = a.y + (int64_t)t.row0 * a.ldy + strip * 128 + 64 * (b0 >> 2) + 4 * n + (b0 & 3);
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = 16 * i + 4 * kq + e;
            if (r >= t.rows || token_at(a, t.row0 + r) < 0) continue;
            uint32_t *const dst = reinterpret_cast<uint32_t *>(y0 + (int64_t)r * a.ldy);
            if constexpr (CB == 4)
                *reinterpret_cast<uint2 *>(dst) = uint2{pack_bf16_rne(acc[i][0][e], acc[i][1][e]), pack_bf16_rne(acc[i][2][e], acc[i][3][e])};
            else
                *dst = pack_bf16_rne(acc[i][0][e], acc[i][1][e]);
        }
}

template <bool F8, int RB, int CB, int D, int KS = 1, bool ONCE = false>
static hipError_t launch_mid(const ExpertsArgs &a, hipStream_t stream)
{
    const int64_t row_tiles = ((int64_t)a.n_rows + 16 * RB - 1) / (16 * RB) + met_experts(a.starts ? a.n_experts : 0, a.n_rows);
    const int64_t grid = (row_tiles * (a.out / (64 * CB)) + 7) / 8 * 8;
    if (!can_launch(grid, 64 * kMidWaves * KS)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_experts_mid<F8, RB, CB, D, KS, ONCE>), dim3((unsigned)grid), dim3(64 * kMidWaves * KS), 0, stream, a);
    return hipGetLastError();
}

// The kernel that a form names; every one that product_form gives is here.
template <bool F8>
static hipError_t launch_form(const ExpertsArgs &a, ProductForm f, hipStream_t stream)
{
    const int which = f.rb * 1000 + f.cb * 100 + f.groups * 10 + f.once;
    if (f.kind == ProductForm::kWide) return launch_wide<F8>(a, stream);
    if (f.kind == ProductForm::kMid) switch (which) {
        case 4410: return launch_mid<F8, 4, 4, 2, 1>(a, stream);
        case 4420: return launch_mid<F8, 4, 4, 2, 2>(a, stream);
        case 4210: return launch_mid<F8, 4, 2, 2, 1>(a, stream);
        case 4220: return launch_mid<F8, 4, 2, 2, 2>(a, stream);
        case 4211: return launch_mid<F8, 4, 2, 2, 1, true>(a, stream);
        case 4221: return launch_mid<F8, 4, 2, 2, 2, true>(a, stream);
        case 2210: return launch_mid<F8, 2, 2, 2, 1>(a, stream);
        case 2220: return launch_mid<F8, 2, 2, 2, 2>(a, stream);
        case 2211: return launch_mid<F8, 2, 2, 2, 1, true>(a, stream);
        case 2221: return launch_mid<F8, 2, 2, 2, 2, true>(a, stream);
        }
    else switch (which) {
        case 2440: return launch_thin<F8, 2, 4, 2, 4>(a, stream);
        case 2441: return launch_thin<F8, 2, 4, 2, 4, true>(a, stream);
        case 1440: return launch_thin<F8, 1, 4, 2, 4>(a, stream);
        case 1441: return launch_thin<F8, 1, 4, 2, 4, true>(a, stream);
        case 1280: return launch_thin<F8, 1, 2, 2, 8>(a, stream);
        case 1180: return launch_thin<F8, 1, 1, 2, 8>(a, stream);
        }
    return hipErrorInvalidValue;
}

hipError_t launch_experts_linear(ExpertsArgs a, bool bits8, hipStream_t stream)
{
    const int met = met_experts(a.starts ? a.n_experts : 0, a.n_rows);
    a.large = large_weights(met, a.out, a.pieces);
    const ProductForm f = product_form(bits8, a.n_rows, met, a.out, a.pieces);
    return bits8 ? launch_form<true>(a, f, stream) : launch_form<false>(a, f, stream);
}

// ------------------------------------------------------------------------------------------------
// Weights into operand order: a thread per 16 bytes of the destination.
// ------------------------------------------------------------------------------------------------
template <bool F8>
__global__ __launch_bounds__(256) void k_experts_pack(const char *__restrict__ w, int64_t pieces_of_16, int row_bytes, int used_bytes,
                                                      int pieces, char *__restrict__ dst)
{
    for (int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x; d < pieces_of_16; d += (int64_t)gridDim.x * 256) {
        const int slot = (int)(d & 63), at_b = (int)(d >> 6) & 15;
        const int b = F8 ? (at_b & 3) + 4 * (at_b >> 3) : at_b & 7, h = F8 ? (at_b >> 2) & 1 : at_b >> 3;  // operand_at
        const int64_t rest = d >> 10;  // (expert * strips + strip) * pieces + piece
        const int64_t es = rest / pieces;
        const int64_t col = 128 * es + 64 * (b >> 2) + 4 * (slot & 15) + (b & 3);  // (strips of all experts are consecutive columns)
        const int at = (int)(rest - es * pieces) * kPieceBytes + 64 * h + 16 * (slot >> 4);
        uint4 v = {0u, 0u, 0u, 0u};
        if (at < used_bytes) v = ldb16(w + col * row_bytes + at);  // (used_bytes is a multiple of 64)
        *reinterpret_cast<uint4 *>(dst + d * 16) = v;
    }
}

hipError_t launch_experts_pack(const char *w, int64_t n_experts, int row_bytes, int used_bytes, int out, bool bits8, char *dst, hipStream_t stream)
{
    const int pieces = row_bytes / kPieceBytes;
    const int64_t n = n_experts * out * pieces * (kPieceBytes / 16);
    const int64_t grid = (n + 255) / 256;
    hipLaunchKernelGGL(bits8 ? k_experts_pack<true> : k_experts_pack<false>, dim3((unsigned)(grid < (1 << 20) ? grid : (1 << 20))), dim3(256), 0, stream, w, n,
                       row_bytes, used_bytes, pieces, dst);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// Rows to 8 bits: 16 lanes have the 128 values of a block, 8 each.  The largest magnitude is found on the bits (bf16 without its sign is ordered
// like its value, infinity above all numbers and NaN above that).
//   q = nearest8(x 448 / d):  with d = m 2^e, 1 <= m < 2, the quotient is (x 448 2^-e) / m: the first factor exact, the division by a
//   reciprocal and one correction, which gives the quotient itself where it has 24 bits or fewer.  A tie of E4M3 does; and where the quotient
//   (11 bits over 8) is no tie it is 2^-13 of itself away from one, far more than what the correction leaves.
// What bounds it is memory: 19675 rows of 4096 43.7 us, 244 MB at 5.6 TB/s; a thread has parts of two blocks so that two requests are under way.
// ------------------------------------------------------------------------------------------------
static __device__ __forceinline__ float value_lo(uint32_t u) { return __uint_as_float(u << 16); }
static __device__ __forceinline__ float value_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }

__global__ __launch_bounds__(256) void k_rows_quantize(const uint16_t *__restrict__ x, int64_t ldx, unsigned total, int in, unsigned blocks,
                                                       uint8_t *__restrict__ q, int64_t ldq, float *__restrict__ scales, int64_t ld_scales)
{
    const int l = threadIdx.x & 15;
    const unsigned at0 = blockIdx.x * (16 * kQuantizeBlocks) + (threadIdx.x >> 4);
    uint4 v[kQuantizeBlocks];
    unsigned row[kQuantizeBlocks], blk[kQuantizeBlocks];
#pragma unroll
    for (int j = 0; j < kQuantizeBlocks; ++j) {
        const unsigned at = min(at0 + 16 * j, total - 1);
        row[j] = at / blocks;
        blk[j] = at - row[j] * blocks;
        const int k = (int)blk[j] * kScaleBlock + 8 * l;
        v[j] = ld16_stream(x + (int64_t)row[j] * ldx + (k < in ? k : 0));
        if (k >= in) v[j] = uint4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int j = 0; j < kQuantizeBlocks; ++j) {
        if (at0 + 16 * j >= total) return;
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
        const float largest = __uint_as_float(top << 16);
        uint32_t o[2] = {0u, 0u};
        float scale = largest;
        if (top < 0x7F80u) {
            const float d = fmaxf(largest, 448.f * 0x1p-126f);
            scale = d / 448.f;
            const uint32_t bits = __float_as_uint(d), e = bits >> 23;  // d = m 2^(e - 127), e >= 9
            const float m = __uint_as_float((bits & 0x007FFFFFu) | 0x3F800000u);
            const float f = 1.75f * __uint_as_float((262u - e) << 23);  // 448 2^(127 - e)
            const float r = __builtin_amdgcn_rcpf(m);
            float c[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float n0 = value_lo(w[i]) * f, n1 = value_hi(w[i]) * f;
                const float t0 = n0 * r, t1 = n1 * r;
                c[2 * i] = fmaf(fmaf(-t0, m, n0), r, t0);
                c[2 * i + 1] = fmaf(fmaf(-t1, m, n1), r, t1);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i], c[4 * i + 1], 0, false);
                o[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i + 2], c[4 * i + 3], p, true);
            }
        } else {
            // an infinity, or a NaN: no scale has a meaning, and the values say so
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t mag = (w[i >> 1] >> (16 * (i & 1))) & 0x7FFFu;
                o[i >> 2] |= (top > 0x7F80u || mag >= 0x7F80u ? 0x7Fu : 0u) << (8 * (i & 3));
            }
        }
        *reinterpret_cast<uint2 *>(q + (int64_t)row[j] * ldq + (int)blk[j] * kScaleBlock + 8 * l) = uint2{o[0], o[1]};
        if (l == 0) scales[(int64_t)row[j] * ld_scales + blk[j]] = scale;
    }
}

hipError_t launch_rows_quantize(const uint16_t *x, int64_t ldx, int64_t rows, int in, uint8_t *q, int64_t ldq, float *scales,
                                int64_t ld_scales, hipStream_t stream)
{
    const int blocks = (in + kScaleBlock - 1) / kScaleBlock;
    const int64_t most = quantize_rows_at_once(blocks);
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t total = (rows - r < most ? rows - r : most) * blocks;
        hipLaunchKernelGGL(k_rows_quantize, dim3((unsigned)((total + 16 * kQuantizeBlocks - 1) / (16 * kQuantizeBlocks))), dim3(256), 0, stream,
                           x + r * ldx, ldx, (unsigned)total, in, (unsigned)blocks, q + r * ldq, ldq, scales + r * ld_scales, ld_scales);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ------------------------------------------------------------------------------------------------
// Picks by expert: a counting sort that keeps the picks' order.  The picks are cut into chunks, one work group each, a chunk into 16 runs, one
// wavefront each.  A wavefront counts 64 picks at a time: lanes with the same expert find each other by ballots over the id's bits, and
// their first lane adds their number to the wavefront's own count of that expert.  The first place of (expert, chunk, wavefront) is then a sum
// over the experts before, the chunks before and the wavefronts before; a second walk over the picks hands the places out.  No atomics whose order shows.
// Up to kGroupAlone chunks of a pick a thread are one launch, each of whose work groups counts all picks by itself, by atomic adds in LDS; else a launch counts and
// a second one, each of whose work groups adds up all chunks' counts, hands out.  A wavefront's S x 64 picks stay in registers between its two walks; S = 0 (beyond 2 M picks) reads them twice.
// What bounds it is the way through memory and LDS, not bytes: device time 3.5 us for 512 picks, 13 for 157400
// (counts 4.2, places 8.8; the chunks' counts all requested at once, 32 a thread: 10).  Up to 8192 picks by one work group instead of up to eight: 4148 of 72
// experts 9.0 / 6.2 us a call, 8192 of 256 14.2 / 7.7, all of one 7.3 / 6.6, mostly of one of 8 9.4 / 9.5.
// ------------------------------------------------------------------------------------------------
constexpr int kGroupWaves = 16;

// lanes with the same id
static __device__ __forceinline__ uint64_t same_id(int id, int bits)
{
    uint64_t m = ~0ull;
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((id >> b) & 1);
        m &= (id >> b) & 1 ? set : ~set;
    }
    return m;
}

// the id of a pick, n_experts for one without an expert and behind the end
static __device__ __forceinline__ int id_at(const int32_t *__restrict__ ids, int64_t ld_ids, int picks, int64_t i, int64_t end, int n_experts)
{
    if (i >= end) return n_experts;
    const int64_t t = (int64_t)((uint32_t)i / (uint32_t)picks);
    const int id = ids[t * ld_ids + (i - t * picks)];
    return (unsigned)id < (unsigned)n_experts ? id : n_experts;
}

// 64 picks of a wavefront's run
struct Picks {
    int id;       // this lane's
    int before;   // lanes below with the same one
    int all;      // .. and of all lanes, in the first of them; else 0
};

static __device__ __forceinline__ Picks match(int id, int n_experts, int bits, int lane)
{
    const uint64_t m = same_id(id, bits);
    const int before = (int)__popcll(m & ((1ull << lane) - 1));
    return Picks{id, before, before == 0 && id < n_experts ? (int)__popcll(m) : 0};
}

// counts of the wavefront's run from pick `from` on into cnt[n_experts] (LDS, zero)
template <int S>
static __device__ __forceinline__ void count_run(const int32_t *__restrict__ ids, int64_t ld_ids, int picks, int64_t from, int64_t end, int n_experts,
                                                 int bits, int lane, int *cnt, Picks (&p)[S ? S : 1])
{
    if constexpr (S > 0) {
#pragma unroll
        for (int s = 0; s < S; ++s) p[s].id = id_at(ids, ld_ids, picks, from + 64 * s + lane, end, n_experts);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            p[s] = match(p[s].id, n_experts, bits, lane);
            if (p[s].all) cnt[p[s].id] += p[s].all;
            in_order();
        }
    } else
        for (int64_t i = from; i < end; i += 64) {
            const Picks q = match(id_at(ids, ld_ids, picks, i + lane, end, n_experts), n_experts, bits, lane);
            if (q.all) cnt[q.id] += q.all;
            in_order();
        }
}

template <int S>
__global__ __launch_bounds__(64 * kGroupWaves) void k_experts_count(const int32_t *__restrict__ ids, int64_t ld_ids, int picks, int64_t n,
                                                                    int64_t chunk, int n_experts, int bits, int32_t *__restrict__ counts)
{
    extern __shared__ int cnt[];  // [kGroupWaves][n_experts]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t run = chunk / kGroupWaves, from = blockIdx.x * chunk + wave * run, end = min(from + run, n);
    for (int e = lane; e < n_experts; e += 64) cnt[wave * n_experts + e] = 0;
    in_order();
    Picks p[S ? S : 1];
    count_run<S>(ids, ld_ids, picks, from, end, n_experts, bits, lane, cnt + wave * n_experts, p);
    __syncthreads();
    for (int e = tid; e < n_experts; e += 64 * kGroupWaves) {
        int s = 0;
#pragma unroll
        for (int w = 0; w < kGroupWaves; ++w) s += cnt[w * n_experts + e];
        counts[(int64_t)blockIdx.x * n_experts + e] = s;
    }
}

template <int S>
__global__ __launch_bounds__(64 * kGroupWaves) void k_experts_place(const int32_t *__restrict__ ids, int64_t ld_ids, int picks, int64_t n,
                                                                    int64_t chunk, int n_experts, int bits,
                                                                    const int32_t *__restrict__ counts, int n_chunks,
                                                                    int32_t *__restrict__ starts, int32_t *__restrict__ order,
                                                                    int32_t *__restrict__ place)
{
    extern __shared__ int cnt[];  // [kGroupWaves][n_experts], the prefix sum's sums of wavefronts, then two sums of every thread
    int *const sums = cnt + kGroupWaves * n_experts, *const some_all = sums + kGroupWaves, *const some_before = some_all + 64 * kGroupWaves;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t run = chunk / kGroupWaves, from = blockIdx.x * chunk + wave * run, end = min(from + run, n);
    for (int e = lane; e < n_experts; e += 64) cnt[wave * n_experts + e] = 0;
    in_order();
    // the chunks' counts: as many threads an expert as there are
    const int share = 64 * kGroupWaves / n_experts;
    const bool several = S == 1 && gridDim.x > 1;  // and none were taken: a chunk is a pick of every thread, and every work group looks at all
    if (several) {
        some_all[tid] = 0;
        some_before[tid] = 0;
        int id[kGroupAlone];
#pragma unroll
        for (int c = 0; c < kGroupAlone; ++c) id[c] = id_at(ids, ld_ids, picks, (int64_t)c * kGroupUnit + tid, n, n_experts);
        __syncthreads();
#pragma unroll
        for (int c = 0; c < kGroupAlone; ++c) {
            // the picks of the first lane's expert at once, as adds to one address wait for each other
            const int e = id[c], first = __builtin_amdgcn_readfirstlane(e), of_first = (int)__popcll(__ballot(e == first));
            const int m = lane == 0 ? of_first : 1;
            if (e < n_experts && (lane == 0 || e != first)) {
                atomicAdd(&some_all[e], m);  // (sums of whole numbers: their order does not show)
                if (c < (int)blockIdx.x) atomicAdd(&some_before[e], m);
            }
        }
    } else if (counts) {
        int all = 0, before = 0;
        const int e = tid % n_experts, q = tid / n_experts;
        if (q < share)
#pragma unroll 8
            for (int c = q; c < n_chunks; c += share) {
                const int v = counts[(int64_t)c * n_experts + e];
                before += c < (int)blockIdx.x ? v : 0;
                all += v;
            }
        some_all[tid] = all;
        some_before[tid] = before;
    }
    Picks p[S ? S : 1];
    count_run<S>(ids, ld_ids, picks, from, end, n_experts, bits, lane, cnt + wave * n_experts, p);
    __syncthreads();
    // thread e: expert e (at most 512 of them)
    int total = 0, before = 0;
    if (tid < n_experts) {
        if (several) {
            total = some_all[tid];
            before = some_before[tid];
        } else if (counts)
            for (int q = 0; q < share; ++q) {
                total += some_all[q * n_experts + tid];
                before += some_before[q * n_experts + tid];
            }
        else
#pragma unroll
            for (int w = 0; w < kGroupWaves; ++w) total += cnt[w * n_experts + tid];
    }
    const int incl = wave_scan(total, lane);
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int first = incl - total, all = 0;
#pragma unroll
    for (int w = 0; w < kGroupWaves; ++w) {
        first += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    if (tid < n_experts) {
        if (blockIdx.x == 0) {
            starts[tid] = first;
            if (tid == n_experts - 1) starts[n_experts] = all;
        }
        int at = first + before;
#pragma unroll
        for (int w = 0; w < kGroupWaves; ++w) {
            const int v = cnt[w * n_experts + tid];
            cnt[w * n_experts + tid] = at;
            at += v;
        }
    }
    // the places behind the last expert's
    for (int64_t i = max((int64_t)all, blockIdx.x * chunk) + tid; i < min((blockIdx.x + 1) * chunk, n); i += 64 * kGroupWaves) order[i] = -1;
    __syncthreads();
    int *const next = cnt + wave * n_experts;
    auto hand_out = [&](const Picks &q, int64_t i) __attribute__((always_inline)) {
        int at = -1;
        if (q.id < n_experts) at = next[q.id] + q.before;
        in_order();  // all have read before the first lanes add
        if (q.all) next[q.id] = at + q.all;
        in_order();
        if (i < end) {
            place[i] = at;
            if (at >= 0 && at < n) order[at] = (int)i;  // (beyond, were the ids changed between the two walks)
        }
    };
    if constexpr (S > 0) {
#pragma unroll
        for (int s = 0; s < S; ++s) hand_out(p[s], from + 64 * s + lane);
    } else
        for (int64_t i = from; i < end; i += 64)
            hand_out(match(id_at(ids, ld_ids, picks, i + lane, end, n_experts), n_experts, bits, lane), i + lane);
}

template <int S>
static hipError_t launch_group(const int32_t *ids, int64_t ld_ids, int64_t n, int64_t chunk, int picks, int n_experts, int32_t *starts,
                               int32_t *order, int32_t *place, int32_t *workspace, hipStream_t stream)
{
    const int chunks = n ? (int)((n + chunk - 1) / chunk) : 1;
    int bits = 0;
    while ((n_experts >> bits) != 0) ++bits;  // of the ids and of n_experts, which stands for none
    const size_t lds = (size_t)kGroupWaves * n_experts * 4;
    if constexpr (S != 1)
        hipLaunchKernelGGL(k_experts_count<S>, dim3((unsigned)chunks), dim3(64 * kGroupWaves), lds, stream, ids, ld_ids, picks, n, chunk, n_experts, bits,
                           workspace);
    hipLaunchKernelGGL(k_experts_place<S>, dim3((unsigned)chunks), dim3(64 * kGroupWaves), lds + (kGroupWaves + (chunks > 1 ? 2 * 64 * kGroupWaves : 0)) * 4,
                       stream, ids, ld_ids, picks, n, chunk, n_experts, bits, S != 1 ? workspace : nullptr, chunks, starts, order, place);
    return hipGetLastError();
}

hipError_t launch_experts_group(const int32_t *ids, int64_t ld_ids, int64_t tokens, int picks, int n_experts, int32_t *starts,
                                int32_t *order, int32_t *place, int32_t *workspace, hipStream_t stream)
{
    const int64_t n = tokens * picks, chunk = group_chunk(n);
    auto go = [&](auto s) { return launch_group<decltype(s)::value>(ids, ld_ids, n, chunk, picks, n_experts, starts, order, place, workspace, stream); };
    switch (chunk / (64 * kGroupWaves)) {
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 4: return go(std::integral_constant<int, 4>{});
    case 8: return go(std::integral_constant<int, 8>{});
    default: return go(std::integral_constant<int, 0>{});
    }
}

// ------------------------------------------------------------------------------------------------
// The weighted sum of a token's rows: a thread has 8 columns of one token, and requests PB of its rows before it adds the first.  Rows are read once
// and past the caches; a pick without one reads the first row, which lies in the caches, and counts nothing.  What bounds it is memory: 19675 tokens'
// 8 picks of 4096 columns, a quarter of them elsewhere, 185 us, 1.13 GB at 6.1 TB/s.
// ------------------------------------------------------------------------------------------------
template <int PB>
__global__ __launch_bounds__(256) void k_experts_combine(const uint16_t *__restrict__ y, int64_t ldy, int n_rows, const int32_t *__restrict__ place,
                                                         const float *__restrict__ weights, unsigned pieces, int picks, unsigned eighths,
                                                         uint16_t *__restrict__ z, int64_t ldz)
{
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const unsigned t = i / eighths, c = (i - t * eighths) * 8;
    const int32_t *const at = place + (int64_t)t * picks;
    const float *const of = weights + (int64_t)t * picks;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < picks; j += PB) {
        uint4 v[PB];
        float w[PB];
        bool there[PB];
#pragma unroll
        for (int q = 0; q < PB; ++q) {
            const int p = at[j + q];
            there[q] = (unsigned)p < (unsigned)n_rows;
            w[q] = of[j + q];
            v[q] = ld16_stream(y + (int64_t)(there[q] ? p : 0) * ldy + c);
        }
#pragma unroll
        for (int q = 0; q < PB; ++q) {
            const uint32_t u[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float lo = fmaf(w[q], value_lo(u[k]), s[2 * k]), hi = fmaf(w[q], value_hi(u[k]), s[2 * k + 1]);
                s[2 * k] = there[q] ? lo : s[2 * k];
                s[2 * k + 1] = there[q] ? hi : s[2 * k + 1];
            }
        }
    }
    st16_stream(z + (int64_t)t * ldz + c, uint4{pack_bf16_rne(s[0], s[1]), pack_bf16_rne(s[2], s[3]), pack_bf16_rne(s[4], s[5]), pack_bf16_rne(s[6], s[7])});
}

hipError_t launch_experts_combine(const uint16_t *y, int64_t ldy, int n_rows, const int32_t *place, const float *weights, int64_t tokens, int picks,
                                  int out, uint16_t *z, int64_t ldz, hipStream_t stream)
{
    const int64_t most = ((int64_t)1 << 31) / (out / 8);  // tokens of a launch, whose pieces are counted in 32 bits
    for (int64_t t = 0; t < tokens; t += most) {
        const int64_t pieces = (tokens - t < most ? tokens - t : most) * (out / 8);
        auto go = [&](auto pb) {
            hipLaunchKernelGGL(k_experts_combine<decltype(pb)::value>, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, stream, y, ldy, n_rows,
                               place + t * picks, weights + t * picks, (unsigned)pieces, n_rows > 0 ? picks : 0, (unsigned)(out / 8), z + t * ldz, ldz);
        };
        if (picks % 4 == 0)
            go(std::integral_constant<int, 4>{});
        else if (picks % 2 == 0)
            go(std::integral_constant<int, 2>{});
        else
            go(std::integral_constant<int, 1>{});
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace lora
