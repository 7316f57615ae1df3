// gfx950 kernels of the frozen layers beside an adapter (include/lora_experts.h): rows to 8 bits, products in block-scaled 8 bits and in
// bf16 over rows grouped by expert, the grouping itself, and the weighted sum behind it.
//
// Both element types walk k in pieces of 128 bytes: 64 bf16 or 128 8-bit values.  A weight tile of 16 columns x one piece is, for either type,
// two operands of 16 bytes a lane (halves of the piece): two 16x16x32 bf16 MFMAs, or one 16x16x128 f8f6f4 MFMA that takes both.  So
// the weights are packed alike:
//   expert e, 128-column strip, piece P, half h, sub-block b, lane slot (kq, n): 16 bytes
//     128 P + 64 h + 16 kq .. of column 128 strip + 64 (b / 4) + 4 n + b mod 4
//   at  e * out * 128 pieces + ((strip * pieces + P) * 2 + h) * 8192 + b * 1024 + (16 kq + n) * 16
// A wavefront's load of an operand is 1 KB of consecutive bytes, and of four sub-blocks lane n ends up with four consecutive columns.
// The token operand uses the same mapping of lanes to k.
#include "lora_device.h"
#include "lora_experts.h"

#include <type_traits>

namespace lora {

typedef __attribute__((ext_vector_type(8))) int i32x8;

static __device__ __forceinline__ uint4 ldb16(const char *p) { return *reinterpret_cast<const uint4 *>(p); }

static __device__ __forceinline__ i32x8 as_i32x8(uint4 lo, uint4 hi)
{
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

// LDS operations of a wavefront complete in order; the compiler keeps them so
static __device__ __forceinline__ void in_order()
{
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// 16 x 16 products over 128 8-bit values of k (both operands E4M3, the instruction's own scales at 1)
static __device__ __forceinline__ f32x4 mfma_e4m3(i32x8 a, i32x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
}

// ------------------------------------------------------------------------------------------------
// Which expert, rows and columns a work group's tile has.  The tiles of a launch are numbered expert by expert, inside it column tile by column tile,
// inside that row tile by row tile, so that a run of them shares its weights; how many there are follows from `starts` on the device
// alone, and every wavefront finds its tile by itself (a prefix sum over the experts' row tiles, 64 experts at a time).
// ------------------------------------------------------------------------------------------------
struct Tile {
    int expert, ct;
    int row0, rows;  // first place, places
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

// tile `at(total)` of all; false if there is none
template <int R, class At>
static __device__ __forceinline__ bool find_tile(const int32_t *__restrict__ starts, int n_experts, int n_rows, int n_ct, int lane, At at,
                                                 Tile &t)
{
    if (!starts) {
        const int mt = (n_rows + R - 1) / R, idx = at(mt * n_ct);
        if (idx < 0) return false;
        t.expert = 0;
        t.ct = idx / mt;
        t.row0 = (idx - t.ct * mt) * R;
        t.rows = min(R, n_rows - t.row0);
        return true;
    }
    int mine = 0, first;
    for (int e = lane; e < n_experts; e += 64) mine += (expert_rows(starts, e, n_rows, first) + R - 1) / R;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d, 64);
    const int idx = at(__builtin_amdgcn_readfirstlane(mine) * n_ct);
    if (idx < 0) return false;
    const int q = idx / n_ct;  // row tile, expert by expert: which expert's
    int before = 0;
    for (int base = 0; base < n_experts; base += 64) {
        const int e = base + lane;
        const int rows = e < n_experts ? expert_rows(starts, e, n_rows, first) : 0;
        const int mt = (rows + R - 1) / R, upto = before + wave_scan(mt, lane);
        const uint64_t hit = __ballot(q < upto);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            const int e_mt = __shfl(mt, l, 64), e_first = __shfl(first, l, 64), e_rows = __shfl(rows, l, 64);
            const int in_e = idx - (__shfl(upto, l, 64) - e_mt) * n_ct;
            const int ct = in_e / e_mt, row = (in_e - ct * e_mt) * R;
            t.expert = __builtin_amdgcn_readfirstlane(base + l);
            t.ct = __builtin_amdgcn_readfirstlane(ct);
            t.row0 = __builtin_amdgcn_readfirstlane(e_first + row);
            t.rows = __builtin_amdgcn_readfirstlane(min(R, e_rows - row));
            return true;
        }
        before = __shfl(upto, 63, 64);
    }
    return false;
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
// meet in LDS in wavefront order.
// ------------------------------------------------------------------------------------------------
template <bool F8, int RB, int WAVES>
constexpr int kThinSlab = WAVES * (16 * RB * 128 + (F8 ? 16 * RB * 4 : 0));
template <bool F8, int RB, int CB, int WAVES>
constexpr int kThinLds = kThinSlab<F8, RB, WAVES> > WAVES * RB * CB * 1024 ? kThinSlab<F8, RB, WAVES> : WAVES *RB *CB * 1024;

template <bool F8, int RB, int CB, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 1) void k_experts_thin(ExpertsArgs a)
{
    constexpr int NX = 2 * RB;                        // x loads of a wavefront per piece: 8 rows each
    constexpr int kSlab = 16 * RB * 128;              // bytes of a wavefront's x region
    constexpr int kRegion = kSlab + (F8 ? 64 * RB : 0);  // .. and the rows' scales
    constexpr int kTiles = RB * CB, R = 16 * RB;
    static_assert(RB <= 4, "a lane for the scale of every row");
    __shared__ __attribute__((aligned(16))) char lds[kThinLds<F8, RB, CB, WAVES>];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, kq = lane >> 4;
    Tile t;
    // work group b runs on XCD b mod 8: every XCD an eighth of the tiles, in one run
    if (!find_tile<R>(a.starts, a.n_experts, a.n_rows, a.out / (16 * CB), lane, [&](int total) {
            const int per_xcd = (total + 7) >> 3, idx = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
            return (int)(blockIdx.x >> 3) >= per_xcd || idx >= total ? -1 : idx;
        }, t))
        return;
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
        const char *wbase = a.w + ((int64_t)t.expert * (a.out >> 7) + strip) * np * 16384 + (int64_t)wave * 16384 + b0 * 1024 + lane * 16;
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
                for (int b = 0; b < CB; ++b) wq[d][h][b] = ldb16(wbase + at * (16384 * WAVES) + h * 8192 + b * 1024);
        };
        auto stage = [&](int d) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < NX; ++q) *reinterpret_cast<uint4 *>(slab + (8 * q + lr) * 128 + ((lc ^ lr) << 4)) = xq[d][q];
            if constexpr (F8)
                if (lane < R) reinterpret_cast<float *>(slab + kSlab)[lane] = sx[d] * sw[d];
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
                        acc[i][b] += s * mfma_e4m3(as_i32x8(xo[0][i], xo[1][i]), as_i32x8(wq[d][0][b], wq[d][1][b]), f32x4{0.f, 0.f, 0.f, 0.f});
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
        uint32_t *dst = reinterpret_cast<uint32_t *>(a.y + (int64_t)(t.row0 + r) * a.ldy + strip * 128 + (b0 >> 2) * 64 + 4 * (l & 15) + (b0 & 3));
        if constexpr (CB == 4)
            *reinterpret_cast<uint2 *>(dst) = uint2{pack_bf16_rne(f[0], f[1]), pack_bf16_rne(f[2], f[3])};
        else
#pragma unroll
            for (int b = 0; b < CB; b += 2) dst[b >> 1] = pack_bf16_rne(f[b], f[b + 1]);
    }
}

template <bool F8, int RB, int CB, int D, int WAVES>
static hipError_t launch_thin(const ExpertsArgs &a, hipStream_t stream)
{
    const int64_t row_tiles = (int64_t)(a.n_rows + 16 * RB - 1) / (16 * RB) + (a.starts ? (a.n_rows < a.n_experts ? a.n_rows : a.n_experts) : 0);
    const int64_t grid = (row_tiles * (a.out / (16 * CB)) + 7) / 8 * 8;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_experts_thin<F8, RB, CB, D, WAVES>), dim3((unsigned)grid), dim3(64 * WAVES), 0, stream, a);
    return hipGetLastError();
}

template <bool F8>
static hipError_t launch_by_rows(const ExpertsArgs &a, hipStream_t stream)
{
    const int per = a.n_rows / a.n_experts;
    if (per <= 16) return launch_thin<F8, 1, 4, 2, 8>(a, stream);
    if (per <= 32) return launch_thin<F8, 2, 4, 2, 8>(a, stream);
    return launch_thin<F8, 4, 4, 2, 8>(a, stream);
}

hipError_t launch_experts_linear(const ExpertsArgs &a, bool bits8, hipStream_t stream)
{
    return bits8 ? launch_by_rows<true>(a, stream) : launch_by_rows<false>(a, stream);
}

// ------------------------------------------------------------------------------------------------
// Weights into operand order: a thread per 16 bytes of the destination.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_experts_pack(const char *__restrict__ w, int64_t pieces_of_16, int row_bytes, int used_bytes,
                                                      int pieces, char *__restrict__ dst)
{
    for (int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x; d < pieces_of_16; d += (int64_t)gridDim.x * 256) {
        const int slot = (int)(d & 63), b = (int)(d >> 6) & 7, h = (int)(d >> 9) & 1;
        const int64_t rest = d >> 10;  // (expert * strips + strip) * pieces + piece
        const int64_t es = rest / pieces;
        const int64_t col = 128 * es + 64 * (b >> 2) + 4 * (slot & 15) + (b & 3);  // (strips of all experts are consecutive columns)
        const int at = (int)(rest - es * pieces) * kPieceBytes + 64 * h + 16 * (slot >> 4);
        uint4 v = {0u, 0u, 0u, 0u};
        if (at < used_bytes) v = ldb16(w + col * row_bytes + at);  // (used_bytes is a multiple of 64)
        *reinterpret_cast<uint4 *>(dst + d * 16) = v;
    }
}

hipError_t launch_experts_pack(const char *w, int64_t n_experts, int row_bytes, int used_bytes, int out, char *dst, hipStream_t stream)
{
    const int pieces = row_bytes / kPieceBytes;
    const int64_t n = n_experts * out * pieces * (kPieceBytes / 16);
    const int64_t grid = (n + 255) / 256;
    hipLaunchKernelGGL(k_experts_pack, dim3((unsigned)(grid < (1 << 20) ? grid : (1 << 20))), dim3(256), 0, stream, w, n, row_bytes, used_bytes, pieces, dst);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// Rows to 8 bits: 16 lanes have the 128 values of a block, 8 each.  The largest magnitude is found on the bits (bf16 without its sign is ordered
// like its value, infinity above all numbers and NaN above that).
//   q = nearest8(x 448 / d):  with d = m 2^e, 1 <= m < 2, the quotient is (x 448 2^-e) / m: the first factor exact, the division by a
//   reciprocal and one correction, which gives the quotient itself where it has 24 bits or fewer.  A tie of E4M3 does; and where the quotient
//   (11 bits over 8) is no tie it is 2^-13 of itself away from one, far more than what the correction leaves.
// ------------------------------------------------------------------------------------------------
static __device__ __forceinline__ float value_lo(uint32_t u) { return __uint_as_float(u << 16); }
static __device__ __forceinline__ float value_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }

__global__ __launch_bounds__(256) void k_rows_quantize(const uint16_t *__restrict__ x, int64_t ldx, int64_t rows, int in, int blocks,
                                                       uint8_t *__restrict__ q, int64_t ldq, float *__restrict__ scales, int64_t ld_scales)
{
    const int64_t at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);  // block of 128
    if (at >= rows * blocks) return;
    const int l = threadIdx.x & 15;
    const int64_t row = at / blocks;
    const int blk = (int)(at - row * blocks), k = blk * kScaleBlock + 8 * l;
    uint4 v = {0u, 0u, 0u, 0u};
    if (k < in) v = ld16(x + row * ldx + k);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
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
        const uint32_t bits = __float_as_uint(d), e = bits >> 23;       // d = m 2^(e - 127), e >= 9
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
            int p = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i], c[4 * i + 1], 0, false);
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
    *reinterpret_cast<uint2 *>(q + row * ldq + k) = uint2{o[0], o[1]};
    if (l == 0) scales[row * ld_scales + blk] = scale;
}

hipError_t launch_rows_quantize(const uint16_t *x, int64_t ldx, int64_t rows, int in, uint8_t *q, int64_t ldq, float *scales,
                                int64_t ld_scales, hipStream_t stream)
{
    const int blocks = (in + kScaleBlock - 1) / kScaleBlock;
    const int64_t grid = (rows * blocks + 15) / 16;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_rows_quantize, dim3((unsigned)grid), dim3(256), 0, stream, x, ldx, rows, in, blocks, q, ldq, scales, ld_scales);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// Picks by expert: a counting sort that keeps the picks' order.  The picks are cut into chunks, one work group each, a chunk into 16 runs, one
// wavefront each.  A wavefront counts 64 picks at a time: lanes with the same expert find each other by ballots over the id's bits, and
// their first lane adds their number to the wavefront's own count of that expert.  The first place of (expert, chunk, wavefront) is then a sum
// over the experts before, the chunks before and the wavefronts before; a second walk over the picks hands the places out.  No atomics.
// ------------------------------------------------------------------------------------------------
constexpr int kGroupWaves = 16;

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

// counts of the wavefront's run [from, to) into cnt[n_experts] (LDS, zeroed here)
static __device__ __forceinline__ void count_run(const int32_t *__restrict__ ids, int64_t ld_ids, int picks, int64_t from, int64_t to,
                                                 int n_experts, int bits, int lane, int *cnt)
{
    for (int e = lane; e < n_experts; e += 64) cnt[e] = 0;
    in_order();
    for (int64_t i = from; i < to; i += 64) {
        const int id = id_at(ids, ld_ids, picks, i + lane, to, n_experts);
        const uint64_t m = same_id(id, bits);
        if (id < n_experts && (m & ((1ull << lane) - 1)) == 0) cnt[id] += __popcll(m);
        in_order();
    }
}

__global__ __launch_bounds__(64 * kGroupWaves) void k_experts_count(const int32_t *__restrict__ ids, int64_t ld_ids, int picks, int64_t n,
                                                                    int64_t chunk, int n_experts, int bits, int32_t *__restrict__ counts)
{
    extern __shared__ int cnt[];  // [kGroupWaves][n_experts]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t run = chunk / kGroupWaves, from = blockIdx.x * chunk + wave * run, end = min(from + run, n);
    count_run(ids, ld_ids, picks, from, end, n_experts, bits, lane, cnt + wave * n_experts);
    __syncthreads();
    for (int e = tid; e < n_experts; e += 64 * kGroupWaves) {
        int s = 0;
#pragma unroll
        for (int w = 0; w < kGroupWaves; ++w) s += cnt[w * n_experts + e];
        counts[(int64_t)blockIdx.x * n_experts + e] = s;
    }
}

__global__ __launch_bounds__(64 * kGroupWaves) void k_experts_place(const int32_t *__restrict__ ids, int64_t ld_ids, int picks, int64_t n,
                                                                    int64_t chunk, int n_experts, int bits,
                                                                    const int32_t *__restrict__ counts, int n_chunks,
                                                                    int32_t *__restrict__ starts, int32_t *__restrict__ order,
                                                                    int32_t *__restrict__ place)
{
    extern __shared__ int cnt[];  // [kGroupWaves][n_experts], then the sums of the wavefronts of the prefix sum
    int *const sums = cnt + kGroupWaves * n_experts;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t run = chunk / kGroupWaves, from = blockIdx.x * chunk + wave * run, end = min(from + run, n);
    count_run(ids, ld_ids, picks, from, end, n_experts, bits, lane, cnt + wave * n_experts);
    __syncthreads();
    // thread e: expert e (at most 1024 of them)
    int total = 0, before = 0;
    if (tid < n_experts) {
        if (counts)
            for (int c = 0; c < n_chunks; ++c) {
                const int v = counts[(int64_t)c * n_experts + tid];
                before += c < (int)blockIdx.x ? v : 0;
                total += v;
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
    for (int64_t p = max((int64_t)all, blockIdx.x * chunk) + tid; p < min((blockIdx.x + 1) * chunk, n); p += 64 * kGroupWaves) order[p] = -1;
    __syncthreads();
    int *const next = cnt + wave * n_experts;
    for (int64_t i = from; i < end; i += 64) {
        const int id = id_at(ids, ld_ids, picks, i + lane, end, n_experts);
        const uint64_t m = same_id(id, bits), below = m & ((1ull << lane) - 1);
        int at = -1;
        if (id < n_experts) at = next[id] + __popcll(below);
        in_order();  // all have read before the first lanes add
        if (id < n_experts && below == 0) next[id] = at + __popcll(m);
        in_order();
        if (i + lane < end) {
            place[i + lane] = at;
            if (at >= 0) order[at] = (int)(i + lane);
        }
    }
}

hipError_t launch_experts_group(const int32_t *ids, int64_t ld_ids, int64_t tokens, int picks, int n_experts, int32_t *starts,
                                int32_t *order, int32_t *place, int32_t *workspace, hipStream_t stream)
{
    const int64_t n = tokens * picks, chunk = group_chunk(n);
    const int chunks = n ? group_chunks(n) : 1;
    int bits = 0;
    while ((n_experts >> bits) != 0) ++bits;  // of the ids and of n_experts, which stands for none
    const size_t lds = (size_t)kGroupWaves * n_experts * 4 + kGroupWaves * 4;
    if (chunks > 1)
        hipLaunchKernelGGL(k_experts_count, dim3((unsigned)chunks), dim3(64 * kGroupWaves), lds, stream, ids, ld_ids, picks, n, chunk, n_experts, bits,
                           workspace);
    hipLaunchKernelGGL(k_experts_place, dim3((unsigned)chunks), dim3(64 * kGroupWaves), lds, stream, ids, ld_ids, picks, n, chunk, n_experts, bits,
                       chunks > 1 ? workspace : nullptr, chunks, starts, order, place);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------
// The weighted sum of a token's rows: a thread has 8 columns of one token.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_experts_combine(const uint16_t *__restrict__ y, int64_t ldy, int n_rows, const int32_t *__restrict__ place,
                                                         const float *__restrict__ weights, int64_t tokens, int picks, int eighths,
                                                         uint16_t *__restrict__ z, int64_t ldz)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= tokens * eighths) return;
    const int64_t t = i / eighths;
    const int c = (int)(i - t * eighths) * 8;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < picks; ++j) {
        const int p = place[t * picks + j];
        if ((unsigned)p >= (unsigned)n_rows) continue;
        const float w = weights[t * picks + j];
        const uint4 v = ld16(y + (int64_t)p * ldy + c);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            s[2 * k] += w * value_lo(u[k]);
            s[2 * k + 1] += w * value_hi(u[k]);
        }
    }
    st16_stream(z + t * ldz + c, uint4{pack_bf16_rne(s[0], s[1]), pack_bf16_rne(s[2], s[3]), pack_bf16_rne(s[4], s[5]), pack_bf16_rne(s[6], s[7])});
}

hipError_t launch_experts_combine(const uint16_t *y, int64_t ldy, int n_rows, const int32_t *place, const float *weights, int64_t tokens, int picks,
                                  int out, uint16_t *z, int64_t ldz, hipStream_t stream)
{
    const int64_t grid = (tokens * (out / 8) + 255) / 256;
    if (grid > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_experts_combine, dim3((unsigned)grid), dim3(256), 0, stream, y, ldy, n_rows, place, weights, tokens, picks, out / 8, z, ldz);
    return hipGetLastError();
}

}  // namespace lora
