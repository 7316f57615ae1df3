// Launch entry points of the operators in include/lora_experts.h (lora_experts.hip), which their host side (lora_experts.cpp) calls.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lora_internal.h"

namespace lora {

constexpr int kScaleBlock = 128;     // values of a row, or of a row and a column of a weight, that share a scale
constexpr int kPieceBytes = 128;     // of a row: what the products walk k in (64 bf16 or 128 8-bit values)
constexpr int kMaxExperts = 512;     // (a work group that groups picks has a count of each for 16 wavefronts in LDS)
constexpr int kQuantizeBlocks = 2;   // of 128 values a thread that rounds to 8 bits has a part of, a sixteenth each
constexpr int kGroupUnit = 1024;      // picks of a work group that groups them: 1, 2, 4, 8 or a multiple of 16 times as many
constexpr int kGroupAlone = 8;        // up to so many work groups each look at all picks; with more a launch counts ahead
constexpr int kGroupMaxChunks = 256;  // of either launch then

// the runtime launches fewer than 2^32 threads
inline bool can_launch(int64_t work_groups, int threads) { return work_groups <= (int64_t)UINT32_MAX / threads; }

// rows of a launch that rounds rows of so many blocks (256 threads for 16 kQuantizeBlocks blocks)
inline int64_t quantize_rows_at_once(int blocks) { return ((int64_t)1 << 28) / blocks; }

// picks of a work group
inline int64_t group_chunk(int64_t n_picks)
{
    if (n_picks <= kGroupAlone * kGroupUnit) return kGroupUnit;
    for (int m = 2; m <= 8; m *= 2)
        if (n_picks <= (int64_t)m * kGroupUnit * kGroupMaxChunks) return m * kGroupUnit;
    const int64_t unit = 16 * kGroupUnit, least = (n_picks + kGroupMaxChunks - 1) / kGroupMaxChunks;
    return (least + unit - 1) / unit * unit;
}
inline int group_chunks(int64_t n_picks) { const int64_t c = group_chunk(n_picks); return (int)((n_picks + c - 1) / c); }
inline bool group_counts(int64_t n_picks) { return n_picks > kGroupAlone * kGroupUnit; }
// as many work groups as any number of picks up to this one has (from 2^19, 2^20, 2^21 and every multiple of 2^22 picks on a work group takes more, and they are fewer)
inline int group_most_chunks(int64_t n_picks) { return n_picks > (int64_t)2 * kGroupUnit * kGroupMaxChunks ? kGroupMaxChunks : group_chunks(n_picks); }

// Rows of x, by expert, times the experts' weights (see include/lora_experts.h).  starts == NULL: one expert that has all rows.
struct ExpertsArgs {
    const char *x;           // rows of `pieces` pieces of 128 bytes, row stride ldx_bytes
    int64_t ldx_bytes;
    const float *x_scales;   // 8 bits: [tokens][pieces], row stride ld_scales
    int64_t ld_scales;
    int tokens;              // rows of x
    const int32_t *starts;   // [experts + 1]
    const int32_t *order;    // place -> pick, or NULL: place -> row of x
    int picks;               // per token
    int n_rows;              // places
    int n_experts;
    const char *w;           // packed
    const float *w_scales;   // 8 bits: [experts][out / 128][pieces]
    int pieces, out;
    bool large;              // the weights that are met do not fit half of the chip's last cache (set by the launcher)
    uint16_t *y;
    int64_t ldy;
};
// experts that some row can meet, 0 for one layer (n_experts = 0 there)
inline int met_experts(int n_experts, int n_rows) { return n_rows < n_experts ? n_rows : n_experts; }

// Weights of more than half of what the chip's last cache holds are read past the caches where an expert has one tile of rows: they would leave
// there whatever else a layer keeps, and another pass would hardly find them.  us, through the caches / past them: 512 rows of 64 experts
// 2048 -> 1536 in bf16 72 / 64 (6.4 TB/s), 1024 78 / 69, 2048 81 / 72, in 8 bits 512 rows 40 / 36; 16 rows 16384 -> 16384 in 8 bits 50 / 44.  Smaller ones: one row
// 8192 -> 8192 (three such layers in turn, 201 MB) 11.9 / 15.5.
inline bool large_weights(int met, int out, int pieces) { return (int64_t)(met ? met : 1) * out * pieces * kPieceBytes > ((int64_t)128 << 20); }

// The kernel of a launch of products: k_experts_thin (16 rb rows x 16 cb columns, `groups` wavefronts), k_experts_mid (16 rb x 64 cb, `groups` groups of
// wavefronts) or k_experts_wide; once: W past the caches.
struct ProductForm {
    enum Kind { kThin, kMid, kWide } kind;
    int rb, cb, groups;
    bool once;
};

// The tiles of a launch: the largest of which there are enough to occupy most compute units, no higher than an expert's rows in the mean ask for.  Row
// tiles are counted as if every expert's last one were half there (the host does not know who picked what).  With one tile of 64 x 256, 64 x 128 or 32 x 128 on a
// compute unit two groups of wavefronts share its pieces (two), unless k is short; with more of them the tiles' own wavefronts are enough (one).
// Device time in us, one layer in 8 bits (wide: k_experts_wide, whose tiles are 256 x 256 or 128 x 256):
//   rows, layer        wide        64 x 256, one / two   64 x 128, one / two   32 x 128, one / two   32 x 64   16 x 64   16 x 32   16 x 16
//   1     4096 4096                                                                                            6.3       5.6       5.3
//   64    4096 4096    36          32 / 25               21 / 17               12.6 / 12.5           8.9       7.3       9.2
//   128   4096 4096    36          32 / 25               21 / 17               12.7 / 12.6           9.4       11.3      14.8
//   256   4096 4096    33          33 / 25               21 / 17               13.4 / 13.1           15.0      19.1      26
//   512   4096 4096    34          33 / 26               22 / 17.5             22 / 21               25        32        52
//   1024  4096 4096    36          35 / 27               32 / 32               39 / 40               49        69        107
//   2048  4096 4096    42          49 / 53               60 / 64               78 / 79               98        136       215
//   64    16384 16384  131         132 / 122             90 / 86               75 / 66               70        90        117
//   256   16384 16384  132         131 / 118             134 / 144             181 / 175             179       252       372
//   115   5568 3584    43          42 / 32               27 / 21               16.3 / 15.5           11.6      13.8      17.4
//   373   5440 640     41                                26 / 21               15.8 / 15.1           11.3      9.1       11.4
//   1149  7232 512     54          54 / 41               33 / 27               20.3 / 19.4           24        24        33
//   689   8128 14848   111         150 / 152             156 / 160             201 / 195             218       316       472
//   10081 704 512      12.1        15.1 / 18.8           15.9 / 18.4           14.6 / 18.2           28        33        59
//   7     3008 4352                                                                                            5.5       4.9       5.8
// and of 64 experts 2048 -> 1536, rows each, in 8 bits: 8 49, - , 47, 39.9, 44, 41, 54; 64 54, 64, 71, 66, 82, 91, 170; in bf16: 8 81, - , 75, 75, 71, 73, 76;
// 32 85, 86, 78, 90, 91, 104, 130; 64 90, 98, 102, 109, 115, 153, 200 (in the same order, one group of wavefronts, through the caches).
// Over 50 random sizes of one layer the choice was 1.7 % from the best of all of these in the mean, over 50 of experts 7 % (a quarter of them with one pick in
// ten here, which the host does not know: up to twice the best).
inline ProductForm product_form(bool bits8, int n_rows, int met, int out, int pieces)
{
    const int per = met ? n_rows / met : n_rows;
    auto fills = [&](int rows, int columns, int least) {
        const int64_t row_tiles = ((int64_t)n_rows + rows - 1) / rows + met / 2;
        return (row_tiles > met ? row_tiles : met) * ((out + columns - 1) / columns) >= least;
    };
    constexpr int kMost = kComputeUnits * 9 / 16;
    const bool large = large_weights(met, out, pieces);
    auto once = [&](int rows) { return large && (met ? per <= rows * 3 / 4 : per <= rows); };
    auto thin = [&](int rb, int cb, int waves) { return ProductForm{ProductForm::kThin, rb, cb, waves, cb == 4 && once(16 * rb)}; };
    auto middle = [&](int rb, int cb) {
        const bool two = pieces >= 16 && !fills(16 * rb, 64 * cb, 2 * kComputeUnits);
        return ProductForm{ProductForm::kMid, rb, cb, two ? 2 : 1, cb == 2 && once(16 * rb)};
    };
    // (more tiles of 64 x 256 than one round: half as many of 128 x 256 or 256 x 256, in one, are earlier.  us, 64 x 256 / wide: 1024 rows 4096 -> 4096 in 8 bits 27 / 33,
    // 1152 49 / 33, 2048 49 / 40, 1100 9152 -> 4480 92 / 67, 2000 of 8 experts 4096 -> 2048 in bf16 77 / 62, 1600 of them 58 / 60.  Few rows an expert, 64 experts
    // 2048 -> 1536, what was taken else / wide: in 8 bits 20 rows 40 / 44, 30 51 / 45, 40 57 / 45, in bf16 30 72 / 78, 40 87 / 79)
    if (per > (bits8 ? 25 : 35) && (fills(256, 256, kMost) || fills(64, 256, kComputeUnits + 1))) return ProductForm{ProductForm::kWide, 0, 0, 0, false};
    if (per > 32 && out % 256 == 0 && fills(64, 256, kMost)) return middle(4, 4);
    if (per > 24 && fills(64, 128, kMost)) return middle(4, 2);
    // (a row an expert, of large weights: 16 x 64 tiles cost up to a tenth more where all picks have an expert here, but where one in ten has, as with experts on
    // eight chips, they are through in half to two thirds of the time.  us, 32 x 128 / 16 x 64, all and one in ten: 90 picks of 78 experts 3584 -> 512 in 8 bits
    // 19.2 / 21.3 and 14.0 / 9.4, 64 of 64 2048 -> 1536 in bf16 50.7 / 50.1 and 17.8 / 11.3, 16 of 64 4096 -> 4096 75.2 / 78.7 and 25.4 / 14.0)
    if ((per > 6 || (large && per > 1 && met)) && fills(32, 128, kMost)) return middle(2, 2);
    if (per > 16 && fills(32, 64, kMost)) return thin(2, 4, 4);
    if (fills(16, 64, kMost)) return thin(1, 4, 4);
    if (fills(16, 32, kMost)) return thin(1, 2, 8);
    return thin(1, 1, 8);
}

// hipErrorInvalidConfiguration, and nothing is launched, where there are more tiles than a launch can have.
hipError_t launch_experts_linear(ExpertsArgs a, bool bits8, hipStream_t stream);

// W [experts][out][row_bytes] -> operand order (see the kernels).  row_bytes: whole pieces, of which the bytes behind used_bytes become zero.
hipError_t launch_experts_pack(const char *w, int64_t n_experts, int row_bytes, int used_bytes, int out, bool bits8, char *dst,
                               hipStream_t stream);

hipError_t launch_rows_quantize(const uint16_t *x, int64_t ldx, int64_t rows, int in, uint8_t *q, int64_t ldq, float *scales,
                                int64_t ld_scales, hipStream_t stream);

// workspace: group_chunks(n) * n_experts ints where group_counts(n)
hipError_t launch_experts_group(const int32_t *ids, int64_t ld_ids, int64_t tokens, int picks, int n_experts, int32_t *starts,
                                int32_t *order, int32_t *place, int32_t *workspace, hipStream_t stream);

hipError_t launch_experts_combine(const uint16_t *y, int64_t ldy, int n_rows, const int32_t *place, const float *weights, int64_t tokens, int picks,
                                  int out, uint16_t *z, int64_t ldz, hipStream_t stream);

}  // namespace lora
