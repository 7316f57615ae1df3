// Launch entry points of the operators in include/lora_experts.h (lora_experts.hip), which their host side (lora_experts.cpp) calls.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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
// hipErrorInvalidConfiguration, and nothing is launched, where there are more tiles than a launch can have.
hipError_t launch_experts_linear(const ExpertsArgs &a, bool bits8, hipStream_t stream);

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
