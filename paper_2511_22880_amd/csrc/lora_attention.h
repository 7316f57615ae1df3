// Launch entry points of the operators in include/lora_attention.h (lora_attention.hip), which their host side (lora_attention.cpp) calls.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lora_internal.h"

namespace lora {

// [tokens][heads][dim] in bf16: strides of a token and a head, in elements
struct HeadRows {
    uint16_t *p;
    int64_t token, head;
};

struct PagedCache {
    char *k, *v;
    float *k_scales, *v_scales;
    int pages, page_shift, kv_heads, dim;
    bool bits8;
};

// Rows turned by their positions: q's into y, and (cache.k given) k's into the cache beside v's.
struct TurnArgs {
    HeadRows q, y, k, v;
    int q_heads, heads;       // of q; of q, k and v together
    uint32_t per_heads;       // 2^32 / heads, rounded up: numbers below 2^16 are divided by it
    int tokens, dim;
    const int32_t *positions, *slots;
    const uint64_t *turns;    // NULL: nothing is turned
    int dims;                 // turned elements of a head
    float magnitude;
    int inverse, interleaved;
    PagedCache cache;
};

hipError_t launch_turn(const TurnArgs &a, hipStream_t stream);

// ---- attention ------------------------------------------------------------------------------------------------
// A tile: the columns (row of a request, query head of a key head's group), row by row, that a work group holds at a time.
constexpr int kFewWaves = 4;  // wavefronts of k_attend_few: with eight a decode step of 256 requests took 419 to 426 us against 408
constexpr int few_keys(bool bits8) { return (bits8 ? 64 : 32) * kFewWaves; }  // that they take in a step: as many bytes either way

struct AttendArgs {
    HeadRows q, y;
    int tokens, group;            // group: query heads per key head
    uint32_t per_group;           // 2^32 / group, rounded up (0 for 1): the upper half of a number's product with it is the quotient or one more
    const int32_t *starts, *lengths, *table;
    int64_t ld_table;
    int requests, room;           // room: slots of a row of the table
    const uint64_t *tree;
    PagedCache cache;
    float scale;                  // its magnitude times log2 e, never zero
    uint32_t flip;                // the sign bits of q that a negative scale exchanges
    float slack;                  // by how much a score may pass the maximum that weights are relative to: 8 / scale
    int least, most;              // columns of the requests that this launch takes: least < rows * group <= most
    int shares;                   // of a key head's work
    bool cut;                     // shares are of steps, and tiles cut where those end; else every tile is a share
    float *parts;                 // workspace: [kv_heads * shares][2][columns][dim], then sums [..][2][columns][2], then 16 bytes each (CutTile)
};

// Which launches a call takes.
struct AttendForm {
    int columns;       // of a tile
    int shares;        // of a key head's work
    int least, most;
    bool cut;          // tiles may be cut (see AttendArgs)
};
struct AttendForms {
    AttendForm f[2];
    int n;
};

// Tiles of a key head, at most: those that rows fill, and a last one for every request of more than `least` columns.
inline int64_t most_tiles(int64_t tokens, int group, int requests, int columns, int least)
{
    const int64_t all = tokens * group, with = all / (least + 1);
    return all / columns + (requests < with ? requests : with);
}

// Whether tiles are cut.  Tiles of few steps are not, if there are not too many of them for a work group each (one that finds none takes 2 us to see that; the host's
// count can be far above what there are): the parts that cut ones leave cost a launch to join them, and for 256 columns 128 KB each way.  The steps are those of
// the longest request that the page table has room for, which is all that the host knows of lengths.  us a call, wide tiles, cut / whole:
//   4 prompts of 307 to 922 tokens, table as wide   45 / 28
// Up to so many steps, 16 / 8:
//   4 prompts on 9 key heads                        35.5 / 47
//   9 prompts beside 92 single tokens               54 / 76
// Up to so many steps, 16 / 32:
//   few requests of so many keys                    23 / 47, 19 / 54
// Up to so many tiles, four / sixteen times the work groups (eight times is between):
//   6 prompts beside 148 single tokens              42 / 55
inline AttendForm attend_form(int columns, int keys, int whole_steps, int work_groups, int64_t tokens, int group, int kv_heads, int requests, int64_t most_keys, int least, int most)
{
    const int64_t steps = most_keys > 0 ? (most_keys + keys - 1) / keys : 1;  // (a tile without keys is one too: its rows are written)
    int64_t tiles = most_tiles(tokens, group, requests, columns, least), shares = work_groups / kv_heads;
    if (most <= columns && tiles > requests) tiles = requests;
    if (tiles < 1) tiles = 1;
    if (steps <= whole_steps && tiles * kv_heads <= 8 * work_groups) return AttendForm{columns, (int)tiles, least, most, false};
    if (shares < 1) shares = 1;
    if (shares > tiles * steps) shares = tiles * steps;
    return AttendForm{columns, (int)shares, least, most, true};
}

// Tiles of up to 32 columns (k_attend_few): shares for two work groups a compute unit.  Of 16 columns two fit at least; for three was level, and three, four or eight
// times as many shares of a decode step took 410, 414 and 433 us against 400.  Of 32 columns two fit with heads of 64 in bf16 (200 registers a wavefront), otherwise one
// (280 to 386), and half of the shares begin when the others end.  us a call, shares for two / for one, trees of 5 to 8 tokens on 4 query heads a key head:
//   requests x keys    64 x 300 to 6000   256 x 200 to 8000   1 x 8000
//   bf16, heads of 128     129 / 117          523 / 514      28.5 / 18.1
//   bf16, heads of 64       63 / 78           264 / 315      15.8 / 12.7
//   8 bits, of 128          99 / 87.5         350 / 352      18.4 / 16.3
//   8 bits, of 64         62.5 / 54           212 / 211      15.1 / 13.2
// (all take those for two.)  More columns share keys through LDS (k_attend_wide): 33 to 64 columns as four tiles of 16 that hold their own keys / as one of 128,
// 6 trees of up to 11 tokens on 4 query heads a key head: 36 / 25 us.
inline AttendForm few_form(int columns, int64_t tokens, int group, int kv_heads, int requests, int64_t most_keys, bool bits8, int most)
{
    return attend_form(columns, few_keys(bits8), 4, 2 * kComputeUnits, tokens, group, kv_heads, requests, most_keys, 0, most);
}
inline AttendForm wide_form(int columns, int64_t tokens, int group, int kv_heads, int requests, int64_t most_keys, int dim, int least)
{
    return attend_form(columns, 8192 / dim, 16, columns == 128 ? 2 * kComputeUnits : kComputeUnits, tokens, group, kv_heads, requests, most_keys, least, INT32_MAX);
}

inline AttendForms attend_forms(int64_t tokens, int group, int kv_heads, int requests, int64_t most_keys, int64_t most_rows, int dim, bool bits8)
{
    const int64_t rows = most_rows > 0 && most_rows < tokens ? most_rows : tokens, columns = rows * group;
    if (columns <= 32) return AttendForms{{few_form(columns <= 16 ? 16 : 32, tokens, group, kv_heads, requests, most_keys, bits8, INT32_MAX), {}}, 1};
    // (128 / 256 columns: pieces of long prompts 1200 / 1034 us, prompts beside single tokens 511 / 488, trees of 280 to 448 columns 71 / 78; where no request has more than 128 half of
    // 256 would idle)
    const int c = columns <= 128 ? 128 : 256;
    // Requests of very different sizes: those of up to 16 columns in a launch of their own, which reads a single token's keys faster than wide tiles of mostly empty
    // columns, in 8 bits above all, where a step of those has half as many bytes.  The second launch costs its start and end, more than that where a tile of each
    // request finds a compute unit at once and there is little to read.  Here too the table's width stands for the longest request.  us a call, two launches / one, 8
    // key heads of 128 in bf16 unless said, tables as wide as the longest request:
    //   single tokens + prompts   384 + 8               466 / 615      20 + 2 of 16000 keys   134 / 171     16 + 1 of 4000 keys   68 / 60
    //                             200 + 40              406 / 512      32 + 2                81.5 / 86       8 + 1 of 2000 keys   53 / 42
    //                             64 + 1                146 / 177      24 + 1                  65 / 70       2 + 2                39 / 28
    //   .. heads of 64            24 + 2                 51 / 73       .. 2 key heads  60 + 2  68 / 103
    //   .. in 8 bits              16 + 1                 48 / 66       8 + 1, heads of 64      26 / 33      200 + 1 of 400 keys   56 / 67
    //   1 to 64 rows              20 requests            58 / 42       100 requests          292 / 274
    //   1 to 500 rows             30 requests            87 / 84       100 requests          352 / 329
    //   trees of 1 to 22 rows behind up to 161 keys, 40 requests, heads of 64   16.6 / 10.7, in 8 bits 23 / 15
    const double bytes = (double)requests * most_keys * kv_heads * dim * 4;
    const int64_t tiles = (int64_t)requests * kv_heads;
    const bool little = (tiles <= 2 * kComputeUnits && most_keys <= 4 * (8192 / dim)) || (!bits8 && requests <= 32 && tiles <= kComputeUnits && bytes <= 300e6);
    if (requests == 1 || group > 16 || tokens > requests * rows / 2 || little)
        return AttendForms{{wide_form(c, tokens, group, kv_heads, requests, most_keys, dim, 0), {}}, 1};
    return AttendForms{{few_form(16, tokens, group, kv_heads, requests, most_keys, bits8, 16), wide_form(c, tokens, group, kv_heads, requests, most_keys, dim, 16)}, 2};
}

inline size_t attend_parts_bytes(const AttendForm &f, int kv_heads, int dim)
{
    return f.cut && f.shares > 1 ? (size_t)kv_heads * f.shares * (2 * f.columns * (dim + 2) * sizeof(float) + 16) : 0;
}

// bytes that a call may need, whatever `most` says: a launch of some of the requests has no more tiles, nor shares, than one of all
inline size_t attend_most_bytes(int64_t tokens, int group, int kv_heads, int requests, int64_t most_keys, int dim, bool bits8)
{
    size_t most = 0;
    for (int columns : {16, 32, 128, 256}) {
        if (columns > 32 && tokens * group <= columns / (columns == 128 ? 4 : 2)) break;  // (no request has so many)
        const size_t n = attend_parts_bytes(columns <= 32 ? few_form(columns, tokens, group, kv_heads, requests, most_keys, bits8, INT32_MAX)
                                                          : wide_form(columns, tokens, group, kv_heads, requests, most_keys, dim, 0), kv_heads, dim);
        if (n > most) most = n;
    }
    return most;
}

// steps of a key head's tiles, at most
inline int64_t most_steps(int64_t tokens, int group, int requests, int64_t most_keys)
{
    return most_tiles(tokens, group, requests, 16, 0) * ((most_keys + 63) / 64 + 1);
}

hipError_t launch_attention(AttendArgs a, const AttendForm &f, hipStream_t stream);

}  // namespace lora
