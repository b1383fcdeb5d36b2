// retopk_paged_plan.h -- host arithmetic of the paged calls: the division by the page
// size and the split of paged_attention over blocks.  No HIP in it, so that a CPU program
// can check the rules over whole ranges of sizes.  Not part of the public C ABI.
#pragma once

#include "retopk_plan.h"

namespace retopk {

// x / page_size for 0 <= x < 2^31 is (x * magic) >> (31 + shift) with shift =
// ceil(log2(page_size)) and magic = ceil(2^(31 + shift) / page_size), below 2^32.  With
// e = magic * page_size - 2^(31 + shift) < page_size <= 2^shift the product is
// x / page_size plus x * e / (page_size * 2^(31 + shift)), less than 1 / page_size: the
// floor is exact.
struct Divisor {
    uint32_t magic;
    int32_t shift;
};
inline Divisor divisor_of(int32_t page_size)
{
    Divisor d = {0u, 0};
    while (((int64_t)1 << d.shift) < page_size) ++d.shift;
    d.magic = (uint32_t)((((uint64_t)1 << (31 + d.shift)) + (uint64_t)page_size - 1) / (uint64_t)page_size);
    return d;
}
constexpr uint32_t divide(uint32_t x, Divisor d)
{
    return (uint32_t)(((uint64_t)x * d.magic) >> (31 + d.shift));
}

// paged_attention: block (chunk, KV head, token) takes chunk_rows positions of one token's
// sequence, counted from its first attended position rounded down to a tile.  The lengths
// are on the device, so the grid is sized for max_len and blocks past a sequence's end
// leave at once.
constexpr int kAttendTile = 32;       // positions of a wave's tile
constexpr int kAttendBlocks = 1024;   // blocks that fill the chip
constexpr int kAttendRowsMin = 256;
constexpr int kAttendRowsMax = 2048;

struct AttendPlan {
    int64_t chunk_rows;        // a multiple of kAttendTile
    int64_t chunks;            // chunks a token needs at most
    int64_t blocks;            // of the whole grid
    int64_t workspace;         // bytes of partial results; 0 with one chunk a token
};

inline AttendPlan attend_plan(int64_t tokens, int64_t n_q_heads, int64_t n_kv_heads, int d, int64_t max_len,
                              int64_t window)
{
    AttendPlan p;
    // a window's first position may lie kAttendTile - 1 past the tile it begins in
    int64_t span = window > 0 && window + kAttendTile - 1 < max_len ? window + kAttendTile - 1 : max_len;
    const int64_t groups = tokens * n_kv_heads;
    int64_t rows = ceil_div(ceil_div(span * groups, kAttendBlocks), kAttendTile) * kAttendTile;
    if (rows < kAttendRowsMin) rows = kAttendRowsMin;
    if (rows > kAttendRowsMax) rows = kAttendRowsMax;
    p.chunk_rows = rows;
    p.chunks = ceil_div(span, rows);
    p.blocks = groups * p.chunks;
    p.workspace = p.chunks > 1 ? tokens * n_q_heads * p.chunks * (d + 2) * 4 : 0;
    return p;
}

}  // namespace retopk
