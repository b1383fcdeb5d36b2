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

// paged_attention: how the positions of all (token, KV head) groups are shared out over waves,
// each of which works alone.  A token's positions count from its first attended one rounded
// down to a tile.  The lengths are on the device, the host knows only max_len, so there are
// three splits:
//   DIRECT    one block a group: no group has more than a few tiles (kAttendDirect; twice and more
//             where the groups alone fill the chip), and the block's waves join their results
//             and write the output themselves.  One launch: 512 positions of 8 KV heads take 9.0 us
//             from 4-bit pages and 10.5 in BALANCED's two, 768 take 11.0 and 10.5, 1024 12.7 and
//             10.5; of f32 pages 256 take 8.1 and 10.9, 384 11.2 and 11.6 (four query heads on each:
//             17.7 and 15.2); 2000 of 1024 groups 43 and 52 from 4-bit pages.
//   BALANCED  the tiles of all groups in one row, token after token, cut into equal parts on
//             the device, one a wave, so that ragged lengths leave no wave idle; a part may
//             span several groups and a group several parts.  At most kAttendTokens tokens,
//             whose tile counts each block sums up for itself.
//   CHUNKED   wave (token, KV head, chunk of kAttendChunk rows) for more tokens than that;
//             waves past a sequence's end leave at once.
// The partial results of BALANCED have numbers wave + group, which no two parts share (each
// part of a wave begins a new group, each part of a group a new wave).  Where all waves of a
// block work on one group they join their results under the number of the first.
constexpr int kAttendTile = 32;       // positions of a tile
constexpr int kAttendDirect = 20;     // tiles
constexpr int kAttendDirectF32 = 8;   // of f32 pages, whose tiles take three times as long
constexpr int kAttendDirectFull = 64; // where there is a wave for every slot
constexpr int kAttendSimds = 1024;    // up to as many tiles a BALANCED wave takes one, of more two at least
constexpr int kAttendStart = 2;       // tiles that the start of a BALANCED group counts as, at most
constexpr int kAttendWaves = 4;       // of a block
constexpr int kAttendTokens = 1024;
constexpr int kAttendChunk = 512;     // rows

enum AttendSplit : int { ATTEND_DIRECT = 0, ATTEND_BALANCED = 1, ATTEND_CHUNKED = 2 };
struct AttendPlan {
    int split;
    int64_t waves;             // in blocks of kAttendWaves, of which the last may be part empty
    int64_t chunks;            // CHUNKED: a group
    int64_t parts;             // partial results of a KV head's query heads; 0: DIRECT
    int64_t ends_bytes;        // BALANCED: the tile counts, at the workspace's start
    int64_t workspace;         // bytes
};

// slots: the waves that run at once; direct: the tiles of a DIRECT group.
inline AttendPlan attend_plan(int64_t tokens, int64_t n_q_heads, int64_t n_kv_heads, int d, int64_t max_len,
                              int64_t window, int64_t slots, int direct)
{
    AttendPlan p = {ATTEND_DIRECT, tokens * n_kv_heads * kAttendWaves, 1, 0, 0, 0};
    // a window's first position may lie kAttendTile - 1 past the tile it begins in
    const int64_t span = window > 0 && window + kAttendTile - 1 < max_len ? window + kAttendTile - 1 : max_len;
    const int64_t groups = tokens * n_kv_heads, tiles = ceil_div(span, kAttendTile);
    if (tiles <= (groups * kAttendWaves >= slots ? kAttendDirectFull : direct)) return p;
    if (tokens <= kAttendTokens && groups * tiles < ((int64_t)1 << 30)) {
        p.split = ATTEND_BALANCED;
        const int64_t all = groups * tiles, pairs = ceil_div(all, 2);
        const int64_t most = all < kAttendSimds ? all : pairs > kAttendSimds ? pairs : kAttendSimds;
        p.waves = most < slots ? most : slots;
        p.parts = p.waves + groups;
        p.ends_bytes = ceil_div(4 * (tokens + 2), 64) * 64;
    } else {
        p.split = ATTEND_CHUNKED;
        p.chunks = ceil_div(span, kAttendChunk);
        p.waves = groups * p.chunks;
        p.parts = p.waves;
    }
    p.workspace = p.ends_bytes + p.parts * (n_q_heads / n_kv_heads) * (d + 2) * 4;
    return p;
}

// Tiles a BALANCED wave takes of `all`.  4096 positions of 8 heads, 1024 tiles, take 19.4 us from f32
// pages with one each and 22.4 with two; 8192 take 27.0 and 24.2 (4 bits: 12.3 and 12.8, 13.9 and 12.9).
constexpr uint32_t attend_part(uint32_t all, uint32_t waves)
{
    const uint32_t n = all / waves + (all % waves != 0), least = all > (uint32_t)kAttendSimds ? 2u : 1u;
    return n < least ? least : n;
}

// Empty tiles put before each group's, since a wave that comes to a new group begins again: as many
// as fit what rounding up leaves of the waves' `per` tiles each, so that no wave takes longer for it.
// 32 ragged sequences, 28 heads on 4, 4 bits: 38.1 us with none, 33.5 with one, 32.2 with two, 32.1 with four.
constexpr uint32_t attend_start(uint32_t all, uint32_t waves, uint32_t per, uint32_t groups)
{
    const uint64_t left = (uint64_t)per * waves - all;
    uint32_t n = 0;
    while (n < (uint32_t)kAttendStart && (uint64_t)groups * (n + 1) <= left) ++n;
    return n;
}

// The parts of a group whose tiles are [from, to), `per` a wave: waves from `first` on, of which
// after `lead` there are `joints` whole blocks that joined theirs.
struct AttendParts {
    int first, count, lead, joints;
};
constexpr AttendParts attend_parts(int from, int to, int per)
{
    const int b0 = from / per, b1 = to > from ? (to - 1) / per : b0 - 1;
    const int64_t block = (int64_t)kAttendWaves * per;
    const int k0 = (int)((from + block - 1) / block), k1 = (int)(to / block);
    if (k1 <= k0) return AttendParts{b0, b1 - b0 + 1, 0, 0};
    const int lead = kAttendWaves * k0 - b0;
    return AttendParts{b0, lead + (k1 - k0) + (b1 - kAttendWaves * k1 + 1), lead, k1 - k0};
}

}  // namespace retopk
