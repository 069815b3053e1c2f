// How tc_attn_chunk cuts its work: plain code, for the kernels, the entry points and tests without a GPU.
//
// An item is a block of up to `rows` rows (token, head) of one request and KV head, and a part of the tiles of keys that any
// of them sees.  Lengths are known on the device alone, so every CTA finds the same cut there, by ChunkCost.
#pragma once

#include <stdint.h>

#include "kv_index.h"

namespace tc {

constexpr int kChunkSms = 148;          // B200; workspaces must not depend on the device that happens to be current
constexpr int kChunkLeastShare = 6;     // tiles of a part at least: beginning, ending and joining one costs as much as some eight
constexpr int kChunkMostParts = 128;    // of a request's keys
constexpr int kChunkSplitItems = 4 * kChunkSms;  // items that a cut may leave of the requests it cuts
constexpr int kChunkEnough = 4 * kChunkSms;      // with so many items nothing is cut: they even out by themselves
constexpr int kChunkEnds = 4;           // what an item costs beside its tiles, in tiles; a cut one twice

struct ChunkShape {
    int32_t group;   // query heads per KV head
    int32_t rows;    // of an item at most, a power of two
    int32_t keys;    // of a tile, a power of two
    int32_t window;  // keys that a row sees up to its own, 2^30 = all
    int32_t sinks;   // first keys that every row sees
    int32_t heads;   // KV heads
    int32_t rows_shift, keys_shift, near_tiles;  // near_tiles: that a block's windows can touch
    uint32_t group_mul, group_shift;             // to divide by `group`
    int32_t turns;                               // slots may take turns (chunk_turns)
};

TC_HD int32_t chunk_low(int32_t a, int32_t b) { return a < b ? a : b; }
TC_HD int32_t chunk_high(int32_t a, int32_t b) { return a > b ? a : b; }
TC_HD int32_t chunk_by_group(const ChunkShape &s, int32_t n)
{
    const uint32_t u = static_cast<uint32_t>(n);
    return static_cast<int32_t>((static_cast<uint32_t>((static_cast<uint64_t>(u) * s.group_mul) >> 32) + u) >> s.group_shift);
}

inline ChunkShape chunk_shape(int32_t group, int32_t rows, int32_t keys, int32_t window, int32_t sinks, int32_t heads)
{
    ChunkShape s{group, rows, keys, window, sinks, heads, 0, 0, 0, 0, 0, 0};
    while (1 << s.rows_shift < rows) s.rows_shift++;
    while (1 << s.keys_shift < keys) s.keys_shift++;
    s.near_tiles = (window + (rows - 1) / group + 1 + keys - 2) / keys + 1;
    while ((1ll << s.group_shift) < group) s.group_shift++;
    s.group_mul = static_cast<uint32_t>(((1ull << 32) * ((1ull << s.group_shift) - static_cast<uint64_t>(group))) / static_cast<uint64_t>(group) + 1);
    return s;
}

// Items of n new tokens of one KV head, uncut.
TC_HD int32_t chunk_blocks(const ChunkShape &s, int32_t n) { return (n * s.group + s.rows - 1) >> s.rows_shift; }

TC_HD int32_t chunk_tiles_of(const ChunkShape &s, int32_t keys) { return (keys + s.keys - 1) >> s.keys_shift; }
// Tiles that a block of a request with `len` keys lists at most.
TC_HD int32_t chunk_tiles(const ChunkShape &s, int32_t len) { return chunk_low(s.near_tiles + chunk_tiles_of(s, chunk_low(s.sinks, len)), chunk_tiles_of(s, len)); }

// Seconds that a warp waits for an item of so many tiles to end: some 60 us a tile.  The slowest measured took 7.1 (256 rows, int8, D = 128, scales
// far apart), so that an item of 2^24 keys takes 0.93 s at full clocks and more under a power cap.
TC_HD int32_t chunk_patience(int32_t tiles) { return 1 + (tiles >> 14); }

// The tiles that a block lists: the first `firsts`, which hold the keys that all rows see, then from tile firsts + skip on.
struct ChunkList {
    int32_t key_end, key_low;  // keys below key_end, from key_low on or below `sinks`, are seen by some row
    int32_t firsts, skip, count;
    int32_t end0, begin1;  // of the list: slot 0 needs none from end0 on, slot 1 none between `firsts` and begin1
};
// pos0: position of the request's first new token; rows row0 .. row0 + rows_here - 1 of its n * group; slot 0 holds the first `slot_rows`.
TC_HD ChunkList chunk_list(const ChunkShape &s, int32_t pos0, int32_t row0, int32_t rows_here, int32_t slot_rows)
{
    ChunkList l;
    const int32_t first = pos0 + chunk_by_group(s, row0), last = pos0 + chunk_by_group(s, row0 + rows_here - 1);
    l.key_end = last + 1;
    l.key_low = chunk_high(0, first - s.window + 1);
    const int32_t low = l.key_low >> s.keys_shift, high = last >> s.keys_shift, sunk = chunk_tiles_of(s, chunk_low(s.sinks, l.key_end));
    l.firsts = chunk_low(sunk, low);
    l.skip = low - l.firsts;
    l.count = l.firsts + high - low + 1;
    l.end0 = l.count, l.begin1 = l.count;
    if (rows_here > slot_rows) {
        l.end0 = ((pos0 + chunk_by_group(s, row0 + slot_rows - 1)) >> s.keys_shift) - l.skip + 1;
        if (sunk > low) l.begin1 = l.firsts;  // keys that every row sees reach into the tiles behind
        else l.begin1 = (chunk_high(0, pos0 + chunk_by_group(s, row0 + slot_rows) - s.window + 1) >> s.keys_shift) - l.skip;
    }
    return l;
}

TC_HD int32_t chunk_parts(int32_t tiles, int32_t share) { return (tiles + share - 1) / share; }
// A request of up to 128 rows leaves one of two slots idle.  Where its keys are cut, both have its rows, and take turns at a part's tiles: each
// leaves a part of its own.  Codes that a CTA widens gain by it (8 tokens behind 120000, 56 rows a KV head, int8: 118 -> 100 us); 16-bit pools
// lose more by twice the parts (70 -> 78 us).
TC_HD bool chunk_turns(const ChunkShape &s, int32_t n, int32_t parts) { return s.turns && n * s.group <= 128 && parts > 1 && 2 * parts <= kChunkMostParts; }
// Whether there is room for all rows of parts.  There is where offsets do not decrease; where they do, requests share tokens and may be more than
// a plan counts, and then nothing is cut.
TC_HD bool chunk_has_room(int64_t part_rows, int64_t rows) { return rows <= part_rows; }
// The cuts that are looked at: into parts of so many tiles that the longest list has up to 1 .. 16, then up to 23, 30 .. 128.
constexpr int kChunkCuts = 32;
TC_HD int32_t chunk_share(int32_t most_tiles, int32_t cut)
{
    const int32_t parts = cut < 16 ? cut + 1 : 16 + (cut - 15) * 7;
    return chunk_high((most_tiles + parts - 1) / parts, parts > 1 ? kChunkLeastShare : 1);
}

// What a cut costs, in tiles.  Two guesses at when the last SM ends, neither of which knows the order: waves of items of average size; and
// waves of items as long as the longest, where those of less than half a share fill what the last wave leaves.  Of 340 drawn batches, the
// cuts so found end 4 % behind the best of all (a simulation); by the first guess alone 7 %, by the second 5 %.
// (Fewer than kChunkEnough blocks, of less than 2^18 tiles.)
struct ChunkCost {
    int32_t items = 0, split = 0, tiles = 0, longest = 0, large = 0, rest = 0;
    // blocks: of one request, of all KV heads
    TC_HD void add(int32_t blocks, int32_t tiles_of, int32_t share, int32_t parts)
    {
        const int32_t ends = (parts > 1 ? 2 : 1) * kChunkEnds, last = tiles_of - (parts - 1) * share;
        items += blocks * parts;
        tiles += blocks * tiles_of;
        if (parts > 1) split += blocks * parts;
        longest = chunk_high(longest, chunk_low(tiles_of, share) + ends);
        large += blocks * (parts - 1);
        if (2 * last > share) large += blocks;
        else rest += blocks * (last + ends);
    }
};
TC_HD float chunk_cost(const ChunkCost &c)
{
    if (c.split > kChunkSplitItems) return 3e38f;
    if (c.items == 0) return 0.f;
    const float longest = static_cast<float>(c.longest);
    const float waves = static_cast<float>((c.items + kChunkSms - 1) / kChunkSms);
    const float even = waves * static_cast<float>(c.tiles + kChunkEnds * (c.items + c.split)) / static_cast<float>(c.items);
    const int32_t large_waves = (c.large + kChunkSms - 1) / kChunkSms;
    const float left = static_cast<float>(c.rest) - static_cast<float>(large_waves * kChunkSms - c.large) * longest;
    const float filled = static_cast<float>(large_waves) * longest + (left > 0.f ? left / kChunkSms : 0.f);
    return 0.3f * (even > longest ? even : longest) + 0.7f * (filled > longest ? filled : longest);
}

// What the host can say of a call: its grid, and its workspace: R pairs of words, then sums and outputs of the parts' rows.
struct ChunkPlan {
    int64_t grid;       // items at most
    int64_t part_rows;  // rows of parts at most; 0: nothing is cut
    int64_t cuts_at, sums_at, parts_at, workspace;
};
inline void plan_chunk(const ChunkShape &s, int64_t R, int64_t n_tokens, int64_t max_new, int64_t max_len, int64_t D, ChunkPlan *p)
{
    *p = ChunkPlan{};
    const int64_t new_most = max_new < n_tokens ? max_new : n_tokens, live = R < n_tokens ? R : n_tokens;
    const int64_t by_each = R * chunk_blocks(s, static_cast<int32_t>(new_most)), by_all = n_tokens * s.group / s.rows + live;
    const int64_t items = (by_each < by_all ? by_each : by_all) * s.heads, tiles = chunk_tiles(s, static_cast<int32_t>(max_len));
    p->grid = items;
    if (tiles <= kChunkLeastShare || items == 0) return;
    p->grid += kChunkSplitItems;
    const int64_t each = s.turns ? 2 : 1, item_rows = each * new_most * s.group < s.rows ? each * new_most * s.group : s.rows, rows = each * R * new_most * s.group * s.heads;
    const int64_t parts = chunk_parts(static_cast<int32_t>(tiles), kChunkLeastShare);
    const int64_t by_items = kChunkSplitItems * item_rows, by_rows = rows * (parts < kChunkMostParts ? parts : kChunkMostParts);
    p->part_rows = by_items < by_rows ? by_items : by_rows;
    auto place = [&](int64_t bytes) {
        const int64_t at = p->workspace;
        p->workspace += (bytes + 255) / 256 * 256;
        return at;
    };
    p->cuts_at = place(R * 8);
    p->sums_at = place(p->part_rows * 4);
    p->parts_at = place(p->part_rows * D * 4);
}

}  // namespace tc
