// How tc_attn_decode cuts its work.  Plain host code, so that it can be tested without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace tc {

// Every part of a row's keys leaves a normalised output and the base-2 logarithm of its sum in the workspace; a
// last kernel joins them.
struct AttnSplit {
    int32_t group;             // query heads per KV head
    int32_t columns;           // rows an item of the stream has: 8, or 16 for groups of more than 8
    int32_t own_blocks;        // blocks of `columns` of a request's group rows
    int32_t prefix_rows;       // rows of queries one prefix CTA takes: 128 (two parts per chunk of keys, one a slot) or
                               // 256; 16: the prefix is part of the stream
    int32_t prefix_blocks;     // blocks of that many (of `columns`) of the R * group rows of one KV head
    int32_t prefix_parts;      // parts that prefix_kernel leaves of every row
    int32_t stream_ctas;       // of four warps each
    int32_t tile_keys;         // keys of a tile of the stream
    int32_t whole_parts;       // prefix_parts, the own keys' part, and that of a prefix in the stream
    int64_t prefix_chunk;      // keys per part of prefix_kernel
    int64_t rows;              // R * Hq
    int64_t stream_tiles;      // at most
    int64_t workspace;         // bytes; in it: [whole_parts][rows] sums and [..][D] outputs, [warps][2][columns] sums
    int64_t sums_at, parts_at, piece_sums_at, pieces_at, before_at;  // and [..][D] outputs of pieces, [R + 5] words at `before`
};

// A prefix that adds at most so many tiles to each warp of the stream is left to it: prefix_kernel takes some 10 us
// to begin and end (128 requests of 32 heads behind 64 tokens 23 us against 33; behind 1000 35 against 74).
constexpr int kPrefixTiles = 4;
// Tiles that a warp of the stream takes at least: one alone is 2 us of latencies (4 requests of 342 tokens:
// 1, 2, 4 tiles 6.5, 8.6, 12.5 us in the stream, and 5.0, 4.8, 4.0 to join the pieces, by a profiler).
constexpr int kLeastShare = 2;
constexpr int kSms = 148;  // B200; the workspace must not depend on the device that happens to be current

// CTAs of stream_kernel that one SM holds, by shared memory and registers.  (D <= 64 with three: 512 requests of about 200
// tokens 58 us for 53 in e4m3, 63 for 60 in bf16.)
inline int stream_ctas(int64_t D, int columns)
{
    if (D > 128) return 1;
    if (columns > 8) return 2;
    return D > 64 ? 3 : 4;
}

inline void split_attn(int64_t R, int64_t Hq, int64_t H, int64_t D, int64_t max_len, int64_t max_prefix, bool quantised, AttnSplit *s)
{
    *s = AttnSplit{};
    s->group = static_cast<int32_t>(Hq / H);
    s->rows = R * Hq;
    s->columns = s->group <= 8 ? 8 : 16;
    s->own_blocks = (s->group + s->columns - 1) / s->columns;
    s->tile_keys = quantised ? 32 : 16;
    auto tiles_of = [&](int64_t keys) { return (keys + s->tile_keys - 1) / s->tile_keys; };
    const int64_t rows = R * s->group, warps = 4ll * kSms * stream_ctas(D, s->columns);  // rows of one KV head
    const bool alone = rows > 16 && D <= 128 && H * ((rows + s->columns - 1) / s->columns) * tiles_of(max_prefix) > kPrefixTiles * warps;
    s->prefix_rows = !alone ? 16 : rows <= 128 ? 128 : 256;
    const int64_t block = s->prefix_rows == 16 ? s->columns : s->prefix_rows;
    s->prefix_blocks = static_cast<int32_t>((rows + block - 1) / block);
    s->prefix_chunk = 128;
    if (s->prefix_rows > 16) {
        // One CTA per SM: the number of parts that costs least, counted in tiles (about 1.5 us; codes take half as long again, which
        // moved no case when it was counted).  The busiest SM's, with
        // four to start and end each part, and what writing the parts and reading them again in join_kernel
        // takes, at some 3 TB/s.  At most 64 parts, and 256 MB of them.
        const int64_t tiles = (max_prefix + 127) / 128, ctas = H * s->prefix_blocks, most = std::max<int64_t>(1, (128ll << 20) / (s->rows * (D + 1) * 4));
        const int slots = s->prefix_rows == 128 ? 2 : 1;
        int64_t best = 1;
        double best_cost = 1e300;
        for (int64_t n = 1; n <= std::min<int64_t>({tiles, 64, most}); n++) {
            const int64_t per = (tiles + n - 1) / n, parts = (tiles + per - 1) / per;
            const double cost = static_cast<double>((ctas * parts + kSms - 1) / kSms * ((per + slots - 1) / slots * slots + 4)) + static_cast<double>(parts * slots) * s->rows * D * 8 / 4.5e6;
            if (cost < best_cost) best = n, best_cost = cost;
        }
        const int64_t per = (tiles + best - 1) / best;
        s->prefix_chunk = per * 128;
        s->prefix_parts = static_cast<int32_t>((tiles + per - 1) / per) * (s->prefix_rows == 128 ? 2 : 1);
    }
    // The stream's warps: what the GPU holds at once, fewer where not even the longest batch would
    // give each its least share.
    const int64_t stream_tiles = R * H * s->own_blocks * tiles_of(max_len) + (s->prefix_rows == 16 ? H * s->prefix_blocks * tiles_of(max_prefix) : 0);
    s->stream_tiles = stream_tiles;
    const int64_t ctas = std::min<int64_t>(static_cast<int64_t>(kSms) * stream_ctas(D, s->columns), (stream_tiles + kLeastShare - 1) / kLeastShare);
    s->stream_ctas = static_cast<int32_t>(ctas);
    const int64_t whole = s->prefix_parts + (max_len > 0) + (max_prefix > 0 && s->prefix_rows == 16), pieces = ctas * 4 * 2 * s->columns;
    auto place = [&](int64_t bytes) {
        const int64_t at = s->workspace;
        s->workspace += (bytes + 255) / 256 * 256;
        return at;
    };
    s->whole_parts = static_cast<int32_t>(whole);
    s->sums_at = place(whole * s->rows * 4);
    s->parts_at = place(whole * s->rows * D * 4);
    s->piece_sums_at = place(pieces * 4);
    s->pieces_at = place(pieces * D * 4);
    s->before_at = place(ctas ? (R + 5) * 4 : 0);
}

}  // namespace tc
