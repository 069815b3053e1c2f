// How tc_attn_decode cuts its work: shared by the entry points and the kernels' launchers.
#pragma once

#include "ops.h"

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

struct AttnParams {
    Layer layer;
    const char *q;
    int64_t q_req, q_head;
    char *out;
    int64_t out_req, out_head;
    float *lse;
    const char *tables;
    int64_t table_width, table_stride;
    const int32_t *lens, *prefix_table, *prefix_len;
    int64_t R, max_len, max_prefix;
    int32_t Hq, q_bf16;
    float scale_log2;  // scale * log2(e)
    FastDiv div_block, div_group, div_heads;
    AttnSplit split;
    float *sums, *parts, *piece_sums, *pieces;
    uint32_t *before;  // {tiles, share, divider of the share}, then the tiles before each request and the prefix
    unsigned int *status;
};

// attn_decode.cu
void split_attn(int64_t R, int64_t Hq, int64_t H, int64_t D, int64_t max_len, int64_t max_prefix, bool quantised, AttnSplit *out);

// attn_prefix.cu: the prefix parts of splits whose prefix_rows is 128 or 256
int launch_prefix(const AttnParams &p, int dtype, int device, cudaStream_t s);

}  // namespace tc
