// The arguments of tc_attn_chunk's kernels: shared by the entry points and the kernels' launchers.
#pragma once

#include <cuda.h>

#include "attn.h"
#include "attn_chunk_split.h"
#include "ops.h"

namespace tc {

struct ChunkParams {
    Layer layer;
    const char *q;
    int64_t q_token, q_head;
    char *out;
    int64_t out_token, out_head;
    float *lse;
    const char *tables;
    int64_t table_stride;
    const int64_t *offsets;
    const int32_t *lens;
    int64_t R, n_tokens, max_new, max_len;
    int32_t Hq, q_bf16;
    int32_t no_singles;  // requests with one new token have their own kernels, launched before this one
    float scale_log2;    // scale * log2(e)
    FastDiv div_block, div_group;
    ChunkShape shape;
    ChunkPlan plan;
    uint2 *cuts;  // of every request that has items: the first of its parts' rows, and the number of its parts
    float *sums, *parts;
    unsigned int *status;
    // Where blocks and tiles fit into one another, pages are fetched as boxes of box_rows tokens of one head; 0: key by key.
    int32_t box_rows;
    FastDiv div_box;
    int32_t q_boxes;  // queries are fetched as boxes, too
    CUtensorMap map_k, map_v, map_q;
};
constexpr uint32_t kUncut = 0xffffffffu;

// attn_chunk.cu, attn_chunk_codes.cu: the items, of unquantised pools and of codes
int launch_chunk_plain(const ChunkParams &p, int dtype, int device, cudaStream_t s);
int launch_chunk_codes(const ChunkParams &p, int device, cudaStream_t s);

// Rows and tile that the kernels take for a head dim.
inline int32_t chunk_rows(int64_t D) { return D > 128 ? 128 : 256; }
inline int32_t chunk_keys(int64_t D) { return D > 128 ? 64 : 128; }

}  // namespace tc
