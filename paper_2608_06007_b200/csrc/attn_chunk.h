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
    int64_t new_from, new_to;  // requests with so many new tokens are this kernel's; others have their own, in the same call
    uint32_t item_spins;       // of waits that may last as long as an item of all the keys there may be
    bool beside;               // launched behind a kernel of the same call that it need not wait for, but for its own end
    float scale_log2;    // scale * log2(e)
    FastDiv div_block, div_group;
    ChunkShape shape;
    ChunkPlan plan;
    uint2 *cuts;  // of every request that has items: the first of its parts' rows, and the number of its parts
    float *sums, *parts;
    uint32_t first_part_row;  // of this kernel's among the call's, which `cuts` counts
    unsigned int *status;
    // Where blocks and tiles fit into one another, pages are fetched as boxes of box_rows tokens of one head; 0: key by key.
    int32_t box_rows;
    FastDiv div_box;
    int32_t q_boxes;  // queries are fetched as boxes, too
    CUtensorMap map_k, map_v, map_q;
    // Codes' tiles that are made fp16 before: wide_list places a request, H tiles a place.  A request's places are the r-th, or where
    // there may be more requests than room the (token0 / new_from)-th: no two of new_from tokens or more have the same.
    char *wide;
    int32_t wide_list, wide_by_request;
    int64_t wide_requests;  // that there is room for
    FastDiv div_wide;
    bool widen_beside;  // the kernel that makes them is launched as `beside` says
};
constexpr uint32_t kUncut = 0xffffffffu;

// attn_chunk.cu, attn_chunk_codes.cu, attn_chunk_wide.cu: the items, of unquantised pools, of codes, and of codes that were made fp16 before
int launch_chunk_plain(const ChunkParams &p, int dtype, int device, cudaStream_t s);
int launch_chunk_codes(const ChunkParams &p, int device, cudaStream_t s);
int launch_chunk_wide(const ChunkParams &p, int device, cudaStream_t s);

// A tile that was made fp16: K and V as the products read them; K's scales, V's exponents and the rest of V's scales of the keys; {mask, 4 words; V's exponent;
// whether scales are far apart; whether V has numbers that are not finite}.
template <int DP> struct WideTile {
    static constexpr int keys = DP > 128 ? 64 : 128, tile = keys * DP * 2;
    static constexpr int64_t scales_at = 2 * tile, header_at = scales_at + 12 * keys, bytes = header_at + 128;
};
inline int64_t wide_tile_bytes(int64_t D) { return D <= 64 ? WideTile<64>::bytes : D <= 128 ? WideTile<128>::bytes : WideTile<256>::bytes; }

// Rows and tile that the kernels take for a head dim.
inline int32_t chunk_rows(int64_t D) { return D > 128 ? 128 : 256; }
inline int32_t chunk_keys(int64_t D) { return D > 128 ? 64 : 128; }

}  // namespace tc
