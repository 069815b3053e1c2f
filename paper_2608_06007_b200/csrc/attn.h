// The arguments of tc_attn_decode's kernels: shared by the entry points and the kernels' launchers.
#pragma once

#include "attn_split.h"
#include "ops.h"

namespace tc {

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
    int32_t window, sinks;  // keys at the end, and at the front, that a row sees; window 0: all
    // kSingles: a request's row of q, out and lse is offsets[r], where offsets[r + 1] is one more; elsewhere it has no part in the call
    const int64_t *offsets;
    int64_t n_tokens, max_new;
    int32_t Hq, q_bf16;
    float scale_log2;  // scale * log2(e)
    FastDiv div_block, div_group, div_heads;
    AttnSplit split;
    float *sums, *parts, *piece_sums, *pieces;
    uint32_t *before;  // {tiles, share, divider of the share}, then the tiles before each request and the prefix
    unsigned int *status;
};

// attn_prefix.cu: the prefix parts of splits whose prefix_rows is 128 or 256
int launch_prefix(const AttnParams &p, int dtype, int device, cudaStream_t s);
// attn_window.cu: a call with a window
int launch_window(const AttnParams &p, int dtype, int device, cudaStream_t s);
// attn_singles.cu: the requests of a tc_attn_chunk call that have one new token; the stream, and then, behind whatever was launched after it, the join
int launch_singles_stream(const AttnParams &p, int dtype, int device, cudaStream_t s);
int launch_singles_join(const AttnParams &p, int dtype, cudaStream_t s);

}  // namespace tc
