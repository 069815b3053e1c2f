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

}  // namespace tc
