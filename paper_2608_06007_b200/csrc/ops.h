// What the operators on a paged layer (kv_append.cu, kv_gather.cu, attn_decode.cu) share: the
// checked description of a layer, and the checks of pointers and strides.
#pragma once

#include <cuda_runtime.h>

#include "exec.h"
#include "kv_index.h"

namespace tc {

constexpr unsigned int kStatusBadIndex = TC_DEVICE_BAD_INDEX;

// A layer whose geometry has been checked.
struct Layer {
    PlaneGeo geo, scale_geo;
    int64_t num_blocks;
    uint32_t B;
    int32_t H, D, dtype, esize;
    char *k, *v;
    float *k_scale, *v_scale;
    uint32_t align;  // of its planes and strides together, up to 32
    bool quantised() const { return dtype == TC_E4M3 || dtype == TC_INT8; }
};

// ---- ops_check.cpp
int dtype_size(int dtype);  // 0 for a number that is no tc_dtype
int check_layer(const tc_kv_layer_t *layer, Layer *out);
// [n][heads] rows of `row_bytes` at p with byte strides (outer, head): alignment of the element, and
// for an output that no two rows overlap.  *align is lowered to what address and strides share.
int check_rows(const char *name, const void *p, const int64_t stride[2], int64_t n, int64_t heads, int64_t row_bytes, int esize, bool output, uint32_t *align);

// Refuses what the current device cannot address: pageable host memory, another device's memory.
int check_memory(const char *name, const void *p, int device);
// ---- launch.cu
// The current device, its status word's address and its SM count (resolved once per device).
int op_device(int *device, unsigned int **status, int *sm_count);

}  // namespace tc
