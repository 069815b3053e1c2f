// Host-side checks of the operators on a paged layer.  No CUDA call here except at the end of the
// file, where pointers are looked up.
#include "ops.h"

#include <algorithm>

namespace tc {

int dtype_size(int dtype)
{
    switch (dtype) {
    case TC_BF16: case TC_FP16: return 2;
    case TC_FP32: return 4;
    case TC_E4M3: case TC_INT8: return 1;
    default: return 0;
    }
}

static uint32_t low_bit(uint64_t v) { return v ? static_cast<uint32_t>(std::min<uint64_t>(v & -v, 32)) : 32u; }

// One plane's strides for rows of `row` bytes; block_stride 0 = tight.
static int plane_geo(const char *name, const tc_kv_pool_t &p, int64_t B, int64_t H, int64_t row, PlaneGeo *out)
{
    if (p.layout != TC_NHD && p.layout != TC_HND) return fail(TC_ERR_INVALID_ARG, "%s.layout %d is not a tc_layout", name, p.layout);
    if (p.num_blocks < 0 || p.num_blocks > INT32_MAX) return fail(TC_ERR_SHAPE, "%s.num_blocks %lld is not in [0, 2^31)", name, (long long)p.num_blocks);
    const __int128 chunk = static_cast<__int128>(B) * H * row;
    if (chunk > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "%s: a block of %lld tokens x %lld heads x %lld bytes is 2 GiB or more", name, (long long)B, (long long)H, (long long)row);
    const int64_t bs = p.block_stride ? p.block_stride : static_cast<int64_t>(chunk);
    if (bs < chunk) return fail(TC_ERR_OVERLAP, "%s.block_stride %lld < block bytes %lld: blocks overlap", name, (long long)bs, (long long)chunk);
    if (static_cast<__int128>(bs) * std::max<int64_t>(p.num_blocks, 1) > (static_cast<__int128>(1) << 56))
        return fail(TC_ERR_TOO_LARGE, "%s: %lld blocks of stride %lld exceed the address space", name, (long long)p.num_blocks, (long long)bs);
    out->block = bs;
    out->token = static_cast<int32_t>(p.layout == TC_NHD ? H * row : row);
    out->head = static_cast<int32_t>(p.layout == TC_NHD ? row : B * row);
    return TC_OK;
}

int check_layer(const tc_kv_layer_t *layer, Layer *out)
{
    if (!layer) return fail(TC_ERR_INVALID_ARG, "layer is required");
    if (layer->struct_size != sizeof *layer) return fail(TC_ERR_INVALID_ARG, "layer.struct_size %u != %zu: header and library disagree", layer->struct_size, sizeof *layer);
    const int esize = dtype_size(layer->dtype);
    if (!esize) return fail(TC_ERR_INVALID_ARG, "layer.dtype %d is not a tc_dtype", layer->dtype);
    for (int64_t n : {layer->B, layer->H, layer->D})
        if (n < 1 || n > (1 << 24)) return fail(TC_ERR_SHAPE, "B, H, D = %lld, %lld, %lld: each must be in [1, 2^24]", (long long)layer->B, (long long)layer->H, (long long)layer->D);
    int rc = plane_geo("pool", layer->pool, layer->B, layer->H, layer->D * esize, &out->geo);
    if (rc != TC_OK) return rc;
    const bool quantised = layer->dtype == TC_E4M3 || layer->dtype == TC_INT8;
    if (quantised) {
        if ((rc = plane_geo("scale_pool", layer->scale_pool, layer->B, layer->H, 4, &out->scale_geo)) != TC_OK) return rc;
        if (layer->scale_pool.num_blocks < layer->pool.num_blocks)
            return fail(TC_ERR_BOUNDS, "scale_pool.num_blocks %lld < pool.num_blocks %lld", (long long)layer->scale_pool.num_blocks, (long long)layer->pool.num_blocks);
        if (!layer->k_scale || !layer->v_scale) return fail(TC_ERR_INVALID_ARG, "a quantised pool needs k_scale and v_scale");
        if ((reinterpret_cast<uintptr_t>(layer->k_scale) | reinterpret_cast<uintptr_t>(layer->v_scale) | static_cast<uintptr_t>(out->scale_geo.block)) & 3)
            return fail(TC_ERR_INVALID_ARG, "the scale planes and their block_stride must be multiples of 4 bytes");
    } else {
        if (layer->k_scale || layer->v_scale) return fail(TC_ERR_INVALID_ARG, "k_scale / v_scale given for a pool that is not quantised");
        out->scale_geo = PlaneGeo{0, 0, 0};
    }
    if (!layer->k || !layer->v) return fail(TC_ERR_INVALID_ARG, "layer.k and layer.v are required");
    const uint32_t align = std::min({low_bit(reinterpret_cast<uintptr_t>(layer->k)), low_bit(reinterpret_cast<uintptr_t>(layer->v)), low_bit(out->geo.block),
                                     low_bit(out->geo.token), low_bit(out->geo.head)});
    if (align < static_cast<uint32_t>(esize)) return fail(TC_ERR_INVALID_ARG, "the pool's planes and block_stride must be multiples of the element's %d bytes", esize);
    out->num_blocks = layer->pool.num_blocks;
    out->B = static_cast<uint32_t>(layer->B);
    out->H = static_cast<int32_t>(layer->H);
    out->D = static_cast<int32_t>(layer->D);
    out->dtype = layer->dtype;
    out->esize = esize;
    out->k = static_cast<char *>(layer->k);
    out->v = static_cast<char *>(layer->v);
    out->k_scale = static_cast<float *>(layer->k_scale);
    out->v_scale = static_cast<float *>(layer->v_scale);
    out->align = align;
    return TC_OK;
}

int check_rows(const char *name, const void *p, const int64_t stride[2], int64_t n, int64_t heads, int64_t row_bytes, int esize, bool output, uint32_t *align)
{
    if (!p) return fail(TC_ERR_INVALID_ARG, "%s is required", name);
    for (int i = 0; i < 2; i++)
        if (stride[i] < 0 || stride[i] > (1ll << 48)) return fail(TC_ERR_SHAPE, "%s_stride[%d] = %lld is not in [0, 2^48]", name, i, (long long)stride[i]);
    // a stride that is never taken does not count
    const int64_t outer = n > 1 ? stride[0] : 0, head = heads > 1 ? stride[1] : 0;
    const uint32_t a = std::min({low_bit(reinterpret_cast<uintptr_t>(p)), low_bit(static_cast<uint64_t>(outer)), low_bit(static_cast<uint64_t>(head))});
    if (a < static_cast<uint32_t>(esize)) return fail(TC_ERR_INVALID_ARG, "%s: address and strides must be multiples of the element's %d bytes", name, esize);
    if (output) {
        const bool heads_inside = (heads == 1 || head >= row_bytes) && (n == 1 || static_cast<__int128>(outer) >= static_cast<__int128>(heads - 1) * head + row_bytes);
        const bool tokens_inside = (n == 1 || outer >= row_bytes) && (heads == 1 || static_cast<__int128>(head) >= static_cast<__int128>(n - 1) * outer + row_bytes);
        if (!heads_inside && !tokens_inside) return fail(TC_ERR_OVERLAP, "%s: strides %lld and %lld make rows of %lld bytes overlap", name, (long long)stride[0], (long long)stride[1], (long long)row_bytes);
    }
    *align = std::min(*align, a);
    return TC_OK;
}

int check_memory(const char *name, const void *p, int device)
{
    cudaPointerAttributes attr;
    if (cudaPointerGetAttributes(&attr, p) != cudaSuccess) {
        cudaGetLastError();
        return fail(TC_ERR_INVALID_ARG, "%s (%p) is not a valid address for this device", name, p);
    }
    if (attr.type == cudaMemoryTypeUnregistered)
        return fail(TC_ERR_INVALID_ARG, "%s (%p) is pageable host memory: pin it (cudaHostAlloc / cudaHostRegister) or use device memory", name, p);
    if (attr.type == cudaMemoryTypeDevice && attr.device != device)
        return fail(TC_ERR_INVALID_ARG, "%s (%p) is memory of device %d but device %d is current", name, p, attr.device, device);
    return TC_OK;
}

}  // namespace tc
