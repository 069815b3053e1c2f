// tc_attn_decode: one query token per request over a shared prefix and the request's own pages.
//
// The keys of a row (request, head) are cut into parts, each of which leaves the softmax-weighted mean of its
// values and log2 of its sum in the workspace; join_kernel weighs the parts against one another.
// prefix_kernel (attn_prefix.cu) takes a prefix that many rows share, stream_kernel all other keys.
// Softmax statistics, scores and outputs are fp32 throughout; only the probabilities are rounded, to 16
// bits, to enter the second matrix product (half a step of 2^-8 or 2^-11 relative to each, no worse than
// the rounding of the values and of the output to those types; in fp16 so down to 2^-21 of the largest, and by at most
// 2^-32 of it below that).
#include <cmath>

#include "attn_stream.cuh"

namespace tc {

template <typename T>
static int launch_decode(const AttnParams &p, int device, cudaStream_t s)
{
    const int rc = p.split.prefix_parts ? launch_prefix(p, std::is_same<T, __half>::value ? TC_FP16 : TC_BF16, device, s) : TC_OK;
    return rc != TC_OK ? rc : launch_stream_and_join<T, kAllKeys>(p, device, s);
}

// What both entry points check; fills p's geometry and split.
static int check_decode(const tc_kv_layer_t *layer, const tc_attn_decode_t *a, AttnParams *p, int64_t window = 0, int64_t sinks = 0)
{
    int rc = check_layer(layer, &p->layer);
    if (rc != TC_OK) return rc;
    if (!a) return fail(TC_ERR_INVALID_ARG, "args is required");
    if (a->struct_size != sizeof *a) return fail(TC_ERR_INVALID_ARG, "args.struct_size %u != %zu: header and library disagree", a->struct_size, sizeof *a);
    if (a->dtype != TC_BF16 && a->dtype != TC_FP16) return fail(TC_ERR_INVALID_ARG, "dtype %d: q and out are TC_BF16 or TC_FP16", a->dtype);
    if (!p->layer.quantised() && p->layer.dtype != a->dtype) return fail(TC_ERR_INVALID_ARG, "an unquantised pool must have the queries' dtype (pool %d, queries %d)", p->layer.dtype, a->dtype);
    const int D = p->layer.D;
    if (D % 16 || D > 256) return fail(TC_ERR_SHAPE, "D = %d: tc_attn_decode takes multiples of 16 up to 256", D);
    if (p->layer.align < 16) return fail(TC_ERR_INVALID_ARG, "tc_attn_decode needs planes and strides that are multiples of 16 bytes");
    if (a->R < 0 || a->R > (1 << 24)) return fail(TC_ERR_SHAPE, "R %lld is not in [0, 2^24]", (long long)a->R);
    if (a->Hq < 1 || a->Hq > (1 << 16) || a->Hq % p->layer.H) return fail(TC_ERR_SHAPE, "Hq %lld is not a multiple of H = %d in [1, 2^16]", (long long)a->Hq, p->layer.H);
    if (a->R * a->Hq > (1 << 30)) return fail(TC_ERR_TOO_LARGE, "R * Hq = %lld rows: too many for one call", (long long)(a->R * a->Hq));
    if (a->max_len < 0 || a->max_len > INT32_MAX - 4096 || a->max_prefix < 0 || a->max_prefix > INT32_MAX - 4096)
        return fail(TC_ERR_SHAPE, "max_len %lld and max_prefix %lld must be in [0, 2^31 - 4096)", (long long)a->max_len, (long long)a->max_prefix);
    if (a->reserved) return fail(TC_ERR_INVALID_ARG, "reserved is %d, not 0", a->reserved);
    if (!(std::fabs(a->scale) <= 1e30f)) return fail(TC_ERR_INVALID_ARG, "scale is not a number of at most 1e30");
    // keys in the tiles that a request has at most: with a window, its own and those of the first tokens, each up to a tile more at either end
    const int64_t most = window ? std::min(a->max_len, std::min(window, a->max_len) + std::min(sinks, a->max_len) + 96) : a->max_len;
    if (a->R * p->layer.H > (1 << 30) / std::max<int64_t>(1, (most + 15) / 16)) return fail(TC_ERR_TOO_LARGE, "R * H * keys = %lld * %d * %lld: too many keys for one call", (long long)a->R, p->layer.H, (long long)most);
    split_attn(a->R, a->Hq, p->layer.H, D, most, a->max_prefix, p->layer.quantised(), &p->split);
    if (p->split.stream_tiles >= (1ll << 31)) return fail(TC_ERR_TOO_LARGE, "%lld tiles of 16 keys: too many for one call", (long long)p->split.stream_tiles);
    return TC_OK;
}

}  // namespace tc

using namespace tc;

extern "C" int tc_attn_workspace(const tc_kv_layer_t *layer, const tc_attn_decode_t *a, int64_t *bytes)
{
    clear_error();
    if (!bytes) return fail(TC_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    AttnParams p{};
    const int rc = check_decode(layer, a, &p);
    if (rc == TC_OK) *bytes = p.split.workspace;
    return rc;
}

// window 0: tc_attn_decode
static int decode(const tc_kv_layer_t *layer, const tc_attn_decode_t *a, int64_t window, int64_t sinks, void *stream)
{
    AttnParams p{};
    int rc = check_decode(layer, a, &p, window, sinks);
    if (rc != TC_OK) return rc;
    p.window = static_cast<int32_t>(std::min<int64_t>(window, INT32_MAX)), p.sinks = static_cast<int32_t>(std::min<int64_t>(sinks, INT32_MAX));
    if (a->R == 0) return TC_OK;
    uint32_t align = 16;
    const int64_t row = p.layer.D * 2ll;
    if ((rc = check_rows("q", a->q, a->q_stride, a->R, a->Hq, row, 2, false, &align)) != TC_OK) return rc;
    if ((rc = check_rows("out", a->out, a->out_stride, a->R, a->Hq, row, 2, true, &align)) != TC_OK) return rc;
    if (align < 16) return fail(TC_ERR_INVALID_ARG, "q, out and their strides must be multiples of 16 bytes");
    if (a->q == a->out) return fail(TC_ERR_OVERLAP, "out is q: the queries are read after the first outputs are written");
    if (reinterpret_cast<uintptr_t>(a->lse) % 4) return fail(TC_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    if (!a->lens || reinterpret_cast<uintptr_t>(a->lens) % 4) return fail(TC_ERR_INVALID_ARG, "lens is required, 4-byte aligned");
    if (a->max_len) {
        if (!a->tables || reinterpret_cast<uintptr_t>(a->tables) % 4 || a->table_stride % 4 || a->table_stride < 0)
            return fail(TC_ERR_INVALID_ARG, "tables is required with max_len > 0; address and table_stride are multiples of 4 bytes");
        if (a->table_width < (a->max_len + p.layer.B - 1) / p.layer.B)
            return fail(TC_ERR_BOUNDS, "table_width %lld holds %lld tokens, max_len is %lld", (long long)a->table_width, (long long)(a->table_width * p.layer.B), (long long)a->max_len);
    }
    if (a->max_prefix && (!a->prefix_table || !a->prefix_len || (reinterpret_cast<uintptr_t>(a->prefix_table) | reinterpret_cast<uintptr_t>(a->prefix_len)) % 4))
        return fail(TC_ERR_INVALID_ARG, "prefix_table and prefix_len are required with max_prefix > 0, 4-byte aligned");
    if (p.split.workspace && (!a->workspace || reinterpret_cast<uintptr_t>(a->workspace) % 16))
        return fail(TC_ERR_INVALID_ARG, "workspace is required, 16-byte aligned");
    if (a->workspace_bytes < p.split.workspace)
        return fail(TC_ERR_BOUNDS, "workspace_bytes %lld < %lld (tc_attn_workspace)", (long long)a->workspace_bytes, (long long)p.split.workspace);
    int device, sms;
    if ((rc = op_device(&device, &p.status, &sms)) != TC_OK) return rc;
    const struct {
        const char *name;
        const void *p;
    } pointers[] = {{"layer.k", layer->k}, {"layer.v", layer->v}, {"layer.k_scale", layer->k_scale}, {"layer.v_scale", layer->v_scale}, {"q", a->q}, {"out", a->out},
                    {"lse", a->lse}, {"lens", a->lens}, {"tables", a->max_len ? a->tables : nullptr}, {"prefix_table", a->max_prefix ? a->prefix_table : nullptr},
                    {"prefix_len", a->max_prefix ? a->prefix_len : nullptr}, {"workspace", p.split.workspace ? a->workspace : nullptr}};
    for (const auto &ptr : pointers)
        if (ptr.p && (rc = check_memory(ptr.name, ptr.p, device)) != TC_OK) return rc;
    p.q = static_cast<const char *>(a->q);
    p.q_req = a->q_stride[0], p.q_head = a->q_stride[1];
    p.out = static_cast<char *>(a->out);
    p.out_req = a->out_stride[0], p.out_head = a->out_stride[1];
    p.lse = a->lse;
    p.tables = reinterpret_cast<const char *>(a->tables);
    p.table_width = a->table_width, p.table_stride = a->table_stride;
    p.lens = a->lens, p.prefix_table = a->prefix_table, p.prefix_len = a->prefix_len;
    p.R = a->R, p.max_len = a->max_len, p.max_prefix = a->max_prefix;
    p.Hq = static_cast<int32_t>(a->Hq);
    p.q_bf16 = a->dtype == TC_BF16;
    p.scale_log2 = static_cast<float>((a->scale != 0.f ? static_cast<double>(a->scale) : 1.0 / std::sqrt(static_cast<double>(p.layer.D))) * 1.4426950408889634);
    p.div_block = make_fastdiv(p.layer.B);
    p.div_group = make_fastdiv(static_cast<uint32_t>(p.split.group));
    p.div_heads = make_fastdiv(static_cast<uint32_t>(p.Hq));
    char *const ws = static_cast<char *>(a->workspace);
    p.sums = reinterpret_cast<float *>(ws + p.split.sums_at);
    p.parts = reinterpret_cast<float *>(ws + p.split.parts_at);
    p.piece_sums = reinterpret_cast<float *>(ws + p.split.piece_sums_at);
    p.pieces = reinterpret_cast<float *>(ws + p.split.pieces_at);
    p.before = reinterpret_cast<uint32_t *>(ws + p.split.before_at);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (window) return launch_window(p, a->dtype, device, s);
    return a->dtype == TC_BF16 ? launch_decode<__nv_bfloat16>(p, device, s) : launch_decode<__half>(p, device, s);
}

extern "C" int tc_attn_decode(const tc_kv_layer_t *layer, const tc_attn_decode_t *a, void *stream)
{
    clear_error();
    return decode(layer, a, 0, 0, stream);
}

extern "C" int tc_attn_decode_window(const tc_kv_layer_t *layer, const tc_attn_decode_t *a, int64_t window, int64_t sinks, void *stream)
{
    clear_error();
    if (window < 1 || sinks < 0) return fail(TC_ERR_SHAPE, "window %lld must be positive and sinks %lld not negative", (long long)window, (long long)sinks);
    if (a && a->struct_size == sizeof *a && a->max_prefix) return fail(TC_ERR_INVALID_ARG, "max_prefix is %lld: with a window there is no shared prefix", (long long)a->max_prefix);
    return decode(layer, a, window, sinks, stream);
}
