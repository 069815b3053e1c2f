// tc_kv_gather: pages of a paged layer, quantised or not, into contiguous rows.
//
// A CTA takes a few consecutive output rows: one thread per row finds its request (bisection of
// the offsets) and its block, then all threads walk the rows' units of 16 output bytes, in output
// order, each read as the 4 to 16 bytes of the pool that hold the same elements.  Bound by HBM.
#include "ops_device.cuh"

#include <algorithm>

namespace tc {

constexpr int kGatherRows = 32;  // most rows of a CTA

struct GatherParams {
    Layer layer;
    const char *tables;
    int64_t table_width, table_stride;
    const int64_t *offsets, *first;
    int64_t R, n_rows;
    char *out[2];
    int64_t row_stride[2], head_stride[2];
    int32_t rows_per_cta, units;   // units of one (token, head) row
    FastDiv div_units, div_heads, div_token;  // by units, H, and planes * H * units
    int32_t planes, plane0;        // outputs asked for: 2, or 1 of which the first is plane0
    unsigned int *status;
};

template <int POOL> struct PoolType;
template <> struct PoolType<TC_BF16> { using type = __nv_bfloat16; };
template <> struct PoolType<TC_FP16> { using type = __half; };
template <> struct PoolType<TC_FP32> { using type = float; };

// N elements of the pool at p as floats (codes: before their scale).
template <int POOL, int N>
__device__ __forceinline__ void load_codes(const char *p, float *x)
{
    if constexpr (POOL == TC_E4M3 || POOL == TC_INT8) {
        uint32_t w[N / 4];
        if constexpr (N == 8) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        }
#pragma unroll
        for (int i = 0; i < N / 4; i++) {
            if constexpr (POOL == TC_E4M3) {
                const float2 a = unpack2<__half>(e4m3_to_half2(w[i])), b = unpack2<__half>(e4m3_to_half2(w[i] >> 16));
                x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = b.x, x[4 * i + 3] = b.y;
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) x[4 * i + j] = static_cast<float>(static_cast<int8_t>(w[i] >> (8 * j)));
            }
        }
    } else {
        load_floats<typename PoolType<POOL>::type, N>(p, x);
    }
}

// VEC: units of 16 output bytes.  Otherwise a unit is one element, at any alignment of the element.
template <int POOL, typename T, bool VEC>
__global__ void __launch_bounds__(256) gather_kernel(const __grid_constant__ GatherParams p)
{
    constexpr int N = VEC ? 16 / static_cast<int>(sizeof(T)) : 1;
    constexpr int kUnroll = 4;
    constexpr bool quantised = POOL == TC_E4M3 || POOL == TC_INT8;
    constexpr int esize = POOL == TC_FP32 ? 4 : quantised ? 1 : 2;
    __shared__ int64_t place[kGatherRows], scale_place[kGatherRows];
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows_per_cta;
    if (threadIdx.x < p.rows_per_cta) {
        const int64_t row = row0 + threadIdx.x;
        int64_t at = -1, scale_at = 0;
        const int64_t r = row < p.n_rows ? request_of(p.offsets, p.R, row) : -1;
        if (r >= 0) {
            const int64_t t = row - p.offsets[r] + (p.first ? p.first[r] : 0);
            bool ok = t >= 0 && t <= INT32_MAX;
            if (ok) {
                uint32_t entry, n;
                token_place(static_cast<uint32_t>(t), p.layer.B, &entry, &n);
                ok = entry < p.table_width;
                if (ok) {
                    const int32_t block = reinterpret_cast<const int32_t *>(p.tables + r * p.table_stride)[entry];
                    ok = block >= 0 && block < p.layer.num_blocks;
                    at = ok ? p.layer.geo.at(block, n, 0) : -1;
                    scale_at = p.layer.scale_geo.at(block, n, 0);
                }
            }
            if (!ok) atomicOr(p.status, kStatusBadIndex);
        }
        if (row == p.n_rows - 1 && p.offsets[p.R] > p.n_rows) atomicOr(p.status, kStatusBadIndex);
        place[threadIdx.x] = at;
        scale_place[threadIdx.x] = scale_at;
    }
    __syncthreads();
    const uint32_t per_token = p.planes * p.layer.H * p.units, total = p.rows_per_cta * per_token;
    for (uint32_t i0 = threadIdx.x; i0 < total; i0 += 256 * kUnroll) {
        float x[kUnroll][N];
        float scale[kUnroll];
        char *dst[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const uint32_t i = i0 + 256 * u;
            dst[u] = nullptr;
            if (i >= total) continue;
            const uint32_t token = quick_div(i, p.div_token), rest = i - token * per_token;
            const uint32_t row = quick_div(rest, p.div_units), unit = rest - row * p.units;
            const uint32_t plane = quick_div(row, p.div_heads), h = row - plane * p.layer.H;
            const int64_t at = place[token];
            if (at < 0) continue;
            const int c = p.plane0 + plane;
            const char *src = (c ? p.layer.v : p.layer.k) + at + static_cast<int64_t>(h) * p.layer.geo.head + unit * N * esize;
            if constexpr (VEC) {
                load_codes<POOL, N>(src, x[u]);
            } else if constexpr (POOL == TC_E4M3) {
                x[u][0] = unpack2<__half>(e4m3_to_half2(*reinterpret_cast<const uint8_t *>(src))).x;
            } else if constexpr (POOL == TC_INT8) {
                x[u][0] = static_cast<float>(*reinterpret_cast<const int8_t *>(src));
            } else {
                x[u][0] = to_float(*reinterpret_cast<const typename PoolType<POOL>::type *>(src));
            }
            if constexpr (quantised)
                scale[u] = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(c ? p.layer.v_scale : p.layer.k_scale) + scale_place[token] + static_cast<int64_t>(h) * p.layer.scale_geo.head);
            dst[u] = (c ? p.out[1] : p.out[0]) + (row0 + token) * (c ? p.row_stride[1] : p.row_stride[0]) + h * (c ? p.head_stride[1] : p.head_stride[0]) + unit * N * static_cast<int>(sizeof(T));
        }
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            if (!dst[u]) continue;
            if constexpr (quantised)
#pragma unroll
                for (int j = 0; j < N; j++) x[u][j] = __fmul_rn(x[u][j], scale[u]);
            if constexpr (VEC) store_floats<T, N>(dst[u], x[u]);
            else *reinterpret_cast<T *>(dst[u]) = from_float<T>(x[u][0]);
        }
    }
}

template <int POOL, typename T>
static int launch_gather(GatherParams &p, bool vector, int sms, cudaStream_t s)
{
    p.units = vector ? p.layer.D * static_cast<int>(sizeof(T)) / 16 : p.layer.D;
    const int64_t per_token = static_cast<int64_t>(p.planes) * p.layer.H * p.units;
    if (per_token * kGatherRows > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "H * D = %lld * %lld: a token's row is too large", (long long)p.layer.H, (long long)p.layer.D);
    // eight units a thread, fewer where that would leave SMs without a CTA
    int64_t rows = std::max<int64_t>(1, std::min<int64_t>(kGatherRows, 2048 / std::max<int64_t>(per_token, 1)));
    rows = std::max<int64_t>(1, std::min(rows, p.n_rows / (2 * sms)));
    p.rows_per_cta = static_cast<int32_t>(rows);
    p.div_units = make_fastdiv(static_cast<uint32_t>(p.units));
    p.div_heads = make_fastdiv(static_cast<uint32_t>(p.layer.H));
    p.div_token = make_fastdiv(static_cast<uint32_t>(per_token));
    const int64_t grid = (p.n_rows + rows - 1) / rows;
    if (grid > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "n_rows %lld: too many for one call", (long long)p.n_rows);
    if (vector) gather_kernel<POOL, T, true><<<static_cast<unsigned>(grid), 256, 0, s>>>(p);
    else gather_kernel<POOL, T, false><<<static_cast<unsigned>(grid), 256, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TC_OK : cuda_fail(e, "kernel launch");
}

template <int POOL>
static int launch_gather_to(GatherParams &p, int dtype, bool vector, int sms, cudaStream_t s)
{
    switch (dtype) {
    case TC_BF16: return launch_gather<POOL, __nv_bfloat16>(p, vector, sms, s);
    case TC_FP16: return launch_gather<POOL, __half>(p, vector, sms, s);
    default: return launch_gather<POOL, float>(p, vector, sms, s);
    }
}

}  // namespace tc

using namespace tc;

extern "C" int tc_kv_gather(const tc_kv_layer_t *layer, const tc_kv_gather_t *a, void *stream)
{
    clear_error();
    GatherParams p{};
    int rc = check_layer(layer, &p.layer);
    if (rc != TC_OK) return rc;
    if (!a) return fail(TC_ERR_INVALID_ARG, "args is required");
    if (a->struct_size != sizeof *a) return fail(TC_ERR_INVALID_ARG, "args.struct_size %u != %zu: header and library disagree", a->struct_size, sizeof *a);
    if (a->dtype != TC_BF16 && a->dtype != TC_FP16 && a->dtype != TC_FP32) return fail(TC_ERR_INVALID_ARG, "dtype %d: k_out and v_out are TC_BF16, TC_FP16 or TC_FP32", a->dtype);
    if (a->R < 0 || a->n_rows < 0) return fail(TC_ERR_SHAPE, "R %lld and n_rows %lld must be >= 0", (long long)a->R, (long long)a->n_rows);
    if (a->R == 0 || a->n_rows == 0) return TC_OK;
    const int e = dtype_size(a->dtype), D = p.layer.D;
    uint32_t align = 16;
    if (!a->k_out && !a->v_out) return fail(TC_ERR_INVALID_ARG, "k_out or v_out is required");
    if (a->k_out && (rc = check_rows("k_out", a->k_out, a->k_stride, a->n_rows, p.layer.H, int64_t(D) * e, e, true, &align)) != TC_OK) return rc;
    if (a->v_out && (rc = check_rows("v_out", a->v_out, a->v_stride, a->n_rows, p.layer.H, int64_t(D) * e, e, true, &align)) != TC_OK) return rc;
    if (a->table_width < 1) return fail(TC_ERR_SHAPE, "table_width %lld < 1", (long long)a->table_width);
    if (a->table_stride < 0 || a->table_stride % 4 || reinterpret_cast<uintptr_t>(a->tables) % 4) return fail(TC_ERR_INVALID_ARG, "tables and table_stride must be multiples of 4 bytes");
    if (!a->tables || !a->offsets) return fail(TC_ERR_INVALID_ARG, "tables and offsets are required");
    if ((reinterpret_cast<uintptr_t>(a->offsets) | reinterpret_cast<uintptr_t>(a->first)) % 8) return fail(TC_ERR_INVALID_ARG, "offsets and first must be 8-byte aligned");
    int device, sms;
    if ((rc = op_device(&device, &p.status, &sms)) != TC_OK) return rc;
    const struct {
        const char *name;
        const void *p;
    } pointers[] = {{"layer.k", layer->k}, {"layer.v", layer->v}, {"layer.k_scale", layer->k_scale}, {"layer.v_scale", layer->v_scale},
                    {"tables", a->tables}, {"offsets", a->offsets}, {"first", a->first}, {"k_out", a->k_out}, {"v_out", a->v_out}};
    for (const auto &ptr : pointers)
        if (ptr.p && (rc = check_memory(ptr.name, ptr.p, device)) != TC_OK) return rc;
    p.tables = reinterpret_cast<const char *>(a->tables);
    p.table_width = a->table_width, p.table_stride = a->table_stride;
    p.offsets = a->offsets, p.first = a->first;
    p.R = a->R, p.n_rows = a->n_rows;
    p.out[0] = static_cast<char *>(a->k_out), p.out[1] = static_cast<char *>(a->v_out);
    for (int i = 0; i < 2; i++) {
        p.row_stride[i] = i ? a->v_stride[0] : a->k_stride[0];
        p.head_stride[i] = i ? a->v_stride[1] : a->k_stride[1];
    }
    p.planes = (a->k_out != nullptr) + (a->v_out != nullptr);
    p.plane0 = a->k_out ? 0 : 1;
    // a unit's 16 output bytes come from 16 / e elements of the pool
    const bool vector = align >= 16 && D % (16 / e) == 0 && p.layer.align >= std::min<uint32_t>(16, 16u / e * p.layer.esize);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (p.layer.dtype) {
    case TC_BF16: return launch_gather_to<TC_BF16>(p, a->dtype, vector, sms, s);
    case TC_FP16: return launch_gather_to<TC_FP16>(p, a->dtype, vector, sms, s);
    case TC_FP32: return launch_gather_to<TC_FP32>(p, a->dtype, vector, sms, s);
    case TC_E4M3: return launch_gather_to<TC_E4M3>(p, a->dtype, vector, sms, s);
    default: return launch_gather_to<TC_INT8>(p, a->dtype, vector, sms, s);
    }
}
