// tc_kv_gather: pages of a paged layer, quantised or not, into contiguous rows.
//
// A CTA takes a few consecutive output rows: one thread per row finds its request (bisection of
// the offsets) and its block, then every thread keeps one place (plane, head, unit of 32 output
// bytes) and steps from token to token, 128 bytes of loads in flight.  Bound by HBM: 98k tokens of 8 heads x
// 128 e4m3 to bf16 (554 MB) take 96 us, 5.8 TB/s, 0.88 of a plain copy; 149k tokens int8 to fp16 (900 MB)
// 147 us, 0.93.  (Two CTAs an SM instead of three: 102 and 156 us.  Units of 16 bytes stored from 8 codes,
// four loads in flight: 178 and 304 us.)
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
    uint32_t rows_per_cta, units, per_token;  // units of one (token, head) row, and of a token: planes * H * units
    uint32_t tokens_per_pass;                 // tokens that 256 threads cover at once
    FastDiv div_units, div_heads, div_token;  // by units, H and per_token
    int32_t planes, plane0;        // outputs asked for: 2, or 1 of which the first is plane0
    unsigned int *status;
};

template <int POOL> struct PoolType;
template <> struct PoolType<TC_BF16> { using type = __nv_bfloat16; };
template <> struct PoolType<TC_FP16> { using type = __half; };
template <> struct PoolType<TC_FP32> { using type = float; };

// N elements of the pool as floats (codes: before their scale).
template <int POOL, int N, int W>
__device__ __forceinline__ void widen_words(const Words<W> &v, float *x)
{
    if constexpr (POOL == TC_E4M3) {
#pragma unroll
        for (int i = 0; i < W; i++) {
            const float2 a = unpack2<__half>(e4m3_to_half2(v.w[i])), b = unpack2<__half>(e4m3_to_half2(v.w[i] >> 16));
            x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = b.x, x[4 * i + 3] = b.y;
        }
    } else if constexpr (POOL == TC_INT8) {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = static_cast<float>(static_cast<int8_t>(v.w[i / 4] >> (8 * (i % 4))));
    } else if constexpr (POOL == TC_FP32) {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = __uint_as_float(v.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < W; i++) {
            const float2 f = unpack2<typename PoolType<POOL>::type>(v.w[i]);
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
}
template <typename T, int N>
__device__ __forceinline__ Words<N * static_cast<int>(sizeof(T)) / 4> narrow_words(const float *x)
{
    Words<N * static_cast<int>(sizeof(T)) / 4> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; i++) r.w[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; i++) r.w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
    }
    return r;
}

// A unit is UNIT output bytes: 32, 16 or 8, or (0) one element at any alignment of the element.
template <int POOL, typename T, int UNIT>
__global__ void __launch_bounds__(256, 3) gather_kernel(const __grid_constant__ GatherParams p)
{
    constexpr bool quantised = POOL == TC_E4M3 || POOL == TC_INT8;
    constexpr int esize = POOL == TC_FP32 ? 4 : quantised ? 1 : 2;
    constexpr int N = UNIT ? UNIT / static_cast<int>(sizeof(T)) : 1;
    constexpr int W = UNIT ? N * esize / 4 : 1;
    constexpr int kUnroll = W <= 4 ? 8 : 4;  // 128 bytes in flight per thread
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
    // A thread keeps its place inside a token (plane, head, unit) and steps from token to token.
    const uint32_t ty = p.tokens_per_pass > 1 ? quick_div(threadIdx.x, p.div_token) : 0;
    if (ty >= p.tokens_per_pass) return;
    for (uint32_t x = threadIdx.x - ty * p.per_token; x < p.per_token; x += 256) {
        const uint32_t row = quick_div(x, p.div_units), unit = x - row * p.units;
        const uint32_t plane = quick_div(row, p.div_heads), h = row - plane * p.layer.H;
        const int c = p.plane0 + plane;
        const char *src = (c ? p.layer.v : p.layer.k) + static_cast<int64_t>(h) * p.layer.geo.head + unit * N * esize;
        const char *scales = reinterpret_cast<const char *>(c ? p.layer.v_scale : p.layer.k_scale) + static_cast<int64_t>(h) * p.layer.scale_geo.head;
        const int64_t stride = c ? p.row_stride[1] : p.row_stride[0];
        char *dst = (c ? p.out[1] : p.out[0]) + row0 * stride + h * (c ? p.head_stride[1] : p.head_stride[0]) + unit * N * static_cast<int>(sizeof(T));
        for (uint32_t t0 = ty; t0 < p.rows_per_cta; t0 += p.tokens_per_pass * kUnroll) {
            Words<W> v[kUnroll];
            float scale[kUnroll];
            bool there[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                const uint32_t t = t0 + u * p.tokens_per_pass;
                const int64_t at = t < p.rows_per_cta ? place[t] : -1;
                there[u] = at >= 0;
                scale[u] = 1.f;
                if (!there[u]) continue;
                if constexpr (UNIT != 0) v[u] = load_words<W>(src + at);
                else if constexpr (esize == 1) v[u].w[0] = *reinterpret_cast<const uint8_t *>(src + at);
                else if constexpr (esize == 2) v[u].w[0] = *reinterpret_cast<const uint16_t *>(src + at);
                else v[u].w[0] = *reinterpret_cast<const uint32_t *>(src + at);
                if constexpr (quantised) scale[u] = *reinterpret_cast<const float *>(scales + scale_place[t]);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                if (!there[u]) continue;
                float f[4 * W > N ? 4 * W : N];
                widen_words<POOL, N, W>(v[u], f);
                if constexpr (quantised)
#pragma unroll
                    for (int j = 0; j < N; j++) f[j] = __fmul_rn(f[j], scale[u]);
                char *to = dst + (t0 + u * p.tokens_per_pass) * stride;
                if constexpr (UNIT != 0) store_words(to, narrow_words<T, N>(f));
                else *reinterpret_cast<T *>(to) = from_float<T>(f[0]);
            }
        }
    }
}

template <int POOL, typename T>
static int launch_gather(GatherParams &p, int unit, int sms, cudaStream_t s)
{
    constexpr int widest = POOL == TC_FP32 && sizeof(T) == 2 ? 16 : 32;  // a unit reads at most 32 bytes of the pool
    unit = std::min(unit, widest);
    p.units = unit ? p.layer.D * static_cast<uint32_t>(sizeof(T)) / unit : p.layer.D;
    const int64_t per_token = static_cast<int64_t>(p.planes) * p.layer.H * p.units;
    if (per_token > INT32_MAX / 2) return fail(TC_ERR_TOO_LARGE, "H * D = %lld * %lld: a token's row is too large", (long long)p.layer.H, (long long)p.layer.D);
    // 32 rows a CTA, fewer where that would leave SMs without two CTAs
    const int64_t rows = std::max<int64_t>(1, std::min<int64_t>(kGatherRows, p.n_rows / (2 * sms)));
    p.rows_per_cta = static_cast<uint32_t>(rows);
    p.per_token = static_cast<uint32_t>(per_token);
    p.tokens_per_pass = std::max<uint32_t>(1, 256 / p.per_token);
    p.div_units = make_fastdiv(p.units);
    p.div_heads = make_fastdiv(static_cast<uint32_t>(p.layer.H));
    p.div_token = make_fastdiv(p.per_token);
    const int64_t grid = (p.n_rows + rows - 1) / rows;
    if (grid > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "n_rows %lld: too many for one call", (long long)p.n_rows);
    if constexpr (widest == 32)
        if (unit == 32) gather_kernel<POOL, T, 32><<<static_cast<unsigned>(grid), 256, 0, s>>>(p);
    if constexpr (sizeof(T) == 2)
        if (unit == 8) gather_kernel<POOL, T, 8><<<static_cast<unsigned>(grid), 256, 0, s>>>(p);
    if (unit == 16) gather_kernel<POOL, T, 16><<<static_cast<unsigned>(grid), 256, 0, s>>>(p);
    if (unit == 0) gather_kernel<POOL, T, 0><<<static_cast<unsigned>(grid), 256, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TC_OK : cuda_fail(e, "kernel launch");
}

template <int POOL>
static int launch_gather_to(GatherParams &p, int dtype, int unit, int sms, cudaStream_t s)
{
    switch (dtype) {
    case TC_BF16: return launch_gather<POOL, __nv_bfloat16>(p, unit, sms, s);
    case TC_FP16: return launch_gather<POOL, __half>(p, unit, sms, s);
    default: return launch_gather<POOL, float>(p, unit, sms, s);
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
    uint32_t align = 32;
    if (!a->k_out && !a->v_out) return fail(TC_ERR_INVALID_ARG, "k_out or v_out is required");
    if (a->k_out && (rc = check_rows("k_out", a->k_out, a->k_stride, a->n_rows, p.layer.H, int64_t(D) * e, e, true, &align)) != TC_OK) return rc;
    if (a->v_out && (rc = check_rows("v_out", a->v_out, a->v_stride, a->n_rows, p.layer.H, int64_t(D) * e, e, true, &align)) != TC_OK) return rc;
    if (a->k_out == a->v_out) return fail(TC_ERR_OVERLAP, "k_out is v_out: both planes would be written there");
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
    // Units of 32 output bytes where both sides are aligned to what one unit reads and writes in one
    // access, else of 16 or 8, else single elements.
    auto fits = [&](int unit) { return align >= static_cast<uint32_t>(unit) && D * e % unit == 0 && p.layer.align >= static_cast<uint32_t>(std::min(32, unit / e * p.layer.esize)); };
    const int unit = fits(32) ? 32 : fits(16) ? 16 : e == 2 && fits(8) ? 8 : 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (p.layer.dtype) {
    case TC_BF16: return launch_gather_to<TC_BF16>(p, a->dtype, unit, sms, s);
    case TC_FP16: return launch_gather_to<TC_FP16>(p, a->dtype, unit, sms, s);
    case TC_FP32: return launch_gather_to<TC_FP32>(p, a->dtype, unit, sms, s);
    case TC_E4M3: return launch_gather_to<TC_E4M3>(p, a->dtype, unit, sms, s);
    default: return launch_gather_to<TC_INT8>(p, a->dtype, unit, sms, s);
    }
}
