// tc_kv_append: rotary positions, quantisation and the scatter into a paged layer, in one pass.
//
// A row is one (token, head) of D numbers.  Its elements come in pairs of 8-element chunks (a, b)
// chosen so that a rotation's partners are in one thread: b = a + rot_dim/2 for the half layout,
// neighbours for the interleaved one and for what is not rotated.  2^k lanes hold a row, so the
// row's largest magnitude is k shuffles away and every number is read once and written once.  The
// threads of one token share its table row in registers over all of its heads.  Bound by HBM.
//
// Products and sums are rounded one by one (no FMA) and the divisions are IEEE, so that the codes are the
// same bits as elementary fp32 operations give: a value next to a rounding border does not depend on
// which kernel wrote it.
#include "ops_device.cuh"

#include <algorithm>

namespace tc {

struct AppendParams {
    Layer layer;
    const char *q, *k, *v;
    char *q_out;
    int64_t q_tok, q_head, o_tok, o_head, k_tok, k_head, v_tok, v_head;
    const int64_t *slots, *positions;
    const char *cos, *sin;
    int64_t n_positions, table_stride;
    int64_t n_tokens;
    int32_t Hq, rot, interleaved;
    int32_t log2_lanes;        // lanes of a row (vector kernel)
    int32_t threads_per_token; // a power of two, 32..256
    unsigned int *status;
};

struct RowPlace {
    const char *src;
    char *dst;
    float *scale;
    bool turn, pool;
};

// Row `row` of a token: H rows of K, H of V, Hq of Q.
__device__ __forceinline__ RowPlace row_place(const AppendParams &p, int row, int64_t token, int64_t block, int32_t n)
{
    RowPlace r;
    const int H = p.layer.H;
    if (row < 2 * H) {
        const bool is_v = row >= H;
        const int h = is_v ? row - H : row;
        r.src = is_v ? p.v + token * p.v_tok + h * p.v_head : p.k + token * p.k_tok + h * p.k_head;
        r.dst = (is_v ? p.layer.v : p.layer.k) + p.layer.geo.at(block, n, h);
        r.scale = p.layer.k_scale ? reinterpret_cast<float *>(reinterpret_cast<char *>(is_v ? p.layer.v_scale : p.layer.k_scale) + p.layer.scale_geo.at(block, n, h)) : nullptr;
        r.turn = !is_v;
        r.pool = true;
    } else {
        const int h = row - 2 * H;
        r.src = p.q + token * p.q_tok + h * p.q_head;
        r.dst = p.q_out + token * p.o_tok + h * p.o_head;
        r.scale = nullptr;
        r.turn = true;
        r.pool = false;
    }
    return r;
}

// The token's slot and position; false: nothing of it is written.
__device__ __forceinline__ bool token_target(const AppendParams &p, int64_t token, int64_t *block, int32_t *n, int64_t *pos)
{
    const int64_t slot = p.slots[token];
    *pos = p.rot ? p.positions[token] : 0;
    if (slot < 0) return false;
    if (!slot_place(slot, p.layer.B, p.layer.num_blocks, block, n) || (p.rot && (*pos < 0 || *pos >= p.n_positions))) {
        atomicOr(p.status, kStatusBadIndex);
        return false;
    }
    return true;
}

__device__ __forceinline__ void turn(float &x, float &y, float c, float s)
{
    const float a = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
    y = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
    x = a;
}

// Scale of a row whose largest magnitude has the bits `most` (bits of magnitudes order like the
// magnitudes, with NaN above infinity): 0 for a row of zeros or of numbers too small to scale,
// NaN for a row that is not finite.  Codes are 0 unless scale > 0.
__device__ __forceinline__ float row_scale(uint32_t most, int dtype)
{
    if (most >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    const float s = __fdiv_rn(__uint_as_float(most), dtype == TC_E4M3 ? 448.f : 127.f);
    return s < 1.17549435e-38f ? 0.f : s;
}

template <typename T>
__device__ __forceinline__ void store_chunk(const AppendParams &p, const RowPlace &r, int at, const float *x, float scale)
{
    if (!r.pool) return store_floats<T, 8>(r.dst + at * static_cast<int>(sizeof(T)), x);
    switch (p.layer.dtype) {
    case TC_BF16: return store_floats<__nv_bfloat16, 8>(r.dst + at * 2, x);
    case TC_FP16: return store_floats<__half, 8>(r.dst + at * 2, x);
    case TC_FP32: return store_floats<float, 8>(r.dst + at * 4, x);
    default: break;
    }
    uint32_t w[4];
    const bool some = scale > 0.f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float a = some ? __fdiv_rn(x[2 * i], scale) : 0.f, b = some ? __fdiv_rn(x[2 * i + 1], scale) : 0.f;
        w[i] = p.layer.dtype == TC_E4M3 ? e4m3_pair(a, b) : int8_pair(a, b);
    }
    *reinterpret_cast<uint2 *>(r.dst + at) = make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

// Rows whose D is a multiple of 8 and whose addresses are multiples of 16 bytes; rot_dim a multiple of 16.
template <typename T>
__global__ void __launch_bounds__(256) append_vector_kernel(const __grid_constant__ AppendParams p)
{
    constexpr int kRows = 2;  // rows in flight per thread: loads of both before the work on either
    const int tpt = p.threads_per_token, lt = threadIdx.x & (tpt - 1);
    const int64_t token = static_cast<int64_t>(blockIdx.x) * (256 / tpt) + threadIdx.x / tpt;
    if (token >= p.n_tokens) return;
    int64_t block, pos;
    int32_t n;
    if (!token_target(p, token, &block, &n, &pos)) return;  // one token's threads are whole warps

    const int lanes = 1 << p.log2_lanes, pair = lt & (lanes - 1), D = p.layer.D;
    const int turned = p.rot >> 4;  // pairs that are rotated
    int a, b;
    if (pair < turned && !p.interleaved) a = 8 * pair, b = a + p.rot / 2;
    else a = 16 * pair, b = a + 8;
    const bool has_a = a < D, has_b = b < D;
    float c[8], s[8];
    if (pair < turned) {
        load_floats<float, 8>(p.cos + pos * p.table_stride + 32 * pair, c);
        load_floats<float, 8>(p.sin + pos * p.table_stride + 32 * pair, s);
    }
    const int rows = 2 * p.layer.H + p.Hq, step = tpt >> p.log2_lanes;
    for (int row0 = lt >> p.log2_lanes; row0 - (lt >> p.log2_lanes) < rows; row0 += kRows * step) {
        float x[kRows][16];
        RowPlace place[kRows];
#pragma unroll
        for (int u = 0; u < kRows; u++) {
            const int row = row0 + u * step;
#pragma unroll
            for (int i = 0; i < 16; i++) x[u][i] = 0.f;
            if (row < rows) {
                place[u] = row_place(p, row, token, block, n);
                if (has_a) load_floats<T, 8>(place[u].src + a * static_cast<int>(sizeof(T)), x[u]);
                if (has_b) load_floats<T, 8>(place[u].src + b * static_cast<int>(sizeof(T)), x[u] + 8);
            }
        }
#pragma unroll
        for (int u = 0; u < kRows; u++) {
            const bool here = row0 + u * step < rows;
            if (here && pair < turned && place[u].turn) {
                if (p.interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; i++) turn(x[u][2 * i], x[u][2 * i + 1], c[i], s[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i++) turn(x[u][i], x[u][8 + i], c[i], s[i]);
                }
            }
            float scale = 0.f;
            if (p.layer.k_scale) {
                uint32_t most = 0;
#pragma unroll
                for (int i = 0; i < 16; i++) most = max(most, __float_as_uint(x[u][i]) & 0x7fffffffu);
                for (int m = 1; m < lanes; m <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, m));
                scale = row_scale(most, p.layer.dtype);
            }
            if (!here) continue;
            if (place[u].pool && place[u].scale && pair == 0) *place[u].scale = scale;
            if (has_a) store_chunk<T>(p, place[u], a, x[u], scale);
            if (has_b) store_chunk<T>(p, place[u], b, x[u] + 8, scale);
        }
    }
}

// Any D up to 512 and any alignment down to the element: a warp per row, element by element.
template <typename T>
__global__ void __launch_bounds__(256) append_scalar_kernel(const __grid_constant__ AppendParams p)
{
    const int rows = 2 * p.layer.H + p.Hq, D = p.layer.D, lane = threadIdx.x & 31;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int64_t token = item / rows;
    if (token >= p.n_tokens) return;
    int64_t block, pos;
    int32_t n;
    if (!token_target(p, token, &block, &n, &pos)) return;
    const RowPlace r = row_place(p, static_cast<int>(item - token * rows), token, block, n);
    const T *src = reinterpret_cast<const T *>(r.src);
    float x[16];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int d = lane + 32 * i;
        x[i] = 0.f;
        if (d < D) {
            x[i] = to_float(src[d]);
            if (r.turn && d < p.rot) {
                const int half = p.rot / 2;
                const bool second = p.interleaved ? (d & 1) : d >= half;
                const int j = p.interleaved ? d >> 1 : (second ? d - half : d);
                const int other = p.interleaved ? d ^ 1 : (second ? d - half : d + half);
                const float c = reinterpret_cast<const float *>(p.cos + pos * p.table_stride)[j], s = reinterpret_cast<const float *>(p.sin + pos * p.table_stride)[j];
                float y = to_float(src[other]);
                if (second) {
                    turn(y, x[i], c, s);
                } else {
                    turn(x[i], y, c, s);
                }
            }
        }
        most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
    }
    most = __reduce_max_sync(0xffffffffu, most);  // also: q may be rotated in place, all lanes have read their partners
    float scale = 0.f;
    if (r.pool && p.layer.k_scale) {
        scale = row_scale(most, p.layer.dtype);
        if (lane == 0) *r.scale = scale;
    }
    const bool some = scale > 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int d = lane + 32 * i;
        if (d >= D) continue;
        if (!r.pool) {
            reinterpret_cast<T *>(r.dst)[d] = from_float<T>(x[i]);
            continue;
        }
        switch (p.layer.dtype) {
        case TC_BF16: reinterpret_cast<__nv_bfloat16 *>(r.dst)[d] = from_float<__nv_bfloat16>(x[i]); break;
        case TC_FP16: reinterpret_cast<__half *>(r.dst)[d] = from_float<__half>(x[i]); break;
        case TC_FP32: reinterpret_cast<float *>(r.dst)[d] = x[i]; break;
        case TC_E4M3: r.dst[d] = static_cast<char>(e4m3_pair(some ? __fdiv_rn(x[i], scale) : 0.f, 0.f)); break;
        default: r.dst[d] = static_cast<char>(int8_pair(some ? __fdiv_rn(x[i], scale) : 0.f, 0.f)); break;
        }
    }
}

template <typename T>
static int launch_append(AppendParams &p, bool vector, cudaStream_t s)
{
    const int64_t rows = 2 * p.layer.H + p.Hq;
    if (vector) {
        int log2_lanes = 0;
        while ((16 << log2_lanes) < p.layer.D) log2_lanes++;
        int tpt = 32;
        while (tpt < 256 && tpt < (rows << log2_lanes)) tpt *= 2;
        p.log2_lanes = log2_lanes;
        p.threads_per_token = tpt;
        const int64_t grid = (p.n_tokens + 256 / tpt - 1) / (256 / tpt);
        if (grid > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "n_tokens %lld: too many for one call", (long long)p.n_tokens);
        append_vector_kernel<T><<<static_cast<unsigned>(grid), 256, 0, s>>>(p);
    } else {
        if (static_cast<__int128>(p.n_tokens) * rows > static_cast<__int128>(INT32_MAX) * 8) return fail(TC_ERR_TOO_LARGE, "n_tokens %lld: too many for one call", (long long)p.n_tokens);
        append_scalar_kernel<T><<<static_cast<unsigned>((p.n_tokens * rows + 7) / 8), 256, 0, s>>>(p);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TC_OK : cuda_fail(e, "kernel launch");
}

}  // namespace tc

using namespace tc;

extern "C" int tc_kv_append(const tc_kv_layer_t *layer, const tc_kv_append_t *a, void *stream)
{
    clear_error();
    AppendParams p{};
    int rc = check_layer(layer, &p.layer);
    if (rc != TC_OK) return rc;
    if (!a) return fail(TC_ERR_INVALID_ARG, "args is required");
    if (a->struct_size != sizeof *a) return fail(TC_ERR_INVALID_ARG, "args.struct_size %u != %zu: header and library disagree", a->struct_size, sizeof *a);
    if (a->flags & ~TC_ROPE_INTERLEAVED) return fail(TC_ERR_INVALID_ARG, "unknown flags 0x%x", a->flags);
    if (a->dtype != TC_BF16 && a->dtype != TC_FP16 && a->dtype != TC_FP32) return fail(TC_ERR_INVALID_ARG, "dtype %d: q, k and v are TC_BF16, TC_FP16 or TC_FP32", a->dtype);
    const int e = dtype_size(a->dtype), D = p.layer.D;
    if (D > 512) return fail(TC_ERR_TOO_LARGE, "D = %d: tc_kv_append takes rows of up to 512 elements", D);
    if (a->n_tokens < 0) return fail(TC_ERR_SHAPE, "n_tokens %lld < 0", (long long)a->n_tokens);
    if (a->rot_dim < 0 || a->rot_dim > D || a->rot_dim % 2) return fail(TC_ERR_SHAPE, "rot_dim %d is not an even number in [0, D = %d]", a->rot_dim, D);
    if (!a->q != !a->q_out) return fail(TC_ERR_INVALID_ARG, "q and q_out come together or not at all");
    if (a->q && (a->Hq < 1 || a->Hq > (1 << 24))) return fail(TC_ERR_SHAPE, "Hq %lld is not in [1, 2^24]", (long long)a->Hq);
    if (a->n_tokens == 0) return TC_OK;
    uint32_t align = std::min<uint32_t>(16, p.layer.align * (p.layer.esize == 1 ? 2 : 1));  // 8 codes are one 8-byte store
    if ((rc = check_rows("k", a->k, a->k_stride, a->n_tokens, p.layer.H, int64_t(D) * e, e, false, &align)) != TC_OK) return rc;
    if ((rc = check_rows("v", a->v, a->v_stride, a->n_tokens, p.layer.H, int64_t(D) * e, e, false, &align)) != TC_OK) return rc;
    if (a->q) {
        if ((rc = check_rows("q", a->q, a->q_stride, a->n_tokens, a->Hq, int64_t(D) * e, e, false, &align)) != TC_OK) return rc;
        if ((rc = check_rows("q_out", a->q_out, a->q_out_stride, a->n_tokens, a->Hq, int64_t(D) * e, e, true, &align)) != TC_OK) return rc;
        if (a->q == a->q_out && ((a->n_tokens > 1 && a->q_stride[0] != a->q_out_stride[0]) || (a->Hq > 1 && a->q_stride[1] != a->q_out_stride[1])))
            return fail(TC_ERR_OVERLAP, "q rotated in place needs the same strides for q and q_out");
    }
    if (!a->slots || reinterpret_cast<uintptr_t>(a->slots) % 8) return fail(TC_ERR_INVALID_ARG, "slots is required, 8-byte aligned");
    if (a->rot_dim) {
        if (!a->positions || reinterpret_cast<uintptr_t>(a->positions) % 8) return fail(TC_ERR_INVALID_ARG, "positions is required with rot_dim > 0, 8-byte aligned");
        if (!a->cos || !a->sin) return fail(TC_ERR_INVALID_ARG, "cos and sin are required with rot_dim > 0");
        if (a->n_positions < 1 || a->n_positions > (1ll << 40)) return fail(TC_ERR_SHAPE, "n_positions %lld is not in [1, 2^40]", (long long)a->n_positions);
        p.table_stride = a->table_stride ? a->table_stride : a->rot_dim * 2ll;
        if (p.table_stride < a->rot_dim * 2ll || p.table_stride > (1 << 20)) return fail(TC_ERR_SHAPE, "table_stride %lld is not in [rot_dim * 2, 2^20]", (long long)p.table_stride);
        const uintptr_t bits = reinterpret_cast<uintptr_t>(a->cos) | reinterpret_cast<uintptr_t>(a->sin) | static_cast<uintptr_t>(p.table_stride);
        if (bits % 4) return fail(TC_ERR_INVALID_ARG, "cos, sin and table_stride must be multiples of 4 bytes");
        if (bits % 16) align = std::min<uint32_t>(align, 4);
    }
    int device, sms;
    if ((rc = op_device(&device, &p.status, &sms)) != TC_OK) return rc;
    const struct {
        const char *name;
        const void *p;
    } pointers[] = {{"layer.k", layer->k}, {"layer.v", layer->v}, {"layer.k_scale", layer->k_scale}, {"layer.v_scale", layer->v_scale}, {"k", a->k}, {"v", a->v},
                    {"q", a->q}, {"q_out", a->q_out}, {"slots", a->slots}, {"positions", a->rot_dim ? a->positions : nullptr},
                    {"cos", a->rot_dim ? a->cos : nullptr}, {"sin", a->rot_dim ? a->sin : nullptr}};
    for (const auto &ptr : pointers)
        if (ptr.p && (rc = check_memory(ptr.name, ptr.p, device)) != TC_OK) return rc;
    p.q = static_cast<const char *>(a->q), p.k = static_cast<const char *>(a->k), p.v = static_cast<const char *>(a->v);
    p.q_out = static_cast<char *>(a->q_out);
    p.q_tok = a->q_stride[0], p.q_head = a->q_stride[1], p.o_tok = a->q_out_stride[0], p.o_head = a->q_out_stride[1];
    p.k_tok = a->k_stride[0], p.k_head = a->k_stride[1], p.v_tok = a->v_stride[0], p.v_head = a->v_stride[1];
    p.slots = a->slots, p.positions = a->positions;
    p.cos = reinterpret_cast<const char *>(a->cos), p.sin = reinterpret_cast<const char *>(a->sin);
    p.n_positions = a->n_positions;
    p.n_tokens = a->n_tokens;
    p.Hq = a->q ? static_cast<int32_t>(a->Hq) : 0;
    p.rot = a->rot_dim;
    p.interleaved = (a->flags & TC_ROPE_INTERLEAVED) != 0;
    const bool vector = align >= 16 && D % 8 == 0 && a->rot_dim % 16 == 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (a->dtype) {
    case TC_BF16: return launch_append<__nv_bfloat16>(p, vector, s);
    case TC_FP16: return launch_append<__half>(p, vector, s);
    default: return launch_append<float>(p, vector, s);
    }
}
