// tc_kv_append: rotary positions, quantisation and the scatter into a paged layer, in one pass.
//
// A row is one (token, head) of D numbers.  Its elements come in pairs of 8-element chunks (a, b)
// chosen so that a rotation's partners are in one thread: b = a + rot_dim/2 for the half layout,
// neighbours for the interleaved one and for what is not rotated.  2^k lanes hold a row, so the
// row's largest magnitude is k shuffles away and every number is read once and written once.  The
// threads of one token share its table row in registers over all of its heads.  Bound by HBM: 32768 tokens of 64
// query and 8 KV heads x 128, bf16 to e4m3 (1.29 GB), take 238 us in a long run, 5.4 TB/s, 0.83 of a plain copy; 222 us, 0.89, 20 passes in a row.  (Slot
// and position waited for before the rows are loaded, one row type per pass: 651 us.)  Few tokens are bound by
// latency: 37 tokens of the 8B model's shape 4 us (the kernel, by a profiler; the call 12).
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
    int32_t threads_per_token; // a power of two, 32..256 (both kernels)
    unsigned int *status;
    float minus_zero;
};

struct RowPlace {
    char *dst;
    float *scale;
    bool turn, pool;
};

// Row `row` of a token: H rows of K, H of V, Hq of Q.
__device__ __forceinline__ const char *row_source(const AppendParams &p, int row, int64_t token)
{
    const int H = p.layer.H;
    if (row < H) return p.k + token * p.k_tok + row * p.k_head;
    if (row < 2 * H) return p.v + token * p.v_tok + (row - H) * p.v_head;
    return p.q + token * p.q_tok + (row - 2 * H) * p.q_head;
}
__device__ __forceinline__ RowPlace row_place(const AppendParams &p, int row, int64_t token, int64_t block, int32_t n)
{
    RowPlace r;
    const int H = p.layer.H;
    if (row < 2 * H) {
        const bool is_v = row >= H;
        const int h = is_v ? row - H : row;
        r.dst = (is_v ? p.layer.v : p.layer.k) + p.layer.geo.at(block, n, h);
        r.scale = p.layer.k_scale ? reinterpret_cast<float *>(reinterpret_cast<char *>(is_v ? p.layer.v_scale : p.layer.k_scale) + p.layer.scale_geo.at(block, n, h)) : nullptr;
        r.turn = !is_v;
        r.pool = true;
    } else {
        const int h = row - 2 * H;
        r.dst = p.q_out + token * p.o_tok + h * p.o_head;
        r.scale = nullptr;
        r.turn = true;
        r.pool = false;
    }
    return r;
}

// Where the token goes; false: nothing of it is written.
__device__ __forceinline__ bool token_target(const AppendParams &p, int64_t slot, int64_t pos, int64_t *block, int32_t *n)
{
    if (slot < 0) return false;
    if (!slot_place(slot, p.layer.B, p.layer.num_blocks, block, n) || (p.rot && (pos < 0 || pos >= p.n_positions))) {
        atomicOr(p.status, kStatusBadIndex);
        return false;
    }
    return true;
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

// Two fp32 operations at once, each rounded by itself.  The assembler contracts a packed product and a
// packed sum into one FMA (measured: a fifth of the rotated numbers differed), so products that a sum
// follows are FMAs already: x * y + (-0), the same number, with a -0 that is known at run time only.
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t &>(r)) : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<uint64_t &>(r)) : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)), "l"(reinterpret_cast<uint64_t &>(c)));
    return r;
}

// x / scale for two numbers, correctly rounded, by Markstein's method: with y the rounded reciprocal, one
// step q + (x - q scale) y brings q within an ulp, a second one rounds it correctly, as long as the
// remainders are exact.  They are where scale >= 2^-80: a quotient below 2^-11 becomes code 0 however
// it is rounded, and above that the remainder's last bit is above 2^-149.  The remainder of x = -0 is +0, and
// so would the quotient be: its sign, which an e4m3 code keeps, is x's.
__device__ __forceinline__ float2 divide2(float2 x, float minus_scale, float y)
{
    const float2 ms = make_float2(minus_scale, minus_scale), y2 = make_float2(y, y);
    float2 q = fma2(x, y2, make_float2(-0.f, -0.f));
    q = fma2(fma2(q, ms, x), y2, q);
    q = fma2(fma2(q, ms, x), y2, q);
    return make_float2(copysignf(q.x, x.x), copysignf(q.y, x.y));
}
constexpr float kDividable = 8.27180613e-25f;  // 2^-80

// The larger magnitude; a NaN wins.
__device__ __forceinline__ float larger(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// A thread's 16 elements of a row: two chunks of 8, held as pairs of rotation partners - lo[i] and hi[i] hold
// elements 2i, 2i + 1 of chunks a and b (half layout), or the even and the odd ones of four neighbours.
struct Pairs {
    float2 lo[4], hi[4];
};
// Chunks of 8 elements of T as they are loaded.
template <typename T> struct Chunk { uint4 v[sizeof(T) / 2]; };

template <typename T>
__device__ __forceinline__ void load_chunk(const char *p, Chunk<T> &c)
{
    c.v[0] = *reinterpret_cast<const uint4 *>(p);
    if constexpr (sizeof(T) == 4) c.v[1] = *reinterpret_cast<const uint4 *>(p + 16);
}
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void widen_chunks(const Chunk<T> (&c)[2], Pairs &x)
{
    const uint32_t *w[2] = {reinterpret_cast<const uint32_t *>(&c[0]), reinterpret_cast<const uint32_t *>(&c[1])};
#pragma unroll
    for (int half = 0; half < 2; half++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            float2 f;  // elements 2i, 2i + 1 of the chunk
            if constexpr (sizeof(T) == 4) f = make_float2(__uint_as_float(w[half][2 * i]), __uint_as_float(w[half][2 * i + 1]));
            else f = unpack2<T>(w[half][i]);
            if constexpr (INTERLEAVED) {
                const int j = 2 * half + i / 2;
                if (i % 2 == 0) x.lo[j].x = f.x, x.hi[j].x = f.y;
                else x.lo[j].y = f.x, x.hi[j].y = f.y;
            } else {
                (half ? x.hi : x.lo)[i] = f;
            }
        }
}
// Elements 2i, 2i + 1 of chunk `half`.
template <bool INTERLEAVED>
__device__ __forceinline__ float2 element2(const Pairs &x, int half, int i)
{
    if constexpr (!INTERLEAVED) return half ? x.hi[i] : x.lo[i];
    const int j = 2 * half + i / 2;
    return i % 2 == 0 ? make_float2(x.lo[j].x, x.hi[j].x) : make_float2(x.lo[j].y, x.hi[j].y);
}
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void store_chunk(char *p, const Pairs &x, int half)
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float2 e = element2<INTERLEAVED>(x, half, i);
        f[2 * i] = e.x, f[2 * i + 1] = e.y;
    }
    store_floats<T, 8>(p, f);
}

// Rows whose D is a multiple of 8 and whose addresses are multiples of 16 bytes; rot_dim a multiple of 16.
// A token's threads hold one row of K or V each and kQueries of Q, all loaded before slot and position
// are known; as many threads as K and V have rows (up to 256) leave nothing idle.  Three CTAs an SM leave 80 registers a
// thread, and up to 104 bytes of the 16-bit kernels' spill: with two, which spill nothing, 32768 tokens took 242 us for
// 222 (e4m3; bf16 pool 234 for 215).  fp32 rows take twice the registers: four queries at once 261 us for 251 with two.
template <typename T, bool INTERLEAVED, bool QUANTISED>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 2 : 3) append_vector_kernel(const __grid_constant__ AppendParams p)
{
    constexpr int kQueries = sizeof(T) == 4 ? 2 : 4;
    const int tpt = p.threads_per_token, lt = threadIdx.x & (tpt - 1);
    const int64_t token = static_cast<int64_t>(blockIdx.x) * (blockDim.x / tpt) + threadIdx.x / tpt;
    if (token >= p.n_tokens) return;
    const int64_t slot = p.slots[token], pos = p.rot ? p.positions[token] : 0;

    const int lanes = 1 << p.log2_lanes, pair = lt & (lanes - 1), D = p.layer.D, H = p.layer.H;
    const int turned = p.rot >> 4;  // pairs that are rotated
    int a, b;
    if (!INTERLEAVED && pair < turned) a = 8 * pair, b = a + p.rot / 2;
    else a = 16 * pair, b = a + 8;
    const bool has_a = a < D, has_b = b < D;
    const int step = tpt >> p.log2_lanes, first = lt >> p.log2_lanes;
    constexpr int e = static_cast<int>(sizeof(T));
    auto load_row = [&](const char *src, bool there, Chunk<T> (&in)[2]) {
        in[0] = Chunk<T>{}, in[1] = Chunk<T>{};
        if (there && has_a) load_chunk<T>(src + a * e, in[0]);
        if (there && has_b) load_chunk<T>(src + b * e, in[1]);
    };
    auto kv_source = [&](int row) { return row < H ? p.k + token * p.k_tok + row * p.k_head : p.v + token * p.v_tok + (row - H) * p.v_head; };
    Chunk<T> kv[2], q[kQueries][2];
    load_row(kv_source(first), first < 2 * H, kv);
    const char *q_src = p.q + token * p.q_tok + first * p.q_head;
    const int64_t q_step = step * p.q_head, o_step = step * p.o_head;
#pragma unroll
    for (int u = 0; u < kQueries; u++) load_row(q_src + u * q_step, first + u * step < p.Hq, q[u]);

    int64_t block;
    int32_t n;
    if (!token_target(p, slot, pos, &block, &n)) return;  // one token's threads are whole warps
    float2 c[4], s[4];
    if (pair < turned) {
        load_floats<float, 8>(p.cos + pos * p.table_stride + 32 * pair, reinterpret_cast<float *>(c));
        load_floats<float, 8>(p.sin + pos * p.table_stride + 32 * pair, reinterpret_cast<float *>(s));
    }
    const float2 zero = make_float2(p.minus_zero, p.minus_zero);
    auto rotate = [&](Pairs &x) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 xs = fma2(x.lo[i], s[i], zero), ys = fma2(x.hi[i], s[i], zero);
            x.lo[i] = add2(fma2(x.lo[i], c[i], zero), make_float2(-ys.x, -ys.y));
            x.hi[i] = add2(fma2(x.hi[i], c[i], zero), xs);
        }
    };

    char *q_dst = p.q_out + token * p.o_tok + first * p.o_head;
    for (int row = first; row < p.Hq;) {
#pragma unroll
        for (int u = 0; u < kQueries; u++) {
            if (row + u * step >= p.Hq) break;
            Pairs x;
            widen_chunks<T, INTERLEAVED>(q[u], x);
            if (pair < turned) rotate(x);
            if (has_a) store_chunk<T, INTERLEAVED>(q_dst + u * o_step + a * e, x, 0);
            if (has_b) store_chunk<T, INTERLEAVED>(q_dst + u * o_step + b * e, x, 1);
        }
        row += kQueries * step, q_src += kQueries * q_step, q_dst += kQueries * o_step;
        if (row >= p.Hq) break;
#pragma unroll
        for (int u = 0; u < kQueries; u++) load_row(q_src + u * q_step, row + u * step < p.Hq, q[u]);
    }

    const int64_t place = p.layer.geo.at(block, n, 0), scale_place = QUANTISED ? p.layer.scale_geo.at(block, n, 0) : 0;
    for (int row0 = 0; row0 < 2 * H; row0 += step) {
        const int row = row0 + first;
        const bool here = row < 2 * H, is_v = row >= H;
        if (row0) load_row(kv_source(row), here, kv);
        Pairs x;
        widen_chunks<T, INTERLEAVED>(kv, x);
        if (pair < turned && !is_v) rotate(x);
        float scale = 0.f;
        if constexpr (QUANTISED) {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 4; i++) most = larger(larger(larger(most, fabsf(x.lo[i].x)), fabsf(x.lo[i].y)), larger(fabsf(x.hi[i].x), fabsf(x.hi[i].y)));
            for (int m = 1; m < lanes; m <<= 1) most = larger(most, __shfl_xor_sync(0xffffffffu, most, m));
            scale = row_scale(__float_as_uint(most), p.layer.dtype);
        }
        if (!here) continue;
        const int h = is_v ? row - H : row;
        char *dst = (is_v ? p.layer.v : p.layer.k) + place + static_cast<int64_t>(h) * p.layer.geo.head;
        if constexpr (!QUANTISED) {
            auto put = [&](auto type) {
                using P = decltype(type);
                if (has_a) store_chunk<P, INTERLEAVED>(dst + a * static_cast<int>(sizeof(P)), x, 0);
                if (has_b) store_chunk<P, INTERLEAVED>(dst + b * static_cast<int>(sizeof(P)), x, 1);
            };
            if (p.layer.dtype == TC_BF16) put(__nv_bfloat16{});
            else if (p.layer.dtype == TC_FP16) put(__half{});
            else put(float{});
        } else {
            if (pair == 0) *reinterpret_cast<float *>(reinterpret_cast<char *>(is_v ? p.layer.v_scale : p.layer.k_scale) + scale_place + static_cast<int64_t>(h) * p.layer.scale_geo.head) = scale;
            if (scale >= kDividable) {
                const float y = __fdiv_rn(1.f, scale);
#pragma unroll
                for (int i = 0; i < 4; i++) x.lo[i] = divide2(x.lo[i], -scale, y), x.hi[i] = divide2(x.hi[i], -scale, y);
            } else {
                const bool some = scale > 0.f;  // rows tinier than divide2 takes; and rows whose codes are 0
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    x.lo[i] = some ? make_float2(__fdiv_rn(x.lo[i].x, scale), __fdiv_rn(x.lo[i].y, scale)) : make_float2(0.f, 0.f);
                    x.hi[i] = some ? make_float2(__fdiv_rn(x.hi[i].x, scale), __fdiv_rn(x.hi[i].y, scale)) : make_float2(0.f, 0.f);
                }
            }
#pragma unroll
            for (int half = 0; half < 2; half++) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 v = element2<INTERLEAVED>(x, half, i);
                    w[i] = p.layer.dtype == TC_E4M3 ? e4m3_pair(v.x, v.y) : int8_pair(v.x, v.y);
                }
                if (half ? has_b : has_a) *reinterpret_cast<uint2 *>(dst + (half ? b : a)) = make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
            }
        }
    }
}

// Any D up to 32 * ITEMS and any alignment down to the element: a warp per row, element by element.  A warp
// keeps its lanes' table entries and goes through its share of the token's rows, the next row loaded ahead.
template <typename T, int ITEMS>
__global__ void __launch_bounds__(256) append_scalar_kernel(const __grid_constant__ AppendParams p)
{
    const int rows = 2 * p.layer.H + p.Hq, D = p.layer.D, lane = threadIdx.x & 31, wpt = p.threads_per_token / 32;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * (8 / wpt) + (threadIdx.x >> 5) / wpt;
    if (token >= p.n_tokens) return;
    const int64_t slot = p.slots[token], pos = p.rot ? p.positions[token] : 0;
    int other[ITEMS];  // where the element's partner is; -1: it is not rotated
#pragma unroll
    for (int i = 0; i < ITEMS; i++) {
        const int d = lane + 32 * i;
        const bool second = p.interleaved ? (d & 1) : d >= p.rot / 2;
        other[i] = d >= p.rot ? -1 : p.interleaved ? d ^ 1 : second ? d - p.rot / 2 : d + p.rot / 2;
    }
    T in[ITEMS], partner[ITEMS];
    auto load_row = [&](int row) {
        const T *src = reinterpret_cast<const T *>(row_source(p, row, token));
        const bool turned = row < p.layer.H || row >= 2 * p.layer.H;
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            const int d = lane + 32 * i;
            in[i] = partner[i] = from_float<T>(0.f);
            if (d < D) in[i] = src[d];
            if (turned && other[i] >= 0) partner[i] = src[other[i]];
        }
    };
    int row = (threadIdx.x >> 5) % wpt;
    if (row < rows) load_row(row);
    int64_t block;
    int32_t n;
    if (!token_target(p, slot, pos, &block, &n)) return;
    float c[ITEMS], s[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; i++) {
        c[i] = s[i] = 0.f;
        if (other[i] < 0) continue;
        const int d = lane + 32 * i, j = p.interleaved ? d >> 1 : min(d, other[i]);
        c[i] = reinterpret_cast<const float *>(p.cos + pos * p.table_stride)[j];
        s[i] = reinterpret_cast<const float *>(p.sin + pos * p.table_stride)[j];
        if (d < other[i]) s[i] = -s[i];  // x cos - x' sin for the first of a pair, x' cos + x sin for the second
    }
    for (; row < rows; row += wpt) {
        const RowPlace r = row_place(p, row, token, block, n);
        float x[ITEMS];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
            x[i] = to_float(in[i]);
            if (r.turn && other[i] >= 0) x[i] = __fadd_rn(__fmul_rn(x[i], c[i]), __fmul_rn(to_float(partner[i]), s[i]));
            most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
        }
        most = __reduce_max_sync(0xffffffffu, most);  // also: q may be rotated in place, all lanes have read their partners
        if (row + wpt < rows) load_row(row + wpt);
        float scale = 0.f;
        if (r.pool && p.layer.k_scale) {
            scale = row_scale(most, p.layer.dtype);
            if (lane == 0) *r.scale = scale;
        }
        const bool some = scale > 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; i++) {
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
}

template <typename T>
static int launch_append(AppendParams &p, bool vector, cudaStream_t s)
{
    const int64_t rows = 2 * p.layer.H + p.Hq;
    if (vector) {
        int log2_lanes = 0;
        while ((16 << log2_lanes) < p.layer.D) log2_lanes++;
        const int64_t wanted = 2ll * p.layer.H << log2_lanes;
        int tpt = 32;
        while (tpt < 256 && tpt < wanted) tpt *= 2;
        p.log2_lanes = log2_lanes;
        p.threads_per_token = tpt;
        const int64_t grid = (p.n_tokens + 256 / tpt - 1) / (256 / tpt);
        if (grid > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "n_tokens %lld: too many for one call", (long long)p.n_tokens);
        const unsigned g = static_cast<unsigned>(grid);
        if (p.layer.quantised()) {
            if (p.interleaved) append_vector_kernel<T, true, true><<<g, 256, 0, s>>>(p);
            else append_vector_kernel<T, false, true><<<g, 256, 0, s>>>(p);
        } else {
            if (p.interleaved) append_vector_kernel<T, true, false><<<g, 256, 0, s>>>(p);
            else append_vector_kernel<T, false, false><<<g, 256, 0, s>>>(p);
        }
    } else {
        int warps = 1;  // of a token: about four rows each
        while (warps < 8 && warps * 4 < rows) warps *= 2;
        p.threads_per_token = 32 * warps;
        const int64_t grid = (p.n_tokens + 8 / warps - 1) / (8 / warps);
        if (grid > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "n_tokens %lld: too many for one call", (long long)p.n_tokens);
        const unsigned g = static_cast<unsigned>(grid);
        if (p.layer.D <= 64) append_scalar_kernel<T, 2><<<g, 256, 0, s>>>(p);
        else if (p.layer.D <= 128) append_scalar_kernel<T, 4><<<g, 256, 0, s>>>(p);
        else append_scalar_kernel<T, 16><<<g, 256, 0, s>>>(p);
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
    p.minus_zero = -0.f;
    p.interleaved = (a->flags & TC_ROPE_INTERLEAVED) != 0;
    const bool vector = align >= 16 && D % 8 == 0 && a->rot_dim % 16 == 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (a->dtype) {
    case TC_BF16: return launch_append<__nv_bfloat16>(p, vector, s);
    case TC_FP16: return launch_append<__half>(p, vector, s);
    default: return launch_append<float>(p, vector, s);
    }
}
