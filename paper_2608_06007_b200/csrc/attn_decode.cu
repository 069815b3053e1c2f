// tc_attn_decode: one query token per request over a shared prefix and the request's own pages.
//
// The keys are cut into parts.  A part's kernel leaves, for each of its rows (request, head), the
// softmax-weighted mean of its values and log2 of its sum; join_kernel weighs the parts against one
// another.  Softmax statistics, scores and outputs are fp32 throughout; only the probabilities are
// rounded, to 16 bits, to enter the second matrix product (half a step of 2^-8 or 2^-11 relative to
// each, no worse than the rounding of the values and of the output to those types).
#include <algorithm>
#include <cmath>

#include "attn.h"
#include "attn_device.cuh"

namespace tc {

constexpr int kSms = 148;  // B200; the workspace must not depend on the device that happens to be current

void split_attn(int64_t R, int64_t Hq, int64_t H, int64_t D, int64_t max_len, int64_t max_prefix, bool quantised, AttnSplit *s)
{
    *s = AttnSplit{};
    s->group = static_cast<int32_t>(Hq / H);
    s->rows = R * Hq;
    s->columns = s->group <= 8 ? 8 : 16;
    s->own_blocks = (s->group + s->columns - 1) / s->columns;
    auto cut = [&](int64_t keys, int64_t ctas, int64_t want, int64_t longest, int64_t *chunk, int32_t *parts) {
        if (keys <= 0) {
            *chunk = 64, *parts = 0;
            return;
        }
        const int64_t tiles = (keys + 63) / 64;
        const int64_t n = std::max<int64_t>(1, std::min<int64_t>(tiles, want / std::max<int64_t>(ctas, 1)));
        int64_t c = std::min((tiles + n - 1) / n * 64, longest);
        // at most 256 MB of parts
        while (c < tiles * 64 && ((keys + c - 1) / c) * s->rows * (D + 1) * 4 > (256ll << 20)) c *= 2;
        *chunk = c;
        *parts = static_cast<int32_t>((keys + c - 1) / c);
    };
    // Own tokens: about six CTAs per SM where there are few requests; at most 1024 keys a part, so that
    // one long request among short ones is not one CTA's work.
    cut(max_len, R * H * s->own_blocks, 6 * kSms, 1024, &s->own_chunk, &s->own_parts);
    const int64_t rows = R * s->group;  // of one KV head
    s->prefix_rows = max_prefix == 0 || rows <= 16 || D > 128 || quantised ? 16 : rows <= 128 ? 128 : 256;
    const int64_t block = s->prefix_rows == 16 ? s->columns : s->prefix_rows;
    s->prefix_blocks = static_cast<int32_t>((rows + block - 1) / block);
    if (s->prefix_rows == 16) {
        cut(max_prefix, H * s->prefix_blocks, 6 * kSms, 1 << 20, &s->prefix_chunk, &s->prefix_parts);
    } else {
        // One CTA per SM: the number of parts that leaves the fewest tiles to the busiest SM, a part costing
        // about two tiles to start and end.
        const int64_t tiles = (max_prefix + 127) / 128, ctas = H * s->prefix_blocks;
        int64_t best = 1, best_cost = INT64_MAX;
        for (int64_t n = 1; n <= std::min<int64_t>(tiles, 64); n++) {
            const int64_t per = (tiles + n - 1) / n, cost = (ctas * ((tiles + per - 1) / per) + kSms - 1) / kSms * (per + 2);
            if (cost < best_cost) best = n, best_cost = cost;
        }
        const int64_t per = (tiles + best - 1) / best;
        s->prefix_chunk = per * 128;
        s->prefix_parts = static_cast<int32_t>((tiles + per - 1) / per) * (s->prefix_rows == 128 ? 2 : 1);
    }
    const int64_t parts = static_cast<int64_t>(s->own_parts) + s->prefix_parts;
    s->sum_bytes = (parts * s->rows * 4 + 255) / 256 * 256;
    s->workspace = s->sum_bytes + parts * s->rows * D * 4;
}

// ------------------------------------------------------------------------------- device helpers
template <bool TRANS>
__device__ __forceinline__ void load_matrix4(uint32_t addr, uint32_t (&r)[4])
{
    if constexpr (TRANS) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
    else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint4 load_shared16(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint2 load_shared8(uint32_t addr)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
}
__device__ __forceinline__ float2 load_shared_f2(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
    return v;
}

// c (16 x 8) += a (16 x 16) * b (16 x 8), fp32 sums
template <typename T> __device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// ------------------------------------------------------------------------------ the parts' kernel
// One warp works alone on tiles of 16 keys; four warps of a CTA share a part and join at its end.
// The keys are the rows of the matrix products, S' = K Q' and O' = V' P' on m16n8k16: the columns are
// the query heads of one KV head (or rows of the batch, for a prefix with few of them), 8 or 16 at
// a time, so few heads leave little of a product idle, and every staged byte of K and V is used once
// per block of columns.  Bound by HBM.  S' comes out with a key's scores along a lane quad; packed
// to 16 bits its 8 x 8 blocks are transposed into the second product's operand by movmatrix.
// A warp has its own ring of stages, filled by 16-byte asynchronous copies whatever the size of
// the pages, and waits for no other warp until the end.
//
// Codes of a quantised pool are staged as they are and become 16-bit numbers on the way into the
// fragments, exactly: K in fp16, V in bf16.  The scales multiply the scores and the probabilities; a
// probability times a scale needs bf16's range.  Queries of such a pool are fp16 with a power of two
// per row taken out, so that the row's largest is in [2^14, 2^15): what is then below fp16's smallest
// step is below 2^-38 of that largest.  A lane reads 16 consecutive codes at once, so the order of the d's
// inside the products is a permutation: the queries use the same one, the outputs undo it.
enum { kPlain = 0, kE4m3 = 1, kInt8 = 2 };

template <int KIND, int DP, int NB>
struct Ring {
    static constexpr int esize = KIND == kPlain ? 2 : 1;
    static constexpr int row = DP * esize, chunks = row / 16;  // bytes and 16-byte chunks of a key
    static constexpr int plane = 16 * row;
    static constexpr int scale_at = 2 * plane, mask_at = scale_at + (KIND == kPlain ? 0 : 128);
    static constexpr int stage = mask_at + 16;
    static constexpr int stages = 3;  // D = 128: two CTAs an SM for 16-bit pools, four for codes
    static constexpr int join = 4 * 8 * NB * (DP + 2) * 4;  // the warps' outputs and statistics at the end
    static constexpr int bytes = 4 * stages * stage > join ? 4 * stages * stage : join;
};

// Where chunk c of key r of a tile is staged: no two of the lanes that one shared-memory pass serves
// meet in a bank, for ldmatrix (eight keys, one chunk) and for the code reads (two keys x four chunks of
// K; keys 0 2 4 6 or their successors x two chunks of V).
template <int KIND, int DP>
__device__ __forceinline__ int place_of(int r, int c)
{
    constexpr int row = DP * (KIND == kPlain ? 2 : 1);
    if constexpr (KIND == kPlain) return r * row + ((c ^ (r & 7)) << 4);
    else if constexpr (DP >= 128) return r * row + ((c ^ ((((r ^ (r >> 2)) & 1) << 2) | (r & 2))) << 4);
    else return r * row + ((c ^ ((r >> 1) & 2)) << 4);
}

// Four codes w as two pairs of fp16 numbers, exactly.
template <int KIND>
__device__ __forceinline__ void widen_half(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    if constexpr (KIND == kE4m3) {
        lo = e4m3_to_half2(w), hi = e4m3_to_half2(w >> 16);
    } else {
        // int8: the bytes of 1024 + (code + 128), less 1152
        const uint32_t u = w ^ 0x80808080u, less = 0x64806480u;
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&less));
        const __half2 y = __hsub2(*reinterpret_cast<const __half2 *>(&b), *reinterpret_cast<const __half2 *>(&less));
        lo = *reinterpret_cast<const uint32_t *>(&x), hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}
// The codes in byte t of v and w as a pair of bf16 numbers, exactly.
template <int KIND>
__device__ __forceinline__ uint32_t widen_bf16(uint32_t v, uint32_t w, int t)
{
    __nv_bfloat162 r;
    if constexpr (KIND == kE4m3) {
        // Sign, exponent and fraction bits in place are the value times 2^-120 (subnormals too); the product
        // with 2^120 is exact.  (Codes 0x7f and 0xff, e4m3's NaN, would be +-480; a quantised row has none.)
        const uint32_t x = __byte_perm(v, w, (t << 4) | ((4 + t) << 12));
        const uint32_t y = (x & 0x80008000u) | ((x >> 4) & 0x07f007f0u), big = 0x7b807b80u;
        r = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&y), *reinterpret_cast<const __nv_bfloat162 *>(&big));
    } else {
        // 128 + the low seven bits, less 128 or (sign bit set) 256: all bf16 numbers
        const uint32_t x = __byte_perm(v, w, t | ((4 + t) << 8));
        const uint32_t a = (x & 0x007f007fu) | 0x43004300u, b = (x & 0x00800080u) | 0x43004300u;
        r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    }
    return *reinterpret_cast<const uint32_t *>(&r);
}

__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// T: the type of the products - the queries' for a plain pool; quantised pools have one kernel (fp16 scores,
// bf16 values) and look at p.q_bf16.
template <typename T, int KIND, int DP, int NB>
__global__ void __launch_bounds__(128) parts_kernel(const __grid_constant__ AttnParams p)
{
    using R = Ring<KIND, DP, NB>;
    using ST = std::conditional_t<KIND == kPlain, T, __half>;
    using VT = std::conditional_t<KIND == kPlain, T, __nv_bfloat16>;
    constexpr int kCols = 8 * NB;
    extern __shared__ __align__(128) unsigned char shared[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int H = p.layer.H, group = p.split.group;

    // Which part: [begin, end) of the keys behind `table`, for rows row0 .. of KV head h.
    const int64_t prefix_ctas = p.split.prefix_rows == 16 ? static_cast<int64_t>(p.split.prefix_parts) * H * p.split.prefix_blocks : 0;
    int64_t id = blockIdx.x, begin, end, row0, row_end, part, table_width;
    int h;
    const int32_t *table;
    const bool prefix = id < prefix_ctas;
    if (prefix) {
        const int64_t block = id % p.split.prefix_blocks;
        id /= p.split.prefix_blocks;
        h = static_cast<int>(id % H);
        part = id / H;
        begin = part * p.split.prefix_chunk;
        int64_t len = *p.prefix_len;
        if (len > p.max_prefix || len < 0) {
            if (threadIdx.x == 0) atomicOr(p.status, kStatusBadIndex);
            len = len < 0 ? 0 : p.max_prefix;
        }
        end = min(begin + p.split.prefix_chunk, len);
        table = p.prefix_table;
        table_width = INT32_MAX;
        row0 = block * kCols;
        row_end = p.R * group;
    } else {
        id -= prefix_ctas;
        const int64_t block = id % p.split.own_blocks;
        id /= p.split.own_blocks;
        h = static_cast<int>(id % H);
        id /= H;
        const int64_t r = id % p.R;
        part = id / p.R;
        begin = part * p.split.own_chunk;
        int64_t len = p.lens[r];
        if (len > p.max_len) {
            if (threadIdx.x == 0) atomicOr(p.status, kStatusBadIndex);
            len = p.max_len;
        }
        end = min(begin + p.split.own_chunk, len);
        part += p.split.prefix_parts;
        table = reinterpret_cast<const int32_t *>(p.tables + r * p.table_stride);
        table_width = p.table_width;
        row0 = r * group + block * kCols;
        row_end = (r + 1) * group;
    }
    if (begin >= end) return;

    const int c = lane & 3, g = lane >> 2, D = p.layer.D;
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(shared)) + warp * R::stages * R::stage;
    const int first = static_cast<int>(begin) + 16 * warp, last = static_cast<int>(end);
    const int tiles = first < last ? (last - first + 63) / 64 : 0;

    const bool one_block = p.layer.B % 16 == 0;  // parts begin at multiples of 64 keys
    // the block that holds key `first + 64 * tile + (lane & 15)`; -1: not a key
    auto look_up = [&](int tile) -> int32_t {
        const int t = first + 64 * tile + (lane & 15);
        if (tile >= tiles || t >= last) return -1;
        const uint32_t entry = quick_div(static_cast<uint32_t>(t), p.div_block);
        int32_t b = -1;
        if (entry < table_width) b = table[entry];
        if (b < 0 || b >= p.layer.num_blocks) {
            atomicOr(p.status, kStatusBadIndex);
            return -1;
        }
        return b;
    };
    auto fill = [&](int tile, int32_t block) {
        const uint32_t at = ring + (tile % R::stages) * R::stage;
        const int t = first + 64 * tile + (lane & 15);
        const int n = t - static_cast<int>(quick_div(static_cast<uint32_t>(t), p.div_block)) * static_cast<int>(p.layer.B);
        const int64_t off = block >= 0 ? p.layer.geo.at(block, n, h) : -1;
        const uint32_t mask = __ballot_sync(0xffffffffu, block >= 0);
        if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(at + R::mask_at), "r"(mask) : "memory");
        if (one_block) {
            // 16 keys of one block: a fixed step from row to row
            const int64_t base = __shfl_sync(0xffffffffu, off, 0);
            const char *k = p.layer.k + base, *v = p.layer.v + base;
#pragma unroll
            for (int i = 0; i < 16 * R::chunks / 32; i++) {
                const int idx = i * 32 + lane, r = idx / R::chunks, ch = idx % R::chunks;
                const bool there = mask >> r & 1 && ch * 16 < D * R::esize;
                const int from = there ? r * p.layer.geo.token + ch * 16 : 0;
                const uint32_t to = at + place_of<KIND, DP>(r, ch);
                copy_async16(to, k + from, there);
                copy_async16(to + R::plane, v + from, there);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16 * R::chunks / 32; i++) {
                const int idx = i * 32 + lane, r = idx / R::chunks, ch = idx % R::chunks;
                const int64_t src = __shfl_sync(0xffffffffu, off, r);
                const bool there = src >= 0 && ch * 16 < D * R::esize;
                const int64_t from = there ? src + ch * 16 : 0;
                const uint32_t to = at + place_of<KIND, DP>(r, ch);
                copy_async16(to, p.layer.k + from, there);
                copy_async16(to + R::plane, p.layer.v + from, there);
            }
        }
        if constexpr (KIND != kPlain) {
            const int64_t from = block >= 0 ? p.layer.scale_geo.at(block, n, h) : 0;
            copy_async4(at + R::scale_at + lane * 4, reinterpret_cast<const char *>(lane < 16 ? p.layer.k_scale : p.layer.v_scale) + from, block >= 0);
        }
    };

    int32_t ahead = look_up(0);
#pragma unroll
    for (int i = 0; i < R::stages - 1; i++) {
        const int32_t b = ahead;
        ahead = look_up(i + 1);
        if (i < tiles) fill(i, b);
        copy_commit();
    }

    // Queries as B fragments: column g, element pairs 2c and 2c + 8 of every 16; for codes the lane's share of every
    // 64 is 16c .. 16c + 15, four to a step.  factor: of the scores of columns 2c and 2c + 1.
    uint32_t qf[NB][DP / 16][2];
    float factor[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; nb++) {
        const int64_t row = row0 + 8 * nb + g;
        const bool there = row < row_end;
        const int64_t r = there ? quick_div(static_cast<uint32_t>(row), p.div_group) : 0;
        const char *q = p.q + r * p.q_req + (h * group + (there ? row - r * group : 0)) * p.q_head;
#pragma unroll
        for (int ks = 0; ks < DP / 16; ks++) {
            const int d0 = KIND == kPlain ? 16 * ks + 2 * c : 64 * (ks / 4) + 16 * c + 4 * (ks % 4);
            const int d1 = KIND == kPlain ? d0 + 8 : d0 + 2;
            qf[nb][ks][0] = there && d0 < D ? *reinterpret_cast<const uint32_t *>(q + d0 * 2) : 0u;
            qf[nb][ks][1] = there && d1 < D ? *reinterpret_cast<const uint32_t *>(q + d1 * 2) : 0u;
        }
        factor[nb][0] = factor[nb][1] = p.scale_log2;
        if constexpr (KIND != kPlain) {
            float most = 0.f;  // of the finite ones
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const float2 f = p.q_bf16 ? unpack2<__nv_bfloat16>(qf[nb][ks][j]) : unpack2<__half>(qf[nb][ks][j]);
                    if (fabsf(f.x) < INFINITY) most = fmaxf(most, fabsf(f.x));
                    if (fabsf(f.y) < INFINITY) most = fmaxf(most, fabsf(f.y));
                }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int e = most > 0.f ? max(static_cast<int>(__float_as_uint(most) >> 23) - 127, -100) : 14;
            const float up = __uint_as_float(static_cast<uint32_t>(14 - e + 127) << 23), down = __uint_as_float(static_cast<uint32_t>(e - 14 + 127) << 23);
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const float2 f = p.q_bf16 ? unpack2<__nv_bfloat16>(qf[nb][ks][j]) : unpack2<__half>(qf[nb][ks][j]);
                    qf[nb][ks][j] = pack2<__half>(f.x * up, f.y * up);
                }
            factor[nb][0] = p.scale_log2 * __shfl_sync(0xffffffffu, down, 8 * c);
            factor[nb][1] = p.scale_log2 * __shfl_sync(0xffffffffu, down, 8 * c + 4);
        }
    }

    float o[NB][DP / 16][4], top[NB][2], sum[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; nb++) {
#pragma unroll
        for (int i = 0; i < DP / 16; i++) o[nb][i][0] = o[nb][i][1] = o[nb][i][2] = o[nb][i][3] = 0.f;
        top[nb][0] = top[nb][1] = -INFINITY, sum[nb][0] = sum[nb][1] = 0.f;
    }

    for (int i = 0; i < tiles; i++) {
        copy_wait<R::stages - 2>();
        __syncwarp();
        const uint32_t at = ring + (i % R::stages) * R::stage;
        uint32_t mask;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(mask) : "r"(at + R::mask_at));

        // s: keys g (0, 1) and g + 8 (2, 3) x columns 2c, 2c + 1
        float s[NB][4] = {};
        if constexpr (KIND == kPlain) {
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks++) {
                uint32_t a[4];
                load_matrix4<false>(at + place_of<KIND, DP>(lane & 15, 2 * ks + (lane >> 4)), a);
#pragma unroll
                for (int nb = 0; nb < NB; nb++) mma16816<ST>(s[nb], a, qf[nb][ks][0], qf[nb][ks][1]);
            }
        } else {
#pragma unroll
            for (int k64 = 0; k64 < DP / 64; k64++) {
                const uint4 v = load_shared16(at + place_of<KIND, DP>(g, 4 * k64 + c)), w = load_shared16(at + place_of<KIND, DP>(g + 8, 4 * k64 + c));
                const uint32_t lo[4] = {v.x, v.y, v.z, v.w}, hi[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    uint32_t a[4];
                    widen_half<KIND>(lo[j], a[0], a[2]);
                    widen_half<KIND>(hi[j], a[1], a[3]);
#pragma unroll
                    for (int nb = 0; nb < NB; nb++) mma16816<ST>(s[nb], a, qf[nb][4 * k64 + j][0], qf[nb][4 * k64 + j][1]);
                }
            }
        }

        float k_scale[2] = {1.f, 1.f}, v_scale[2] = {1.f, 1.f};
        if constexpr (KIND != kPlain) {
#pragma unroll
            for (int j = 0; j < 2; j++) {
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(k_scale[j]) : "r"(at + R::scale_at + (g + 8 * j) * 4));
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v_scale[j]) : "r"(at + R::scale_at + 64 + (g + 8 * j) * 4));
            }
        }
        float most[NB][2];
        bool move = false;
        const bool key[2] = {(mask >> g & 1) != 0, (mask >> (g + 8) & 1) != 0};
#pragma unroll
        for (int nb = 0; nb < NB; nb++)
#pragma unroll
            for (int j = 0; j < 2; j++) {
                s[nb][j] = key[0] ? s[nb][j] * (KIND == kPlain ? factor[nb][j] : factor[nb][j] * k_scale[0]) : -INFINITY;
                s[nb][j + 2] = key[1] ? s[nb][j + 2] * (KIND == kPlain ? factor[nb][j] : factor[nb][j] * k_scale[1]) : -INFINITY;
                most[nb][j] = fmaxf(s[nb][j], s[nb][j + 2]);
                move = move || most[nb][j] > top[nb][j] + 8.f;
            }
        // A running maximum moves only when a score exceeds it by more than 8 (2^8 in probabilities): up
        // to there they stay small enough for either 16-bit type and the outputs need no rescaling.
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int nb = 0; nb < NB; nb++) {
                float f[2];
#pragma unroll
                for (int j = 0; j < 2; j++) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) most[nb][j] = fmaxf(most[nb][j], __shfl_xor_sync(0xffffffffu, most[nb][j], x));
                    const float m = fmaxf(top[nb][j], most[nb][j]);
                    f[j] = m == top[nb][j] ? 1.f : exp2_approx(top[nb][j] - m);
                    top[nb][j] = m;
                    sum[nb][j] *= f[j];
                }
#pragma unroll
                for (int k = 0; k < DP / 16; k++) o[nb][k][0] *= f[0], o[nb][k][1] *= f[1], o[nb][k][2] *= f[0], o[nb][k][3] *= f[1];
            }
        }
        uint32_t pf[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; nb++) {
            const float m0 = top[nb][0] == -INFINITY ? 0.f : top[nb][0], m1 = top[nb][1] == -INFINITY ? 0.f : top[nb][1];
            const float e0 = exp2_approx(s[nb][0] - m0), e1 = exp2_approx(s[nb][1] - m1), e2 = exp2_approx(s[nb][2] - m0), e3 = exp2_approx(s[nb][3] - m1);
            sum[nb][0] += e0 + e2, sum[nb][1] += e1 + e3;
            pf[nb][0] = transposed(KIND == kPlain ? pack2<VT>(e0, e1) : pack2<VT>(e0 * v_scale[0], e1 * v_scale[0]));
            pf[nb][1] = transposed(KIND == kPlain ? pack2<VT>(e2, e3) : pack2<VT>(e2 * v_scale[1], e3 * v_scale[1]));
        }

        if constexpr (KIND == kPlain) {
#pragma unroll
            for (int k = 0; k < DP / 16; k++) {
                uint32_t a[4];  // d's 16k .. + 7 and + 8 .., keys 0-7 and 8-15
                load_matrix4<true>(at + R::plane + place_of<KIND, DP>((lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)), a);
#pragma unroll
                for (int nb = 0; nb < NB; nb++) mma16816<VT>(o[nb][k], a, pf[nb][0], pf[nb][1]);
            }
        } else {
            constexpr int bytes = DP >= 128 ? 16 : 8;  // codes a lane reads of each of its four keys
#pragma unroll
            for (int u = 0; u < DP / (8 * bytes); u++) {
                uint32_t w[4][bytes / 4];
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const int kk = 2 * c + (k & 1) + 8 * (k >> 1);
                    if constexpr (bytes == 16) {
                        const uint4 v = load_shared16(at + R::plane + place_of<KIND, DP>(kk, 8 * u + g));
                        w[k][0] = v.x, w[k][1] = v.y, w[k][2] = v.z, w[k][3] = v.w;
                    } else {
                        const uint2 v = load_shared8(at + R::plane + place_of<KIND, DP>(kk, g >> 1) + (g & 1) * 8);
                        w[k][0] = v.x, w[k][1] = v.y;
                    }
                }
#pragma unroll
                for (int t = 0; t < bytes; t += 2) {
                    const uint32_t a[4] = {widen_bf16<KIND>(w[0][t / 4], w[1][t / 4], t & 3), widen_bf16<KIND>(w[0][t / 4], w[1][t / 4], (t & 3) + 1),
                                           widen_bf16<KIND>(w[2][t / 4], w[3][t / 4], t & 3), widen_bf16<KIND>(w[2][t / 4], w[3][t / 4], (t & 3) + 1)};
#pragma unroll
                    for (int nb = 0; nb < NB; nb++) mma16816<VT>(o[nb][(bytes * u + t) / 2], a, pf[nb][0], pf[nb][1]);
                }
            }
        }
        __syncwarp();
        const int32_t b = ahead;
        ahead = look_up(i + R::stages);
        if (i + R::stages - 1 < tiles) fill(i + R::stages - 1, b);
        copy_commit();
    }
    copy_wait<0>();

    // Join the four warps: outputs and (maximum, sum) of each in shared memory.
    __syncthreads();
    float *mine = reinterpret_cast<float *>(shared) + warp * kCols * (DP + 2);
#pragma unroll
    for (int nb = 0; nb < NB; nb++)
#pragma unroll
        for (int j = 0; j < 2; j++) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) sum[nb][j] += __shfl_xor_sync(0xffffffffu, sum[nb][j], x);
            float *col = mine + (8 * nb + 2 * c + j) * (DP + 2);
#pragma unroll
            for (int k = 0; k < DP / 16; k++)
#pragma unroll
                for (int half = 0; half < 2; half++) {
                    constexpr int bytes = DP >= 128 ? 16 : 8;
                    const int d = KIND == kPlain ? 16 * k + g + 8 * half : 8 * bytes * (2 * k / bytes) + g * bytes + 2 * k % bytes + half;
                    col[d] = o[nb][k][2 * half + j];
                }
            if (g == 0) col[DP] = top[nb][j], col[DP + 1] = sum[nb][j];
        }
    __syncthreads();
    for (int i = warp; i < kCols; i += 4) {
        const int64_t row = row0 + i;
        if (row >= row_end) break;
        const float *w[4];
        float m = -INFINITY, f[4], total = 0.f;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            w[k] = reinterpret_cast<const float *>(shared) + (k * kCols + i) * (DP + 2);
            m = fmaxf(m, w[k][DP]);
        }
#pragma unroll
        for (int k = 0; k < 4; k++) {
            f[k] = w[k][DP] == -INFINITY && w[k][DP + 1] == 0.f ? 0.f : exp2f(w[k][DP] - m);
            total += f[k] * w[k][DP + 1];
        }
        const int64_t r = quick_div(static_cast<uint32_t>(row), p.div_group);
        const int64_t at = part * p.split.rows + r * p.Hq + h * group + (row - r * group);
        const float inv = total == 0.f ? 0.f : 1.f / total;
        for (int d = lane; d < D; d += 32) p.parts[at * D + d] = (f[0] * w[0][d] + f[1] * w[1][d] + f[2] * w[2][d] + f[3] * w[3][d]) * inv;
        if (lane == 0) p.sums[at] = total == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m) + log2f(total);
    }
}

// The parts' outputs, each by its share of the whole sum.  WARPS warps of a CTA take a row, each some of its
// parts: one where there are few parts, four where one warp's chain of loads would be long.
template <typename T, int WARPS>
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ AttnParams p)
{
    constexpr int kAhead = 4;  // parts loaded at once
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = p.layer.D, share = warp % WARPS;
    __shared__ float others[WARPS == 1 ? 1 : 4][WARPS == 1 ? 1 : 32 * 8 + 1];
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (4 / WARPS) + warp / WARPS;
    if (row >= p.split.rows) return;  // WARPS > 1: a CTA is one row
    const int64_t r = row / p.Hq, head = row - r * p.Hq;
    int64_t len = p.lens[r];
    if (len < 0) return;
    len = min(len, p.max_len);
    const int64_t shared_len = p.split.prefix_parts ? min(max(static_cast<int64_t>(*p.prefix_len), int64_t(0)), p.max_prefix) : 0;
    const int front = static_cast<int>((shared_len + p.split.prefix_chunk - 1) / p.split.prefix_chunk) * (p.split.prefix_rows == 128 ? 2 : 1);
    const int back = static_cast<int>((len + p.split.own_chunk - 1) / p.split.own_chunk);
    const int n = front + back;
    auto index = [&](int i) -> int64_t { return static_cast<int64_t>(i < front ? i : p.split.prefix_parts + i - front) * p.split.rows + row; };
    float m = -INFINITY;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, p.sums[index(i)]);
#pragma unroll
    for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    const float base = m == -INFINITY ? 0.f : m;
    float acc[8] = {}, total = 0.f;
    const int from = n * share / WARPS, to = n * (share + 1) / WARPS;
    for (int i0 = from; i0 < to; i0 += 32) {
        const int mine = i0 + lane;
        const float weight = mine < to ? exp2f(p.sums[index(mine)] - base) : 0.f;
        total += weight;
        for (int j0 = 0; j0 < min(32, to - i0); j0 += kAhead) {
            float w[kAhead];
            float4 v[kAhead][2];
#pragma unroll
            for (int j = 0; j < kAhead; j++) {
                w[j] = __shfl_sync(0xffffffffu, weight, j0 + j);  // 0 past the end and for a part without keys, whose outputs were not written
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    v[j][k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (w[j] != 0.f && lane * 4 + 128 * k < D) v[j][k] = *reinterpret_cast<const float4 *>(p.parts + index(i0 + j0 + j) * D + lane * 4 + 128 * k);
                }
            }
#pragma unroll
            for (int j = 0; j < kAhead; j++)
#pragma unroll
                for (int k = 0; k < 2; k++)
                    if (w[j] != 0.f) acc[4 * k] += w[j] * v[j][k].x, acc[4 * k + 1] += w[j] * v[j][k].y, acc[4 * k + 2] += w[j] * v[j][k].z, acc[4 * k + 3] += w[j] * v[j][k].w;
        }
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) total += __shfl_xor_sync(0xffffffffu, total, x);
    if constexpr (WARPS > 1) {
#pragma unroll
        for (int k = 0; k < 8; k++) others[warp][k * 32 + lane] = acc[k];
        if (lane == 0) others[warp][256] = total;
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int w = 1; w < WARPS; w++) {
#pragma unroll
            for (int k = 0; k < 8; k++) acc[k] += others[w][k * 32 + lane];
            total += others[w][256];
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    char *dst = p.out + r * p.out_req + head * p.out_head;
#pragma unroll
    for (int k = 0; k < 2; k++)
        if (lane * 4 + 128 * k < D)
            *reinterpret_cast<uint2 *>(dst + (lane * 4 + 128 * k) * 2) = make_uint2(pack2<T>(acc[4 * k] * inv, acc[4 * k + 1] * inv), pack2<T>(acc[4 * k + 2] * inv, acc[4 * k + 3] * inv));
    if (p.lse && lane == 0) p.lse[row] = total == 0.f ? -INFINITY : (base + log2f(total)) * 0.6931471805599453f;
}

// --------------------------------------------------------------------------------------- launching
template <typename T, int KIND, int DP, int NB>
static int launch_parts(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    using R = Ring<KIND, DP, NB>;
    static bool raised[kMaxDevices];  // set once per device; setting it twice does no harm
    if (!raised[device]) {
        const cudaError_t e = cudaFuncSetAttribute(parts_kernel<T, KIND, DP, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, R::bytes);
        if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(dynamic shared memory)");
        raised[device] = true;
    }
    parts_kernel<T, KIND, DP, NB><<<grid, 128, R::bytes, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TC_OK : cuda_fail(e, "kernel launch");
}

template <typename T, int KIND, int NB>
static int launch_parts_for(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    if (p.layer.D <= 64) return launch_parts<T, KIND, 64, NB>(p, grid, device, s);
    if (p.layer.D <= 128) return launch_parts<T, KIND, 128, NB>(p, grid, device, s);
    return launch_parts<T, KIND, 256, NB>(p, grid, device, s);
}

template <typename T, int KIND>
static int launch_parts_columns(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    return p.split.columns == 8 ? launch_parts_for<T, KIND, 1>(p, grid, device, s) : launch_parts_for<T, KIND, 2>(p, grid, device, s);
}

template <typename T>
static int launch_decode(const AttnParams &p, int device, cudaStream_t s)
{
    int rc = TC_OK;
    if (p.split.prefix_rows > 16 && (rc = launch_prefix(p, std::is_same<T, __half>::value ? TC_FP16 : TC_BF16, device, s)) != TC_OK) return rc;
    const int64_t ctas = (p.split.prefix_rows == 16 ? static_cast<int64_t>(p.split.prefix_parts) * p.layer.H * p.split.prefix_blocks : 0) + static_cast<int64_t>(p.split.own_parts) * p.R * p.layer.H * p.split.own_blocks;
    if (ctas > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "%lld parts: too many for one call", (long long)ctas);
    if (ctas) {
        const unsigned grid = static_cast<unsigned>(ctas);
        switch (p.layer.dtype) {
        case TC_E4M3: rc = launch_parts_columns<__half, kE4m3>(p, grid, device, s); break;
        case TC_INT8: rc = launch_parts_columns<__half, kInt8>(p, grid, device, s); break;
        default: rc = launch_parts_columns<T, kPlain>(p, grid, device, s); break;
        }
        if (rc != TC_OK) return rc;
    }
    if (p.split.prefix_parts + p.split.own_parts > 8) join_kernel<T, 4><<<static_cast<unsigned>(p.split.rows), 128, 0, s>>>(p);
    else join_kernel<T, 1><<<static_cast<unsigned>((p.split.rows + 3) / 4), 128, 0, s>>>(p);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? TC_OK : cuda_fail(e, "kernel launch");
}

// What both entry points check; fills p's geometry and split.
static int check_decode(const tc_kv_layer_t *layer, const tc_attn_decode_t *a, AttnParams *p)
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
    if (!(a->scale == a->scale) || std::isinf(a->scale)) return fail(TC_ERR_INVALID_ARG, "scale is not a finite number");
    split_attn(a->R, a->Hq, p->layer.H, D, a->max_len, a->max_prefix, p->layer.quantised(), &p->split);
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

extern "C" int tc_attn_decode(const tc_kv_layer_t *layer, const tc_attn_decode_t *a, void *stream)
{
    clear_error();
    AttnParams p{};
    int rc = check_decode(layer, a, &p);
    if (rc != TC_OK) return rc;
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
    p.sums = static_cast<float *>(a->workspace);
    p.parts = reinterpret_cast<float *>(static_cast<char *>(a->workspace) + p.split.sum_bytes);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return a->dtype == TC_BF16 ? launch_decode<__nv_bfloat16>(p, device, s) : launch_decode<__half>(p, device, s);
}
