// tc_attn_decode: one query token per request over a shared prefix and the request's own pages.
//
// The keys of a row (request, head) are cut into parts, each of which leaves the softmax-weighted mean of its
// values and log2 of its sum in the workspace; join_kernel weighs the parts against one another.
// prefix_kernel (attn_prefix.cu) takes a prefix that many rows share, stream_kernel all other keys.
// Softmax statistics, scores and outputs are fp32 throughout; only the probabilities are rounded, to 16
// bits, to enter the second matrix product (half a step of 2^-8 or 2^-11 relative to each, no worse than
// the rounding of the values and of the output to those types; in fp16 so down to 2^-21 of the largest, and by at most
// 2^-32 of it below that).
#include <algorithm>
#include <atomic>
#include <cmath>

#include "attn.h"
#include "attn_device.cuh"

namespace tc {

constexpr float kLn2 = 0.6931471805599453f;
// ------------------------------------------------------------------------------- device helpers
template <bool TRANS>
__device__ __forceinline__ void load_matrix4(uint32_t addr, uint32_t (&r)[4])
{
    if constexpr (TRANS) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
    else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
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

// ---------------------------------------------------------------------------------- the stream
// All tiles of keys - of every request, KV head and block of columns in turn, then of a prefix that
// few rows share - are one sequence, of which every warp of the grid takes an equal stretch, whatever
// the lengths.  It has its own ring of stages, filled by 16-byte asynchronous copies whatever the size
// of the pages, and works alone: the copies run ahead across the ends of items, so that short
// requests cost no gaps.  An item that is one warp's leaves a whole part, one that is cut leaves pieces,
// at most two a warp.  Bound by HBM for 16-bit pools (297k tokens of 4 heads x 128, 608 MB: a call takes 105 us, 5.8 TB/s,
// 0.88 of a plain copy), by latency and issue for codes (the same in int8, 313 MB: 73 us in a long run, 4.3 TB/s; 69 us 20 in a row).
//
// The keys are the rows of the matrix products, S' = K Q' and O' = V' P' on m16n8k16: the columns are
// the query heads of one KV head (or rows of the batch, for the prefix), 8 or 16 at a time, so few
// heads leave little of a product idle, and every staged byte of K and V is used once per block of
// columns.  S' comes out with a key's scores along a lane quad; packed to 16 bits its 8 x 8 blocks are
// transposed into the second product's operand by movmatrix.
//
// Codes of a quantised pool are staged as they are and become fp16 on the way into the fragments,
// exactly.  ldmatrix hands a lane four codes of one key's row (K), its 8-bit transpose four keys' codes of
// one d (V); which key is which row of S' is chosen so that both products agree on the order of the keys.
// The key's scale multiplies the scores.  The value's goes into the exponent, w = exp2(s + log2 v_scale
// - top), so that fp16 probabilities have the largest contribution as their reference whatever the scales
// are.  The sum has exp2(s - ref) with a running maximum of its own: scales reach from 2^-126 to 2^127, so neither is the
// other times a number that fp32 holds.  (These exponentials cost 3 % at D = 256, 12 % with 16 columns there, nothing
// else that was measured; w over its scale instead, where an item's scales allow it, was slower.)  Queries of such a pool are fp16 with a power of two
// per row taken out, so that the row's largest is in [2^14, 2^15): what is then below fp16's smallest
// step is below 2^-38 of that largest.

// A tile is 16 keys, or 32 for codes, whose widening takes twice the instructions a byte: two groups of 16
// side by side keep the warps busier than a third more warps would (D = 128, 297k tokens of 4 heads, by a profiler: 62 us against 70).
template <int KIND, int DP>
struct Ring {
    static constexpr int esize = KIND == kPlain ? 2 : 1;
    static constexpr int groups = KIND == kPlain ? 1 : 2, keys = 16 * groups;
    static constexpr int row = DP * esize, chunks = row / 16;  // bytes and 16-byte chunks of a key
    static constexpr int plane = 16 * row, group = 2 * plane, tile = groups * group;  // 16 keys' K, then their V
    static constexpr int head = KIND == kPlain ? 16 : 16 + 8 * keys;  // {mask, flags, request, item}, then scales of K and of V
    // One tile is in flight while one is worked on.  D = 128 and 8 columns: three CTAs an SM (a third stage and two CTAs
    // were slower where requests are short, by a profiler: 512 of about 200 keys 102 against 88 us).
    static constexpr int stages = 2;
    static constexpr int bytes = 4 * stages * (tile + head);
    static constexpr int copies = 16 * chunks / 32, rows_per_copy = 32 / chunks;  // of 16 keys, by a warp
};

// Where chunk c of key r of a tile is staged: no two of the rows that one shared-memory pass serves meet in a
// bank - eight keys in order (16-bit), keys 0 1 4 5 8 9 12 13 or their successors but one (codes).
template <int KIND, int DP>
__device__ __forceinline__ int place_of(int r, int c)
{
    constexpr int row = DP * (KIND == kPlain ? 2 : 1);
    if constexpr (KIND == kPlain) return r * row + ((c ^ (r & 7)) << 4);
    else if constexpr (DP >= 128) return r * row + ((c ^ (((r >> 2) << 1 | (r & 1)) & 7)) << 4);
    else return r * row + ((c ^ (r >> 2 & 3)) << 4);
}

// 16 keys x 32 d's of 8 bits, transposed: r[0], r[1]: d's g and g + 8, keys 4c .. 4c + 3; r[2], r[3]: 16 d's on.
__device__ __forceinline__ void load_codes_transposed(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// Length of a request (r < R) or of the prefix (r == R; 0 where prefix_kernel takes it), in keys.
__device__ __forceinline__ int stream_length(const AttnParams &p, int64_t r, bool tell)
{
    const int64_t most = r < p.R ? p.max_len : p.max_prefix;
    if (most == 0 || (r == p.R && p.split.prefix_rows != 16)) return 0;
    int64_t len = r < p.R ? p.lens[r] : *p.prefix_len;
    if (tell && (len > most || (r == p.R && len < 0))) atomicOr(p.status, kStatusBadIndex);
    return static_cast<int>(min(max(len, int64_t(0)), most));
}
__device__ __forceinline__ int stream_items(const AttnParams &p, int64_t r) { return p.layer.H * (r < p.R ? p.split.own_blocks : p.split.prefix_blocks); }
__device__ __forceinline__ uint32_t tiles_of(const AttnParams &p, uint32_t keys) { return p.split.tile_keys == 16 ? (keys + 15) >> 4 : (keys + 31) >> 5; }
// Tiles that each warp takes of `total` (below 2^31): warp w has [w * share, (w + 1) * share).
__device__ __forceinline__ uint32_t stream_share(const AttnParams &p, uint32_t total) { return max((total + p.split.stream_ctas * 4 - 1) / (p.split.stream_ctas * 4), static_cast<uint32_t>(kLeastShare)); }
__device__ __forceinline__ uint32_t stream_tiles(const AttnParams &p, int64_t r, bool tell) { return tiles_of(p, stream_length(p, r, tell)) * stream_items(p, r); }

enum : uint32_t { kFirst = 1, kLast = 2, kWhole = 4, kSecond = 8 };

// T: the type of the products - the queries' for a plain pool, fp16 for a quantised one, which looks at p.q_bf16.
template <typename T, int KIND, int DP, int NB>
__global__ void __launch_bounds__(128, DP > 128 ? 1 : NB > 1 ? 2 : DP == 64 ? 4 : 3) stream_kernel(const __grid_constant__ AttnParams p)
{
    using R = Ring<KIND, DP>;
    using ST = std::conditional_t<KIND == kPlain, T, __half>;
    using VT = ST;
    constexpr int kCols = 8 * NB;
    constexpr float kLift = probability_lift<VT>();
    extern __shared__ __align__(128) unsigned char shared[];
    __shared__ uint32_t sums_of[4], start_at[4], start_off[4];
    allow_next();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = p.split.group;

    // Every CTA adds the tiles of all requests up, each thread over a run of them, and finds where its warps
    // begin; CTA 0 also leaves the sums for join_kernel.
    const int64_t per = (p.R + 1 + 127) / 128, mine0 = threadIdx.x * per, mine1 = min(mine0 + per, p.R + 1);
    uint32_t my_tiles = 0;
    for (int64_t r = mine0; r < mine1; r++) my_tiles += stream_tiles(p, r, blockIdx.x == 0);
    uint32_t upto = my_tiles;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, upto, x);
        if (lane >= x) upto += v;
    }
    if (lane == 31) sums_of[warp] = upto;
    __syncthreads();
    uint32_t total = 0;
#pragma unroll
    for (int w = 0; w < 4; w++) {
        if (w < warp) upto += sums_of[w];
        total += sums_of[w];
    }
    const uint32_t before = upto - my_tiles, share = stream_share(p, total);
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const uint32_t from = (w * gridDim.x + blockIdx.x) * share;
        if (from < before || from >= upto) continue;
        uint32_t at = before;
        for (int64_t r = mine0; r < mine1; r++) {
            const uint32_t n = stream_tiles(p, r, false);
            if (from < at + n) {
                start_at[w] = static_cast<uint32_t>(r), start_off[w] = from - at;
                break;
            }
            at += n;
        }
    }
    if (blockIdx.x == 0) {
        uint32_t at = before;
        for (int64_t r = mine0; r < mine1; r++) {
            p.before[4 + r] = at;
            at += stream_tiles(p, r, false);
        }
        if (threadIdx.x == 0) {
            // the share, and what quick_div needs to divide by it (as make_fastdiv on the host)
            const uint32_t shift = share > 1 ? 32 - __clz(share - 1) : 0;
            const uint32_t mul = static_cast<uint32_t>((((1ull << shift) - share) << 32) / share + 1);
            *reinterpret_cast<uint4 *>(p.before) = make_uint4(total, share, mul, shift);
        }
    }
    __syncthreads();
    // spread over the SMs first, so that few shares do not meet on few of them
    const uint32_t index = warp * gridDim.x + blockIdx.x;
    if (static_cast<uint64_t>(index) * share >= total) return await_last();
    const int todo = static_cast<int>(min(share, total - index * share));

    const int c = lane & 3, g = lane >> 2, D = p.layer.D;
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(shared)) + warp * R::stages * R::tile;
    const uint32_t heads = static_cast<uint32_t>(__cvta_generic_to_shared(shared)) + 4 * R::stages * R::tile + warp * R::stages * R::head;
    const bool one_block = p.layer.B % 16 == 0;  // 16 keys lie in one block

    // The next tile to be copied: tile `l_tile` of `l_tiles` of item `l_item` of request l_r.
    int64_t l_r = start_at[warp];
    int l_len = stream_length(p, l_r, false), l_tiles = static_cast<int>(tiles_of(p, l_len));
    int l_item = static_cast<int>(start_off[warp] / l_tiles), l_tile = static_cast<int>(start_off[warp] - l_item * l_tiles);
    const int32_t *l_table = l_r < p.R ? reinterpret_cast<const int32_t *>(p.tables + l_r * p.table_stride) : p.prefix_table;
    auto head_of = [&](int64_t r, int item) {
        const int blocks = r < p.R ? p.split.own_blocks : p.split.prefix_blocks;
        return blocks == 1 ? item : item / blocks;
    };
    const int first_item = l_item;
    bool l_first = true, l_from_start = l_tile == 0, l_second = false;
    int l_left = todo;
    // this lane's rows and chunk of every copy
    const int my_row = lane / R::chunks, my_chunk = lane % R::chunks;
    const bool in_row = my_chunk * 16 < D * R::esize;
    int spot[R::copies];
#pragma unroll
    for (int i = 0; i < R::copies; i++) spot[i] = place_of<KIND, DP>(i * R::rows_per_copy + my_row, my_chunk);
    const int64_t v_from_k = p.layer.v - p.layer.k, copy_step = static_cast<int64_t>(R::rows_per_copy) * p.layer.geo.token;
    // What the table says of the tile's key of this lane; kNoKey: it is none.  Looked at a tile later, so that nothing
    // waits for the load.
    constexpr int32_t kNoKey = INT32_MIN;
    const int my_key = lane % R::keys;
    auto look_up = [&]() -> int32_t {
        const int t = R::keys * l_tile + my_key;
        if (l_left <= 0 || t >= l_len) return kNoKey;
        const uint32_t entry = quick_div(static_cast<uint32_t>(t), p.div_block);
        return l_r == p.R || entry < p.table_width ? l_table[entry] : -1;
    };
    // Copies the next tile to stage `to`, its keys' blocks given, and steps on.
    auto fill = [&](int to, int32_t said) {
        if (said != kNoKey && (said < 0 || said >= p.layer.num_blocks)) atomicOr(p.status, kStatusBadIndex);
        const int32_t block = said >= 0 && said < p.layer.num_blocks ? said : -1;
        const uint32_t at = ring + to * R::tile, head = heads + to * R::head;
        const int t = R::keys * l_tile + my_key;
        const int n = t - static_cast<int>(quick_div(static_cast<uint32_t>(t), p.div_block)) * static_cast<int>(p.layer.B);
        const int h = head_of(l_r, l_item);
        const uint32_t mask = __ballot_sync(0xffffffffu, block >= 0);
        const bool end = l_tile + 1 == l_tiles, last = end || l_left == 1;
        if (lane == 0)
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(head),
                         "r"(mask), "r"((l_first ? kFirst : 0u) | (last ? kLast : 0u) | (last && end && l_from_start ? kWhole : 0u) | (l_second ? kSecond : 0u)), "r"(static_cast<uint32_t>(l_r)), "r"(l_item)
                         : "memory");
#pragma unroll
        for (int sub = 0; sub < R::groups; sub++) {
            const uint32_t dst = at + sub * R::group;
            if (one_block) {
                // a fixed step from key to key
                const int n0 = __shfl_sync(0xffffffffu, n, 16 * sub), b0 = __shfl_sync(0xffffffffu, block, 16 * sub);
                const char *k = p.layer.k + p.layer.geo.at(max(b0, 0), n0 + my_row, h) + my_chunk * 16;
                const uint32_t rows = in_row ? mask >> (16 * sub + my_row) : 0u;
#pragma unroll
                for (int i = 0; i < R::copies; i++, k += copy_step) {
                    const bool there = rows >> (i * R::rows_per_copy) & 1;
                    copy_async16(dst + spot[i], k, there);  // where it is not there, nothing is read
                    copy_async16(dst + spot[i] + R::plane, k + v_from_k, there);
                }
            } else {
                const int64_t off = block >= 0 ? p.layer.geo.at(block, n, h) : -1;
#pragma unroll
                for (int i = 0; i < R::copies; i++) {
                    const int64_t src = __shfl_sync(0xffffffffu, off, 16 * sub + i * R::rows_per_copy + my_row);
                    const bool there = src >= 0 && in_row;
                    const char *k = p.layer.k + (there ? src + my_chunk * 16 : 0);
                    copy_async16(dst + spot[i], k, there);
                    copy_async16(dst + spot[i] + R::plane, k + v_from_k, there);
                }
            }
        }
        if constexpr (KIND != kPlain) {
            const int64_t from = block >= 0 ? p.layer.scale_geo.at(block, n, h) : 0;
            copy_async4(head + 16 + lane * 4, reinterpret_cast<const char *>(p.layer.k_scale) + from, block >= 0);
            copy_async4(head + 16 + 4 * R::keys + lane * 4, reinterpret_cast<const char *>(p.layer.v_scale) + from, block >= 0);
        }
        l_left--;
        l_first = last;
        l_tile++;
        if (end) {
            l_tile = 0, l_from_start = true, l_second = true;
            if (++l_item == stream_items(p, l_r) && l_left > 0) {
                // the next request that has keys; `l_left` says that there is one
                l_item = 0;
                for (int64_t base = l_r + 1; base <= p.R; base += 32) {
                    const int len = base + lane <= p.R ? stream_length(p, base + lane, false) : 0;
                    const uint32_t some = __ballot_sync(0xffffffffu, len > 0);
                    if (!some) continue;
                    const int at_lane = __ffs(some) - 1;
                    l_r = base + at_lane;
                    l_len = __shfl_sync(0xffffffffu, len, at_lane);
                    break;
                }
                l_tiles = static_cast<int>(tiles_of(p, l_len));
                l_table = l_r < p.R ? reinterpret_cast<const int32_t *>(p.tables + l_r * p.table_stride) : p.prefix_table;
            }
        }
    };

    int32_t ahead = look_up();
#pragma unroll
    for (int i = 0; i < R::stages - 1; i++) {
        if (i < todo) {
            fill(i, ahead);
            ahead = look_up();
        }
        copy_commit();
    }

    // Rows of an item: columns 0 .. row_end - row0 of KV head h.
    struct Item {
        int64_t row0, row_end;
        int h;
    };
    auto item_of = [&](int64_t r, int item) {
        Item it;
        const int blocks = r < p.R ? p.split.own_blocks : p.split.prefix_blocks;
        it.h = head_of(r, item);
        const int block = item - it.h * blocks;
        it.row0 = (r < p.R ? r * group : 0) + block * kCols;
        it.row_end = (r < p.R ? r + 1 : p.R) * group;
        return it;
    };
    // Queries as B fragments: column g, element pairs 2c and 2c + 8 of every 16; for codes 4c and 4c + 2.  factor: of the scores of columns 2c and 2c + 1.
    uint32_t qf[NB][DP / 16][2];
    float factor[NB][2];
    auto load_queries = [&](int64_t r, int item, uint32_t (&q)[NB][DP / 16][2]) {
        const Item it = item_of(r, item);
#pragma unroll
        for (int nb = 0; nb < NB; nb++) {
            const int64_t row = it.row0 + 8 * nb + g;
            const bool there = row < it.row_end;
            const int64_t req = there ? quick_div(static_cast<uint32_t>(row), p.div_group) : 0;
            const char *src = p.q + req * p.q_req + (it.h * group + (there ? row - req * group : 0)) * p.q_head;
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks++) {
                const int d0 = 16 * ks + (KIND == kPlain ? 2 : 4) * c;
                const int d1 = KIND == kPlain ? d0 + 8 : d0 + 2;
                q[nb][ks][0] = there && d0 < D ? *reinterpret_cast<const uint32_t *>(src + d0 * 2) : 0u;
                q[nb][ks][1] = there && d1 < D ? *reinterpret_cast<const uint32_t *>(src + d1 * 2) : 0u;
            }
        }
    };
    auto take_queries = [&]() {
#pragma unroll
        for (int nb = 0; nb < NB; nb++) {
            factor[nb][0] = factor[nb][1] = p.scale_log2;
            if constexpr (KIND != kPlain) {
                float most = 0.f;  // of the finite ones
#pragma unroll
                for (int ks = 0; ks < DP / 16; ks++)
#pragma unroll
                    for (int j = 0; j < 2; j++) most = finite_magnitude(most, query_pair(qf[nb][ks][j], p.q_bf16));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
                float up, down;
                query_powers(most, up, down);
#pragma unroll
                for (int ks = 0; ks < DP / 16; ks++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        const float2 f = query_pair(qf[nb][ks][j], p.q_bf16);
                        qf[nb][ks][j] = pack2<__half>(f.x * up, f.y * up);
                    }
                factor[nb][0] = p.scale_log2 * __shfl_sync(0xffffffffu, down, 8 * c);
                factor[nb][1] = p.scale_log2 * __shfl_sync(0xffffffffu, down, 8 * c + 4);
            }
        }
    };
    load_queries(start_at[warp], first_item, qf);

    float o[NB][DP / 16][4], top[NB][2], sum[NB][2];
    float ref[NB][2];  // codes: the running maximum of the scores, which the sum is relative to; `top` has V's scales in it
    // this lane's keys of 16, rows g and g + 8 of S'
    const int key0 = KIND == kPlain ? g : 4 * (g >> 1) + (g & 1), key1 = KIND == kPlain ? g + 8 : key0 + 2;
    int stage = 0, next_fill = R::stages - 1;
    for (int i = 0; i < todo; i++) {
        copy_wait<R::stages - 2>();
        __syncwarp();  // every lane is done with the tile before, whose stage is filled again
        if (l_left > 0) {
            fill(next_fill, ahead);
            ahead = look_up();
        }
        copy_commit();
        next_fill = next_fill + 1 == R::stages ? 0 : next_fill + 1;
        __syncwarp();  // with two stages that was the next tile, whose head is looked at below
        const uint32_t at = ring + stage * R::tile, head_at = heads + stage * R::head;
        uint32_t mask, flags, head_r, head_item;
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(mask), "=r"(flags), "=r"(head_r), "=r"(head_item) : "r"(head_at));
        if (flags & kFirst) {
            take_queries();
#pragma unroll
            for (int nb = 0; nb < NB; nb++) {
#pragma unroll
                for (int k = 0; k < DP / 16; k++) o[nb][k][0] = o[nb][k][1] = o[nb][k][2] = o[nb][k][3] = 0.f;
                top[nb][0] = top[nb][1] = ref[nb][0] = ref[nb][1] = -INFINITY, sum[nb][0] = sum[nb][1] = 0.f;
            }
        }

        // s: keys key0 (0, 1) and key1 (2, 3) of each 16 x columns 2c, 2c + 1
        float s[R::groups][NB][4] = {};
        if constexpr (KIND == kPlain) {
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks++) {
                uint32_t a[4];
                load_matrix4<false>(at + place_of<KIND, DP>(lane & 15, 2 * ks + (lane >> 4)), a);
#pragma unroll
                for (int nb = 0; nb < NB; nb++) mma16816<ST>(s[0][nb], a, qf[nb][ks][0], qf[nb][ks][1]);
            }
        } else {
            const int i = lane & 7, key = 4 * (i >> 1) + (i & 1) + ((lane >> 2) & 2);
#pragma unroll
            for (int ks = 0; ks < DP / 16; ks += 2) {
                const uint32_t from = at + place_of<KIND, DP>(key, ks + (lane >> 4));
                uint32_t w[R::groups][4];  // chunk ks: rows g and g + 8; chunk ks + 1
#pragma unroll
                for (int sub = 0; sub < R::groups; sub++) load_matrix4<false>(from + sub * R::group, w[sub]);
#pragma unroll
                for (int j = 0; j < 2; j++)
#pragma unroll
                    for (int sub = 0; sub < R::groups; sub++) {
                        uint32_t a[4];
                        widen<KIND>(w[sub][2 * j], a[0], a[2]);
                        widen<KIND>(w[sub][2 * j + 1], a[1], a[3]);
#pragma unroll
                        for (int nb = 0; nb < NB; nb++) mma16816<ST>(s[sub][nb], a, qf[nb][ks + j][0], qf[nb][ks + j][1]);
                    }
            }
        }
        // An item's last scores are taken: its queries make room for the next one's, loaded while this tile ends.
        if ((flags & kLast) && i + 1 < todo) {
            const uint32_t next = heads + (stage + 1 == R::stages ? 0 : stage + 1) * R::head;
            uint32_t next_mask, next_flags, r, item;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(next_mask), "=r"(next_flags), "=r"(r), "=r"(item) : "r"(next));
            load_queries(r, static_cast<int>(item), qf);
        }

        float k_scale[R::groups][2], v_log[R::groups][2];
        uint32_t v_sign[R::groups][2];
        if constexpr (KIND != kPlain) {
#pragma unroll
            for (int sub = 0; sub < R::groups; sub++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const uint32_t key = head_at + 16 + (16 * sub + (j ? key1 : key0)) * 4;
                    float v;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(k_scale[sub][j]) : "r"(key));
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(key + 4 * R::keys));
                    // 0: -infinity, a weight of 0; NaN: the weight and with it the outputs, but not the sum
                    v_log[sub][j] = __log2f(fabsf(v)), v_sign[sub][j] = __float_as_uint(v) & 0x80000000u;
                }
        }
        float most[NB][2], most_ref[NB][2];  // of what `top` and `ref` are of
        bool move = false;
#pragma unroll
        for (int nb = 0; nb < NB; nb++) most[nb][0] = most[nb][1] = most_ref[nb][0] = most_ref[nb][1] = -INFINITY;
#pragma unroll
        for (int sub = 0; sub < R::groups; sub++) {
            const bool key[2] = {(mask >> (16 * sub + key0) & 1) != 0, (mask >> (16 * sub + key1) & 1) != 0};
#pragma unroll
            for (int nb = 0; nb < NB; nb++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    float &a = s[sub][nb][j], &b = s[sub][nb][j + 2];
                    if constexpr (KIND == kPlain) a *= factor[nb][j], b *= factor[nb][j];
                    else a *= factor[nb][j] * k_scale[sub][0], b *= factor[nb][j] * k_scale[sub][1];
                    if (!key[0]) a = -INFINITY;
                    if (!key[1]) b = -INFINITY;
                    if constexpr (KIND == kPlain) {
                        most[nb][j] = fmaxf(most[nb][j], fmaxf(a, b));
                    } else {
                        most[nb][j] = fmaxf(most[nb][j], fmaxf(a + v_log[sub][0], b + v_log[sub][1]));
                        most_ref[nb][j] = fmaxf(most_ref[nb][j], fmaxf(a, b));
                    }
                }
        }
#pragma unroll
        for (int nb = 0; nb < NB; nb++)
#pragma unroll
            for (int j = 0; j < 2; j++) move = move || most[nb][j] > top[nb][j] + 8.f || (KIND != kPlain && most_ref[nb][j] > ref[nb][j] + 8.f);
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
                    if constexpr (KIND == kPlain) {
                        sum[nb][j] *= f[j];
                    } else {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) most_ref[nb][j] = fmaxf(most_ref[nb][j], __shfl_xor_sync(0xffffffffu, most_ref[nb][j], x));
                        const float r = fmaxf(ref[nb][j], most_ref[nb][j]);
                        if (r != ref[nb][j]) sum[nb][j] *= exp2_approx(ref[nb][j] - r);
                        ref[nb][j] = r;
                    }
                }
#pragma unroll
                for (int k = 0; k < DP / 16; k++) o[nb][k][0] *= f[0], o[nb][k][1] *= f[1], o[nb][k][2] *= f[0], o[nb][k][3] *= f[1];
            }
        }
        uint32_t pf[R::groups][NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; nb++) {
            const float m0 = top[nb][0] == -INFINITY ? 0.f : top[nb][0] - kLift, m1 = top[nb][1] == -INFINITY ? 0.f : top[nb][1] - kLift;
            const float r0 = ref[nb][0] == -INFINITY ? 0.f : ref[nb][0], r1 = ref[nb][1] == -INFINITY ? 0.f : ref[nb][1];
#pragma unroll
            for (int sub = 0; sub < R::groups; sub++) {
                float (&x)[4] = s[sub][nb];
                if constexpr (KIND != kPlain) {
                    sum[nb][0] += exp2_approx(x[0] - r0) + exp2_approx(x[2] - r0), sum[nb][1] += exp2_approx(x[1] - r1) + exp2_approx(x[3] - r1);
                    x[0] += v_log[sub][0], x[1] += v_log[sub][0], x[2] += v_log[sub][1], x[3] += v_log[sub][1];
                }
                float e0 = exp2_approx(x[0] - m0), e1 = exp2_approx(x[1] - m1), e2 = exp2_approx(x[2] - m0), e3 = exp2_approx(x[3] - m1);
                if constexpr (KIND == kPlain) sum[nb][0] += e0 + e2, sum[nb][1] += e1 + e3;
                if constexpr (KIND != kPlain) {
                    e0 = __uint_as_float(__float_as_uint(e0) ^ v_sign[sub][0]), e1 = __uint_as_float(__float_as_uint(e1) ^ v_sign[sub][0]);
                    e2 = __uint_as_float(__float_as_uint(e2) ^ v_sign[sub][1]), e3 = __uint_as_float(__float_as_uint(e3) ^ v_sign[sub][1]);
                }
                pf[sub][nb][0] = transposed(pack2<VT>(e0, e1));
                pf[sub][nb][1] = transposed(pack2<VT>(e2, e3));
            }
        }

        if constexpr (KIND == kPlain) {
#pragma unroll
            for (int k = 0; k < DP / 16; k++) {
                uint32_t a[4];  // d's 16k .. + 7 and + 8 .., keys 0-7 and 8-15
                load_matrix4<true>(at + R::plane + place_of<KIND, DP>((lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)), a);
#pragma unroll
                for (int nb = 0; nb < NB; nb++) mma16816<VT>(o[nb][k], a, pf[0][nb][0], pf[0][nb][1]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < DP / 16; k += 2) {
                const uint32_t from = at + R::plane + place_of<KIND, DP>(lane & 15, k + (lane >> 4));
                uint32_t w[R::groups][4];
#pragma unroll
                for (int sub = 0; sub < R::groups; sub++) load_codes_transposed(from + sub * R::group, w[sub]);
#pragma unroll
                for (int sub = 0; sub < R::groups; sub++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        uint32_t a[4];
                        widen<KIND>(w[sub][2 * j], a[0], a[2]);
                        widen<KIND>(w[sub][2 * j + 1], a[1], a[3]);
#pragma unroll
                        for (int nb = 0; nb < NB; nb++) mma16816<VT>(o[nb][k + j], a, pf[sub][nb][0], pf[sub][nb][1]);
                    }
            }
        }
        stage = stage + 1 == R::stages ? 0 : stage + 1;

        if (flags & kLast) {
            // The item's part of the keys: a whole part, or one of this warp's two pieces.
            const Item it = item_of(head_r, static_cast<int>(head_item));
            const bool whole = flags & kWhole;
            const int64_t slot = p.split.whole_parts - 1 - (head_r < p.R && p.max_prefix > 0 && p.split.prefix_rows == 16);  // own keys, then the prefix
            const int64_t piece = (static_cast<int64_t>(index) * 2 + (flags & kSecond ? 1 : 0)) * kCols;
#pragma unroll
            for (int nb = 0; nb < NB; nb++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    float all = sum[nb][j];
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) all += __shfl_xor_sync(0xffffffffu, all, x);
                    const int col = 8 * nb + 2 * c + j;
                    const int64_t row = it.row0 + col;
                    if (row >= it.row_end) continue;
                    const int64_t req = quick_div(static_cast<uint32_t>(row), p.div_group);
                    const int64_t where = whole ? slot * p.split.rows + req * p.Hq + it.h * group + (row - req * group) : piece + col;
                    float *dst = (whole ? p.parts : p.pieces) + where * D;
                    const float base = KIND == kPlain ? top[nb][j] : ref[nb][j];
                    const float inv = all == 0.f ? 0.f : 1.f / all, log = all == 0.f ? -INFINITY : (base == -INFINITY ? 0.f : base - (KIND == kPlain ? kLift : 0.f)) + log2f(all);
                    float by = inv;
                    if constexpr (KIND != kPlain) {
                        // outputs are relative to `top`: from there to `ref`, in two steps where fp32 does not hold one
                        float step = top[nb][j] - kLift - (base == -INFINITY ? 0.f : base);
                        if (!(fabsf(step) < 80.f)) {
                            step *= 0.5f;
#pragma unroll
                            for (int k = 0; k < DP / 16; k++) o[nb][k][j] *= exp2_approx(step), o[nb][k][2 + j] *= exp2_approx(step);
                        }
                        by *= exp2_approx(step);
                    }
                    if (whole && p.max_prefix == 0) {
                        // these are all of the row's keys: its output
                        char *out = p.out + req * p.out_req + (it.h * group + (row - req * group)) * p.out_head;
#pragma unroll
                        for (int k = 0; k < DP / 16; k++)
#pragma unroll
                            for (int half = 0; half < 2; half++) {
                                const float x = o[nb][k][2 * half + j] * by;
                                if (16 * k >= D) continue;
                                if (KIND == kPlain ? std::is_same<T, __nv_bfloat16>::value : p.q_bf16) reinterpret_cast<__nv_bfloat16 *>(out)[16 * k + g + 8 * half] = __float2bfloat16_rn(x);
                                else reinterpret_cast<__half *>(out)[16 * k + g + 8 * half] = __float2half_rn(x);
                            }
                        if (g == 0 && p.lse) p.lse[req * p.Hq + it.h * group + (row - req * group)] = log * kLn2;
                        continue;
                    }
#pragma unroll
                    for (int k = 0; k < DP / 16; k++)
#pragma unroll
                        for (int half = 0; half < 2; half++)
                            if (16 * k < D) dst[16 * k + g + 8 * half] = o[nb][k][2 * half + j] * by;
                    if (g == 0) (whole ? p.sums : p.piece_sums)[where] = log;
                }
        }
    }
    copy_wait<0>();
    await_last();  // join_kernel waits for this kernel alone
}

// The parts' outputs, each by its share of the whole sum, with a running maximum.  WARPS warps take a row, each
// some of its parts: one where there are few parts, more where one warp's chain of loads would be long.
// Every lane finds one part - its sum, and where its outputs are - and then the warp reads the outputs of kAhead
// parts at once: what a part without keys (sum -infinity) left in its place is read but not used.
// The latencies of these few loads are all the time there is, so a row's lengths are loaded a row ahead, and where a
// warp takes a row, four loads in flight leave registers for eight CTAs an SM.  Against five CTAs with eight loads, a
// call of 512 requests of 32 heads, e4m3, D = 128, took 149 us for 157 behind a prefix of 4000 and 76 for 81 without.
constexpr int kJoinCtas = 8;
constexpr float kLess = 12.f;  // weights are 2^-12 at most: the outputs of up to that many parts may be next to the largest number
template <typename T, int DP, int WARPS>
__global__ void __launch_bounds__(WARPS == 1 ? 128 : 32 * WARPS, WARPS == 1 ? kJoinCtas : 1) join_kernel(const __grid_constant__ AttnParams p)
{
    constexpr int kVectors = DP <= 128 ? 1 : 2, kAhead = (WARPS == 1 ? 4 : 8) / kVectors;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = p.layer.D, share_of = WARPS == 1 ? 0 : warp;
    __shared__ __align__(16) float others[WARPS == 1 ? 1 : WARPS][WARPS == 1 ? 4 : DP + 4];
    const uint32_t rows = static_cast<uint32_t>(p.split.rows), row_step = WARPS == 1 ? gridDim.x * 4 : gridDim.x;
    uint32_t row = WARPS == 1 ? blockIdx.x * 4 + warp : blockIdx.x;
    if (row >= rows) return;
    const bool prefix_streams = p.max_prefix && p.split.prefix_rows == 16, streams = p.split.stream_ctas > 0;
    int32_t own_len = p.lens[quick_div(row, p.div_heads)];
    const int32_t prefix_len = p.max_prefix ? *p.prefix_len : 0;
    await_last();  // what is read from here on the kernels before this one have written
    const uint4 shares = streams ? *reinterpret_cast<const uint4 *>(p.before) : make_uint4(0, 0, 0, 0);
    const uint32_t prefix_at = prefix_streams ? p.before[4 + p.R] : 0, share = shares.y;
    uint32_t own_at = streams ? p.before[4 + quick_div(row, p.div_heads)] : 0;
    const FastDiv div_share{shares.z, shares.w};
    const uint32_t prefix_keys = min(max(prefix_len, 0), static_cast<int32_t>(p.max_prefix)), chunk = static_cast<uint32_t>(p.split.prefix_chunk);
    const uint32_t front = p.split.prefix_parts ? (prefix_keys + chunk - 1) / chunk * (p.split.prefix_rows == 128 ? 2 : 1) : 0;
    // What the stream left of an item: one whole part, or pieces of warps w0 .. w1.  A warp's first item is its piece 0; only
    // the item's first warp may have begun with another item.
    struct Left {
        uint32_t count, first, next;  // parts; index of the first and the second of them
        bool whole;
    };

    for (; row < rows; row += row_step) {
        const uint32_t r = quick_div(row, p.div_heads), head = row - r * p.Hq, h = quick_div(head, p.div_group), in_group = head - h * p.split.group;
        const int32_t len = own_len;
        const uint32_t at = own_at;
        if (row + row_step < rows) {
            const uint32_t next = quick_div(row + row_step, p.div_heads);
            own_len = p.lens[next];
            if (streams) own_at = p.before[4 + next];
        }
        if (len < 0) continue;
        if (len > p.max_len && head == 0 && lane == 0) atomicOr(p.status, kStatusBadIndex);
        auto left = [&](uint32_t keys, uint32_t begin, uint32_t in_q, uint32_t blocks, uint32_t whole_slot) {
            Left l{0, 0, 0, false};
            const uint32_t tiles = tiles_of(p, keys), columns = p.split.columns, block = blocks > 1 ? in_q / columns : 0, col = in_q - block * columns;
            if (!tiles) return l;
            const uint32_t first = begin + (h * blocks + block) * tiles, w0 = quick_div(first, div_share), w1 = quick_div(first + tiles - 1, div_share);
            l.count = w1 - w0 + 1;
            l.whole = w0 == w1;
            l.first = l.whole ? whole_slot : w0 * 2 * columns + col + (w0 * share < first ? columns : 0);
            l.next = (w0 + 1) * 2 * columns + col;
            return l;
        };
        const Left own = left(min(len, static_cast<int32_t>(p.max_len)), at, in_group, p.split.own_blocks, p.split.whole_parts - (prefix_streams ? 2 : 1));
        if (p.max_prefix == 0 && own.whole) continue;  // the stream has written the output
        Left shared{0, 0, 0, false};
        if (prefix_streams) shared = left(prefix_keys, prefix_at, r * p.split.group + in_group, p.split.prefix_blocks, p.split.whole_parts - 1);
        const uint32_t n = front + own.count + shared.count, from = n * share_of / WARPS, to = n * (share_of + 1) / WARPS;

        float acc[4 * kVectors] = {}, all = 0.f, top = -INFINITY;
        for (uint32_t i0 = from; i0 < to; i0 += 32) {
            // this lane's part: prefix_kernel's, then those of the own keys, then those of a prefix in the stream
            const uint32_t i = min(i0 + lane, to - 1), q = i - front;
            const bool mine = q < own.count;
            const Left &l = mine ? own : shared;
            const uint32_t k = mine ? q : q - own.count;
            const bool whole = i < front || l.whole;
            const int64_t index = i < front ? static_cast<int64_t>(i) * rows + row
                                  : l.whole ? static_cast<int64_t>(l.first) * rows + row
                                            : static_cast<int64_t>(k == 0 ? l.first : l.next + (k - 1) * 2 * p.split.columns);
            const float *outputs = (whole ? p.parts : p.pieces) + index * D;
            const float sum = i0 + lane < to ? (whole ? p.sums : p.piece_sums)[index] : -INFINITY;
            const int here = static_cast<int>(min(to - i0, 32u));
            float weight = 0.f;
#pragma unroll 1
            for (int j0 = 0; j0 < here; j0 += kAhead) {
                float4 v[kAhead][kVectors];
#pragma unroll
                for (int j = 0; j < kAhead; j++) {
                    const float *src = reinterpret_cast<const float *>(__shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(outputs), min(j0 + j, here - 1))) + lane * 4;
#pragma unroll
                    for (int x = 0; x < kVectors; x++) {
                        v[j][x] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (j0 + j < here && lane * 4 + 128 * x < D) v[j][x] = *reinterpret_cast<const float4 *>(src + 128 * x);
                    }
                }
                if (j0 == 0) {
                    float m = sum;
#pragma unroll
                    for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                    if (m > top) {
                        const float f = exp2_approx(top - m);
#pragma unroll
                        for (int x = 0; x < 4 * kVectors; x++) acc[x] *= f;
                        all *= f;
                        top = m;
                    }
                    weight = sum == -INFINITY ? 0.f : exp2_approx(sum - (top == -INFINITY ? 0.f : top) - kLess);  // NaN where the sum is
                    float add = weight;
#pragma unroll
                    for (int x = 16; x; x >>= 1) add += __shfl_xor_sync(0xffffffffu, add, x);
                    all += add;
                }
#pragma unroll
                for (int j = 0; j < kAhead; j++) {
                    const float w = __shfl_sync(0xffffffffu, weight, (j0 + j) & 31);
                    if (w == 0.f || j0 + j >= here) continue;
#pragma unroll
                    for (int x = 0; x < kVectors; x++) acc[4 * x] += w * v[j][x].x, acc[4 * x + 1] += w * v[j][x].y, acc[4 * x + 2] += w * v[j][x].z, acc[4 * x + 3] += w * v[j][x].w;
                }
            }
        }
        if constexpr (WARPS > 1) {
#pragma unroll
            for (int x = 0; x < kVectors; x++)
                if (lane * 4 + 128 * x < DP) *reinterpret_cast<float4 *>(&others[warp][lane * 4 + 128 * x]) = make_float4(acc[4 * x], acc[4 * x + 1], acc[4 * x + 2], acc[4 * x + 3]);
            if (lane == 0) others[warp][DP] = all, others[warp][DP + 1] = top;
            __syncthreads();
            if (warp) return;  // a CTA takes one row
            for (int w = 0; w < WARPS; w++) top = fmaxf(top, others[w][DP + 1]);
            const float base = top == -INFINITY ? 0.f : top;
            all = 0.f;
#pragma unroll
            for (int x = 0; x < 4 * kVectors; x++) acc[x] = 0.f;
            for (int w = 0; w < WARPS; w++) {
                const float part = others[w][DP], part_top = others[w][DP + 1];
                if (part == 0.f) continue;
                const float f = part_top == -INFINITY ? 1.f : exp2_approx(part_top - base);  // -infinity: all of its sums are NaN
                all += f * part;
#pragma unroll
                for (int x = 0; x < kVectors; x++)
                    if (lane * 4 + 128 * x < DP)
#pragma unroll
                        for (int k = 0; k < 4; k++) acc[4 * x + k] += f * others[w][lane * 4 + 128 * x + k];
            }
        }
        const float inv = all == 0.f ? 0.f : 1.f / all;
        char *dst = p.out + r * p.out_req + head * p.out_head;
#pragma unroll
        for (int x = 0; x < kVectors; x++)
            if (lane * 4 + 128 * x < D)
                *reinterpret_cast<uint2 *>(dst + (lane * 4 + 128 * x) * 2) = make_uint2(pack2<T>(acc[4 * x] * inv, acc[4 * x + 1] * inv), pack2<T>(acc[4 * x + 2] * inv, acc[4 * x + 3] * inv));
        if (p.lse && lane == 0) p.lse[row] = all == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + kLess + log2f(all)) * kLn2;
        if (WARPS > 1) return;
    }
}

// --------------------------------------------------------------------------------------- launching
template <typename T, int KIND, int DP, int NB>
static int launch_stream(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    using R = Ring<KIND, DP>;
    static std::atomic<bool> raised[kMaxDevices];  // set once per device; setting it twice does no harm
    if (!raised[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(stream_kernel<T, KIND, DP, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, R::bytes);
        if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(dynamic shared memory)");
        raised[device].store(true, std::memory_order_relaxed);
    }
    return launch_attn(stream_kernel<T, KIND, DP, NB>, grid, 128, R::bytes, p.split.prefix_parts > 0, p, s);
}

template <typename T, int KIND, int NB>
static int launch_stream_for(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    if (p.layer.D <= 64) return launch_stream<T, KIND, 64, NB>(p, grid, device, s);
    if (p.layer.D <= 128) return launch_stream<T, KIND, 128, NB>(p, grid, device, s);
    return launch_stream<T, KIND, 256, NB>(p, grid, device, s);
}

template <typename T, int KIND>
static int launch_stream_columns(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    return p.split.columns == 8 ? launch_stream_for<T, KIND, 1>(p, grid, device, s) : launch_stream_for<T, KIND, 2>(p, grid, device, s);
}

template <typename T>
static int launch_decode(const AttnParams &p, int device, cudaStream_t s)
{
    int rc = TC_OK;
    if (p.split.prefix_parts && (rc = launch_prefix(p, std::is_same<T, __half>::value ? TC_FP16 : TC_BF16, device, s)) != TC_OK) return rc;
    if (p.split.stream_ctas) {
        const unsigned grid = static_cast<unsigned>(p.split.stream_ctas);
        switch (p.layer.dtype) {
        case TC_E4M3: rc = launch_stream_columns<__half, kE4m3>(p, grid, device, s); break;
        case TC_INT8: rc = launch_stream_columns<__half, kInt8>(p, grid, device, s); break;
        default: rc = launch_stream_columns<T, kPlain>(p, grid, device, s); break;
        }
        if (rc != TC_OK) return rc;
    }
    // parts of a row: the prefix kernel's, and about as many as warps share one item of the stream
    const int64_t parts = p.split.prefix_parts + p.split.stream_ctas * 4 / std::max<int64_t>(p.R * p.layer.H * p.split.own_blocks, 1);
    const unsigned rows = static_cast<unsigned>(p.split.rows);
    // Few rows of many parts: 16 warps a row.  One context of 65536 int8 tokens 29 us so, 92 with a warp a row; three of 65k to
    // 131k 69 and 98; 64 requests of some 256 tokens (2048 rows) 59 so and 27 with a warp a row.
    const bool wide = parts > 32 && rows < 1024;
    const unsigned few = std::min<unsigned>((rows + 3) / 4, kSms * kJoinCtas);
    const bool follows = p.split.prefix_parts || p.split.stream_ctas;
    if (p.layer.D <= 128) return wide ? launch_attn(join_kernel<T, 128, 16>, rows, 512, 0, follows, p, s) : launch_attn(join_kernel<T, 128, 1>, few, 128, 0, follows, p, s);
    return wide ? launch_attn(join_kernel<T, 256, 16>, rows, 512, 0, follows, p, s) : launch_attn(join_kernel<T, 256, 1>, few, 128, 0, follows, p, s);
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
    if (a->reserved) return fail(TC_ERR_INVALID_ARG, "reserved is %d, not 0", a->reserved);
    if (!(std::fabs(a->scale) <= 1e30f)) return fail(TC_ERR_INVALID_ARG, "scale is not a number of at most 1e30");
    if (a->R * p->layer.H > (1 << 30) / std::max<int64_t>(1, (a->max_len + 15) / 16)) return fail(TC_ERR_TOO_LARGE, "R * H * max_len = %lld * %d * %lld: too many keys for one call", (long long)a->R, p->layer.H, (long long)a->max_len);
    split_attn(a->R, a->Hq, p->layer.H, D, a->max_len, a->max_prefix, p->layer.quantised(), &p->split);
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
    p.div_heads = make_fastdiv(static_cast<uint32_t>(p.Hq));
    char *const ws = static_cast<char *>(a->workspace);
    p.sums = reinterpret_cast<float *>(ws + p.split.sums_at);
    p.parts = reinterpret_cast<float *>(ws + p.split.parts_at);
    p.piece_sums = reinterpret_cast<float *>(ws + p.split.piece_sums_at);
    p.pieces = reinterpret_cast<float *>(ws + p.split.pieces_at);
    p.before = reinterpret_cast<uint32_t *>(ws + p.split.before_at);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return a->dtype == TC_BF16 ? launch_decode<__nv_bfloat16>(p, device, s) : launch_decode<__half>(p, device, s);
}
