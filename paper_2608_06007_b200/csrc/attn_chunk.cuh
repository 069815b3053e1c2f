// tc_attn_chunk: attention of chunks of new tokens over a paged cache, on the fifth-generation tensor cores.
//
// Mathematics.  The rows of a request and KV head are its (new token, query head of the group) pairs, token by token, 256 at a time (head
// dims above 128: 128), so that a tile of K and V meets all heads that share it.  Over the tiles of keys that some row sees, one
// pass: S = Q K' to tensor memory; a thread has a row, t = max(t, S scale), P = 2^(S scale - t) to tensor memory, l += sum P; O += P V there.
// All exponents are of 2, the scale has log2(e) in it.  t moves only when a score exceeds it by more than 8: till then P is at most 2^8, and O
// is not touched; what O and l hold is rescaled when it does, and the last t and l give the outputs and their logarithm.  S, t, l and O are
// fp32; P is rounded once to the products' 16 bits, fp16 with 2^7 taken in (probability_lift), so that what is below 2^-21 of the
// row's largest is what its smallest steps lose.
// Codes are fp16 exactly.  K's scale multiplies the scores.  V's multiplies the probabilities in fp32, before their one rounding,
// as a power of two that the whole tile has, which goes into the exponent, and a rest below 1; where scales within a tile are more than 2^16 apart,
// or a tile's largest is 2^40 below one before, each key has a power of its own (far_maxima, far_probabilities).  Queries that
// meet codes are fp16 with a power of two per row taken out.
//
// What a row does not see must not reach it, not even as 0 x NaN: of a tile in which rows differ, the warps that fetch V look whether
// it has numbers that are not finite, and the rows' sums over such a tile are made one number at a time (spoiled_tile).  Keys
// that no row sees are 0 in shared memory, or cut off by the tile's mask.
//
// Warps.  Eight of softmax, a thread a row; four that fetch (codes: eight that also widen); one each issues S and O products; one finds
// the items.  Two slots of 128 rows go through a tile, so that one's products run beside the other's exponentials.  Items are
// independent CTAs of a grid as large as the largest batch that the bounds allow; a CTA that nears the end of one takes over
// another that has not been launched (try_cancel) and goes on without a gap, since the lengths are known on the device alone.
//
// What bounds it.  Two slots' products take 2048 clocks a tile of 128 keys at D = 128, and as many the exponentials, at 16 a clock
// and SM; a slot's softmax is a chain of some 3000 (load 250, maximum 450, exponentials 1600, the rest and stores 600), of which two run side by
// side.  Measured: 2048 tokens behind 6144 of 32 heads over 8 KV heads, bf16: 215 us, 1.12 PFLOP/s, 0.67 of a library's large product, and 247 us, 0.97
// PFLOP/s, under the power cap of a long run; 8192 behind 24576, 64 heads: 6.8 ms, 1.13 PFLOP/s, and 7.1.  Two threads a row (16 warps of softmax) were slower, 290 us: half the registers, and both
// halves of a row wait for one another.  K and V have their own warps: with one for both, V's wait for a free stage held K's next back.
// Codes that each CTA widens itself: 33 tokens behind 120000 of 28 heads over 4, int8: 151 us.  A slot's chain bounds it, 6100 clocks a
// tile: its scores wait for the product before, whose probabilities lie in their place (1800), two passes (1500, 2400), the product; the eight
// widening warps take 3500.  One pass with the old maximum, probabilities in registers till it is known, was slower, 168 us: its code is long
// and six warps of four kinds share a scheduler's instruction cache.  Requests of many blocks go another way (attn_chunk_wide.cu).
#pragma once

#include <algorithm>
#include <atomic>

#include "attn_chunk.h"
#include "attn_tensor.cuh"

namespace tc {

constexpr float kChunkLn2 = 0.6931471805599453f;

// Codes that attn_chunk_wide.cu has made fp16, tile by tile, before: their scales still come with the scores.
constexpr int kWide = 3;
template <int KIND> constexpr bool kWidens = KIND == kE4m3 || KIND == kInt8;

// A CTA's warps: eight of softmax, those that fetch pages (codes: four for K and four for V), then four that issue products and find items.
template <int KIND> struct ChunkWarps {
    static constexpr int softmax = 8, loaders = kWidens<KIND> ? 8 : 4, all = softmax + loaders + 4, threads = 32 * all;
    // registers of a thread: at the launch, of the softmax, of the others
    static constexpr int launch_registers = kWidens<KIND> ? 96 : 128, softmax_registers = kWidens<KIND> ? 112 : 192, other_registers = kWidens<KIND> ? 80 : 64;
    static_assert(32 * softmax * softmax_registers + (threads - 32 * softmax) * other_registers <= threads * launch_registers && threads * launch_registers <= 65536, "a split that never ends");
};

template <int KIND, int DP>
struct ChunkMemory {
    static constexpr int slots = DP > 128 ? 1 : 2, keys = DP > 128 ? 64 : 128;
    static constexpr int tile = keys * DP * 2, q_tile = 128 * DP * 2;  // bytes
    static constexpr int queries = slots * q_tile;
    static constexpr int stages = DP == 64 ? 6 : 4;  // K and V in turn, so that each stage is always one's
    // Tiles whose masks and scales are kept: those of a tile must not be replaced before its last product is issued, and
    // K and V have their own warps, of which K's may be four tiles ahead.
    static constexpr int infos = 8;
    // {mask, 4 words; whether V has numbers that are not finite, up to 4 words}; codes: V's exponent, whether scales are far apart; each
    // warp's largest and smallest of V's scales; scales of K; keys' exponents; scales of V over the power of two
    static constexpr int info = KIND == kPlain ? 32 : 80 + 12 * keys, scales = 80;
    // Powers of two taken out of the queries, of four items: an item's are written when its scores may be, and read by a slot whose softmax may be at
    // the item before the last.  (It is no further behind: an item is published when all warps have taken the one before the last.)
    static constexpr int down_sets = 4, downs = KIND == kPlain ? 0 : down_sets * slots * 128 * 4;
    static constexpr int table = 2 * ChunkWarps<KIND>::threads * 4;  // items, and rows of parts, before each thread's requests
    static constexpr int item = 80;
    static constexpr int rest = infos * info + downs + table + 2 * item + 16 + 512;
    // more than half of an SM's, so that no two CTAs meet on one: the second would wait for tensor memory with an item in hand
    static constexpr int least = 120 * 1024;
    static constexpr int used = queries + stages * tile + rest + 1024;
    static constexpr int bytes = used > least ? used : least;
};

// One item as it lies in shared memory.
struct alignas(16) ChunkItem {
    int32_t valid, r, h, row0;       // valid: 0 = the end, 2 = the slots take turns at the tiles; r: of tiles that were made fp16, their place
    int32_t rows, pos0, begin, end;  // the part: tiles [begin, end) of the list
    ChunkList list;                  // 7 words
    uint32_t part_row;               // of the request's row 0 of this part; kUncut: outputs are written
    int64_t token0;                  // row of q that is the request's first new token
    int32_t firsts, skip;            // of the request's list of tiles, where those lie ready
};
static_assert(sizeof(ChunkItem) == 80);

struct ChunkRequest {
    int64_t token0;
    int32_t n, len;  // n = 0: nothing is done for it
};
__device__ __forceinline__ ChunkRequest chunk_request(const ChunkParams &p, int64_t r, bool tell)
{
    ChunkRequest q;
    const int64_t to = p.offsets[r + 1];
    q.token0 = p.offsets[r], q.len = p.lens[r];
    const int64_t n = to - q.token0;
    const bool bad = q.token0 < 0 || to < q.token0 || to > p.n_tokens || n > p.max_new || (q.len >= 0 && (q.len > p.max_len || q.len < n));
    if (tell && bad) atomicOr(p.status, kStatusBadIndex);
    q.n = bad || q.len < 0 || n < p.new_from || n > p.new_to ? 0 : static_cast<int32_t>(n);
    return q;
}

// Which of the places for tiles made fp16 are request r's.
__device__ __forceinline__ int64_t wide_place(const ChunkParams &p, int64_t r, int64_t token0) { return p.wide_by_request ? r : quick_div(static_cast<uint32_t>(token0), p.div_wide); }

// Any of two 16-bit numbers infinite or NaN.
template <typename T> __device__ __forceinline__ uint32_t not_finite(uint32_t w)
{
    constexpr uint32_t exponent = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u, last = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
    return ((w & exponent) + last) & 0x80008000u;
}

constexpr int32_t kNoKey = INT32_MIN;  // no entry of a table

// A box of a tensor map's tokens t .. of one head and block, elements x .. , to shared memory.
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap *map, int x, int t, int h, int block, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(t), "r"(h), "r"(block), "r"(bar) : "memory");
}

__device__ __forceinline__ void copy_box3(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// A run of bytes, a multiple of 16, to shared memory.
__device__ __forceinline__ void copy_run(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// A scale of V as a power of two, of its own or its tile's, and the rest, which multiplies the probabilities.
constexpr int kLeastExponent = -126;
struct ScaleOfV {
    float scale;
    uint32_t size;  // bits of its magnitude; of a NaN 0, so that it is passed over
    // 2 to this power is above the magnitude
    __device__ __forceinline__ static int exponent_of(uint32_t size) { return static_cast<int>(size >> 23) - 126; }
    // far: the key's own, else the tile's; a key of scale 0 takes no part in the maximum where each has its own
    __device__ __forceinline__ float exponent(bool far, int tile) const { return scale == 0.f ? -4096.f : static_cast<float>(far ? exponent_of(size) : tile); }
    __device__ __forceinline__ float rest(bool far, int tile) const
    {
        const int e = far ? exponent_of(size) : tile, half = e >> 1;  // 2^-e, from 2^-129 to 2^126, in two factors
        return scale * __uint_as_float(static_cast<uint32_t>(127 - half) << 23) * __uint_as_float(static_cast<uint32_t>(127 - (e - half)) << 23);
    }
};

__device__ __forceinline__ ScaleOfV scale_of_v(float scale)
{
    const uint32_t size = __float_as_uint(scale) & 0x7fffffffu;
    return ScaleOfV{scale, size > 0x7f800000u ? 0u : size};
}

// Bits 0 .. n - 1.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// What a row sees of a tile: the tile's mask, and keys below `upper`, from `lower` on or below `firsts`.
struct RowView {
    uint32_t mask_at;
    int upper, lower, firsts;
    __device__ __forceinline__ uint32_t word(int c) const
    {
        uint32_t there;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(there) : "r"(mask_at + 4 * c));
        return there & low_bits(upper - 32 * c) & (~low_bits(lower - 32 * c) | low_bits(firsts - 32 * c));
    }
};

// Rare: V has numbers that are not finite in a tile that not every row sees all of.  The second product would give 0 times such
// a number to rows that do not see its key, so here each row adds up what it sees.
template <typename T, int DP, int KEYS>
__device__ __noinline__ void spoiled_tile(uint32_t p_at, uint32_t o_at, uint32_t v, RowView view, bool first)
{
#pragma unroll 1
    for (int c = 0; c < DP / 16; c++) {
        uint32_t acc[16];
#pragma unroll
        for (int i = 0; i < 16; i++) acc[i] = 0;
        if (!first) tensor_load16(o_at + 16 * c, acc);
        tensor_loaded();
#pragma unroll 1
        for (int k = 0; k < KEYS; k++) {
            uint32_t pair, x[8];
            asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(pair) : "r"(p_at + (k >> 1)));
            tensor_loaded();
            const float2 both = unpack2<T>(pair);
            const bool seen = view.word(k >> 5) >> (k & 31) & 1;
            const float weight = k & 1 ? both.y : both.x;
            const int chunk = 2 * c;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(v + swizzled<KEYS>(k, chunk)));
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]) : "r"(v + swizzled<KEYS>(k, chunk + 1)));
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float2 f = unpack2<T>(x[i]);
                const float a = __uint_as_float(acc[2 * i]), b = __uint_as_float(acc[2 * i + 1]);
                acc[2 * i] = __float_as_uint(seen ? fmaf(weight, f.x, a) : a), acc[2 * i + 1] = __float_as_uint(seen ? fmaf(weight, f.y, b) : b);
            }
            __syncwarp();
        }
        tensor_store16(o_at + 16 * c, acc);
    }
    tensor_stored();
}

// Rare: scales of V so far apart that what is next to nothing among the probabilities can be much of the sum.  Each key has its
// own power of two here, and the sum exponentials of its own; the scores stay in tensor memory and are gone through twice, 16 at a time:
// for the row's maxima, then for the probabilities.  scales: of the tile's K, then exponents and the rest of V's.
template <int KEYS>
__device__ __noinline__ float2 far_maxima(uint32_t s_at, RowView view, uint32_t scales, float factor)
{
    float highest = -INFINITY, most = -INFINITY;
#pragma unroll 1
    for (int c = 0; c < KEYS / 16; c++) {
        uint32_t v[16];
        tensor_load16(s_at + 16 * c, v);
        const uint32_t here = view.word(c >> 1) >> 16 * (c & 1);
        tensor_loaded();
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 k4 = load_shared_f4(scales + 4 * (16 * c + i)), e4 = load_shared_f4(scales + 4 * KEYS + 4 * (16 * c + i));
            const float k[4] = {k4.x, k4.y, k4.z, k4.w}, e[4] = {e4.x, e4.y, e4.z, e4.w};
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const float x = here >> (i + j) & 1 ? __uint_as_float(v[i + j]) * (factor * k[j]) : -INFINITY;
                highest = fmaxf(highest, x), most = fmaxf(most, x + e[j]);
            }
        }
    }
    return make_float2(highest, most);
}
// Probabilities relative to m, to p_at; the sum of exponentials relative to `ref`.
template <int KEYS>
__device__ __noinline__ float far_probabilities(uint32_t s_at, uint32_t p_at, RowView view, uint32_t scales, float factor, float ref, float m)
{
    float sum = 0.f;
#pragma unroll 1
    for (int c = 0; c < KEYS / 16; c++) {
        uint32_t v[16], w[8];
        tensor_load16(s_at + 16 * c, v);
        const uint32_t here = view.word(c >> 1) >> 16 * (c & 1);
        tensor_loaded();
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 k4 = load_shared_f4(scales + 4 * (16 * c + i)), e4 = load_shared_f4(scales + 4 * KEYS + 4 * (16 * c + i));
            const float4 f4 = load_shared_f4(scales + 8 * KEYS + 4 * (16 * c + i));
            const float k[4] = {k4.x, k4.y, k4.z, k4.w}, e[4] = {e4.x, e4.y, e4.z, e4.w}, f[4] = {f4.x, f4.y, f4.z, f4.w};
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                x[j] = here >> (i + j) & 1 ? __uint_as_float(v[i + j]) * (factor * k[j]) : -INFINITY;
                sum += exp2_approx(x[j] - ref);
                x[j] = exp2_approx(x[j] + e[j] - m) * f[j];
            }
            w[i / 2] = pack2<__half>(x[0], x[1]), w[i / 2 + 1] = pack2<__half>(x[2], x[3]);
        }
        tensor_store8(p_at + 8 * c, w);
    }
    return sum;
}

// Where a wait ran out: boxes and runs may still be on their way to this CTA's shared memory, whoever asked for them.  Their barriers' phases end when
// they are there; one that has none runs out.  bars_at: of `full`, in what the kernel has laid out.
template <int STAGES>
__device__ __noinline__ void copies_landed(uint32_t bars_at)
{
    extern __shared__ unsigned char raw[];
    const uint32_t full = ((static_cast<uint32_t>(__cvta_generic_to_shared(raw)) + 1023) & ~1023u) + bars_at, i = threadIdx.x, q_full = full + 16 * STAGES + 64;
    // q_full, answered, landed
    const uint32_t bar = i < STAGES ? full + 8 * i : i == STAGES ? q_full : i == STAGES + 1 ? q_full + 56 : q_full + 80 + 8 * (i & 1);
    if (i < STAGES + 4) barrier_wait(bar, barrier_passed(bar, 0));
}

// T: the type of the products, fp16 for codes.
template <typename T, int KIND, int DP>
__global__ void __launch_bounds__(ChunkWarps<KIND>::threads, 1) chunk_kernel(const __grid_constant__ ChunkParams p)
{
    using M = ChunkMemory<KIND, DP>;
    using W = ChunkWarps<KIND>;
    // kMine: keys of a tile that a warp fetches
    constexpr int kKeys = M::keys, kSlots = M::slots, kMine = kKeys / 4, kWords = kKeys / 32, kLoad = W::softmax, kIssue = kLoad + W::loaders;
    // Tiles made fp16: 8 prompts in a window of 2048, int8, 1.92 ms so, 2.11 where the compiler unrolls its waits.  Where codes are widened here it is
    // the other way, for want of registers: 33 tokens behind 120000, int8, 191 us so and 151.
    constexpr bool kRolled = KIND == kWide;
    constexpr float kLift = probability_lift<T>();
    extern __shared__ unsigned char raw[];
    allow_next();
    const uint32_t base = (static_cast<uint32_t>(__cvta_generic_to_shared(raw)) + 1023) & ~1023u;
    unsigned char *const gen = raw + (base - static_cast<uint32_t>(__cvta_generic_to_shared(raw)));
    constexpr int kRingAt = M::queries, kInfoAt = kRingAt + M::stages * M::tile, kDownsAt = kInfoAt + M::infos * M::info, kTableAt = kDownsAt + M::downs,
                  kItemsAt = kTableAt + M::table, kAnswerAt = kItemsAt + 2 * M::item, kBarsAt = kAnswerAt + 16;
    static_assert(kInfoAt % 16 == 0 && kItemsAt % 16 == 0 && kAnswerAt % 16 == 0);
    const uint32_t ring = base + kRingAt, info = base + kInfoAt;
    const uint32_t full = base + kBarsAt, empty = full + 8 * M::stages, s_full = empty + 8 * M::stages, s_taken = s_full + 16, p_ready = s_taken + 16, o_added = p_ready + 16;
    const uint32_t q_full = o_added + 16, q_empty = q_full + 8, item_full = q_empty + 8, item_empty = item_full + 16, wanted = item_empty + 16, answered = wanted + 8, last_at = answered + 8, landed = last_at + 16, tensor_at = landed + 16;
    static_assert(8 * (2 * M::stages + 20) + 8 <= 512);
    uint32_t *const items_before = reinterpret_cast<uint32_t *>(gen + kTableAt), *const rows_before = items_before + W::threads;
    ChunkItem *const items = reinterpret_cast<ChunkItem *>(gen + kItemsAt);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, D = p.layer.D, H = p.layer.H;
    const ChunkShape &shape = p.shape;

    if (threadIdx.x == 0) {
        // boxes announce themselves to whoever waits for their bytes; copies key by key for their lanes, and a lane of each warp what it has written beside them
        const int ready = KIND == kWide ? 1 : KIND != kPlain ? 128 : p.box_rows ? 2 : 2 * 33;
        for (int i = 0; i < M::stages; i++) barrier_init(full + 8 * i, ready), barrier_init(empty + 8 * i, 1);
        for (int i = 0; i < 2; i++) barrier_init(landed + 8 * i, 1);
        for (int i = 0; i < 2; i++) barrier_init(s_full + 8 * i, 1), barrier_init(s_taken + 8 * i, 128), barrier_init(p_ready + 8 * i, 128), barrier_init(o_added + 8 * i, 1);
        for (int i = 0; i < 2; i++) barrier_init(item_full + 8 * i, 1), barrier_init(item_empty + 8 * i, kSlots * 4 + W::loaders + 2 + (KIND != kPlain && p.q_boxes ? 1 : 0)), barrier_init(last_at + 8 * i, 1);
        barrier_init(q_full, KIND != kPlain ? 32 * W::loaders : p.q_boxes ? 1 : 4 * 33), barrier_init(q_empty, 1), barrier_init(wanted, 1), barrier_init(answered, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssue) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tensor_at) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }

    // Both slots have an item's rows and take turns at its tiles; parts that an item so leaves.
    constexpr bool kTurns = kWidens<KIND> && kSlots == 2;
    auto turns = [](const ChunkItem &item) { return kTurns && item.valid == 2; };
    auto each_leaves = [&](int32_t n, int32_t parts) { return kTurns && chunk_turns(shape, n, parts) ? 2 : 1; };

    // ------------------------------------------------------------------- the cut, the same in every CTA
    // Each thread has a run of requests, of which it keeps the first.
    __shared__ int32_t sum_items[W::all], sum_tiles[W::all], best_share[16];
    __shared__ float best_cost[16];
    __shared__ uint32_t warp_items[W::all], warp_rows[W::all];
    const int64_t per = (p.R + W::threads - 1) / W::threads, run0 = min(threadIdx.x * per, p.R), run1 = min(run0 + per, p.R);
    struct Extent {
        int32_t n, blocks, tiles;  // new tokens, items of all heads, uncut, and tiles of one
    };
    auto extent_of = [&](int64_t r, bool tell) {
        const ChunkRequest q = chunk_request(p, r, tell);
        return q.n ? Extent{q.n, chunk_blocks(shape, q.n) * H, chunk_tiles(shape, q.len)} : Extent{0, 0, 0};
    };
    const Extent first = run0 < run1 ? extent_of(run0, true) : Extent{0, 0, 0};
    int32_t share = 1 << 30;
    if (p.plan.part_rows) {
        int32_t n_items = first.blocks, most = first.tiles;
        for (int64_t r = run0 + 1; r < run1; r++) {
            const Extent e = extent_of(r, false);
            n_items = min(n_items + e.blocks, 1 << 20), most = max(most, e.tiles);
        }
        n_items = __reduce_add_sync(0xffffffffu, min(n_items, 1 << 20));
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) sum_items[warp] = n_items, sum_tiles[warp] = most;
        items_before[threadIdx.x] = first.blocks, rows_before[threadIdx.x] = first.tiles;  // for the search
        __syncthreads();
        n_items = lane < W::all ? sum_items[lane] : 0, most = lane < W::all ? sum_tiles[lane] : 0;
        n_items = __reduce_add_sync(0xffffffffu, n_items), most = __reduce_max_sync(0xffffffffu, most);
        if (n_items < kChunkEnough && most > kChunkLeastShare) {
            if (warp < 16) {
                // warp w looks at cuts w and w + 16
                ChunkCost sum[2];
                const int32_t shares[2] = {chunk_share(most, warp), chunk_share(most, warp + 16)};
                const float inverse[2] = {1.f / shares[0], 1.f / shares[1]};
                for (int64_t r = lane; r < p.R; r += 32) {
                    const Extent e = per == 1 ? Extent{1, static_cast<int32_t>(items_before[r]), static_cast<int32_t>(rows_before[r])} : extent_of(r, false);
#pragma unroll
                    for (int c = 0; c < 2; c++) sum[c].add(e.blocks, e.tiles, shares[c], static_cast<int32_t>((static_cast<float>(e.tiles + shares[c] - 1) + 0.5f) * inverse[c]));
                }
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    sum[c].items = __reduce_add_sync(0xffffffffu, sum[c].items), sum[c].split = __reduce_add_sync(0xffffffffu, sum[c].split);
                    sum[c].tiles = __reduce_add_sync(0xffffffffu, sum[c].tiles), sum[c].longest = __reduce_max_sync(0xffffffffu, sum[c].longest);
                    sum[c].large = __reduce_add_sync(0xffffffffu, sum[c].large), sum[c].rest = __reduce_add_sync(0xffffffffu, sum[c].rest);
                }
                const float cost0 = chunk_cost(sum[0]), cost1 = chunk_cost(sum[1]);
                if (lane == 0) best_cost[warp] = min(cost0, cost1), best_share[warp] = cost1 < cost0 ? shares[1] : shares[0];
            }
            __syncthreads();
            float cost = 3e38f;
            for (int w = 0; w < 16; w++)
                if (best_cost[w] < cost || (best_cost[w] == cost && best_share[w] > share)) cost = best_cost[w], share = best_share[w];
        } else {
            __syncthreads();
        }
    }
    uint32_t total;
    for (;;) {
        uint32_t my_items = 0, my_rows = 0;
        for (int64_t r = run0; r < run1; r++) {
            const Extent e = r == run0 ? first : extent_of(r, true);
            const int32_t parts = e.tiles > share ? chunk_parts(e.tiles, share) : 1;
            my_items += e.blocks * parts;
            if (parts > 1) my_rows += static_cast<uint32_t>(e.n) * p.Hq * parts * each_leaves(e.n, parts);
        }
        uint32_t upto = my_items, rows_upto = my_rows;
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) {
            const uint32_t a = __shfl_up_sync(0xffffffffu, upto, x), b = __shfl_up_sync(0xffffffffu, rows_upto, x);
            if (lane >= x) upto += a, rows_upto += b;
        }
        if (lane == 31) warp_items[warp] = upto, warp_rows[warp] = rows_upto;
        __syncthreads();
        const uint32_t theirs = lane < W::all ? warp_items[lane] : 0, their_rows = lane < W::all ? warp_rows[lane] : 0;
        total = __reduce_add_sync(0xffffffffu, theirs);
        if (!chunk_has_room(p.plan.part_rows, __reduce_add_sync(0xffffffffu, their_rows))) {
            share = 1 << 30;
            __syncthreads();
            continue;
        }
        upto += __reduce_add_sync(0xffffffffu, lane < warp ? theirs : 0), rows_upto += __reduce_add_sync(0xffffffffu, lane < warp ? their_rows : 0);
        items_before[threadIdx.x] = upto - my_items, rows_before[threadIdx.x] = rows_upto - my_rows;
        break;
    }
    fence_before();
    __syncthreads();
    fence_after();
    // All 512 columns are this CTA's, so they begin at 0; a constant lets the products' operands stay in uniform registers.
    // A softmax holds a tile's scores in registers and gives their one buffer back at once, beside the two slots' probabilities;
    // of codes, whose warps leave it few registers, it goes through them twice where they lie, and puts the probabilities in their place.
    constexpr bool kInPlace = kWidens<KIND> && kSlots == 2;
    constexpr uint32_t tensor = 0, kScores = 0, kScoresStep = kInPlace ? 128 : 0, kProbabilities = kInPlace ? 0 : 128, kProbabilitiesStep = kInPlace ? 128 : 64, kOutputs = 256;
    bool fine = true;  // no wait of this thread has run out

    // Item `it` of this CTA's; false when there is none, or a wait ran out.
    auto take_item = [&](int it, ChunkItem &item) {
        if (!__all_sync(0xffffffffu, barrier_wait<kRolled>(item_full + 8 * (it & 1), (it >> 1) & 1, p.item_spins))) {
            fine = false;
            return false;
        }
        const uint4 *src = reinterpret_cast<const uint4 *>(items + (it & 1));
        uint4 *dst = reinterpret_cast<uint4 *>(&item);
#pragma unroll
        for (int i = 0; i < 5; i++) dst[i] = src[i];
        __syncwarp();
        if (lane == 0) barrier_arrive(item_empty + 8 * (it & 1));
        return item.valid != 0;
    };
    // Copy u (K of this CTA's tile u / 2, then V) is in stage u % stages: whether it is there, and whether copy u - stages is done with.
    auto copied = [&](uint32_t u) { return barrier_wait<kRolled>(full + 8 * (u % M::stages), (u / M::stages) & 1); };
    auto stage_free = [&](uint32_t u) { return u < M::stages || barrier_wait<kRolled>(empty + 8 * (u % M::stages), (u / M::stages - 1) & 1); };
    // All rows of an item's queries, as boxes of whole tokens (one lane).
    auto copy_query_boxes = [&](const ChunkItem &item, uint32_t bar) {
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(item.rows > 128 ? M::queries : M::q_tile) : "memory");
        const int token = static_cast<int>(item.token0) + static_cast<int>(quick_div(static_cast<uint32_t>(item.row0), p.div_group)), step = static_cast<int>(quick_div(128, p.div_group));
        for (int slot = 0; slot < (item.rows > 128 ? kSlots : 1); slot++)
            for (int c = 0; c < DP / 64; c++) copy_box3(base + slot * M::q_tile + c * (128 * 128), &p.map_q, 64 * c, item.h * shape.group, token + slot * step, bar);
    };
    auto tile_of = [](const ChunkItem &item, int i) { return i < item.list.firsts ? i : i + item.list.skip; };
    // Does slot `slot` need tile i of the list?
    auto needs = [&](const ChunkItem &item, int slot, int i) {
        if (kSlots == 1) return true;
        if (turns(item)) return ((i - item.begin) & 1) == slot;
        return slot == 0 ? i < item.list.end0 : item.rows > 128 && (i < item.list.firsts || i >= item.list.begin1);
    };
    // Is there a key in tile i that some row sees and another does not?
    auto ragged = [&](const ChunkItem &item, int i) {
        const int k0 = tile_of(item, i) * kKeys;
        return k0 + kKeys - 1 > item.pos0 + static_cast<int>(quick_div(item.row0, p.div_group)) || (k0 < item.list.key_end - shape.window && k0 + kKeys > shape.sinks);
    };

    if (warp < kLoad) {
        // ---------------------------------------------------------------------------- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(W::softmax_registers));
        const int slot = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tensor + (static_cast<uint32_t>((warp & 3) * 32) << 16), p_at = lanes + kProbabilities + slot * kProbabilitiesStep, o_at = lanes + kOutputs + slot * 128;
        uint32_t steps = 0, tiles = 0, loads = 0;  // of this slot; of the CTA; items that had queries
        for (int it = 0; slot < kSlots && fine; it++) {
            ChunkItem item;
            if (!take_item(it, item)) break;
            const bool some = item.begin < item.end;
            const int count = item.end - item.begin;
            if (slot == 1 && item.rows <= 128 && !turns(item)) {
                tiles += max(count, 0), loads += some;
                continue;
            }
            const int first_row = turns(item) ? 0 : slot * 128, row = item.row0 + min(first_row + r, item.rows - 1);
            const int token = static_cast<int>(quick_div(static_cast<uint32_t>(row), p.div_group)), pos = item.pos0 + token;
            float factor = fabsf(p.scale_log2);  // of this thread's row of scores
            const uint32_t down_at = base + kDownsAt + 4 * ((loads % M::down_sets) * kSlots * 128 + first_row + r);
            loads += some;
            float top = -INFINITY;
            float ref = -INFINITY;  // codes: the running maximum of the scores, which the sum is relative to; `top` has the tiles' powers in it
            float2 sum = make_float2(0.f, 0.f);
            bool mine = false;  // O holds something of this item
            auto scale_outputs = [&](float f) {
#pragma unroll 1
                for (int c = 0; c < DP / 16 && fine; c++) {
                    uint32_t v[16];
                    tensor_load16(o_at + 16 * c, v);
                    tensor_loaded();
#pragma unroll
                    for (int i = 0; i < 16; i++) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                    tensor_store16(o_at + 16 * c, v);
                }
            };
            auto raise_ref = [&](float highest) {
                const float to = fmaxf(ref, highest), less = exp2_approx(ref - (to == -INFINITY ? 0.f : to));
                sum.x *= less, sum.y *= less;
                ref = to;
            };
            for (int i = item.begin; i < item.end && fine; i++, tiles++) {
                if (!needs(item, slot, i)) continue;
                // one slot: the scores have two buffers in turn
                const uint32_t b = kSlots == 1 ? steps & 1 : slot, parity = kSlots == 1 ? (steps >> 1) & 1 : steps & 1, s_at = lanes + kScores + slot * kScoresStep + (kSlots == 1 ? (steps & 1) * kKeys : 0);
                fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(s_full + 8 * b, parity));
                if (!fine) break;
                fence_after();
                const uint32_t about = info + (tiles % M::infos) * M::info;
                // P is free and O at rest when this slot's last product is done
                bool rest = steps == 0;
                auto await_rest = [&]() {
                    if (rest) return;
                    fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(o_added + 8 * slot, (steps - 1) & 1));
                    fence_after();
                    rest = true;
                };
                // the row's running maximum moves; O is rescaled
                auto move_top = [&](float most) {
                    const float m = fmaxf(top, most), f = m == top ? 1.f : exp2_approx(top - m);
                    top = m;
                    if constexpr (KIND == kPlain) sum.x *= f, sum.y *= f;
                    if (mine) {
                        await_rest();
                        scale_outputs(f);
                    }
                };
                const bool edge = ragged(item, i);
                RowView view{about, 1 << 30, -(1 << 30), 0};
                if (edge) {
                    const int k0 = tile_of(item, i) * kKeys;
                    view.upper = pos + 1 - k0, view.lower = view.upper - shape.window, view.firsts = shape.sinks - k0;
                }
                float exponent = 0.f;
                uint32_t far = 0;
                if constexpr (KIND != kPlain) {
                    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=f"(exponent), "=r"(far) : "r"(about + 32));
                    if (!mine) {
                        float down;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(down) : "r"(down_at));
                        factor *= down;
                    }
                }
                if (KIND != kPlain && far) {
                    const uint32_t scales = about + M::scales;
                    const float2 maxima = far_maxima<kKeys>(s_at, view, scales, factor);
                    raise_ref(maxima.x);
                    move_top(maxima.y);
                    await_rest();
                    if (!fine) break;
                    sum.x += far_probabilities<kKeys>(s_at, p_at, view, scales, factor, ref == -INFINITY ? 0.f : ref, top == -INFINITY ? 0.f : top - kLift);
                    tensor_stored();
                    fence_before();
                    barrier_arrive(s_taken + 8 * b);
                } else if constexpr (kWidens<KIND>) {
                    // 32 scores at a time, in a loop whose code stays small: six warps of four kinds share a scheduler's instruction cache
                    auto scores = [&](int c, float2 (&x)[16]) {
                        tensor_load32(s_at + 32 * c, reinterpret_cast<uint32_t(&)[32]>(x));
                        const uint32_t word = view.word(c);
                        tensor_loaded();
                        const float2 f2 = make_float2(factor, factor), zero = make_float2(0.f, 0.f);
#pragma unroll
                        for (int j = 0; j < 8; j++) {
                            const float4 k = load_shared_f4(about + M::scales + 128 * c + 16 * j);
                            x[2 * j] = fused2(x[2 * j], fused2(f2, make_float2(k.x, k.y), zero), zero);
                            x[2 * j + 1] = fused2(x[2 * j + 1], fused2(f2, make_float2(k.z, k.w), zero), zero);
                        }
                        if (word != 0xffffffffu) {
#pragma unroll
                            for (int j = 0; j < 16; j++) {
                                if (!(word >> (2 * j) & 1)) x[j].x = -INFINITY;
                                if (!(word >> (2 * j + 1) & 1)) x[j].y = -INFINITY;
                            }
                        }
                    };
                    float highest = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < kWords; c++) {
                        float2 x[16];
                        scores(c, x);
                        float m2[2] = {highest, -INFINITY};
#pragma unroll
                        for (int j = 0; j < 16; j++) m2[j & 1] = larger3(m2[j & 1], x[j].x, x[j].y);
                        highest = fmaxf(m2[0], m2[1]);
                    }
                    const float most = highest + exponent;
                    // a running maximum moves only when a score exceeds it by more than 8 (2^8 in probabilities)
                    if (__any_sync(0xffffffffu, most > top + 8.f || highest > ref + 8.f)) {
                        raise_ref(highest);
                        move_top(most);
                    }
                    if constexpr (!kInPlace) await_rest();  // P is free
                    if (!fine) break;
                    const float m = top == -INFINITY ? 0.f : top - kLift;
                    const float2 minus = make_float2(exponent - m, exponent - m);
                    float2 here = make_float2(0.f, 0.f);
#pragma unroll 1
                    for (int c = 0; c < kWords; c++) {
                        float2 x[16];
                        scores(c, x);
                        uint32_t w[16];
                        float4 f4;  // the rest of V's scales
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            float2 e = sum2(x[j], minus);
                            e = make_float2(exp2_approx(e.x), exp2_approx(e.y));
                            here = sum2(here, e);
                            if (j % 2 == 0) f4 = load_shared_f4(about + M::scales + 8 * kKeys + 128 * c + 8 * j);
                            e = fused2(e, j % 2 ? make_float2(f4.z, f4.w) : make_float2(f4.x, f4.y), make_float2(0.f, 0.f));
                            w[j] = pack2<T>(e.x, e.y);
                        }
                        tensor_store16(p_at + 16 * c, w);  // in place: 16 columns of the 32 c that have been read
                    }
                    // `here` is relative to m - exponent, which is at most 48 above ref: exponent is no less than 40 below any before
                    const float all = here.x + here.y;
                    sum.x = fmaf(all, all == 0.f ? 0.f : exp2_approx(m - exponent - (ref == -INFINITY ? 0.f : ref)), sum.x);
                    tensor_stored();
                    fence_before();
                    barrier_arrive(s_taken + 8 * b);
                } else {
                    union {
                        uint32_t w[kWords][32];
                        float f[kWords][32];
                        float2 f2[kWords][16];
                    } s;
#pragma unroll
                    for (int c = 0; c < kWords; c++) tensor_load32(s_at + 32 * c, s.w[c]);
                    uint32_t mask[kWords], all_seen = 0xffffffffu;
#pragma unroll
                    for (int c = 0; c < kWords; c++) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(mask[c]) : "r"(about + 4 * c));
                    tensor_loaded();
                    fence_before();
                    barrier_arrive(s_taken + 8 * b);
                    if (edge) {
#pragma unroll
                        for (int c = 0; c < kWords; c++) mask[c] = view.word(c);
                    }
                    if constexpr (KIND != kPlain) {
                        const float2 zero = make_float2(0.f, 0.f);
#pragma unroll
                        for (int j = 0; j < kKeys / 4; j++) {
                            const float4 k = load_shared_f4(about + M::scales + 16 * j);
                            float2 *x = &s.f2[j / 8][j % 8 * 2];
                            x[0] = fused2(x[0], make_float2(k.x, k.y), zero), x[1] = fused2(x[1], make_float2(k.z, k.w), zero);
                        }
                    }
#pragma unroll
                    for (int c = 0; c < kWords; c++) all_seen &= mask[c];
                    if (!__all_sync(0xffffffffu, all_seen == 0xffffffffu)) {
#pragma unroll
                        for (int c = 0; c < kWords; c++) {
                            if (__all_sync(0xffffffffu, mask[c] == 0xffffffffu)) continue;
#pragma unroll
                            for (int j = 0; j < 32; j++)
                                if (!(mask[c] >> j & 1)) s.f[c][j] = -INFINITY;
                        }
                    }
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < kWords; c++) {
                        m4[c] = fmaxf(s.f[c][0], s.f[c][1]);
#pragma unroll
                        for (int j = 2; j < 32; j += 2) m4[c] = larger3(m4[c], s.f[c][j], s.f[c][j + 1]);
                    }
                    const float highest = fmaxf(larger3(m4[0], m4[1], m4[2]), m4[3]) * factor, most = highest + exponent;
                    bool move = most > top + 8.f;
                    if constexpr (KIND != kPlain) move = move || highest > ref + 8.f;
                    // a running maximum moves only when a score exceeds it by more than 8 (2^8 in probabilities)
                    if (__any_sync(0xffffffffu, move)) {
                        if constexpr (KIND != kPlain) raise_ref(highest);
                        move_top(most);
                    }
                    // asked before the exponentials, answered behind them: as a rule the product before is done by now
                    const bool asked = steps == 0 || barrier_passed(o_added + 8 * slot, (steps - 1) & 1);
                    const float m = top == -INFINITY ? 0.f : top - kLift;
                    const float2 minus = make_float2(exponent - m, exponent - m), f2 = make_float2(factor, factor);
                    float2 here = make_float2(0.f, 0.f);
#pragma unroll
                    for (int c = 0; c < kWords; c++) {
                        float4 f4;  // the rest of V's scales
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            float2 e = fused2(s.f2[c][j], f2, minus);
                            e = make_float2(exp2_approx(e.x), exp2_approx(e.y));
                            here = sum2(here, e);
                            if constexpr (KIND != kPlain) {
                                if (j % 2 == 0) f4 = load_shared_f4(about + M::scales + 8 * kKeys + 128 * c + 8 * j);
                                e = fused2(e, j % 2 ? make_float2(f4.z, f4.w) : make_float2(f4.x, f4.y), make_float2(0.f, 0.f));
                            }
                            s.w[c][j] = pack2<T>(e.x, e.y);  // (in the place of scores that are done with)
                        }
                    }
                    if constexpr (KIND == kPlain) {
                        sum = sum2(sum, here);
                    } else {
                        // `here` is relative to m - exponent, which is at most 48 above ref: exponent is no less than 40 below any before
                        const float all = here.x + here.y;
                        sum.x = fmaf(all, all == 0.f ? 0.f : exp2_approx(m - exponent - (ref == -INFINITY ? 0.f : ref)), sum.x);
                    }
                    if (!__all_sync(0xffffffffu, asked)) await_rest();
                    fence_after();
                    if (!fine) break;
#pragma unroll
                    for (int c = 0; c < kWords; c++) tensor_store16(p_at + 16 * c, reinterpret_cast<const uint32_t(&)[16]>(s.w[c]));
                    tensor_stored();
                }
                if (edge) {
                    const uint32_t u = 2 * tiles + 1, stage = u % M::stages;
                    fine = __all_sync(0xffffffffu, copied(u));
                    if (!fine) break;
                    uint32_t bad[4];
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(bad[0]), "=r"(bad[1]), "=r"(bad[2]), "=r"(bad[3]) : "r"(about + 16) : "memory");
                    if (bad[0] | bad[1] | bad[2] | bad[3]) spoiled_tile<T, DP, kKeys>(p_at, o_at, ring + stage * M::tile, view, !mine);
                }
                fence_before();
                barrier_arrive(p_ready + 8 * slot);
                mine = true;
                steps++;
            }
            if (!fine) break;
            // The rows' outputs, or the part: outputs by the sum, and its logarithm.
            const float all = sum.x + sum.y, lowest = KIND == kPlain ? top - kLift : ref;
            const bool store = first_row + r < item.rows, cut = item.part_row != kUncut;
            const int head = item.h * shape.group + (row - token * shape.group);
            const int64_t at = static_cast<int64_t>(item.part_row) + (turns(item) ? slot * item.rows * H : 0) + static_cast<int64_t>(token) * p.Hq + head;
            const float log = all == 0.f ? -INFINITY : (lowest == -INFINITY ? 0.f : lowest) + log2f(all);
            char *const out = p.out + (item.token0 + token) * p.out_token + head * p.out_head;
            if (mine) {
                fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(o_added + 8 * slot, (steps - 1) & 1));
                if (!fine) break;
                fence_after();
                float inv = 1.f / all;
                if constexpr (KIND != kPlain) {
                    // outputs are relative to `top`: from there to `ref`, in two steps where fp32 does not hold one
                    float step = top - kLift - (lowest == -INFINITY ? 0.f : lowest);
                    if (__any_sync(0xffffffffu, !(fabsf(step) < 80.f))) {
                        step *= 0.5f;
                        scale_outputs(exp2_approx(step));
                        tensor_stored();
                    }
                    inv *= exp2_approx(step);
                }
#pragma unroll 1
                for (int c = 0; c < DP / 32; c++) {
                    uint32_t v[32];
                    tensor_load32(o_at + 32 * c, v);
                    tensor_loaded();
#pragma unroll
                    for (int j = 0; j < 32; j++) v[j] = all == 0.f ? 0u : __float_as_uint(__uint_as_float(v[j]) * inv);  // (without weight 0, whatever V is)
                    if (cut) {
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            if (store && 32 * c + j < D) *reinterpret_cast<uint4 *>(p.parts + at * D + 32 * c + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int k = 0; k < 4; k++) {
                                const float a = __uint_as_float(v[j + 2 * k]), z = __uint_as_float(v[j + 2 * k + 1]);
                                w[k] = KIND == kPlain ? pack2<T>(a, z) : p.q_bf16 ? pack2<__nv_bfloat16>(a, z) : pack2<__half>(a, z);
                            }
                            if (store && 32 * c + j < D) *reinterpret_cast<uint4 *>(out + (32 * c + j) * 2) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                }
                fence_before();  // O has been read when the next item's first probabilities are announced
            } else if (store && !cut) {
                for (int j = 0; j < D; j += 8) *reinterpret_cast<uint4 *>(out + j * 2) = make_uint4(0, 0, 0, 0);
            }
            if (store && cut) p.sums[at] = log;
            if (store && !cut && p.lse) p.lse[(item.token0 + token) * p.Hq + head] = log * kChunkLn2;
        }
    } else if (warp < kIssue) {
        // --------------------------------------------------------------------------- the pages
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(W::other_registers));
        const int thread = threadIdx.x - 32 * kLoad;
        uint32_t tiles = 0, loads = 0, looks = 0;  // of the CTA; items that had queries; tiles of V that were looked at
        auto place_in_block = [&](int t) { return t - static_cast<int>(quick_div(static_cast<uint32_t>(t), p.div_block)) * static_cast<int>(p.layer.B); };
        // where 8 elements of a row of queries are, or NULL: past the last row or past D
        auto query_at = [&](const ChunkItem &item, int rr, int chunk) -> const char * {
            if (rr >= item.rows || chunk * 8 >= D) return nullptr;
            const uint32_t row = item.row0 + rr, token = quick_div(row, p.div_group);
            return p.q + (item.token0 + token) * p.q_token + (item.h * shape.group + static_cast<int>(row - token * shape.group)) * p.q_head + chunk * 16;
        };
        // Queries that meet codes: fp16 with a power of two taken out of each row; eight lanes have a row.
        auto prepare_queries = [&](const ChunkItem &item) {
            if (p.q_boxes) {
                if (fine) fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(landed, loads & 1));
            } else if (loads && fine) {
                fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(q_empty, (loads - 1) & 1));
            }
            const int rows = item.rows > 128 ? kSlots * 128 : 128;
#pragma unroll 2
            for (int r0 = (warp - kLoad) * 4; r0 < rows && fine; r0 += 4 * W::loaders) {
                const int rr = r0 + (lane >> 3);
                unsigned char *const to = gen + (rr >> 7) * M::q_tile;
                uint4 v[DP / 64];
                float most = 0.f, up, down;
#pragma unroll
                for (int j = 0; j < DP / 64; j++) {
                    const int ch = 8 * j + (lane & 7);
                    const char *src = p.q_boxes ? nullptr : query_at(item, rr, ch);
                    v[j] = make_uint4(0, 0, 0, 0);
                    if (p.q_boxes) v[j] = *reinterpret_cast<const uint4 *>(to + swizzled(rr & 127, ch));
                    else if (src) v[j] = *reinterpret_cast<const uint4 *>(src);
                }
#pragma unroll
                for (int j = 0; j < DP / 64; j++)
                    for (uint32_t x : {v[j].x, v[j].y, v[j].z, v[j].w}) most = finite_magnitude(most, query_pair(x, p.q_bf16));
#pragma unroll
                for (int x = 1; x < 8; x <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
                query_powers(most, up, down);
#pragma unroll
                for (int j = 0; j < DP / 64; j++) {
                    uint32_t x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const float2 f = query_pair(x[k], p.q_bf16);
                        x[k] = pack2<__half>(f.x * up, f.y * up);
                    }
                    *reinterpret_cast<uint4 *>(to + swizzled(rr & 127, 8 * j + (lane & 7))) = make_uint4(x[0], x[1], x[2], x[3]);
                }
                if ((lane & 7) == 0) *reinterpret_cast<float *>(gen + kDownsAt + 4 * ((loads % M::down_sets) * kSlots * 128 + rr)) = down;
            }
            fence_shared_to_async();
            if (fine) barrier_arrive(q_full);
            loads++;
        };
        // near the item's end the next one is asked for
        auto near_end = [&](const ChunkItem &item, int i) {
            if (warp == kLoad && lane == 0 && i == max(item.begin, item.end - 2)) barrier_arrive(wanted);
        };

        if constexpr (KIND == kPlain) {
            // Two warps fetch K, two V, each half of every tile's keys.  Where pages fit, a lane has a page and fetches boxes of it, 64 elements wide, that
            // land swizzled; what they bring beside the keys that are seen is harmless in K, whose scores are masked, and
            // is made zero in V.  Elsewhere keys are copied in chunks of 16 bytes.
            const int kv = (warp - kLoad) >> 1, sub = warp & 1;
            constexpr int kHalf = kKeys / 2, kHalfWords = kHalf / 32, chunks = DP / 8;
            const char *const plane = kv ? p.layer.v : p.layer.k;
            const CUtensorMap *const map = kv ? &p.map_v : &p.map_k;
            // Copies announce themselves when they have landed; lane 0 says for its warp what was written beside them.
            auto announce = [&](uint32_t bar) {
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive(bar);
            };
            // Where the heads of a group are a power of two, its rows are boxes of whole tokens, and one warp fetches them.
            auto take_queries = [&](const ChunkItem &item) {
                if (p.q_boxes && warp != kLoad) {
                    loads++;
                    return;
                }
                if (loads) fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(q_empty, (loads - 1) & 1));
                if (!fine) return;
                if (p.q_boxes) {
                    if (lane == 0) copy_query_boxes(item, q_full);
                    __syncwarp();
                    loads++;
                    return;
                }
#pragma unroll 4
                for (int j = 0; j < kSlots * DP / 8; j++) {
                    const int idx = j * 128 + thread, rr = idx / chunks, ch = idx % chunks;
                    const char *src = query_at(item, rr, ch);
                    copy_async16(base + (rr >> 7) * M::q_tile + swizzled(rr & 127, ch), src ? src : p.q, src != nullptr);
                }
                announce(q_full);
                loads++;
            };
            // What the table says of this lane's page, or of its keys; kNoKey: it is none that is seen.  Looked at a tile later.
            const int box_rows = p.box_rows, pages = box_rows ? kHalf / box_rows : 0;
            auto first_key = [&](const ChunkItem &item, int i) { return tile_of(item, i) * kKeys + sub * kHalf; };
            auto entry = [&](const ChunkItem &item, int i, int t, int rows) -> int32_t {
                if (i >= item.end || t >= item.list.key_end || (t + rows <= item.list.key_low && t >= shape.sinks)) return kNoKey;
                return reinterpret_cast<const int32_t *>(p.tables + item.r * p.table_stride)[quick_div(static_cast<uint32_t>(t), p.div_block)];
            };
            auto look_up = [&](const ChunkItem &item, int i, int32_t (&said)[kHalfWords]) {
                const int t = first_key(item, i);
                if (box_rows) {
                    said[0] = lane < pages ? entry(item, i, t + lane * box_rows, box_rows) : kNoKey;
                } else {
#pragma unroll
                    for (int x = 0; x < kHalfWords; x++) said[x] = entry(item, i, t + lane + 32 * x, 1);
                }
            };
            auto checked = [&](int32_t said) -> int32_t {
                const bool in = said >= 0 && said < p.layer.num_blocks;
                if (!in && said != kNoKey) atomicOr(p.status, kStatusBadIndex);
                return in ? said : -1;
            };
            for (int it = 0; fine; it++) {
                ChunkItem item;
                if (!take_item(it, item)) break;
                int32_t ahead[kHalfWords];
                look_up(item, item.begin, ahead);
                for (int i = item.begin; i < item.end && fine; i++, tiles++) {
                    near_end(item, i);
                    const int t0 = first_key(item, i);
                    const uint32_t u = 2 * tiles + kv, stage = u % M::stages, bar = full + 8 * (u % M::stages), about = info + (tiles % M::infos) * M::info, to = ring + stage * M::tile;
                    int32_t blk[kHalfWords];
                    uint32_t mask[kHalfWords];
                    blk[0] = checked(ahead[0]);
#pragma unroll
                    for (int x = 0; x < kHalfWords; x++) {
                        const int t = t0 + lane + 32 * x;
                        bool there = t < item.list.key_end && (t >= item.list.key_low || t < shape.sinks);
                        if (box_rows) {
                            there = __shfl_sync(0xffffffffu, blk[0], quick_div(static_cast<uint32_t>(lane + 32 * x), p.div_box)) >= 0 && there;
                        } else {
                            if (x) blk[x] = checked(ahead[x]);
                            there = blk[x] >= 0;
                        }
                        mask[x] = __ballot_sync(0xffffffffu, there);
                    }
                    look_up(item, i + 1, ahead);
                    if (kv && i == item.begin) take_queries(item);
                    if (fine) fine = __all_sync(0xffffffffu, stage_free(u));
                    if (!fine) break;
                    if (kv == 0 && lane == 0) {
#pragma unroll
                        for (int x = 0; x < kHalfWords; x++) asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 4 * (sub * kHalfWords + x)), "r"(mask[x]) : "memory");
                    }
                    const bool look = kv && ragged(item, i);
                    // what is written beside a copy is written before it is announced: the products may follow its last byte at once
                    auto say_bad = [&](uint32_t bad) {
                        if (lane == 0) asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(about + 16 + 8 * sub), "r"(bad), "r"(0) : "memory");
                    };
                    if (kv && !look) say_bad(0);
                    if (box_rows) {
                        const uint32_t lands = look ? landed + 8 * sub : bar;
                        if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(lands), "n"(kHalf * DP * 2) : "memory");
                        __syncwarp();
                        if (lane < pages) {
                            const int t = t0 + lane * box_rows;
#pragma unroll
                            for (int c = 0; c < DP / 64; c++)
                                copy_box(to + c * (kKeys * 128) + (sub * kHalf + lane * box_rows) * 128, map, 64 * c, place_in_block(t), item.h, blk[0] >= 0 ? blk[0] : static_cast<int32_t>(p.layer.num_blocks), lands);
                        }
                        __syncwarp();
                    } else {
                        int64_t off[kHalfWords];
#pragma unroll
                        for (int x = 0; x < kHalfWords; x++) off[x] = blk[x] >= 0 ? p.layer.geo.at(blk[x], place_in_block(t0 + lane + 32 * x), item.h) : -1;
#pragma unroll
                        for (int j = 0; j < kHalf * chunks / 32; j++) {
                            const int idx = j * 32 + lane, rr = idx / chunks, ch = idx % chunks;
                            const int64_t src = __shfl_sync(0xffffffffu, off[j * 32 / chunks / 32], rr & 31);
                            const bool there = src >= 0 && ch * 8 < D;
                            copy_async16(to + swizzled<kKeys>(sub * kHalf + rr, ch), plane + (there ? src + ch * 16 : 0), there);
                        }
                    }
                    if (look) {
                        if (box_rows) {
                            fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(landed + 8 * sub, looks & 1));
                            looks++;
                            if (!fine) break;
                        } else {
                            copy_wait<0>();
                        }
                        uint32_t any = 0;
                        const bool whole = mask[0] == 0xffffffffu && mask[kHalfWords - 1] == 0xffffffffu;
#pragma unroll 1
                        for (int j0 = 0; j0 < kHalf * chunks / 32; j0 += 8) {
                            uint32_t x[8][4];
#pragma unroll
                            for (int j = 0; j < 8; j++) {
                                const int idx = (j0 + j) * 32 + lane;
                                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[j][0]), "=r"(x[j][1]), "=r"(x[j][2]), "=r"(x[j][3]) : "r"(to + swizzled<kKeys>(sub * kHalf + idx / chunks, idx % chunks)) : "memory");
                            }
#pragma unroll
                            for (int j = 0; j < 8; j++) {
                                const int idx = (j0 + j) * 32 + lane, rr = idx / chunks;
                                const uint32_t odd = not_finite<T>(x[j][0]) | not_finite<T>(x[j][1]) | not_finite<T>(x[j][2]) | not_finite<T>(x[j][3]);
                                if (whole || ((kHalfWords == 2 && rr >= 32 ? mask[kHalfWords - 1] : mask[0]) >> (rr & 31) & 1)) any |= odd;
                                else asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(to + swizzled<kKeys>(sub * kHalf + rr, idx % chunks)), "r"(0) : "memory");
                            }
                        }
                        __syncwarp();
                        say_bad(__any_sync(0xffffffffu, any != 0));
                        fence_shared_to_async();
                    }
                    if (!box_rows) announce(bar);
                    else if (look) {
                        __syncwarp();
                        if (lane == 0) barrier_arrive(bar);
                    }
                    if (!kv && i == item.begin) take_queries(item);
                }
                if (item.begin >= item.end && warp == kLoad && lane == 0) barrier_arrive(wanted);
            }
            copy_wait<0>();
        } else if constexpr (KIND == kWide) {
            // Tiles lie ready, swizzled: one warp fetches K, with scales and masks, one V; all four take part in the queries.
            const int kv = warp - kLoad;
            for (int it = 0; fine; it++) {
                ChunkItem item;
                if (!take_item(it, item)) break;
                // tile i's place among the request's
                auto place = [&](int i) {
                    const int t = tile_of(item, i), listed = t < item.firsts ? t : t - item.skip;
                    return p.wide + ((static_cast<int64_t>(item.r) * p.wide_list + listed) * H + item.h) * WideTile<DP>::bytes;
                };
                // lane by lane: of K the mask, the exponent and whether scales are far apart, of V whether it has numbers that are not finite; each is
                // written by the warp whose copy it is read with, since neither waits for the other
                auto header = [&](int i) {
                    const bool some = (kv == 0 ? lane < 6 : kv == 1 && lane == 6) && i < item.end;
                    return some ? reinterpret_cast<const uint32_t *>(place(i) + WideTile<DP>::header_at)[lane] : 0u;
                };
                uint32_t ahead = header(item.begin);
                int e_most = kLeastExponent;  // the largest of a tile so far
                if (kv >= 2 && item.begin < item.end) prepare_queries(item);
                for (int i = item.begin; i < item.end && fine && kv < 2; i++, tiles++) {
                    const uint32_t u = 2 * tiles + kv, stage = u % M::stages, bar = full + 8 * stage, about = info + (tiles % M::infos) * M::info;
                    near_end(item, i);
                    const char *const from = place(i);
                    uint32_t word = ahead;
                    ahead = header(i + 1);
                    fine = __all_sync(0xffffffffu, stage_free(u));
                    if (!fine) break;
                    if (kv == 0) {
                        const int e = static_cast<int>(__shfl_sync(0xffffffffu, word, 4));
                        if (lane == 5) word |= e < e_most - 40;
                        e_most = max(e_most, e);
                        if (lane == 4) word = __float_as_uint(static_cast<float>(e));
                        const int to = lane < 4 ? 4 * lane : 32 + 4 * (lane - 4);
                        if (lane < 6) asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + to), "r"(word) : "memory");
                    } else if (lane >= 6 && lane < 10) {
                        if (!ragged(item, i)) word = 0;  // what all rows see the products take, whatever it is
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 16 + 4 * (lane - 6)), "r"(word) : "memory");
                    }
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(M::tile + (kv ? 0 : 12 * kKeys)) : "memory");
                        copy_run(ring + stage * M::tile, from + kv * M::tile, M::tile, bar);
                        if (kv == 0) copy_run(about + M::scales, from + WideTile<DP>::scales_at, 12 * kKeys, bar);
                    }
                    __syncwarp();
                    if (i == item.begin) prepare_queries(item);
                }
                if (item.begin >= item.end && warp == kLoad && lane == 0) barrier_arrive(wanted);
            }
        } else {
            // Codes: four warps fetch and widen K, four V, each its own keys of every tile, through registers, a tile ahead; both are fp16
            // exactly.  K's scales multiply the scores, V's the probabilities, in fp32, before those are rounded to fp16 once: what is
            // left of a scale over a power of two that the tile's largest sets, 2^exponent, which is in the maximum that probabilities
            // are relative to.  They keep their precision down to 2^-14, so where scales span no more than 2^16 a key of a small one may have all
            // the weight.  Where they span more the tile is `far`, and each key has an exponent of its own; so it is where a tile's largest
            // scale is 2^-40 of one before.
            const int kv = warp >= kLoad + 4, w = warp & 3;
            // all of K's four warps, wherever a wait of one ran out
            auto together = [&](bool yes) {
                if (kv) return yes;
                uint32_t all;
                asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"(static_cast<uint32_t>(yes)) : "memory");
                return all != 0;
            };
            // what the table says of this lane's key of a tile; kNoKey: it is none.  Looked at a tile later
            auto key_of = [&](const ChunkItem &item, int i) { return tile_of(item, i) * kKeys + w * kMine + lane; };
            auto look_up = [&](const ChunkItem &item, int i) -> int32_t {
                const int t = key_of(item, i);
                if (i >= item.end || lane >= kMine || t >= item.list.key_end || (t < item.list.key_low && t >= shape.sinks)) return kNoKey;
                return reinterpret_cast<const int32_t *>(p.tables + item.r * p.table_stride)[quick_div(static_cast<uint32_t>(t), p.div_block)];
            };
            auto checked = [&](int32_t said) -> int32_t {
                const bool in = said >= 0 && said < p.layer.num_blocks;
                if (!in && said != kNoKey) atomicOr(p.status, kStatusBadIndex);
                return in ? said : -1;
            };
            const char *const plane = kv ? p.layer.v : p.layer.k;
            constexpr int chunks = DP / 16, kUnits = kMine * chunks / 32;  // 16-byte chunks of codes that a lane has of a tile
            for (int it = 0;; it++) {
                uint4 codes[kUnits];
                ChunkItem item;
                const bool took = fine && take_item(it, item);
                if (!together(took)) break;
                const bool some = item.begin < item.end;
                int64_t next_off = -1;
                float next_k = 0.f, next_v = 0.f;
                uint32_t next_mask = 0;
                int32_t ahead = look_up(item, item.begin);
                // where this lane's key of a tile is, and its scales: a tile ahead of their use, and the table two
                auto fetch = [&](int i) {
                    const int32_t blk = checked(ahead);
                    ahead = look_up(item, i + 1);
                    next_off = -1, next_k = next_v = 0.f;
                    if (blk >= 0) {
                        const int n = place_in_block(key_of(item, i));
                        next_off = p.layer.geo.at(blk, n, item.h);
                        const int64_t at = p.layer.scale_geo.at(blk, n, item.h);
                        if (!kv) next_k = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.layer.k_scale) + at);
                        next_v = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.layer.v_scale) + at);
                    }
                    next_mask = __ballot_sync(0xffffffffu, blk >= 0);
                };
                auto load_unit = [&](int j) {
                    const int idx = j * 32 + lane, rr = idx / chunks, ch = idx % chunks;
                    const int64_t src = __shfl_sync(0xffffffffu, next_off, rr);
                    codes[j] = make_uint4(0, 0, 0, 0);
                    if (src >= 0 && ch * 16 < D) codes[j] = *reinterpret_cast<const uint4 *>(plane + src + ch * 16);
                };
                int e_most = kLeastExponent;  // the largest of a tile so far
                fetch(item.begin);
                // (loaded behind the queries, which need the registers)
                if (next_off >= 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(plane + next_off));
                if (some) prepare_queries(item);
#pragma unroll
                for (int j = 0; j < kUnits; j++) load_unit(j);
                for (int i = item.begin; i < item.end; i++, tiles++) {
                    const uint32_t u = 2 * tiles + kv, stage = u % M::stages, about = info + (tiles % M::infos) * M::info;
                    near_end(item, i);
                    const float scale_k = next_k;
                    const float scale_v = next_v;
                    const uint32_t mask = next_mask;
                    fetch(i + 1);
                    if (fine) fine = __all_sync(0xffffffffu, stage_free(u));
                    if (!kv) {
                        if (lane == 0) {
                            if constexpr (kMine == 32) asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 4 * w), "r"(mask) : "memory");
                            else asm volatile("st.shared.u16 [%0], %1;" ::"r"(about + 2 * w), "h"(static_cast<uint16_t>(mask)) : "memory");
                        }
                        if (lane < kMine) asm volatile("st.shared.f32 [%0], %1;" ::"r"(about + M::scales + 4 * (w * kMine + lane)), "f"(scale_k) : "memory");
                    }
                    if (!kv) {
                        const ScaleOfV v = scale_of_v(scale_v);
                        const uint32_t warp_most = __reduce_max_sync(0xffffffffu, v.size), warp_least = __reduce_min_sync(0xffffffffu, v.size ? v.size : 0x7f800000u);
                        if (lane == 0) {
                            asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 48 + 4 * w), "r"(warp_most) : "memory");
                            asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 64 + 4 * w), "r"(warp_least) : "memory");
                        }
                        fine = together(fine);  // the four warps come here for every tile, and leave together where a wait ran out
                        if (!fine) break;
                        uint32_t all[4], low[4];
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(all[0]), "=r"(all[1]), "=r"(all[2]), "=r"(all[3]) : "r"(about + 48) : "memory");
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(low[0]), "=r"(low[1]), "=r"(low[2]), "=r"(low[3]) : "r"(about + 64) : "memory");
                        const int e = ScaleOfV::exponent_of(max(max(all[0], all[1]), max(all[2], all[3])));
                        const bool far = e < e_most - 40 || ScaleOfV::exponent_of(min(min(low[0], low[1]), min(low[2], low[3]))) < e - 16;
                        e_most = max(e_most, e);
                        if (w == 0 && lane == 0) asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(about + 32), "f"(static_cast<float>(e)), "r"(static_cast<uint32_t>(far)) : "memory");
                        if (lane < kMine) {
                            const uint32_t at = about + M::scales + 4 * (w * kMine + lane);
                            asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 4 * kKeys), "f"(v.exponent(far, e)) : "memory");
                            asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 8 * kKeys), "f"(v.rest(far, e)) : "memory");
                        }
                    } else if (!fine) {
                        break;
                    }
                    const uint32_t to = ring + stage * M::tile;
                    const bool look = kv && ragged(item, i);
                    uint32_t bad = look && !(fabsf(scale_v) < INFINITY);
#pragma unroll
                    for (int j = 0; j < kUnits; j++) {
                        const int idx = j * 32 + lane, rr = idx / chunks, ch = idx % chunks;
                        // two 16-byte chunks; the lanes of every other 64 d's write theirs in the other order, into other banks
                        const bool odd = ch & 4;
                        const uint4 c = codes[j];
                        uint32_t x[8];
                        widen<KIND>(odd ? c.z : c.x, x[0], x[1]);
                        widen<KIND>(odd ? c.w : c.y, x[2], x[3]);
                        widen<KIND>(odd ? c.x : c.z, x[4], x[5]);
                        widen<KIND>(odd ? c.y : c.w, x[6], x[7]);
                        load_unit(j);
                        if (look) {
#pragma unroll
                            for (int k = 0; k < 8; k++) bad |= not_finite<__half>(x[k]);
                        }
                        const uint32_t a = to + swizzled<kKeys>(w * kMine + rr, 2 * ch + odd), b = to + swizzled<kKeys>(w * kMine + rr, 2 * ch + !odd);
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(b), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
                    }
                    if (kv) {
                        const uint32_t any = __any_sync(0xffffffffu, bad != 0);
                        if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 16 + 4 * w), "r"(any) : "memory");
                    }
                    __syncwarp();
                    fence_shared_to_async();
                    barrier_arrive(full + 8 * (u % M::stages));
                }
                if (!some && warp == kLoad && lane == 0) barrier_arrive(wanted);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(W::other_registers));
        // ----------------------------------------------------------------------- matrix products
        // Two warps, one for each product, so that neither waits for what only the other needs.  They stay together and
        // elect the thread that issues: with uniform control the operands are uniform registers already.
        if (warp == kIssue) {
            // a negative scale: the queries enter with the other sign
            const uint32_t qk = instruction<T>(kKeys, false) | (p.scale_log2 < 0.f ? 1u << 13 : 0u);
            uint32_t tiles = 0, loads = 0, steps[2] = {0, 0};
            int before = -1;  // the slot whose scores were the last
            for (int it = 0; fine; it++) {
                ChunkItem item;
                if (!take_item(it, item)) break;
                if (item.begin >= item.end) continue;
                fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(q_full, loads & 1));
                for (int i = item.begin; i < item.end && fine; i++, tiles++) {
                    const uint32_t u = 2 * tiles, stage = u % M::stages;
                    fine = copied(u);
                    if constexpr (KIND == kPlain) fence_shared_to_async();  // what copies key by key have written, to the products
#pragma unroll
                    for (int slot = 0; slot < kSlots; slot++) {
                        if (!needs(item, slot, i)) continue;
                        uint32_t b, column = tensor + kScores;
                        if constexpr (kSlots == 1) {
                            b = steps[0] & 1, column += b * kKeys;
                            if (steps[0] >= 2 && fine) fine = barrier_wait<kRolled>(s_taken + 8 * b, ((steps[0] >> 1) - 1) & 1);
                        } else if constexpr (kInPlace) {
                            // the slot's columns are free when its last product has taken the probabilities that lay in them
                            b = slot, column += slot * kScoresStep;
                            if (steps[slot] && fine) fine = barrier_wait<kRolled>(o_added + 8 * slot, (steps[slot] - 1) & 1);
                        } else {
                            // the buffer is free when the scores of the step before have been taken
                            b = slot;
                            if (before >= 0 && fine) fine = barrier_wait<kRolled>(s_taken + 8 * before, (steps[before] - 1) & 1);
                        }
                        fine = __all_sync(0xffffffffu, fine);
                        if (!fine) break;
                        fence_after();
                        const uint64_t q_operand = operand(base + (turns(item) ? 0 : slot * M::q_tile), 16), k_operand = operand(ring + stage * M::tile, 16);
                        if (elected()) {
#pragma unroll
                            for (int k = 0; k < DP / 16; k++)
                                mma_shared(column, q_operand + (((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4), k_operand + (((k >> 2) * (kKeys * 128) + (k & 3) * 32) >> 4), qk, k > 0);
                            commit_to(s_full + 8 * b);
                        }
                        __syncwarp();
                        steps[slot]++;
                        before = slot;
                    }
                    if (!fine) break;
                    if (elected()) {
                        commit_to(empty + 8 * (u % M::stages));
                        if (i + 1 == item.end) commit_to(q_empty);
                    }
                    __syncwarp();
                }
                loads++;
            }
        } else if (warp == kIssue + 1) {
            const uint32_t pv = instruction<T>(DP, true);
            uint32_t tiles = 0, steps[2] = {0, 0};
            for (int it = 0; fine; it++) {
                ChunkItem item;
                if (!take_item(it, item)) break;
                bool holds[2] = {false, false};  // O of a slot holds something of this item
                for (int i = item.begin; i < item.end && fine; i++, tiles++) {
                    const uint32_t u = 2 * tiles + 1, stage = u % M::stages;
                    fine = __all_sync(0xffffffffu, copied(u));
                    if (!fine) break;
                    if constexpr (KIND == kPlain) fence_shared_to_async();
                    uint32_t bad[4];
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(bad[0]), "=r"(bad[1]), "=r"(bad[2]), "=r"(bad[3]) : "r"(info + (tiles % M::infos) * M::info + 16) : "memory");
                    const bool spoiled = __any_sync(0xffffffffu, (bad[0] | bad[1] | bad[2] | bad[3]) != 0);
                    const uint64_t v_operand = operand(ring + stage * M::tile, kKeys * 128);
#pragma unroll
                    for (int slot = 0; slot < kSlots; slot++) {
                        if (!needs(item, slot, i)) continue;
                        fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(p_ready + 8 * slot, steps[slot] & 1));
                        if (!fine) break;
                        fence_after();
                        if (elected()) {
                            if (!spoiled) {  // else the softmax has added it up
#pragma unroll
                                for (int k = 0; k < kKeys / 16; k++)
                                    mma_tensor(tensor + kOutputs + slot * 128, tensor + kProbabilities + slot * kProbabilitiesStep + 8 * k, v_operand + k * (2048 >> 4), pv, holds[slot] || k > 0);
                            }
                            commit_to(o_added + 8 * slot);
                        }
                        __syncwarp();
                        holds[slot] = true;
                        steps[slot]++;
                    }
                    if (!fine) break;
                    if (elected()) commit_to(empty + 8 * (u % M::stages));
                    __syncwarp();
                }
            }
        } else if (warp == kIssue + 2) {
            // -------------------------------------------------------------------------- the items
            // This CTA's first is its own; then it takes over CTAs that have not been launched yet, one whenever the copies of the
            // last item near their end.
            const uint32_t answer = base + kAnswerAt;
            uint32_t id = blockIdx.x, asked = 0;
            bool more = true;
            for (int it = 0; fine;) {
                if (more && id < total) {
                    // the last thread whose requests begin at or before the item, then the request
                    int t = -1;
#pragma unroll
                    for (int j = 0; j < W::all; j++) t += __popc(__ballot_sync(0xffffffffu, items_before[j * 32 + lane] <= id));
                    uint32_t at = items_before[t], rows_at = rows_before[t];
                    const int64_t to = min((t + 1) * per, p.R);
                    ChunkItem item;
                    item.valid = 0;
                    for (int64_t r = t * per; r < to; r++) {
                        const ChunkRequest q = chunk_request(p, r, false);
                        if (!q.n) continue;
                        const int32_t tiles = chunk_tiles(shape, q.len), parts = tiles > share ? chunk_parts(tiles, share) : 1, blocks = chunk_blocks(shape, q.n);
                        const uint32_t here = static_cast<uint32_t>(blocks) * parts * H;
                        if (id >= at + here) {
                            at += here;
                            if (parts > 1) rows_at += static_cast<uint32_t>(q.n) * p.Hq * parts * each_leaves(q.n, parts);
                            continue;
                        }
                        // heads first, so that CTAs side by side read pages side by side; the last block, which sees most, first
                        uint32_t rest = id - at;
                        item.h = rest % H, rest /= H;
                        const int32_t part = rest % parts, block = blocks - 1 - static_cast<int32_t>(rest / parts);
                        const int32_t each = each_leaves(q.n, parts);  // parts that an item leaves
                        item.valid = each, item.r = static_cast<int32_t>(r);
                        item.row0 = block * shape.rows;
                        item.rows = min(static_cast<int32_t>(min(static_cast<int64_t>(q.n) * shape.group - item.row0, static_cast<int64_t>(shape.rows))), shape.rows);
                        item.pos0 = q.len - q.n;
                        item.list = chunk_list(shape, item.pos0, item.row0, item.rows, 128);
                        item.begin = static_cast<int32_t>(min(static_cast<int64_t>(part) * share, static_cast<int64_t>(item.list.count)));
                        item.end = static_cast<int32_t>(min(static_cast<int64_t>(item.begin) + share, static_cast<int64_t>(item.list.count)));
                        item.part_row = parts > 1 ? rows_at + static_cast<uint32_t>(part * each) * q.n * p.Hq : kUncut;
                        item.token0 = q.token0;
                        item.firsts = item.skip = 0;
                        if constexpr (KIND == kWide) {
                            const ChunkList whole = chunk_list(shape, item.pos0, 0, q.n * shape.group, q.n * shape.group);
                            item.r = static_cast<int32_t>(wide_place(p, r, q.token0));
                            item.firsts = whole.firsts, item.skip = whole.skip;
                        }
                        // for chunk_join_kernel, by whoever has the request's first item
                        if (p.plan.part_rows && id == at && lane == 0) p.cuts[r] = make_uint2(p.first_part_row + rows_at, static_cast<uint32_t>(parts * each));
                        break;
                    }
                    if (item.valid) {
                        if (it >= 2) fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(item_empty + 8 * (it & 1), ((it >> 1) - 1) & 1));
                        if (!fine) break;
                        if (lane == 0) {
                            items[it & 1] = item;
                            barrier_arrive(item_full + 8 * (it & 1));
                        }
                        __syncwarp();
                        fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(wanted, it & 1, p.item_spins));
                        if (!fine) break;
                        it++;
                    }
                }
                if (!more) {
                    // no item: the end
                    if (it >= 2) fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(item_empty + 8 * (it & 1), ((it >> 1) - 1) & 1));
                    if (lane == 0) {
                        items[it & 1].valid = 0;
                        barrier_arrive(item_full + 8 * (it & 1));
                    }
                    break;
                }
                if (elected()) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the answer before has been read
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], 16;" ::"r"(answered) : "memory");
                    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(answered) : "memory");
                }
                __syncwarp();
                fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(answered, asked & 1));
                asked++;
                if (!fine) break;
                uint32_t got, next = 0;
                asm volatile("{\n\t.reg .pred p;\n\t.reg .b128 a;\n\tld.shared.b128 a, [%2];\n\tclusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\tselp.u32 %0, 1, 0, p;\n\t"
                             "mov.u32 %1, 0;\n\t@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, _, _, _}, a;\n\t}"
                             : "=r"(got), "=r"(next) : "r"(answer) : "memory");
                __syncwarp();
                more = got != 0, id = next;
            }
        }
        if (KIND != kPlain && warp == kIssue + 3 && p.q_boxes) {
            // ------------------------------------------------------------------- queries that meet codes
            // fetched as they are; the warps that fetch K and V take the powers of two out
            uint32_t loads = 0;
            for (int it = 0; fine; it++) {
                ChunkItem item;
                if (!take_item(it, item)) break;
                if (item.begin >= item.end) continue;
                if (loads) fine = __all_sync(0xffffffffu, barrier_wait<kRolled>(q_empty, (loads - 1) & 1));
                if (fine && lane == 0) copy_query_boxes(item, landed);
                __syncwarp();
                loads++;
            }
        }
        if (warp <= kIssue + 1 && !fine) {
            // products may be in flight: let them end before the tensor memory is given back
            const uint32_t last = last_at + 8 * (warp - kIssue);
            if (elected()) commit_to(last);
            __syncwarp();
            barrier_wait<kRolled>(last, 0);
        }
    }
    if (p.beside) await_last();  // who waits for this kernel waits for those before it, too
    if (!fine) atomicOr(p.status, static_cast<unsigned int>(TC_DEVICE_BULK_WAIT_TIMEOUT));
    fence_before();
    if (!__syncthreads_and(fine)) {
        copies_landed<M::stages>(kBarsAt);
        __syncthreads();
    }
    if (warp == kIssue) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tensor) : "memory");
}

template <typename T, int KIND, int DP>
int launch_chunk_shape(const ChunkParams &p, int device, cudaStream_t s)
{
    using M = ChunkMemory<KIND, DP>;
    static_assert(M::bytes <= 232448 - 1024, "more shared memory than a CTA can have beside its static arrays");
    static std::atomic<bool> raised[kMaxDevices];  // set once per device; setting it twice does no harm
    if (!raised[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(chunk_kernel<T, KIND, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, M::bytes);
        if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(dynamic shared memory)");
        // the warps' shares of registers must not be more than a CTA is launched with
        cudaFuncAttributes attr;
        const cudaError_t f = cudaFuncGetAttributes(&attr, chunk_kernel<T, KIND, DP>);
        if (f != cudaSuccess) return cuda_fail(f, "cudaFuncGetAttributes");
        if (attr.numRegs != ChunkWarps<KIND>::launch_registers) return fail(TC_ERR_CUDA, "tc_attn_chunk's kernel was built with %d registers a thread, not %d", attr.numRegs, ChunkWarps<KIND>::launch_registers);
        raised[device].store(true, std::memory_order_relaxed);
    }
    return launch_attn(chunk_kernel<T, KIND, DP>, static_cast<unsigned>(p.plan.grid), ChunkWarps<KIND>::threads, M::bytes, p.beside, p, s);
}

template <typename T, int KIND>
int launch_chunk_type(const ChunkParams &p, int device, cudaStream_t s)
{
    if (p.layer.D <= 64) return launch_chunk_shape<T, KIND, 64>(p, device, s);
    if (p.layer.D <= 128) return launch_chunk_shape<T, KIND, 128>(p, device, s);
    return launch_chunk_shape<T, KIND, 256>(p, device, s);
}

}  // namespace tc
