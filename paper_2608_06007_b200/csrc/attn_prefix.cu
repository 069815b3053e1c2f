// The shared prefix of tc_attn_decode on the fifth-generation tensor cores.
//
// All rows of queries of one KV head - R requests x Hq / H heads - meet every key of the prefix, so
// this is a dense attention over pages.  A CTA has two slots of 128 rows in tensor memory, each with its probabilities P
// (64 columns) and its outputs O (128); one buffer of scores S (128) serves both in turn, since a softmax takes
// its scores into registers at once.  So the next scores of a slot are there when its softmax
// ends, and neither the tensor cores nor the softmax wait for one another.  With more than 128
// rows the slots hold different rows and both take every tile of 128 keys, so a tile is read once for
// 256 rows; with fewer, both hold the same rows and take the tiles in turn.
//
//   warps 0-3, 4-7   softmax of slot 0 and 1: a thread owns one row and holds a tile's 128 scores in registers, so no
//                    shuffle is needed.  The probabilities, rounded to 16 bits, go to tensor memory, where the
//                    second product takes them.  The running maximum moves only when a tile exceeds it
//                    by more than 2^8 (then O is rescaled).
//   warps 8-11       fill a ring of K and V tiles from the pages: 16-byte asynchronous copies into the
//                    swizzled layout, whatever the page size; one lane looks a key's block up.  Codes are
//                    staged as they are first and widened to fp16 by the warp that fetched them.
//   warps 12, 13     issue the matrix products, S = Q K' and O += P V.
//
// Bound by the softmax: 128 requests x 64 heads x 128 behind 32768 tokens (1.4e11 flop): a call takes 168 us in a long run, 0.82 PFLOP/s,
// 0.51 of the measured rate (148 to 154 us, 0.56, 20 in a row); per tile and slot of 1024 clocks of products the softmax takes some 2900 for both
// slots, 2048 of them exponentials.  Kernel times that a profiler gave there, for 142 us: scores over probabilities, a buffer per
// slot 160 us; one buffer, both products from one warp 155; scores issued between the halves of the second product
// 186; a part of the exponentials as polynomials 154.  Codes: bound by the four warps that widen them
// (512 requests x 32 heads behind 4000 e4m3 tokens 70 us, bf16 48, by a profiler; the calls 148 and 131).
//
// Scales of a quantised pool: K's multiply the scores, V's are taken into the values, over a power of two per tile that
// goes into the probabilities.  The sum, without it, has a running maximum of its own: scales reach from 2^-126 to 2^127.
// Every wait is bounded; one that runs out sets TC_DEVICE_BULK_WAIT_TIMEOUT and the CTA leaves.
#include <algorithm>
#include <atomic>

#include "attn.h"
#include "attn_device.cuh"
#include "barrier.cuh"

namespace tc {

constexpr int kTile = 128;       // keys of a tile, and rows of a slot
constexpr int kPrefixThreads = 512;  // 128 registers each; the softmax's 256 take 192, the others keep 64
constexpr int kInfos = 4;            // tiles whose masks and scales are kept

template <int KIND, int DP, bool TWO>
struct PrefixShape {
    static constexpr int tile = kTile * DP * 2;        // bytes of a K or V tile, and of a slot's queries
    static constexpr int queries = (TWO ? 2 : 1) * tile;
    static constexpr int codes = KIND == kPlain ? 0 : kTile * DP;   // bytes of a staged tile of codes
    static constexpr int staged = KIND == kPlain ? 0 : 3;
    // Scores run a tile and a half ahead of the outputs (TWO), or three tiles.
    static constexpr int stages = KIND != kPlain ? (TWO ? 3 : 4) : TWO ? 4 : 6;
    static constexpr int info = KIND == kPlain ? 16 : 64 + 8 * kTile;  // mask; V's exponent, whether scales are far apart; each warp's largest and smallest; scales of K; keys' exponents
    static constexpr int bytes = queries + stages * tile + staged * codes + kInfos * info + 256 + 1024;  // barriers, slack for the alignment
};

// Shared-memory operand descriptor: 128-byte swizzle, 8-row atoms of 1024 bytes `sbo` apart; lbo: from one
// 64-element column of atoms to the next (only where the 64 elements run along M or N).
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lbo)
{
    return static_cast<uint64_t>((addr >> 4) & 0x3fff) | static_cast<uint64_t>(lbo >> 4) << 16 | static_cast<uint64_t>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Instruction descriptor: fp32 sums of 16-bit products, M = 128.
template <typename A> __device__ constexpr uint32_t instruction(int n, bool b_rows_along_n)
{
    const uint32_t type = sizeof(A) && std::is_same<A, __nv_bfloat16>::value ? 1 : 0;
    return 1u << 4 | type << 7 | type << 10 | (b_rows_along_n ? 1u << 16 : 0u) | static_cast<uint32_t>(n / 8) << 17 | (128u / 16) << 24;
}
__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
__device__ __forceinline__ void mma_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
// Arrives at the barrier when all products issued so far by this thread are done.
__device__ __forceinline__ void commit_to(uint32_t bar) { asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory"); }

#define TC_R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define TC_W8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])
// 32 columns of this thread's lane.  The registers hold them after tensor_loaded().
__device__ __forceinline__ void tensor_load32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : TC_R8(r, 0), TC_R8(r, 8), TC_R8(r, 16), TC_R8(r, 24) : "r"(addr));
}
__device__ __forceinline__ void tensor_load16(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : TC_R8(r, 0), TC_R8(r, 8) : "r"(addr));
}
__device__ __forceinline__ void tensor_store16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::TC_W8(r, 0), TC_W8(r, 8), "r"(addr) : "memory");
}
__device__ __forceinline__ void tensor_store8(uint32_t addr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::TC_W8(r, 0), "r"(addr) : "memory");
}
__device__ __forceinline__ void tensor_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tensor_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_shared_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One lane of a converged warp.
__device__ __forceinline__ bool elected()
{
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}

// Byte of element d of row r in a swizzled tile of 128 rows: columns of 64 elements, 128 bytes a row, the
// 16-byte chunks of a row permuted by its place in its group of eight.
__device__ __forceinline__ uint32_t swizzled(int r, int chunk) { return (chunk >> 3) * (kTile * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4); }

__device__ __forceinline__ float larger3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float2 fused2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<uint64_t &>(r)) : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)), "l"(reinterpret_cast<uint64_t &>(c)));
    return r;
}
__device__ __forceinline__ float2 sum2(float2 a, float2 b)
{
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t &>(r)) : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)));
    return r;
}
__device__ __forceinline__ float4 load_shared_f4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}

struct RowState {
    float top, ref, sum;
};

// Rare: scales of V so far apart that what is next to nothing among the probabilities can be much of the sum.
// Each key has its own power of two here, and the sum exponentials of its own; the scores
// stay in tensor memory and are gone through twice, 16 at a time.  False when a wait ran out.  A function of its
// own: in line, never run, it slowed the other tiles (512 requests behind 4000 e4m3 147 -> 150 us a call).
template <int DP>
__device__ __noinline__ bool far_tile(RowState &state, uint32_t s_at, uint32_t p_at, uint32_t o_at, uint32_t about, float factor, uint32_t o_added, int mine)
{
    constexpr float kLift = probability_lift<__half>();
    float highest = -INFINITY, most = -INFINITY, base = 0.f, m = 0.f, sum = state.sum;
#pragma unroll 1
    for (int pass = 0; pass < 2; pass++) {
        if (pass) {
            const float ref = fmaxf(state.ref, highest);
            base = ref == -INFINITY ? 0.f : ref;
            sum *= exp2_approx(state.ref - base);
            state.ref = ref;
            const float to = fmaxf(state.top, most), f = to == state.top ? 1.f : exp2_approx(state.top - to);
            state.top = to;
            m = to == -INFINITY ? 0.f : to - kLift;
            if (mine) {
                if (!__all_sync(0xffffffffu, barrier_wait(o_added, (mine - 1) & 1))) return false;
                fence_after();
#pragma unroll 1
                for (int c = 0; c < DP / 16; c++) {
                    uint32_t v[16];
                    tensor_load16(o_at + 16 * c, v);
                    tensor_loaded();
#pragma unroll
                    for (int i = 0; i < 16; i++) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                    tensor_store16(o_at + 16 * c, v);
                }
            }
        }
#pragma unroll 1
        for (int c = 0; c < 8; c++) {
            uint32_t v[16], w[8], here;
            tensor_load16(s_at + 16 * c, v);
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(here) : "r"(about + 4 * (c >> 1)));
            here >>= 16 * (c & 1);
            tensor_loaded();
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const float4 k4 = load_shared_f4(about + 64 + 4 * (16 * c + i));
                const float4 e4 = load_shared_f4(about + 64 + 4 * kTile + 4 * (16 * c + i));
                const float k[4] = {k4.x, k4.y, k4.z, k4.w}, e[4] = {e4.x, e4.y, e4.z, e4.w};
                float x[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    x[j] = here >> (i + j) & 1 ? __uint_as_float(v[i + j]) * (factor * k[j]) : -INFINITY;
                    if (!pass) {
                        highest = fmaxf(highest, x[j]), most = fmaxf(most, x[j] + e[j]);
                    } else {
                        sum += exp2_approx(x[j] - base);
                        x[j] = exp2_approx(x[j] + e[j] - m);
                    }
                }
                w[i / 2] = pack2<__half>(x[0], x[1]), w[i / 2 + 1] = pack2<__half>(x[2], x[3]);
            }
            if (pass) tensor_store8(p_at + 8 * c, w);
        }
    }
    state.sum = sum;
    return true;
}

// T: the type of the products, fp16 for codes.
template <typename T, int KIND, int DP, bool TWO>
__global__ void __launch_bounds__(kPrefixThreads, 1) prefix_kernel(const __grid_constant__ AttnParams p)
{
    using Shape = PrefixShape<KIND, DP, TWO>;
    constexpr float kLift = probability_lift<T>();
    extern __shared__ unsigned char raw[];
    allow_next();
    const uint32_t base = (static_cast<uint32_t>(__cvta_generic_to_shared(raw)) + 1023) & ~1023u;
    unsigned char *const gen = raw + (base - static_cast<uint32_t>(__cvta_generic_to_shared(raw)));
    const uint32_t ring = base + Shape::queries, staging = ring + Shape::stages * Shape::tile, info = staging + Shape::staged * Shape::codes, bars = info + kInfos * Shape::info;
    const uint32_t full = bars, empty = full + 8 * Shape::stages, s_full = empty + 8 * Shape::stages, s_taken = s_full + 16, p_ready = s_taken + 16, o_added = p_ready + 16, tensor_at = o_added + 16;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, H = p.layer.H, group = p.split.group, D = p.layer.D;

    // Which rows, which keys.
    int64_t id = blockIdx.x;
    const int64_t block = id % p.split.prefix_blocks;
    id /= p.split.prefix_blocks;
    const int h = static_cast<int>(id % H);
    const int64_t part = id / H;
    int64_t len = *p.prefix_len;
    if (len > p.max_prefix || len < 0) {
        if (threadIdx.x == 0) atomicOr(p.status, kStatusBadIndex);
        len = len < 0 ? 0 : p.max_prefix;
    }
    const int begin = static_cast<int>(part * p.split.prefix_chunk);
    const int end = static_cast<int>(min(static_cast<int64_t>(begin) + p.split.prefix_chunk, len));
    if (begin >= end) return;
    const int tiles = __shfl_sync(0xffffffffu, (end - begin + kTile - 1) / kTile, 0);
    const int64_t row0 = block * (TWO ? 256 : 128), row_end = p.R * group;
    const int steps = TWO ? 2 * tiles : tiles;  // step t: slot t & 1, tile t / 2 (TWO) or t

    if (threadIdx.x == 0) {
        barrier_init(tensor_at + 8, 1), barrier_init(tensor_at + 16, 1);
        for (int i = 0; i < Shape::stages; i++) barrier_init(full + 8 * i, 128), barrier_init(empty + 8 * i, 1);
        for (int i = 0; i < 2; i++) barrier_init(s_full + 8 * i, 1), barrier_init(s_taken + 8 * i, 128), barrier_init(p_ready + 8 * i, 128), barrier_init(o_added + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tensor_at) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // Queries: zero past the last row and past D; a negative scale is taken into their sign.
    const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
    auto query = [&](int r, int chunk) {
        const int64_t row = row0 + r;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < row_end && chunk * 8 < D) {
            const int64_t req = quick_div(static_cast<uint32_t>(row), p.div_group);
            v = *reinterpret_cast<const uint4 *>(p.q + req * p.q_req + (h * group + (row - req * group)) * p.q_head + chunk * 16);
            v.x ^= flip, v.y ^= flip, v.z ^= flip, v.w ^= flip;
        }
        return v;
    };
    float factor = fabsf(p.scale_log2);  // of this thread's row of scores
    if constexpr (KIND == kPlain) {
        for (int i = threadIdx.x; i < (TWO ? 256 : 128) * (DP / 8); i += kPrefixThreads)
            *reinterpret_cast<uint4 *>(gen + (i / (DP / 8) >> 7) * Shape::tile + swizzled(i / (DP / 8) & 127, i % (DP / 8))) = query(i / (DP / 8), i % (DP / 8));
    } else if (warp < 8) {
        const int r = TWO ? threadIdx.x : threadIdx.x & 127;
        float most = 0.f, up, down;
        for (int i = 0; i < DP / 8; i++) {
            const uint4 v = query(r, i);
            for (uint32_t w : {v.x, v.y, v.z, v.w}) most = finite_magnitude(most, query_pair(w, p.q_bf16));
        }
        query_powers(most, up, down);
        factor *= down;
        if (TWO || warp < 4)
            for (int i = 0; i < DP / 8; i++) {
                const uint4 v = query(r, i);
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float2 f = query_pair(w[j], p.q_bf16);
                    w[j] = pack2<__half>(f.x * up, f.y * up);
                }
                *reinterpret_cast<uint4 *>(gen + (r >> 7) * Shape::tile + swizzled(r & 127, i)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
    }
    fence_shared_to_async();
    fence_before();
    __syncthreads();
    fence_after();
    // All 512 columns are this CTA's, so they begin at 0; a constant lets the products' operands stay in
    // uniform registers.
    constexpr uint32_t tensor = 0;
    bool fine = true;  // no wait of this thread has run out

    if (warp < 8) {
        // ---------------------------------------------------------------------------- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int slot = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tensor + (static_cast<uint32_t>((warp & 3) * 32) << 16), s_at = lanes, p_at = lanes + 128 + slot * 64, o_at = lanes + 256 + slot * 128;
        float top = -INFINITY;
        float ref = -INFINITY;  // codes: the running maximum of the scores, which the sum is relative to; `top` has the tiles' powers in it
        float2 sum = make_float2(0.f, 0.f);
        int mine = 0;
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
        for (int t = slot; t < steps && fine; t += 2, mine++) {
            fine = __all_sync(0xffffffffu, barrier_wait(s_full + 8 * slot, mine & 1));
            if (!fine) break;
            fence_after();
            const int tile = TWO ? t >> 1 : t;
            const uint32_t about = info + (tile % kInfos) * Shape::info;
            // P is free and O at rest when this slot's last product is done
            bool rest = mine == 0;
            auto await_rest = [&]() {
                if (rest) return;
                fine = __all_sync(0xffffffffu, barrier_wait(o_added + 8 * slot, (mine - 1) & 1));
                fence_after();
                rest = true;
            };
            union {
                uint32_t w[4][32];
                float f[4][32];
                float2 f2[4][16];
            } s;
#pragma unroll
            for (int c = 0; c < 4; c++) tensor_load32(s_at + 32 * c, s.w[c]);
            uint32_t mask[4];
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(mask[0]), "=r"(mask[1]), "=r"(mask[2]), "=r"(mask[3]) : "r"(about));
            float exponent = 0.f;
            uint32_t far = 0;
            if constexpr (KIND != kPlain) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=f"(exponent), "=r"(far) : "r"(about + 16));
            tensor_loaded();
            if constexpr (KIND != kPlain) {
                if (far) {
                    RowState state{top, ref, sum.x + sum.y};
                    fine = far_tile<DP>(state, s_at, p_at, o_at, about, factor, o_added + 8 * slot, mine);
                    top = state.top, ref = state.ref, sum = make_float2(state.sum, 0.f);
                    if (!fine) break;
                    tensor_stored();
                    fence_before();
                    barrier_arrive(s_taken + 8 * slot);
                    barrier_arrive(p_ready + 8 * slot);
                    continue;
                }
            }
            fence_before();
            barrier_arrive(s_taken + 8 * slot);
            if constexpr (KIND != kPlain) {
                const float2 f2 = make_float2(factor, factor), zero = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < 32; i++) {
                    const float4 k = load_shared_f4(about + 64 + 16 * i);
                    float2 *x = &s.f2[i / 8][i % 8 * 2];
                    x[0] = fused2(x[0], fused2(f2, make_float2(k.x, k.y), zero), zero);
                    x[1] = fused2(x[1], fused2(f2, make_float2(k.z, k.w), zero), zero);
                }
            }
            if ((mask[0] & mask[1] & mask[2] & mask[3]) != 0xffffffffu) {
#pragma unroll
                for (int c = 0; c < 4; c++)
#pragma unroll
                    for (int i = 0; i < 32; i++)
                        if (!(mask[c] >> i & 1)) s.f[c][i] = -INFINITY;
            }
            float m4[4];
#pragma unroll
            for (int c = 0; c < 4; c++) {
                m4[c] = fmaxf(s.f[c][0], s.f[c][1]);
#pragma unroll
                for (int i = 2; i < 32; i += 2) m4[c] = larger3(m4[c], s.f[c][i], s.f[c][i + 1]);
            }
            const float highest = fmaxf(larger3(m4[0], m4[1], m4[2]), m4[3]), most = KIND == kPlain ? highest * factor : highest + exponent;
            bool move = most > top + 8.f;
            if constexpr (KIND != kPlain) move = move || highest > ref + 8.f;
            if (__any_sync(0xffffffffu, move)) {
                if constexpr (KIND != kPlain) raise_ref(highest);
                const float m = fmaxf(top, most), f = m == top ? 1.f : exp2_approx(top - m);
                top = m;
                if constexpr (KIND == kPlain) sum.x *= f, sum.y *= f;
                if (mine) {
                    await_rest();
                    scale_outputs(f);
                }
            }
            const float m = top == -INFINITY ? 0.f : top - kLift;
            const float2 minus = make_float2(exponent - m, exponent - m), f2 = make_float2(factor, factor);
            uint32_t w[4][16];
            float2 here = make_float2(0.f, 0.f);
#pragma unroll
            for (int c = 0; c < 4; c++) {
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    float2 e = KIND == kPlain ? fused2(s.f2[c][i], f2, minus) : sum2(s.f2[c][i], minus);
                    e = make_float2(exp2_approx(e.x), exp2_approx(e.y));
                    here = sum2(here, e);
                    w[c][i] = pack2<T>(e.x, e.y);
                }
            }
            if constexpr (KIND == kPlain) {
                sum = sum2(sum, here);
            } else {
                // `here` is relative to m - exponent, which is at most 48 above ref: exponent is no less than 40 below any before
                const float all = here.x + here.y;
                sum.x = fmaf(all, all == 0.f ? 0.f : exp2_approx(m - exponent - (ref == -INFINITY ? 0.f : ref)), sum.x);
            }
            await_rest();  // by now it has been given, as a rule
            if (!fine) break;
#pragma unroll
            for (int c = 0; c < 4; c++) tensor_store16(p_at + 16 * c, w[c]);
            tensor_stored();
            fence_before();
            barrier_arrive(p_ready + 8 * slot);
        }
        // The part: outputs by the sum, and its logarithm.  A slot without a tile says -infinity.
        const float all = sum.x + sum.y;
        const int64_t row = row0 + (TWO ? slot * 128 : 0) + r;
        const int64_t out_part = TWO ? part : 2 * part + slot;
        const bool store = row < row_end;
        const int64_t req = store ? quick_div(static_cast<uint32_t>(row), p.div_group) : 0;
        const int64_t at = out_part * p.split.rows + req * p.Hq + h * group + (row - req * group);
        if (mine && fine) fine = __all_sync(0xffffffffu, barrier_wait(o_added + 8 * slot, (mine - 1) & 1));
        const float base = KIND == kPlain ? top - kLift : ref;
        if (mine && fine) {
            fence_after();
            float inv = all == 0.f ? 0.f : 1.f / all;
            if constexpr (KIND != kPlain) {
                // outputs are relative to `top`: from there to `ref`, in two steps where fp32 does not hold one
                float step = top - kLift - (base == -INFINITY ? 0.f : base);
                if (__any_sync(0xffffffffu, !(fabsf(step) < 80.f))) {
                    step *= 0.5f;
                    scale_outputs(exp2_approx(step));
                    tensor_stored();
                }
                inv *= exp2_approx(step);
            }
#pragma unroll(KIND == kPlain ? 1 : DP / 32)
            for (int c = 0; c < DP / 32; c++) {
                uint32_t v[32];
                tensor_load32(o_at + 32 * c, v);
                tensor_loaded();
#pragma unroll
                for (int i = 0; i < 32; i += 4)
                    if (store && 32 * c + i < D)
                        *reinterpret_cast<float4 *>(p.parts + at * D + 32 * c + i) = make_float4(__uint_as_float(v[i]) * inv, __uint_as_float(v[i + 1]) * inv,
                                                                                                 __uint_as_float(v[i + 2]) * inv, __uint_as_float(v[i + 3]) * inv);
            }
        }
        if (store) p.sums[at] = !mine || all == 0.f ? -INFINITY : (base == -INFINITY ? 0.f : base) + log2f(all);
    } else if (warp < 12) {
        // --------------------------------------------------------------------------- the pages
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        const int w = warp - 8;
        // what the table says of this lane's key of a tile; kNoKey: it is none.  Looked at a tile later
        constexpr int32_t kNoKey = INT32_MIN;
        auto look_up = [&](int tile) -> int32_t {
            const int t = begin + tile * kTile + w * 32 + lane;
            return tile < tiles && t < end ? p.prefix_table[quick_div(static_cast<uint32_t>(t), p.div_block)] : kNoKey;
        };
        auto checked = [&](int32_t said) -> int32_t {
            const bool in = said >= 0 && said < p.layer.num_blocks;
            if (!in && said != kNoKey) atomicOr(p.status, kStatusBadIndex);
            return in ? said : -1;
        };
        auto place_in_block = [&](int tile) {
            const int t = begin + tile * kTile + w * 32 + lane;
            return t - static_cast<int>(quick_div(static_cast<uint32_t>(t), p.div_block)) * static_cast<int>(p.layer.B);
        };
        if constexpr (KIND == kPlain) {
            int32_t ahead = look_up(0);
            int told = 0;  // copies whose arrival has been passed on
            // Copy u (K of tile u / 2, then V) goes to stage u % stages; up to three are in flight.
            auto pass_on = [&](int u) {
                fence_shared_to_async();
                barrier_arrive(full + 8 * (u % Shape::stages));
            };
            for (int tile = 0; tile < tiles && fine; tile++) {
                const int32_t blk = checked(ahead);
                ahead = look_up(tile + 1);
                const int64_t off = blk >= 0 ? p.layer.geo.at(blk, place_in_block(tile), h) : -1;
                const uint32_t mask = __ballot_sync(0xffffffffu, blk >= 0);
                for (int kv = 0; kv < 2; kv++) {
                    const int u = 2 * tile + kv, stage = u % Shape::stages;
                    if (u >= Shape::stages && !__all_sync(0xffffffffu, barrier_passed(empty + 8 * stage, (u / Shape::stages - 1) & 1))) {
                        // nothing to issue: pass on what is in flight as soon as it is there
                        copy_wait<0>();
                        while (told < u) pass_on(told++);
                        fine = __all_sync(0xffffffffu, barrier_wait(empty + 8 * stage, (u / Shape::stages - 1) & 1));
                        if (!fine) break;
                    }
                    // the tile whose mask this one's replaces is past its last use: its V is older than this stage's last copy
                    if (kv == 0 && lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(info + (tile % kInfos) * Shape::info + 4 * w), "r"(mask) : "memory");
                    const char *plane = kv ? p.layer.v : p.layer.k;
                    const uint32_t to = ring + stage * Shape::tile;
                    constexpr int chunks = DP / 8;
#pragma unroll
                    for (int i = 0; i < chunks; i++) {
                        const int idx = i * 32 + lane, rr = idx / chunks, ch = idx % chunks;
                        const int64_t src = __shfl_sync(0xffffffffu, off, rr);
                        const bool there = src >= 0 && ch * 8 < D;
                        copy_async16(to + swizzled(w * 32 + rr, ch), plane + (there ? src + ch * 16 : 0), there);
                    }
                    copy_commit();
                    copy_wait<2>();
                    if (told + 2 <= u) pass_on(told++);
                }
            }
            copy_wait<0>();
            if (fine)
                while (told < 2 * tiles) pass_on(told++);
        } else {
            // Codes: a warp fetches and widens its own 32 keys of every tile.  V's are multiplied by their scales over a
            // power of two that the tile's largest scale sets, 2^exponent, which puts the values below 2^16: rounded
            // to fp16 twice (the factor and the product), half a step of 2^-11 each, like the probabilities
            // that they meet.  Products below fp16's normal numbers are off by half of 2^-24, which is 2^-15 of the
            // key's scale at most, since a tile whose scales span more than 2^16 is `far`: there each key
            // has an exponent of its own.  So it is where a tile's largest scale is 2^-40 of one before.  K's scales are left to the
            // scores, in fp32, for the sake of the logarithms.
            constexpr int chunks = DP / 16;
            const uint32_t mine = staging + w * 32 * DP;
            int32_t ahead = look_up(0);
            int64_t off = -1;
            float next_k = 0.f, next_v = 0.f, scale_v = 0.f;
            uint32_t next_mask = 0;
            auto fetch = [&](int u) {
                if (u < 2 * tiles) {
                    if ((u & 1) == 0) {
                        const int tile = u >> 1, n = place_in_block(tile);
                        const int32_t blk = checked(ahead);
                        ahead = look_up(tile + 1);
                        off = blk >= 0 ? p.layer.geo.at(blk, n, h) : -1;
                    }
                    const char *plane = u & 1 ? p.layer.v : p.layer.k;
#pragma unroll
                    for (int i = 0; i < chunks; i++) {
                        const int idx = i * 32 + lane, rr = idx / chunks, ch = idx % chunks;
                        const int64_t src = __shfl_sync(0xffffffffu, off, rr);
                        const bool there = src >= 0 && ch * 16 < D;
                        copy_async16(mine + (u % Shape::staged) * Shape::codes + rr * DP + ch * 16, plane + (there ? src + ch * 16 : 0), there);
                    }
                }
                copy_commit();
            };
            // masks and scales of a tile, a tile ahead of their use
            auto fetch_scales = [&](int tile) {
                const int t = begin + tile * kTile + w * 32 + lane;
                next_k = next_v = 0.f;
                bool there = tile < tiles && t < end;
                if (there) {
                    const int32_t blk = p.prefix_table[quick_div(static_cast<uint32_t>(t), p.div_block)];
                    there = blk >= 0 && blk < p.layer.num_blocks;
                    if (there) {
                        const int64_t at = p.layer.scale_geo.at(blk, place_in_block(tile), h);
                        next_k = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.layer.k_scale) + at);
                        next_v = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.layer.v_scale) + at);
                    }
                }
                next_mask = __ballot_sync(0xffffffffu, there);
            };
            int e_most = -133;  // the largest exponent of a tile so far
            fetch_scales(0);
            for (int u = 0; u < Shape::staged - 1; u++) fetch(u);
            for (int u = 0; u < 2 * tiles; u++) {
                copy_wait<Shape::staged - 2>();
                __syncwarp();
                const int stage = u % Shape::stages, tile = u >> 1;
                if (u >= Shape::stages && fine) fine = __all_sync(0xffffffffu, barrier_wait(empty + 8 * stage, (u / Shape::stages - 1) & 1));
                const uint32_t about = info + (tile % kInfos) * Shape::info;
                if ((u & 1) == 0) {
                    // the tile whose mask and scales these replace is past its last use: its V is older than this stage's last copy
                    const float scale_k = next_k;
                    scale_v = next_v;
                    if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 4 * w), "r"(next_mask) : "memory");
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(about + 64 + 4 * (w * 32 + lane)), "f"(scale_k) : "memory");
                    fetch_scales(tile + 1);
                    const uint32_t bits = __float_as_uint(scale_v) & 0x7fffffffu, size = bits > 0x7f800000u ? 0 : bits;  // a NaN is passed over
                    const uint32_t warp_most = __reduce_max_sync(0xffffffffu, size), warp_least = __reduce_min_sync(0xffffffffu, size ? size : 0x7f800000u);
                    if (lane == 0) {
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 32 + 4 * w), "r"(warp_most) : "memory");
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(about + 48 + 4 * w), "r"(warp_least) : "memory");
                    }
                    asm volatile("bar.sync 1, 128;" ::: "memory");  // the four warps come here for every tile, whatever a wait said
                    uint32_t all[4], low[4];
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(all[0]), "=r"(all[1]), "=r"(all[2]), "=r"(all[3]) : "r"(about + 32));
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(low[0]), "=r"(low[1]), "=r"(low[2]), "=r"(low[3]) : "r"(about + 48));
                    int e = static_cast<int>(max(max(all[0], all[1]), max(all[2], all[3])) >> 23) - 127 - 6;  // a tile of zeros: the least
                    const bool far = e < e_most - 40 || static_cast<int>(min(min(low[0], low[1]), min(low[2], low[3])) >> 23) - 127 - 6 < e - 16;
                    e_most = max(e_most, e);
                    if (w == 0 && lane == 0) asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(about + 16), "f"(static_cast<float>(e)), "r"(static_cast<uint32_t>(far)) : "memory");
                    if (far) {
                        // each key's own; one of zeros takes no part in the probabilities
                        e = static_cast<int>(size >> 23) - 127 - 6;
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(about + 64 + 4 * kTile + 4 * (w * 32 + lane)), "f"(scale_v == 0.f ? -4096.f : static_cast<float>(e)) : "memory");
                    }
                    // 2^-e, up to 2^133, in two factors
                    scale_v *= __uint_as_float(static_cast<uint32_t>(127 + min(-e, 127)) << 23);
                    scale_v *= __uint_as_float(static_cast<uint32_t>(127 + max(-e - 127, 0)) << 23);
                }
                const uint32_t from = mine + (u % Shape::staged) * Shape::codes, to = ring + stage * Shape::tile;
                const uint32_t factor2 = pack2<__half>(scale_v, scale_v);
                // four 16-byte chunks of codes at a time, loads first
#pragma unroll
                for (int i0 = 0; i0 < chunks && fine; i0 += 4) {
                    uint32_t c[4][4];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int idx = (i0 + i) * 32 + lane;
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(c[i][0]), "=r"(c[i][1]), "=r"(c[i][2]), "=r"(c[i][3]) : "r"(from + idx / chunks * DP + idx % chunks * 16));
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int idx = (i0 + i) * 32 + lane, rr = idx / chunks, ch = idx % chunks;
                        // two 16-byte chunks; the lanes of the upper 64 d's write theirs in the other order, into other banks
                        const bool odd = ch >= 4;
                        uint32_t x[8];
                        widen<KIND>(odd ? c[i][2] : c[i][0], x[0], x[1]);
                        widen<KIND>(odd ? c[i][3] : c[i][1], x[2], x[3]);
                        widen<KIND>(odd ? c[i][0] : c[i][2], x[4], x[5]);
                        widen<KIND>(odd ? c[i][1] : c[i][3], x[6], x[7]);
                        if (u & 1) {
                            const uint32_t f = __shfl_sync(0xffffffffu, factor2, rr);
#pragma unroll
                            for (int j = 0; j < 8; j++) {
                                const __half2 v = __hmul2(*reinterpret_cast<const __half2 *>(&x[j]), *reinterpret_cast<const __half2 *>(&f));
                                x[j] = *reinterpret_cast<const uint32_t *>(&v);
                            }
                        }
                        const uint32_t a = to + swizzled(w * 32 + rr, 2 * ch + odd), b = to + swizzled(w * 32 + rr, 2 * ch + !odd);
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(b), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
                    }
                }
                fence_shared_to_async();
                if (fine) barrier_arrive(full + 8 * stage);
                __syncwarp();
                fetch(u + Shape::staged - 1);
            }
            copy_wait<0>();
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // ----------------------------------------------------------------------- matrix products
        // Two warps, one for each product, so that neither waits for what only the other needs.  They stay together and
        // elect the thread that issues: with uniform control the operands are uniform registers already
        // (issued from one lane's branch, products took twice as long).
        if (warp == 12) {
            const uint32_t qk = instruction<T>(kTile, false);
            for (int t = 0; t < steps && fine; t++) {
                const int slot = t & 1, tile = TWO ? t >> 1 : t, u = 2 * tile, stage = u % Shape::stages;
                if (!TWO || slot == 0) fine = barrier_wait(full + 8 * stage, (u / Shape::stages) & 1);
                // the buffer is free when the scores of the step before have been taken
                if (t && fine) fine = barrier_wait(s_taken + 8 * (slot ^ 1), ((t - 1) >> 1) & 1);
                fine = __all_sync(0xffffffffu, fine);
                if (!fine) break;
                fence_after();
                const uint64_t q_operand = operand(base + (TWO ? slot * Shape::tile : 0), 16), k_operand = operand(ring + stage * Shape::tile, 16);
                if (elected()) {
#pragma unroll
                    for (int i = 0; i < DP / 16; i++) {
                        const uint32_t at = ((i >> 2) * (kTile * 128) + (i & 3) * 32) >> 4;
                        mma_shared(tensor, q_operand + at, k_operand + at, qk, i > 0);
                    }
                    commit_to(s_full + 8 * slot);
                    if (!TWO || slot == 1) commit_to(empty + 8 * stage);
                }
                __syncwarp();
            }
        } else if (warp == 13) {
            const uint32_t pv = instruction<T>(DP, true);
            for (int t = 0; t < steps && fine; t++) {
                const int slot = t & 1, tile = TWO ? t >> 1 : t, u = 2 * tile + 1, stage = u % Shape::stages;
                if (!TWO || slot == 0) fine = barrier_wait(full + 8 * stage, (u / Shape::stages) & 1);
                if (fine) fine = barrier_wait(p_ready + 8 * slot, (t >> 1) & 1);
                fine = __all_sync(0xffffffffu, fine);
                if (!fine) break;
                fence_after();
                const uint64_t v_operand = operand(ring + stage * Shape::tile, kTile * 128);
                if (elected()) {
#pragma unroll
                    for (int i = 0; i < kTile / 16; i++) mma_tensor(tensor + 256 + slot * 128, tensor + 128 + slot * 64 + 8 * i, v_operand + i * (2048 >> 4), pv, t > 1 || i > 0);
                    if (!TWO || slot == 1) commit_to(empty + 8 * stage);
                    commit_to(o_added + 8 * slot);
                }
                __syncwarp();
            }
        }
        if (warp < 14 && !fine) {
            // products may be in flight: let them end before the tensor memory is given back
            const uint32_t last = tensor_at + 8 + 8 * (warp - 12);
            if (elected()) commit_to(last);
            __syncwarp();
            barrier_wait(last, 0);
        }
    }
    if (!fine) atomicOr(p.status, static_cast<unsigned int>(TC_DEVICE_BULK_WAIT_TIMEOUT));
    fence_before();
    __syncthreads();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tensor) : "memory");
}

template <typename T, int KIND, int DP, bool TWO>
static int launch_prefix_shape(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    using Shape = PrefixShape<KIND, DP, TWO>;
    static_assert(Shape::bytes <= 232448, "more shared memory than a CTA can have");
    static std::atomic<bool> raised[kMaxDevices];  // set once per device; setting it twice does no harm
    if (!raised[device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(prefix_kernel<T, KIND, DP, TWO>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::bytes);
        if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(dynamic shared memory)");
        raised[device].store(true, std::memory_order_relaxed);
    }
    return launch_attn(prefix_kernel<T, KIND, DP, TWO>, grid, kPrefixThreads, Shape::bytes, false, p, s);
}

template <typename T, int KIND>
static int launch_prefix_type(const AttnParams &p, unsigned grid, int device, cudaStream_t s)
{
    const bool two = p.split.prefix_rows == 256;
    if (p.layer.D <= 64) return two ? launch_prefix_shape<T, KIND, 64, true>(p, grid, device, s) : launch_prefix_shape<T, KIND, 64, false>(p, grid, device, s);
    return two ? launch_prefix_shape<T, KIND, 128, true>(p, grid, device, s) : launch_prefix_shape<T, KIND, 128, false>(p, grid, device, s);
}

int launch_prefix(const AttnParams &p, int dtype, int device, cudaStream_t s)
{
    const int64_t chunks = p.split.prefix_rows == 256 ? p.split.prefix_parts : p.split.prefix_parts / 2;
    const int64_t ctas = chunks * p.layer.H * p.split.prefix_blocks;
    if (ctas > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "%lld parts: too many for one call", (long long)ctas);
    const unsigned grid = static_cast<unsigned>(ctas);
    switch (p.layer.dtype) {
    case TC_E4M3: return launch_prefix_type<__half, kE4m3>(p, grid, device, s);
    case TC_INT8: return launch_prefix_type<__half, kInt8>(p, grid, device, s);
    default: return dtype == TC_BF16 ? launch_prefix_type<__nv_bfloat16, kPlain>(p, grid, device, s) : launch_prefix_type<__half, kPlain>(p, grid, device, s);
    }
}

}  // namespace tc
