// tc_attn_chunk over codes that many blocks of rows meet: every tile is made fp16 once, and the items take it as it lies.
//
// A block of 256 rows widens what it meets, which costs its CTA more than the products and the softmax do.  Where a request has many
// blocks, they would widen the same tiles again and again; here one CTA a tile does it for all: bytes to read once, twice as many to write
// once, and then to read from L2 as often as blocks meet them.  Bound by HBM: 3800 tiles of 128 keys x 128 of int8, 125 MB and
// 250 MB written: 83 us, 4.5 TB/s.  The items behind it take some 5000 clocks a tile, where 16-bit pools take 3600: each thread loads
// 128 scales of K and as many of V from shared memory a tile, 2000 clocks of its bandwidth for eight warps.
#include "attn_chunk.cuh"

namespace tc {

// A CTA has a tile of one request and KV head: four warps K, four V, each a quarter of the keys.
template <int KIND, int DP> __device__ __forceinline__ void widen_tile(const ChunkParams &p)
{
    using W = WideTile<DP>;
    constexpr int kKeys = W::keys, kMine = kKeys / 4, chunks = DP / 16, kUnits = kMine * chunks / 32;
    __shared__ uint32_t most_of[4], least_of[4], bad_of[4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, kv = warp >> 2, w = warp & 3, H = p.layer.H, D = p.layer.D;
    const int h = blockIdx.x % H, listed = static_cast<int>(blockIdx.x / H % p.wide_list);
    int64_t r = blockIdx.x / H / p.wide_list;
    if (!p.wide_by_request) {
        // the request whose place this is
        __shared__ int found;
        if (threadIdx.x == 0) found = -1;
        __syncthreads();
        for (int64_t i = threadIdx.x; i < p.R; i += 256) {
            const ChunkRequest q = chunk_request(p, i, false);
            if (q.n && wide_place(p, i, q.token0) == r) found = static_cast<int>(i);
        }
        __syncthreads();
        if (found < 0) return;
        r = found;
    }
    const ChunkRequest q = chunk_request(p, r, false);
    if (!q.n) return;
    const ChunkList list = chunk_list(p.shape, q.len - q.n, 0, q.n * p.shape.group, q.n * p.shape.group);
    if (listed >= list.count) return;
    const int t = (listed < list.firsts ? listed : listed + list.skip) * kKeys + w * kMine + lane;
    int32_t blk = -1;
    if (lane < kMine && t < list.key_end && (t >= list.key_low || t < p.shape.sinks)) {
        blk = reinterpret_cast<const int32_t *>(p.tables + r * p.table_stride)[quick_div(static_cast<uint32_t>(t), p.div_block)];
        if (blk < 0 || blk >= p.layer.num_blocks) atomicOr(p.status, kStatusBadIndex), blk = -1;
    }
    int64_t off = -1;
    float scale_k = 0.f, scale_v = 0.f;
    if (blk >= 0) {
        const int n = t - static_cast<int>(quick_div(static_cast<uint32_t>(t), p.div_block)) * static_cast<int>(p.layer.B);
        off = p.layer.geo.at(blk, n, h);
        const int64_t at = p.layer.scale_geo.at(blk, n, h);
        scale_k = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.layer.k_scale) + at);
        scale_v = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.layer.v_scale) + at);
    }
    const char *const plane = kv ? p.layer.v : p.layer.k;
    uint4 codes[kUnits];
#pragma unroll
    for (int j = 0; j < kUnits; j++) {
        const int idx = j * 32 + lane, ch = idx % chunks;
        const int64_t src = __shfl_sync(0xffffffffu, off, idx / chunks);
        codes[j] = make_uint4(0, 0, 0, 0);
        if (src >= 0 && ch * 16 < D) codes[j] = *reinterpret_cast<const uint4 *>(plane + src + ch * 16);
    }
    const uint32_t mask = __ballot_sync(0xffffffffu, blk >= 0);
    // V's exponents, as where a CTA widens its own tiles
    const ScaleOfV v = scale_of_v(scale_v);
    const uint32_t warp_most = __reduce_max_sync(0xffffffffu, v.size), warp_least = __reduce_min_sync(0xffffffffu, v.size ? v.size : 0x7f800000u);
    if (kv && lane == 0) most_of[w] = warp_most, least_of[w] = warp_least;
    __syncthreads();
    const int e = ScaleOfV::exponent_of(max(max(most_of[0], most_of[1]), max(most_of[2], most_of[3])));
    const bool far = ScaleOfV::exponent_of(min(min(least_of[0], least_of[1]), min(least_of[2], least_of[3]))) < e - 16;
    char *const to = p.wide + ((wide_place(p, r, q.token0) * p.wide_list + listed) * H + h) * W::bytes;
    uint32_t bad = !(fabsf(scale_v) < INFINITY);
#pragma unroll
    for (int j = 0; j < kUnits; j++) {
        const int idx = j * 32 + lane, rr = idx / chunks, ch = idx % chunks;
        uint32_t x[8];
        widen<KIND>(codes[j].x, x[0], x[1]);
        widen<KIND>(codes[j].y, x[2], x[3]);
        widen<KIND>(codes[j].z, x[4], x[5]);
        widen<KIND>(codes[j].w, x[6], x[7]);
#pragma unroll
        for (int k = 0; k < 8; k++) bad |= not_finite<__half>(x[k]);
        char *const tile = to + kv * W::tile;
        *reinterpret_cast<uint4 *>(tile + swizzled<kKeys>(w * kMine + rr, 2 * ch)) = make_uint4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<uint4 *>(tile + swizzled<kKeys>(w * kMine + rr, 2 * ch + 1)) = make_uint4(x[4], x[5], x[6], x[7]);
    }
    bad = __any_sync(0xffffffffu, bad != 0);
    if (kv && lane == 0) bad_of[w] = bad;
    if (!kv) {
        float *const scales = reinterpret_cast<float *>(to + W::scales_at);
        if (lane < kMine) {
            scales[w * kMine + lane] = scale_k;
            // (where a later part finds the tile far from those before it, all of its keys have the tile's exponent)
            scales[kKeys + w * kMine + lane] = v.exponent(far, e), scales[2 * kKeys + w * kMine + lane] = v.rest(far, e);
        }
        if (lane == 0) {
            if constexpr (kMine == 32) reinterpret_cast<uint32_t *>(to + W::header_at)[w] = mask;
            else reinterpret_cast<uint16_t *>(to + W::header_at)[w] = static_cast<uint16_t>(mask);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t *const header = reinterpret_cast<uint32_t *>(to + W::header_at);
        header[4] = static_cast<uint32_t>(e), header[5] = far, header[6] = bad_of[0] | bad_of[1] | bad_of[2] | bad_of[3];
    }
}

template <int KIND, int DP>
__global__ void __launch_bounds__(256) chunk_widen_kernel(const __grid_constant__ ChunkParams p)
{
    widen_tile<KIND, DP>(p);
    if (p.widen_beside && blockIdx.x == 0) await_last();  // this kernel has not ended before those before it have
}

template <int DP>
static int launch_wide_shape(const ChunkParams &p, int device, cudaStream_t s)
{
    const unsigned grid = static_cast<unsigned>(p.wide_requests * p.wide_list * p.layer.H);
    const int rc = p.layer.dtype == TC_E4M3 ? launch_attn(chunk_widen_kernel<kE4m3, DP>, grid, 256, 0, p.widen_beside, p, s) : launch_attn(chunk_widen_kernel<kInt8, DP>, grid, 256, 0, p.widen_beside, p, s);
    return rc != TC_OK ? rc : launch_chunk_shape<__half, kWide, DP>(p, device, s);
}

int launch_chunk_wide(const ChunkParams &p, int device, cudaStream_t s)
{
    if (p.layer.D <= 64) return launch_wide_shape<64>(p, device, s);
    if (p.layer.D <= 128) return launch_wide_shape<128>(p, device, s);
    return launch_wide_shape<256>(p, device, s);
}

}  // namespace tc
