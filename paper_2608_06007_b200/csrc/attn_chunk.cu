// tc_attn_chunk: the entry points, unquantised pools, and the kernel that joins the parts of requests whose keys are cut.
#include <cmath>
#include <numeric>

#include "attn_chunk.cuh"

namespace tc {

int launch_chunk_plain(const ChunkParams &p, int dtype, int device, cudaStream_t s)
{
    return dtype == TC_BF16 ? launch_chunk_type<__nv_bfloat16, kPlain>(p, device, s) : launch_chunk_type<__half, kPlain>(p, device, s);
}

// The parts' outputs, each by its share of the whole sum.  A warp takes a row; a lane finds the weights of up to four parts,
// then the warp reads the outputs of four parts at once.  Where nothing was cut it ends after a look at `cuts`.
constexpr float kLess = 12.f;  // weights are 2^-12 at most: the outputs of up to that many parts may be next to the largest number
static_assert(kChunkMostParts <= 128);
template <typename T, int DP>
__global__ void __launch_bounds__(128) chunk_join_kernel(const __grid_constant__ ChunkParams p)
{
    constexpr int kVectors = DP / 128;
    const int lane = threadIdx.x & 31, D = p.layer.D;
    const int64_t first_warp = blockIdx.x * 4ll + (threadIdx.x >> 5), warps = gridDim.x * 4ll;
    await_last();
    for (int64_t r0 = 0; r0 < p.R; r0 += 32) {
        const ChunkRequest mine = r0 + lane < p.R ? chunk_request(p, r0 + lane, false) : ChunkRequest{0, 0, 0};
        const uint2 cut = mine.n ? p.cuts[r0 + lane] : make_uint2(0, 0);
        // (where a call's kernel gave up, or offsets made more items than its grid holds, nobody may have said)
        const bool said = cut.y > 1 && cut.y <= kChunkMostParts && cut.x + static_cast<int64_t>(cut.y) * mine.n * p.Hq <= p.plan.part_rows;
        for (uint32_t some = __ballot_sync(0xffffffffu, said); some; some &= some - 1) {
            const int who = __ffs(some) - 1;
            const uint32_t base = __shfl_sync(0xffffffffu, cut.x, who);
            const int32_t parts = static_cast<int32_t>(__shfl_sync(0xffffffffu, cut.y, who));
            const int64_t rows = static_cast<int64_t>(__shfl_sync(0xffffffffu, mine.n, who)) * p.Hq, token0 = __shfl_sync(0xffffffffu, mine.token0, who);
            for (int64_t row = first_warp; row < rows; row += warps) {
                const int64_t token = row / p.Hq, head = row - token * p.Hq;
                float sum[4], top = -INFINITY, all = 0.f, acc[4 * kVectors] = {};
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    sum[k] = lane + 32 * k < parts ? p.sums[base + (lane + 32 * k) * rows + row] : -INFINITY;
                    top = fmaxf(top, sum[k]);
                }
#pragma unroll
                for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const bool some = sum[k] != -INFINITY;
                    sum[k] = some ? exp2_approx(sum[k] - (top == -INFINITY ? 0.f : top) - kLess) : -1.f;  // NaN where the sum is; -1: no part, or one without weight
                    if (some) all += sum[k];
                }
#pragma unroll
                for (int x = 16; x; x >>= 1) all += __shfl_xor_sync(0xffffffffu, all, x);
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    for (int j0 = 32 * k; j0 < min(parts, 32 * k + 32); j0 += 4) {
                        float4 v[4][kVectors];
#pragma unroll
                        for (int j = 0; j < 4; j++)
#pragma unroll
                            for (int x = 0; x < kVectors; x++) {
                                v[j][x] = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (j0 + j < parts && lane * 4 + 128 * x < D) v[j][x] = *reinterpret_cast<const float4 *>(p.parts + (base + (j0 + j) * rows + row) * D + lane * 4 + 128 * x);
                            }
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const float w = __shfl_sync(0xffffffffu, sum[k], (j0 + j) & 31);
                            // what a part without keys left in its place is read but not used; one whose weight is 0 in fp32 may not be finite
                            if (w < 0.f || j0 + j >= parts) continue;
#pragma unroll
                            for (int x = 0; x < kVectors; x++) acc[4 * x] += w * v[j][x].x, acc[4 * x + 1] += w * v[j][x].y, acc[4 * x + 2] += w * v[j][x].z, acc[4 * x + 3] += w * v[j][x].w;
                        }
                    }
                }
                const float inv = all == 0.f ? 0.f : 1.f / all;
                char *const dst = p.out + (token0 + token) * p.out_token + head * p.out_head;
#pragma unroll
                for (int x = 0; x < kVectors; x++)
                    if (lane * 4 + 128 * x < D)
                        *reinterpret_cast<uint2 *>(dst + (lane * 4 + 128 * x) * 2) = make_uint2(pack2<T>(acc[4 * x] * inv, acc[4 * x + 1] * inv), pack2<T>(acc[4 * x + 2] * inv, acc[4 * x + 3] * inv));
                if (p.lse && lane == 0) p.lse[token0 * p.Hq + row] = all == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + kLess + log2f(all)) * kChunkLn2;
            }
        }
    }
}

// Tensor maps, where a call's geometry fits them: queries as [token][head][d], whose boxes are the whole tokens that an item's slot of 128
// rows holds; pages of an unquantised pool as [block][head][token][d], in boxes of as many tokens as divide a block and half a tile.
// Elsewhere q_boxes or box_rows stays 0.
constexpr int32_t kLeastBox = 4;  // tokens: 16 prompts in blocks of 20 take 404 us so, 544 key by key
static int describe_boxes(ChunkParams *p)
{
    p->box_rows = p->q_boxes = 0;
    const Layer &l = p->layer;
    const int32_t group = p->shape.group, rows = static_cast<int32_t>(std::gcd<int64_t>(l.B, p->shape.keys / 2));
    const bool queries = 128 % group == 0, pages = !l.quantised() && rows >= kLeastBox && l.num_blocks > 0;
    if (!queries && !pages) return TC_OK;
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<Encode> known;  // looked up once; twice does no harm
    Encode encode = known.load(std::memory_order_relaxed);
    if (!encode) {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return cuda_fail(e, "cudaGetDriverEntryPointByVersion(cuTensorMapEncodeTiled)");
        if (found != cudaDriverEntryPointSuccess || !f) return fail(TC_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
        encode = reinterpret_cast<Encode>(f);
        known.store(encode, std::memory_order_relaxed);
    }
    // 64 elements wide, swizzled as the products read them; false for a geometry that tensor maps do not hold
    auto map = [&](CUtensorMap *m, const void *at, int rank, const cuuint64_t *extent, const cuuint64_t *stride, const cuuint32_t *box) {
        const cuuint32_t step[4] = {1, 1, 1, 1};
        for (int i = 0; i + 1 < rank; i++)
            if (stride[i] == 0 || stride[i] >= (1ull << 40)) return false;
        return encode(m, p->q_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, static_cast<cuuint32_t>(rank), const_cast<void *>(at), extent, stride, box, step,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    using Size = cuuint64_t;
    if (queries) {
        const Size row = l.D * 2ll, extent[3] = {static_cast<Size>(l.D), static_cast<Size>(p->Hq), static_cast<Size>(p->n_tokens)};
        const Size stride[2] = {p->Hq > 1 ? static_cast<Size>(p->q_head) : row, p->n_tokens > 1 ? static_cast<Size>(p->q_token) : row * p->Hq};
        const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(group), static_cast<cuuint32_t>(128 / group)};
        p->q_boxes = map(&p->map_q, p->q, 3, extent, stride, box);
    }
    if (pages) {
        const Size extent[4] = {static_cast<Size>(l.D), l.B, static_cast<Size>(l.H), static_cast<Size>(l.num_blocks)};
        const Size stride[3] = {static_cast<Size>(l.geo.token), static_cast<Size>(l.geo.head), static_cast<Size>(l.geo.block)};
        const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(rows), 1, 1};
        if (map(&p->map_k, l.k, 4, extent, stride, box) && map(&p->map_v, l.v, 4, extent, stride, box)) p->box_rows = rows, p->div_box = make_fastdiv(static_cast<uint32_t>(rows));
    }
    return TC_OK;
}

// Requests with one new token go to the stream where there may be some number of them: it reads codes at some 4 TB/s and 16-bit numbers
// at 6, where items of 256 rows, of which these have a few, take a tile as slowly as if they were full (64 requests, 51 of them single, 200k tokens
// of 8 heads x 128, e4m3: a call of 386 us so, 570 without, before requests of many blocks had kernels of their own).  Its two launches cost some 12 us,
// and nothing else tells a call of fewer requests from one of prompts.  300 tokens behind 2000 beside R - 1 single ones behind 8000 (30000), us with it and
// without: bf16 R = 4: 92 and 69 (137, 132), R = 8: 119, 107 (211, 225), R = 16: 158, 156 (344, 419); e4m3 R = 4: 102, 136 (129, 232), R = 8: 120, 210 (184, 437).
// Prompts of 200 alone, bf16, R = 8: 46, 34.  So codes would gain from fewer than eight on, where some are single, and 16-bit pools lose up to there.
constexpr int64_t kLeastSingles = 8;
// Bytes of tiles made fp16 at most.  8 prompts of up to 15061 tokens in a window of 2048, int8, of 8 heads x 128: 1.93 ms so, with 493 MB of them, 3.12 where
// each block widens its own; 64 requests, four of them of 104 to 374 new tokens behind up to 10883, e4m3: 280 us, of which these tiles take 32, and 387.
constexpr int64_t kMostWide = 1ll << 30;

// What a call launches, in one workspace.
struct ChunkCall {
    ChunkParams most;     // requests that meet the pages as they lie
    ChunkParams wide;     // those whose codes are made fp16 before
    AttnParams singles;   // those with one new token
    bool has_wide, has_singles;
    int64_t singles_at, wide_at, workspace;
};

// What both entry points check; fills the kernels' geometry and plans.
static int check_chunk(const tc_kv_layer_t *layer, const tc_attn_chunk_t *a, ChunkCall *c)
{
    ChunkParams *const p = &c->most;
    int rc = check_layer(layer, &p->layer);
    if (rc != TC_OK) return rc;
    if (!a) return fail(TC_ERR_INVALID_ARG, "args is required");
    if (a->struct_size != sizeof *a) return fail(TC_ERR_INVALID_ARG, "args.struct_size %u != %zu: header and library disagree", a->struct_size, sizeof *a);
    if (a->dtype != TC_BF16 && a->dtype != TC_FP16) return fail(TC_ERR_INVALID_ARG, "dtype %d: q and out are TC_BF16 or TC_FP16", a->dtype);
    if (!p->layer.quantised() && p->layer.dtype != a->dtype) return fail(TC_ERR_INVALID_ARG, "an unquantised pool must have the queries' dtype (pool %d, queries %d)", p->layer.dtype, a->dtype);
    const int D = p->layer.D;
    if (D % 16 || D > 256) return fail(TC_ERR_SHAPE, "D = %d: tc_attn_chunk takes multiples of 16 up to 256", D);
    if (p->layer.align < 16) return fail(TC_ERR_INVALID_ARG, "tc_attn_chunk needs planes and strides that are multiples of 16 bytes");
    if (a->R < 0 || a->R > (1 << 24)) return fail(TC_ERR_SHAPE, "R %lld is not in [0, 2^24]", (long long)a->R);
    if (a->Hq < 1 || a->Hq > (1 << 16) || a->Hq % p->layer.H) return fail(TC_ERR_SHAPE, "Hq %lld is not a multiple of H = %d in [1, 2^16]", (long long)a->Hq, p->layer.H);
    if (a->n_tokens < 0 || a->n_tokens > (1 << 30)) return fail(TC_ERR_SHAPE, "n_tokens %lld is not in [0, 2^30]", (long long)a->n_tokens);
    if (a->max_len < 0 || a->max_len > (1 << 24)) return fail(TC_ERR_SHAPE, "max_len %lld is not in [0, 2^24]", (long long)a->max_len);
    if (a->max_new < 0 || a->max_new > a->max_len) return fail(TC_ERR_SHAPE, "max_new %lld is not in [0, max_len = %lld]", (long long)a->max_new, (long long)a->max_len);
    if (a->window < 0 || a->sinks < 0) return fail(TC_ERR_SHAPE, "window %lld and sinks %lld must not be negative", (long long)a->window, (long long)a->sinks);
    if (a->sinks && !a->window) return fail(TC_ERR_INVALID_ARG, "sinks without a window: every key is seen");
    if (a->reserved) return fail(TC_ERR_INVALID_ARG, "reserved is %d, not 0", a->reserved);
    if (!(std::fabs(a->scale) <= 1e30f)) return fail(TC_ERR_INVALID_ARG, "scale is not a number of at most 1e30");
    p->shape = chunk_shape(static_cast<int32_t>(a->Hq / p->layer.H), chunk_rows(D), chunk_keys(D), static_cast<int32_t>(a->window ? std::min<int64_t>(a->window, 1 << 30) : 1 << 30),
                           static_cast<int32_t>(std::min<int64_t>(a->sinks, 1 << 30)), p->layer.H);
    p->shape.turns = p->layer.quantised() && p->shape.rows == 256;
    const ChunkShape &s = p->shape;
    const int64_t new_most = std::min(a->max_new, a->n_tokens);
    if (new_most * s.group > INT32_MAX - 4096 || a->R * chunk_blocks(s, static_cast<int32_t>(new_most)) > INT32_MAX / s.heads)
        return fail(TC_ERR_TOO_LARGE, "R = %lld requests of up to %lld tokens x %lld heads: too many for one call", (long long)a->R, (long long)new_most, (long long)a->Hq);
    p->R = a->R, p->n_tokens = a->n_tokens, p->max_new = a->max_new, p->max_len = a->max_len;
    const int64_t most = a->window ? std::min(a->max_len, std::min(a->window, a->max_len) + std::min(a->sinks, a->max_len) + 96) : a->max_len;
    // (what the stream's 32-bit counts of rows and tiles do not hold goes without it)
    bool fits = a->R * a->Hq <= (1 << 30) && a->R * p->layer.H <= (1 << 30) / std::max<int64_t>(1, (most + 15) / 16);
    if (fits && (a->max_new == 1 || a->R >= kLeastSingles)) {
        c->singles.layer = p->layer;
        split_attn(a->R, a->Hq, p->layer.H, D, most, 0, p->layer.quantised(), &c->singles.split);
        c->has_singles = fits = c->singles.split.stream_tiles < (1ll << 31);
    }
    p->new_from = c->has_singles ? 2 : 1, p->new_to = a->max_new;
    // Codes that three blocks of a request's rows meet, or more, are made fp16 once, where the requests that may have as many fit into
    // kMostWide; else those of the requests with the most new tokens.  16 requests of four query heads a KV head, e4m3, us so and where each block widens
    // its own: two blocks behind 2000 176 and 188, three 221 and 261, four 266 and 335; behind 16000 (4 requests) 276 and 292, 342 and 403, 396 and 527.
    // With nothing cached the tiles are few and it costs some 15: 67 and 52, 82 and 64, 96 and 84; two blocks lose there what they gain behind 2000.
    if (p->layer.quantised() && a->max_new > 1 && new_most * s.group > 2 * s.rows) {
        const int64_t near = (std::min<int64_t>(s.window, a->max_len) + new_most) / s.keys + 2 + chunk_tiles_of(s, static_cast<int32_t>(std::min<int64_t>(s.sinks, a->max_len)));
        const int64_t list = std::min<int64_t>(near, chunk_tiles_of(s, static_cast<int32_t>(a->max_len))), bytes = list * s.heads * wide_tile_bytes(D), room = kMostWide / bytes;
        int64_t from = std::max<int64_t>(2 * s.rows / s.group + 1, p->new_from);
        if (std::min(a->R, a->n_tokens / from) > room) from = a->n_tokens / (room + 1) + 1;
        if (room > 0 && from <= new_most) {
            ChunkParams *const w = &c->wide;
            c->has_wide = true;
            *w = *p;
            w->new_from = from, p->new_to = from - 1;
            w->wide_by_request = a->R <= a->n_tokens / from;
            w->wide_requests = std::min(a->R, a->n_tokens / from);
            w->wide_list = static_cast<int32_t>(list);
            w->div_wide = make_fastdiv(static_cast<uint32_t>(from));
            plan_chunk(s, w->wide_requests, a->n_tokens, a->max_new, a->max_len, D, &w->plan);
        }
    }
    // `cuts`, then the sums and outputs of the parts' rows of all kernels
    ChunkPlan &plan = p->plan;
    if (a->max_new > 1 && p->new_from <= p->new_to) plan_chunk(s, a->R, a->n_tokens, p->new_to, a->max_len, D, &plan);
    auto place = [&](int64_t bytes) {
        const int64_t at = c->workspace;
        c->workspace += (bytes + 255) / 256 * 256;
        return at;
    };
    const int64_t part_rows = plan.part_rows + c->wide.plan.part_rows;  // (max_len decides whether anything may be cut: of both or of neither)
    if (part_rows) plan.cuts_at = place(a->R * 8), plan.sums_at = place(part_rows * 4), plan.parts_at = place(part_rows * D * 4);
    c->singles_at = place(c->has_singles ? c->singles.split.workspace : 0);
    c->wide_at = place(c->has_wide ? c->wide.wide_requests * c->wide.wide_list * s.heads * wide_tile_bytes(D) : 0);
    if (a->max_new == 1 && !fits) return fail(TC_ERR_TOO_LARGE, "R * H * keys = %lld * %d * %lld: too many for one call", (long long)a->R, p->layer.H, (long long)most);
    return TC_OK;
}

template <typename T>
static int launch_chunk(const ChunkCall &c, int dtype, int device, cudaStream_t s)
{
    const ChunkParams &p = c.most;
    int rc = TC_OK;
    if (c.has_singles) {
        if ((rc = launch_singles_stream(c.singles, dtype, device, s)) != TC_OK) return rc;
        if (p.max_new == 1) return launch_singles_join(c.singles, dtype, s);
    }
    if (p.new_from <= p.new_to) rc = p.layer.quantised() ? launch_chunk_codes(p, device, s) : launch_chunk_plain(p, dtype, device, s);
    if (rc == TC_OK && c.has_wide) rc = launch_chunk_wide(c.wide, device, s);
    if (rc == TC_OK && c.has_singles) rc = launch_singles_join(c.singles, dtype, s);
    ChunkParams all = p;
    if (c.has_wide) all.new_to = c.wide.new_to, all.plan.part_rows += c.wide.plan.part_rows;
    if (rc != TC_OK || !all.plan.part_rows) return rc;
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>((p.n_tokens * p.Hq + 3) / 4, kChunkSms * 8));
    return p.layer.D <= 128 ? launch_attn(chunk_join_kernel<T, 128>, grid, 128, 0, true, all, s) : launch_attn(chunk_join_kernel<T, 256>, grid, 128, 0, true, all, s);
}

}  // namespace tc

using namespace tc;

extern "C" int tc_attn_chunk_workspace(const tc_kv_layer_t *layer, const tc_attn_chunk_t *a, int64_t *bytes)
{
    clear_error();
    if (!bytes) return fail(TC_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    ChunkCall c{};
    const int rc = check_chunk(layer, a, &c);
    if (rc == TC_OK) *bytes = c.workspace;
    return rc;
}

extern "C" int tc_attn_chunk(const tc_kv_layer_t *layer, const tc_attn_chunk_t *a, void *stream)
{
    clear_error();
    ChunkCall c{};
    int rc = check_chunk(layer, a, &c);
    if (rc != TC_OK) return rc;
    ChunkParams &p = c.most;
    const int64_t need = c.workspace;
    if (a->R == 0 || a->n_tokens == 0 || a->max_new == 0) return TC_OK;
    uint32_t align = 16;
    const int64_t row = p.layer.D * 2ll;
    if ((rc = check_rows("q", a->q, a->q_stride, a->n_tokens, a->Hq, row, 2, false, &align)) != TC_OK) return rc;
    if ((rc = check_rows("out", a->out, a->out_stride, a->n_tokens, a->Hq, row, 2, true, &align)) != TC_OK) return rc;
    if (align < 16) return fail(TC_ERR_INVALID_ARG, "q, out and their strides must be multiples of 16 bytes");
    if (a->q == a->out) return fail(TC_ERR_OVERLAP, "out is q: the queries are read after the first outputs are written");
    if (reinterpret_cast<uintptr_t>(a->lse) % 4) return fail(TC_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    if (!a->lens || reinterpret_cast<uintptr_t>(a->lens) % 4) return fail(TC_ERR_INVALID_ARG, "lens is required, 4-byte aligned");
    if (!a->offsets || reinterpret_cast<uintptr_t>(a->offsets) % 8) return fail(TC_ERR_INVALID_ARG, "offsets is required, 8-byte aligned");
    if (!a->tables || reinterpret_cast<uintptr_t>(a->tables) % 4 || a->table_stride % 4 || a->table_stride < 0)
        return fail(TC_ERR_INVALID_ARG, "tables is required; address and table_stride are multiples of 4 bytes");
    if (a->table_width < (a->max_len + p.layer.B - 1) / p.layer.B)
        return fail(TC_ERR_BOUNDS, "table_width %lld holds %lld tokens, max_len is %lld", (long long)a->table_width, (long long)(a->table_width * p.layer.B), (long long)a->max_len);
    if (need && (!a->workspace || reinterpret_cast<uintptr_t>(a->workspace) % 16)) return fail(TC_ERR_INVALID_ARG, "workspace is required, 16-byte aligned");
    if (a->workspace_bytes < need)
        return fail(TC_ERR_BOUNDS, "workspace_bytes %lld < %lld (tc_attn_chunk_workspace)", (long long)a->workspace_bytes, (long long)need);
    if (const int64_t items = std::max(p.plan.grid, c.wide.plan.grid); items > INT32_MAX) return fail(TC_ERR_TOO_LARGE, "%lld items: too many for one call", (long long)items);
    int device, sms;
    if ((rc = op_device(&device, &p.status, &sms)) != TC_OK) return rc;
    const struct {
        const char *name;
        const void *p;
    } pointers[] = {{"layer.k", layer->k}, {"layer.v", layer->v}, {"layer.k_scale", layer->k_scale}, {"layer.v_scale", layer->v_scale}, {"q", a->q}, {"out", a->out},
                    {"lse", a->lse}, {"lens", a->lens}, {"offsets", a->offsets}, {"tables", a->tables}, {"workspace", need ? a->workspace : nullptr}};
    for (const auto &ptr : pointers)
        if (ptr.p && (rc = check_memory(ptr.name, ptr.p, device)) != TC_OK) return rc;
    p.q = static_cast<const char *>(a->q);
    p.q_token = a->q_stride[0], p.q_head = a->q_stride[1];
    p.out = static_cast<char *>(a->out);
    p.out_token = a->out_stride[0], p.out_head = a->out_stride[1];
    p.lse = a->lse;
    p.tables = reinterpret_cast<const char *>(a->tables);
    p.table_stride = a->table_stride;
    p.offsets = a->offsets, p.lens = a->lens;
    p.Hq = static_cast<int32_t>(a->Hq);
    p.q_bf16 = a->dtype == TC_BF16;
    p.item_spins = static_cast<uint32_t>(chunk_patience(chunk_tiles(p.shape, static_cast<int32_t>(a->max_len)))) * kWaitSpins;
    p.scale_log2 = static_cast<float>((a->scale != 0.f ? static_cast<double>(a->scale) : 1.0 / std::sqrt(static_cast<double>(p.layer.D))) * 1.4426950408889634);
    p.div_block = make_fastdiv(p.layer.B);
    p.div_group = make_fastdiv(static_cast<uint32_t>(p.shape.group));
    if ((rc = describe_boxes(&p)) != TC_OK) return rc;
    char *const ws = static_cast<char *>(a->workspace);
    p.cuts = reinterpret_cast<uint2 *>(ws + p.plan.cuts_at);
    p.sums = reinterpret_cast<float *>(ws + p.plan.sums_at);
    p.parts = reinterpret_cast<float *>(ws + p.plan.parts_at);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    p.beside = c.has_singles;
    if (c.has_wide) {
        const ChunkParams w = c.wide;
        c.wide = p;
        c.wide.new_from = w.new_from, c.wide.new_to = w.new_to, c.wide.plan = w.plan;
        c.wide.wide_by_request = w.wide_by_request, c.wide.wide_requests = w.wide_requests, c.wide.wide_list = w.wide_list, c.wide.div_wide = w.div_wide;
        c.wide.wide = ws + c.wide_at;
        c.wide.first_part_row = static_cast<uint32_t>(p.plan.part_rows);
        c.wide.sums += p.plan.part_rows, c.wide.parts += p.plan.part_rows * p.layer.D;
        c.wide.beside = false;  // its tiles have to be there
        c.wide.widen_beside = c.has_singles || p.new_from <= p.new_to;
    }
    if (c.has_singles) {
        AttnParams &q = c.singles;
        q.q = p.q, q.q_req = p.q_token, q.q_head = p.q_head;
        q.out = p.out, q.out_req = p.out_token, q.out_head = p.out_head;
        q.lse = p.lse;
        q.tables = p.tables, q.table_width = a->table_width, q.table_stride = p.table_stride;
        q.lens = p.lens, q.offsets = p.offsets, q.n_tokens = p.n_tokens, q.max_new = p.max_new;
        q.R = p.R, q.max_len = p.max_len;
        q.window = p.shape.window, q.sinks = p.shape.sinks;
        q.Hq = p.Hq, q.q_bf16 = p.q_bf16, q.scale_log2 = p.scale_log2;
        q.div_block = p.div_block, q.div_group = p.div_group, q.div_heads = make_fastdiv(static_cast<uint32_t>(p.Hq));
        q.status = p.status;
        char *const at = ws + c.singles_at;
        q.sums = reinterpret_cast<float *>(at + q.split.sums_at), q.parts = reinterpret_cast<float *>(at + q.split.parts_at);
        q.piece_sums = reinterpret_cast<float *>(at + q.split.piece_sums_at), q.pieces = reinterpret_cast<float *>(at + q.split.pieces_at);
        q.before = reinterpret_cast<uint32_t *>(at + q.split.before_at);
    }
    return a->dtype == TC_BF16 ? launch_chunk<__nv_bfloat16>(c, a->dtype, device, s) : launch_chunk<__half>(c, a->dtype, device, s);
}
