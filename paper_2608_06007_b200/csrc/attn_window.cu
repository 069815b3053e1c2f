// tc_attn_decode_window: one query token per request over its last tokens and its first ones.  The keys that it sees are two runs, so
// the stream's tiles are those of both, one behind the other, and all else is as without a window (attn_stream.cuh).  Bound by HBM, by
// issue for codes: 64 requests of 4096 keys and 4 sinks, bf16, 797 MB: 134 us, 6.0 TB/s; 512 of 1024, e4m3: 155 us, 4.9 TB/s (164 in
// a long run).
#include "attn_stream.cuh"

namespace tc {

int launch_window(const AttnParams &p, int dtype, int device, cudaStream_t s)
{
    return dtype == TC_BF16 ? launch_stream_and_join<__nv_bfloat16, kWindow>(p, device, s) : launch_stream_and_join<__half, kWindow>(p, device, s);
}

}  // namespace tc
