// The requests of a tc_attn_chunk call that have one new token: few rows a request, so that reading their keys is all the time there is, and the
// stream of tc_attn_decode_window takes them.
#include "attn_stream.cuh"

namespace tc {

int launch_singles_stream(const AttnParams &p, int dtype, int device, cudaStream_t s)
{
    return dtype == TC_BF16 ? launch_stream_alone<__nv_bfloat16, kSingles>(p, device, s) : launch_stream_alone<__half, kSingles>(p, device, s);
}

int launch_singles_join(const AttnParams &p, int dtype, cudaStream_t s)
{
    return dtype == TC_BF16 ? launch_join<__nv_bfloat16, kSingles>(p, s) : launch_join<__half, kSingles>(p, s);
}

}  // namespace tc
