// tc_attn_chunk over pools of codes.
#include "attn_chunk.cuh"

namespace tc {

int launch_chunk_codes(const ChunkParams &p, int device, cudaStream_t s)
{
    return p.layer.dtype == TC_E4M3 ? launch_chunk_type<__half, kE4m3>(p, device, s) : launch_chunk_type<__half, kInt8>(p, device, s);
}

}  // namespace tc
