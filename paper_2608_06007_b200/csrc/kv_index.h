// Addresses inside one layer of a paged pool: the arithmetic that the operators' kernels do on
// indices read from device memory.  Plain host code too, so that it can be tested without a GPU.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define TC_HD __host__ __device__ __forceinline__
#else
#define TC_HD inline
#endif

namespace tc {

// Byte strides of one plane: token n of block b, head h starts at b*block + n*token + h*head.
struct PlaneGeo {
    int64_t block;
    int32_t token, head;
    TC_HD int64_t at(int64_t b, int32_t n, int32_t h) const { return b * block + static_cast<int64_t>(n) * token + static_cast<int64_t>(h) * head; }
};

// Token t of a table: its block's entry and its place in the block (t / B is a 32-bit division:
// lengths are int32).
TC_HD void token_place(uint32_t t, uint32_t B, uint32_t *entry, uint32_t *n)
{
    *entry = t / B;
    *n = t - *entry * B;
}

// slot = block * B + n; false where it is outside the pool.
TC_HD bool slot_place(int64_t slot, uint32_t B, int64_t num_blocks, int64_t *block, int32_t *n)
{
    if (slot < 0) return false;
    *block = (slot >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(slot) / B) : slot / static_cast<int64_t>(B);
    *n = static_cast<int32_t>(slot - *block * B);
    return *block < num_blocks;
}

// The request that row `row` belongs to: the last r with offsets[r] <= row, by bisection over
// [0, R); -1 where row >= offsets[R] or row < offsets[0].  Ends after log2(R) steps and stays inside
// offsets[0..R] whatever the numbers are.
TC_HD int64_t request_of(const int64_t *offsets, int64_t R, int64_t row)
{
    if (R <= 0 || row < offsets[0] || row >= offsets[R]) return -1;
    int64_t lo = 0, hi = R;
    while (hi - lo > 1) {
        const int64_t mid = lo + (hi - lo) / 2;
        if (offsets[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace tc
