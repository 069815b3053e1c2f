"""What tc_attn_chunk's kernels do when a wait has run out, by a kernel of its own: copies in flight land before they are left."""
import ctypes
import os
import subprocess
import time

import pytest
import torch

from paper_2608_06007_b200 import build

pytestmark = pytest.mark.gpu

LANDING = """
#include "attn_chunk.cuh"
namespace tc {
constexpr int kStages = 4, kBytes = 16384, kBarsAt = 6 * kBytes;
__global__ void landing(const unsigned char *src, unsigned char *dst, int *got)
{
    extern __shared__ unsigned char raw[];
    const uint32_t base = (static_cast<uint32_t>(__cvta_generic_to_shared(raw)) + 1023) & ~1023u, full = base + kBarsAt, q_full = full + 16 * kStages + 64, landed = q_full + 80;
    const unsigned char *gen = raw + (base - static_cast<uint32_t>(__cvta_generic_to_shared(raw)));
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2 * kStages + 20; i++) barrier_init(full + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        // two announced; one whose barrier somebody else has yet to arrive at; the queries', and half a look at V's
        const uint32_t bars[6] = {full, full + 8, full + 16, q_full, landed, landed + 8};
        for (int i = 0; i < 6; i++) {
            if (i == 2) asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bars[i]), "r"(kBytes) : "memory");
            else asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bars[i]), "r"(kBytes) : "memory");
            copy_run(base + i * kBytes, src + i * kBytes, kBytes, bars[i]);
        }
    }
    __syncthreads();
    copies_landed<kStages>(kBarsAt);
    __syncthreads();
    for (int i = threadIdx.x; i < 6 * kBytes; i += blockDim.x) dst[i] = gen[i];
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; i++) got[i] = barrier_passed(full + 8 * i, 0), got[2 + i] = barrier_passed(landed + 8 * i, 0);
        got[4] = barrier_passed(q_full, 0), got[5] = barrier_passed(full + 24, 0);
        got[6] = barrier_wait(full + 24, 0, 16), got[7] = barrier_wait<true>(full + 24, 0, 16);  // a few turns, then given up
    }
}
}
extern "C" __attribute__((visibility("default"))) int run(const unsigned char *src, unsigned char *dst, int *got)
{
    const int bytes = tc::kBarsAt + 1024 + 512;
    if (cudaFuncSetAttribute(tc::landing, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)) return 1;
    tc::landing<<<1, 128, bytes>>>(src, dst, got);
    return static_cast<int>(cudaDeviceSynchronize());
}
"""


def test_copies_in_flight_land_before_a_kernel_that_gives_up_ends(tmp_path):
    src, lib = tmp_path / "landing.cu", tmp_path / "landing.so"
    src.write_text(LANDING)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), *build.NVCC_FLAGS, "-I", build.CSRC, "-I", build.INCLUDE, "-shared", "-cudart", "static", "-o", str(lib), str(src)])
    bytes_ = torch.randint(0, 256, (6 * 16384,), dtype=torch.uint8, device="cuda")
    copied, got = torch.zeros_like(bytes_), torch.full((8,), 7, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    begin = time.monotonic()
    assert ctypes.CDLL(str(lib)).run(*(ctypes.c_void_p(t.data_ptr()) for t in (bytes_, copied, got))) == 0
    assert 0.2 < time.monotonic() - begin < 20  # barriers that have no copy run out, all at once
    assert torch.equal(copied, bytes_)
    assert got.tolist() == [1, 1, 1, 1, 1, 0, 0, 0]
