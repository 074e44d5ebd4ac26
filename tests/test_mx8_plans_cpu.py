"""Every plan of the MXFP8 x MXFP4 product has a kernel: without a GPU a call ends at its first HIP call, one without a kernel does before."""
import os
import random

import pytest
import torch

from paper_2601_07475_amd import binding as B

pytestmark = [pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libarcq.so not built"),
              pytest.mark.skipif(torch.cuda.device_count() > 0, reason="the calls' operands are no memory: only where nothing can be launched")]

FAKE = 0x10000
# prompts into down projections (rows, features, channels), whole and over several ranks, whose tiles leave compute units idle
PROMPTS = [(M, N, K) for N, K in ((5120, 27648), (5120, 25600), (5120, 20480), (7168, 18432), (4096, 28672), (2048, 28672), (1024, 28672),
                                  (16384, 53248), (3584, 18944), (6144, 28672), (8192, 28672), (4096, 14336))
           for M in (1, 16, 33, 100, 200, 256, 385, 512, 600, 640, 768, 1000, 1024, 1200, 1280, 1500, 1700, 2048, 2500, 3000, 3400, 4097, 5376, 6909, 8192)]


def drawn(n):
    rng = random.Random(4)
    for _ in range(n):
        M, N, K = (int(2.0 ** rng.uniform(lo, hi)) for lo, hi in ((0, 14), (0, 16), (5, 16)))
        yield M, N, max(32, K // 32 * 32)


def call(M, N, K, S, dtype, workspace):
    """(status, message)"""
    need = B.arcq_mx8_gemm_workspace_size(M, N, K)
    dt = B.DTYPE_F16 if dtype is torch.float16 else B.DTYPE_F32
    status = B.lib().arcq_mx8_gemm(FAKE, FAKE, FAKE, FAKE, M, N, K, S, FAKE, dt, N, FAKE if workspace else None, need if workspace else 0, None)
    return status, B.lib().arcq_last_error().decode()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("workspace", [False, True])
def test_every_plan_has_a_kernel(dtype, workspace):
    sizes = [*PROMPTS, *drawn(3000)]
    seen = set()
    for i, (M, N, K) in enumerate(sizes):
        S = min(K, 256) if i % 3 == 0 else 0
        status, message = call(M, N, K, S, dtype, workspace)
        route = B.arcq_mx8_gemm_route(M, N, K, S, dtype, workspace)
        assert status == B.HIP_ERROR and "device" in message, (M, N, K, S, route, message)
        seen.add(route[:3])
        assert workspace or route[3] == 1
        assert route[3] * M * N * 4 <= 64 << 20 or route[3] == 1            # what the header promises of a workspace
        assert B.arcq_mx8_gemm_workspace_size(M, N, K) <= 64 << 20
    tiles = {(B.ROUTE_TILES, 64 * m, 64 * n) for m, n in ((1, 2), (1, 4), (2, 2), (3, 2), (2, 4), (3, 4))}
    assert tiles <= seen and any(r[0] == B.ROUTE_STREAM for r in seen)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_smallest_products_stream(dtype):
    """A launch is all that they take: the kernel with the least to set up."""
    for M, N, K in ((1, 8, 32), (1, 512, 128), (1, 4096, 64), (16, 64, 64), (32, 512, 128), (64, 64, 64), (128, 512, 128)):
        assert B.arcq_mx8_gemm_route(M, N, K, 0, dtype, True)[0] == B.ROUTE_STREAM


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("workspace", [False, True])
def test_route_of_nothing(dtype, workspace):
    """No rows, no features: the answer for one, as of the other products' routes; once a division by zero."""
    for M, N in ((0, 8), (4, 0), (0, 0)):
        assert B.arcq_mx8_gemm_route(M, N, 64, 0, dtype, workspace) == (B.ROUTE_STREAM, 16, 16, 1)
