"""No-GPU checks of workspace sizes: one that is made for the most tokens serves fewer, too."""
import ctypes
import os

import pytest

from paper_2601_07475_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libarcq.so not built")

P = ctypes.c_void_p
FAKE, OFF16 = P(0x10000), P(0x10010)


def sizes(size, most):
    return [size(m) for m in range(1, most + 1)]


@pytest.mark.parametrize("K,E", [(8192, 256), (4096, 64), (2048, 65), (512, 1024), (1000, 256), (65536, 16), (65536, 1), (8, 1024), (4096, 8), (16384, 300)])
def test_router(K, E):
    got = sizes(lambda m: B.arcq_moe_route_workspace_size(m, K, E), 700) + [B.arcq_moe_route_workspace_size(m, K, E) for m in (1000, 2047, 2048, 4095, 4096, 4097, 10 ** 6, 2 ** 31 - 1)]
    assert got == sorted(got)
    # and a call asks for no more than what was made for as many tokens: a workspace that is off its alignment is what it finds wrong, not one that is too small
    for m in (1, 33, 65, 700):
        need = B.arcq_moe_route_workspace_size(m, K, E)
        if need:
            call = lambda ws, bytes_: B.lib().arcq_moe_route(FAKE, m, K, K, FAKE, K, E, None, 1, 0, FAKE, FAKE, ws, bytes_, None)  # noqa: E731
            assert call(OFF16, need) == B.BAD_ALIGN and call(FAKE, need - 1) == B.WORKSPACE_TOO_SMALL


def test_router_sums_fit():
    """The sums of every run of K of as many tokens as a launch takes: (runs, tokens, experts) in 64 bits, runs as the launch has them."""
    for K, E in ((8192, 256), (4096, 64), (65536, 16), (1024, 1000)):
        for m in list(range(1, 300)) + [1000, 4096]:
            tiles = (m + 15) // 16 * ((E + 15) // 16)
            runs = max(1, min(512 // tiles, K // 512))
            if K * E > 65536 or E > 64:
                assert B.arcq_moe_route_workspace_size(m, K, E) >= runs * m * E * 8


@pytest.mark.parametrize("top,E,K,I,N", [(8, 256, 2048, 2048, 512), (2, 8, 4096, 14336, 4096), (8, 128, 4096, 1792, 4096), (4, 30, 5120, 1392, 5120), (1, 1024, 64, 8192, 1280),
                                         (1, 1024, 64, 8192, 1), (16, 1024, 256, 65536, 300), (2, 2, 256, 4096, 256), (3, 7, 96, 96, 1000), (1, 1, 32, 1024, 100000), (5, 40, 32, 3136, 1800)])
@pytest.mark.parametrize("reorder", [False, True])
def test_experts(top, E, K, I, N, reorder):
    got = sizes(lambda m: B.arcq_moe_workspace_size(m, top, E, K, I, N, reorder), 70)
    assert got == sorted(got)
    for m in range(1, 65):
        # h of every slot in 32 bits, and results of every run, as the launch has them, where they are added up by a launch of their own
        groups, runs = (N + 255) // 256 * min(E, m * top), 0
        if m > 4 or I < 128:
            runs = max(1, min(512 // groups, (I + 127) // 128 // 8, 8))
        assert got[m - 1] >= 4 * m * top * ((I + 127) // 128 * 128) + 4 * runs * m * top * N + 2 * m * K * reorder
        call = lambda ws, bytes_: B.lib().arcq_moe(FAKE, m, K, K, FAKE if reorder else None, FAKE, FAKE, top, E, FAKE, FAKE, FAKE, I, 0, FAKE, FAKE, FAKE, N, 0, 4,  # noqa: E731
                                                   None, 0, FAKE, 0, N, ws, bytes_, None)
        assert call(OFF16, got[m - 1]) == B.BAD_ALIGN and call(FAKE, got[m - 1] - 1) == B.WORKSPACE_TOO_SMALL
