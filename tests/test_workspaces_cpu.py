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
