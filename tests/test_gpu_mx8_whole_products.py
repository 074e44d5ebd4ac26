"""MXFP8 x MXFP4: no product loses bits to a larger one beside it, whatever the output's type and the kernel that runs.

The matrix unit lines eight products of eight consecutive k up at the largest, and keeps 13 bits below its exponent.  The operands here have in every
eight k one large element of A under a weight of 0.5 and seven small ones under weights of 2, and the large ones cancel in pairs: the result is what the
small ones leave, and nothing is left of it where they were cut.
"""
import numpy as np
import pytest
import torch

from oracle import mxfp8 as M8
from paper_2601_07475_amd import binding as B

from test_gpu_mx8 import STREAM_SHAPES, TILE_SHAPES, output
from test_gpu_parity import dev, say

pytestmark = pytest.mark.gpu

HALF, TWO = 1, 4                    # E2M1 codes


def pack_nibbles(c):
    return (c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)


def test_one_sum_by_hand():
    """256 x 0.5 + 7 x (7 x 2^-9) x 2, and the same with -256: 49 / 128 is left, in fp16 too; the first half alone is 128.19140625."""
    say("mx8_gemm, one sum by hand")
    a = np.zeros((300, 32), np.uint8)
    a[:, 0], a[:, 1:8], a[:, 8], a[:, 9:16] = 0x78, 0x07, 0xF8, 0x07        # 256, 7 subnormal steps, -256
    only = a.copy()
    only[:, 8:] = 0
    w = np.zeros((300, 32), np.uint8)
    w[:, :16] = TWO
    w[:, [0, 8]] = HALF
    one = np.full((300, 1), 127, np.uint8)
    for codes, value in ((a, 49 / 128), (only, 128.19140625)):
        want, _ = M8.gemm(codes, one, pack_nibbles(w), one)
        assert np.all(want == value)
        for dtype in (torch.float16, torch.float32):
            expected = torch.tensor(value, dtype=dtype).item()              # fp32: exact, all of it are multiples of 2^-8 below 2^8
            for M in (1, 16, 40, 300):                                      # streamed, and on tiles
                y = B.arcq_mx8_gemm(dev(codes[:M]), dev(one[:M]), dev(pack_nibbles(w)), dev(one), out_dtype=dtype)
                assert bool((y == expected).all()), (M, dtype, y[0, 0].item(), expected)


def operands(M, N, K, S, seed):
    rng = np.random.default_rng(seed)
    pairs = K // 16
    rows = np.arange(pairs)[:, None] * 16
    at = rng.integers(0, 8, pairs)                                          # the large element's place in its eight
    a = rng.integers(0, 8, (M, K)).astype(np.uint8)                         # subnormals: 0 to 7 x 2^-9
    big = rng.integers(0x78, 0x7F, (M, pairs)).astype(np.uint8)             # 256 to 448
    a[:, rows[:, 0] + at], a[:, rows[:, 0] + 8 + at] = big, big | 0x80
    sign = rng.integers(0, 2, (N, pairs)).astype(np.uint8) * 8
    sign[::2] = 0                                                           # every second feature: nothing of the rest cancels either
    w = np.repeat(sign, 16, axis=1) | TWO
    w[:, rows[:, 0] + at], w[:, rows[:, 0] + 8 + at] = sign | HALF, sign | HALF
    w = np.concatenate([w, w[:, K - S:]], axis=1)
    asc = np.full((M, K // 32), 127, np.uint8)
    wsc = np.full((N, (K + S) // 32), 127, np.uint8)
    return a, asc, pack_nibbles(w), wsc


@pytest.mark.parametrize("M,N,K,S,dtype,workspace,route", TILE_SHAPES + STREAM_SHAPES[:-1])
def test_nothing_is_cut(M, N, K, S, dtype, workspace, route):
    say(f"mx8_gemm, small products beside large ones, M={M} N={N} K={K} S={S} {dtype} on {route}")
    a, asc, wc, wsc = operands(M, N, K, S, seed=M + N)
    want, mag = M8.gemm(a, asc, wc, wsc)
    need = B.arcq_mx8_gemm_workspace_size(M, N, K)
    ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
    _, y = output(M, N, dtype, 1)
    B.arcq_mx8_gemm(dev(a), dev(asc), dev(wc), dev(wsc), y=y, workspace=ws)
    got = y.double().cpu().numpy()
    # K / 32 block sums and as many additions to the accumulator lose less than a step each, 2^-23 of at most mag; joining waves and runs: 64 more
    bound = mag * (K / 16 + 64) * 2.0 ** -23
    # the tolerance tells a cut from none: where nothing cancels, less than half of the result
    assert np.all(bound[:, ::2] < 0.5 * want[:, ::2])
    if dtype is torch.float16:
        bound = bound + (np.abs(want) + bound) * 2.0 ** -11 + 2.0 ** -25
    over = np.abs(got - want) - bound
    assert over.max() <= 0, f"{over.max()} over the bound at {np.unravel_index(over.argmax(), over.shape)}"
