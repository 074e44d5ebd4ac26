"""fp16 rows times MXFP4 weights: every scale byte from 2^-127 to 2^127, in tails of a chunk and in whole ones."""
import numpy as np
import pytest
import torch

from oracle import mxfp4 as MX
from oracle import mxfp8 as M8
from paper_2601_07475_amd import binding as B

from test_gpu_parity import dev, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("reorder", [False, True])
@pytest.mark.parametrize("M,K", [(4, 64), (3, 128), (4, 160), (12, 640), (29, 672)])
def test_every_scale_byte(M, K, reorder):
    say(f"mx_gemv, bytes 0 to 254, M={M} K={K} reorder={reorder}")
    rng = np.random.default_rng(K)
    N = 255
    codes = rng.integers(0, 256, (N, K // 2)).astype(np.uint8)
    scales = ((np.arange(N)[:, None] + 7 * np.arange(K // 32)) % 255).astype(np.uint8)
    assert {0, 254} <= set(scales[:, 0]) and np.array_equal(MX.e8m0_decode(np.array([0, 254], np.uint8)), [2.0 ** -127, 2.0 ** 127])
    X = np.zeros((M, K), np.float16)
    X[np.arange(M), rng.integers(0, K, M)] = np.resize(np.float16([1, 2.0 ** -24, -3, 32768]), M)
    perm = rng.permutation(K).astype(np.int32) if reorder else None
    # a row has one channel, so a result is one product rounded once: a subnormal at one end, infinite at the other
    want, _ = M8.gemv(X, perm, codes, scales)
    with np.errstate(over="ignore"):
        want = want.astype(np.float32)
    assert np.isinf(want).any() and np.any((want != 0) & (np.abs(want) < 2.0 ** -126))
    got = B.arcq_mx_gemv(dev(X), None if perm is None else dev(perm), dev(codes), dev(scales), out_dtype=torch.float32).cpu().numpy()
    assert np.array_equal(got, want)
