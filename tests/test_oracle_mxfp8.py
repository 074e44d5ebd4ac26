"""Pins of the MXFP8 oracle: against the library's float8 type, exact fractions, and the format's defining inequalities."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import arcquant as A
from oracle import brute
from oracle import mxfp4 as MX
from oracle import mxfp8 as M8


def test_element_rounding_is_the_float8_types_on_every_fp16():
    x = np.arange(65536, dtype=np.uint32).astype(np.uint16).view(np.float16)
    x = x[np.isfinite(x)].astype(np.float64)
    want = torch.from_numpy(np.clip(x, -448, 448)).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(M8.e4m3_byte(M8.e4m3_nearest(x)), want)


def block_by_fractions(v, up):
    """(scale byte, codes) of a block in exact rationals, the code by looking through all 127 magnitudes."""
    amax = max(abs(Fraction(float(t))) for t in v)
    e = 0
    if amax:
        e = -200
        while Fraction(2) ** (e + 1) <= amax:
            e += 1
        e -= 8
        if up and amax > 448 * Fraction(2) ** e:
            e += 1
    grid = [Fraction(brute.e4m3_value(b)) for b in range(0x7F)]
    codes = []
    for t in v:
        w = abs(Fraction(float(t))) / Fraction(2) ** e
        best = min(range(0x7F), key=lambda b: (abs(grid[b] - w), b & 1))
        codes.append(best | (0x80 if np.signbit(t) else 0))
    return e + 127, codes


@pytest.mark.parametrize("up", [False, True])
def test_blocks_against_exact_rationals(up):
    rng = np.random.default_rng(5)
    blocks = [rng.standard_normal(32) * 10.0 ** rng.uniform(-6, 4) for _ in range(12)]
    blocks += [np.zeros(32), np.full(32, -0.0), np.full(32, 2.0 ** -24), np.full(32, 65504.0)]
    blocks += [np.r_[m * 2.0 ** 3, rng.standard_normal(31)] for m in (1.0, 1.75, 1.75 + 2.0 ** -10, 1.8125, 1.9375, 2 - 2.0 ** -10)]
    v = np.array(blocks).astype(np.float16)
    sb, codes = M8.quantize_blocks(v, "up" if up else "nearest")
    for i in range(len(v)):
        e, c = block_by_fractions(v[i], up)
        assert sb[i] == e and codes[i].tolist() == c, i


def test_scale_inequalities_and_error():
    rng = np.random.default_rng(6)
    v = (rng.standard_normal((500, 32)) * 10.0 ** rng.uniform(-3, 3, (500, 1))).astype(np.float16).astype(np.float64)
    for mode in ("nearest", "up"):
        sb, codes = M8.quantize_blocks(v, mode)
        X, amax = MX.e8m0_decode(sb), np.abs(v).max(-1)
        assert np.all(amax < 512 * X) and np.all(256 * X <= amax) if mode == "nearest" else np.all(amax <= 448 * X) and np.all(224 * X < amax)
        err = np.abs(M8.dequantize(codes, sb.reshape(-1, 1)) - v)
        clipped = np.abs(v) > 448 * X[:, None]
        half_step = np.maximum(np.abs(v) * 2.0 ** -4, X[:, None] * 2.0 ** -10)
        assert np.all(err[~clipped] <= half_step[~clipped])
        assert mode == "nearest" or not clipped.any()


def test_reorder_norm_and_products_as_identities():
    rng = np.random.default_rng(7)
    M, K, N, S = 5, 96, 7, 32
    X = (rng.standard_normal((M, K)) * 3).astype(np.float16)
    R = rng.standard_normal((M, K)).astype(np.float16)
    gamma = (1 + 0.1 * rng.standard_normal(K)).astype(np.float16)
    perm = rng.permutation(K)
    c, s = M8.quantize_act(X, perm)
    c2, s2 = M8.quantize_act(X[:, perm])
    assert np.array_equal(c, c2) and np.array_equal(s, s2)
    c, s, h = M8.add_rmsnorm_quantize_act(X, R, gamma, 1e-5, perm)
    assert np.array_equal(h, X + R)                                         # numpy adds fp16 with one rounding
    c2, s2 = M8.quantize_act(A.rmsnorm(h, gamma, 1e-5), perm)
    assert np.array_equal(c, c2) and np.array_equal(s, s2)
    W = (rng.standard_normal((N, K)) * 0.02).astype(np.float16)
    wc, ws = MX.pack_weight(W, perm, S)
    wc0, ws0 = MX.pack_weight(W, perm, 0)
    y, mag = M8.gemm(c, s, wc, ws)
    assert np.array_equal(y, M8.gemm(c, s, wc0, ws0)[0]) and np.all(np.abs(y) <= mag)
    # the S columns change nothing for fp16 rows either, and with weights on the grid the product is the plain one
    assert np.array_equal(M8.gemv(X, perm, wc, ws)[0], M8.gemv(X, perm, wc0, ws0)[0])
    packed = rng.choice([0, 0.5, 1, 1.5, 2, 3, 4, 6], (N, K)) * rng.choice([-1, 1], (N, K))
    packed[:, ::8] = 6                                                      # a 6 in every block: its scale is 1
    grid = np.empty_like(packed)
    grid[:, perm] = packed
    gc, gs = MX.pack_weight(grid.astype(np.float16), perm, S)
    assert np.array_equal(M8.gemv(X, perm, gc, gs)[0], X.astype(np.float64) @ grid.T)
    nc, ns = A.pack_weight(grid.astype(np.float16), perm, S, np.float32(1.0))
    assert np.array_equal(M8.gemv(X, perm, nc, ns, np.float32(1.0))[0], X.astype(np.float64) @ grid.T)


def test_aligned_loss_by_hand():
    """One group: exponents of 448 (8) and 6 (2) on top, 2^(10 - 13) for each of seven others, times the blocks' scales."""
    ac, asc = np.zeros((1, 32), np.uint8), np.array([[128]], np.uint8)
    ac[0, 0], ac[0, 1] = 0x7E, 0x01                                         # 448, 2^-9
    wc, wsc = np.zeros((2, 16), np.uint8), np.array([[127], [126]], np.uint8)
    wc[:, 0] = 0x17                                                         # 6, 0.5
    assert np.array_equal(M8.aligned_loss(ac, asc, wc, wsc), [[7 * 2.0 ** -3 * 2, 7 * 2.0 ** -3]])
    ac[0, 0] = 0                                                            # what is left: the subnormal, exponents -6 and 0
    assert np.array_equal(M8.aligned_loss(ac, asc, wc, wsc), [[7 * 2.0 ** -19 * 2, 7 * 2.0 ** -19]])
    assert not M8.aligned_loss(np.zeros_like(ac), asc, wc, wsc).any()
