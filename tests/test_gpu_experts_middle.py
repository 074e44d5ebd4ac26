"""The values between the two products of a mixture's experts: 23 bits of them arrive, whatever size they are, on every kernel of the second product."""
import numpy as np
import pytest
import torch

from oracle import arcquant as A
from oracle import layers as L
from oracle import mxfp4 as MX
from paper_2601_07475_amd import binding as B

from test_gpu_epilogue import ACT, assert_within
from test_gpu_experts import call, choices, random_experts
from test_gpu_parity import dev, say

# tokens as rows of one tile, two and four of them, with sixteen waves a workgroup and with eight; gathered, 8 and 16 rows at a time, from less than a chunk to several
# runs of the channels between
KINDS = [(1, 256, 2), (2, 1120, 2), (3, 288, 1), (4, 2080, 2), (5, 416, 2), (8, 544, 2), (8, 1312, 1), (3, 64, 1), (7, 96, 2), (5, 2080, 16), (8, 160, 9), (12, 96, 2), (20, 2080, 2), (40, 288, 2),
         (70, 1056, 1)]


def one_channel_each(fmt, M, I, top, N, seed):
    """Tokens of one channel, features of one channel between: sums without roundings.  -> the call's operands, y in 64 bits, sum of magnitudes, largest terms."""
    rng = np.random.default_rng(seed)
    K, E = 64, max(3, top)
    x = np.zeros((M, K), dtype=np.float16)
    x[np.arange(M), rng.integers(0, K, M)] = 1.0 + rng.integers(1, 1024, M) / 1024.0
    up, down = random_experts(fmt, E, 2 * I, K, 0, rng), random_experts(fmt, E, N, I, 0, rng)
    up[0][up[0] & 0x07 == 0] |= 0x02                                    # no zeros
    up[0][up[0] & 0x70 == 0] |= 0x20
    at = rng.integers(0, I, (E, N))
    at[:, :min(I, N)] = rng.permutation(I)[:min(I, N)]
    code = rng.integers(1, 8, (E, N)) | rng.integers(0, 2, (E, N)) << 3
    down[0][:] = 0
    np.put_along_axis(down[0], (at // 2)[:, :, None], (code << 4 * (at % 2)).astype(np.uint8)[:, :, None], 2)
    if fmt == "nvfp4":
        up, down = ((c, s, np.ldexp(np.float32(1.0), rng.integers(-4, 5, E)).astype(np.float32)) for c, s, _ in (up, down))
    ids, w = choices(rng, M, E, top, False)
    w += 0.25
    return x, ids, w, up, down


def sums(fmt, x, ids, w, up, down, middle=lambda h: h):
    """y in 64 bits, the magnitudes of its terms, and what a term may be off by where only the largest value near by limits it."""
    def dequantized(p, e, K):
        return (MX.dequantize(p[0][e], p[1][e]) if p[2] is None else A.dequantize(p[0][e], p[1][e], p[2][e]))[:, :K].astype(np.float64)
    M, (E, N) = x.shape[0], down[0].shape[:2]
    I = up[0].shape[1] // 2
    y, mag, floor = np.zeros((M, N)), np.zeros((M, N)), np.zeros((M, N))
    W, D = ([dequantized(p, e, k) for e in range(E)] for p, k in ((up, x.shape[1]), (down, I)))
    for m in range(M):
        for e, weight in zip(ids[m], w[m].astype(np.float64)):
            v = W[e] @ x[m].astype(np.float64)
            h = weight * v[:I] * v[I:]
            y[m] += D[e] @ middle(h)
            mag[m] += np.abs(D[e]) @ np.abs(h)
            floor[m] += np.abs(D[e]).sum(1) * 2.0 ** -38 * np.abs(h).max()
    return y, mag, floor


def bound(mag, floor, top):
    """Each term: the values' products in fp32 (two roundings; those of 11-bit inputs with 4-bit codes and their scales are exact), 2^-23 from the two numbers, a rounding each for
    their sum, its unit and the weights' scale; then one addition for each term and each run of channels, of which there are at most 16."""
    return mag * (2 * L.HALF + 2.0 ** -23 + 3 * L.HALF + (top + 16) * L.HALF) + floor


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,I,top", KINDS)
@pytest.mark.parametrize("N", [2080, 4112])
def test_every_value_arrives(fmt, M, I, top, N):
    """A feature is one value: nothing of it is hidden behind other terms' roundings."""
    say(f"moe, every value {fmt} M={M} I={I} top={top} N={N}")
    x, ids, w, up, down = one_channel_each(fmt, M, I, top, N, I + M)
    want, mag, floor = sums(fmt, x, ids, w, up, down)
    assert_within(call(fmt, dev(x), None, ids, w, up, down, activation=B.ACT_NONE, out_dtype=torch.float32), want, bound(mag, floor, top))


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,I,top", [(1, 256, 2), (8, 544, 2), (5, 2080, 16), (20, 96, 2)])
def test_a_value_of_fewer_bits_would_show(fmt, M, I, top):
    """One fp16 number for a value, and 16 bits of it, are beyond the bound in many features; 24 bits are within it.
    (The bound is 25 to 39 half steps of 2^-24, so 2^-19 of the magnitudes; n bits round by up to 2^-n, evenly.)"""
    x, ids, w, up, down = one_channel_each(fmt, M, I, top, 300, 1)

    def bits(n):
        return lambda h: np.ldexp(np.round(np.ldexp(np.frexp(h)[0], n)), np.frexp(h)[1] - n)
    want, mag, floor = sums(fmt, x, ids, w, up, down)
    off = bound(mag, floor, top)
    for n, least, most in ((11, 0.9, 1.0), (16, 0.3, 1.0), (24, 0.0, 0.0)):
        share = np.mean(np.abs(sums(fmt, x, ids, w, up, down, bits(n))[0] - want) > off)
        assert least <= share <= most, (n, share)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,I,top", KINDS)
def test_values_of_any_size(fmt, M, I, top):
    """The same layer with values between from 2^-70 to 2^90, tokens of very different sizes beside each other among them."""
    say(f"moe, values of any size {fmt} M={M} I={I} top={top}")
    rng = np.random.default_rng(I)
    K, N, E = 96, 40, max(3, top)
    x = rng.standard_normal((M, K)).astype(np.float16)
    x[1::2] *= np.float16(2.0 ** -6)
    up, down = random_experts(fmt, E, 2 * I, K, 0, rng), random_experts(fmt, E, N, I, 0, rng)
    ids, w = choices(rng, M, E, top, False)
    for power in (-35, -12, -6, 8, 12, 30, 45):
        moved = (up[0], up[1] + np.uint8(power % 256), None) if fmt == "mx" else (*up[:2], np.ldexp(up[2], power))
        for act in ("none", "relu"):
            want, off = L.experts(x, None, ids, w, moved, down, act)
            # (the bound goes by the values themselves, not by a fixed size)
            assert np.median(off / np.abs(want).max(1, keepdims=True)) < 0.1
            assert_within(call(fmt, dev(x), None, ids, w, moved, down, activation=ACT[act], out_dtype=torch.float32), want, off)


@pytest.mark.gpu
@pytest.mark.parametrize("M,I,top", [(1, 4128, 1), (2, 2080, 2), (4, 4128, 2), (8, 2080, 1), (8, 4128, 2), (5, 2080, 16), (20, 4128, 1), (64, 2080, 2)])
@pytest.mark.parametrize("way", ["up", "down", "here and there"])
def test_values_that_grow(M, I, top, way):
    """From channel to channel, by 2^50 in all: of a row, and of runs of its channels.  MXFP4 blocks whose scales fold, and some that do not."""
    say(f"moe, values that grow {way} M={M} I={I} top={top}")
    rng = np.random.default_rng(I + M)
    K, N, E = 64, 33, max(2, top)
    x = rng.standard_normal((M, K)).astype(np.float16)
    up, down = random_experts("mx", E, 2 * I, K, 0, rng), random_experts("mx", E, N, I, 0, rng)
    power = np.linspace(-25, 25, I)
    power = {"up": power, "down": power[::-1], "here and there": np.where(rng.random(I) < 0.01, 25, -25)}[way].astype(int)
    up[1][:, :I] += power.astype(np.uint8)[None, :, None]
    # weights that shrink as values grow: terms of the same size all along
    down[1][:] = (down[1].astype(int) - np.round(power.reshape(-1, 32).mean(1)).astype(int)).astype(np.uint8)
    ids, w = choices(rng, M, E, top, False)
    want, off = L.experts(x, None, ids, w, up, down, "none")
    assert_within(call("mx", dev(x), None, ids, w, up, down, activation=B.ACT_NONE, out_dtype=torch.float32), want, off)
    zero = x.copy()
    zero[::2] = 0
    want, off = L.experts(zero, None, ids, w, up, down, "relu")
    assert_within(call("mx", dev(zero), None, ids, w, up, down, activation=B.ACT_RELU, out_dtype=torch.float32), want, off)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_a_large_value_is_not_lost_nor_spreads(fmt):
    """Values past 2^20: finite where they are, and no other token's concern."""
    say("moe, one large value", fmt)
    rng = np.random.default_rng(3)
    for M, I in ((2, 256), (8, 288), (12, 64), (40, 288)):
        K, N, E = 128, 40, 2
        up, down = random_experts(fmt, E, 2 * I, K, 0, rng), random_experts(fmt, E, N, I, 0, rng)
        x = rng.standard_normal((M, K)).astype(np.float16)
        ids, w = choices(rng, M, E, 2, False)
        before = call(fmt, dev(x), None, ids, w, up, down, out_dtype=torch.float32)
        x[0] = np.float16(30000.0) * np.sign(x[0])
        want, off = L.experts(x, None, ids, w, up, down)
        y = call(fmt, dev(x), None, ids, w, up, down, out_dtype=torch.float32)
        assert_within(y, want, off)
        assert torch.equal(y[1:], before[1:])
