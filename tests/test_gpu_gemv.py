"""GPU parity of the products of fp16 rows with packed 4-bit weights against the oracle, within a bound derived from their roundings."""
import numpy as np
import pytest
import torch

from oracle import arcquant as A
from oracle import mxfp4 as MX
from oracle import mxfp8 as M8
from paper_2601_07475_amd import binding as B
from paper_2601_07475_amd import workloads as wk

from test_gpu_mx8 import assert_product, output, strided
from test_gpu_parity import dev, say

pytestmark = pytest.mark.gpu


def pack(fmt, W, perm, S):
    """(codes, scales, tensor scale or None)"""
    if fmt == "mx":
        return (*MX.pack_weight(W, perm, S), None)
    ts = wk.tensor_scale(W)
    return (*A.pack_weight(W, perm, S, ts), ts)


def call(fmt, x, perm, w, **kw):
    wc, wsc, ts = w
    wc, wsc = (dev(t) if isinstance(t, np.ndarray) else t for t in (wc, wsc))
    return B.arcq_mx_gemv(x, perm, wc, wsc, **kw) if fmt == "mx" else B.arcq_gemv(x, perm, wc, wsc, float(ts), **kw)


# M, N, K, S: one of everything, tails of features and of chunks (half a piece of 32 codes for NVFP4), every tile of rows, more rows than one
# pass takes, one to four weight tiles a wave, whole groups only and none, S = 0 and S = K
SHAPES = [(1, 1, 32, 0), (1, 17, 64, 32), (2, 16, 96, 96), (3, 100, 128, 0), (1, 4096, 512, 64), (5, 333, 544, 32), (16, 250, 1056, 0), (17, 64, 2592, 64),
          (32, 4101, 640, 0), (33, 70, 1120, 96), (64, 4100, 256, 0), (65, 40, 608, 32), (130, 33, 4128, 0), (1, 8200, 1024, 0), (7, 9000, 736, 224),
          (1, 64, 14336, 256), (16, 48, 28672, 1024), (1, 20, 65536, 0), (4, 12300, 160, 0), (20, 8300, 512, 0)]


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,N,K,S", SHAPES)
@pytest.mark.parametrize("reorder", [False, True])
def test_products(fmt, M, N, K, S, reorder):
    if fmt == "nvfp4":
        K -= 16 * ((M + N) % 2) if K > 32 and S < K else 0              # K a multiple of 16 only
    dtype = torch.float16 if (M + N + reorder) % 2 else torch.float32
    say(f"gemv {fmt} M={M} N={N} K={K} S={S} reorder={reorder} {dtype}")
    rng = np.random.default_rng(M * K + N)
    X = wk.activations(wk.Workload("t", M, K, N, S, max(1, K // 100), "loguniform20_100", 0.02, 4))
    W = (rng.standard_normal((N, K)) * 0.02).astype(np.float16)
    perm = rng.permutation(K).astype(np.int32) if reorder else None
    w = pack(fmt, W, np.arange(K) if perm is None else perm, S)
    want, mag = M8.gemv(X, perm, *w)
    raw, y = output(M, N, dtype, N % 4)
    x = strided(X, 8 * (M % 3))
    call(fmt, x, dev(perm) if reorder else None, w, y=y)
    torch.cuda.synchronize()
    assert_product(y, want, mag, K)
    y.fill_(12345.0)
    assert bool((raw == 12345.0).all())


# Workgroups that take one tile of weight rows after the other, over rounds of K that end in a part of one: the next tile's weights and rows are
# asked for while the last, shorter turn of this one is multiplied.
@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,N,K", [(1, 8400, 4736), (1, 16700, 4192), (3, 8300, 4256), (6, 16600, 4352), (16, 33000, 4704), (20, 16500, 4896), (32, 8200, 9216),
                                   (9, 4100, 4064), (9, 4096, 4096), (16, 100, 8224), (5, 2000, 10272),
                                   (2, 1001, 20512), (14, 4400, 14336), (32, 850, 9312), (40, 130, 16416), (23, 8482, 4128)])
def test_tile_after_tile(fmt, M, N, K):
    say(f"gemv {fmt} M={M} N={N} K={K}")
    block = 32 if fmt == "mx" else 16
    rng = np.random.default_rng(M + N + K)
    x = rng.standard_normal((M, K)).astype(np.float16)
    codes = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    scales = rng.integers(118, 124, (N, K // block), dtype=np.uint8) if fmt == "mx" else rng.integers(40, 60, (N, K // block), dtype=np.uint8)
    w = (codes, scales, None if fmt == "mx" else np.float32(0.125))
    want, mag = M8.gemv(x, None, *w)
    raw, y = output(M, N, torch.float32, 3)
    call(fmt, dev(x), None, w, y=y)
    torch.cuda.synchronize()
    assert_product(y, want, mag, K)


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_scales_over_their_whole_range(fmt):
    """Weights whose blocks differ by many powers of two, and rows with subnormals: sums are of either end of the range."""
    say(f"gemv {fmt}, scales over the whole range")
    M, N, K = 6, 50, 1184
    rng = np.random.default_rng(3)
    X = (rng.standard_normal((M, K)) * 2.0 ** rng.integers(-20, 12, (M, K))).astype(np.float16)
    X[1] = (rng.standard_normal(K) * 2.0 ** -22).astype(np.float16)     # subnormals only
    W = (rng.standard_normal((N, K // 16, 16)) * 2.0 ** rng.integers(-22, 13, (N, K // 16, 1))).reshape(N, K).astype(np.float16)
    W[3] = 0
    W[4, :16] = 65504
    w = pack(fmt, W, np.arange(K), 0)
    want, mag = M8.gemv(X, None, *w)
    got = call(fmt, dev(X), None, w, out_dtype=torch.float32).double().cpu().numpy()
    assert np.all(np.abs(got - want) <= mag * (K / 16 + 64) * 2.0 ** -23 + 2.0 ** -149)
    assert np.all(got[:, 3] == 0)


def test_every_scale_byte():
    """All 255 exponents of MXFP4 and all 127 scales of NVFP4, one weight row each, against one channel at a time."""
    say("gemv, every scale byte")
    for fmt, bytes_ in (("mx", np.arange(40, 215)), ("nvfp4", np.arange(0, 0x7F))):
        N, block = len(bytes_), 32 if fmt == "mx" else 16
        K = 2 * block
        codes = np.random.default_rng(1).integers(0, 256, (N, K // 2)).astype(np.uint8)
        scales = np.stack([bytes_, np.roll(bytes_, 1)], 1).astype(np.uint8)
        X = np.zeros((4, K), dtype=np.float16)
        X[0, 0], X[1, 5], X[2, K - 1], X[3, block] = 1, 3, -0.5, 2.0 ** -24
        w = (codes, scales, None if fmt == "mx" else np.float32(1.0))
        want, _ = M8.gemv(X, None, *w)
        got = call(fmt, dev(X), None, w, out_dtype=torch.float32).double().cpu().numpy()
        assert np.array_equal(got, want), fmt                           # single products: exact


def test_unaligned_weights_and_scales():
    """Codes at 8-byte addresses, scale bytes at odd ones."""
    say("gemv, operands at the least alignment")
    M, N, K, S = 3, 70, 1184, 32
    rng = np.random.default_rng(6)
    X = rng.standard_normal((M, K)).astype(np.float16)
    W = (rng.standard_normal((N, K)) * 0.02).astype(np.float16)
    for fmt in ("nvfp4", "mx"):
        w = pack(fmt, W, np.arange(K), S)
        want, mag = M8.gemv(X, None, *w)
        buf = torch.zeros(w[0].size + 64, dtype=torch.uint8, device="cuda")
        sbuf = torch.zeros(w[1].size + 64, dtype=torch.uint8, device="cuda")
        for off, soff in ((8, 1), (24, 3)):
            wc, wsc = buf[off:off + w[0].size].view(w[0].shape), sbuf[soff:soff + w[1].size].view(w[1].shape)
            wc.copy_(dev(w[0]))
            wsc.copy_(dev(w[1]))
            assert_product(call(fmt, dev(X), None, (wc, wsc, w[2]), out_dtype=torch.float32), want, mag, K)


def test_no_rows_and_no_features():
    x = torch.empty((0, 64), dtype=torch.float16, device="cuda")
    w, s = torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros((8, 2), dtype=torch.uint8, device="cuda")
    assert B.arcq_mx_gemv(x, None, w, s).shape == (0, 8)
    one = torch.ones((1, 64), dtype=torch.float16, device="cuda")
    assert B.arcq_mx_gemv(one, None, w[:0], s[:0]).shape == (1, 0)
    assert B.arcq_gemv(one, None, w[:0], torch.zeros((0, 4), dtype=torch.uint8, device="cuda"), 1.0).shape == (1, 0)


def test_more_rows_than_a_launch_takes():
    """70000 rows go in two runs, which share the workspace for the reordered rows."""
    say("gemv, 70000 rows")
    M, N, K = 70000, 20, 64
    rng = np.random.default_rng(8)
    X = rng.standard_normal((M, K)).astype(np.float16)
    perm = rng.permutation(K).astype(np.int32)
    w = pack("mx", (rng.standard_normal((N, K)) * 0.02).astype(np.float16), perm, 0)
    assert B.arcq_mx_gemv_workspace_size(M, N, K, True) == 65536 * K * 2
    want, mag = M8.gemv(X, perm, *w)
    assert_product(call("mx", dev(X), dev(perm), w, out_dtype=torch.float32), want, mag, K)


def test_operands_in_host_memory():
    """Refused before the library sees their addresses."""
    x, w, s = torch.zeros((2, 64), dtype=torch.float16), torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 2), dtype=torch.uint8)
    xd, wd, sd, codes, scales = x.cuda(), w.cuda(), s.cuda(), torch.zeros((2, 64), dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8)
    y, perm = torch.zeros((2, 8), dtype=torch.float16), torch.arange(64, dtype=torch.int32)
    for args in ((x, None, wd, sd), (xd, perm, wd, sd), (xd, None, w, sd), (xd, None, wd, s)):
        with pytest.raises(AssertionError):
            B.arcq_mx_gemv(*args)
    with pytest.raises(AssertionError):
        B.arcq_mx_gemv(xd, None, wd, sd, y=y)
    with pytest.raises(AssertionError):
        B.arcq_mx_gemv(xd, perm.cuda(), wd, sd, workspace=torch.zeros(4096, dtype=torch.uint8))
    for kw in ({"codes": codes}, {"scales": scales}, {"perm": perm}):
        with pytest.raises(AssertionError):
            B.arcq_mx8_quantize_act(xd, **kw)
        with pytest.raises(AssertionError):
            B.arcq_mx8_add_rmsnorm_quantize_act(xd, None, xd[0], 1e-5, **kw)
    for residual, gamma, hidden in ((x, xd[0], None), (xd, x[0], None), (xd, xd[0], x)):
        with pytest.raises(AssertionError):
            B.arcq_mx8_add_rmsnorm_quantize_act(xd, residual, gamma, 1e-5, hidden=hidden)
    for args in ((codes, scales.cuda(), wd, sd), (codes.cuda(), scales, wd, sd), (codes.cuda(), scales.cuda(), w, sd)):
        with pytest.raises(AssertionError):
            B.arcq_mx8_gemm(*args)
