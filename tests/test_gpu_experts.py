"""GPU parity of a mixture of experts (router, experts) against the oracle: choices exactly, values within bounds derived from their roundings."""
import numpy as np
import pytest
import torch

from oracle import arcquant as A
from oracle import layers as L
from oracle import mxfp4 as MX
from paper_2601_07475_amd import binding as B

from test_gpu_epilogue import ACT, assert_within
from test_gpu_mx8 import output, strided
from test_gpu_parity import dev, say

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------------------ router

def check_route(x, r, top, bias, flags, extra=0):
    want_ids, want_w = L.route(x, r, top, bias, bool(flags & B.MOE_SIGMOID), bool(flags & B.MOE_RENORMALIZE))
    M, E = x.shape[0], r.shape[0]
    raw_i = torch.full((M * top + 64,), -77, dtype=torch.int32, device="cuda")
    raw_w = torch.full((M * top + 64,), 12345.0, device="cuda")
    ids, w = raw_i[32:32 + M * top].view(M, top), raw_w[32:32 + M * top].view(M, top)
    need = B.arcq_moe_route_workspace_size(M, x.shape[1], E)
    ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    B.arcq_moe_route(strided(x, 8 * extra), strided(r, 8 * (extra % 2)), top, None if bias is None else dev(bias), flags, ids, w, ws)
    torch.cuda.synchronize()
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    # a score in fp32 or more: the exponential's argument and value, the sum, the quotients: fewer than 16 half steps
    assert np.all(np.abs(w.double().cpu().numpy() - want_w) <= want_w * 16 * L.HALF + 2.0 ** -126)
    ids.fill_(-77)
    w.fill_(12345.0)
    assert bool((raw_i == -77).all()) and bool((raw_w == 12345.0).all())


@pytest.mark.parametrize("M,K,E,top", [(1, 8, 1, 1), (1, 4096, 8, 2), (2, 264, 5, 5), (3, 1000, 64, 8), (4, 72, 1024, 16), (5, 2048, 65, 1), (17, 520, 100, 10), (64, 4096, 256, 8),
                                       (100, 1032, 31, 4), (300, 256, 16, 16), (33, 8192, 129, 6), (1, 65536, 3, 2), (1, 8192, 512, 8), (7, 128, 17, 3), (2000, 64, 8, 2)])
def test_router(M, K, E, top):
    rng = np.random.default_rng(M + K + E)
    x = rng.standard_normal((M, K)).astype(np.float16)
    r = (rng.standard_normal((E, K)) / np.sqrt(K)).astype(np.float16)
    bias = (0.2 * rng.standard_normal(E)).astype(np.float32)
    for flags in range(4):
        for b in (None, bias):
            say(f"router M={M} K={K} E={E} top={top} flags={flags} bias={b is not None}")
            check_route(x, r, top, b, flags, extra=flags)


@pytest.mark.parametrize("M,K,E,top", [(5000, 32, 8, 2), (4099, 64, 70, 3)])
def test_router_of_many_tokens(M, K, E, top):
    say(f"router M={M} K={K} E={E}")
    rng = np.random.default_rng(M)
    check_route(rng.standard_normal((M, K)).astype(np.float16), rng.standard_normal((E, K)).astype(np.float16), top, None, B.MOE_RENORMALIZE)


def test_router_ties():
    """Sums that are equal exactly: the lower index first, among many and among all."""
    say("router, ties")
    rng = np.random.default_rng(3)
    for M, E in ((1, 130), (6, 130), (40, 1000)):
        x = rng.integers(-2, 3, (M, 64)).astype(np.float16)
        r = rng.integers(-1, 2, (E, 64)).astype(np.float16)
        r[E // 2:] = r[:E - E // 2]
        for flags in (0, B.MOE_RENORMALIZE):
            check_route(x, r, 16, None, flags)
        check_route(x, np.zeros_like(r), 7, None, 0)
        check_route(x, np.zeros_like(r), 7, np.linspace(0, 1, E).astype(np.float32), B.MOE_SIGMOID)


def test_router_near_ties():
    """Scores that differ in the 40th bit: fp32 sums could not tell them apart."""
    say("router, near ties")
    for M in (1, 20):
        x = np.zeros((M, 512), dtype=np.float16)
        x[:, 0], x[:, 1:3] = 60000, 2.0 ** -10
        r = np.zeros((40, 512), dtype=np.float16)
        r[:, 0] = 1.0
        r[:, 1] = 2.0 ** -10 * np.random.default_rng(1).permutation(40)
        r[:, 500:] = 1.0                                                # (of channels that are zero)
        check_route(x, r, 16, None, B.MOE_RENORMALIZE)


def test_router_extremes():
    """Far scores, and some that overflow an exponential on the way."""
    say("router, far scores")
    rng = np.random.default_rng(5)
    for M in (2, 30):
        x, r = (300 * rng.standard_normal((M, 256))).astype(np.float16), (30 * rng.standard_normal((90, 256))).astype(np.float16)
        for flags in range(4):
            want_ids, want_w = L.route(x, r, 1, None, bool(flags & B.MOE_SIGMOID), bool(flags & B.MOE_RENORMALIZE))
            ids, w = B.arcq_moe_route(dev(x), dev(r), 1, flags=flags)
            assert np.array_equal(ids.cpu().numpy(), want_ids)
            assert np.allclose(w.cpu().numpy(), want_w, rtol=16 * L.HALF, atol=2.0 ** -126)


def test_router_of_what_is_not_finite():
    """Experts at most once each, within range, and no other row touched."""
    say("router, inf and nan")
    for M in (3, 40):
        x = torch.randn((M, 64), device="cuda").half()
        r = torch.randn((70, 64), device="cuda").half()
        want, _ = B.arcq_moe_route(x, r, 8)
        x[1, 3], x[2, 5] = float("nan"), float("inf")
        for bias in (None, torch.zeros(70, device="cuda")):
            for flags in range(4):
                ids, _ = B.arcq_moe_route(x, r, 8, bias=bias, flags=flags)
                rows = ids.cpu().numpy()
                for row in rows:
                    live = row[row >= 0]
                    assert len(set(live)) == len(live) and (live < 70).all()
                assert np.array_equal(rows[0], want[0].cpu().numpy()) and np.array_equal(rows[3:], want[3:].cpu().numpy())


# ----------------------------------------------------------------------------------------------------------------- experts

def random_experts(fmt, E, rows, K, S, rng):
    """Packed weights of random codes, scales near one over the root of K, and their repeated columns (noise: they have to be passed over)."""
    block = 32 if fmt == "mx" else 16
    codes = rng.integers(0, 256, (E, rows, (K + S) // 2), dtype=np.uint8)
    if fmt == "mx":
        at = 127 - int(round(np.log2(3 * np.sqrt(K))))
        return codes, rng.integers(at - 1, at + 2, (E, rows, (K + S) // block), dtype=np.uint8), None
    return codes, rng.integers(40, 64, (E, rows, (K + S) // block), dtype=np.uint8), ((rng.random(E) + 0.5) / (3 * np.sqrt(K))).astype(np.float32)


def call(fmt, x, perm, ids, w, up, down, **kw):
    up, down = (tuple(None if t is None else dev(t) if isinstance(t, np.ndarray) else t for t in p) for p in (up, down))
    ids, w = (dev(t) if isinstance(t, np.ndarray) else t for t in (ids, w))
    if fmt == "mx":
        return B.arcq_mx_moe(x, perm, ids, w, *up[:2], *down[:2], **kw)
    return B.arcq_moe(x, perm, ids, w, *up, *down, **kw)


def choices(rng, M, E, top, drop):
    ids = np.stack([rng.permutation(E)[:top] for _ in range(M)]).astype(np.int32)
    if drop:
        ids[rng.random((M, top)) < 0.3] = -1
        ids[rng.random(M) < 0.2] = -1
    return ids, rng.random((M, top)).astype(np.float32)


def check(fmt, M, K, I, N, E, top, S=0, S2=0, act="silu", residual=False, reorder=False, drop=False, dtype=torch.float16, in_place=False, seed=0, ids=None, w=None):
    say(f"moe {fmt} M={M} K={K} I={I} N={N} E={E} top={top} S={S} S2={S2} {act} residual={residual} reorder={reorder} drop={drop} {dtype}")
    rng = np.random.default_rng(seed + M + K + I)
    x = rng.standard_normal((M, K)).astype(np.float16)
    perm = rng.permutation(K).astype(np.int32) if reorder else None
    up, down = random_experts(fmt, E, 2 * I, K, S, rng), random_experts(fmt, E, N, I, S2, rng)
    if ids is None:
        ids, w = choices(rng, M, E, top, drop)
    r = rng.standard_normal((M, N)).astype(np.float16 if dtype is torch.float16 else np.float32) if residual else None
    want, off = L.experts(x, perm, ids, w, up, down, act, r)
    raw, y = output(M, N, dtype, N % 3)
    res = None
    if residual:
        res = y if in_place else output(M, N, dtype, 1)[1]
        res.copy_(dev(r))
    need = B.arcq_moe_workspace_size(M, ids.shape[1], E, K, I, N, reorder)
    buf = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    call(fmt, strided(x, 8 * (M % 3)), None if perm is None else dev(perm), ids, w, up, down, activation=ACT[act], residual=res, y=y, workspace=buf[:need])
    torch.cuda.synchronize()
    assert_within(y, want, off)
    assert bool((buf[need:] == 0xFF).all())
    y.fill_(12345.0)
    assert bool((raw == 12345.0).all())
    return want


# one of everything; one token and many; tails of chunks on either side; odd features; experts with one to more than 32 tokens; more experts than tokens use
SIZES = [(1, 32, 32, 1, 1, 1), (1, 64, 32, 17, 3, 3), (2, 160, 96, 40, 4, 1), (1, 512, 256, 130, 9, 8), (5, 544, 160, 33, 6, 2), (8, 256, 288, 64, 2, 2), (9, 128, 128, 48, 3, 2),
         (17, 96, 64, 20, 2, 1), (33, 64, 96, 31, 1, 1), (40, 64, 32, 16, 2, 2), (64, 64, 64, 24, 1, 1), (64, 32, 64, 16, 40, 16), (3, 1056, 1120, 100, 12, 4), (16, 160, 64, 300, 5, 2),
         (1, 2080, 544, 50, 2, 2), (4, 32, 32, 5, 1024, 16), (70, 64, 32, 16, 4, 2), (130, 32, 32, 9, 3, 3), (12, 4128, 32, 10, 2, 1), (6, 32, 4128, 20, 3, 2), (25, 288, 160, 36, 1, 1)]


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,K,I,N,E,top", SIZES)
def test_experts(fmt, M, K, I, N, E, top):
    which = M + K + I + N
    if fmt == "nvfp4" and K > 32 and I > 32:
        K, I = K - 16 * (M % 2), I - 16 * (M // 2 % 2)                  # multiples of 16 only
    block = 32 if fmt == "mx" else 16
    check(fmt, M, K, I, N, E, top, S=block * (which % 3 % (K // block + 1)), S2=block * (which % 2), act=L.NAMES[which % 5], residual=which % 2 == 0,
          dtype=torch.float16 if which % 4 < 2 else torch.float32, in_place=which % 4 == 2)
    check(fmt, M, K, I, N, E, top, act="silu", residual=which % 2 == 1, reorder=True, drop=True, dtype=torch.float32 if which % 4 < 2 else torch.float16, seed=1)


# up to 64 and up to 256 choices of up to 16 tokens, K in two, four and eight parts of whole and broken groups of three, four and five chunks; too many tokens for that
@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("K", [256, 1024, 1184, 1280, 1760, 2048, 2304, 2816, 3552, 4096, 4640, 6144, 8160])
@pytest.mark.parametrize("M,top", [(3, 2), (9, 8)])
def test_long_rows(fmt, K, M, top):
    check(fmt, M, K, 48 if fmt == "nvfp4" else 64, 17, 10, top, S=32 * (K % 3), act="gelu", dtype=torch.float32, drop=True)


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,K,I,N,E,top", [(16, 4608, 160, 40, 4, 2), (14, 128, 32, 40, 4, 2), (16, 256, 128, 33, 20, 16),       # gathered, 16 rows at a time; 256 choices
                                           (1, 64, 160, 4112, 3, 2), (3, 64, 416, 5000, 2, 2), (7, 64, 544, 4112, 2, 1),        # columns for half as many waves a workgroup
                                           (5, 256, 2080, 40, 20, 16), (2, 128, 96, 40, 3, 2), (8, 64, 1056, 300, 2, 2),        # slots by themselves, in runs of I and not
                                           (40, 64, 4128, 33, 3, 1), (20, 96, 2080, 600, 2, 2),
                                           (67, 288, 160, 40, 4, 2), (81, 512, 288, 40, 4, 4), (129, 256, 1056, 24, 3, 2)])     # last tokens of another kind than the first
def test_kinds(fmt, M, K, I, N, E, top):
    check(fmt, M, K, I, N, E, top, S=32, S2=32, residual=True, dtype=torch.float32, in_place=True)
    check(fmt, M, K, I, N, E, top, reorder=True, drop=True, residual=True)


@pytest.mark.parametrize("M,K,I,N,E,top", [(2, 1184, 288, 40, 3, 2), (3, 2304, 672, 20, 2, 2), (7, 4640, 1056, 20, 2, 1), (9, 2816, 160, 20, 9, 8), (16, 4608, 288, 20, 2, 1), (12, 160, 544, 20, 2, 2),
                                           (40, 672, 1184, 40, 3, 2), (5, 416, 2080, 24, 20, 16)])
def test_scales_far_apart(M, K, I, N, E, top):
    """MXFP4 blocks that no 16-bit code can take the scale of, here and there and in a row's last blocks."""
    rng = np.random.default_rng(K)
    say(f"moe, scales far apart {M} {K} {I}")
    x = rng.standard_normal((M, K)).astype(np.float16)
    up, down = random_experts("mx", E, 2 * I, K, 32, rng), random_experts("mx", E, N, I, 0, rng)
    for s in (up[1], down[1]):
        s[rng.random(s.shape) < 0.02] = 80
        s[rng.random(s.shape) < 0.01] = 128
        s[:, ::3, -2:] = 94
        s[0, 1::4] = np.maximum(s[0, 1::4], 97)
    ids, w = choices(rng, M, E, top, False)
    want, off = L.experts(x, None, ids, w, up, down)
    assert_within(call("mx", dev(x), None, ids, w, up, down, out_dtype=torch.float32), want, off)


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_tokens_that_are_not_finite(fmt):
    """A token with NaN or infinities in it changes no other token's result."""
    say("moe, inf and nan", fmt)
    rng = np.random.default_rng(8)
    for M, K, I, top in ((2, 512, 160, 2), (7, 1024, 288, 1), (12, 512, 96, 2), (40, 256, 288, 2)):
        up, down = ([dev(t) if t is not None else None for t in random_experts(fmt, 3, r, k, 0, rng)] for r, k in ((2 * I, K), (40, I)))
        x = dev(rng.standard_normal((M, K)).astype(np.float16))
        ids, w = (dev(t) for t in choices(rng, M, 3, top, False))
        want = call(fmt, x, None, ids, w, up, down, out_dtype=torch.float32)
        x[0, 5], x[0, 9], x[0, K - 1] = float("nan"), float("inf"), float("-inf")
        got = call(fmt, x, None, ids, w, up, down, out_dtype=torch.float32)
        assert torch.equal(got[1:], want[1:]) and not bool(torch.isfinite(got[0]).any())


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_tokens_without_experts(fmt):
    """No choice, or none that there is: the residual, or zeros; the weights there are not read."""
    M, K, I, N, E, top = 5, 64, 32, 20, 3, 2
    ids = np.array([[-1, -1], [3, 7], [-2 ** 31, 2 ** 31 - 1], [1, -1], [-1, 2]], dtype=np.int32)
    w = np.where((ids >= 0) & (ids < E), np.float32(0.5), np.float32(np.nan)).astype(np.float32)
    for residual in (False, True):
        for dtype in (torch.float16, torch.float32):
            check(fmt, M, K, I, N, E, top, residual=residual, dtype=dtype, ids=ids, w=np.nan_to_num(w, nan=9.0))
    rng = np.random.default_rng(1)
    x = dev(rng.standard_normal((M, K)).astype(np.float16))
    up, down = random_experts(fmt, E, 2 * I, K, 0, rng), random_experts(fmt, E, N, I, 0, rng)
    y = call(fmt, x, None, ids, w, up, down)
    assert bool(torch.isfinite(y).all()) and bool((y[:3] == 0).all()) and bool((y[3:] != 0).any())
    r = torch.randn((M, N), device="cuda").half()
    assert torch.equal(call(fmt, x, None, np.full((M, top), -1, dtype=np.int32), w, up, down, residual=r), r)


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M", [1, 3, 20])
def test_an_expert_twice(fmt, M):
    """Both weights count, and the same inputs give the same bits every time."""
    rng = np.random.default_rng(7)
    ids = np.array([[2, 0, 2, 1], [1, 1, 1, 1], [0, -1, 0, 2]], dtype=np.int32)[rng.integers(0, 3, M)]
    w = rng.random((M, 4)).astype(np.float32)
    check(fmt, M, 96, 64, 20, 3, 4, ids=ids, w=w, dtype=torch.float32)
    check(fmt, M, 96, 64, 20, 3, 4, ids=ids, w=w, residual=True)


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_same_bits_every_time(fmt):
    rng = np.random.default_rng(9)
    M, K, I, N, E, top = 48, 512, 288, 272, 6, 3
    x = dev(rng.standard_normal((M, K)).astype(np.float16))
    up, down = ([dev(t) if t is not None else None for t in random_experts(fmt, E, r, k, 0, rng)] for r, k in ((2 * I, K), (N, I)))
    ids, w = (dev(t) for t in choices(rng, M, E, top, False))
    first = call(fmt, x, None, ids, w, up, down, out_dtype=torch.float32)
    for _ in range(5):
        assert torch.equal(call(fmt, x, None, ids, w, up, down, out_dtype=torch.float32), first)
    # a token's result is its own: whatever the others choose
    alone = call(fmt, x[5:6], None, ids[5:6], w[5:6], up, down, out_dtype=torch.float32)
    assert float((alone - first[5:6]).abs().max()) <= 1e-4 * float(first.abs().max())


def test_range_of_the_middle():
    """Values between the products far above and below what one fp16 number holds."""
    say("moe, middle values from 2^-30 to 2^19")
    rng = np.random.default_rng(11)
    M, K, I, N, E = 3, 32, 64, 33, 1
    x = np.ones((M, K), dtype=np.float16)
    codes = np.zeros((E, 2 * I, K // 2), dtype=np.uint8)
    codes[:, :, 0] = 0x02                                               # 1.0 times x[0]
    scales = np.full((E, 2 * I, 1), 127, dtype=np.uint8)
    scales[0, :I, 0] = 127 + np.linspace(-20, 9, I).astype(int)         # g = 2^-20 .. 2^9
    scales[0, I:, 0] = 127 + np.linspace(-10, 10, I).astype(int)
    down = random_experts("mx", E, N, I, 0, rng)
    down[1][:] = 127
    ids, w = np.zeros((M, 1), dtype=np.int32), np.array([[1.0], [1.9], [-0.3]], dtype=np.float32)
    for act in ("none", "relu", "silu"):
        want, off = L.experts(x, None, ids, w, (codes, scales, None), down, act)
        assert_within(call("mx", dev(x), None, ids, w, (codes, scales, None), down, activation=ACT[act], out_dtype=torch.float32), want, off)


def test_unaligned_weights_and_scales():
    """Codes at 8-byte addresses, scale bytes at odd ones."""
    say("moe, operands at the least alignment")
    M, K, I, N, E, top = 4, 288, 160, 24, 3, 2
    rng = np.random.default_rng(6)
    x = rng.standard_normal((M, K)).astype(np.float16)
    ids, w = choices(rng, M, E, top, False)
    for fmt in ("nvfp4", "mx"):
        up, down = random_experts(fmt, E, 2 * I, K, 32, rng), random_experts(fmt, E, N, I, 0, rng)
        want, off = L.experts(x, None, ids, w, up, down)
        moved = []
        for p, at, sat in ((up, 8, 1), (down, 24, 3)):
            buf, sbuf = (torch.zeros(t.size + 64, dtype=torch.uint8, device="cuda") for t in p[:2])
            wc, wsc = buf[at:at + p[0].size].view(p[0].shape), sbuf[sat:sat + p[1].size].view(p[1].shape)
            wc.copy_(dev(p[0]))
            wsc.copy_(dev(p[1]))
            moved.append((wc, wsc, p[2]))
        assert_within(call(fmt, dev(x), None, ids, w, *moved, out_dtype=torch.float32), want, off)


@pytest.mark.parametrize("M", [2, 7, 12, 40])
def test_every_scale_byte(M):
    """Exponents of MXFP4 and all scales of NVFP4, on either side of the activation; tokens as one tile of rows and gathered."""
    say("moe, scale bytes", M)
    rng = np.random.default_rng(2)
    for fmt, bytes_, block in (("mx", np.arange(90, 150), 32), ("nvfp4", np.arange(0, 0x7F), 16)):
        K, N = 8 * block, len(bytes_)
        I = (len(bytes_) + 31) // 32 * 32 + 128
        x = (rng.standard_normal((M, K)) * 0.5).astype(np.float16)
        ids, w = np.zeros((M, 1), dtype=np.int32), np.ones((M, 1), dtype=np.float32)
        flat = np.ones(1, dtype=np.float32) if fmt == "nvfp4" else None
        up = rng.integers(0, 256, (1, 2 * I, K // 2), dtype=np.uint8), np.full((1, 2 * I, 8), 120 if fmt == "mx" else 0x30, dtype=np.uint8), flat
        down = rng.integers(0, 256, (1, N, I // 2), dtype=np.uint8), np.repeat(bytes_[None, :, None], I // block, 2).astype(np.uint8), flat
        want, off = L.experts(x, None, ids, w, up, down, "none")
        assert_within(call(fmt, dev(x), None, ids, w, up, down, activation=B.ACT_NONE, out_dtype=torch.float32), want, off)
        up[1][0, :N, :] = bytes_[:, None] if fmt == "nvfp4" else np.clip(bytes_, 112, 134)[:, None]
        down[1][:] = 120 if fmt == "mx" else 0x30
        want, off = L.experts(x, None, ids, w, up, down, "relu")
        assert_within(call(fmt, dev(x), None, ids, w, up, down, activation=B.ACT_RELU, out_dtype=torch.float32), want, off)


def test_operands_past_4_gib():
    """Experts whose codes lie beyond 32-bit offsets."""
    say("moe, 4.3 GiB of codes")
    M, K, I, N, E = 2, 8192, 2048, 16, 260
    torch.manual_seed(0)
    up_c = torch.randint(0, 256, (E, 2 * I, K // 2), dtype=torch.uint8, device="cuda")
    up_s = torch.randint(118, 121, (E, 2 * I, K // 32), dtype=torch.uint8, device="cuda")
    down_c = torch.randint(0, 256, (E, N, I // 2), dtype=torch.uint8, device="cuda")
    down_s = torch.randint(118, 121, (E, N, I // 32), dtype=torch.uint8, device="cuda")
    assert up_c.numel() > 1 << 32
    x = torch.randn((M, K), device="cuda").half()
    w = torch.ones((M, 1), device="cuda")
    y = B.arcq_mx_moe(x, None, torch.full((M, 1), E - 1, dtype=torch.int32, device="cuda"), w, up_c, up_s, down_c, down_s, out_dtype=torch.float32)
    one = [t[E - 1:].contiguous() for t in (up_c, up_s, down_c, down_s)]
    assert torch.equal(y, B.arcq_mx_moe(x, None, torch.zeros((M, 1), dtype=torch.int32, device="cuda"), w, *one, out_dtype=torch.float32))
    assert float(y.abs().max()) > 0


# ------------------------------------------------------------------------------------------------------- together, as in use

def layer(fmt, seed=0):
    rng = np.random.default_rng(seed)
    M, K, I, E, top, S = 6, 512, 160, 12, 3, 64
    perm = rng.permutation(K).astype(np.int32)
    W = (rng.standard_normal((E * 2 * I, K)) / np.sqrt(K)).astype(np.float16)
    D = (rng.standard_normal((E * K, I)) / np.sqrt(I)).astype(np.float16)
    own = torch.arange(I, dtype=torch.int32, device="cuda")
    if fmt == "mx":
        up, down = B.arcq_mx_pack_weight(dev(W), dev(perm), S), B.arcq_mx_pack_weight(dev(D), own, 32)
        host = [MX.pack_weight(W, perm, S), MX.pack_weight(D, np.arange(I), 32)]
        ts = None
    else:
        ts = np.full(E, 0.0005, dtype=np.float32)
        up, down = B.arcq_pack_weight(dev(W), dev(perm), S, 0.0005), B.arcq_pack_weight(dev(D), own, 32, 0.0005)
        host = [A.pack_weight(W, perm, S, np.float32(0.0005)), A.pack_weight(D, np.arange(I), 32, np.float32(0.0005))]
    shape = lambda p, rows: (*(t.reshape(E, rows, -1) for t in p), ts if isinstance(p[0], np.ndarray) or ts is None else dev(ts))  # noqa: E731
    router = (rng.standard_normal((E, K)) / np.sqrt(K)).astype(np.float16)
    x, hidden = rng.standard_normal((M, K)).astype(np.float16), rng.standard_normal((M, K)).astype(np.float32)
    return perm, shape(up, 2 * I), shape(down, K), [shape(host[0], 2 * I), shape(host[1], K)], router, x, hidden, top, I


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_whole_layer(fmt):
    """Weights from the packers, router, experts and the addition to the hidden state in place, eager and replayed, against the oracle."""
    say("moe, whole layer", fmt)
    perm, up, down, host, router, x, hidden, top, I = layer(fmt)
    M, K = x.shape
    E = router.shape[0]
    xd, rd, pd = dev(x), dev(router), dev(perm)
    ids, w = torch.empty((M, top), dtype=torch.int32, device="cuda"), torch.empty((M, top), device="cuda")
    h = dev(hidden)
    scratch = torch.empty(B.arcq_moe_workspace_size(M, top, E, K, I, K, True) + B.arcq_moe_route_workspace_size(M, K, E) + 256, dtype=torch.uint8, device="cuda")
    parts = (up[0], up[1], up[2], down[0], down[1], down[2]) if fmt == "nvfp4" else (up[0], up[1], down[0], down[1])

    def eager():
        B.arcq_moe_route(xd, rd, top, flags=B.MOE_RENORMALIZE, ids=ids, weights=w, workspace=scratch)
        (B.arcq_moe if fmt == "nvfp4" else B.arcq_mx_moe)(xd, pd, ids, w, *parts, residual=h, y=h, workspace=scratch)

    def verify(a, b):
        """against the oracle, with the weights that the router gave (within their own bound)"""
        want_ids, want_w = L.route(a, router, top, None, False, True)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        got_w = w.cpu().numpy()
        assert np.all(np.abs(got_w - want_w) <= want_w * 16 * L.HALF)
        want, off = L.experts(a, perm, want_ids, got_w, host[0], host[1], "silu", b)
        assert_within(h, want, off)

    eager()
    torch.cuda.synchronize()
    verify(x, hidden)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.prepare_moe_route(xd, rd, top, ids, w, flags=B.MOE_RENORMALIZE, workspace=scratch)()
        if fmt == "nvfp4":
            B.prepare_moe(xd, pd, ids, w, *parts, h, scratch, residual=h)()
        else:
            B.prepare_mx_moe(xd, pd, ids, w, *parts, h, scratch, residual=h)()
    rng = np.random.default_rng(5)
    for _ in range(3):
        a, b = rng.standard_normal(x.shape).astype(np.float16), rng.standard_normal(hidden.shape).astype(np.float32)
        xd.copy_(dev(a))
        h.copy_(dev(b))
        scratch.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        verify(a, b)
        got = h.clone()
        h.copy_(dev(b))
        eager()
        torch.cuda.synchronize()
        assert torch.equal(got, h)
    side = torch.cuda.Stream()
    h.copy_(dev(b))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager()
    side.synchronize()
    assert torch.equal(got, h)


def test_two_graphs_share_a_workspace():
    """Two layers captured apart, replayed one after the other on the same scratch memory."""
    say("moe, two graphs")
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    made = []
    for seed in (1, 2):
        perm, up, down, host, router, x, hidden, top, I = layer("mx", seed)
        xd, rd, pd, y = dev(x), dev(router), dev(perm), torch.empty(x.shape, device="cuda")
        ids, w = torch.empty((x.shape[0], top), dtype=torch.int32, device="cuda"), torch.empty((x.shape[0], top), device="cuda")
        B.arcq_moe_route(xd, rd, top, ids=ids, weights=w, workspace=scratch)
        want = B.arcq_mx_moe(xd, pd, ids, w, *up[:2], *down[:2], out_dtype=torch.float32)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.prepare_moe_route(xd, rd, top, ids, w, workspace=scratch)()
            B.prepare_mx_moe(xd, pd, ids, w, *up[:2], *down[:2], y, scratch)()
        made.append((g, y, want, (up, down, xd, rd, pd, ids, w)))
    for _ in range(3):
        for g, y, *_ in made:
            y.fill_(7.0)
            g.replay()
        torch.cuda.synchronize()
        for _, y, want, _ in made:
            assert torch.equal(y, want)


@pytest.mark.parametrize("fmt,M", [("nvfp4", 2), ("mx", 12), ("nvfp4", 48), ("mx", 100)])
def test_replayed_and_at_the_same_time(fmt, M):
    """Each kind of kernel in a graph, replayed with other tokens and choices; two calls at once on streams and workspaces of their own."""
    say("moe, graphs and two streams", fmt, M)
    rng = np.random.default_rng(M)
    K, I, N, E, top = 512, 288, 272, 7, 3
    up, down = ([dev(t) if t is not None else None for t in random_experts(fmt, E, r, k, 0, rng)] for r, k in ((2 * I, K), (N, I)))
    parts = (*up, *down) if fmt == "nvfp4" else (*up[:2], *down[:2])
    prepare, eager = (B.prepare_moe, B.arcq_moe) if fmt == "nvfp4" else (B.prepare_mx_moe, B.arcq_mx_moe)
    perm = dev(rng.permutation(K).astype(np.int32))

    def tokens():
        return (dev(rng.standard_normal((M, K)).astype(np.float16)), *(dev(t) for t in choices(rng, M, E, top, True)))

    x, ids, w = tokens()
    need = B.arcq_moe_workspace_size(M, top, E, K, I, N, True)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    y, r = torch.empty((M, N), device="cuda"), torch.randn((M, N), device="cuda")
    eager(x, perm, ids, w, *parts, residual=r, y=y, workspace=ws[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        prepare(x, perm, ids, w, *parts, y, ws[0], residual=r)()
    for _ in range(4):
        for to, t in zip((x, ids, w), tokens()):
            to.copy_(t)
        ws[0].fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager(x, perm, ids, w, *parts, residual=r))
    sets, streams = [tokens() for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    want = [eager(a, perm, b, c, *parts, out_dtype=torch.float32) for a, b, c in sets]
    ys = [torch.zeros((M, N), device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for (a, b, c), stream, out, scratch in zip(sets, streams, ys, ws):
            with torch.cuda.stream(stream):
                eager(a, perm, b, c, *parts, y=out, workspace=scratch)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ys, want))


def test_operands_that_do_not_fit():
    """Refused before the library sees their addresses."""
    perm, up, down, host, router, x, hidden, top, I = layer("mx")
    xd, pd = dev(x), dev(perm)
    ids, w = B.arcq_moe_route(xd, dev(router), top)
    good = [xd, pd, ids, w, up[0], up[1], down[0], down[1]]
    assert B.arcq_mx_moe(*good).shape == x.shape
    for at, bad in ((0, x), (0, xd.float()), (0, xd.T), (1, pd.cpu()), (1, pd.long()), (2, ids.cpu()), (2, ids.long()), (3, w.half()), (3, w.cpu()), (4, up[0].cpu()), (7, down[1].cpu()),
                    (6, down[0].transpose(0, 1)), (2, torch.cat([ids, ids], 1)[:, ::2])):
        with pytest.raises((AssertionError, B.ArcqError)):
            B.arcq_mx_moe(*good[:at], bad if torch.is_tensor(bad) else torch.from_numpy(bad), *good[at + 1:])
    for at, bad in ((1, pd[:-4]), (2, ids[:, :2].contiguous()), (3, w[:3]), (4, up[0][:3]), (6, down[0][:, :, :1].contiguous()), (5, up[1][:, :, :1].contiguous())):
        with pytest.raises(B.ArcqError):
            B.arcq_mx_moe(*good[:at], bad, *good[at + 1:])
    for kw in ({"activation": 7}, {"residual": xd[:2]}, {"workspace": torch.empty(256, dtype=torch.uint8, device="cuda")}):
        with pytest.raises(B.ArcqError):
            B.arcq_mx_moe(*good, **kw)
    for kw in ({"top_k": 0}, {"top_k": 13}, {"top_k": 17}, {"flags": 4}, {"bias": torch.zeros(3, device="cuda")}):
        with pytest.raises(B.ArcqError):
            B.arcq_moe_route(xd, dev(router), **{"top_k": top, **kw})
    with pytest.raises(B.ArcqError):
        B.arcq_moe_route(xd, dev(router)[:, :-8], top)
    # nothing to do
    assert B.arcq_mx_moe(xd[:0], pd, ids[:0], w[:0], *good[4:]).shape == (0, x.shape[1])
    assert B.arcq_moe_route(xd[:0], dev(router), top)[0].shape == (0, top)
