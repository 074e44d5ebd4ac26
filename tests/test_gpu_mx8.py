"""GPU parity of the MXFP8 path against the oracle: quantizers byte by byte, products within a bound derived from their roundings."""
import numpy as np
import pytest
import torch

from oracle import mxfp4 as MX
from oracle import mxfp8 as M8
from paper_2601_07475_amd import binding as B
from paper_2601_07475_amd import workloads as wk

from test_gpu_parity import assert_same_bytes, dev, guarded_empty, guards_intact, say

pytestmark = pytest.mark.gpu


def inputs(M, K, seed):
    """Rows with outlier channels, and among them the blocks where a scale or an element can go wrong."""
    wl = wk.Workload("t", M, K, 1, 0, max(1, K // 100), "loguniform20_100", 0.02, seed)
    X = wk.activations(wl)
    X[0, :32] = 0                                                       # nothing in a block
    if M > 1:
        X[1, :32] = -0.0
        X[1, K - 32:] = np.float16(2.0 ** -24)                          # the smallest subnormals alone
    if M > 2:
        X[2, :32] = np.linspace(440, 512, 32).astype(np.float16)        # around the largest element
        X[2, K - 32:] = 65504
    return X


def strided(a, extra):
    """The array on the GPU inside rows `extra` elements longer, whose rest is NaN."""
    t = torch.full((a.shape[0], a.shape[1] + extra), float("nan"), dtype=torch.float16, device="cuda")
    t[:, :a.shape[1]] = dev(a)
    return t[:, :a.shape[1]]


def fp16_output(M, K, extra=0):
    """(whole buffer, the [M, K] view of it) with everything at NaN's bit pattern 0x7E7E."""
    raw = torch.full((M * (K + extra) + 256,), 0x7E7E, dtype=torch.int16, device="cuda").view(torch.float16)
    return raw, raw[128:128 + M * (K + extra)].view(M, K + extra)[:, :K]


def untouched(raw, view):
    """Everything of raw outside view still has its fill."""
    bits = raw.view(torch.int16).clone()
    inside = torch.as_strided(bits, view.shape, view.stride(), 128)
    inside.fill_(0x7E7E)
    return bool((bits == 0x7E7E).all())


def quantize(fn, M, K, **kw):
    raw_c, codes = guarded_empty((M, K))
    raw_s, scales = guarded_empty((M, K // 32))
    out = fn(codes=codes, scales=scales, **kw)
    torch.cuda.synchronize()
    assert guards_intact(raw_c, M * K) and guards_intact(raw_s, M * K // 32)
    return codes.cpu().numpy(), scales.cpu().numpy(), out


# a block, lane tails, one to four halves a lane and their limits, more rows than workgroups (with two, with one buffer)
SHAPES = [(1, 32), (3, 64), (5, 1056), (130, 4096), (33, 5120), (4, 14336), (3, 16384), (3, 16416), (2, 28672), (2, 32768), (2, 32800),
          (3, 65536), (5000, 96), (2600, 4096), (530, 20512), (300, 40960)]


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("reorder", [False, True])
def test_quantizer_bytes(M, K, reorder):
    up = (M + K // 32 + reorder) % 2
    say(f"mx8_quantize_act M={M} K={K} reorder={reorder} up={up}")
    X = inputs(M, K, seed=K % 89)
    perm = np.random.default_rng(K).permutation(K).astype(np.int32) if reorder else None
    want_c, want_s = M8.quantize_act(X, perm, "up" if up else "nearest")
    got_c, got_s, _ = quantize(B.arcq_mx8_quantize_act, M, K, x=strided(X, 8 * (M % 3)), perm=dev(perm) if reorder else None,
                               flags=B.SCALE_ROUND_UP if up else 0)
    assert_same_bytes(got_s, want_s, "scales")
    assert_same_bytes(got_c, want_c, "codes")


def norm_inputs(M, K, seed):
    X, R = inputs(M, K, seed), inputs(M, K, seed + 1)
    X, R = (np.clip(t, -30000, 30000) for t in (X, R))                  # their sum stays finite
    R[0, 32:64] = -X[0, 32:64]                                          # sums of zero
    wl = wk.Workload("t", M, K, 1, 0, 1, "const50", 0.02, seed)
    return X, R, wk.rmsnorm_gamma(wl)


@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("reorder", [False, True])
@pytest.mark.parametrize("add", [False, True])
def test_norm_bytes(M, K, reorder, add):
    if M * K > 5e6 and not add:
        M //= 4
    up, exact = (M + K // 32 + reorder) % 2, (K // 32 + add) % 2
    say(f"mx8_add_rmsnorm_quantize_act M={M} K={K} reorder={reorder} add={add} up={up} exact={exact}")
    X, R, gamma = norm_inputs(M, K, seed=K % 83)
    perm = np.random.default_rng(K).permutation(K).astype(np.int32) if reorder else None
    want_c, want_s, want_h = M8.add_rmsnorm_quantize_act(X, R if add else None, gamma, 1e-5, perm, "up" if up else "nearest")
    raw, hidden = fp16_output(M, K, 16)
    kw = dict(x=strided(X, 8), residual=strided(R, 24) if add else None, gamma=dev(gamma), eps=1e-5, perm=dev(perm) if reorder else None,
              hidden=hidden if add else None, flags=(B.SCALE_ROUND_UP if up else 0) | (B.RMSNORM_EXACT_SUM if exact else 0))
    got_c, got_s, _ = quantize(B.arcq_mx8_add_rmsnorm_quantize_act, M, K, **kw)
    assert_same_bytes(got_s, want_s, "scales")
    assert_same_bytes(got_c, want_c, "codes")
    assert untouched(raw, hidden)
    if add:
        assert_same_bytes(hidden.contiguous().view(torch.int16).cpu().numpy(), want_h.view(np.int16), "hidden")
    # the integer sum and the fp64 sum with its bracket give the same bytes
    kw["flags"] ^= B.RMSNORM_EXACT_SUM
    other_c, other_s, _ = quantize(B.arcq_mx8_add_rmsnorm_quantize_act, M, K, **kw)
    assert_same_bytes(other_s, want_s, "scales, the other sum")
    assert_same_bytes(other_c, want_c, "codes, the other sum")


@pytest.mark.parametrize("over", ["x", "residual"])
@pytest.mark.parametrize("M,K,reorder", [(3000, 256, True), (700, 20512, False), (300, 40960, True)])
def test_norm_in_place(M, K, reorder, over):
    say(f"mx8_add_rmsnorm_quantize_act in place of {over} M={M} K={K}")
    X, R, gamma = norm_inputs(M, K, seed=3)
    perm = torch.randperm(K, device="cuda").int() if reorder else None
    x, r = strided(X, 8), strided(R, 16)
    c, s, h = B.arcq_mx8_add_rmsnorm_quantize_act(x, r, dev(gamma), 1e-5, perm)
    for _ in range(2):
        x, r = strided(X, 8), strided(R, 16)
        target = x if over == "x" else r
        c2, s2, h2 = B.arcq_mx8_add_rmsnorm_quantize_act(x, r, dev(gamma), 1e-5, perm, hidden=target)
        assert h2 is target and torch.equal(c, c2) and torch.equal(s, s2) and torch.equal(h, target)
        assert torch.equal(r if over == "x" else x, dev(R if over == "x" else X))


def test_rows_whose_mean_sits_on_a_border():
    """Rows whose exact mean of squares is halfway between two fp32 values: the plain sum cannot decide them."""
    say("rows on a rounding border of the mean")
    K = 64
    X = np.zeros((4, K), dtype=np.float16)
    # sum of squares 2^24 + 1 (and + 3): halfway between fp32 neighbours; dividing by K = 64 keeps it there
    X[0, :2] = [4096, 1]
    X[1, :4] = [4096, 1, 1, 1]
    X[2, :3] = [4096, 1, 2.0 ** -24]                                    # just above: only an exact sum sees it
    X[3, :] = 1
    gamma = np.ones(K, dtype=np.float16)
    want_c, want_s, _ = M8.add_rmsnorm_quantize_act(X, None, gamma, 0.0)
    got_c, got_s, _ = quantize(B.arcq_mx8_add_rmsnorm_quantize_act, 4, K, x=dev(X), residual=None, gamma=dev(gamma), eps=0.0)
    assert_same_bytes(got_s, want_s, "scales")
    assert_same_bytes(got_c, want_c, "codes")


def test_rows_of_zeros():
    say("rows of zeros, with eps")
    X = np.zeros((2, 4096), dtype=np.float16)
    X[1, 7] = 2.0 ** -24
    gamma = np.full(4096, 2.0, dtype=np.float16)
    want_c, want_s, want_h = M8.add_rmsnorm_quantize_act(X, X, gamma, 1e-6)
    got_c, got_s, out = quantize(B.arcq_mx8_add_rmsnorm_quantize_act, 2, 4096, x=dev(X), residual=dev(X), gamma=dev(gamma), eps=1e-6)
    assert_same_bytes(got_s, want_s, "scales")
    assert_same_bytes(got_c, want_c, "codes")
    assert np.array_equal(out[2].cpu().numpy(), want_h)


# ------------------------------------------------------------------------------------------------------------------ products

def assert_product(y, want, mag, K, dropped=0.0):
    """dropped: what the kernel's summation may lose beside fp32 accumulation, an array like want."""
    got = y.double().cpu().numpy()
    # each of the K / 32 block sums and each addition to the accumulator loses less than a step, 2^-23 of at most mag; joining waves and runs: 64 more
    bound = mag * (K / 16 + 64) * 2.0 ** -23 + dropped
    if y.dtype is torch.float16:
        bound = bound + (np.abs(want) + bound) * 2.0 ** -11 + 2.0 ** -25        # half a step, of a subnormal too
    over = np.abs(got - want) - bound
    assert np.isfinite(got).all() and over.max() <= 0, f"{over.max()} over the bound at {np.unravel_index(over.argmax(), over.shape)}"
    if y.dtype is torch.float32 or np.ndim(dropped) == 0:
        rms = np.sqrt(np.mean(want ** 2))
        err = np.max(np.abs(got - want) / np.maximum(np.abs(want), max(rms, 1e-300)))
        assert err <= (2e-5 if y.dtype is torch.float32 else 1e-3), err


def assert_fp16_product(y, ac, asc, wc, wsc, want, mag):
    """fp16 results of arcq_mx8_gemm: the bits that the matrix unit drops looked up for some rows, bounded for all: less than 2^-13 of the
    largest of eight products for each of seven others, 2^-10 of the sum of the eight magnitudes."""
    M, K = ac.shape
    rows = np.unique(np.linspace(0, M - 1, max(1, min(M, int(4e7) // (wc.shape[0] * K)))).astype(int))
    assert_product(y[torch.from_numpy(rows).cuda()], want[rows], mag[rows], K, M8.aligned_loss(ac[rows], asc[rows], wc, wsc))
    assert_product(y, want, mag, K, mag * 2.0 ** -10)


def packed_weights(N, K, S, seed, perm=None):
    W = (np.random.default_rng(seed).standard_normal((N, K)) * 0.02).astype(np.float16)
    return MX.pack_weight(W, np.arange(K) if perm is None else perm, S)


def output(M, N, dtype, extra):
    """A guarded output of a product: (whole buffer, view)."""
    raw = torch.full((M * (N + extra) + 64,), 12345.0, dtype=dtype, device="cuda")
    return raw, raw[32:32 + M * (N + extra)].view(M, N + extra)[:, :N]


def run_gemm(M, N, K, S, dtype, seed, extra=0, workspace=True):
    X = wk.activations(wk.Workload("t", M, K, N, 0, max(1, K // 100), "loguniform20_100", 0.02, seed))
    ac, asc = M8.quantize_act(X)
    wc, wsc = packed_weights(N, K, S, seed + 1)
    want, mag = M8.gemm(ac, asc, wc, wsc)
    need = B.arcq_mx8_gemm_workspace_size(M, N, K)
    ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
    raw, y = output(M, N, dtype, extra)
    B.arcq_mx8_gemm(dev(ac), dev(asc), dev(wc), dev(wsc), y=y, workspace=ws)
    torch.cuda.synchronize()
    if dtype is torch.float16:
        assert_fp16_product(y, ac, asc, wc, wsc, want, mag)
    else:
        assert_product(y, want, mag, K)
    y.fill_(12345.0)
    assert bool((raw == 12345.0).all())                                 # nothing beside the output
    return need


# M, N, K, S: one of everything, tails of rows, features, blocks and units, few and many rows, S = 0 and S = K
GEMM_SHAPES = [(1, 1, 32, 0), (1, 17, 64, 32), (3, 16, 96, 96), (16, 250, 512, 64), (17, 333, 1056, 0), (33, 64, 4128, 32), (64, 4100, 544, 0),
               (65, 129, 1568, 128), (100, 1000, 2048, 0), (128, 128, 256, 0), (129, 257, 160, 32), (255, 511, 3104, 64), (256, 256, 128, 0),
               (300, 2000, 992, 0), (513, 700, 736, 32), (777, 515, 4352, 224), (1000, 3000, 1024, 0), (1, 5000, 14336, 0), (16, 2048, 8192, 256),
               (200, 256, 16384, 0), (2049, 1, 320, 0), (1, 40000, 96, 0), (4100, 260, 448, 0)]


@pytest.mark.parametrize("M,N,K,S", GEMM_SHAPES)
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_gemm(M, N, K, S, dtype):
    say(f"mx8_gemm M={M} N={N} K={K} S={S} {dtype}")
    run_gemm(M, N, K, S, dtype, seed=M + K, extra=(N * 7) % 5, workspace=(M + N) % 2 == 0)


F16, F32 = torch.float16, torch.float32
# M, N, K, S, type, workspace, (kernel, tile rows, tile columns, runs): every tile, K off its unit of 128 so that rows of scale bytes start at any address
TILE_SHAPES = [(154, 66, 1888, 0, F16, True, (B.ROUTE_TILES, 64, 128, 3)), (149, 69, 2016, 96, F32, True, (B.ROUTE_TILES, 64, 128, 4)),
               (1306, 2949, 544, 0, F16, False, (B.ROUTE_TILES, 64, 256, 1)), (6055, 261, 544, 0, F32, False, (B.ROUTE_TILES, 64, 256, 1)),
               (6055, 261, 544, 0, F16, False, (B.ROUTE_TILES, 128, 128, 1)), (393, 8112, 608, 0, F32, False, (B.ROUTE_TILES, 128, 128, 1)),
               (2113, 2756, 544, 96, F16, False, (B.ROUTE_TILES, 128, 256, 1)), (2113, 2756, 544, 96, F32, False, (B.ROUTE_TILES, 128, 256, 1)),
               (6552, 555, 544, 0, F16, False, (B.ROUTE_TILES, 192, 128, 1)), (6552, 555, 544, 0, F32, False, (B.ROUTE_TILES, 192, 128, 1)),
               (2965, 2695, 544, 96, F16, False, (B.ROUTE_TILES, 192, 256, 1)), (2965, 2695, 544, 96, F32, False, (B.ROUTE_TILES, 192, 256, 1)),
               (7457, 1649, 544, 0, F16, False, (B.ROUTE_TILES, 256, 256, 1)),
               (520, 2050, 8224, 0, F16, True, (B.ROUTE_TILES, 128, 128, 3)), (300, 4100, 8224, 0, F32, True, (B.ROUTE_TILES, 64, 256, 3)),
               (520, 4100, 6176, 0, F32, True, (B.ROUTE_TILES, 128, 256, 3))]
# the streaming kernel with K in several runs, and with more rows than a launch takes
STREAM_SHAPES = [(15, 112, 20640, 0, F16, True, (B.ROUTE_STREAM, 16, 16, 8)), (30, 40, 16416, 0, F32, True, (B.ROUTE_STREAM, 32, 16, 8)),
                 (16, 1030, 28704, 224, F16, True, (B.ROUTE_STREAM, 16, 16, 3)), (128, 70, 8224, 0, F32, True, (B.ROUTE_STREAM, 32, 16, 6)),
                 (15, 112, 20640, 0, F32, False, (B.ROUTE_STREAM, 16, 16, 1)), (65600, 40, 96, 0, F32, True, (B.ROUTE_TILES, 128, 128, 1))]


@pytest.mark.parametrize("M,N,K,S,dtype,workspace,route", TILE_SHAPES + STREAM_SHAPES)
def test_gemm_tiles(M, N, K, S, dtype, workspace, route):
    say(f"mx8_gemm M={M} N={N} K={K} S={S} {dtype} on {route}")
    assert B.arcq_mx8_gemm_route(M, N, K, S, dtype, workspace) == route
    run_gemm(M, N, K, S, dtype, seed=M, extra=3, workspace=workspace)


def test_gemm_scale_bytes_at_any_address():
    """Scale bytes of both operands at odd addresses of their own, on tiles and streamed."""
    say("mx8_gemm, scale bytes at odd addresses")
    for M, N, K, S in ((200, 300, 1056, 32), (5, 300, 1056, 32), (129, 257, 2048, 0)):
        X = wk.activations(wk.Workload("t", M, K, N, 0, 10, "loguniform20_100", 0.02, 5))
        ac, asc = M8.quantize_act(X)
        wc, wsc = packed_weights(N, K, S, 6)
        want, mag = M8.gemm(ac, asc, wc, wsc)
        buf = [torch.full((t.size + 8,), 0xFF, dtype=torch.uint8, device="cuda") for t in (asc, wsc)]      # 0xFF: NaN, beside the operands
        for offs in ((1, 2), (3, 1), (2, 3)):
            views = []
            for b, o, t in zip(buf, offs, (asc, wsc)):
                b.fill_(0xFF)
                views.append(b[o:o + t.size].view(t.shape))
                views[-1].copy_(dev(t))
            y = B.arcq_mx8_gemm(dev(ac), views[0], dev(wc), views[1], out_dtype=torch.float32)
            assert_product(y, want, mag, K)


@pytest.mark.parametrize("up", [0, 1])
def test_gemm_extreme_scales(up):
    """Blocks of very different size in one row, up to both ends of what the quantizer writes."""
    say("mx8_gemm, scales over the whole range")
    M, N, K = 70, 40, 640
    rng = np.random.default_rng(8)
    X = (rng.standard_normal((M, K // 32, 32)) * 2.0 ** rng.integers(-22, 14, (M, K // 32, 1))).reshape(M, K).astype(np.float16)
    W = (rng.standard_normal((N, K // 32, 32)) * 2.0 ** rng.integers(-22, 13, (N, K // 32, 1))).reshape(N, K).astype(np.float16)
    wc, wsc = MX.pack_weight(W, np.arange(K), 0)
    c, s, _ = quantize(B.arcq_mx8_quantize_act, M, K, x=dev(X), flags=up * B.SCALE_ROUND_UP)
    want, mag = M8.gemm(c, s, wc, wsc)
    for rows in (M, 5):
        y = B.arcq_mx8_gemm(dev(c[:rows]), dev(s[:rows]), dev(wc), dev(wsc), out_dtype=torch.float32)
        got = y.double().cpu().numpy()
        assert np.all(np.abs(got - want[:rows]) <= mag[:rows] * (K / 16 + 64) * 2.0 ** -23)


def test_packed_weights_serve_both_precisions():
    """The layer's weights, packed once with S for the 4-bit path, under 4-bit and under 8-bit activations: both come near fp16 rows."""
    say("one set of packed weights, both precisions")
    M, N, K, S = 48, 192, 1024, 64
    rng = np.random.default_rng(12)
    X = wk.activations(wk.Workload("t", M, K, N, S, 10, "loguniform20_100", 0.02, 9))
    perm = wk.calibrate_perm(X)
    W = (rng.standard_normal((N, K)) * 0.02).astype(np.float16)
    x, p = dev(X), dev(perm)
    wc, wsc = B.arcq_mx_pack_weight(dev(W), p, S)
    y4 = B.arcq_mx_gemm(*B.arcq_mx_quantize_act(x, p, S), wc, wsc, out_dtype=torch.float32)
    y8 = B.arcq_mx8_gemm(*B.arcq_mx8_quantize_act(x, p), wc, wsc, out_dtype=torch.float32)
    xp, w = X.astype(np.float64)[:, perm], MX.dequantize(wc.cpu().numpy(), wsc.cpu().numpy())[:, :K]
    full = xp @ w.T
    # An element is off by at most 2^-4 of it (rounding) or an eighth (one in (448, 512] steps of its block saturates), one below the
    # smallest normal by 2^-10 of the block's step, which is at most 2^-8 of its maximum; fp32 accumulation is far below.
    amax = np.repeat(np.abs(xp).reshape(M, K // 32, 32).max(-1), 32, axis=1)
    bound = (np.abs(xp) / 8 + amax * 2.0 ** -18) @ np.abs(w).T * (1 + 2.0 ** -10)
    assert np.all(np.abs(y8.double().cpu().numpy() - full) <= bound)
    # 4 bits: half a step of E2M1 is at most a sixth of a block's maximum, saturation a quarter of it
    bound4 = (amax / 4) @ np.abs(w).T * (1 + 2.0 ** -10)
    assert np.all(np.abs(y4.double().cpu().numpy() - full) <= bound4)


def test_empty_calls_launch_nothing():
    x = torch.empty((0, 64), dtype=torch.float16, device="cuda")
    g = torch.ones(64, dtype=torch.float16, device="cuda")
    c, s = B.arcq_mx8_quantize_act(x)
    assert c.shape == (0, 64) and s.shape == (0, 2)
    c, s, h = B.arcq_mx8_add_rmsnorm_quantize_act(x, x, g, 1e-5)
    assert h.shape == (0, 64)
    w, ws = torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros((8, 2), dtype=torch.uint8, device="cuda")
    assert B.arcq_mx8_gemm(c, s, w, ws).shape == (0, 8)
    a, asc = torch.zeros((3, 64), dtype=torch.uint8, device="cuda"), torch.zeros((3, 2), dtype=torch.uint8, device="cuda")
    assert B.arcq_mx8_gemm(a, asc, w[:0], ws[:0]).shape == (3, 0)
