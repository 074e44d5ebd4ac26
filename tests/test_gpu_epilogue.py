"""GPU parity of the products with bias, activation and residual against the oracle, within a bound derived from their roundings."""
import numpy as np
import pytest
import torch

from oracle import layers as L
from oracle import mxfp8 as M8
from paper_2601_07475_amd import binding as B
from paper_2601_07475_amd import workloads as wk

from test_gpu_gemv import pack
from test_gpu_mx8 import output, strided
from test_gpu_parity import dev, say

pytestmark = pytest.mark.gpu
ACT = dict(zip(L.NAMES, (B.ACT_NONE, B.ACT_RELU, B.ACT_GELU, B.ACT_GELU_TANH, B.ACT_SILU)))


def assert_within(y, want, off):
    """off: what fp32 arithmetic may lose; y's own rounding comes on top: half a step, of a subnormal too."""
    got = y.double().cpu().numpy()
    half = torch.finfo(y.dtype).eps / 2
    bound = off + (np.abs(want) + off) * half + (2.0 ** -25 if y.dtype is torch.float16 else 2.0 ** -149)
    over = np.abs(got - want) - bound
    assert np.isfinite(got).all() and over.max(initial=-1.0) <= 0, f"{over.max()} over the bound at {np.unravel_index(over.argmax(), over.shape)}"


class Product:
    """One of the three products: operands, its sums in 64 bits, and calls of it."""

    def __init__(self, kind, M, N, K, S, seed, reorder=False):
        self.kind, self.M, self.N, self.K = kind, M, N, K
        rng = np.random.default_rng(seed)
        X = wk.activations(wk.Workload("t", M, K, N, S, max(1, K // 100), "loguniform20_100", 0.02, seed))
        W = (rng.standard_normal((N, K)) * 0.5 / np.sqrt(K)).astype(np.float16)
        perm = rng.permutation(K).astype(np.int32) if reorder else None
        w = pack("nvfp4" if kind == "gemv" else "mx", W, np.arange(K) if perm is None else perm, S)
        self.w = dev(w[0]), dev(w[1])
        if kind == "mx8":
            a = M8.quantize_act(X)
            self.head = (dev(a[0]), dev(a[1]), *self.w)
            self.sums, self.mag = M8.gemm(*a, *w[:2])
        else:
            self.head = (strided(X, 8 * (M % 3)), None if perm is None else dev(perm), *self.w)
            self.head += (float(w[2]),) if kind == "gemv" else ()
            self.sums, self.mag = M8.gemv(X, perm, *w)
        self.need = (B.arcq_mx8_gemm_workspace_size(M, N, K) if kind == "mx8" else
                     (B.arcq_gemv_workspace_size if kind == "gemv" else B.arcq_mx_gemv_workspace_size)(M, N, K, reorder))

    def __call__(self, **kw):
        fn = {"gemv": B.arcq_gemv_epilogue, "mx_gemv": B.arcq_mx_gemv_epilogue, "mx8": B.arcq_mx8_gemm_epilogue}[self.kind]
        return fn(*self.head, **kw)

    def plain(self, **kw):
        return {"gemv": B.arcq_gemv, "mx_gemv": B.arcq_mx_gemv, "mx8": B.arcq_mx8_gemm}[self.kind](*self.head, **kw)


def check(p, act, bias, residual, dtype, extra=3, in_place=False, workspace=True, seed=0):
    rng = np.random.default_rng(seed)
    M, N = p.M, p.N
    b = (2.0 * rng.standard_normal(N)).astype(np.float16) if bias else None
    r = (3.0 * rng.standard_normal((M, N))).astype(np.float16 if dtype is torch.float16 else np.float32) if residual else None
    want, off = L.finish(p.sums, p.mag, p.K, b, act, r)
    raw, y = output(M, N, dtype, extra)
    res = None
    if residual and in_place:
        y.copy_(dev(r))
        res = y
    elif residual:
        res = output(M, N, dtype, 5)[1]
        res.copy_(dev(r))
    ws = torch.full((max(p.need, 256),), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
    p(bias=None if b is None else dev(b), activation=ACT[act], residual=res, y=y, workspace=ws)
    torch.cuda.synchronize()
    assert_within(y, want, off)
    if residual and not in_place:
        assert torch.equal(res, dev(r))
    y.fill_(12345.0)
    assert bool((raw == 12345.0).all())


# one of everything; odd features; every tile of rows; one to four weight tiles; K in several runs; more rows than one pass takes
ROWS = [(1, 1, 32, 0), (2, 17, 64, 32), (4, 1030, 512, 64), (5, 333, 544, 32), (16, 250, 1056, 0), (17, 64, 2592, 64), (33, 70, 1120, 96), (9, 4100, 4064, 0),
        (1, 64, 14336, 256), (3, 512, 28672, 0), (16, 1023, 8224, 0), (30, 850, 9312, 0), (7, 9000, 736, 224)]


@pytest.mark.parametrize("kind", ["gemv", "mx_gemv"])
@pytest.mark.parametrize("M,N,K,S", ROWS)
def test_rows(kind, M, N, K, S):
    for n, act in enumerate(L.NAMES):
        which = M + N + n
        dtype = torch.float16 if which % 2 else torch.float32
        say(f"{kind}_epilogue M={M} N={N} K={K} S={S} {act} {dtype}")
        if n == 0 or n == 3:
            p = Product(kind, M, N, K, S, M + N, reorder=n == 3)
        check(p, act, which % 3 != 0, which % 4 != 1, dtype, extra=N % 4, in_place=which % 5 == 0, seed=n)


# streaming with one and two tiles of rows and several weight tiles, K in runs; tiles of every size and both types, with ragged edges and K;
# tiles with K in runs; one feature, one row
TILES = [(1, 1, 32, 0), (3, 100, 128, 0), (16, 3001, 416, 32), (31, 4100, 1056, 0), (15, 112, 20640, 0), (1, 481, 16032, 0), (65, 65, 64, 0), (130, 333, 544, 96),
         (300, 500, 2592, 0), (777, 1030, 1056, 0), (1000, 2600, 352, 0), (2500, 1800, 128, 0), (300, 512, 14336, 0), (140, 5000, 288, 0), (4097, 2111, 96, 0)]


@pytest.mark.parametrize("M,N,K,S", TILES)
def test_mx8(M, N, K, S):
    p = Product("mx8", M, N, K, S, M + N)
    for n, act in enumerate(L.NAMES):
        for dtype in (torch.float16, torch.float32):
            which = M + N + n + (dtype is torch.float32)
            say(f"mx8_epilogue M={M} N={N} K={K} S={S} {act} {dtype}", B.arcq_mx8_gemm_route(M, N, K, S, dtype, which % 3 > 0))
            check(p, act, which % 3 != 1, which % 4 != 2, dtype, extra=N % 4, in_place=which % 5 == 0, workspace=which % 3 > 0, seed=n)


def test_every_mx8_tile_runs():
    """The shapes above reach the streaming kernel and every tile, in one run of K and in several."""
    routes = {(dt, B.arcq_mx8_gemm_route(M, N, K, S, dt, True)) for M, N, K, S in TILES + MORE for dt in (torch.float16, torch.float32)}
    tiles = {(dt, r[1], r[2]) for dt, r in routes if r[0] == B.ROUTE_TILES}
    assert any(r[0] == B.ROUTE_STREAM and r[3] > 1 for _, r in routes) and any(r[0] == B.ROUTE_TILES and r[3] > 1 for _, r in routes)
    six = {(64, 128), (64, 256), (128, 128), (128, 256), (192, 128), (192, 256)}
    assert {t[1:] for t in tiles if t[0] is torch.float16} == six | {(256, 256)} and {t[1:] for t in tiles if t[0] is torch.float32} == six


MORE = [(415, 8410, 64, 0), (587, 8381, 64, 0), (516, 7293, 64, 0), (912, 8555, 160, 0), (2320, 3345, 64, 0), (268, 6591, 64, 0), (2765, 1375, 64, 0)]


@pytest.mark.parametrize("M,N,K,S", MORE)
def test_mx8_large_tiles(M, N, K, S):
    p = Product("mx8", M, N, K, S, 5)
    for dtype, act in ((torch.float16, "silu"), (torch.float32, "gelu")):
        say(f"mx8_epilogue M={M} N={N} K={K} {dtype}", B.arcq_mx8_gemm_route(M, N, K, S, dtype, True))
        check(p, act, True, True, dtype, extra=1)


@pytest.mark.parametrize("kind", ["gemv", "mx_gemv", "mx8"])
def test_nothing_behind_the_product_is_the_plain_call(kind):
    say(kind)
    p = Product(kind, 6, 200, 512, 32, 1)
    for dtype in (torch.float16, torch.float32):
        assert torch.equal(p(out_dtype=dtype), p.plain(out_dtype=dtype))


@pytest.mark.parametrize("kind,M,N", [("gemv", 5, 1), ("mx_gemv", 40, 90), ("mx8", 300, 700), ("mx8", 20, 40)])
def test_activations_over_their_range(kind, M, N):
    """Sums from -300 to 300, and tiny ones: nothing overflows on the way, and far arguments have their limits."""
    say(kind, M, N)
    K = 64
    rng = np.random.default_rng(4)
    p = Product(kind, M, N, K, 0, 1)
    b = np.resize(np.concatenate([np.linspace(-300, 300, 61), np.linspace(-8, 8, 33), [1e-4, -1e-4, 6e-8, -6e-8, 0.0]]), N).astype(np.float16)
    rng.shuffle(b)
    for act in L.NAMES:
        want, off = L.finish(p.sums, p.mag, K, b, act)
        for dtype in (torch.float16, torch.float32):
            assert_within(p(bias=dev(b), activation=ACT[act], out_dtype=dtype), want, off)


def test_more_rows_than_a_launch_takes():
    say("mx_gemv_epilogue, 70000 rows")
    p = Product("mx_gemv", 70000, 20, 64, 0, 8, reorder=True)
    check(p, "gelu_tanh", True, True, torch.float16)


def test_more_mx8_rows_than_a_launch_takes():
    say("mx8_gemm_epilogue, 70000 rows")
    p = Product("mx8", 70000, 24, 64, 32, 9)
    check(p, "silu", True, True, torch.float32)
    check(p, "none", True, True, torch.float16, in_place=True, workspace=False)


def test_other_streams_and_graphs():
    """Captured on a stream of its own, replayed with other inputs between eager calls; two graphs with one workspace, one after the other."""
    say("epilogues in graphs")
    for kind, M, N, K in (("gemv", 3, 512, 28672), ("mx_gemv", 16, 1023, 8224), ("mx8", 300, 512, 14336), ("mx8", 200, 300, 96)):
        p = Product(kind, M, N, K, 0, 3)
        bias = torch.randn(N, device="cuda").half()
        ys = [torch.randn((M, N), device="cuda").half() for _ in range(2)]
        res = [torch.randn((M, N), device="cuda").half() for _ in range(2)]
        ws = torch.empty(max(p.need, 256), dtype=torch.uint8, device="cuda")
        prepare = {"gemv": B.prepare_gemv_epilogue, "mx_gemv": B.prepare_mx_gemv_epilogue, "mx8": B.prepare_mx8_gemm_epilogue}[kind]
        graphs = []
        for i in range(2):
            p(bias=bias, activation=B.ACT_SILU, residual=res[i], y=ys[i], workspace=ws)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                prepare(*p.head, ys[i], bias=bias, activation=B.ACT_SILU, residual=res[i], workspace=ws)()
            graphs.append(g)
        for turn in range(3):
            for i in range(2):
                res[i].normal_()
                ys[i].fill_(7.0)
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            for i in range(2):
                assert torch.equal(ys[i], p(bias=bias, activation=B.ACT_SILU, residual=res[i], workspace=ws)), (kind, turn)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = p(bias=bias, activation=B.ACT_SILU, residual=res[0], workspace=ws)        # (without, K would go in one run)
        side.synchronize()
        assert torch.equal(again, ys[0])


def test_operands_that_do_not_fit():
    """Refused before the library sees their addresses."""
    p = Product("mx8", 4, 40, 64, 0, 1)
    y, b, r = torch.zeros((4, 40), device="cuda").half(), torch.zeros(40, device="cuda").half(), torch.zeros((4, 40), device="cuda").half()
    for kw in ({"bias": b.cpu()}, {"bias": b.float()}, {"residual": r.cpu()}, {"residual": r.float(), "y": y}, {"residual": r.T}, {"bias": torch.cat([b, b])[::2]}):
        with pytest.raises((AssertionError, B.ArcqError)):
            p(**kw)
    for kw in ({"bias": b[:39]}, {"residual": r[:3]}, {"residual": r[:, :39]}, {"activation": 5}, {"activation": -1}):
        with pytest.raises(B.ArcqError):
            p(**kw)
    wide = torch.zeros((4, 80), device="cuda").half()
    with pytest.raises(B.ArcqError):
        p(residual=wide[:, :40], y=torch.as_strided(wide, (4, 40), (40, 1)))
    assert p(residual=wide[:, :40], y=wide[:, :40]).data_ptr() == wide.data_ptr()


def test_no_rows_and_no_features():
    one = torch.ones((1, 64), dtype=torch.float16, device="cuda")
    w, s = torch.zeros((8, 32), dtype=torch.uint8, device="cuda"), torch.zeros((8, 2), dtype=torch.uint8, device="cuda")
    b = torch.ones(8, dtype=torch.float16, device="cuda")
    assert B.arcq_mx_gemv_epilogue(one[:0], None, w, s, bias=b, residual=one[:0, :8]).shape == (0, 8)
    assert B.arcq_mx_gemv_epilogue(one, None, w[:0], s[:0], bias=b[:0], activation=B.ACT_GELU).shape == (1, 0)
