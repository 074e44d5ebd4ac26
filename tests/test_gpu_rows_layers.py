"""The operators with 8- and 16-bit activations together, as a program uses them: a layer's projections behind their norms, a decode
step on the same packed weights, on other streams and in captured graphs."""
import numpy as np
import pytest
import torch

from oracle import arcquant as A
from oracle import mxfp4 as MX
from oracle import mxfp8 as M8
from paper_2601_07475_amd import binding as B
from paper_2601_07475_amd import workloads as wk

from test_gpu_graph import _replays_match
from test_gpu_mx8 import assert_fp16_product, assert_product
from test_gpu_parity import assert_same_bytes, dev, say

pytestmark = pytest.mark.gpu

D, FF, S = 512, 1376, 32        # hidden and inner size of a small model, outlier columns


def model(seed):
    rng = np.random.default_rng(seed)
    up, down = ((rng.standard_normal(s) * 0.05).astype(np.float16) for s in ((FF, D), (D, FF)))
    p_up, p_down = (rng.permutation(n).astype(np.int32) for n in (D, FF))
    gamma = (1 + 0.1 * rng.standard_normal(D)).astype(np.float16)
    return dict(gamma=gamma, p_up=p_up, p_down=p_down, up=MX.pack_weight(up, p_up, S), down=MX.pack_weight(down, p_down, S),
                up_nv=A.pack_weight(up, p_up, S, wk.tensor_scale(up)), ts=wk.tensor_scale(up))


@pytest.mark.parametrize("M", [1, 19, 300])
def test_mlp_with_8_bit_activations(M):
    """hidden -> norm -> up -> quantize -> down -> next layer's addition and norm, in place; each step against the oracle on what it got."""
    say(f"MLP with MXFP8 activations, M={M}")
    m = model(1)
    rng = np.random.default_rng(2)
    x, r = (dev((rng.standard_normal((M, D)) * 2).astype(np.float16)) for _ in range(2))
    g, pu, pd = dev(m["gamma"]), dev(m["p_up"]), dev(m["p_down"])
    up, down = [dev(t) for t in m["up"]], [dev(t) for t in m["down"]]
    rn = r.cpu().numpy()
    c, s, h = B.arcq_mx8_add_rmsnorm_quantize_act(x, r, g, 1e-5, pu, hidden=r)
    wc, wsc, wh = M8.add_rmsnorm_quantize_act(x.cpu().numpy(), rn, m["gamma"], 1e-5, m["p_up"])
    assert_same_bytes(c.cpu().numpy(), wc, "codes")
    assert_same_bytes(s.cpu().numpy(), wsc, "scales")
    assert np.array_equal(r.cpu().numpy(), wh)
    y = B.arcq_mx8_gemm(c, s, *up)
    assert_fp16_product(y, wc, wsc, *m["up"], *M8.gemm(wc, wsc, *m["up"]))
    c, s = B.arcq_mx8_quantize_act(y, pd)
    wc, wsc = M8.quantize_act(y.cpu().numpy(), m["p_down"])
    assert_same_bytes(c.cpu().numpy(), wc, "codes")
    assert_same_bytes(s.cpu().numpy(), wsc, "scales")
    z = B.arcq_mx8_gemm(c, s, *down)
    assert_fp16_product(z, wc, wsc, *m["down"], *M8.gemm(wc, wsc, *m["down"]))
    zn = z.cpu().numpy()
    c, s, h = B.arcq_mx8_add_rmsnorm_quantize_act(z, r, g, 1e-5, pu, hidden=z)
    wc, wsc, wh = M8.add_rmsnorm_quantize_act(zn, wh, m["gamma"], 1e-5, m["p_up"])
    assert_same_bytes(c.cpu().numpy(), wc, "codes")
    assert_same_bytes(s.cpu().numpy(), wsc, "scales")
    assert np.array_equal(z.cpu().numpy(), wh)


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_decode_step_on_the_weights_of_the_4_bit_path(fmt):
    """A prompt through the 4-bit GEMM and the next token through fp16 rows, on the same packed weights."""
    say(f"4-bit prompt, fp16 decode, {fmt}")
    m = model(3)
    X = wk.activations(wk.Workload("t", 40, D, FF, S, 5, "loguniform20_100", 0.05, 5))
    x, pu = dev(X), dev(m["p_up"])
    if fmt == "mx":
        w = [dev(t) for t in m["up"]]
        prompt = B.arcq_mx_gemm(*B.arcq_mx_quantize_act(x, pu, S), *w, out_dtype=torch.float32)
        token = B.arcq_mx_gemv(x[-1:], pu, *w, out_dtype=torch.float32)
        want, mag = M8.gemv(X[-1:], m["p_up"], *m["up"])
    else:
        w, ts = [dev(t) for t in m["up_nv"]], float(m["ts"])
        sx = float(wk.tensor_scale(X))
        prompt = B.arcq_gemm(*B.arcq_quantize_act(x, pu, S, sx), sx, *w, ts, out_dtype=torch.float32)
        token = B.arcq_gemv(x[-1:], pu, *w, ts, out_dtype=torch.float32)
        want, mag = M8.gemv(X[-1:], m["p_up"], *m["up_nv"], m["ts"])
    assert_product(token, want, mag, D)
    # the prompt's last row is the same product with quantized activations
    a, b = prompt[-1].double(), token[0].double()
    assert float((a - b).norm() / b.norm()) < 0.25


def test_steps_in_a_captured_graph():
    say("graph capture of the 8-bit layer and the fp16 decode step")
    m, M = model(4), 150
    g, pu, pd = dev(m["gamma"]), dev(m["p_up"]), dev(m["p_down"])
    up, down, nv = ([dev(t) for t in m[k]] for k in ("up", "down", "up_nv"))
    ins = [(torch.randn((M, D), device="cuda") * 2).half() for _ in range(4)]
    x, r = ins[0].clone(), ins[1].clone()
    h, y, z = (torch.empty(s, dtype=torch.float16, device="cuda") for s in ((M, D), (M, FF), (M, D)))
    v, v2 = (torch.empty((7, FF), dtype=torch.float32, device="cuda") for _ in range(2))
    c1, s1, c2, s2 = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in ((M, D), (M, D // 32), (M, FF), (M, FF // 32)))
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def step():
        B.arcq_mx8_add_rmsnorm_quantize_act(x, r, g, 1e-5, pu, hidden=h, codes=c1, scales=s1)
        B.arcq_mx8_gemm(c1, s1, *up, y=y, workspace=ws)
        B.arcq_mx8_quantize_act(y, pd, codes=c2, scales=s2)
        B.arcq_mx8_gemm(c2, s2, *down, y=z, workspace=ws)
        B.arcq_mx_gemv(x[:7], pu, *up, y=v, workspace=ws)
        B.arcq_gemv(x[:7], pu, *nv, float(m["ts"]), y=v2, workspace=ws)

    _replays_match(step, step, [h, y, z, v, v2, c1, s1, c2, s2], lambda i: x.copy_(ins[i]))


def test_two_streams_at_once():
    """The same calls on two streams, each with a workspace of its own, give what one after the other gives."""
    say("two streams")
    m = model(6)
    pu, up = dev(m["p_up"]), [dev(t) for t in m["up"]]
    xs = [(torch.randn((33, D), device="cuda") * 2).half() for _ in range(2)]

    def step(x, ws):
        c, s = B.arcq_mx8_quantize_act(x, pu)
        return B.arcq_mx8_gemm(c, s, *up, workspace=ws), B.arcq_mx_gemv(x, pu, *up, workspace=ws)

    spaces = [torch.empty(1 << 22, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = [step(x, w) for x, w in zip(xs, spaces)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for x, w, st in zip(xs, spaces, streams):
            with torch.cuda.stream(st):
                got.append(step(x, w))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for p, q in zip(got, want) for a, b in zip(p, q))


def test_runs_of_k_in_a_captured_graph():
    """Few features over many channels: partial results in the workspace and a second launch, replayed."""
    say("graph capture of products with K in several runs")
    M, N, K = 9, 200, 12320
    assert B.arcq_mx8_gemm_route(M, N, K, 0, torch.float16, True)[3] > 1 and B.arcq_mx_gemv_workspace_size(M, N, K, False) > 0
    gen = torch.Generator(device="cuda").manual_seed(3)
    ins = [torch.randn((M, K), device="cuda", generator=gen).half() for _ in range(4)]
    x, perm = ins[0].clone(), torch.randperm(K, device="cuda", generator=gen).int()
    wc = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    mx, nv = (torch.randint(lo, hi, (N, K // b), dtype=torch.uint8, device="cuda", generator=gen) for lo, hi, b in ((115, 122, 32), (40, 60, 16)))
    c, s = torch.empty((M, K), dtype=torch.uint8, device="cuda"), torch.empty((M, K // 32), dtype=torch.uint8, device="cuda")
    ys = [torch.empty((M, N), dtype=t, device="cuda") for t in (torch.float16, torch.float32, torch.float32)]
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def step():
        B.arcq_mx8_quantize_act(x, perm, codes=c, scales=s)
        B.arcq_mx8_gemm(c, s, wc, mx, y=ys[0], workspace=ws)
        B.arcq_mx_gemv(x, perm, wc, mx, y=ys[1], workspace=ws)
        B.arcq_gemv(x, None, wc, nv, 0.5, y=ys[2], workspace=ws)

    _replays_match(step, step, [c, s, *ys], lambda i: x.copy_(ins[i]))


def test_weights_past_32_bit_offsets():
    """131200 features over 65536 channels, 4.3 GB of codes: the last rows of weights against the oracle."""
    say("weights of more than 4 GiB")
    N, K, M = 131200, 65536, 2
    gen = torch.Generator(device="cuda").manual_seed(4)
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    mx, nv = (torch.randint(lo, hi, (N, K // b), dtype=torch.uint8, device="cuda", generator=gen) for lo, hi, b in ((115, 122, 32), (40, 60, 16)))
    x = torch.randn((M, K), device="cuda", generator=gen).half()
    c, s = B.arcq_mx8_quantize_act(x)
    got = [B.arcq_gemv(x, None, codes, nv, 0.5, out_dtype=torch.float32), B.arcq_mx_gemv(x, None, codes, mx, out_dtype=torch.float32),
           B.arcq_mx8_gemm(c, s, codes, mx, out_dtype=torch.float32)]
    X, cn, sn = x.cpu().numpy(), c.cpu().numpy(), s.cpu().numpy()
    for rows in (slice(0, 20), slice(N - 20, N)):
        w, wm, wn = codes[rows].cpu().numpy(), mx[rows].cpu().numpy(), nv[rows].cpu().numpy()
        for y, (want, mag) in zip(got, (M8.gemv(X, None, w, wn, np.float32(0.5)), M8.gemv(X, None, w, wm), M8.gemm(cn, sn, w, wm))):
            assert_product(y[:, rows], want, mag, K)


def test_rows_past_32_bit_offsets():
    """65600 rows of 65536 channels, 4.3 GB of MXFP8 codes and 8.6 GB of fp16: quantized, normalised and multiplied; the last rows against the oracle."""
    say("activations of more than 4 GiB")
    M, N, K = 65600, 40, 65536
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((M, K), dtype=torch.float16, device="cuda")
    for r in range(0, M, 4100):
        x[r:r + 4100] = torch.randn((4100, K), device="cuda", generator=gen)
    w = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda", generator=gen)
    mx = torch.randint(115, 122, (N, K // 32), dtype=torch.uint8, device="cuda", generator=gen)
    gamma = (1 + 0.1 * torch.randn(K, device="cuda", generator=gen)).half()
    c, s = B.arcq_mx8_quantize_act(x)
    nc, ns, _ = B.arcq_mx8_add_rmsnorm_quantize_act(x, None, gamma, 1e-5)
    y = B.arcq_mx8_gemm(c, s, w, mx, out_dtype=torch.float32)
    v = B.arcq_mx_gemv(x, None, w, mx, out_dtype=torch.float32)
    wn, mn = w.cpu().numpy(), mx.cpu().numpy()
    for rows in (slice(0, 3), slice(65500, 65510), slice(65534, 65538), slice(M - 3, M)):
        X, cn, sn = x[rows].cpu().numpy(), c[rows].cpu().numpy(), s[rows].cpu().numpy()
        for got, want in zip((cn, sn), M8.quantize_act(X)):
            assert_same_bytes(got, want, "quantized")
        for got, want in zip((nc[rows].cpu().numpy(), ns[rows].cpu().numpy()), M8.add_rmsnorm_quantize_act(X, None, gamma.cpu().numpy(), 1e-5)[:2]):
            assert_same_bytes(got, want, "normalised")
        assert_product(y[rows], *M8.gemm(cn, sn, wn, mn), K)
        assert_product(v[rows], *M8.gemv(X, None, wn, mn), K)


def test_prepared_calls():
    """Arguments checked and converted once: captured and replayed, the plain calls' results."""
    say("prepared calls")
    m, M = model(9), 21
    g, pu = dev(m["gamma"]), dev(m["p_up"])
    up, nv, ts = [dev(t) for t in m["up"]], [dev(t) for t in m["up_nv"]], float(m["ts"])
    ins = [(torch.randn((M, D), device="cuda") * 2).half() for _ in range(4)]
    x, r = ins[0].clone(), ins[1].clone()
    h, y = torch.empty((M, D), dtype=torch.float16, device="cuda"), torch.empty((M, FF), dtype=torch.float16, device="cuda")
    v, w = (torch.empty((M, FF), dtype=torch.float32, device="cuda") for _ in range(2))
    c1, s1, c2, s2 = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in ((M, D), (M, D // 32), (M, D), (M, D // 32)))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def capture():
        B.prepare_mx8_add_rmsnorm_quantize_act(x, r, g, 1e-5, pu, 0, h, c1, s1)()
        B.prepare_mx8_quantize_act(x, None, B.SCALE_ROUND_UP, c2, s2)()
        B.prepare_mx8_gemm(c1, s1, *up, y, ws)()
        B.prepare_gemv(x, pu, *nv, ts, v, ws)()
        B.prepare_mx_gemv(x, pu, *up, w, ws)()

    def eager():
        B.arcq_mx8_add_rmsnorm_quantize_act(x, r, g, 1e-5, pu, hidden=h, codes=c1, scales=s1)
        B.arcq_mx8_quantize_act(x, None, B.SCALE_ROUND_UP, c2, s2)
        B.arcq_mx8_gemm(c1, s1, *up, y=y, workspace=ws)
        B.arcq_gemv(x, pu, *nv, ts, y=v, workspace=ws)
        B.arcq_mx_gemv(x, pu, *up, y=w, workspace=ws)

    _replays_match(capture, eager, [h, y, v, w, c1, s1, c2, s2], lambda i: x.copy_(ins[i]))
    with pytest.raises(B.ArcqError):
        B.prepare_mx_gemv(x, pu, *up, w)()          # 21 rows are reordered into a workspace
    for hidden, codes in ((None, c1), (h, None)):
        with pytest.raises(AssertionError):
            B.prepare_mx8_add_rmsnorm_quantize_act(x, r, g, 1e-5, pu, 0, hidden, codes, s1)
    with pytest.raises(AssertionError):
        B.prepare_mx8_quantize_act(x, None, 0, c2, None)
