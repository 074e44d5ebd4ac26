"""Activations where little is left of their argument: right to a few units of what is left, on every kernel that applies one."""
import numpy as np
import pytest
import torch

from oracle import layers as L
from paper_2601_07475_amd import binding as B

from test_gpu_epilogue import ACT, assert_within
from test_gpu_experts import call
from test_gpu_parity import dev, say


def off(act, v):
    """What a value of act(v) may be off by.  GELU of a negative v is its tail and nothing else."""
    if act == "gelu":
        return L.gelu_tail(v) * 20.0 * L.HALF + np.abs(L.activation(act, v)) * L.HALF + 2.0 ** -126
    return L.activation_slack(act, v)


def test_the_bound_sees_the_tail():
    """An erfc that is right to 1.5e-7 but not relatively, or GELU by 1 + erf in fp32, is beyond it."""
    v = np.linspace(-6.0, -3.0, 301)
    z = -v / np.sqrt(2.0)
    t = 1.0 / (1.0 + 0.3275911 * z)
    p = t * (0.254829592 + t * (-0.284496736 + t * (1.421413741 + t * (-1.453152027 + t * 1.061405429))))
    assert np.mean(np.abs(v * p * np.exp(-z * z) / 2.0 - L.activation("gelu", v)) > off("gelu", v)) > 0.9
    plain = torch.nn.functional.gelu(torch.from_numpy(v).float()).double().numpy()
    assert np.mean(np.abs(plain - L.activation("gelu", v)) > off("gelu", v)) > 0.5
    near = torch.nn.functional.gelu(torch.from_numpy(v)).numpy() * (1.0 + 15.0 * L.HALF)
    assert np.all(np.abs(near - L.activation("gelu", v)) <= off("gelu", v))


def arguments(n):
    v = np.concatenate([-np.linspace(0.01, 13.0, 2000), np.linspace(0.01, 13.0, 500), -np.exp(np.linspace(-15, 0, 300)), np.exp(np.linspace(-15, 0, 100)), [0.0, 20.0, -20.0, 60000.0, -60000.0]])
    v = np.random.default_rng(n).permutation(v.astype(np.float16))
    return np.resize(v, n)


# products: rows of each kernel, runs of K, tiles; sums of zeros, so that the activation's argument is the bias
SHAPES = [("gemv", 1, 3001, 64), ("gemv", 20, 1500, 64), ("gemv", 3, 500, 28672), ("mx_gemv", 4, 2999, 64), ("mx_gemv", 16, 1001, 8224), ("mx8", 2, 3000, 64), ("mx8", 300, 2904, 64),
          ("mx8", 300, 512, 14336), ("mx8", 15, 112, 20640)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,M,N,K", SHAPES)
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_products(kind, M, N, K, act):
    say(f"{kind} {M}x{K}x{N} {act} of the bias")
    bias = arguments(N)
    block = 16 if kind == "gemv" else 32
    w = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda"), torch.full((N, K // block), 0x38 if kind == "gemv" else 127, dtype=torch.uint8, device="cuda")
    kw = {"bias": dev(bias), "activation": ACT[act], "out_dtype": torch.float32}
    if kind == "mx8":
        kw["workspace"] = torch.empty(max(B.arcq_mx8_gemm_workspace_size(M, N, K), 256), dtype=torch.uint8, device="cuda")
        y = B.arcq_mx8_gemm_epilogue(torch.zeros((M, K), dtype=torch.uint8, device="cuda"), torch.full((M, K // 32), 127, dtype=torch.uint8, device="cuda"), *w, **kw)
    else:
        x = torch.zeros((M, K), dtype=torch.float16, device="cuda")
        y = B.arcq_gemv_epilogue(x, None, *w, 1.0, **kw) if kind == "gemv" else B.arcq_mx_gemv_epilogue(x, None, *w, **kw)
    v = np.broadcast_to(bias.astype(np.float64), (M, N))
    assert_within(y, L.activation(act, v), off(act, v))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
@pytest.mark.parametrize("M,K,I", [(1, 256, 256), (4, 64, 160), (8, 256, 128), (16, 256, 128), (40, 64, 96)])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_experts(fmt, M, K, I, act):
    """g of one channel, u = 1, a feature of one channel between: y is the activation.  On top of its own bound: the products by u and the weight (exact here), 2^-23 of
    what is between the products and 2^-38 of the largest there, three roundings of the sum, its unit and the scale, and up to 16 zeros that are added."""
    say(f"moe {fmt} {M}x{K} {act} by itself")
    rng = np.random.default_rng(M + I)
    block = 32 if fmt == "mx" else 16
    x = np.zeros((M, K), dtype=np.float16)
    x[:, 0], x[:, 1] = arguments(M * 7)[:M] / np.float16(6.0) + np.float16(0.25), 1.0
    codes = np.zeros((1, 2 * I, K // 2), dtype=np.uint8)
    code = rng.integers(1, 8, I) | 8
    codes[0, :I, 0], codes[0, I:, 0] = code, 0x20
    one = 127 if fmt == "mx" else 0x38
    ts = None if fmt == "mx" else np.ones(1, dtype=np.float32)
    up = codes, np.full((1, 2 * I, K // block), one, dtype=np.uint8), ts
    down = np.zeros((1, I, I // 2), dtype=np.uint8), np.full((1, I, I // block), one, dtype=np.uint8), ts
    down[0][0, np.arange(I), np.arange(I) // 2] = np.where(np.arange(I) % 2, 0x20, 0x02)
    g = x[:, :1].astype(np.float64) * -np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])[code & 7]
    ids, w = np.zeros((M, 1), dtype=np.int32), np.ones((M, 1), dtype=np.float32)
    y = call(fmt, dev(x), None, ids, w, up, down, activation=ACT[act], out_dtype=torch.float32)
    want = L.activation(act, g)
    assert_within(y, want, off(act, g) + np.abs(want) * (2.0 ** -23 + 19 * L.HALF) + 2.0 ** -38 * np.abs(want).max(1, keepdims=True))
