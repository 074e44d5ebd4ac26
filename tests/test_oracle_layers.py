"""The float64 statements of whole layers, against definitions written out element by element."""
import math

import numpy as np
import pytest
import torch

from oracle import arcquant as A
from oracle import layers as L
from oracle import mxfp4 as MX


def test_activations_are_what_torch_has():
    v = np.concatenate([np.linspace(-30, 30, 4001), [-1e4, 1e4, 0.0]])
    t = torch.from_numpy(v)
    F = torch.nn.functional
    for name, want in (("relu", F.relu(t)), ("gelu", F.gelu(t)), ("gelu_tanh", F.gelu(t, approximate="tanh")), ("silu", F.silu(t)), ("none", t)):
        assert np.allclose(L.activation(name, v), want.numpy(), rtol=1e-12, atol=1e-15), name


def test_steepest_slope():
    v = np.linspace(-20, 20, 400001)
    for name in L.NAMES[1:]:
        assert np.max(np.abs(np.diff(L.activation(name, v)) / np.diff(v))) < L.STEEPEST


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_route_by_hand(sigmoid, biased):
    rng = np.random.default_rng(1)
    x, r = rng.standard_normal((3, 16)).astype(np.float16), rng.standard_normal((5, 16)).astype(np.float16)
    bias = rng.standard_normal(5).astype(np.float32) if biased else None
    ids, w = L.route(x, r, 2, bias, sigmoid, True)
    for m in range(3):
        l = [sum(float(x[m, k]) * float(r[e, k]) for k in range(16)) for e in range(5)]
        s = [1 / (1 + math.exp(-v)) for v in l] if sigmoid else [math.exp(v) / sum(math.exp(u) for u in l) for v in l]
        order = sorted(range(5), key=lambda e: (-(s[e] + (float(bias[e]) if biased else 0.0)), e))[:2]
        assert list(ids[m]) == order
        assert np.allclose(w[m], [s[e] / sum(s[i] for i in order) for e in order], rtol=1e-12)


def test_route_ties_go_to_the_lowest_index():
    x = np.ones((1, 8), dtype=np.float16)
    r = np.zeros((6, 8), dtype=np.float16)
    r[[1, 4]] = 1.0
    ids, w = L.route(x, r, 4)
    assert ids.tolist() == [[1, 4, 0, 2]] and w[0, 0] == w[0, 1] and w[0, 2] == w[0, 3]


@pytest.mark.parametrize("fmt", ["nvfp4", "mx"])
def test_experts_by_hand(fmt):
    rng = np.random.default_rng(2)
    M, K, I, N, E = 3, 32, 32, 4, 2
    x = rng.standard_normal((M, K)).astype(np.float16)
    perm = rng.permutation(K)
    U, D = rng.standard_normal((E, 2 * I, K)).astype(np.float16), rng.standard_normal((E, N, I)).astype(np.float16)

    def pack(W, perm):
        if fmt == "mx":
            parts = [MX.pack_weight(w, perm, 32) for w in W]
            return np.stack([p[0] for p in parts]), np.stack([p[1] for p in parts]), None
        parts = [A.pack_weight(w, perm, 16, np.float32(0.001)) for w in W]
        return np.stack([p[0] for p in parts]), np.stack([p[1] for p in parts]), np.full(E, 0.001, dtype=np.float32)

    up, down = pack(U, perm), pack(D, np.arange(I))
    ids = np.array([[1, 0], [-1, 1], [2, -1]], dtype=np.int32)
    w = rng.random((M, 2)).astype(np.float32)
    res = rng.standard_normal((M, N)).astype(np.float16)
    y, off = L.experts(x, perm, ids, w, up, down, "relu", res)
    deq = (lambda c, s, ts: MX.dequantize(c, s)) if fmt == "mx" else A.dequantize
    for m in range(M):
        for n in range(N):
            total = float(res[m, n])
            for j in range(2):
                e = ids[m, j]
                if not 0 <= e < E:
                    continue
                Wu, Wd = (deq(p[0][e], p[1][e], None if p[2] is None else p[2][e]) for p in (up, down))
                for i in range(I):
                    g = sum(float(Wu[i, k]) * float(x[m, perm[k]]) for k in range(K))
                    u = sum(float(Wu[I + i, k]) * float(x[m, perm[k]]) for k in range(K))
                    total += float(w[m, j]) * max(g, 0.0) * u * float(Wd[n, i])
            assert abs(total - y[m, n]) <= 1e-9 * (1 + abs(total))
    assert (off >= 0).all() and np.array_equal(y[2], res[2].astype(np.float64))


def test_bounds_hold_for_float32():
    """An fp32 evaluation in torch lies within them."""
    rng = np.random.default_rng(3)
    M, K, N = 5, 256, 40
    a, w = rng.standard_normal((M, K)).astype(np.float16), (rng.standard_normal((N, K)) * 0.5).astype(np.float16)
    b, r = rng.standard_normal(N).astype(np.float16), rng.standard_normal((M, N)).astype(np.float32)
    total, mag = a.astype(np.float64) @ w.astype(np.float64).T, np.abs(a).astype(np.float64) @ np.abs(w).astype(np.float64).T
    F = torch.nn.functional
    acts = {"none": lambda t: t, "relu": F.relu, "gelu": F.gelu, "gelu_tanh": lambda t: F.gelu(t, approximate="tanh"), "silu": F.silu}
    for name, act in acts.items():
        y, off = L.finish(total, mag, K, b, name, r)
        got = act(torch.from_numpy(a).float() @ torch.from_numpy(w).float().T + torch.from_numpy(b).float()) + torch.from_numpy(r)
        assert (np.abs(got.double().numpy() - y) <= off + np.abs(y) * L.HALF).all(), name
