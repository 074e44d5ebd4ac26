"""Whole layers on packed 4-bit weights, in float64 numpy.  Test infrastructure only.

activation   the four activations (and none), by their definitions
finish       what a product does behind its sums: act(sum + bias) + residual
route        the router of a mixture of experts: scores, the best experts of each token, their weights
experts      the experts' part: sum of weight (act(x G^T) * (x U^T)) D^T over a token's experts, + residual

finish and experts also return the bound that the roundings of an fp32 implementation leave: every product of length K is off by less than
mag (K / 16 + 64) 2^-23 (mag: the same sum of magnitudes), as for the plain products.
"""
import math

import numpy as np

from . import arcquant as A
from . import mxfp4 as MX

NAMES = ("none", "relu", "gelu", "gelu_tanh", "silu")
STEEPEST = 1.13             # largest slope of any of them (GELU's, at sqrt(2))
HALF = 2.0 ** -24           # half a step of fp32

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _sigmoid(t):
    e = np.exp(-np.abs(t))
    return np.where(t >= 0, 1.0, e) / (1.0 + e)


def activation(name, v):
    v = np.asarray(v, dtype=np.float64)
    if name == "none":
        return v
    if name == "relu":
        return np.maximum(v, 0.0)
    if name == "gelu":
        return v * _erfc(-v / math.sqrt(2.0)) / 2.0
    if name == "gelu_tanh":
        return v * _sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
    if name == "silu":
        return v * _sigmoid(v)
    raise ValueError(name)


def gelu_tail(v):
    """|v| Phi(-|v|)"""
    return np.abs(v) * _erfc(np.abs(v) / math.sqrt(2.0)) / 2.0


def activation_slack(name, v):
    """What evaluating it in fp32 may be off by at a v in fp32.
    silu, gelu_tanh: v / (1 + E), E = 2^(-t log2 e): the exponent's rounding and the constant's put 1.5 |t| half steps on E (tanh's t itself has four
    roundings: 4 |t| more), the exponential, the sum, the reciprocal and the product 2 + 1 + 2 + 1; where E overflows the result is 0.
    gelu: v less a tail of |v| / 2 erfc(|v| / sqrt(2)), each of which is within half a step, and the tail's value within 20: its argument t = 1 / (1 + p z) within 3 behind the sum's
    and z's roundings, 2 more by the reciprocal, times at most 3 (z = 0, where z's own error does not count: 9 in all), the polynomial's fit 1, its roundings 4, t 1, the
    exponential with what is put back on it 4, the products 1."""
    v = np.asarray(v, dtype=np.float64)
    if name in ("none", "relu"):
        return np.zeros_like(v)
    if name == "gelu":
        return gelu_tail(v) * 20.0 * HALF + np.abs(v) * HALF + 2.0 ** -126
    t = np.abs(v) if name == "silu" else 1.6 * (np.abs(v) + 0.044715 * np.abs(v) ** 3)
    out = np.abs(activation(name, v))
    return out * ((1.5 if name == "silu" else 5.5) * np.minimum(t, 200.0) + 6.0) * HALF + 2.0 ** -110


def sum_error(mag, K):
    return mag * (K / 16 + 64) * 2.0 ** -23


def middle_error(h):
    """What the values h [I] between the two products are off by on their way, whatever their size: three products in fp32 (four half steps), then two fp16
    numbers.  The first leaves at most 2^-11 of its value, which the second rounds at half a step of its own, 2^-12 of that: 2^-23 in all.  Both count in units
    that take the largest value of the row, or of some of its channels, to 2^13 at least, and fp16 has no steps below 2^-24, so half of one is 2^-38 of that value."""
    return h * (4 * HALF + 2.0 ** -23) + 2.0 ** -38 * h.max(initial=0.0)


def finish(total, mag, K, bias=None, act="none", residual=None):
    """total, mag: a product's sums and their magnitudes -> (y, how far an fp32 evaluation may be off, before y's own rounding)."""
    off = sum_error(mag, K)
    v = total
    if bias is not None:
        v = v + np.asarray(bias, dtype=np.float64)
        off = off + (np.abs(v) + off) * HALF
    off = STEEPEST * off * (act != "none") + off * (act == "none") + activation_slack(act, np.abs(v) + off)
    y = activation(act, v)
    if residual is not None:
        y = y + np.asarray(residual, dtype=np.float64)
        off = off + (np.abs(y) + off) * HALF
    return y, off


def route(x, router, top, bias=None, sigmoid=False, renormalize=False):
    """x [M, K], router [E, K] -> ids [M, top], weights float64 [M, top]."""
    logits = np.asarray(x, dtype=np.float64) @ np.asarray(router, dtype=np.float64).T
    if sigmoid:
        score = _sigmoid(logits)
    else:
        score = np.exp(logits - logits.max(1, keepdims=True))
        score /= score.sum(1, keepdims=True)
    rank = logits if bias is None else score + np.asarray(bias, dtype=np.float64)
    ids = np.argsort(-rank, axis=1, kind="stable")[:, :top]
    w = np.take_along_axis(score, ids, 1)
    return ids.astype(np.int32), w / w.sum(1, keepdims=True) if renormalize else w


def _weights(codes, scales, K, tensor_scale):
    w = MX.dequantize(codes, scales) if tensor_scale is None else A.dequantize(codes, scales, tensor_scale)
    return w[:, :K].astype(np.float64)


def experts(x, perm, ids, weights, up, down, act="silu", residual=None):
    """x fp16 [M, K]; up, down: (codes [E, rows, ...], scales, tensor scales [E] or None) -> (y float64 [M, N], bound as in finish)."""
    x = np.asarray(x).astype(np.float64)
    x = x if perm is None else x[:, np.asarray(perm)]
    M, K = x.shape
    E, N = down[0].shape[:2]
    I = up[0].shape[1] // 2
    y, off, mag = np.zeros((M, N)), np.zeros((M, N)), np.zeros((M, N))
    for m in range(M):
        for e, w in zip(ids[m], weights[m].astype(np.float64)):
            if e < 0 or e >= E:
                continue
            W = _weights(up[0][e], up[1][e], K, None if up[2] is None else up[2][e])
            D = _weights(down[0][e], down[1][e], I, None if down[2] is None else down[2][e])
            v, dv = W @ x[m], sum_error(np.abs(W) @ np.abs(x[m]), K)
            g, u, dg, du = v[:I], v[I:], dv[:I], dv[I:]
            a = activation(act, g)
            da = (STEEPEST if act != "none" else 1.0) * dg + activation_slack(act, np.abs(g) + dg)
            h = w * a * u
            dh = np.abs(w) * (da * (np.abs(u) + du) + np.abs(a) * du)
            dh = dh + middle_error(np.abs(h) + dh)
            y[m] += D @ h
            mag[m] += np.abs(D) @ (np.abs(h) + dh)
            off[m] += np.abs(D) @ dh
    off = off + sum_error(mag, I * ids.shape[1])
    if residual is not None:
        y = y + np.asarray(residual, dtype=np.float64)
        off = off + (np.abs(y) + off) * HALF
    return y, off
