"""MXFP8 activations against packed 4-bit weights, step by step, in numpy.  Test infrastructure only.

MXFP8 is the 8-bit block format that the paper compares its two 4-bit stages with (Section 3.4): g = 32 E4M3 elements (bias 7,
max 448, finite flavour) and one E8M0 scale (value 2^(byte - 127)) per block, no tensor scale.  Scale rule of the OCP Microscaling
specification: shared exponent = floor(log2(max |v|)) - 8 (8 is E4M3's largest exponent), elements round to nearest even
on the E4M3 grid and saturate at 448 (a block maximum in (448 X, 512 X) clips); an all-zero block has byte 127.
scale_rounding="up": X is the smallest power of two with max |v| <= 448 X.

The residual's addition rounds once to fp16; the norm is oracle.arcquant.rmsnorm.  Products are taken in float64 over the K primary
columns of the packed weights, whose S repeated columns belong to the 4-bit path alone.
"""
import numpy as np

from . import arcquant as A
from . import formats as F
from . import mxfp4 as MX

G = 32
EMAX_ELEM = 8     # largest exponent of E4M3 (448 = 1.75 * 2^8)
E4M3_MAX = 448.0


def e4m3_nearest(w):
    """float64 w -> nearest E4M3 value (ties to even, saturating), with the sign of w."""
    w = np.asarray(w, dtype=np.float64)
    a = np.minimum(np.abs(w), E4M3_MAX)
    _, e = np.frexp(a)                                  # a in [2^(e-1), 2^e)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)     # 3 mantissa bits; below 2^-6 the subnormals' step
    return np.copysign(np.rint(a / step) * step, w)


def e4m3_byte(v):
    """float64 values of the E4M3 grid -> bytes."""
    table = F.e4m3_decode(np.arange(0x7F, dtype=np.uint8)).astype(np.float64)
    at = np.searchsorted(table, np.abs(v))
    if not np.array_equal(table[at], np.abs(v)):
        raise ValueError("not on the grid")
    return (at.astype(np.uint8) | (np.signbit(v).astype(np.uint8) << 7)).astype(np.uint8)


def quantize_blocks(v, scale_rounding="nearest"):
    """v float [..., 32] finite -> (sbyte uint8 [...], codes uint8 [..., 32])."""
    if scale_rounding not in ("nearest", "up"):
        raise ValueError("scale_rounding must be 'nearest' or 'up'")
    v = np.asarray(v, dtype=np.float64)
    if not np.all(np.isfinite(v)):
        raise ValueError("non-finite input")
    amax = np.abs(v).max(axis=-1)
    _, e = np.frexp(amax)
    shared = np.where(amax > 0, e - 1 - EMAX_ELEM, 0)
    if scale_rounding == "up":
        shared = shared + ((amax > 0) & (amax > E4M3_MAX * np.ldexp(1.0, shared)))
    return (shared + 127).astype(np.uint8), e4m3_byte(e4m3_nearest(np.ldexp(v, -shared[..., None])))


def quantize_act(X, perm=None, scale_rounding="nearest"):
    """X fp16 [M, K] -> codes uint8 [M, K], scales uint8 [M, K / 32]."""
    X = np.asarray(X)
    assert X.dtype == np.float16 and X.ndim == 2 and X.shape[1] % G == 0
    M, K = X.shape
    Xp = X if perm is None else X[:, np.asarray(perm)]
    sb, codes = quantize_blocks(Xp.astype(np.float64).reshape(M, K // G, G), scale_rounding)
    return codes.reshape(M, K), sb


def add_rmsnorm_quantize_act(X, residual, gamma, eps, perm=None, scale_rounding="nearest"):
    """-> codes, scales, hidden (X itself without a residual)."""
    hidden = X if residual is None else (X.astype(np.float32) + residual.astype(np.float32)).astype(np.float16)
    codes, scales = quantize_act(A.rmsnorm(hidden, gamma, eps), perm, scale_rounding)
    return codes, scales, hidden


def dequantize(codes, scales):
    """float64 [M, K] (exact)."""
    codes = np.asarray(codes)
    v = F.e4m3_decode(codes & 0x7F).astype(np.float64)
    v = np.where(codes & 0x80, -v, v)
    M, K = v.shape
    return (v.reshape(M, K // G, G) * MX.e8m0_decode(scales)[..., None]).reshape(M, K)


def gemm(a_codes, a_scales, w_codes, w_scales):
    """Activations [M, K], weights packed [N, K + S] -> (Y float64 [M, N], the same of the magnitudes)."""
    a, w = dequantize(a_codes, a_scales), MX.dequantize(w_codes, w_scales)[:, :a_codes.shape[1]]
    return a @ w.T, np.abs(a) @ np.abs(w).T


def gemv(X, perm, w_codes, w_scales, w_tensor_scale=None):
    """fp16 rows, weights packed [N, K + S]: NVFP4 with its tensor scale, MXFP4 without -> (Y float64 [M, N], of the magnitudes)."""
    x = np.asarray(X).astype(np.float64)
    x = x if perm is None else x[:, np.asarray(perm)]
    w = MX.dequantize(w_codes, w_scales) if w_tensor_scale is None else A.dequantize(w_codes, w_scales, w_tensor_scale)
    w = w[:, :x.shape[1]].astype(np.float64)
    return x @ w.T, np.abs(x) @ np.abs(w).T


def aligned_loss(a_codes, a_scales, w_codes, w_scales):
    """Largest error, element by element, of products whose eight products of eight consecutive k are lined up at the largest of their
    exponent sums (an element's exponent, that of the smallest normal below it) and cut 13 bits below it: less than a unit there for each of
    seven others.  float64 [M, N]; for a few rows of activations (it looks at every product)."""
    K = a_codes.shape[1]
    mag = a_codes & 0x7F
    ea = np.where(mag == 0, -1000, np.maximum(mag >> 3, 1).astype(np.int64) - 7)
    ea = ea + np.repeat(a_scales.astype(np.int64) - 127, G, axis=1)
    c = MX.unpack_nibbles(w_codes)[:, :K] & 7
    ew = np.where(c == 0, -1000, np.maximum(c >> 1, 1).astype(np.int64) - 1)
    ew = ew + np.repeat(w_scales[:, :K // G].astype(np.int64) - 127, G, axis=1)
    out = np.zeros((a_codes.shape[0], w_codes.shape[0]))
    for k in range(0, K, 8):
        top = np.full(out.shape, -2000, dtype=np.int64)
        for i in range(k, k + 8):
            np.maximum(top, ea[:, i, None] + ew[None, :, i], out=top)
        out += np.where(top > -500, 7.0 * np.exp2(np.maximum(top, -500) - 13.0), 0.0)
    return out
