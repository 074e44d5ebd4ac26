"""No-GPU checks of the entry points with 8-bit and 16-bit activations: bad arguments are rejected before any HIP call."""
import ctypes
import os

import pytest

from paper_2601_07475_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libarcq.so not built")

P = ctypes.c_void_p                   # never dereferenced: every call below fails validation first, or has nothing to do
FAKE, OFF2, OFF4, OFF8, OFF16 = P(0x10000), P(0x10002), P(0x10004), P(0x10008), P(0x10010)
BIG = B.MAX_K + 32


def last():
    return B.lib().arcq_last_error().decode()


def quantize(x=FAKE, M=4, K=512, ldx=512, perm=FAKE, flags=0, codes=FAKE, scales=FAKE):
    return B.lib().arcq_mx8_quantize_act(x, M, K, ldx, perm, flags, codes, scales, None)


def norm(x=FAKE, M=4, K=512, ldx=512, residual=FAKE, ldr=512, hidden=P(0x40000), ldh=512, gamma=FAKE, eps=1e-5, perm=FAKE, flags=0,
         codes=FAKE, scales=FAKE):
    return B.lib().arcq_mx8_add_rmsnorm_quantize_act(x, M, K, ldx, residual, ldr, hidden, ldh, gamma, eps, perm, flags, codes, scales, None)


def gemm(a=FAKE, asc=FAKE, w=FAKE, wsc=FAKE, M=4, N=8, K=64, S=32, y=FAKE, dt=0, ldy=8, ws=None, wsb=0):
    return B.lib().arcq_mx8_gemm(a, asc, w, wsc, M, N, K, S, y, dt, ldy, ws, wsb, None)


def gemv(x=FAKE, M=2, K=64, ldx=64, perm=None, w=FAKE, wsc=FAKE, ts=1.0, N=8, S=32, y=FAKE, dt=0, ldy=8, ws=None, wsb=0):
    return B.lib().arcq_gemv(x, M, K, ldx, perm, w, wsc, ts, N, S, y, dt, ldy, ws, wsb, None)


def mx_gemv(x=FAKE, M=2, K=64, ldx=64, perm=None, w=FAKE, wsc=FAKE, N=8, S=32, y=FAKE, dt=0, ldy=8, ws=None, wsb=0):
    return B.lib().arcq_mx_gemv(x, M, K, ldx, perm, w, wsc, N, S, y, dt, ldy, ws, wsb, None)


def test_mx8_packed_sizes():
    assert B.arcq_mx8_packed_sizes(16, 512) == (16 * 512, 16 * 16)
    assert B.arcq_mx8_packed_sizes(0, 32) == (0, 0)
    assert B.arcq_mx8_packed_sizes(1 << 20, 65536) == (1 << 36, 1 << 31)
    for rows, K in ((4, 0), (4, 16), (4, 48), (4, BIG), (-1, 64)):
        with pytest.raises(B.ArcqError) as e:
            B.arcq_mx8_packed_sizes(rows, K)
        assert e.value.status == B.BAD_SHAPE


def test_mx8_quantizer_argument_errors():
    assert quantize(K=48, ldx=48) == B.BAD_SHAPE and quantize(K=BIG, ldx=BIG) == B.BAD_SHAPE and quantize(K=0) == B.BAD_SHAPE
    assert quantize(M=-1) == B.BAD_SHAPE and quantize(M=1 << 31) == B.BAD_SHAPE
    assert quantize(ldx=504) == B.BAD_SHAPE and "leading dimension" in last()
    for flags in (B.LAYOUT_INTERLEAVED, B.RMSNORM_EXACT_SUM, 8):
        assert quantize(flags=flags) == B.INVALID_ARG
    assert quantize(x=None) == quantize(codes=None) == quantize(scales=None) == B.INVALID_ARG
    assert quantize(x=OFF8) == B.BAD_ALIGN and quantize(ldx=516) == B.BAD_ALIGN
    assert quantize(codes=OFF8) == B.BAD_ALIGN and "codes" in last()
    assert quantize(perm=OFF4) == B.BAD_ALIGN and "perm" in last()
    assert quantize(M=0, x=None, perm=None, codes=None, scales=None) == B.OK and last() == ""


def test_mx8_norm_argument_errors():
    assert norm(K=48) == B.BAD_SHAPE and norm(M=-1) == B.BAD_SHAPE and norm(ldx=504) == B.BAD_SHAPE
    assert norm(ldr=504) == B.BAD_SHAPE and "residual" in last()
    assert norm(ldh=504) == B.BAD_SHAPE and "hidden" in last()
    for eps in (-1e-6, float("inf"), float("nan")):
        assert norm(eps=eps) == B.INVALID_ARG and "eps" in last()
    for flags in (B.LAYOUT_INTERLEAVED, 8):
        assert norm(flags=flags) == B.INVALID_ARG
    # the sum has to go somewhere, and without a residual there is none
    assert norm(hidden=None) == B.INVALID_ARG and norm(residual=None) == B.INVALID_ARG and "together" in last()
    for null in ("x", "gamma", "codes", "scales"):
        assert norm(**{null: None}) == B.INVALID_ARG
    for off in ("x", "residual", "hidden", "gamma", "codes", "perm"):
        assert norm(**{off: OFF8}) == B.BAD_ALIGN, off
    assert norm(ldx=516) == norm(ldr=516) == norm(ldh=516) == B.BAD_ALIGN
    # in place over an input of another pitch: rows of the sum would lie over rows still to be read
    assert norm(hidden=FAKE, residual=P(0x80000), ldh=520) == B.BAD_SHAPE and norm(hidden=FAKE, x=P(0x80000), ldh=520) == B.BAD_SHAPE
    assert norm(M=0, x=None, residual=None, hidden=None, gamma=None, perm=None, codes=None, scales=None) == B.OK


def test_mx8_gemm_argument_errors():
    assert gemm(K=0) == gemm(K=48) == gemm(K=BIG) == B.BAD_SHAPE
    assert gemm(S=16) == gemm(S=96) == gemm(S=-32) == B.BAD_SHAPE
    assert gemm(M=-1) == gemm(N=-1) == gemm(M=1 << 31) == B.BAD_SHAPE and gemm(ldy=7) == B.BAD_SHAPE
    assert gemm(dt=2) == B.INVALID_ARG
    for null in ("a", "asc", "w", "wsc", "y"):
        assert gemm(**{null: None}) == B.INVALID_ARG
    assert gemm(a=OFF8) == B.BAD_ALIGN and gemm(w=OFF8) == B.BAD_ALIGN and gemm(y=OFF2) == B.BAD_ALIGN
    assert gemm(ws=OFF16, wsb=1 << 30) == B.BAD_ALIGN and "workspace" in last()
    assert gemm(M=0, a=None, asc=None, y=None) == B.OK and gemm(N=0, w=None, wsc=None, y=None, ldy=0) == B.OK
    n = ctypes.c_size_t(9)
    assert B.lib().arcq_mx8_gemm_workspace_size(4, 8, 48, ctypes.byref(n)) == B.BAD_SHAPE
    assert B.lib().arcq_mx8_gemm_workspace_size(4, 8, 64, None) == B.INVALID_ARG
    assert B.arcq_mx8_gemm_workspace_size(0, 8, 64) == 0 and B.arcq_mx8_gemm_workspace_size(4, 0, 64) == 0


@pytest.mark.parametrize("call,block", [(gemv, 16), (mx_gemv, 32)])
def test_gemv_argument_errors(call, block):
    assert call(K=block // 2) == call(K=block + block // 2, ldx=64) == call(K=BIG, ldx=BIG) == call(K=0) == B.BAD_SHAPE
    assert call(S=block // 2) == call(S=96) == call(S=-block) == B.BAD_SHAPE
    assert call(M=-1) == call(N=-1) == call(M=1 << 31) == call(N=1 << 31) == B.BAD_SHAPE
    assert call(ldx=56) == B.BAD_SHAPE and call(ldy=7) == B.BAD_SHAPE
    assert call(dt=2) == B.INVALID_ARG
    for null in ("x", "w", "wsc", "y"):
        assert call(**{null: None}) == B.INVALID_ARG
    assert call(x=OFF8) == call(ldx=68) == call(w=OFF4) == call(y=OFF2) == call(perm=OFF4, ws=FAKE, wsb=1 << 20) == B.BAD_ALIGN
    assert call(M=0, x=None, y=None) == B.OK and call(N=0, w=None, wsc=None, y=None, ldy=0) == B.OK
    size = B.arcq_gemv_workspace_size if block == 16 else B.arcq_mx_gemv_workspace_size
    for M, N, K in ((2, 8, 64), (64, 4096, 28672)):
        need = size(M, N, K, True)
        if need:
            short = dict(M=M, N=N, K=K, S=0, ldx=K, ldy=N, perm=FAKE)
            assert call(**short) == B.WORKSPACE_TOO_SMALL
            assert call(**short, ws=FAKE, wsb=need - 1) == B.WORKSPACE_TOO_SMALL and "workspace" in last()
            assert call(**short, ws=OFF16, wsb=need) == B.BAD_ALIGN
    assert size(64, 4096, 28672, True) > 0
    assert size(0, 8, 64, True) == size(8, 0, 64, True) == 0
    with pytest.raises(B.ArcqError):
        size(4, 8, block // 2, False)


@pytest.mark.parametrize("call,block", [(gemv, 16), (mx_gemv, 32)])
def test_gemv_workspace_of_few_features(call, block):
    """K in several runs where features alone do not fill the chip: partial results, with and without an order of the channels."""
    size = B.arcq_gemv_workspace_size if block == 16 else B.arcq_mx_gemv_workspace_size
    M, N, K = 3, 512, 28672
    need = size(M, N, K, False)
    assert need > 0 and need % (M * N * 4) == 0 and size(M, N, K, True) == need + M * K * 2
    short = dict(M=M, N=N, K=K, S=0, ldx=K, ldy=N)
    assert call(**short) == call(**short, ws=FAKE, wsb=need - 1) == B.WORKSPACE_TOO_SMALL
    assert call(**short, ws=OFF16, wsb=need) == B.BAD_ALIGN
    assert size(M, 64, 512, False) == size(M, 65536, 4096, False) == 0


def test_gemv_tensor_scale():
    for bad in (0.0, -1.0, float("inf"), float("nan"), 2.0 ** -70, 2.0 ** 70):
        assert gemv(ts=bad) == B.INVALID_ARG
