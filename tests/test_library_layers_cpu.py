"""No-GPU checks of the products with an epilogue, of the router and of the experts: bad arguments are rejected before any HIP call."""
import ctypes
import os

import pytest

from paper_2601_07475_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libarcq.so not built")

P = ctypes.c_void_p                   # never dereferenced: every call below fails validation first, or has nothing to do
FAKE, OFF1, OFF2, OFF4, OFF8, OFF16 = P(0x10000), P(0x10001), P(0x10002), P(0x10004), P(0x10008), P(0x10010)
BIG = B.MAX_K + 32


def last():
    return B.lib().arcq_last_error().decode()


def mx8(a=FAKE, asc=FAKE, w=FAKE, wsc=FAKE, M=4, N=8, K=64, S=32, bias=FAKE, act=4, res=FAKE, ldr=8, y=P(0x40000), dt=0, ldy=8, ws=None, wsb=0):
    return B.lib().arcq_mx8_gemm_epilogue(a, asc, w, wsc, M, N, K, S, bias, act, res, ldr, y, dt, ldy, ws, wsb, None)


def gemv(x=FAKE, M=2, K=64, ldx=64, perm=None, w=FAKE, wsc=FAKE, ts=1.0, N=8, S=32, bias=FAKE, act=4, res=FAKE, ldr=8, y=P(0x40000), dt=0, ldy=8, ws=None, wsb=0):
    return B.lib().arcq_gemv_epilogue(x, M, K, ldx, perm, w, wsc, ts, N, S, bias, act, res, ldr, y, dt, ldy, ws, wsb, None)


def mx_gemv(x=FAKE, M=2, K=64, ldx=64, perm=None, w=FAKE, wsc=FAKE, N=8, S=32, bias=FAKE, act=4, res=FAKE, ldr=8, y=P(0x40000), dt=0, ldy=8, ws=None, wsb=0):
    return B.lib().arcq_mx_gemv_epilogue(x, M, K, ldx, perm, w, wsc, N, S, bias, act, res, ldr, y, dt, ldy, ws, wsb, None)


def route(x=FAKE, M=3, K=64, ldx=64, r=FAKE, ldr=64, E=8, bias=None, top=2, flags=0, ids=FAKE, w=FAKE, ws=FAKE, wsb=1 << 30):
    return B.lib().arcq_moe_route(x, M, K, ldx, r, ldr, E, bias, top, flags, ids, w, ws, wsb, None)


def moe(x=FAKE, M=3, K=64, ldx=64, perm=None, ids=FAKE, w=FAKE, top=2, E=8, uc=FAKE, us=FAKE, ut=FAKE, I=64, S=32, dc=FAKE, ds=FAKE, dt_=FAKE, N=8, S2=0, act=4,
        res=FAKE, ldr=8, y=P(0x40000), dt=0, ldy=8, ws=FAKE, wsb=1 << 30):
    return B.lib().arcq_moe(x, M, K, ldx, perm, ids, w, top, E, uc, us, ut, I, S, dc, ds, dt_, N, S2, act, res, ldr, y, dt, ldy, ws, wsb, None)


def mx_moe(x=FAKE, M=3, K=64, ldx=64, perm=None, ids=FAKE, w=FAKE, top=2, E=8, uc=FAKE, us=FAKE, I=64, S=32, dc=FAKE, ds=FAKE, N=8, S2=0, act=4,
           res=FAKE, ldr=8, y=P(0x40000), dt=0, ldy=8, ws=FAKE, wsb=1 << 30):
    return B.lib().arcq_mx_moe(x, M, K, ldx, perm, ids, w, top, E, uc, us, I, S, dc, ds, N, S2, act, res, ldr, y, dt, ldy, ws, wsb, None)


@pytest.mark.parametrize("call", [mx8, gemv, mx_gemv, moe, mx_moe])
def test_what_follows_a_product(call):
    for act in (-1, 5, 100):
        assert call(act=act) == B.INVALID_ARG and "activation" in last()
    assert call(ldr=7) == B.BAD_SHAPE and "residual" in last()
    assert call(res=OFF2) == B.BAD_ALIGN and "residual" in last()
    # in place over a residual of another pitch: rows of y would lie over rows still to be read
    assert call(res=P(0x40000), ldr=16) == B.BAD_SHAPE and "in place" in last()
    assert call(M=0, x=None, y=None, res=None) == B.OK if call not in (mx8,) else call(M=0, a=None, y=None, res=None) == B.OK
    assert call(N=0, y=None, ldy=0, ldr=0) == B.OK
    assert call(y=None) == B.INVALID_ARG and call(ldy=7) == B.BAD_SHAPE and call(dt=2) == B.INVALID_ARG and call(y=OFF2) == B.BAD_ALIGN
    if call not in (moe, mx_moe):
        assert call(bias=OFF1) == B.BAD_ALIGN and "bias" in last()


@pytest.mark.parametrize("call", [mx8, gemv, mx_gemv])
def test_products_check_what_the_plain_calls_check(call):
    assert call(K=0) == call(K=40) == call(S=8) == call(M=-1) == call(N=-1) == B.BAD_SHAPE
    assert call(w=None) == call(wsc=None) == B.INVALID_ARG and call(w=OFF4) == B.BAD_ALIGN
    if call is gemv:
        assert call(ts=float("nan")) == B.INVALID_ARG
    if call is not mx8:
        need = B.arcq_gemv_workspace_size(64, 4096, 28672, True)
        short = dict(M=64, N=4096, K=28672, S=0, ldx=28672, ldy=4096, ldr=4096, perm=FAKE)
        assert need > 0 and call(**short) == call(**short, ws=FAKE, wsb=16) == B.WORKSPACE_TOO_SMALL
    else:
        assert call(ws=OFF16, wsb=1 << 30) == B.BAD_ALIGN and "workspace" in last()


def test_router_argument_errors():
    assert route(K=0) == route(K=12) == route(K=BIG, ldx=BIG, ldr=BIG) == route(M=-1) == route(M=1 << 31) == B.BAD_SHAPE
    assert route(E=0) == route(E=B.MOE_MAX_EXPERTS + 1) == B.BAD_SHAPE and "E = " in last()
    assert route(top=0) == route(top=9) == route(top=B.MOE_MAX_TOP_K + 1, E=64) == route(top=-1) == B.BAD_SHAPE and "top_k" in last()
    assert route(ldx=56) == B.BAD_SHAPE and route(ldr=56) == B.BAD_SHAPE and "router" in last()
    assert route(flags=4) == B.INVALID_ARG and "flags" in last()
    for null in ("x", "r", "ids", "w"):
        assert route(**{null: None}) == B.INVALID_ARG, null
    assert route(x=OFF8) == route(r=OFF8) == route(ldx=68) == route(ldr=68) == route(ids=OFF2) == route(w=OFF2) == route(bias=OFF2) == B.BAD_ALIGN
    assert route(M=0, x=None, r=None, ids=None, w=None, ws=None, wsb=0) == B.OK and last() == ""
    n = ctypes.c_size_t(9)
    assert B.lib().arcq_moe_route_workspace_size(4, 60, 8, ctypes.byref(n)) == B.BAD_SHAPE
    assert B.lib().arcq_moe_route_workspace_size(4, 64, 8, None) == B.INVALID_ARG
    assert B.arcq_moe_route_workspace_size(0, 64, 8) == 0
    for M, K, E in ((64, 8192, 256), (1, 8192, 512), (2000, 4096, 64)):
        need = B.arcq_moe_route_workspace_size(M, K, E)
        if need:
            short = dict(M=M, K=K, E=E, ldx=K, ldr=K)
            assert route(**short, ws=None, wsb=0) == route(**short, wsb=need - 1) == B.WORKSPACE_TOO_SMALL and "workspace" in last()
            assert route(**short, ws=OFF16, wsb=need) == B.BAD_ALIGN


@pytest.mark.parametrize("call,block", [(moe, 16), (mx_moe, 32)])
def test_experts_argument_errors(call, block):
    assert call(K=block // 2) == call(K=BIG, ldx=BIG) == call(K=0) == call(S=block // 2) == call(S=96) == call(S=-block) == B.BAD_SHAPE
    assert call(I=0) == call(I=block // 2) == call(I=BIG) == call(S2=block // 2) == call(S2=96) == B.BAD_SHAPE
    assert call(M=-1) == call(M=1 << 31) == call(N=-1) == call(N=1 << 25) == B.BAD_SHAPE
    assert call(E=0) == call(E=B.MOE_MAX_EXPERTS + 1) == call(top=0) == call(top=B.MOE_MAX_TOP_K + 1) == B.BAD_SHAPE
    assert call(ldx=56) == B.BAD_SHAPE
    nulls = ["x", "ids", "w", "uc", "us", "dc", "ds", "y"] + (["ut", "dt_"] if block == 16 else [])
    for null in nulls:
        assert call(**{null: None}) == B.INVALID_ARG, null
    offs = {"x": OFF8, "ldx": 68, "uc": OFF4, "dc": OFF4, "perm": OFF8, "ids": OFF2, "w": OFF2, "y": OFF2} | ({"ut": OFF2, "dt_": OFF1} if block == 16 else {})
    for name, off in offs.items():
        assert call(**{name: off}) == B.BAD_ALIGN, name
    need = B.arcq_moe_workspace_size(3, 2, 8, 64, 64, 8, False)
    assert need >= 2 * 3 * 2 * 64 * 2
    assert call(wsb=need - 1) == call(ws=None) == B.WORKSPACE_TOO_SMALL and "workspace" in last()
    assert call(ws=OFF16) == B.BAD_ALIGN
    more = B.arcq_moe_workspace_size(3, 2, 8, 64, 64, 8, True)
    assert more > need and call(perm=FAKE, wsb=need) == B.WORKSPACE_TOO_SMALL


def test_experts_workspace():
    size = B.arcq_moe_workspace_size
    assert size(0, 2, 8, 64, 64, 64, True) == size(2, 2, 8, 64, 64, 0, True) == 0
    assert size(10 ** 6, 8, 32, 4096, 14336, 4096, True) == size(64, 8, 32, 4096, 14336, 4096, True) <= 64 << 20      # tokens go so many at a time
    n = ctypes.c_size_t(9)
    raw = B.lib().arcq_moe_workspace_size
    for bad in ((4, 0, 8, 64, 64, 8), (4, 17, 32, 64, 64, 8), (-1, 2, 8, 64, 64, 8), (4, 2, 0, 64, 64, 8), (4, 2, 8, 40, 64, 8), (4, 2, 8, 64, 8, 8), (4, 2, 8, 64, 64, -1)):
        assert raw(*bad, 0, ctypes.byref(n)) == B.BAD_SHAPE, bad
    assert raw(4, 2, 8, 64, 64, 8, 0, None) == B.INVALID_ARG
