"""Refusals of the 8-bit product, the row quantisation and the channels-last GroupNorm: status codes returned before anything is enqueued
(no GPU), and their workspace queries."""
import ctypes

import pytest

P, ODD, NUL = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x100002), ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    t.lib()
    return t


def test_product_refusals(tao):
    f = tao.lib().tao_bound_linear_int8

    def call(A=P, sa=P, W=P, sw=P, bias=NUL, y=P, tau=P, M=4, N=8, K=32, lda=32, ldw=32, ldy=8, batch=1, sA=0, sW=0, sY=0, model=None):
        return f(A, sa, W, sw, bias, y, tau, M, N, K, lda, ldw, ldy, batch, sA, sW, sY, model, None)
    for k in ("M", "N", "K", "batch", "sA", "sW", "sY"):
        assert call(**{k: -1}) == tao.ERR_SHAPE, k
    assert call(lda=31) == call(ldw=31) == call(ldy=7) == tao.ERR_SHAPE
    assert call(batch=2, sA=128, sY=31) == tao.ERR_SHAPE                               # overlapping outputs
    assert call(M=2 ** 31, lda=32) == call(M=2 ** 20, N=2 ** 16, ldy=2 ** 16) == tao.ERR_SHAPE
    assert call(lda=2 ** 59) == call(batch=2, sA=2 ** 60, sY=64) == tao.ERR_SHAPE
    assert call(K=131072, lda=131072, ldw=131072) == tao.ERR_K_RANGE
    assert tao.INT8_MAX_K * 2 ** 14 < 2 ** 31 <= (tao.INT8_MAX_K + 1) * 2 ** 14
    for k in ("A", "sa", "W", "sw"):
        assert call(**{k: NUL}) == tao.ERR_NULL, k
    assert call(y=NUL, tau=NUL) == tao.ERR_NULL
    for k in ("sa", "sw", "bias", "y", "tau"):
        assert call(**{k: ODD}) == tao.ERR_ALIGN, k
    assert call(model=ctypes.byref(tao.FpModel(u=0.5))) == tao.ERR_MODEL
    for k in ("M", "N", "batch"):                                                      # nothing to do
        assert call(**{k: 0}, A=NUL, sa=NUL, W=NUL, sw=NUL, y=NUL, tau=NUL) == tao.OK, k


def test_product_check_refusals(tao):
    f, need = tao.lib().tao_bound_check_linear_int8, tao.lib().tao_check_workspace_bytes(32)

    def call(y_ref=NUL, claimed=P, alpha=1.0, eps=1e-12, out=P, ws=P, bytes=need, **k):
        a = dict(M=4, N=8, K=32, lda=32, ldw=32, ldy=8)
        a.update(k)
        return f(P, P, P, P, NUL, y_ref, claimed, a["M"], a["N"], a["K"], a["lda"], a["ldw"], a["ldy"], 1, 0, 0, 0, alpha, eps, None, out, ws, bytes, None)
    assert call(M=-1) == call(lda=5) == tao.ERR_SHAPE
    for v in (-1.0, float("nan"), float("inf")):
        assert call(alpha=v) == call(eps=v) == tao.ERR_SHAPE
    assert call(claimed=NUL) == call(out=NUL) == tao.ERR_NULL
    assert call(claimed=ODD) == call(y_ref=ODD) == call(out=ctypes.c_void_p(0x100004)) == tao.ERR_ALIGN
    assert call(ws=NUL) == call(bytes=need - 1) == call(ws=ctypes.c_void_p(0x100080)) == tao.ERR_WORKSPACE
    assert call(K=131072, lda=131072, ldw=131072) == tao.ERR_K_RANGE


def test_quantisation_refusals(tao):
    f = tao.lib().tao_quantize_rows
    assert f(P, P, P, -1, 4, 4, 4, None) == f(P, P, P, 4, -1, 4, 4, None) == f(P, P, P, 4, 8, 7, 8, None) == f(P, P, P, 4, 8, 8, 7, None) == tao.ERR_SHAPE
    assert f(P, P, P, 2, 8, 2 ** 60, 8, None) == tao.ERR_SHAPE
    assert f(NUL, P, P, 4, 8, 8, 8, None) == f(P, NUL, P, 4, 8, 8, 8, None) == f(P, P, NUL, 4, 8, 8, 8, None) == tao.ERR_NULL
    assert f(ODD, P, P, 4, 8, 8, 8, None) == f(P, P, ODD, 4, 8, 8, 8, None) == tao.ERR_ALIGN
    assert f(NUL, NUL, NUL, 0, 8, 8, 8, None) == tao.OK


def test_groupnorm_act_refusals(tao):
    L = tao.lib()
    need = L.tao_groupnorm_act_workspace_bytes(2, 4096, 8, 4)
    assert need > 0
    assert L.tao_groupnorm_act_workspace_bytes(2, 16, 8, 4) == 0      # one workgroup a group: nothing to keep

    def call(act=tao.ACT_SILU, x=P, g=P, b=P, eps=1e-5, y=P, tau=P, batch=2, positions=4096, channels=8, groups=4, ldx=8, ldy=8, model=None, ws=P, bytes=need):
        return L.tao_bound_groupnorm_act(act, x, g, b, eps, y, tau, batch, positions, channels, groups, ldx, ldy, model, ws, bytes, None)
    assert call(act=tao.ACT_GELU_ERF) == call(act=-1) == call(act=99) == tao.ERR_KIND
    assert call(groups=3) == call(groups=0) == call(batch=-1) == call(positions=-1) == call(channels=-4) == tao.ERR_SHAPE
    assert call(ldx=7) == call(ldy=7) == call(eps=-1.0) == call(eps=float("nan")) == call(ldx=2 ** 59) == tao.ERR_SHAPE
    assert call(positions=2 ** 31) == call(positions=2 ** 30) == call(batch=2 ** 29, positions=16) == tao.ERR_SHAPE
    assert call(batch=2 ** 20, positions=1) == call(batch=2 ** 20, positions=1, channels=4096, groups=1, ldx=4096, ldy=4096) == tao.ERR_SHAPE
    assert L.tao_groupnorm_act_workspace_bytes(2 ** 20, 1, 8, 4) == L.tao_groupnorm_act_workspace_bytes(2 ** 20, 1, 4096, 1) == 0
    assert L.tao_groupnorm_act_workspace_bytes(1, 64, 2 ** 20, 2 ** 20) < 2 ** 30     # a group keeps parts of the blocks it lies in, not of all
    assert call(positions=2 ** 24) == tao.ERR_K_RANGE
    assert call(x=NUL) == call(y=NUL, tau=NUL) == tao.ERR_NULL
    assert call(x=ODD) == call(g=ODD) == call(b=ODD) == call(y=ODD) == call(tau=ODD) == tao.ERR_ALIGN
    assert call(ws=NUL) == call(bytes=need - 1) == call(ws=ctypes.c_void_p(0x100080)) == tao.ERR_WORKSPACE
    assert call(model=ctypes.byref(tao.FpModel(c_exp=2.0 ** 24))) == tao.ERR_MODEL
    for k in ("batch", "positions", "channels"):
        assert call(**{k: 0}, x=NUL, y=NUL, tau=NUL, ws=NUL, bytes=0) == tao.OK, k

    cneed = L.tao_bound_check_groupnorm_act_workspace_bytes(2, 4096, 8, 4)
    assert cneed == need + L.tao_check_workspace_bytes(2 * 4096 * 8)

    def check(act=tao.ACT_SILU, y_ref=NUL, claimed=P, alpha=1.0, eps=0.0, out=P, ws=P, bytes=cneed, groups=4):
        return L.tao_bound_check_groupnorm_act(act, P, P, P, 1e-5, y_ref, claimed, 2, 4096, 8, groups, 8, 8, alpha, eps, None, out, ws, bytes, None)
    assert check(act=3) == tao.ERR_KIND and check(groups=5) == tao.ERR_SHAPE
    for v in (-1.0, float("nan"), float("inf")):
        assert check(alpha=v) == check(eps=v) == tao.ERR_SHAPE
    assert check(claimed=NUL) == check(out=NUL) == tao.ERR_NULL
    assert check(claimed=ODD) == check(y_ref=ODD) == check(out=ctypes.c_void_p(0x100004)) == tao.ERR_ALIGN
    assert check(ws=NUL) == check(bytes=cneed - 1) == check(ws=ctypes.c_void_p(0x100080)) == tao.ERR_WORKSPACE
    assert L.tao_groupnorm_act_workspace_bytes(2, 16, 9, 4) == 0 and L.tao_groupnorm_act_workspace_bytes(0, 16, 8, 4) == 0
