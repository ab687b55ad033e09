"""Refusals of the rotary tables, the norm and rotation of heads and the product with 4-bit weights: status codes returned before anything is
enqueued (no GPU), and their workspace queries."""
import ctypes
import os
import subprocess
import sys

import pytest

P, ODD, NUL = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x100002), ctypes.c_void_p(0)
FOUR = ctypes.c_void_p(0x100004)
BAD = (-1.0, float("nan"), float("inf"))


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    t.lib()
    return t


def test_table_refusals(tao):
    f = tao.lib().tao_bound_rope_tables

    def call(positions=P, inv=P, scale=1.0, c=P, s=P, tc=P, ts=P, npos=8, half=4, model=None):
        return f(positions, inv, scale, c, s, tc, ts, npos, half, model, None)
    assert call(npos=-1) == call(half=-1) == call(npos=2 ** 31) == call(half=2 ** 31) == call(npos=2 ** 30, half=2 ** 11) == tao.ERR_SHAPE
    for v in (float("nan"), float("inf"), 1e39):
        assert call(scale=v) == tao.ERR_SHAPE
    assert call(inv=NUL) == call(c=NUL, s=NUL, tc=NUL, ts=NUL) == tao.ERR_NULL
    for k in ("inv", "c", "s", "tc", "ts"):
        assert call(**{k: ODD}) == tao.ERR_ALIGN, k
    assert call(positions=FOUR) == tao.ERR_ALIGN
    assert call(model=ctypes.byref(tao.FpModel(u=0.5))) == call(model=ctypes.byref(tao.FpModel(c_cos=-1.0))) == tao.ERR_MODEL
    assert call(npos=0, inv=NUL) == call(half=0, c=NUL, s=NUL, tc=NUL, ts=NUL) == tao.OK


HEADS = dict(norm=1, x=P, gq=P, gk=P, eps=1e-6, c=P, s=P, tc=NUL, ts=NUL, pos=P, tokens=3, hq=4, hk=2, d=16, rot=8, npos=5, ldt=96, ldh=16, ldyt=96, ldyh=16, inter=0)


def head_args(k):
    a = dict(HEADS)
    a.update(k)
    front = (a["norm"], a["x"], a["gq"], a["gk"], a["eps"], a["c"], a["s"], a["tc"], a["ts"], a["pos"])
    return front, (a["tokens"], a["hq"], a["hk"], a["d"], a["rot"], a["npos"], a["ldt"], a["ldh"], a["ldyt"], a["ldyh"], a["inter"])


def shared_head_refusals(tao, call):
    for k in ("tokens", "hq", "hk", "d", "rot", "ldt", "ldh", "ldyt", "ldyh"):
        assert call(**{k: -1}) == tao.ERR_SHAPE, k
    assert call(rot=7) == call(rot=18) == call(npos=0) == call(d=2 ** 30, ldyh=2 ** 30, ldyt=2 ** 40) == tao.ERR_SHAPE
    assert call(ldyh=15) == call(ldyt=95) == call(ldyt=0) == call(ldyt=16, ldyh=47) == tao.ERR_SHAPE          # outputs would overlap
    assert call(tokens=2 ** 33, ldyt=2 ** 10) == call(ldt=2 ** 59) == call(ldh=2 ** 59) == call(tokens=2 ** 40, hq=0, hk=0) == call(hq=2 ** 30) == tao.ERR_SHAPE
    for v in BAD:
        assert call(eps=v) == tao.ERR_SHAPE
    for norm in (0, 2, 3, 4, 6, -1):
        assert call(norm=norm) == tao.ERR_KIND
    assert call(norm=tao.NORM_NONE) == call(norm=tao.NORM_NONE, gk=NUL) == tao.ERR_KIND                       # a gain without a norm
    for k in ("x", "c", "s"):
        assert call(**{k: NUL}) == tao.ERR_NULL, k
    assert call(tc=P) == call(ts=P) == tao.ERR_NULL
    for k in ("x", "gq", "gk", "c", "s"):
        assert call(**{k: ODD}) == tao.ERR_ALIGN, k
    assert call(tc=ODD, ts=P) == call(tc=P, ts=ODD) == call(pos=FOUR) == tao.ERR_ALIGN
    assert call(d=2 ** 24, ldh=2 ** 24, ldt=2 ** 27, ldyh=2 ** 24, ldyt=2 ** 27) == tao.ERR_K_RANGE
    assert call(model=ctypes.byref(tao.FpModel(u=0.5))) == tao.ERR_MODEL


def test_head_refusals(tao):
    f = tao.lib().tao_bound_norm_rope

    def call(y=P, tau=P, model=None, **k):
        front, back = head_args(k)
        return f(*front, y, tau, *back, model, None)
    shared_head_refusals(tao, call)
    assert call(y=NUL, tau=NUL) == tao.ERR_NULL
    assert call(y=ODD) == call(tau=ODD) == tao.ERR_ALIGN
    for k in ({"tokens": 0}, {"hq": 0, "hk": 0}, {"d": 0, "rot": 0}):
        assert call(x=NUL, c=NUL, s=NUL, y=NUL, tau=NUL, **k) == tao.OK, k
    # the other kinds of norm stay with tao_bound_norm, and it knows nothing of "none"
    assert tao.lib().tao_bound_norm(tao.NORM_NONE, P, P, P, P, 1e-6, P, 4, 8, 8, None, None) == tao.ERR_KIND


def test_head_check_refusals(tao):
    f, need = tao.lib().tao_bound_check_norm_rope, tao.lib().tao_check_workspace_bytes(3 * 6 * 16)

    def call(y_ref=NUL, claimed=P, alpha=1.0, eps_rel=1e-12, model=None, out=P, ws=P, bytes=need, **k):
        front, back = head_args(k)
        return f(*front, y_ref, claimed, *back, alpha, eps_rel, model, out, ws, bytes, None)
    shared_head_refusals(tao, call)
    for v in BAD:
        assert call(alpha=v) == call(eps_rel=v) == tao.ERR_SHAPE
    assert call(claimed=NUL) == call(out=NUL) == tao.ERR_NULL
    assert call(claimed=ODD) == call(y_ref=ODD) == call(out=FOUR) == tao.ERR_ALIGN
    assert call(ws=NUL) == call(bytes=need - 1) == call(ws=ctypes.c_void_p(0x100080)) == tao.ERR_WORKSPACE


INT4 = dict(A=P, W=P, scale=P, zero=P, group=32, bias=NUL, M=4, N=8, K=65, lda=65, ldw=33, ldy=8)


def shared_int4_refusals(tao, call):
    for k in ("M", "N", "K"):
        assert call(**{k: -1}) == tao.ERR_SHAPE, k
    assert call(lda=64) == call(ldw=32) == call(ldy=7) == tao.ERR_SHAPE
    for group in (0, -32, 1, 31, 33, 48, 64 - 16):
        assert call(group=group) == tao.ERR_SHAPE, group
    assert call(M=2 ** 31) == call(N=2 ** 31, ldy=2 ** 31) == call(M=2 ** 20, N=2 ** 16, ldy=2 ** 16) == call(K=2 ** 31, lda=2 ** 31, ldw=2 ** 30) == tao.ERR_SHAPE
    assert call(lda=2 ** 59) == call(ldw=2 ** 58) == call(ldy=2 ** 59) == tao.ERR_SHAPE
    assert call(K=2 ** 24, lda=2 ** 24, ldw=2 ** 23, group=128) == tao.ERR_K_RANGE
    for k in ("A", "W", "scale"):
        assert call(**{k: NUL}) == tao.ERR_NULL, k
    for k in ("A", "scale", "bias"):
        assert call(**{k: ODD}) == tao.ERR_ALIGN, k
    assert call(model=ctypes.byref(tao.FpModel(u=0.5))) == tao.ERR_MODEL


def test_int4_refusals(tao):
    L = tao.lib()

    def call(y=P, tau=P, model=None, ws=NUL, bytes=0, **k):
        a = dict(INT4)
        a.update(k)
        return L.tao_bound_linear_int4(a["A"], a["W"], a["scale"], a["zero"], a["group"], a["bias"], y, tau, a["M"], a["N"], a["K"], a["lda"], a["ldw"], a["ldy"], model, ws, bytes, None)
    shared_int4_refusals(tao, call)
    assert call(y=NUL, tau=NUL) == tao.ERR_NULL
    assert call(y=ODD) == call(tau=ODD) == tao.ERR_ALIGN
    for k in ("M", "N"):
        assert call(**{k: 0}, A=NUL, W=NUL, scale=NUL, y=NUL, tau=NUL) == tao.OK, k
    assert L.tao_linear_int4_workspace_bytes(-1, 8, 8) == L.tao_linear_int4_workspace_bytes(0, 8, 8) == 0


def test_int4_check_refusals(tao):
    L = tao.lib()
    need = L.tao_bound_check_linear_int4_workspace_bytes(4, 8, 65)
    assert need >= L.tao_check_workspace_bytes(32)

    def call(y_ref=NUL, claimed=P, alpha=1.0, eps_rel=1e-12, model=None, out=P, ws=P, bytes=need, **k):
        a = dict(INT4)
        a.update(k)
        return L.tao_bound_check_linear_int4(a["A"], a["W"], a["scale"], a["zero"], a["group"], a["bias"], y_ref, claimed, a["M"], a["N"], a["K"], a["lda"], a["ldw"], a["ldy"],
                                             alpha, eps_rel, model, out, ws, bytes, None)
    shared_int4_refusals(tao, call)
    for v in BAD:
        assert call(alpha=v) == call(eps_rel=v) == tao.ERR_SHAPE
    assert call(claimed=NUL) == call(out=NUL) == tao.ERR_NULL
    assert call(claimed=ODD) == call(y_ref=ODD) == call(out=FOUR) == tao.ERR_ALIGN
    assert call(ws=NUL) == call(bytes=need - 1) == call(ws=ctypes.c_void_p(0x100080)) == tao.ERR_WORKSPACE


@pytest.mark.parametrize("M,N,K", [(16, 10300, 200), (2, 96, 12288), (5, 4200, 6200)])
def test_int4_workspace_refusals(tao, M, N, K):
    """Products that take digits, parts of the reduction, or both: their workspace missing, short and off its alignment."""
    L = tao.lib()
    need, check = L.tao_linear_int4_workspace_bytes(M, N, K), L.tao_bound_check_linear_int4_workspace_bytes(M, N, K)
    assert 0 < need < check
    for ws, size in ((NUL, need), (NUL, 0), (P, need - 1), (P, 0), (ctypes.c_void_p(0x100080), need)):
        assert L.tao_bound_linear_int4(P, P, P, NUL, 128, NUL, P, P, M, N, K, K, K // 2, N, None, ws, size, None) == tao.ERR_WORKSPACE
    for ws, size in ((NUL, check), (P, check - 1), (P, need), (ctypes.c_void_p(0x100080), check)):
        assert L.tao_bound_check_linear_int4(P, P, P, NUL, 128, NUL, NUL, P, M, N, K, K, K // 2, N, 1.0, 1e-12, None, P, ws, size, None) == tao.ERR_WORKSPACE


def test_int4_takes_every_number_of_tokens_that_it_says():
    """2^31 - 1 tokens by one column are no bad shape.  (Their operands fit no card: in a process without devices, where the call ends before its launch.)"""
    code = """
import ctypes, torch
import paper_2510_16028_amd as t
assert torch.cuda.device_count() == 0
P = ctypes.c_void_p(0x100000)
for M, N, K in ((2 ** 31 - 1, 1, 33), (2 ** 31 - 1, 31, 127), (2 ** 31 - 8, 1, 64), (1, 2 ** 31 - 1, 64)):
    assert t.lib().tao_linear_int4_workspace_bytes(M, N, K) == 0
    print(t.lib().tao_bound_linear_int4(P, P, P, None, K, None, P, P, M, N, K, K, (K + 1) // 2, N, None, None, 0, None))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1"), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    import paper_2510_16028_amd as tao
    assert r.stdout.split() == [str(tao.ERR_LAUNCH)] * 4
