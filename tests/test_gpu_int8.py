"""The 8-bit product with scales and the quantisation of its rows against their oracles: outputs bit for bit, bounds one-sided within 1e-6,
profiles equal to the streaming check of the stored output and bound."""
import numpy as np
import pytest
import torch

import oracle
from oracle import int8
from opmap import assert_profile_equal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


def operands(M, N, K, seed=0, bias=False, extremes=True):
    rng = np.random.default_rng(seed)
    A, W = rng.integers(-128, 128, (M, K), dtype=np.int8), rng.integers(-128, 128, (N, K), dtype=np.int8)
    if extremes and M and N and K:
        A[0], W[0] = -128, -128
        A[-1, -1], W[-1, -1] = 127, -128
    sa, sw = rng.uniform(0.001, 0.1, M).astype(np.float32), rng.uniform(-0.1, 0.1, N).astype(np.float32)
    return A, sa, W, sw, rng.normal(0, 1, N).astype(np.float32) if bias else None


def cuda(*arrays):
    return [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def assert_bound(tau, exact, what=""):
    """tau at or above the formula's value (extended precision, good to a few 2^-63) and within 1e-6; one step where it is subnormal."""
    t, e = tau.astype(np.longdouble), np.asarray(exact)
    assert np.array_equal(np.isnan(t), np.isnan(e)), what
    ok = ~np.isnan(e)
    t, e = t[ok], e[ok]
    big = e > np.finfo(np.float32).max
    assert np.isinf(t[big]).all(), what
    t, e = t[~big], e[~big]
    assert (t >= e * (1 - np.longdouble(2) ** -60)).all(), what
    most = e * (1 + np.longdouble(1e-6)) + np.longdouble(2) ** -149
    assert ((t <= most) | (np.isinf(t) & (most > np.finfo(np.float32).max))).all(), "%s: %g" % (what, float((t / np.maximum(e, 1e-300) - 1).max()))


SHAPES = [(1, 1, 1), (1, 7, 3), (2, 16, 64), (5, 33, 100), (16, 40, 65), (17, 16, 128), (33, 129, 257), (64, 64, 64), (65, 130, 1000),
          (127, 129, 31), (128, 256, 512), (130, 250, 1001), (200, 1000, 96), (257, 263, 2048), (1, 4096, 4096), (8, 1111, 3000), (300, 511, 4099), (513, 770, 640)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("with_bias", [False, True])
def test_product(tao, M, N, K, with_bias):
    A, sa, W, sw, b = operands(M, N, K, M + N + K, with_bias)
    y, tau = tao.tao_bound_linear_int8(*cuda(A, sa, W, sw), bias=cuda(b)[0])
    ye, te = int8.linear_int8(A, sa, W, sw, b)
    assert np.array_equal(y.cpu().numpy().view(np.uint32), ye.view(np.uint32))
    assert_bound(tau.cpu().numpy(), te)


@pytest.mark.parametrize("K", [0, 1, 15, 16, 17, 127, 128, 129, 1024, 1025, 16384, 131071])
def test_reduction_lengths_and_the_largest_sums(tao, K):
    M, N = 19, 35
    A, sa, W, sw, b = operands(M, N, K, K, True)
    if K:
        A[1], A[2] = -128, 127
        W[1], W[2] = -128, 127
    y, tau = tao.tao_bound_linear_int8(*cuda(A, sa, W, sw), bias=cuda(b)[0])
    ye, te = int8.linear_int8(A, sa, W, sw, b)
    assert np.array_equal(y.cpu().numpy().view(np.uint32), ye.view(np.uint32))
    assert_bound(tau.cpu().numpy(), te)


@pytest.mark.parametrize("M,N,K", [(3, 50, 96), (70, 90, 200), (256, 300, 192)])
@pytest.mark.parametrize("pad,at", [(0, 0), (1, 0), (3, 5), (16, 0), (16, 16), (7, 1)])
def test_strides_and_addresses(tao, M, N, K, pad, at):
    """Rows further apart than they are long, from any address; what lies between and behind them is 127 and must not count."""
    A, sa, W, sw, b = operands(M, N, K, pad + at, True)

    def placed(a):
        rows, k = a.shape
        flat = np.full(at + rows * (k + pad) + 64, 127, np.int8)
        for r in range(rows):
            flat[at + r * (k + pad): at + r * (k + pad) + k] = a[r]
        return torch.from_numpy(flat).cuda()[at: at + rows * (k + pad)].view(rows, k + pad)[:, :k]
    Ad, Wd = placed(A), placed(W)
    sad, swd, bd = cuda(sa, sw, b)
    y, tau = tao.tao_bound_linear_int8(Ad, sad, Wd, swd, bias=bd)
    ye, te = int8.linear_int8(A, sa, W, sw, b)
    assert np.array_equal(y.cpu().numpy().view(np.uint32), ye.view(np.uint32))
    assert_bound(tau.cpu().numpy(), te)


def test_wide_output_rows_keep_what_lies_between_them(tao):
    for M, N, K in ((5, 33, 64), (130, 257, 128), (300, 260, 256)):
        A, sa, W, sw, _ = operands(M, N, K, 3)
        Ad, sad, Wd, swd = cuda(A, sa, W, sw)
        y, tau = torch.full((M, N + 9), 7.0, device="cuda"), torch.full((M, N + 9), 7.0, device="cuda")
        rc = tao.lib().tao_bound_linear_int8(Ad.data_ptr(), sad.data_ptr(), Wd.data_ptr(), swd.data_ptr(), None, y.data_ptr(), tau.data_ptr(),
                                             M, N, K, K, K, N + 9, 1, 0, 0, 0, None, tao._stream())
        assert rc == 0
        ye, te = int8.linear_int8(A, sa, W, sw)
        assert np.array_equal(y[:, :N].cpu().numpy(), ye)
        assert_bound(tau[:, :N].cpu().numpy(), te)
        assert bool((y[:, N:] == 7).all()) and bool((tau[:, N:] == 7).all())


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("M,N,K", [(4, 20, 64), (70, 65, 130), (200, 256, 256)])
def test_batches(tao, shared, M, N, K):
    parts = [operands(M, N, K, s, True) for s in range(3)]
    A, sa = (np.stack([p[i] for p in parts]) for i in (0, 1))
    W, sw = (parts[0][i] if shared else np.stack([p[i] for p in parts]) for i in (2, 3))
    b = parts[0][4]
    y, tau = tao.tao_bound_linear_int8(*cuda(A, sa, W, sw), bias=cuda(b)[0])
    claimed = y.clone()
    claimed[1, 2, 3] += 1.0
    pf = tao.tao_bound_check_linear_int8(*cuda(A, sa, W, sw), claimed, bias=cuda(b)[0])
    for z in range(3):
        ye, te = int8.linear_int8(A[z], sa[z], W if shared else W[z], sw if shared else sw[z], b)
        assert np.array_equal(y[z].cpu().numpy().view(np.uint32), ye.view(np.uint32))
        assert_bound(tau[z].cpu().numpy(), te)
    assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy()))
    assert pf["violations"] == 1


def test_one_of_the_two_outputs(tao):
    A, sa, W, sw, b = operands(40, 70, 128, 1, True)
    a, bias = cuda(A, sa, W, sw), cuda(b)[0]
    y, tau = tao.tao_bound_linear_int8(*a, bias=bias)
    y1, none = tao.tao_bound_linear_int8(*a, bias=bias, with_tau=False)
    none2, t1 = tao.tao_bound_linear_int8(*a, bias=bias, with_y=False)
    assert none is None and none2 is None and torch.equal(y, y1) and torch.equal(tau, t1)


def test_scales_that_are_no_ordinary_numbers(tao):
    A, sa, W, sw, b = operands(40, 70, 96, 5, True)
    sa[3], sa[4], sa[5], sa[6], sa[7] = np.nan, np.inf, 0.0, 1e-42, 3e38
    sw[2], sw[9], sw[10], sw[11] = np.nan, -np.inf, 0.0, -1e-30
    b[20], b[21] = np.inf, np.nan
    y, tau = tao.tao_bound_linear_int8(*cuda(A, sa, W, sw), bias=cuda(b)[0])
    ye, te = int8.linear_int8(A, sa, W, sw, b)
    y, tau = y.cpu().numpy(), tau.cpu().numpy()
    same = (y.view(np.uint32) == ye.view(np.uint32)) | (np.isnan(y) & np.isnan(ye))
    assert same.all()
    finite = np.isfinite(sa)[:, None] & np.isfinite(sw)[None, :] & np.isfinite(b)[None, :]
    assert_bound(tau[finite], te[finite])
    assert not np.isfinite(tau[~finite]).any()
    claimed = torch.from_numpy(y.copy()).cuda()
    pf = tao.tao_bound_check_linear_int8(*cuda(A, sa, W, sw), claimed, bias=cuda(b)[0])
    assert_profile_equal(pf, oracle.check_and_profile(y, y, tau))
    assert pf["violations"] >= (~finite).sum()


@pytest.mark.parametrize("model", [dict(mode=1, lam=4.0), dict(flags=1), dict(u=2.0 ** -11), dict(flags=1, u=2.0 ** -20)])
def test_models(tao, model):
    A, sa, W, sw, b = operands(33, 65, 700, 8, True)
    sa[0], sw[0] = 1e-40, 1e-30
    m = tao.FpModel(**model)
    _, tau = tao.tao_bound_linear_int8(*cuda(A, sa, W, sw), bias=cuda(b)[0], model=m)
    _, te = int8.linear_int8(A, sa, W, sw, b, model=m)
    assert_bound(tau.cpu().numpy(), te)


CHECKED = [(1, 1, 1), (3, 100, 70), (16, 512, 512), (60, 200, 333), (150, 300, 640), (300, 260, 1024), (700, 1000, 96), (1, 5000, 128), (1025, 513, 256)]


@pytest.mark.parametrize("M,N,K", CHECKED)
@pytest.mark.parametrize("ref", [False, True])
def test_check_is_the_streaming_check_of_the_stored_bound(tao, M, N, K, ref):
    A, sa, W, sw, b = operands(M, N, K, M * N, True)
    a, bias = cuda(A, sa, W, sw), cuda(b)[0]
    y, tau = tao.tao_bound_linear_int8(*a, bias=bias)
    g = torch.Generator(device="cuda").manual_seed(M + N)
    f = torch.tensor([0.0, 0.0, 0.5, -0.99, 1.0, 1.01, -3.0, 1e6], device="cuda")[torch.randint(0, 8, y.shape, generator=g, device="cuda")]
    claimed = (y.double() + f.double() * tau.double()).float()
    claimed.view(-1)[0] = float("nan")
    claimed.view(-1)[-1] = float("inf")
    y_ref = (y * (1 + 2.0 ** -23)).contiguous() if ref else None
    for alpha, eps_rel in ((1.0, 1e-12), (2.0, 0.0)):
        pf = tao.tao_bound_check_linear_int8(*a, claimed, bias=bias, y_ref=y_ref, alpha=alpha, eps_rel=eps_rel)
        other = y if y_ref is None else y_ref
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), other.cpu().numpy(), tau.cpu().numpy(), alpha, eps_rel))
    honest = tao.tao_bound_check_linear_int8(*a, y.clone(), bias=bias)
    assert honest["accept"] == 1 and honest["max_rel"] == 0.0 and honest["n"] == M * N


@pytest.mark.parametrize("M,N,K", [(20, 300, 200), (150, 300, 640), (1500, 1000, 128), (2100, 2100, 64)])
def test_the_largest_error_among_many(tao, M, N, K):
    """Claims whose largest error is one of many almost as large, the last of a rising row, the first of a falling one, or the only one."""
    a = cuda(*operands(M, N, K, 5, True))
    y, tau = tao.tao_bound_linear_int8(*a)
    d, n = y.double(), y.numel()
    ramp = torch.arange(1, n + 1, device="cuda", dtype=torch.float64).view(y.shape) / n
    one = y.clone()
    one.view(-1)[n // 3] *= 1.5
    for claimed in ((d * (1 + 1e-3)).float(), (d * (1 + 1e-3 * ramp)).float(), (d * (1 + 1e-3 * (1 + 1 / n - ramp))).float(), one, torch.nextafter(y, torch.zeros_like(y)), 0 * y):
        pf = tao.tao_bound_check_linear_int8(*a[:4], claimed, a[4], eps_rel=1e-9)
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy(), 1.0, 1e-9))


def test_checks_of_nothing(tao):
    for M, N in ((0, 5), (5, 0)):
        A, sa, W, sw, _ = operands(M, N, 16)
        pf = tao.tao_bound_check_linear_int8(*cuda(A, sa, W, sw), torch.empty((M, N), device="cuda"))
        assert pf["n"] == 0 and pf["accept"] == 1 and pf["hist"].sum() == 0
        y, tau = tao.tao_bound_linear_int8(*cuda(A, sa, W, sw))
        assert y.shape == (M, N)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 5), (7, 64), (2, 255), (5, 256), (64, 257), (9, 1000), (3, 1024), (4, 2049), (6, 4096), (2, 5001), (3, 12288), (1, 40000), (700, 33), (20000, 17), (8, 2), (2, 16385), (3, 32769), (17000, 1030), (5, 4)])
def test_quantised_rows_bit_for_bit(tao, rows, cols):
    rng = np.random.default_rng(rows * cols)
    x = (rng.normal(0, 1, (rows, cols)) * np.exp(rng.normal(0, 3, (rows, 1)))).astype(np.float32)
    if rows > 6:
        x[0] = 0; x[1, cols // 2] = np.inf; x[2, -1] = np.nan; x[3] = 0; x[3, -1] = 1e-45; x[4] *= np.float32(1e-41); x[5, 0] = -np.inf; x[6] = 3e38
    q, s = tao.tao_quantize_rows(cuda(x)[0])
    qe, se = int8.quantize_rows(x)
    assert np.array_equal(s.cpu().numpy().view(np.uint32) & 0x7fffffff, se.view(np.uint32) & 0x7fffffff) or np.array_equal(s.cpu().numpy(), se, equal_nan=True)
    assert np.array_equal(q.cpu().numpy(), qe)


def test_quantised_rows_of_every_alignment(tao):
    rng = np.random.default_rng(0)
    for cols, ld, at, ldq, atq in ((100, 100, 1, 100, 3), (100, 103, 0, 101, 1), (256, 260, 4, 272, 0), (1000, 1000, 2, 1000, 0), (4096, 4100, 0, 4100, 4), (5000, 5001, 3, 5003, 5)):
        rows = 5
        base = torch.from_numpy(rng.normal(0, 2, at + rows * ld).astype(np.float32)).cuda()
        x = base[at:].view(rows, ld)[:, :cols]
        store = torch.full((atq + rows * ldq,), 99, dtype=torch.int8, device="cuda")
        q = store[atq:].view(rows, ldq)[:, :cols]
        tao.tao_quantize_rows(x, q=q)
        qe, _ = int8.quantize_rows(x.cpu().numpy())
        assert np.array_equal(q.cpu().numpy(), qe)
        assert bool((store[atq:].view(rows, ldq)[:, cols:] == 99).all()) and bool((store[:atq] == 99).all())


@pytest.mark.parametrize("rows,cols", [(8, 4096), (3000, 777), (40, 20000)])
def test_quantised_rows_are_those_of_a_tensor_program(tao, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp(torch.randn((rows, 1), generator=g, device="cuda"))
    scale = x.abs().amax(dim=1) / 127
    q, s = tao.tao_quantize_rows(x)
    assert torch.equal(s, scale) and torch.equal(q, torch.round(x / scale[:, None]).to(torch.int8))


@pytest.mark.parametrize("largest", [127.0, 1.0, 3.7e-5, 2.9e30, 1e-38, 2.0 ** -93, 2.0 ** -94])
def test_quotients_in_the_middle_of_two_whole_numbers(tao, largest):
    """The rounded quotient decides, at ties to even: arguments at and next to every middle, also where the scale is next to having no reciprocal."""
    m = np.float32(largest)
    s = m * (np.float32(1) / np.float32(127))
    k = (np.arange(-127, 127) + 0.5).astype(np.float32)
    x = [m]
    for step in range(-3, 4):
        v = (k * s).astype(np.float32)
        for _ in range(abs(step)):
            v = np.nextafter(v, np.float32(np.inf if step > 0 else -np.inf))
        x.append(v)
    x = np.hstack(x).astype(np.float32)
    assert np.abs(x).max() == m
    for cols in (len(x), 1000, 200, 60):
        rows = np.stack([np.concatenate([[m], c]) for c in np.array_split(x[1:], max(1, len(x) // cols)) for c in [np.resize(c, cols - 1)]]).astype(np.float32)
        q, scale = tao.tao_quantize_rows(cuda(rows)[0])
        qe, se = int8.quantize_rows(rows)
        assert np.array_equal(scale.cpu().numpy(), se) and np.array_equal(q.cpu().numpy(), qe)


@pytest.mark.parametrize("M,N,K", [(70, 33, 96), (40, 40, 100)])
def test_offsets_beyond_32_bits(tao, M, N, K):
    """Rows of A and W so far apart that the last ones lie more than 2^31 elements on; the same for rows to be quantised and their values."""
    A, sa, W, sw, _ = cuda(*operands(M, N, K, 3, False))
    expect = tao.tao_bound_linear_int8(A, sa, W, sw)
    far = lambda t: torch.empty((len(t), 2 ** 31 // len(t) + 2 ** 20), dtype=t.dtype, device="cuda")[:, 16:16 + t.shape[1]].copy_(t)
    for a, w in ((far(A), W), (A, far(W)), (far(A), far(W))):
        got = tao.tao_bound_linear_int8(a, sa, w, sw)
        assert torch.equal(got[0], expect[0]) and torch.equal(got[1], expect[1])
    x = torch.randn((M, K), device="cuda")
    q, s = tao.tao_quantize_rows(x)
    q2, s2 = tao.tao_quantize_rows(far(x), q=far(torch.zeros_like(q)))
    assert torch.equal(q, q2) and torch.equal(s, s2)


def test_refusals_of_the_binding(tao):
    A, sa, W, sw, b = cuda(*operands(8, 16, 32, 0, True))
    call = tao.tao_bound_linear_int8
    for bad in (lambda: call(A.float(), sa, W, sw), lambda: call(A, sa.double(), W, sw), lambda: call(A.cpu(), sa, W, sw),
                lambda: tao.tao_bound_check_linear_int8(A, sa, W, sw, None)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: call(A, sa, W[:, :31], sw), lambda: call(A, sa[:7], W, sw), lambda: call(A, sa, W, sw, bias=b[:3]),
                lambda: call(A.t(), sa, W, sw), lambda: call(A, sa, W, sw, y=torch.empty((8, 15), device="cuda")),
                lambda: call(A, sa, W, sw, with_y=False, with_tau=False),
                lambda: call(A.expand(3, 8, 32), sa.expand(3, 8).contiguous(), W.expand(3, 16, 32), sw.expand(3, 16).contiguous()),
                lambda: tao.tao_bound_check_linear_int8(A, sa, W, sw, torch.empty((16, 8), device="cuda")),
                lambda: tao.tao_bound_check_linear_int8(A, sa, W, sw, torch.empty((8, 16), device="cuda"), ws=torch.empty(64, dtype=torch.uint8, device="cuda")),
                lambda: tao.tao_quantize_rows(torch.empty((4, 8), device="cuda"), q=torch.empty((4, 7), dtype=torch.int8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(tao.TaoError):
        big = torch.zeros((1, 131072), dtype=torch.int8, device="cuda")
        call(big, sa[:1], big, sw[:1])
