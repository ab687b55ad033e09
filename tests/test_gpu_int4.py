"""The product with 4-bit weights and group scales against its oracle: outputs within the documented distance of the formula, bounds one-sided within
1e-6, profiles equal to the streaming check of the stored output and bound; and a run of the operators of a decode step."""
import numpy as np
import pytest
import torch

import oracle
from oracle import int4, rotary
from opmap import assert_profile_equal
from test_gpu_int8 import assert_bound, cuda

pytestmark = pytest.mark.gpu
F, L, U = np.float32, np.longdouble, 2.0 ** -24


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


def operands(M, N, K, group, seed=0, zero=False, bias=False, spread=1.0):
    rng = np.random.default_rng(seed + M + N + K)
    G = -(-K // group)
    A = (rng.normal(0, 1, (M, K)) * np.exp(rng.normal(0, spread, (M, K)))).astype(F)
    q = rng.integers(0, 16, (N, K)).astype(np.uint8)
    s = (rng.uniform(0.001, 0.1, (N, G)) * rng.choice([-1, 1], (N, G))).astype(F)
    z = rng.integers(0, 16, (N, G)).astype(np.uint8) if zero else None
    return A, q, s, group, z, rng.normal(0, 1, N).astype(F) if bias else None


def run(tao, A, q, s, group, z, b, **more):
    Ad, Wd, sd, zd, bd = cuda(A, int4.pack(q), s, z, b)
    return tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd, **more)


def assert_product(got, A, q, s, group, z, b, model=None, what=""):
    y, tau = (t.cpu().numpy() for t in got)
    ye, te, size = int4.linear_int4(A, q, s, group, z, b, model=model)
    assert_bound(tau, te, what)
    ok = np.isfinite(size)
    # K <= 32: one rounding of the formula in binary64 (a sum of K products there); else the documented 15 u of the sum of magnitudes
    far = np.abs(ye) * L(U) + size * L(2) ** -46 if A.shape[1] <= 32 else size * 15 * L(U)
    assert (np.abs(y.astype(L) - ye)[ok] <= far[ok] * (1 + L(2) ** -20) + L(2) ** -149).all(), "%s %g" % (what, float((np.abs(y.astype(L) - ye)[ok] / np.maximum(size[ok], 1e-300) / U).max()))
    assert (np.abs(y.astype(L) - ye)[ok & (te > 1e-30)] <= te[ok & (te > 1e-30)] * (1 + L(2) ** -20)).all(), what


SHAPES = [(1, 1, 1, 32), (1, 7, 3, 3), (2, 16, 64, 32), (5, 33, 100, 32), (1, 64, 128, 128), (3, 40, 129, 64), (8, 129, 257, 128), (9, 64, 64, 64), (1, 300, 1000, 1000), (16, 31, 96, 96), (17, 70, 513, 512),
          (33, 128, 512, 128), (1, 1000, 4096, 128), (2, 96, 12288, 128), (64, 65, 640, 32), (65, 32, 1001, 32), (130, 250, 320, 64), (4, 515, 2050, 256), (7, 4100, 200, 32), (31, 33, 63, 63), (6, 48, 5000, 160)]


@pytest.mark.parametrize("M,N,K,group", SHAPES)
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("bias", [False, True])
def test_product(tao, M, N, K, group, zero, bias):
    o = operands(M, N, K, group, 0, zero, bias)
    assert_product(run(tao, *o), *o)


@pytest.mark.parametrize("K", [0, 1, 2, 15, 16, 17, 31, 32, 33, 34, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1023, 1025])
def test_reduction_lengths(tao, K):
    for group in (32, 64, max(K, 1)):
        o = operands(3, 37, K, group, K, True, True)
        assert_product(run(tao, *o), *o)


# products of so many tiles that digits are formed once: eight tokens a tile, sixteen over 64 columns, over 128 with two and with one group of wavefronts, and parts of the reduction
ONCE = [(5, 8300, 130, 32), (9, 4200, 257, 64), (8, 8209, 128, 128), (16, 10300, 200, 128), (15, 10250, 384, 96), (40, 11000, 130, 32), (33, 11001, 192, 64), (100, 10000, 129, 128), (81, 10013, 160, 160), (5, 4200, 6200, 160)]


@pytest.mark.filterwarnings("ignore:invalid value")
@pytest.mark.parametrize("M,N,K,group", ONCE)
@pytest.mark.parametrize("zero", [False, True])
def test_products_of_many_tiles(tao, M, N, K, group, zero):
    """... ordinary ones; rows of A and W further apart than they are long, from any address, with tokens and scales that are no numbers, an activation far above the others, and zero points
    outside the codes; then the check of claims at and around their bounds."""
    A, q, s, _, z, b = o = operands(M, N, K, group, 1, zero, not zero)
    assert_product(run(tao, *o), *o)
    A[1, 5], A[2, K // 2], A[3, 0] = np.nan, np.inf, 1e7
    s[7, 0], s[N - 1, -1] = np.nan, 0.0
    q[::3, 0] = 8 if z is None else z[::3, 0]
    if zero:
        z[5::200, 0] = 255
    W = int4.pack(q)
    Ad, Wd = torch.full((M, K + 3), float("nan"), device="cuda")[:, 1:K + 1], torch.full((N, W.shape[1] + 5), 255, dtype=torch.uint8, device="cuda")[:, 3:W.shape[1] + 3]
    Ad.copy_(torch.from_numpy(A))
    Wd.copy_(torch.from_numpy(W))
    sd, zd, bd = cuda(s, z, b)
    y, tau = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd)
    assert_product((y, tau), A, q, s, group, z, b)
    f = torch.tensor([0.0, 0.5, -0.99, 1.01, -3.0, 0.0, 0.0], device="cuda")[torch.arange(M * N, device="cuda") % 7].view(M, N)
    claimed = (y.double() + f.double() * tau.double()).float()
    pf = tao.tao_bound_check_linear_int4(Ad, Wd, sd, group, claimed, zero=zd, bias=bd)
    assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy()))


def test_more_tokens_than_digits_are_kept_of(tao):
    """A product whose digits take more than the workspace keeps of them at a time: the tokens go through in slabs."""
    M, N, K, group = 20000, 48, 1000, 64
    need = tao.tao_linear_int4_workspace_bytes(M, N, K)
    assert need < 8 * M * K                                  # (eight bytes of digits an activation)
    A, q, s, _, z, b = operands(M, N, K, group, 2, True, True)
    got = run(tao, A, q, s, group, z, b)
    for rows in (slice(0, 40), slice(8000, 8300), slice(16200, 16500), slice(M - 40, M)):
        assert_product([t[rows] for t in got], A[rows], q, s, group, z, b)


@pytest.mark.parametrize("M", [1, 2, 3, 5, 8, 9, 16, 24, 25, 32, 40, 100])
def test_numbers_of_tokens(tao, M):
    o = operands(M, 100, 300, 64, M, True, False, spread=3.0)
    assert_product(run(tao, *o), *o)


def test_codes_one_by_one(tao):
    """Every code with every zero point, and zero points outside the codes: one weight a row, so nothing can hide in a sum."""
    for K in (1, 40, 300):
        N, G = 256, -(-K // 64)
        A, s = np.zeros((2, K), F), np.full((N, G), 0.5, F)
        A[0, K - 1], A[1, 0] = 1.0, -3.0
        q, z = np.repeat(np.arange(N)[:, None] % 16, K, 1).astype(np.uint8), np.repeat(np.arange(N)[:, None] // 16, G, 1).astype(np.uint8)
        for zz in (z, z * 17, None):
            y, tau = run(tao, A, q, s, 64, zz, None)
            w = (q[:, 0].astype(int) - (8 if zz is None else zz[:, 0].astype(int))) * 0.5
            assert np.array_equal(y.cpu().numpy(), np.stack([w, -3 * w]).astype(F))
            assert_product((y, tau), A, q, s, 64, zz, None)


def test_columns_of_zero_weights(tao):
    """Codes equal to their zero points: exactly 0, with a bound of 0."""
    A, q, s, group, z, _ = operands(9, 40, 384, 128, 1, True)
    q[:20] = np.repeat(z[:20], 128, 1)
    y, tau = run(tao, A, q, s, group, z, None)
    assert not y[:, :20].any() and not tau[:, :20].any() and bool((tau[:, 20:] > 0).all())


@pytest.mark.parametrize("spread", [0.0, 6.0, 12.0])
def test_tokens_of_any_range(tao, spread):
    """Elements whose sizes differ by many octaves: what a sum keeps of the small ones is part of the bound's 1e-6."""
    rng = np.random.default_rng(4)
    o = list(operands(11, 64, 700, 128, 4, True, False, spread=spread))
    if spread == 12.0:                                       # single bits, and all significant bits, at every place
        o[0] = (o[0].view(np.uint32) & np.uint32(0xff800000) | rng.choice([0, 1, 0x7fffff, 0x400000, 0x00ffff, 0x7f0000, 0x7fff], o[0].shape).astype(np.uint32)).view(F)
    assert_product(run(tao, *o), *o)


@pytest.mark.parametrize("K,group", [(20, 20), (200, 64), (1024, 128)])
def test_values_that_are_no_ordinary_numbers(tao, K, group):
    M, N = 20, 40
    A, q, s, _, z, b = operands(M, N, K, group, 5, True, True)
    A[0, 3], A[1, 5], A[2, 0] = np.inf, np.nan, -np.inf
    A[3], A[4], A[5, ::2], A[6] = 0, 1e-42, 1e-36, 3e38
    A[7, 1], A[8, 2], A[9], A[10, 0] = 1e-45, 1e-38, A[9] * F(1e-35), 2.0 ** 120
    A[11] *= F(2.0 ** -100)
    A[12] *= F(2.0 ** 108)
    A[13, K // 2] = 2.0 ** -101
    s[2, 0], s[3, -1], s[4, 0], s[5], s[6] = np.nan, np.inf, 0.0, 1e-42, 1e38
    b[10], b[11], b[12] = np.nan, -np.inf, 3e38
    got = run(tao, A, q, s, group, z, b)
    y, tau = (t.cpu().numpy() for t in got)
    ye, te, size = int4.linear_int4(A, q, s, group, z, b)
    assert_bound(tau, te)
    with np.errstate(all="ignore"):
        ok = np.isfinite(te) & (np.abs(ye) < 3e38)
        assert (np.abs(y.astype(L) - ye)[ok] <= 15 * U * size[ok] * (1 + 1e-6) + L(2) ** -149).all()
    pf = tao.tao_bound_check_linear_int4(*cuda(A, int4.pack(q), s), group, got[0].clone(), zero=cuda(z)[0], bias=cuda(b)[0])
    assert_profile_equal(pf, oracle.check_and_profile(y, y, tau))


@pytest.mark.parametrize("model", [dict(mode=1, lam=4.0), dict(flags=1), dict(u=2.0 ** -16), dict(flags=1, u=2.0 ** -20)])
@pytest.mark.parametrize("K,group", [(30, 32), (700, 128)])
def test_models(tao, model, K, group):
    o = list(operands(7, 65, K, group, 8, True, True))
    o[0][0] = 1e-40
    o[2][0] = 1e-30
    m = tao.FpModel(**model)
    y, tau = run(tao, *o, model=m)
    assert_bound(tau.cpu().numpy(), int4.linear_int4(*o, model=m)[1])


@pytest.mark.parametrize("lam", [0.2, 0.4, 0.5, 1.0, 2.0, 4.0])
@pytest.mark.parametrize("M,N,K,group", [(3, 40, 33, 32), (8, 40, 128, 128), (8, 100, 224, 32), (3, 60, 1024, 128), (8, 8209, 200, 128), (2, 96, 12288, 128)])
def test_outputs_are_covered_by_the_bound_of_any_lambda(tao, lam, M, N, K, group):
    """Probabilistic bounds far below 15 u of the magnitudes, and tokens whose low bits all point the same way next to an activation, with a weight of 0, that makes a tile's whole numbers coarse: by 1 to 32 u of the
    sum.  The output stays inside the bound, and alpha = 2 admits claims at either end of it.  (A bound of the formula is at least one rounding: Gamma(K') >= 2^-24.)"""
    m = tao.FpModel(mode=1, lam=lam)
    G, big = -(-K // group), 5
    q, z = np.full((N, K), 15, np.uint8), np.zeros((N, G), np.uint8)
    q[:, big::max(group, 128)] = 0
    s = np.full((N, G), 0.37, F) * (1 + np.arange(N, dtype=F)[:, None] / N)
    if K == 33:
        s[:, 1] = 1e-20                                      # (one column: next to nothing)
    for octave in (5, 6, 7, 8, 9, 10):
        A = np.tile((1 + np.array([3, 1, 7, 3, 11], F) * F(2.0 ** -23))[np.arange(M) % 5, None], (1, K)).astype(F)
        A[:, big::max(group, 128)] = 1.5 * 2.0 ** octave
        y, tau = run(tao, A, q, s, group, z, None, model=m)
        ye, te, size = int4.linear_int4(A, q, s, group, z, None, model=m)
        assert_bound(tau.cpu().numpy(), te)
        assert (np.abs(y.cpu().numpy().astype(L) - ye) <= np.maximum(te, np.abs(ye) * L(U)) * (1 + L(2) ** -20)).all(), "%d: %g u" % (octave, float((np.abs(y.cpu().numpy() - ye) / size).max() / U))
        if te.min() < 2 * np.abs(ye).max() * U:
            continue                                         # (claims of binary32 inside the bound: only its rounding would fit)
        for end in (-1, 1):
            claimed = (ye + end * (te - np.abs(ye) * L(U) * 1.01)).astype(F)       # rounded, they are inside
            pf = tao.tao_bound_check_linear_int4(*cuda(A, int4.pack(q), s), group, cuda(claimed)[0], zero=cuda(z)[0], alpha=2.0, model=m)
            assert pf["accept"] == 1, octave


@pytest.mark.parametrize("M,N,K,group", [(3, 50, 96, 32), (9, 70, 257, 64), (20, 40, 512, 128)])
@pytest.mark.parametrize("pad,at,pada,ata", [(0, 0, 0, 0), (1, 0, 3, 1), (3, 5, 0, 2), (16, 0, 4, 0), (16, 16, 4, 4), (7, 1, 1, 3), (4, 4, 2, 0)])
def test_strides_and_addresses(tao, M, N, K, group, pad, at, pada, ata):
    """Rows further apart than they are long, from any address; what lies between is NaN in A and 255 in W and must not count."""
    A, q, s, _, z, b = operands(M, N, K, group, pad + at, True, True)
    W = int4.pack(q)

    def placed(a, pad, at, fill):
        rows, k = a.shape
        flat = np.full(at + rows * (k + pad) + 64, fill, a.dtype)
        for r in range(rows):
            flat[at + r * (k + pad): at + r * (k + pad) + k] = a[r]
        return torch.from_numpy(flat).cuda()[at: at + rows * (k + pad)].view(rows, k + pad)[:, :k]
    sd, zd, bd = cuda(s, z, b)
    got = tao.tao_bound_linear_int4(placed(A, pada, ata, np.nan), placed(W, pad, at, 255), sd, group, zero=zd, bias=bd)
    assert_product(got, A, q, s, group, z, b)


@pytest.mark.parametrize("K,group", [(7, 32), (40, 32), (257, 64), (1030, 1030)])
@pytest.mark.parametrize("at,pad", [(0, 0), (1, 0), (3, 5), (2, 2)])
def test_any_size_at_any_address(tao, K, group, at, pad):
    """The kernel of any size (models with underflow terms take it) with rows from any address; then tiles that leave outputs open: an activation far above the others of its block."""
    A, q, s, _, z, b = operands(3, 20, K, group, K + at, True, True)
    W, m = int4.pack(q), tao.FpModel(flags=1)
    Ad, sd, zd, bd = cuda(A, s, z, b)
    store = torch.full((at + 20 * (W.shape[1] + pad),), 255, dtype=torch.uint8, device="cuda")
    Wd = store[at:].view(20, W.shape[1] + pad)[:, :W.shape[1]].copy_(torch.from_numpy(W))
    assert_product(tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd, model=m), A, q, s, group, z, b, model=m)
    A[:, K // 2] *= 1e6
    q[::2, K // 2] = z[::2, K // 2 // group]
    Wd.copy_(torch.from_numpy(int4.pack(q)))
    assert_product(tao.tao_bound_linear_int4(cuda(A)[0], Wd, sd, group, zero=zd, bias=bd), A, q, s, group, z, b)


def test_wide_output_rows_keep_what_lies_between_them(tao):
    for M, N, K in ((5, 33, 64), (30, 257, 128), (2, 64, 31)):
        A, q, s, group, z, _ = operands(M, N, K, 32, 3)
        Ad, Wd, sd = cuda(A, int4.pack(q), s)
        y, tau = torch.full((M, N + 9), 7.0, device="cuda"), torch.full((M, N + 9), 7.0, device="cuda")
        ws = torch.empty(max(256, tao.tao_linear_int4_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
        rc = tao.lib().tao_bound_linear_int4(Ad.data_ptr(), Wd.data_ptr(), sd.data_ptr(), None, 32, None, y.data_ptr(), tau.data_ptr(), M, N, K, K, (K + 1) // 2, N + 9, None,
                                             ws.data_ptr(), ws.numel(), tao._stream())
        assert rc == 0
        assert_product((y[:, :N], tau[:, :N]), A, q, s, 32, None, None)
        assert bool((y[:, N:] == 7).all()) and bool((tau[:, N:] == 7).all())
        # claims and outputs of such rows are checked in place
        claimed, ref = y.clone(), y.clone()
        claimed[M - 1, 3] += 1.0
        out, need = tao.new_profile_buffer(y.device), tao.tao_bound_check_linear_int4_workspace_bytes(M, N, K)
        wsc = torch.empty(need, dtype=torch.uint8, device="cuda")
        for r in (None, ref.data_ptr()):
            rc = tao.lib().tao_bound_check_linear_int4(Ad.data_ptr(), Wd.data_ptr(), sd.data_ptr(), None, 32, None, r, claimed.data_ptr(), M, N, K, K, (K + 1) // 2, N + 9, 1.0, 1e-12, None,
                                                       out.data_ptr(), wsc.data_ptr(), need, tao._stream())
            pf = tao.read_profile(out)
            assert rc == 0 and pf["n"] == M * N and pf["violations"] == 1


def test_leading_dimensions_and_one_of_the_two_outputs(tao):
    A, q, s, group, z, b = operands(24, 70, 256, 64, 1, True, True)
    Ad, Wd, sd, zd, bd = cuda(A, int4.pack(q), s, z, b)
    y, tau = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd)
    y3, t3 = tao.tao_bound_linear_int4(Ad.view(2, 3, 4, 256), Wd, sd, group, zero=zd, bias=bd)
    assert y3.shape == (2, 3, 4, 70) and torch.equal(y3.view(24, 70), y) and torch.equal(t3.view(24, 70), tau)
    one = tao.tao_bound_linear_int4(Ad[0], Wd, sd, group, zero=zd, bias=bd)
    assert one[0].shape == (70,)
    y1, none = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd, with_tau=False)
    none2, t1 = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd, with_y=False)
    assert none is None and none2 is None and torch.equal(y, y1) and torch.equal(tau, t1)


CHECKED = [(1, 1, 1, 32), (3, 100, 70, 32), (16, 512, 512, 128), (1, 5000, 128, 128), (33, 300, 640, 64), (8, 2100, 256, 128), (70, 1000, 96, 96), (2, 40000, 64, 32)]


@pytest.mark.parametrize("M,N,K,group", CHECKED)
@pytest.mark.parametrize("ref", [False, True])
def test_check_is_the_streaming_check_of_the_stored_bound(tao, M, N, K, group, ref):
    A, q, s, _, z, b = operands(M, N, K, group, M * N, True, True)
    Ad, Wd, sd, zd, bd = cuda(A, int4.pack(q), s, z, b)
    y, tau = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd)
    g = torch.Generator(device="cuda").manual_seed(M + N)
    f = torch.tensor([0.0, 0.0, 0.5, -0.99, 1.0, 1.01, -3.0, 1e6], device="cuda")[torch.randint(0, 8, y.shape, generator=g, device="cuda")]
    claimed = (y.double() + f.double() * tau.double()).float()
    claimed.view(-1)[0] = float("nan")
    claimed.view(-1)[-1] = float("inf")
    y_ref = (y * (1 + 2.0 ** -23)).contiguous() if ref else None
    for alpha, eps_rel in ((1.0, 1e-12), (2.0, 0.0)):
        pf = tao.tao_bound_check_linear_int4(Ad, Wd, sd, group, claimed, zero=zd, bias=bd, y_ref=y_ref, alpha=alpha, eps_rel=eps_rel)
        other = y if y_ref is None else y_ref
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), other.cpu().numpy(), tau.cpu().numpy(), alpha, eps_rel))
    honest = tao.tao_bound_check_linear_int4(Ad, Wd, sd, group, y.clone(), zero=zd, bias=bd)
    assert honest["accept"] == 1 and honest["max_rel"] == 0.0 and honest["n"] == M * N


def test_checks_of_nothing(tao):
    for M, N in ((0, 5), (5, 0)):
        A, q, s, group, _, _ = operands(M, N, 64, 32)
        a = cuda(A, int4.pack(q), s)
        pf = tao.tao_bound_check_linear_int4(*a, group, torch.empty((M, N), device="cuda"))
        assert pf["n"] == 0 and pf["accept"] == 1 and pf["hist"].sum() == 0
        assert tao.tao_bound_linear_int4(*a, group)[0].shape == (M, N)


@pytest.mark.parametrize("M,N,K", [(10, 33, 96), (9, 40, 100)])
def test_offsets_beyond_32_bits(tao, M, N, K):
    """Rows of A and W so far apart that the last ones lie more than 2^31 elements on."""
    A, q, s, group, z, b = operands(M, N, K, 32, 3, True)
    Ad, Wd, sd, zd = cuda(A, int4.pack(q), s, z)
    expect = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd)
    far = lambda t: torch.empty((len(t), 2 ** 31 // len(t) + 2 ** 20), dtype=t.dtype, device="cuda")[:, 16:16 + t.shape[1]].copy_(t)
    for a, w in ((far(Ad), Wd), (Ad, far(Wd))):
        got = tao.tao_bound_linear_int4(a, w, sd, group, zero=zd)
        assert torch.equal(got[0], expect[0]) and torch.equal(got[1], expect[1])


@pytest.mark.parametrize("M,N,K", [(70000000, 3, 40), (3, 140000000, 33)])
def test_more_tiles_than_a_launch_has(tao, M, N, K):
    """Outputs whose tiles would have 2^32 threads and more: the first and last of them, and those next to the seams, against the same product in part."""
    g = torch.Generator(device="cuda").manual_seed(1)
    A, s = torch.randn((M, K), generator=g, device="cuda"), torch.rand((N, 2), generator=g, device="cuda")
    W = torch.randint(0, 256, (N, (K + 1) // 2), generator=g, device="cuda", dtype=torch.uint8)
    y, tau = tao.tao_bound_linear_int4(A, W, s, 32)
    long, seam = max(M, N), (1 << 22) * (1 if M > N else 16)
    for at in {0, seam - 50, seam, 2 * seam - 50, long - 100}:
        if at + 100 > long:
            continue
        rows, cols = (slice(at, at + 100), slice(None)) if M > N else (slice(None), slice(at, at + 100))
        a, w, sc = A[rows].contiguous(), W[cols].contiguous(), s[cols].contiguous()
        q = torch.stack([w & 15, w >> 4], dim=2).flatten(1)[:, :K]
        assert_product((y[rows, cols], tau[rows, cols]), a.cpu().numpy(), q.cpu().numpy(), sc.cpu().numpy(), 32, None, None)


def at_the_end(a):
    """A copy whose last byte is the last one of an allocation of whole pages."""
    store = torch.empty(20 << 20, dtype=torch.uint8, device="cuda")
    return store[len(store) - a.nbytes:].view(torch.from_numpy(a).dtype).view(a.shape).copy_(torch.from_numpy(a))


@pytest.mark.parametrize("M", [1, 3, 7, 30])
@pytest.mark.parametrize("K", [31, 33, 48, 66, 95, 128, 130, 288])
@pytest.mark.parametrize("zero", [False, True])
def test_operands_that_end_where_their_memory_ends(tao, M, K, zero):
    """Nothing behind an operand is read, not even to be thrown away (rows shorter than the bytes that a tile brings, tiles beyond the last row, no zero points)."""
    for group in (32, 64, K):
        A, q, s, _, z, b = operands(M, 21, K, group, K, zero, True)
        W, k = int4.pack(q), dict(zero=None if z is None else at_the_end(z), bias=at_the_end(b))
        assert_product(tao.tao_bound_linear_int4(at_the_end(A), at_the_end(W), at_the_end(s), group, **k), A, q, s, group, z, b)


def test_refusals_of_the_binding(tao):
    A, q, s, group, z, b = operands(8, 16, 64, 32, 0, True, True)
    A, W, s, z, b = cuda(A, int4.pack(q), s, z, b)
    call, check = tao.tao_bound_linear_int4, tao.tao_bound_check_linear_int4
    for bad in (lambda: call(A.double(), W, s, 32), lambda: call(A, W.to(torch.int8), s, 32), lambda: call(A.cpu(), W, s, 32), lambda: call(A, W, s, 32, zero=z.float()), lambda: check(A, W, s, 32, None)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: call(A, W[:, :31], s, 32), lambda: call(A, W, s[:, :1], 32), lambda: call(A, W, s, 64), lambda: call(A, W, s, 0), lambda: call(A, W, s, 32, zero=z[:8]),
                lambda: call(A, W, s, 32, bias=b[:3]), lambda: call(A.t(), W, s, 32), lambda: call(A, W, s, 32, y=torch.empty((8, 15), device="cuda")),
                lambda: call(A, W, s, 32, with_y=False, with_tau=False), lambda: check(A, W, s, 32, torch.empty((16, 8), device="cuda")),
                lambda: check(A, W, s, 32, torch.empty((8, 16), device="cuda"), ws=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(tao.TaoError):                        # rows that overlap: read by no call, as their lengths are not the ones that strides say
        call(A[:1].expand(8, 64), W, s, 32)
    with pytest.raises(tao.TaoError):
        call(A, W[:1].expand(16, 32), s, 32)
    with pytest.raises(tao.TaoError):
        call(A, W, torch.ones((16, 4), device="cuda"), 16)


def step(tao, A, W, s, z, inv, pos, gq, gk, y=None):
    """Queries, keys and values of a decode step from 4-bit weights; then the tables of the positions, and norm and rotation of the queries and keys where they lie."""
    y, tau = tao.tao_bound_linear_int4(A, W, s, 128, zero=z)
    tables = tao.tao_bound_rope_tables(inv, pos)
    rows = torch.arange(len(pos), device="cuda")
    x = y.view(len(pos), -1, 64)[:, :10]
    h = tao.tao_bound_norm_rope(x, tables[0], tables[1], gamma=gq, gamma_k=gk, heads_k=2, positions=rows, tau_cos=tables[2], tau_sin=tables[3])
    return (y, tau) + tables + h


def test_a_decode_step(tao):
    """The three operators together, eagerly and as a captured graph that is replayed on new inputs."""
    rng = np.random.default_rng(9)
    M, K, N = 6, 256, 12 * 64
    q, s, z = rng.integers(0, 16, (N, K)).astype(np.uint8), rng.uniform(0.001, 0.02, (N, 2)).astype(F), rng.integers(6, 11, (N, 2)).astype(np.uint8)
    inv = (1e6 ** (-np.arange(32) / 32)).astype(F)
    gq, gk = (rng.normal(1, 0.1, 64).astype(F) for _ in range(2))
    A = [rng.normal(0, 1, (M, K)).astype(F) for _ in range(3)]
    pos = [rng.integers(0, 50000, M) for _ in range(3)]
    fixed = cuda(int4.pack(q), s, z, inv)
    gains = cuda(gq, gk)
    eager = []
    for a, p in zip(A, pos):
        ad, pd = cuda(a, p)
        got = step(tao, ad, *fixed, pd, *gains)
        assert_product(got[:2], a, q, s, 128, z, None)
        tables = rotary.rope_tables(p, inv)
        for g, e in zip(got[4:6], tables[2:]):
            assert_bound(g.cpu().numpy(), e)
        arrays = [t.cpu().numpy() for t in got]
        y, tau = rotary.norm_rope(arrays[0].reshape(M, -1, 64)[:, :10], arrays[2], arrays[3], 64, gamma_q=gq, gamma_k=gk, heads_k=2, tau_cos=arrays[4], tau_sin=arrays[5])
        assert_bound(arrays[7], tau)
        assert (np.abs(arrays[6].astype(L) - y) <= tau).all()
        for alpha, off, accept in ((1.0, 0.0, 1), (1.0, 2.0, 0), (2.0, 1.9, 1)):
            claim = (got[6].double() + off * got[7].double()).float()
            pf = tao.tao_bound_check_norm_rope(got[0].view(M, -1, 64)[:, :10], got[2], got[3], claim, gamma=gains[0], gamma_k=gains[1], heads_k=2, positions=torch.arange(M, device="cuda"),
                                               tau_cos=got[4], tau_sin=got[5], alpha=alpha)
            assert pf["accept"] == accept
        eager.append([t.clone() for t in got])
    static_a, static_p = cuda(A[0], pos[0])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(tao, static_a, *fixed, static_p, *gains)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(tao, static_a, *fixed, static_p, *gains)
    for round_ in range(2):
        for a, p, expect in zip(A, pos, eager):
            static_a.copy_(torch.from_numpy(a))
            static_p.copy_(torch.from_numpy(p))
            graph.replay()
            torch.cuda.synchronize()
            other = step(tao, static_a * 2, *fixed, static_p, *gains)       # eager work between the replays
            for g, e in zip(captured, expect):
                assert torch.equal(g, e)
            del other


def test_calls_on_two_streams(tao):
    o = operands(9, 300, 1024, 128, 2, True)
    A, W, s, z = cuda(o[0], int4.pack(o[1]), o[2], o[4])
    y, tau = tao.tao_bound_linear_int4(A, W, s, 128, zero=z)
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream() for _ in range(2)], []
    for n in range(6):
        with torch.cuda.stream(streams[n % 2]):
            results.append((tao.tao_bound_linear_int4(A, W, s, 128, zero=z),
                            tao.tao_bound_check_linear_int4(A, W, s, 128, y, zero=z, readback=False,
                                                            ws=torch.empty(tao.tao_bound_check_linear_int4_workspace_bytes(9, 300, 1024), dtype=torch.uint8, device="cuda"))))
    torch.cuda.synchronize()
    for (y2, t2), pf in results:
        assert torch.equal(y, y2) and torch.equal(tau, t2) and tao.read_profile(pf)["accept"] == 1


# ------------------------------------------------------------------ workspaces: digits (16 tokens, 64 columns), parts of the reduction, both

WORKSPACES = [(16, 10300, 200, 128), (2, 96, 12288, 128), (5, 4200, 6200, 160)]


@pytest.mark.parametrize("M,N,K,group", WORKSPACES)
def test_two_streams_have_workspaces_of_their_own(tao, M, N, K, group):
    """Products and checks of different operands enqueued in turn on two streams, each with the workspace that the binding keeps for its stream."""
    assert tao.tao_linear_int4_workspace_bytes(M, N, K) > 0
    streams, data, expect, got = [torch.cuda.Stream() for _ in range(2)], [], [], []
    for n in range(2):
        A, q, s, _, z, _ = operands(M, N, K, group, 40 + n, True)
        data.append(cuda(A, int4.pack(q), s, z))
        own = torch.empty(tao.tao_linear_int4_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
        expect.append(tao.tao_bound_linear_int4(data[n][0], data[n][1], data[n][2], group, zero=data[n][3], ws=own))
        assert_product(expect[n], A, q, s, group, z, None)
    torch.cuda.synchronize()
    for i in range(12):
        n = i % 2
        A, W, s, z = data[n]
        with torch.cuda.stream(streams[n]):
            got.append((n, tao.tao_bound_linear_int4(A, W, s, group, zero=z), tao.tao_bound_check_linear_int4(A, W, s, group, expect[n][0], zero=z, readback=False)))
    torch.cuda.synchronize()
    kept = [tao._ws_cache[(torch.cuda.current_device(), stream.cuda_stream)] for stream in streams]
    assert min(k.numel() for k in kept) >= tao.tao_bound_check_linear_int4_workspace_bytes(M, N, K) and kept[0].data_ptr() != kept[1].data_ptr()
    for n, (y, tau), pf in got:
        assert torch.equal(y, expect[n][0]) and torch.equal(tau, expect[n][1])
        pf = tao.read_profile(pf)
        assert pf["accept"] == 1 and pf["max_rel"] == 0.0 and pf["n"] == M * N


@pytest.mark.parametrize("M,N,K,group", WORKSPACES)
def test_captured_products_keep_their_workspaces(tao, M, N, K, group):
    """Two graphs of a product and its check on one stream, replayed in turn on new inputs, with eager products between the replays that use the shared workspace and make it grow."""
    A, q, s, _, z, _ = operands(M, N, K, group, 50, True)
    W, sd, zd = cuda(int4.pack(q), s, z)
    inputs = [torch.from_numpy((A * F(f)).astype(F)).cuda() for f in (1.0, -0.75, 3.1)]
    expect = [tao.tao_bound_linear_int4(a, W, sd, group, zero=zd) for a in inputs]
    assert_product(expect[1], (A * F(-0.75)).astype(F), q, s, group, z, None)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        for n in range(2):
            a, claim = inputs[0].clone(), expect[0][0].clone()
            tao.tao_bound_check_linear_int4(a, W, sd, group, claim, zero=zd, readback=False)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = tao.tao_bound_linear_int4(a, W, sd, group, zero=zd)
                pf = tao.tao_bound_check_linear_int4(a, W, sd, group, claim, zero=zd, readback=False)
            graphs.append((graph, a, claim, out, pf))
    torch.cuda.current_stream().wait_stream(stream)
    for i in range(6):
        for n, (graph, a, claim, out, pf) in enumerate(graphs):
            k = (i + n) % 3
            a.copy_(inputs[k])
            claim.copy_(expect[k][0])
            if i == 4:
                claim[M - 1, N - 1] = float("nan")
            graph.replay()
            between = tao.tao_bound_linear_int4(inputs[(k + 1) % 3].repeat(1 + i, 1), W, sd, group, zero=zd)       # eager, on the same stream, of more tokens each time
            torch.cuda.synchronize()
            assert torch.equal(out[0], expect[k][0]) and torch.equal(out[1], expect[k][1])
            assert tao.read_profile(pf)["violations"] == (1 if i == 4 else 0)
            if i == 0:
                assert torch.equal(between[0], expect[(k + 1) % 3][0])


# ------------------------------------------------------------------ the borders of digits that are formed once (and of joined parts): every shape of tile

ROWS = [(8, 8209, 130, 32), (16, 10300, 200, 128), (40, 11000, 130, 64), (100, 10000, 129, 128), (5, 4200, 6200, 160)]
JOINED = [(2, 96, 12288, 128), (24, 2100, 8300, 128)]


@pytest.mark.parametrize("M,N,K,group", ROWS + JOINED)
@pytest.mark.parametrize("zero", [False, True])
def test_larger_products_whose_operands_end_where_their_memory_ends(tao, M, N, K, group, zero):
    assert tao.tao_linear_int4_workspace_bytes(M, N, K) > 0
    A, q, s, _, z, b = o = operands(M, N, K, group, 3, zero, True)
    expect = run(tao, *o)
    assert_product(expect, *o)
    got = tao.tao_bound_linear_int4(at_the_end(A), at_the_end(int4.pack(q)), at_the_end(s), group, zero=None if z is None else at_the_end(z), bias=at_the_end(b))
    assert torch.equal(got[0], expect[0]) and torch.equal(got[1], expect[1])


def strided_rows(t, step, at=0):
    """A copy of t whose rows lie `step` elements apart; what lies between is not touched."""
    return torch.empty(at + len(t) * step, dtype=t.dtype, device="cuda").as_strided(t.shape, (step, 1), at).copy_(t)


@pytest.mark.parametrize("M,N,K,group", ROWS[:3] + ROWS[4:] + JOINED[:1])
def test_larger_products_beyond_32_bits(tao, M, N, K, group):
    """Rows of A, of W, and of the outputs and claims so far apart that the last ones lie more than 2^31 elements on."""
    assert tao.tao_linear_int4_workspace_bytes(M, N, K) > 0
    A, q, s, _, z, b = operands(M, N, K, group, 4, True, True)
    Ad, Wd, sd, zd, bd = cuda(A, int4.pack(q), s, z, b)
    expect = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd)
    for a, w in ((strided_rows(Ad, 2 ** 31 // M + 2 ** 20), Wd), (Ad, strided_rows(Wd, 2 ** 31 // N + 2 ** 18, 16))):
        got = tao.tao_bound_linear_int4(a, w, sd, group, zero=zd, bias=bd)
        assert torch.equal(got[0], expect[0]) and torch.equal(got[1], expect[1])
        del a, w
    step = 2 ** 31 // M + 2 ** 20
    assert (M - 1) * step > 2 ** 31 - 2 ** 31 // M
    y, tau = strided_rows(0 * expect[0], step), strided_rows(0 * expect[0], step)
    product, check = outputs_through_the_c_abi(tao, Ad, Wd, sd, zd, bd, group, y, tau, step)
    assert product() == 0 and torch.equal(y, expect[0]) and torch.equal(tau, expect[1])
    y[M - 1, N - 1] += 2 * tau[M - 1, N - 1]
    pf = check(y)
    assert pf["n"] == M * N and pf["violations"] == 1


def outputs_through_the_c_abi(tao, A, W, s, z, b, group, y, tau, ldy):
    """The product into rows ldy apart, and the check of claims laid out like that."""
    (M, K), N = A.shape, len(W)
    ws = torch.empty(max(256, tao.tao_bound_check_linear_int4_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    front = [t.data_ptr() if t is not None else None for t in (A, W, s, z)] + [group, None if b is None else b.data_ptr()]
    dims = (M, N, K, K, (K + 1) // 2, ldy)
    L = tao.lib()

    def product():
        return L.tao_bound_linear_int4(*front, y.data_ptr(), tau.data_ptr(), *dims, None, ws.data_ptr(), ws.numel(), tao._stream())

    def check(claimed):
        out = tao.new_profile_buffer(A.device)
        assert L.tao_bound_check_linear_int4(*front, None, claimed.data_ptr(), *dims, 1.0, 1e-12, None, out.data_ptr(), ws.data_ptr(), ws.numel(), tao._stream()) == 0
        return tao.read_profile(out)
    return product, check


@pytest.mark.parametrize("M,N,K,group", ROWS + JOINED + [(20000, 48, 1000, 64)])
def test_larger_products_into_wide_rows(tao, M, N, K, group):
    """Outputs in rows of N + 9 elements, claims checked there too; what lies between stays as it was.  The last size goes through in slabs of tokens."""
    assert tao.tao_linear_int4_workspace_bytes(M, N, K) > 0
    A, q, s, _, z, b = operands(M, N, K, group, 5, True, True)
    Ad, Wd, sd, zd, bd = cuda(A, int4.pack(q), s, z, b)
    expect = tao.tao_bound_linear_int4(Ad, Wd, sd, group, zero=zd, bias=bd)
    y, tau = torch.full((M, N + 9), 7.0, device="cuda"), torch.full((M, N + 9), 7.0, device="cuda")
    product, check = outputs_through_the_c_abi(tao, Ad, Wd, sd, zd, bd, group, y, tau, N + 9)
    assert product() == 0 and torch.equal(y[:, :N], expect[0]) and torch.equal(tau[:, :N], expect[1])
    assert bool((y[:, N:] == 7).all()) and bool((tau[:, N:] == 7).all())
    at = (0, M // 2, M - 1)
    for i in at:
        y[i, N - 1] += 2 * tau[i, N - 1]
    pf = check(y)
    assert pf["n"] == M * N and pf["violations"] == len(set(at))


def test_more_outputs_than_a_launch_has_wavefronts_for(tao):
    """The kernel of any size and the check that joins: their wavefronts and lanes take a second output, in a last trip that is not whole."""
    M, N, K, seam = 7, 42859, 8, 262144
    assert seam < M * N < 2 * seam
    A, q, s, _, z, b = operands(M, N, K, K, 6, True, True)
    got = run(tao, A, q, s, K, z, b)
    cols = np.concatenate([np.arange(40), np.arange(seam // M - 40, seam // M + 40), np.arange(N - 40, N)])       # (outputs go out column by column)
    assert_product([t[:, torch.from_numpy(cols).cuda()] for t in got], A, q[cols], s[cols], K, z[cols], b[cols])
    y, tau = got
    claimed = y.clone().view(-1)
    at = torch.tensor([0, seam - 1, seam, M * N - 1], device="cuda")
    claimed[at] += 3 * tau.view(-1)[at]
    claimed = claimed.view(M, N)
    pf = tao.tao_bound_check_linear_int4(*cuda(A, int4.pack(q), s), K, claimed, zero=cuda(z)[0], bias=cuda(b)[0])
    assert pf["violations"] == 4
    assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy()))
