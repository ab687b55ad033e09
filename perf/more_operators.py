"""Operators of a decoder's projections and positions that a verifier re-executes, bounds and checks in one call: the tables of
the rotary embedding from positions, the RMS norm of every query and key head with the rotation of (part of) it, and the matrix
product of binary32 activations with 4-bit weights that have a scale, and possibly a zero point, for each group.

`run` takes a case through the library where `own` is true and through elementary torch operations where it is
false; `exact` is the same in 64 bits from the definitions.  Everything is synthetic and made on the GPU from the seed.

    tables     c = m cos(p f), s = m sin(p f) of position p and frequency f (m: the scaling of long contexts); their bounds hold
               a rounding of p, of the angle, the function's own error, a rounding for m
    rotation   h = x r g, r = 1/sqrt(mean(x^2) + eps) per head (or h = x), then y_a = h_a c - h_b s, y_b = h_b c + h_a s on
               the pairs of the head's first elements; the others are h
    product    y = sum_k a_k (q_k - z_g) s_g + b, g = k / group; each term is rounded K + 1 times at most (K + 2 with a bias)
"""
import math

import torch

own = False

U = 2.0 ** -24
C_DIV = C_RSQRT = 2.0                  # accuracies of the default model, in units of U
C_SIN = C_COS = 4.0
EPS_REL = 1e-12
NBINS = 2048
NONE = dict(check=False, claim="none")


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # a decode step of 64 sequences, each at a position of its own
        dict(name="tables_step", kind="tables", npos=64, half=64, far=40960, scale=1.0),
        # the whole table of a context that was made 32 times longer, with the amplitude that goes with it
        dict(name="tables_long", kind="tables", npos=131072, half=64, far=0, scale=1.3465735902799727),
        # one token: the 32 query and 8 key heads that the fused projection of a decode step leaves
        dict(name="heads_token", kind="heads", tokens=1, heads_q=32, heads_k=8, d=128, rot=128, norm=True, interleaved=False, errors=False, fused=True, **NONE),
        # a prefill's queries and keys, read where the fused projection left them
        dict(name="heads_prefill", kind="heads", tokens=2048, heads_q=32, heads_k=8, d=128, rot=128, norm=True, interleaved=False, errors=False, fused=True, **NONE),
        # no norm, part of a head in neighbouring pairs, a table with bounds of its own; sizes that fit no vector
        dict(name="heads_partial", kind="heads", tokens=777, heads_q=13, heads_k=0, d=90, rot=26, norm=False, interleaved=True, errors=True, fused=False, **NONE),
        # a prefill's queries and keys checked against a proposer that leaves the bound in places
        dict(name="heads_check", kind="heads", tokens=2048, heads_q=32, heads_k=8, d=128, rot=128, norm=True, interleaved=False, errors=False, fused=False, check=True, claim="perturbed"),
        # one token: the output projection of a decode step
        dict(name="int4_token", kind="int4", M=1, K=4096, N=4096, group=128, zero=False, bias=False, **NONE),
        # one token: the down projection, weights with zero points
        dict(name="int4_down", kind="int4", M=1, K=12288, N=4096, group=128, zero=True, bias=False, **NONE),
        # sixteen sequences in decode: the gate projection
        dict(name="int4_batch", kind="int4", M=16, K=4096, N=12288, group=128, zero=True, bias=True, **NONE),
        # sizes that fit no tile, no vector and no group
        dict(name="int4_ragged", kind="int4", M=5, K=1001, N=3001, group=32, zero=True, bias=True, **NONE),
        # a short prompt
        dict(name="int4_prompt", kind="int4", M=128, K=4096, N=4096, group=64, zero=False, bias=False, **NONE),
        # eight sequences in decode, the proposer's claim checked on the spot
        dict(name="int4_check", kind="int4", M=8, K=4096, N=12288, group=128, zero=False, bias=False, check=True, claim="honest"),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm, odd ones among them."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tables", "heads", "heads", "int4", "int4", "int4"])
    check = kind != "tables" and rng.random() < 0.4
    claim = rng.choice(["honest", "perturbed"]) if check else "none"
    if kind == "tables":
        half = rng.choice([16, 32, 48, 64, 64, _spread(rng, 1, 128)])
        return dict(kind=kind, npos=_spread(rng, 1, (1 << 23) // half), half=half, far=rng.choice([0, 4096, 131072, 1 << 20]), scale=rng.choice([1.0, 1.0, 1.0 + rng.random()]))
    if kind == "heads":
        d = rng.choice([64, 80, 96, 128, 128, 128, 256, _spread(rng, 2, 320)])
        while True:
            heads_q = _spread(rng, 1, 64)
            heads_k = rng.choice([0, _spread(rng, 1, heads_q)])
            tokens = _spread(rng, 1, 16384)
            if tokens * (heads_q + heads_k) * d <= 2048 * 40 * 128:
                break
        rot = rng.choice([d, d, d // 2, d // 4]) // 2 * 2
        return dict(kind=kind, tokens=tokens, heads_q=heads_q, heads_k=heads_k, d=d, rot=max(rot, 2), norm=rng.random() < 0.7, interleaved=rng.random() < 0.3,
                    errors=rng.random() < 0.3, fused=not check and rng.random() < 0.5, check=check, claim=claim)
    while True:
        M, K, N = rng.choice([1, _spread(rng, 1, 256)]), _spread(rng, 64, 16384), _spread(rng, 16, 16384)
        if rng.random() < 0.7:                          # widths of real layers are mostly multiples of 64
            K, N = (K + 63) // 64 * 64, (N + 63) // 64 * 64
        if M * K * N <= 128 * 4096 * 4096 and K * N <= 1 << 26:
            break
    return dict(kind=kind, M=M, K=K, N=N, group=rng.choice([32, 64, 128, 128, 256, K]), zero=rng.random() < 0.5, bias=rng.random() < 0.3, check=check, claim=claim)


# ------------------------------------------------------------------ inputs

def _randn(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda") * std


def _claims(g, y, tau, claim):
    """A proposer's output beside the verifier's y: a step of binary32 or two away, or f times the bound away.  A claim
    that rounding has put close to its bound is replaced by y, and so is one of an exact element."""
    if claim == "honest":
        moved = y.view(torch.int32) + torch.randint(-1, 2, y.shape, generator=g, device="cuda", dtype=torch.int32)
        claimed = torch.where((y.abs() > 1e-30) & (tau > 0), moved.view(torch.float32), y)
    else:
        f = torch.tensor([0.0, 0.5, 0.7, 2.0, -0.5, -0.7, -3.0, 0.0], device="cuda")
        claimed = (y.double() + (f[torch.randint(0, 8, y.shape, generator=g, device="cuda")] * tau).double()).float()
    share = (claimed.double() - y.double()).abs() / tau.double()
    return torch.where((share > 0.8) & (share < 1.25), y, claimed)


def _frequencies(g, half):
    theta = 1e6 * (0.5 + torch.rand((1,), generator=g, device="cuda"))
    return theta ** (-torch.arange(half, device="cuda", dtype=torch.float32) / half)


def _prepare_tables(c, g):
    # positions in order, or those of sequences of different lengths
    if c["far"]:
        positions = torch.randint(0, c["far"], (c["npos"],), generator=g, device="cuda")
    else:
        positions = torch.arange(c["npos"], device="cuda")
    return dict(positions=positions, inv_freq=_frequencies(g, c["half"]), scale=c["scale"])


def _prepare_heads(c, g):
    T, H, d, half = c["tokens"], c["heads_q"] + c["heads_k"], c["d"], c["rot"] // 2
    # queries and keys, with the values behind them where the projection is fused; heads of different sizes
    wide = _randn(g, (T, H + (c["heads_k"] or 1) if c["fused"] else H, d)) * torch.exp(_randn(g, (1, 1, d), 0.5))
    npos = min(4096, max(64, T))
    angles = torch.arange(npos, device="cuda").double()[:, None] * _frequencies(g, half).double()
    s = dict(x=wide[:, :H], cos=angles.cos().float(), sin=angles.sin().float(), tau_cos=None, tau_sin=None, gamma=None, gamma_k=None, eps=1e-6,
             positions=torch.randint(0, npos, (T,), generator=g, device="cuda"))
    if c["errors"]:
        s["tau_cos"], s["tau_sin"] = (t.abs() * (4 * U) + angles.float() * U for t in (s["cos"], s["sin"]))
    if c["norm"]:
        s["gamma"] = 1 + _randn(g, (d,), 0.1)
        s["gamma_k"] = 1 + _randn(g, (d,), 0.1) if c["heads_k"] else None
    if c["check"]:
        s["y_ref"], tau = _plain_heads(c, s)
        s["claimed"] = _claims(g, s["y_ref"], tau, c["claim"])
    return s


def _prepare_int4(c, g):
    M, K, N = c["M"], c["K"], c["N"]
    G = -(-K // c["group"])
    # nibbles of the usual spread around the middle, two to a byte; tokens of different sizes with a few large channels
    a = _randn(g, (M, K)) * torch.exp(_randn(g, (M, 1), 0.5))
    a[:, :: max(1, K // 16)] *= 8.0
    s = dict(A=a, W=torch.clamp(torch.round(_randn(g, (N, -(-K // 2) * 2), 3.0)) + 8, 0, 15).to(torch.uint8),
             scale=(0.5 + torch.rand((N, G), generator=g, device="cuda")) * 0.01,
             zero=torch.randint(6, 11, (N, G), generator=g, device="cuda", dtype=torch.uint8) if c["zero"] else None,
             bias=_randn(g, (N,), 0.5) if c["bias"] else None, group=c["group"])
    s["W"] = s["W"][:, 0::2] + 16 * s["W"][:, 1::2]
    if c["check"]:
        s["y_ref"], tau = _plain_int4(s)
        s["claimed"] = _claims(g, s["y_ref"], tau, c["claim"])
    return s


_PREPARE = dict(tables=_prepare_tables, heads=_prepare_heads, int4=_prepare_int4)


def _results(c):
    """The buffers that a program keeps for the results, and its workspace."""
    import paper_2510_16028_amd as tao
    device = torch.device("cuda", torch.cuda.current_device())
    bytes_ = lambda n: torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)
    made = lambda *shape: torch.empty(shape, device=device)
    if c["kind"] == "tables":
        return dict(cos=made(c["npos"], c["half"]), sin=made(c["npos"], c["half"]), tau_cos=made(c["npos"], c["half"]), tau_sin=made(c["npos"], c["half"]))
    if c["kind"] == "heads":
        shape = (c["tokens"], c["heads_q"] + c["heads_k"], c["d"])
        if c["check"]:
            return dict(out=tao.new_profile_buffer(device), ws=bytes_(tao.tao_check_workspace_bytes(shape[0] * shape[1] * shape[2])))
        return dict(y=made(*shape), tau=made(*shape))
    if c["check"]:
        return dict(out=tao.new_profile_buffer(device), ws=bytes_(tao.tao_bound_check_linear_int4_workspace_bytes(c["M"], c["N"], c["K"])))
    return dict(y=made(c["M"], c["N"]), tau=made(c["M"], c["N"]), ws=bytes_(tao.tao_linear_int4_workspace_bytes(c["M"], c["N"], c["K"])))


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return _PREPARE[case["kind"]](case, g)


def prepare(case, seed):
    return case, _inputs(case, seed), _results(case) if own else None


# ------------------------------------------------------------------ the plain forms

def _gamma(k):
    return k * U / (1 - k * U)


def _plain_tables(s):
    # angles of far positions, their cosines and their errors in 64 bits
    p, m = s["positions"].double()[:, None], s["scale"]
    angle = p * s["inv_freq"].double()
    e = torch.where(p.abs() > 1 / U, _gamma(2), _gamma(1)) * angle.abs()
    c, si = torch.cos(angle), torch.sin(angle)

    def bound(value, other, own_error):
        b = torch.minimum(torch.minimum(other.abs() * e + 0.5 * e * e, e), 1 + value.abs())
        b = b + own_error * U * (value.abs() + b)
        return abs(m) * (b if m == 1 else b + U * (value.abs() + b))
    return [(m * c).float(), (m * si).float(), bound(c, si, C_COS).float(), bound(si, c, C_SIN).float()]


def _plain_heads(c, s):
    x, d, rot = s["x"], c["d"], c["rot"]
    F, r, h = 0.0, 1.0, x
    if c["norm"]:
        squares = (x * x).sum(dim=-1, keepdim=True)
        v = squares / d
        e_v = ((_gamma(d - 1) * (1 + U) + U) * squares / d + C_DIV * U * v) / (1 - C_DIV * U)
        w = v + s["eps"]
        e_w = (e_v + U * w) / (1 - U)
        low = w - e_w
        low = torch.where(low > 0, low, float("nan"))
        r = w ** -0.5
        e_r = 0.5 * e_w * low ** -1.5 + C_RSQRT * U * low ** -0.5
        R = r + e_r
        F = e_r + U * R + U * R * (1 + U) ** 2
        g = s["gamma"][None, :].expand(c["heads_q"], d)
        if c["heads_k"]:
            g = torch.cat([g, s["gamma_k"][None, :].expand(c["heads_k"], d)])
        h = x * g
    # y = r rotated(h); an element's error before the rotation is F |h|
    at = s["positions"]
    co, si = s["cos"][at][:, None, :], s["sin"][at][:, None, :]
    tc, ts = (0.0, 0.0) if s["tau_cos"] is None else (s["tau_cos"][at][:, None, :], s["tau_sin"][at][:, None, :])
    if c["interleaved"]:
        a, b = h[..., 0:rot:2], h[..., 1:rot:2]
    else:
        a, b = h[..., :rot // 2], h[..., rot // 2:rot]
    k = _gamma(2) * (r + F) + F
    k_c, k_s = k * (co.abs() + tc) + r * tc, k * (si.abs() + ts) + r * ts
    ya, yb = r * (a * co - b * si), r * (b * co + a * si)
    ta, tb = a.abs() * k_c + b.abs() * k_s, b.abs() * k_c + a.abs() * k_s
    join = (lambda p, q: torch.stack([p, q], dim=-1).flatten(-2)) if c["interleaved"] else (lambda p, q: torch.cat([p, q], dim=-1))
    rest = h[..., rot:]
    return torch.cat([join(ya, yb), r * rest], dim=-1), torch.cat([join(ta, tb), F * rest.abs()], dim=-1)


def _weights(s, K):
    """(q - z) s in binary32: a whole number and one rounding."""
    q = torch.stack([s["W"] & 15, s["W"] >> 4], dim=-1).flatten(1)[:, :K].float()
    of = torch.arange(K, device=q.device) // s["group"]
    return (q - (8.0 if s["zero"] is None else s["zero"].float()[:, of])) * s["scale"][:, of]


def _plain_int4(s):
    K = s["A"].shape[1]
    w = _weights(s, K)
    y, m = s["A"] @ w.t(), s["A"].abs() @ w.abs().t()
    if s["bias"] is None:
        return y, _gamma(K + 1) * m
    return y + s["bias"], _gamma(K + 2) * (m + s["bias"].abs())


def _profile(claimed, ref, tau):
    """Elements outside their bounds, and the profile of the relative errors on bins of an eighth of an octave."""
    cd, rd = claimed.double().flatten(), ref.double().flatten()
    d = (cd - rd).abs()
    n = d.numel()
    violations = (~(d <= tau.double().flatten())).sum()
    e = (d / (rd.abs() + EPS_REL)).float()
    nan = torch.isnan(e)
    bins = torch.where(nan, NBINS - 1, e.view(torch.int32) >> 20)
    hist = torch.bincount(bins, minlength=NBINS)
    upto = torch.cumsum(hist, 0)
    ranks = torch.tensor([max(1, -(-n * a // b)) for a, b in ((1, 2), (99, 100), (999, 1000))], device=d.device)
    at = torch.searchsorted(upto, ranks)
    return dict(violations=violations.view(1), accept=(violations == 0).int().view(1), nan_count=nan.sum().view(1),
                max_rel=torch.where(nan, 0.0, e).amax().view(1), percentile_bins=at.int(), hist=hist)


def _run_plain(c, s):
    if c["kind"] == "tables":
        return _plain_tables(s)
    y, tau = _plain_heads(c, s) if c["kind"] == "heads" else _plain_int4(s)
    return _profile(s["claimed"], s["y_ref"], tau) if c["check"] else [y, tau]


# ------------------------------------------------------------------ the library's calls

def _fields(out):
    """The fields of a tao_profile in device memory."""
    words, halves = out[:24].view(torch.int64), out[24:56].view(torch.int32)
    return dict(violations=words[1:2], accept=halves[1:2], nan_count=words[2:3], max_rel=out[24:28].view(torch.float32),
                percentile_bins=halves[2:5], hist=out[64:].view(torch.int64))


def _run_own(c, s, r):
    import paper_2510_16028_amd as tao
    if c["kind"] == "tables":
        return list(tao.tao_bound_rope_tables(s["inv_freq"], s["positions"], scale=s["scale"], **r))
    if c["kind"] == "heads":
        given = dict(norm=tao.NORM_RMSNORM if c["norm"] else tao.NORM_NONE, gamma=s["gamma"], gamma_k=s["gamma_k"], heads_k=c["heads_k"], eps=s["eps"],
                     positions=s["positions"], tau_cos=s["tau_cos"], tau_sin=s["tau_sin"], interleaved=c["interleaved"])
        if c["check"]:
            return _fields(tao.tao_bound_check_norm_rope(s["x"], s["cos"], s["sin"], s["claimed"], y_ref=s["y_ref"], eps_rel=EPS_REL, readback=False, **given, **r))
        return list(tao.tao_bound_norm_rope(s["x"], s["cos"], s["sin"], **given, **r))
    given = dict(zero=s["zero"], bias=s["bias"])
    if c["check"]:
        return _fields(tao.tao_bound_check_linear_int4(s["A"], s["W"], s["scale"], s["group"], s["claimed"], y_ref=s["y_ref"], eps_rel=EPS_REL, readback=False, **given, **r))
    return list(tao.tao_bound_linear_int4(s["A"], s["W"], s["scale"], s["group"], **given, **r))


def run(state):
    case, s, r = state
    return _run_own(case, s, r) if r is not None else _run_plain(case, s)


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_tables(c, s):
    rows, scale = [], float(torch.tensor(c["scale"], dtype=torch.float32))
    for p in s["positions"].split(1 << 14):
        theta = torch.outer(p.double(), s["inv_freq"].double())
        steps = 1.0 + (p.double().abs() > 2.0 ** 24).double()
        moved = (theta.abs() * (steps * U / (1.0 - steps * U))[:, None])
        out = []
        for value, slope, own_error in ((theta.cos(), theta.sin(), 4.0), (theta.sin(), theta.cos(), 4.0)):
            through = torch.stack([slope.abs() * moved + moved ** 2 / 2.0, moved, 1.0 + value.abs()]).amin(0)
            through = through + own_error * U * (value.abs() + through)
            if scale != 1.0:
                through = (through + U * (value.abs() + through)) * abs(scale)
            out.append((value * scale, through))
        rows.append((out[0][0], out[1][0], out[0][1], out[1][1]))
    return [torch.cat(t) for t in zip(*rows)]


def _exact_heads(c, s):
    """The chain of the norm step by step, then each pair's products with their errors."""
    ys, taus = [], []
    d, rot, half = c["d"], c["rot"], c["rot"] // 2
    eps = float(torch.tensor(s["eps"], dtype=torch.float32))
    for x, at in zip(s["x"].split(512), s["positions"].split(512)):
        p = x.double()
        err = torch.zeros_like(p)
        if c["norm"]:
            total = (p * p).sum(-1, keepdim=True)
            g_n = (d - 1) * U / (1.0 - (d - 1) * U)
            err_total = g_n * total * (1.0 + U) + U * total
            mean = total / d
            err_mean = (err_total / d + 2.0 * U * mean) / (1.0 - 2.0 * U)
            w = mean + eps
            err_w = (err_mean + U * w) / (1.0 - U)
            w_lo = torch.where(w > err_w, w - err_w, torch.full_like(w, math.nan))
            root = 1.0 / w.sqrt()
            err_root = err_w / (2.0 * w_lo * w_lo.sqrt()) + 2.0 * U / w_lo.sqrt()
            most = root + err_root
            gain = s["gamma"].double().repeat(c["heads_q"], 1)
            if c["heads_k"]:
                gain = torch.vstack([gain, s["gamma_k"].double().repeat(c["heads_k"], 1)])
            size = (p * gain).abs()
            p = p * gain * root
            err = size * err_root + U * size * most + U * size * most * (1.0 + U) ** 2
        if c["interleaved"]:
            ia = torch.arange(0, rot, 2, device="cuda")
            ib = ia + 1
        else:
            ia = torch.arange(half, device="cuda")
            ib = ia + half
        cos, sin = (s[k].double()[at].unsqueeze(1) for k in ("cos", "sin"))
        ec, es = (torch.zeros_like(cos), torch.zeros_like(sin)) if s["tau_cos"] is None else (s[k].double()[at].unsqueeze(1) for k in ("tau_cos", "tau_sin"))
        y, tau = p.clone(), err.clone()

        def product(v, ev, t, et):                           # its value's largest size, and how far it may be off
            return (v.abs() + ev) * (t.abs() + et), ev * (t.abs() + et) + v.abs() * et
        g2 = 2.0 * U / (1.0 - 2.0 * U)
        pa, ea, pb, eb = p[..., ia], err[..., ia], p[..., ib], err[..., ib]
        for to, first, second, sign in ((ia, (pa, ea), (pb, eb), -1.0), (ib, (pb, eb), (pa, ea), 1.0)):
            m1, e1 = product(*first, cos, ec)
            m2, e2 = product(*second, sin, es)
            y[..., to] = first[0] * cos + sign * second[0] * sin
            tau[..., to] = e1 + e2 + g2 * (m1 + m2)
        ys.append(y)
        taus.append(tau)
    return torch.cat(ys), torch.cat(taus)


def _exact_int4(c, s):
    K, N, group = c["K"], c["N"], c["group"]
    a = s["A"].double()
    y, size = torch.zeros((c["M"], N), dtype=torch.float64, device="cuda"), torch.zeros((c["M"], N), dtype=torch.float64, device="cuda")
    step = max(group, 1024 // group * group)                 # whole groups at a time
    for k0 in range(0, K, step):
        k1 = min(K, k0 + step)
        digits = torch.empty((N, (k1 - k0 + 1) // 2 * 2), dtype=torch.float64, device="cuda")
        packed = s["W"][:, k0 // 2:(k1 + 1) // 2].double()   # (groups begin at even places)
        digits[:, 1::2] = torch.floor(packed / 16.0)
        digits[:, 0::2] = packed - 16.0 * digits[:, 1::2]
        of = torch.div(torch.arange(k0, k1, device="cuda"), group, rounding_mode="floor")
        middle = torch.full((N, k1 - k0), 8.0, dtype=torch.float64, device="cuda") if s["zero"] is None else s["zero"].double().index_select(1, of)
        w = (digits[:, :k1 - k0] - middle) * s["scale"].double().index_select(1, of)
        y += torch.mm(a[:, k0:k1], w.t().contiguous())
        size += torch.mm(a[:, k0:k1].abs(), w.abs().t().contiguous())
    steps = K + 1.0
    if s["bias"] is not None:
        b = s["bias"].double()
        y, size, steps = y + b, size + b.abs(), steps + 1.0
    return y, size * (steps * U / (1.0 - steps * U))


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "tables":
        return _exact_tables(c, s)
    y, tau = _exact_heads(c, s) if c["kind"] == "heads" else _exact_int4(c, s)
    if not c["check"]:
        return [y, tau]
    y = s["y_ref"]
    away = (s["claimed"].double() - y.double()).abs()
    error = (away / (y.double().abs() + EPS_REL)).float().flatten()
    outside = int((away > tau).sum())
    # counts between the lower edges of the bins, up to that of the infinite errors
    ordered = error.sort().values
    edges = (torch.arange(2041, device="cuda", dtype=torch.int32) << 20).view(torch.float32)
    counts = torch.zeros(NBINS, dtype=torch.int64, device="cuda")
    counts[:2040] = torch.diff(torch.searchsorted(ordered, edges))
    ranks = [max(1, math.ceil(error.numel() * a / b)) for a, b in ((1, 2), (99, 100), (999, 1000))]
    bins = torch.stack([ordered[k - 1] for k in ranks]).view(torch.int32) // (1 << 20)
    one = lambda v, t: torch.tensor([v], dtype=t, device="cuda")
    return dict(violations=one(outside, torch.int64), accept=one(int(outside == 0), torch.int32), nan_count=one(0, torch.int64),
                max_rel=ordered[-1:], percentile_bins=bins.int(), hist=counts)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Bytes: operands, claims and re-executed outputs read once, outputs and bounds written once (of a table, the rows that are looked
    up).  Operations: the product's multiplications and additions, once for the output and once for the bound; for the others a
    nominal count per element (cosine, sine and bounds; norm, rotation and bound)."""
    c, profile = case, 64 + 8 * NBINS
    if c["kind"] == "tables":
        n = c["npos"] * c["half"]
        return dict(bytes=8 * c["npos"] + 4 * c["half"] + 16 * n, flops=80 * n)
    if c["kind"] == "heads":
        n = c["tokens"] * (c["heads_q"] + c["heads_k"]) * c["d"]
        rows = min(c["tokens"], min(4096, max(64, c["tokens"])))
        tables = rows * c["rot"] // 2 * (16 if c["errors"] else 8) + 8 * c["tokens"]
        return dict(bytes=12 * n + tables + (8 * c["d"] if c["norm"] else 0) + (profile if c["check"] else 0), flops=20 * n)
    M, K, N = c["M"], c["K"], c["N"]
    G = -(-K // c["group"])
    operands = 4 * M * K + N * (-(-K // 2)) + N * G * (5 if c["zero"] else 4) + (4 * N if c["bias"] else 0)
    return dict(bytes=operands + 8 * M * N + (profile if c["check"] else 0), flops=4 * M * K * N)
