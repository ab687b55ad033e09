"""Operators that a verifier re-executes, bounds and checks in one call: the 8-bit matrix product with a scale for
each token and channel, the quantisation of its rows, and group norm with an activation on channels-last features.

`run` takes a case through the library where `own` is true and through elementary torch operations where it is
false; `exact` is the same in 64 bits from the definitions.  Everything is synthetic and made on the GPU from the seed.

    product    y = S sa_i sw_j + b_j, S = sum_k A_ik W_jk in whole numbers; two roundings for the scales, one more
               where S is too large for binary32, one for the bias
    quantised  s = max|x| / 127, q = round(x / s)
    group norm p = (x - mean) / sqrt(var + eps) * gamma + beta per sample and group, then SiLU, ReLU or nothing
"""
import math

import torch

own = False

U = 2.0 ** -24
C_DIV = C_RSQRT = C_EXP = 2.0          # accuracies of the default model, in units of U
EPS_REL = 1e-12
NBINS = 2048


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # one token against a large weight: a projection of a decode step
        dict(name="int8_token", kind="int8", M=1, K=4096, N=4096, bias=False, check=False, claim="none"),
        # the fused query, key and value projection of an encoder block at sequence length 512
        dict(name="int8_encoder", kind="int8", M=512, K=768, N=2304, bias=True, check=False, claim="none"),
        # sizes that fit no tile and no vector
        dict(name="int8_ragged", kind="int8", M=1111, K=1001, N=3001, bias=True, check=False, claim="none"),
        # the stress product, output and bound handed over
        dict(name="int8_stress", kind="int8", M=8192, K=8192, N=8192, bias=False, check=False, claim="none"),
        # a handful of tokens in decode, an honest proposer's claim checked on the spot
        dict(name="int8_decode_check", kind="int8", M=8, K=4096, N=12288, bias=False, check=True, claim="honest"),
        # the gate projection of a decoder layer's prefill, a proposer that leaves the bound in places
        dict(name="int8_prefill_check", kind="int8", M=2048, K=4096, N=12288, bias=True, check=True, claim="perturbed"),
        # activations of a handful of tokens, and those of a prefill's down projection
        dict(name="quantize_decode", kind="quantize", rows=8, cols=4096),
        dict(name="quantize_prefill", kind="quantize", rows=2048, cols=12288),
        # the innermost stage of an image decoder: few pixels, many channels
        dict(name="groupnorm_inner", kind="norm", batch=2, positions=64, channels=1280, groups=32, act="silu", check=False, claim="none"),
        # its last stage: 512 x 512 pixels of 128 channels
        dict(name="groupnorm_outer", kind="norm", batch=1, positions=512 * 512, channels=128, groups=32, act="silu", check=False, claim="none"),
        # the entry of a transformer block on 64 x 64 features, checked (ten channels a group)
        dict(name="groupnorm_entry_check", kind="norm", batch=2, positions=64 * 64, channels=320, groups=32, act="none", check=True, claim="honest"),
        # a middle stage of a batch, checked, a proposer that leaves the bound in places
        dict(name="groupnorm_batch_check", kind="norm", batch=4, positions=128 * 128, channels=512, groups=32, act="silu", check=True, claim="perturbed"),
    ]


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm, odd ones among them."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["int8", "int8", "int8", "quantize", "norm", "norm"])
    check = rng.random() < 0.5
    claim = rng.choice(["honest", "perturbed"]) if check else "none"
    if kind == "int8":
        while True:
            M, K, N = _spread(rng, 1, 8192), _spread(rng, 16, 16384), _spread(rng, 16, 16384)
            if rng.random() < 0.6:                      # widths of real layers are mostly multiples of 64
                K, N = (K + 63) // 64 * 64, (N + 63) // 64 * 64
            if M * K * N <= 2048 * 4096 * 12288 and M * N <= 1 << 25:
                break
        return dict(kind=kind, M=M, K=K, N=N, bias=rng.random() < 0.5, check=check, claim=claim)
    if kind == "quantize":
        cols = _spread(rng, 16, 16384)
        return dict(kind=kind, rows=_spread(rng, 1, max(1, (1 << 24) // cols)), cols=cols)
    while True:
        groups = rng.choice([1, 4, 8, 16, 32, 32, 32, 64])
        per = _spread(rng, 1, 80)
        batch, positions = _spread(rng, 1, 16), _spread(rng, 16, 512 * 512)
        if groups * per >= 16 and batch * positions * groups * per <= 1 << 25 and positions * per <= 1 << 21:
            break
    return dict(kind=kind, batch=batch, positions=positions, channels=groups * per, groups=groups,
                act=rng.choice(["silu", "silu", "relu", "none"]), check=check, claim=claim)


# ------------------------------------------------------------------ inputs

def _randn(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda") * std


def _claims(g, y, tau, claim):
    """A proposer's output beside the verifier's y: a step of binary32 or two away, or f times the bound away.  A claim
    that rounding has put close to its bound is replaced by y."""
    if claim == "honest":
        moved = y.view(torch.int32) + torch.randint(-1, 2, y.shape, generator=g, device="cuda", dtype=torch.int32)
        claimed = torch.where(y.abs() > 1e-30, moved.view(torch.float32), y)
    else:
        f = torch.tensor([0.0, 0.5, 0.7, 2.0, -0.5, -0.7, -3.0, 0.0], device="cuda")
        claimed = (y.double() + (f[torch.randint(0, 8, y.shape, generator=g, device="cuda")] * tau).double()).float()
    share = (claimed.double() - y.double()).abs() / tau.double()
    return torch.where((share > 0.8) & (share < 1.25), y, claimed)


def _prepare_int8(c, g):
    M, K, N = c["M"], c["K"], c["N"]
    # rows of activations of different sizes, weights of the usual spread, both already in 8 bits
    s = dict(A=torch.randint(-127, 128, (M, K), generator=g, device="cuda", dtype=torch.int8),
             W=torch.clamp(torch.round(_randn(g, (N, K), 32.0)), -127, 127).to(torch.int8),
             sa=(1.0 + torch.rand((M,), generator=g, device="cuda")) * 0.02,
             sw=(1.0 + torch.rand((N,), generator=g, device="cuda")) * 0.0005,
             bias=_randn(g, (N,), 0.5) if c["bias"] else None)
    if c["check"]:
        y, tau = _plain_product(s)
        s["claimed"] = _claims(g, y, tau, c["claim"])
    return s


def _prepare_quantize(c, g):
    # tokens of different sizes with a few large channels, as activations have them
    x = _randn(g, (c["rows"], c["cols"])) * torch.exp(_randn(g, (c["rows"], 1)))
    x[:, :: max(1, c["cols"] // 16)] *= 8.0
    return dict(x=x)


def _prepare_norm(c, g):
    B, P, C = c["batch"], c["positions"], c["channels"]
    s = dict(x=_randn(g, (B, P, C)) + _randn(g, (B, 1, C), 0.5), gamma=1 + _randn(g, (C,), 0.1), beta=_randn(g, (C,), 0.1), eps=1e-5)
    if c["check"]:
        y, tau = _plain_norm(c, s)
        s["y_ref"] = y
        s["claimed"] = _claims(g, y, tau, c["claim"])
    return s


_PREPARE = dict(int8=_prepare_int8, quantize=_prepare_quantize, norm=_prepare_norm)


def _results(c):
    """The buffers that a program keeps for the results, and its workspace."""
    import paper_2510_16028_amd as tao
    device = torch.device("cuda", torch.cuda.current_device())
    empty = lambda n: torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)
    if c["kind"] == "quantize":
        return dict(q=torch.empty((c["rows"], c["cols"]), dtype=torch.int8, device=device), scale=torch.empty((c["rows"],), device=device))
    shape = (c["M"], c["N"]) if c["kind"] == "int8" else (c["batch"], c["positions"], c["channels"])
    geometry = None if c["kind"] == "int8" else (c["batch"], c["positions"], c["channels"], c["groups"])
    if c["check"]:
        need = tao.tao_check_workspace_bytes(shape[0] * shape[1]) if geometry is None else tao.tao_bound_check_groupnorm_act_workspace_bytes(*geometry)
        return dict(out=tao.new_profile_buffer(device), ws=empty(need))
    r = dict(y=torch.empty(shape, device=device), tau=torch.empty(shape, device=device))
    if geometry is not None:
        r["ws"] = empty(tao.tao_groupnorm_act_workspace_bytes(*geometry))
    return r


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return _PREPARE[case["kind"]](case, g)


def prepare(case, seed):
    return case, _inputs(case, seed), _results(case) if own else None


# ------------------------------------------------------------------ the plain forms

def _gamma(k):
    return k * U / (1 - k * U)


def _whole_sums(A, W):
    """sum_k A_ik W_jk: every partial sum is a whole number, which binary32 holds up to 2^24."""
    t = torch.float32 if A.shape[1] * 127 * 127 <= 1 << 24 else torch.float64
    return A.to(t) @ W.to(t).t()


def _plain_product(s):
    S = _whole_sums(s["A"], s["W"])
    large = S.abs() * U > 1
    v = S.float() * s["sa"][:, None] * s["sw"]
    g = torch.where(large, _gamma(3), _gamma(2)).float()
    if s["bias"] is None:
        return v, g * v.abs()
    y = v + s["bias"]
    spread = g * v.abs()
    return y, spread + U * (y.abs() + spread)


def _plain_quantize(s):
    x = s["x"]
    scale = x.abs().amax(dim=1) / 127
    q = torch.clamp(torch.round(x / torch.where(scale > 0, scale, 1.0)[:, None]), -127, 127)
    return [q * scale[:, None], scale]


def _plain_norm(c, s):
    B, P, C, G = c["batch"], c["positions"], c["channels"], c["groups"]
    x = s["x"].view(B, P, G, C // G)
    n, over = P * (C // G), (1, 3)
    gn = _gamma(n - 1)
    # the statistics: sums of up to millions of terms, in 64 bits
    mean = x.sum(dim=over, keepdim=True, dtype=torch.float64) / n
    e_mean = (gn * x.abs().sum(dim=over, keepdim=True, dtype=torch.float64) / n + C_DIV * U * mean.abs()) / (1 - C_DIV * U)
    d = (x - mean).float()
    s1 = d.abs().sum(dim=over, keepdim=True, dtype=torch.float64)
    s2 = (d * d).sum(dim=over, keepdim=True, dtype=torch.float64)
    # errors of d, of its square's sum, of the variance and of its inverse root
    up, ep = U / (1 - U), e_mean / (1 - U)
    sum_big2 = (1 + up) ** 2 * s2 + 2 * (1 + up) * ep * s1 + n * ep * ep
    e_sum = gn * (1 + U) * sum_big2 + up * (2 + up) * s2 + ep * (2 + 2 * up) * s1 + n * ep * ep + U * sum_big2
    var = s2 / n
    e_var = (e_sum / n + C_DIV * U * var) / (1 - C_DIV * U)
    w = var + torch.tensor(s["eps"], dtype=torch.float32).item()
    e_w = (e_var + U * w) / (1 - U)
    low = w - e_w
    low = torch.where(low > 0, low, float("nan"))
    r = w ** -0.5
    e_r = 0.5 * e_w * low ** -1.5 + C_RSQRT * U * low ** -0.5
    k = e_r + U * (r + e_r)
    k1 = (1 + U) * ((1 + up) * k + r * up) + U * r
    k0 = (1 + U) * ep * (k + r)
    gamma, beta = s["gamma"].view(G, -1), s["beta"].view(G, -1)
    p = d * r.float() * gamma + beta
    e = gamma.abs() * (k1.float() * d.abs() + k0.float())
    e = e + U * (p.abs() + e)
    if c["act"] == "silu":
        sig = 1 / (1 + torch.exp(-p))
        y = p * sig
        slope = (sig * (1 + p * (1 - sig))).abs()
        b = torch.minimum(slope * e + 0.25 * e * e, 1.1 * e)
        f = (C_EXP * U / (1 - C_EXP * U) + U) / (1 - U)
        f = f / (1 - U) + U
        f = f / (1 - f)
        tau = b + f * (y.abs() + b)
    elif c["act"] == "relu":
        y = torch.clamp(p, min=0.0)
        tau = torch.clamp(torch.minimum(e, p + e), min=0.0)
    else:
        y, tau = p, e
    return y.view(B, P, C), tau.view(B, P, C)


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
    if c["kind"] == "quantize":
        return _plain_quantize(s)
    y, tau = _plain_product(s) if c["kind"] == "int8" else _plain_norm(c, s)
    return _profile(s["claimed"], s.get("y_ref", y), tau) if c["check"] else [y, tau]


# ------------------------------------------------------------------ the library's calls

def _fields(out):
    """The fields of a tao_profile in device memory."""
    words, halves = out[:24].view(torch.int64), out[24:56].view(torch.int32)
    return dict(violations=words[1:2], accept=halves[1:2], nan_count=words[2:3], max_rel=out[24:28].view(torch.float32),
                percentile_bins=halves[2:5], hist=out[64:].view(torch.int64))


def _run_own(c, s, r):
    import paper_2510_16028_amd as tao
    if c["kind"] == "quantize":
        q, scale = tao.tao_quantize_rows(s["x"], q=r["q"], scale=r["scale"])
        return [q * scale[:, None], scale]
    if c["kind"] == "int8":
        if c["check"]:
            return _fields(tao.tao_bound_check_linear_int8(s["A"], s["sa"], s["W"], s["sw"], s["claimed"], bias=s["bias"], eps_rel=EPS_REL,
                                                           out=r["out"], ws=r["ws"], readback=False))
        return list(tao.tao_bound_linear_int8(s["A"], s["sa"], s["W"], s["sw"], bias=s["bias"], y=r["y"], tau=r["tau"]))
    act = dict(silu=tao.ACT_SILU, relu=tao.ACT_RELU, none=tao.ACT_EXACT)[c["act"]]
    if c["check"]:
        return _fields(tao.tao_bound_check_groupnorm_act(s["x"], s["claimed"], c["groups"], s["gamma"], s["beta"], s["eps"], act=act, y_ref=s["y_ref"],
                                                         eps_rel=EPS_REL, out=r["out"], ws=r["ws"], readback=False))
    return list(tao.tao_bound_groupnorm_act(s["x"], c["groups"], s["gamma"], s["beta"], s["eps"], act=act, y=r["y"], tau=r["tau"], ws=r["ws"]))


def run(state):
    case, s, r = state
    return _run_own(case, s, r) if r is not None else _run_plain(case, s)


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "quantize":
        x = s["x"].double()
        scale = (x.abs().max(dim=1).values / 127.0).float().double()        # the scale is a binary32 value, and so is the quotient
        steps = (x / scale.unsqueeze(1)).float().double().round().clamp(-127.0, 127.0)
        return [steps * scale.unsqueeze(1), scale]
    if c["kind"] == "int8":
        sums = torch.mm(s["A"].double(), s["W"].double().t().contiguous())
        v = sums * torch.outer(s["sa"].double(), s["sw"].double())
        roundings = 2.0 + (sums.abs() > 2.0 ** 24).double()
        tau = v.abs() * (roundings * U / (1.0 - roundings * U))
        y = v
        if s["bias"] is not None:
            y = v + s["bias"].double()
            tau = tau + U * (y.abs() + tau)
        if c["check"]:
            # the re-executed output is the binary32 one: each step rounded
            y = (sums.float().double() * s["sa"].double().unsqueeze(1)).float().double()
            y = (y * s["sw"].double()).float()
            if s["bias"] is not None:
                y = (y.double() + s["bias"].double()).float()
    else:
        y, tau = _exact_norm(c, s)
        y = s["y_ref"] if c["check"] else y
    if not c["check"]:
        return [y, tau]
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


def _exact_norm(c, s):
    """The chain of the two-pass algorithm, each step's error with what it is made of, one sample at a time."""
    eps = float(torch.tensor(s["eps"], dtype=torch.float32))
    G, per = c["groups"], c["channels"] // c["groups"]
    n = c["positions"] * per
    g_n = (n - 1) * U / (1.0 - (n - 1) * U)
    gamma, beta = s["gamma"].double().view(G, 1, per), s["beta"].double().view(G, 1, per)
    ys, taus = [], []
    for sample in s["x"]:
        x = sample.double().view(c["positions"], G, per).permute(1, 0, 2).contiguous()
        total = lambda t: t.flatten(1).sum(1).view(G, 1, 1)
        mu = total(x) / n
        err_mu = (g_n * total(x.abs()) / n + 2.0 * U * mu.abs()) / (1.0 - 2.0 * U)
        dev = x - mu
        err_dev = (err_mu + U * dev.abs()) / (1.0 - U)
        large = dev.abs() + err_dev
        err_squares = total(err_dev * (dev.abs() + large) + U * large ** 2) + g_n * total(large ** 2 * (1.0 + U))
        variance = total(dev ** 2) / n
        err_variance = (err_squares / n + 2.0 * U * variance) / (1.0 - 2.0 * U)
        w = variance + eps
        err_w = (err_variance + U * w) / (1.0 - U)
        w_lo = torch.where(w > err_w, w - err_w, torch.full_like(w, math.nan))
        root = 1.0 / w.sqrt()
        err_root = err_w / (2.0 * w_lo * w_lo.sqrt()) + 2.0 * U / w_lo.sqrt()
        err_h = large * err_root + root * err_dev + U * large * (root + err_root)
        err_p = gamma.abs() * err_h + U * gamma.abs() * (dev.abs() * root + err_h)
        p = dev * root * gamma + beta
        err = err_p + U * (p.abs() + err_p)
        if c["act"] == "silu":
            sig = torch.sigmoid(p)
            y = p * sig
            through = torch.minimum((sig + y * (1.0 - sig)).abs() * err + err ** 2 / 4.0, 1.1 * err)
            steps = 2.0 * U / (1.0 - 2.0 * U) + U                            # the exponential, and adding one
            steps = steps / (1.0 - U) / (1.0 - U) + U                        # the quotient
            tau = through + steps / (1.0 - steps) * (y.abs() + through)
        elif c["act"] == "relu":
            y = p.relu()
            tau = torch.minimum(err, p + err).relu()
        else:
            y, tau = p, err
        back = lambda t: t.permute(1, 0, 2).reshape(c["positions"], c["channels"])
        ys.append(back(y))
        taus.append(back(tau))
    return torch.stack(ys), torch.stack(taus)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    """Bytes: operands, claims and re-executed outputs read once, outputs and bounds written once.  Operations: the product's
    multiplications and additions; for the others a nominal count per element (scaling and rounding; the statistics and the bound)."""
    c, profile = case, 64 + 8 * NBINS
    if c["kind"] == "quantize":
        n = c["rows"] * c["cols"]
        return dict(bytes=5 * n + 4 * c["rows"], flops=4 * n)
    if c["kind"] == "int8":
        M, K, N = c["M"], c["K"], c["N"]
        operands = M * K + N * K + 4 * (M + N + (N if c["bias"] else 0))
        return dict(bytes=operands + (4 * M * N + profile if c["check"] else 8 * M * N), flops=2 * M * K * N)
    n = c["batch"] * c["positions"] * c["channels"]
    return dict(bytes=12 * n + 8 * c["channels"] + (profile if c["check"] else 0), flops=40 * n)
