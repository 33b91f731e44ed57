"""The training operators whose speed is judged beside the convolutions: layer
normalisation, forward and backward, and the orthogonalised update of the
weight matrices (Newton-Schulz products, alone and inside a whole step).

A case is a dict of plain values; ``kind`` says which operator it is:

  norm_fwd  layer normalisation of ``rows`` rows of ``c`` values:
            y = (x - mean) * rstd * gamma + beta, and each row's mean and rstd
  norm_bwd  its gradients: dx, and dgamma and dbeta summed over the rows
  ns        ``steps`` Newton-Schulz steps on one ``rows`` x ``cols`` matrix
  muon      one update of all weight matrices of a network of ``c0`` input
            fields, ``c5`` channels at the end and ``features`` inputs of the
            head: momentum, Newton-Schulz, weight decay, the new weights

With ``own`` false, ``run`` evaluates the definitions with elementary torch
operations in float32, rounded once at the end; with ``own`` true it makes
the framework's calls.  ``exact`` evaluates the definitions in float64.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5

#: Newton-Schulz: x -> a x + b (x x') x + c (x x')^2 x
COEF = (3.4445, -4.7750, 2.0315)
NS_EPS = 1e-7

#: the update's hyperparameters (rates decay linearly as in the framework's Adam step)
ETA0, ETA_MIN, T_DECAY, MU, DECAY, T = 0.02, 0.001, 100000, 0.95, 0.01, 1000

HEAD_WIDTHS = (128, 64, 3)


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # the smallest call: the hidden layer of the head at batch 8, where launch and
        # host are what a user waits for
        dict(name="norm_fwd_8x128_f32", kind="norm_fwd", rows=8, c=128, dtype="f32"),
        # the head's input, one row per cube: few rows as long as the flattened stack output
        dict(name="norm_fwd_8x65536_bf16", kind="norm_fwd", rows=8, c=65536, dtype="bf16"),
        # the first layer's activation of eight 128^3 cubes, normalised over its 16 channels
        dict(name="norm_fwd_128cube_c16_bf16", kind="norm_fwd", rows=8 * 128 ** 3, c=16, dtype="bf16"),
        # the head's input in fp32, with the gradients of its 65,536 scales and offsets
        dict(name="norm_bwd_8x65536_f32", kind="norm_bwd", rows=8, c=65536, dtype="f32"),
        # ragged rows: no length that a 16-byte vector or a wave divides
        dict(name="norm_bwd_4097x777_f32", kind="norm_bwd", rows=4097, c=777, dtype="f32"),
        # the largest pass over memory: the gradients at the first layer's activation
        dict(name="norm_bwd_128cube_c16_bf16", kind="norm_bwd", rows=8 * 128 ** 3, c=16, dtype="bf16"),
        # the first convolution's 27 x 16 weights: the latency of a call
        dict(name="ns_27x16_f32", kind="ns", rows=27, cols=16, steps=5, dtype="f32"),
        # the head's first layer: a long axis of 65,536 and a short one of 128
        dict(name="ns_65536x128_f32", kind="ns", rows=65536, cols=128, steps=5, dtype="f32"),
        # a wide matrix of odd sides, in bf16
        dict(name="ns_517x2051_bf16", kind="ns", rows=517, cols=2051, steps=5, dtype="bf16"),
        # a large square matrix, where the matrix products are all of the time
        dict(name="ns_4096x4096_f32", kind="ns", rows=4096, cols=4096, steps=5, dtype="f32"),
        # the update of the network on 64^3 cubes, with the bf16 copy of the weights
        dict(name="muon_net64_bf16", kind="muon", c0=1, c5=128, features=8192, dtype="bf16"),
        # the update of the network on 128^3 cubes in fp32
        dict(name="muon_net128_f32", kind="muon", c0=1, c5=128, features=65536, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ones' ranges: rows from 1 to 2^24 and row
    lengths from 4 to 2^18 with at most 2^28 values (rows of two values have a dx
    that is all cancellation), matrices from 1 x 1 to 65,536 x 4,096 at no more
    products than the listed square one has, networks of 1 or 4 input fields and
    heads of 512 to 65,536 inputs."""
    while True:
        kind = rng.choice(["norm_fwd", "norm_fwd", "norm_bwd", "norm_bwd", "ns", "ns", "ns", "muon"])
        dtype = rng.choice(["f32", "bf16"])
        if kind in ("norm_fwd", "norm_bwd"):
            case = dict(kind=kind, rows=_log(rng, 1, 1 << 24), c=_log(rng, 4, 1 << 18), dtype=dtype)
            if case["rows"] * case["c"] > (1 << 28 if dtype == "bf16" else 1 << 27):
                continue
        elif kind == "ns":
            case = dict(kind=kind, rows=_log(rng, 1, 65536), cols=_log(rng, 1, 65536), steps=rng.choice([4, 5, 5, 5, 6]),
                        dtype=dtype)
            if case["rows"] * case["cols"] > 1 << 24 or min(case["rows"], case["cols"]) > 4096:
                continue
            if work(case)["flops"] > work(dict(kind="ns", rows=4096, cols=4096, steps=5, dtype="f32"))["flops"]:
                continue
        else:
            case = dict(kind=kind, c0=rng.choice([1, 1, 4]), c5=rng.choice([128, 128, 256]), features=128 * _log(rng, 4, 512),
                        dtype=dtype)
        return case


# ---------------------------------------------------------------------------
# shapes and work
# ---------------------------------------------------------------------------

def _matrices(case):
    """(rows, cols) of every weight matrix: a convolution's is [taps * c_in][c_out]."""
    c5 = case["c5"]
    conv = [(27 * case["c0"], 16), (64 * 16, 32), (64 * 32, 64), (27 * 64, 64), (8 * 64, c5), (8 * c5, c5)]
    dims = [case["features"], *HEAD_WIDTHS]
    return conv + [(dims[i], dims[i + 1]) for i in range(len(HEAD_WIDTHS))]


def _groups(case):
    """(starts, rows, cols, values in all): every matrix starts on a multiple of 16 values."""
    shapes = _matrices(case) if case["kind"] == "muon" else [(case["rows"], case["cols"])]
    starts, at = [], 0
    for r, c in shapes:
        starts.append(at)
        at += -(-r * c // 16) * 16
    return starts, [r for r, _ in shapes], [c for _, c in shapes], at


def _ns_flops(r, c, steps):
    """The products of the shorter side's Gram matrices (symmetric: half of them)
    and polynomials, the iteration carried out on the m x m matrices for two steps
    at a time, so that the long side is touched (steps + 1) / 2 times."""
    m, n = min(r, c), max(r, c)
    passes = (steps + 1) // 2
    return passes * (m * m * n + 2 * m * m * n) + (5 * (steps // 2) + steps % 2) * m ** 3


def work(case):
    """Bytes: every input read once, every output written once."""
    es = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind == "norm_fwd":
        n = case["rows"] * case["c"]
        return dict(bytes=2 * n * es + 8 * case["c"] + 8 * case["rows"], flops=7 * n)
    if kind == "norm_bwd":
        n = case["rows"] * case["c"]
        return dict(bytes=3 * n * es + 12 * case["c"] + 8 * case["rows"], flops=12 * n)
    if kind == "ns":
        return dict(bytes=2 * case["rows"] * case["cols"] * es, flops=_ns_flops(case["rows"], case["cols"], case["steps"]))
    n = sum(r * c for r, c in _matrices(case))
    # reads v, g, m; writes v, m and the bf16 copy
    return dict(bytes=n * (20 + (2 if case["dtype"] == "bf16" else 0)),
                flops=sum(_ns_flops(r, c, 5) for r, c in _matrices(case)) + 8 * n)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _tdt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _norm_data(case, seed):
    """Activations after a leaky ReLU (their mean is not zero) with a scale and
    an offset of their own in each row, trained scales around 1, and an
    upstream gradient."""
    g, t = _gen(seed), _tdt(case)
    r, c = case["rows"], case["c"]
    x = torch.randn((r, c), generator=g, device=DEV)
    x = torch.where(x > 0, x, 0.01 * x)
    x *= 0.5 + torch.rand((r, 1), generator=g, device=DEV)
    x += 0.2 * torch.randn((r, 1), generator=g, device=DEV)
    x = x.to(t)
    gamma = 1 + 0.1 * torch.randn(c, generator=g, device=DEV)
    beta = 0.1 * torch.randn(c, generator=g, device=DEV)
    dy = torch.randn((r, c), generator=g, device=DEV).to(t) if case["kind"] == "norm_bwd" else None
    return x, gamma, beta, dy


def _gradient(r, c, g):
    """A gradient as training has it: a few strong directions of falling
    strength over the noise of the batch."""
    k = min(16, r, c)
    s = 4.0 / torch.arange(1, k + 1, device=DEV, dtype=torch.float32)
    lead = torch.randn((r, k), generator=g, device=DEV) * s @ torch.randn((k, c), generator=g, device=DEV)
    return 1e-3 * (lead / math.sqrt(k) + torch.randn((r, c), generator=g, device=DEV))


def _ns_data(case, seed):
    return _gradient(case["rows"], case["cols"], _gen(seed)).to(_tdt(case))


def _muon_data(case, seed):
    """A step in the middle of training: weights at their initial scale and
    momentum that has settled around the gradient (padding is zero)."""
    g = _gen(seed)
    starts, rows, cols, n = _groups(case)
    v, gr, m = (torch.zeros(n, device=DEV) for _ in range(3))
    for o, r, c in zip(starts, rows, cols):
        v[o:o + r * c] = math.sqrt(2.0 / r) * torch.randn(r * c, generator=g, device=DEV)
        gr[o:o + r * c] = _gradient(r, c, g).reshape(-1)
        m[o:o + r * c] = 0.3 * _gradient(r, c, g).reshape(-1)
    return v, gr, m


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("norm_fwd", "norm_bwd"):
        x, gamma, beta, dy = _norm_data(case, seed)
        r, c = x.shape
        q = dict(case=case, x=x, gamma=gamma, beta=beta)
        if kind == "norm_fwd":
            q.update(y=torch.empty_like(x), mean=torch.empty(r, device=DEV), rstd=torch.empty(r, device=DEV))
        else:
            # what the forward pass kept
            h = x.float()
            mean = h.mean(1)
            rstd = torch.rsqrt((h - mean[:, None]).square().mean(1) + EPS)
            q.update(dy=dy, mean=mean, rstd=rstd, dx=torch.empty_like(x), dgamma=torch.empty(c, device=DEV),
                     dbeta=torch.empty(c, device=DEV))
        return q
    if kind == "ns":
        x = _ns_data(case, seed)
        return dict(case=case, g=x, o=torch.empty_like(x))
    v, gr, m = _muon_data(case, seed)
    return dict(case=case, v=v, g=gr, m=m, v16=torch.zeros_like(v, dtype=torch.bfloat16) if case["dtype"] == "bf16" else None,
                t=T)


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _norm_fwd(q):
    x = q["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = torch.rsqrt(d.square().mean(1) + EPS)
    y = d * rstd[:, None] * q["gamma"] + q["beta"]
    return dict(y=y.to(q["x"].dtype), mean=mean, rstd=rstd)


def _norm_bwd(q):
    dy, rstd = q["dy"].float(), q["rstd"][:, None]
    xhat = (q["x"].float() - q["mean"][:, None]) * rstd
    g = dy * q["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dict(dx=dx.to(q["x"].dtype), dgamma=(dy * xhat).sum(0), dbeta=dy.sum(0))


def _orthogonal(x, steps):
    """steps Newton-Schulz steps on x / ||x||, in float32."""
    a, b, c = COEF
    x = x / (torch.sqrt(x.square().sum()) + NS_EPS)
    wide = x.shape[0] <= x.shape[1]
    for _ in range(steps):
        if wide:
            s = x @ x.t()
            x = a * x + (b * s + c * (s @ s)) @ x
        else:
            s = x.t() @ x
            x = a * x + x @ (b * s + c * (s @ s))
    return x


def _rate(t):
    return (ETA0 - ETA_MIN) * (1 - min(t, T_DECAY) / T_DECAY) + ETA_MIN


def _muon(q):
    eta = _rate(q["t"])
    starts, rows, cols, _ = _groups(q["case"])
    for o, r, c in zip(starts, rows, cols):
        at = slice(o, o + r * c)
        m = MU * q["m"][at] + (1 - MU) * q["g"][at]
        u = (1 - MU) * q["g"][at] + MU * m
        s = math.sqrt(max(1.0, c / r))
        w = q["v"][at]
        q["v"][at] = w - eta * (s * _orthogonal(u.view(r, c), 5).reshape(-1) + DECAY * w)
        q["m"][at] = m
    if q["v16"] is not None:
        q["v16"].copy_(q["v"])
    q["t"] += 1
    return dict(v=q["v"], m=q["m"], v16=q["v16"])


# ---------------------------------------------------------------------------
# the calls
# ---------------------------------------------------------------------------

def _calls(q):
    """The framework's calls.  What a program makes once and keeps (the groups'
    host arrays and a workspace) is made on the state's first pass."""
    from paper_1808_04728_amd import binding as B
    case = q["case"]
    kind, dt = case["kind"], case["dtype"]

    def space(n):
        return torch.empty(max(16, n), dtype=torch.uint8, device=DEV)

    if kind == "norm_fwd":
        r, c = case["rows"], case["c"]
        if "ws" not in q:
            q["ws"] = space(B.cf_layernorm_fwd_workspace_size(r, c, dt))
        B.cf_layernorm_fwd(r, c, dt, q["x"], q["gamma"], q["beta"], EPS, q["y"], q["mean"], q["rstd"], q["ws"])
        return dict(y=q["y"], mean=q["mean"], rstd=q["rstd"])
    if kind == "norm_bwd":
        r, c = case["rows"], case["c"]
        if "ws" not in q:
            q["ws"] = space(B.cf_layernorm_bwd_workspace_size(r, c, dt))
        B.cf_layernorm_bwd(r, c, dt, q["dy"], q["x"], q["gamma"], q["mean"], q["rstd"], q["dx"], q["dgamma"], q["dbeta"],
                           q["ws"])
        return dict(dx=q["dx"], dgamma=q["dgamma"], dbeta=q["dbeta"])
    if "ws" not in q:
        starts, rows, cols, _ = _groups(case)
        q["groups"] = B.make_matrices(starts, rows, cols)
        if kind == "ns":
            q["hp"] = B.make_ns_hparams(steps=case["steps"], coef=COEF, eps=NS_EPS)
            q["ws"] = space(B.cf_newton_schulz_workspace_size(q["groups"], dt))
        else:
            q["hp"] = B.make_muon_hparams(T_DECAY, eta0=ETA0, eta_min=ETA_MIN, mu=MU, weight_decay=DECAY, steps=5, coef=COEF,
                                          eps=NS_EPS)
            q["ws"] = space(B.cf_muon_workspace_size(q["groups"]))
    if kind == "ns":
        B.cf_newton_schulz(q["groups"], dt, q["hp"], q["g"], q["o"], q["ws"])
        return q["o"]
    B.cf_muon_step(q["groups"], q["t"], q["hp"], q["v"], q["g"], q["m"], q["v16"], q["ws"])
    q["t"] += 1
    return dict(v=q["v"], m=q["m"], v16=q["v16"])


def run(state):
    if own:
        return _calls(state)
    kind = state["case"]["kind"]
    if kind == "norm_fwd":
        return _norm_fwd(state)
    if kind == "norm_bwd":
        return _norm_bwd(state)
    if kind == "ns":
        return _orthogonal(state["g"].float(), state["case"]["steps"]).to(state["g"].dtype)
    return _muon(state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _orthogonal64(x, steps):
    """U p(S) V' of x / ||x|| = U S V', p the polynomial applied ``steps`` times,
    through the eigenvalues' side alone: with h = x x' every step multiplies x by
    q = a + b h + c h^2, which commutes with h."""
    a, b, c = COEF
    x = x / (x.norm() + NS_EPS)
    wide = x.shape[0] <= x.shape[1]
    y = x if wide else x.t().contiguous()
    h = y @ y.t()
    p = None
    for _ in range(steps):
        q = torch.addmm(b * h, h, h, alpha=c)
        q.diagonal().add_(a)
        p = q if p is None else q @ p
        h = q @ h @ q
    return p @ x if wide else x @ p


def exact(case, seed):
    kind = case["kind"]
    if kind in ("norm_fwd", "norm_bwd"):
        x, gamma, beta, dy = _norm_data(case, seed)
        rows, c = x.shape
        gamma, beta = gamma.double(), beta.double()
        part = max(1, (1 << 26) // c)  # rows at a time
        out, dgamma, dbeta = [], torch.zeros_like(gamma), torch.zeros_like(gamma)
        for i in range(0, rows, part):
            h = x[i:i + part].double()
            var, mean = torch.var_mean(h, dim=1, unbiased=False, keepdim=True)
            if kind == "norm_fwd":
                rstd = (var + EPS) ** -0.5
                out.append((torch.addcmul(beta, (h - mean) * rstd, gamma), mean[:, 0], rstd[:, 0]))
                continue
            # the pass reads the forward's float32 mean and rstd
            h = x[i:i + part].float()
            mean = h.mean(1)
            rstd = torch.rsqrt((h - mean[:, None]).square().mean(1) + EPS).double()[:, None]
            xh = (h.double() - mean.double()[:, None]) * rstd
            d = dy[i:i + part].double()
            dgamma += (d * xh).sum(0)
            dbeta += d.sum(0)
            d = d * gamma
            out.append((rstd * (d - d.sum(1, keepdim=True) / c - xh * ((d * xh).sum(1, keepdim=True) / c)),))
        parts = [torch.cat(p) for p in zip(*out)]
        if kind == "norm_fwd":
            return dict(y=parts[0], mean=parts[1], rstd=parts[2])
        return dict(dx=parts[0], dgamma=dgamma, dbeta=dbeta)
    if kind == "ns":
        return _orthogonal64(_ns_data(case, seed).double(), case["steps"])
    v, gr, m = (t.double() for t in _muon_data(case, seed))
    starts, rows, cols, _ = _groups(case)
    m = torch.lerp(gr, m, MU)
    u = torch.lerp(gr, m, MU)
    eta = ETA_MIN + (ETA0 - ETA_MIN) * (1 - T / T_DECAY)
    for o, r, c in zip(starts, rows, cols):
        w = v[o:o + r * c]
        w *= 1 - eta * DECAY
        w -= eta * max(1.0, c / r) ** 0.5 * _orthogonal64(u[o:o + r * c].view(r, c), 5).reshape(-1)
    return dict(v=v, m=m, v16=v if case["dtype"] == "bf16" else None)
