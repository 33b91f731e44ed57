"""Further training operators whose speed is judged: group normalisation with its
activation, the matrix product with bias, activation and residual in its epilogue,
each forward and backward, and the AdamW update of many tensors at once.

A case is a dict of plain values; ``kind`` says which operator it is:

  gn_fwd    group normalisation of ``n`` samples of ``vox`` voxels of ``c`` channels in
            ``groups`` groups, then an activation: y, and each group's mean and rstd
  gn_bwd    its gradients: dx, and dgamma and dbeta summed over samples and voxels
  lin_fwd   y = act(x W + b) + r of ``m`` rows, ``k`` inputs and ``n`` outputs, and
            the pre-activation z = x W + b
  lin_bwd   its gradients: dx = (dz W' + r) * act'(z) (z of the layer before, r the
            gradient that reaches x past this layer), dW = x' dz, db
  adamw     one AdamW update of a list of tensors (``model`` says which): parameters,
            their bf16 copy, and both moments, in fp32 or in 8 bits

With ``own`` false, ``run`` evaluates the definitions with elementary torch
operations in float32 (float64 next to a border), rounded once at the end; with
``own`` true it makes the framework's calls.  ``exact`` evaluates the definitions
in float64.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
ALPHA = 0.01

#: the update's hyperparameters (the rate decays linearly as in the framework's other updates)
ETA0, ETA_MIN, T_DECAY, B1, B2, ADAM_EPS, DECAY, T, SEED = 1e-3, 1e-4, 100000, 0.9, 0.999, 1e-8, 0.01, 1000, 20

#: values that share a scale where moments are held in 8 bits
BLOCK = 256


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # the smallest call: the last convolution's output of one 64^3 cube (4^3 voxels)
        dict(name="gn_fwd_4cube_c128_f32", kind="gn_fwd", n=1, vox=4 ** 3, c=128, groups=8, act="silu", dtype="f32"),
        # the first layer's activation of eight 128^3 cubes
        dict(name="gn_fwd_128cube_c16_bf16", kind="gn_fwd", n=8, vox=128 ** 3, c=16, groups=4, act="lrelu", dtype="bf16"),
        # cubes of an odd side, three to a batch, with groups of 8 channels
        dict(name="gn_bwd_31cube_c48_f32", kind="gn_bwd", n=3, vox=31 ** 3, c=48, groups=6, act="silu", dtype="f32"),
        # the gradients at the first layer's activation: the largest pass over memory
        dict(name="gn_bwd_128cube_c16_bf16", kind="gn_bwd", n=8, vox=128 ** 3, c=16, groups=4, act="lrelu", dtype="bf16"),
        # the voxels of one small cube through a voxel-wise layer: the latency of a call
        dict(name="lin_fwd_64x128x512_bf16", kind="lin_fwd", m=64, k=128, n=512, act="gelu", residual=False, dtype="bf16"),
        # the widening layer of a voxel-wise block on eight cubes of 16^3 voxels
        dict(name="lin_fwd_32768x1024x4096_bf16", kind="lin_fwd", m=32768, k=1024, n=4096, act="gelu", residual=False,
             dtype="bf16"),
        # no side that a vector or a tile divides, with the residual, in fp32
        dict(name="lin_fwd_4097x515x1027_f32", kind="lin_fwd", m=4097, k=515, n=1027, act="lrelu", residual=True, dtype="f32"),
        # the gradients of the narrowing layer of that block
        dict(name="lin_bwd_32768x4096x1024_bf16", kind="lin_bwd", m=32768, k=4096, n=1024, act="gelu", residual=False,
             dtype="bf16"),
        # the gradients of a middling layer on eleven^3 voxels of odd widths, in fp32
        dict(name="lin_bwd_1331x130x517_f32", kind="lin_bwd", m=11 ** 3, k=130, n=517, act="silu", residual=True, dtype="f32"),
        # the parameters of the network on 64^3 cubes: many small tensors, one launch's latency
        dict(name="adamw_net64_f32", kind="adamw", model="net", size=8192, state="f32", dtype="bf16"),
        # a list of tensors of odd lengths with moments in 8 bits
        dict(name="adamw_odd_40_8bit", kind="adamw", model="odd", size=40, state="8bit", dtype="f32"),
        # twelve voxel-wise blocks of 1024 channels widened to 4096, moments in 8 bits
        dict(name="adamw_blocks_12_8bit", kind="adamw", model="blocks", size=12, state="8bit", dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ones' ranges: 1 to 16 samples of 1 to 2^21 voxels of
    1 to 512 channels, at most 2^28 values and at least 16 a group (a group of two has
    a dx that is all cancellation); products of 1 to 65,536 rows and 1 to 8,192
    inputs and outputs with at most the listed ones' operations; networks, lists of 1
    to 64 tensors of odd lengths and 1 to 12 blocks."""
    while True:
        kind = rng.choice(["gn_fwd", "gn_fwd", "gn_bwd", "gn_bwd", "lin_fwd", "lin_fwd", "lin_fwd", "lin_bwd", "lin_bwd",
                           "lin_bwd", "adamw", "adamw"])
        dtype = rng.choice(["f32", "bf16"])
        act = rng.choice(["none", "lrelu", "silu", "gelu"])
        if kind in ("gn_fwd", "gn_bwd"):
            per, groups = _log(rng, 1, 64), _log(rng, 1, 32)
            case = dict(kind=kind, n=_log(rng, 1, 16), vox=_log(rng, 1, 1 << 21), c=per * groups, groups=groups, act=act,
                        dtype=dtype)
            if case["c"] > 512 or case["vox"] * per < 16:
                continue
            if case["n"] * case["vox"] * case["c"] > (1 << 28 if dtype == "bf16" else 1 << 27):
                continue
        elif kind in ("lin_fwd", "lin_bwd"):
            case = dict(kind=kind, m=_log(rng, 1, 65536), k=_log(rng, 1, 8192), n=_log(rng, 1, 8192), act=act,
                        residual=rng.random() < 0.5, dtype=dtype)
            if case["m"] * case["k"] * case["n"] > 32768 * 1024 * 4096:
                continue
        else:
            model = rng.choice(["net", "odd", "odd", "blocks"])
            size = 128 * _log(rng, 4, 512) if model == "net" else _log(rng, 1, 64 if model == "odd" else 12)
            case = dict(kind=kind, model=model, size=size, state=rng.choice(["f32", "8bit"]), dtype=dtype)
        return case


# ---------------------------------------------------------------------------
# shapes and work
# ---------------------------------------------------------------------------

def _tensors(case):
    """(values, whether it decays) of every tensor of a model: ``net`` the convolution
    stack and head with ``size`` inputs of the head, weights then biases; ``odd``
    ``size`` tensors from 1 to 2^20 values; ``blocks`` of two matrices, their biases,
    and a normalisation's scales and offsets."""
    size = case["size"]
    if case["model"] == "net":
        conv = [(27, 16), (64 * 16, 32), (64 * 32, 64), (27 * 64, 64), (8 * 64, 128), (8 * 128, 128)]
        dims = [size, 128, 64, 3]
        shapes = conv + [(dims[i], dims[i + 1]) for i in range(3)]
        return [(r * c, True) for r, c in shapes] + [(c, False) for _, c in shapes]
    if case["model"] == "odd":
        return [(1 + int(2 ** (20 * ((i * 37 + 11) % 64) / 63)), i % 3 != 0) for i in range(size)]
    block = [(1024 * 4096, True), (4096, False), (4096 * 1024, True), (1024, False), (1024, False), (1024, False)]
    return block * size


def work(case):
    """Bytes: every input read once, every output written once."""
    es = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind in ("gn_fwd", "gn_bwd"):
        v, c, q = case["n"] * case["vox"] * case["c"], case["c"], case["n"] * case["groups"]
        if kind == "gn_fwd":
            return dict(bytes=2 * v * es + 8 * c + 8 * q, flops=10 * v)
        return dict(bytes=3 * v * es + 16 * c + 8 * q, flops=20 * v)
    if kind in ("lin_fwd", "lin_bwd"):
        m, k, n = case["m"], case["k"], case["n"]
        if kind == "lin_fwd":
            return dict(bytes=(m * k + k * n + (2 + case["residual"]) * m * n) * es + 4 * n, flops=2 * m * k * n)
        z = case["act"] != "none"
        return dict(bytes=((2 + z + case["residual"]) * m * k + m * n + k * n) * es + 4 * k * n + 4 * n, flops=4 * m * k * n)
    v = sum(count for count, _ in _tensors(case))
    state = 16 if case["state"] == "f32" else 4 + 16 / BLOCK
    return dict(bytes=v * (12 + state + (2 if case["dtype"] == "bf16" else 0)), flops=16 * v)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _tdt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _gn_data(case, seed):
    """Convolution outputs: every sample and channel has a scale and an offset of its
    own; trained scales around 1, and an upstream gradient."""
    g, t = _gen(seed), _tdt(case)
    n, v, c = case["n"], case["vox"], case["c"]
    x = torch.randn((n, v, c), generator=g, device=DEV)
    x *= 0.5 + torch.rand((n, 1, c), generator=g, device=DEV)
    x += 0.5 * torch.randn((n, 1, c), generator=g, device=DEV)
    x = x.to(t)
    gamma = 1 + 0.2 * torch.randn(c, generator=g, device=DEV)
    beta = 0.2 * torch.randn(c, generator=g, device=DEV)
    dy = torch.randn((n, v, c), generator=g, device=DEV).to(t) if case["kind"] == "gn_bwd" else None
    return x, gamma, beta, dy


def _gn_stats(x, groups):
    """float32 mean and rstd [n][groups], a sample at a time in float64."""
    n, v, c = x.shape
    h = [torch.var_mean(s.double().view(v, groups, c // groups), dim=(0, 2), unbiased=False) for s in x]
    return torch.stack([m for _, m in h]).float(), torch.stack([(s + EPS) ** -0.5 for s, _ in h]).float()


def _lin_data(case, seed):
    """Activations and weights at their initial scale, biases of trained size."""
    g, t = _gen(seed), _tdt(case)
    m, k, n = case["m"], case["k"], case["n"]

    def normal(*shape, s=1.0):
        return (s * torch.randn(shape, generator=g, device=DEV)).to(t)

    x, w = normal(m, k), normal(k, n, s=1 / math.sqrt(k))
    if case["kind"] == "lin_fwd":
        return x, w, 0.1 * torch.randn(n, generator=g, device=DEV), normal(m, n) if case["residual"] else None
    dz = normal(m, n)
    z = normal(m, k) if case["act"] != "none" else None
    return x, w, dz, z, normal(m, k) if case["residual"] else None


def _adamw_layout(case):
    """Every tensor starts on a block of its own in flat arrays: (first block, values,
    decay) a tensor, and the blocks in all."""
    out, at = [], 0
    for count, decays in _tensors(case):
        out.append((at, count, DECAY if decays else 0.0))
        at += -(-count // BLOCK)
    return out, at


def _codes(x):
    """float8 codes (to nearest) and power-of-two scales of blocks, for a state to begin from."""
    top = x.abs().amax(1, keepdim=True)
    e = torch.clamp(torch.ceil(torch.log2(torch.clamp(top, min=1e-38) / 448)), min=-126)
    s = torch.exp2(e)
    return (x / s).to(torch.float8_e4m3fn), s


def _adamw_data(case, seed):
    """A step in the middle of training: weights at their initial scale, and moments
    that have settled around the gradient; padding behind a tensor is zero."""
    g = _gen(seed)
    tensors, nb = _adamw_layout(case)
    first = torch.tensor([b for b, _, _ in tensors] + [nb], device=DEV)
    tensor = torch.repeat_interleave(torch.arange(len(tensors), device=DEV), first.diff())
    index = (torch.arange(nb, device=DEV) - first[tensor])[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    live = index < torch.tensor([count for _, count, _ in tensors], device=DEV)[tensor][:, None]
    size = torch.exp2(4 * torch.rand((nb, 1), generator=g, device=DEV) - 12)  # of a block's gradients

    def normal(s):
        return torch.where(live, s * torch.randn((nb, BLOCK), generator=g, device=DEV), 0.0)

    q = dict(p=normal(0.05), g=normal(size), m=normal(0.3 * size), v=normal(size).square() + 0.2 * normal(size).square())
    q.update(index=index, tensor=tensor, decay=torch.tensor([d for _, _, d in tensors], device=DEV)[tensor][:, None])
    if case["state"] == "8bit":
        q["m"], q["ms"] = _codes(q["m"])
        q["r"], q["rs"] = _codes(q.pop("v").sqrt())
    return q


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("gn_fwd", "gn_bwd"):
        x, gamma, beta, dy = _gn_data(case, seed)
        n, v, c = x.shape
        q = dict(case=case, x=x, gamma=gamma, beta=beta)
        if kind == "gn_fwd":
            q.update(y=torch.empty_like(x), mean=torch.empty((n, case["groups"]), device=DEV),
                     rstd=torch.empty((n, case["groups"]), device=DEV))
        else:
            mean, rstd = _gn_stats(x, case["groups"])  # what the forward pass kept
            q.update(dy=dy, mean=mean, rstd=rstd, dx=torch.empty_like(x), dgamma=torch.empty(c, device=DEV),
                     dbeta=torch.empty(c, device=DEV))
        return q
    if kind == "lin_fwd":
        x, w, b, r = _lin_data(case, seed)
        y = torch.empty((case["m"], case["n"]), dtype=x.dtype, device=DEV)
        return dict(case=case, x=x, w=w, b=b, r=r, y=y, z=torch.empty_like(y))
    if kind == "lin_bwd":
        x, w, dz, z, r = _lin_data(case, seed)
        return dict(case=case, x=x, w=w, dz=dz, z=z, r=r, dx=torch.empty_like(x),
                    dw=torch.empty((case["k"], case["n"]), device=DEV), db=torch.empty(case["n"], device=DEV))
    q = dict(case=case, t=T, **_adamw_data(case, seed))
    q["p16"] = torch.zeros_like(q["p"], dtype=torch.bfloat16) if case["dtype"] == "bf16" else None
    return q


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _act(u, act):
    if act == "lrelu":
        return torch.where(u > 0, u, ALPHA * u)
    if act == "silu":
        return u / (1 + torch.exp(-u))
    if act == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    return u


def _slope(u, act):
    """act'(u); u > 0 is the border of the leaky ReLU."""
    if act == "lrelu":
        return torch.where(u > 0, 1.0, ALPHA)
    if act == "silu":
        s = 1 / (1 + torch.exp(-u))
        return s * (1 + u * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(u)


def _spread(s, c):
    """[n][groups] to [n][1][c]."""
    return s.repeat_interleave(c // s.shape[1], dim=1)[:, None, :]


def _gn_fwd(q):
    case = q["case"]
    n, v, c = q["x"].shape
    x = q["x"].float().view(n, v, case["groups"], -1)
    mean = x.mean((1, 3), keepdim=True)
    d = x - mean
    rstd = torch.rsqrt(d.square().mean((1, 3), keepdim=True) + EPS)
    u = (d * rstd).view(n, v, c) * q["gamma"] + q["beta"]
    return dict(y=_act(u, case["act"]).to(q["x"].dtype), mean=mean[:, 0, :, 0], rstd=rstd[:, 0, :, 0])


def _gn_bwd(q):
    case = q["case"]
    n, v, c = q["x"].shape
    mean, rstd = _spread(q["mean"], c), _spread(q["rstd"], c)
    xh = (q["x"].float() - mean) * rstd
    if case["act"] == "lrelu":  # the side of the border in float64
        u = (q["x"].double() - mean) * rstd.double() * q["gamma"].double() + q["beta"].double()
        du = q["dy"].float() * torch.where(u > 0, 1.0, ALPHA)
    else:
        du = q["dy"].float() * _slope(xh * q["gamma"] + q["beta"], case["act"])
    g = du * q["gamma"]
    m1 = _spread(g.view(n, v, case["groups"], -1).mean((1, 3)), c)
    m2 = _spread((g * xh).view(n, v, case["groups"], -1).mean((1, 3)), c)
    return dict(dx=(rstd * (g - m1 - xh * m2)).to(q["x"].dtype), dgamma=(du * xh).sum((0, 1)), dbeta=du.sum((0, 1)))


def _lin_fwd(q):
    z = q["x"].float() @ q["w"].float() + q["b"]
    y = _act(z, q["case"]["act"])
    if q["r"] is not None:
        y = y + q["r"].float()
    return dict(y=y.to(q["x"].dtype), z=z.to(q["x"].dtype))


def _lin_bwd(q):
    dz = q["dz"].float()
    dx = dz @ q["w"].float().t()
    if q["r"] is not None:
        dx = dx + q["r"].float()
    if q["z"] is not None:
        dx = dx * _slope(q["z"].float(), q["case"]["act"])
    return dict(dx=dx.to(q["x"].dtype), dw=q["x"].float().t() @ dz, db=dz.sum(0))


def _mix(h):
    """32 bits in, 32 bits out (held in int64)."""
    h = h ^ (h >> 16)
    h = h * 0x6A09E667 & 0xFFFFFFFF
    h = h ^ (h >> 15)
    h = h * 0xBB67AE85 & 0xFFFFFFFF
    return h ^ (h >> 16)


def _bits(q):
    """The update's random bits of every value: from the seed, the step, the tensor's
    place in the list and the value's place in the tensor."""
    step = _mix((SEED + q["t"] * 0x9E3779B9) & 0xFFFFFFFF)
    key = _mix((step + q["tensor"] * 0x9E3779B9) & 0xFFFFFFFF)
    return _mix((key[:, None] + q["index"] * 0x9E3779B9) & 0xFFFFFFFF)


def _scale(x):
    """The smallest power of two that brings a block's largest value to 448 or below."""
    f, e = torch.frexp(x.abs().amax(1, keepdim=True))  # f in [0.5, 1)
    e = torch.where(f > 0, torch.clamp(e - 9 + (f > 0.875).int(), min=-126), -126)
    return torch.ldexp(torch.ones_like(f), e)


def _stochastic(x, bits16):
    """Values of at most 448 to float8 codes: up with the chance of the part left over."""
    a = x.abs()
    low = a < 2.0 ** -6  # steps of 2^-9 below, as above it up to 2^-5
    b = torch.where(low, a + 2.0 ** -6, a).view(torch.int32) + (bits16 << 4).int()
    a = (b & ~0xFFFFF).view(torch.float32)
    a = torch.where(low, a - 2.0 ** -6, a)
    return torch.where(x < 0, -a, a).to(torch.float8_e4m3fn)


def _rate(t):
    return (ETA0 - ETA_MIN) * (1 - min(t, T_DECAY) / T_DECAY) + ETA_MIN


def _adamw(q):
    eta, k, eight = _rate(q["t"]), q["t"] + 1, q["case"]["state"] == "8bit"
    g = q["g"]
    if eight:
        m, r = q["m"].float() * q["ms"], q["r"].float() * q["rs"]
        v = r * r
    else:
        m, v = q["m"], q["v"]
    m = m * B1 + g * (1 - B1)
    v = v * B2 + (g * g) * (1 - B2)
    r = v.sqrt()
    step = (m / (r * (1 / math.sqrt(1 - B2 ** k)) + ADAM_EPS)) * (eta / (1 - B1 ** k))
    q["p"] = q["p"] * (1 - eta * q["decay"]) - step
    if q["p16"] is not None:
        q["p16"] = q["p"].to(torch.bfloat16)
    if eight:
        bits = _bits(q)
        q["ms"], q["rs"] = _scale(m), _scale(r)
        q["m"] = _stochastic(m / q["ms"], bits & 0xFFFF)
        r = _stochastic(r / q["rs"], bits >> 16)
        # a second moment that is not zero is not held as zero
        q["r"] = torch.where((v > 0) & (r.float() == 0), 2.0 ** -9, r.float()).to(torch.float8_e4m3fn)
    else:
        q["m"], q["v"] = m, v
    q["t"] += 1
    return _adamw_state(q)


def _adamw_state(q):
    return {name: q[name] for name in ("p", "p16", "m", "ms", "v", "r", "rs") if q.get(name) is not None}


# ---------------------------------------------------------------------------
# the calls
# ---------------------------------------------------------------------------

def _calls(q):
    """The framework's calls.  What a program makes once and keeps (workspaces, the list
    of tensors) is made on the state's first pass."""
    from paper_1808_04728_amd import binding as B
    case = q["case"]
    kind, dt = case["kind"], case["dtype"]

    def space(*sizes):
        return torch.empty(max(16, *sizes), dtype=torch.uint8, device=DEV)

    if kind in ("gn_fwd", "gn_bwd"):
        shape = (case["n"], case["vox"], case["c"], case["groups"], dt)
        if kind == "gn_fwd":
            if "ws" not in q:
                q["ws"] = space(B.cf_groupnorm_fwd_workspace_size(*shape), 16)
            B.cf_groupnorm_fwd(*shape, q["x"], q["gamma"], q["beta"], EPS, case["act"], ALPHA, q["y"], q["mean"], q["rstd"],
                               q["ws"])
            return dict(y=q["y"], mean=q["mean"], rstd=q["rstd"])
        if "ws" not in q:
            q["ws"] = space(B.cf_groupnorm_bwd_workspace_size(*shape), 16)
        B.cf_groupnorm_bwd(*shape, q["dy"], q["x"], q["gamma"], q["beta"], q["mean"], q["rstd"], case["act"], ALPHA, q["dx"],
                           q["dgamma"], q["dbeta"], q["ws"])
        return dict(dx=q["dx"], dgamma=q["dgamma"], dbeta=q["dbeta"])
    if kind in ("lin_fwd", "lin_bwd"):
        shape = (case["m"], case["k"], case["n"], dt)
        if kind == "lin_fwd":
            if "ws" not in q:
                q["ws"] = space(B.cf_linear_fwd_workspace_size(*shape), 16)
            B.cf_linear_fwd(*shape, q["x"], q["w"], q["b"], case["act"], ALPHA, q["r"], q["y"], q["z"], q["ws"])
            return dict(y=q["y"], z=q["z"])
        if "ws" not in q:
            q["ws"] = space(B.cf_linear_bwd_data_workspace_size(*shape), B.cf_linear_bwd_weight_workspace_size(*shape))
        B.cf_linear_bwd_data(*shape, q["dz"], q["w"], q["r"], q["z"], case["act"], ALPHA, q["dx"], q["ws"])
        B.cf_linear_bwd_weight(*shape, q["x"], q["dz"], q["dw"], q["db"], q["ws"])
        return dict(dx=q["dx"], dw=q["dw"], db=q["db"])
    if "list" not in q:
        def part(name, b, count):
            return None if q.get(name) is None else q[name].view(-1)[b * BLOCK:b * BLOCK + count]

        def scales(name, b, count):
            return None if q.get(name) is None else q[name].view(-1)[b:b - (-count // BLOCK)]

        q["list"] = B.make_adamw_tensors([
            dict(p=part("p", b, n), g=part("g", b, n), m=part("m", b, n), v=part("r" if "r" in q else "v", b, n),
                 m_scale=scales("ms", b, n), v_scale=scales("rs", b, n), p16=part("p16", b, n), weight_decay=d)
            for b, n, d in _adamw_layout(case)[0]])
        q["hp"] = B.make_adamw_hparams(T_DECAY, eta0=ETA0, eta_min=ETA_MIN, beta1=B1, beta2=B2, eps=ADAM_EPS, seed=SEED)
    B.cf_adamw_step(q["list"], q["t"], q["hp"])
    q["t"] += 1
    return _adamw_state(q)


def run(state):
    if own:
        return _calls(state)
    plain = dict(gn_fwd=_gn_fwd, gn_bwd=_gn_bwd, lin_fwd=_lin_fwd, lin_bwd=_lin_bwd, adamw=_adamw)
    return plain[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _curve64(u, act):
    """(act(u), act'(u)) in float64, through tanh and erfc."""
    if act == "lrelu":
        d = ALPHA + (1 - ALPHA) * (u > 0).double()
        return u * d, d
    if act == "silu":
        s = 0.5 + 0.5 * torch.tanh(0.5 * u)
        return u * s, s + u * s * (0.5 - 0.5 * torch.tanh(0.5 * u))
    if act == "gelu":
        s = 0.5 * torch.erfc(-u / 2 ** 0.5)
        return u * s, s + u * torch.exp(-u * u / 2) / (2 * math.pi) ** 0.5
    return u, torch.ones_like(u)


def _gn64(case, seed):
    x, gamma, beta, dy = _gn_data(case, seed)
    n, v, c = x.shape
    groups, per = case["groups"], case["c"] // case["groups"]
    gamma, beta = gamma.double().view(groups, per), beta.double().view(groups, per)
    if dy is not None:
        mean32, rstd32 = _gn_stats(x, groups)  # the pass reads the forward's float32 mean and rstd
    out, dgamma, dbeta = [], torch.zeros_like(gamma), torch.zeros_like(gamma)
    for i in range(n):
        h = x[i].double().view(v, groups, per)
        if dy is None:
            var, mean = torch.var_mean(h, dim=(0, 2), unbiased=False)
            rstd = (var + EPS) ** -0.5
            u = torch.addcmul(beta, (h - mean[:, None]) * rstd[:, None], gamma)
            out.append((_curve64(u, case["act"])[0].view(v, c), mean, rstd))
            continue
        rstd = rstd32[i].double()[:, None]
        h = (h - mean32[i].double()[:, None]) * rstd
        d = dy[i].double().view(v, groups, per) * _curve64(torch.addcmul(beta, h, gamma), case["act"])[1]
        dgamma += (d * h).sum(0)
        dbeta += d.sum(0)
        d = d * gamma
        count = v * per
        out.append(((rstd * (d - d.sum((0, 2))[:, None] / count - h * ((d * h).sum((0, 2))[:, None] / count))).view(v, c),))
    parts = [torch.stack(p) for p in zip(*out)]
    if dy is None:
        return dict(y=parts[0], mean=parts[1], rstd=parts[2])
    return dict(dx=parts[0], dgamma=dgamma.view(-1), dbeta=dbeta.view(-1))


def exact(case, seed):
    kind = case["kind"]
    if kind in ("gn_fwd", "gn_bwd"):
        return _gn64(case, seed)
    if kind == "lin_fwd":
        x, w, b, r = _lin_data(case, seed)
        z = torch.addmm(b.double(), x.double(), w.double())
        y = _curve64(z, case["act"])[0]
        return dict(y=y if r is None else y + r.double(), z=z)
    if kind == "lin_bwd":
        x, w, dz, z, r = (None if t is None else t.double() for t in _lin_data(case, seed))
        dx = torch.mm(w, dz.t().contiguous()).t()
        if r is not None:
            dx = dx + r
        if z is not None:
            dx = dx * _curve64(z, case["act"])[1]
        return dict(dx=dx, dw=torch.mm(x.t().contiguous(), dz), db=torch.mv(dz.t().contiguous(), torch.ones_like(dz[:, 0])))
    q = {name: t.double() if t.is_floating_point() else t for name, t in _adamw_data(case, seed).items()}
    eight = case["state"] == "8bit"
    m = torch.lerp(q["g"], q["m"] * q["ms"] if eight else q["m"], B1)
    v = torch.lerp(q["g"] ** 2, (q["r"] * q["rs"]) ** 2 if eight else q["v"], B2)
    eta = ETA_MIN + (ETA0 - ETA_MIN) * (1 - T / T_DECAY)
    p = q["p"] - eta * (q["decay"] * q["p"] + (m / (1 - B1 ** (T + 1))) / ((v / (1 - B2 ** (T + 1))) ** 0.5 + ADAM_EPS))
    out = dict(p=p, p16=p if case["dtype"] == "bf16" else None)
    if not eight:
        return dict(out, m=m, v=v)
    r = v ** 0.5
    # codes are rounded at random: the values that they stand for on average
    for name, x in (("m", m), ("r", r)):
        top = x.abs().amax(1, keepdim=True)
        s = 2.0 ** torch.clamp(torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448)), min=-126)
        out[name], out[name + "s"] = x / s, s
    return out
