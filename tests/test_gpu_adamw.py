"""GPU parity of the AdamW update through the C ABI: bit by bit against the same fp32
operations in numpy (the header gives their order, and the codes' random bits), and
against the formulas in float64.

Against float64 (fp32 moments).  Each of m, v and r = sqrt(v) has relative errors of
at most 2, 3 and 2.5 half steps of its terms, the quotient 3 more, its factor one, p
three roundings: within 12 2^-24 of the terms |m| + |g|, |step| and |p| added up."""
import numpy as np
import pytest
import torch

from paper_1808_04728_amd import binding as B

gpu = pytest.mark.gpu

BLOCK = B.CF_ADAMW_BLOCK
GUARD = 64
F = np.float32
HP = dict(eta0=2e-3, eta_min=1e-4, beta1=0.9, beta2=0.999, eps=1e-8)
COUNTS = [1, 3, 4, 255, 256, 257, 1000, 1023, 1024, 1025, 4099, 70001]


def mix(h):
    h = h ^ (h >> np.uint32(16))
    h = h * np.uint32(0x6A09E667)
    h = h ^ (h >> np.uint32(15))
    h = h * np.uint32(0xBB67AE85)
    return h ^ (h >> np.uint32(16))


def random_bits(seed, t, l, n):
    g = 0x9E3779B9
    one = lambda x: np.array([x & 0xFFFFFFFF], np.uint32)  # noqa: E731
    key = mix(one(int(mix(one(seed + t * g))[0]) + l * g))
    return mix(key + np.arange(n, dtype=np.uint64).astype(np.uint32) * np.uint32(g))


def decode(codes):
    """fp32 values of e4m3 codes."""
    c = codes.astype(np.int64)
    s, e, f = np.where(c & 128, -1.0, 1.0), (c >> 3) & 15, c & 7
    x = np.where(e > 0, (8 + f) * 2.0 ** (e - 10.0), f * 2.0 ** -9)
    return np.where((c & 127) == 127, np.nan, s * x).astype(F)


def encode(x, scale, bits16):
    """Codes of x / scale, rounded by the random bits."""
    a = np.abs(x / scale)
    bad = ~np.isfinite(a)
    a = np.where(bad, F(0), a).astype(F)
    low = a < F(2.0 ** -6)
    t = np.where(low, a + F(2.0 ** -6), a).astype(F).view(np.uint32)
    c = ((t + (bits16 << np.uint32(4))) >> np.uint32(20)) - np.where(low, 968, 960).astype(np.uint32)
    c = np.where(bad, 0x7F, c)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def block_scales(x):
    n = x.size
    nb = -(-n // BLOCK)
    pad = np.zeros(nb * BLOCK, F)
    pad[:n] = np.where(np.isfinite(x), np.abs(x), 0)
    top = pad.reshape(nb, BLOCK).max(1)
    bits = top.view(np.uint32)
    field = (bits >> np.uint32(23)).astype(np.int64) - 8 + ((bits & np.uint32(0x7FFFFF)) > 0x600000)
    return (np.maximum(field, 1).astype(np.uint32) << np.uint32(23)).view(F)


def spread(s, n):
    return np.repeat(s, BLOCK)[:n]


def step32(q, l, t, hp, seed, decay):
    """The header's fp32 operations on one tensor's arrays (a dict), in numpy."""
    b1, b2, k = hp["beta1"], hp["beta2"], t + 1
    eta = (hp["eta0"] - hp["eta_min"]) * (1 - min(t, 100) / 100) + hp["eta_min"]
    n = q["p"].size
    eight = "ms" in q
    with np.errstate(all="ignore"):
        if eight:
            m, r = decode(q["m"]) * spread(q["ms"], n), decode(q["v"]) * spread(q["vs"], n)
            v = r * r
        else:
            m, v = q["m"], q["v"]
        g = q["g"]
        m = m * F(b1) + g * F(1 - b1)
        v = v * F(b2) + (g * g) * F(1 - b2)
        r = np.sqrt(v)
        d = (m / (r * F(1 / np.sqrt(1 - b2 ** k)) + F(hp["eps"]))) * F(eta / (1 - b1 ** k))
        out = dict(q, p=q["p"] * (F(1) - F(eta) * F(decay)) - d)
        if eight:
            h = random_bits(seed, t, l, n)
            out["ms"], out["vs"] = block_scales(m), block_scales(r)
            out["m"] = encode(m, spread(out["ms"], n), h & np.uint32(0xFFFF))
            c = encode(r, spread(out["vs"], n), h >> np.uint32(16))
            out["v"] = np.where((c == 0) & (v > 0), 1, c).astype(np.uint8)
        else:
            out["m"], out["v"] = m, v
    assert all(out[x].dtype == (np.uint8 if eight and x in "mv" else F) for x in ("p", "m", "v"))
    return out


class Guarded:
    """A buffer of n values between guard bands."""

    def __init__(self, a):
        a = torch.as_tensor(a)
        self.n = a.numel()
        self.buf = torch.full((self.n + 2 * GUARD,), 7, dtype=a.dtype, device="cuda")
        self.t = self.buf[GUARD:GUARD + self.n]
        self.t.copy_(a)

    def get(self):
        b = self.buf.cpu()
        assert (b[:GUARD].float() == 7).all() and (b[GUARD + self.n:].float() == 7).all(), "written outside a tensor"
        return b[GUARD:GUARD + self.n]


def make(counts, eight, seed=0, g16=False):
    rng = np.random.Generator(np.random.PCG64(seed))
    out = []
    for n in counts:
        size = F(2.0 ** rng.integers(-14, -4))
        g = (size * rng.standard_normal(n)).astype(F)
        q = dict(p=(0.05 * rng.standard_normal(n)).astype(F), g=g)
        m, v = (0.3 * size * rng.standard_normal(n)).astype(F), (size * rng.standard_normal(n)).astype(F) ** 2
        if eight:
            q["ms"], q["vs"] = block_scales(m), block_scales(np.sqrt(v))
            bits = np.full(n, 0x8000, np.uint32)
            q["m"], q["v"] = encode(m, spread(q["ms"], n), bits), encode(np.sqrt(v), spread(q["vs"], n), bits)
        else:
            q["m"], q["v"] = m, v
        if g16:
            q["g"] = torch.as_tensor(g).bfloat16().float().numpy()
        out.append(q)
    return out


def to_device(qs, g16=False, p16=True):
    dev = []
    for q in qs:
        d = {k: Guarded(v) for k, v in q.items()}
        if g16:
            d["g"] = Guarded(torch.as_tensor(q["g"]).bfloat16())
        if p16:
            d["p16"] = Guarded(torch.zeros(q["p"].size, dtype=torch.bfloat16))
        dev.append(d)
    return dev


NAMES = dict(p="p", g="g", m="m", v="v", ms="m_scale", vs="v_scale", p16="p16")


def tensors_of(dev, decay):
    return B.make_adamw_tensors([dict({NAMES[k]: v.t for k, v in d.items()}, weight_decay=w) for d, w in zip(dev, decay)])


def same_bits(dev, qs):
    for d, q in zip(dev, qs):
        for k in q:
            got = d[k].get()
            if k == "g":
                continue
            got = got.numpy()
            assert np.array_equal(got.view(np.uint8), q[k].view(np.uint8)), (k, q["p"].size)
        if "p16" in d:
            assert torch.equal(d["p16"].get(), torch.as_tensor(q["p"]).bfloat16())


@gpu
@pytest.mark.parametrize("g16", [False, True])
@pytest.mark.parametrize("eight", [False, True])
def test_bits(eight, g16):
    qs = make(COUNTS, eight, 1, g16)
    decay = [0.1 * (i % 3) for i in range(len(qs))]
    dev = to_device(qs, g16)
    ts = tensors_of(dev, decay)
    for t in (0, 1, 57, 1000):
        B.cf_adamw_step(ts, t, B.make_adamw_hparams(100, seed=5, **HP))
        qs = [step32(q, l, t, HP, 5, w) for l, (q, w) in enumerate(zip(qs, decay))]
        same_bits(dev, qs)


@gpu
def test_mixed_list_of_many():
    """More tensors than a launch takes, of both kinds, empty ones among them."""
    rng = np.random.Generator(np.random.PCG64(7))
    counts = [int(c) for c in rng.integers(0, 900, 130)]
    qs = [make([c], i % 3 == 0, i)[0] for i, c in enumerate(counts)]
    dev = to_device(qs, p16=False)
    ts = tensors_of(dev, [0.01] * len(qs))
    for t in range(2):
        B.cf_adamw_step(ts, t, B.make_adamw_hparams(100, seed=9, **HP))
        qs = [step32(q, l, t, HP, 9, 0.01) for l, q in enumerate(qs)]
    same_bits(dev, qs)


@gpu
@pytest.mark.parametrize("eight", [False, True])
def test_large(eight):
    """Workgroups of several turns."""
    qs = make([9_000_001], eight, 3)
    dev = to_device(qs)
    B.cf_adamw_step(tensors_of(dev, [0.1]), 4, B.make_adamw_hparams(100, seed=1, **HP))
    same_bits(dev, [step32(qs[0], 0, 4, HP, 1, 0.1)])


@gpu
def test_against_float64():
    qs = make([5000], False, 4)
    dev = to_device(qs)
    t, decay, q = 3, 0.1, {k: v.astype(np.float64) for k, v in qs[0].items()}
    B.cf_adamw_step(tensors_of(dev, [decay]), t, B.make_adamw_hparams(100, **HP))
    eta = (HP["eta0"] - HP["eta_min"]) * (1 - t / 100) + HP["eta_min"]
    m, v = 0.9 * q["m"] + 0.1 * q["g"], 0.999 * q["v"] + 0.001 * q["g"] ** 2
    d = eta * (m / (1 - 0.9 ** 4)) / (np.sqrt(v / (1 - 0.999 ** 4)) + 1e-8)
    terms = eta * ((0.9 * abs(q["m"]) + 0.1 * abs(q["g"])) / (1 - 0.9 ** 4)) / (np.sqrt(v / (1 - 0.999 ** 4)) + 1e-8)
    p = (1 - eta * decay) * q["p"] - d
    u = 12 * 2.0 ** -24
    assert np.all(abs(dev[0]["m"].get().numpy() - m) <= u * (0.9 * abs(q["m"]) + 0.1 * abs(q["g"])))
    assert np.all(abs(dev[0]["v"].get().numpy() - v) <= u * v)
    assert np.all(abs(dev[0]["p"].get().numpy() - p) <= u * (terms + abs(q["p"])))


@gpu
def test_first_step_from_zero():
    """Zero bytes are the moments before the first update, whatever finite scales hold."""
    n = 700
    g = torch.randn(n, generator=torch.Generator().manual_seed(2))
    p0 = torch.zeros(n, device="cuda")
    z = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    s = [torch.ones(3, device="cuda") for _ in range(2)]
    p = p0.clone()
    ts = B.make_adamw_tensors([dict(p=p, g=g.cuda(), m=z[0], v=z[1], m_scale=s[0], v_scale=s[1])])
    B.cf_adamw_step(ts, 0, B.make_adamw_hparams(10, eta0=1e-2, eta_min=1e-2))
    # the first step is eta sign(g) but for eps / |g| of it
    assert float((p.cpu() + 1e-2 * g.sign()).abs().max()) <= 1e-2 * (1e-8 / float(g.abs().min()) + 12 * 2.0 ** -24)


@gpu
def test_zero_gradients_and_blocks():
    n = 600
    dev = to_device([dict(p=np.ones(n, F), g=np.zeros(n, F), m=np.zeros(n, np.uint8), v=np.zeros(n, np.uint8),
                          ms=np.ones(3, F), vs=np.ones(3, F))])
    B.cf_adamw_step(tensors_of(dev, [0.0]), 0, B.make_adamw_hparams(10))
    d = dev[0]
    assert (d["p"].get() == 1).all() and not d["m"].get().any() and not d["v"].get().any()
    assert (d["ms"].get() == 2.0 ** -126).all() and (d["vs"].get() == 2.0 ** -126).all()


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_not_finite_stays_at_its_value(bad):
    qs = make([1000], True, 6)
    qs[0]["g"][300] = bad
    dev = to_device(qs)
    B.cf_adamw_step(tensors_of(dev, [0.0]), 2, B.make_adamw_hparams(100, seed=3, **HP))
    ref = step32(qs[0], 0, 2, HP, 3, 0.0)
    hit = np.zeros(1000, bool)
    hit[300] = True
    for k in ("m", "v"):
        got = dev[0][k].get().numpy()
        assert np.array_equal(np.isnan(decode(got)), hit) and np.array_equal(got[~hit], ref[k][~hit])
    for k in ("ms", "vs"):
        assert np.array_equal(dev[0][k].get().numpy(), ref[k])
    assert np.array_equal(dev[0]["p"].get().numpy()[~hit], ref["p"][~hit])


@gpu
def test_codes_are_unbiased():
    """A constant second moment decays in 8 bits as in 32: over 400 steps without
    gradient v falls by 0.999^400 = 0.670.  A step moves sqrt(v) by a random number of
    codes of variance below step^2 / 4, so 400 steps and 65536 values leave the mean's
    spread below 20 / 2 / 256 = 4 % of a code's step (at most 1/8), 0.5 % of the value; four
    of those, and the squares' excess, the variance 100 steps^2 / 64 / 65536, are within 3 %."""
    n = 1 << 16
    rng = np.random.Generator(np.random.PCG64(11))
    r = (0.5 + 0.5 * rng.random(n)).astype(F)
    vs = block_scales(r)
    dev = to_device([dict(p=np.zeros(n, F), g=np.zeros(n, F), m=np.zeros(n, np.uint8), v=encode(r, spread(vs, n), np.full(n, 0x8000, np.uint32)),
                          ms=np.ones(n // BLOCK, F), vs=vs)], p16=False)
    r0 = decode(dev[0]["v"].get().numpy()).astype(np.float64) * spread(vs, n)
    ts = tensors_of(dev, [0.0])
    for t in range(400):
        B.cf_adamw_step(ts, t, B.make_adamw_hparams(1000, seed=13))
    r1 = decode(dev[0]["v"].get().numpy()).astype(np.float64) * spread(dev[0]["vs"].get().numpy(), n)
    assert abs(r1.mean() / (r0.mean() * 0.999 ** 200) - 1) < 0.03


@gpu
def test_captured_on_a_stream():
    qs = make([5000, 300], True, 8)
    dev, ref = to_device(qs), to_device(qs)
    hp = B.make_adamw_hparams(100, seed=4, **HP)
    ts, tr = tensors_of(dev, [0.1, 0.0]), tensors_of(ref, [0.1, 0.0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.cf_adamw_step(ts, 2, hp, stream=s)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        B.cf_adamw_step(tr, 2, hp)
        for a, b in zip(dev, ref):
            assert all(torch.equal(a[k].get(), b[k].get()) for k in a)


@gpu
def test_past_a_piece():
    """A tensor past 2^30 values (one entry of a launch): random bits and blocks go on."""
    n = (1 << 30) + 1000
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.ones(-(-n // BLOCK), device="cuda") for _ in range(2))
    tail = 2000
    gt = torch.as_tensor(make([tail], False, 9)[0]["g"]).bfloat16()
    g[n - tail:] = gt.cuda()
    B.cf_adamw_step(B.make_adamw_tensors([dict(p=p, g=g, m=m, v=v, m_scale=ms, v_scale=vs, weight_decay=0.1)]), 0,
                    B.make_adamw_hparams(100, seed=6, **HP))
    # the last blocks: those from the first multiple of 256 in the tail on
    beg = -(-(n - tail) // BLOCK) * BLOCK
    k = n - beg
    zero = dict(p=np.zeros(k, F), g=gt.float().numpy()[tail - k:], m=np.zeros(k, np.uint8), v=np.zeros(k, np.uint8),
                ms=np.ones(-(-k // BLOCK), F), vs=np.ones(-(-k // BLOCK), F))
    one = np.array([0], np.uint32)
    base = random_bits(6, 0, 0, 1)
    assert base.size == one.size
    ref = step32(zero, 0, 0, HP, 6, 0.1)
    assert np.array_equal(p[beg:].cpu().numpy(), ref["p"])
    h = mix(mix(mix(np.array([6], np.uint32))) + (np.arange(beg, n, dtype=np.uint64) & 0xFFFFFFFF).astype(np.uint32) * np.uint32(0x9E3779B9))
    mm = zero["g"] * F(1 - 0.9)
    assert np.array_equal(m[beg:].cpu().numpy(), encode(mm, spread(ref["ms"], k), h & np.uint32(0xFFFF)))
    assert not p[: beg - BLOCK * 8].any()


@gpu
def test_shared_gradient():
    g = torch.randn(500, device="cuda")
    ps = [torch.zeros(500, device="cuda") for _ in range(2)]
    st = [[torch.zeros(500, device="cuda") for _ in range(2)] for _ in range(2)]
    ts = B.make_adamw_tensors([dict(p=p, g=g, m=a, v=b) for p, (a, b) in zip(ps, st)])
    B.cf_adamw_step(ts, 0, B.make_adamw_hparams(10))
    assert torch.equal(ps[0], ps[1]) and ps[0].any()


# ---- refusals (no kernel is launched) ------------------------------------------------

A = 0x7F0000000000
M = 1 << 24


def entry(**kw):
    q = dict(p=A, g=A + M, m=A + 2 * M, v=A + 3 * M, m_scale=None, v_scale=None, p16=None, count=1000, weight_decay=0.0, g_dtype=0)
    q.update(kw)
    return B.cf_adamw_tensor(*[q[k] for k in ("p", "g", "m", "v", "m_scale", "v_scale", "p16", "count", "weight_decay", "g_dtype")])


def expect(status, entries, t=0, **hp):
    arr = (B.cf_adamw_tensor * max(1, len(entries)))(*entries)
    with pytest.raises(B.CfError) as e:
        B.cf_adamw_step((len(entries), arr), t, B.make_adamw_hparams(**dict(dict(t_decay=10), **hp)), stream=0)
    assert e.value.status == status, str(e.value)


def test_refusals():
    bad = B.CF_ERR_INVALID_ARG
    for hp in (dict(t_decay=0), dict(eta0=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=float("inf"))):
        expect(bad, [entry()], **hp)
    expect(bad, [entry()], t=-1)
    for kw in (dict(count=-1), dict(count=1 << 40), dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(g_dtype=2),
               dict(m_scale=A + 4 * M), dict(v_scale=A + 4 * M), dict(p=None), dict(g=None), dict(m=None), dict(v=None)):
        expect(bad, [entry(**kw)])
    for k in ("p", "g", "m", "v", "p16"):
        expect(B.CF_ERR_ALIGNMENT, [entry(**{k: A + 9 * M + 4})])
    expect(B.CF_ERR_ALIGNMENT, [entry(m_scale=A + 4 * M + 2, v_scale=A + 5 * M)])
    for kw in (dict(g=A), dict(m=A + 16), dict(v=A + 2 * M), dict(p16=A + M), dict(p16=A + 2 * M + 16),
               dict(m_scale=A, v_scale=A + 5 * M), dict(m_scale=A + 5 * M, v_scale=A + 5 * M)):
        expect(B.CF_ERR_ALIAS, [entry(**kw)])
    other = dict(p=A + 4 * M, g=A + M, m=A + 5 * M, v=A + 6 * M)
    expect(B.CF_ERR_ALIAS, [entry(), entry()])
    expect(B.CF_ERR_ALIAS, [entry(), entry(**dict(other, p=A + 3984))])
    expect(B.CF_ERR_ALIAS, [entry(), entry(**dict(other, v=A + M))])
    expect(B.CF_ERR_ALIAS, [entry(**other), entry(**dict(other, p=A + 7 * M, m=A + 8 * M, v=A + 9 * M, g=A + 4 * M))])
    arr = (B.cf_adamw_tensor * 1)(entry())
    for n in (-1, 1 << 17):
        with pytest.raises(B.CfError):
            B.cf_adamw_step((n, arr), 0, B.make_adamw_hparams(10), stream=0)
    with pytest.raises(B.CfError):
        B._check(B.lib().cf_adamw_step(1, arr, 0, None, None))
    with pytest.raises(B.CfError):
        B._check(B.lib().cf_adamw_step(1, None, 0, B.make_adamw_hparams(10), None))


def test_nothing_to_do():
    B.cf_adamw_step((0, (B.cf_adamw_tensor * 1)()), 0, B.make_adamw_hparams(10), stream=0)
    arr = (B.cf_adamw_tensor * 1)(entry(count=0, p=None, g=None))
    B.cf_adamw_step((1, arr), 0, B.make_adamw_hparams(10), stream=0)


def test_tensors_are_checked():
    z = torch.zeros
    ok = dict(p=z(10), g=z(10), m=z(10), v=z(10))
    assert B.make_adamw_tensors([ok])[0] == 1
    for k, x in (("g", z(9)), ("m", z(10, dtype=torch.uint8)), ("v", z(10).double()), ("p", z(20)[::2]), ("g", None),
                 ("p16", z(10)), ("m_scale", z(1))):
        with pytest.raises(ValueError):
            B.make_adamw_tensors([dict(ok, **{k: x})])
    eight = dict(ok, m=z(10, dtype=torch.uint8), v=z(10, dtype=torch.float8_e4m3fn), m_scale=z(1), v_scale=z(1))
    B.make_adamw_tensors([eight])
    with pytest.raises(ValueError):
        B.make_adamw_tensors([dict(eight, v_scale=z(2))])
