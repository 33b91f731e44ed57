"""GPU parity of the matrix products with bias, activation and residual, and of their
gradients, through the C ABI.

Small whole numbers make every product and sum exact in fp32 whatever its order, so
those results are compared bit by bit.  Otherwise, with T the sum of the absolute
terms of an output, an fp32 sum of L + 2 terms in any order is within
(L + 8) 2^-23 T (the matrix units may cut instead of rounding); activations are within
2^-21 |z| of the formulas and their derivatives, at most 1.13, within 2^-20; a bf16
output adds half a step, 2^-8 |value|."""
import math

import numpy as np
import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

ALPHA = 0.01
GUARD = 64
ACTS = ["none", "lrelu", "silu", "gelu"]
SHAPES = [(1, 1, 1), (1, 7, 3), (3, 1, 5), (5, 8, 1), (64, 128, 512), (63, 65, 67), (64, 64, 64), (65, 32, 129), (128, 256, 128),
          (257, 100, 255), (256, 512, 256), (1, 4096, 1000), (1000, 3, 1000), (33, 1000, 8), (300, 520, 260), (129, 2048, 64),
          (1331, 130, 517), (512, 192, 1024), (2048, 64, 72), (96, 4104, 40), (7, 16, 8192), (4100, 40, 24), (40, 24, 4100),
          (16384, 16, 16), (20000, 5, 3), (4096, 1024, 1024), (4104, 264, 4088), (520, 4200, 4104), (8192, 72, 4096)]


def _t(dt):
    return torch.bfloat16 if dt == "bf16" else torch.float32


def _curve(u, act, alpha=ALPHA):
    if act == "lrelu":
        return torch.where(u > 0, u, alpha * u), torch.where(u > 0, 1.0, alpha).to(u.dtype)
    if act == "silu":
        s = torch.sigmoid(u)
        return u * s, s * (1 + u * (1 - s))
    if act == "gelu":
        q = 0.5 * torch.erfc(-u / math.sqrt(2))
        return u * q, q + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    return u, torch.ones_like(u)


class Guarded:
    """An output between two guard bands; every value starts as NaN."""

    def __init__(self, shape, dtype):
        n = int(np.prod(shape))
        self.buf = torch.full((n + 2 * GUARD,), float("nan"), dtype=dtype, device="cuda")
        self.buf[:GUARD] = 7.0
        self.buf[GUARD + n:] = 7.0
        self.t = self.buf[GUARD:GUARD + n].view(shape)
        self.n = n

    def get(self):
        b = self.buf.float().cpu()
        assert (b[:GUARD] == 7).all() and (b[GUARD + self.n:] == 7).all(), "written outside the output"
        return self.t.double().cpu()


def _ws(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda").fill_(0xff)  # NaN patterns


def _gen(*key):
    return torch.Generator().manual_seed(sum(k * p for k, p in zip(key, (1, 7919, 104729, 13))))


def _whole(g, shape, dt, most=2):
    return torch.randint(-most, most + 1, shape, generator=g).to(_t(dt))


def _real(g, shape, dt, s=1.0):
    return (s * torch.randn(shape, generator=g)).to(_t(dt))


def _fwd(x, w, b, act, r, dt, with_z=True, stream=None):
    m, k, n = x.shape[0], x.shape[1], w.shape[1]
    y, z = Guarded((m, n), _t(dt)), Guarded((m, n), _t(dt)) if with_z else None
    dev = [None if t is None else t.cuda() for t in (x, w, b, r)]
    B.cf_linear_fwd(m, k, n, dt, dev[0], dev[1], dev[2], act, ALPHA, dev[3], y.t, z.t if z else None,
                    _ws(B.cf_linear_fwd_workspace_size(m, k, n, dt)), stream=stream)
    return y, z


def _data(dz, w, r, z, act, dt):
    m, n, k = dz.shape[0], dz.shape[1], w.shape[0]
    dx = Guarded((m, k), _t(dt))
    dev = [None if t is None else t.cuda() for t in (dz, w, r, z)]
    B.cf_linear_bwd_data(m, k, n, dt, dev[0], dev[1], dev[2], dev[3], act, ALPHA, dx.t,
                         _ws(B.cf_linear_bwd_data_workspace_size(m, k, n, dt)))
    return dx


def _weight(x, dz, dt, with_db=True):
    m, k, n = x.shape[0], x.shape[1], dz.shape[1]
    dw, db = Guarded((k, n), torch.float32), Guarded((n,), torch.float32) if with_db else None
    B.cf_linear_bwd_weight(m, k, n, dt, x.cuda(), dz.cuda(), dw.t, db.t if db else None,
                           _ws(B.cf_linear_bwd_weight_workspace_size(m, k, n, dt)))
    return dw, db


def _round(t, dt):
    return t.to(_t(dt)).double()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_whole_numbers(m, k, n, dt):
    g = _gen(m, k, n, 1)
    x, w, dz = _whole(g, (m, k), dt), _whole(g, (k, n), dt), _whole(g, (m, n), dt)
    b, r, rx = _whole(g, (n,), "f32", 50), _whole(g, (m, n), dt, 50), _whole(g, (m, k), dt, 50)
    x64, w64, dz64 = x.double(), w.double(), dz.double()
    z64 = x64 @ w64 + b.double()
    y, z = _fwd(x, w, b, "none", r, dt)
    assert torch.equal(z.get(), _round(z64, dt))
    assert torch.equal(y.get(), _round(z64 + r.double(), dt))
    y, _ = _fwd(x, w, None, "none", None, dt, with_z=False)
    assert torch.equal(y.get(), _round(x64 @ w64, dt))
    dx = _data(dz, w, rx, None, "none", dt)
    assert torch.equal(dx.get(), _round(dz64 @ w64.t() + rx.double(), dt))
    # a slope of 1 / 2 at every negative value and at zero
    zin = _whole(g, (m, k), dt)
    dev = torch.empty((m, k), dtype=_t(dt), device="cuda")
    B.cf_linear_bwd_data(m, k, n, dt, dz.cuda(), w.cuda(), None, zin.cuda(), "lrelu", 0.5, dev,
                         _ws(B.cf_linear_bwd_data_workspace_size(m, k, n, dt)))
    assert torch.equal(dev.double().cpu(), _round(dz64 @ w64.t() * torch.where(zin.double() > 0, 1.0, 0.5), dt))
    dw, db = _weight(x, dz, dt)
    assert torch.equal(dw.get(), x64.t() @ dz64)
    assert torch.equal(db.get(), dz64.sum(0))
    dw, _ = _weight(x, dz, dt, with_db=False)
    assert torch.equal(dw.get(), x64.t() @ dz64)


def _check(got, ref, lim, dt):
    lim = lim + (2.0 ** -8 * ref.abs() if dt == "bf16" else 2.0 ** -24 * ref.abs())
    assert not torch.isnan(got).any()
    assert bool(((got - ref).abs() <= lim).all()), float(((got - ref).abs() - lim).max())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_real_numbers(m, k, n, dt):
    g = _gen(m, k, n, 2)
    x, w, dz = _real(g, (m, k), dt), _real(g, (k, n), dt, k ** -0.5), _real(g, (m, n), dt)
    b, r, rx, zin = _real(g, (n,), "f32"), _real(g, (m, n), dt), _real(g, (m, k), dt), _real(g, (m, k), dt, 3.0)
    x64, w64, dz64 = x.double(), w.double(), dz.double()
    z64 = x64 @ w64 + b.double()
    ez = (k + 8) * 2.0 ** -23 * (x64.abs() @ w64.abs() + b.double().abs())
    s64 = dz64 @ w64.t()
    es = (n + 8) * 2.0 ** -23 * (dz64.abs() @ w64.abs().t() + rx.double().abs())
    for act in ACTS:
        y, z = _fwd(x, w, b, act, r, dt)
        _check(z.get(), z64, ez, dt)
        # the sum with the residual is rounded too
        y64 = _curve(z64, act)[0] + r.double()
        _check(y.get(), y64, 1.13 * ez + 2.0 ** -21 * z64.abs() + 2.0 ** -23 * y64.abs(), dt)
        dx = _data(dz, w, rx, zin, act, dt)
        _check(dx.get(), (s64 + rx.double()) * _curve(zin.double(), act)[1], 1.13 * es + 2.0 ** -20 * (s64 + rx.double()).abs(), dt)
    dw, db = _weight(x, dz, dt)
    _check(dw.get(), x64.t() @ dz64, (m + 8) * 2.0 ** -23 * (x64.abs().t() @ dz64.abs()), "f32")
    _check(db.get(), dz64.sum(0), (m + 8) * 2.0 ** -23 * dz64.abs().sum(0), "f32")


def test_gradients_against_differences():
    """dx, dW and db of sum(c y) against central differences in float64 (a third
    derivative's h^2 / 6 and 2^-52 / h, below 1e-6 at h = 1e-4)."""
    m, k, n = 5, 6, 7
    g = _gen(m, k, n, 3)
    z0, w, b, c = (_real(g, s, "f32") for s in ((m, k), (k, n), (n,), (m, n)))
    for act in ("silu", "gelu"):
        x = _curve(z0.double(), act)[0].float()
        dx = _data(c, w, None, z0, act, "f32").get()
        dw, db = (t.get() for t in _weight(x, c, "f32"))

        def loss(z, w, b):
            return float(((_curve(z, act)[0] @ w + b) * c.double()).sum())

        args = [z0.double(), w.double(), b.double()]
        for i, got in enumerate((dx, dw, db)):
            num = torch.zeros_like(args[i])
            for j in range(num.numel()):
                d = []
                for h in (1e-4, -1e-4):
                    a = [t.clone() for t in args]
                    a[i].view(-1)[j] += h
                    d.append(loss(*a))
                num.view(-1)[j] = (d[0] - d[1]) / 2e-4
            assert float((got - num).abs().max()) <= 1e-5 * float(num.abs().max())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(70, 40, 50), (256, 128, 256)])
def test_in_place(m, k, n, dt):
    g = _gen(m, k, n, 4)
    x, w, dz = _real(g, (m, k), dt), _real(g, (k, n), dt), _real(g, (m, n), dt)
    b, r, rx, zin = _real(g, (n,), "f32"), _real(g, (m, n), dt), _real(g, (m, k), dt), _real(g, (m, k), dt)
    y, _ = _fwd(x, w, b, "silu", r, dt)
    rc = r.cuda()
    B.cf_linear_fwd(m, k, n, dt, x.cuda(), w.cuda(), b.cuda(), "silu", ALPHA, rc, rc, None,
                    _ws(B.cf_linear_fwd_workspace_size(m, k, n, dt)))
    assert torch.equal(rc, y.t)
    dx = _data(dz, w, rx, zin, "silu", dt)
    for over in (0, 1):
        t = [rx.cuda(), zin.cuda()]
        B.cf_linear_bwd_data(m, k, n, dt, dz.cuda(), w.cuda(), t[0], t[1], "silu", ALPHA, t[over],
                             _ws(B.cf_linear_bwd_data_workspace_size(m, k, n, dt)))
        assert torch.equal(t[over], dx.t)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(70, 41, 50), (512, 256, 256)])
def test_not_finite(m, k, n, dt):
    """A NaN or an infinity reaches the outputs whose formula has it, and no others."""
    g = _gen(m, k, n, 5)
    for bad in (float("nan"), float("inf")):
        x, w, dz = _real(g, (m, k), dt), _real(g, (k, n), dt), _real(g, (m, n), dt)
        x[3, 5], dz[4, 6] = bad, bad
        y, z = _fwd(x, w, None, "none", None, dt)
        rows = torch.zeros(m, dtype=torch.bool)
        rows[3] = True
        want = x.double() @ w.double()
        assert torch.equal(torch.isfinite(z.get()).all(1), ~rows)
        if math.isinf(bad):
            assert torch.equal(z.get()[3], want[3])
        dx = _data(dz, w, None, None, "none", dt).get()
        rows = torch.zeros(m, dtype=torch.bool)
        rows[4] = True
        assert torch.equal(torch.isfinite(dx).all(1), ~rows) and torch.equal(torch.isfinite(dx).any(1), ~rows)
        dw, db = (t.get() for t in _weight(x, dz, dt))
        hit = torch.zeros((k, n), dtype=torch.bool)
        hit[5, :] = hit[:, 6] = True
        assert torch.equal(~torch.isfinite(dw), hit)
        assert torch.equal(~torch.isfinite(db), hit.all(0))


def test_empty():
    w = torch.ones((4, 3), device="cuda")
    y = torch.full((3,), 5.0, device="cuda")
    B.cf_linear_fwd(0, 4, 3, "f32", w, w, None, "none", 0.0, None, y)
    B.cf_linear_bwd_data(0, 4, 3, "f32", w, w, None, None, "none", 0.0, y)
    dw, db = torch.full((4, 3), 2.0, device="cuda"), torch.full((3,), 2.0, device="cuda")
    B.cf_linear_bwd_weight(0, 4, 3, "f32", None, None, dw, db)
    assert not dw.any() and not db.any() and (y == 5).all()


@pytest.mark.parametrize("dt,m,k,n", [("f32", 100, 30, 60), ("bf16", 300, 72, 136), ("bf16", 2048, 256, 512), ("f32", 2048, 64, 64)])
def test_captured_on_a_stream(dt, m, k, n):
    g = _gen(m, k, n, 6)
    x, w, dz, zin = (_real(g, s, dt).cuda() for s in ((m, k), (k, n), (m, n), (m, k)))
    b = _real(g, (n,), "f32").cuda()
    y, z, dx = torch.empty_like(dz), torch.empty_like(dz), torch.empty_like(x)
    dw, db = torch.empty((k, n), device="cuda"), torch.empty(n, device="cuda")
    ws = _ws(max(B.cf_linear_fwd_workspace_size(m, k, n, dt), B.cf_linear_bwd_data_workspace_size(m, k, n, dt),
                 B.cf_linear_bwd_weight_workspace_size(m, k, n, dt)))

    def run(stream):
        B.cf_linear_fwd(m, k, n, dt, x, w, b, "gelu", ALPHA, None, y, z, ws, stream=stream)
        B.cf_linear_bwd_data(m, k, n, dt, dz, w, None, zin, "gelu", ALPHA, dx, ws, stream=stream)
        B.cf_linear_bwd_weight(m, k, n, dt, x, dz, dw, db, ws, stream=stream)

    outs = (y, z, dx, dw, db)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run(s)
    for i in range(4):
        x.mul_(1.25).add_(0.1 * i)
        for t in outs + (ws,):
            t.fill_(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        run(None)
        assert all(torch.equal(a, c) for a, c in zip(got, outs))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_past_32_bits(dt):
    """Rows past 2^31 values: the last ones as they are alone."""
    m, k, n = (1 << 25) + 3, 8, 72
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randint(-2, 3, (m, k), generator=g, device="cuda").to(_t(dt))
    w = torch.randint(-2, 3, (k, n), generator=g, device="cuda").to(_t(dt))
    y = torch.empty((m, n), dtype=_t(dt), device="cuda")
    B.cf_linear_fwd(m, k, n, dt, x, w, None, "none", 0.0, None, y, None, _ws(B.cf_linear_fwd_workspace_size(m, k, n, dt)))
    at = torch.cat([torch.arange(0, 300), torch.arange(m // 2, m // 2 + 300), torch.arange(m - 300, m)]).cuda()
    assert torch.equal(y[at].double(), x[at].double() @ w.double())
    dx = torch.empty_like(x)
    B.cf_linear_bwd_data(m, k, n, dt, y, w, None, None, "none", 0.0, dx, _ws(B.cf_linear_bwd_data_workspace_size(m, k, n, dt)))
    assert torch.equal(dx[at].double(), (y[at].double() @ w.double().t()).to(_t(dt)).double())
    # dW = x' y: sums of 2^25 whole terms of at most 64; slices of 2^16 of them are exact, and
    # 2^9 slices are joined in a tree whose paths are at most 8 + 6 additions: 14 2^-24 < 2^-20
    dw = torch.empty((k, n), device="cuda")
    B.cf_linear_bwd_weight(m, k, n, dt, x, y, dw, None, _ws(B.cf_linear_bwd_weight_workspace_size(m, k, n, dt)))
    ref = sum(x[i:i + (1 << 22)].double().t().contiguous() @ y[i:i + (1 << 22)].double() for i in range(0, m, 1 << 22))
    assert float((dw.double() - ref).abs().max()) <= 2.0 ** -20 * float(ref.abs().max())


# 4096 x 4096 outputs of 64 terms are one round of the large tiles, whose epilogues look
# activations and slopes up.  Terms that are zeros, or one that is 1, leave the epilogue alone:
# its value to 2^-14 of itself and 2^-21 |u|, or its slope to 2^-16, and half a step of bf16.
@pytest.mark.parametrize("part", range(4))
def test_gelu_of_large_tiles(part):
    m = n = 4096
    u = torch.linspace(-10, 10, 4 * n, dtype=torch.float64)[part::4].float()
    u[:8] = torch.tensor([0.0, -0.0, 40.0, -40.0, 1e30, -1e30, math.inf, math.nan])
    x, w = torch.zeros(m, 64, device="cuda").bfloat16(), torch.ones(64, n, device="cuda").bfloat16()
    y = torch.full((m, n), 7.0, device="cuda").bfloat16()
    z = torch.empty_like(y)
    ws = torch.empty(max(16, B.cf_linear_fwd_workspace_size(m, 64, n, "bf16")), dtype=torch.uint8, device="cuda")
    B.cf_linear_fwd(m, 64, n, "bf16", x, w, u.cuda(), "gelu", 0.0, None, y, z, ws)
    assert torch.equal(y[:1].expand(m, n)[:, :7], y[:, :7]) and torch.equal(y[:1, 8:].expand(m, n - 8), y[:, 8:])
    got, d = y[m // 2].double().cpu(), u.double()
    assert got[6] == math.inf and math.isnan(got[7]) and bool(torch.isnan(y[:, 7]).all())
    want = d * 0.5 * torch.erfc(-d / math.sqrt(2))
    want[5] = 0.0
    keep = torch.ones(n, dtype=torch.bool)
    keep[6:8] = False
    err, bound = (got - want).abs(), (2.0 ** -8 + 2.0 ** -14) * want.abs() + 2.0 ** -21 * d.abs().clamp(max=8.0)
    assert bool((err <= bound)[keep].all()), float((err / bound)[keep].max())
    assert torch.equal(z[5].cpu()[keep], u.bfloat16()[keep])


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes_of_large_tiles(act):
    m = k = 4096
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    z = bits.view(torch.bfloat16).repeat(m * k // 65536).view(m, k).cuda()
    dz, w = torch.zeros(m, 64, device="cuda").bfloat16(), torch.zeros(k, 64, device="cuda").bfloat16()
    dz[:, 0] = 1
    w[:, 0] = 1
    dx = torch.full((m, k), 7.0, device="cuda").bfloat16()
    ws = torch.empty(max(16, B.cf_linear_bwd_data_workspace_size(m, k, 64, "bf16")), dtype=torch.uint8, device="cuda")
    B.cf_linear_bwd_data(m, k, 64, "bf16", dz, w, None, z, act, 0.0, dx, ws)
    rows = dx.view(-1, 65536).view(torch.int16)
    assert torch.equal(rows, rows[:1].expand_as(rows))
    got, u = dx.view(-1)[:65536].double().cpu(), bits.view(torch.bfloat16).double()
    assert bool(torch.isnan(got[torch.isnan(u)]).all())
    fin = torch.isfinite(u)
    got, u = got[fin], u[fin]
    if act == "gelu":
        want = 0.5 * torch.erfc(-u / math.sqrt(2)) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    else:
        s = torch.sigmoid(u)
        want = s * (1 + u * torch.sigmoid(-u))
    want = torch.where(u.abs() > 1e4, (u > 0).double(), want)
    err, bound = (got - want).abs(), 2.0 ** -8 * want.abs() + 2.0 ** -16
    assert bool((err <= bound).all()), float((err / bound).max())


# Outputs in both directions that take the tiles of 256, 128 and 64, whole and ragged; the
# formulas in float64 on the GPU.
LARGE = [(4096, 64, 4096, "bf16"), (4090, 72, 4104, "bf16"), (3901, 35, 4099, "bf16"), (4096, 128, 2048, "bf16"),
         (4001, 130, 2101, "bf16"), (1536, 64, 1536, "bf16"), (2048, 96, 2048, "f32"), (4001, 70, 2051, "f32"),
         (1024, 40, 1021, "f32")]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,terms,cols,dt", LARGE)
def test_epilogues_of_all_tiles(rows, terms, cols, dt, act):
    g = torch.Generator(device="cuda").manual_seed(rows + terms)

    def real(shape, s=1.0, t=None):
        return (s * torch.randn(shape, generator=g, device="cuda")).to(_t(t or dt))

    x, w, b, r, zin = real((rows, terms)), real((terms, cols), terms ** -0.5), real((cols,), 1.0, "f32"), real((rows, cols)), real((rows, cols), 3.0)
    s64, sabs = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    step = 2.0 ** -8 if dt == "bf16" else 2.0 ** -24

    def check(got, ref, lim):
        err, lim = (got.double() - ref).abs(), lim + step * ref.abs()
        assert bool((err <= lim).all()), float((err / lim).max())

    for res in (None, r):
        y, z = torch.full((rows, cols), math.nan, device="cuda", dtype=_t(dt)), torch.full((rows, cols), math.nan, device="cuda", dtype=_t(dt))
        B.cf_linear_fwd(rows, terms, cols, dt, x, w, b, act, ALPHA, res, y, z, _ws(B.cf_linear_fwd_workspace_size(rows, terms, cols, dt)))
        z64 = s64 + b.double()
        e = (terms + 8) * 2.0 ** -23 * (sabs + b.double().abs())
        check(z, z64, e)
        y64 = _curve(z64, act)[0] + (0.0 if res is None else res.double())
        # (the large tiles' GELU: 2^-20 z^2 of itself more, at most where the step of bf16 is 2^-8)
        table = 2.0 ** -14 * _curve(z64, act)[0].abs() if act == "gelu" and dt == "bf16" else 0.0
        check(y, y64, 1.13 * e + 2.0 ** -21 * z64.abs() + 2.0 ** -23 * y64.abs() + table)
        # the same numbers as a data gradient: dx = (x w^T ..) with w given as [cols][terms]
        dx = torch.full((rows, cols), math.nan, device="cuda", dtype=_t(dt))
        B.cf_linear_bwd_data(rows, cols, terms, dt, x, w.t().contiguous(), res, None if act == "none" else zin, act, ALPHA, dx,
                             _ws(B.cf_linear_bwd_data_workspace_size(rows, cols, terms, dt)))
        d64 = s64 + (0.0 if res is None else res.double())
        e = (terms + 8) * 2.0 ** -23 * (sabs + (0.0 if res is None else res.double().abs()))
        check(dx, d64 * _curve(zin.double(), act)[1], 1.13 * e + (2.0 ** -20 + (2.0 ** -15 if dt == "bf16" else 0.0)) * d64.abs())
    if act == "none":
        dw, db = torch.full((rows, cols), math.nan, device="cuda"), torch.full((cols,), math.nan, device="cuda")
        xt = x.t().contiguous()
        B.cf_linear_bwd_weight(terms, rows, cols, dt, xt, w, dw, db, _ws(B.cf_linear_bwd_weight_workspace_size(terms, rows, cols, dt)))
        step = 2.0 ** -24
        check(dw, s64, (terms + 8) * 2.0 ** -23 * sabs)
        check(db, w.double().sum(0), (terms + 8) * 2.0 ** -23 * w.double().abs().sum(0))


def test_other_stream_and_its_tensors():
    """Calls on a stream of their own, behind the work that fills their inputs there."""
    side = torch.cuda.Stream()
    m, k, n = 1100, 264, 520
    with torch.cuda.stream(side):
        x, w = torch.zeros(m, k, device="cuda").bfloat16(), torch.zeros(k, n, device="cuda").bfloat16()
        for _ in range(20):
            x += 0.125
            w += 0.0625
        y = torch.empty(m, n, device="cuda").bfloat16()
        B.cf_linear_fwd(m, k, n, "bf16", x, w, None, "none", 0.0, None, y, None,
                        _ws(B.cf_linear_fwd_workspace_size(m, k, n, "bf16")))
    side.synchronize()
    assert torch.equal(y, torch.full_like(y, 2.5 * 1.25 * k))
