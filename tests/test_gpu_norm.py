"""GPU parity of layer normalisation, forward and backward, through the C ABI,
against the formulas in float64.

Tolerances.  fp32: the framework's 1e-5 of the largest value an output could
have without cancellation (y: of max |y|; dx: of max_r rstd_r max |g_r|, since
short rows cancel almost entirely; dgamma and dbeta: of the largest sum of
absolute terms).  bf16 adds half a unit in the last of its eight bits of each
value, 2^-8 |value| to be clear of ties.  mean and rstd are fp32 for both."""
import numpy as np
import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

TOL = 1e-5
EPS = 1e-5
GUARD = 64

SHAPES = [(1, 1), (5, 1), (3, 2), (7, 3), (1, 5), (64, 4), (33, 16), (1000, 16), (4099, 8), (257, 31), (130, 64), (77, 65),
          (9, 255), (6, 256), (5, 257), (11, 512), (4, 1000), (3, 1023), (3, 1025), (5, 2049), (3, 4100), (2, 8192), (9, 8195),
          (2, 16384), (3, 16385), (1, 65536), (9, 65537), (1, 131073), (2, 300001), (40, 20000), (2049, 777), (300, 3000),
          (500, 7), (100, 21), (101, 43), (50, 90), (41, 180), (30, 370), (21, 700), (5, 1400), (700, 17), (3, 5100), (300, 17000)]


def _t(dt):
    return torch.bfloat16 if dt == "bf16" else torch.float32


def _data(rows, c, dt, seed=0):
    g = torch.Generator().manual_seed(seed * 7919 + rows * 31 + c)
    x = torch.randn((rows, c), generator=g) * (0.5 + torch.rand((rows, 1), generator=g)) + torch.randn((rows, 1), generator=g)
    dy = torch.randn((rows, c), generator=g)
    gamma, beta = 1 + 0.3 * torch.randn(c, generator=g), 0.3 * torch.randn(c, generator=g)
    return x.to(_t(dt)), dy.to(_t(dt)), gamma, beta


def _fwd64(x, gamma, beta, eps=EPS):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    return (x - mean) * rstd * gamma.double() + beta.double(), mean[:, 0], rstd[:, 0]


def _bwd64(x, dy, gamma, mean, rstd):
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    d = dy.double()
    g = d * gamma.double()
    dx = rstd.double()[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (d * xh).sum(0), d.sum(0), g, xh


class Guarded:
    """An output of n values between two guard bands; every value starts as NaN."""

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


def _run_fwd(x, gamma, beta, dt, eps=EPS, stream=None):
    rows, c = x.shape
    y, mean, rstd = Guarded((rows, c), _t(dt)), Guarded((rows,), torch.float32), Guarded((rows,), torch.float32)
    ws = _ws(B.cf_layernorm_fwd_workspace_size(rows, c, dt))
    B.cf_layernorm_fwd(rows, c, dt, x.cuda(), gamma.cuda(), beta.cuda(), eps, y.t, mean.t, rstd.t, ws, stream=stream)
    return y, mean, rstd


def _run_bwd(x, dy, gamma, mean, rstd, dt):
    rows, c = x.shape
    dx, dg, db = Guarded((rows, c), _t(dt)), Guarded((c,), torch.float32), Guarded((c,), torch.float32)
    ws = _ws(B.cf_layernorm_bwd_workspace_size(rows, c, dt))
    B.cf_layernorm_bwd(rows, c, dt, dy.cuda(), x.cuda(), gamma.cuda(), mean.cuda(), rstd.cuda(), dx.t, dg.t, db.t, ws)
    return dx, dg, db


def _close(got, ref, scale, dt):
    err = (got - ref).abs()
    lim = TOL * scale + (2.0 ** -8 * ref.abs() if dt == "bf16" else 0.0)
    assert not torch.isnan(got).any()
    assert (err <= lim).all(), float((err - lim).max())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
def test_forward(rows, c, dt):
    x, _, gamma, beta = _data(rows, c, dt)
    y, mean, rstd = _run_fwd(x, gamma, beta, dt)
    ry, rm, rr = _fwd64(x, gamma, beta)
    # a mean's error, relative to the row's spread, is an error of y
    scale = max(float(ry.abs().max()), float((x.double().abs().amax(1) * rr).max()) if c > 1 else 1.0)
    _close(mean.get(), rm, float(x.double().abs().max()), "f32")
    if c > 1:
        _close(rstd.get(), rr, float(rr.max()), "f32")
        _close(y.get(), ry, scale, dt)
    else:
        assert torch.equal(y.get(), beta.expand(rows, 1).to(_t(dt)).double())  # a single value is its own mean


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
def test_backward(rows, c, dt):
    x, dy, gamma, beta = _data(rows, c, dt, 1)
    _, mean, rstd = _fwd64(x, gamma, beta)
    mean, rstd = mean.float(), rstd.float()
    dx, dg, db = _run_bwd(x, dy, gamma, mean, rstd, dt)
    rx, rg, rb, g, xh = _bwd64(x, dy, gamma, mean, rstd)
    _close(dx.get(), rx, float((rstd.double() * g.abs().amax(1)).max()), dt)
    d = dy.double().abs()
    _close(dg.get(), rg, float((d * xh.abs()).sum(0).max()) if c > 1 else 1.0, "f32")
    _close(db.get(), rb, float(d.sum(0).max()), "f32")
    if c == 1:
        assert (dx.get() == 0).all()


@pytest.mark.parametrize("rows,c", [(4, 7), (3, 48), (2, 5000), (2, 140001)])
def test_gradients_against_differences(rows, c):
    """Directional derivatives of sum(w * y) in float64 against the kernels' gradients."""
    x, w, gamma, beta = _data(rows, c, "f32", 2)
    _, mean, rstd = _fwd64(x, gamma, beta)
    dx, dg, db = (t.get() for t in _run_bwd(x, w, gamma, mean.float(), rstd.float(), "f32"))
    g = torch.Generator().manual_seed(5)
    ux, ug, ub = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((rows, c), (c,), (c,)))
    h = 1e-5

    def f(s):
        return (w.double() * _fwd64(x.double() + s * ux, gamma.double() + s * ug, beta.double() + s * ub)[0]).sum()

    num = (f(h) - f(-h)) / (2 * h)
    ana = (dx * ux).sum() + (dg * ug).sum() + (db * ub).sum()
    size = (dx * ux).abs().sum() + (dg * ug).abs().sum() + (db * ub).abs().sum()
    assert abs(num - ana) <= 1e-5 * size


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(70, 16), (9, 333), (3, 5001), (3, 20000), (3, 140000)])
def test_infinite_and_nan_rows_stay_apart(rows, c, dt):
    x, dy, gamma, beta = _data(rows, c, dt, 3)
    x[0, c // 2] = float("inf")
    x[2, c - 1] = float("nan")
    y, mean, rstd = _run_fwd(x, gamma, beta, dt)
    ry, rm, rr = _fwd64(x, gamma, beta)
    got = y.t.double().cpu()
    y.t.nan_to_num_(0.0)
    y.get()
    bad = torch.zeros(rows, dtype=torch.bool)
    bad[0] = bad[2] = True
    assert torch.isnan(ry[bad]).all() and torch.isnan(got[bad]).all()
    _close(got[~bad], ry[~bad], max(float(ry[~bad].abs().max()), float((x[~bad].double().abs().amax(1) * rr[~bad]).max())), dt)
    m, s = rm.float(), rr.float()
    dx, dg, db = _run_bwd(x, dy, gamma, m, s, dt)
    gx = dx.t.double().cpu()
    rx, _, rb, g, _ = _bwd64(x, dy, gamma, m, s)
    assert torch.isnan(gx[bad]).all()
    _close(gx[~bad], rx[~bad], float((s.double() * g.abs().amax(1))[~bad].max()), dt)
    assert torch.isnan(dg.t).all()  # every column has a value of the bad rows
    _close(db.get(), rb, float(dy.double().abs().sum(0).max()), "f32")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(50, 16), (7, 777), (3, 9000), (3, 150001)])
def test_large_offset_and_constant_rows(rows, c, dt):
    """Rows far from zero keep their variance (it is not a difference of moments); constant rows give beta."""
    x, _, gamma, beta = _data(rows, c, "f32", 4)
    x = x + 64.0
    x[1] = 3.0
    x = x.to(_t(dt))
    y, mean, rstd = _run_fwd(x, gamma, beta, dt)
    ry, rm, rr = _fwd64(x, gamma, beta)
    assert float(((rstd.get() - rr).abs() / rr).max()) <= 1e-4  # 64 / spread units of 2^-24, squared distances
    err = (y.get() - ry).abs()
    lim = 2.0 ** -22 * 70.0 * rr[:, None] * (1 + gamma.double().abs().max()) + 1e-4 * ry.abs().max() * 0.1 + \
        (2.0 ** -8 * ry.abs() if dt == "bf16" else 0.0)
    assert (err <= lim).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(100, 16), (40, 513), (5, 6000), (5, 70000), (2, 200000)])
def test_in_place_repeat_and_side_stream(rows, c, dt):
    x, dy, gamma, beta = _data(rows, c, dt, 5)
    y, mean, rstd = _run_fwd(x, gamma, beta, dt)
    dx, dg, db = _run_bwd(x, dy, gamma, mean.t.cpu(), rstd.t.cpu(), dt)
    s = torch.cuda.Stream()
    dev = [t.cuda() for t in (x, dy, gamma, beta)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        xs, dys, ga, be = dev
        m2, r2 = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        yin = xs.clone()
        ws = _ws(max(B.cf_layernorm_fwd_workspace_size(rows, c, dt), B.cf_layernorm_bwd_workspace_size(rows, c, dt)))
        B.cf_layernorm_fwd(rows, c, dt, yin, ga, be, EPS, yin, m2, r2, ws)
        din, g2, b2 = dys.clone(), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        B.cf_layernorm_bwd(rows, c, dt, din, xs, ga, m2, r2, din, g2, b2, ws)
        xin = xs.clone()
        g3, b3 = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        B.cf_layernorm_bwd(rows, c, dt, dys, xin, ga, m2, r2, xin, g3, b3, ws)
    s.synchronize()
    for a, b in ((yin, y.t), (m2, mean.t), (r2, rstd.t), (din, dx.t), (xin, dx.t), (g2, dg.t), (b2, db.t), (g3, dg.t), (b3, db.t)):
        assert torch.equal(a, b)


def test_no_rows():
    one = torch.ones(16, device="cuda")
    dg, db = torch.full((16,), 3.0, device="cuda"), torch.full((16,), 3.0, device="cuda")
    B.cf_layernorm_fwd(0, 16, "f32", None, None, None, EPS, None, None, None)
    B.cf_layernorm_bwd(0, 16, "f32", None, None, one, None, None, None, dg, db, None)
    assert (dg == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_graph_replays(dt):
    """Captured calls replay to the eager bits, with eager work in between."""
    rows, c = 300, 96
    x, dy, gamma, beta = (t.cuda() for t in _data(rows, c, dt, 6))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = _ws(B.cf_layernorm_bwd_workspace_size(rows, c, dt))

    def calls():
        B.cf_layernorm_fwd(rows, c, dt, x, gamma, beta, EPS, y, mean, rstd)
        B.cf_layernorm_bwd(rows, c, dt, dy, x, gamma, mean, rstd, dx, dg, db, ws)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(3):
        x.copy_(_data(rows, c, dt, 10 + k)[0])
        calls()
        want = [t.clone() for t in (y, mean, rstd, dx, dg, db)]
        for t in (y, mean, rstd, dx, dg, db):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, mean, rstd, dx, dg, db)))


def test_offsets_past_32_bits():
    """More than 2^32 values: the last rows land where they belong."""
    rows, c = (1 << 28) + 3, 17
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    x = torch.zeros((rows, c), dtype=torch.bfloat16, device="cuda")
    tail, dy, gamma, beta = _data(64, c, "bf16", 7)
    x[-64:] = tail.cuda()
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.cf_layernorm_fwd(rows, c, "bf16", x, gamma.cuda(), beta.cuda(), EPS, x, mean, rstd)
    ry, _, rr = _fwd64(tail, gamma, beta)
    _close(x[-64:].double().cpu(), ry, max(float(ry.abs().max()), float((tail.double().abs().amax(1) * rr).max())), "bf16")
    assert torch.equal(x[5], beta.to(torch.bfloat16).cuda())


@pytest.mark.parametrize("c", [4, 3])
def test_more_rows_than_one_launch_takes(c):
    """bf16 rows of 2^32 values and more in all, in place: rows around the places where
    2^32 values and half of all end, and the last ones."""
    rows = 2 ** 32 // c + 9
    x = torch.empty(rows * c, dtype=torch.bfloat16, device="cuda").fill_(0.5)
    at = sorted({0, 1, rows // 2 - 1, rows // 2, rows // 2 + 1, rows // 2 + 2, 2 ** 32 // c - 1, 2 ** 32 // c, rows - 2, rows - 1})
    gen = torch.Generator().manual_seed(c)
    vals = torch.randn((len(at), c), generator=gen).bfloat16()
    for i, r in enumerate(at):
        x[r * c:(r + 1) * c] = vals[i].cuda()
    g = torch.rand(c, generator=gen) + 0.5
    b = torch.randn(c, generator=gen)
    mean = torch.full((rows,), 9.0, device="cuda")
    rstd = torch.full((rows,), 9.0, device="cuda")
    B.cf_layernorm_fwd(rows, c, "bf16", x, g.cuda(), b.cuda(), 1e-5, x, mean, rstd, None)
    v = vals.double()
    mu = v.mean(1, keepdim=True)
    rs = 1.0 / torch.sqrt(((v - mu) ** 2).mean(1, keepdim=True) + 1e-5)
    want = (v - mu) * rs * g.double() + b.double()
    got = torch.stack([x[r * c:(r + 1) * c] for r in at]).double().cpu()
    # one rounding to bf16 of values whose fp32 error is far below it
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()
    assert float((mean[at].double().cpu() - mu[:, 0]).abs().max()) <= 1e-6
    # the constant rows between: mean 0.5, y = beta
    flat = torch.cat([mean[at[0] + 2:rows // 2 - 1], mean[rows // 2 + 3:2 ** 32 // c - 1]])
    assert bool((flat == 0.5).all())
    assert torch.equal(x[2 * c:3 * c].cpu(), b.bfloat16())
