"""GPU parity of the Newton-Schulz orthogonalisation and of the momentum update
around it, through the C ABI, against the formulas in float64.

Tolerance.  A rounding of relative size 2^-24 anywhere in the first step is an
absolute error of that size in the singular values' scale, and the polynomial
multiplies small singular values by a = 3.4445 a step: the result's error is held
to 4 a^steps 2^-24 of its Frobenius norm (1.2e-4 for five steps), for a
handful of such roundings.  bf16 outputs add half a unit in the last of eight
bits, 2^-9."""
import math

import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

GUARD = 64
SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (3, 64), (64, 3), (16, 27), (27, 16), (31, 33), (32, 32), (65, 64), (64, 65), (96, 97),
          (100, 300), (300, 100), (128, 128), (127, 2000), (129, 257), (1024, 32), (2000, 5), (5, 2000), (200, 192), (257, 255),
          (512, 512), (513, 700), (8192, 128), (128, 4097), (20000, 64), (1000, 999), (1, 70000), (70001, 2)]


def tol(steps, dt="f32", coef=B.NS_COEF):
    return 4 * max(1.0, abs(coef[0])) ** steps * 2.0 ** -24 + (2.0 ** -9 if dt == "bf16" else 0.0)


def _t(dt):
    return torch.bfloat16 if dt == "bf16" else torch.float32


def ns64(x, steps=5, coef=B.NS_COEF, eps=1e-7):
    a, b, c = coef
    x = x.double()
    x = x / (x.norm() + eps)
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            h = x @ x.t()
            x = a * x + (b * h + c * (h @ h)) @ x
        else:
            h = x.t() @ x
            x = a * x + x @ (b * h + c * (h @ h))
    return x


def matrix(r, c, kind="signal", seed=0):
    g = torch.Generator().manual_seed(seed * 7919 + r * 31 + c)
    noise = torch.randn((r, c), generator=g)
    if kind == "noise":
        return noise
    if kind == "rank1":
        return torch.randn((r, 1), generator=g) @ torch.randn((1, c), generator=g)
    k = min(8, r, c)
    lead = torch.randn((r, k), generator=g) * (4.0 / torch.arange(1, k + 1)) @ torch.randn((k, c), generator=g)
    return 1e-3 * (lead / math.sqrt(k) + noise)


def run_ns(ms, dt="f32", steps=5, coef=B.NS_COEF, eps=1e-7, stream=None, in_place=False, gap=0):
    """The matrices of ms in flat arrays with gaps; checks that the gaps stay."""
    off, at = [], GUARD
    for x in ms:
        off.append(at)
        at = (at + x.numel() + 7) // 8 * 8 + gap
    flat = torch.full((at + GUARD,), 7.0, dtype=_t(dt))
    inside = torch.zeros(at + GUARD, dtype=torch.bool)
    for o, x in zip(off, ms):
        flat[o:o + x.numel()] = x.reshape(-1).to(_t(dt))
        inside[o:o + x.numel()] = True
    g = flat.cuda()
    out = g if in_place else torch.full_like(g, 9.0)
    mats = B.make_matrices(off, [x.shape[0] for x in ms], [x.shape[1] for x in ms])
    ws = torch.empty(max(16, B.cf_newton_schulz_workspace_size(mats, dt)), dtype=torch.uint8, device="cuda").fill_(0xff)
    B.cf_newton_schulz(mats, dt, B.make_ns_hparams(steps, coef, eps), g, out, ws, stream=stream)
    res = out.cpu()
    assert (res[~inside] == (7.0 if in_place else 9.0)).all(), "written outside the matrices"
    bits = torch.int16 if dt == "bf16" else torch.int32  # (an input may hold NaN)
    assert in_place or torch.equal(g.cpu().view(bits), flat.view(bits))
    return [res[o:o + x.numel()].view(x.shape) for o, x in zip(off, ms)]


def check(got, x, dt="f32", steps=5, coef=B.NS_COEF, eps=1e-7):
    ref = ns64(x.to(_t(dt)), steps, coef, eps)
    err = float((got.double() - ref).norm())
    assert err <= tol(steps, dt, coef) * float(ref.norm()), (err, float(ref.norm()))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("r,c", SHAPES)
def test_shapes(r, c, dt):
    x = matrix(r, c)
    check(run_ns([x], dt)[0], x, dt)


@pytest.mark.parametrize("r,c", [(20000, 256), (200, 30011), (400, 12000), (9000, 900)])
def test_gram_products_in_slices(r, c):
    """Long sides whose Gram products are cut and summed, alone and beside a matrix of
    few slices."""
    x, y = matrix(r, c, "noise"), matrix(160, 700, "noise")
    one = run_ns([x])[0]
    check(one, x)
    both = run_ns([x, y])
    assert torch.equal(both[0], one)
    assert torch.equal(both[1], run_ns([y])[0])
    check(both[1], y)


@pytest.mark.parametrize("kind", ["noise", "rank1"])
@pytest.mark.parametrize("r,c", [(16, 27), (60, 200), (300, 128), (128, 128), (260, 400)])
def test_spectra(r, c, kind):
    x = matrix(r, c, kind)
    check(run_ns([x])[0], x)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7, 10])
@pytest.mark.parametrize("r,c", [(40, 24), (130, 300)])
def test_steps(r, c, steps):
    x = matrix(r, c)
    check(run_ns([x], steps=steps)[0], x, steps=steps)


@pytest.mark.parametrize("coef", [(1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (3.0, -16.0 / 5, 6.0 / 5)])
def test_coefficients(coef):
    """Other polynomials; with many steps the rows become orthonormal."""
    x = matrix(48, 200, "noise")
    check(run_ns([x], coef=coef)[0], x, coef=coef)
    if coef == (2.0, -1.5, 0.5):
        o = run_ns([x], coef=coef, steps=16)[0].double()
        assert float((o @ o.t() - torch.eye(48, dtype=torch.float64)).abs().max()) <= 1e-5


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e6, 1e30])
@pytest.mark.parametrize("r,c", [(24, 40), (300, 200)])
def test_scale_of_the_input(r, c, scale):
    x = matrix(r, c, "noise") * scale
    check(run_ns([x], eps=0.0)[0], x, eps=0.0)


@pytest.mark.parametrize("r,c", [(16, 27), (140, 130)])
def test_zero_infinite_and_nan_matrices_stay_apart(r, c):
    good = matrix(r, c)
    zero, inf, nan = torch.zeros(r, c), matrix(r, c, seed=1), matrix(r, c, seed=2)
    inf[r // 2, c // 2] = float("-inf")
    nan[0, 0] = float("nan")
    out = run_ns([zero, inf, good, nan, good])
    assert (out[0] == 0).all()
    assert torch.isnan(out[1]).all() and torch.isnan(out[3]).all()
    check(out[2], good)
    assert torch.equal(out[2], out[4])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_many_matrices(dt):
    """More matrices than one set of launches takes, of all sizes, some empty."""
    shapes = [(27, 16), (1024, 32), (0, 5), (2048, 64), (1, 1), (130, 140), (64, 3), (128, 64), (5, 0), (300, 20)] * 4
    ms = [matrix(r, c, seed=i) if r * c else torch.zeros(r, c) for i, (r, c) in enumerate(shapes)]
    for x, got in zip(ms, run_ns(ms, dt, gap=24)):
        if x.numel():
            check(got, x, dt)
            assert torch.equal(got, run_ns([x], dt)[0])  # alone or with others: the same bits


@pytest.mark.parametrize("r,c", [(27, 16), (4096, 64), (300, 500)])
def test_transpose_in_place_repeat_and_side_stream(r, c):
    x = matrix(r, c)
    one = run_ns([x])[0]
    assert torch.equal(one, run_ns([x], in_place=True)[0])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        assert torch.equal(one, run_ns([x])[0])
    t = run_ns([x.t().contiguous()])[0]
    assert float((t.t().double() - one.double()).norm()) <= tol(5) * float(one.double().norm())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("nesterov,scale,decay", [(True, B.CF_MUON_SCALE_SHAPE, 0.0), (False, B.CF_MUON_SCALE_RMS, 0.1)])
def test_muon_steps(nesterov, scale, decay, bf16):
    """Three updates of a small network against float64, each from the device's own state."""
    shapes = [(27, 16), (1024, 32), (512, 128), (64, 3), (3, 64), (200, 260), (1, 40)]
    off, at = [], 16
    for r, c in shapes:
        off.append(at)
        at = (at + r * c + 15) // 16 * 16
    n = at + GUARD
    g = torch.Generator().manual_seed(3)
    v, m = torch.randn(n, generator=g).cuda(), torch.zeros(n, device="cuda")
    v16 = torch.full((n,), 5.0, dtype=torch.bfloat16, device="cuda") if bf16 else None
    mats = B.make_matrices(off, [r for r, _ in shapes], [c for _, c in shapes])
    hp = B.make_muon_hparams(100, eta0=0.02, eta_min=0.001, mu=0.9, weight_decay=decay, nesterov=nesterov, scale=scale)
    ws = torch.empty(B.cf_muon_workspace_size(mats), dtype=torch.uint8, device="cuda").fill_(0xff)
    for t in (0, 1, 250):
        gr = torch.randn(n, generator=g)
        for o, (r, c) in zip(off, shapes):
            gr[o:o + r * c] = matrix(r, c, seed=t).reshape(-1)
        v0, m0 = v.cpu(), m.cpu()
        gd = gr.cuda()
        B.cf_muon_step(mats, t, hp, v, gd, m, v16, ws)
        v1, m1 = v.cpu(), m.cpu()
        assert torch.equal(gd.cpu(), gr)
        eta = 0.019 * (1 - min(t, 100) / 100) + 0.001
        out = torch.ones(n, dtype=torch.bool)
        for o, (r, c) in zip(off, shapes):
            s = slice(o, o + r * c)
            out[s] = False
            gd64, md, vd = gr[s].double(), m0[s].double(), v0[s].double()
            mn = 0.9 * md + 0.1 * gd64
            assert float((m1[s].double() - mn).abs().max()) <= 2.0 ** -22 * float((md.abs() + gd64.abs()).max())
            u = 0.1 * gd64 + 0.9 * mn if nesterov else mn
            k = math.sqrt(max(1.0, c / r)) if scale == B.CF_MUON_SCALE_SHAPE else 0.2 * math.sqrt(max(r, c))
            o64 = ns64(u.view(r, c)).reshape(-1)
            vn = vd - eta * (k * o64 + decay * vd)
            lim = eta * k * tol(5) * float(o64.norm()) + 2.0 ** -23 * float(vd.norm())
            assert float((v1[s].double() - vn).norm()) <= lim
            if bf16:
                assert torch.equal(v16[s].cpu(), v1[s].to(torch.bfloat16))
        assert torch.equal(v1[out], v0[out]) and torch.equal(m1[out], m0[out])
        if bf16:
            assert (v16.cpu()[out] == 5).all()


def test_graph_replays():
    """Captured steps replay to the eager bits, with eager work in between."""
    shapes = [(27, 16), (256, 128), (150, 300)]
    off = [0, 512, 512 + 256 * 128]
    n = off[-1] + 150 * 300
    mats = B.make_matrices(off, [r for r, _ in shapes], [c for _, c in shapes])
    hp = B.make_muon_hparams(100)
    ws = torch.empty(B.cf_muon_workspace_size(mats), dtype=torch.uint8, device="cuda")
    gen = torch.Generator().manual_seed(9)
    v, gr, m = (torch.randn(n, generator=gen).cuda() for _ in range(3))
    B.cf_muon_step(mats, 5, hp, v, gr, m, None, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cf_muon_step(mats, 5, hp, v, gr, m, None, ws)
    for _ in range(3):
        gr.copy_(torch.randn(n, generator=gen))
        v0, m0 = v.clone(), m.clone()
        B.cf_muon_step(mats, 5, hp, v, gr, m, None, ws)
        want_v, want_m = v.clone(), m.clone()
        v.copy_(v0)
        m.copy_(m0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(v, want_v) and torch.equal(m, want_m)
