"""Layer normalisation of many rows: workgroups that go round their rows several times,
tensors that pass the last-level cache by, the longest rows of a workgroup, blocks of many
long rows.  Against the formulas in float64 on the GPU, with guard bands around the outputs.

Tolerances: those of the other normalisation tests, 1e-5 of the largest value an output
could have without cancellation, and for bf16 half a unit in the last of eight bits (2^-8 of
a value, to be clear of ties)."""
import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

TOL = 1e-5
EPS = 1e-5
GUARD = 64


def _t(dt):
    return torch.bfloat16 if dt == "bf16" else torch.float32


def data(rows, c, dt):
    g = torch.Generator(device="cuda").manual_seed(rows * 31 + c)
    x = torch.randn((rows, c), generator=g, device="cuda")
    x *= 0.5 + torch.rand((rows, 1), generator=g, device="cuda")
    x += torch.randn((rows, 1), generator=g, device="cuda")
    dy = torch.randn((rows, c), generator=g, device="cuda")
    gamma, beta = (torch.randn(c, generator=g, device="cuda") * 0.3 for _ in range(2))
    return x.to(_t(dt)), dy.to(_t(dt)), 1 + gamma, beta


class Out:
    """A NaN-filled output (or a copy of `like`) between two guard bands."""

    def __init__(self, shape, dtype, like=None):
        n = 1
        for s in shape:
            n *= s
        self.buf = torch.full((n + 2 * GUARD,), 7.0, dtype=dtype, device="cuda")
        self.t = self.buf[GUARD:GUARD + n].view(shape)
        if like is None:
            self.t.fill_(float("nan"))
        else:
            self.t.copy_(like)

    def get(self):
        assert bool((self.buf[:GUARD] == 7).all()) and bool((self.buf[-GUARD:] == 7).all()), "written outside the output"
        return self.t


def ws(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda").fill_(0xff)  # NaN patterns


def close(got, want, scale, dt):
    lim = TOL * scale
    err = (got.double() - want).abs()
    assert bool((err <= (lim + 2.0 ** -8 * want.abs() if dt == "bf16" else lim)).all()), float(err.max())


def statistics(x):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    return mean, ((x - mean).square().mean(1, keepdim=True) + EPS).rsqrt()


def check_forward(rows, c, dt, in_place=False):
    x, _, gamma, beta = data(rows, c, dt)
    y = Out((rows, c), x.dtype, x if in_place else None)
    mean, rstd = Out((rows,), torch.float32), Out((rows,), torch.float32)
    B.cf_layernorm_fwd(rows, c, dt, y.t if in_place else x, gamma, beta, EPS, y.t, mean.t, rstd.t,
                       ws(B.cf_layernorm_fwd_workspace_size(rows, c, dt)))
    m, r = statistics(x)
    close(mean.get(), m[:, 0], float(x.abs().max()), "f32")
    close(rstd.get(), r[:, 0], float(r.max()), "f32")
    want = (x.double() - m) * r * gamma.double() + beta.double()
    close(y.get(), want, max(float(want.abs().max()), float((x.double().abs().amax(1, keepdim=True) * r).max())), dt)


def check_backward(rows, c, dt, in_place=None):
    x, dy, gamma, _ = data(rows, c, dt)
    m, r = (t[:, 0].float() for t in statistics(x))
    dx = Out((rows, c), x.dtype, {None: None, "x": x, "dy": dy}[in_place])
    dg, db = Out((c,), torch.float32), Out((c,), torch.float32)
    B.cf_layernorm_bwd(rows, c, dt, dx.t if in_place == "dy" else dy, dx.t if in_place == "x" else x, gamma, m, r, dx.t, dg.t,
                       db.t, ws(B.cf_layernorm_bwd_workspace_size(rows, c, dt)))
    r64, d = r.double()[:, None], dy.double()
    xh = (x.double() - m.double()[:, None]) * r64
    close(dg.get(), (d * xh).sum(0), float((d * xh).abs().sum(0).max()), "f32")
    close(db.get(), d.sum(0), float(d.abs().sum(0).max()), "f32")
    d *= gamma.double()
    want = r64 * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
    close(dx.get(), want, float((r64 * d.abs().amax(1, keepdim=True)).max()), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(1500011, 2), (1000003, 3), (400003, 5), (400000, 16), (300007, 21), (100001, 40), (60013, 90),
                                    (40009, 100), (20011, 190), (20001, 370), (10007, 700), (10001, 1000), (5003, 1537), (5001, 2900),
                                    (3001, 4096), (3003, 8100), (1201, 12301)])
def test_backward_goes_round_its_rows(rows, c, dt):
    check_backward(rows, c, dt)


# more than 256 MiB in all, rows a multiple of a vector: teams, workgroups
@pytest.mark.parametrize("dt,rows,c", [("f32", 2000003, 16), ("bf16", 3000001, 24), ("f32", 40007, 960), ("bf16", 40007, 1888),
                                       ("f32", 8003, 4100), ("bf16", 5003, 13000)])
def test_past_the_cache(dt, rows, c):
    check_forward(rows, c, dt)
    check_forward(rows, c, dt, in_place=True)
    for in_place in (None, "x", "dy"):
        check_backward(rows, c, dt, in_place)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(300, 20000), (300, 20003), (257, 30001), (300, 40000), (300, 65535), (300, 65536)])
def test_forward_of_the_longest_rows_of_a_workgroup(rows, c, dt):
    check_forward(rows, c, dt)


# rows in chunks of one and of many pieces, and blocks of 16 and of many rows
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(1500, 70000), (1501, 70003), (3000, 20000), (3001, 20001), (17, 300001)])
def test_many_long_rows(rows, c, dt):
    check_forward(rows, c, dt)
    check_backward(rows, c, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_many_long_rows_in_place(dt):
    check_forward(1500, 70003, dt, in_place=True)
    for in_place in ("x", "dy"):
        check_backward(3000, 20001, dt, in_place)
