"""SiLU and GELU, and their slopes, over the whole range of pre-activations through every
kernel that computes them: all bf16 values, and fp32 values past the ends of e^u's range,
where an exponential overflows or vanishes and the activations do not.

The pre-activations are given exactly: products of zeros with the values as bias, data
gradients of 1 with the values as z, normalisations of zeros (backward: with a dy of one
1 a channel) with the values as beta.  So what is left is what the header allows, 2^-21 |u|
of the activations and 2^-20 of the slopes, and the output's rounding, half a step of its
type."""
import math

import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
# half the distance of subnormal values, 2^-126 2^-23 and 2^-126 2^-7: there a rounding is off by
# as much whatever the value (bf16 values of 2^-133 to 2^-126 halved by GELU)
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134}
ACTS = ["silu", "gelu"]


def _t(dt):
    return torch.bfloat16 if dt == "bf16" else torch.float32


def _ws(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda").fill_(0xff)  # NaN patterns


def _dense(n):
    """fp32 values from -130 to 130."""
    return torch.linspace(-130, 130, n, dtype=torch.float64, device="cuda").float()


def _patterns():
    """All bf16 values, as fp32."""
    return torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16).float()


def _sweeps(n):
    """Rows of n values: one of the dense range, and where n is 65536 one of all bf16 values."""
    return [_dense(n)] + ([_patterns()] if n == 65536 else [])


def _curve(u, act):
    """(act(u), act'(u)) in float64 for finite u."""
    if act == "silu":
        s, r = torch.sigmoid(u), torch.sigmoid(-u)
        return u * s, s * (1 + u * r)
    q = 0.5 * torch.erfc(-u / math.sqrt(2))
    return u * q, q + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)


def _check(got, ref, lim, dt, fin):
    """got within lim and its rounding of ref where u is finite, and finite there."""
    got, ref, lim = got.double()[fin], ref[fin], lim[fin]
    assert bool(torch.isfinite(got).all()), f"{int((~torch.isfinite(got)).sum())} values are not finite"
    err, lim = (got - ref).abs(), lim + STEP[dt] * ref.abs() + TINY[dt]
    assert bool((err <= lim).all()), float((err - lim).max())


def _check_acts(y, u, act, dt):
    u = u.double().expand(y.shape)
    assert bool(torch.isnan(y[torch.isnan(u)]).all())
    _check(y, _curve(u, act)[0], 2.0 ** -21 * u.abs(), dt, torch.isfinite(u))


def _check_slopes(d, u, act, dt):
    u = u.double().expand(d.shape)
    assert bool(torch.isnan(d[torch.isnan(u)]).all())
    _check(d, _curve(u, act)[1], torch.full_like(u, 2.0 ** -20), dt, torch.isfinite(u))


# Tiles of 64 (3 rows) and 128 (300 rows in bf16, 200 in fp32), sums cut into slices with rows of
# whole pieces and ragged ones, and rows past the tiles' offsets.
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt,m,k,n", [("f32", 3, 16, 65536), ("bf16", 3, 16, 65536), ("f32", 200, 64, 65536),
                                      ("bf16", 300, 64, 65536), ("f32", 64, 4096, 512), ("bf16", 64, 4096, 512),
                                      ("f32", 64, 4096, 509), ("bf16", 64, 4096, 509), ("f32", 1, 1, (1 << 22) + 3),
                                      ("bf16", 1, 1, (1 << 22) + 3)])
def test_products_forward(dt, m, k, n, act):
    x, w = torch.zeros((m, k), dtype=_t(dt), device="cuda"), torch.zeros((k, n), dtype=_t(dt), device="cuda")
    ws = _ws(B.cf_linear_fwd_workspace_size(m, k, n, dt))
    for u in _sweeps(n):
        y = torch.full((m, n), math.nan, dtype=_t(dt), device="cuda")
        B.cf_linear_fwd(m, k, n, dt, x, w, u, act, 0.0, None, y, None, ws)
        _check_acts(y, u[None], act, dt)


# The same (rows, terms, columns) of data gradients; rows of 2^22 terms are past the tiles' offsets.
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt,m,n,k", [("f32", 3, 16, 65536), ("bf16", 3, 16, 65536), ("f32", 200, 64, 65536),
                                      ("bf16", 300, 64, 65536), ("f32", 64, 4096, 512), ("bf16", 64, 4096, 512),
                                      ("f32", 64, 4096, 509), ("bf16", 64, 4096, 509), ("f32", 24, 1 << 22, 24),
                                      ("bf16", 24, 1 << 22, 24)])
def test_products_data_gradient(dt, m, n, k, act):
    dz, w = torch.zeros((m, n), dtype=_t(dt), device="cuda"), torch.zeros((k, n), dtype=_t(dt), device="cuda")
    dz[:, 0] = 1
    w[:, 0] = 1
    ws = _ws(B.cf_linear_bwd_data_workspace_size(m, k, n, dt))
    for u in [s[None].expand(m, k) for s in _sweeps(k)] if k == 65536 else [_dense(m * k).view(m, k)]:
        z = u.to(_t(dt)).contiguous()
        dx = torch.full((m, k), math.nan, dtype=_t(dt), device="cuda")
        B.cf_linear_bwd_data(m, k, n, dt, dz, w, None, z, act, 0.0, dx, ws)
        _check_slopes(dx, z, act, dt)


# Groups of one workgroup of 256 threads and of 1024; slices whose rows the second pass joins, and
# so many groups that a launch of its own does; voxels of more values than a workgroup's turn.
NORMS = [(4, 65536, 1024), (200, 65536, 1024), (100, 1024, 8), (3000, 1024, 1024), (3, 65536, 8)]


def _betas(c):
    return _sweeps(c) if c == 65536 else list(_dense(16 * c).view(16, c))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vox,c,groups", NORMS)
def test_normalisation_forward(vox, c, groups, dt, act):
    x, gamma = torch.zeros((1, vox, c), dtype=_t(dt), device="cuda"), torch.ones(c, device="cuda")
    mean, rstd = torch.empty(groups, device="cuda"), torch.empty(groups, device="cuda")
    ws = _ws(B.cf_groupnorm_fwd_workspace_size(1, vox, c, groups, dt))
    for u in _betas(c):
        y = torch.full_like(x, math.nan)
        B.cf_groupnorm_fwd(1, vox, c, groups, dt, x, gamma, u.contiguous(), EPS, act, 0.0, y, mean, rstd, ws)
        _check_acts(y, u, act, dt)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vox,c,groups", NORMS)
def test_normalisation_backward(vox, c, groups, dt, act):
    x, gamma = torch.zeros((1, vox, c), dtype=_t(dt), device="cuda"), torch.ones(c, device="cuda")
    dy = torch.zeros_like(x)
    dy[0, vox // 2] = 1
    mean, rstd = torch.zeros(groups, device="cuda"), torch.ones(groups, device="cuda")
    ws = _ws(B.cf_groupnorm_bwd_workspace_size(1, vox, c, groups, dt))
    for u in _betas(c):
        u = torch.where(torch.isfinite(u), u, 0.0).contiguous()
        dx = torch.full_like(x, math.nan)
        dgamma, dbeta = torch.full((c,), math.nan, device="cuda"), torch.full((c,), math.nan, device="cuda")
        B.cf_groupnorm_bwd(1, vox, c, groups, dt, dy, x, gamma, u, mean, rstd, act, 0.0, dx, dgamma, dbeta, ws)
        # a sum of one term and zeros
        _check_slopes(dbeta, u, act, "f32")
        assert not dgamma.any()
        # dx = du - its group's mean: the slope's error, and twice an fp32 sum's, c / groups + 8
        # steps of 2^-24 of at most 1.13
        s = _curve(u.double(), act)[1]
        du = s * dy.double()
        ref = du - (s.view(groups, -1).sum(1) / (vox * (c // groups))).repeat_interleave(c // groups)
        lim = torch.full_like(ref, 2.0 ** -19 + (c // groups + 8) * 2.0 ** -23)
        _check(dx, ref, lim, dt, torch.ones_like(ref, dtype=torch.bool))
