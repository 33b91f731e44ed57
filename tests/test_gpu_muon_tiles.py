"""GPU parity of the Newton-Schulz products on each of their tiles (sides of 32 to 256, for
the products of the short side, those of the long side and the Gram product, whole and in
slices), by matrices of odd sides, against the formulas in float64.  test_muon_plan.py
checks on the host that these sizes take each tile.

Tolerance: that of the other Newton-Schulz tests for the whole matrix, 4 a^5 2^-24 of the
result's norm (1.2e-4); and since one wrong piece of a large matrix is little of its norm,
every element within ten times that share of the elements' root mean square (roundings
spread evenly over the matrix: 1.6e7 of them stay within 6 standard deviations).  bf16
outputs add half a unit in the last of eight bits, 2^-9 of the norm and 2^-8 of an element
to be clear of ties."""
import math

import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

TOL = 4 * B.NS_COEF[0] ** 5 * 2.0 ** -24
SHAPES = [(131, 133), (133, 131), (145, 2051), (2051, 145), (165, 2657), (165, 6641), (6641, 165), (165, 16601), (16601, 165),
          (49801, 165), (165, 49801), (351, 2807), (719, 723), (871, 2171), (1427, 1423), (1941, 1943), (2829, 2831), (2905, 2903),
          (3979, 3975), (4895, 4901)]


def matrix(r, c, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + r * 31 + c)
    lead = torch.randn((r, 8), generator=g, device="cuda") * (4.0 / torch.arange(1, 9, device="cuda"))
    noise = torch.randn((r, c), generator=g, device="cuda")
    return 1e-3 * (lead @ torch.randn((8, c), generator=g, device="cuda") / math.sqrt(8) + noise)


def ns64(x):
    """Five steps in float64, with the polynomials of the shorter side's Gram matrix."""
    a, b, c = B.NS_COEF
    x = x.double()
    x = x / (x.norm() + 1e-7)
    wide = x.shape[0] <= x.shape[1]
    h = x @ x.t().contiguous() if wide else x.t().contiguous() @ x
    p = None
    for _ in range(5):
        q = b * h + c * (h @ h)
        q.diagonal().add_(a)
        p = q if p is None else q @ p
        h = q @ h @ q
    return p @ x if wide else x @ p


def close(got, want, share, part=0.0):
    """share: of the norm and, tenfold, of the root mean square; part: of each element."""
    err = got.double() - want
    assert not torch.isnan(err).any()
    norm = float(want.norm())
    assert float(err.norm()) <= (share + part / 2) * norm, float(err.norm()) / norm
    rms = norm / math.sqrt(want.numel())
    assert bool((err.abs() <= 10 * share * rms + part * want.abs()).all()), float(err.abs().max()) / rms


def workspace(n, fill):
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(fill)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("r,c", SHAPES)
def test_orthogonalised(r, c, dt):
    x = matrix(r, c).to(torch.bfloat16 if dt == "bf16" else torch.float32)
    mats = B.make_matrices([0], [r], [c])
    n = B.cf_newton_schulz_workspace_size(mats, dt)
    out = []
    for fill in (0xff, 0x3c):  # NaN patterns, ordinary numbers
        o = torch.full_like(x, float("nan"))
        B.cf_newton_schulz(mats, dt, B.make_ns_hparams(), x, o, workspace(n, fill))
        out.append(o)
    assert torch.equal(out[0], out[1])
    close(out[0], ns64(x), TOL, 2.0 ** -8 if dt == "bf16" else 0.0)


@pytest.mark.parametrize("r,c", SHAPES)
def test_updated(r, c):
    """The momentum update with a bf16 copy."""
    eta, mu, decay = 0.02, 0.9, 0.1
    g, m, v = matrix(r, c, 1), 0.3 * matrix(r, c, 2), matrix(r, c, 3)
    mats = B.make_matrices([0], [r], [c])
    hp = B.make_muon_hparams(100, eta0=eta, eta_min=0.001, mu=mu, weight_decay=decay)
    want_m = mu * m.double() + (1 - mu) * g.double()
    gain = math.sqrt(max(1.0, c / r))
    want_v = v.double() - eta * (gain * ns64((1 - mu) * g.double() + mu * want_m) + decay * v.double())
    v16 = torch.empty((r, c), dtype=torch.bfloat16, device="cuda")
    v0 = v.clone()
    B.cf_muon_step(mats, 0, hp, v, g, m, v16, workspace(B.cf_muon_workspace_size(mats), 0xff))
    assert float((m.double() - want_m).abs().max()) <= 2.0 ** -22 * float((m.abs() + g.abs()).max())
    # v's own size beside the step's: two roundings of 2^-24
    step, want_step = v.double() - v0.double(), want_v - v0.double()
    err, norm = step - want_step, float(want_step.norm())
    size = float(v.abs().max())
    assert float(err.norm()) <= TOL * norm + 2.0 ** -23 * float(v.double().norm())
    assert bool((err.abs() <= 10 * TOL * norm / math.sqrt(r * c) + 2.0 ** -23 * size).all())
    assert torch.equal(v16, v.to(torch.bfloat16))


@pytest.mark.parametrize("r,c", [(300, 500), (1427, 1423)])
def test_many_steps_give_orthonormal_rows(r, c):
    """With 2 x - 1.5 x^3 + 0.5 x^5 singular values go to 1, where the derivative is zero: only
    the last products' roundings are left.  Singular values from 0.3 to 1 (in units of the norm,
    from 0.3 / sqrt(m)) need 16 steps at most."""
    m = min(r, c)
    gen = torch.Generator().manual_seed(r)
    u, v = (torch.linalg.qr(torch.randn((k, m), generator=gen, dtype=torch.float64))[0] for k in (r, c))
    x = ((u * torch.linspace(0.3, 1.0, m, dtype=torch.float64)) @ v.t()).float().cuda()
    mats = B.make_matrices([0], [r], [c])
    o = torch.empty_like(x)
    B.cf_newton_schulz(mats, "f32", B.make_ns_hparams(16, (2.0, -1.5, 0.5)), x, o,
                       workspace(B.cf_newton_schulz_workspace_size(mats, "f32"), 0xff))
    o = o.double()
    h = o @ o.t().contiguous() if r <= c else o.t().contiguous() @ o
    assert float((h - torch.eye(m, dtype=torch.float64, device="cuda")).abs().max()) <= 1e-5


def test_largest_short_side():
    """Offsets of a 16384 x 16384 matrix's products, 2^28 values of 4 bytes each."""
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB of device memory")
    m = 16384
    x = matrix(m, m, 5)
    mats = B.make_matrices([0], [m], [m])
    o = torch.empty_like(x)
    B.cf_newton_schulz(mats, "f32", B.make_ns_hparams(), x, o, workspace(B.cf_newton_schulz_workspace_size(mats, "f32"), 0xff))
    close(o, ns64(x), TOL)
