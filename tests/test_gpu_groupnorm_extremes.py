"""Group normalisation of groups whose values come near the end of fp32's range, where the
formulas are finite: the same results from every kernel that may take a group.

Tolerances: those of the other normalisation tests, 1e-5 of the largest value an output
could have without cancellation, and for bf16 half a unit in the last of eight bits.  The
groups' sums and the squares of the deviations are powers of two that fp32 holds exactly."""
import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

TOL = 1e-5
EPS = 1e-5

# one workgroup of 256 threads and of 1024; slices that the second pass joins; so many groups that a
# launch of its own joins them; voxels of more values than a workgroup's turn
SHAPES = [(2, 64, 128, 8), (1, 1024, 2048, 128), (1, 1 << 14, 16, 4), (3, 1 << 12, 16, 4), (1, 4096, 1024, 1024), (1, 64, 8192, 8)]


def _t(dt):
    return torch.bfloat16 if dt == "bf16" else torch.float32


def _ws(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda").fill_(0xff)  # NaN patterns


def _affine(c):
    gen = torch.Generator(device="cuda").manual_seed(c)
    return [torch.randn(c, generator=gen, device="cuda") for _ in range(2)]


def _fwd(x, gamma, beta, groups, dt):
    n, vox, c = x.shape
    y, mean, rstd = torch.empty_like(x), torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
    B.cf_groupnorm_fwd(n, vox, c, groups, dt, x, gamma, beta, EPS, "none", 0.0, y, mean, rstd,
                       _ws(B.cf_groupnorm_fwd_workspace_size(n, vox, c, groups, dt)))
    return y.double(), mean.double(), rstd.double()


@pytest.mark.parametrize("n,vox,c,groups", SHAPES)
def test_mean_whose_square_is_infinite(n, vox, c, groups):
    gamma, beta = _affine(c)
    sign = torch.tensor([1.0, 1.0, -1.0, -1.0], device="cuda").repeat(vox // 4)[:, None].expand(vox, c)
    base = torch.tensor([1.0, -1.0], device="cuda").repeat((n + 1) // 2)[:n] * 2.0 ** 67
    y, mean, rstd = _fwd((base[:, None, None] + 2.0 ** 50 * sign).contiguous(), gamma, beta, groups, "f32")
    assert torch.equal(mean, base.double()[:, None].expand(n, groups))
    assert float((rstd * 2.0 ** 50 - 1).abs().max()) <= TOL
    want = sign.double() * gamma.double() + beta.double()
    assert float((y - want).abs().max()) <= TOL * float(want.abs().max())


# (and, in slices, sizes whose last slice and vector are parts of ones)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,vox,c,groups", SHAPES + [(1, 4099, 16, 4), (2, 70001, 12, 3), (1, 9001, 3, 1), (1, 40, 3333, 3), (2, 3001, 520, 520)])
def test_constant_groups_whose_square_is_infinite(n, vox, c, groups, dt):
    gamma, beta = _affine(c)
    y, mean, rstd = _fwd(torch.full((n, vox, c), -2.0 ** 67, dtype=_t(dt), device="cuda"), gamma, beta, groups, dt)
    assert (mean == -2.0 ** 67).all()
    assert float((rstd * EPS ** 0.5 - 1).abs().max()) <= TOL
    assert torch.equal(y, beta.to(_t(dt)).double().expand(n, vox, c))
