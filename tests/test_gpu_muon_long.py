"""GPU parity of the Newton-Schulz products of matrices whose long side has so many
columns that a row of a tile is more than 2^32 bytes from the tile's first.

Tolerance: that of the other Newton-Schulz tests, 4 a^steps 2^-24 of the result's norm for
five steps, and half a unit in the last of a bf16 output's eight bits."""
import pytest
import torch

from paper_1808_04728_amd import binding as B

pytestmark = pytest.mark.gpu

BLOCK = 1 << 16  # columns at a time


def tol(dt):
    return 4 * B.NS_COEF[0] ** 5 * 2.0 ** -24 + (2.0 ** -9 if dt == "bf16" else 0.0)


def orthogonal64(h, norm, steps=5):
    """The m x m factor P with O = P G from G's Gram matrix, in float64."""
    a, b, c = B.NS_COEF
    norm = norm + 1e-7
    h = h / (norm * norm)
    eye = torch.eye(h.shape[0], dtype=torch.float64, device=h.device)
    p = eye / norm
    for _ in range(steps):
        q = a * eye + b * h + c * (h @ h)
        p, h = q @ p, q @ h @ q
    return p


def test_rows_past_32_bits():
    """Rows of eight common signals of falling strength and noise of their own (rows that
    are noise alone would have about the same Gram matrix whichever of them are read)."""
    m, n = 256, 8_600_011
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 64 GB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(11)
    mix = torch.randn((m, 8), generator=gen, device="cuda") * (4.0 / torch.arange(1, 9, device="cuda"))
    g = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    h = torch.zeros((m, m), dtype=torch.float64, device="cuda")
    for j in range(0, n, BLOCK):
        k = min(BLOCK, n - j)
        x = mix @ torch.randn((8, k), generator=gen, device="cuda") + torch.randn((m, k), generator=gen, device="cuda")
        g[:, j:j + k] = x.to(torch.bfloat16)
        y = g[:, j:j + k].double()
        h += y @ y.t().contiguous()
    mats = B.make_matrices([0], [m], [n])
    ws = torch.empty(B.cf_newton_schulz_workspace_size(mats, "bf16"), dtype=torch.uint8, device="cuda")
    o = torch.empty_like(g)
    B.cf_newton_schulz(mats, "bf16", B.make_ns_hparams(), g, o, ws)
    p = orthogonal64(h, h.diagonal().sum().sqrt())
    err = ref = 0.0
    for j in range(0, n, BLOCK):
        want = p @ g[:, j:j + BLOCK].double()
        err += float((o[:, j:j + BLOCK].double() - want).square().sum())
        ref += float(want.square().sum())
    assert err ** 0.5 <= tol("bf16") * ref ** 0.5, (err ** 0.5, ref ** 0.5)


# the skinny kernels, and tiles of 64 that reach just below 2^32 bytes, with the longest side
@pytest.mark.parametrize("r,c,dt", [(100, 1 << 24, "f32"), ((1 << 24) - 3, 100, "bf16"), (200, 1 << 24, "f32"),
                                    ((1 << 24) - 5, 131, "bf16")])
def test_longest_side(r, c, dt):
    m, n = min(r, c), max(r, c)
    mats = B.make_matrices([0], [r], [c])
    need = B.cf_newton_schulz_workspace_size(mats, dt)
    if torch.cuda.mem_get_info()[0] < need + 16 * m * n + (8 << 30):
        pytest.skip("needs about 80 GB of device memory")
    gen = torch.Generator(device="cuda").manual_seed(m)
    mix = torch.randn((m, 8), generator=gen, device="cuda") * (4.0 / torch.arange(1, 9, device="cuda"))
    g = torch.empty((r, c), dtype=torch.bfloat16 if dt == "bf16" else torch.float32, device="cuda")

    def part(t, j):  # columns of the long side, from the short side's rows
        return t[:, j:j + BLOCK] if r < c else t[j:j + BLOCK].t()

    h = torch.zeros((m, m), dtype=torch.float64, device="cuda")
    for j in range(0, n, BLOCK):
        k = min(BLOCK, n - j)
        part(g, j).copy_(mix @ torch.randn((8, k), generator=gen, device="cuda") + torch.randn((m, k), generator=gen, device="cuda"))
        y = part(g, j).double()
        h += y @ y.t().contiguous()
    o = torch.empty_like(g)
    B.cf_newton_schulz(mats, dt, B.make_ns_hparams(), g, o, torch.empty(need, dtype=torch.uint8, device="cuda"))
    p = orthogonal64(h, h.diagonal().sum().sqrt())
    err = ref = 0.0
    for j in range(0, n, BLOCK):
        want = p @ part(g, j).double().contiguous()
        e = (part(o, j).double() - want).square().sum()
        # no block is wrong that the whole would hide
        assert float(e) <= 4 * tol(dt) ** 2 * float(want.square().sum()), j
        err += float(e)
        ref += float(want.square().sum())
    assert err ** 0.5 <= tol(dt) * ref ** 0.5, (err ** 0.5, ref ** 0.5)
