"""Host-side refusals of the group normalisation entry points (no kernel is launched)."""
import math
import os

import pytest

from paper_1808_04728_amd import binding as B

A = 0x7F0000000000  # fake, 16-byte aligned device addresses (never dereferenced)
M = 1 << 24

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libcosmoflow_hip.so not built")


def expect(status, fn, *args):
    with pytest.raises(B.CfError) as e:
        fn(*args)
    assert e.value.status == status, str(e.value)
    assert B.cf_last_error() != ""


def fwd(n=2, vox=5000, c=48, groups=6, dtype="f32", x=A, gamma=A + M, beta=A + 2 * M, eps=1e-5, act="silu", alpha=0.01,
        y=A + 3 * M, mean=A + 4 * M, rstd=A + 5 * M, ws=A + 6 * M, ws_bytes=M):
    B.cf_groupnorm_fwd(n, vox, c, groups, dtype, x, gamma, beta, eps, act, alpha, y, mean, rstd, ws, ws_bytes, 0)


def bwd(n=2, vox=5000, c=48, groups=6, dtype="f32", dy=A, x=A + M, gamma=A + 2 * M, beta=A + 3 * M, mean=A + 4 * M,
        rstd=A + 5 * M, act="silu", alpha=0.01, dx=A + 6 * M, dgamma=A + 7 * M, dbeta=A + 8 * M, ws=A + 9 * M, ws_bytes=M):
    B.cf_groupnorm_bwd(n, vox, c, groups, dtype, dy, x, gamma, beta, mean, rstd, act, alpha, dx, dgamma, dbeta, ws, ws_bytes, 0)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_sizes(call):
    for bad in (dict(n=-1), dict(vox=-1), dict(c=0), dict(c=-6), dict(groups=0), dict(groups=-1), dict(groups=5), dict(groups=96)):
        expect(B.CF_ERR_INVALID_ARG, lambda: call(**bad))
    for bad in (dict(vox=1 << 31), dict(n=1 << 20), dict(c=1 << 24, groups=1), dict(n=1 << 10, vox=1 << 26)):
        expect(B.CF_ERR_UNSUPPORTED, lambda: call(**bad))
    for bad in (dict(dtype="f64"), dict(act="tanh"), dict(act=9)):
        with pytest.raises(ValueError):
            call(**bad)
    expect(B.CF_ERR_INVALID_ARG,
           lambda: B._check(B.lib().cf_groupnorm_fwd(1, 1, 1, 1, 0, A, A, A, 0.0, 4, 0.0, A, A, A, None, 0, None)))
    expect(B.CF_ERR_INVALID_ARG,
           lambda: B._check(B.lib().cf_groupnorm_fwd(1, 1, 1, 1, 7, A, A, A, 0.0, 0, 0.0, A, A, A, None, 0, None)))


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("alpha", [math.nan, math.inf])
def test_alpha(call, alpha):
    expect(B.CF_ERR_INVALID_ARG, lambda: call(act="lrelu", alpha=alpha))


@pytest.mark.parametrize("eps", [-1e-6, math.nan, math.inf])
def test_eps(eps):
    expect(B.CF_ERR_INVALID_ARG, lambda: fwd(eps=eps))


@pytest.mark.parametrize("name", ["x", "gamma", "beta", "y", "mean", "rstd"])
def test_forward_pointers(name):
    expect(B.CF_ERR_INVALID_ARG, lambda: fwd(**{name: None}))
    expect(B.CF_ERR_ALIGNMENT, lambda: fwd(**{name: A + 40 * M + 4}))


@pytest.mark.parametrize("name", ["dy", "x", "gamma", "beta", "mean", "rstd", "dx", "dgamma", "dbeta"])
def test_backward_pointers(name):
    expect(B.CF_ERR_INVALID_ARG, lambda: bwd(**{name: None}))
    expect(B.CF_ERR_ALIGNMENT, lambda: bwd(**{name: A + 40 * M + 8}))


def test_overlaps():
    size = 2 * 5000 * 48 * 4
    for bad in (dict(y=A + 16), dict(y=A + size - 16), dict(mean=A), dict(rstd=A + 4 * M), dict(y=A + M), dict(ws=A + 3 * M)):
        expect(B.CF_ERR_ALIAS, lambda: fwd(**bad))
    for bad in (dict(dx=A + 16), dict(dx=A + M + 16), dict(dgamma=A + 8 * M), dict(dbeta=A + 2 * M), dict(dx=A + 4 * M),
                dict(ws=A)):
        expect(B.CF_ERR_ALIAS, lambda: bwd(**bad))
    expect(B.CF_ERR_ALIAS, lambda: bwd(n=0, dgamma=A, dbeta=A))


def test_workspace():
    need = B.cf_groupnorm_fwd_workspace_size(2, 5000, 48, 6, "f32")
    assert need > 0
    expect(B.CF_ERR_WORKSPACE, lambda: fwd(ws=None, ws_bytes=need))
    expect(B.CF_ERR_WORKSPACE, lambda: fwd(ws_bytes=need - 1))
    expect(B.CF_ERR_ALIGNMENT, lambda: fwd(ws=A + 6 * M + 4))
    need = B.cf_groupnorm_bwd_workspace_size(2, 5000, 48, 6, "f32")
    expect(B.CF_ERR_WORKSPACE, lambda: bwd(ws=None))
    expect(B.CF_ERR_WORKSPACE, lambda: bwd(ws_bytes=need - 1))
    expect(B.CF_ERR_ALIGNMENT, lambda: bwd(ws=A + 9 * M + 4))
    for shape in ((-1, 4, 4, 2), (1, -1, 4, 2), (1, 4, 0, 1), (1, 4, 4, 3), (0, 4, 4, 2), (1, 0, 4, 2)):
        assert B.cf_groupnorm_fwd_workspace_size(*shape, "f32") == 0
        assert B.cf_groupnorm_bwd_workspace_size(*shape, "bf16") == 0
