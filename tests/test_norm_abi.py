"""Host-side refusals of the layer normalisation entry points (no kernel is launched)."""
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


def fwd(rows=64, c=48, dtype="f32", x=A, gamma=A + M, beta=A + 2 * M, eps=1e-5, y=A + 3 * M, mean=A + 4 * M, rstd=A + 5 * M,
        ws=None, ws_bytes=0):
    B.cf_layernorm_fwd(rows, c, dtype, x, gamma, beta, eps, y, mean, rstd, ws, ws_bytes, 0)


def bwd(rows=64, c=48, dtype="f32", dy=A, x=A + M, gamma=A + 2 * M, mean=A + 3 * M, rstd=A + 4 * M, dx=A + 5 * M,
        dgamma=A + 6 * M, dbeta=A + 7 * M, ws=A + 8 * M, ws_bytes=M):
    B.cf_layernorm_bwd(rows, c, dtype, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, ws_bytes, 0)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_sizes(call):
    expect(B.CF_ERR_INVALID_ARG, lambda: call(rows=-1))
    expect(B.CF_ERR_INVALID_ARG, lambda: call(c=0))
    expect(B.CF_ERR_INVALID_ARG, lambda: call(c=-3))
    expect(B.CF_ERR_UNSUPPORTED, lambda: call(c=(1 << 30) + 1))
    expect(B.CF_ERR_UNSUPPORTED, lambda: call(rows=1 << 36, c=16))
    expect(B.CF_ERR_INVALID_ARG, lambda: B._check(B.lib().cf_layernorm_fwd(1, 1, 7, A, A, A, 0.0, A, A, A, None, 0, None)))
    with pytest.raises(ValueError):
        call(dtype="f64")


@pytest.mark.parametrize("eps", [-1e-6, math.nan, math.inf])
def test_eps(eps):
    expect(B.CF_ERR_INVALID_ARG, lambda: fwd(eps=eps))


@pytest.mark.parametrize("name", ["x", "gamma", "beta", "y", "mean", "rstd"])
def test_forward_pointers(name):
    expect(B.CF_ERR_INVALID_ARG, lambda: fwd(**{name: None}))
    expect(B.CF_ERR_ALIGNMENT, lambda: fwd(**{name: A + 40 * M + 4}))


@pytest.mark.parametrize("name", ["dy", "x", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta"])
def test_backward_pointers(name):
    expect(B.CF_ERR_INVALID_ARG, lambda: bwd(**{name: None}))
    expect(B.CF_ERR_ALIGNMENT, lambda: bwd(**{name: A + 40 * M + 8}))


def test_workspace():
    assert B.cf_layernorm_fwd_workspace_size(64, 48, "f32") == 0
    need = B.cf_layernorm_fwd_workspace_size(3, 1 << 20, "f32")
    assert need > 0
    big = 1 << 33
    wide = dict(rows=3, c=1 << 20, x=big, gamma=2 * big, beta=3 * big, y=4 * big, mean=5 * big, rstd=6 * big)
    expect(B.CF_ERR_WORKSPACE, lambda: fwd(**wide, ws=None, ws_bytes=need))
    expect(B.CF_ERR_WORKSPACE, lambda: fwd(**wide, ws=7 * big, ws_bytes=need - 1))
    expect(B.CF_ERR_ALIGNMENT, lambda: fwd(**wide, ws=7 * big + 4, ws_bytes=need))
    expect(B.CF_ERR_ALIAS, lambda: fwd(**wide, ws=big, ws_bytes=need))
    need = B.cf_layernorm_bwd_workspace_size(64, 48, "f32")
    expect(B.CF_ERR_WORKSPACE, lambda: bwd(ws=None))
    expect(B.CF_ERR_WORKSPACE, lambda: bwd(ws_bytes=need - 1))
    expect(B.CF_ERR_ALIGNMENT, lambda: bwd(ws=A + 8 * M + 4))
    expect(B.CF_ERR_ALIAS, lambda: bwd(ws=A))
    for rows, c in ((-1, 4), (4, 0), (4, -1), (0, 4)):
        assert B.cf_layernorm_fwd_workspace_size(rows, c, "f32") == 0
        assert B.cf_layernorm_bwd_workspace_size(rows, c, "bf16") == 0


def test_aliasing():
    """y may be x, dx may be dy or x, exactly; any other overlap is refused."""
    expect(B.CF_ERR_ALIAS, lambda: fwd(y=A + 16))
    expect(B.CF_ERR_ALIAS, lambda: fwd(mean=A))
    expect(B.CF_ERR_ALIAS, lambda: fwd(y=A + M))
    expect(B.CF_ERR_ALIAS, lambda: fwd(rstd=A + 4 * M))
    expect(B.CF_ERR_ALIAS, lambda: bwd(dx=A + 16))
    expect(B.CF_ERR_ALIAS, lambda: bwd(dx=A + M - 16))
    expect(B.CF_ERR_ALIAS, lambda: bwd(dx=A + 2 * M))
    expect(B.CF_ERR_ALIAS, lambda: bwd(dgamma=A + 2 * M))
    expect(B.CF_ERR_ALIAS, lambda: bwd(dbeta=A + 6 * M))


def test_no_rows_is_a_no_op():
    fwd(rows=0, x=None, y=None, gamma=None, beta=None, mean=None, rstd=None)
    assert B.cf_last_error() == ""
    expect(B.CF_ERR_INVALID_ARG, lambda: bwd(rows=0, dgamma=None))
    expect(B.CF_ERR_ALIAS, lambda: bwd(rows=0, dbeta=A + 6 * M))
