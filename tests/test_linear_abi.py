"""Host-side refusals of the matrix products with an epilogue (no kernel is launched)."""
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


def fwd(m=64, k=48, n=32, dtype="f32", x=A, w=A + M, bias=A + 2 * M, act="silu", alpha=0.01, residual=A + 3 * M, y=A + 4 * M,
        z=A + 5 * M, ws=A + 6 * M, ws_bytes=M):
    B.cf_linear_fwd(m, k, n, dtype, x, w, bias, act, alpha, residual, y, z, ws, ws_bytes, 0)


def data(m=64, k=48, n=32, dtype="f32", dz=A, w=A + M, residual=A + 2 * M, z=A + 3 * M, act="silu", alpha=0.01, dx=A + 4 * M,
         ws=A + 5 * M, ws_bytes=M):
    B.cf_linear_bwd_data(m, k, n, dtype, dz, w, residual, z, act, alpha, dx, ws, ws_bytes, 0)


def weight(m=64, k=48, n=32, dtype="f32", x=A, dz=A + M, dw=A + 2 * M, db=A + 3 * M, ws=A + 4 * M, ws_bytes=M):
    B.cf_linear_bwd_weight(m, k, n, dtype, x, dz, dw, db, ws, ws_bytes, 0)


@pytest.mark.parametrize("call", [fwd, data, weight])
def test_sizes(call):
    for bad in (dict(m=-1), dict(k=0), dict(n=0), dict(k=-4), dict(n=-4)):
        expect(B.CF_ERR_INVALID_ARG, lambda: call(**bad))
    for bad in (dict(k=(1 << 24) + 1), dict(n=(1 << 24) + 1), dict(m=1 << 30, k=1 << 10), dict(m=1 << 30, n=1 << 10),
                dict(k=1 << 20, n=1 << 20)):
        expect(B.CF_ERR_UNSUPPORTED, lambda: call(**bad))
    with pytest.raises(ValueError):
        call(dtype="f64")


@pytest.mark.parametrize("call", [fwd, data])
def test_activation(call):
    for alpha in (math.nan, math.inf):
        expect(B.CF_ERR_INVALID_ARG, lambda: call(act="lrelu", alpha=alpha))
    with pytest.raises(ValueError):
        call(act="relu6")
    expect(B.CF_ERR_INVALID_ARG, lambda: data(z=None))
    expect(B.CF_ERR_INVALID_ARG,
           lambda: B._check(B.lib().cf_linear_fwd(1, 1, 1, 0, A, A + M, None, -1, 0.0, None, A + 2 * M, None, None, 0, None)))
    expect(B.CF_ERR_INVALID_ARG,
           lambda: B._check(B.lib().cf_linear_fwd(1, 1, 1, 5, A, A + M, None, 0, 0.0, None, A + 2 * M, None, None, 0, None)))


@pytest.mark.parametrize("call,required,optional", [(fwd, ("x", "w", "y"), ("bias", "residual", "z")),
                                                    (data, ("dz", "w", "dx"), ("residual", "z")),
                                                    (weight, ("x", "dz", "dw"), ("db",))])
def test_pointers(call, required, optional):
    for name in required:
        expect(B.CF_ERR_INVALID_ARG, lambda: call(**{name: None}))
    for name in required + optional:
        expect(B.CF_ERR_ALIGNMENT, lambda: call(**{name: A + 40 * M + 4}))


def test_overlaps():
    for bad in (dict(y=A), dict(y=A + M), dict(y=A + 3 * M + 16), dict(z=A + 4 * M), dict(z=A + 3 * M), dict(y=A + 2 * M),
                dict(z=A + 16)):
        expect(B.CF_ERR_ALIAS, lambda: fwd(**bad))
    for bad in (dict(dx=A), dict(dx=A + M), dict(dx=A + 2 * M + 16), dict(dx=A + 3 * M + 16)):
        expect(B.CF_ERR_ALIAS, lambda: data(**bad))
    for bad in (dict(dw=A), dict(dw=A + M + 16), dict(db=A + 2 * M), dict(db=A)):
        expect(B.CF_ERR_ALIAS, lambda: weight(**bad))
    expect(B.CF_ERR_ALIAS, lambda: weight(m=0, db=A + 2 * M))


SIZES = [(64, 48, 32), (4096, 1024, 512), (70000, 30, 50), (1, 8192, 3), (33, 8192, 40)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_workspace(dt):
    big = 1 << 36
    for m, k, n in SIZES:
        need = B.cf_linear_fwd_workspace_size(m, k, n, dt)
        at = dict(m=m, k=k, n=n, dtype=dt, x=A, w=A + big, bias=None, residual=None, y=A + 2 * big, z=None)
        if need:
            expect(B.CF_ERR_WORKSPACE, lambda: fwd(**at, ws=None, ws_bytes=need))
            expect(B.CF_ERR_WORKSPACE, lambda: fwd(**at, ws=A + 3 * big, ws_bytes=need - 1))
            expect(B.CF_ERR_ALIGNMENT, lambda: fwd(**at, ws=A + 3 * big + 4, ws_bytes=need))
            expect(B.CF_ERR_ALIAS, lambda: fwd(**at, ws=A + 2 * big, ws_bytes=need))
        need = B.cf_linear_bwd_data_workspace_size(m, k, n, dt)
        at = dict(m=m, k=k, n=n, dtype=dt, dz=A, w=A + big, residual=None, z=A + 2 * big, dx=A + 3 * big)
        if need:
            expect(B.CF_ERR_WORKSPACE, lambda: data(**at, ws=None, ws_bytes=need))
            expect(B.CF_ERR_WORKSPACE, lambda: data(**at, ws=A + 4 * big, ws_bytes=need - 1))
            expect(B.CF_ERR_ALIAS, lambda: data(**at, ws=A, ws_bytes=need))
        need = B.cf_linear_bwd_weight_workspace_size(m, k, n, dt)
        at = dict(m=m, k=k, n=n, dtype=dt, x=A, dz=A + big, dw=A + 2 * big, db=A + 3 * big)
        if need:
            expect(B.CF_ERR_WORKSPACE, lambda: weight(**at, ws=None, ws_bytes=need))
            expect(B.CF_ERR_WORKSPACE, lambda: weight(**at, ws=A + 4 * big, ws_bytes=need - 1))
            expect(B.CF_ERR_ALIAS, lambda: weight(**at, ws=A + 2 * big, ws_bytes=need))
    for m, k, n in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), (0, 4, 4)):
        for q in (B.cf_linear_fwd_workspace_size, B.cf_linear_bwd_data_workspace_size, B.cf_linear_bwd_weight_workspace_size):
            assert q(m, k, n, dt) == 0
