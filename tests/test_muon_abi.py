"""Host-side refusals of the orthogonalised updates (no kernel is launched)."""
import math
import os

import pytest

from paper_1808_04728_amd import binding as B

A = 0x7F0000000000  # fake, 16-byte aligned device addresses (never dereferenced)
M = 1 << 30

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libcosmoflow_hip.so not built")

ONE = ([0], [64], [48])


def expect(status, fn, *args):
    with pytest.raises(B.CfError) as e:
        fn(*args)
    assert e.value.status == status, str(e.value)
    assert B.cf_last_error() != ""


def ns(mats=ONE, dtype="f32", g=A, o=A + M, ws=A + 2 * M, ws_bytes=M, **hp):
    B.cf_newton_schulz(B.make_matrices(*mats), dtype, B.make_ns_hparams(**hp), g, o, ws, ws_bytes, 0)


def muon(mats=ONE, t=0, v=A, g=A + M, m=A + 2 * M, v16=A + 3 * M, ws=A + 4 * M, ws_bytes=M, t_decay=10, **hp):
    B.cf_muon_step(B.make_matrices(*mats), t, B.make_muon_hparams(t_decay, **hp), v, g, m, v16, ws, ws_bytes, 0)


@pytest.mark.parametrize("call", [ns, muon])
def test_matrices(call):
    expect(B.CF_ERR_INVALID_ARG, lambda: call(([-8], [4], [4])))
    expect(B.CF_ERR_INVALID_ARG, lambda: call(([0], [-4], [4])))
    expect(B.CF_ERR_INVALID_ARG, lambda: call(([0], [4], [-4])))
    expect(B.CF_ERR_ALIGNMENT, lambda: call(([4], [4], [4])))
    expect(B.CF_ERR_UNSUPPORTED, lambda: call(([0], [16385], [16385])))
    expect(B.CF_ERR_UNSUPPORTED, lambda: call(([0], [1], [(1 << 24) + 1])))
    expect(B.CF_ERR_ALIAS, lambda: call(([0, 8], [4, 4], [4, 4])))
    expect(B.CF_ERR_ALIAS, lambda: call(([16, 0], [4, 4], [4, 4])))
    with pytest.raises(ValueError):
        call(([0, 16], [4], [4]))


def test_null_arguments():
    L, ms, hp = B.lib(), B.make_matrices(*ONE), B.make_ns_hparams()
    mh = B.make_muon_hparams(10)
    assert L.cf_newton_schulz(1, None, 0, hp, A, A + M, A + 2 * M, M, None) == B.CF_ERR_INVALID_ARG
    assert L.cf_newton_schulz(1, ms, 0, None, A, A + M, A + 2 * M, M, None) == B.CF_ERR_INVALID_ARG
    assert L.cf_newton_schulz(-1, ms, 0, hp, A, A + M, A + 2 * M, M, None) == B.CF_ERR_INVALID_ARG
    assert L.cf_newton_schulz(1, ms, 5, hp, A, A + M, A + 2 * M, M, None) == B.CF_ERR_INVALID_ARG
    assert L.cf_newton_schulz((1 << 16) + 1, ms, 0, hp, A, A + M, A + 2 * M, M, None) == B.CF_ERR_UNSUPPORTED
    assert L.cf_muon_step(1, None, 0, mh, A, A + M, A + 2 * M, None, A + 3 * M, M, None) == B.CF_ERR_INVALID_ARG
    assert L.cf_muon_step(1, ms, 0, None, A, A + M, A + 2 * M, None, A + 3 * M, M, None) == B.CF_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [ns, muon])
@pytest.mark.parametrize("bad", [dict(steps=0), dict(steps=33), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
                                 dict(coef=(math.nan, 0, 0)), dict(coef=(1, math.inf, 0))])
def test_iteration(call, bad):
    expect(B.CF_ERR_INVALID_ARG, lambda: call(**bad))


@pytest.mark.parametrize("call", [ns, muon])
def test_coefficients_that_grow(call):
    expect(B.CF_ERR_UNSUPPORTED, lambda: call(coef=(4.0, 0.0, 0.0)))
    expect(B.CF_ERR_UNSUPPORTED, lambda: call(coef=(3.4445, -4.7750, 9.0)))
    expect(B.CF_ERR_UNSUPPORTED, lambda: call(coef=(1e200, 1e200, 1e200)))


@pytest.mark.parametrize("bad", [dict(mu=-0.1), dict(mu=1.0), dict(mu=math.nan), dict(weight_decay=-1.0), dict(eta0=math.inf),
                                 dict(eta_min=math.nan), dict(weight_decay=math.inf), dict(scale=2), dict(scale=-1),
                                 dict(nesterov=2), dict(t=-1), dict(t_decay=0)])
def test_muon_hyperparameters(bad):
    expect(B.CF_ERR_INVALID_ARG, lambda: muon(**bad))


def test_pointers_and_workspace():
    need = B.cf_newton_schulz_workspace_size(B.make_matrices(*ONE), "f32")
    assert need > 0
    for name in ("g", "o"):
        expect(B.CF_ERR_INVALID_ARG, lambda: ns(**{name: None}))
        expect(B.CF_ERR_ALIGNMENT, lambda: ns(**{name: A + 9 * M + 4}))
    for name in ("v", "g", "m"):
        expect(B.CF_ERR_INVALID_ARG, lambda: muon(**{name: None}))
        expect(B.CF_ERR_ALIGNMENT, lambda: muon(**{name: A + 9 * M + 4}))
    expect(B.CF_ERR_ALIGNMENT, lambda: muon(v16=A + 9 * M + 4))
    expect(B.CF_ERR_WORKSPACE, lambda: ns(ws=None))
    expect(B.CF_ERR_WORKSPACE, lambda: ns(ws_bytes=need - 1))
    expect(B.CF_ERR_ALIGNMENT, lambda: ns(ws=A + 2 * M + 8))
    need = B.cf_muon_workspace_size(B.make_matrices(*ONE))
    expect(B.CF_ERR_WORKSPACE, lambda: muon(ws=None))
    expect(B.CF_ERR_WORKSPACE, lambda: muon(ws_bytes=need - 1))
    expect(B.CF_ERR_ALIGNMENT, lambda: muon(ws=A + 4 * M + 8))
    expect(B.CF_ERR_ALIAS, lambda: ns(o=A + 16))
    expect(B.CF_ERR_ALIAS, lambda: ns(ws=A))
    expect(B.CF_ERR_ALIAS, lambda: ns(ws=A + M))
    for a in ("v", "g", "m", "v16"):
        expect(B.CF_ERR_ALIAS, lambda: muon(**{a: A + 4 * M}))
    expect(B.CF_ERR_ALIAS, lambda: muon(g=A))
    assert B.cf_newton_schulz_workspace_size(B.make_matrices([0], [-1], [4]), "f32") == 0
    assert B.cf_muon_workspace_size(B.make_matrices([4], [4], [4])) == 0


def test_nothing_to_do():
    for mats in (([], [], []), ([0], [0], [5]), ([0, 0], [7, 0], [0, 0])):
        ns(mats, g=None, o=None, ws=None, ws_bytes=0)
        muon(mats, v=None, g=None, m=None, v16=None, ws=None, ws_bytes=0)
        assert B.cf_newton_schulz_workspace_size(B.make_matrices(*mats), "bf16") == 0
        assert B.cf_muon_workspace_size(B.make_matrices(*mats)) == 0
