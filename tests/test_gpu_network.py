"""The network with layer normalisation and its two updates, end to end: the same
bits as its parts run one by one, gradients through head and normalisation against
float64, parameters after an update against float64, and a loss that falls.

Tolerances.  Gradients (fp32): twelve sums on the way (two statistics and the output
of the normalisation, three products forward and six backward, the normalisation's
backward), each with an error of at most 4 sqrt(K) 2^-24 of its terms' norm for
K <= 1024 terms of mixed signs: 12 * 4 * 32 * 2^-24 = 9.2e-5, taken as 1e-4 of the
gradient's norm.  Matrices after an update: the orthogonalisation's 4 a^5 2^-24 of the
update's norm, and half a unit of each parameter."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_1808_04728_amd import binding as B
from paper_1808_04728_amd import inputs
from paper_1808_04728_amd.head import FCHead
from paper_1808_04728_amd.network import NORM_EPS, Network, layout, main, synthetic
from paper_1808_04728_amd.stack import ConvStack

gpu = pytest.mark.gpu
LAYERS = inputs.stack_layers()


def make(size=32, batch=2, dtype="f32", norm="sample", seed=0):
    net = Network(LAYERS, size, batch, dtype=dtype, norm=norm)
    x, *params = synthetic(size, batch, layers=LAYERS, features=net.head.dims[0], seed=seed)
    net.stack.set_input(x)
    net.set_params(*params)
    return net, x, params


def test_layout():
    off = layout([27 * 16, 16, 3, 1, 0, 17])
    assert off == [0, 432, 448, 464, 480, 480, 512]


def test_norm_is_checked():
    with pytest.raises(ValueError):
        Network(LAYERS, 32, 1, norm="batch")


@gpu
@pytest.mark.parametrize("norm", ["sample", "voxel"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_as_the_parts(dtype, norm):
    net, x, (cw, cb, fw, fb, target) = make(dtype=dtype, norm=norm)
    loss = net.step()
    st = ConvStack(LAYERS, 32, 2, dtype=dtype)
    st.set_input(x)
    st.set_params(cw, cb)
    head = FCHead(2, net.head.dims[0], net.head.dims[1:], dtype=dtype)
    head.set_params(fw, fb, target)
    h = st.forward()
    rows, c = (2, h.numel() // 2) if norm == "sample" else (h.numel() // 128, 128)
    one, zero = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    y, dout = torch.empty((2, h.numel() // 2), dtype=h.dtype, device="cuda"), torch.empty_like(h)
    mean, rstd = (torch.empty(rows, device="cuda") for _ in range(2))
    dg, db = torch.empty_like(one), torch.empty_like(one)
    ws = torch.empty(max(16, B.cf_layernorm_fwd_workspace_size(rows, c, dtype),
                         B.cf_layernorm_bwd_workspace_size(rows, c, dtype)), dtype=torch.uint8, device="cuda")
    B.cf_layernorm_fwd(rows, c, dtype, h, one, zero, NORM_EPS, y, mean, rstd, ws)
    dy = head.step(y)
    B.cf_layernorm_bwd(rows, c, dtype, dy, h, one, mean, rstd, dout, dg, db, ws)
    st.backward(dout)
    assert torch.equal(loss[0], head.loss[0])
    assert torch.equal(net.dgamma, dg) and torch.equal(net.dbeta, db)
    for a, b in zip(net.stack.L, st.L):
        assert torch.equal(a["dw"], b["dw"]) and torch.equal(a["db"], b["db"])
    for i in range(3):
        assert torch.equal(net.head.dw[i], head.dw[i]) and torch.equal(net.head.db[i], head.db[i])
    with pytest.raises(RuntimeError):
        net.stack.update(B.make_hparams(10))


@gpu
@pytest.mark.parametrize("norm", ["sample", "voxel"])
def test_gradients_against_float64(norm):
    net, _, (cw, cb, fw, fb, target) = make(norm=norm, seed=5)
    rng = np.random.Generator(np.random.PCG64(77))
    net.gamma.copy_(torch.as_tensor(rng.uniform(0.5, 1.5, net.c)))
    net.beta.copy_(torch.as_tensor(rng.uniform(-0.5, 0.5, net.c)))
    loss = net.step()
    x = net.stack.output().double().cpu().reshape(net.rows, net.c).requires_grad_()
    g = net.gamma.double().cpu().requires_grad_()
    b = net.beta.double().cpu().requires_grad_()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    h = ((x - mean) / torch.sqrt(var + NORM_EPS) * g + b).reshape(2, -1)
    for w, bias in zip(fw, fb):
        h = torch.nn.functional.leaky_relu(h @ torch.as_tensor(w).double() + torch.as_tensor(bias).double(), 0.01)
    ref = ((h - torch.as_tensor(target).double()) ** 2).mean()
    ref.backward()
    assert abs(float(loss[0]) - float(ref)) <= 1e-4 * float(ref)
    for got, want in ((net.dout, x.grad), (net.dgamma, g.grad), (net.dbeta, b.grad)):
        err = float((got.double().cpu().reshape(-1) - want.reshape(-1)).norm())
        assert err <= 1e-4 * float(want.norm()), (err, float(want.norm()))


def ns64(x, steps=5, coef=B.NS_COEF, eps=1e-7):
    a, b, c = coef
    x = x / (x.norm() + eps)
    for _ in range(steps):
        h = x.t() @ x
        x = a * x + x @ (b * h + c * (h @ h))
    return x


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_update_against_float64(dtype):
    net, _, _ = make(dtype=dtype, seed=9)
    mu, eta, decay = 0.95, 0.02, 0.1
    hv = B.make_hparams(100)
    for t in range(2):
        net.step()
        before = [b.double().cpu() for b in (net.param, net.grad, net.momentum)]
        vec = [b[net.vec0:].double().cpu().numpy() for b in (net.param, net.grad, net.momentum)]
        second = net.second.double().cpu().numpy()
        net.update(B.make_muon_hparams(100, eta0=eta, eta_min=eta, mu=mu, weight_decay=decay), hv)
        after = net.param.double().cpu()
        for q in net.mats:
            sl = slice(q.offset, q.offset + q.rows * q.cols)
            v, g, m = (b[sl].view(q.rows, q.cols) for b in before)
            m = mu * m + (1 - mu) * g
            u = ns64((1 - mu) * g + mu * m) if q.rows >= q.cols else ns64(((1 - mu) * g + mu * m).t()).t()
            upd = eta * (math.sqrt(max(1.0, q.cols / q.rows)) * u + decay * v)
            err = float((after[sl].view(q.rows, q.cols) - (v - upd)).norm())
            bound = 4 * B.NS_COEF[0] ** 5 * 2.0 ** -24 * float(upd.norm()) + 2.0 ** -24 * float(v.norm())
            assert err <= bound, (t, q.rows, q.cols, err, bound)
            if dtype == "bf16":
                assert torch.equal(net.w16[sl], net.param[sl].bfloat16())
        v1, _, _, _ = oracle.adam_larc_step(list(net.vec_offsets[1]), t, 100, *vec, second)
        got = net.param[net.vec0:].double().cpu().numpy()
        assert np.all(np.abs(got - v1) <= np.spacing(np.abs(v1.astype(np.float32))))


@gpu
@pytest.mark.parametrize("norm", ["sample", "voxel"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loss_falls(dtype, norm):
    net, _, _ = make(dtype=dtype, norm=norm)
    hm, hv = B.make_muon_hparams(30, eta0=0.02), B.make_hparams(30)
    losses = []
    for _ in range(30):
        losses.append(float(net.step()[0]))
        net.update(hm, hv)
    assert all(math.isfinite(v) for v in losses)
    assert losses[-1] < 0.5 * losses[0], losses


@gpu
def test_command(capsys):
    main(["--size", "32", "--batch", "1", "--steps", "3"])
    assert "step 3: loss" in capsys.readouterr().out
