"""Group normalisation, the block over a voxel's channels and AdamW as the network runs
them together: each stage against its formula in float64 on the stage's own inputs, the
same bits on one stream and two, deferred sums or not, captured or not, and what is
refused.

Tolerances (fp32, relative to the norm).  A sum of K terms of mixed signs is off by at
most 4 sqrt(K) 2^-24 of its terms' norm, 7.6e-6 for K <= 1024 terms.  A group
normalisation forward is three such sums, its mean relative to the largest value (factor
KAPPA = rms / deviation of the groups); its backward three more on top.  From the stack's
output to its gradient there are 5 products and 3 sums forward and 10 products and 4 sums
backward: 22 * 7.6e-6 = 1.7e-4.  AdamW's first step of fp32 values: u = g / (|g| + eps) to
8 roundings of 2^-24, and half a unit of the parameter for each of its two updates."""
import math
import os

import numpy as np
import pytest
import torch

from paper_1808_04728_amd import binding as B
from paper_1808_04728_amd import inputs
from paper_1808_04728_amd.mixer import ChannelMixer
from paper_1808_04728_amd.network import NORM_EPS, Network, main, synthetic
from paper_1808_04728_amd.stack import GROUP_NORM_EPS, ConvStack

gpu = pytest.mark.gpu
built = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libcosmoflow_hip.so not built")
SUM = 4 * 32 * 2.0 ** -24
LAYERS = [dict(l, norm=math.gcd(l["cout"], 8), act=a)
          for l, a in zip(inputs.stack_layers(), ("silu", "gelu", "lrelu", "none", "silu", "gelu"))]
MIXED = [LAYERS[0], inputs.stack_layers()[1], *LAYERS[2:4], *inputs.stack_layers()[4:]]


def make(layers=LAYERS, size=32, batch=2, dtype="f32", seed=3, **kw):
    net = Network(layers, size, batch, dtype=dtype, **kw)
    x, *params = synthetic(size, batch, layers=layers, features=net.head.dims[0], seed=seed)
    net.stack.set_input(x)
    c, h = net.c if kw.get("norm") != "sample" else 128, kw.get("mixer", 0)
    mixer = None
    if h:
        mixer = ([inputs.normal((c, h), seed + 1, (2 / c) ** 0.5), inputs.normal((h, c), seed + 2, h ** -0.5)],
                 [inputs.normal((h,), seed + 3, 0.1), inputs.normal((c,), seed + 4, 0.1)])
    net.set_params(*params, mixer=mixer)
    return net


# ---- what is refused ----------------------------------------------------------------

@built
@pytest.mark.parametrize("layer", [dict(norm=3), dict(norm=-1), dict(norm=4, act="relu"), dict(act="silu")])
def test_layers_are_checked(layer):
    with pytest.raises(ValueError):
        ConvStack([dict(inputs.stack_layers()[0], **layer)], 16, 1, device="cpu", overlap_wgrad=False)


@built
@pytest.mark.parametrize("kw", [dict(norm="group", groups=0), dict(norm="group", groups=3), dict(optimizer="sgd"),
                                dict(mixer=-1)])
def test_options_are_checked(kw):
    with pytest.raises(ValueError):
        Network(inputs.stack_layers(), 32, 1, device="cpu", **kw)


@built
def test_hyperparameters_are_checked():
    muon, adamw = (Network(inputs.stack_layers(), 32, 1, device="cpu", optimizer=o) for o in ("muon", "adamw8"))
    for net, hp in ((muon, (B.make_adamw_hparams(10),)), (muon, (B.make_muon_hparams(10),)),
                    (adamw, (B.make_muon_hparams(10), B.make_hparams(10))),
                    (adamw, (B.make_adamw_hparams(10), B.make_hparams(10)))):
        with pytest.raises(ValueError):
            net.update(*hp)
        assert net.t == 0
    with pytest.raises(ValueError):
        muon.set_params([], [], [], [], np.zeros((1, 3), np.float32), mixer=([], []))


@built
@pytest.mark.parametrize("miss", ["gamma", "dgamma"])
def test_gamma_is_bound(miss):
    s = ConvStack(LAYERS, 32, 1, device="cpu", overlap_wgrad=False)
    keys = ("w", "w32", "b", "dw", "db", "gamma", "dgamma")
    ps = [{k: torch.zeros_like(l[k]) for k in keys} for l in s.L]
    own = s.L[0]["gamma"]
    del ps[0][miss]
    with pytest.raises(ValueError):
        s.bind_params(ps)
    assert s.L[0]["gamma"] is own
    ps[0][miss] = torch.zeros_like(own)
    s.bind_params(ps)
    assert s.L[0][miss] is ps[0][miss]


# ---- stage by stage -----------------------------------------------------------------

def act64(u, act, alpha=0.01):
    return {"none": lambda: u, "lrelu": lambda: torch.where(u > 0, u, alpha * u), "silu": lambda: u * torch.sigmoid(u),
            "gelu": lambda: u * 0.5 * torch.erfc(-u / math.sqrt(2))}[act]()


def norm64(x, gamma, beta, groups, act, eps):
    n, c = x.shape[0], x.shape[-1]
    h = x.reshape(n, -1, groups, c // groups)
    var, mean = torch.var_mean(h, (1, 3), correction=0, keepdim=True)
    return act64(((h - mean) / torch.sqrt(var + eps)).reshape(x.shape) * gamma + beta, act)


def leaf(t, *shape):
    return (t.reshape(*shape) if shape else t).detach().double().cpu().requires_grad_()


def close(got, want, tol, what):
    got, want = got.detach().double().cpu().reshape(-1), want.detach().reshape(-1)
    err, size = float((got - want).norm()), float(want.norm())
    assert err <= tol * size, (what, err / size, tol)


def conv64(x, w, stride):
    k = w.shape[0]
    pads = []
    for n in reversed(x.shape[1:4]):
        t = max((-(-n // stride) - 1) * stride + k - n, 0)
        pads += [t // 2, t - t // 2]
    x = torch.nn.functional.pad(x.permute(0, 4, 1, 2, 3), pads)
    return torch.nn.functional.conv3d(x, w.permute(4, 3, 0, 1, 2), stride=stride).permute(0, 2, 3, 4, 1)


@gpu
@pytest.mark.parametrize("layers", [LAYERS, MIXED], ids=["all", "some"])
@pytest.mark.parametrize("overlap", [False, True])
def test_stack_stage_by_stage(layers, overlap):
    st = ConvStack(layers, 32, 2, overlap_wgrad=overlap)
    x, cw, cb, *_ = synthetic(32, 2, layers=layers, features=1024, seed=11)
    st.set_input(x)
    st.set_params(cw, [inputs.normal(b.shape, 5, 0.3) for b in cb])
    for i, l in enumerate(st.L):
        if l["groups"]:
            l["gamma"].copy_(torch.as_tensor(1 + inputs.normal(l["gamma"].shape, 50 + i, 0.3)))
    out = st.forward()
    dout = torch.as_tensor(inputs.normal(tuple(out.shape), 60)).cuda()
    st.backward(dout)
    torch.cuda.synchronize()
    for i, l in enumerate(st.L):
        if not l["groups"]:
            continue
        s, name = l["spec"], f"layer {i + 1}"
        xin, w = leaf(st.layer_input(i)), leaf(l["w"])
        u = conv64(xin, w, s["stride"])
        close(l["u"], u, 4 * math.sqrt(s["k"] ** 3 * s["cin"]) * 2.0 ** -24, name + " u")
        gout = st.L[i + 1]["dx"] if i + 1 < len(st.L) else dout
        gout = gout.double().cpu()
        if s["pool"]:
            gout = torch.nn.functional.interpolate(gout.permute(0, 4, 1, 2, 3), scale_factor=2).permute(0, 2, 3, 4, 1) / 8
        un, g, b = leaf(l["u"]), leaf(l["gamma"]), leaf(l["b"])
        y = norm64(un, g, b, l["groups"], l["act"], GROUP_NORM_EPS)
        var, mean = torch.var_mean(un.detach().reshape(2, -1, l["groups"], s["cout"] // l["groups"]), (1, 3), correction=0)
        kappa = float(torch.sqrt(1 + mean * mean / (var + GROUP_NORM_EPS)).max())
        close(l["z"], y, 3 * SUM * kappa, name + " y")
        y.backward(gout)
        for t, want in (("dz", un.grad), ("dgamma", g.grad), ("db", b.grad)):
            close(l[t], want, 6 * SUM * kappa, f"{name} {t}")
        u.backward(l["dz"].double().cpu())
        terms = u.numel() // s["cout"]
        close(l["dw"], w.grad, 4 * math.sqrt(terms) * 2.0 ** -24, name + " dw")
        if i:
            close(l["dx"], xin.grad, 4 * math.sqrt(s["k"] ** 3 * s["cout"]) * 2.0 ** -24, name + " dx")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_stack_same_bits_on_two_streams_and_undeferred(dtype):
    x, cw, cb, *_ = synthetic(32, 2, layers=MIXED, features=1024, seed=12)
    runs = []
    for kw in (dict(overlap_wgrad=False), dict(overlap_wgrad=True), dict(overlap_wgrad=False, defer_reductions=False)):
        st = ConvStack(MIXED, 32, 2, dtype=dtype, **kw)
        st.set_input(x)
        st.set_params(cw, cb)
        out = st.forward()
        st.backward(torch.as_tensor(inputs.normal(tuple(out.shape), 61)).cuda().to(out.dtype))
        torch.cuda.synchronize()
        runs.append((out.clone(), st.flat_grad.clone()))
        assert bool(torch.isfinite(st.flat_grad).all()) and all(float(l["dw"].abs().max()) > 0 for l in st.L)
    for o, g in runs[1:]:
        assert torch.equal(o, runs[0][0]) and torch.equal(g, runs[0][1])


@gpu
@pytest.mark.parametrize("norm", ["sample", "voxel", "group"])
def test_block_and_norm_against_float64(norm):
    net = make(norm=norm, mixer=200, groups=4)
    net.gamma.copy_(torch.as_tensor(1 + inputs.normal((net.c,), 70, 0.3)))
    net.beta.copy_(torch.as_tensor(inputs.normal((net.c,), 71, 0.3)))
    loss = net.step()
    m = net.mixer
    x = leaf(net.stack.output(), -1, 128)
    w, b = [leaf(t) for t in m.w], [leaf(t) for t in m.b]
    g, be = leaf(net.gamma), leaf(net.beta)
    h = x + act64(x @ w[0] + b[0], "gelu") @ w[1] + b[1]
    if norm == "group":
        h = norm64(h.reshape(2, -1, 128), g, be, 4, "none", NORM_EPS)
    else:
        h = h.reshape(net.rows, net.c)
        var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
        h = (h - mean) / torch.sqrt(var + NORM_EPS) * g + be
    h = h.reshape(2, -1)
    for i in range(3):
        h = torch.nn.functional.leaky_relu(h @ net.head.w[i].double().cpu() + net.head.b[i].double().cpu(), 0.01)
    ref = ((h - net.head.target.double().cpu()) ** 2).mean()
    ref.backward()
    tol = 22 * SUM
    assert abs(float(loss[0]) - ref.item()) <= tol * ref.item()
    for what, got, want in (("dx", m.dx, x.grad), ("dgamma", net.dgamma, g.grad), ("dbeta", net.dbeta, be.grad),
                            *((f"dw{i}", m.dw[i], w[i].grad) for i in range(2)),
                            *((f"db{i}", m.db[i], b[i].grad) for i in range(2))):
        close(got, want, tol, what)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_zero_block_is_the_identity(dtype):
    x = torch.as_tensor(inputs.normal((37, 48), 1)).cuda().to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    m = ChannelMixer(37, 48, 30, dtype=dtype)
    m.set_params([inputs.normal((48, 30), 2), np.zeros((30, 48))], [np.zeros(30), np.zeros(48)])
    assert torch.equal(m.forward(x), x)
    assert torch.equal(m.backward(x), x)
    assert not m.dw[0].any() and not m.db[0].any() and m.dw[1].any()


# ---- updates, graphs, the command ---------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_first_adamw_step(dtype):
    eta, decay, eps = 0.01, 0.1, 1e-8
    after = []
    for o in ("adamw", "adamw8"):
        net = make(dtype=dtype, norm="group", mixer=40, optimizer=o, weight_decay=decay)
        net.step()
        p, g = net.param.double().cpu(), net.grad.double().cpu()
        net.update(B.make_adamw_hparams(100, eta0=eta, eta_min=eta, eps=eps))
        after.append(net.param.clone())
        got = net.param.double().cpu()
        wd = torch.zeros_like(p)
        for q in net.mats:
            wd[q.offset:q.offset + q.rows * q.cols] = decay
        want = p - eta * wd * p - eta * g / (g.abs() + eps)
        bound = 2.0 ** -24 * (8 * eta + 2 * p.abs())
        assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())
        if dtype == "bf16":
            for q in net.mats:
                sl = slice(q.offset, q.offset + q.rows * q.cols)
                assert torch.equal(net.w16[sl], net.param[sl].bfloat16())
        assert all(bool(s.any()) for s in net.state)
    # the step comes from the moments before they are rounded to a byte
    assert torch.equal(*after)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured(dtype):
    net = make(layers=MIXED, dtype=dtype, norm="group", mixer=64, optimizer="adamw8")
    hp = B.make_adamw_hparams(10)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        net.step()
    for _ in range(4):
        net.step()
        torch.cuda.synchronize()
        want = net.grad.clone(), net.head.loss.clone()
        net.grad.zero_()
        net.head.loss.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(net.grad, want[0]) and torch.equal(net.head.loss, want[1])
        net.update(hp)  # eager work between the replays, and other weights for the next
    assert net.t == 4


@gpu
@pytest.mark.parametrize("args", [["--norm", "group", "--mixer", "32", "--optimizer", "adamw8", "--conv-norm", "silu"],
                                  ["--optimizer", "adamw", "--dtype", "f32"], ["--mixer", "8", "--conv-norm", "gelu"]])
def test_command(capsys, args):
    main(["--size", "32", "--batch", "1", "--steps", "3", *args])
    out = capsys.readouterr().out
    losses = [float(l.split()[-1]) for l in out.splitlines() if "loss" in l]
    assert "step 3: loss" in out and all(math.isfinite(v) for v in losses)
