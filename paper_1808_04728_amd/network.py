"""The whole network as it trains: convolution stack, a block over the channels of each
voxel if asked for, normalisation of its output, fully-connected head, and one update of
all parameters.

  forward   stack -> [mixer] -> normalisation -> head -> loss
  backward  head -> normalisation -> [mixer] -> stack
  update    "muon": matrices (the weights) take momentum with orthogonalised steps, one
            cf_muon_step call; vectors (biases, the normalisations' gamma and beta) Adam +
            LARC, one cf_adam_larc_step call
            "adamw", "adamw8": one cf_adamw_step call for all of them, its two moments in
            fp32 or in a byte a value; matrices decay, vectors do not

The normalisation runs over a sample's whole output (``norm="sample"``: batch rows of
d*h*w*c values), over the channels of each voxel (``norm="voxel"``: batch*d*h*w rows of
c) or over groups of channels of a sample (``norm="group"``).  The head then sees inputs
of one scale whatever the updates do to the convolutions.

All parameters live in flat buffers, matrices first and vectors after them, each on
a multiple of 16 elements: fp32 values, fp32 gradients, and for a bf16 network the
bf16 weights that the products read.

``python -m paper_1808_04728_amd.network`` trains on synthetic cubes.
"""
from __future__ import annotations

import argparse
import math
import time

import numpy as np
import torch

from . import binding as B
from . import inputs
from .head import FCHead
from .mixer import ChannelMixer
from .stack import ConvStack

NORM_EPS = 1e-5


def layout(sizes):
    """Element offsets of tensors of these sizes, each on a multiple of 16, and the end."""
    off = [0]
    for n in sizes:
        off.append(off[-1] + (n + 15) // 16 * 16)
    return off


class Network:
    def __init__(self, layers, size, batch, widths=inputs.HEAD_WIDTHS, dtype="f32", norm="sample", alpha=0.01,
                 device="cuda", groups=8, mixer=0, optimizer="muon", weight_decay=0.01):
        """groups: of norm="group".  mixer: hidden values of the block over a voxel's channels
        (0: no such block).  weight_decay: of the matrices, with "adamw" and "adamw8"."""
        if norm not in ("sample", "voxel", "group"):
            raise ValueError(f"norm: {norm}")
        if optimizer not in ("muon", "adamw", "adamw8"):
            raise ValueError(f"optimizer: {optimizer}")
        self.dtype, self.norm, self.groups, self.optimizer = dtype, norm, groups, optimizer
        self.stack = ConvStack(layers, size, batch, dtype=dtype, alpha=alpha, device=device)
        out = self.stack.output()
        features, channels = out.numel() // batch, out.shape[-1]
        if norm == "group" and (groups < 1 or channels % groups):
            raise ValueError(f"groups: {groups} of {channels} channels")
        self.vox = features // channels
        self.rows, self.c = (batch, features) if norm == "sample" else (out.numel() // channels, channels)
        self.head = FCHead(batch, features, widths, dtype=dtype, alpha=alpha, device=device)
        self.mixer = ChannelMixer(batch * self.vox, channels, mixer, dtype=dtype, device=device) if mixer else None
        self._alloc_params(device, weight_decay)
        self.y = torch.empty((batch, features), dtype=out.dtype, device=device)
        self.dout = torch.empty_like(out)
        self.mean = torch.empty(batch * groups if norm == "group" else self.rows, dtype=torch.float32, device=device)
        self.rstd = torch.empty_like(self.mean)
        if norm == "group":
            shape = (batch, self.vox, self.c, groups, dtype)
            nws = max(16, B.cf_groupnorm_fwd_workspace_size(*shape), B.cf_groupnorm_bwd_workspace_size(*shape))
        else:
            nws = max(16, B.cf_layernorm_fwd_workspace_size(self.rows, self.c, dtype),
                      B.cf_layernorm_bwd_workspace_size(self.rows, self.c, dtype))
        if optimizer == "muon":
            nws = max(nws, B.cf_muon_workspace_size(self.mats), B.cf_adam_larc_workspace_size(self.vec_offsets))
        self.ws = torch.empty(nws, dtype=torch.uint8, device=device)
        self.t = 0

    def _alloc_params(self, device, weight_decay):
        convs, mixed = self.stack.L, self.mixer.w if self.mixer else []
        normed = [i for i, l in enumerate(convs) if l["groups"]]
        shapes = [tuple(l["w32"].shape) for l in convs] + [tuple(w.shape) for w in [*self.head.w, *mixed]]
        vectors = [l["b"].numel() for l in convs] + [b.numel() for b in self.head.b]
        vectors += [b.numel() for b in self.mixer.b] if self.mixer else []
        vectors += [self.c, self.c] + [convs[i]["gamma"].numel() for i in normed]
        off = layout([int(np.prod(s)) for s in shapes] + vectors)
        nm = len(shapes)
        self.vec0 = off[nm]
        self.vec_offsets = B.adam_offsets([o - self.vec0 for o in off[nm:]])
        # a convolution's weights are the matrix of its taps and inputs by its outputs
        self.mats = B.make_matrices(off[:nm], [int(np.prod(s[:-1])) for s in shapes], [s[-1] for s in shapes])
        self.param = torch.zeros(off[-1], dtype=torch.float32, device=device)
        self.grad = torch.zeros_like(self.param)
        self.w16 = torch.zeros(self.vec0, dtype=torch.bfloat16, device=device) if self.dtype == "bf16" else None

        def view(buf, i):
            n = int(np.prod(shapes[i])) if i < nm else vectors[i - nm]
            return buf[off[i]:off[i] + n].view(shapes[i] if i < nm else (n,))

        ps = [dict(w=view(self.w16 if self.w16 is not None else self.param, i), w32=view(self.param, i),
                   b=view(self.param, nm + i), dw=view(self.grad, i), db=view(self.grad, nm + i)) for i in range(nm)]
        nl, nh = len(convs), len(self.head.w)
        for j, i in enumerate(normed):
            ps[i].update(gamma=view(self.param, 2 * nm + 2 + j), dgamma=view(self.grad, 2 * nm + 2 + j))
            ps[i]["gamma"].fill_(1.0)
        self.stack.bind_params(ps[:nl])
        self.head.bind_params(ps[nl:nl + nh])
        if self.mixer:
            self.mixer.bind_params(ps[nl + nh:])
        self._head_params, self._mixer_params = ps[nl:nl + nh], ps[nl + nh:]
        self.gamma, self.beta = view(self.param, 2 * nm), view(self.param, 2 * nm + 1)
        self.dgamma, self.dbeta = view(self.grad, 2 * nm), view(self.grad, 2 * nm + 1)
        self.gamma.fill_(1.0)
        if self.optimizer == "muon":
            self.momentum = torch.zeros_like(self.param)  # of matrices, and Adam's first moment
            self.second = torch.zeros(off[-1] - self.vec0, dtype=torch.float32, device=device)
            self.state = [self.momentum, self.second]
            return
        count = len(off) - 1
        if self.optimizer == "adamw":
            self.state = [torch.zeros_like(self.param) for _ in range(2)]
            moments = [dict(m=view(self.state[0], i), v=view(self.state[1], i)) for i in range(count)]
        else:
            self.state = [torch.zeros(off[-1], dtype=torch.uint8, device=device) for _ in range(2)]
            blocks = [-(-int(np.prod(n)) // B.CF_ADAMW_BLOCK) for n in shapes + vectors]
            at = np.cumsum([0] + blocks)
            self.state += [torch.zeros(int(at[-1]), dtype=torch.float32, device=device) for _ in range(2)]
            moments = [dict(m=view(self.state[0], i), v=view(self.state[1], i), m_scale=self.state[2][at[i]:at[i + 1]],
                            v_scale=self.state[3][at[i]:at[i + 1]]) for i in range(count)]
        self.tensors = B.make_adamw_tensors(
            [dict(p=view(self.param, i), g=view(self.grad, i),
                  p16=view(self.w16, i) if self.w16 is not None and i < nm else None,
                  weight_decay=weight_decay if i < nm else 0.0, **moments[i]) for i in range(count)])

    def set_params(self, conv_weights, conv_biases, fc_weights, fc_biases, target, mixer=None):
        """Weights are rounded to the network's dtype, their fp32 values hold exactly those;
        gamma = 1, beta = 0; resets the optimizer state.  mixer: its (weights, biases); by
        default He-normal first and zero second weights: the block starts as the identity."""
        self.stack.set_params(conv_weights, conv_biases)
        self.head.set_params(fc_weights, fc_biases, target)
        if self.mixer:
            c, h = self.mixer.c, self.mixer.hidden
            self.mixer.set_params(*(mixer if mixer is not None else (
                [inputs.normal((c, h), 4000, (2.0 / c) ** 0.5), np.zeros((h, c), np.float32)],
                [np.zeros(h, np.float32), np.zeros(c, np.float32)])))
        elif mixer is not None:
            raise ValueError("mixer: the network has none")
        for p in self._head_params + self._mixer_params:
            p["w32"].copy_(p["w"].float())
        self.gamma.fill_(1.0)
        self.beta.zero_()
        for s in self.state:
            s.zero_()
        self.t = 0

    def step(self, stream=None):
        """Forward and backward of the stack's input (stack.set_input) and the head's target:
        fills every gradient; returns the device loss tensor (one fp32 in element 0)."""
        s = B.raw_stream(stream)
        x = self.stack.forward(stream)
        if self.mixer:
            x = self.mixer.forward(x, s)
        if self.norm == "group":
            shape = (self.head.m, self.vox, self.c, self.groups, self.dtype)
            B.cf_groupnorm_fwd(*shape, x, self.gamma, self.beta, NORM_EPS, "none", 0.0, self.y, self.mean, self.rstd,
                               self.ws, stream=s)
        else:
            B.cf_layernorm_fwd(self.rows, self.c, self.dtype, x, self.gamma, self.beta, NORM_EPS, self.y, self.mean,
                               self.rstd, self.ws, stream=s)
        dy = self.head.step(self.y, stream)
        if self.norm == "group":
            B.cf_groupnorm_bwd(*shape, dy, x, self.gamma, self.beta, self.mean, self.rstd, "none", 0.0, self.dout,
                               self.dgamma, self.dbeta, self.ws, stream=s)
        else:
            B.cf_layernorm_bwd(self.rows, self.c, self.dtype, dy, x, self.gamma, self.mean, self.rstd, self.dout,
                               self.dgamma, self.dbeta, self.ws, stream=s)
        dout = self.mixer.backward(self.dout, s) if self.mixer else self.dout
        self.stack.backward(dout, stream)
        return self.head.loss

    def update(self, hp_matrices, hp_vectors=None, stream=None):
        """One update of all parameters from the gradients of the last step: with "muon"
        binding.make_muon_hparams and binding.make_hparams, else binding.make_adamw_hparams
        alone."""
        muon = self.optimizer == "muon"
        if isinstance(hp_matrices, B.cf_muon_hparams) != muon or (hp_vectors is not None) != muon:
            raise ValueError(f"hyperparameters of another optimizer than {self.optimizer}")
        s = B.raw_stream(stream)
        if muon:
            B.cf_muon_step(self.mats, self.t, hp_matrices, self.param, self.grad, self.momentum, self.w16, self.ws,
                           stream=s)
            v = self.vec0
            B.cf_adam_larc_step(self.vec_offsets, self.t, hp_vectors, self.param[v:], self.grad[v:], self.momentum[v:],
                                self.second, None, self.ws, stream=s)
        else:
            B.cf_adamw_step(self.tensors, self.t, hp_matrices, stream=s)
        self.t += 1


def synthetic(size, batch, widths=inputs.HEAD_WIDTHS, layers=None, features=None, seed=0):
    """Input cubes, He-normal parameters and targets from the simulations' ranges."""
    x = np.stack([inputs.grf_lognormal_poisson(size, seed + i) for i in range(batch)])[..., None]
    cw = [inputs.he_normal(l["k"], l["cin"], l["cout"], seed + 1000 + i) for i, l in enumerate(layers)]
    cb = [np.zeros(l["cout"], np.float32) for l in layers]
    dims = [features, *widths]
    fw = [inputs.normal((dims[i], dims[i + 1]), seed + 2000 + i, (2.0 / dims[i]) ** 0.5) for i in range(len(widths))]
    fb = [np.zeros(n, np.float32) for n in widths]
    rng = np.random.Generator(np.random.PCG64(seed + 3000))
    lo, hi = np.asarray(inputs.PARAM_RANGES).T
    target = rng.uniform(lo, hi, (batch, len(lo))).astype(np.float32)
    return x, cw, cb, fw, fb, target


def main(argv=None):
    ap = argparse.ArgumentParser(description="train the network on synthetic cubes")
    ap.add_argument("--size", type=int, default=64, help="side of the input cubes")
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    ap.add_argument("--norm", choices=("sample", "voxel", "group"), default="sample")
    ap.add_argument("--groups", type=int, default=8, help="of --norm group and --conv-norm")
    ap.add_argument("--conv-norm", choices=("lrelu", "silu", "gelu"), help="group normalisation and this activation in every convolution layer")
    ap.add_argument("--mixer", type=int, default=0, help="hidden values of a block over each voxel's channels")
    ap.add_argument("--optimizer", choices=("muon", "adamw", "adamw8"), default="muon")
    ap.add_argument("--rate", type=float, default=0.002, help="first rate of the matrices, or of all parameters")
    a = ap.parse_args(argv)
    layers = inputs.stack_layers()
    if a.conv_norm:
        layers = [dict(l, norm=math.gcd(l["cout"], a.groups), act=a.conv_norm) for l in layers]
    net = Network(layers, a.size, a.batch, dtype=a.dtype, norm=a.norm, groups=a.groups, mixer=a.mixer,
                  optimizer=a.optimizer)
    x, *params = synthetic(a.size, a.batch, layers=layers, features=net.head.dims[0])
    net.stack.set_input(x)
    net.set_params(*params)
    if a.optimizer == "muon":
        hp = B.make_muon_hparams(a.steps, eta0=a.rate, eta_min=a.rate / 20), B.make_hparams(a.steps)
    else:
        hp = (B.make_adamw_hparams(a.steps, eta0=a.rate, eta_min=a.rate / 20),)
    t0 = None
    for i in range(a.steps):
        loss = net.step()
        net.update(*hp)
        if i == 0 or (i + 1) % 10 == 0 or i + 1 == a.steps:
            print(f"step {i + 1}: loss {float(loss[0]):.6f}", flush=True)
        if i == 0:
            t0 = time.perf_counter()
    if a.steps > 1:
        print(f"{(time.perf_counter() - t0) / (a.steps - 1) * 1e3:.3f} ms a step")


if __name__ == "__main__":
    main()
