"""The whole network as it trains: convolution stack, layer normalisation of its
output, fully-connected head, and one update of all parameters.

  forward   stack -> layer normalisation -> head -> loss
  backward  head -> layer normalisation -> stack
  update    matrices (convolution and fully-connected weights): momentum with
            orthogonalised steps, one cf_muon_step call; vectors (biases, the
            normalisation's gamma and beta): Adam + LARC, one cf_adam_larc_step call

The normalisation runs over a sample's whole output (``norm="sample"``: batch rows of
d*h*w*c values) or over the channels of each voxel (``norm="voxel"``: batch*d*h*w
rows of c).  The head then sees inputs of one scale whatever the updates do to the
convolutions.

All parameters live in flat buffers, matrices first and vectors after them, each on
a multiple of 16 elements: fp32 values, fp32 gradients, and for a bf16 network the
bf16 weights that the products read.

``python -m paper_1808_04728_amd.network`` trains on synthetic cubes.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

from . import binding as B
from . import inputs
from .head import FCHead
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
                 device="cuda"):
        if norm not in ("sample", "voxel"):
            raise ValueError(f"norm: {norm}")
        self.dtype = dtype
        self.stack = ConvStack(layers, size, batch, dtype=dtype, alpha=alpha, device=device)
        out = self.stack.output()
        features = out.numel() // batch
        self.rows, self.c = (batch, features) if norm == "sample" else (out.numel() // out.shape[-1], out.shape[-1])
        self.head = FCHead(batch, features, widths, dtype=dtype, alpha=alpha, device=device)
        self._alloc_params(device)
        self.y = torch.empty((batch, features), dtype=out.dtype, device=device)
        self.dout = torch.empty_like(out)
        self.mean = torch.empty(self.rows, dtype=torch.float32, device=device)
        self.rstd = torch.empty_like(self.mean)
        nws = max(16, B.cf_layernorm_fwd_workspace_size(self.rows, self.c, dtype),
                  B.cf_layernorm_bwd_workspace_size(self.rows, self.c, dtype), B.cf_muon_workspace_size(self.mats),
                  B.cf_adam_larc_workspace_size(self.vec_offsets))
        self.ws = torch.empty(nws, dtype=torch.uint8, device=device)
        self.t = 0

    def _alloc_params(self, device):
        shapes = [tuple(l["w32"].shape) for l in self.stack.L] + [tuple(w.shape) for w in self.head.w]
        vectors = [l["b"].numel() for l in self.stack.L] + [b.numel() for b in self.head.b] + [self.c, self.c]
        off = layout([int(np.prod(s)) for s in shapes] + vectors)
        nm = len(shapes)
        self.vec0 = off[nm]
        self.vec_offsets = B.adam_offsets([o - self.vec0 for o in off[nm:]])
        # a convolution's weights are the matrix of its taps and inputs by its outputs
        self.mats = B.make_matrices(off[:nm], [int(np.prod(s[:-1])) for s in shapes], [s[-1] for s in shapes])
        self.param = torch.zeros(off[-1], dtype=torch.float32, device=device)
        self.grad = torch.zeros_like(self.param)
        self.momentum = torch.zeros_like(self.param)  # of matrices, and Adam's first moment
        self.second = torch.zeros(off[-1] - self.vec0, dtype=torch.float32, device=device)
        self.w16 = torch.zeros(self.vec0, dtype=torch.bfloat16, device=device) if self.dtype == "bf16" else None

        def view(buf, i):
            n = int(np.prod(shapes[i])) if i < nm else vectors[i - nm]
            return buf[off[i]:off[i] + n].view(shapes[i] if i < nm else (n,))

        ps = [dict(w=view(self.w16 if self.w16 is not None else self.param, i), w32=view(self.param, i),
                   b=view(self.param, nm + i), dw=view(self.grad, i), db=view(self.grad, nm + i)) for i in range(nm)]
        nl = len(self.stack.L)
        self.stack.bind_params(ps[:nl])
        self.head.bind_params(ps[nl:])
        self._head_params = ps[nl:]
        self.gamma, self.beta = view(self.param, 2 * nm), view(self.param, 2 * nm + 1)
        self.dgamma, self.dbeta = view(self.grad, 2 * nm), view(self.grad, 2 * nm + 1)
        self.gamma.fill_(1.0)

    def set_params(self, conv_weights, conv_biases, fc_weights, fc_biases, target):
        """Weights are rounded to the network's dtype, their fp32 values hold exactly those;
        gamma = 1, beta = 0; resets the optimizer state."""
        self.stack.set_params(conv_weights, conv_biases)
        self.head.set_params(fc_weights, fc_biases, target)
        for p in self._head_params:
            p["w32"].copy_(p["w"].float())
        self.gamma.fill_(1.0)
        self.beta.zero_()
        self.momentum.zero_()
        self.second.zero_()
        self.t = 0

    def step(self, stream=None):
        """Forward and backward of the stack's input (stack.set_input) and the head's target:
        fills every gradient; returns the device loss tensor (one fp32 in element 0)."""
        s = B.raw_stream(stream)
        x = self.stack.forward(stream)
        B.cf_layernorm_fwd(self.rows, self.c, self.dtype, x, self.gamma, self.beta, NORM_EPS, self.y, self.mean,
                           self.rstd, self.ws, stream=s)
        dy = self.head.step(self.y, stream)
        B.cf_layernorm_bwd(self.rows, self.c, self.dtype, dy, x, self.gamma, self.mean, self.rstd, self.dout,
                           self.dgamma, self.dbeta, self.ws, stream=s)
        self.stack.backward(self.dout, stream)
        return self.head.loss

    def update(self, hp_matrices, hp_vectors, stream=None):
        """One update of all parameters from the gradients of the last step
        (binding.make_muon_hparams, binding.make_hparams)."""
        s = B.raw_stream(stream)
        B.cf_muon_step(self.mats, self.t, hp_matrices, self.param, self.grad, self.momentum, self.w16, self.ws, stream=s)
        v = self.vec0
        B.cf_adam_larc_step(self.vec_offsets, self.t, hp_vectors, self.param[v:], self.grad[v:], self.momentum[v:],
                            self.second, None, self.ws, stream=s)
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
    ap.add_argument("--norm", choices=("sample", "voxel"), default="sample")
    ap.add_argument("--rate", type=float, default=0.002, help="first rate of the matrices")
    a = ap.parse_args(argv)
    layers = inputs.stack_layers()
    net = Network(layers, a.size, a.batch, dtype=a.dtype, norm=a.norm)
    x, *params = synthetic(a.size, a.batch, layers=layers, features=net.head.dims[0])
    net.stack.set_input(x)
    net.set_params(*params)
    hm, hv = B.make_muon_hparams(a.steps, eta0=a.rate, eta_min=a.rate / 20), B.make_hparams(a.steps)
    t0 = None
    for i in range(a.steps):
        loss = net.step()
        net.update(hm, hv)
        if i == 0 or (i + 1) % 10 == 0 or i + 1 == a.steps:
            print(f"step {i + 1}: loss {float(loss[0]):.6f}", flush=True)
        if i == 0:
            t0 = time.perf_counter()
    if a.steps > 1:
        print(f"{(time.perf_counter() - t0) / (a.steps - 1) * 1e3:.3f} ms a step")


if __name__ == "__main__":
    main()
