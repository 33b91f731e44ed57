"""A residual block over the channels of every voxel, driven through the C ABI.

  forward   y = x + gelu(x W1 + b1) W2 + b2, rows of c channels through `hidden` values
  backward  dz1 = (dy W2^T) gelu'(z1);  dx = dy + dz1 W1^T;  dW, db of both products

Two products forward and four backward, each one ``binding`` call that applies bias,
activation, its slope and the residual sum as it writes.  PyTorch allocates the buffers
once and supplies the stream.
"""
from __future__ import annotations

import torch

from . import binding as B


def _t(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class ChannelMixer:
    def __init__(self, rows, c, hidden, dtype="f32", device="cuda"):
        if hidden < 1:
            raise ValueError(f"hidden: {hidden}")
        self.rows, self.c, self.hidden, self.dtype = rows, c, hidden, dtype
        t = _t(dtype)
        shapes = [(c, hidden), (hidden, c)]
        self.w = [torch.zeros(s, dtype=t, device=device) for s in shapes]
        self.b = [torch.zeros(s[1], dtype=torch.float32, device=device) for s in shapes]
        self.dw = [torch.empty(s, dtype=torch.float32, device=device) for s in shapes]
        self.db = [torch.empty(s[1], dtype=torch.float32, device=device) for s in shapes]
        self.z = torch.empty((rows, hidden), dtype=t, device=device)  # in front of the activation
        self.a = torch.empty_like(self.z)
        self.dz = torch.empty_like(self.z)
        self.y = torch.empty((rows, c), dtype=t, device=device)
        self.dx = torch.empty_like(self.y)
        ws = max(f(rows, k, n, dtype) for k, n in shapes
                 for f in (B.cf_linear_fwd_workspace_size, B.cf_linear_bwd_data_workspace_size,
                           B.cf_linear_bwd_weight_workspace_size))
        self.ws = torch.empty(max(ws, 16), dtype=torch.uint8, device=device)
        self.x = None

    def bind_params(self, params):
        """Use the caller's tensors for the parameters and their gradients: one dict of w (the
        block's dtype), b, dw and db (fp32) a product, in the shapes of the block's own,
        contiguous and 16-byte aligned (ValueError)."""
        B.check_params([dict(w=w, b=b, dw=dw, db=db) for w, b, dw, db in zip(self.w, self.b, self.dw, self.db)], params)
        for k in ("w", "b", "dw", "db"):
            setattr(self, k, [p[k] for p in params])

    def set_params(self, weights, biases):
        for i, (w, b) in enumerate(zip(weights, biases)):
            self.w[i].copy_(torch.as_tensor(w, dtype=torch.float32).to(self.w[i].dtype))
            self.b[i].copy_(torch.as_tensor(b, dtype=torch.float32))

    def forward(self, x, stream=None):
        """x: rows * c values of the block's dtype, contiguous; kept for backward.  Returns y."""
        assert x.is_contiguous() and x.numel() == self.rows * self.c and x.dtype == self.y.dtype
        self.x = x
        m, c, h = self.rows, self.c, self.hidden
        B.cf_linear_fwd(m, c, h, self.dtype, x, self.w[0], self.b[0], "gelu", 0.0, None, self.a, self.z, self.ws,
                        stream=stream)
        B.cf_linear_fwd(m, h, c, self.dtype, self.a, self.w[1], self.b[1], "none", 0.0, x, self.y, None, self.ws,
                        stream=stream)
        return self.y

    def backward(self, dy, stream=None):
        """dy: gradient of y (not modified).  Fills dw and db, returns the gradient of x."""
        assert dy.is_contiguous() and dy.numel() == self.rows * self.c and dy.dtype == self.y.dtype
        m, c, h = self.rows, self.c, self.hidden
        B.cf_linear_bwd_weight(m, h, c, self.dtype, self.a, dy, self.dw[1], self.db[1], self.ws, stream=stream)
        B.cf_linear_bwd_data(m, h, c, self.dtype, dy, self.w[1], None, self.z, "gelu", 0.0, self.dz, self.ws,
                             stream=stream)
        B.cf_linear_bwd_weight(m, c, h, self.dtype, self.x, self.dz, self.dw[0], self.db[0], self.ws, stream=stream)
        B.cf_linear_bwd_data(m, c, h, self.dtype, self.dz, self.w[0], dy, None, "none", 0.0, self.dx, self.ws,
                             stream=stream)
        return self.dx
