"""Parameters that a caller hands to the stack and the head: what does not fit is refused
before anything is taken, what fits is used as it is (no kernel is launched)."""
import os

import pytest
import torch

from paper_1808_04728_amd import binding as B
from paper_1808_04728_amd import inputs
from paper_1808_04728_amd.head import FCHead
from paper_1808_04728_amd.stack import ConvStack

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libcosmoflow_hip.so not built")


def head(dtype="bf16"):
    h = FCHead(2, 64, (16, 8, 3), dtype=dtype, device="cpu")
    return h, [dict(w=h.w[i], b=h.b[i], dw=h.dw[i], db=h.db[i]) for i in range(3)]


def stack(dtype="bf16"):
    s = ConvStack(inputs.stack_layers(), 32, 1, dtype=dtype, device="cpu", overlap_wgrad=False)
    return s, [{k: l[k] for k in ("w", "w32", "b", "dw", "db")} for l in s.L]


def fresh(own):
    return [{k: torch.zeros_like(t) for k, t in p.items()} for p in own]


@pytest.mark.parametrize("make", [head, stack])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_taken_as_they_are(make, dtype):
    net, own = make(dtype)
    ps = fresh(own)
    net.bind_params(ps)
    now = [dict(w=net.w[i], b=net.b[i], dw=net.dw[i], db=net.db[i]) for i in range(3)] if make is head else net.L
    assert all(now[i][k] is ps[i][k] for i in range(len(ps)) for k in ps[i])


def unaligned(t):
    return torch.zeros(t.numel() + 1, dtype=t.dtype)[1:].view(t.shape)


BAD = {
    "short list": lambda ps: ps.pop(),
    "long list": lambda ps: ps.append(ps[-1]),
    "missing": lambda ps: ps[-1].pop("db"),
    "shape": lambda ps: ps[-1].update(dw=ps[-1]["dw"].unsqueeze(0)),
    "dtype": lambda ps: ps[-1].update(w=ps[-1]["w"].double()),
    "strides": lambda ps: ps[-1].update(b=torch.zeros(2 * ps[-1]["b"].numel())[::2]),
    "alignment": lambda ps: ps[-1].update(w=unaligned(ps[-1]["w"])),
    "gradient's alignment": lambda ps: ps[1].update(dw=unaligned(ps[1]["dw"])),
    "device": lambda ps: ps[0].update(b=ps[0]["b"].to("meta")),
    "not a tensor": lambda ps: ps[0].update(b=None),
}


@pytest.mark.parametrize("make", [head, stack])
@pytest.mark.parametrize("bad", sorted(BAD))
def test_refused_before_any_is_taken(make, bad):
    net, own = make()
    ps = fresh(own)
    BAD[bad](ps)
    with pytest.raises(ValueError):
        net.bind_params(ps)
    now = [dict(w=net.w[i], b=net.b[i], dw=net.dw[i], db=net.db[i]) for i in range(3)] if make is head else net.L
    assert all(now[i][k] is own[i][k] for i in range(len(own)) for k in own[i])
    if make is stack:
        assert net.flat_param is not None
