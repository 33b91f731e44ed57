"""The list of an AdamW call lies on one device: what make_adamw_tensors refuses."""
import pytest
import torch

from paper_1808_04728_amd import binding as B


def entry(device, n=300, eight=False):
    z = lambda k, t=torch.float32: torch.zeros(k, dtype=t, device=device)  # noqa: E731
    d = dict(p=z(n), g=z(n), m=z(n), v=z(n))
    if eight:
        d.update(m=z(n, torch.uint8), v=z(n, torch.uint8), m_scale=z(2), v_scale=z(2))
    return d


@pytest.mark.parametrize("eight", [False, True])
def test_list_over_two_devices(eight):
    here, there = entry("cpu", eight=eight), entry("meta", eight=eight)
    assert B.make_adamw_tensors([here, entry("cpu", 5)])[0] == 2
    for tensors in ([here, there], [there, here], [here, here, there], [here, dict(here, p=there["p"])],
                    [dict(here, p16=torch.zeros(300, dtype=torch.bfloat16, device="meta"))]):
        with pytest.raises(ValueError, match="on meta|on cpu"):
            B.make_adamw_tensors(tensors)
