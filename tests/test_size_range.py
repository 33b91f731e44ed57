"""Sizes that do not fit the 32 bits of their C argument are refused by the binding, not cut to
their low bits, which may be a size that the call takes (no kernel is launched)."""
import os

import pytest

from paper_1808_04728_amd import binding as B

A = 0x7F0000000000  # fake, 16-byte aligned device addresses (never dereferenced)
M = 1 << 24

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libcosmoflow_hip.so not built")

P = [A + i * M for i in range(9)]
GROUPNORM = [
    lambda n, c, g: B.cf_groupnorm_fwd_workspace_size(n, 5000, c, g, "f32"),
    lambda n, c, g: B.cf_groupnorm_bwd_workspace_size(n, 5000, c, g, "f32"),
    # (without a workspace: a call of cut sizes would be refused for that, and not run)
    lambda n, c, g: B.cf_groupnorm_fwd(n, 5000, c, g, "f32", *P[:3], 1e-5, "none", 0.0, *P[3:6], None, 0, 0),
    lambda n, c, g: B.cf_groupnorm_bwd(n, 5000, c, g, "f32", *P[:6], "none", 0.0, *P[6:9], None, 0, 0),
]
LINEAR = [
    lambda m, k, n: B.cf_linear_fwd_workspace_size(m, k, n, "f32"),
    lambda m, k, n: B.cf_linear_bwd_data_workspace_size(m, k, n, "f32"),
    lambda m, k, n: B.cf_linear_bwd_weight_workspace_size(m, k, n, "f32"),
    lambda m, k, n: B.cf_linear_fwd(m, k, n, "f32", P[0], P[1], None, "none", 0.0, None, P[2], None, None, 0, 0),
    lambda m, k, n: B.cf_linear_bwd_data(m, k, n, "f32", P[0], P[1], None, None, "none", 0.0, P[2], None, 0, 0),
    lambda m, k, n: B.cf_linear_bwd_weight(m, k, n, "f32", *P[:4], None, 0, 0),
]


@pytest.mark.parametrize("calls,sizes", [(GROUPNORM, (2, 48, 6)), (LINEAR, (40, 2048, 1024)), (LINEAR, (40, 2048, 2048))])
def test_past_32_bits(calls, sizes):
    for call in calls:
        for i in range(3):
            for more in (1 << 32, -1 << 32, 3 << 40, 1 << 31):
                bad = list(sizes)
                bad[i] += more
                with pytest.raises(ValueError, match="past 32 bits"):
                    call(*bad)
