"""Norms on the GPU where values leave the ordinary range: gates far from 0 (needs a GB300).

Tolerances as in the norms' other tests.  A sigmoid below 2^-126 is 0 in fp32: a SiLU gate below -87 is off by less than
2^-126 times 90, the largest |g| of which the product with an unrounded sigmoid still is above 2^-132.
"""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref
from tests.test_gpu_norm import BWD, check_forward, make

pytestmark = pytest.mark.gpu
TINY = 90 * 2.0 ** -126


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("types", ["bf16", "mixed", "f32"])
@pytest.mark.parametrize("D", [256, 203])
def test_gates_far_from_zero(D, types, act):
    """To the lowest and largest number of the type: a gate is 0 on one side, 1 or itself on the other."""
    block, t = make(12, D, types, "rms", "none", act, 1)
    lowest = torch.finfo(t["gate"].dtype).min
    for row, value in enumerate((lowest, -1e30, -1e6, -500.0, -100.0, -90.0, -88.0, -87.0, -60.0, 60.0, 1e6)):
        t["gate"][row, ::2] = value
    if act == "sigmoid":
        t["gate"][11, ::2] = -lowest
        t["gate"][10, ::3] = -math.inf
        t["gate"][9, ::3] = math.inf
    r, _ = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    check_forward(block, t, r, None)
    got = fem.fem_norm_bwd(block, r, t["y"], t["gate"], t["dr"])
    assert all(got[i].isfinite().all() for i in (0, 1, 3))
    # dgate = e act'(gate), e = scale dr w N(y); what a slope is off by counts by the magnitudes that it is summed from
    g, e = t["gate"].double(), block.scale * t["dr"].double() * ref._norm(t["y"].double(), "rms", block.eps) * block.weights["w_post"].double()
    p, q = torch.sigmoid(g), torch.sigmoid(-g)
    slope, size = (p * q, p * q) if act == "sigmoid" else (p + g * p * q, p * (1 + g.abs() * q))
    fine = g.isfinite()
    off = (got[2].double() - e * slope).abs()
    allowed = ref.half_step(t["gate"].dtype) * (e * slope).abs() + BWD * ref.UNIT * (e * size).abs() * 2 + TINY * e.abs()
    assert (off <= allowed)[fine].all()
    if act == "silu":
        assert torch.equal(r[0, ::2], t["x"][0, ::2])
