"""What limits the gated recurrence on the GPU: slow rates, and states that are not finite (needs a GB300)."""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests.test_gpu_recur import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


@pytest.mark.parametrize("rate,S,T,C", [(1e-4, 1, 40000, 64), (1e-4, 64, 20000, 512), (1e-5, 1, 200000, 64)])
@pytest.mark.parametrize("mean", [False, True])
def test_slow_rates(rate, S, T, C, mean):
    """A constant input over more than one horizon, or two, in chunks and whole lines.  With r = e^-s every state is
    w (1 - r^t) / (1 - r), w = 1 - r where `mean`.  A decay is off by 2^-25, a composed one by its rounding more, up to 2^-24, and a
    state by its own: 5 2^-25 a step, of which 1 / s count."""
    s = torch.full((S, T, C), rate, device="cuda")
    exact = s[0, 0, 0].double().item()  # as fp32 has it
    h, last = fem.fem_recur_fwd(s, torch.ones_like(s), mean=mean)
    steps = torch.arange(1, T + 1, device="cuda", dtype=torch.float64)[:, None]
    want = -torch.expm1(-exact * steps) / (1.0 if mean else -math.expm1(-exact))
    worst = max(((x.double() - want).abs() / want).max().item() for x in h)
    worst = max(worst, ((last.double() - want[-1]).abs() / want[-1]).max().item())
    assert worst <= 5 * 2.0 ** -25 / exact + 2.0 ** -20


@pytest.mark.parametrize("S,T,C", [(2, 8, 64), (2, 700, 64), (2, 700, 63), (64, 700, 512), (3, 700, 14)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_state_that_is_not_finite_stays_so(S, T, C, dtype, value):
    """However a sequence is cut, through decays whose product is 0 and a rate of infinity; the others keep their bits."""
    s, u, dh = (x.view(S, T, C) for x in make(S * T, C, dtype, T + C, rate=3.0))
    s[1, T // 2, 3] = math.inf
    clean, _ = fem.fem_recur_fwd(s, u)
    u[1, 2, 3] = value
    h, last = fem.fem_recur_fwd(s, u)
    touched = torch.zeros(h.shape, dtype=torch.bool, device="cuda")
    touched[1, 2:, 3] = True
    assert not h[touched].isfinite().any() and not last[1, 3].isfinite() and torch.equal(h[~touched], clean[~touched])
    dh[1, T - 3, 3] = value
    ds, du, _ = fem.fem_recur_bwd(s, u, clean, dh)
    assert not du[1, :T - 2, 3].isfinite().any() and du[1, T - 2:, 3].isfinite().all()
    assert ds[:, :, torch.arange(C, device="cuda") != 3].isfinite().all() and du[0].isfinite().all()
