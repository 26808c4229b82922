"""Rotary positions where a thread has more heads than it loads at once, on the GPU against their 64-bit form (needs a
GB300): prompts, whose heads a thread goes through in rounds of four.  Tolerance as in the rotary positions' other tests."""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref
from tests.test_gpu_rope import UNITS, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


def check(got, x, pos, rates, plan):
    want, magnitude = ref.rope(x, pos, rates, plan.interleaved, plan.amplitude)
    half = ref.half_step(x.dtype)
    over = ((got.double() - want).abs() / (half * want.abs() + UNITS * ref.UNIT * magnitude * (1 + half) + 1e-37)).nan_to_num(nan=math.inf)
    assert over.max() <= 1, (over.max().item(), over.argmax().item())
    assert torch.equal(got[..., plan.rotary_dim:], x[..., plan.rotary_dim:])


# heads of whole pieces, halves that end off 16 bytes, rows off 16 bytes; 40 heads are shared out evenly, 37 and 11 are not
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("N,Hq,Hk,d,r", [(20000, 37, 3, 16, 16), (20000, 30, 7, 24, 10), (4001, 32, 8, 128, 128), (6007, 12, 11, 80, 74),
                                         (6007, 11, 12, 80, 48), (20011, 9, 2, 33, 18), (1009, 64, 64, 72, 72)])
def test_more_heads_than_are_under_way(N, Hq, Hk, d, r, interleaved, dtype):
    qkv = make((N, Hq + 2 * Hk, d), dtype, N + d)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    gen = torch.Generator(device="cuda").manual_seed(N)
    pos = torch.randint(-1000, 1 << 24, (N,), generator=gen, device="cuda").to(torch.int32)
    plan = fem.Rope(r, interleaved=interleaved, amplitude=1.25)
    out = tuple(torch.full(t.shape, math.nan, dtype=dtype, device="cuda") for t in (q, k))
    for got, x in zip(fem.fem_rope(plan, q, k, positions=pos, out=out), (q, k)):
        check(got, x, pos, ref.rope_rates(r), plan)
    whole, rest = qkv.clone(), qkv[:, Hq + Hk:].clone()
    q, k = whole[:, :Hq], whole[:, Hq:Hq + Hk]
    fem.fem_rope(plan, q, k, positions=pos, out=(q, k))  # in place: the same bits, and nothing else touched
    assert torch.equal(q, out[0]) and torch.equal(k, out[1]) and torch.equal(whole[:, Hq + Hk:], rest)
