"""Rotary positions on the GPU against their 64-bit form (needs a GB300).

Tolerance: the output's half step, and 10 roundings of fp32 of A (|a| + |b|): cosine and sine are off by 4 units at most
and by what the remainder of the turn is rounded (pi/4 units), then come the amplitude (1), each product (1) and their
sum (1); the rates' and positions' part is under a unit for positions below 2^24.
"""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
UNITS = 10


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


def make(shape, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def compare(got, x, pos, rates, plan, inverse=False):
    want, size = ref.rope(x, pos, rates, plan.interleaved, plan.amplitude, inverse)
    ref.check(got, want, size, UNITS)
    r = plan.rotary_dim
    assert torch.equal(got[..., r:], x[..., r:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("N,Hq,Hk,d,r", [(1, 1, 1, 16, 16), (3, 4, 1, 64, 32), (37, 12, 3, 128, 128), (5, 5, 2, 80, 74),
                                         (9, 3, 3, 2, 2), (2, 7, 1, 33, 18), (130, 2, 1, 256, 64), (4, 1, 1, 1024, 1024),
                                         (3, 2, 1, 1023, 1022), (700, 33, 9, 64, 64), (6, 3, 2, 8, 8), (6, 3, 1, 24, 24),
                                         (7, 3, 1, 24, 16), (7, 3, 1, 40, 16), (6, 2, 2, 24, 8)])
def test_rows(N, Hq, Hk, d, r, interleaved, dtype):
    """Queries and keys as views of one projection's output, positions in any order."""
    qkv = make((N, Hq + 2 * Hk, d), dtype, N + d)
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    gen = torch.Generator(device="cuda").manual_seed(N)
    pos = torch.randint(-1000, 1 << 24, (N,), generator=gen, device="cuda").to(torch.int32)
    plan = fem.Rope(r, interleaved=interleaved, amplitude=1.25)
    for inverse in (False, True):
        out = tuple(torch.full(t.shape, math.nan, dtype=dtype, device="cuda") for t in (q, k))
        got = fem.fem_rope(plan, q, k, positions=pos, inverse=inverse, out=out)
        for g, x in zip(got, (q, k)):
            compare(g, x, pos, ref.rope_rates(r), plan, inverse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,T,Hq,Hk,d,r", [(1, 1, 2, 2, 64, 64), (3, 129, 4, 2, 64, 32), (2, 50, 6, 0, 48, 30)])
@pytest.mark.parametrize("scaling", [None, "linear", "base", "parts"])
def test_heads(B, T, Hq, Hk, d, r, dtype, scaling):
    """The read's layout; positions given or counted; every scaling."""
    q = make((B, Hq, T, d), dtype, 1)
    k = make((B, Hk, T, d), dtype, 2) if Hk else None
    plan = fem.Rope(r, base=500.0, scaling=scaling, factor=4.0, context=256.0, low=1.0, high=8.0)
    rates = ref.rope_rates(r, 500.0, scaling, 4.0, 256.0, 1.0, 8.0)
    counted = torch.arange(T, device="cuda").expand(B, T)
    given = (counted * 3 + 100 * torch.arange(B, device="cuda")[:, None]).to(torch.int32).contiguous()
    for pos, arg in ((counted, None), (given, given)):
        got = fem.fem_rope(plan, q, k, positions=arg)
        compare(got[0], q, pos, rates, plan)
        if k is not None:
            compare(got[1], k, pos, rates, plan)
        else:
            assert got[1] is None


def test_far_positions_are_exact():
    """The angle is a 64-bit product: at positions up to 2^28 a rate in doubles is off by less than 2^-24 rad, and
    4 more units of what it turns count."""
    pos = torch.tensor([0, 1, -1, 1 << 24, (1 << 24) + 1, (1 << 28) - 1, -(1 << 28)], dtype=torch.int32, device="cuda")
    x = make((7, 2, 128), torch.float32, 3)
    plan = fem.Rope(128)
    got, _ = fem.fem_rope(plan, x, positions=pos)
    want, size = ref.rope(x, pos, ref.rope_rates(128), False)
    ref.check(got, want, size, UNITS + 4)


def test_there_and_back():
    """Twice 10 units of the pair, whose length a rotation keeps: sqrt(2) for |a| + |b| each way."""
    x = make((40, 3, 64), torch.float32, 4)
    plan = fem.Rope(64, interleaved=True)
    y, _ = fem.fem_rope(plan, x)
    z, _ = fem.fem_rope(plan, y, inverse=True)
    _, size = ref.rope(x, torch.arange(40, device="cuda"), ref.rope_rates(64), True)
    ref.check(z, x, 2 * size, 2 * UNITS)


@pytest.mark.parametrize("d,r,interleaved", [(64, 64, False), (64, 32, True), (40, 22, False)])
def test_in_place_and_odd_views(d, r, interleaved):
    """In place, at addresses and strides that are not multiples of 16 bytes, the same bits as out of place; what lies
    around the view stays."""
    plan = fem.Rope(r, interleaved=interleaved)
    for lead in (0, 1, 8):
        whole = make((6, 5, d + 11), torch.bfloat16, 5)
        q, k = whole[1:5, :3, lead:lead + d], whole[1:5, 3:4, lead:lead + d]
        want = fem.fem_rope(plan, q.contiguous(), k.contiguous())
        before = whole.clone()
        got = fem.fem_rope(plan, q, k, out=(q, k))
        assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
        before[1:5, :3, lead:lead + d], before[1:5, 3:4, lead:lead + d] = q, k
        assert torch.equal(whole, before)


def test_infinities_and_nan_stay_in_their_pairs():
    x = make((4, 2, 64), torch.float32, 6)
    clean, _ = fem.fem_rope(fem.Rope(64), x)
    x[1, 0, 5], x[2, 1, 40] = math.inf, math.nan
    got, _ = fem.fem_rope(fem.Rope(64), x)
    touched = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    touched[1, 0, [5, 37]] = touched[2, 1, [8, 40]] = True
    assert torch.equal(got[~touched], clean[~touched])
    assert not torch.isfinite(got[touched]).any()


def test_empty_calls():
    plan = fem.Rope(16)
    got = fem.fem_rope(plan, torch.empty((0, 2, 16), device="cuda"), torch.empty((0, 1, 16), device="cuda"))
    assert got[0].shape == (0, 2, 16) and got[1].shape == (0, 1, 16)


def test_offsets_past_32_bits():
    """A token stride of 2^31 + 8 elements."""
    step = (1 << 31) + 8
    whole = torch.empty(step + 2 * 64, dtype=torch.bfloat16, device="cuda")
    q = whole.as_strided((2, 2, 64), (step, 64, 1))
    q.copy_(make((2, 2, 64), torch.bfloat16, 7))
    pos = torch.tensor([3, 5], dtype=torch.int32, device="cuda")
    want, _ = fem.fem_rope(fem.Rope(64), q.contiguous(), positions=pos)
    got, _ = fem.fem_rope(fem.Rope(64), q, positions=pos, out=(q, None))
    assert torch.equal(got, want)


def test_streams_and_graphs():
    """Another stream's outputs are its own memory; a captured call follows its inputs."""
    plan = fem.Rope(64)
    q, k = make((50, 4, 64), torch.bfloat16, 8), make((50, 2, 64), torch.bfloat16, 9)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    want = fem.fem_rope(plan, q, k, positions=pos)
    side = torch.cuda.Stream()
    late = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for t in late:
        t.fill_(7)
    del late, t
    got = fem.fem_rope(plan, q, k, positions=pos, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))

    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kept = fem.fem_rope(plan, q, k, positions=pos)
    pos += 11
    q.neg_()
    graph.replay()
    torch.cuda.synchronize()
    want = fem.fem_rope(plan, q, k, positions=pos)
    assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_refusals():
    plan = fem.Rope(64)
    q, k = make((4, 2, 64), torch.bfloat16, 10), make((4, 1, 64), torch.bfloat16, 11)
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (dict(q=q.half()), dict(q=q[0]), dict(k=k.float()), dict(k=k[:3]), dict(k=k[..., :32]), dict(positions=pos.long()),
                dict(positions=pos[:3]), dict(q=q.transpose(0, 2)), dict(out=(q[:3], k)), dict(out=(q, k[..., :8]))):
        with pytest.raises(ValueError):
            fem.fem_rope(plan, **{**dict(q=q, k=k, positions=pos), **bad})
    with pytest.raises(fem.FemError):
        fem.fem_rope(plan, q[..., :32], k[..., :32])  # fewer elements than turn
    with pytest.raises(fem.FemError):
        fem.fem_rope(plan, q, out=(q[:1].expand(4, 2, 64), None))  # one address for four rows
