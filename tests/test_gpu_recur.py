"""The gated recurrence and its gradients on the GPU against their 64-bit forms (needs a GB300).

Tolerance: the output's half step, and 28 roundings of fp32 of the magnitudes that the reference sums with the decayed
errors of the steps before.  A step's decay is off by at most 2 units; its w by up to 21 (just above a rate of 1/8, where
e^(-s) is off by 2 ulp and its rounded exponent by a quarter, 2.3 units of 1, and w is 0.1175 and rounded once more), w u by
one more and the sum by one; joining stretches multiplies decays, 1 unit a step, and adds once more.  (A decay far from 1
is off by s units more of itself, and s e^(-s) is less than a unit.)
"""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
UNITS = 28


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


def make(n, c, dtype, seed, rate=0.3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = rate * torch.nn.functional.softplus(torch.randn((n, c), generator=gen, device="cuda") * 2)
    return s.to(dtype), *(torch.randn((n, c), generator=gen, device="cuda").to(dtype) for _ in range(2))


def states(seqs, c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((seqs, c), generator=gen, device="cuda") for _ in range(2)]


def offsets_of(lens, first=0):
    got = [first]
    for n in lens:
        got.append(got[-1] + n)
    return torch.tensor(got, dtype=torch.int32, device="cuda")


CASES = [([1], 1), ([1] * 65, 64), ([5], 3), ([16, 17], 130), ([31, 33, 0, 1, 2], 64), ([127], 66), ([128, 129], 32),
         ([500, 3], 100), ([0, 0, 7], 8), ([1000], 257), ([2500, 40, 0, 700], 72), ([4100], 33), ([2000, 30], 8), ([1300, 30], 24),
         ([150] * 70 + [600, 0], 256), ([90] * 20, 2000)]


@pytest.mark.parametrize("lens,c", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mean", [False, True])
def test_packed(lens, c, dtype, mean):
    """Forward and backward with states; outputs are poisoned beforehand."""
    n = sum(lens)
    s, u, dh = make(n, c, dtype, n + c)
    h0, dl = states(len(lens), c, c)
    off = offsets_of(lens)
    out = torch.full_like(s, math.nan)
    last = torch.full_like(h0, math.nan)
    h, last = fem.fem_recur_fwd(s, u, offsets=off, max_len=max(lens), h0=h0, mean=mean, out=out, state_out=last)
    want, want_last, hm, lm = ref.recur(s.cpu(), u.cpu(), lens, h0.cpu(), mean)
    ref.check(h, want, hm, UNITS)
    ref.check(last, want_last, lm, UNITS)
    got = fem.fem_recur_bwd(s, u, h, dh, offsets=off, max_len=max(lens), h0=h0, dstate=dl, mean=mean)
    grads, sizes = ref.recur_grads(s.cpu(), u.cpu(), h.cpu(), dh.cpu(), lens, h0.cpu(), dl.cpu(), mean)
    for g, w, m in zip(got, grads, sizes):
        ref.check(g, w, m, UNITS)
    fem.check_device_error()


@pytest.mark.parametrize("B,T,C", [(1, 1, 16), (3, 40, 64), (2, 300, 40), (1, 5000, 64), (40, 130, 256)])
@pytest.mark.parametrize("mean", [False, True])
def test_batches(B, T, C, mean):
    """[B, T, C] as a part of a projection's output, without states."""
    wide = torch.empty((B, T, 2 * C + 8), device="cuda")
    s, u, dh = (x.view(B, T, C) for x in make(B * T, C, torch.float32, T))
    wide[..., :C], wide[..., C + 8:] = s, u
    h, last = fem.fem_recur_fwd(wide[..., :C], wide[..., C + 8:], mean=mean)
    lens = [T] * B
    flat = lambda x: x.reshape(B * T, C).cpu()  # noqa: E731
    want, want_last, hm, lm = ref.recur(flat(s), flat(u), lens, None, mean)
    ref.check(h.view(B * T, C), want, hm, UNITS)
    ref.check(last, want_last, lm, UNITS)
    ds, du, dh0 = fem.fem_recur_bwd(wide[..., :C], wide[..., C + 8:], h, dh, mean=mean)
    assert dh0 is None
    grads, sizes = ref.recur_grads(flat(s), flat(u), flat(h), flat(dh), lens, None, None, mean)
    ref.check(ds.view(B * T, C), grads[0], sizes[0], UNITS)
    ref.check(du.view(B * T, C), grads[1], sizes[1], UNITS)


@pytest.mark.parametrize("c,width", [(64, 67), (63, 64), (7, 9)])
def test_odd_strides(c, width):
    """Rows whose starts are not aligned: the same values as contiguous ones, and nothing written between them."""
    s, u, _ = make(200, c, torch.bfloat16, c)
    wide = [torch.zeros((200, width), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    views = [w[:, 1:1 + c] for w in wide]
    views[0].copy_(s), views[1].copy_(u)
    wide[2].fill_(3)
    off = offsets_of([150, 50])
    h, last = fem.fem_recur_fwd(views[0], views[1], offsets=off, max_len=150, out=views[2])
    want, want_last, hm, lm = ref.recur(s.cpu(), u.cpu(), [150, 50])
    ref.check(h, want, hm, UNITS)
    ref.check(last, want_last, lm, UNITS)
    assert (wide[2][:, 0] == 3).all() and (wide[2][:, 1 + c:] == 3).all()


@pytest.mark.parametrize("mean", [False, True])
def test_near_and_far_rates(mean):
    """No decay at all, decays to nothing, a reset by an infinite rate."""
    n, c = 700, 64
    _, u, _ = make(n, c, torch.float32, 1)
    s = torch.zeros((n, c), device="cuda")
    s[:, 16:32] = 200.0
    s[:, 32:48] = 1e-6
    s[350, 48:] = math.inf
    h, last = fem.fem_recur_fwd(s, u, offsets=offsets_of([n]), max_len=n, mean=mean)
    want, _, hm, _ = ref.recur(s.cpu(), u.cpu(), [n], None, mean)
    ref.check(h, want, hm, UNITS)


def test_nan_stays_in_its_channel_and_sequence():
    s, u, _ = make(600, 64, torch.float32, 2)
    off = offsets_of([300, 300])
    clean, _ = fem.fem_recur_fwd(s, u, offsets=off, max_len=300)
    u[100, 5] = math.nan
    u[310, 9] = math.inf
    h, _ = fem.fem_recur_fwd(s, u, offsets=off, max_len=300)
    touched = torch.zeros(h.shape, dtype=torch.bool, device="cuda")
    touched[100:300, 5] = touched[310:, 9] = True
    assert torch.equal(h[~touched], clean[~touched])
    assert h[100:300, 5].isnan().all() and not h[310:, 9].isfinite().any()


def test_lengths_beyond_max_len_are_right():
    lens = [3000, 10, 500]
    s, u, dh = make(sum(lens), 64, torch.float32, 3)
    off = offsets_of(lens)
    want, _, hm, _ = ref.recur(s.cpu(), u.cpu(), lens)
    for bound in (0, 1, 100, 100000, None):
        h, _ = fem.fem_recur_fwd(s, u, offsets=off, max_len=bound)
        ref.check(h, want, hm, UNITS)
        ds, du, _ = fem.fem_recur_bwd(s, u, h, dh, offsets=off, max_len=bound)
        grads, sizes = ref.recur_grads(s.cpu(), u.cpu(), h.cpu(), dh.cpu(), lens)
        ref.check(ds, grads[0], sizes[0], UNITS)
        ref.check(du, grads[1], sizes[1], UNITS)


@pytest.mark.parametrize("steps", [1, 40])
def test_a_pool_of_states(steps):
    """States in place in a pool, a sequence without one, rows of the pool that no sequence has; a long pass and its
    parts agree."""
    lens, c = [steps] * 4, 96
    n = sum(lens)
    s, u, _ = make(n, c, torch.bfloat16, 4)
    pool = states(9, c, 5)[0]
    rows = torch.tensor([7, -1, 0, 3], dtype=torch.int32, device="cuda")
    before, off = pool.clone(), offsets_of(lens)
    h0 = torch.zeros((4, c), device="cuda")
    h0[[0, 2, 3]] = before[[7, 0, 3]]
    want, want_last, hm, lm = ref.recur(s.cpu(), u.cpu(), lens, h0.cpu())
    h, got = fem.fem_recur_fwd(s, u, offsets=off, max_len=steps, h0=pool, state_rows=rows)
    assert got is pool
    ref.check(h, want, hm, UNITS)
    ref.check(pool[[7, 0, 3]], want_last[[0, 2, 3]], lm[[0, 2, 3]], UNITS)
    others = [1, 2, 4, 5, 6, 8]
    assert torch.equal(pool[others], before[others])
    # the same from outside: states kept apart
    kept = torch.zeros_like(pool)
    h2, _ = fem.fem_recur_fwd(s, u, offsets=off, max_len=steps, h0=before, state_rows=rows, state_out=kept)
    assert torch.equal(h2, h) and torch.equal(kept[[7, 0, 3]], pool[[7, 0, 3]]) and not kept[others].any()


def test_token_by_token_is_the_whole():
    """Serving: one step of every sequence a call, states in place."""
    S, T, c = 5, 60, 128
    s, u, _ = (x.view(S, T, c) for x in make(S * T, c, torch.float32, 6))
    pool = torch.zeros((S, c), device="cuda")
    one = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    rows = torch.arange(S, dtype=torch.int32, device="cuda")
    got = torch.stack([fem.fem_recur_fwd(s[:, t].contiguous(), u[:, t].contiguous(), offsets=one, max_len=1, h0=pool,
                                         state_rows=rows)[0] for t in range(T)], 1)
    want, _, hm, _ = ref.recur(s.reshape(-1, c).cpu(), u.reshape(-1, c).cpu(), [T] * S)
    ref.check(got.view(-1, c), want, hm, UNITS)


def test_rows_of_no_sequence_stay():
    s, u, dh = make(100, 64, torch.bfloat16, 7)
    off = offsets_of([20, 30], first=10)
    out = torch.full_like(s, 5.0)
    fem.fem_recur_fwd(s, u, offsets=off, max_len=30, out=out)
    assert (out[:10] == 5).all() and (out[60:] == 5).all()
    want, *_ = fem.fem_recur_fwd(s[10:60].contiguous(), u[10:60].contiguous(), offsets=off - 10, max_len=30)
    assert torch.equal(out[10:60], want)


def test_indices_outside_are_left_out_and_recorded():
    """The kernels compare every offset and state row with its array before they use it."""
    s, u, dh = make(40, 64, torch.float32, 8)
    want, _ = fem.fem_recur_fwd(s, u, offsets=offsets_of([20, 20]), max_len=20)
    for bad in ([0, 20, 41], [0, 20, 10], [-1, 20, 40], [30, 20, 40], [0, 20, 1 << 30]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        out = torch.zeros_like(s)
        fem.fem_recur_fwd(s, u, offsets=off, max_len=20, out=out)
        with pytest.raises(fem.FemError):
            fem.check_device_error()
        right = [q for q in range(2) if bad[q:q + 2] == [20 * q, 20 * q + 20]]
        for q in right:
            assert torch.equal(out[20 * q:20 * q + 20], want[20 * q:20 * q + 20])
        fem.fem_recur_bwd(s, u, want, dh, offsets=off, max_len=20)
        with pytest.raises(fem.FemError):
            fem.check_device_error()
    pool = torch.zeros((3, 64), device="cuda")
    rows = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    h, _ = fem.fem_recur_fwd(s, u, offsets=offsets_of([20, 20]), max_len=20, h0=pool, state_rows=rows)
    with pytest.raises(fem.FemError):
        fem.check_device_error()
    assert torch.equal(h, want) and not pool[[0, 2]].any()
    fem.check_device_error()


def test_the_conditioners_convolution_is_a_special_case():
    """The same operator's dense fp32 form: both within their own bound of the definition."""
    s, u, _ = (x.view(2, 900, 64) for x in make(1800, 64, torch.float32, 9))
    a, _ = fem.fem_recur_fwd(s, u)
    b = fem.fem_tdc_conv(s, u)
    assert (a - b).abs().max() <= 1e-4 * max(1.0, a.abs().max().item())


@pytest.mark.parametrize("lens", [[3000], [100, 2000, 37] * 4])
def test_the_same_bits_again(lens):
    s, u, dh = make(sum(lens), 200, torch.bfloat16, 10)
    off = offsets_of(lens)
    first = None
    for _ in range(3):
        h, last = fem.fem_recur_fwd(s, u, offsets=off, max_len=max(lens))
        got = (h, last, *fem.fem_recur_bwd(s, u, h, dh, offsets=off, max_len=max(lens))[:2])
        assert first is None or all(torch.equal(a, b) for a, b in zip(got, first))
        first = got


def test_streams_and_graphs():
    s, u, dh = (x.view(2, 400, 64) for x in make(800, 64, torch.bfloat16, 11))
    want, want_last = fem.fem_recur_fwd(s, u)
    side = torch.cuda.Stream()
    late = [torch.empty_like(t) for t in (want, want_last)]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for t in late:
        t.fill_(7)
    del late, t
    h, last = fem.fem_recur_fwd(s, u, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(h, want) and torch.equal(last, want_last)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h, last = fem.fem_recur_fwd(s, u, mean=True)
            grads = fem.fem_recur_bwd(s, u, h, dh, mean=True)
    u.neg_()
    dh.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    h2, last2 = fem.fem_recur_fwd(s, u, mean=True)
    grads2 = fem.fem_recur_bwd(s, u, h2, dh, mean=True)
    assert torch.equal(h, h2) and torch.equal(last, last2)
    assert all(torch.equal(a, b) for a, b in zip(grads[:2], grads2[:2]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_sequences_of_some_steps(dtype):
    """So many that a thread walks each channel of one alone, and a longer one than was said."""
    lens, c = [40] * 255 + [131, 0, 1], 512
    n = sum(lens)
    s, u, dh = make(n, c, dtype, 15)
    h0, dlast = states(len(lens), c, 16)
    off = offsets_of(lens)
    h, last = fem.fem_recur_fwd(s, u, offsets=off, max_len=40, h0=h0, mean=True)
    want, want_last, hm, lm = ref.recur(s.cpu(), u.cpu(), lens, h0.cpu(), True)
    ref.check(h, want, hm, UNITS)
    ref.check(last, want_last, lm, UNITS)
    got = fem.fem_recur_bwd(s, u, h, dh, offsets=off, max_len=40, h0=h0, dstate=dlast, mean=True)
    grads, sizes = ref.recur_grads(s.cpu(), u.cpu(), h.cpu(), dh.cpu(), lens, h0.cpu(), dlast.cpu(), True)
    for g, w, m in zip(got, grads, sizes):
        ref.check(g, w, m, UNITS)


def test_many_short_sequences_beside_a_long_one():
    """The chunks are counted by the long one's length, the others have none of them to do."""
    lens, c = [1] * 3000 + [2000] + [0] * 500, 64
    n = sum(lens)
    s, u, dh = make(n, c, torch.bfloat16, 14)
    off = offsets_of(lens)
    h, last = fem.fem_recur_fwd(s, u, offsets=off, max_len=2000)
    assert torch.equal(h[:3000], u[:3000])  # a first step has nothing to decay
    want, want_last, hm, lm = ref.recur(s[3000:].cpu(), u[3000:].cpu(), [2000])
    ref.check(h[3000:], want, hm, UNITS)
    ref.check(last[3000:3001], want_last, lm, UNITS)
    assert not last[3001:].any() and torch.equal(last[:3000], u[:3000].float())
    ds, du, _ = fem.fem_recur_bwd(s, None, h, dh, offsets=off, max_len=2000)
    assert torch.equal(du[:3000], dh[:3000]) and not ds[:3000].any()
    grads, sizes = ref.recur_grads(s[3000:].cpu(), u[3000:].cpu(), h[3000:].cpu(), dh[3000:].cpu(), [2000])
    ref.check(ds[3000:], grads[0], sizes[0], UNITS)
    ref.check(du[3000:], grads[1], sizes[1], UNITS)
    fem.check_device_error()


def test_arrays_past_32_bits():
    """More than 2^32 elements: the last rows against a call on them alone, from the state before."""
    n, c, tail = 131200, 32768, 40
    s = torch.full((n, c), 0.5, dtype=torch.bfloat16, device="cuda")
    u = torch.empty((n, c), dtype=torch.bfloat16, device="cuda").normal_()
    h, last = fem.fem_recur_fwd(s[None], u[None], state_out=None)
    start = h[0, n - tail - 1].float()[None]
    want, _ = fem.fem_recur_fwd(s[n - tail:][None], u[n - tail:][None], h0=start)
    # the start is rounded to bf16, and half of that is left after a step and a half
    err = (h[0, n - tail:].float() - want[0].float()).abs()
    decayed = torch.exp(-0.5 * torch.arange(1, tail + 1, device="cuda"))[:, None] * start.abs() * 2.0 ** -8
    assert (err <= decayed + 2.0 ** -7 * want[0].float().abs() + 1e-5).all()


def test_empty_calls():
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.empty((0, 16), dtype=dtype, device="cuda")
        h0 = states(2, 16, 12)[0]
        h, last = fem.fem_recur_fwd(x, x, offsets=offsets_of([0, 0]), max_len=0, h0=h0)
        assert h.shape == (0, 16) and torch.equal(last, h0)
        ds, du, dh0 = fem.fem_recur_bwd(x, x, x, x, offsets=offsets_of([0, 0]), max_len=0, h0=h0, dstate=h0)
        assert torch.equal(dh0, h0)
        h, last = fem.fem_recur_fwd(x, x, offsets=offsets_of([]), max_len=0)
        assert last.shape == (0, 16)


def test_refusals():
    s, u, dh = make(40, 64, torch.float32, 13)
    off = offsets_of([20, 20])
    h0 = torch.zeros((2, 64), device="cuda")
    rows = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (dict(u=u[:39]), dict(u=u.bfloat16()), dict(s=s.half()), dict(offsets=off.long()), dict(offsets=off[None]),
                dict(offsets=None), dict(h0=h0[:1]), dict(h0=h0.double()), dict(h0=h0[:, :32]), dict(state_rows=rows, state_out=False),
                dict(h0=h0, state_rows=rows[:1]), dict(h0=h0, state_out=torch.zeros((3, 64), device="cuda")),
                dict(out=s.t().contiguous().t())):
        with pytest.raises(ValueError):
            fem.fem_recur_fwd(**{**dict(s=s, u=u, offsets=off, max_len=20), **bad})
    x = s.view(2, 20, 64)
    with pytest.raises(ValueError):
        fem.fem_recur_fwd(x.transpose(0, 1), x.transpose(0, 1))  # rows that are not evenly spaced
    with pytest.raises(ValueError):
        fem.fem_recur_bwd(s, u, s, dh, offsets=off, h0=h0, dstate=h0[:1])
    with pytest.raises(ValueError):
        fem.fem_recur_bwd(s, None, s, dh, offsets=off, mean=True)
