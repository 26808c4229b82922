"""The gated recurrence where lines of steps are many tiles long, on the GPU against its 64-bit form (needs a GB300): in
CTAs of four and eight warps, of 32, 16 and 8 lanes' channels, whole and in chunks, rows on and off 16 bytes.

Tolerance: the output's half step and as many roundings of the reference's magnitudes as in the recurrence's other tests.
"""
import math
import random

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref
from tests.test_gpu_recur import UNITS, make, offsets_of, states

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


def check(name, got, want, magnitude):
    half = ref.half_step(got.dtype)
    over = ((got.double() - want).abs() / (half * want.abs() + UNITS * ref.UNIT * magnitude * (1 + half) + 1e-37)).nan_to_num(nan=math.inf)
    assert over.max() <= 1, (name, over.max().item(), over.argmax().item())


def padded(x, lens):
    """[N, C] as [T, S, C] in 64 bits, zeros behind a sequence's end, where a rate of zero keeps a state."""
    y = torch.zeros((max(lens), len(lens), x.shape[-1]), dtype=torch.float64, device=x.device)
    for q, part in enumerate(x.double().split(lens)):
        y[:len(part), q] = part
    return y


def packed(y, lens):
    return torch.cat([y[:n, q] for q, n in enumerate(lens)])


def forward(s, u, lens, h0, mean):
    """All sequences at once; values and magnitudes as the reference's one by one."""
    s, u = padded(s, lens), padded(u, lens)
    h, hm = torch.zeros_like(s), torch.zeros_like(s)
    x = h0.double()
    size, err = x.abs(), torch.zeros_like(x)
    here = torch.arange(len(s), device=s.device)[:, None, None] < torch.tensor(lens, device=s.device)[None, :, None]
    for t in range(len(s)):
        a = torch.exp(-s[t])
        f = u[t] * -torch.expm1(-s[t]) if mean else u[t]
        x, size = a * x + f, a * size + f.abs()
        err = a * err + size * here[t]
        h[t], hm[t] = x, err
    return packed(h, lens), x, packed(hm, lens), err


def gradients(s, u, h, dh, lens, h0, dstate, mean):
    s, u, h, dh = (padded(x, lens) for x in (s, u, h, dh))
    ds, du, dsm, dum = (torch.zeros_like(s) for _ in range(4))
    m = dstate.double()
    size, err = m.abs(), torch.zeros_like(m)
    here = torch.arange(len(s), device=s.device)[:, None, None] < torch.tensor(lens, device=s.device)[None, :, None]
    for t in range(len(s) - 1, -1, -1):
        a, w = torch.exp(-s[t]), -torch.expm1(-s[t])
        total, before = dh[t] + m, h[t - 1] if t else h0.double()
        size = size + dh[t].abs()
        du[t], dum[t] = (total * w, (size + err) * w) if mean else (total, size + err)
        m, size, err = a * total, a * size, a * (err + size * here[t])
        ds[t] = m * (u[t] - before) if mean else -m * before
        dsm[t] = (size + err) * (before.abs() + (u[t].abs() if mean else 0.0))
    return [packed(x, lens) for x in (ds, du)] + [m], [packed(x, lens) for x in (dsm, dum)] + [err + size]


def compare(lens, c, dtype, mean, s, u, dh, **kw):
    h0, dl = states(len(lens), c, c)
    out, last = torch.full((sum(lens), c), math.nan, dtype=dtype, device="cuda"), torch.full_like(h0, math.nan)
    h, last = fem.fem_recur_fwd(s, u, h0=h0, mean=mean, out=out.view(s.shape), state_out=last, **kw)
    flat = lambda x: x.reshape(-1, c)  # noqa: E731
    want, want_last, hm, lm = forward(flat(s), flat(u), lens, h0, mean)
    check("h", out, want, hm)
    check("last", last, want_last, lm)
    got = fem.fem_recur_bwd(s, u, h, dh, h0=h0, dstate=dl, mean=mean, **kw)
    grads, sizes = gradients(flat(s), flat(u), out, flat(dh), lens, h0, dl, mean)
    for name, g, w, m in zip(("ds", "du", "dh0"), got, grads, sizes):
        check(name, g.view(w.shape), w, m)
    fem.check_device_error()


SHAPES = [(8, 1030, 2048), (20, 1030, 1000), (9, 1030, 1001), (3, 700, 2048), (64, 300, 512), (200, 700, 48), (700, 500, 30), (700, 500, 14),
          (2, 5000, 256), (1, 5000, 33), (1, 5000, 8)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("S,T,C", SHAPES)
def test_batches_of_many_tiles(S, T, C, dtype, mean):
    s, u, dh = (x.view(S, T, C) for x in make(S * T, C, dtype, S + T))
    compare([T] * S, C, dtype, mean, s, u, dh)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("S,T,C", [(40, 1500, 512), (11, 3000, 333), (5, 4000, 64), (300, 400, 24)])
def test_packed_sequences_of_many_tiles(S, T, C, dtype, mean):
    rng = random.Random(S)
    lens = [T] + [rng.choice([0, 1, rng.randint(1, T), rng.randint(1, T)]) for _ in range(S - 1)]
    s, u, dh = make(sum(lens), C, dtype, S)
    compare(lens, C, dtype, mean, s, u, dh, offsets=offsets_of(lens), max_len=T)
