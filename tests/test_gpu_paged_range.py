"""The paged read where scores and values leave the range of fp32 between key tiles (needs a GB300).

Scores: q is 8 in its first channels and 0 elsewhere, so that with d = 64 a key's score is the sum of its
first channels (sqrt(2) less at d = 128).  The bounds are the ones of the other paged reads: what is
recomputed, and what is not, has to meet them alike.
"""
import math

import pytest
import torch

from paper_2602_07160_gb300 import fem
from tests.test_gpu_paged_read import DEV, check, lib, make  # noqa: F401  (lib: builds and loads the library)

pytestmark = pytest.mark.gpu


def rewrite(cache, table, k, v):
    """The keys and values [ctx, d] of the only head of sequence 0."""
    pos = torch.arange(len(k), device=DEV)
    slots = table[0].long()[pos // cache.page_size] * cache.page_size + pos % cache.page_size
    fem.fem_cache_write(cache, k.to(torch.bfloat16)[:, None].contiguous(), v.to(torch.bfloat16)[:, None].contiguous(), slots)


# (keys, the outlying value's key, the keys whose scores lie higher)
JUMPS = {"one_warp": (192, 20, (64, 192)),        # the warp that has the value meets the higher scores
         "another_warp": (192, 20, (64, 80)),     # only the warp beside it does
         "another_cta": (40000, 20, (30000, 40000))}


@pytest.mark.parametrize("fmt,d", [("bf16", 64), ("bf16", 128), ("e4m3", 64), ("e4m3", 128)])
@pytest.mark.parametrize("where", sorted(JUMPS))
@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("beta", [5.0, 8.0, 20.0])
def test_a_prior_that_jumps_over_an_outlying_value(fmt, d, where, n, beta):
    """A value far above the others in an early key, and later scores higher by more than a weight's range:
    the value's term, e^(beta v) times next to nothing, is still the larger one."""
    ctx, at, (lo, hi) = JUMPS[where]
    q, cache, off, cl, table = make(fmt, 1, 2, d, 64, [(n, ctx)], seed=40)
    q.zero_()
    q[..., 0] = 8.0
    g = torch.Generator().manual_seed(41)
    for nats in (90.0, 100.0, 110.0, 140.0):
        k = torch.zeros((ctx, d))
        k[:, 0] = torch.randn(ctx, generator=g)
        k[lo:hi, 0] += nats
        k[:, 0] *= math.sqrt(d) / 8
        v = torch.rand((ctx, d), generator=g) * 0.5 - 0.5
        v[:16] = torch.rand((16, d), generator=g) * 2 - 1
        v[lo:hi] = -0.5
        # some ten nats over the later keys' term, in half of the channels
        v[at, ::2] = (nats + 10.0) / beta - 0.5
        rewrite(cache, table, k.to(DEV), v.to(DEV))
        check(q, cache, torch.full((1, d), beta, device=DEV), off, cl, table, causal=True, max_q=n, rms=False)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("beta", [None, 0.0, 0.1, 0.7, 8.0])
@pytest.mark.parametrize("ctx", [1024, 30 * 1024])
@pytest.mark.parametrize("nats", [84.0, 84.5, 85.0, 86.0, 87.0, 88.0, 88.5, 89.0])
def test_weights_that_are_finite_and_whose_sum_is_not(fmt, beta, ctx, nats):
    """Scores that rise in a row's last key tile until its weights against the maximum so far are still in
    fp32's range and their sum is not; a read in one piece, and one that is joined."""
    n, d = 60, 64
    q, cache, off, cl, table = make(fmt, 1, 2, d, 64, [(n, ctx)], seed=42)
    q.zero_()
    q[..., 0] = 8.0
    k = torch.zeros((ctx, d))
    k[ctx - 128:, 0] = nats
    for spread in (0.02, 1.0):
        v = spread * torch.randn((ctx, d), generator=torch.Generator().manual_seed(43))
        rewrite(cache, table, k.to(DEV), v.to(DEV))
        b = None if beta is None else torch.full((1, d), beta, device=DEV)
        check(q, cache, b, off, cl, table, causal=True, max_q=n, rms=False)


@pytest.mark.parametrize("beta", [None, 0.7])
def test_pieces_whose_sums_are_finite_and_together_are_not(beta):
    """One key of a high score in each of two key tiles, eight tiles apart in a long context, that end
    the stretches of two CTAs in one of the steps below."""
    n, d, tiles = 20, 64, 608
    ctx = 128 * tiles
    q, cache, off, cl, table = make("bf16", 1, 2, d, 64, [(n, ctx)], seed=48)
    q.zero_()
    q[..., 0] = 8.0
    v = torch.randn((ctx, d), generator=torch.Generator().manual_seed(49))
    for step in range(8):
        k = torch.zeros((ctx, d))
        k[[128 * (100 + step) + 3, 128 * (108 + step) + 3], 0] = 88.5
        rewrite(cache, table, k.to(DEV), v.to(DEV))
        b = None if beta is None else torch.full((1, d), beta, device=DEV)
        check(q, cache, b, off, cl, table, causal=True, max_q=n, rms=False)


@pytest.mark.parametrize("beta", [None, 0.1, 0.7, 8.0])
@pytest.mark.parametrize("nats", [86.5, 87.0, 87.5, 88.0, 88.5])
def test_weights_near_the_end_of_the_range_before_the_maximum_rises(beta, nats):
    """Two key tiles that hold a few keys of the same high score each: the first tile's weights, up to the
    end of fp32's range against the maximum so far, are worth as much as the second's."""
    n, ctx, d = 60, 1024, 64
    q, cache, off, cl, table = make("bf16", 1, 2, d, 64, [(n, ctx)], seed=44)
    q.zero_()
    q[..., 0] = 8.0
    k = torch.zeros((ctx, d))
    k[[515, 600, 650, 720], 0] = nats  # a key of either half of key tiles 4 and 5
    v = torch.randn((ctx, d), generator=torch.Generator().manual_seed(45))
    rewrite(cache, table, k.to(DEV), v.to(DEV))
    b = None if beta is None else torch.full((1, d), beta, device=DEV)
    check(q, cache, b, off, cl, table, causal=True, max_q=n, rms=False)


@pytest.mark.parametrize("beta", [None, 0.1, 0.7, 8.0])
@pytest.mark.parametrize("base", [15104.0, 30208.0, 60416.0])
def test_a_maximum_that_rises_among_scores_of_tens_of_thousands(beta, base):
    """Scores so large that a maximum in 8 bits could lie a weight's range over the true one."""
    n, ctx, d = 40, 1024, 64
    q, cache, off, cl, table = make("bf16", 1, 2, d, 64, [(n, ctx)], seed=46)
    q.zero_()
    q[..., :3] = 8.0
    b = None if beta is None else torch.full((1, d), beta, device=DEV)
    v = torch.randn((ctx, d), generator=torch.Generator().manual_seed(47))
    for step in range(0, 48):
        k = torch.zeros((ctx, d))
        k[:, 0] = base                    # to multiples of 128 or 256, in bf16
        k[:, 1] = 2.0 * step              # where the maximum falls between them
        k[[520, 640, 700], 2] = 42.0      # the largest scores, in key tiles 4 and 5
        k[[521, 641, 701], 2] = 40.0      # an eighth of their weight
        rewrite(cache, table, k.to(DEV), v.to(DEV))
        check(q, cache, b, off, cl, table, causal=True, max_q=n, rms=False)


@pytest.mark.parametrize("spread", [0.25, 1.0, 2.0])
def test_scores_whose_fp32_steps_are_tens(spread):
    """Equal scores of 2^30 and up, where fp32's steps are 64 and 128, over values far under the first ones':
    the rounding of a maximum takes no part of the weights with it."""
    n, ctx, d = 40, 1024, 64
    q, cache, off, cl, table = make("bf16", 1, 2, d, 64, [(n, ctx)], seed=50)
    q.zero_()
    q[..., 0] = 8.0
    v = spread * torch.rand((ctx, d), generator=torch.Generator().manual_seed(51)) - 5.0 - spread / 2
    v[:16] = 0.0
    for step in range(64):
        k = torch.zeros((ctx, d))
        k[16:, 0] = 2.0 ** 30 * (1 + step / 64)
        rewrite(cache, table, k.to(DEV), v.to(DEV))
        check(q, cache, torch.full((1, d), 8.0, device=DEV), off, cl, table, causal=True, max_q=n, rms=False)


@pytest.mark.parametrize("fmt,d", [("bf16", 64), ("e4m3", 128)])
@pytest.mark.parametrize("n,ctx", [(1, 20), (1, 300), (1, 5000), (4, 300), (40, 300), (40, 5000)])
@pytest.mark.parametrize("spread", [0.001, 0.01, 0.1, 1.0])
def test_channels_whose_first_values_are_zero(fmt, d, n, ctx, spread):
    """Half of the channels begin with zeros, which say nothing of the values that follow: those are read
    as well as any."""
    q, cache, off, cl, table = make(fmt, 1, 2, d, 64, [(n, ctx)], seed=52)
    g = torch.Generator().manual_seed(53)
    v = spread * torch.randn((ctx, d), generator=g)
    v[:16, ::2] = 0
    rewrite(cache, table, torch.randn((ctx, d), generator=g).to(DEV), v.to(DEV))
    for beta in (1e-4, 0.01, 0.1, 0.75, 2.0, 20.0):
        check(q, cache, torch.full((1, d), beta, device=DEV), off, cl, table, causal=True, max_q=n, rms=False)
