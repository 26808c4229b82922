"""The read over a paged cache against a plain 64-bit statement (needs a GB300).

Tolerances.  An fp32 cache is read in fp32: 1e-4, the fp32 read's bound.  With bf16 outputs an
entry may be off by its own rounding, 2^-9 |o|, and by the roundings of the prior weights and of
the value bank to 8-bit significands, each at most 2^-9 of a term: together at most 2^-8 of the
weighted |bank|, which is at most 2 max |v| of the channel (the bank is read where 1 + beta a / L
is at least 1/4, or against max |v| > 1/beta).  So |o - ref| <= 2^-8 |ref| + 2^-7 max |v|; roundings of
either sign average out, so the root mean square stays under a quarter of that.  lse is fp32:
1e-5 (1 + |lse|).
"""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import paged_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


def make(fmt, H, Hq, d, page, lens, seed=0, q_scale=1.0, v_scale=1.0, poison=True):
    """(q, cache, q_offsets, ctx_lens, table): lens are (new tokens, context) per sequence.  Pages
    and rows past a sequence's length hold NaN, and table entries past it no page."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-ctx // page) for _, ctx in lens]
    pages = sum(need) + 2
    dtype = TYPES[fmt]
    cache = fem.PagedCache.empty(pages, H, d, page, dtype)
    if poison:
        if fmt == "e4m3":
            cache.k_exp.fill_(255)
            cache.v_exp.fill_(255)
        else:
            cache.k.fill_(math.nan)
            cache.v.fill_(math.nan)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table, at = torch.full((len(lens), max(max(need), 1) + 1), -1, dtype=torch.int32), 0
    slots = []
    for s, (m, (_, ctx)) in enumerate(zip(need, lens)):
        table[s, :m] = order[at:at + m]
        at += m
        pos = torch.arange(ctx)
        slots.append(table[s].long()[pos // page] * page + pos % page)
    slots = torch.cat(slots).to(DEV)
    k = torch.randn((len(slots), H, d), generator=g).to(cache.row_dtype).to(DEV)
    v = (v_scale * torch.randn((len(slots), H, d), generator=g)).to(cache.row_dtype).to(DEV)
    fem.fem_cache_write(cache, k, v, slots)
    N = sum(n for n, _ in lens)
    q = (q_scale * torch.randn((N, Hq + 2, d), generator=g)).to(cache.row_dtype).to(DEV)[:, 1:1 + Hq]  # a strided view
    offsets = torch.tensor([sum(n for n, _ in lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
    ctx = torch.tensor([c for _, c in lens], dtype=torch.int32, device=DEV)
    return q, cache, offsets, ctx, table.to(DEV)


def make_beta(kind, H, d, seed=0):
    if kind is None:
        return None
    lo, hi = kind
    u = torch.rand((H, d), generator=torch.Generator().manual_seed(seed))
    beta = torch.exp(math.log(lo) + u * math.log(hi / lo)).float()
    beta[0, :3] = 0.0
    return beta.to(DEV)


def check(q, cache, beta, offsets, ctx, table, causal, max_q, v_abs=None, rms=True):
    N, Hq, d = q.shape
    out = torch.full((N, Hq, d), math.nan, dtype=q.dtype, device=DEV)
    lse = torch.full((N, Hq), math.nan, dtype=torch.float32, device=DEV)
    fem.fem_paged_read(q, cache, beta, offsets, ctx, table, max_q=max_q, causal=causal, out=out, lse=lse)
    fem.check_device_error()
    ref, ref_lse, big = R.read(q, cache, beta, offsets, ctx, table, causal)
    empty = torch.isinf(ref_lse)
    assert torch.equal(torch.isinf(lse), empty)
    assert torch.isfinite(out).all()
    assert (out[empty] == 0).all()
    err_l = (lse.double() - ref_lse)[~empty].abs()
    assert (err_l <= 1e-5 * (1 + ref_lse[~empty].abs())).all(), err_l.max()
    err = (out.double() - ref).abs()
    if q.dtype == torch.float32:
        assert err.max() <= 1e-4, err.max()
    else:
        tol = 2.0 ** -8 * ref.abs() + 2.0 ** -7 * big
        worst = (err / tol.clamp_min(1e-30)).max().item()
        assert worst <= 1.0, worst
        if rms and err.numel():
            assert err.square().mean().sqrt() <= 0.25 * tol.square().mean().sqrt()
    return out, lse


LENS = {
    "one": [(1, 1)],
    "tokens": [(1, 1), (1, 15), (1, 16), (1, 17), (1, 64), (1, 127), (1, 128), (1, 129), (1, 700), (1, 0)],
    "drafts": [(2, 2), (5, 40), (3, 129), (0, 50), (8, 300), (4, 2)],
    "chunks": [(17, 17), (130, 400), (1, 77), (64, 64), (0, 0), (33, 257), (128, 128), (40, 20)],
    "long_chunk": [(300, 1000)],
}


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("lens", sorted(LENS))
@pytest.mark.parametrize("H,Hq,d,page", [(2, 2, 64, 16), (2, 8, 128, 64), (1, 3, 64, 128), (1, 8, 128, 32)])
@pytest.mark.parametrize("kind", [None, (0.1, 5.0)])
def test_read(fmt, lens, H, Hq, d, page, kind):
    lens = LENS[lens]
    args = make(fmt, H, Hq, d, page, lens, seed=d + page)
    check(args[0], args[1], make_beta(kind, H, d), *args[2:], causal=True, max_q=max(n for n, _ in lens))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens", ["tokens", "drafts", "chunks"])
def test_read_without_a_mask(fmt, lens):
    """Every new token sees the whole context (cached states of another length)."""
    lens = LENS[lens]
    args = make(fmt, 2, 4, 64, 64, lens, seed=5)
    check(args[0], args[1], make_beta((0.1, 5.0), 2, 64), *args[2:], causal=False, max_q=max(n for n, _ in lens))


@pytest.mark.parametrize("fmt,d", [("bf16", 16), ("bf16", 96), ("e4m3", 32), ("e4m3", 256), ("f32", 48), ("f32", 256)])
def test_read_other_head_dimensions(fmt, d):
    lens = [(1, 33), (5, 200), (20, 20)]
    args = make(fmt, 2, 4, d, 32, lens, seed=d)
    check(args[0], args[1], make_beta((0.05, 20.0), 2, d), *args[2:], causal=True, max_q=20)


@pytest.mark.parametrize("lens", ["tokens", "drafts", "chunks"])
@pytest.mark.parametrize("beta", [1e-6, 1e-3, 0.05, 1.0, 20.0, 300.0])
@pytest.mark.parametrize("v_scale", [0.01, 1.0, 30.0])
def test_read_any_beta_and_spread(lens, beta, v_scale):
    """One beta for every channel, over values of small, unit and large spread, peaked priors."""
    lens = LENS[lens]
    q, cache, off, ctx, table = make("bf16", 2, 4, 64, 16, lens, seed=3, q_scale=4.0, v_scale=v_scale)
    b = torch.full((2, 64), beta, device=DEV)
    check(q, cache, b, off, ctx, table, causal=True, max_q=max(n for n, _ in lens), rms=False)


@pytest.mark.parametrize("n,ctx", [(1, 5000), (6, 5000), (200, 5000)])
def test_read_peaked_prior_far_under_the_largest_value(n, ctx):
    """Rows whose prior sits on one key whose value lies far below the others': e^(beta (v - max v))
    is under fp32's range, and the result is still that key's value."""
    H, d = 1, 64
    q, cache, off, cl, table = make("bf16", H, 2, d, 64, [(n, ctx)], seed=1)
    pos = torch.arange(ctx, device=DEV)
    where, row = table[0].long()[pos // 64], pos % 64
    key = ctx - n - 1  # a key every row sees
    cache.k[where, 0, row] = 0
    cache.k[where[key], 0, row[key]] = 24.0
    q.fill_(8.0)       # score 8 * 24 * 64 / 8 = 1536 at the key, 0 elsewhere
    cache.v[where, 0, row] = torch.rand((ctx, d), device=DEV).to(torch.bfloat16) + 20.0
    cache.v[where[key], 0, row[key]] = -20.0
    for beta in (0.5, 20.0):
        b = torch.full((H, d), beta, device=DEV)
        out, lse = check(q, cache, b, off, cl, table, causal=True, max_q=n, rms=False)


def test_read_ignores_what_a_row_does_not_see():
    """Infinities and NaN in later keys and values of the chunk leave earlier rows alone."""
    lens = [(40, 200), (6, 100)]
    for fmt_d in (64, 128):
        q, cache, off, ctx, table = make("bf16", 1, 2, fmt_d, 32, lens, seed=9)
        beta = make_beta((0.1, 5.0), 1, fmt_d)
        for b in (None, beta):
            clean, clean_lse = fem.fem_paged_read(q, cache, b, off, ctx, table, max_q=40)
            kept = (cache.k.clone(), cache.v.clone())
            for s, (n, c) in enumerate(lens):
                for i, bad in ((c - 1, math.nan), (c - 2, math.inf)):
                    cache.k[table[s, i // 32].long(), :, i % 32] = bad
                    cache.v[table[s, i // 32].long(), :, i % 32] = bad
            out, lse = fem.fem_paged_read(q, cache, b, off, ctx, table, max_q=40)
            a = 0
            for n, c in lens:
                rows = slice(a, a + n - 2)
                tol = 2.0 ** -6 * (1 + clean[rows].double().abs())
                assert torch.isfinite(out[rows]).all()
                assert ((out[rows].double() - clean[rows].double()).abs() <= tol).all()
                assert ((lse[rows] - clean_lse[rows]).abs() <= 1e-4).all()
                a += n
            cache.k.copy_(kept[0])
            cache.v.copy_(kept[1])
    fem.check_device_error()


def test_rows_nobody_owns_are_not_written():
    q, cache, off, ctx, table = make("bf16", 2, 4, 128, 64, [(3, 90), (2, 50)], seed=2)
    off = off + 2  # rows 0, 1 belong to nobody, nor do the last two
    big = torch.cat([q, q])[:9].contiguous()
    out = torch.full(big.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full(big.shape[:2], 7.0, device=DEV)
    fem.fem_paged_read(big, cache, None, off, ctx, table, max_q=3, out=out, lse=lse)
    fem.check_device_error()
    assert (out[:2] == 7).all() and (out[7:] == 7).all() and (lse[:2] == 7).all() and (lse[7:] == 7).all()
    ref, ref_lse, _ = R.read(big, cache, None, off, ctx, table, True)
    assert (out[2:7].double() - ref[2:7]).abs().max() < 0.05


@pytest.mark.parametrize("n", [1, 4, 150])
def test_pages_that_are_not_there(n):
    """A table entry that names no page: its keys are left out, and the call reports it."""
    for page in (16, 64, 128):
        q, cache, off, ctx, table = make("e4m3", 2, 4, 64, page, [(n, 400), (n, 333)], seed=page)
        table[0, 1] = cache.num_pages
        table[1, 0] = -5
        beta = make_beta((0.1, 5.0), 2, 64)
        out, lse = fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n)
        with pytest.raises(fem.FemError) as e:
            fem.check_device_error()
        assert e.value.status == 1
        ref, ref_lse, big = R.read(q, cache, beta, off, ctx, table, True)
        assert ((lse.double() - ref_lse).abs() <= 1e-5 * (1 + ref_lse.abs())).all()
        assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -7 * big).all()


def test_lengths_outside_the_buffers_are_cut_and_reported():
    q, cache, off, ctx, table = make("bf16", 1, 1, 64, 16, [(2, 40)], seed=4)
    out, lse = fem.fem_paged_read(q, cache, None, off, ctx, table, max_q=2)
    fem.check_device_error()
    fem.fem_paged_read(q, cache, None, off + 1, ctx, table, max_q=2)      # the last row is past q
    with pytest.raises(fem.FemError):
        fem.check_device_error()
    fem.fem_paged_read(q, cache, None, off, ctx * 0 + 2 ** 30, table, max_q=2)  # past the table
    with pytest.raises(fem.FemError):
        fem.check_device_error()


@pytest.mark.parametrize("n", [1, 3, 100])
def test_max_q_may_be_loose(n):
    lens = [(n, 300), (1, 20)]
    args = make("bf16", 2, 4, 128, 32, lens, seed=6)
    beta = make_beta((0.1, 5.0), 2, 128)
    for max_q in (n, 500, 1):  # below the longest, too: read correctly all the same
        check(args[0], args[1], beta, *args[2:], causal=True, max_q=max_q)


@pytest.mark.parametrize("n", [1, 5, 200])
def test_same_inputs_same_bits_and_streams(n):
    lens = [(n, 2000 + n), (n, 700 + n)]
    q, cache, off, ctx, table = make("e4m3", 2, 8, 128, 64, lens, seed=8)
    beta = make_beta((0.1, 5.0), 2, 128)
    first, first_lse = fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        out, lse = (torch.full_like(first, math.nan), torch.full_like(first_lse, math.nan))
        side.wait_stream(torch.cuda.current_stream())
        fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n, out=out, lse=lse, stream=side)
        side.synchronize()
        assert torch.equal(out, first) and torch.equal(lse, first_lse)


@pytest.mark.parametrize("n", [1, 150])
def test_read_in_a_graph_follows_the_device_arrays(n):
    """A captured call reads lengths and tables from the device at replay."""
    q, cache, off, ctx, table = make("bf16", 2, 4, 128, 64, [(n, 500), (n, 900)], seed=12)
    beta = make_beta((0.1, 5.0), 2, 128)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n, out=out, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n, out=out, lse=lse)
    ctx -= 37
    graph.replay()
    torch.cuda.synchronize()
    want, want_lse = fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=n)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("H,Hq,d", [(1, 5, 64), (1, 7, 128), (2, 24, 64), (1, 40, 128), (1, 130, 64), (1, 300, 64)])
@pytest.mark.parametrize("n", [1, 3, 90])
def test_any_number_of_query_heads(H, Hq, d, n):
    """Groups that are no power of two, wider than a row tile's tokens, wider than a row tile."""
    lens = [(n, n + 200), (1, 1), (n, n)]
    args = make("e4m3", H, Hq, d, 32, lens, seed=Hq)
    check(args[0], args[1], make_beta((0.1, 5.0), H, d), *args[2:], causal=True, max_q=n)


@pytest.mark.parametrize("n,S", [(1, 200), (2, 1000), (20, 300)])
def test_many_sequences(n, S):
    """More sequences than a block has threads, some without rows, some without a cache."""
    lens = [(0, 5) if s % 7 == 3 else (1, 0) if s % 31 == 30 else (1 + s % n, 1 + s % n + (s * 13) % 150) for s in range(S)]
    args = make("bf16", 1, 2, 64, 16, lens, seed=S)
    check(args[0], args[1], make_beta((0.1, 5.0), 1, 64), *args[2:], causal=True, max_q=n)


@pytest.mark.parametrize("n", [1, 4, 60])
@pytest.mark.parametrize("jump", [40.0, 80.0, 300.0, 40000.0])
def test_scores_that_jump(n, jump):
    """Scores that rise or fall by far more than the weights' range from one key tile to another."""
    for sign in (1.0, -1.0):
        q, cache, off, ctx, table = make("bf16", 1, 2, 64, 64, [(n, 900)], seed=21)
        pos = torch.arange(900, device=DEV)
        where, row = table[0].long()[pos // 64], pos % 64
        q.zero_()
        q[..., 0] = 8.0                       # score: k_0 in natural units
        k0 = torch.where(pos >= 450, sign * jump, 0.0) + torch.sin(pos.float())
        cache.k[where, 0, row] = 0
        cache.k[where, 0, row, 0] = k0.to(torch.bfloat16)
        for beta in (None, torch.full((1, 64), 0.7, device=DEV), torch.full((1, 64), 8.0, device=DEV)):
            check(q, cache, beta, off, ctx, table, causal=True, max_q=n, rms=False)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("big", [50.0, 3.0e4])
def test_values_far_from_the_first_ones(n, big):
    """Channels whose first values are tiny, zero or negative and whose later ones are not."""
    q, cache, off, ctx, table = make("bf16", 1, 2, 64, 16, [(n, 300)], seed=22, q_scale=3.0)
    pos = torch.arange(300, device=DEV)
    where, row = table[0].long()[pos // 16], pos % 16
    g = torch.Generator().manual_seed(5)
    v = torch.randn((300, 64), generator=g).to(DEV)
    v[:16, :16] = 0
    v[:16, 16:32] *= 1e-4
    v[:16, 32:48] = -big
    v[200, 8:40] = big
    cache.v[where, 0, row] = v.to(torch.bfloat16)
    for beta in (1e-5, 1e-3, 0.3, 4.0):
        check(q, cache, torch.full((1, 64), beta, device=DEV), off, ctx, table, causal=True, max_q=n, rms=False)


def test_read_over_a_cache_past_32_bits():
    """Pages past 2^31 elements of the cache are read at their own place."""
    H, d, page = 8, 128, 64
    pages = (1 << 31) // (H * d * page) + 8
    k = torch.empty((pages, H, page, d), dtype=torch.bfloat16, device=DEV)
    cache = fem.PagedCache(k, torch.empty_like(k))
    g = torch.Generator().manual_seed(2)
    table = torch.tensor([[pages - 1, 3, pages - 4]], dtype=torch.int32, device=DEV)
    for p in table[0].tolist():
        cache.k[p] = torch.randn((H, page, d), generator=g).to(torch.bfloat16).to(DEV)
        cache.v[p] = torch.randn((H, page, d), generator=g).to(torch.bfloat16).to(DEV)
    beta = make_beta((0.1, 5.0), H, d)
    for n in (1, 100):
        q = torch.randn((n, H, d), generator=g).to(torch.bfloat16).to(DEV)
        off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        check(q, cache, beta, off, torch.tensor([170], dtype=torch.int32, device=DEV), table, causal=True, max_q=n)


@pytest.mark.parametrize("n", [1, 50])
def test_infinite_and_nan_rows(n):
    """A query of NaN gives NaN in its own row alone; a key of -inf has no weight."""
    q, cache, off, ctx, table = make("bf16", 1, 2, 128, 32, [(n, 333), (n, 100)], seed=30)
    q[0, 0] = math.nan
    beta = make_beta((0.1, 5.0), 1, 128)
    for b in (None, beta):
        out, lse = fem.fem_paged_read(q, cache, b, off, ctx, table, max_q=n)
        assert torch.isnan(out[0, 0]).all() and torch.isnan(lse[0, 0])
        ref, ref_lse, big = R.read(q, cache, b, off, ctx, table, True)
        ok = torch.isfinite(ref_lse)
        assert ok.sum().item() == ok.numel() - 1
        assert torch.isfinite(out[ok]).all()
        assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -7 * big)[ok].all()
    fem.check_device_error()


def test_matches_the_contiguous_reads():
    """The same tokens through fem_decode and fem_fwd (contiguous, one head per key/value head)."""
    H, d, T = 4, 128, 700
    lens = [(T, T)]
    q, cache, off, ctx, table = make("bf16", H, H, d, 64, lens, seed=13)
    beta = make_beta((0.1, 5.0), H, d)
    out, lse = fem.fem_paged_read(q, cache, beta, off, ctx, table, max_q=T)
    k, v = fem.fem_cache_gather(cache, table, torch.zeros(1, dtype=torch.int32, device=DEV), off, T)
    as_bhtd = [t.transpose(0, 1).contiguous()[None] for t in (q, k, v)]
    ref, ref_lse = fem.fem_fwd(*as_bhtd, beta, causal=True)
    assert (out.transpose(0, 1)[None].float() - ref).abs().max() <= 4e-2
    assert (lse.transpose(0, 1)[None] - ref_lse).abs().max() <= 2e-3
    one = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    tok, tok_lse = fem.fem_paged_read(q[-1:], cache, beta, one, ctx, table, max_q=1)
    dec, dec_lse = fem.fem_decode(as_bhtd[0][:, :, -1].contiguous(), as_bhtd[1], as_bhtd[2], beta)
    assert (tok[0].float() - dec[0]).abs().max() <= 2e-2
    assert (tok_lse[0] - dec_lse[0]).abs().max() <= 1e-4


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens", ["tokens", "chunks"])
@pytest.mark.parametrize("q_scale", [1.0, 6.0])
@pytest.mark.parametrize("d", [64, 128])
def test_read_with_small_and_large_beta_in_one_head(fmt, lens, q_scale, d):
    """beta 1e-4 to 20 side by side: the largest |E| of one channel decides nothing about another's."""
    lens = LENS[lens]
    q, cache, off, ctx, table = make(fmt, 2, 8, d, 32, lens, seed=17, q_scale=q_scale)
    check(q, cache, make_beta((1e-4, 20.0), 2, d, seed=3), off, ctx, table, causal=True, max_q=max(n for n, _ in lens),
          rms=False)


@pytest.mark.parametrize("beta", [0.3, 5.0])
@pytest.mark.parametrize("n", [1, 40])
def test_a_few_channels_of_a_row_again(n, beta):
    """Values whose first ones mislead in a few channels: those alone are recomputed."""
    q, cache, off, ctx, table = make("bf16", 1, 4, 128, 64, [(n, 1500)], seed=23, poison=False)
    order = table[0, :24].long()
    v = cache.v[order]  # [pages, 1, 64, 128]: positions in order
    v[0, 0, :16, 3:9] = 0.01 * v[0, 0, :16, 3:9]
    v[2:, 0, :, 5] -= 40.0
    v[2:, 0, :, 7] += 40.0
    cache.v[order] = v
    b = torch.full((1, 128), beta, device=DEV)
    check(q, cache, b, off, ctx, table, causal=True, max_q=n, rms=False)
