"""Writing a paged cache and reading it back, against plain 64-bit statements (needs a GB300).

Both are defined to the bit (a rounding of each element by itself), so codes, scales and values
read back have to be equal.
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


def _tokens(N, H, d, dtype, seed, spread=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((N, H, d), generator=g)
    if spread:  # rows of very different magnitudes
        x = x * torch.exp(6.0 * torch.randn((N, H, 1), generator=g))
    return x.to(dtype).to(DEV)


def _expect(cache, k, v, slots):
    """The cache's tensors after the write, as (values of the codes, bytes)."""
    want = []
    for t, e, new in ((cache.k, cache.k_exp, k), (cache.v, cache.v_exp, v)):
        t = t.to(torch.float32).double().clone()
        e = None if e is None else e.clone()
        code, byte = R.quantise(new) if e is not None else (new.double(), None)
        for i, s in enumerate(slots.tolist()):
            if 0 <= s < cache.num_pages * cache.page_size:
                t[s // cache.page_size, :, s % cache.page_size] = code[i]
                if e is not None:
                    e[s // cache.page_size, :, s % cache.page_size] = byte[i]
        want.append((t, e))
    return want


def _check(cache, want):
    for (t, e), (wt, we) in zip(((cache.k, cache.k_exp), (cache.v, cache.v_exp)), want):
        if e is not None:
            assert torch.equal(e, we)
        assert torch.equal(t.to(torch.float32).double(), wt)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("N,H,d,page", [(1, 1, 16, 16), (1, 8, 128, 64), (37, 3, 64, 32), (200, 5, 96, 128),
                                        (65, 2, 256, 256), (513, 12, 64, 16), (40, 7, 240, 64), (9, 4, 32, 16)])
def test_write(fmt, N, H, d, page):
    pages = N // page + 3
    cache = fem.PagedCache.empty(pages, H, d, page, TYPES[fmt])
    k, v = (_tokens(N, H, d, cache.row_dtype, 7 * N + d + i) for i in range(2))
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(N))[:N].to(DEV)
    slots[::5] = -1  # padding, left out
    want = _expect(cache, k, v, slots)
    fem.fem_cache_write(cache, k, v, slots)
    fem.check_device_error()
    _check(cache, want)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_write_takes_views_of_one_projection(fmt):
    N, H, d = 70, 4, 128
    qkv = _tokens(N, 3 * H + 1, d, torch.bfloat16, 3)
    cache = fem.PagedCache.empty(3, H, d, 64, TYPES[fmt])
    slots = torch.arange(N, device=DEV) + 11
    k, v = qkv[:, H:2 * H], qkv[:, 2 * H:3 * H]
    want = _expect(cache, k, v, slots)
    fem.fem_cache_write(cache, k, v, slots)
    _check(cache, want)
    # heads outermost
    kt, vt = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (k, v))
    other = fem.PagedCache.empty(3, H, d, 64, TYPES[fmt])
    fem.fem_cache_write(other, kt, vt, slots)
    _check(other, want)
    # one token of many: the token axis has no stride to speak of
    one = fem.PagedCache.empty(3, H, d, 64, TYPES[fmt])
    fem.fem_cache_write(one, k[5:6], v[5:6], slots[5:6])
    _check(one, _expect(fem.PagedCache.empty(3, H, d, 64, TYPES[fmt]), k[5:6], v[5:6], slots[5:6]))


def test_write_e4m3_edges():
    """Rows of zeros, of subnormal and of the largest magnitudes, ties, one outlier, infinities and NaN."""
    d = 64
    rows = []
    rows.append(torch.zeros(d))
    rows.append(torch.full((d,), 2.0 ** -130))               # far under the smallest scale: all codes 0
    rows.append(torch.linspace(-1, 1, d) * 2.0 ** -100)
    rows.append(torch.full((d,), 3.38e38))                   # bf16's largest
    rows.append(torch.linspace(-1, 1, d) * 2.0 ** 127)
    rows.append(torch.arange(d).float() + 0.5)               # ties at the larger codes
    rows.append(torch.full((d,), 448.0))
    rows.append(torch.full((d,), 450.0))                     # one bf16 step past 448
    rows.append(torch.cat([torch.full((1,), 1000.0), torch.full((d - 1,), 1e-3)]))
    rows.append(torch.cat([torch.full((1,), math.inf), torch.ones(d - 1)]))
    rows.append(torch.cat([torch.ones(d - 1), torch.full((1,), math.nan)]))
    rows.append(torch.cat([torch.ones(d - 1), torch.full((1,), -math.inf)]))
    k = torch.stack(rows).to(torch.bfloat16).to(DEV)[:, None]
    v = (-k).contiguous()
    cache = fem.PagedCache.empty(1, 1, d, 16, torch.float8_e4m3fn)
    slots = torch.arange(len(rows), device=DEV)
    want = _expect(cache, k, v, slots)
    fem.fem_cache_write(cache, k, v, slots)
    _check(cache, want)
    table = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    gk, gv = fem.fem_cache_gather(cache, table, torch.zeros(1, dtype=torch.int32, device=DEV),
                                  torch.tensor([0, len(rows)], dtype=torch.int32, device=DEV), len(rows))
    for got, (t, e) in ((gk, want[0]), (gv, want[1])):
        ref = R.values(t, e)[0, 0, :len(rows)]
        assert torch.equal(torch.isnan(got[:, 0]), torch.isnan(ref))
        assert torch.isfinite(got[:9]).all()
        assert torch.equal(torch.nan_to_num(got[:, 0].double()), torch.nan_to_num(ref))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("H,d,page,lens", [(1, 16, 16, [1]), (3, 64, 32, [1, 31, 32, 33]), (8, 128, 64, [200, 0, 65, 1]),
                                           (2, 256, 256, [300, 511]), (5, 96, 128, [129, 7])])
def test_gather(fmt, H, d, page, lens):
    need = [-(-x // page) for x in lens]
    pages = sum(need) + 2
    cache = fem.PagedCache.empty(pages, H, d, page, TYPES[fmt])
    N = pages * page
    k, v = (_tokens(N, H, d, cache.row_dtype, 5 * N + i) for i in range(2))
    fem.fem_cache_write(cache, k, v, torch.arange(N, device=DEV))
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(d)).to(torch.int32)
    table, at = torch.full((len(lens), max(need)), -7, dtype=torch.int32), 0
    for s, m in enumerate(need):
        table[s, :m] = order[at:at + m]
        at += m
    table = table.to(DEV)
    starts = [x // 3 for x in lens]
    counts = [x - s for x, s in zip(lens, starts)]
    offsets = torch.tensor([sum(counts[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
    total = sum(counts)
    gk, gv = fem.fem_cache_gather(cache, table, torch.tensor(starts, dtype=torch.int32, device=DEV), offsets, total)
    fem.check_device_error()
    for got, which in ((gk, "k"), (gv, "v")):
        ref = torch.cat([R.sequence(cache, which, table[s], x)[0][:, starts[s]:].transpose(0, 1)
                         for s, x in enumerate(lens) if x])
        assert torch.equal(got.double(), ref)


def test_long_cache_offsets_pass_32_bits():
    """Pages past 2^31 elements (and 2^32 bytes) of a cache are written and read at their own place."""
    H, d, page = 8, 128, 64
    pages = (1 << 31) // (H * d * page) + 40
    k = torch.empty((pages, H, page, d), dtype=torch.bfloat16, device=DEV)
    cache = fem.PagedCache(k, torch.empty_like(k))
    at = [0, 1, pages - 1, pages - 2, (1 << 31) // (H * d * page)]
    for p in at:
        k[p].zero_()
    N = 5 * page
    new = _tokens(N, H, d, torch.bfloat16, 1)
    slots = torch.cat([torch.arange(page) + p * page for p in at]).to(DEV)
    fem.fem_cache_write(cache, new, (new * 2).contiguous(), slots)
    table = torch.tensor([at], dtype=torch.int32, device=DEV)
    gk, gv = fem.fem_cache_gather(cache, table, torch.zeros(1, dtype=torch.int32, device=DEV),
                                  torch.tensor([0, N], dtype=torch.int32, device=DEV), N)
    fem.check_device_error()
    assert torch.equal(gk, new) and torch.equal(gv, new * 2)
    assert torch.equal(k[at[2]].transpose(0, 1), new[2 * page:3 * page])


def test_nothing_to_do():
    cache = fem.PagedCache.empty(2, 2, 64, 16)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    fem.fem_cache_write(cache, none, none, torch.empty(0, dtype=torch.int64, device=DEV))
    z = torch.zeros(1, dtype=torch.int32, device=DEV)
    k, v = fem.fem_cache_gather(cache, z[None], z, torch.zeros(2, dtype=torch.int32, device=DEV), 0)
    assert k.shape == (0, 2, 64)
    fem.check_device_error()


def test_slots_and_pages_outside_are_left_out_and_reported():
    cache = fem.PagedCache.empty(2, 2, 64, 16, torch.float8_e4m3fn)
    k = _tokens(3, 2, 64, torch.bfloat16, 0, spread=False)
    slots = torch.tensor([1, 32, -3], device=DEV)
    want = _expect(cache, k, k, slots)
    fem.fem_cache_write(cache, k, k, slots)
    with pytest.raises(fem.FemError) as e:
        fem.check_device_error()
    assert e.value.status == 1
    _check(cache, want)
    table = torch.tensor([[0, 5]], dtype=torch.int32, device=DEV)
    gk, _ = fem.fem_cache_gather(cache, table, torch.zeros(1, dtype=torch.int32, device=DEV),
                                 torch.tensor([0, 20], dtype=torch.int32, device=DEV), 20)
    with pytest.raises(fem.FemError):
        fem.check_device_error()
    fem.check_device_error()  # the word is cleared
    assert torch.count_nonzero(gk[16:]).item() == 0 and torch.count_nonzero(gk[1]).item() > 0


def test_write_runs_on_the_given_stream():
    cache = fem.PagedCache.empty(4, 4, 128, 64)
    k = _tokens(100, 4, 128, torch.bfloat16, 2)
    slots = torch.arange(100, device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    fem.fem_cache_write(cache, k, k, slots, stream=side)
    side.synchronize()
    _check(cache, _expect(fem.PagedCache.empty(4, 4, 128, 64), k, k, slots))
