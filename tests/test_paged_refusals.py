"""What the paged-cache entry points refuse, on the host and before any CUDA call (CPU only)."""
import ctypes

import pytest
import torch

from paper_2602_07160_gb300 import build, fem


@pytest.fixture(scope="module")
def lib():
    build.build()
    return fem.load()


P = lambda x: ctypes.c_void_p(x) if x else None  # noqa: E731  fake, never dereferenced


def _cache(**kw):
    a = dict(k=16, v=16, k_exp=0, v_exp=0, format=0, num_pages=4, H=2, page_size=64, d=64)
    a.update(kw)
    return ctypes.byref(fem._CacheStruct(*(a[n] for n, _ in fem._CacheStruct._fields_)))


BAD_CACHES = [(dict(k=0), 1), (dict(v=0), 1), (dict(k=24), 1), (dict(format=3), 1), (dict(format=-1), 1),
              (dict(num_pages=0), 1), (dict(H=0), 1), (dict(d=0), 1), (dict(page_size=0), 1), (dict(format=1), 1),
              (dict(format=1, k_exp=16), 1), (dict(k_exp=16), 1), (dict(page_size=48), 2), (dict(page_size=8), 2),
              (dict(page_size=512), 2), (dict(d=72), 2), (dict(d=272), 2), (dict(H=70000), 2)]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_cache_errors_are_synchronous(lib, bad, code):
    c = _cache(**bad)
    assert lib.fem_cache_write(c, P(16), P(16), 64, 64, 64, 64, P(16), 1, None) == code
    assert lib.fem_cache_gather(c, P(16), 1, P(16), P(16), 1, P(16), P(16), 1, None) == code
    assert lib.fem_paged_read(c, P(16), 64, 64, None, P(16), P(16), P(16), 1, 1, 1, 2, 1, 1, P(16), None, None) == code


def test_null_cache(lib):
    assert lib.fem_cache_write(None, P(16), P(16), 64, 64, 64, 64, P(16), 1, None) == 1


def test_write_argument_errors(lib):
    def call(k=16, v=16, sn=128, sh=64, slots=16, N=1):
        return lib.fem_cache_write(_cache(), P(k), P(v), sn, sh, 128, 64, P(slots), N, None)
    assert call(k=0) == 1 and call(v=0) == 1 and call(slots=0) == 1 and call(N=-1) == 1
    assert call(k=24) == 1 and call(slots=20) == 1
    assert call(sn=100) == 1 and call(sh=4) == 1 and call(sn=-128) == 1
    assert call(N=0) == 0 and call(k=0, v=0, slots=0, N=0) == 0


def test_gather_argument_errors(lib):
    def call(table=16, pages=1, starts=16, offsets=16, S=1, k=16, v=16, total=1):
        return lib.fem_cache_gather(_cache(), P(table), pages, P(starts), P(offsets), S, P(k), P(v), total, None)
    assert call(table=0) == 1 and call(pages=0) == 1 and call(starts=0) == 1 and call(offsets=0) == 1
    assert call(S=0) == 1 and call(k=0) == 1 and call(v=0) == 1 and call(k=8) == 1 and call(total=-1) == 1
    assert call(total=0, k=0, v=0) == 0


def test_read_argument_errors(lib):
    def call(q=16, sn=128, sh=64, beta=0, off=16, ctx=16, table=16, pages=1, S=1, N=1, Hq=4, max_q=1, causal=1, out=16,
             lse=0):
        return lib.fem_paged_read(_cache(), P(q), sn, sh, P(beta), P(off), P(ctx), P(table), pages, S, N, Hq, max_q,
                                  causal, P(out), P(lse), None)
    for bad in (dict(q=0), dict(off=0), dict(ctx=0), dict(table=0), dict(out=0), dict(pages=0), dict(S=0), dict(N=-1),
                dict(Hq=0), dict(Hq=3), dict(max_q=-1), dict(causal=2), dict(q=24), dict(out=8), dict(beta=18),
                dict(lse=18), dict(sn=4), dict(sh=-64)):
        assert call(**bad) == 1, bad
    assert call(N=(1 << 31) - 1) == 2
    assert call(N=0, q=0, out=0) == 0


def test_the_binding_checks_its_tensors():
    k = torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        fem.PagedCache(k, k)                                # not on a GPU
    with pytest.raises(ValueError):
        fem.PagedCache(k, k[:1])
    with pytest.raises(ValueError):
        fem.PagedCache(k.half(), k.half())
    with pytest.raises(ValueError):
        fem.PagedCache(k, k, k_exp=torch.zeros((2, 2, 16), dtype=torch.uint8))
    with pytest.raises(ValueError):
        fem.PagedCache(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn))
