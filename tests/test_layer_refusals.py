"""What the entry points around the read refuse, on the host and before any CUDA call (CPU only)."""
import ctypes
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref


@pytest.fixture(scope="module")
def lib():
    build.build()
    return fem.load()


P = lambda x: ctypes.c_void_p(x) if x else None  # noqa: E731  fake, never dereferenced


def heads(p=16, sb=0, st=256, sh=64):
    return None if p is None else fem._heads_bytes(p, sb, st, sh)


def test_rope_arguments(lib):
    def call(q=heads(), qo=heads(), Hq=4, k=heads(), ko=heads(), Hk=2, B=1, T=3, d=64, type=0, turns=16, rotary=64,
             inter=0, pos=16, inverse=0):
        return lib.fem_rope(q, qo, Hq, k, ko, Hk, B, T, d, type, P(turns), rotary, inter, 1.0, P(pos), inverse, None)
    for bad in (dict(q=None), dict(qo=None), dict(q=heads(0)), dict(qo=heads(0)), dict(k=heads(0)), dict(ko=None),
                dict(q=heads(17)), dict(q=heads(18), type=2), dict(q=heads(st=-1)), dict(qo=heads(st=0)), dict(qo=heads(sh=0)),
                dict(ko=heads(sh=0)), dict(B=2), dict(Hq=0), dict(Hk=0), dict(B=-1), dict(T=-1), dict(d=0), dict(type=1),
                dict(type=3), dict(turns=0), dict(turns=20), dict(rotary=0), dict(rotary=63), dict(rotary=66), dict(inter=2),
                dict(pos=18), dict(inverse=-1)):
        assert call(**bad) == 1, bad
    assert call(d=1026) == 2
    assert call(B=1 << 16, T=1 << 16) == 2
    assert call(T=0) == 0 and call(B=0) == 0 and call(T=0, q=None, qo=None) == 0


def test_rope_turns(lib):
    table = (ctypes.c_uint64 * 512)()

    def call(rotary=64, base=10000.0, scaling=0, factor=2.0, context=4096.0, low=1.0, high=32.0, t=table):
        return lib.fem_rope_turns(rotary, base, scaling, factor, context, low, high, t)
    inf, nan = math.inf, math.nan
    for bad in (dict(rotary=0), dict(rotary=7), dict(rotary=1026), dict(base=0.0), dict(base=-1.0), dict(base=inf),
                dict(base=nan), dict(scaling=-1), dict(scaling=4), dict(scaling=1, factor=0.0), dict(scaling=2, factor=nan),
                dict(scaling=3, context=0.0), dict(scaling=3, low=32.0), dict(scaling=3, high=inf), dict(t=None),
                dict(base=1e-300, scaling=1, factor=1e-300)):
        assert call(**bad) == 1, bad
    assert call(factor=nan, low=5.0, high=1.0) == 0  # a plain table asks for neither


@pytest.mark.parametrize("scaling", [None, "linear", "base", "parts"])
@pytest.mark.parametrize("rotary", [2, 20, 128])
def test_rope_turns_are_the_rates(lib, scaling, rotary):
    """The table in whole turns of 2^64 against the rates in 64 bits: three roundings of a double and one unit."""
    table = (ctypes.c_uint64 * (rotary // 2))()
    factor = 8.0
    assert lib.fem_rope_turns(rotary, 10000.0, fem.Rope.SCALINGS[scaling], factor, 4096.0, 1.0, 32.0, table) == 0
    for got, rate in zip(table, ref.rope_rates(rotary, 10000.0, scaling, factor).tolist()):
        want = rate / (2 * math.pi) % 1.0
        assert abs(got / 2.0 ** 64 - want) <= 8 * 2.0 ** -53 * want + 2.0 ** -64


def test_recur_arguments(lib):
    def fwd(s=16, u=16, ss=8, us=8, off=0, S=2, T=4, N=8, C=8, type=0, mean=0, h0=0, hl=0, rows=0, num=2, h=16, hs=8):
        return lib.fem_recur_fwd(P(s), P(u), ss, us, P(off), S, T, N, C, type, mean, P(h0), P(hl), P(rows), num, P(h), hs, None)
    bad = (dict(s=0), dict(u=0), dict(h=0), dict(s=17), dict(h=18, type=2), dict(ss=-1), dict(hs=7), dict(hs=0), dict(off=18),
           dict(S=-1), dict(T=-1), dict(N=-1), dict(N=9), dict(C=0), dict(type=1), dict(mean=2), dict(h0=18), dict(hl=18),
           dict(rows=18), dict(h0=16, num=1), dict(hl=16, num=-1, rows=16))
    for b in bad:
        assert fwd(**b) == 1, b
    assert fwd(S=1 << 27, T=0, N=0) == 2
    for b in (dict(ss=1 << 20), dict(us=1 << 20), dict(hs=1 << 20), dict(C=1 << 20, ss=1 << 20, us=1 << 20, hs=1 << 20)):
        assert fwd(**b) == 2, b
    assert fwd(S=0, T=0, N=0, s=0, u=0, h=0) == 0

    def bwd(s=16, u=16, h=16, dh=16, st=8, off=0, S=2, T=4, N=8, C=8, type=0, mean=1, h0=0, dl=0, ds=16, du=16, dst=8, dh0=0):
        return lib.fem_recur_bwd(P(s), P(u), P(h), P(dh), st, 8, 8, 8, P(off), S, T, N, C, type, mean, P(h0), P(dl), P(ds), P(du),
                                 dst, 8, P(dh0), None)
    for b in (dict(s=0), dict(u=0), dict(h=0), dict(dh=0), dict(ds=0), dict(du=0), dict(st=-8), dict(dst=4), dict(h0=17),
              dict(dl=18), dict(dh0=18), dict(N=7), dict(mean=-1)):
        assert bwd(**b) == 1, b
    assert bwd(st=1 << 20) == 2 and bwd(dst=1 << 20) == 2
    assert bwd(S=0, T=0, N=0) == 0


def norm(**kw):
    a = dict(B=1, T=3, H=1, d=64, x_type=0, y_type=0, post=1, pre=1, gate_act=0, scale=1.0, eps=1e-6, w_post=0, b_post=0, w_pre=0,
             b_pre=0)
    a.update(kw)
    return fem._norm_bytes(*a.values())


BAD_NORMS = [(dict(B=-1), 1), (dict(T=-1), 1), (dict(H=0), 1), (dict(d=0), 1), (dict(x_type=1), 1), (dict(y_type=4), 1),
             (dict(x_type=0, y_type=2), 2), (dict(post=3), 1), (dict(pre=-1), 1), (dict(gate_act=3), 1), (dict(eps=0.0), 1),
             (dict(eps=-1.0), 1), (dict(eps=math.nan), 1), (dict(scale=math.inf), 1), (dict(w_post=18), 1), (dict(b_pre=17), 1),
             (dict(H=1, d=16385), 2), (dict(H=1 << 20, d=1 << 20), 2), (dict(B=1 << 16, T=1 << 16), 2)]


@pytest.mark.parametrize("bad,code", BAD_NORMS)
def test_norm_descriptions(lib, bad, code):
    n = norm(**bad)
    assert lib.fem_norm_fwd(n, P(16), heads(), None, P(16), P(16), None) == code
    assert lib.fem_norm_bwd(n, P(16), heads(), None, None, P(16), P(16), heads(), None, *[P(0)] * 4, None) == code


def test_norm_arguments(lib):
    def fwd(n=norm(), x=16, y=heads(), gate=None, r=16, z=16):
        return lib.fem_norm_fwd(n, P(x), y, gate, P(r), P(z), None)
    for b in (dict(n=None), dict(x=0), dict(x=17), dict(y=heads(0)), dict(y=heads(17)), dict(r=0), dict(r=17), dict(z=0),
              dict(z=17), dict(y=None, gate=heads()), dict(gate=heads(0)), dict(n=norm(pre=0)), dict(n=norm(pre=0), y=None, z=0),
              dict(y=heads(sh=-1))):
        assert fwd(**b) == 1, b
    assert fwd(n=norm(T=0), x=0, r=0, z=0) == 0

    def bwd(n=norm(), r=16, y=heads(), gate=None, dr=16, dz=16, dx=16, dy=heads(), dgate=None, wp=0, bp=0, wq=0, bq=0):
        return lib.fem_norm_bwd(n, P(r), y, gate, P(dr), P(dz), P(dx), dy, dgate, P(wp), P(bp), P(wq), P(bq), None)
    for b in (dict(n=None), dict(r=0), dict(dx=0), dict(dx=17), dict(dr=17), dict(dz=0), dict(dy=None), dict(y=None),
              dict(gate=heads()), dict(dgate=heads()), dict(dy=heads(st=0)), dict(wp=18), dict(y=None, dy=None, wp=16),
              dict(n=norm(pre=0), dz=0, wq=16), dict(n=norm(pre=0), dz=16)):
        assert bwd(**b) == 1, b
    assert bwd(n=norm(B=0)) == 0


def test_the_binding_checks_its_tensors():
    x = torch.zeros((4, 64))
    for call in (lambda: fem.fem_recur_fwd(x[None], x[None]), lambda: fem.fem_norm_fwd(fem.BlockNorm(64), x, x),
                 lambda: fem.fem_rope(fem.Rope(16, device="cpu"), x.view(4, 1, 64))):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError):
        fem.BlockNorm(64, post="batch")
    with pytest.raises(ValueError):
        fem.BlockNorm(0)
    with pytest.raises(ValueError):
        fem.BlockNorm(64, w_post=x[0])  # not on a GPU
    with pytest.raises(ValueError):
        fem.Rope(16, scaling="other", device="cpu")
    with pytest.raises(fem.FemError):
        fem.Rope(15, device="cpu")
