"""The binding of the operators around the read against a stand-in library and stand-in devices (CPU only)."""
import copy
import types

import pytest
import torch

from paper_2602_07160_gb300 import fem

D = 64


class Library:
    """Takes every call and does nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    """Host tensors, whose device index is -1, pass for those of the current device."""
    lib = Library()
    monkeypatch.setattr(fem, "load", lambda: lib)
    monkeypatch.setattr(fem, "_current", lambda index: None)
    monkeypatch.setattr(fem, "_stream_number", lambda stream, index: 0)
    return lib


class Weight:
    """What BlockNorm looks at of a CUDA parameter; `data` is what a module replaces when it changes type or device."""

    def __init__(self, data, index=-1):
        self.data, self.index = data, index

    device = types.SimpleNamespace(type="cuda")
    dtype = property(lambda self: self.data.dtype)
    shape = property(lambda self: self.data.shape)
    get_device = lambda self: self.index  # noqa: E731
    is_contiguous = lambda self: self.data.is_contiguous()  # noqa: E731
    data_ptr = lambda self: self.data.data_ptr()  # noqa: E731


CHANGES = {"bf16": lambda w: setattr(w, "data", w.data.bfloat16()), "shorter": lambda w: setattr(w, "data", w.data[:D - 1].clone()),
           "longer": lambda w: setattr(w, "data", torch.ones(D + 1)), "of two axes": lambda w: setattr(w, "data", w.data.view(1, D)),
           "strided": lambda w: setattr(w, "data", torch.ones(2 * D)[::2]), "elsewhere": lambda w: setattr(w, "index", 0)}


@pytest.mark.parametrize("name", ["w_post", "b_post", "w_pre", "b_pre"])
@pytest.mark.parametrize("change", list(CHANGES))
def test_a_weight_that_changed_is_refused(library, name, change):
    """`module.bfloat16()` and `module.cpu()` replace what is behind a parameter that the object keeps."""
    weights = {n: Weight(torch.ones(D)) for n in ("w_post", "b_post", "w_pre", "b_pre")}
    block = fem.BlockNorm(D, **weights)
    x = torch.zeros((3, D))
    calls = (lambda: fem.fem_norm_fwd(block, x, x), lambda: fem.fem_norm_bwd(block, x, x, dz=x))
    for call in calls:
        call()
    assert library.calls == ["fem_norm_fwd", "fem_norm_bwd"]
    CHANGES[change](weights[name])
    for call in calls:
        with pytest.raises(ValueError, match=name):
            call()
    assert library.calls == ["fem_norm_fwd", "fem_norm_bwd"]


@pytest.mark.parametrize("name,value", [("width", 32), ("post", "layer"), ("pre", "none"), ("gate", "silu"), ("scale", 2.0), ("eps", 1e-3),
                                        ("index", 0), ("weights", {})])
def test_a_norm_stays_as_it_was_made(name, value):
    """Its calls take what the constructor made of these: a later assignment would be half seen."""
    block = fem.BlockNorm(D, w_post=Weight(torch.ones(D)))
    before = getattr(block, name)
    with pytest.raises(AttributeError):
        setattr(block, name, value)
    assert getattr(block, name) == before
    with pytest.raises(TypeError):
        block.weights["b_pre"] = Weight(torch.ones(D))


def test_a_copied_norm_reads_its_own_weights(library):
    block = fem.BlockNorm(D, w_post=Weight(torch.ones(D)))
    twin = copy.deepcopy(block)
    assert twin.weights["w_post"] is not block.weights["w_post"]
    assert twin._addresses() == [twin.weights["w_post"].data_ptr(), 0, 0, 0] != block._addresses()


@pytest.mark.parametrize("name,value", [("rotary_dim", 128), ("interleaved", 1), ("amplitude", 2.0), ("turns", None), ("index", 0)])
def test_a_rope_stays_as_it_was_made(name, value):
    """Its table has a rate for each of the pairs that it was made for, and the kernel reads one for each that a call names."""
    rope = fem.Rope(16, device="cpu")
    before = getattr(rope, name)
    with pytest.raises(AttributeError):
        setattr(rope, name, value)
    assert getattr(rope, name) is before


M = 1 << 32
BF16 = torch.bfloat16


def far(*shape, dtype=BF16):
    """A tensor of any size, without its memory."""
    return torch.empty(shape, dtype=dtype, device="meta")


ROPE_SIZES = [((M, 1, 16), None), ((1, M, 16), None), ((M + 3, 2, 16), (M + 3, 1, 16)), ((3, 2, 16), (3, M + 1, 16)), ((M, 1, 3, 16), None),
              ((1, 2, M + 3, 16), None), ((1, 2, 3, M + 16), None)]


@pytest.mark.parametrize("q,k", ROPE_SIZES)
def test_rope_sizes_past_32_bits_are_refused(library, q, k):
    """The C entry takes 32 bits of each: what a call had beyond them was left out without an error."""
    rope = fem.Rope.__new__(fem.Rope)
    rope.__dict__.update(turns=far(8, dtype=torch.int64), index=-1, rotary_dim=16, interleaved=0, amplitude=1.0)
    with pytest.raises(fem.FemError) as error:
        fem.fem_rope(rope, far(*q), None if k is None else far(*k))
    assert error.value.status == 2 and library.calls == []
    with pytest.raises(fem.FemError):
        fem.Rope(M + 16, device="cpu")


RECUR_SIZES = [((1, M, 16), None), ((M + 3, 1, 16), None), ((3, 2, M + 16), None), ((M + 40, 16), 3), ((40, M + 16), 3),
               ((1 << 16, 1 << 16, 16), None)]


@pytest.mark.parametrize("shape,seqs", RECUR_SIZES)
def test_recurrence_sizes_past_32_bits_are_refused(library, shape, seqs):
    s = far(*shape)
    offsets = None if seqs is None else far(seqs + 1, dtype=torch.int32)
    for call in (lambda: fem.fem_recur_fwd(s, s, offsets=offsets, state_out=False), lambda: fem.fem_recur_bwd(s, s, s, s, offsets=offsets)):
        with pytest.raises(fem.FemError) as error:
            call()
        assert error.value.status == 2 and library.calls == []


def test_more_states_or_sequences_than_32_bits_are_refused(library):
    s, offsets = far(40, 16), far(4, dtype=torch.int32)
    pool, rows = far(M + 5, 16, dtype=torch.float32), far(3, dtype=torch.int32)
    for call in (lambda: fem.fem_recur_fwd(s, s, offsets=offsets, h0=pool, state_rows=rows),
                 lambda: fem.fem_recur_fwd(s, s, offsets=offsets, state_rows=rows, state_out=pool),
                 lambda: fem.fem_recur_fwd(s, s, offsets=far(M + 3, dtype=torch.int32))):
        with pytest.raises(fem.FemError) as error:
            call()
        assert error.value.status == 2 and library.calls == []


def test_a_bound_past_32_bits_is_still_a_bound(library, monkeypatch):
    """max_len bounds the lengths from above: more than there can be is no more than that."""
    s, offsets = far(40, 16), far(4, dtype=torch.int32)
    seen = []
    monkeypatch.setattr(library, "fem_recur_fwd", lambda *a: seen.append(a[6]) or 0, raising=False)
    for bound in (40, (1 << 31) - 1, M + 8):
        fem.fem_recur_fwd(s, s, offsets=offsets, max_len=bound)
    assert seen == [40, (1 << 31) - 1, (1 << 31) - 1]


@pytest.mark.parametrize("shape,y", [((M, 16), None), ((2, M // 2, 16), (2, 4, M // 2, 4)), ((M, 16), (M, 4, 4)), ((3, M + 16), None)])
def test_norm_sizes_past_32_bits_are_refused(library, shape, y):
    block = fem.BlockNorm(shape[-1])
    x = far(*shape)
    y = x if y is None else far(*y)
    for call in (lambda: fem.fem_norm_fwd(block, x, y), lambda: fem.fem_norm_bwd(block, x, y, dz=x)):
        with pytest.raises(fem.FemError) as error:
            call()
        assert error.value.status == 2 and library.calls == []


@pytest.mark.parametrize("shape", [(1, M, 1), (M + 2, 3, 1), (2, 3, M + 1)])
def test_conditioner_sizes_past_32_bits_are_refused(library, monkeypatch, shape):
    """The dense convolution of the recurrence's kind, through the same 32 bits."""
    monkeypatch.setattr(torch.Tensor, "device", types.SimpleNamespace(type="cuda"))
    s = far(*shape, dtype=torch.float32)
    with pytest.raises(fem.FemError) as error:
        fem.fem_tdc_conv(s, s, out=s, stream=types.SimpleNamespace(cuda_stream=0))
    assert error.value.status == 2 and library.calls == []
