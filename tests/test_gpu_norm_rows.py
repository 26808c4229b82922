"""Norms over many rows on the GPU against 64-bit forms: every block goes round its loop more often than it has stages of
copies, with several rows of 32 to 512 threads at a time and a last round that is not full (needs a GB300).

Tolerances as in the norms' other tests; sums over rows of whole numbers are exact in any order.
"""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref
from tests.test_gpu_norm import TYPES, check_backward, check_forward, make, randn, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


@pytest.fixture(autouse=True)
def compared_on_the_gpu(monkeypatch):
    """The reference's comparison, where the tensors are."""
    def check(got, want, magnitude, units, dtype=None):
        half = ref.half_step(got.dtype if dtype is None else dtype)
        got, want, magnitude = got.double(), want.double(), magnitude.double()
        assert got.shape == want.shape
        over = ((got - want).abs() / (half * want.abs() + units * ref.UNIT * magnitude * (1 + half) + 1e-37)).nan_to_num(nan=math.inf)
        assert over.numel() > 0 and over.max() <= 1, (over.max().item(), over.argmax().item())
    monkeypatch.setattr(ref, "check", check)


# threads a row go by its length, and blocks take 1 to 20 rows at a time
SIZES = [(30011, 200), (30011, 203), (20003, 256), (20011, 384), (16001, 512), (10007, 768), (8005, 1000), (8009, 1001), (8017, 1024),
         (5003, 1536), (4001, 2000), (4003, 2001), (4007, 2048), (2003, 4096), (2011, 4097), (1009, 8192), (607, 8200)]


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("rows,D", SIZES)
def test_many_rows(rows, D, types):
    for kind, act in (("rms", "silu"), ("layer", "sigmoid")):
        block, t = make(rows, D, types, kind, kind, act, rows + D)
        run(block, t)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("shape", [(3, 16, 1367, 128), (2, 5, 3001, 25), (5, 6, 2003, 64)])
def test_many_rows_of_heads(shape, types):
    """Rows followed from one sequence into the next; heads that are copied in pieces, and heads read singly."""
    B, H, T, d = shape
    rows, D = B * T, H * d
    block, t = make(rows, D, types, "rms", "layer", "silu", 2, shape=shape)
    r, z = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    check_forward(block, t, r, z)
    check_backward(block, t, r, fem.fem_norm_bwd(block, r, t["y"], t["gate"], t["dr"], t["dz"]))


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("rows,D", SIZES)
def test_sums_of_whole_numbers(rows, D, types):
    """db_pre = sum dz, and without norms dw_post = sum dr y and db_post = sum dr: no row is left out or counted twice."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    xt, yt = TYPES[types]
    whole = lambda t: torch.randint(-3, 4, (rows, D), generator=gen, device="cuda").to(t)  # noqa: E731
    x, y, dr, dz = whole(xt), whole(yt), whole(xt), whole(yt)
    ones, zeros = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    block = fem.BlockNorm(D, post="none", pre="none", w_post=ones, b_post=zeros)
    dx, dy, _, dw, db, *_ = fem.fem_norm_bwd(block, x, y, dr=dr)
    assert torch.equal(dx, dr) and torch.equal(dy, dr.to(yt))
    assert torch.equal(dw.double(), (dr.double() * y.double()).sum(0)) and torch.equal(db.double(), dr.double().sum(0))
    block = fem.BlockNorm(D, pre="layer", w_pre=ones, b_pre=zeros)
    assert torch.equal(fem.fem_norm_bwd(block, x, dr=dr, dz=dz)[6].double(), dz.double().sum(0))


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("rows,D", [(20011, 384), (8009, 1001), (4007, 2048), (2011, 4097)])
def test_many_rows_in_place(rows, D, types):
    """The stream over itself, its next rows under way; and dx over dr at the C entry."""
    block, t = make(rows, D, types, "rms", "rms", "silu", 3)
    r, z = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    want = fem.fem_norm_bwd(block, r, t["y"], t["gate"], t["dr"], t["dz"])
    x = t["x"].clone()
    got = fem.fem_norm_fwd(block, x, t["y"], t["gate"], out=x)
    assert torch.equal(x, r) and torch.equal(got[1], z)
    heads = lambda v: fem._heads_bytes(v.data_ptr(), 0, D, 0)  # noqa: E731
    dr, dy, dgate, sums = t["dr"].clone(), torch.empty_like(t["y"]), torch.empty_like(t["gate"]), [randn(torch.Generator(device="cuda"), D) for _ in range(4)]
    rc = fem.load().fem_norm_bwd(block._describe((1, rows, 1, D), *TYPES[types]), r.data_ptr(), heads(t["y"]), heads(t["gate"]), dr.data_ptr(),
                                 t["dz"].data_ptr(), dr.data_ptr(), heads(dy), heads(dgate), sums[0].data_ptr(), None, sums[2].data_ptr(), None,
                                 torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0
    for a, b in ((dr, want[0]), (dy, want[1]), (dgate, want[2]), (sums[0], want[3]), (sums[2], want[5])):
        assert torch.equal(a, b)
