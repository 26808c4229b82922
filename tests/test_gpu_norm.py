"""Norms fused with gate and residual, and their gradients, on the GPU against 64-bit forms (needs a GB300).

Tolerance: the output's half step, and a number of fp32 roundings of what goes into a value, every term by its
magnitude.  A row's sums take at most 16 additions in a thread and 10 more over threads, and a square root and a
division round 2 to 3 units each: a norm's factor is off by under 40 units, a normalised value by 64 with its own
subtractions and products, and a gradient, in which two sums and two factors meet, by 256.  An approximated sigmoid is
off by under 8 units.
"""
import math

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
FWD, BWD = 64, 256
NAMES = ("w_post", "b_post", "w_pre", "b_pre")
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "mixed": (torch.float32, torch.bfloat16), "f32": (torch.float32, torch.float32)}


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return fem.load()


def randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def make(rows, D, types, post, pre, act, seed, shape=None, bias=True, weights=True):
    """A block and its tensors; y and gate in `shape` where given."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    xt, yt = TYPES[types]
    shape = shape or (rows, D)
    w = {n: None for n in NAMES}
    for end, kind in (("post", post), ("pre", pre)):
        if weights:
            w["w_" + end] = 1 + 0.3 * randn(gen, D)
        if bias and kind == "layer":
            w["b_" + end] = 0.2 * randn(gen, D)
    block = fem.BlockNorm(D, post=post, pre=pre, gate=act, scale=0.7, eps=1e-5, **w)
    t = dict(x=(randn(gen, rows, D) * 2 + 0.3).to(xt), y=(randn(gen, *shape) + 0.2).to(yt),
             gate=None if act == "none" else randn(gen, *shape).mul_(2).to(yt), dr=randn(gen, rows, D).to(xt),
             dz=None if pre == "none" else randn(gen, rows, D).to(yt))
    return block, t


def as_rows(t):
    return None if t is None else (t if t.dim() == 2 else ref.rows_of(t)).double()


def norm_size(v, kind, eps, err):
    """Magnitude of the errors of a normalised row whose elements are off by `err` units each."""
    if kind == "none":
        return err
    c = v - v.mean(-1, keepdim=True) if kind == "layer" else v
    inv = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)
    spread = v.abs().mean(-1, keepdim=True) if kind == "layer" else 0.0
    unit = c * inv
    e = err + v.abs() + spread
    return inv * (e + e.mean(-1, keepdim=True) + unit.abs() * (unit.abs() * e).mean(-1, keepdim=True))


def check_forward(block, t, r, z):
    w = {n: None if v is None else v.double() for n, v in block.weights.items()}
    x, y, g = t["x"].double(), as_rows(t.get("y")), as_rows(t.get("gate"))
    want_r, want_z = ref.block(x, y, g, w, block.post, block.pre, block.gate, block.scale, block.eps)
    one = lambda n, none: none if w[n] is None else w[n].abs()  # noqa: E731
    size = x.abs()
    if y is not None:
        branch = norm_size(y, block.post, block.eps, y.abs()) * one("w_post", 1.0) + one("b_post", 0.0)
        size = size + block.scale * branch * (1.0 if g is None else ref._gate(g, block.gate).abs())
        ref.check(r, want_r, size, FWD)
    if block.pre != "none":
        out = norm_size(want_r, block.pre, block.eps, size) * one("w_pre", 1.0) + one("b_pre", 0.0)
        ref.check(z, want_z, out, FWD)


def check_backward(block, t, r, got, units=BWD):
    """Against automatic differentiation in 64 bits; magnitudes by the gradients' formulas."""
    leaf = {n: v.double().requires_grad_(True) for n, v in block.weights.items() if v is not None}
    w = {n: leaf.get(n) for n in NAMES}
    rr = r.double().requires_grad_(True)
    y, g = as_rows(t.get("y")), as_rows(t.get("gate"))
    for name, v in (("y", y), ("gate", g)):
        if v is not None:
            leaf[name] = v.requires_grad_(True)
    dr = t["dr"].double() if t["dr"] is not None else torch.zeros_like(rr)
    want, size = {}, {}
    dx, dxs = dr, dr.abs()
    rows = r.shape[0]
    depth = rows + 64.0  # additions that a weight's sum takes, at most, in units of the terms' magnitudes
    if block.pre != "none":
        dz = t["dz"].double()
        z = ref._norm(rr, block.pre, block.eps)
        unit = z.detach()
        f = dz * (1.0 if w["w_pre"] is None else w["w_pre"].detach())
        c = rr.detach() - (rr.detach().mean(-1, keepdim=True) if block.pre == "layer" else 0.0)
        rho = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + block.eps)
        grad, = torch.autograd.grad(z, rr, f)
        dx = dr + grad
        off = norm_size(rr.detach(), block.pre, block.eps, rr.detach().abs())  # what the unit row is off by
        dxs = dxs + rho * (f.abs() + f.abs().mean(-1, keepdim=True) + (unit.abs() + off) * (f.abs() * (unit.abs() + off)).mean(-1, keepdim=True))
        want["dw_pre"], size["dw_pre"] = (dz * unit).sum(0), (dz.abs() * (unit.abs() + off)).sum(0) * (1 + depth / units)
        want["db_pre"], size["db_pre"] = dz.sum(0), dz.abs().sum(0) * (1 + depth / units)
    want["dx"], size["dx"] = dx, dxs
    if y is not None:
        unit = ref._norm(y, block.post, block.eps)
        v = unit * (1.0 if w["w_post"] is None else w["w_post"]) + (0.0 if w["b_post"] is None else w["b_post"])
        if g is not None:
            v = v * ref._gate(g, block.gate)
        names = [n for n in ("y", "gate", "w_post", "b_post") if n in leaf]
        for n, grad in zip(names, torch.autograd.grad(block.scale * v, [leaf[n] for n in names], dx, retain_graph=True)):
            want["d" + n] = grad
        with torch.no_grad():
            unit, wp = unit.detach(), 1.0 if w["w_post"] is None else w["w_post"].detach().abs()
            bp = 0.0 if w["b_post"] is None else w["b_post"].detach().abs()
            off = norm_size(y, block.post, block.eps, y.abs())
            gate = torch.ones_like(y) if g is None else ref._gate(g, block.gate).abs()
            e = block.scale * dxs
            if g is not None:
                p = torch.sigmoid(g)
                slope = {"identity": torch.ones_like(g), "sigmoid": p * (1 - p), "silu": p * (1 + g.abs() * (1 - p))}[block.gate]
                size["dgate"] = e * ((unit.abs() + off) * wp + bp) * slope
            terms = e * gate * (unit.abs() + off)
            size["dw_post"] = terms.sum(0) * (1 + depth / units)
            size["db_post"] = (e * gate).sum(0) * (1 + depth / units)
            f = e * gate * wp
            if block.post == "none":
                size["dy"] = f
            else:
                c = y - (y.mean(-1, keepdim=True) if block.post == "layer" else 0.0)
                inv = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + block.eps)
                u = unit.abs() + off
                size["dy"] = inv * (f + f.mean(-1, keepdim=True) + u * (f * u).mean(-1, keepdim=True))
            if "dw_post" not in want:
                want["dw_post"] = (dx * block.scale * (1.0 if g is None else ref._gate(g, block.gate)) * unit).sum(0)
    names = ("dx", "dy", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")
    for name, value in zip(names, got):
        if value is None:
            assert name not in want or name.startswith("db"), name
            continue
        value = value if name not in ("dy", "dgate") or value.dim() == 2 else ref.rows_of(value)
        ref.check(value, want[name].detach(), size[name].detach(), units)


def run(block, t):
    r, z = fem.fem_norm_fwd(block, t["x"], t.get("y"), t.get("gate"))
    check_forward(block, t, r, z)
    got = fem.fem_norm_bwd(block, r, t.get("y"), t.get("gate"), t["dr"], t["dz"])
    check_backward(block, t, r, got)
    return r, z, got


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("rows,D", [(1, 1), (2, 8), (3, 197), (9, 256), (5, 384), (4, 512), (11, 768), (2, 1000), (7, 1024),
                                    (3, 1537), (5, 2048), (2, 4096), (2, 4097), (3, 8192), (1, 16384), (2, 16383), (700, 64)])
def test_sizes(rows, D, types):
    block, t = make(rows, D, types, "rms", "rms", "silu", rows + D)
    run(block, t)
    block, t = make(rows, D, types, "layer", "layer", "sigmoid", rows + D)
    run(block, t)


@pytest.mark.parametrize("post", ["none", "rms", "layer"])
@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("act", ["none", "identity", "sigmoid", "silu"])
@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_kinds(post, pre, act, types):
    for D in (320, 203):
        block, t = make(6, D, types, post, pre, act, 1)
        run(block, t)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("shape", [(10, 4, 64), (3, 6, 5, 64), (2, 5, 4, 25), (1, 3, 1, 128)])
def test_heads(shape, types):
    """y and gate as the reads give them: [N, H, d] and [B, H, T, d]."""
    rows, D = (shape[0], shape[1] * shape[2]) if len(shape) == 3 else (shape[0] * shape[2], shape[1] * shape[3])
    block, t = make(rows, D, types, "rms", "layer", "silu", 2, shape=shape)
    if len(shape) == 4:
        for n in ("x", "dr", "dz"):
            t[n] = t[n].view(shape[0], shape[2], D)
    r, z = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    got = fem.fem_norm_bwd(block, r, t["y"], t["gate"], t["dr"], t["dz"])
    assert r.shape == t["x"].shape and got[1].shape == shape and got[2].shape == shape
    flat = {n: v.view(rows, D) if n in ("x", "dr", "dz") else v for n, v in t.items()}
    check_forward(block, flat, r.view(rows, D), z.view(rows, D))
    check_backward(block, flat, r.view(rows, D), (got[0].view(rows, D), *got[1:]))


@pytest.mark.parametrize("lead,width", [(0, 200), (8, 272), (1, 199), (3, 203)])
def test_parts_of_a_projection(lead, width):
    """y and gate side by side in wider rows, at any element."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    wide = randn(gen, 9, 2 * width + 16).bfloat16()
    block, t = make(9, width, "bf16", "rms", "rms", "silu", 4)
    t["y"], t["gate"] = wide[:, lead:lead + width], wide[:, lead + width:lead + 2 * width]
    run(block, t)


@pytest.mark.parametrize("types", list(TYPES))
def test_without_weights_and_without_a_block(types):
    block, t = make(5, 640, types, "rms", "layer", "none", 5, weights=False, bias=False)
    run(block, t)
    block, t = make(5, 640, "f32" if types == "mixed" else types, "rms", "rms", "none", 6)
    t["y"] = None
    r, z, got = run(block, t)
    assert r is t["x"] and got[1] is None and got[3] is None and got[5] is not None


def test_no_gradient_past_the_next_block():
    block, t = make(5, 256, "bf16", "rms", "rms", "identity", 7)
    t["dr"] = None
    run(block, t)


def test_many_rows_of_sums():
    """More rows than blocks: every block's sums take several rows."""
    block, t = make(3000, 72, "f32", "layer", "layer", "silu", 8)
    run(block, t)


@pytest.mark.parametrize("post", ["rms", "layer"])
def test_rows_of_zeros_and_of_one_value(post):
    """A row without spread: the norm's factor is 1 / sqrt(eps), and a layer norm's output its bias."""
    block, t = make(4, 128, "f32", post, post, "none", 9)
    t["x"][0], t["y"][0] = 0, 0
    t["x"][1], t["y"][1] = 3, -2
    r, z, got = run(block, t)
    assert all(torch.isfinite(v).all() for v in (r, z, *got) if v is not None)


def test_far_means():
    """A layer norm takes its variance about the mean: values of 1000 with a spread of 1."""
    block, t = make(6, 512, "f32", "layer", "layer", "none", 10)
    t["x"] += 1000
    t["y"] += 1000
    run(block, t)


def test_nan_stays_in_its_row():
    block, t = make(40, 96, "bf16", "rms", "layer", "silu", 11)
    clean = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    t["y"][3, 5], t["x"][7, 1] = math.nan, math.inf
    got = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    rows = [i for i in range(40) if i not in (3, 7)]
    for a, b in zip(got, clean):
        assert torch.equal(a[rows], b[rows]) and not torch.isfinite(a[[3, 7]]).all()
    back = fem.fem_norm_bwd(block, got[0], t["y"], t["gate"], t["dr"], t["dz"])
    again = fem.fem_norm_bwd(block, clean[0], t["y"].nan_to_num(), t["gate"], t["dr"], t["dz"])
    for a, b in zip(back[:3], again[:3]):
        assert torch.equal(a[rows], b[rows])


def test_in_place():
    block, t = make(33, 384, "bf16", "rms", "rms", "silu", 12)
    want = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    z = torch.empty_like(t["x"])
    got = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"], out=t["x"], z_out=z)
    assert got[0] is t["x"] and torch.equal(t["x"], want[0]) and torch.equal(z, want[1])


def test_the_same_bits_again_and_graphs():
    """Fixed orders of summation; two captured backward passes have workspaces of their own."""
    block, t = make(2000, 200, "bf16", "rms", "rms", "silu", 13)
    r, _ = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    call = lambda: fem.fem_norm_bwd(block, r, t["y"], t["gate"], t["dr"], t["dz"])  # noqa: E731
    want = call()
    assert all(a is b or torch.equal(a, b) for a, b in zip(call(), want))
    side = [torch.cuda.Stream() for _ in range(2)]
    graphs, kept = [], []
    torch.cuda.synchronize()
    for stream in side:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            kept.append(call())
        graphs.append(graph)
    t["dz"].neg_()
    want = call()
    torch.cuda.synchronize()
    for graph, stream in zip(graphs, side):
        with torch.cuda.stream(stream):
            graph.replay()
    torch.cuda.synchronize()
    for got in kept:
        assert all(a is b or torch.equal(a, b) for a, b in zip(got, want))


def test_another_stream():
    block, t = make(500, 512, "bf16", "rms", "rms", "silu", 14)
    want = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    back = fem.fem_norm_bwd(block, want[0], t["y"], t["gate"], t["dr"], t["dz"])
    side = torch.cuda.Stream()
    late = [torch.empty_like(v) for v in (*want, *back) if v is not None]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    for v in late:
        v.fill_(7)
    del late, v
    got = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"], stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    again = fem.fem_norm_bwd(block, want[0], t["y"], t["gate"], t["dr"], t["dz"], stream=side)
    torch.cuda.synchronize()
    assert all(a is b or torch.equal(a, b) for a, b in zip(again, back))


def test_empty_calls():
    block, t = make(0, 64, "bf16", "layer", "layer", "silu", 15)
    r, z = fem.fem_norm_fwd(block, t["x"], t["y"], t["gate"])
    assert r.shape == z.shape == (0, 64)
    got = fem.fem_norm_bwd(block, r, t["y"], t["gate"], t["dr"], t["dz"])
    assert all(v.shape == (64,) and not v.any() for v in got[3:])


def test_rows_past_32_bits():
    """2^31 elements and more: the last rows as in a call of their own."""
    rows, D = (1 << 18) + 5, 8200
    block, _ = make(1, D, "bf16", "rms", "rms", "none", 16)
    x = torch.empty((rows, D), dtype=torch.bfloat16, device="cuda").normal_()
    r, z = fem.fem_norm_fwd(block, x, x)
    want = fem.fem_norm_fwd(block, x[-7:].contiguous(), x[-7:].contiguous())
    assert torch.equal(r[-7:], want[0]) and torch.equal(z[-7:], want[1])
    back = fem.fem_norm_bwd(block, r, x, None, z, z)
    want = fem.fem_norm_bwd(block, r[-7:].contiguous(), x[-7:].contiguous(), None, z[-7:].contiguous(), z[-7:].contiguous())
    assert torch.equal(back[0][-7:], want[0]) and torch.equal(back[1][-7:], want[1])


def test_weights_are_read_at_each_call():
    """Changed in place, and replaced behind the tensor."""
    block, t = make(40, 64, "bf16", "rms", "rms", "none", 18)
    before, _ = fem.fem_norm_fwd(block, t["x"], t["y"])
    for change in (lambda w: w.mul_(2), lambda w: setattr(w, "data", torch.full((64,), 3.0, device="cuda"))):
        change(block.weights["w_post"])
        same = fem.BlockNorm(64, scale=0.7, eps=1e-5, **{n: None if w is None else w.clone() for n, w in block.weights.items()})
        got, want = (fem.fem_norm_fwd(b, t["x"], t["y"]) for b in (block, same))
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and not torch.equal(got[0], before)


@pytest.mark.parametrize("D", [1000, 1001, 200])
def test_an_infinite_weight_stays_in_its_channel(D):
    """Threads with no channel have no weight either."""
    block, t = make(5, D, "f32", "rms", "none", "none", 19, weights=True)
    fine, _ = fem.fem_norm_fwd(block, t["x"], t["y"])
    fine_grads = fem.fem_norm_bwd(block, fine, t["y"], None, t["dr"])
    block.weights["w_post"][0] = math.inf
    r, _ = fem.fem_norm_fwd(block, t["x"], t["y"])
    assert torch.equal(r[:, 1:], fine[:, 1:]) and torch.isinf(r[:, 0]).all()
    dx, dy, _, dw, *_ = fem.fem_norm_bwd(block, r, t["y"], None, t["dr"])
    assert torch.equal(dx, fine_grads[0]) and torch.equal(dw, fine_grads[3])
    pre, t = make(5, D, "f32", "none", "rms", "none", 20)
    _, z0 = fem.fem_norm_fwd(pre, t["x"])
    pre.weights["w_pre"][0] = math.inf
    _, z = fem.fem_norm_fwd(pre, t["x"])
    assert torch.equal(z[:, 1:], z0[:, 1:])


def test_some_of_the_weights_gradients():
    """At the C entry each of them may be left out, and all."""
    rows, D = 300, 256
    block, t = make(rows, D, "f32", "layer", "layer", "silu", 21)
    x, y, g, dr, dz = (t[n] for n in ("x", "y", "gate", "dr", "dz"))
    want = fem.fem_norm_bwd(block, x, y, g, dr, dz)
    describe = block._describe((1, rows, 1, D), torch.float32, torch.float32)
    heads = lambda v: fem._heads_bytes(v.data_ptr(), 0, D, 0)
    for keep in ((), (0,), (1,), (2,), (3,), (0, 2), (1, 3)):
        got = [torch.empty_like(x) for _ in range(3)]
        sums = [torch.empty(D, device="cuda") if i in keep else None for i in range(4)]
        rc = fem.load().fem_norm_bwd(describe, x.data_ptr(), heads(y), heads(g), dr.data_ptr(), dz.data_ptr(), got[0].data_ptr(),
                                     heads(got[1]), heads(got[2]), *(None if s is None else s.data_ptr() for s in sums),
                                     torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert rc == 0 and all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(s is None or torch.equal(s, b) for s, b in zip(sums, want[3:]))


def test_refusals():
    block, t = make(6, 64, "bf16", "rms", "rms", "silu", 17)
    x, y, g = t["x"], t["y"], t["gate"]
    for bad in (dict(x=x.half()), dict(x=x[:, :32]), dict(x=x.t()), dict(y=y.half()), dict(y=y[:5]), dict(gate=None), dict(gate=g.float()),
                dict(gate=g[:5]), dict(y=None), dict(y=y.view(2, 3, 64)), dict(out=x[:5]), dict(z_out=x.float())):
        with pytest.raises(ValueError):
            fem.fem_norm_fwd(block, **{**dict(x=x, y=y, gate=g), **bad})
    with pytest.raises(fem.FemError):
        fem.fem_norm_fwd(block, x, y.float(), g.float())  # a bf16 stream of a float32 branch
    with pytest.raises(ValueError):
        fem.fem_norm_bwd(block, x, y, g, t["dr"])
    with pytest.raises(ValueError):
        fem.fem_norm_bwd(block, x, y, g, t["dr"][:5], t["dz"])
