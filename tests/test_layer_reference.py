"""The formulas of the gradients around the read against differences of the forward passes, in 64 bits (CPU only)."""
import pytest
import torch

from tests import layer_reference as ref

F64 = torch.float64


def differences(f, x, g, step=1e-6):
    """Gradient of <g, f(x)> by central differences."""
    out = torch.zeros_like(x)
    for i in range(x.numel()):
        d = torch.zeros_like(x).view(-1)
        d[i] = step
        out.view(-1)[i] = ((f(x + d.view_as(x)) - f(x - d.view_as(x))) * g).sum() / (2 * step)
    return out


@pytest.mark.parametrize("mean", [False, True])
def test_recurrence(mean):
    gen = torch.Generator().manual_seed(1)
    lens, C = [3, 0, 1, 4], 2
    s = torch.rand((8, C), generator=gen, dtype=F64)
    u, dh = (torch.randn((8, C), generator=gen, dtype=F64) for _ in range(2))
    h0, dl = (torch.randn((4, C), generator=gen, dtype=F64) for _ in range(2))
    h, *_ = ref.recur(s, u, lens, h0, mean)
    (ds, du, dh0), _ = ref.recur_grads(s, u, h, dh, lens, h0, dl, mean)

    def both(s=s, u=u, h0=h0):
        h, last, *_ = ref.recur(s, u, lens, h0, mean)
        return torch.cat([h, last])
    g = torch.cat([dh, dl])
    assert torch.allclose(ds, differences(lambda v: both(s=v), s, g), atol=1e-7)
    assert torch.allclose(du, differences(lambda v: both(u=v), u, g), atol=1e-7)
    assert torch.allclose(dh0, differences(lambda v: both(h0=v), h0, g), atol=1e-7)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_back_is_the_gradient(interleaved):
    gen = torch.Generator().manual_seed(2)
    x, g = (torch.randn((3, 2, 10), generator=gen, dtype=F64) for _ in range(2))
    pos, rates = torch.tensor([0, -7, 1000]), ref.rope_rates(8)
    back, _ = ref.rope(g, pos, rates, interleaved, 1.25, inverse=True)
    want = differences(lambda v: ref.rope(v, pos, rates, interleaved, 1.25)[0], x, g, 1e-4)
    assert torch.allclose(back, want, atol=1e-8)


@pytest.mark.parametrize("kind", ["none", "rms", "layer"])
@pytest.mark.parametrize("act", ["identity", "sigmoid", "silu"])
def test_automatic_gradients_of_the_block(kind, act):
    """What the GPU's gradients are compared with."""
    gen = torch.Generator().manual_seed(3)
    x, y, gate, dr, dz = (torch.randn((2, 5), generator=gen, dtype=F64) for _ in range(5))
    w = {n: torch.randn(5, generator=gen, dtype=F64) for n in ("w_post", "b_post", "w_pre", "b_pre")}
    run = lambda y: torch.cat(ref.block(x, y, gate, w, kind, "layer", act, 0.5, 1e-3))  # noqa: E731
    leaf = y.clone().requires_grad_(True)
    got, = torch.autograd.grad(run(leaf), leaf, torch.cat([dr, dz]))
    assert torch.allclose(got, differences(run, y, torch.cat([dr, dz])), atol=1e-7)
