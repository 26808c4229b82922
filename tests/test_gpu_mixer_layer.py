"""The layer of examples/mixer_layer.py, all its operators together: its outputs and gradients against the same layer in
64 bits by automatic differentiation, and served against trained (needs a GB300).

Tolerances: the read is held to 1e-4 of its outputs' scale and its backward pass to 1e-4 of each gradient's (their own
tests); the products and the operators around them add a few hundred roundings of 2^-24, 2e-5.  An output goes through
one read, a gradient through the read, its backward pass and up to three products after them: 2e-4 and 5e-4 of scale.
"""
import importlib.util
import math
import os

import pytest
import torch

from paper_2602_07160_gb300 import build, fem
from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    build.build()
    fem.load()
    spec = importlib.util.spec_from_file_location("mixer_layer", os.path.join(ROOT, "examples", "mixer_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def plain_layer(layer, x, z, w):
    """The layer from its formulas, in 64 bits; w: its weights."""
    B, T, D = x.shape
    H, d = layer.H, layer.d
    s, u = torch.nn.functional.softplus(z @ w["w_rate"]), z @ w["w_in"]
    h, state = [], torch.zeros(B, layer.C, dtype=torch.float64, device=x.device)
    for t in range(T):
        a = torch.exp(-s[:, t])
        state = a * state + (1 - a) * u[:, t]
        h.append(state)
    c = z + torch.stack(h, 1) @ w["w_cond"]
    split = lambda y: y.view(B, T, H, d).transpose(1, 2)  # noqa: E731
    q, k, v = (split(y) for y in (c @ w["w_qkv"]).chunk(3, -1))
    pos = torch.arange(T, device=x.device).expand(B, T)
    q, k = (ref.rope(y, pos, ref.rope_rates(d // 2), True)[0] for y in (q, k))
    score = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(torch.ones(T, T, device=x.device).triu(1).bool(), -math.inf)
    prior = torch.log_softmax(score, -1)
    beta = w["beta"][None, :, None, :]
    top = v.amax(2, keepdim=True).detach()
    out = top + torch.log(torch.exp(prior) @ torch.exp(beta * (v - top))) / beta
    rows = lambda y: y.transpose(1, 2).reshape(B * T, D)  # noqa: E731
    gate = split(z @ w["w_gate"])
    r, z2 = ref.block(x.reshape(B * T, D), rows(out), rows(gate), {"b_post": None, **{n: w[n] for n in ("w_post", "w_pre", "b_pre")}},
                      "rms", "layer", "silu", 0.5, 1e-6)
    return r.view(B, T, D), z2.view(B, T, D)


@pytest.mark.parametrize("B,T,prompt", [(2, 70, 40), (1, 130, 129), (3, 33, 1)])
def test_layer(example, B, T, prompt):
    layer, (x, z, dr, dz2), got, grads, worst = example.run(B=B, T=T, H=3, d=16, C=20, prompt=prompt, seed=T)
    w = {n: t.double().requires_grad_(True) for n, t in
         [(n, getattr(layer, n)) for n in ("w_rate", "w_in", "w_cond", "w_qkv", "w_gate", "beta")] +
         [(n, layer.norm.weights[n]) for n in ("w_post", "w_pre", "b_pre")]}
    leaves = {"x": x.double().requires_grad_(True), "z": z.double().requires_grad_(True), **w}
    want = plain_layer(layer, leaves["x"], leaves["z"], w)
    for a, b in zip(got, want):
        assert (a - b).abs().max() <= 2e-4 * b.abs().max()
    exact = torch.autograd.grad((want[0] * dr).sum() + (want[1] * dz2).sum(), list(leaves.values()))
    assert set(grads) == set(leaves)
    for name, b in zip(leaves, exact):
        assert (grads[name] - b).abs().max() <= 5e-4 * b.abs().max(), name
    assert worst <= 2e-4 * max(t.abs().max().item() for t in got)


def test_command(example, capsys):
    example.main(["--tokens", "60", "--batch", "1"])
    assert "served token by token" in capsys.readouterr().out
