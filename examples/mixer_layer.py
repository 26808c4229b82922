"""One mixer layer trained and served: what stands around the read, put together.

    python examples/mixer_layer.py [--tokens 200] [--batch 2]

A layer takes the residual stream x and its normed copy z. A conditioner's gated recurrence over z joins z before the
projection to queries, keys and values; rotary positions turn queries and keys; the free-energy read mixes; the block's
output is normed, gated and added to the stream, and the next layer's input normed, in one pass. ``forward`` and
``backward`` are the training step (fp32, whole sequences), ``serve`` the same layer over a paged cache and a pool of the
conditioner's states, a chunk of the prompts and then a token at a time. Weights are random, hidden states synthetic.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_07160_gb300 import fem  # noqa: E402


class Layer:
    """Weights of one layer: H heads of d, a conditioner of C channels."""

    def __init__(self, H, d, C, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        D = H * d
        normal = lambda *shape: torch.randn(shape, generator=g, device=device)  # noqa: E731
        self.H, self.d, self.C, self.D = H, d, C, D
        self.w_rate, self.w_in = normal(D, C) / D ** 0.5, normal(D, C) / D ** 0.5
        self.w_cond = 0.3 * normal(C, D) / C ** 0.5
        self.w_qkv, self.w_gate = normal(D, 3 * D) / D ** 0.5, normal(D, D) / D ** 0.5
        self.beta = torch.nn.functional.softplus(1.8 + 0.3 * normal(H, d))
        self.rope = fem.Rope(d // 2, interleaved=True, device=device)
        self.norm = fem.BlockNorm(D, post="rms", pre="layer", gate="silu", w_post=1 + 0.1 * normal(D), w_pre=1 + 0.1 * normal(D),
                                  b_pre=0.1 * normal(D), scale=0.5)


def heads(x, layer):
    """[B, T, H d] as [B, H, T, d], a view."""
    return x.view(*x.shape[:2], layer.H, layer.d).transpose(1, 2)


def forward(layer, x, z):
    """x, z: [B, T, D]. Returns the stream after the layer, its normed copy, and what the backward pass needs."""
    pre = z @ layer.w_rate
    s, u = torch.nn.functional.softplus(pre), z @ layer.w_in
    h, _ = fem.fem_recur_fwd(s, u, mean=True, state_out=False)
    c = z + h @ layer.w_cond
    q, k, v = (heads(t, layer) for t in (c @ layer.w_qkv).chunk(3, -1))
    (q, k), v = fem.fem_rope(layer.rope, q, k), v.contiguous()
    out, lse = fem.fem_fwd_f32(q, k, v, layer.beta)
    gate = heads(z @ layer.w_gate, layer)
    r, z2 = fem.fem_norm_fwd(layer.norm, x, out, gate)
    return r, z2, (z, pre, s, u, h, c, q, k, v, out, lse, gate, r)


def backward(layer, saved, dr, dz2):
    """Gradients of <dr, r> + <dz2, z2>: a dict of those of x, z and the weights."""
    z, pre, s, u, h, c, q, k, v, out, lse, gate, r = saved
    rows = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    flat = lambda t: t.transpose(1, 2).reshape(*z.shape[:2], -1)  # noqa: E731
    dx, dout, dgate, dw_post, _, dw_pre, db_pre = fem.fem_norm_bwd(layer.norm, r, out, gate, dr, dz2)
    dq, dk, dv, dbeta = fem.fem_bwd_f32(q, k, v, layer.beta, out, lse, dout)
    dq, dk = fem.fem_rope(layer.rope, dq, dk, inverse=True)
    dqkv = torch.cat([flat(t) for t in (dq, dk, dv)], -1)
    dc, dgate = dqkv @ layer.w_qkv.T, flat(dgate)
    dh = dc @ layer.w_cond.T
    ds, du, _ = fem.fem_recur_bwd(s, u, h, dh, mean=True)
    dpre = ds * torch.sigmoid(pre)
    return dict(x=dx, z=dc + dgate @ layer.w_gate.T + dpre @ layer.w_rate.T + du @ layer.w_in.T, beta=dbeta, w_post=dw_post, w_pre=dw_pre,
                b_pre=db_pre, w_gate=rows(z).T @ rows(dgate), w_qkv=rows(c).T @ rows(dqkv), w_cond=rows(h).T @ rows(dc),
                w_rate=rows(z).T @ rows(dpre), w_in=rows(z).T @ rows(du))


def serve(layer, x, z, prompt, page=16):
    """The same layer over x, z [B, T, D], sequence by sequence of rows: `prompt` tokens in one call, then one a call."""
    B, T, D = x.shape
    device, per = x.device, -(-T // page)
    cache = fem.PagedCache.empty(B * per, layer.H, layer.d, page, torch.float32, device)
    pages = torch.randperm(B * per, device=device).to(torch.int32).view(B, per)
    pool = torch.zeros(B + 1, layer.C, device=device)  # a row more than there are sequences
    state_rows = torch.arange(B, 0, -1, device=device, dtype=torch.int32)
    outs = []
    at = 0
    while at < T:
        n = prompt if at == 0 else 1
        pos = torch.arange(at, at + n, device=device, dtype=torch.int32).repeat(B)
        offsets = torch.arange(0, (B + 1) * n, n, device=device, dtype=torch.int32)
        xs, zs = (t[:, at:at + n].contiguous().view(B * n, D) for t in (x, z))
        s, u = torch.nn.functional.softplus(zs @ layer.w_rate), zs @ layer.w_in
        h, _ = fem.fem_recur_fwd(s, u, offsets=offsets, max_len=n, h0=pool, state_rows=state_rows, mean=True)
        qkv = ((zs + h @ layer.w_cond) @ layer.w_qkv).view(B * n, 3 * layer.H, layer.d)
        q, k, v = qkv.split(layer.H, 1)
        fem.fem_rope(layer.rope, q, k, positions=pos, out=(q, k))  # in place, in the projection's output
        at += n
        slots = (pages.long()[:, pos[:n].long() // page] * page + pos[:n].long() % page).view(-1)
        fem.fem_cache_write(cache, k, v, slots)
        ctx = torch.full((B,), at, device=device, dtype=torch.int32)
        out, _ = fem.fem_paged_read(q, cache, layer.beta, offsets, ctx, pages, max_q=n)
        r, z2 = fem.fem_norm_fwd(layer.norm, xs, out, (zs @ layer.w_gate).view(B * n, layer.H, layer.d))
        outs.append((r.view(B, n, D), z2.view(B, n, D)))
    fem.check_device_error()
    return tuple(torch.cat(t, 1) for t in zip(*outs))


def run(B=2, T=200, H=4, d=32, C=48, prompt=150, seed=0):
    """A training step and the serving pass: the gradients, and the largest difference between the two outputs."""
    layer = Layer(H, d, C, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn(B, T, H * d, generator=g, device="cuda")
    _, z = fem.fem_norm_fwd(fem.BlockNorm(H * d, pre="layer"), x)  # the first layer has no block before it
    r, z2, saved = forward(layer, x, z)
    dr, dz2 = (torch.randn(r.shape, generator=g, device="cuda") for _ in range(2))
    grads = backward(layer, saved, dr, dz2)
    served = serve(layer, x, z, prompt)
    worst = max((a - b).abs().max().item() for a, b in zip(served, (r, z2)))
    return layer, (x, z, dr, dz2), (r, z2), grads, worst


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=200)
    ap.add_argument("--batch", type=int, default=2)
    a = ap.parse_args(argv)
    *_, grads, worst = run(B=a.batch, T=a.tokens, prompt=max(1, a.tokens - 50))
    print("gradients' norms: " + ", ".join(f"{name} {t.norm().item():.3g}" for name, t in grads.items()))
    print(f"served token by token: within {worst:.2e} of the training pass")


if __name__ == "__main__":
    main()
