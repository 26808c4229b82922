"""Plain 64-bit forms of the operators around the read, and the bounds their fp32 arithmetic keeps to.

Tolerances count roundings: an output of type t is off by at most eps(t) / 2 of its value, and the fp32 arithmetic
before it by some number of 2^-24 of the sum of the magnitudes that went into it, which each function returns beside the
value.  The numbers are derived where they are used.
"""
import math

import torch

UNIT = 2.0 ** -24  # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def check(got, want, magnitude, units, dtype=None):
    """got within half a step of its type and `units` roundings of `magnitude` of want."""
    dtype = got.dtype if dtype is None else dtype
    got, want, magnitude = got.double().cpu(), want.double().cpu(), magnitude.double().cpu()
    assert got.shape == want.shape
    tol = half_step(dtype) * want.abs() + units * UNIT * magnitude * (1 + half_step(dtype)) + 1e-37
    over = ((got - want).abs() / tol).nan_to_num(nan=math.inf)
    assert over.numel() == 0 or over.max() <= 1, (over.max().item(), (got - want).abs().max().item())


# --- rotary positions

def rope_rates(rotary, base=10000.0, scaling=None, factor=1.0, context=4096.0, low=1.0, high=32.0):
    rates = []
    for i in range(rotary // 2):
        b = base * factor ** (rotary / (rotary - 2)) if scaling == "base" and rotary > 2 else base
        theta = b ** (-2 * i / rotary)
        if scaling == "linear":
            theta /= factor
        if scaling == "parts":
            g = min(1.0, max(0.0, (context * theta / (2 * math.pi) - low) / (high - low)))
            theta = g * theta + (1 - g) * theta / factor
        rates.append(theta)
    return torch.tensor(rates, dtype=torch.float64)


def rope(x, positions, rates, interleaved, amplitude=1.0, inverse=False):
    """x [N, H, d] or [B, H, T, d] (positions [N] or [B, T]); returns the result and |a| + |b| of every element."""
    x = x.double()
    r = 2 * rates.numel()
    angle = positions.double()[..., None] * rates.to(x.device)
    angle = (-angle if inverse else angle).unsqueeze(1)  # over heads
    cos, sin = amplitude * torch.cos(angle), amplitude * torch.sin(angle)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y, size = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    size[..., a] = size[..., b] = abs(amplitude) * (x[..., a].abs() + x[..., b].abs())
    return y, size


# --- the gated recurrence

def recur(s, u, lens, h0=None, mean=False):
    """Packed s, u [N, C] and the sequences' lengths: h, the last states, and the bound's magnitudes of both: each step
    adds an error of some roundings of the magnitudes in its state, and passes on its predecessor's, decayed."""
    s, u = s.double(), u.double()
    h, hm = torch.zeros_like(s), torch.zeros_like(s)
    last, lm = (torch.zeros((len(lens), s.shape[1]), dtype=torch.float64, device=s.device) for _ in range(2))
    at = 0
    for q, n in enumerate(lens):
        x = h0[q].double() if h0 is not None else torch.zeros_like(last[q])
        size, err = x.abs(), torch.zeros_like(x)
        for t in range(at, at + n):
            a = torch.exp(-s[t])
            f = u[t] * -torch.expm1(-s[t]) if mean else u[t]
            x = a * x + f
            size = a * size + f.abs()
            err = a * err + size
            h[t], hm[t] = x, err
        last[q], lm[q] = x, err
        at += n
    return h, last, hm, lm


def recur_grads(s, u, h, dh, lens, h0=None, dstate=None, mean=False):
    """ds, du, dh0 by the formulas, each with its magnitude."""
    s, u, h, dh = (t.double() for t in (s, u, h, dh))
    ds, du, dsm, dum = (torch.zeros_like(s) for _ in range(4))
    dh0, dm0 = (torch.zeros((len(lens), s.shape[1]), dtype=torch.float64, device=s.device) for _ in range(2))
    at = 0
    for q, n in enumerate(lens):
        m = dstate[q].double() if dstate is not None else torch.zeros_like(dh0[q])
        size, err = m.abs(), torch.zeros_like(m)
        for t in range(at + n - 1, at - 1, -1):
            a, w = torch.exp(-s[t]), -torch.expm1(-s[t])
            total, before = dh[t] + m, h[t - 1] if t > at else (h0[q].double() if h0 is not None else torch.zeros_like(m))
            size = size + dh[t].abs()
            du[t], dum[t] = (total * w, (size + err) * w) if mean else (total, size + err)
            m, size, err = a * total, a * size, a * (err + size)
            ds[t] = m * (u[t] - before) if mean else -m * before
            dsm[t] = (size + err) * (before.abs() + (u[t].abs() if mean else 0.0))
        dh0[q], dm0[q] = m, err + size
        at += n
    return (ds, du, dh0), (dsm, dum, dm0)


# --- norms with gate and residual

def rows_of(x):
    """[N, H, d] or [B, H, T, d] as [rows, H d]."""
    return x.flatten(1) if x.dim() == 3 else x.transpose(1, 2).reshape(x.shape[0] * x.shape[2], -1)


def _norm(v, kind, eps):
    if kind == "none":
        return v
    c = v - v.mean(-1, keepdim=True) if kind == "layer" else v
    return c / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)


def _gate(g, act):
    return {"identity": lambda: g, "sigmoid": lambda: torch.sigmoid(g), "silu": lambda: g * torch.sigmoid(g)}[act]()


def block(x, y, gate, w, post, pre, act, scale, eps):
    """r and z of rows x, y, gate [rows, D] (y, gate may be None), weights w a dict of [D] or None."""
    one = lambda name, none: w[name] if w[name] is not None else none  # noqa: E731
    r = x
    if y is not None:
        v = _norm(y, post, eps) * one("w_post", 1.0) + one("b_post", 0.0)
        if gate is not None:
            v = v * _gate(gate, act)
        r = x + scale * v
    z = None if pre == "none" else _norm(r, pre, eps) * one("w_pre", 1.0) + one("b_pre", 0.0)
    return r, z
