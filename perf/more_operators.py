"""The operators around the read in a layer, as cases that can be timed and compared.

Three operators, each with its backward pass:

* ``rope``: rotary positions of queries and keys, halves or neighbours paired, all or part of a head, frequencies
  scaled for long contexts; its backward pass is the rotation back;
* ``recur``, ``recur_bwd``: the gated linear recurrence h_t = e^(-s_t) h_(t-1) + w(s_t) u_t of every channel, w = 1 or
  1 - e^(-s_t), over sequences of any lengths and with states carried between calls, and its gradients;
* ``norm``, ``norm_bwd``: a block's end and the next one's start in one pass, r = x + scale act(g) (w N(y) + b) and
  z = w' N(r) + b', N a root-mean-square or layer norm or nothing, and its gradients.

Where ``own`` is false ``run`` computes each in elementary torch operations in 32 bits; where it is true it calls the
library.
"""
import math
import random

import torch

own = False

BASE = 10000.0
EPS = 1e-6


def listed():
    return [
        # one decode step of eight sequences at far positions, eight key heads: the smallest call, where latency counts
        {"name": "rope_tokens", "op": "rope", "layout": "rows", "batch": 8, "tokens": 1, "q_heads": 32, "heads": 8, "d": 128,
         "rotary": 128, "type": "bf16", "interleaved": False, "scaling": "parts", "factor": 8.0, "first": 100000, "back": False},
        # a long prompt's queries and keys as the projection leaves them, contexts stretched from 4096 positions
        {"name": "rope_prompt", "op": "rope", "layout": "rows", "batch": 1, "tokens": 16383, "q_heads": 32, "heads": 8, "d": 128,
         "rotary": 128, "type": "bf16", "interleaved": False, "scaling": "parts", "factor": 16.0, "first": 50000, "back": False},
        # gradients on their way back through half of every head, neighbours paired, in the read's layout and fp32
        {"name": "rope_back_part_f32", "op": "rope", "layout": "heads", "batch": 4, "tokens": 2048, "q_heads": 16, "heads": 16, "d": 64,
         "rotary": 32, "type": "f32", "interleaved": True, "scaling": "none", "factor": 1.0, "first": 0, "back": True},
        # one decode step of 64 sequences, states from and to a pool
        {"name": "recur_tokens", "op": "recur", "type": "bf16", "seqs": 64, "lo": 1, "hi": 1, "channels": 2048, "mean": True,
         "states": True, "lens": 1},
        # prompts of several lengths in one call, an odd number of channels, fp32, states kept for what follows
        {"name": "recur_ragged_f32", "op": "recur", "type": "f32", "seqs": 7, "lo": 50, "hi": 5000, "channels": 1001, "mean": False,
         "states": True, "lens": 2},
        # one very long sequence of few channels: the conditioner's hidden width
        {"name": "recur_long", "op": "recur", "type": "bf16", "seqs": 1, "lo": 131072, "hi": 131072, "channels": 256, "mean": False,
         "states": False, "lens": 3},
        # a training batch of the headline length
        {"name": "recur_train", "op": "recur", "type": "bf16", "seqs": 8, "lo": 8192, "hi": 8192, "channels": 2048, "mean": True,
         "states": False, "lens": 4},
        # its gradients
        {"name": "recur_back", "op": "recur_bwd", "type": "bf16", "seqs": 8, "lo": 8192, "hi": 8192, "channels": 2048, "mean": True,
         "states": False, "lens": 5},
        # gradients of packed documents that began from given states, fp32
        {"name": "recur_back_ragged_f32", "op": "recur_bwd", "type": "f32", "seqs": 12, "lo": 100, "hi": 3000, "channels": 768,
         "mean": False, "states": True, "lens": 6},
        # one decode step of eight sequences: latency
        {"name": "norm_tokens", "op": "norm", "layout": "rows", "batch": 1, "tokens": 8, "heads": 1, "d": 2048, "x_type": "bf16",
         "y_type": "bf16", "post": "rms", "pre": "rms", "act": "silu"},
        # a training batch at the headline's width, the mixer's output in the read's layout, fp32 residual stream
        {"name": "norm_train", "op": "norm", "layout": "heads", "batch": 4, "tokens": 8192, "heads": 16, "d": 128, "x_type": "f32",
         "y_type": "bf16", "post": "rms", "pre": "layer", "act": "identity"},
        # gradients through a gated block, the same number of rows, bf16 throughout
        {"name": "norm_back", "op": "norm_bwd", "layout": "rows", "batch": 4, "tokens": 8192, "heads": 1, "d": 2048, "x_type": "bf16",
         "y_type": "bf16", "post": "rms", "pre": "rms", "act": "silu"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "recur", "recur_bwd", "norm", "norm_bwd"])
    if op == "rope":
        d, heads = rng.choice([16, 64, 80, 128, 256]), rng.choice([1, 2, 4, 8, 12, 16])
        layout, group = rng.choice(["rows", "heads"]), rng.choice([1, 2, 4])
        tokens = _log(rng, 1, 2 ** 27 // ((group + 2) * heads * d * 4))
        batch = rng.randint(1, max(1, min(8, 16384 // tokens)))
        scaling = rng.choice(["none", "none", "linear", "base", "parts"])
        return {"op": op, "layout": layout, "batch": batch, "tokens": max(1, tokens // batch), "q_heads": group * heads, "heads": heads,
                "d": d, "rotary": rng.choice([d, d // 2, d - 6]), "type": rng.choice(["bf16", "bf16", "f32"]),
                "interleaved": rng.random() < 0.5, "scaling": scaling, "factor": 1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]),
                "first": rng.choice([0, rng.randrange(200000)]), "back": rng.random() < 0.4}
    if op in ("recur", "recur_bwd"):
        channels = rng.choice([32, 64, 256, 333, 768, 1000, 1024, 2048, 4096])
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 1, min(131072, 2 ** 26 // (channels * seqs)))
        return {"op": op, "type": rng.choice(["bf16", "bf16", "f32"]), "seqs": seqs, "lo": rng.choice([hi, max(1, hi // 10)]), "hi": hi,
                "channels": channels, "mean": rng.random() < 0.5, "states": rng.random() < 0.5, "lens": rng.randrange(1 << 30)}
    layout = rng.choice(["rows", "rows", "heads"])
    heads, d = (rng.choice([6, 12, 16]), rng.choice([64, 128])) if layout == "heads" else (1, rng.choice([197, 384, 768, 1000, 2048, 4097, 8192]))
    tokens = _log(rng, 1, min(32768, 2 ** 25 // (heads * d)))
    x_type, y_type = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
    return {"op": op, "layout": layout, "batch": 1, "tokens": tokens, "heads": heads, "d": d, "x_type": x_type, "y_type": y_type,
            "post": rng.choice(["none", "rms", "rms", "layer"]), "pre": rng.choice(["rms", "rms", "layer"]),
            "act": rng.choice(["none", "identity", "sigmoid", "silu"])}


# --- inputs

def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _lens(case):
    """The sequences' lengths; they go by the case alone.  Ragged ones have an empty one among them."""
    if case["lo"] == case["hi"]:
        return [case["hi"]] * case["seqs"]
    rng = random.Random(case["lens"])
    got = [rng.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
    if case["seqs"] > 2:
        got[case["seqs"] // 2] = 0
    return got


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": case}
    {"rope": _prepare_rope, "recur": _prepare_recur, "recur_bwd": _prepare_recur, "norm": _prepare_norm,
     "norm_bwd": _prepare_norm}[case["op"]](case, gen, state)
    return state


def _prepare_rope(case, gen, state):
    batch, tokens, hq, h, d = (case[n] for n in ("batch", "tokens", "q_heads", "heads", "d"))
    if case["layout"] == "rows":  # queries, keys and values of one projection's output
        qkv = _normal(gen, batch * tokens, hq + 2 * h, d).to(_type(case["type"]))
        state["q"], state["k"] = qkv[:, :hq], qkv[:, hq:hq + h]
    else:
        state["q"], state["k"] = (_normal(gen, batch, n, tokens, d).to(_type(case["type"])) for n in (hq, h))
    first = case["first"] + torch.randint(0, 1000, (batch,), generator=gen, device="cuda") if case["first"] else \
        torch.zeros(batch, dtype=torch.int64, device="cuda")
    pos = (first[:, None] + torch.arange(tokens, device="cuda")).to(torch.int32)
    state["pos"] = pos.view(-1) if case["layout"] == "rows" else pos
    context = 4096
    state["scaling"] = {"none": {}, "linear": {"scaling": "linear", "factor": case["factor"]},
                        "base": {"scaling": "base", "factor": case["factor"]},
                        "parts": {"scaling": "parts", "factor": case["factor"], "context": context, "low": 1.0, "high": 32.0,
                                  "amplitude": 0.1 * math.log(case["factor"]) + 1.0}}[case["scaling"]]
    if own:
        from paper_2602_07160_gb300 import fem
        state["fem"] = fem
        state["plan"] = fem.Rope(case["rotary"], base=BASE, interleaved=case["interleaved"], device="cuda", **state["scaling"])


def _prepare_recur(case, gen, state):
    lens, c, kind = _lens(case), case["channels"], _type(case["type"])
    n, seqs = sum(lens), case["seqs"]
    uniform = case["lo"] == case["hi"]
    # rates whose horizon runs from a step to a thousand, channel by channel
    horizon = 10.0 ** (-3.0 * torch.rand((c,), generator=gen, device="cuda"))
    s = (torch.nn.functional.softplus(_normal(gen, n, c)) * horizon).to(kind)
    u = _normal(gen, n, c).to(kind)
    state["offsets"], state["most"] = None, max(lens)
    state["starts"] = torch.tensor([sum(lens[:i]) for i in range(seqs + 1)], dtype=torch.int32, device="cuda")
    state["lens"] = torch.tensor(lens, device="cuda")
    state["seq"] = torch.repeat_interleave(torch.arange(seqs, device="cuda"), state["lens"])
    state["at"] = torch.arange(n, device="cuda") - state["starts"].long()[state["seq"]]
    if not uniform:
        state["offsets"] = state["starts"]
    shape = (seqs, case["hi"], c) if uniform else (n, c)
    state["s"], state["u"] = s.view(shape), u.view(shape)
    state["h0"] = state["rows"] = state["dstate"] = state["pool"] = None
    if case["states"]:
        if case["op"] == "recur":  # a pool of states, of which every sequence has a row
            state["h0"] = _normal(gen, seqs + 5, c)
            state["rows"] = torch.randperm(seqs + 5, generator=gen, device="cuda")[:seqs].to(torch.int32)
            state["pool"] = torch.zeros_like(state["h0"])
        else:
            state["h0"], state["dstate"] = _normal(gen, seqs, c), _normal(gen, seqs, c)
    if case["op"] == "recur_bwd":
        h, _ = _plain_states(state)
        state["h"] = h.to(kind).view(shape)
        state["dh"] = _normal(gen, n, c).to(kind).view(shape)
    if own:
        from paper_2602_07160_gb300 import fem
        state["fem"] = fem


def _prepare_norm(case, gen, state):
    batch, tokens, heads, d = (case[n] for n in ("batch", "tokens", "heads", "d"))
    width, xt, yt = heads * d, _type(case["x_type"]), _type(case["y_type"])
    inner = (batch, heads, tokens, d) if case["layout"] == "heads" else (batch * tokens, width)
    outer = (batch, tokens, width) if case["layout"] == "heads" else (batch * tokens, width)
    spread = torch.exp(_normal(gen, width) * 0.5)  # a residual stream's channels differ in size
    state["x"] = (_normal(gen, *outer) * 2 * spread).to(xt)
    state["y"] = (_normal(gen, *inner) + 0.1).to(yt)
    state["gate"] = None if case["act"] == "none" else _normal(gen, *inner).to(yt)
    state["scale"] = 0.5
    weights = {}
    for end in ("post", "pre"):
        weights["w_" + end] = 1 + 0.2 * _normal(gen, width)
        weights["b_" + end] = 0.1 * _normal(gen, width) if case[end] == "layer" else None
    state["weights"] = weights
    if case["op"] == "norm_bwd":
        state["r"] = state.pop("x")
        state["dr"], state["dz"] = _normal(gen, *outer).to(xt), _normal(gen, *outer).to(yt)
    if own:
        from paper_2602_07160_gb300 import fem
        state["fem"] = fem
        state["plan"] = fem.BlockNorm(width, post=case["post"], pre=case["pre"], gate=case["act"], scale=state["scale"], eps=EPS, **weights)


# --- a pass

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _own_rope(state):
    q, k = state["fem"].fem_rope(state["plan"], state["q"], state["k"], positions=state["pos"], inverse=state["case"]["back"])
    return {"q": q, "k": k}


def _own_recur(state):
    keep = state["pool"] if state["case"]["states"] else False
    h, last = state["fem"].fem_recur_fwd(state["s"], state["u"], offsets=state["offsets"], max_len=state["most"], h0=state["h0"],
                                         state_rows=state["rows"], mean=state["case"]["mean"], state_out=keep)
    return {"h": h, "state": last} if state["case"]["states"] else {"h": h}


def _own_recur_bwd(state):
    ds, du, dh0 = state["fem"].fem_recur_bwd(state["s"], state["u"], state["h"], state["dh"], offsets=state["offsets"],
                                             max_len=state["most"], h0=state["h0"], dstate=state["dstate"], mean=state["case"]["mean"])
    return {"ds": ds, "du": du, "dh0": dh0} if state["case"]["states"] else {"ds": ds, "du": du}


def _own_norm(state):
    r, z = state["fem"].fem_norm_fwd(state["plan"], state["x"], state["y"], state["gate"])
    return {"r": r, "z": z}


def _own_norm_bwd(state):
    names = ("dx", "dy", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")
    got = state["fem"].fem_norm_bwd(state["plan"], state["r"], state["y"], state["gate"], state["dr"], state["dz"])
    return {name: t for name, t in zip(names, got) if t is not None}


# --- the plain forms

def _frequencies(case, scaling):
    """Radians per position of every pair, in 64 bits, and the factor of cosine and sine."""
    r, base, f = case["rotary"], BASE, case["factor"]
    if case["scaling"] == "base" and r > 2:
        base = BASE * f ** (r / (r - 2))
    theta = base ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
    if case["scaling"] == "linear":
        theta = theta / f
    if case["scaling"] == "parts":  # fast pairs as they are, slow ones stretched, those between in part
        turns = scaling["context"] * theta / (2 * math.pi)
        keep = ((turns - scaling["low"]) / (scaling["high"] - scaling["low"])).clamp(0, 1)
        theta = keep * theta + (1 - keep) * theta / f
    return theta, scaling.get("amplitude", 1.0)


def _plain_rope(state):
    case = state["case"]
    r = case["rotary"]
    theta, amplitude = _frequencies(case, state["scaling"])
    angle = state["pos"].double()[..., None] * theta
    cos, sin = (f(angle).mul_(amplitude).float() for f in (torch.cos, torch.sin))
    if case["back"]:
        sin = -sin
    axis = 1  # the heads'
    cos, sin = cos.unsqueeze(axis), sin.unsqueeze(axis)
    first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    got = {}
    for name in ("q", "k"):
        x = state[name].float()
        y = x.clone(memory_format=torch.contiguous_format)
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., second] * cos + x[..., first] * sin
        got[name] = y.to(state[name].dtype)
    return got


def _scan(a, b):
    """x_t = a_t x_(t-1) + b_t along axis 1 from x_0 = b_0, by doubling steps; overwrites both."""
    step = 1
    while step < a.shape[1]:
        b[:, step:] = b[:, step:] + a[:, step:] * b[:, :-step]
        a[:, step:] = a[:, step:] * a[:, :-step]
        step *= 2
    return b


def _padded(state, name):
    """A packed input as [seqs, most, channels] in 32 bits, zeros past a sequence's end (a rate of zero keeps a state)."""
    x = state[name]
    if state["offsets"] is None:
        return x.float()
    y = torch.zeros((state["case"]["seqs"], state["most"], x.shape[-1]), device=x.device)
    y[state["seq"], state["at"]] = x.float()
    return y


def _packed(state, x):
    return x if state["offsets"] is None else x[state["seq"], state["at"]]


def _plain_states(state):
    """Every state in the inputs' layout and each sequence's last, in 32 bits."""
    s, b = _padded(state, "s"), _padded(state, "u")
    a = torch.exp(-s)
    b = b * -torch.expm1(-s) if state["case"]["mean"] else b.clone()
    if state["h0"] is not None:
        h0 = state["h0"] if state["rows"] is None else state["h0"][state["rows"].long()]
        b[:, 0] += a[:, 0] * h0
    h = _scan(a, b)
    return _packed(state, h), h[:, -1]


def _plain_recur(state):
    h, last = _plain_states(state)
    h = h.to(state["s"].dtype)
    if not state["case"]["states"]:
        return {"h": h}
    state["pool"][state["rows"].long()] = last
    return {"h": h, "state": state["pool"]}


def _plain_recur_bwd(state):
    mean = state["case"]["mean"]
    s, h, g = _padded(state, "s"), _padded(state, "h"), _padded(state, "dh")
    a = torch.exp(-s)
    # m_t = a_t (dh_t + m_(t+1)), the cotangent that step t sends to the state before it
    ra, rb = a.flip(1), (a * g).flip(1)
    if state["dstate"] is not None:
        rb[:, 0] += ra[:, 0] * state["dstate"]
    m = _scan(ra.clone(), rb).flip(1)
    total = g.clone()  # dh_t + m_(t+1)
    total[:, :-1] += m[:, 1:]
    if state["dstate"] is not None:
        total[:, -1] += state["dstate"]
    before = torch.zeros_like(h)
    before[:, 1:] = h[:, :-1]
    if state["h0"] is not None:
        before[:, 0] = state["h0"]
    if mean:
        ds, du = m * (_padded(state, "u") - before), total * -torch.expm1(-s)
    else:
        ds, du = -m * before, total
    got = {"ds": _packed(state, ds).to(state["s"].dtype), "du": _packed(state, du).to(state["s"].dtype)}
    if state["case"]["states"]:
        got["dh0"] = m[:, 0].contiguous()
    return got


def _rows(x, layout):
    """[batch, heads, tokens, d] as rows [batch tokens, heads d]."""
    return x.transpose(1, 2).flatten(0, 1).flatten(1) if layout == "heads" else x


def _unrows(x, like, layout):
    if layout != "heads":
        return x
    b, h, t, d = like.shape
    return x.view(b, t, h, d).transpose(1, 2).contiguous()


def _normed(x, kind):
    """x normalised over its last axis, and the factor that did it."""
    if kind == "none":
        return x, None
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    inv = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * inv, inv


def _weighted(x, weights, end):
    y = x * weights["w_" + end]
    return y if weights["b_" + end] is None else y + weights["b_" + end]


def _act(g, act):
    """The gate and its slope."""
    if act == "identity":
        return g, torch.ones_like(g)
    p = torch.sigmoid(g)
    return (p, p * (1 - p)) if act == "sigmoid" else (g * p, p * (1 + g * (1 - p)))


def _plain_norm(state):
    case, weights = state["case"], state["weights"]
    x = state["x"].float().reshape(-1, case["heads"] * case["d"])
    y = _weighted(_normed(_rows(state["y"].float(), case["layout"]), case["post"])[0], weights, "post")
    if state["gate"] is not None:
        y = y * _act(_rows(state["gate"].float(), case["layout"]), case["act"])[0]
    r = x + state["scale"] * y
    z = _weighted(_normed(r, case["pre"])[0], weights, "pre")
    return {"r": r.to(state["x"].dtype).view(state["x"].shape), "z": z.to(state["y"].dtype).view(state["x"].shape)}


def _norm_back(g, unit, inv, kind):
    """The cotangent of a norm's input from that of its output."""
    if kind == "none":
        return g
    if kind == "layer":
        g = g - g.mean(-1, keepdim=True)
    return inv * (g - unit * (g * unit).mean(-1, keepdim=True))


def _plain_norm_bwd(state):
    case, weights = state["case"], state["weights"]
    r = state["r"].float().reshape(-1, case["heads"] * case["d"])
    dr, dz = state["dr"].float().view_as(r), state["dz"].float().view_as(r)
    unit, inv = _normed(r, case["pre"])
    dx = dr + _norm_back(dz * weights["w_pre"], unit, inv, case["pre"])
    got = {"dx": dx.to(state["r"].dtype).view(state["r"].shape), "dw_pre": (dz * unit).sum(0)}
    if weights["b_pre"] is not None:
        got["db_pre"] = dz.sum(0)
    unit, inv = _normed(_rows(state["y"].float(), case["layout"]), case["post"])
    e = state["scale"] * dx
    if state["gate"] is not None:
        gate, slope = _act(_rows(state["gate"].float(), case["layout"]), case["act"])
        dgate = e * _weighted(unit, weights, "post") * slope
        got["dgate"] = _unrows(dgate.to(state["y"].dtype), state["y"], case["layout"])
        e = e * gate
    got["dw_post"] = (e * unit).sum(0)
    if weights["b_post"] is not None:
        got["db_post"] = e.sum(0)
    dy = _norm_back(e * weights["w_post"], unit, inv, case["post"])
    got["dy"] = _unrows(dy.to(state["y"].dtype), state["y"], case["layout"])
    names = ("dx", "dy", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")
    return {name: got[name] for name in names if name in got}


_OWN = {"rope": _own_rope, "recur": _own_recur, "recur_bwd": _own_recur_bwd, "norm": _own_norm, "norm_bwd": _own_norm_bwd}
_PLAIN = {"rope": _plain_rope, "recur": _plain_recur, "recur_bwd": _plain_recur_bwd, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd}


def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "rope":
        rows = case["batch"] * case["tokens"]
        n = rows * (case["q_heads"] + case["heads"])
        return {"bytes": 2 * n * case["d"] * size[case["type"]] + 4 * rows + 4 * case["rotary"], "flops": 3 * n * case["rotary"]}
    if case["op"] in ("recur", "recur_bwd"):
        n, c, seqs, mean = sum(_lens(case)), case["channels"], case["seqs"], case["mean"]
        moved = 3 if case["op"] == "recur" else 6 if mean else 5
        return {"bytes": moved * n * c * size[case["type"]] + ((2 if case["op"] == "recur" else 3) * seqs * c * 4 if case["states"] else 0),
                "flops": (4 if case["op"] == "recur" else 8) * n * c}
    rows, width = case["batch"] * case["tokens"], case["heads"] * case["d"]
    xs, ys, gates = size[case["x_type"]], size[case["y_type"]], 0 if case["act"] == "none" else 1
    vectors = sum(1 + (case[end] == "layer") for end in ("post", "pre"))
    if case["op"] == "norm":
        return {"bytes": rows * width * (2 * xs + (2 + gates) * ys) + 4 * width * vectors, "flops": 14 * rows * width}
    return {"bytes": rows * width * (3 * xs + (3 + 2 * gates) * ys) + 8 * width * vectors, "flops": 40 * rows * width}


# --- the operators' definitions in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, state)
    if case["op"] in ("recur", "recur_bwd"):
        return _exact_recur(case, state)
    return _exact_norm(case, state)


def _exact_rope(case, state):
    r, pairs = case["rotary"], case["rotary"] // 2
    rate = []
    for i in range(pairs):
        w = BASE ** (-2 * i / r)
        if case["scaling"] == "linear":
            w /= case["factor"]
        elif case["scaling"] == "base" and r > 2:
            w = (BASE * case["factor"] ** (r / (r - 2))) ** (-2 * i / r)
        elif case["scaling"] == "parts":
            kept = min(1.0, max(0.0, (4096 * w / (2 * math.pi) - 1.0) / 31.0))
            w = w * kept + w / case["factor"] * (1.0 - kept)
        rate.append(w)
    pos = state["pos"].double()
    angle = pos[..., None] * torch.tensor(rate, dtype=torch.float64, device="cuda")
    size = torch.full_like(angle, 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "parts" else 1.0)
    turn = torch.polar(size, -angle if case["back"] else angle)[:, None]
    got = {}
    for name in ("q", "k"):
        x = state[name].double().contiguous()
        part = x[..., :r]
        pair = part.unflatten(-1, (pairs, 2)) if case["interleaved"] else part.unflatten(-1, (2, pairs)).transpose(-1, -2)
        back = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        back = back if case["interleaved"] else back.transpose(-1, -2)
        got[name] = torch.cat([back.flatten(-2), x[..., r:]], -1)
    return got


def _exact_recur(case, state):
    """Sequence by sequence and step by step; sequences of one length together."""
    c, lens = case["channels"], _lens(case)
    if case["lo"] == case["hi"]:
        groups = [list(range(case["seqs"]))]
    else:
        groups = [[i] for i in range(case["seqs"])]
    if sum(lens[g[0]] for g in groups) > 200000:
        return None
    flat = {name: state[name].reshape(-1, c) for name in ("s", "u", "h", "dh") if name in state}
    starts = [sum(lens[:i]) for i in range(len(lens))]
    outs = {name: torch.zeros((sum(lens), c), dtype=torch.float64, device="cuda") for name in (("h",) if case["op"] == "recur" else ("ds", "du"))}
    ends = torch.zeros((case["seqs"], c), dtype=torch.float64, device="cuda")
    for g in groups:
        n, first = lens[g[0]], starts[g[0]]
        part = {k: x[first:first + n * len(g)].view(len(g), n, c).transpose(0, 1).double().contiguous() for k, x in flat.items()}
        decay = torch.exp(-part["s"])
        take = -torch.expm1(-part["s"]) if case["mean"] else torch.ones_like(decay)
        start = torch.zeros((len(g), c), dtype=torch.float64, device="cuda")
        if state["h0"] is not None:
            start = (state["h0"] if state["rows"] is None else state["h0"][state["rows"].long()])[g].double()
        if case["op"] == "recur":
            feed, hidden = take * part["u"], torch.empty_like(decay)
            now = start
            for d, f, out in zip(decay.unbind(0), feed.unbind(0), hidden.unbind(0)):
                now = torch.addcmul(f, d, now, out=out)
            outs["h"][first:first + n * len(g)] = hidden.transpose(0, 1).reshape(-1, c)
            ends[g] = now
            continue
        coming = state["dstate"][g].double() if state["dstate"] is not None else torch.zeros_like(start)
        sums = torch.empty_like(decay)  # the whole cotangent of every state
        for d, gr, out in zip(reversed(decay.unbind(0)), reversed(part["dh"].unbind(0)), reversed(sums.unbind(0))):
            torch.add(gr, coming, out=out)
            coming = out * d
        earlier = torch.cat([start[None], part["h"]])[:n]
        slope = decay * part["u"] if case["mean"] else torch.zeros_like(decay)
        outs["ds"][first:first + n * len(g)] = (sums * (slope - decay * earlier)).transpose(0, 1).reshape(-1, c)
        outs["du"][first:first + n * len(g)] = (sums * take).transpose(0, 1).reshape(-1, c)
        ends[g] = coming
    got = {name: x.view(state["s"].shape) for name, x in outs.items()}
    if case["states"]:
        if case["op"] == "recur":
            pool = torch.zeros_like(state["pool"], dtype=torch.float64)
            pool[state["rows"].long()] = ends
            got["state"] = pool
        else:
            got["dh0"] = ends
    return got


def _exact_norm(case, state):
    """The forward pass in 64 bits, and the gradients by automatic differentiation of it."""
    width, heads = case["heads"] * case["d"], case["layout"] == "heads"
    leaf = {n: t.double() for n, t in state["weights"].items() if t is not None}
    leaf["y"] = state["y"].double()
    if state["gate"] is not None:
        leaf["gate"] = state["gate"].double()
    back = case["op"] == "norm_bwd"

    def normal(v, kind):
        if kind == "none":
            return v
        centre = v - v.mean(-1, keepdim=True) if kind == "layer" else v
        return centre / torch.sqrt(centre.square().mean(-1, keepdim=True) + EPS)

    def branch(v):
        y = v["y"].permute(0, 2, 1, 3).reshape(-1, width) if heads else v["y"]
        y = normal(y, case["post"]) * v["w_post"] + v.get("b_post", 0.0)
        if "gate" in v:
            g = v["gate"].permute(0, 2, 1, 3).reshape(-1, width) if heads else v["gate"]
            y = y * {"identity": lambda t: t, "sigmoid": torch.sigmoid, "silu": lambda t: t * torch.sigmoid(t)}[case["act"]](g)
        return y * state["scale"]

    def out(r, v):
        return normal(r, case["pre"]) * v["w_pre"] + v.get("b_pre", 0.0)

    if not back:
        r = state["x"].double().reshape(-1, width) + branch(leaf)
        return {"r": r.view(state["x"].shape), "z": out(r, leaf).view(state["x"].shape)}
    for t in leaf.values():
        t.requires_grad_(True)
    r = state["r"].double().reshape(-1, width).requires_grad_(True)
    pre = [n for n in ("w_pre", "b_pre") if n in leaf]
    grads = torch.autograd.grad(out(r, leaf), [r] + [leaf[n] for n in pre], state["dz"].double().reshape(-1, width))
    got = {"d" + n: g for n, g in zip(pre, grads[1:])}
    dx = grads[0] + state["dr"].double().reshape(-1, width)
    rest = [n for n in ("y", "gate", "w_post", "b_post") if n in leaf]
    got |= {"d" + n: g for n, g in zip(rest, torch.autograd.grad(branch(leaf), [leaf[n] for n in rest], dx))}
    got["dx"] = dx.view(state["r"].shape)
    names = ("dx", "dy", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")
    return {name: got[name] for name in names if name in got}
