"""The paged key/value cache's operators, as cases that can be timed and compared.

Three operators of the serving path:

* ``write``: new tokens' keys and values into the pages of a cache, as bf16 or quantised to e4m3 with one
  power-of-two scale per token and head;
* ``gather``: stretches of cached sequences read back as contiguous bf16 keys and values;
* ``read``: the free-energy read (plain softmax attention where ``beta`` is absent) of new tokens over the
  cache, from one token per sequence to whole prompts, with fewer key/value heads than query heads.

Where ``own`` is false ``run`` computes each in elementary torch operations in 32 bits; where it is true it
calls the library.
"""
import math
import random

import torch

own = False

E_MIN = -100  # smallest scale exponent
E_TOP = 120   # largest: 448 * 2**120 is past bf16's range, so codes stop at 240 there


def listed():
    return [
        # one decode step of eight sequences: the write's smallest call, where latency counts
        {"name": "write_tokens_bf16", "op": "write", "format": "bf16", "tokens": 8, "heads": 8, "d": 128, "page": 64},
        # a prompt's keys and values at the width of the headline workload (16 heads of 128), into 8 bits
        {"name": "write_prompt_e4m3", "op": "write", "format": "e4m3", "tokens": 8192, "heads": 16, "d": 128, "page": 64},
        # short stretches of a few sequences, heads of 64, an odd total
        {"name": "gather_short_e4m3", "op": "gather", "format": "e4m3", "seqs": 3, "heads": 12, "d": 64, "page": 16,
         "lo": 100, "hi": 700, "lens": 3},
        # whole sequences of the headline length read back for a pass that wants them contiguous
        {"name": "gather_long_e4m3", "op": "gather", "format": "e4m3", "seqs": 4, "heads": 16, "d": 128, "page": 64,
         "lo": 7000, "hi": 8192, "lens": 4},
        # one decode step of a few short conversations, as many key/value heads as query heads: latency
        {"name": "token_few_short", "op": "read", "format": "bf16", "seqs": 4, "n_lo": 1, "n_hi": 1, "ctx_lo": 64,
         "ctx_hi": 1024, "q_heads": 16, "heads": 16, "d": 128, "page": 64, "beta": True, "causal": True, "lens": 5},
        # one decode step of a full batch over an 8-bit cache, four query heads to a key/value head
        {"name": "token_batch_e4m3", "op": "read", "format": "e4m3", "seqs": 48, "n_lo": 1, "n_hi": 1, "ctx_lo": 2048,
         "ctx_hi": 8192, "q_heads": 32, "heads": 8, "d": 128, "page": 64, "beta": True, "causal": True, "lens": 6},
        # one decode step of a single very long conversation
        {"name": "token_long", "op": "read", "format": "bf16", "seqs": 1, "n_lo": 1, "n_hi": 1, "ctx_lo": 131071,
         "ctx_hi": 131071, "q_heads": 32, "heads": 8, "d": 128, "page": 64, "beta": True, "causal": True, "lens": 7},
        # a few drafted tokens per sequence, heads of 64, plain attention, one sequence with nothing cached yet
        {"name": "drafts_d64_mean", "op": "read", "format": "e4m3", "seqs": 9, "n_lo": 1, "n_hi": 5, "ctx_lo": 900,
         "ctx_hi": 4000, "q_heads": 12, "heads": 4, "d": 64, "page": 16, "beta": False, "causal": True, "lens": 8,
         "empty": True},
        # a chunk of a prompt over what is cached of it
        {"name": "chunk_512", "op": "read", "format": "bf16", "seqs": 1, "n_lo": 512, "n_hi": 512, "ctx_lo": 8192,
         "ctx_hi": 8192, "q_heads": 16, "heads": 4, "d": 128, "page": 64, "beta": True, "causal": True, "lens": 9},
        # chunks of several prompts at once, lengths as they come, 12 heads of 64, 8-bit cache
        {"name": "chunks_ragged_e4m3", "op": "read", "format": "e4m3", "seqs": 6, "n_lo": 100, "n_hi": 700,
         "ctx_lo": 1000, "ctx_hi": 5000, "q_heads": 12, "heads": 12, "d": 64, "page": 32, "beta": True, "causal": True,
         "lens": 10},
        # a whole prompt of the headline length and width
        {"name": "prompt_8192", "op": "read", "format": "bf16", "seqs": 1, "n_lo": 8192, "n_hi": 8192, "ctx_lo": 8192,
         "ctx_hi": 8192, "q_heads": 16, "heads": 16, "d": 128, "page": 64, "beta": True, "causal": True, "lens": 11},
        # decoder tokens over cached encoder states of another length (197 image tokens), no mask, plain attention
        {"name": "cross_197_mean", "op": "read", "format": "bf16", "seqs": 32, "n_lo": 40, "n_hi": 80, "ctx_lo": 197,
         "ctx_hi": 197, "q_heads": 6, "heads": 6, "d": 64, "page": 64, "beta": False, "causal": False, "lens": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "gather", "token", "token", "drafts", "chunk", "chunk"])
    case = {"op": op if op in ("write", "gather") else "read", "format": rng.choice(["bf16", "e4m3"]),
            "heads": rng.choice([1, 2, 4, 8, 12, 16]), "d": rng.choice([64, 128]), "page": rng.choice([16, 32, 64, 128])}
    if op == "write":
        return {**case, "tokens": _log(rng, 1, 8192)}
    case["lens"] = rng.randrange(1 << 30)
    if op == "gather":
        hi = _log(rng, 16, 8192)
        return {**case, "seqs": rng.randint(1, 4), "lo": max(1, hi // 2), "hi": hi}
    group = rng.choice([1, 2, 4, 8] if case["heads"] <= 4 else [1, 2, 4] if case["heads"] <= 8 else [1])
    case["q_heads"] = group * case["heads"]
    case["beta"] = rng.random() < 0.7
    case["causal"] = rng.random() < 0.8
    if op == "chunk":
        n = _log(rng, 17, 4096)
        seqs = rng.randint(1, max(1, min(8, 8192 // n)))
        ctx = max(n, _log(rng, 100, min(16384, 8192 * 8192 // (2 * n * seqs))))
    else:
        n = 1 if op == "token" else rng.randint(2, 8)
        seqs = _log(rng, 1, 48)
        ctx = _log(rng, 16, min(131072, 8192 * 48 // seqs))
    return {**case, "seqs": seqs, "n_lo": max(1, n // 2), "n_hi": n, "ctx_lo": max(n, ctx // 2), "ctx_hi": max(n, ctx)}


def _lens(case):
    """(new tokens, context) of each sequence; they go by the case alone."""
    rng = random.Random(case["lens"])
    if case["op"] == "gather":
        return [(0, rng.randint(case["lo"], case["hi"])) for _ in range(case["seqs"])]
    got = [(rng.randint(case["n_lo"], case["n_hi"]), rng.randint(case["ctx_lo"], case["ctx_hi"])) for _ in range(case["seqs"])]
    got = [(n, max(n, ctx)) for n, ctx in got]
    if case.get("empty"):
        got[len(got) // 2] = (1, 0)
    return got


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _quantise(x):
    """e4m3 codes and biased scale exponents of x [..., d], one scale for each last axis, in 32 bits."""
    x = x.float()
    amax = x.abs().amax(-1)
    bad = ~torch.isfinite(x).all(-1)
    frac, expo = torch.frexp(torch.where(bad, torch.zeros_like(amax), amax))  # amax = frac 2^expo, frac in [1/2, 1)
    e = torch.where(frac <= 0.875, expo - 9, expo - 8).clamp(E_MIN, E_TOP).to(torch.int32)
    e = torch.where(amax == 0, torch.full_like(e, E_MIN), e)
    top = torch.where(e == E_TOP, 240.0, 448.0)[..., None]
    codes = torch.ldexp(x, -e[..., None]).clamp(-top, top)
    codes = torch.where(bad[..., None], torch.zeros_like(codes), codes).to(torch.float8_e4m3fn)
    return codes, torch.where(bad, 255, e + 127).to(torch.uint8)


def _scales(expo):
    e = expo.to(torch.int32)
    return torch.where(e == 255, math.nan, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e - 127))


def _cache(case, gen, pages, filled):
    """Pages [pages, heads, page, d] of keys and of values: what a prompt left there, or zeros."""
    shape = (pages, case["heads"], case["page"], case["d"])
    got = {}
    for name in ("k", "v"):
        x = _normal(gen, *shape) if filled else torch.zeros(shape, device="cuda")
        if case["format"] == "e4m3":
            got[name], got[name + "_exp"] = _quantise(x)
        else:
            got[name], got[name + "_exp"] = x.to(torch.bfloat16), None
    return got


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    page, heads, d = case["page"], case["heads"], case["d"]
    state = {"case": case}
    if case["op"] == "write":
        n = case["tokens"]
        pages = -(-n // page) + 2
        state |= _cache(case, gen, pages, False)
        kv = _normal(gen, n, 2 * heads, d).to(torch.bfloat16)  # one projection's output: keys, then values
        state["new_k"], state["new_v"] = kv[:, :heads], kv[:, heads:]
        state["slots"] = torch.randperm(pages * page, generator=gen, device="cuda")[:n]
    else:
        lens = _lens(case)
        need = [-(-ctx // page) for _, ctx in lens]
        pages, width = sum(need) + 3, max(need)
        state |= _cache(case, gen, pages, True)
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        table, at = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda"), 0
        for s, m in enumerate(need):
            table[s, :m] = order[at:at + m]
            at += m
        state["table"] = table
        state["ctx"] = torch.tensor([ctx for _, ctx in lens], dtype=torch.int32, device="cuda")
        counts = [ctx if case["op"] == "gather" else n for n, ctx in lens]
        offsets = [sum(counts[:s]) for s in range(len(lens) + 1)]
        state["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        state["rows"], state["most"] = offsets[-1], max(counts)
        state["row_seq"] = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(counts, device="cuda"))
        state["row_pos"] = torch.arange(offsets[-1], device="cuda") - state["offsets"].long()[state["row_seq"]]
        state["starts"] = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
        state["width"] = max(ctx for _, ctx in lens)
        if case["op"] == "read":
            q = _normal(gen, offsets[-1], case["q_heads"] + 2 * heads, d).to(torch.bfloat16)
            state["q"] = q[:, :case["q_heads"]]  # queries, keys and values of one projection's output
            u = torch.rand((heads, d), generator=gen, device="cuda")
            state["beta"] = torch.exp(math.log(0.1) + u * math.log(50.0)) if case["beta"] else None  # 0.1 to 5
    if own:
        from paper_2602_07160_gb300 import fem
        state["fem"] = fem
        state["cache"] = fem.PagedCache(state["k"], state["v"], state["k_exp"], state["v_exp"])
    return state


def run(state):
    case = state["case"]
    if case["op"] == "write":
        return (_run_write if own else _plain_write)(state)
    if case["op"] == "gather":
        return (_run_gather if own else _plain_gather)(state)
    return (_run_read if own else _plain_read)(state)


def _run_write(state):
    state["fem"].fem_cache_write(state["cache"], state["new_k"], state["new_v"], state["slots"])
    return {name: state[name] for name in ("k", "v", "k_exp", "v_exp") if state[name] is not None}


def _run_gather(state):
    k, v = state["fem"].fem_cache_gather(state["cache"], state["table"], state["starts"], state["offsets"], state["rows"])
    return {"k": k, "v": v}


def _run_read(state):
    out, lse = state["fem"].fem_paged_read(state["q"], state["cache"], state["beta"], state["offsets"], state["ctx"],
                                           state["table"], max_q=state["most"], causal=state["case"]["causal"])
    return {"out": out, "lse": lse}


def _plain_write(state):
    page = state["case"]["page"]
    at, inside = torch.div(state["slots"], page, rounding_mode="floor"), state["slots"] % page
    names = ("k", "v")
    if state["case"]["format"] == "e4m3":
        codes = [_quantise(state["new_" + n]) for n in names]
        state["k"].view(torch.uint8)[at, :, inside] = codes[0][0].view(torch.uint8)
        state["v"].view(torch.uint8)[at, :, inside] = codes[1][0].view(torch.uint8)
        state["k_exp"][at, :, inside], state["v_exp"][at, :, inside] = codes[0][1], codes[1][1]
        return {name: state[name] for name in ("k", "v", "k_exp", "v_exp")}
    state["k"][at, :, inside], state["v"][at, :, inside] = state["new_k"], state["new_v"]
    return {name: state[name] for name in names}


def _plain_pages(state, name):
    """Cached values [seqs, heads, positions, d] in 32 bits, sequence by sequence in order of position."""
    table = state["table"].clamp_min(0).long()
    x = state[name][table].float()
    if state[name + "_exp"] is not None:
        x = x * _scales(state[name + "_exp"][table])[..., None]
    s, p, h, page, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(s, h, p * page, d)[:, :, :state["width"]]


def _plain_gather(state):
    seq, pos = state["row_seq"], state["row_pos"]
    return {"k": _plain_pages(state, "k")[seq, :, pos].to(torch.bfloat16),
            "v": _plain_pages(state, "v")[seq, :, pos].to(torch.bfloat16)}


def _plain_read(state):
    case, ctx, offsets = state["case"], state["ctx"].long(), state["offsets"].long()
    heads, d, most, width = case["heads"], case["d"], state["most"], state["width"]
    group, seqs = case["q_heads"] // heads, case["seqs"]
    k, v = _plain_pages(state, "k"), _plain_pages(state, "v")
    rows = (offsets[:-1, None] + torch.arange(most, device=k.device)).clamp_max(state["rows"] - 1)
    q = state["q"][rows].float().view(seqs, most, heads, group, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(seqs, heads, most * group, d)
    score = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    limit = ctx[:, None].expand(seqs, most)
    if case["causal"]:
        limit = ctx[:, None] - (offsets[1:] - offsets[:-1])[:, None] + torch.arange(1, most + 1, device=k.device)
        limit = torch.minimum(limit, ctx[:, None])
    key = torch.arange(width, device=k.device)
    hidden = (key >= limit[..., None]).repeat_interleave(group, dim=1)[:, None]
    score = score.masked_fill_(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    some = torch.where(total > 0, total, 1.0)
    cached = (key < ctx[:, None])[:, None, :, None]
    v = torch.where(cached, v, 0.0)
    if state["beta"] is None:
        out = (p @ v) / some
    else:
        beta = state["beta"][None, :, None, :]
        shift = torch.where(cached, v, -math.inf).amax(2, keepdim=True)
        shift = torch.where(shift == -math.inf, 0.0, shift)
        mixed = (p @ torch.exp(beta * (v - shift))) / some
        out = shift + torch.log(torch.where(total > 0, mixed, 1.0)) / beta
        out = torch.where(total > 0, out, 0.0)
    out = out.view(seqs, heads, most, group, d).permute(0, 2, 1, 3, 4).reshape(seqs, most, heads * group, d)
    lse = lse.view(seqs, heads, most, group).permute(0, 2, 1, 3).reshape(seqs, most, heads * group)
    return {"out": out[state["row_seq"], state["row_pos"]].to(torch.bfloat16), "lse": lse[state["row_seq"], state["row_pos"]]}


def work(case):
    heads, d = case["heads"], case["d"]
    cached = 2 * heads * (d + 1 if case["format"] == "e4m3" else 2 * d)  # bytes of one position's keys and values
    if case["op"] == "write":
        return {"bytes": case["tokens"] * (cached + 2 * heads * d * 2 + 8), "flops": 0}
    lens = _lens(case)
    positions = sum(ctx for _, ctx in lens)
    table = 4 * sum(-(-ctx // case["page"]) for _, ctx in lens)
    if case["op"] == "gather":
        return {"bytes": positions * (cached + 2 * heads * d * 2) + table, "flops": 0}
    rows = sum(n for n, _ in lens) * case["q_heads"]
    pairs = sum(n * ctx - (n * (n - 1) // 2 if case["causal"] and ctx >= n else 0) for n, ctx in lens)
    return {"bytes": positions * cached + table + rows * (4 * d + 4), "flops": 4 * pairs * case["q_heads"] * d}


# --- the operators' definitions in 64 bits

def _exact_codes(x):
    """The value of each e4m3 code of x [..., d], in 64 bits, and the scales' biased exponents."""
    x = x.double()
    amax = x.abs().amax(-1)
    e = torch.ceil(torch.log2(amax.clamp_min(1e-300) / 448.0))
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, torch.where(amax <= 448.0 * torch.exp2(e - 1), e - 1, e))
    e = e.clamp(E_MIN, E_TOP)
    y = x * torch.exp2(-e)[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)  # codes: 4 bits, from 2^-9
    return torch.round(y / step) * step, (e + 127).to(torch.uint8)


def _exact_sequence(state, name, s, ctx):
    """Positions 0 .. ctx - 1 of sequence s, [heads, ctx, d] in 64 bits."""
    page = state["case"]["page"]
    at = torch.arange(ctx, device="cuda")
    where = state["table"][s].long()[at // page]
    x = state[name][where, :, at % page].to(torch.float32).double()
    if state[name + "_exp"] is not None:
        x = x * torch.exp2(state[name + "_exp"][where, :, at % page].double() - 127)[..., None]
    return x.transpose(0, 1)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "write":
        page, got = case["page"], {}
        for name in ("k", "v"):
            new = state["new_" + name]
            codes, expo = _exact_codes(new) if case["format"] == "e4m3" else (new.double(), None)
            got[name] = state[name].to(torch.float32).double()
            got[name][state["slots"] // page, :, state["slots"] % page] = codes
            if expo is not None:
                got[name + "_exp"] = state[name + "_exp"].clone()
                got[name + "_exp"][state["slots"] // page, :, state["slots"] % page] = expo
        return got
    lens = _lens(case)
    if case["op"] == "gather":
        return {name: torch.cat([_exact_sequence(state, name, s, ctx).transpose(0, 1) for s, (_, ctx) in enumerate(lens)])
                for name in ("k", "v")}
    heads, d = case["heads"], case["d"]
    group = case["q_heads"] // heads
    outs, lses, first = [], [], 0
    for s, (n, ctx) in enumerate(lens):
        q = state["q"][first:first + n].double().view(n, heads, group, d)
        first += n
        out = torch.zeros((n, heads, group, d), dtype=torch.float64, device="cuda")
        lse = torch.full((n, heads, group), -math.inf, dtype=torch.float64, device="cuda")
        if ctx:
            k, v = _exact_sequence(state, "k", s, ctx), _exact_sequence(state, "v", s, ctx)
            last = ctx - n + torch.arange(n, device="cuda") if case["causal"] else torch.full((n,), ctx - 1, device="cuda")
            shown = torch.arange(ctx, device="cuda") <= last[:, None]
            for h in range(heads):
                for g in range(group):
                    logits = torch.where(shown, q[:, h, g] @ k[h].T / math.sqrt(d), -math.inf)
                    norm = torch.logsumexp(logits, 1)
                    prior = torch.exp(logits - norm[:, None])
                    lse[:, h, g] = norm
                    if state["beta"] is None:
                        out[:, h, g] = prior @ v[h]
                    else:
                        b = state["beta"][h].double()
                        out[:, h, g] = torch.log(prior @ torch.exp(b * v[h])) / b
        outs.append(out.reshape(n, heads * group, d))
        lses.append(lse.reshape(n, heads * group))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
