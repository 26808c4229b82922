"""Plain 64-bit statements of the paged cache's operators, for the tests.

Everything here is elementary torch in float64 (integers where the format is), sequence by
sequence and head by head, and shares nothing with the library."""
import math

import torch


def quantise(x):
    """e4m3 codes (as their values, float64) and scale bytes of x [..., d], one scale per last axis.

    The scale 2^e is the smallest power of two with max |x| <= 448 2^e, e in [-100, 120]; codes are
    rounded to the nearest of e4m3's values, ties to even."""
    x = x.double()
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x)
    amax = x.abs().amax(-1)
    e = torch.full_like(amax, -100.0)
    for cand in range(-100, 120):  # the definition, step by step
        e = torch.where(amax > 448.0 * 2.0 ** cand, torch.full_like(e, cand + 1.0), e)
    y = x * torch.exp2(-e)[..., None]
    # e4m3: 3 fraction bits from 2^-6 up, steps of 2^-9 below
    mag = y.abs().clamp_min(2.0 ** -6)
    step = torch.exp2(torch.floor(torch.log2(mag)) - 3)
    code = torch.round(y / step) * step
    top = torch.where(e == 120, 240.0, 448.0)[..., None]
    code = torch.where(code > top, top, torch.where(code < -top, -top, code))
    return code, torch.where(bad, torch.full_like(e, 255.0), e + 127).to(torch.uint8)


def values(codes, exps):
    """Cached values in float64 (exps None: codes are the values)."""
    x = codes.to(torch.float32).double()
    if exps is None:
        return x
    e = exps.double()
    return x * torch.where(e == 255, torch.full_like(e, math.nan), torch.exp2(e - 127))[..., None]


def sequence(cache, which, table_row, ctx):
    """Positions 0 .. ctx - 1 of one sequence, [H, ctx, d] in float64; positions whose page is not
    in the cache come with True in the second result."""
    x = cache.k if which == "k" else cache.v
    e = cache.k_exp if which == "k" else cache.v_exp
    at = torch.arange(ctx, device=x.device)
    page = table_row.long()[at // cache.page_size]
    gone = (page < 0) | (page >= cache.num_pages)
    page = torch.where(gone, torch.zeros_like(page), page)
    row = at % cache.page_size
    return values(x[page, :, row], None if e is None else e[page, :, row]).transpose(0, 1), gone


def _mix(logp, seen, v, beta):
    """sum_i p_i v_ij, or (1/beta_j) log sum_i p_i exp(beta_j v_ij), of rows of log weights [n, ctx]."""
    seen, zero = seen[..., None], torch.zeros((), dtype=torch.float64, device=v.device)
    p = torch.exp(logp)[..., None]
    mean = torch.where(seen, p * v, zero).sum(1)
    if beta is None:
        return mean
    # in the log domain no spread of beta v loses anything; around the mean, no small beta does
    direct = torch.logsumexp(torch.where(seen, logp[..., None] + beta * v, -math.inf), 1) / beta
    x = beta * torch.where(seen, v - mean[:, None], zero)
    w = (p * torch.where(seen, torch.expm1(x.clamp_max(1.0)), zero)).sum(1)
    near = mean + torch.log1p(w.clamp_min(-0.9)) / beta
    small = torch.where(seen, x.abs(), zero).amax(1) < 1.0
    return torch.where(beta == 0, mean, torch.where(small, near, direct))


def read(q, cache, beta, q_offsets, ctx_lens, table, causal):
    """The read: (out [N, Hq, d], lse [N, Hq]) in float64, and the largest |v| each row's channel
    could see, [N, Hq, d].  Rows no sequence owns are NaN."""
    N, Hq, d = q.shape
    G = Hq // cache.H
    dev = q.device
    out = torch.full((N, Hq, d), math.nan, dtype=torch.float64, device=dev)
    big = torch.zeros((N, Hq, d), dtype=torch.float64, device=dev)
    lse = torch.full((N, Hq), math.nan, dtype=torch.float64, device=dev)
    for s, ctx in enumerate(ctx_lens.tolist()):
        a, b = q_offsets[s].item(), q_offsets[s + 1].item()
        n = b - a
        if n == 0:
            continue
        if ctx == 0:
            out[a:b], lse[a:b] = 0.0, -math.inf
            continue
        k, gone = sequence(cache, "k", table[s], ctx)
        v, _ = sequence(cache, "v", table[s], ctx)
        pos = torch.arange(ctx, device=dev)
        last = ctx - n + torch.arange(n, device=dev) if causal else torch.full((n,), ctx - 1, device=dev)
        seen = (pos <= last[:, None]) & ~gone
        none = ~seen.any(1)
        step = max(1, (1 << 25) // (ctx * d))  # rows at a time: each weighs every (key, channel) by itself
        for h in range(cache.H):
            vh = torch.where(gone[:, None], torch.zeros_like(v[h]), v[h])
            for g in range(G):
                logit = torch.where(seen, q[a:b, h * G + g].double() @ k[h].T / math.sqrt(d), -math.inf)
                norm = torch.logsumexp(logit, 1)
                lse[a:b, h * G + g] = norm
                logp = torch.where(none[:, None], torch.full_like(logit, -math.inf), logit - norm[:, None])
                o = torch.cat([_mix(logp[r:r + step], seen[r:r + step], vh, None if beta is None else beta[h].double())
                               for r in range(0, n, step)])
                o[none] = 0.0
                out[a:b, h * G + g] = o
                big[a:b, h * G + g] = torch.where(gone[:, None], torch.zeros_like(vh), vh).abs().amax(0)
        lse[a:b][none] = -math.inf
    return out, lse, big
