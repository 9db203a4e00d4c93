"""The serving operators' definitions in 64 bits, from their formulas, with the bound that each result's rounding gives (used
by the GPU tests and pinned by the CPU tests)."""
import math

import torch

U16 = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}    # unit roundoffs
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}          # half a step below the smallest normal number
U32 = 2.0 ** -24


# ---- queries, keys and values ------------------------------------------------------------------------------

def turned64(x, positions, freqs, axis_of, *, rot, pairs, kind=None, w=None, b=None, eps=1e-5):
    """Heads x (T, h, D) normed and turned, positions (axes, T), and the bound on what fp32 arithmetic adds to the
    rounding.  A norm's sums are trees of fewer than 16 roundings, its factor and weight a few more, so 32 half steps
    of the normed values (of their spread before the mean is taken off); cosine and sine are off by less than 4 half
    steps of 1 (a rest of at most half a quarter turn rounded to fp32, times a rounded constant, 2^-23.7 in all; the
    series' own rest and last roundings, 2^-23.8), products and sum by 3 more."""
    x = x.double()
    mag = x.abs()
    if kind is not None:
        mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
        r = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
        w64 = torch.ones_like(x[0, 0]) if w is None else w.double()
        b64 = torch.zeros_like(w64) if b is None else b.double()
        mag = (x.abs() + mean.abs() + (x.abs().mean(-1, keepdim=True) if kind == "layer" else 0)) * r * w64.abs() + b64.abs()
        x = (x - mean) * r * w64 + b64
    err = (32 if kind else 0) * U32 * mag
    half = rot // 2
    if half:
        axis = torch.zeros(half, dtype=torch.long, device=x.device) if axis_of is None else axis_of.long().clamp(0, positions.shape[0] - 1)
        t = (positions.double()[axis].t() * freqs.double())[:, None]
        first = torch.arange(half, device=x.device) * (2 if pairs else 1)
        second = first + (1 if pairs else half)
        a, c = x[..., first], x[..., second]
        ea = err[..., first] + err[..., second] + 8 * U32 * (a.abs() + c.abs())
        x, err = x.clone(), err.clone()
        x[..., first], x[..., second] = a * torch.cos(t) - c * torch.sin(t), c * torch.cos(t) + a * torch.sin(t)
        err[..., first] = err[..., second] = ea
    return x, err


def places64(starts, lens, T):
    """(sequence, place) of every token, (-1, 0) of those of no sequence."""
    out = [(-1, 0)] * T
    for b in range(len(lens)):
        for t in range(max(starts[b], 0), min(starts[b + 1], T)):
            out[t] = (b, max(lens[b], 0) - starts[b + 1] + t)
    return out


def slot64(table, page_size, n_pages, b, place):
    """(page, slot) of a place, or None."""
    if b < 0 or place < 0 or place >= table.shape[1] * page_size:
        return None
    page = int(table[b, place // page_size])
    return (page, place % page_size) if 0 <= page < n_pages else None


# ---- attention ------------------------------------------------------------------------------------------------

def paged64(q, k, v, table, page_size, starts, lens, max_len, scale):
    """out, lse and the bounds of both; q (T, H, D), k and v (pages, page_size, N, D).  Rows of no sequence are NaN.

    A score is a sum of D products, in chains of at most D / 8 + 8 roundings of its magnitude: d.  Probabilities are off
    by d and by their own rounding to 16 bits (in f16 by 2^-25 of the largest at least), sums of n of them by n / 16 + 32
    roundings (a lane adds eight in 128 keys, then waves and parts); the output is rounded once more."""
    T, H, D = q.shape
    P, N = k.shape[0], k.shape[2]
    u, tiny = U16[q.dtype], TINY[q.dtype]
    out = torch.full((T, H, D), math.nan, dtype=torch.float64, device=q.device)
    lse = torch.full((T, H), math.nan, dtype=torch.float64, device=q.device)
    bound, lbound = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(len(lens)):
        s0, s1 = max(starts[b], 0), min(starts[b + 1], T)
        n, own = s1 - s0, min(max(lens[b], 0), max_len)
        for i in range(n):
            t, see = s0 + i, own - n + i + 1
            places = torch.arange(max(see, 0), device=q.device)
            pages = table[b][places // page_size].long()
            ok = (pages >= 0) & (pages < P)
            pages, slots = pages[ok], (places % page_size)[ok]
            for g in range(N):
                hs = slice(g * H // N, (g + 1) * H // N)
                if not len(pages):
                    out[t, hs], lse[t, hs] = 0.0, -math.inf
                    continue
                kk, vv, qq = k[pages, slots, g].double(), v[pages, slots, g].double(), q[t, hs].double()
                s = (qq @ kk.t().contiguous()) * scale
                d = ((qq.abs() @ kk.abs().t().contiguous()) * scale).amax(-1, keepdim=True) * (D / 8 + 8) * U32
                m = s.amax(-1, keepdim=True)
                e = torch.exp(s - m)
                p = e / e.sum(-1, keepdim=True)
                r = (len(pages) / 16 + 32) * U32
                out[t, hs], lse[t, hs] = p @ vv, (m + torch.log(e.sum(-1, keepdim=True)))[:, 0]
                mag = p @ vv.abs()
                bound[t, hs] = (u + 2 * d + r) * mag + u * out[t, hs].abs() + tiny + tiny * vv.abs().sum(0) / e.sum(-1, keepdim=True)
                lbound[t, hs] = (d + r)[:, 0] + 4 * U32 * (1 + lse[t, hs].abs())
    return out, lse, bound, lbound


# ---- log probabilities ------------------------------------------------------------------------------------------

def logprobs64(row, token, temperature, n_top):
    """(logp, rank, entropy, top, top_logp) of one row, by the header's rules, and the bounds of logp (per unit of
    distance from the largest logit, and beside it) and entropy: a lane adds up to 16 of every 4096 values, joins a few
    more; exp2 and its argument are off by two half steps each, relative to the argument where it is large."""
    V = row.numel()
    v = row.double().cpu()
    v = torch.where(torch.isnan(v), -math.inf, v) + 0.0
    T = min(max(temperature, 2.0 ** -126), 1e30) if temperature > 0 else 0.0
    order = sorted(range(V), key=lambda i: (-v[i].item(), i)) if V <= 4096 else torch.sort(v, descending=True, stable=True).indices.tolist()
    top = v[order[0]].item()
    if top == -math.inf:
        logp, entropy = torch.full((V,), -math.inf, dtype=torch.float64), 0.0
    elif T == 0.0:
        logp, entropy = torch.full((V,), -math.inf, dtype=torch.float64), 0.0
        logp[order[0]] = 0.0
    elif top == math.inf:
        n = int((v == math.inf).sum())
        logp, entropy = torch.where(v == math.inf, -math.log(n), -math.inf), math.log(n)
    else:
        x = (v - top) / T                     # from the largest logit: beside 1e30 a logarithm would be lost in 64 bits too
        logp = x - torch.logsumexp(x, -1)
        p = torch.exp(logp)
        entropy = -float(torch.special.xlogy(p, p).sum())
    drawn = [i for i in order[:n_top] if v[i] > -math.inf]
    fill = n_top - len(drawn)
    inside = 0 <= token < V
    return (float(logp[token]) if inside else -math.inf, order.index(token) if inside else -1, entropy,
            drawn + [-1] * fill, [float(logp[i]) for i in drawn] + [-math.inf] * fill)


def logp_bound(vocab, logp):
    return (vocab / 256 + 64) * U32 + 4 * U32 * (abs(logp) if math.isfinite(logp) else 0.0)


def entropy_bound(vocab, entropy):
    return (vocab / 256 + 64) * 4 * U32 * (1 + entropy)
