"""The step operators' definitions in 64 bits, element by element from their formulas, with the bound that each
result's rounding gives (used by the GPU tests and pinned by the CPU tests)."""
import math

import torch

U16 = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}    # unit roundoffs
U32 = 2.0 ** -24


def norm64(u, kind, w, b, eps):
    if kind == "layer":
        u = u - u.mean(-1, keepdim=True)
    u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + eps)
    if w is not None:
        u = u * w.double()
    return u if b is None else u + b.double()


def block64(y, h, *, kind, post, post_w=None, post_b=None, gate=None, res=1.0, pre_w=None, pre_b=None, eps=1e-5):
    v = torch.zeros_like(h, dtype=torch.float64) if y is None else y.double()
    if post and y is not None:
        v = norm64(v, kind, post_w, post_b, eps)
    if gate is not None:
        v = v * gate.double()
    hp = v if h is None else res * h.double() + v
    return hp, norm64(hp, kind, pre_w, pre_b, eps)


def lora64(x, a, b, ids, ranks, scales, y0):
    """y and the sum of magnitudes |B| |A| |x| that its rounding is measured against."""
    T, n = x.shape[0], a.shape[0]
    y = torch.zeros((T, b.shape[1]), dtype=torch.float64, device=x.device) if y0 is None else y0.double().clone()
    mag = y.abs()
    for t in range(T):
        i = int(ids[t])
        if not 0 <= i < n:
            continue
        r = a.shape[1] if ranks is None else min(max(int(ranks[i]), 0), a.shape[1])
        s = 1.0 if scales is None else float(scales[i])
        A, B = a[i, :r].double(), b[i, :, :r].double()
        y[t] += s * (B @ (A @ x[t].double()))
        mag[t] += abs(s) * (B.abs() @ (A.abs() @ x[t].double().abs()))
    return y, mag


def attn64(q, kp, vp, k, v, starts, lens, scale):
    """out, lse and sum p |v| of every row; q (T, H, D), kp (P, N, D), k (B, S, N, D)."""
    T, H, D = q.shape
    N = k.shape[2]
    out = torch.zeros((T, H, D), dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=q.device)
    for b in range(len(lens)):
        n, own = starts[b + 1] - starts[b], min(max(lens[b], 0), k.shape[1])
        for i in range(n):
            t, see = starts[b] + i, own - n + i + 1
            for g in range(N):
                hs = slice(g * H // N, (g + 1) * H // N)
                kk, vv = kp[:, g].double(), vp[:, g].double()
                if see > 0:
                    kk, vv = torch.cat([kk, k[b, :see, g].double()]), torch.cat([vv, v[b, :see, g].double()])
                if not kk.shape[0]:
                    continue
                s = (q[t, hs].double() @ kk.t().contiguous()) * scale
                lse[t, hs] = torch.logsumexp(s, -1)
                p = torch.softmax(s, -1)
                out[t, hs], mag[t, hs] = p @ vv, p @ vv.abs()
    return out, lse, mag


def dist64(row, temperature):
    """The distribution of a row of logits, by the header's rules."""
    v = row.double()
    v = torch.where(torch.isnan(v), -math.inf, v)
    top = v.max()
    p = torch.zeros_like(v)
    if top == -math.inf:
        return p
    if not temperature > 0:
        p[int((v == top).nonzero()[0])] = 1.0
        return p
    if top == math.inf:
        p[v == math.inf] = 1.0
    else:
        p = torch.exp((v - top) / temperature)
    return p / p.sum()


def verify64(target, draft, tokens, counts, temps, uniform, noise):
    """(out, accepted, logp) of every sequence and how near its closest decision came (relative)."""
    B, rows, V = target.shape
    n = rows - 1
    result = []
    for b in range(B):
        c, T = min(max(counts[b], 0), n), temps[b]
        out, logp, near, a = [-1] * rows, [0.0] * rows, math.inf, 0
        while True:
            p = dist64(target[b, a], T)
            w = p
            if a < c:
                x = tokens[b][a]
                q = torch.zeros_like(p)
                if draft is not None:
                    q = dist64(draft[b, a], T)
                elif 0 <= x < V:
                    q[x] = 1.0
                if 0 <= x < V:
                    left, right = uniform[b][a] * float(q[x]), float(p[x])
                    if max(left, right) > 0:
                        near = min(near, abs(left - right) / max(left, right))
                    if left < right:
                        out[a], logp[a], a = x, math.log(float(p[x])), a + 1
                        continue
                w = (p - q).clamp(min=0)
                w = torch.where(w > 1e-6 * p, w, 0.0) if draft is not None else w
                if not float(w.max()) > 0:
                    w = p
            break
        score = w / noise[b].double()
        top = score.topk(min(2, V)).values.tolist()
        if top[0] > 0:
            token = int((score == score.max()).nonzero()[0])
            if len(top) > 1:
                near = min(near, (top[0] - top[1]) / top[0])
            out[a], logp[a] = token, math.log(float(p[token])) if float(p[token]) > 0 else -math.inf
        else:
            logp[a] = -math.inf
        result.append((out, a, logp, near))
    return result
