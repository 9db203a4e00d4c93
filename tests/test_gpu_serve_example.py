"""examples/paged_decode.py: every row's logits and scores against the whole model in 64 bits, requests coming and going."""
import importlib.util
import os

import pytest
import torch

from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_decode", os.path.join(ROOT, "examples", "paged_decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def forward64(m, tokens):
    """Logits of every token of one request, on the CPU."""
    D = lambda t: t.double().cpu()  # noqa: E731

    def norm(v, w):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-5) * D(w)

    T, G = len(tokens), m.heads // m.kv_heads
    angle = torch.arange(T, dtype=torch.float64)[:, None] * D(m.freqs)
    cos, sin = torch.cos(angle), torch.sin(angle)

    def turned(v):
        a, b = v[..., :m.dim // 2], v[..., m.dim // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    h = D(m.embed)[tokens]
    seen = torch.ones(T, T, dtype=torch.bool).tril()
    for w in m.layers:
        x = norm(h, w["before_attn"])
        q, k, v = ((x @ D(w[p]).t()).view(T, -1, m.dim).transpose(0, 1) for p in "qkv")
        q, k = turned(norm(q, w["q_norm"])), turned(norm(k, w["k_norm"]))
        k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
        s = (q @ k.transpose(1, 2) * m.dim ** -0.5).masked_fill(~seen, -torch.inf)
        h = h + (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(T, -1) @ D(w["o"]).t()
        x = norm(h, w["before_mlp"])
        h = h + (torch.nn.functional.silu(x @ D(w["g"]).t()) * (x @ D(w["u"]).t())) @ D(w["d"]).t()
    return norm(h, m.norm) @ D(m.head).t()


def test_serves_as_the_whole_model_does(example):
    m = example.Model(vocab=211, seed=5)
    server = example.Server(m, seqs=3, pages=9, page_size=8, longest=40, alternatives=3)
    prompts = [[(5 * i * i + r) % 37 for i in range(n)] for r, n in enumerate((1, 20, 7, 16, 3))]
    rows = [[] for _ in prompts]

    def each(places, counts, tokens):
        row = 0
        for r, c in zip(places, counts):
            for _ in range(c):
                i, row = row, row + 1
                rows[r].append((server.logits[i].double().cpu(), server.top[i].tolist(), server.top_logp[i].tolist(),
                                float(server.entropy[i]), int(server.given[i]), float(server.logp[i]), int(server.rank[i])))

    history, scored = example.serve(server, prompts, 9, each)
    assert sorted(server.free) == list(range(9))
    for r, prompt in enumerate(prompts):
        assert len(history[r]) == len(prompt) + 9 and len(rows[r]) == len(history[r]) - 1
        want = forward64(m, history[r][:-1])
        answer = 0.0
        for i, (logits, top, top_logp, entropy, given, logp, rank) in enumerate(rows[r]):
            # 16-bit activations, keys and probabilities: about 2^-11 each, some twenty of them on a path of two layers
            assert float((logits - want[i]).norm() / want[i].norm()) < 1e-2
            p = torch.log_softmax(logits, -1)             # the scores against the logits they were taken from
            order = torch.sort(logits, descending=True, stable=True).indices
            assert top == order[:3].tolist() and all(abs(a - float(p[x])) < 1e-5 for a, x in zip(top_logp, top))
            assert abs(entropy + float((p.exp() * p).sum())) < 1e-4
            if i + 1 < len(prompt):
                assert given == prompt[i + 1] and abs(logp - float(p[given])) < 1e-5 and order[rank] == given
            else:
                assert given == -1 and rank == -1 and history[r][i + 1] == top[0]
                answer += top_logp[0]
        assert abs(answer - scored[r][1]) < 1e-4
