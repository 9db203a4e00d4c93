"""examples/batched_decode.py: every step's logits against the whole model in 64 bits, and its tokens against them."""
import importlib.util
import os

import pytest
import torch

from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("batched_decode", os.path.join(ROOT, "examples", "batched_decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def forward64(m, tokens, n_prompt, adapter):
    """Logits of every token of one request, prompt (without the adapter) and all, on the CPU."""
    D = lambda t: t.double().cpu()  # noqa: E731

    def norm(v, w):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-5) * D(w)

    h = D(m.embed)[tokens]
    T, G = len(tokens), m.heads // m.kv_heads
    seen = torch.ones(T, T, dtype=torch.bool).tril()
    for w in m.layers:
        def project(p, x):
            y = x @ D(w[p]).t()
            y[n_prompt:] += x[n_prompt:] @ D(w["a"][p][adapter]).t() @ D(w["b"][p][adapter]).t()
            return y

        x = norm(h, w["before_attn"])
        q, k, v = (project(p, x).view(T, -1, m.dim).transpose(0, 1) for p in "qkv")
        k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
        s = (q @ k.transpose(1, 2) * m.dim ** -0.5).masked_fill(~seen, -torch.inf)
        a = (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(T, -1)
        h = h + norm(project("o", a), w["after_attn"])
        x = norm(h, w["before_mlp"])
        h = h + norm(project("d", torch.nn.functional.silu(project("g", x)) * project("u", x)), w["after_mlp"])
    return norm(h, m.norm) @ D(m.head).t()


@pytest.mark.parametrize("drafts,temperature", [(0, 0.0), (3, 0.0), (4, 0.9)])
def test_decodes_as_the_whole_model_does(example, drafts, temperature):
    m = example.Model(vocab=211, seed=3)
    prompt, firsts, steps = [(5 * i * i + i) % 37 for i in range(90)], [3, 200, 3, 77, 9], 6
    rows = []                                             # (fed tokens, logits, accepted) of every step
    history, share = example.decode(m, prompt, firsts, drafts, steps, temperature, seed=1,
                                    each=lambda t, l, a: rows.append((t.tolist(), l.double().cpu().view(5, drafts + 1, -1), a)))
    assert 0.0 <= share <= 1.0
    worst = 0.0
    for b in range(5):
        want = forward64(m, prompt + history[b], 90, b % m.adapters)[90:]
        at = 0
        for fed, logits, accepted in rows:
            for i in range(accepted[b] + 1):
                assert fed[b][i] == history[b][at + i]
                y, ref = logits[b, i], want[at + i]
                worst = max(worst, float((y - ref).norm() / ref.norm()))
                if temperature == 0.0:
                    assert history[b][at + i + 1] == int(y.argmax())
            at += accepted[b] + 1
        assert at + 1 == len(history[b])
    # 16-bit activations and probabilities: about 2^-11 each, some twenty of them on a path of two layers
    assert worst < 1e-2, worst
