"""Step operators over more rows than one launch holds workgroups for: a launch of 2^32 threads or more would be cut to what
is left over 2^32, without an error."""
import pytest
import torch

import step_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
NAN = float("nan")


@pytest.mark.parametrize("T,d", [((1 << 26) + 5, 8), ((1 << 24) + 3, 520)])
def test_norms(T, d):
    """Rows of 64 threads, and of 256: 1000 kinds of rows over and over."""
    kinds = 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    some = torch.randn((kinds, d), generator=g, device="cuda")
    of = torch.arange(T, device="cuda") % kinds
    every = lambda t: t.repeat(-(-T // kinds), 1)[:T]  # noqa: E731  (torch gathers 16-byte rows wrongly past 2^26)
    y = every(some)
    h = torch.full((T, d), NAN, device="cuda")
    x = torch.full((T, d), NAN, dtype=torch.bfloat16, device="cuda")
    gate = torch.randn((kinds, d), generator=g, device="cuda").to(torch.bfloat16)
    gates = every(gate) if d == 8 else gate[:1]
    wsr.wsr_block_norm(wsr.make_block(kind=wsr.WSR_NORM_RMS, fmt=wsr.WSR_BF16, flags=wsr.WSR_BLOCK_POST, n_tokens=T, d=d, y=y, y_tok_stride=4 * d,
                                      gate=gates, gate_tok_stride=2 * d if d == 8 else 0, h_out=h, h_out_tok_stride=4 * d, x=x,
                                      x_tok_stride=2 * d), stream())
    torch.cuda.synchronize()
    for t in (0, T - 7):                                    # against the formula, at both ends
        kind = of[t:t + 7]
        eh, ex = su.block64(some[kind], None, kind="rms", post=True, gate=gate[kind] if d == 8 else gate[:1])
        assert ((h[t:t + 7].double() - eh).abs() <= 64 * su.U32 * (1 + eh.abs())).all()
        assert ((x[t:t + 7].double() - ex).abs() <= su.U16[torch.bfloat16] * ex.abs() + 1e-5).all()
    step = kinds << 14                                      # equal rows have equal bits, whichever launch took them
    for t in range(0, T, step):
        n = min(step, T - t)
        assert torch.equal(h[t:t + n].view(torch.int32), h[:kinds].repeat(-(-n // kinds), 1)[:n].view(torch.int32))
        assert torch.equal(x[t:t + n].view(torch.int16), x[:kinds].repeat(-(-n // kinds), 1)[:n].view(torch.int16))


def test_attention_rows():
    """2^20 tokens of 65 heads behind a single key: every output is its value, every lse its score."""
    T, H, D, B = 1 << 20, 65, 64, 20000
    g = torch.Generator(device="cuda").manual_seed(2)
    q, kp, vp = (torch.randn((1, H, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    starts[-1] = T
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = torch.full((T, H, D), NAN, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, H), NAN, device="cuda")
    p = wsr.make_attn(fmt=wsr.WSR_BF16, n_heads=H, n_kv_heads=H, head_dim=D, n_seqs=B, n_tokens=T, scale=0.125, q=q, q_head_stride=2 * D,
                      k_prefix=kp, v_prefix=vp, prefix_len=1, prefix_tok_stride=2 * H * D, prefix_head_stride=2 * D, max_len=0,
                      starts=starts, lens=lens, out=out, out_tok_stride=2 * H * D, out_head_stride=2 * D, lse=lse)
    ws = torch.empty(wsr.wsr_attn_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    wsr.wsr_prefix_attention(p, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    want = (q[0].double() * kp[0].double()).sum(-1) * 0.125
    for t in range(0, T, 1 << 16):
        assert (out[t:t + (1 << 16)] == vp[0]).all()
        assert ((lse[t:t + (1 << 16)].double() - want).abs() <= 1e-5).all()


def test_verification_rows():
    """65536 sequences with room for 63 drafts over 16384 logits that all of them share."""
    B, n, V = 1 << 16, 63, 16384
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn(V, generator=g, device="cuda")
    noise = torch.empty(V, device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    tokens = torch.randint(0, V, (B, n), generator=g, device="cuda").to(torch.int32)
    counts = torch.arange(B, device="cuda").remainder(n + 1).to(torch.int32)
    uniform = torch.zeros((B, n), device="cuda")            # every draft is accepted
    out = torch.full((B, n + 1), -7, dtype=torch.int32, device="cuda")
    accepted = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    p = wsr.make_verify(n_seqs=B, n_drafts=n, vocab=V, target=logits, tokens=tokens, counts=counts, uniform=uniform, noise=noise, out=out,
                        accepted=accepted)
    ws = torch.empty(wsr.wsr_verify_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    wsr.wsr_verify_drafts(p, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    assert torch.equal(accepted, counts)
    place, c = torch.arange(n + 1, device="cuda"), counts[:, None]
    pad = torch.nn.functional.pad(tokens, (0, 1))
    want = torch.where(place < c, pad, -1)
    score = torch.softmax(logits.double(), -1) / noise.double()
    assert float(score.topk(2).values[1]) < 0.999 * float(score.max())
    want = torch.where(place == c, int(score.argmax()), want).to(torch.int32)
    assert torch.equal(out, want)
