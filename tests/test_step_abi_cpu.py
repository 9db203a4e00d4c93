"""The step operators' C ABI on a machine without a GPU: the library exports what include/wsr_step.h declares and
rejects bad arguments before touching the HIP runtime (no call here gets as far as a launch)."""
import ctypes
import os
import re

import pytest
import torch

import step_util as su
from paper_2608_12114_amd import wsr
from paper_2608_12114_amd import wsr_step as ws

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "wsr_step.h")).read()
L = ws.step_lib()
A = 0x10000          # an aligned fake address, never dereferenced
ARG, ALIGN, SIZE, OK = wsr.WSR_E_ARG, wsr.WSR_E_ALIGN, wsr.WSR_E_SIZE, wsr.WSR_OK


def test_exports_every_declared_symbol():
    body = re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)
    names = sorted(set(re.findall(r"\b(wsr_[a-z0-9_]+)\s*\(", body)))
    assert len(names) == 8, names
    for n in names:
        assert hasattr(L, n) and hasattr(wsr, n), n


def test_structures_match_the_header():
    for cls in (ws.wsr_block, ws.wsr_lora, ws.wsr_attn, ws.wsr_verify):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (cls.__name__, cls.__name__), HEADER, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        names = []
        for decl in body.split(";"):
            decl = re.sub(r"\b(const|int32_t|int64_t|float|void)\b", "", decl).replace("*", "")
            names += [n.strip() for n in decl.split(",") if n.strip()]
        assert names == [n for n, _ in cls._fields_], cls


def _block(**over):
    return ws.make_block(**{**dict(kind=0, fmt=1, n_tokens=2, d=64, y=A, y_tok_stride=256, h=A, h_tok_stride=256, h_out=A,
                                   h_out_tok_stride=256, x=A, x_tok_stride=128), **over})


@pytest.mark.parametrize("over,st", [
    (dict(kind=2), ARG), (dict(fmt=3), ARG), (dict(flags=2), ARG), (dict(reserved=1), ARG), (dict(n_tokens=-1), ARG),
    (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG), (dict(d=60), ALIGN), (dict(d=32776), SIZE), (dict(d=-8), ARG),
    (dict(y_tok_stride=-16), ALIGN), (dict(y_tok_stride=8), ALIGN), (dict(y=A + 4), ALIGN), (dict(pre_w=A + 2), ALIGN),
    (dict(gate=A + 8), ALIGN), (dict(x_tok_stride=112), ARG), (dict(h_out_tok_stride=240), ARG), (dict(h_tok_stride=512), ARG),
    (dict(y=None, h=None), ARG), (dict(x=None, h_out=None), ARG), (dict(n_tokens=1 << 40, y_tok_stride=1 << 40), SIZE),
    (dict(n_tokens=0, y=None, h=None), OK), (dict(d=0), OK)])
def test_block_norm_refusals(over, st):
    assert L.wsr_block_norm(_block(**over), None) == st, ws.wsr_step_last_error()
    assert bool(ws.wsr_step_last_error()) == (st != OK)


def test_null_structures():
    assert L.wsr_block_norm(None, None) == ARG
    assert L.wsr_prefix_attention(None, A, 1 << 20, None) == ARG and L.wsr_attn_workspace_bytes(None) == 0
    assert L.wsr_verify_drafts(None, A, 1 << 20, None) == ARG and L.wsr_verify_workspace_bytes(None) == 0
    assert L.wsr_lora_sweep(None, 1, 1, A, 1, None, None, A, 1 << 20, None) == ARG
    assert L.wsr_lora_workspace_bytes(None, 1, 1) == 0
    with pytest.raises(wsr.WsrError) as e:
        wsr.wsr_block_norm(_block(kind=9))
    assert e.value.status == ARG and "kind" in str(e.value)


def _lora(**over):
    return {**dict(fmt=2, rank=16, M=64, K=64, a=A, a_stride=2048, b=A, b_stride=2048, x=A, x_tok_stride=128, y0=A,
                   y0_tok_stride=256, y=A, y_tok_stride=256), **over}


@pytest.mark.parametrize("over,st", [
    (dict(fmt=4), ARG), (dict(rank=0), ARG), (dict(rank=257), ARG), (dict(M=-1), ARG), (dict(K=12), ALIGN),
    (dict(K=1 << 30), SIZE), (dict(M=1 << 31), SIZE), (dict(a=A + 8), ALIGN), (dict(x=A + 2), ALIGN), (dict(b=A + 1), ALIGN),
    (dict(y=A + 2), ALIGN), (dict(a_stride=2056), ALIGN), (dict(b_stride=3), ALIGN), (dict(x_tok_stride=-16), ALIGN),
    (dict(y_tok_stride=252), ARG), (dict(y0_tok_stride=512), ARG), (dict(y=None), ARG), (dict(b=None), ARG), (dict(x=None), ARG),
    (dict(a_stride=1 << 60), SIZE)])
def test_lora_refusals(over, st):
    mods = ws.make_loras([_lora(), _lora(**over)])
    need = wsr.wsr_lora_workspace_bytes(ws.make_loras([_lora()] * 2), 4)
    assert L.wsr_lora_sweep(mods, 2, 4, A, 3, None, None, A, need, None) == st
    assert "projection 1" in ws.wsr_step_last_error()


def test_lora_call_refusals():
    mods = ws.make_loras([_lora()])
    need = wsr.wsr_lora_workspace_bytes(mods, 4)
    f = L.wsr_lora_sweep
    assert f(mods, -1, 4, A, 3, None, None, A, need, None) == ARG
    assert f(mods, 1, -1, A, 3, None, None, A, need, None) == ARG
    assert f(mods, 1, (1 << 20) + 1, A, 3, None, None, A, 1 << 40, None) == SIZE
    assert f(mods, 1, 4, None, 3, None, None, A, need, None) == ARG
    assert f(mods, 1, 4, A, 8193, None, None, A, need, None) == SIZE
    assert f(mods, 1, 4, A, -1, None, None, A, need, None) == SIZE
    assert f(mods, 1, 4, A + 2, 3, None, None, A, need, None) == ALIGN
    assert f(mods, 1, 4, A, 3, None, None, A, need - 1, None) == SIZE
    assert f(mods, 1, 4, A, 3, None, None, A + 16, need, None) == ALIGN
    assert f(mods, 1, 4, A, 3, None, None, None, need, None) == ARG
    assert f(mods, 1, 0, None, 3, None, None, None, 0, None) == OK
    assert f(None, 0, 4, None, 3, None, None, None, 0, None) == OK


def _attn(**over):
    return ws.make_attn(**{**dict(fmt=2, n_heads=8, n_kv_heads=2, head_dim=64, n_seqs=3, n_tokens=4, scale=0.125, q=A,
                                  q_tok_stride=1024, q_head_stride=128, k_prefix=A, v_prefix=A, prefix_len=10,
                                  prefix_tok_stride=256, prefix_head_stride=128, k=A, v=A, max_len=5, kv_seq_stride=1280,
                                  kv_tok_stride=256, kv_head_stride=128, starts=A, lens=A, out=A, out_tok_stride=1024,
                                  out_head_stride=128, lse=A), **over})


@pytest.mark.parametrize("over,st", [
    (dict(fmt=3), ARG), (dict(head_dim=96), SIZE), (dict(n_heads=9), ARG), (dict(n_kv_heads=0), ARG), (dict(n_heads=1), ARG),
    (dict(n_seqs=-1), ARG), (dict(n_tokens=-1), ARG), (dict(prefix_len=-1), ARG), (dict(max_len=-1), ARG),
    (dict(max_len=1 << 31), SIZE), (dict(n_tokens=1 << 21), SIZE), (dict(scale=0.0), ARG), (dict(scale=float("inf")), ARG),
    (dict(scale=float("nan")), ARG), (dict(starts=None), ARG), (dict(n_seqs=0), ARG), (dict(q_tok_stride=1000), ALIGN),
    (dict(kv_tok_stride=-16), ALIGN), (dict(prefix_tok_stride=(16 << 20) + 16), SIZE), (dict(kv_seq_stride=1 << 62), SIZE),
    (dict(q=A + 8), ALIGN), (dict(v=A + 2), ALIGN), (dict(lens=A + 2), ALIGN), (dict(lse=A + 1), ALIGN), (dict(q=None), ARG),
    (dict(lens=None), ARG), (dict(v_prefix=None), ARG), (dict(k=None), ARG), (dict(out=None), ARG), (dict(out_head_stride=112), ARG),
    (dict(out_tok_stride=0), ARG), (dict(reserved=1), ARG), (dict(n_tokens=0), OK)])
def test_attention_refusals(over, st):
    need = wsr.wsr_attn_workspace_bytes(_attn())
    assert need > 0
    assert L.wsr_prefix_attention(_attn(**over), A, max(need, 1 << 40), None) == st, ws.wsr_step_last_error()


def test_attention_row_numbers_fit():
    """2^20 tokens of 4096 heads on one key head are more rows than are counted in 32 bits."""
    wide = _attn(n_heads=4096, n_kv_heads=1, n_tokens=1 << 20, q_head_stride=16, out_head_stride=128)
    assert L.wsr_prefix_attention(wide, A, 1 << 40, None) == SIZE
    assert wsr.wsr_attn_workspace_bytes(wide) == 0


def test_attention_workspace():
    need = wsr.wsr_attn_workspace_bytes(_attn())
    assert L.wsr_prefix_attention(_attn(), A, need - 1, None) == SIZE
    assert L.wsr_prefix_attention(_attn(), A + 16, need, None) == ALIGN
    assert L.wsr_prefix_attention(_attn(), None, need, None) == ARG


def _verify(**over):
    return ws.make_verify(**{**dict(n_seqs=2, n_drafts=3, vocab=100, target=A, target_seq_stride=1600, target_row_stride=400,
                                    draft=A, draft_seq_stride=1200, draft_row_stride=400, tokens=A, counts=A, temperature=A,
                                    uniform=A, noise=A, noise_seq_stride=400, out=A, accepted=A, logp=A), **over})


@pytest.mark.parametrize("over,st", [
    (dict(n_seqs=-1), ARG), (dict(n_drafts=-1), ARG), (dict(n_drafts=64), SIZE), (dict(vocab=0), ARG),
    (dict(vocab=(1 << 24) + 1), SIZE), (dict(n_seqs=1 << 17), SIZE), (dict(target_row_stride=402), ALIGN),
    (dict(noise_seq_stride=-4), ALIGN), (dict(target=A + 2), ALIGN), (dict(tokens=A + 1), ALIGN), (dict(target=None), ARG),
    (dict(noise=None), ARG), (dict(out=None), ARG), (dict(accepted=None), ARG), (dict(tokens=None), ARG), (dict(uniform=None), ARG),
    (dict(target_seq_stride=1 << 62), SIZE), (dict(n_seqs=0), OK)])
def test_verify_refusals(over, st):
    need = wsr.wsr_verify_workspace_bytes(_verify())
    assert L.wsr_verify_drafts(_verify(**over), A, max(need, 1 << 40), None) == st, ws.wsr_step_last_error()


def test_verify_workspace():
    need = wsr.wsr_verify_workspace_bytes(_verify())
    assert L.wsr_verify_drafts(_verify(), A, need - 1, None) == SIZE
    assert L.wsr_verify_drafts(_verify(), A + 16, need, None) == ALIGN
    assert L.wsr_verify_drafts(_verify(), None, need, None) == ARG


# ---- the 64-bit definitions the GPU tests compare with, on hand-made values ---------------------------------

def test_definitions_by_hand():
    y, h = torch.tensor([[3.0, 4.0]]), torch.tensor([[1.0, 1.0]])
    hp, x = su.block64(y, h, kind="rms", post=True, gate=torch.tensor([2.0, 0.0]), res=0.5, eps=0.0)
    r = 3 / (12.5 ** 0.5) * 2 + 0.5                      # mean square of (3, 4) is 12.5
    assert torch.allclose(hp, torch.tensor([[r, 0.5]], dtype=torch.float64))
    assert torch.allclose(x, hp / ((r * r + 0.25) / 2) ** 0.5)
    _, x = su.block64(None, torch.tensor([[1.0, 3.0]]), kind="layer", post=False, eps=0.0)
    assert torch.allclose(x, torch.tensor([[-1.0, 1.0]], dtype=torch.float64))
    one = lambda *v: torch.tensor(v, dtype=torch.float32)  # noqa: E731
    y, _ = su.lora64(one(1, 2)[None], one(1, 1)[None, None], one(5, 7)[None, :, None], [0], None, [2.0], one(1, 1)[None])
    assert y.tolist() == [[31.0, 43.0]]                  # 1 + 2 * 5 * 3, 1 + 2 * 7 * 3
    q, k, v = torch.zeros(2, 1, 2), torch.zeros(1, 3, 1, 2), one(1, 2, 4).view(1, 3, 1, 1).expand(1, 3, 1, 2)
    out, lse, _ = su.attn64(q, torch.zeros(0, 1, 2), torch.zeros(0, 1, 2), k, v, [0, 2], [3], 1.0)
    assert out[:, 0, 0].tolist() == pytest.approx([1.5, 7 / 3]) and lse.exp()[:, 0].tolist() == pytest.approx([2, 3])
    t = torch.log(one(0.5, 0.5, 0.25)).expand(1, 2, 3)
    r = su.verify64(t, None, [[2]], [1], [1.0], [[0.1]], torch.ones(1, 3))
    assert r[0][:2] == ([2, 0], 1)                       # 0.1 * 1 < 0.2; then the lowest of the equal scores
    r = su.verify64(t, None, [[2]], [1], [1.0], [[0.3]], one(1, 0.5, 1)[None])
    assert r[0][:2] == ([1, -1], 0)
