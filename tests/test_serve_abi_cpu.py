"""The serving operators' C ABI on a machine without a GPU: the library exports what include/wsr_serve.h declares and rejects
bad arguments before touching the HIP runtime (no call here gets as far as a launch)."""
import ctypes
import math
import os
import re

import pytest
import torch

import serve_util as su
from paper_2608_12114_amd import wsr
from paper_2608_12114_amd import wsr_serve as ws

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "wsr_serve.h")).read()
L = ws.serve_lib()
A = 0x10000          # an aligned fake address, never dereferenced
ARG, ALIGN, SIZE, OK = wsr.WSR_E_ARG, wsr.WSR_E_ALIGN, wsr.WSR_E_SIZE, wsr.WSR_OK


def test_exports_every_declared_symbol():
    body = re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)
    names = sorted(set(re.findall(r"\b(wsr_[a-z0-9_]+)\s*\(", body)))
    assert len(names) == 6, names
    for n in names:
        assert hasattr(L, n) and hasattr(wsr, n), n


def test_structures_match_the_header(tmp_path):
    """Names and order from the header's text, sizes and offsets from a C compiler."""
    classes = (ws.wsr_pages, ws.wsr_qkv, ws.wsr_paged, ws.wsr_logprobs)
    lines = []
    for cls in classes:
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (cls.__name__, cls.__name__), HEADER, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        names = []
        for decl in body.split(";"):
            decl = re.sub(r"\b(const|int32_t|int64_t|float|void|wsr_pages)\b", "", decl).replace("*", "")
            names += [n.strip() for n in decl.split(",") if n.strip()]
        assert names == [n for n, _ in cls._fields_], cls
        lines += [f'printf("%zu ", sizeof({cls.__name__}));'] + [f'printf("%zu ", offsetof({cls.__name__}, {n}));' for n in names]
    src = tmp_path / "t.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "wsr_serve.h"\nint main(void) {' + "".join(lines) + "return 0; }\n")
    import subprocess
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in classes:
        want += [ctypes.sizeof(cls)] + [getattr(cls, n).offset for n, _ in cls._fields_]
    assert got == want


def _pages(**over):
    return ws.make_pages(**{**dict(k=A, v=A, n_pages=8, page_size=16, page_stride=16 * 512, tok_stride=512, head_stride=256,
                                   table=A, table_stride=16, max_pages=4), **over})


BAD_PAGES = [(dict(n_pages=-1), ARG), (dict(page_size=0), SIZE), (dict(page_size=(1 << 20) + 1), SIZE), (dict(max_pages=-1), ARG),
             (dict(max_pages=1 << 27), SIZE), (dict(k=None), ARG), (dict(v=None), ARG), (dict(table=None), ARG), (dict(k=A + 8), ALIGN),
             (dict(v=A + 2), ALIGN), (dict(table=A + 2), ALIGN), (dict(page_stride=8), ALIGN), (dict(tok_stride=-16), ALIGN),
             (dict(head_stride=24), ALIGN), (dict(table_stride=6), ALIGN), (dict(page_stride=1 << 62), SIZE), (dict(reserved=1), ARG)]


def _qkv(cache=None, **over):
    return ws.make_qkv(**{**dict(fmt=wsr.WSR_BF16, flags=1, kind=0, n_heads=4, n_kv_heads=2, head_dim=128, rot_dim=128, n_seqs=2, n_tokens=3,
                                 q=A, q_tok_stride=2048, k=A, k_tok_stride=1024, v=A, v_tok_stride=1024, freqs=A, starts=A, lens=A,
                                 q_out=A, q_out_tok_stride=1024, q_out_head_stride=256, cache=cache or _pages()), **over})


@pytest.mark.parametrize("over,st", [
    (dict(fmt=0), ARG), (dict(fmt=3), ARG), (dict(flags=4), ARG), (dict(kind=2), ARG), (dict(reserved=1), ARG), (dict(eps=-1.0), ARG),
    (dict(eps=math.nan), ARG), (dict(head_dim=96), SIZE), (dict(rot_dim=4), SIZE), (dict(rot_dim=136), SIZE), (dict(rot_dim=-8), SIZE),
    (dict(n_axes=0), ARG), (dict(n_axes=5), ARG), (dict(n_axes=2), ARG), (dict(n_heads=-1), ARG), (dict(n_kv_heads=-1), ARG),
    (dict(n_heads=4097), SIZE), (dict(n_tokens=-1), ARG), (dict(n_seqs=-1), ARG), (dict(n_tokens=(1 << 20) + 1), SIZE),
    (dict(n_seqs=(1 << 20) + 1), SIZE), (dict(k=None), ARG), (dict(v=None), ARG), (dict(starts=None), ARG), (dict(lens=None), ARG),
    (dict(n_seqs=0), ARG), (dict(q_out=None), ARG), (dict(freqs=None), ARG), (dict(q=A + 4), ALIGN), (dict(k=A + 8), ALIGN),
    (dict(v=A + 8), ALIGN), (dict(q_w=A + 2), ALIGN), (dict(k_b=A + 2), ALIGN), (dict(q_out=A + 8), ALIGN), (dict(freqs=A + 2), ALIGN),
    (dict(axis_of=A + 1), ALIGN), (dict(positions=A + 2), ALIGN), (dict(starts=A + 2), ALIGN), (dict(lens=A + 3), ALIGN),
    (dict(q_tok_stride=8), ALIGN), (dict(k_tok_stride=-16), ALIGN), (dict(v_tok_stride=4), ALIGN), (dict(pos_axis_stride=2), ALIGN),
    (dict(q_out_tok_stride=240), ARG), (dict(q_out_head_stride=240), ARG), (dict(q_out_head_stride=8), ALIGN),
    (dict(q_tok_stride=1 << 62), SIZE), (dict(n_tokens=0), OK), (dict(q=None, k=None, v=None, cache=ws.wsr_pages()), OK),
    (dict(n_heads=0, n_kv_heads=0, cache=ws.wsr_pages()), OK)])
def test_append_refusals(over, st):
    assert L.wsr_append_qkv(_qkv(**over), None) == st, ws.wsr_serve_last_error()
    assert bool(ws.wsr_serve_last_error()) == (st != OK)


@pytest.mark.parametrize("over,st", BAD_PAGES + [(dict(tok_stride=240), ARG), (dict(head_stride=240), ARG), (dict(page_stride=240), ARG)])
def test_append_refuses_caches(over, st):
    assert L.wsr_append_qkv(_qkv(_pages(**over)), None) == st, ws.wsr_serve_last_error()


def _paged(cache=None, **over):
    return ws.make_paged(**{**dict(fmt=wsr.WSR_F16, n_heads=4, n_kv_heads=2, head_dim=128, n_seqs=2, n_tokens=3, scale=0.1, max_len=64, q=A,
                                   q_tok_stride=1024, q_head_stride=256, starts=A, lens=A, out=A, out_tok_stride=1024,
                                   out_head_stride=256, lse=A, cache=cache or _pages()), **over})


@pytest.mark.parametrize("over,st", [
    (dict(fmt=0), ARG), (dict(head_dim=96), SIZE), (dict(n_heads=5), ARG), (dict(n_kv_heads=0), ARG), (dict(n_heads=1), ARG),
    (dict(n_heads=8192), ARG), (dict(n_seqs=-1), ARG), (dict(n_tokens=-1), ARG), (dict(max_len=-1), ARG),
    (dict(max_len=65), SIZE), (dict(n_tokens=(1 << 20) + 1), SIZE), (dict(n_tokens=1 << 20, n_heads=64), SIZE), (dict(scale=0.0), ARG),
    (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG), (dict(starts=None), ARG), (dict(n_seqs=0), ARG), (dict(reserved=1), ARG),
    (dict(q=None), ARG), (dict(out=None), ARG), (dict(lens=None), ARG), (dict(q=A + 8), ALIGN), (dict(out=A + 4), ALIGN),
    (dict(lens=A + 2), ALIGN), (dict(starts=A + 1), ALIGN), (dict(lse=A + 2), ALIGN), (dict(q_tok_stride=8), ALIGN),
    (dict(q_head_stride=-16), ALIGN), (dict(out_tok_stride=240), ARG), (dict(out_head_stride=240), ARG), (dict(q_tok_stride=1 << 62), SIZE),
    (dict(n_tokens=0), OK)])
def test_paged_refusals(over, st):
    need = wsr.wsr_paged_workspace_bytes(_paged())
    assert need > 0
    assert L.wsr_paged_attention(_paged(**over), A, max(need, 1 << 40), None) == st, ws.wsr_serve_last_error()


@pytest.mark.parametrize("over,st", BAD_PAGES)
def test_paged_refuses_caches(over, st):
    p = _paged(_pages(**over), max_len=1)
    assert L.wsr_paged_attention(p, A, 1 << 40, None) == st, ws.wsr_serve_last_error()
    assert wsr.wsr_paged_workspace_bytes(p) == 0


def _logprobs(**over):
    return ws.make_logprobs(**{**dict(n_rows=3, vocab=1000, n_top=4, logits=A, row_stride=4000, tokens=A, temperature=A, logp=A, rank=A,
                                      entropy=A, top=A, top_logp=A), **over})


@pytest.mark.parametrize("over,st", [
    (dict(n_rows=-1), ARG), (dict(vocab=0), ARG), (dict(n_top=-1), ARG), (dict(n_top=65), SIZE), (dict(vocab=(1 << 24) + 1), SIZE),
    (dict(n_rows=(1 << 20) + 1), SIZE), (dict(n_rows=1 << 20, vocab=(1 << 20) + 1), SIZE), (dict(reserved=1), ARG),
    (dict(row_stride=-4), ALIGN), (dict(row_stride=6), ALIGN),
    (dict(row_stride=1 << 62), SIZE), (dict(logits=A + 2), ALIGN), (dict(tokens=A + 1), ALIGN), (dict(temperature=A + 2), ALIGN),
    (dict(top=A + 2), ALIGN), (dict(logits=None), ARG), (dict(top=None), ARG), (dict(tokens=None), ARG),
    (dict(tokens=None, logp=None), ARG), (dict(n_rows=0), OK)])
def test_logprobs_refusals(over, st):
    need = wsr.wsr_logprobs_workspace_bytes(_logprobs())
    assert need > 0
    assert L.wsr_token_logprobs(_logprobs(**over), A, max(need, 1 << 40), None) == st, ws.wsr_serve_last_error()


def test_workspaces_and_null_structures():
    for f, p, size in ((L.wsr_paged_attention, _paged(), wsr.wsr_paged_workspace_bytes), (L.wsr_token_logprobs, _logprobs(), wsr.wsr_logprobs_workspace_bytes)):
        need = size(p)
        assert f(p, A, need - 1, None) == SIZE
        assert f(p, A + 16, need, None) == ALIGN
        assert f(p, None, need, None) == ARG
        assert f(None, A, 1 << 20, None) == ARG and size(None) == 0
    assert L.wsr_append_qkv(None, None) == ARG
    with pytest.raises(wsr.WsrError) as e:
        wsr.wsr_append_qkv(_qkv(kind=9))
    assert e.value.status == ARG and "kind" in str(e.value)


# ---- the 64-bit definitions the GPU tests compare with, on hand-made values ---------------------------------

def test_definitions_by_hand():
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0]]])
    turn = lambda **o: su.turned64(x, torch.tensor([[1]]), torch.tensor([math.pi / 2]), None, rot=2, **o)[0][0, 0].tolist()  # noqa: E731
    assert turn(pairs=False) == pytest.approx([-2, 1, 3, 4], abs=1e-6) == turn(pairs=True)
    y = su.turned64(x, torch.tensor([[0], [1]]), torch.tensor([1.0, math.pi]), torch.tensor([0, 1]), rot=4, pairs=False)[0][0, 0]
    assert y.tolist() == pytest.approx([1, -2, 3, -4], abs=1e-6)         # the second pair (2, 4) by half a turn
    y = su.turned64(x, torch.tensor([[0]]), torch.tensor([1.0]), None, rot=0, pairs=False, kind="layer", eps=0.0)[0][0, 0]
    assert y.tolist() == pytest.approx([(v - 2.5) / 1.25 ** 0.5 for v in (1, 2, 3, 4)])
    assert su.places64([0, 2, 3], [5, 1], 4) == [(0, 3), (0, 4), (1, 0), (-1, 0)]
    table = torch.tensor([[3, -1]])
    assert su.slot64(table, 4, 4, 0, 2) == (3, 2) and su.slot64(table, 4, 4, 0, 4) is None and su.slot64(table, 4, 3, 0, 2) is None
    k, v = torch.zeros(2, 2, 1, 2), torch.tensor([4.0, 8.0, 1.0, 2.0]).view(2, 2, 1, 1).expand(2, 2, 1, 2)
    out, lse, _, _ = su.paged64(torch.zeros(2, 1, 2, dtype=torch.float16), k, v, torch.tensor([[1, 0]]), 2, [0, 2], [3], 4, 1.0)
    assert out[:, 0, 0].tolist() == pytest.approx([1.5, 7 / 3]) and lse.exp()[:, 0].tolist() == pytest.approx([2, 3])
    out, lse, _, _ = su.paged64(torch.zeros(1, 1, 2, dtype=torch.float16), k, v, torch.tensor([[1, 7]]), 2, [0, 1], [3], 4, 1.0)
    assert out[0, 0, 0] == pytest.approx(1.5)                            # page 7 is a hole
    row = torch.log(torch.tensor([0.25, 0.5, 0.25, 0.0]))
    logp, rank, entropy, top, top_logp = su.logprobs64(row, 2, 1.0, 4)
    assert (rank, top) == (2, [1, 0, 2, -1]) and logp == pytest.approx(math.log(0.25)) and entropy == pytest.approx(1.5 * math.log(2))
    assert top_logp[0] == pytest.approx(math.log(0.5)) and top_logp[3] == -math.inf
    assert su.logprobs64(row, 3, 0.0, 1) == (-math.inf, 3, 0.0, [1], [0.0]) and su.logprobs64(row, 4, 1.0, 0)[:2] == (-math.inf, -1)


@pytest.mark.parametrize("D,heads,kv,seqs", [(64, 8, 8, 8), (64, 64, 8, 32), (128, 32, 8, 2), (128, 64, 8, 300), (256, 16, 2, 24), (128, 8, 1, 1)])
@pytest.mark.parametrize("max_len", [100, 768, 1000, 1536, 1537, 1 << 20])
def test_a_workspace_for_many_tokens_serves_fewer(D, heads, kv, seqs, max_len):
    def need(tokens, n=seqs, **over):
        return wsr.wsr_paged_workspace_bytes(_paged(_pages(page_size=64, max_pages=1 << 14), n_heads=heads, n_kv_heads=kv, head_dim=D,
                                                    n_seqs=n, n_tokens=tokens, max_len=max_len, **over))

    sizes = [need(t) for t in (*range(1, 70), *range(70, 3000, 37), 20000)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    sizes = [need(n, n, starts=None) for n in range(1, 500)]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("vocab", [1000, 4097, 32000, 128256, 1 << 24])
@pytest.mark.parametrize("n_top", [0, 1, 20, 64])
def test_a_workspace_for_many_rows_serves_fewer(vocab, n_top):
    sizes = [wsr.wsr_logprobs_workspace_bytes(_logprobs(vocab=vocab, n_rows=r, n_top=n_top)) for r in (*range(1, 800), 1000, 1536, 1537, 4000, 1 << 16)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    fewer = [wsr.wsr_logprobs_workspace_bytes(_logprobs(vocab=vocab, n_rows=33, n_top=n)) for n in range(65)]
    assert fewer == sorted(fewer)
