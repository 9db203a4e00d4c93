"""Projections without rows (M = 0) in wsr_lora_sweep, on a machine without a GPU: their pointers may be null, so they
take part in no launch and no workspace."""
import pytest

from paper_2608_12114_amd import wsr
from paper_2608_12114_amd import wsr_step as ws

L = ws.step_lib()
A = 0x10000          # an aligned fake address, never dereferenced
FULL = dict(fmt=2, rank=16, M=64, K=4096, a=A, a_stride=16 * 8192, b=A, b_stride=2048, x=A, x_tok_stride=8192, y0=A, y0_tok_stride=256,
            y=A, y_tok_stride=256)
EMPTY = dict(fmt=2, rank=64, M=0, K=1 << 20)


def _bytes(specs, tokens):
    return wsr.wsr_lora_workspace_bytes(ws.make_loras(specs), tokens)


@pytest.mark.parametrize("tokens", [1, 4, 40, 300])
@pytest.mark.parametrize("at", [0, 1, 2])
@pytest.mark.parametrize("fmt", [1, 2])
def test_no_workspace(tokens, at, fmt):
    full = [FULL, {**FULL, "K": 8}]
    assert _bytes(full[:at] + [{**EMPTY, "fmt": fmt}] + full[at:], tokens) == _bytes(full, tokens)


def test_many_runs_of_projections():
    """More projections than a table holds, every other one empty: as many runs as the others alone make."""
    full = [{**FULL, "fmt": 1 + i // 100 % 2} for i in range(500)]
    mixed = [s for f in full for s in (EMPTY, f)] + [EMPTY]
    assert _bytes(mixed, 9) == _bytes(full, 9)


@pytest.mark.parametrize("tokens", [1, 4, 40, 300])
def test_nothing_is_launched(tokens):
    """A sweep of empty projections has nothing to do: it succeeds where no launch could."""
    mods = ws.make_loras([EMPTY] * 300)
    need = wsr.wsr_lora_workspace_bytes(mods, tokens)
    assert L.wsr_lora_sweep(mods, 300, tokens, A, 3, None, None, A, need, None) == wsr.WSR_OK, ws.wsr_step_last_error()
