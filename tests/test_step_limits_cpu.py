"""What the step operators refuse for its size, on a machine without a GPU: counts that the kernels hold in 32 bits."""
import pytest

from paper_2608_12114_amd import wsr
from paper_2608_12114_amd import wsr_step as ws
from test_step_abi_cpu import A, SIZE, _attn, _lora

L = ws.step_lib()


@pytest.mark.parametrize("prefix,most,fits", [(1 << 30, 1 << 30, False), (1 << 30, (1 << 30) - 4095, False),
                                              (1 << 30, (1 << 30) - 4096, True), ((1 << 30) - 4096, 1 << 30, True)])
def test_attention_counts_a_rows_keys_in_32_bits(prefix, most, fits):
    p = _attn(prefix_len=prefix, max_len=most)
    assert (wsr.wsr_attn_workspace_bytes(p) > 0) == fits
    if not fits:
        assert L.wsr_prefix_attention(p, A, 1 << 40, None) == SIZE and "keys" in ws.wsr_step_last_error()


@pytest.mark.parametrize("seqs,heads,fits", [(1 << 20, 15, True), (1 << 20, 16, False), (1 << 18, 64, False), (1 << 16, 64, True)])
def test_attention_workgroups_of_one_launch(seqs, heads, fits):
    """A launch of 2^32 threads or more would be cut short without an error."""
    p = _attn(n_seqs=seqs, n_tokens=seqs, n_heads=heads, n_kv_heads=heads, starts=None, prefix_len=0)
    assert (wsr.wsr_attn_workspace_bytes(p) > 0) == fits
    if not fits:
        assert L.wsr_prefix_attention(p, A, 1 << 40, None) == SIZE and "launch" in ws.wsr_step_last_error()


def test_adapters_rows_of_a_call():
    mods = ws.make_loras([_lora(M=(1 << 31) - 1, y_tok_stride=1 << 34, y0_tok_stride=1 << 34)] * 33)
    assert L.wsr_lora_sweep(mods, 33, 4, A, 3, None, None, A, 1 << 40, None) == SIZE and "rows" in ws.wsr_step_last_error()
