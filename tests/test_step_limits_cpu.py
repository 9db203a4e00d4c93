"""What the step operators refuse for its size, on a machine without a GPU: counts that the kernels hold in 32 bits."""
import pytest

from paper_2608_12114_amd import wsr
from paper_2608_12114_amd import wsr_step as ws
from test_step_abi_cpu import A, SIZE, _attn

L = ws.step_lib()


@pytest.mark.parametrize("prefix,most,fits", [(1 << 30, 1 << 30, False), (1 << 30, (1 << 30) - 4095, False),
                                              (1 << 30, (1 << 30) - 4096, True), ((1 << 30) - 4096, 1 << 30, True)])
def test_attention_counts_a_rows_keys_in_32_bits(prefix, most, fits):
    p = _attn(prefix_len=prefix, max_len=most)
    assert (wsr.wsr_attn_workspace_bytes(p) > 0) == fits
    if not fits:
        assert L.wsr_prefix_attention(p, A, 1 << 40, None) == SIZE and "keys" in ws.wsr_step_last_error()
