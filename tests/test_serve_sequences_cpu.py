"""Workspaces of paged attention for many sequences, on a machine without a GPU."""
import pytest

from paper_2608_12114_amd import wsr
from test_serve_abi_cpu import _paged, _pages


@pytest.mark.parametrize("D,heads,kv", [(64, 4, 1), (64, 64, 8), (128, 32, 8), (128, 8, 1), (256, 16, 2)])
@pytest.mark.parametrize("max_len", [100, 768, 1000, 1536, 1537, 1 << 20])
def test_a_workspace_for_many_sequences_serves_fewer(D, heads, kv, max_len):
    def need(tokens, n, **over):
        return wsr.wsr_paged_workspace_bytes(_paged(_pages(page_size=64, max_pages=1 << 14), n_heads=heads, n_kv_heads=kv, head_dim=D,
                                                    n_seqs=n, n_tokens=tokens, max_len=max_len, **over))

    sizes = [need(n, n, starts=None) for n in (*range(1, 700), 5000, 1 << 17)]
    assert sizes == sorted(sizes)
    for n in (192, 193, 512, 513, 5000):
        sizes = [need(t, n) for t in (*range(1, 700, 7), *range(700, 20000, 97))]
        assert sizes == sorted(sizes)
        # up to 512 sequences each workgroup may read all of them; more leave two sums each
        assert n <= 512 or sizes[0] >= 8 * n
