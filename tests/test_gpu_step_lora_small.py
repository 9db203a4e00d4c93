"""wsr_lora_sweep on both sides of its choice of one launch or two for up to three tokens."""
import pytest
import torch

from gpu_util import needs_gpu
from test_gpu_step_lora import Case

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,rank,K", [(1, 16, 14336), (1, 16, 14344), (1, 64, 3584), (1, 64, 3592), (1, 65, 256), (2, 16, 4096), (2, 16, 4104),
                                      (2, 33, 1984), (3, 8, 4096), (3, 8, 4104), (3, 64, 512), (4, 1, 64)])
def test_bytes_of_a(T, rank, K, dt):
    """448 KiB of A for one token, 256 for two, 192 for three; 64 ranks; three tokens."""
    for ranks in (None, [rank, max(1, rank // 2), 1]):
        c = Case([(300, K), (257, min(K, 136))], T, 3, rank, dt, seed=K, ranks=ranks)
        c.run()
        c.check()


@pytest.mark.parametrize("M", [512 * 256, 512 * 256 + 1])
def test_rows(M):
    """512 workgroups of 256 rows, and one more."""
    c = Case([(M, 64)], 2, 2, 8, torch.bfloat16, seed=60, y0="in place")
    c.ids[0] = -1
    c.run()
    c.check()


@pytest.mark.parametrize("n", [8, 9])
def test_projections(n):
    c = Case([(40 + i, 72 + 8 * i) for i in range(n)], 3, 2, 12, torch.float16, seed=61)
    c.run()
    c.check()


@pytest.mark.parametrize("T,n,rank", [(1, 1, 64), (2, 2, 1), (3, 2, 9), (3, 3, 1)])
def test_one_launch_and_two_agree(T, n, rank):
    """A projection alone, in one launch, and beside one of long rows, in two: skipped and used tokens in turn."""
    for shapes in ([(300, 512)], [(300, 512), (16, 1 << 18)]):
        c = Case(shapes, T, n, rank, torch.bfloat16, seed=30)
        c.ids[1::2] = -1
        c.run()
        c.check()
