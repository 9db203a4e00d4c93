"""wsr_paged_attention in each of its forms, on both sides of the choices between them: tiles of 16 to 128 rows, one launch and
two, units cut into few and many parts, sequences found in one and several steps."""
import pytest
import torch

import serve_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr
from test_gpu_serve_paged import BF16, F16, INF, NAN, Case

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("G,n", [(8, 1), (8, 3), (4, 8), (8, 7), (5, 13), (8, 40), (3, 101)])
@pytest.mark.parametrize("room", [0, 2000])
def test_tiles(D, G, n, room):
    """8 to 320 rows of a sequence, with and without room for a second launch; a tile's last rows empty."""
    c = Case([n, max(1, n // 2), n], [n + 700, n, n + 123], 2 * G, 2, D, F16, page=12, room=room, seed=n)
    c.run()
    c.check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,n", [(8, 1), (8, 3), (8, 8), (4, 40)])
def test_units_cut_into_parts(D, G, n):
    """A long sequence beside short ones: parts of different numbers, some of them joined, others stored at once."""
    c = Case([n] * 5, [n + 5000, n, n + 40, n + 1700, n + 2600], G, 1, D, BF16, page=33, seed=D)
    c.run()
    c.check()


@pytest.mark.parametrize("n,lens", [(1, 1500), (6, 900), (40, 1300), (64, 2500)])
@pytest.mark.parametrize("page", [1, 19, 64])
def test_holes_in_every_form(n, lens, page):
    row = -(-(lens + n) // page)
    holes = [((0, i), (-1, 1 << 30)[i % 2]) for i in range(row) if i * page % 256 < 100] + [((1, i), -7) for i in range(row)]
    c = Case([n, n, n], [lens + n, 200 + n, n], 8, 2, 128, F16, page=page, holes=holes)
    c.run()
    c.check()
    assert torch.isneginf(c.lse[n:2 * n]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [3, 8, 40])
@pytest.mark.parametrize("value", [INF, NAN])
def test_broken_values_in_every_form(n, D, value):
    """An infinity or NaN among the values of a place that only the later queries see."""
    lens = 1400 + n
    c = Case([n], [lens], 8, 1, D, F16, page=8)
    place = lens - n // 2
    c.v[int(c.table[0, place // 8]), place % 8, 0, 5] = value
    c.run()
    first = next(i for i in range(n) if place < lens - n + i + 1)
    hit = torch.zeros_like(c.out, dtype=torch.bool)
    hit[first:, :, 5] = True
    assert (torch.isnan(c.out[hit]) if value != value else c.out[hit] == value).all()
    c.v[int(c.table[0, place // 8]), place % 8, 0, 5] = 0.0
    out, _, bound, _ = su.paged64(c.q, c.k, c.v, c.table, 8, c.starts, c.lens, c.max_len, c.scale)
    assert ((c.out.double() - out).abs()[~hit] <= bound[~hit]).all()


@pytest.mark.parametrize("n", [8, 40])
def test_rows_without_keys_in_every_form(n):
    """More queries than keys, and lengths of zero, among tiles that others fill."""
    c = Case([n, n, 1, n], [n // 2, 0, 300, n + 900], 8, 1, 128, BF16, page=5, first=2, after=3)
    c.run()
    c.check()


@pytest.mark.parametrize("seqs", [64, 65, 300, 5000])
@pytest.mark.parametrize("room", [0, 3000])
def test_numbers_of_sequences(seqs, room):
    counts = [1 + (b % 7 == 0) - (b % 5 == 0) for b in range(seqs)]
    c = Case(counts, [n + (13 * b) % 37 for b, n in enumerate(counts)], 2, 1, 64, F16, page=8, room=room)
    c.run()
    c.check()


def test_starts_are_clamped():
    """What the device says past the rows of q is clamped to them."""
    c = Case([2, 3], [40, 9], 4, 2, 64, F16)
    c.dev_starts.copy_(torch.tensor([-5, 2, 1 << 30]))
    c.run()
    c.check()


def test_one_sequence_beside_many_key_heads():
    """Units enough for one launch without a cut where sequences are few."""
    c = Case([1, 1], [1400, 1000], 256, 256, 64, BF16)
    c.run()
    c.check()


@pytest.mark.parametrize("N,seqs,n,room", [(8, 32, 1, 0), (8, 32, 1, 2500), (7, 19, 1, 0), (8, 16, 1, 0), (8, 8, 17, 0), (4, 8, 24, 0)])
def test_as_many_parts_as_there_is_room_for(N, seqs, n, room):
    """Equal lengths, whose units come out in whole parts: all that the workspace holds, on both sides of few units."""
    c = Case([n] * seqs, [2048] * seqs, 8 * N, N, 64, F16, page=32, room=room)
    c.run()
    c.check()


MANY = 64, 8                                  # heads: enough tiles of 128 rows, from some 120 tokens on


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,lens", [(120, 130), (121, 900), (150, 2900)])
def test_tiles_of_most_rows(D, n, lens):
    """128 rows, in one part and in several; of unequal sequences, whose last tiles are part empty."""
    c = Case([n, n - 3, n + 1], [lens, n - 3, lens + 77], *MANY, D, (F16, BF16)[n % 2], page=20, seed=n)
    c.run()
    c.check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("page", [1, 19])
def test_holes_in_tiles_of_most_rows(D, page):
    n, lens = 121, 1000
    holes = [((0, i), (-1, 1 << 30)[i % 2]) for i in range(lens // page) if i * page % 256 < 100] + [((1, i), -7) for i in range(-(-(lens + 50) // page))]
    c = Case([n, n, n], [lens, lens + 50, n // 2], *MANY, D, F16, page=page, holes=holes)
    c.run()
    c.check()
    assert torch.isneginf(c.lse[n:2 * n]).all()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("value", [INF, NAN])
def test_broken_values_in_tiles_of_most_rows(D, value):
    n, lens = 170, 800
    c = Case([n, n], [lens, n], *MANY, D, F16, page=8)
    place = lens - n // 2
    at = int(c.table[0, place // 8]), place % 8, 3, 5
    c.v[at] = value
    c.run()
    hit = torch.zeros_like(c.out, dtype=torch.bool)
    hit[n - n // 2:n, 24:32, 5] = True
    assert (torch.isnan(c.out[hit]) if value != value else c.out[hit] == value).all()
    c.v[at] = 0.0
    out, _, bound, _ = su.paged64(c.q, c.k, c.v, c.table, 8, c.starts, c.lens, c.max_len, c.scale)
    assert ((c.out.double() - out).abs()[~hit] <= bound[~hit]).all()


@pytest.mark.parametrize("H,N,D,n", [(8, 2, 64, 1), (8, 8, 128, 1), (64, 8, 128, 3), (64, 2, 64, 40), (16, 2, 256, 12)])
@pytest.mark.parametrize("room", [0, 3000])
def test_anything_on_the_device_stays_inside(H, N, D, n, room):
    """Starts that fall, lengths and pages of any value: whatever comes out, nothing around the outputs is touched."""
    seqs = 300 if n == 1 else 70
    c = Case([n] * seqs, [n + 20] * seqs, H, N, D, F16, page=24, room=room)
    c.k.fill_(0.5), c.v.fill_(0.25)
    g = torch.Generator().manual_seed(H * D + n)
    any32 = lambda t, lo=-2 ** 31, hi=2 ** 31 - 1: t.copy_(torch.randint(lo, hi, t.shape, generator=g))  # noqa: E731
    T, edge = n * seqs, 50
    wide, wide_lse = c.out.new_full((T + 2 * edge, H, D), 77.0), c.lse.new_full((T + 2 * edge, H), 77.0)
    ws = torch.full((wsr.wsr_paged_workspace_bytes(wsr.make_paged(**c.fields)) + (2 << 20),), 255, dtype=torch.uint8, device="cuda")
    for starts in ((-5, T + 5), (0, T + 1), (-2 ** 31, 2 ** 31 - 1), (T, T + 1)):
        any32(c.dev_starts, *starts), any32(c.dev_lens), any32(c.table)
        c.table[:, ::2] = torch.randint(0, c.k.shape[0], c.table[:, ::2].shape, generator=g).to(c.table)
        p = wsr.make_paged(**{**c.fields, "out": wide[edge:], "lse": wide_lse[edge:]})
        wsr.wsr_paged_attention(p, ws[1 << 20:], ws.numel() - (2 << 20), stream())
        torch.cuda.synchronize()
        for t in (wide, wide_lse):
            assert (t[:edge] == 77.0).all() and (t[-edge:] == 77.0).all()
        assert (ws[:1 << 20] == 255).all() and (ws[-(1 << 20):] == 255).all()
