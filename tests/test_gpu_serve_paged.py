"""wsr_paged_attention against its formula in 64 bits: single tokens, drafts and chunks over ragged lengths, pages of any size,
holes, broken values in masked places, other layouts and offsets past 4 GiB."""
import pytest
import torch

import serve_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
FMT = {torch.float16: wsr.WSR_F16, torch.bfloat16: wsr.WSR_BF16}
F16, BF16, NAN, INF = torch.float16, torch.bfloat16, float("nan"), float("inf")


class Case:
    def __init__(self, counts, lens, H, N, D, dt, *, page=16, head_major=False, seed=0, first=0, after=0, room=0, scale=None, holes=()):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
        B, T = len(counts), first + sum(counts) + after
        self.lens, self.page, self.scale = list(lens), page, D ** -0.5 if scale is None else scale
        self.starts = [first + sum(counts[:i]) for i in range(B + 1)]
        self.q = (r(T, H, D).float() * 2).to(dt)
        row = max([1] + [-(-n // page) for n in lens]) + -(-room // page)
        pool = B * row + 3
        self.max_len = row * page
        self.table = torch.randperm(pool, generator=g, device="cuda")[:B * row].view(B, row).to(torch.int32)
        view = lambda t: t.transpose(1, 2) if head_major else t  # noqa: E731
        shape = (pool, N, page, D) if head_major else (pool, page, N, D)
        self.k, self.v = view(r(*shape)), view(r(*shape))
        used = torch.zeros(pool, page, dtype=torch.bool, device="cuda")
        for at, entry in holes:
            self.table[at] = entry
        for b, n in enumerate(self.lens):                        # what no sequence's keys are may hold anything
            places = torch.arange(min(max(n, 0), self.max_len), device="cuda")
            pages = self.table[b][places // page].long()
            ok = (pages >= 0) & (pages < pool)
            used[pages[ok], (places % page)[ok]] = True
        self.k[~used], self.v[~used] = NAN, NAN
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.dev_starts, self.dev_lens = ints(self.starts), ints(self.lens)
        self.out = torch.full((T, H, D), 77.0, dtype=dt, device="cuda")
        self.lse = torch.full((T, H), 77.0, device="cuda")
        self.fields = dict(fmt=FMT[dt], n_heads=H, n_kv_heads=N, head_dim=D, n_seqs=B, n_tokens=T, scale=self.scale, max_len=self.max_len,
                           q=self.q, q_tok_stride=2 * H * D, q_head_stride=2 * D, starts=self.dev_starts, lens=self.dev_lens, out=self.out,
                           out_tok_stride=2 * H * D, out_head_stride=2 * D, lse=self.lse, cache=self.pages())

    def pages(self):
        return wsr.make_pages(k=self.k, v=self.v, n_pages=self.k.shape[0], page_size=self.page, page_stride=2 * self.k.stride(0),
                              tok_stride=2 * self.k.stride(1), head_stride=2 * self.k.stride(2), table=self.table,
                              table_stride=4 * self.table.shape[1], max_pages=self.table.shape[1])

    def run(self, sync=True, on=None, **over):
        self.paged = wsr.make_paged(**{**self.fields, **over})
        self.ws = torch.full((wsr.wsr_paged_workspace_bytes(self.paged),), 255, dtype=torch.uint8, device="cuda")
        wsr.wsr_paged_attention(self.paged, self.ws, self.ws.numel(), on or stream())
        if sync:
            torch.cuda.synchronize()

    def check(self):
        out, lse, bound, lbound = su.paged64(self.q, self.k, self.v, self.table, self.page, self.starts, self.lens, self.max_len, self.scale)
        none = torch.isnan(lse) & (torch.arange(lse.shape[0], device="cuda")[:, None] < self.starts[0]) | (
            torch.arange(lse.shape[0], device="cuda")[:, None] >= self.starts[-1])
        assert (self.out[none] == 77.0).all() and (self.lse[none] == 77.0).all()       # rows of no sequence stay
        ok, got = ~none, self.out.double()
        err = (got - out).abs()[ok]
        assert (err <= bound[ok]).all(), float((err / bound[ok].clamp(min=1e-30)).max())
        empty = torch.isinf(lse) & ok
        assert torch.equal(torch.isinf(self.lse) & ok, empty) and (self.out[empty] == 0).all()
        err = (self.lse.double() - lse).abs()[ok & ~empty]
        assert (err <= lbound[ok & ~empty]).all(), float(err.max())


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,N", [(8, 2), (4, 4), (7, 1), (24, 1)])
@pytest.mark.parametrize("counts,lens,page", [
    ([1], [1], 16), ([1], [33], 5), ([1, 1, 1], [5, 64, 700], 16), ([1] * 9, range(1, 10), 1), ([3, 1, 5], [3, 170, 433], 7),
    ([2] * 17, [2 + 41 * i for i in range(17)], 64), ([40, 7], [40, 300], 33)])
def test_matches_formula(counts, lens, page, H, N, D, dt):
    c = Case(list(counts), lens, H, N, D, dt, page=page, seed=page + H, head_major=page == 33)
    c.run()
    c.check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("counts,lens,H,N", [
    ([1], [9001], 8, 2), ([1, 1], [3000, 5], 64, 8), ([300], [300], 8, 2), ([129, 1, 64], [2000, 90, 64], 12, 4), ([1] * 130, None, 4, 2),
    ([5] * 70, None, 16, 2)])
def test_long_and_many(counts, lens, H, N, D):
    """Lengths over many shares, tiles of chunks, and more than 64 sequences."""
    lens = lens or [n + (37 * i) % 300 for i, n in enumerate(counts)]
    c = Case(counts, lens, H, N, D, BF16, page=24, room=100)
    c.run()
    c.check()


def test_rows_that_see_nothing_and_rows_of_no_sequence():
    c = Case([1, 2, 0, 4, 1], [0, 1, 30, 2, -3], 8, 2, 128, F16, page=4, first=3, after=2)
    c.run()
    c.check()
    c = Case([3, 3], [0, 0], 4, 4, 64, BF16)
    c.run()
    assert (c.out == 0).all() and torch.isneginf(c.lse).all()
    c.run(cache=wsr.make_pages(table=c.table, table_stride=4 * c.table.shape[1], page_size=16, max_pages=c.table.shape[1]))
    assert (c.out == 0).all() and torch.isneginf(c.lse).all()


@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_holes(page):
    """Keys in pages outside the pool take part in nothing; a sequence of nothing but holes sees nothing."""
    lens = [500, 200, 90]
    row = -(-500 // page)
    holes = [((0, i), (-1, 10 ** 6, -(1 << 31), (1 << 31) - 1)[i % 4]) for i in range(row) if i * page % 128 >= 64 or i < 2]
    holes += [((1, i), -1) for i in range(row)] + [((2, 0), -5)]
    c = Case([1, 3, 2], lens, 8, 2, 128, F16, page=page, holes=holes)
    c.run()
    c.check()
    assert torch.isneginf(c.lse[1:4]).all()


def test_lengths_past_the_room():
    """Lengths are clamped to max_len, whatever the device says."""
    c = Case([1, 2], [64, 64], 4, 2, 64, BF16, page=16)
    c.dev_lens.copy_(torch.tensor([(1 << 31) - 1, 65]))
    c.run()
    c.check()
    c.max_len = 37
    c.run(max_len=37)
    c.lens = [64, 64]
    c.check()


@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("counts,lens", [([4], [70]), ([1], [70]), ([33], [600])])
def test_broken_values_reach_those_that_see_them(value, counts, lens):
    c = Case(counts, lens, 4, 2, 64, F16, page=8)
    n, own = counts[0], lens[0]
    place = own - max(1, n // 2)                                 # seen by the later half of the queries
    page, slot = int(c.table[0, place // 8]), place % 8
    c.v[page, slot, 1, 5] = value
    c.run()
    hit = torch.zeros_like(c.out, dtype=torch.bool)
    hit[max(n - n // 2 - 1 + (n == 1), 0) if n > 1 else 0:, 2:, 5] = True
    first = next(i for i in range(n) if place < own - n + i + 1)
    hit[:] = False
    hit[first:, 2:, 5] = True
    assert torch.equal(c.out[hit], torch.full_like(c.out[hit], value)) if value == value else torch.isnan(c.out[hit]).all()
    c.v[page, slot, 1, 5] = 0.0
    out, _, bound, _ = su.paged64(c.q, c.k, c.v, c.table, 8, c.starts, c.lens, c.max_len, c.scale)
    assert ((c.out.double() - out).abs()[~hit] <= bound[~hit]).all()


def test_broken_keys_and_queries():
    c = Case([2, 1], [50, 40], 4, 2, 64, BF16, page=8)
    c.k[int(c.table[0, 1]), 3, 0, 7] = NAN                       # a key that both of the first sequence's queries see
    c.q[2, 3] = INF
    c.run()
    assert torch.isnan(c.out[:2, :2]).all() and torch.isnan(c.lse[:2, :2]).all()
    assert torch.isnan(c.out[2, 3]).all() and torch.isnan(c.lse[2, 3])
    assert torch.isfinite(c.out[:2, 2:]).all() and torch.isfinite(c.out[2, :3]).all()


def test_large_scores():
    """Scores of thousands: the softmax is taken against the largest."""
    c = Case([1, 3], [300, 200], 4, 2, 128, F16, scale=30.0)
    c.run()
    c.check()


def test_shared_pages_and_strides():
    """Two sequences on the same pages, queries and outputs with gaps, no lse, no starts."""
    c = Case([1, 1, 1], [100, 90, 33], 4, 2, 128, F16, page=16)
    c.table[1] = c.table[0]
    wide = torch.full((3, 6, 160), 5.0, dtype=F16, device="cuda")
    q = torch.randn(3, 9, 136, device="cuda").to(F16)
    c.q = q[:, :4, :128]
    c.run(out=wide, out_tok_stride=2 * 960, out_head_stride=320, lse=None, starts=None, q=q, q_tok_stride=2 * 9 * 136, q_head_stride=2 * 136)
    out, _, bound, _ = su.paged64(c.q, c.k, c.v, c.table, 16, c.starts, c.lens, c.max_len, c.scale)
    assert ((wide[:, :4, :128].double() - out).abs() <= bound).all()
    wide[:, :4, :128] = 5.0
    assert (wide == 5.0).all()


def test_offsets_past_4_gib():
    """Pages on both sides of 4 GiB of the pool, read as their copies near its start."""
    c = Case([1], [40], 4, 2, 64, F16, page=16)
    step = 16 * 2 * 64
    pool = torch.zeros(2, 5 * (1 << 29) // step, 16, 2, 64, dtype=F16, device="cuda")
    last = pool.shape[1] - 1
    c.run()
    want = c.out.clone()
    for i, page in enumerate((last, 3, last - 1)):
        pool[0, page], pool[1, page] = c.k[int(c.table[0, i])], c.v[int(c.table[0, i])]
        c.table[0, i] = page
    c.k, c.v = pool[0], pool[1]
    c.out.zero_()
    c.run(cache=c.pages())
    assert torch.equal(c.out, want)


def test_same_bits_every_time():
    c = Case([1, 4, 30], [3000, 900, 700], 16, 2, 128, BF16)
    c.run()
    first = c.out.clone(), c.lse.clone()
    for _ in range(3):
        c.run()
        assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])
