"""wsr_append_qkv against its formula in 64 bits: norms, both kinds of pairs, several axes, far positions, odd pages, holes,
tokens of no sequence, and everything that is not written left as it was."""
import pytest
import torch

import serve_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
FMT = {torch.float16: wsr.WSR_F16, torch.bfloat16: wsr.WSR_BF16}
F16, BF16 = torch.float16, torch.bfloat16


class Case:
    def __init__(self, counts, lens, H, N, D, dt, *, rot=None, pairs=False, kind=None, bias=False, weights=True, axes=1, page=16,
                 head_major=False, seed=0, first=0, after=0, holes=(), positions=None, spread=1.0, pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s, to=torch.float32: torch.randn(s, generator=g, device="cuda").to(to)  # noqa: E731
        self.H, self.N, self.D, self.dt, self.page, self.pairs, self.kind = H, N, D, dt, page, pairs, kind
        self.rot = D if rot is None else rot
        B, T = len(counts), first + sum(counts) + after
        self.T, self.lens = T, list(lens)
        self.starts = [first + sum(counts[:i]) for i in range(B + 1)]
        wide = lambda h: (r(T, h * D + pad) * spread)[:, :h * D]  # noqa: E731
        self.q, self.k, self.v = wide(H), wide(N), wide(N)
        w = lambda: (1 + 0.2 * r(D)).to(dt) if kind and weights else None  # noqa: E731
        b = lambda: (0.1 * r(D)).to(dt) if kind and bias else None  # noqa: E731
        self.w = dict(q_w=w(), q_b=b(), k_w=w(), k_b=b())
        half = self.rot // 2
        self.freqs = (1e4 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / max(half, 1))).float()
        self.axis_of = None
        if axes > 1:
            self.axis_of = torch.randint(-1, axes + 1, (half,), generator=g, device="cuda").to(torch.int32)
        self.positions = positions
        if positions is None and axes > 1:
            self.positions = torch.randint(-5, 4000, (axes, T), generator=g, device="cuda").to(torch.int32)
        row = max([1] + [-(-max(n, 1) // page) for n in lens])
        pool = B * row + 3
        self.table = torch.randperm(pool, generator=g, device="cuda")[:B * row].view(B, row).to(torch.int32)
        for at, page_index in holes:
            self.table[at] = page_index
        shape = (pool, N, page, D) if head_major else (pool, page, N, D)
        view = lambda t: t.transpose(1, 2) if head_major else t  # noqa: E731
        self.kc, self.vc = view(r(*shape, to=dt)), view(r(*shape, to=dt))
        self.out = r(T, H, D, to=dt)
        self.before = [t.clone() for t in (self.out, self.kc, self.vc)]
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.dev_starts, self.dev_lens = ints(self.starts), ints(self.lens)
        self.pages = wsr.make_pages(k=self.kc, v=self.vc, n_pages=pool, page_size=page, page_stride=2 * self.kc.stride(0),
                                    tok_stride=2 * self.kc.stride(1), head_stride=2 * self.kc.stride(2), table=self.table,
                                    table_stride=4 * row, max_pages=row)
        self.fields = dict(
            fmt=FMT[dt], flags=(wsr.WSR_QKV_NORM if kind else 0) | (wsr.WSR_QKV_PAIRS if pairs else 0),
            kind=wsr.WSR_NORM_LAYER if kind == "layer" else wsr.WSR_NORM_RMS, n_heads=H, n_kv_heads=N, head_dim=D, rot_dim=self.rot,
            n_axes=axes, n_seqs=B, n_tokens=T, q=self.q, q_tok_stride=4 * self.q.stride(0), k=self.k, k_tok_stride=4 * self.k.stride(0),
            v=self.v, v_tok_stride=4 * self.v.stride(0), freqs=self.freqs, axis_of=self.axis_of, positions=self.positions,
            pos_axis_stride=4 * T, starts=self.dev_starts, lens=self.dev_lens, q_out=self.out, q_out_tok_stride=2 * H * D,
            q_out_head_stride=2 * D, cache=self.pages, **self.w)

    def run(self, sync=True, on=None, **over):
        wsr.wsr_append_qkv(wsr.make_qkv(**{**self.fields, **over}), on or stream())
        if sync:
            torch.cuda.synchronize()

    def want(self):
        T, N, D = self.T, self.N, self.D
        where = su.places64(self.starts, self.lens, T)
        at = torch.tensor([[p for _, p in where]], device="cuda") if self.positions is None else self.positions
        turn = lambda x, w, b: su.turned64(  # noqa: E731
            x.reshape(T, -1, D), at, self.freqs, self.axis_of, rot=self.rot, pairs=self.pairs, kind=self.kind, w=self.w[w], b=self.w[b])
        q, k = turn(self.q, "q_w", "q_b"), turn(self.k, "k_w", "k_b")
        v = (self.v.reshape(T, N, D).double(), torch.zeros(T, N, D, dtype=torch.float64, device="cuda"))
        full = [[t.double(), torch.zeros(t.shape, dtype=torch.float64, device="cuda"), torch.zeros(t.shape, dtype=torch.bool, device="cuda")]
                for t in self.before]
        table = self.table.cpu()
        for t, (b, place) in enumerate(where):
            if b < 0:
                continue
            for f, (x, e) in zip(full[:1], (q,)):
                f[0][t], f[1][t], f[2][t] = x[t], e[t], True
            slot = su.slot64(table, self.page, self.kc.shape[0], b, place)
            if slot:
                for f, (x, e) in zip(full[1:], (k, v)):
                    f[0][slot], f[1][slot], f[2][slot] = x[t], e[t], True
        return full

    def check(self):
        for got, old, (want, err, written) in zip((self.out, self.kc, self.vc), self.before, self.want()):
            assert torch.equal(got[~written].view(torch.int16), old[~written].view(torch.int16))      # bit for bit
            # one rounding to 16 bits (half a step of the result, or of the smallest numbers) beside fp32's own
            bound = err * (1 + su.U16[self.dt]) + su.U16[self.dt] * want.abs() + su.TINY[self.dt]
            off = (got.double() - want).abs()[written]
            assert (off <= bound[written]).all(), float((off / bound[written].clamp(min=1e-30)).max())


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("D,H,N", [(64, 8, 2), (128, 4, 4), (256, 2, 1), (128, 7, 1), (64, 3, 5)])
@pytest.mark.parametrize("kind,bias", [(None, False), ("rms", False), ("layer", True)])
@pytest.mark.parametrize("pairs", [False, True])
def test_matches_formula(D, H, N, kind, bias, pairs, dt):
    c = Case([1, 5, 1, 18], [1, 9, 40, 18], H, N, D, dt, kind=kind, bias=bias, pairs=pairs, page=7, seed=D + H)
    c.run()
    c.check()


@pytest.mark.parametrize("rot", [0, 8, 24, 64, 120, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("page,head_major", [(1, False), (16, True), (100, False)])
def test_parts_of_a_head_and_layouts(rot, pairs, page, head_major):
    c = Case([3, 2], [3, 130], 5, 2, 128, BF16, rot=rot, pairs=pairs, kind="rms", page=page, head_major=head_major, pad=12)
    c.run()
    c.check()


@pytest.mark.parametrize("axes", [2, 3, 4])
@pytest.mark.parametrize("pairs", [False, True])
def test_several_axes(axes, pairs):
    """Axis numbers outside the axes are clamped to them; positions may be negative."""
    c = Case([4, 30], [4, 200], 4, 2, 64, F16, axes=axes, pairs=pairs, seed=axes)
    c.run()
    c.check()


@pytest.mark.parametrize("far", [0, 1 << 20, (1 << 24) + 1, (1 << 31) - 70])
def test_far_positions(far):
    """An angle of 2^31 keeps its place in the turn: fp32 would have lost whole turns from 2^26 on."""
    at = torch.arange(64, dtype=torch.int64, device="cuda").add(far).to(torch.int32)[None]
    c = Case([64], [64], 2, 1, 128, F16, positions=at, spread=4.0)
    c.run()
    # 64-bit arithmetic itself leaves 2^-52 of 2^31 turns, 2^-21: 8 half steps of 1 in 32 bits
    full = c.want()
    for got, (want, err, _) in zip((c.out, c.kc), full):
        bound = err * 2 + su.U16[F16] * want.abs() + su.TINY[F16] + (2.0 ** -20 * 32 if far > 1 << 30 else 0.0)
        assert ((got.double() - want).abs() <= bound).all()


def test_places_that_are_not_there():
    """Holes, places past the table and below 0, tokens before the first and behind the last sequence: nothing is stored, and
    queries of tokens that belong to a sequence are."""
    c = Case([2, 6, 0, 3, 1], [1, 40, 9, 33, -4], 4, 2, 64, BF16, kind="rms", page=4, first=3, after=5,
             holes=[((1, 9), -1), ((1, 8), 10 ** 6), ((3, 7), -(1 << 31))])
    c.run()
    c.check()
    c = Case([5], [8], 4, 2, 64, F16, page=2)
    c.dev_lens.fill_(11)                                         # behind the table's last entry
    c.lens = [11]
    c.run()
    c.check()
    c.dev_lens.fill_((1 << 31) - 1)
    c.run()
    c.lens = [(1 << 31) - 1]
    c.out.copy_(c.before[0])
    c.before = [t.clone() for t in (c.out, c.kc, c.vc)]
    c.run()
    assert torch.equal(c.kc.view(torch.int16), c.before[1].view(torch.int16)) and torch.isfinite(c.out).all()


def test_only_queries_and_only_keys():
    c = Case([3, 4], [30, 4], 4, 2, 128, F16, kind="layer", bias=True)
    c.run(k=None, v=None, cache=wsr.make_pages())
    c.before[1:] = [c.kc.clone(), c.vc.clone()]
    assert torch.equal(c.kc, c.before[1]) and not torch.equal(c.out, c.before[0])
    queries, c.before[0] = c.out.clone(), c.out.clone()
    c.out.fill_(7.0)
    c.run(q=None, q_out=None, n_heads=0)
    assert (c.out == 7.0).all() and not torch.equal(c.kc, c.before[1])
    c.out.copy_(queries)
    c.check()


def test_no_starts_one_token_each():
    c = Case([1] * 9, range(1, 10), 8, 2, 128, BF16, kind="rms", page=3)
    c.run(starts=None)
    c.check()


def test_broken_values_stay_in_their_head():
    c = Case([4], [20], 4, 2, 64, F16, kind="rms")
    c.q[1, 64 + 3], c.k[2, 5], c.v[3, 64 + 9] = float("inf"), float("nan"), -float("inf")
    c.run()
    want = c.want()
    bad = torch.zeros_like(c.out, dtype=torch.bool)
    bad[1, 1] = True
    ok = (c.out.double() - want[0][0]).abs() <= want[0][1] * 2 + su.U16[F16] * want[0][0].abs() + su.TINY[F16]
    assert ok[~bad].all() and not torch.isfinite(c.out[1, 1]).all()
    where = [su.slot64(c.table.cpu(), 16, c.kc.shape[0], 0, 16 + t) for t in range(4)]
    assert torch.isnan(c.kc[where[2]][0]).all() and torch.isfinite(c.kc[where[2]][1]).all()
    assert c.vc[where[3]][1, 9] == -float("inf") and torch.isfinite(c.vc[where[3]]).sum() == 127


def test_many_sequences():
    """Enough sequences for two levels of the search for a token's."""
    counts = [(7 * i) % 3 for i in range(5000)]
    c = Case(counts, [n + i % 5 for i, n in enumerate(counts)], 1, 1, 64, F16, page=4, first=2, after=3)
    c.run()
    c.check()


def test_offsets_past_4_gib():
    """Pages on both sides of 4 GiB of the pool."""
    c = Case([3], [3], 2, 1, 64, F16, page=2)
    pool = torch.zeros(2, (5 << 30) // 2, dtype=F16, device="cuda")
    step = 2 * 64 * 2
    last = pool.shape[1] * 2 // step - 1
    c.table[0, 0], c.table[0, 1] = last, 0
    c.run(cache=wsr.make_pages(k=pool[0], v=pool[1], n_pages=last + 1, page_size=2, page_stride=step, tok_stride=128, head_stride=128,
                               table=c.table, table_stride=8, max_pages=2))
    got = pool.view(2, last + 1, 2, 64)[:, [last, last, 0], [0, 1, 0]]
    c.table[0, 0], c.table[0, 1] = 0, 1
    c.run()
    same = torch.stack([c.kc[[0, 0, 1], [0, 1, 0], 0], c.vc[[0, 0, 1], [0, 1, 0], 0]])
    assert torch.equal(got, same) and torch.count_nonzero(pool) <= 6 * 64
