"""wsr_lora_sweep against its formula in 64 bits: ranks 1 to 256, odd rows, one token to hundreds in any order of
adapters, tokens without one, unread parts full of NaN, in place and strided, and under a captured graph."""
import math

import pytest
import torch

import step_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
FMT = {torch.float16: wsr.WSR_F16, torch.bfloat16: wsr.WSR_BF16}


class Case:
    def __init__(self, shapes, T, n, rank, dt, seed=0, ranks=None, scales=True, y0="apart", b_pad=0, pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.T, self.n, self.dt, self.rank = T, n, dt, rank
        self.ids = torch.randint(0, max(1, n), (T,), generator=g, device="cuda").to(torch.int32)
        self.ranks = None if ranks is None else torch.tensor(ranks, dtype=torch.int32, device="cuda")
        self.scales = 0.5 + torch.rand(max(1, n), generator=g, device="cuda") if scales else None
        self.mods = []
        for M, K in shapes:
            m = {"M": M, "K": K, "x": r(T, K + pad).to(dt)[:, :K], "a": (r(n, rank, K) * max(K, 1) ** -0.5).to(dt),
                 "b_store": (r(n * M * rank + b_pad) * 0.05).to(dt)}
            m["b"] = m["b_store"][b_pad:].view(n, M, rank)
            m["y0"] = None if y0 == "none" else r(T, M + pad)[:, :M]
            m["y"] = m["y0"].clone() if y0 == "in place" else torch.full((T, M + pad), float("nan"), device="cuda")[:, :M]
            if y0 == "in place":
                m["y0"], m["src"] = m["y"], m["y0"]
            else:
                m["src"] = m["y0"]
            self.mods.append(m)
        self.table = wsr.make_loras(
            dict(fmt=FMT[dt], rank=rank, M=m["M"], K=m["K"], a=m["a"], a_stride=2 * rank * m["K"], b=m["b"],
                 b_stride=2 * m["M"] * rank, x=m["x"], x_tok_stride=2 * m["x"].stride(0) if m["K"] else 0, y0=m["y0"],
                 y0_tok_stride=0 if m["y0"] is None else 4 * m["y0"].stride(0), y=m["y"], y_tok_stride=4 * m["y"].stride(0))
            for m in self.mods)
        self.ws = torch.full((wsr.wsr_lora_workspace_bytes(self.table, T),), 255, dtype=torch.uint8, device="cuda")

    def run(self, sync=True):
        wsr.wsr_lora_sweep(self.table, self.T, self.ids, self.n, self.ranks, self.scales, self.ws, self.ws.numel(), stream())
        if sync:
            torch.cuda.synchronize()

    def check(self):
        for m in self.mods:
            y, mag = su.lora64(m["x"], m["a"], m["b"], self.ids.tolist(), None if self.ranks is None else self.ranks.tolist(),
                               None if self.scales is None else self.scales.tolist(), m["src"])
            # fp32 sums of K and of rank terms: roundings add up like a walk, measured against the magnitudes
            bound = su.U32 * (8 + 2 * math.sqrt(m["K"]) + 2 * math.sqrt(self.rank)) * mag + 1e-30
            err = (m["y"].double() - y).abs()
            assert (err <= bound).all(), (m["M"], m["K"], float((err / bound).max()))


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,n,rank", [(1, 1, 16), (1, 3, 1), (2, 1, 3), (5, 5, 4), (16, 2, 8), (17, 1, 16), (31, 3, 24),
                                      (64, 1, 16), (64, 64, 5), (65, 1, 16), (65, 4, 64), (130, 33, 12), (300, 2, 128), (70, 3, 256)])
def test_matches_formula(T, n, rank, dt):
    c = Case([(96, 64), (131, 200), (1024, 1160)], T, n, rank, dt, seed=T + rank)
    c.run()
    c.check()


@pytest.mark.parametrize("T", [3, 40, 150])
def test_tokens_without_an_adapter(T):
    """Numbers outside [0, n_adapters) take no adapter: y = y0, and nothing is read for them."""
    c = Case([(260, 72)], T, 2, 8, torch.bfloat16, seed=1)
    c.ids[::3] = -1
    c.ids[1::7] = 2
    c.ids[2] = 2 ** 31 - 1
    c.run()
    c.check()


@pytest.mark.parametrize("y0", ["none", "in place", "apart"])
@pytest.mark.parametrize("T", [9, 100])
def test_base_outputs(y0, T):
    c = Case([(77, 136), (512, 512)], T, 3, 16, torch.float16, seed=2, y0=y0, pad=8)
    c.ids[0] = -5
    c.run()
    c.check()


@pytest.mark.parametrize("T", [6, 90])
@pytest.mark.parametrize("rank", [16, 18])
def test_unread_ranks_may_hold_anything(T, rank):
    c = Case([(130, 264)], T, 4, rank, torch.bfloat16, seed=3, ranks=[rank + 5, 7, 0, -3])
    m = c.mods[0]
    m["a"][1, 7:], m["b"][1, :, 7:] = float("nan"), float("inf")
    m["a"][2:], m["b"][2:] = float("nan"), float("nan")
    c.ids[:4] = torch.arange(4, dtype=torch.int32)
    c.run()
    c.check()


def test_odd_places_of_b():
    """B at 2-byte alignment, ranks that are no multiple of four."""
    for rank, pad in ((16, 1), (8, 3), (7, 1), (6, 2)):
        c = Case([(65, 64)], 20, 2, rank, torch.float16, seed=4, b_pad=pad)
        c.run()
        c.check()


def test_many_projections_no_scales_and_empty_ones():
    c = Case([(40, 32), (0, 64), (24, 0), (8, 8)] + [(48, 40)] * 240, 4, 2, 4, torch.float16, seed=5, scales=False)
    c.run()
    c.check()


def test_no_adapters_at_all():
    c = Case([(40, 32)], 70, 1, 4, torch.float16, seed=6)
    c.n = 0
    c.run()
    assert torch.equal(c.mods[0]["y"], c.mods[0]["src"])


def test_adapters_beyond_32_bits():
    """The last adapter of the pool lies past 4 GiB."""
    T, M, K, rank, dt = 3, 64, 64, 8, torch.bfloat16
    c = Case([(M, K)], T, 2, rank, dt, seed=7)
    m = c.mods[0]
    far = (1 << 32) + 4096
    store = torch.zeros(far + 65536, dtype=torch.uint8, device="cuda")
    a1 = store[far:far + 2 * rank * K].view(dt).view(rank, K)
    store[:2 * rank * K].view(dt).view(rank, K).copy_(m["a"][0])
    a1.copy_(m["a"][1])
    c.table[0].a, c.table[0].a_stride = store.data_ptr(), far
    c.run()
    c.check()


def test_graph_replay_with_other_adapters():
    for T in (12, 80):
        c = Case([(136, 256), (300, 64)], T, 5, 16, torch.bfloat16, seed=8)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c.run(sync=False)
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run(sync=False)
        for k in range(4):
            c.ids.copy_(torch.randint(-1, 5, (T,), device="cuda"))
            for m in c.mods:
                m["y"].fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            c.check()
            first = [m["y"].clone() for m in c.mods]
            c.run()
            assert all(torch.equal(f, m["y"]) for f, m in zip(first, c.mods))


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,n,rank", [(8, 4, 16), (40, 5, 8), (150, 30, 12), (20, 3, 96)])
def test_broken_adapter_reaches_its_own_tokens_only(T, n, rank, dt):
    """Infinities and NaN in one adapter's weights, and in one token's activations, leave the others' results alone."""
    c = Case([(130, 128), (64, 72)], T, n, rank, dt, seed=10)
    c.ids[:n] = torch.arange(n, dtype=torch.int32)
    c.ids[n + 1] = -1
    for m in c.mods:
        m["b"][1, ::3, 0], m["b"][1, 1::3, rank - 1], m["a"][2, 1, 5] = float("nan"), float("inf"), float("inf")
        m["x"][0, 3] = float("nan")
    c.run()
    whole = torch.ones(T, dtype=torch.bool, device="cuda")
    whole[0] = False
    whole &= (c.ids != 1) & (c.ids != 2)
    assert whole.sum() > 0
    for m in c.mods:
        y, mag = su.lora64(m["x"], m["a"], m["b"], c.ids.tolist(), None, c.scales.tolist(), m["src"])
        bound = su.U32 * (8 + 2 * math.sqrt(m["K"]) + 2 * math.sqrt(rank)) * mag
        assert ((m["y"].double() - y).abs() <= bound)[whole].all()
        assert torch.isfinite(m["y"][whole]).all() and not torch.isfinite(m["y"][0]).any()
        assert not torch.isfinite(m["y"][c.ids == 1][:, ::3]).any() and not torch.isfinite(m["y"][c.ids == 2]).any()


def test_steady_bits():
    """The order of tokens inside an adapter's tiles is free; the results are not."""
    c = Case([(136, 264)], 500, 3, 16, torch.bfloat16, seed=11)
    c.run()
    want = c.mods[0]["y"].clone()
    for _ in range(3):
        c.mods[0]["y"].fill_(float("nan"))
        c.run()
        assert torch.equal(c.mods[0]["y"], want)


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e6])
def test_inner_vectors_of_any_size(size):
    """f16 activations and weights give inner vectors far from 1: their terms are scaled, not cut."""
    c = Case([(96, 64)], 5, 2, 16, torch.float16, seed=12, y0="none")
    c.mods[0]["a"].mul_(min(size, 1.0) ** 0.25 if size < 1 else 30.0)
    c.mods[0]["x"].mul_(min(size, 1.0) ** 0.15 if size < 1 else 300.0)
    c.run()
    c.check()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,n,rank", [(500, 5, 24), (333, 20, 12), (200, 9, 64)])
def test_bits_do_not_depend_on_a_tokens_place(T, n, rank, dt):
    """The same tokens in another order, so in other tiles beside other adapters, get the same bits."""
    c = Case([(136, 264)], T, n, rank, dt, seed=13)
    m = c.mods[0]
    m["b"][1, ::40, 0] = float("inf")
    c.run()
    want, x, y0, ids = m["y"].clone(), m["x"].clone(), m["y0"].clone(), c.ids.clone()
    for seed in range(3):
        to = torch.randperm(T, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        m["x"].copy_(x[to]), m["y0"].copy_(y0[to]), c.ids.copy_(ids[to])
        m["y"].fill_(float("nan"))
        c.run()
        assert torch.equal(m["y"].view(torch.int32), want[to].view(torch.int32))


@pytest.mark.parametrize("T", [1, 20, 100])
def test_an_infinite_weight_gives_infinities(T):
    """An infinity in the last ranks of a single adapter, whose ranks may leave the last product part empty."""
    for rank in (8, 16, 24, 32):
        c = Case([(64, 64)], T, 1, rank, torch.bfloat16, seed=14)
        m = c.mods[0]
        m["b"][0, 5, rank - 1] = float("inf")
        c.run()
        assert torch.isinf(m["y"][:, 5]).all()
        assert torch.isfinite(m["y"][:, torch.arange(64, device="cuda") != 5]).all()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,n,rank,ranks", [(1, 2, 64, None), (5, 3, 33, [33, 7, 0]), (16, 16, 16, None), (16, 5, 100, [100, 64, 65, 1, 99]),
                                            (7, 2, 24, None)])
def test_few_tokens_over_long_rows(T, n, rank, ranks, dt):
    """Rows of A too long for the form of one launch; whole and odd numbers of rows, tokens without an adapter."""
    c = Case([(131, 16392), (640, 24576), (8, 8200)], T, n, rank, dt, seed=T + rank, ranks=ranks, y0="in place", pad=8)
    if T > 2:
        c.ids[2] = -1
    c.run()
    c.check()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_broken_adapters_among_few_tokens_over_long_rows(dt):
    """As above, in the form of two launches for up to 16 tokens."""
    T, n, rank = 9, 4, 16
    c = Case([(130, 16384), (64, 20000)], T, n, rank, dt, seed=20)
    c.ids[:n] = torch.arange(n, dtype=torch.int32)
    for m in c.mods:
        m["b"][1, ::3, 0], m["b"][1, 1::3, rank - 1], m["a"][2, 1, 5] = float("nan"), float("inf"), float("inf")
    c.run()
    whole = (c.ids != 1) & (c.ids != 2)
    for m in c.mods:
        y, mag = su.lora64(m["x"], m["a"], m["b"], c.ids.tolist(), None, c.scales.tolist(), m["src"])
        bound = su.U32 * (8 + 2 * math.sqrt(m["K"]) + 2 * math.sqrt(rank)) * mag
        assert ((m["y"].double() - y).abs() <= bound)[whole].all()
        assert torch.isinf(m["y"][c.ids == 1][:, 1::3]).all()


@pytest.mark.parametrize("T,n,rank", [(1, 1, 64), (3, 2, 9), (6, 2, 1)])
def test_one_launch_and_two_agree(T, n, rank):
    """The same projection alone (one launch) and beside one of long rows (two): both within the bound, skipped and
    used tokens in turn."""
    for shapes in ([(300, 512)], [(300, 512), (16, 1 << 18)]):
        c = Case(shapes, T, n, rank, torch.bfloat16, seed=30)
        c.ids[1::2] = -1
        c.run()
        c.check()
