"""examples/paged_decode.py: requests and pages, on a machine without a GPU (a step's kernels are left out)."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SPEC = importlib.util.spec_from_file_location("paged_decode", os.path.join(ROOT, "examples", "paged_decode.py"))
example = importlib.util.module_from_spec(SPEC)
SPEC.loader.exec_module(example)


class Server(example.Server):
    """Pages as the example's server holds them, and tokens that count on."""

    def __init__(self, seqs, pages, page_size, longest):
        self.seqs, self.page_size, self.row = seqs, page_size, -(-longest // page_size)
        self.free, self.held = list(range(pages)), [[] for _ in range(seqs)]
        self.pages, self.steps, self.fullest = pages, 0, 0

    def run(self, counts, lens, tokens, given, stream):
        assert len(tokens) == len(given) == sum(counts) <= example.MOST and min(counts) >= 0
        for b, n in enumerate(lens):
            assert n <= self.row * self.page_size
            self.hold(b, n)
        pages = sum(self.held, []) + self.free
        assert sorted(pages) == list(range(self.pages))        # every page once
        self.steps, self.fullest = self.steps + 1, max(self.fullest, self.pages - len(self.free))
        self.logp, self.top, self.top_logp = torch.zeros(len(tokens)), torch.tensor(tokens)[:, None] + 1, torch.full((len(tokens), 1), -0.5)


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: None)


def check(prompts, n, history, scored, server):
    for p, h, s in zip(prompts, history, scored):
        assert h == p + [p[-1] + 1 + i for i in range(n)] and s == [0.0, -0.5 * n]
    assert sorted(server.free) == list(range(server.pages)) and not any(server.held)


@pytest.mark.parametrize("pages", [8, 9, 15, 16, 40])
@pytest.mark.parametrize("n", [1, 7, 40])
def test_requests_wait_for_pages(pages, n):
    """More places than pages for them: a request begins when the pages of its whole answer are there, and all are answered."""
    prompts = [[r] * (1 + 11 * r % 23) for r in range(12)]
    server = Server(seqs=6, pages=pages, page_size=8, longest=64)
    history, scored = example.serve(server, prompts, n)
    check(prompts, n, history, scored, server)
    assert server.fullest <= pages


def test_the_program_s_own_requests():
    """The command's requests at any number of tokens."""
    for requests, n in ((24, 40), (24, 100), (24, 400), (1, 1), (60, 3)):
        prompts, sizes = example.workload(requests, n)
        server = Server(**sizes)
        history, scored = example.serve(server, prompts, n)
        check(prompts, n, history, scored, server)


@pytest.mark.parametrize("prompts,n", [
    ([[1] * 60], 6), ([[1], [2] * 65], 1),          # more places than a row of the table has
    ([[1] * 30, [2] * 40], 10),                     # more pages than there are
    ([[1], []], 3), ([[1]], 0)])
def test_requests_that_cannot_be_served(prompts, n):
    server = Server(seqs=2, pages=6, page_size=8, longest=64)
    with pytest.raises(ValueError):
        example.serve(server, prompts, n)
    assert server.steps == 0 and len(server.free) == 6


def test_a_request_that_just_fits():
    server = Server(seqs=2, pages=8, page_size=8, longest=64)
    history, _ = example.serve(server, [[3] * 60, [4] * 60], 5)         # the last token's key is never stored
    assert [len(h) for h in history] == [65, 65] and server.fullest == 8
