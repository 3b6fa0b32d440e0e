"""The serving example's scheduler on the CPU: every request is answered whatever the page pool, without endless restarts."""
from types import SimpleNamespace

import numpy as np
import pytest

from examples.serve_decoder import serve
from tests import attn_reference as R

VOCAB = 512


def answer(text):
    return (sum(text) * 31 + len(text)) % VOCAB


class Steps:
    """Stands for a decoder: the bookkeeping of a step by its definition, answers from the tokens a row has in the cache."""

    def __init__(self, rows, n_pages, max_tokens, max_pages, page=16, limit=20000):
        self.attn = SimpleNamespace(cfg=SimpleNamespace(max_requests=rows, max_tokens=max_tokens, n_pages=n_pages, max_pages=max_pages,
                                                        page_tokens=page))
        self.table, self.free = np.full((rows, max_pages), -1, np.int32), np.arange(n_pages, dtype=np.int32)
        self.n_free, self.ctx, self.text = n_pages, [0] * rows, [[] for _ in range(rows)]
        self.page, self.left = page, limit

    def step(self, new_len, tokens):
        self.left -= 1
        assert self.left >= 0, "no end in sight"
        assert len(tokens) == sum(max(n, 0) for n in new_len) <= self.attn.cfg.max_tokens
        s = R.slots(new_len, self.ctx, self.table, self.free, self.n_free, self.page, len(tokens))
        self.table, self.free, self.n_free, self.ctx = s["table"], s["free"], int(s["n_free"][0]), s["kv_len"].tolist()
        for r, n in enumerate(new_len):
            if n < 0:
                self.text[r] = []
            elif s["admitted"][r]:
                self.text[r] += tokens[s["q_start"][r]:s["q_start"][r + 1]]
        return [answer(t) for t in self.text], s["admitted"].tolist()


def expected(prompt, n_new):
    text = list(prompt)
    for _ in range(n_new):
        text.append(answer(text))
    return text[len(prompt):]


def run(dec, prompts, n_new, **kw):
    assert serve(dec, prompts, n_new, **kw) == [expected(p, n_new) for p in prompts]
    assert dec.n_free == dec.attn.cfg.n_pages and sorted(dec.free.tolist()) == list(range(dec.n_free))


@pytest.mark.parametrize("requests,n_new", [(12, 24), (16, 48), (24, 48), (12, 96)])
def test_the_examples_own_workload_ends(requests, n_new):
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, VOCAB, int(rng.integers(1, 150))).tolist() for _ in range(requests)]
    run(Steps(8, 40, 128, 32), prompts, n_new)


@pytest.mark.parametrize("seed", range(300))
def test_random_pools_end(seed):
    rng = np.random.default_rng(seed)
    n_new, page = int(rng.integers(1, 40)), int(rng.choice([16, 32]))
    prompts = [rng.integers(0, VOCAB, int(rng.integers(1, 120))).tolist() for _ in range(int(rng.integers(1, 15)))]
    largest = max(R.ceil_div(len(p) + n_new - 1, page) for p in prompts)
    pages = largest + int(rng.integers(0, 2 * largest + 1))               # the largest request fits just so, or more do
    run(Steps(int(rng.integers(1, 9)), pages, int(rng.integers(1, 130)), largest + int(rng.integers(0, 3)), page), prompts, n_new,
        chunk=int(rng.integers(1, 60)))


def test_a_request_that_holds_pages_is_not_stopped_by_one_that_holds_none():
    """The younger request in the lower row asks first and counts against the older one's needs."""
    run(Steps(2, 8, 64, 8), [[1] * 28, [2] * 118, [3] * 21], 7, chunk=49)


def test_requests_that_cannot_be_served_are_refused():
    for dec, prompts, n_new in ((Steps(2, 4, 64, 9), [[1] * 60], 6), (Steps(2, 9, 64, 4), [[1], [1] * 60], 6), (Steps(2, 4, 64, 4), [[1], []], 6),
                                (Steps(2, 4, 64, 4), [[1]], 0)):
        with pytest.raises(ValueError):
            serve(dec, prompts, n_new)
    run(Steps(2, 4, 64, 4), [[1] * 59], 6)                                  # 64 tokens in the cache: four pages
