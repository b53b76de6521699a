"""The host's part of verifying drafts, selecting pages and evicting by attention: its mirror of the lengths, which pages it has
bounded, what it refuses (no GPU: the launches are off)."""
import random

import pytest
import torch

from paper_2509_04377_amd import synth
from paper_2509_04377_amd.engine import LayeredCache, PagedCache, host_only

B = 16


def _cache(lens, budget, **kw):
    wl = synth.LLAMA32_1B.with_(dtype="f32", layers=1, num_kv_heads=2, num_q_heads=4, num_seqs=len(lens), budget=budget, steps=200)
    cache = PagedCache.create(torch.float32, len(lens), 2, 4, 64, B, synth.page_layout(wl, lens, 1), budget, device="cpu", **kw)
    cache.set_host_lens(lens)
    return cache


def _one_by_one(n, tokens, budget):
    for _ in range(tokens):
        n -= B if n > 0 and n % B == 0 and n >= budget else 0
        n += 1
    return n


@pytest.mark.parametrize("seed", range(4))
def test_lengths_behind_a_path_are_those_of_single_steps(seed):
    r = random.Random(seed)
    S, budget = 7, 64
    lens = [r.choice([0, 1, 15, 16, 48, 63, 64, 90]) for _ in range(S)]
    cache = _cache(lens, budget)
    want = list(cache.host_lens)
    drafts = torch.zeros((S, 64, 2, 64))
    with host_only():
        for _ in range(6):
            n = [r.choice([0, 0, 1, 16, 17, 40, 64]) for _ in range(S)]
            cache.accept_path(drafts, drafts, torch.zeros((S, 64), dtype=torch.int32), torch.tensor(n, dtype=torch.int32), n)
            want = [_one_by_one(a, b, budget) for a, b in zip(want, n)]
            assert cache.host_lens == want


def test_a_sequence_at_the_end_of_its_path_keeps_its_pages(monkeypatch):
    cache = _cache([64, 64, 63, 64, 10], 64)
    seen = []
    monkeypatch.setattr(PagedCache, "score_and_evict", lambda self: seen.append(self.block_table.data_ptr() if self.desc.num_seqs < 5 else 0))
    drafts = torch.zeros((5, 4, 2, 64))
    n = [1, 0, 4, 2, 0]
    with host_only():
        cache.accept_path(drafts, drafts, torch.zeros((5, 4), dtype=torch.int32), torch.tensor(n, dtype=torch.int32), n)
    rows = [cache.block_table[s].data_ptr() for s in range(5)]
    assert seen == [rows[0], rows[3], rows[2]] and cache.host_lens == [49, 64, 51, 50, 10]
    part = cache.rows(1, 3)
    assert part.desc.num_seqs == 2 and part.desc.max_blocks == cache.desc.max_blocks and part.host_lens == [64, 51]
    assert part.seq_lens.data_ptr() == cache.seq_lens[1:].data_ptr() and part.scores.shape[0] == 2


def test_path_lengths_that_are_refused():
    cache = _cache([10, 20], 64)
    drafts, path = torch.zeros((2, 4, 2, 64)), torch.zeros((2, 4), dtype=torch.int32)
    for n in ([1], [1, 2, 3], [-1, 2], [5, 1]):
        with pytest.raises(ValueError, match="host_path_lens"), host_only():
            cache.accept_path(drafts, drafts, path, torch.zeros(2, dtype=torch.int32), n)
    assert cache.host_lens == [10, 20]


def test_a_path_that_leaves_the_table_is_refused():
    """Without evictions (a budget beyond the table) a row holds what its table holds; at a budget it never gets that far."""
    cache = _cache([10, 20], 64)
    drafts, path, n = torch.zeros((2, 64, 2, 64)), torch.zeros((2, 64), dtype=torch.int32), [54, 44]
    cache.budget = 10 ** 6
    assert cache.desc.max_blocks * B == 64
    with host_only():
        with pytest.raises(ValueError, match="left of a table row"):
            cache.accept_path(drafts, drafts, path, torch.tensor([50, 45], dtype=torch.int32), [50, 45])
        assert cache.host_lens == [10, 20]
        cache.accept_path(drafts, drafts, path, torch.tensor(n, dtype=torch.int32), n)
        assert cache.host_lens == [64, 64]
        cache.budget = 64
        cache.accept_path(drafts, drafts, path, torch.tensor([64, 64], dtype=torch.int32), [64, 64])
    assert cache.host_lens == [_one_by_one(64, 64, 64)] * 2


@pytest.mark.parametrize("seed", range(3))
def test_every_page_behind_the_newest_has_bounds(monkeypatch, seed):
    """A model of the pages: which have bounds is noted by the launch that would have made them; an eviction takes any."""
    r = random.Random(seed)
    lens, budget = [0, 40, 64, 64, 31], 64
    cache = _cache(lens, budget)
    cache.select_pages(3)
    pages = [[False] * -(-n // B) for n in cache.host_lens]   # per sequence: has bounds
    n_now = list(cache.host_lens)

    def launch(fn, *a):
        if fn.__name__ == "pe_page_bounds":
            for s, p in enumerate(pages):
                full = n_now[s] // B
                for j in range(max(0, full - a[4]) if a[4] else 0, full):
                    p[j] = True
        elif fn.__name__ == "pe_append_kv":
            for s, p in enumerate(pages):
                p += [False] if n_now[s] % B == 0 else []
                n_now[s] += 1
        elif fn.__name__ == "pe_append_path":
            for s, p in enumerate(pages):
                take = min(a[4][s] - done[s], B - n_now[s] % B)
                p += [False] if take and n_now[s] % B == 0 else []
                n_now[s], done[s] = n_now[s] + take, done[s] + take
        elif fn.__name__ == "pe_select_pages":
            assert all(p[:-1] == [True] * len(p[:-1]) for p in pages)
        elif "evict" in fn.__name__:
            first = (a[2].data_ptr() - cache.block_table.data_ptr()) // (4 * cache.block_table.stride(0))
            for s in range(first, first + a[0].num_seqs):
                if n_now[s] and n_now[s] % B == 0 and n_now[s] >= budget:
                    del pages[s][r.randrange(len(pages[s]))]
                    n_now[s] -= B

    from paper_2509_04377_amd import engine
    monkeypatch.setattr(engine, "_launch", launch)
    x = torch.zeros((5, 64, 2, 64))
    for step in range(120):
        if r.random() < 0.2:
            n, done = [r.choice([0, 1, 16, 30]) for _ in range(5)], [0] * 5
            cache.accept_path(x, x, torch.zeros((5, 64), dtype=torch.int32), torch.tensor(n, dtype=torch.int32), n)
        cache.decode_step(x[:, 0], x[:, 0], x[:, :2], x)
        assert n_now == cache.host_lens


def test_what_does_not_go_together():
    cache = _cache([10, 20], 64)
    cache.evict_by_attention()
    with pytest.raises(ValueError, match="over all pages"):
        cache.select_pages(4)
    cache.select_pages(0)
    with pytest.raises(RuntimeError, match="nothing to choose a page by"):
        cache.score_and_evict()
    cache = _cache([10, 20], 64)
    cache.select_pages(4)
    with pytest.raises(ValueError, match="over all pages"):
        cache.evict_by_attention()
    cache.select_pages(0)
    cache.evict_by_attention()


def test_layers_advance_together():
    lens = [64, 50, 0]
    wl = synth.LLAMA32_1B.with_(dtype="f32", layers=2, num_kv_heads=2, num_q_heads=4, num_seqs=3, budget=64, steps=200)
    model = LayeredCache(torch.float32, 2, 3, 2, 4, 64, B, synth.page_layout(wl, lens * 2, 1), 64, device="cpu")
    model.set_host_lens(lens)
    drafts, n = torch.zeros((2, 3, 20, 2, 64)), [17, 3, 20]
    with host_only():
        model.accept_path(drafts, drafts, torch.zeros((3, 20), dtype=torch.int32), torch.tensor(n, dtype=torch.int32), n)
    assert model.host_lens == [_one_by_one(a, b, 64) for a, b in zip(lens, n)] == model.folded.host_lens[3:]
