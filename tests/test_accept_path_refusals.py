"""What accept_path refuses it refuses before anything has joined the cache (no GPU: launches are only counted)."""
import pytest
import torch

from paper_2509_04377_amd import engine, synth
from paper_2509_04377_amd.engine import LayeredCache, PagedCache, triggers

B, BUDGET = 16, 64


def _cache(lens, layers=0):
    wl = synth.LLAMA32_1B.with_(dtype="f32", layers=max(layers, 1), num_kv_heads=2, num_q_heads=4, num_seqs=len(lens), budget=BUDGET, steps=200)
    layout = synth.page_layout(wl, list(lens) * max(layers, 1), 1)
    if layers:
        c = LayeredCache(torch.float32, layers, len(lens), 2, 4, 64, B, layout, BUDGET, device="cpu")
    else:
        c = PagedCache.create(torch.float32, len(lens), 2, 4, 64, B, layout, BUDGET, device="cpu")
    c.set_host_lens(lens)
    return c


def _accept(c, n, layers=0):
    shape = (layers,) * bool(layers) + (len(n), 64, 2, 64)
    drafts = torch.zeros(shape)
    c.accept_path(drafts, drafts, torch.zeros((len(n), 64), dtype=torch.int32), torch.tensor(n, dtype=torch.int32), n)


@pytest.mark.parametrize("layers", [0, 2])
@pytest.mark.parametrize("lens,n", [([41, 50], [40, 3]), ([64, 10], [1, 0]), ([0, 63], [5, 2]), ([0, 0], [0, 64]), ([17, 80], [64, 1])])
def test_by_attention_before_any_step(monkeypatch, layers, lens, n):
    """Refused exactly where an eviction would be due, with nothing launched and no length changed."""
    calls = []
    monkeypatch.setattr(engine, "_launch", lambda fn, *a: calls.append(fn.__name__))
    c = _cache(lens, layers)
    c.evict_by_attention()
    before = list(c.host_lens)

    def due(length, tokens):
        for _ in range(tokens):
            if triggers([length], B, BUDGET)[0]:
                return True
            length += 1
        return False

    if any(due(a, b) for a, b in zip(before, n)):
        with pytest.raises(RuntimeError, match="no attention step before the first eviction"):
            _accept(c, n, layers)
        assert not calls and c.host_lens == before
    else:
        _accept(c, n, layers)
        assert c.host_lens == [a + b for a, b in zip(before, n)]
        assert calls and all(name == "pe_append_path" for name in calls)
    # behind a step the same path is taken
    for x in [c.folded] + c.per_layer if layers else [c]:
        x.attention.started = True
    c.host_lens = before
    _accept(c, n, layers)


def test_every_length_and_path(monkeypatch):
    """The refusal against the loop's own evictions, counted one by one."""
    calls = []
    monkeypatch.setattr(engine, "_launch", lambda fn, *a: calls.append(fn.__name__))
    for budget in (16, 64):
        for length in range(82):
            for tokens in (0, 1, 2, 15, 16, 17, 48, 64):
                c = _cache([length])
                c.budget, c.host_lens = budget, [length]
                if length + tokens > c.desc.max_blocks * B and length > BUDGET:
                    continue
                c.evict_by_attention()
                c.attention.started = True
                calls.clear()
                _accept(c, [tokens])
                evicts = "pe_evict_blocks_ex" in calls
                c.host_lens, c.attention.started = [length], False
                if evicts:
                    with pytest.raises(RuntimeError):
                        _accept(c, [tokens])
                    assert c.host_lens == [length]
                else:
                    _accept(c, [tokens])


def test_lengths_of_all_layers_follow_a_call_that_fails_on_its_way(monkeypatch):
    """A call of the library's that raises behind an eviction: the driver's lengths are what is left, as the folded cache's are."""
    c = _cache([64, 10], 2)

    def launch(fn, *a):
        if fn.__name__ == "pe_append_path":
            raise ValueError("k_draft must be contiguous")

    monkeypatch.setattr(engine, "_launch", launch)
    with pytest.raises(ValueError):
        _accept(c, [1, 1], 2)
    assert c.host_lens == [48, 10] and c.folded.host_lens == [48, 10, 48, 10]
