"""A step whose outputs take the queries' place, where weights have to be made before the first eviction: the queries are still needed."""
import pytest
import torch

from paper_2509_04377_amd import engine, synth
from paper_2509_04377_amd.engine import LayeredCache, PagedCache

from _paged64 import DTYPES

HK, G, B, BUDGET, LENS, LAYERS = 2, 4, 16, 64, [64, 90, 23], 2


def _cache(dt, D, layers, device, shared=False):
    wl = synth.LLAMA32_1B.with_(dtype=dt, layers=max(layers, 1), num_kv_heads=HK, num_q_heads=HK * G, num_seqs=len(LENS), head_dim=D, budget=BUDGET,
                                steps=200)
    layout = synth.page_layout(wl, LENS * max(layers, 1), 5, shared=shared)
    make = (LayeredCache, (layers,)) if layers else (PagedCache.create, ())
    c = make[0](DTYPES[dt], *make[1], len(LENS), HK, HK * G, D, B, layout, BUDGET, device=device, shared=shared)
    if device != "cpu":
        for l in range(max(layers, 1)):
            (c.per_layer[l] if layers else c).prefill_prune(*synth.prompt_kv(wl, l, LENS, 5, device=device), max(LENS))
    c.set_host_lens(LENS)
    c.evict_by_attention()
    return c


@pytest.mark.parametrize("layers", [0, LAYERS])
def test_nothing_is_written_over_the_queries_before_they_are_read_last(monkeypatch, layers):
    seen = []
    monkeypatch.setattr(engine, "_launch", lambda fn, *a: seen.append((fn.__name__, a)))
    c = _cache("f32", 64, layers, "cpu")
    lead = (layers,) if layers else ()
    nk, q = torch.zeros(lead + (len(LENS), HK, 64)), torch.zeros(lead + (len(LENS), HK * G, 64))
    c.decode_step(nk, nk, q, q)
    reads = [a for name, a in seen if name == "pe_paged_decode_weights"]
    n = max(layers, 1)
    assert len(reads) == 2 * n
    for l in range(n):
        assert reads[l][1].data_ptr() == reads[n + l][1].data_ptr() == reads[n + l][10].data_ptr() != reads[l][10].data_ptr()


@pytest.mark.gpu
@pytest.mark.parametrize("layers", [0, LAYERS])
@pytest.mark.parametrize("dt,D,shared", [("bf16", 128, False), ("f32", 64, True)])
def test_steps_in_place_of_the_queries(dt, D, shared, layers):
    print("case in place", dt, D, shared, layers, flush=True)
    got = []
    for in_place in (False, True):
        c, g, outs = _cache(dt, D, layers, "cuda", shared), torch.Generator().manual_seed(4), []
        lead = (layers,) if layers else ()
        for step in range(36):
            nk, nv, q = (torch.randn(lead + (len(LENS), h, D), generator=g).to(DTYPES[dt]).cuda() for h in (HK, HK, HK * G))
            out = q if in_place else torch.empty_like(q)
            c.decode_step(nk, nv, q, out)
            outs.append(out)
        f = c.folded if layers else c
        got.append(outs + [f.scores, f.block_table, f.seq_lens])
    for i, (a, b) in enumerate(zip(*got)):
        assert torch.equal(a, b), i
