"""Selected pages and evictions by attention that are switched under a live GraphedStepper: a replayed step uses what an eager one would use,
and nothing of what has been given back.  On the CPU with launches and graphs that are only noted, on the GPU against eager steps."""
import contextlib
import weakref

import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd import engine, synth
from paper_2509_04377_amd.engine import GraphedStepper, LayeredCache

from _paged64 import DTYPES

DEV = "cuda"
LAYERS, HK, G, B, BUDGET = 2, 2, 4, 16, 64
LENS = [64, 50, 23]
SWITCHES = {6: lambda m: m.select_pages(3), 20: lambda m: m.select_pages(0), 26: lambda m: m.select_pages(3), 38: lambda m: m.select_pages(2),
            46: lambda m: m.select_pages(0), 52: lambda m: m.evict_by_attention(0.5), 72: lambda m: m.evict_by_attention(0.9)}


def _model(dt, D, device, shared=False):
    wl = synth.LLAMA32_1B.with_(dtype=dt, layers=LAYERS, num_kv_heads=HK, num_q_heads=HK * G, num_seqs=len(LENS), head_dim=D, budget=BUDGET,
                                steps=200)
    layout = synth.page_layout(wl, LENS * LAYERS, 5, shared=shared)
    return wl, LayeredCache(DTYPES[dt], LAYERS, len(LENS), HK, HK * G, D, B, layout, BUDGET, device=device, shared=shared)


class _Noted:
    """Stands in for a HIP graph: what is launched while it is captured, it launches again."""
    log, capturing = [], None

    def __init__(self):
        self.launches = []

    def replay(self):
        _Noted.log += self.launches


def _noting(monkeypatch):
    def launch(fn, *args):
        if not engine.HostOnly.active:
            at = tuple(a.data_ptr() if isinstance(a, torch.Tensor) else tuple(getattr(a, n) for n, _ in a._fields_)
                       if isinstance(a, (pe.pe_cache_desc, pe.pe_evict_opts)) else a for a in args)
            (_Noted.capturing.launches if _Noted.capturing else _Noted.log).append((fn.__name__, at))

    @contextlib.contextmanager
    def capture(graph):
        _Noted.capturing = graph
        yield
        _Noted.capturing = None

    monkeypatch.setattr(engine, "_launch", launch)
    monkeypatch.setattr(torch.cuda, "CUDAGraph", _Noted)
    monkeypatch.setattr(torch.cuda, "graph", capture)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    monkeypatch.setattr(_Noted, "log", [])


def test_replayed_launches_are_those_of_eager_steps(monkeypatch):
    """Two models over the same tensors, one eager, one through a stepper, switched alike; old selections and weights are kept here, so that no
    two of them are at one address."""
    _noting(monkeypatch)
    _, one = _model("f32", 64, "cpu")
    bufs = [torch.zeros((LAYERS, len(LENS), h, 64)) for h in (HK, HK, HK * G, HK * G)]
    one.set_host_lens(LENS)
    stepper, kept = GraphedStepper(one, *bufs), []
    for step in range(95):
        if step in SWITCHES:
            kept += [(c.selection, c.attention) for c in [one.folded] + one.per_layer]
            SWITCHES[step](one)
        if step == 60:
            one.folded.evict_opts = pe.pe_evict_opts(pe.PE_POLICY_LOWEST_SCORE, 1, 1, 0, 0)
        # (the same step, eager, of the same state: only the host's part of it has to be put back)
        state = [(c, dict(c.__dict__)) for c in [one.folded] + one.per_layer], one.host_lens
        inner = [(x, dict(x.__dict__)) for c in [one.folded] + one.per_layer for x in (c.selection, c.attention) if x is not None]
        _Noted.log.clear()
        one.decode_step(*bufs)
        want = list(_Noted.log)
        for c, fields in state[0] + inner:
            c.__dict__.update(fields)
        one.host_lens = state[1]
        _Noted.log.clear()
        stepper.step()
        assert [name for name, _ in _Noted.log] == [name for name, _ in want], step
        for (name, got), (_, eager) in zip(_Noted.log, want):
            # (scratch that a step makes for itself has an address of its own: the output of weights in front of an eviction)
            differ = [i for i, (a, b) in enumerate(zip(got, eager)) if a != b]
            assert not differ or (name == "pe_paged_decode_weights" and differ == [10]), (step, name, differ)


def test_a_stepper_holds_what_its_graphs_point_into_and_lets_go_of_it(monkeypatch):
    _noting(monkeypatch)
    _, one = _model("f32", 64, "cpu")
    bufs = [torch.zeros((LAYERS, len(LENS), h, 64)) for h in (HK, HK, HK * G, HK * G)]
    one.set_host_lens(LENS)
    stepper = GraphedStepper(one, *bufs)
    for _ in range(3):
        stepper.step()
    plain = len(stepper.graphs)
    for n in (3, 3, 2):
        one.select_pages(n)
        mine = weakref.ref(one.folded.selection)
        stepper.step()
        assert len(stepper.graphs) > plain
        one.select_pages(0)
        assert mine() is not None      # a replay may still be on its way
        stepper.step()
        assert mine() is None and len(stepper.graphs) <= plain + 1   # (a plain step of another kind may have come)
        plain = len(stepper.graphs)


def _drive(dt, D, shared, graphs):
    wl, m = _model(dt, D, DEV, shared)
    for l in range(LAYERS):
        m.prefill_prune_layer(l, *synth.prompt_kv(wl, l, LENS, 5, device=DEV), max(LENS))
    m.set_host_lens(LENS)
    bufs = [torch.empty((LAYERS, len(LENS), h, D), dtype=DTYPES[dt], device=DEV) for h in (HK, HK, HK * G, HK * G)]
    stepper = GraphedStepper(m, *bufs) if graphs else None
    got, g = [], torch.Generator().manual_seed(3)
    for step in range(95):
        if step in SWITCHES:
            SWITCHES[step](m)
            junk = [torch.full((n,), float("nan"), device=DEV) for n in (64, 300, 2000, 20000)]   # takes what has been given back
        for x in bufs[:3]:
            x.copy_(torch.randn(x.shape, generator=g).to(x.dtype))
        stepper.step() if graphs else m.decode_step(*bufs)
        got.append(bufs[3].clone())
        if step in SWITCHES:
            assert all(bool(x.isnan().all()) for x in junk), step
    torch.cuda.synchronize()
    return got + [m.folded.block_table.clone(), m.folded.seq_lens.clone(), m.folded.k_pool.clone(), m.folded.scores.clone()]


@pytest.mark.gpu
@pytest.mark.parametrize("dt,D,shared", [("bf16", 128, False), ("f32", 64, True)])
def test_switched_modes_in_replayed_steps(dt, D, shared):
    print("case switched", dt, D, shared, flush=True)
    eager, replayed = (_drive(dt, D, shared, graphs) for graphs in (False, True))
    for i, (a, b) in enumerate(zip(eager, replayed)):
        assert torch.equal(a, b), i
