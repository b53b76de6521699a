"""Generation with the caches of engine.py: prompts pruned, drafts verified and accepted, steps over selected pages, evictions by the
attention that pages got -- one after the other on one cache, against plain computations in 64 bits and against single steps."""
import math

import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd import synth
from paper_2509_04377_amd.engine import GraphedStepper, LayeredCache, PagedCache

from _paged64 import DTYPES, assert_close, attend
from test_gpu_tree import _trees, _words
from test_host_marshalling import _Recorder

pytestmark = pytest.mark.gpu
DEV = "cuda"
S, Hk, G, B, BUDGET = 5, 2, 4, 16, 64
LENS = [90, 64, 41, 7, 63]


def _cache(dt, D, shared, lens=LENS, layers=0):
    wl = synth.LLAMA32_1B.with_(dtype=dt, layers=max(layers, 1), num_kv_heads=Hk, num_q_heads=Hk * G, num_seqs=len(lens), head_dim=D,
                                budget=BUDGET, steps=200)
    layout = synth.page_layout(wl, list(lens) * max(layers, 1), 5, shared=shared)
    if layers:
        c = LayeredCache(DTYPES[dt], layers, len(lens), Hk, Hk * G, D, B, layout, BUDGET, shared=shared)
    else:
        c = PagedCache.create(DTYPES[dt], len(lens), Hk, Hk * G, D, B, layout, BUDGET, shared=shared)
    for l in range(max(layers, 1)):
        k, v, cu = synth.prompt_kv(wl, l, lens, 5, device=DEV)
        (c.per_layer[l] if layers else c).prefill_prune(k, v, cu, max(lens))
    c.set_host_lens(lens)
    return c


def _inputs(seed, shape, dt):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(DTYPES[dt]).to(DEV)


def _rows(cache, table=None, lens=None):
    """k, v [s][h]: float64 tokens of every row of the cache as its table (or that one) has them."""
    table = (cache.block_table if table is None else table).cpu()
    lens = (cache.seq_lens if lens is None else lens).cpu()
    pools = [p.double().cpu() for p in (cache.k_pool, cache.v_pool)]
    out = []
    for pool in pools:
        per_seq = []
        for s in range(table.shape[0]):
            n = int(lens[s])
            pages = -(-n // B)
            if cache.shared:
                t = pool[table[s, :pages].long()].reshape(-1, Hk, pool.shape[-1])[:n]
                per_seq.append([t[:, h] for h in range(Hk)])
            else:
                per_seq.append([pool[table[s, h, :pages].long()].reshape(-1, pool.shape[-1])[:n] for h in range(Hk)])
        out.append(per_seq)
    return out


def _check_step(out, q, k, v, dtype):
    for s in range(q.shape[0]):
        for h in range(q.shape[1]):
            want, _, bound = attend(q[s, h:h + 1].double().cpu(), k[s][h // G], v[s][h // G])
            assert_close(out[s, h:h + 1], want, bound, dtype)


def _random_path(sees, r):
    """A way from a root down: every node's ancestors are in its mask."""
    leaf = int(torch.randint(0, sees.shape[0], (1,), generator=r))
    return [j for j in range(leaf + 1) if sees[leaf, j]]


@pytest.mark.parametrize("dt,D,shared,mode", [(*c, m) for c in (("bf16", 128, False), ("f32", 64, True))
                                              for m in ("plain", "cached", "fused", "oldest")
                                              if not (c[2] and m == "fused")])   # (pe_score_evict has no head-shared form)
def test_an_accepted_path_leaves_what_single_steps_leave(dt, D, shared, mode):
    """Tables, lengths, pages in use, scores' mirror: as from appending token by token with an eviction wherever one is due, each
    sequence by itself; paths from none to several pages, twice the same draft, and single steps in between."""
    print("case accept", mode, dt, D, shared, flush=True)
    a, b = _cache(dt, D, shared), _cache(dt, D, shared)
    for c in (a, b):
        c.cached_scores, c.fused_evict = mode == "cached", mode == "fused"
        if mode == "oldest":
            c.evict_opts = pe.pe_evict_opts(pe.PE_POLICY_OLDEST, 1, 0, 0, 0)
    parts = [b.rows(s, s + 1) for s in range(S)]
    T = 40
    for turn, lens in enumerate(([0, 1, 23, 9, 1], [40, 40, 0, 40, 17], [8, 16, 32, 0, 16], [0, 0, 0, 0, 0], [1, 1, 1, 1, 1])):
        kd, vd = _inputs(10 + turn, (S, T, Hk, D), dt), _inputs(20 + turn, (S, T, Hk, D), dt)
        path = torch.randint(0, T, (S, T), generator=torch.Generator().manual_seed(turn)).int()
        a.accept_path(kd, vd, path.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), lens)
        for s, part in enumerate(parts):
            for i in range(lens[s]):
                trig = part.triggers()
                if trig[0]:
                    part.score_and_evict()
                    part.evicted(trig)
                d = int(path[s, i])
                part.append_kv(kd[s:s + 1, d].contiguous(), vd[s:s + 1, d].contiguous())
                part.host_lens = [part.host_lens[0] + 1]
        torch.cuda.synchronize()
        assert a.host_lens == [p.host_lens[0] for p in parts] == a.seq_lens.tolist()
        for name in ("block_table", "seq_lens", "spare_used", "freed_phys", "k_pool", "v_pool"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (turn, name)
    assert a.host_lens[0] <= BUDGET


@pytest.mark.parametrize("dt,D,shared", [("bf16", 128, False), ("bf16", 64, True), ("f32", 64, False)])
def test_verification_and_selected_steps_one_after_the_other(dt, D, shared):
    """Prompt, then in turn: a tree of drafts over the cache, the accepted ones into it (evictions where pages fill), a few
    steps over the three best pages, which are looked up by hand, and one over all of them."""
    print("case generation", dt, D, shared, flush=True)
    dtype, T, Hq = DTYPES[dt], 12, Hk * G
    c = _cache(dt, D, shared)
    r = torch.Generator().manual_seed(3)
    for turn in range(4):
        q, kd, vd = _inputs(turn, (S, T, Hq, D), dt), _inputs(40 + turn, (S, T, Hk, D), dt), _inputs(50 + turn, (S, T, Hk, D), dt)
        sees = _trees(S, T, r)
        out = torch.empty_like(q)
        c.tree_decode(q, kd, vd, _words(sees).to(DEV), out)
        k, v = _rows(c)
        for s in range(S):
            for h in range(Hq):
                kk, vv = (torch.cat((x[s][h // G], y[s, :, h // G].double().cpu())) for x, y in ((k, kd), (v, vd)))
                m = torch.cat((torch.ones((T, k[s][h // G].shape[0]), dtype=torch.bool), sees[s]), 1)
                want, _, bound = attend(q[s, :, h].double().cpu(), kk, vv, m)
                assert_close(out[s, :, h], want, bound, dtype)
        ways = [_random_path(sees[s], r) for s in range(S)]
        lens = [len(w) for w in ways]
        path = torch.tensor([w + [0] * (T - len(w)) for w in ways], dtype=torch.int32, device=DEV)
        c.accept_path(kd, vd, path, torch.tensor(lens, dtype=torch.int32, device=DEV), lens)
        c.select_pages(3)
        for step in range(6):
            nk, nv, q1 = _inputs(60 + step, (S, Hk, D), dt), _inputs(70 + step, (S, Hk, D), dt), _inputs(80 + step + 9 * turn, (S, Hq, D), dt)
            o1 = torch.empty_like(q1)
            c.decode_step(nk, nv, q1, o1)
            assert c.seq_lens.tolist() == c.host_lens
            k, v = _rows(c)
            chosen = torch.full_like(c.selection.table, -1).cpu()
            table = c.block_table.cpu()
            for s, n in enumerate(c.host_lens):
                pages, rows = -(-n // B), 1 if shared else Hk
                for row in range(rows):
                    heads = range(Hk) if shared else (row,)
                    score = torch.zeros(max(pages - 1, 0), dtype=torch.float64)
                    for h in heads:
                        kk = k[s][h][:(pages - 1) * B].view(max(pages - 1, 0), B, D)
                        for x in q1[s, h * G:(h + 1) * G].double().cpu():
                            score += torch.maximum(x * kk.amin(1), x * kk.amax(1)).sum(1)
                    score = score.float()
                    best = sorted(sorted(range(pages - 1), key=lambda j: (-float(score[j]), j))[:2] + [pages - 1])
                    at = (s,) if shared else (s, row)
                    chosen[at][:len(best)] = table[at][best]
            assert torch.equal(c.selection.table.cpu(), chosen), (turn, step)
            _check_step(o1, q1, *_rows(c, c.selection.table, c.selection.lens), dtype)
        c.select_pages(0)
        q1, o1 = _inputs(99, (S, Hq, D), dt), torch.empty((S, Hq, D), dtype=dtype, device=DEV)
        c.decode_step(nk, nv, q1, o1)
        _check_step(o1, q1, *_rows(c), dtype)
    assert max(c.host_lens) == BUDGET or c.spare_used.max() > 0


@pytest.mark.parametrize("dt,D,shared", [("bf16", 128, False), ("f32", 64, True)])
def test_evictions_by_attention(dt, D, shared):
    """Each step's output and weights against 64 bits (from the weights before it), and each eviction: the page with the least of
    what the array held, the newest excepted; accepted drafts in between."""
    print("case by attention", dt, D, shared, flush=True)
    dtype, Hq = DTYPES[dt], Hk * G
    c = _cache(dt, D, shared, [64, 80, 63, 20])
    n_seq = 4
    c.evict_by_attention(0.75)
    evictions = 0
    for step in range(40):
        nk, nv, q = _inputs(step, (n_seq, Hk, D), dt), _inputs(100 + step, (n_seq, Hk, D), dt), _inputs(200 + step, (n_seq, Hq, D), dt) * 2
        before, table, trig, lens = c.scores.clone().cpu(), c.block_table.cpu().clone(), c.triggers(), list(c.host_lens)
        k, v = _rows(c)
        if step == 0:   # the first eviction comes before any step: this step's queries decide
            before[:] = math.inf
            for s in range(n_seq):
                for h in range(Hk):
                    w = sum(attend(q[s, x:x + 1].double().cpu(), k[s][h], v[s][h])[1][0] for x in range(h * G, (h + 1) * G))
                    pages = -(-lens[s] // B)
                    before[s, h, :pages] = torch.nn.functional.pad(w, (0, pages * B - lens[s])).view(pages, B).sum(1).float()
        out = torch.empty_like(q)
        c.decode_step(nk, nv, q, out)
        k, v = _rows(c)
        _check_step(out, q, k, v, dtype)
        now = c.scores.cpu()
        for s in range(n_seq):
            old = before[s].clone()
            if trig[s]:
                evictions += 1
                pages = lens[s] // B
                for row in range(1 if shared else Hk):
                    at = (s,) if shared else (s, row)
                    gone = int(c.evicted_logical[at])
                    held = before[s].double().mean(0).float() if shared else before[s, row]
                    least = float(held[:pages - 1].min())
                    assert 0 <= gone < pages - 1 and float(held[gone]) <= least + (1e-3 if step == 0 else 0.0)
                    left = [j for j in range(pages) if j != gone]
                    assert c.block_table[at][:pages - 1].tolist() == table[at][left].tolist()
                    for h in range(Hk) if shared else (row,):
                        old[h, :pages - 1], old[h, pages - 1:] = before[s, h][left], math.inf
            n = c.host_lens[s]
            pages = -(-n // B)
            for h in range(Hk):
                got, off = torch.zeros(pages, dtype=torch.float64), 0.0
                for x in range(h * G, (h + 1) * G):
                    one = torch.ones((n, 1), dtype=torch.float64)
                    _, w, rel = attend(q[s, x:x + 1].double().cpu(), k[s][h], one)
                    got += torch.nn.functional.pad(w[0], (0, pages * B - n)).view(pages, B).sum(1)
                    off = max(off, float(rel[0, 0]))
                was = old[h, :pages].double()
                was[~torch.isfinite(was)] = 0.0
                want = 0.75 * was + got
                # (step 0: the weights before it are this test's own, rounded, and within `off` of the kernel's, as are those it adds)
                slack = (off * (got + 0.75 * was if step == 0 else got) + 12 * 2.0 ** -24 * want)
                assert bool(((now[s, h, :pages].double() - want).abs() <= slack).all()), (step, s, h)
                assert bool((now[s, h, pages:] == math.inf).all())
        if step % 13 == 12:
            n = [5, 0, 17, 30]
            kd, vd = _inputs(300 + step, (n_seq, 30, Hk, D), dt), _inputs(400 + step, (n_seq, 30, Hk, D), dt)
            path = torch.arange(30, dtype=torch.int32, device=DEV).repeat(n_seq, 1)
            c.accept_path(kd, vd, path, torch.tensor(n, dtype=torch.int32, device=DEV), n)
            assert c.seq_lens.tolist() == c.host_lens
    assert evictions >= 4


def _drive(model, kind, stepper, layers, n_seq, dt, D):
    """Steps of all layers with an accepted path in between; every output."""
    Hq = Hk * G
    bufs = [torch.empty((layers, n_seq, h, D), dtype=DTYPES[dt], device=DEV) for h in (Hk, Hk, Hq, Hq)]
    if kind == "selected":
        model.select_pages(3)
    else:
        model.evict_by_attention(0.5)
    graph = GraphedStepper(model, *bufs) if stepper else None
    got = []
    for step in range(44):
        for i, x in enumerate(bufs[:3]):
            x.copy_(_inputs(1000 * i + step, tuple(x.shape), dt))
        graph.step() if graph else model.decode_step(*bufs)
        got.append(bufs[3].clone())
        if step in (9, 30):
            n = [3, 20, 0]
            kd, vd = (_inputs(7 + step + i, (layers, n_seq, 20, Hk, D), dt) for i in range(2))
            path = torch.arange(20, dtype=torch.int32, device=DEV).repeat(n_seq, 1)
            model.accept_path(kd, vd, path, torch.tensor(n, dtype=torch.int32, device=DEV), n)
    torch.cuda.synchronize()
    return got + [model.folded.block_table.clone(), model.folded.seq_lens.clone(), model.folded.spare_used.clone()]


@pytest.mark.parametrize("kind", ["selected", "attention"])
@pytest.mark.parametrize("dt,D,shared", [("bf16", 64, False), ("f32", 64, True)])
def test_layers_and_graphs(kind, dt, D, shared):
    """All layers from one driver give what the layers give by themselves, and replayed graphs what eager launches give."""
    print("case layers", kind, dt, shared, flush=True)
    layers, lens = 3, [64, 50, 90]
    eager = _drive(_cache(dt, D, shared, lens, layers), kind, False, layers, 3, dt, D)
    replayed = _drive(_cache(dt, D, shared, lens, layers), kind, True, layers, 3, dt, D)
    assert all(torch.equal(a, b) for a, b in zip(eager, replayed))

    model = _cache(dt, D, shared, lens, layers)
    one = model.per_layer[1]
    one.host_lens = [min(n, BUDGET) for n in lens]
    if kind == "selected":
        one.select_pages(3)
    else:
        one.evict_by_attention(0.5)
    for step in range(44):
        nk, nv, q = (_inputs(1000 * i + step, (layers, 3, h, D), dt)[1] for i, h in enumerate((Hk, Hk, Hk * G)))
        out = torch.empty_like(q)
        one.decode_step(nk, nv, q, out)
        assert torch.equal(out, eager[step][1]), step
        if step in (9, 30):
            n = [3, 20, 0]
            kd, vd = (_inputs(7 + step + i, (layers, 3, 20, Hk, D), dt)[1] for i in range(2))
            path = torch.arange(20, dtype=torch.int32, device=DEV).repeat(3, 1)
            one.accept_path(kd, vd, path, torch.tensor(n, dtype=torch.int32, device=DEV), n)


CALLS = {"prefill_prune", "score_triggered_blocks", "evict_blocks", "evict_blocks_ex", "tree_decode", "append_path", "page_bounds",
         "select_pages", "paged_decode", "paged_decode_weights", "append_paged_decode"}


def _everything(shared):
    got = []
    for kind in ("selected", "attention", None):
        c = _cache("bf16", 64, shared)
        if kind == "selected":
            c.select_pages(2)
        elif kind == "attention":
            c.evict_by_attention()
        for step in range(20):
            nk, nv, q = (_inputs(100 * i + step, (S, h, 64), "bf16") for i, h in enumerate((Hk, Hk, Hk * G)))
            out = torch.empty_like(q)
            c.decode_step(nk, nv, q, out)
            got.append(out)
        q, kd, vd = (_inputs(i, (S, 9, h, 64), "bf16") for i, h in enumerate((Hk * G, Hk, Hk)))
        words, n = _words(_trees(S, 9, torch.Generator().manual_seed(1))).to(DEV), [1, 9, 0, 4, 5]
        lens = torch.tensor(n, dtype=torch.int32, device=DEV)
        for given in (None, lens):
            out = torch.zeros_like(q)
            c.tree_decode(q, kd, vd, words, out, given)
            got.append(out)
        c.accept_path(kd, vd, torch.arange(9, dtype=torch.int32, device=DEV).repeat(S, 1), lens, n)
        got += [c.block_table, c.seq_lens, c.spare_used, c.k_pool, c.v_pool, c.freed_phys]
        got += [c.selection.table, c.selection.lens] if c.selection else [c.scores] if c.attention else []
    return got


@pytest.mark.parametrize("shared", [False, True], ids=["per_head", "shared"])
def test_every_call_goes_the_native_way_and_as_through_ctypes(monkeypatch, shared):
    print("case marshalling", shared, flush=True)
    pe.lib()
    recorder = _Recorder(pe._host)
    monkeypatch.setattr(pe, "_host", recorder)
    native = _everything(shared)
    assert {name for name, _ in recorder.seen} == CALLS and all(status == pe.PE_OK for _, status in recorder.seen)
    monkeypatch.setattr(pe, "_host", pe._NoHost())
    through_ctypes = _everything(shared)
    assert len(native) == len(through_ctypes)
    assert all(torch.equal(a, b) for a, b in zip(native, through_ctypes))
