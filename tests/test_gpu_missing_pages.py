"""Rows that lack pages, as a plan leaves them that found too few, stepped all the same: nothing outside the pools is read or written, and the
other rows are what they are."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd.engine import FreePages, LayeredCache, LayeredQuantCache, PagedCache, QuantCache, empty_layout

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt,D,B", [(torch.bfloat16, 128, 16), (torch.float32, 64, 32), (torch.bfloat16, 64, 128), (torch.float32, 128, 16)])
def test_scores(dt, D, B, shared):
    """A missing page is read as page 0, by all ways to a score."""
    print("case scores", dt, D, B, shared, flush=True)
    S, Hk, n = 3, 2, 6
    heads, rows = ((Hk,), ()) if shared else ((), (Hk,))
    P = S * (1 if shared else Hk) * n + 1
    g = torch.Generator().manual_seed(D + B)
    kp, vp = (torch.randn((P, B) + heads + (D,), generator=g).to(dt).to(DEV) for _ in range(2))
    whole = (torch.randperm(P - 1, generator=g).int() + 1).view((S,) + rows + (n,)).to(DEV)
    table, zero = whole.clone(), whole.clone()
    for where in ((0,), (1, ...) + (slice(2, 4),), (2, ...) + (n - 1,)):   # all pages of a sequence, two, the last one
        table[where], zero[where] = -1, 0
    desc = pe.make_desc(dt, S, Hk, Hk, D, B, n, P, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    lens = _i32([n * B] * S)

    def all_ways(t):
        got = []
        for call in (lambda o: pe.pe_score_blocks(desc, kp, vp, t, lens, o), lambda o: pe.pe_score_recent_blocks(desc, kp, vp, t, lens, 3, o),
                     lambda o: pe.pe_score_triggered_blocks(desc, kp, vp, t, lens, 2 * B, o)):
            o = torch.full((S, Hk, n), 7.0, device=DEV)
            call(o)
            got.append(o)
        if not shared:   # in one pass with the eviction, whose choice goes by the same scores
            o, at, freed, t2, l2 = torch.full((S, Hk, n), 7.0, device=DEV), *(torch.full((S, Hk), -9, dtype=torch.int32, device=DEV) for _ in range(2)), t.clone(), lens.clone()
            pe.pe_score_evict(desc, kp, vp, t2, l2, 2 * B, o, at, freed)
            got += [o, at, l2]
            assert torch.equal(freed, t.gather(2, at.long()[..., None])[..., 0])
        torch.cuda.synchronize()
        return got

    for a, b in zip(all_ways(table), all_ways(zero)):
        assert torch.equal(a, b)


FORMS = [("paged", torch.bfloat16, 128, 4, {}), ("paged", torch.bfloat16, 64, 1, {}), ("paged", torch.float32, 64, 2, {}), ("paged", torch.bfloat16, 64, 8, {"decode_splits": 3}),
         ("paged", torch.float32, 128, 4, {"decode_splits": 2}), ("apart", torch.bfloat16, 64, 4, {}), ("selected", torch.bfloat16, 64, 4, {}),
         ("attention", torch.float32, 64, 4, {}), ("layers", torch.bfloat16, 64, 4, {}), ("layers", torch.float32, 128, 1, {}),
         ("quant", torch.bfloat16, 128, 4, {}), ("quant", torch.float32, 64, 8, {}), ("quant_layers", torch.bfloat16, 64, 2, {})]


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("kind,dt,D,G,opts", FORMS)
def test_steps_leave_a_place_without_a_sequence_alone(kind, dt, D, G, opts, shared):
    """Sequences 0 and 2 step over evictions with place 1 emptied, and are what they are where a third one steps there. Nothing of place 1 changes."""
    print("case steps", kind, dt, D, G, shared, flush=True)
    S, Hk, B, budget, lens = 3, 2, 16, 48, [40, 48, 7]
    layers = 2 if "layers" in kind else 1
    rows, width, n_spare = 1 if shared else Hk, 4, 4
    P = layers * S * rows * (width + n_spare)

    def life(ends):
        g = torch.Generator().manual_seed(5)
        layout = empty_layout(layers * S, Hk, width, n_spare, P, DEV, shared)
        args, cls = (Hk, Hk * G, D, B, layout, budget), QuantCache if "quant" in kind else PagedCache
        if layers > 1:
            c = (LayeredQuantCache if "quant" in kind else LayeredCache)(dt, layers, S, *args, shared=shared)
        else:
            c = cls.create(dt, S, *args, shared=shared, **({} if "quant" in kind else {"decode_opts": opts}))
        f = c.folded if layers > 1 else c
        plans = c.admit(_i32(lens), sum(lens), FreePages.of(torch.randperm(P, generator=g).int().to(DEV)))
        plans = plans if layers > 1 else [plans]
        stage = PagedCache.create(dt, S, *args[:-2], empty_layout(S, Hk, width, 1, P, DEV, shared), budget, shared=shared)
        for l in range(layers):
            k, v = (torch.randn((sum(lens), Hk, D), generator=g).to(dt).to(DEV) for _ in range(2))
            if "quant" in kind:
                stage.seq_lens.zero_()
                p = stage.admit(_i32(lens), sum(lens), FreePages.of(torch.arange(P, dtype=torch.int32, device=DEV)))
                stage.prefill_prune(k, v, p.cu_seqlens, max(lens))
                stage.set_host_lens(lens)
                c.take_layer(l, stage) if layers > 1 else c.take(stage)
            else:
                (c.per_layer[l] if layers > 1 else c).prefill_prune(k, v, plans[l].cu_seqlens, max(lens))
        c.set_host_lens(lens)
        if kind == "selected":
            c.select_pages(2)
        if kind == "attention":
            c.evict_by_attention()
        pools = [f.k.view(torch.uint8), f.v.view(torch.uint8), f.scales, f.k_tail, f.v_tail] if "quant" in kind else [f.k_pool, f.v_pool]
        def step_all(o):
            nk, nv, q = (torch.randn(lead + (h, D), generator=g).to(dt).to(DEV) for h in (Hk, Hk, Hk * G))
            c.decode_step(nk, nv, q, o, **({"fused": False} if kind == "apart" else {}))
            return o.view((layers, S) + o.shape[len(lead):])[:, [0, 2]]

        lead = (layers, S) if layers > 1 else (S,)
        if kind == "attention":   # place 1 would evict at once: all of them look once more where it does, so all three take that step
            step_all(torch.zeros(lead + (Hk * G, D), dtype=dt, device=DEV))
        if ends:
            pages = c.end([1])
            assert len(pages) == layers * rows * (3 + n_spare)
            of_pages = lambda t: t[pages.long()].clone() if t.shape[0] == P else t.view(layers, S, *t.shape[1:])[:, 1].clone()   # noqa: E731
            still = [of_pages(t) for t in pools]
        outs = []
        for step in range(40):
            outs.append(step_all(torch.zeros(lead + (Hk * G, D), dtype=dt, device=DEV)))
            assert f.seq_lens.tolist() == c.host_lens * layers, step
        if ends:
            assert c.host_lens[1] == -1
            for t, nothing in ((f.block_table, -1), (f.spare, -1), (f.spare_used, 0)):
                assert bool((t.view((layers, S) + t.shape[1:])[:, 1] == nothing).all())
            assert all(torch.equal(a, of_pages(t)) for a, t in zip(still, pools))
        held = [t.view((layers, S) + t.shape[1:])[:, [0, 2]].clone() for t in (f.block_table, f.spare_used, f.seq_lens)]
        return outs + held

    assert all(torch.equal(a, b) for a, b in zip(life(True), life(False)))


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_a_sequence_without_pages_is_stepped(shared, quant):
    """Nobody was told that the list did not hold sequence 1: it reaches the budget without a page, and sequence 0 is what it is alone."""
    print("case without pages", shared, quant, flush=True)
    S, Hk, G, D, B, budget, width, n_spare = 2, 2, 2, 64, 16, 32, 3, 3
    rows = 1 if shared else Hk
    P = rows * (width + n_spare)
    lens = [30, 32]

    def life(told):
        g = torch.Generator().manual_seed(6)
        c = (QuantCache if quant else PagedCache).create(torch.bfloat16, S, Hk, Hk * G, D, B, empty_layout(S, Hk, width, n_spare, P, DEV, shared), budget,
                                                         shared=shared)
        plan = c.admit(_i32(lens), 62, FreePages.of(torch.randperm(P, generator=g).int().to(DEV)))
        assert plan.admitted.tolist() == [1, 0]
        k, v = (torch.randn((62, Hk, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
        if quant:
            stage = PagedCache.create(torch.bfloat16, S, Hk, Hk * G, D, B, empty_layout(S, Hk, width, 1, 2 * P, DEV, shared), budget, shared=shared)
            p = stage.admit(_i32(lens), 62, FreePages.of(torch.arange(2 * P, dtype=torch.int32, device=DEV)))
            stage.prefill_prune(k, v, p.cu_seqlens, 32)
            c.take(stage)
        else:
            c.prefill_prune(k, v, plan.cu_seqlens, 32)
        c.set_host_lens(lens)
        if told:
            c.end([1])
        outs = []
        for step in range(40):
            nk, nv, q = (torch.randn((S, h, D), generator=g).to(torch.bfloat16).to(DEV) for h in (Hk, Hk, Hk * G))
            o = torch.zeros_like(q)
            c.decode_step(nk, nv, q, o)
            outs.append(o[0])
        return outs + [c.block_table[0], c.seq_lens[0]]

    assert all(torch.equal(a, b) for a, b in zip(life(False), life(True)))
