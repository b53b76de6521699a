"""Admissions as a program makes them over its life: prompts kept whole beyond the budget, sequences that come while others run."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd.engine import FreePages, GraphedStepper, LayeredCache, LayeredQuantCache, PagedCache, QuantCache, empty_layout

pytestmark = pytest.mark.gpu
DEV = "cuda"
S, Hk, G, D, B, BUDGET = 3, 2, 2, 64, 16, 64


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _randn(g, *shape):
    return torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)


@pytest.mark.parametrize("layers", [0, 2])
@pytest.mark.parametrize("shared", [False, True])
def test_whole_prompts_beyond_the_budget(shared, layers):
    """The mirror says what the device holds, at every step over evictions, and a step evicts as the same calls one by one do."""
    width, n_spare, lens = 10, 4, [100, 64, 21]
    rows, n = 1 if shared else Hk, max(layers, 1)
    P = n * S * rows * (width + n_spare)
    layout = empty_layout(n * S, Hk, width, n_spare, P, DEV, shared)
    args = (Hk, Hk * G, D, B, layout, BUDGET)
    m = LayeredCache(torch.bfloat16, layers, S, *args, shared=shared) if layers else PagedCache.create(torch.bfloat16, S, *args, shared=shared)
    g = torch.Generator().manual_seed(1)
    got = m.admit(_i32(lens), sum(lens), FreePages.of(torch.randperm(P, generator=g).int().to(DEV)), whole=True)
    rope = pe.make_rope(D, 1e4)
    for c, plan in zip(m.per_layer if layers else [m], got if layers else [got]):
        q, k, v = _randn(g, sum(lens), Hk * G, D), _randn(g, sum(lens), Hk, D), _randn(g, sum(lens), Hk, D)
        c.rotate_store(rope, plan, q, k, v, torch.empty_like(q))
    m.set_host_lens(lens, whole=True)
    f = m.folded if layers else m
    assert f.seq_lens.tolist() == lens * n
    evicted = 0
    for step in range(50):
        lead = (layers, S) if layers else (S,)
        nk, nv, q = _randn(g, *lead, Hk, D), _randn(g, *lead, Hk, D), _randn(g, *lead, Hk * G, D)
        evicted += sum(m._triggers() if layers else m.triggers())
        m.decode_step(nk, nv, q, torch.empty_like(q))
        assert f.seq_lens.tolist() == m.host_lens * n, step
        used = f.block_table.view(n * S, rows, width)
        for r, held in enumerate(f.seq_lens.tolist()):
            pages = -(-held // B)
            assert bool((used[r, :, :pages] >= 0).all()) and bool((used[r, :, pages:] == -1).all()), (step, r)
    assert evicted >= 6 and max(m.host_lens) <= 112


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_a_prompt_beside_sequences_that_run(shared, quant):
    """One sequence comes while another one decodes over evictions and a third finds no pages: the first two are what each is by itself."""
    width, n_spare, n_steps = 4, 4, 40
    rows = 1 if shared else Hk
    need = rows * (width + n_spare)
    ids = torch.randperm(8 * need, generator=torch.Generator().manual_seed(2)).int().to(DEV)
    layout = lambda n: empty_layout(S, Hk, width, n, len(ids), DEV, shared)   # noqa: E731
    g = torch.Generator().manual_seed(3)
    prompts = [[_randn(g, n, Hk, D) for _ in range(2)] for n in (90, 75, 200)]
    steps = [(_randn(g, S, Hk, D), _randn(g, S, Hk, D), _randn(g, S, Hk * G, D)) for _ in range(2 * n_steps)]

    def life(first, second, room):
        """first, second: which sequences come in front of the steps, and in the middle of them.  The outputs of every step."""
        make = lambda cls, n: cls.create(torch.bfloat16, S, Hk, Hk * G, D, B, layout(n), BUDGET, shared=shared)   # noqa: E731
        c, out = make(QuantCache if quant else PagedCache, n_spare), []
        free = FreePages.of(ids[:room].contiguous())
        for half, who in enumerate((first, second)):
            lens = [prompts[s][0].shape[0] if s in who else 0 for s in range(S)]
            k, v = (torch.cat([prompts[s][i] for s in who] or [prompts[0][i][:0]]) for i in range(2))
            plan = c.admit(_i32(lens), sum(lens), free)
            was = c.admitted.tolist()
            if quant:
                stage = make(PagedCache, 1)
                p = stage.admit(_i32(lens), sum(lens), FreePages.of(ids))
                stage.prefill_prune(k, v, p.cu_seqlens, max(lens))
                stage.set_host_lens([n if a == 1 else 0 for n, a in zip(lens, was)])   # (the third fits there, but not here)
                c.take(stage)
            else:
                c.prefill_prune(k, v, plan.cu_seqlens, max(lens))
            c.set_host_lens([n if a == 1 else None for n, a in zip(lens, was)])
            lens_now = c.seq_lens.tolist()
            assert all(c.host_lens[s] == lens_now[s] for s in range(S)), (half, lens_now, c.host_lens)
            for nk, nv, q in steps[half * n_steps:(half + 1) * n_steps]:
                o = torch.empty_like(q)
                c.decode_step(nk, nv, q, o)
                assert c.seq_lens.tolist() == c.host_lens
                out.append(o.view(S, -1))
            # the places without a sequence have had the steps' tokens, for which they have no page: empty again
            for s in range(S):
                if s not in first + second or (s in second and half == 0) or was[s] == 0 and s not in first:
                    c.seq_lens[s] = 0
                    c.block_table[s] = -1
                    c.set_host_lens([0 if i == s else None for i in range(S)])
        return out

    both = life([0], [1, 2], 2 * need)          # the list does not hold the third
    alone = life([0], [], 8 * need), life([], [1], 8 * need)
    for i, o in enumerate(both):
        assert torch.equal(o[0], alone[0][i][0]), i
        assert i < n_steps or torch.equal(o[1], alone[1][i][1]), i


@pytest.mark.parametrize("dt,B", [(torch.bfloat16, 16), (torch.float32, 128)])
@pytest.mark.parametrize("shared", [False, True])
def test_pages_of_admitted_sequences_only(dt, B, shared):
    """pe_quant_pages_admitted: what it writes is what pe_quant_pages does, and of the other sequences nothing."""
    lens, width = [2 * B + 3, 3 * B, 5, B], 3
    rows, heads = (1, (Hk,)) if shared else (Hk, ())
    P = len(lens) * rows * width
    g = torch.Generator().manual_seed(4)
    desc = pe.make_desc(dt, len(lens), Hk, Hk, D, B, width, P, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    kp, vp = (torch.randn((P, B) + heads + (D,), generator=g).to(dt).to(DEV) for _ in range(2))
    table = torch.randperm(P, generator=g).int().view((len(lens),) + (() if shared else (Hk,)) + (width,)).to(DEV)

    def run(mask):
        k, v = (torch.full((P, B) + heads + (D,), 9, dtype=torch.uint8, device=DEV) for _ in range(2))
        scales = torch.full((P,) + heads + (2,), 9.0, device=DEV)
        tails = [torch.full((len(lens), Hk, B, D), 9.0, dtype=dt, device=DEV) for _ in range(2)]
        scores = torch.full((len(lens), Hk, width), 9.0, device=DEV)
        pe.pe_quant_pages(desc, pe.make_quant_cache(desc, k, v, scales, *tails), kp, vp, table, _i32(lens), table, scores,
                          None if mask is None else _i32(mask))
        torch.cuda.synchronize()
        return (k, v, scales), tails + [scores]

    whole = run(None)
    for mask in ([1, 0, 2, 0], [0, 1, 0, 1], [0] * 4, [1] * 4):
        got = run(mask)
        for s, m in enumerate(mask):
            pages = table[s].flatten().long()
            for a, b in zip(got[0], whole[0]):
                assert torch.equal(a[pages], b[pages]) if m else bool((a[pages] == 9).all()), (mask, s)
            for a, b in zip(got[1], whole[1]):
                assert torch.equal(a[s], b[s]) if m else bool((a[s] == 9).all()), (mask, s)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("shared", [False, True])
def test_replayed_steps_between_admissions(shared, quant):
    """Sequences end and others begin between the steps of a stepper: every replay against the eager step of a model of its own."""
    layers, width, n_spare = 2, 4, 4
    rows = 1 if shared else Hk
    P = layers * S * rows * (width + n_spare)
    made, frees = [], []
    for _ in range(2):
        m = (LayeredQuantCache if quant else LayeredCache)(torch.bfloat16, layers, S, Hk, Hk * G, D, B, empty_layout(layers * S, Hk, width, n_spare, P, DEV, shared),
                                                           BUDGET, shared=shared)
        assert m.end(range(S)).numel() == 0
        made.append(m)
        frees.append(FreePages.of(torch.randperm(P, generator=torch.Generator().manual_seed(7)).int().to(DEV)))
    bufs = [torch.zeros((layers, S, h, D), dtype=torch.bfloat16, device=DEV) for h in (Hk, Hk, Hk * G, Hk * G)]
    out = torch.zeros_like(bufs[3])
    stepper = GraphedStepper(made[0], *bufs)
    comes = {0: [90, 0, 30], 25: [0, 64, 0], 45: [20, 0, 0], 60: [0, 0, 130]}
    ends = {40: [0], 58: [2], 70: [1]}
    for step in range(90):
        if step in comes:
            lens = comes[step]
            kv = [[_randn(torch.Generator().manual_seed(100 * step + 10 * l + i), sum(lens), Hk, D) for i in range(2)] for l in range(layers)]
            for i, m in enumerate(made):
                plans = m.admit(_i32(lens), sum(lens), frees[i])
                assert plans[0].admitted.tolist() == [int(n > 0) for n in lens]
                for l in range(layers):
                    if quant:
                        stage = PagedCache.create(torch.bfloat16, S, Hk, Hk * G, D, B, empty_layout(S, Hk, width, 1, 99, DEV, shared), BUDGET, shared=shared)
                        p = stage.admit(_i32(lens), sum(lens), FreePages.of(torch.arange(99, dtype=torch.int32, device=DEV)))
                        stage.prefill_prune(*kv[l], p.cu_seqlens, max(lens))
                        stage.set_host_lens(lens)
                        m.take_layer(l, stage)
                    else:
                        m.prefill_prune_layer(l, *kv[l], plans[l].cu_seqlens, max(lens))
                m.set_host_lens([n or None for n in lens])
        g = torch.Generator().manual_seed(step)
        for t in bufs[:3]:
            t.copy_(torch.randn(t.shape, generator=g))
        assert stepper.step() == made[1].decode_step(bufs[0], bufs[1], bufs[2], out)
        torch.cuda.synchronize()
        live = [s for s, n in enumerate(made[1].host_lens) if n >= 0]
        assert torch.equal(bufs[3][:, live], out[:, live]), step
        a, b = made[0].folded, made[1].folded
        assert made[0].host_lens == made[1].host_lens and a.seq_lens.tolist() == b.seq_lens.tolist() == made[1].host_lens * layers, step
        assert torch.equal(a.block_table, b.block_table) and torch.equal(a.spare_used, b.spare_used)
        if step in ends:
            for i, m in enumerate(made):
                frees[i] = FreePages.of(torch.cat((frees[i].pages[int(frees[i].used):], m.end(ends[step]))))
    assert len(stepper.graphs) <= 4
