"""The new calls as a program runs them together: prompts planned on the device, turned, pruned or stored whole, rounded, and decoded over
evictions, beside the unrounded cache that takes the same decisions."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd.engine import FreePages, GraphedStepper, LayeredCache, LayeredQuantCache, PagedCache, QuantCache, empty_layout

from _paged64 import DTYPES, assert_close
from _paged64 import attend as attend_unrounded
from _quant64 import E4M3, attend
from _tokens64 import frequencies, rotate

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _held(c, s, h, n):
    """What the first n tokens of a row stand for, in float64."""
    B = c.desc.block_size
    shared = c.desc.layout == pe.PE_LAYOUT_SHARED
    page = (c.block_table[s] if shared else c.block_table[s, h])[:n // B].long()
    rows = []
    for i, (pool, tail) in enumerate(((c.k, c.k_tail), (c.v, c.v_tail))):
        x = pool.view(torch.uint8)[page]
        x = (x[:, :, h] if shared else x).view(E4M3).to(torch.float32).double()
        scale = (c.scales[page, h, i] if shared else c.scales[page, i]).double()
        rows.append(torch.cat(((x * scale[:, None, None]).flatten(0, 1), tail[s, h, :n % B].double())).cpu())
    return rows


def _check(c, q, out, lens):
    G = c.desc.num_q_heads // c.desc.num_kv_heads
    for s, n in enumerate(lens):
        for h in range(c.desc.num_kv_heads):
            k, v = _held(c, s, h, n)
            want, bound = attend(q[s, h * G:(h + 1) * G].double().cpu(), k, v, q.dtype)
            assert_close(out[s, h * G:(h + 1) * G], want, bound, q.dtype)


@pytest.mark.parametrize("roped", [False, True])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt,D,B,opts", [("bf16", 64, 16, None), ("bf16", 128, 32, None), ("f32", 64, 16, None),
                                         ("bf16", 64, 16, (pe.PE_POLICY_LOWEST_SCORE, 1, 1)), ("bf16", 64, 16, (pe.PE_POLICY_OLDEST, 0, 0))])
def test_prompts_then_steps_over_evictions(dt, D, B, opts, shared, roped):
    dtype, S, Hk, G, budget, lens = DTYPES[dt], 4, 2, 3, 4 * B, [9 * B + 5, 4 * B, B - 1, 2 * B + 3]
    g = torch.Generator().manual_seed(D + B)
    width, n_spare = budget // B, budget // B
    P = S * (1 if shared else Hk) * (width + n_spare)
    free = torch.randperm(P, generator=g).int()
    layout = lambda: empty_layout(S, Hk, width, n_spare, P, DEV, shared)   # noqa: E731
    rope, f = (pe.make_rope(D, 10000.0), frequencies(D, 10000.0)) if roped else (None, None)
    quant = QuantCache.create(dtype, S, Hk, Hk * G, D, B, layout(), budget, shared=shared, rope=rope)
    plain = PagedCache.create(dtype, S, Hk, Hk * G, D, B, layout(), budget, shared=shared)
    plain.cached_scores = opts is None
    if opts:
        quant.evict_opts = plain.evict_opts = pe.pe_evict_opts(opts[0], opts[1], opts[2], 0, 0)
    total = sum(lens)
    plans = [c.admit(_i32(lens), total, FreePages.of(free.to(DEV))) for c in (quant, plain)]
    assert plans[0].cu_seqlens.tolist() == [sum(lens[:i]) for i in range(S + 1)] and torch.equal(quant.block_table, plain.block_table)
    q, k, v = (torch.randn((total, h, D), generator=g).to(dtype).to(DEV) for h in (Hk * G, Hk, Hk))
    if roped:
        raw = k.clone()
        plain.rotate(rope, plans[0].positions, q, k, q, k)
        assert_close(k, *rotate(raw.cpu(), plans[0].positions.cpu(), f, False), dtype)
    plain.prefill_prune(k, v, plans[0].cu_seqlens, max(lens))
    plain.set_host_lens(lens)
    quant.take(plain)
    assert quant.seq_lens.tolist() == plain.seq_lens.tolist() == quant.host_lens
    out, want = (torch.empty((S, Hk * G, D), dtype=dtype, device=DEV) for _ in range(2))
    gone = 0
    for step in range(3 * B + 2):
        nk, nv = (torch.randn((S, Hk, D), generator=g).to(dtype).to(DEV) for _ in range(2))
        nq = torch.randn((S, Hk * G, D), generator=g).to(dtype).to(DEV)
        if roped:
            quant.positions.copy_(_i32([n + step for n in lens]))
        gone += sum(quant.triggers())
        quant.decode_step(nk, nv, nq, out)
        if roped:   # what the cache got is what the unrounded one gets
            slot = (quant.seq_lens - 1).long() % B
            nk, nq = quant.k_tail[torch.arange(S, device=DEV), :, slot].contiguous(), quant.turned
        plain.decode_step(nk, nv, nq, want)
        assert torch.equal(quant.block_table, plain.block_table) and torch.equal(quant.seq_lens, plain.seq_lens), step
        assert quant.seq_lens.tolist() == quant.host_lens == plain.host_lens
        assert torch.equal(quant.evicted_logical, plain.evicted_logical)
        if step % 7 == 0 or step > 3 * B - 2:
            _check(quant, nq, out, quant.host_lens)
        assert bool(torch.isfinite(out).all()) and float((out - want).abs().max()) < 0.5 * float(want.abs().max())   # rounded to 3 bits behind the first
    assert gone > S


def _model(dt, D, shared, layers, S, Hk, G, B, budget, lens, seed, roped):
    g = torch.Generator().manual_seed(seed)
    dtype, width = DTYPES[dt], budget // B
    R, n_spare = layers * S, width
    P = R * (1 if shared else Hk) * (width + n_spare)
    rope = pe.make_rope(D, 10000.0, interleaved=True) if roped else None
    model = LayeredQuantCache(dtype, layers, S, Hk, Hk * G, D, B, empty_layout(R, Hk, width, n_spare, P, DEV, shared), budget, shared=shared, rope=rope)
    free = FreePages.of(torch.randperm(P, generator=g).int().to(DEV))
    plans = model.admit(_i32(lens), sum(lens), free)
    assert all(p.cu_seqlens.tolist()[-1] == sum(lens) for p in plans) and model.folded.seq_lens.tolist() == [min(n, budget) for n in lens] * layers
    used = model.folded.block_table[model.folded.block_table >= 0].tolist() + model.folded.spare.flatten().tolist()
    assert len(set(used)) == len(used) and int(free.used) == len(used)   # no page twice, in no layer
    # (one staging cache for a layer at a time)
    rows = 1 if shared else Hk
    stage = PagedCache.create(dtype, S, Hk, Hk * G, D, B, empty_layout(S, Hk, width, 1, S * rows * (width + 1), DEV, shared), budget, shared=shared)
    for l, c in enumerate(model.per_layer):
        stage.seq_lens.zero_()
        p = stage.admit(_i32(lens), sum(lens), FreePages.of(torch.arange(S * rows * (width + 1), dtype=torch.int32, device=DEV)))
        k, v = (torch.randn((sum(lens), Hk, D), generator=g).to(dtype).to(DEV) for _ in range(2))
        stage.prefill_prune(k, v, p.cu_seqlens, max(lens))
        stage.set_host_lens(lens)
        model.take_layer(l, stage)
    return model


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("roped", [False, True])
def test_replayed_steps_of_all_layers(shared, roped):
    """A graphed model beside an eager one, over evictions; the eager one's last layer against 64 bits."""
    layers, S, Hk, G, D, B, budget, lens = 2, 3, 2, 4, 64, 16, 64, [200, 50, 7]
    made = [_model("bf16", D, shared, layers, S, Hk, G, B, budget, lens, 3, roped) for _ in range(2)]
    bufs = [torch.zeros((layers, S, h, D), dtype=torch.bfloat16, device=DEV) for h in (Hk, Hk, Hk * G, Hk * G)]
    out = torch.zeros_like(bufs[3])
    stepper, g = GraphedStepper(made[0], *bufs), torch.Generator().manual_seed(9)
    for step in range(70):
        for t in bufs[:3]:
            t.copy_(torch.randn(t.shape, generator=g))
        if roped:
            for m in made:
                m.positions.copy_(_i32([n + step for n in lens]))
        assert stepper.step() == made[1].decode_step(bufs[0], bufs[1], bufs[2], out)
        torch.cuda.synchronize()
        assert torch.equal(bufs[3], out), step
        a, b = made[0].folded, made[1].folded
        for name in ("block_table", "seq_lens", "scores", "spare_used", "freed_phys", "k_tail"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (step, name)
        assert b.seq_lens.tolist() == made[1].host_lens * layers
        if step % 23 == 0:
            c = made[1].per_layer[-1]
            _check(c, c.turned if roped else bufs[2][-1], out[-1], made[1].host_lens)
    assert len(stepper.graphs) <= 4


def test_all_layers_of_an_unrounded_cache_are_admitted():
    """LayeredCache: pages from one list, then a prune and steps, beside a cache whose layout came from the host."""
    layers, S, Hk, Hq, D, B, budget, lens = 2, 3, 2, 4, 64, 16, 64, [100, 64, 9]
    R, width, n_spare = layers * S, budget // B, budget // B
    P = R * Hk * (width + n_spare)
    g = torch.Generator().manual_seed(1)
    ids = torch.randperm(P, generator=g).int()
    one = LayeredCache(torch.float32, layers, S, Hk, Hq, D, B, empty_layout(R, Hk, width, n_spare, P, DEV), budget)
    one.admit(_i32(lens), sum(lens), FreePages.of(ids.to(DEV)))
    layout = empty_layout(R, Hk, width, n_spare, P, "cpu")
    at = 0
    for r in range(R):   # the same deal, on the host
        need = -(-min(lens[r % S], budget) // B)
        for h in range(Hk):
            layout.block_table[r, h, :need] = ids[at:at + need]
            layout.spare[r, h] = ids[at + need:at + need + n_spare]
            at += need + n_spare
    two = LayeredCache(torch.float32, layers, S, Hk, Hq, D, B, layout, budget)
    assert torch.equal(one.folded.block_table, two.folded.block_table) and torch.equal(one.folded.spare, two.folded.spare)
    cu = _i32([sum(lens[:i]) for i in range(S + 1)])
    for l in range(layers):
        k, v = (torch.randn((sum(lens), Hk, D), generator=g).to(DEV) for _ in range(2))
        for m in (one, two):
            m.prefill_prune_layer(l, k, v, cu, max(lens))
    for m in (one, two):
        m.set_host_lens(lens)
    for step in range(40):
        nk, nv = (torch.randn((layers, S, Hk, D), generator=g).to(DEV) for _ in range(2))
        q = torch.randn((layers, S, Hq, D), generator=g).to(DEV)
        outs = [torch.empty_like(q) for _ in range(2)]
        for m, out in zip((one, two), outs):
            m.decode_step(nk, nv, q, out)
        assert torch.equal(*outs) and torch.equal(one.folded.block_table, two.folded.block_table), step


@pytest.mark.parametrize("dt,shared", [("bf16", False), ("f32", True)])
def test_prompts_kept_whole_in_chunks(dt, shared):
    """Chunks of prompts planned, turned and stored into the pages, then attention over them; a sequence that the list does not hold stays out."""
    dtype, S, Hk, G, D, B = DTYPES[dt], 3, 2, 2, 64, 16
    g = torch.Generator().manual_seed(5)
    width, P = 8, 64
    cache = PagedCache.create(dtype, S, Hk, Hk * G, D, B, empty_layout(S, Hk, width, 1, P, DEV, shared), width * B, shared=shared)
    free = FreePages.of(torch.randperm(P, generator=g).int().to(DEV))
    rope, f = pe.make_rope(48, 10000.0), frequencies(48, 10000.0)
    keys, values = ([[] for _ in range(S)] for _ in range(2))
    lens = [0] * S
    for new in ([37, 5, 0], [1, 60, 16], [30, 1, 1], [0, 3, 500]):
        total = sum(new) + 9                                       # a padded batch
        plan = cache.admit(_i32(new), total, free, whole=True)
        q, k, v = (torch.randn((total, h, D), generator=g).to(dtype) for h in (Hk * G, Hk, Hk))
        qo = torch.empty_like(q, device=DEV)
        cache.rotate_store(rope, plan, q.to(DEV), k.to(DEV), v.to(DEV), qo)
        y, _ = rotate(k, plan.positions.cpu(), f, False)
        at = 0
        for s, n in enumerate(new):
            if n < 500:                                            # (does not fit its table row)
                keys[s].append(y[at:at + n].to(dtype))
                values[s].append(v[at:at + n])
                lens[s] += n
            at += n
        assert cache.seq_lens.tolist() == lens
    q = torch.randn((S, Hk * G, D), generator=g).to(dtype)
    out = torch.empty_like(q, device=DEV)
    cache.paged_decode(q.to(DEV), out)
    for s in range(S):
        k, v = torch.cat(keys[s]).double(), torch.cat(values[s]).double()
        for h in range(Hk):
            qs = q[s, h * G:(h + 1) * G].double()
            want, w, bound = attend_unrounded(qs, k[:, h], v[:, h])
            # the stored keys are the rotation's, rounded: at most a step from the reference's rounding of it, each (its error can turn a tie)
            step = torch.finfo(dtype).eps * 1.01
            off = 2 * (qs.abs() @ k[:, h].abs().T * D ** -0.5).amax(1, keepdim=True) * step
            assert_close(out[s, h * G:(h + 1) * G], want, bound + off * (w @ v[:, h].abs()), dtype)
