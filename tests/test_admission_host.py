"""The host's part of admissions: its mirror of the lengths behind prompts that are pruned or kept whole, beside sequences that run on
(no GPU: the launches are off)."""
import pytest
import torch

from paper_2509_04377_amd.engine import FreePages, LayeredCache, LayeredQuantCache, PagedCache, QuantCache, empty_layout, host_only

S, Hk, Hq, D, B, BUDGET, WIDTH = 3, 2, 4, 64, 16, 64, 12


@pytest.fixture(autouse=True)
def no_gpu_memory(monkeypatch):
    """Workspaces and tensors on the CPU, whose addresses no call will see."""
    from paper_2509_04377_amd import binding as pe
    monkeypatch.setattr(pe, "_addr", lambda t, name, dtype=None: t.data_ptr())
    monkeypatch.setattr(pe, "alloc_workspace", lambda *a, **kw: torch.empty(0))


def _make(kind, num_seqs=S):
    cls = dict(paged=PagedCache, quant=QuantCache, layers=LayeredCache, quant_layers=LayeredQuantCache)[kind]
    layers = (2,) if "layers" in kind else ()
    rows = num_seqs * (layers[0] if layers else 1)
    args = (torch.float32,) + layers + (num_seqs, Hk, Hq, D, B, empty_layout(rows, Hk, WIDTH, 2, 64, "cpu"), BUDGET)
    return cls(*args, device="cpu") if layers else cls.create(*args, device="cpu")


KINDS = ["paged", "quant", "layers", "quant_layers"]


def _mirrors(c):
    return [c.host_lens] + ([c.folded.host_lens[i:i + S] for i in (0, S)] if hasattr(c, "folded") else [])


@pytest.mark.parametrize("kind", KINDS)
def test_lengths_that_are_told(kind):
    c = _make(kind)
    for lens, whole, want in (([100, 64, 3], False, [64, 64, 3]), ([100, None, 0], True, [100, 64, 0]), ([None, 70, None], False, [100, 64, 0]),
                              ([None, 0, None], True, [100, 0, 0])):
        c.set_host_lens(lens, whole)
        assert all(m == want for m in _mirrors(c)), (lens, whole)
    for lens in ([1, 2], [1, 2, 3, 4]):
        with pytest.raises(ValueError, match="one length per sequence"):
            c.set_host_lens(lens)
    assert c.host_lens == [100, 0, 0]


@pytest.mark.parametrize("kind", KINDS)
def test_steps_go_on_from_what_was_told(kind):
    """A prompt kept whole beyond the budget loses a page where it has filled one, as the device counts."""
    c = _make(kind)
    c.set_host_lens([100, 64, 3], whole=True)
    want = [100, 64, 3]
    shape = (2, S) if "layers" in kind else (S,)
    new, q = torch.zeros(shape + (Hk, D)), torch.zeros(shape + (Hq, D))
    with host_only():
        for step in range(40):
            want = [n - B if n > 0 and n % B == 0 and n >= BUDGET else n for n in want]
            c.decode_step(new, new, q, torch.zeros_like(q))
            want = [n + 1 for n in want]
            if step == 20:
                c.set_host_lens([None, 7, None])
                want[1] = 7
            assert c.host_lens == want, step


@pytest.mark.parametrize("kind", ["paged", "layers"])
def test_what_was_counted_of_a_place_is_forgotten(kind):
    c = _make(kind)
    f = c.folded if kind == "layers" else c
    f.host_scored = [4] * f.desc.num_seqs
    c.set_host_lens([None, 9, None])
    assert f.host_scored is None   # (the pages that a cached score is of are another sequence's)


@pytest.mark.parametrize("kind", ["paged", "layers"])
def test_attention_stays_with_sequences_that_run_on(kind):
    c = _make(kind)
    c.evict_by_attention()
    caches = [c.folded] + c.per_layer if kind == "layers" else [c]
    for x in caches:
        x.attention.started = True
        x.scores.fill_(2.0)
    c.set_host_lens([None, 9, None])
    for x in caches:
        rows = x.scores.view(-1, S, Hk, WIDTH)
        assert x.attention.started and bool((rows[:, [0, 2]] == 2.0).all()) and bool(torch.isinf(rows[:, 1]).all())
    c.set_host_lens([5, 9, 1])
    assert not any(x.attention.started for x in caches)


@pytest.mark.parametrize("kind", KINDS)
def test_a_part_of_a_cache_admits_nobody(kind):
    """Its new lengths would lie in an array that the cache does not read."""
    c = _make(kind)
    f = c.folded if "layers" in kind else c
    free = FreePages.of(torch.arange(8, dtype=torch.int32))
    before = f.seq_lens.data_ptr()
    for part in [f.rows(0, 2)] + (c.per_layer if "layers" in kind else []):
        with pytest.raises(ValueError, match="the whole cache's"):
            part.admit(torch.ones(part.desc.num_seqs, dtype=torch.int32), 2, free)
    with host_only():
        c.admit(torch.ones(S, dtype=torch.int32), S, free)
    assert f.seq_lens.data_ptr() != before
    for l, part in enumerate(c.per_layer if "layers" in kind else []):
        assert part.seq_lens.data_ptr() == f.seq_lens[l * S:].data_ptr() and part.seq_lens_alt.data_ptr() == f.seq_lens_alt[l * S:].data_ptr()


class _Took(Exception):
    pass


def _plan_room(**small):
    """pe_plan_tokens on tensors of the right sizes, but for those that lack one number."""
    from paper_2509_04377_amd import binding as pe
    T, R = 7, S * Hk
    need = dict(seq_lens=S, new_lens=S, first_positions=S, free_pages=9, free_used=1, block_table=R * WIDTH, spare=R * 2, seq_lens_out=S,
                free_used_out=1, cu_seqlens_out=S + 1, positions_out=T, slots_out=T * Hk, admitted=S, spare_used=R, freed_phys=R, only=S)
    t = {name: torch.zeros(n - small.get(name, 0), dtype=torch.int64 if name == "slots_out" else torch.int32) for name, n in need.items()}
    t["spare"] = t["spare"].view(-1, 2) if "spare" not in small else torch.zeros((R - 1, 2), dtype=torch.int32)
    desc = pe.make_desc(torch.float32, S, Hk, Hq, D, B, WIDTH, 64)
    pe.pe_plan_tokens(desc, *(t[n] for n in ("seq_lens", "new_lens", "first_positions")), T, 0, *(t[n] for n in (
        "free_pages", "free_used", "block_table", "spare", "seq_lens_out", "free_used_out", "cu_seqlens_out", "positions_out", "slots_out",
        "admitted", "spare_used", "freed_phys", "only")))


@pytest.mark.parametrize("name", ["seq_lens", "new_lens", "first_positions", "free_used", "block_table", "spare", "seq_lens_out", "free_used_out",
                                  "cu_seqlens_out", "positions_out", "slots_out", "admitted", "spare_used", "freed_phys", "only"])
def test_a_plan_needs_room_for_its_tokens(name, monkeypatch):
    """Nothing is launched that would write (or read) behind a tensor's end."""
    from paper_2509_04377_amd import binding as pe

    class _Library:
        addr_plan_tokens_ex = 1

        def pe_plan_tokens_ex(self, *args):
            raise _Took

    library = _Library()
    monkeypatch.setattr(pe, "lib", lambda: library)
    monkeypatch.setattr(pe, "_host", pe._NoHost())
    monkeypatch.setattr(pe, "_stream", lambda: None)
    with pytest.raises(_Took):      # all are large enough
        _plan_room()
    with pytest.raises(ValueError, match=name + " must have room for"):
        _plan_room(**{name: 1})


@pytest.mark.parametrize("kind", ["paged", "quant"])
def test_a_plan_to_write_into_that_is_too_small(kind, monkeypatch):
    from paper_2509_04377_amd import binding as pe
    c = _make(kind)
    free = FreePages.of(torch.arange(8, dtype=torch.int32))
    monkeypatch.setattr(pe, "_stream", lambda: None)
    new = torch.ones(S, dtype=torch.int32)
    plan = c.new_plan(5)
    before = c.seq_lens, free.used
    with pytest.raises(ValueError, match="positions_out must have room for 6"):
        c.admit(new, 6, free, plan=plan)
    assert c.seq_lens is before[0] and free.used is before[1] and c.admitted is None   # as it was


@pytest.mark.parametrize("quant", ["quant", "quant_layers"])
def test_only_caches_of_one_shape_are_taken(quant):
    """Another width or number of sequences would have the other cache's table read behind its rows, other types and pages its pools."""
    to = _make(quant)
    take = (lambda c: to.take_layer(1, c)) if quant == "quant_layers" else to.take
    made = dict(dtype=torch.float32, num_seqs=S, num_kv_heads=Hk, num_q_heads=Hq, head_dim=D, block_size=B, width=WIDTH, shared=False)
    for what, change in (("dtype", dict(dtype=torch.bfloat16)), ("num_seqs", dict(num_seqs=2)), ("num_kv_heads", dict(num_kv_heads=4)),
                         ("head_dim", dict(head_dim=128)), ("block_size", dict(block_size=32)), ("max_blocks", dict(width=WIDTH - 1)),
                         ("max_blocks", dict(width=WIDTH + 1)), ("layout", dict(shared=True)), (None, dict(num_q_heads=8))):
        a = dict(made, **change)
        layout = empty_layout(a["num_seqs"], a["num_kv_heads"], a["width"], 1, 64, "cpu", a["shared"])
        c = PagedCache.create(a["dtype"], a["num_seqs"], a["num_kv_heads"], a["num_q_heads"], a["head_dim"], a["block_size"], layout, BUDGET, device="cpu",
                              shared=a["shared"])
        with host_only():
            if what is None:
                take(c)
            else:
                with pytest.raises(ValueError, match="another shape: " + what):
                    take(c)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("kind", KINDS)
def test_sequences_that_end(kind, shared):
    """Their pages come back once, their places are as if nobody had been there, and the mirror leaves them out of steps."""
    cls = dict(paged=PagedCache, quant=QuantCache, layers=LayeredCache, quant_layers=LayeredQuantCache)[kind]
    n, rows, spares = 2 if "layers" in kind else 1, 1 if shared else Hk, 3
    args = (Hk, Hq, D, B, empty_layout(n * S, Hk, WIDTH, spares, 999, "cpu", shared), BUDGET)
    c = cls(torch.float32, n, S, *args, device="cpu", shared=shared) if n > 1 else cls.create(torch.float32, S, *args, device="cpu", shared=shared)
    f = c.folded if n > 1 else c
    ids = torch.arange(n * S * rows * (WIDTH + spares), dtype=torch.int32).view(n, S, rows, WIDTH + spares)
    f.block_table.view(n, S, rows, WIDTH)[:] = ids[..., :WIDTH]     # (behind the length too: what is left there of earlier ones)
    f.spare.view(n, S, rows, spares)[:] = ids[..., WIDTH:]
    f.spare_used.view(n, S, rows)[:] = torch.tensor([0, 2, 3])[:, None]
    f.seq_lens.view(n, S)[:] = torch.tensor([33, 64, 5])
    f.freed_phys.view(n, S, rows)[:, 1, 0] = 900
    c.set_host_lens([33, 64, 5])
    before = [t.clone() for t in (f.block_table, f.spare, f.spare_used, f.seq_lens, f.freed_phys)]
    got = c.end(iter([1, 2, 1]))
    want = [x for l in range(n) for s, held, used in ((1, 4, 2), (2, 1, 3)) for h in range(rows)
            for x in ids[l, s, h, :held].tolist() + ids[l, s, h, WIDTH + used:].tolist()] + [900] * n
    assert sorted(got.tolist()) == sorted(want) and got.dtype == torch.int32
    assert c.host_lens == [33, -1, -1]
    for t, was, nothing in zip((f.block_table, f.spare, f.spare_used, f.seq_lens, f.freed_phys), before, (-1, -1, 0, -1, -1)):
        t, was = t.view((n, S) + t.shape[1:]), was.view((n, S) + t.shape[1:])
        assert torch.equal(t[:, 0], was[:, 0]) and bool((t[:, 1:] == nothing).all())
    assert c.end([2]).numel() == 0
    lead = (n, S) if n > 1 else (S,)
    new, q = torch.zeros(lead + (Hk, D)), torch.zeros(lead + (Hq, D))
    with host_only():
        for step in range(40):
            c.decode_step(new, new, q, torch.zeros_like(q))
    assert c.host_lens == [_stepped(33, 40), -1, -1]
    for bad in ([3], [-1], [0, 7]):
        with pytest.raises(ValueError, match="places are 0 to 2"):
            c.end(bad)
    with pytest.raises(ValueError, match="the whole cache's"):
        f.rows(0, 2).end([0])


def _stepped(n, steps):
    for _ in range(steps):
        n += 1 - (B if n % B == 0 and n >= BUDGET else 0)
    return n


def test_no_path_where_there_is_no_sequence():
    c = _make("paged")
    c.end([1])
    drafts = torch.zeros((S, 4, Hk, D))
    path, lens = torch.zeros((S, 4), dtype=torch.int32), torch.tensor([1, 1, 0], dtype=torch.int32)
    with host_only():
        with pytest.raises(ValueError, match="no sequence"):
            c.accept_path(drafts, drafts, path, lens, [1, 1, 0])
        c.accept_path(drafts, drafts, path, lens, [3, 0, 2])
    assert c.host_lens == [3, -1, 2]
