"""The plan of a batch's tokens (pe_plan_tokens) against a plain one, sequence by sequence: whole numbers, equal or wrong."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _tokens64 import plan

pytestmark = pytest.mark.gpu
DEV = "cuda"
JUNK = -77


def _i32(x):
    return torch.tensor(x, dtype=torch.int32)


def _run(lens, new, Hk, B, shared=False, budget=0, n_spare=0, short=None, first=None, pad=0, used=3, extra_blocks=1, seed=0, clip=0, total=None,
         max_blocks=None, dtype=torch.bfloat16, graph=False):
    g = torch.Generator().manual_seed(seed)
    S, rows = len(lens), 1 if shared else Hk
    kept = [max(n, min(n + max(m, 0), budget)) if budget else n + max(m, 0) for n, m in zip(lens, new)]
    width = max(1, max(-(-k // B) for k in kept) + extra_blocks) if max_blocks is None else max_blocks
    have = [min(width, -(-n // B)) for n in lens]
    pages = sum(have) * rows
    ids = torch.randperm(pages + 400 * rows * S, generator=g).int()
    table = torch.full((S, rows, width), -1, dtype=torch.int32)
    at = 0
    for s in range(S):
        for h in range(rows):
            table[s, h, :have[s]] = ids[at:at + have[s]]
            at += have[s]
    need = sum((-(-k // B) - -(-n // B) + (n_spare if n == 0 and m > 0 else 0)) * rows for k, n, m in zip(kept, lens, new))
    free = ids[at:at + max(1, used + need + (5 if short is None else -short))]
    spare = torch.full((S, rows, max(1, n_spare)), JUNK, dtype=torch.int32)
    tokens = sum(max(m, 0) for m in new)
    total = max(0, tokens + pad - clip) if total is None else total
    t, sp = table.tolist(), spare.tolist()
    want = plan(lens, new, first, total, budget, free.tolist(), used, t, sp, n_spare, B)

    desc = pe.make_desc(dtype, S, Hk, Hk, 64, B, width, 1 << 20, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    shape = (lambda x: x[:, 0].contiguous()) if shared else (lambda x: x)
    dt, ds = shape(table).to(DEV), shape(spare).to(DEV)
    lens_out, used_out, cu = (torch.full((n,), JUNK, dtype=torch.int32, device=DEV) for n in (S, 1, S + 1))
    pos = torch.full((total + 1,), JUNK, dtype=torch.int32, device=DEV)
    slots = torch.full((total + 1,) + (() if shared else (rows,)), JUNK, dtype=torch.int64, device=DEV)
    args = [_i32(lens).to(DEV), _i32(new).to(DEV), None if first is None else _i32(first).to(DEV), total, budget, free.to(DEV), _i32([used]).to(DEV),
            dt, ds if n_spare else None, lens_out, used_out, cu, pos, slots]
    pe.pe_plan_tokens(desc, *args)
    torch.cuda.synchronize()
    got = [lens_out.tolist(), int(used_out), cu.tolist(), pos[:total].tolist(), slots[:total].view(total, rows).tolist()]
    assert got == list(want)
    assert int(pos[total]) == JUNK and slots[total].flatten().tolist() == [JUNK] * rows   # nothing behind the room given
    assert dt.view(S, rows, width).tolist() == t
    assert ds.view(S, rows, -1).tolist() == sp
    return want


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("B", [16, 32, 64, 128])
def test_prompts(B, shared):
    _run([0] * 7, [1, B, B - 1, 0, B + 1, 3 * B, 517], 3, B, shared)


@pytest.mark.parametrize("shared", [False, True])
def test_one_token_each(shared):
    _run([15, 16, 17, 0, 31, 32, 160], [1] * 7, 4, 16, shared)


def test_chunks_behind_what_is_there_and_positions_that_ran_ahead():
    _run([5, 0, 47, 48, 100], [40, 3, 1, 16, 0], 2, 16, first=[1000, 0, 70000, 2 ** 31 - 16, 7])


@pytest.mark.parametrize("n_spare", [1, 3])
@pytest.mark.parametrize("shared", [False, True])
def test_spare_pages_for_sequences_that_begin(n_spare, shared):
    _run([0, 7, 0, 0, 64], [33, 2, 0, 16, 1], 3, 16, shared, n_spare=n_spare)


@pytest.mark.parametrize("shared", [False, True])
def test_a_budget_leaves_slots_to_the_prune(shared):
    _run([0, 0, 0, 48, 80], [200, 64, 63, 30, 5], 2, 16, shared, budget=64, n_spare=1)


@pytest.mark.parametrize("short", [1, 2, 9, 30])
def test_too_few_free_pages(short):
    """The first sequence that the list does not hold, and every later one that needs pages, are left; one that needs none is served."""
    _run([0, 0, 20, 30, 0, 0], [40, 100, 2, 1, 17, 50], 2, 16, short=short, n_spare=1)


def test_rows_that_are_too_short():
    _run([0, 0, 30], [200, 33, 50], 2, 16, max_blocks=4)


def test_an_empty_list():
    _run([10, 0], [3, 4], 2, 16, used=50, short=53)
    _run([10, 0], [3, 4], 2, 16, used=-5)


def test_padding_and_too_little_room():
    _run([0, 9], [20, 30], 2, 16, pad=301)
    _run([0, 9], [20, 30], 2, 16, clip=27)
    _run([0, 9], [0, 0], 2, 16)
    _run([0, 9], [-4, 30], 2, 16)


@pytest.mark.parametrize("S", [255, 256, 257, 700])
def test_many_sequences(S):
    """More than a workgroup sums at a time."""
    g = torch.Generator().manual_seed(S)
    lens = torch.randint(0, 60, (S,), generator=g).tolist()
    new = torch.randint(-1, 40, (S,), generator=g).tolist()
    _run(lens, new, 2, 16, n_spare=1, seed=S)
    _run(lens, new, 2, 16, short=300, seed=S)


def test_many_tokens():
    _run([0, 3, 0], [5000, 20001, 7777], 5, 16, extra_blocks=3)


@pytest.mark.parametrize("Hk", [1, 7, 8, 63, 4095, 4096, 5003])
def test_many_heads(Hk):
    _run([0, 3, 16], [20, 1, 17], Hk, 16)


def test_missing_pages_give_no_slot():
    """A row of a sequence that goes on without its page."""
    lens, new, B, width = _i32([20]), _i32([3]), 16, 3
    table = torch.tensor([[[7, -1, -1], [8, 9, -1]]], dtype=torch.int32, device=DEV)
    desc = pe.make_desc(torch.bfloat16, 1, 2, 2, 64, B, width, 64)
    out = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (1, 1, 2, 3)]
    slots = torch.zeros((3, 2), dtype=torch.int64, device=DEV)
    pe.pe_plan_tokens(desc, lens.to(DEV), new.to(DEV), None, 3, 0, _i32([1, 2]).to(DEV), _i32([0]).to(DEV), table, None, *out, slots)
    assert slots.tolist() == [[-1, 9 * B + 4 + i] for i in range(3)] and out[0].tolist() == [23] and out[1].tolist() == [0]


def test_outputs_that_are_not_asked_for():
    B = 16
    table = torch.full((2, 2, 4), -1, dtype=torch.int32, device=DEV)
    desc = pe.make_desc(torch.bfloat16, 2, 2, 2, 64, B, 4, 64)
    lens_out, used = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    pe.pe_plan_tokens(desc, _i32([0, 0]).to(DEV), _i32([17, 1]).to(DEV), None, 0, 0, torch.arange(9, dtype=torch.int32, device=DEV),
                      _i32([1]).to(DEV), table, None, lens_out, used, None, None, None)
    assert table.tolist() == [[[1, 2, -1, -1], [3, 4, -1, -1]], [[5, -1, -1, -1], [6, -1, -1, -1]]]
    assert lens_out.tolist() == [17, 1] and used.tolist() == [7]


def test_slots_beyond_32_bits():
    B = 128
    table = torch.full((1, 1, 2), -1, dtype=torch.int32, device=DEV)
    desc = pe.make_desc(torch.bfloat16, 1, 1, 1, 64, B, 2, 2 ** 31 - 1)
    out = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (1, 1, 2, 2)]
    slots = torch.zeros((2, 1), dtype=torch.int64, device=DEV)
    pe.pe_plan_tokens(desc, _i32([0]).to(DEV), _i32([2]).to(DEV), None, 2, 0, _i32([2 ** 31 - 2]).to(DEV), _i32([0]).to(DEV), table, None, *out, slots)
    assert slots.tolist() == [[(2 ** 31 - 2) * B], [(2 ** 31 - 2) * B + 1]]


def test_replayed_with_other_lengths():
    """One graph for every step: lengths, and with them what is dealt, change between replays."""
    S, Hk, B, width, total = 3, 2, 16, 8, 12
    desc = pe.make_desc(torch.bfloat16, S, Hk, Hk, 64, B, width, 4096)
    free = torch.randperm(600, generator=torch.Generator().manual_seed(1)).int()
    lens, new, used = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (S, S, 1))
    table = torch.full((S, Hk, width), -1, dtype=torch.int32, device=DEV)
    lens_out, used_out, cu, pos = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (S, 1, S + 1, total))
    slots = torch.zeros((total, Hk), dtype=torch.int64, device=DEV)
    call = lambda: pe.pe_plan_tokens(desc, lens, new, None, total, 0, free_d, used, table, None, lens_out, used_out, cu, pos, slots)   # noqa: E731
    free_d = free.to(DEV)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    t, at, have = [[[-1] * width for _ in range(Hk)] for _ in range(S)], 0, [0] * S
    for step, add in enumerate(([3, 4, 5], [1, 1, 1], [0, 9, 3], [1, 0, 0], [4, 4, 4])):
        new.copy_(_i32(add))
        graph.replay()
        torch.cuda.synchronize()
        want = plan(have, add, None, total, 0, free.tolist(), at, t, None, 0, B)
        assert [lens_out.tolist(), int(used_out), cu.tolist(), pos.tolist(), slots.tolist()] == list(want), step
        assert table.tolist() == t
        have, at = want[0], want[1]
        lens.copy_(lens_out)
        used.copy_(used_out)
