"""The prune behind a plan that did not serve everyone: rows without their pages, and sequences that are not the prune's to write."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd.engine import FreePages, PagedCache, empty_layout

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
JUNK = -7.0
# by the rule for launches: selection and copy in one launch; in two
LENS = {"one": [300, 70, 1, 129], "two": [33000, 70, 1, 129]}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class _Prompts:
    """Prompts, and pools with a page of guard in front and behind."""

    def __init__(self, dt, shared, lens, budget, seed, Hk=2, D=64, B=16):
        self.lens, self.budget, self.Hk, self.D, self.B, self.shared = lens, budget, Hk, D, B, shared
        self.dtype, self.rows = DTYPES[dt], () if shared else (Hk,)
        g = torch.Generator().manual_seed(seed)
        self.k, self.v = (torch.randn((sum(lens), Hk, D), generator=g).to(self.dtype).to(DEV) for _ in range(2))
        self.cu = _i32([sum(lens[:i]) for i in range(len(lens) + 1)])
        width = -(-budget // B)
        self.P = len(lens) * (1 if shared else Hk) * width
        self.table = torch.randperm(self.P, generator=g).int().view((len(lens),) + self.rows + (width,)).to(DEV)
        self.desc = pe.make_desc(self.dtype, len(lens), Hk, Hk, D, B, width, self.P, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)

    def prune(self, table, **how):
        """(pools with their guards, lengths, kept indices)"""
        shape = (self.P + 2, self.B) + ((self.Hk,) if self.shared else ()) + (self.D,)
        kp, vp = (torch.full(shape, JUNK, dtype=self.dtype, device=DEV) for _ in range(2))
        lens = torch.full((len(self.lens),), -5, dtype=torch.int32, device=DEV)
        kept = torch.full((len(self.lens),) + self.rows + (self.budget,), -9, dtype=torch.int32, device=DEV)
        ws = pe.alloc_workspace(pe.PE_OP_PREFILL_PRUNE, self.desc, sum(self.lens))
        pe.pe_prefill_prune(self.desc, self.k, self.v, self.cu, sum(self.lens), max(self.lens), self.budget, kp[1:-1], vp[1:-1], table, lens, kept,
                            ws, **how)
        torch.cuda.synchronize()
        return kp, vp, lens, kept


@pytest.mark.parametrize("way", ["one", "two"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_tokens_without_a_page_are_dropped(dt, shared, way):
    """All entries of a row missing, or its last one: the other pages are what they are with all of them, and nothing else is written."""
    print("case", dt, shared, way, flush=True)
    c = _Prompts(dt, shared, LENS[way], 64, 1)
    whole = c.prune(c.table)
    table = c.table.clone()
    gone = [(0, -1), (1, slice(None)), (3, 2)]
    for s, j in gone:
        table[(s, j) if shared else (s, 1, j)] = -1
    got = c.prune(table)
    lost = torch.cat([c.table[(s, j) if shared else (s, 1, j)].flatten() for s, j in gone]).long() + 1
    for a, b in zip(got[:2], whole[:2]):
        b[lost] = JUNK
        assert torch.equal(a, b)
        assert bool((a[0] == JUNK).all()) and bool((a[-1] == JUNK).all())
    assert torch.equal(got[2], whole[2]) and torch.equal(got[3], whole[3])


@pytest.mark.parametrize("way", ["one", "two"])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_only_sequences_that_begin_are_written(dt, shared, way):
    """Running sequences (2) and those that were left (0) keep pages, lengths and indices, with a full table of theirs and with none."""
    print("case", dt, shared, way, flush=True)
    c = _Prompts(dt, shared, LENS[way], 64, 2)
    whole = c.prune(c.table)
    for mask, table in (([1, 0, 2, 1], c.table), ([0, 1, 0, 0], torch.where(torch.arange(4, device=DEV).view((4,) + (1,) * (c.table.dim() - 1)) == 1, c.table, -1)),
                        ([0, 0, 0, 0], torch.full_like(c.table, -1))):
        got = c.prune(table, admitted=_i32(mask))
        for s, m in enumerate(mask):
            pages = c.table[s].flatten().long() + 1
            for a, b in zip(got[:2], whole[:2]):
                assert torch.equal(a[pages], b[pages]) if m == 1 else bool((a[pages] == JUNK).all()), (mask, s)
            assert int(got[2][s]) == (int(whole[2][s]) if m == 1 else -5)
            assert torch.equal(got[3][s], whole[3][s]) if m == 1 else bool((got[3][s] == -9).all())
        assert all(bool((p[i] == JUNK).all()) for p in got[:2] for i in (0, -1))
    assert all(torch.equal(a, b) for a, b in zip(c.prune(c.table, admitted=_i32([1] * 4)), whole))


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_list_that_ends_beside_running_sequences(dt, shared):
    """Sequence 0 runs; 1 begins; the list does not hold 2, nor 3 behind it; 0 also brings a chunk.  Only sequence 1 is written."""
    dtype, S, Hk, D, B, budget = DTYPES[dt], 4, 2, 64, 16, 64
    rows, width = 1 if shared else Hk, 8
    P = rows * (4 + 1 + 4 + 1) + rows + 2     # sequence 0 (4 pages, a spare one), 1 likewise, what is left is too little for 2
    g = torch.Generator().manual_seed(3)
    cache = PagedCache.create(dtype, S, Hk, Hk, D, B, empty_layout(S, Hk, width, 1, P, DEV, shared), budget, shared=shared)
    cache.k_pool.fill_(JUNK)
    cache.v_pool.fill_(JUNK)
    free = FreePages.of(torch.randperm(P, generator=g).int().to(DEV))

    def prompts(lens):
        plan = cache.admit(_i32(lens), sum(lens), free)
        k, v = (torch.randn((sum(lens), Hk, D), generator=g).to(dtype).to(DEV) for _ in range(2))
        cache.prefill_prune(k, v, plan.cu_seqlens, max(lens))
        return plan, k, v

    first, _, _ = prompts([90, 0, 0, 0])
    assert first.admitted.tolist() == [1, 0, 0, 0] and cache.seq_lens.tolist() == [64, 0, 0, 0]
    before = cache.k_pool.clone(), cache.v_pool.clone()
    plan, k, v = prompts([12, 77, 70, 50])
    assert plan.admitted.tolist() == [2, 1, 0, 0] and plan.cu_seqlens.tolist() == [0, 12, 89, 159, 209]
    assert cache.seq_lens.tolist() == [64, 64, 0, 0] and bool((cache.block_table[2:] == -1).all())
    mine = cache.block_table[1].flatten()
    mine = mine[mine >= 0].long()
    others = torch.ones(P, dtype=torch.bool, device=DEV)
    others[mine] = False
    alone = PagedCache.create(dtype, 1, Hk, Hk, D, B, empty_layout(1, Hk, width, 1, P, DEV, shared), budget, shared=shared)
    alone.block_table.copy_(cache.block_table[1:2])
    alone.k_pool.fill_(JUNK)
    alone.v_pool.fill_(JUNK)
    alone.prefill_prune(k[12:89].contiguous(), v[12:89].contiguous(), _i32([0, 77]), 77)
    for got, was, want in zip((cache.k_pool, cache.v_pool), before, (alone.k_pool, alone.v_pool)):
        assert torch.equal(got[mine], want[mine]) and torch.equal(got[others], was[others])
    # a part of the sequences, by their part of the answer
    part, _, _ = prompts([0, 0, 0, 16])
    assert part.admitted.tolist() == [0, 0, 0, 1] and cache.seq_lens.tolist() == [64, 64, 0, 16]
    assert cache.rows(1, 3).admitted.tolist() == [0, 0] and cache.rows(2, 4).admitted.tolist() == [0, 1]
