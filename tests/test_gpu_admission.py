"""Admissions as a program makes them over its life: prompts kept whole beyond the budget, sequences that come while others run."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd.engine import FreePages, LayeredCache, PagedCache, QuantCache, empty_layout

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
