"""Calls for trees, weights and paths that the header allows at its edges: counts outside their range, outputs that begin in the middle of a
16-byte group, more pages selected than a table has."""
import math

import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import DTYPES, Cache
from test_gpu_tree import _case, _check, _want

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _shifted(shape, dtype, fill):
    """A dense tensor that begins one element behind an allocation's beginning."""
    n = math.prod(shape)
    return torch.full((n + 1,), fill, dtype=dtype, device=DEV)[1:].view(shape)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hk,splits", [(5, 2, 1), (5, 2, 3), (60, 3, 1), (60, 3, 2)])
def test_draft_counts_are_clamped_and_outputs_begin_anywhere(dt, T, Hk, splits):
    print("case edges", dt, T, Hk, splits, flush=True)
    G, lens, counts = 8, [0, 100, 700], [T, 0, T]
    c, q, kd, vd, sees, words = _case(T, lens, counts, T, Hk, G, 128, 16, DTYPES[dt], False)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    desc = c.desc(pe, Hk * G, decode_splits=splits)
    kp, vp, table, sl = c.to(DEV)
    out = _shifted(q.shape, q.dtype, 7.0)
    given = torch.tensor([T + 1000, -3, 0x7fffffff], dtype=torch.int32, device=DEV)
    pe.pe_tree_decode(desc, T, q.to(DEV), kd.to(DEV), vd.to(DEV), given, words.to(DEV), kp, vp, table, sl, 128 ** -0.5, out,
                      pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T))
    _check(out, want, bound, counts, q.dtype)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("splits", [1, 3])
def test_weights_and_outputs_begin_anywhere_and_take_the_queries_place(dt, splits):
    print("case edges of weights", dt, splits, flush=True)
    c = Cache(3, [0, 1, 700], 2, 64, 16, DTYPES[dt], True)
    q = torch.randn((3, 10, 64), generator=torch.Generator().manual_seed(3)).to(c.dtype).to(DEV)
    desc = c.desc(pe, 10, decode_splits=splits)
    kp, vp, table, sl = c.to(DEV)
    ws = pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, desc)
    got = []
    for shifted in (False, True):
        shape = (3, 2, c.max_blocks)
        w_in = _shifted(shape, torch.float32, 1.5) if shifted else torch.full(shape, 1.5, device=DEV)
        w_out = _shifted(shape, torch.float32, 9.0) if shifted else torch.full(shape, 9.0, device=DEV)
        out = _shifted(q.shape, q.dtype, 7.0) if shifted else torch.full_like(q, 7.0)
        pe.pe_paged_decode_weights(desc, q, kp, vp, table, sl, 0.125, 0.5, w_in, w_out, out, ws)
        got.append((out, w_out))
    place, w = q.clone(), torch.full((3, 2, c.max_blocks), 1.5, device=DEV)
    pe.pe_paged_decode_weights(desc, place, kp, vp, table, sl, 0.125, 0.5, w, w, place, ws)
    got.append((place, w))
    for out, w in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(w, got[0][1])


def test_paths_whose_counts_are_no_counts_are_left_alone():
    print("case edges of paths", flush=True)
    c = Cache(4, [5, 6, 7], 2, 64, 16, torch.bfloat16, False)
    kp, vp, table, lens = c.to(DEV)
    before = [x.clone() for x in (kp, vp, table, lens)]
    kd = torch.randn((3, 4, 2, 64), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    path = torch.zeros((3, 4), dtype=torch.int32, device=DEV)
    n = torch.tensor([-1, 0x7fffffff, 3], dtype=torch.int32, device=DEV)
    done = torch.tensor([0, 4, -2], dtype=torch.int32, device=DEV)
    freed, used = torch.full((3, 2), -1, dtype=torch.int32, device=DEV), torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    spare = torch.zeros((3, 2, 1), dtype=torch.int32, device=DEV)
    pe.pe_append_path(c.desc(pe, 2), kd, kd, path, n, done, kp, vp, table, lens, freed, spare, used)
    for a, b in zip((kp, vp, table, lens), before):
        assert torch.equal(a.nan_to_num(9.0) if a.is_floating_point() else a, b.nan_to_num(9.0) if b.is_floating_point() else b)
    assert done.tolist() == [0, 4, -2] and int(used.sum()) == 0


def test_more_pages_than_a_table_has():
    print("case edges of selections", flush=True)
    c = Cache(5, [0, 1, 70, 33], 2, 64, 16, torch.bfloat16, False, extra_blocks=0)
    _, _, table, lens = c.to(DEV)
    q = torch.randn((4, 4, 64), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    bounds = torch.full((c.pages, 2, 64), float("nan"), dtype=torch.bfloat16, device=DEV)   # (none is read)
    desc, k = c.desc(pe, 4), c.max_blocks + 3
    to, idx, n = (torch.full(s, -9, dtype=torch.int32, device=DEV) for s in ((4, 2, k), (4, 2, k), (4,)))
    pe.pe_select_pages(desc, q, bounds, table, lens, k, to, n, idx, pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, desc))
    assert torch.equal(to[..., :c.max_blocks], table) and bool((to[..., c.max_blocks:] == -1).all()) and torch.equal(n, lens)
    want = torch.where(to >= 0, torch.arange(k, device=DEV).int().expand(to.shape), torch.full_like(to, -1))
    assert torch.equal(idx, want)
