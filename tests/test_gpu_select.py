"""Bounds of pages' keys and the pages selected by them, against plain computations in 64 bits."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import DTYPES, NAN, Cache, assert_close, attend

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _bounds(c, fill):
    """What pe_page_bounds is to leave in an array that held `fill`: the full pages' smallest and largest keys."""
    shape = (c.pages, 2) + tuple(c.k_pool.shape[2:])
    want = torch.full(shape, fill, dtype=c.dtype)
    rows = c.table if not c.shared else c.table[:, None]
    for s, n in enumerate(c.lens):
        for r in range(rows.shape[1]):
            for j in range(n // c.B):
                page = int(rows[s, r, j])
                want[page, 0], want[page, 1] = c.k_pool[page].amin(0), c.k_pool[page].amax(0)
    return want


def _scores(c, q, s):
    """[rows of the sequence][full pages], fp64 sums rounded once to fp32, straight from the keys."""
    G, n = q.shape[1] // c.Hk, c.lens[s] // c.B
    per_head = []
    for h in range(c.Hk):
        k = c.k[s][h][:n * c.B].view(n, c.B, c.D)
        lo, hi = k.amin(1), k.amax(1)
        per_head.append(sum(torch.maximum(x * lo, x * hi).sum(1) for x in q[s, h * G:(h + 1) * G].double()))
    per_head = torch.stack(per_head)
    return (per_head.sum(0, keepdim=True) if c.shared else per_head).float()


def _selection(c, q, k):
    """(logical indices [S][rows][k], lengths [S])"""
    S, rows = len(c.lens), 1 if c.shared else c.Hk
    idx, lens = torch.full((S, rows, k), -1, dtype=torch.int32), torch.zeros(S, dtype=torch.int32)
    for s, n in enumerate(c.lens):
        pages = -(-n // c.B)
        lens[s] = n if pages <= k else (k - 1) * c.B + n - (pages - 1) * c.B
        scores = _scores(c, q, s)
        for r in range(rows):
            if pages <= k:
                best = list(range(pages))
            else:
                order = sorted(range(pages - 1), key=lambda j: (-float(scores[r, j]), j))
                best = sorted(order[:k - 1]) + [pages - 1]
            idx[s, r, :len(best)] = torch.tensor(best, dtype=torch.int32)
    return idx, lens


def _select(c, q, bounds, k, idx=True):
    desc = c.desc(pe, q.shape[1])
    _, _, table, lens = c.to(DEV)
    shape = tuple(c.table.shape[:-1]) + (k,)
    to = torch.full(shape, -9, dtype=torch.int32, device=DEV)
    at = torch.full(shape, -9, dtype=torch.int32, device=DEV) if idx else None
    n = torch.full((len(c.lens),), -9, dtype=torch.int32, device=DEV)
    ws = pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, desc)
    ws.fill_(0x7f)
    pe.pe_select_pages(desc, q.to(DEV), bounds, table, lens, k, to, n, at, ws)
    return to, n, at


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D,B,Hk,shared", [(64, 16, 2, False), (128, 16, 3, True), (64, 32, 1, True), (128, 64, 2, False), (64, 128, 2, False),
                                           (128, 128, 5, True)])
def test_bounds_of_full_pages(dt, D, B, Hk, shared):
    """All of them, and the most recent ones; what else is in the array stays."""
    print("case bounds", dt, D, B, Hk, shared, flush=True)
    c = Cache(D + B, [0, 1, B - 1, B, 5 * B + 3, 9 * B, 2 * B - 1], Hk, D, B, DTYPES[dt], shared)
    kp, _, table, lens = c.to(DEV)
    want = _bounds(c, 7.0)
    got = torch.full(want.shape, 7.0, dtype=c.dtype, device=DEV)
    pe.pe_page_bounds(c.desc(pe, Hk), kp, table, lens, 0, got)
    assert torch.equal(got.cpu(), want)
    for recent in (1, 3, 100):
        got.fill_(7.0)
        pe.pe_page_bounds(c.desc(pe, Hk), kp, table, lens, recent, got)
        some = want.clone()
        rows = c.table if not shared else c.table[:, None]
        for s, n in enumerate(c.lens):
            for r in range(rows.shape[1]):
                for j in range(max(0, n // B - recent)):
                    some[int(rows[s, r, j])] = 7.0
        assert torch.equal(got.cpu(), some), recent


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D,B,Hk,G,k,shared", [(64, 16, 2, 1, 1, False), (128, 16, 2, 4, 2, False), (64, 32, 3, 4, 7, True), (128, 16, 1, 8, 33, False),
                                               (128, 64, 2, 3, 5, True), (64, 128, 1, 7, 3, False), (64, 16, 5, 2, 64, True),
                                               (128, 16, 2, 4, 500, False)])
def test_selection_and_attention(dt, D, B, Hk, G, k, shared):
    """Fewer pages than are selected, as many, more; rows without a token; the newest page full, or with one token. The bounds of what is
    not to be read are NaN. The selected pages attended to against 64 bits."""
    print("case select", dt, D, B, Hk, G, k, shared, flush=True)
    lens = [0, 1, B, k * B, k * B + 1, 3 * k * B, (k + 70) * B - 3, 300 * B + 5 if B < 64 else 9 * B]
    c = Cache(D + B + k, lens, Hk, D, B, DTYPES[dt], shared)
    g = torch.Generator().manual_seed(k)
    q = torch.randn((len(lens), Hk * G, D), generator=g).to(c.dtype)
    bounds = _bounds(c, NAN).to(DEV)
    to, n, at = _select(c, q, bounds, k)
    idx, want_lens = _selection(c, q, k)
    idx = idx[:, 0] if shared else idx
    assert torch.equal(n.cpu(), want_lens)
    assert torch.equal(at.cpu(), idx)
    want = torch.where(idx >= 0, c.table.gather(-1, idx.clamp(min=0).long()), torch.full_like(idx, -1))
    assert torch.equal(to.cpu(), want)
    to2, n2, _ = _select(c, q, bounds, k, idx=False)
    assert torch.equal(to2, to) and torch.equal(n2, n)
    sel = pe.make_desc(c.dtype, len(lens), Hk, Hk * G, D, B, k, c.pages, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    kp, vp = c.k_pool.to(DEV), c.v_pool.to(DEV)
    out = torch.full(q.shape, 7.0, dtype=c.dtype, device=DEV)
    pe.pe_paged_decode(sel, q.to(DEV), kp, vp, to, n, D ** -0.5, out, pe.alloc_workspace(pe.PE_OP_PAGED_DECODE, sel))
    for s, length in enumerate(lens):
        for h in range(Hk * G):
            pages = [int(j) for j in (idx[s] if shared else idx[s, h // G]) if j >= 0]
            tokens = [t for j in pages for t in range(j * B, min(length, (j + 1) * B))]
            o, _, b = attend(q[s, h:h + 1].double(), c.k[s][h // G][tokens], c.v[s][h // G][tokens])
            assert_close(out[s, h:h + 1], o, b, c.dtype)


@pytest.mark.parametrize("n,k", [(700, 256), (2100, 31), (9000, 4000), (20000, 2), (33000, 600)])
def test_ties_go_to_the_lowest_index(n, k):
    """Few different scores over many pages: among equal ones the first are taken. (Scores are set through one element of the bounds, and are
    of either sign; -0 and 0 are equal.)"""
    print("case ties", n, k, flush=True)
    B, D = 16, 64
    g = torch.Generator().manual_seed(n)
    level = torch.randint(-2, 4, (n,), generator=g).float()
    table = torch.randperm(n, generator=g).int().view(1, 1, n)
    bounds = torch.zeros((n, 2, D))
    bounds[table[0, 0].long(), 1, 3] = level
    bounds[table[0, 0].long(), 0, 3] = level - 1
    bounds[table[0, 0].long(), 0, 5] = -0.0
    q = torch.zeros((1, 2, D))
    q[0, :, 3] = 1.0
    q[0, :, 5] = -1.0
    desc = pe.make_desc(torch.float32, 1, 1, 2, D, B, n, n)
    to, at = (torch.full((1, 1, k), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    out_n = torch.zeros(1, dtype=torch.int32, device=DEV)
    pe.pe_select_pages(desc, q.to(DEV), bounds.to(DEV), table.to(DEV), torch.tensor([n * B - 2], dtype=torch.int32, device=DEV), k, to, out_n, at,
                       pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, desc))
    order = torch.sort(level[:n - 1], descending=True, stable=True).indices[:k - 1].sort().values
    want = torch.cat((order, torch.tensor([n - 1]))).int()
    assert torch.equal(at.cpu()[0, 0], want)
    assert torch.equal(to.cpu()[0, 0], table[0, 0][want.long()])
    assert int(out_n) == k * B - 2


def test_selection_in_a_graph_follows_lengths_and_queries():
    print("case select graph", flush=True)
    c = Cache(3, [500, 2000], 2, 128, 16, torch.bfloat16, False)
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(3)).bfloat16().to(DEV)
    kp, _, table, lens = c.to(DEV)
    bounds = torch.zeros((c.pages, 2, 128), dtype=torch.bfloat16, device=DEV)
    desc, k = c.desc(pe, 8), 20
    ws = pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, desc)
    outs = [(torch.zeros((2, 2, k), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV),
             torch.zeros((2, 2, k), dtype=torch.int32, device=DEV)) for _ in range(2)]

    def call(o):
        pe.pe_page_bounds(desc, kp, table, lens, 0, bounds)
        pe.pe_select_pages(desc, q, bounds, table, lens, k, *o, ws)

    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[0])
    for n in (2000, 1999, 320, 321, 0):
        lens[1] = n
        q.normal_()
        graph.replay()
        call(outs[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs)), n
