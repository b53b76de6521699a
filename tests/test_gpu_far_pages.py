"""Trees, paths, page weights, bounds and selections over pages that lie behind 2^32 bytes and elements of their pools: bit for bit what the
same pages at the start of a small pool give.  And two of these calls at once, on streams of their own."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import Cache
from test_gpu_tree import _trees, _words

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 0.09


def _far(c, pages):
    """The cache's pages as the last ones of pools of so many, which hold nothing else."""
    base = pages - c.pages
    pools = []
    for x in (c.k_pool, c.v_pool):
        pool = torch.empty((pages,) + x.shape[1:], dtype=x.dtype, device=DEV)
        pool[base:] = x.to(DEV)
        pools.append(pool)
    table = torch.where(c.table >= 0, c.table + base, c.table).to(DEV)
    return pools + [table, c.seq_lens.to(DEV)], base


def _desc(c, Hq, pages, **kw):
    return pe.make_desc(c.dtype, len(c.lens), c.Hk, Hq, c.D, c.B, c.max_blocks, pages,
                        pe.PE_LAYOUT_SHARED if c.shared else pe.PE_LAYOUT_PER_HEAD, **kw)


def _all_calls(c, dev, pages, base, T, G, bounds_too):
    """What the calls give; ids of pages relative to `base`."""
    S, Hq = len(c.lens), c.Hk * G
    g = torch.Generator().manual_seed(T)
    kp, vp, table, lens = dev
    q, kd, vd = (torch.randn((S, T, h, c.D), generator=g).to(c.dtype).to(DEV) for h in (Hq, c.Hk, c.Hk))
    words = _words(_trees(S, T, g)).to(DEV)
    desc, got = _desc(c, Hq, pages), []
    out = torch.empty_like(q)
    pe.pe_tree_decode(desc, T, q, kd, vd, None, words, kp, vp, table, lens, SCALE, out, pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T))
    got.append(out)
    q1, out1 = q[:, 0].contiguous(), torch.empty((S, Hq, c.D), dtype=c.dtype, device=DEV)
    weights = torch.empty((S, c.Hk, c.max_blocks), device=DEV)
    pe.pe_paged_decode_weights(desc, q1, kp, vp, table, lens, SCALE, 1.0, None, weights, out1,
                               pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, desc))
    got += [out1, weights]
    if bounds_too:
        heads = (c.Hk,) if c.shared else ()
        bounds = torch.empty((pages, 2) + heads + (c.D,), dtype=c.dtype, device=DEV)
        pe.pe_page_bounds(desc, kp, table, lens, 0, bounds)
        to, n = torch.empty(table.shape[:-1] + (3,), dtype=torch.int32, device=DEV), torch.empty_like(lens)
        pe.pe_select_pages(desc, q1, bounds, table, lens, 3, to, n, None, pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, desc))
        full = sorted({int(p) for s, m in enumerate(c.lens) for p in c.table[s].reshape(-1, c.max_blocks)[:, :m // c.B].flatten()})
        got += [torch.where(to >= 0, to - base, to), n, bounds[torch.tensor(full, device=DEV) + base]]
    per_row = c.table.shape[:-1]
    spare = torch.full(per_row + (1,), base + c.pages - 1, dtype=torch.int32, device=DEV)   # (none is needed)
    freed, used = (torch.full(per_row, v, dtype=torch.int32, device=DEV) for v in (-1, 0))
    path, n = torch.tensor([[T - 1, 0]] * S, dtype=torch.int32, device=DEV), torch.full((S,), 2, dtype=torch.int32, device=DEV)
    pe.pe_append_path(desc, kd, vd, path, n, torch.zeros_like(n), kp, vp, table, lens, freed, spare, used)
    torch.cuda.synchronize()
    got += [lens.clone(), used, kp[base:].nan_to_num(7.0), vp[base:].nan_to_num(7.0)]
    return got


@pytest.mark.parametrize("dt,D,B,Hk,G,T,shared,pages", [
    (torch.bfloat16, 128, 16, 2, 4, 3, False, (1 << 21) + 700), (torch.bfloat16, 128, 32, 4, 8, 64, True, (1 << 18) + 700),
    (torch.float32, 64, 16, 2, 2, 20, False, (1 << 22) + 700), (torch.bfloat16, 64, 16, 1, 4, 2, False, (1 << 24) + 700)])
def test_pages_behind_32_bits(dt, D, B, Hk, G, T, shared, pages):
    """(The last: bounds of more than 2^32 bytes too.)"""
    print("case far", dt, D, B, Hk, G, T, shared, pages, flush=True)
    c = Cache(5, [3 * B + 1, 40 * B + 3, B + 2, 700, 5, 2 * B + 7, 1, 130], Hk, D, B, dt, shared)
    assert pages * B * D * (Hk if shared else 1) > 1 << 32
    near = _all_calls(c, c.to(DEV), c.pages, 0, T, G, True)
    dev, base = _far(c, pages)
    far = _all_calls(c, dev, pages, base, T, G, True)
    for i, (a, b) in enumerate(zip(near, far)):
        assert torch.equal(a, b), i


def test_two_calls_at_once():
    """A tree, page weights and a selection on three streams, each with its own workspace, over one cache."""
    print("case streams", flush=True)
    T, G, Hk, D, B = 16, 4, 2, 128, 16
    c = Cache(6, [2000, 77, 4000, 0], Hk, D, B, torch.bfloat16, False)
    kp, vp, table, lens = c.to(DEV)
    g = torch.Generator().manual_seed(2)
    q, kd, vd = (torch.randn((4, T, h, D), generator=g).bfloat16().to(DEV) for h in (Hk * G, Hk, Hk))
    q1, words, desc = q[:, 0].contiguous(), _words(_trees(4, T, g)).to(DEV), c.desc(pe, Hk * G)
    bounds = torch.empty((c.pages, 2, D), dtype=torch.bfloat16, device=DEV)
    pe.pe_page_bounds(desc, kp, table, lens, 0, bounds)

    def calls():
        out, out1, w = torch.zeros_like(q), torch.zeros_like(q1), torch.zeros((4, Hk, c.max_blocks), device=DEV)
        to, n = torch.zeros((4, Hk, 9), dtype=torch.int32, device=DEV), torch.zeros_like(lens)
        ws = [pe.alloc_workspace(op, desc, t) for op, t in ((pe.PE_OP_TREE_DECODE, T), (pe.PE_OP_DECODE_WEIGHTS, 0), (pe.PE_OP_SELECT_PAGES, 0))]
        run = [lambda: pe.pe_tree_decode(desc, T, q, kd, vd, None, words, kp, vp, table, lens, SCALE, out, ws[0]),
               lambda: pe.pe_paged_decode_weights(desc, q1, kp, vp, table, lens, SCALE, 1.0, None, w, out1, ws[1]),
               lambda: pe.pe_select_pages(desc, q1, bounds, table, lens, 9, to, n, None, ws[2])]
        return run, [out, out1, w, to, n], ws

    run, want, _ = calls()
    for f in run:
        f()
    torch.cuda.synchronize()
    run, got, keep = calls()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in run]
    for _ in range(10):
        for f, stream in zip(run, streams):
            with torch.cuda.stream(stream):
                f()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(keep) == 3
