"""Attention over a cache in 8 bits (pe_quant_decode) against 64 bits: types, layouts, lengths, groups, splits, scales, junk."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import DTYPES, assert_close
from _quant64 import QuantCache, attend

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _run(seed, lens, Hk, G, D, B, dt, shared=False, splits=0, scale=None, place=None, **kw):
    dtype = DTYPES[dt]
    c = QuantCache(seed, lens, Hk, D, B, dtype, shared, **kw)
    desc = c.desc(pe, Hk * G, decode_splits=splits)
    g = torch.Generator().manual_seed(seed + 7)
    q = torch.randn((len(lens), Hk * G, D), generator=g).to(dtype)
    cache = c.quant(pe, desc, DEV)
    _, _, table, sl = c.to(DEV)
    qd = q.to(DEV)
    out = place(qd) if place else torch.full_like(qd, 7.0)
    ws = pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc)
    if ws is not None:
        ws.fill_(0xff)
    pe.pe_quant_decode(desc, cache, qd, table, sl, D ** -0.5 if scale is None else scale, out, ws)
    torch.cuda.synchronize()
    for s in range(len(lens)):
        for h in range(Hk):
            want, bound = attend(q[s, h * G:(h + 1) * G].double(), c.k[s][h], c.v[s][h], dtype, scale)
            assert_close(out[s, h * G:(h + 1) * G], want, bound, dtype)
    return out


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B", [16, 32, 64, 128])
def test_lengths(B, D, dt, shared):
    _run(B + D, [0, 1, 15, 16, 17, B - 1, B, B + 1, 2 * B + 15, 3 * B, 7 * B + 3, 529], 2, 4, D, B, dt, shared)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8])
def test_groups(G, dt, D, shared):
    _run(G, [33, 200, 0, 64], 3, G, D, 16, dt, shared)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt,D,G", [("bf16", 128, 4), ("bf16", 64, 8), ("f32", 128, 2), ("f32", 64, 5)])
@pytest.mark.parametrize("splits", [1, 2, 3, 8, 9, 12, 13, 40])
def test_splits(splits, dt, D, G, shared):
    """Merged by the last to arrive, by a launch of one wave, and of several; splits without tokens among them."""
    _run(splits, [1500, 3, 0, 700, 16], 2, G, D, 16, dt, shared, splits=splits)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_any_scales(D, dt):
    _run(5, [70, 16, 300], 2, 4, D, 16, dt, odd_scales=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [2.0 ** 30, 2.0 ** -30])
def test_large_and_small_elements(scale, dt):
    _run(6, [70, 16, 300], 2, 4, 64, 16, dt, scale=2.0 ** -3 / scale, **{"extra_pages": 2})   # logits of any size
    c_scale = dict(lens=[70, 16, 300], Hk=2, G=4, D=64, B=16, dt=dt)
    dtype = DTYPES[dt]
    c = QuantCache(8, c_scale["lens"], 2, 64, 16, dtype, False, scale=scale)
    desc = c.desc(pe, 8)
    q = (torch.randn((3, 8, 64), generator=torch.Generator().manual_seed(9)) / scale).to(dtype)
    out = torch.empty_like(q, device=DEV)
    pe.pe_quant_decode(desc, c.quant(pe, desc, DEV), q.to(DEV), *c.to(DEV)[2:], 0.125, out, pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc))
    for s in range(3):
        for h in range(2):
            want, bound = attend(q[s, h * 4:h * 4 + 4].double(), c.k[s][h], c.v[s][h], dtype, 0.125)
            assert_close(out[s, h * 4:h * 4 + 4], want, bound, dtype)


@pytest.mark.parametrize("splits", [1, 4, 16])
def test_in_the_queries_place_and_anywhere(splits):
    want = _run(10, [500, 90], 2, 4, 64, 16, "bf16", splits=splits)
    assert torch.equal(_run(10, [500, 90], 2, 4, 64, 16, "bf16", splits=splits, place=lambda q: q), want)
    odd = lambda q: torch.zeros(q.numel() + 1, dtype=q.dtype, device=DEV)[1:].view(q.shape)   # noqa: E731
    assert torch.equal(_run(10, [500, 90], 2, 4, 64, 16, "bf16", splits=splits, place=odd), want)


def test_the_cache_is_what_its_numbers_stand_for():
    """Scales that are powers of two: the same attention as over a bfloat16 cache of the same values."""
    lens, Hk, G, D, B = [600, 33, 1024], 2, 4, 128, 16
    c = QuantCache(11, lens, Hk, D, B, torch.bfloat16, False)
    desc = c.desc(pe, Hk * G)
    for s, n in enumerate(lens):
        for h in range(Hk):
            for j in range(-(-n // B)):
                part = slice(j * B, min(n, (j + 1) * B))
                for pool, x in ((c.k_pool, c.k), (c.v_pool, c.v)):
                    pool[c.table[s, h, j], :part.stop - part.start] = x[s][h][part].to(torch.bfloat16)
    q = torch.randn((3, Hk * G, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    kp, vp, table, sl = c.to(DEV)
    a, b = torch.empty_like(q), torch.empty_like(q)
    pe.pe_quant_decode(desc, c.quant(pe, desc, DEV), q, table, sl, D ** -0.5, a, pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc))
    pe.pe_paged_decode(desc, q, kp, vp, table, sl, D ** -0.5, b, pe.alloc_workspace(pe.PE_OP_PAGED_DECODE, desc))
    # two roundings of sums in 32 bits to bfloat16: neighbours at most
    d = (a.float() - b.float()).abs() - 2.0 ** -7 * b.float().abs()
    assert float(d.max()) <= 2.0 ** -18


def test_many_rows_and_long_ones():
    _run(12, [40 + i % 60 for i in range(130)], 4, 2, 64, 16, "bf16")
    _run(13, [9000], 1, 4, 128, 32, "bf16")
    _run(14, [4000, 1], 2, 8, 64, 16, "f32", shared=True)


@pytest.mark.parametrize("G", [1, 4, 5, 8])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_long_pieces(D, dt, G):
    """Rows whole: two tiles in flight for D = 64, odd and even numbers of them, waves without any."""
    _run(G, [1024, 1040, 1153, 1300, 2000, 2 * 8 * 16 * 5, 17], 1, G, D, 16, dt, splits=1)
    _run(G, [3000, 5], 1, G, D, 128, dt, shared=True, splits=2)


def test_lengths_that_the_table_does_not_hold():
    """A caller's mistake: the row ends with its table; a negative length is none."""
    c = QuantCache(20, [64, 64, 64], 1, 64, 16, torch.bfloat16, False, extra_blocks=0)
    desc = c.desc(pe, 2)
    q = torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    sl = torch.tensor([70000, -3, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 7.0, device=DEV)
    pe.pe_quant_decode(desc, c.quant(pe, desc, DEV), q.to(DEV), c.table.to(DEV), sl, 0.125, out, pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc))
    for s in (0, 2):
        assert_close(out[s], *attend(q[s].double(), c.k[s][0], c.v[s][0], torch.bfloat16, 0.125), torch.bfloat16)
    assert bool((out[1] == 0).all())


def test_two_graphs_with_one_workspace():
    """Two layers' calls, captured apart, with the same workspace, replayed in turn on one stream."""
    made = []
    ws = None
    for seed in (21, 22):
        c = QuantCache(seed, [700, 900, 31], 2, 128, 16, torch.bfloat16, False)
        desc = c.desc(pe, 8, decode_splits=5)
        ws = pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc) if ws is None else ws
        q = torch.randn((3, 8, 128), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
        made.append((c, desc, c.quant(pe, desc, DEV), q, q.to(DEV), c.to(DEV), torch.empty_like(q, device=DEV)))
    torch.cuda.synchronize()
    graphs = []
    for c, desc, cache, q, qd, d, out in made:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            pe.pe_quant_decode(desc, cache, qd, d[2], d[3], 128 ** -0.5, out, ws)
    for _ in range(5):
        for g, m in zip(graphs, made):
            m[-1].fill_(3.0)
            g.replay()
    torch.cuda.synchronize()
    for c, desc, cache, q, qd, d, out in made:
        for s in range(3):
            for h in range(2):
                want, bound = attend(q[s, h * 4:h * 4 + 4].double(), c.k[s][h], c.v[s][h], torch.bfloat16)
                assert_close(out[s, h * 4:h * 4 + 4], want, bound, torch.bfloat16)


@pytest.mark.parametrize("splits", [0, 3, 16])
def test_replayed_while_the_cache_grows(splits):
    """One graph, the lengths and the output's old contents changing between replays, eager calls in between."""
    lens, Hk, G, D, B = [300, 45, 160], 2, 4, 128, 16
    c = QuantCache(15, lens, Hk, D, B, torch.bfloat16, False)
    desc = c.desc(pe, Hk * G, decode_splits=splits)
    cache = c.quant(pe, desc, DEV)
    _, _, table, sl = c.to(DEV)
    q = torch.randn((3, Hk * G, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    out, eager = torch.empty_like(q), torch.empty_like(q)
    ws, ws2 = (pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc) for _ in range(2))
    pe.pe_quant_decode(desc, cache, q, table, sl, 0.1, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pe.pe_quant_decode(desc, cache, q, table, sl, 0.1, out, ws)
    for step, n in enumerate(([300, 45, 160], [288, 16, 0], [16, 32, 144], [300, 0, 16])):
        sl.copy_(torch.tensor(n, dtype=torch.int32))
        q.mul_(0.9)
        for _ in range(2):
            graph.replay()
        pe.pe_quant_decode(desc, cache, q, table, sl, 0.1, eager, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), step


def test_two_at_once_on_two_streams():
    made = []
    for seed in (16, 17):
        c = QuantCache(seed, [700, 900, 31], 2, 128, 16, torch.bfloat16, False)
        desc = c.desc(pe, 8, decode_splits=6)
        q = torch.randn((3, 8, 128), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
        made.append((c, desc, c.quant(pe, desc, DEV), q, q.to(DEV), c.to(DEV), torch.empty_like(q, device=DEV),
                     pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for c, desc, cache, q, qd, d, out, ws, stream in made:
            with torch.cuda.stream(stream):
                pe.pe_quant_decode(desc, cache, qd, d[2], d[3], 128 ** -0.5, out, ws)
    torch.cuda.synchronize()
    for c, desc, cache, q, qd, d, out, ws, stream in made:
        for s in range(3):
            for h in range(2):
                want, bound = attend(q[s, h * 4:h * 4 + 4].double(), c.k[s][h], c.v[s][h], torch.bfloat16)
                assert_close(out[s, h * 4:h * 4 + 4], want, bound, torch.bfloat16)
