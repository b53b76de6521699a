"""Attention with the weight that each page got, against plain attention in 64 bits, and the eviction by it."""
import math

import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import DTYPES, NAN, Cache, assert_close, attend

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _want(c, q, before, decay):
    """(out, its bound, weights, their bound): a page's weight is off by its tokens' (attend() relative to A = 1), the sum over the heads and
    pages' tokens, and the two roundings of the sum with what was there."""
    S, Hq, D = q.shape
    G = Hq // c.Hk
    out, bound = torch.zeros((S, Hq, D), dtype=torch.float64), torch.zeros((S, Hq, D), dtype=torch.float64)
    w = torch.full((S, c.Hk, c.max_blocks), math.inf, dtype=torch.float64)
    wb = torch.zeros_like(w)
    for s, n in enumerate(c.lens):
        pages = -(-n // c.B)
        for h in range(c.Hk):
            got, off = torch.zeros(pages, dtype=torch.float64), torch.zeros(pages, dtype=torch.float64)
            for x in range(h * G, (h + 1) * G):
                o, p, b = attend(q[s, x:x + 1].double(), c.k[s][h], c.v[s][h])
                _, _, rel = attend(q[s, x:x + 1].double(), c.k[s][h], torch.ones((n, 1), dtype=torch.float64))
                out[s, x], bound[s, x] = o[0], b[0]
                if n:
                    one = torch.zeros(pages * c.B, dtype=torch.float64)
                    one[:n] = p[0]
                    one = one.view(pages, c.B).sum(1)
                    got += one
                    off += one * float(rel[0, 0])
            if n:
                old = torch.zeros(pages, dtype=torch.float64) if before is None else before[s, h, :pages].double().clone()
                old[~torch.isfinite(old)] = 0.0
                w[s, h, :pages] = old * decay + got
                wb[s, h, :pages] = off + (G + 4) * 2.0 ** -24 * (old * decay + got).abs()
    return out, bound, w, wb


def _run(c, q, before, decay, splits=0, alias=False):
    desc = c.desc(pe, q.shape[1], decode_splits=splits)
    kp, vp, table, lens = c.to(DEV)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    w_in = None if before is None else before.to(DEV)
    w_out = w_in if alias else torch.full((len(c.lens), c.Hk, c.max_blocks), NAN, device=DEV)
    ws = pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, desc)
    if ws is not None:
        ws.fill_(0xff)   # NaN wherever nothing is written
    pe.pe_paged_decode_weights(desc, q.to(DEV), kp, vp, table, lens, q.shape[2] ** -0.5, decay, w_in, w_out, out, ws)
    return out, w_out


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D,B,Hk,G,shared", [(64, 16, 2, 1, False), (128, 16, 2, 4, True), (64, 32, 3, 4, False), (128, 64, 1, 8, False),
                                             (64, 128, 2, 7, True), (128, 128, 2, 3, False), (128, 32, 5, 2, True), (64, 16, 1, 5, False)])
def test_weights_against_64_bits(dt, D, B, Hk, G, shared):
    """Empty rows, one token, pages that end inside a step or a round, every split count; weights that were there, +inf and NaN among
    them, and none; in place."""
    print("case weights", dt, D, B, Hk, G, shared, flush=True)
    lens = [0, 1, 15, 16, 127, 128, 129, 700, 1600]
    c = Cache(D + B + G, lens, Hk, D, B, DTYPES[dt], shared, extra_blocks=2)
    g = torch.Generator().manual_seed(B)
    q = torch.randn((len(lens), Hk * G, D), generator=g).to(c.dtype)
    before = torch.rand((len(lens), Hk, c.max_blocks), generator=g) * 5
    before[:, :, -3:] = math.inf
    before[7, 0, 0], before[8, 0, 1] = NAN, math.inf
    for decay, old in ((1.0, before), (0.5, before), (0.25, None), (0.0, before)):
        out, bound, w, wb = _want(c, q, old, decay)
        for splits, alias in ((0, False), (1, False), (2, True), (5, False)):
            got, gw = _run(c, q, old, decay, splits, alias and old is not None)
            assert_close(got, out, bound, c.dtype)
            gw = gw.cpu().double()
            inf = torch.isinf(w)
            assert bool((gw[inf] == math.inf).all())
            assert bool(((gw - w).abs()[~inf] <= wb[~inf]).all()), float(((gw - w).abs()[~inf] - wb[~inf]).max())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_long_rows(dt):
    """More tokens than a split's parts have room for: the split count grows with the table."""
    print("case long", dt, flush=True)
    c = Cache(5, [20001, 8000], 1, 64, 16, DTYPES[dt], False)
    q = torch.randn((2, 8, 64), generator=torch.Generator().manual_seed(5)).to(c.dtype)
    out, bound, w, wb = _want(c, q, None, 1.0)
    for splits in (0, 1, 3, 7):
        got, gw = _run(c, q, None, 1.0, splits)
        assert_close(got, out, bound, c.dtype)
        gw, inf = gw.cpu().double(), torch.isinf(w)
        assert torch.equal(torch.isinf(gw), inf) and bool(((gw - w).abs()[~inf] <= wb[~inf]).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_large_logits(dt):
    """References that move often: what a part was relative to when it was kept counts."""
    print("case large", dt, flush=True)
    c = Cache(6, [900, 64], 2, 64, 16, DTYPES[dt], True, scale=30.0)
    q = torch.randn((2, 6, 64), generator=torch.Generator().manual_seed(6)).to(c.dtype)
    out, bound, w, wb = _want(c, q, None, 1.0)
    for splits in (1, 3):
        got, gw = _run(c, q, None, 1.0, splits)
        assert_close(got, out, bound, c.dtype)
        gw, inf = gw.cpu().double(), torch.isinf(w)
        assert bool(((gw - w).abs()[~inf] <= wb[~inf] + 2.0 ** -126).all())


def test_weights_sum_to_the_query_heads_and_repeat():
    print("case sums", flush=True)
    c = Cache(7, [2048] * 6, 4, 128, 16, torch.bfloat16, False, extra_blocks=0)
    q = torch.randn((6, 16, 128), generator=torch.Generator().manual_seed(7)).bfloat16()
    for splits in (1, 4):
        out, w = _run(c, q, None, 1.0, splits)
        again, w2 = _run(c, q, None, 1.0, splits)
        assert torch.equal(out, again) and torch.equal(w, w2)
        assert bool(((w.double().sum(-1) - 4.0).abs() < 4 * (2048 + 200) * 2.0 ** -23).all())


def test_weights_in_a_graph():
    """Replays add up in place, and follow the lengths."""
    print("case weights graph", flush=True)
    c = Cache(8, [700, 33], 2, 128, 16, torch.bfloat16, False)
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(8)).bfloat16().to(DEV)
    kp, vp, table, lens = c.to(DEV)
    desc = c.desc(pe, 8)
    ws = pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, desc)
    state = [(torch.full((2, 2, c.max_blocks), math.inf, device=DEV), torch.zeros_like(q)) for _ in range(2)]
    call = lambda w, out: pe.pe_paged_decode_weights(desc, q, kp, vp, table, lens, 128 ** -0.5, 0.5, w, w, out, ws)   # noqa: E731
    call(*state[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*state[0])
    state[1][0].fill_(math.inf)
    for n in (700, 650, 3, 0, 700):
        lens[0] = n
        graph.replay()
        call(*state[1])
        torch.cuda.synchronize()
        assert torch.equal(*[s[0] for s in state]) and torch.equal(*[s[1] for s in state]), n
