"""Attention of a tree of drafts over the paged cache, and the accepted path's way into it, against plain computations in 64 bits."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import DTYPES, NAN, Cache, assert_close, attend

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _trees(S, T, g, kind="tree"):
    """bool [S, T, T]: which drafts a draft attends to."""
    sees = torch.zeros((S, T, T), dtype=torch.bool)
    for s in range(S):
        for i in range(T):
            if kind == "chain":
                sees[s, i, :i + 1] = True
            elif kind == "any":   # no tree at all: any set, the later ones and the empty one among them
                sees[s, i] = torch.rand(T, generator=g) < (0.0 if i % 5 == 4 else 0.4)
            else:
                parent = int(torch.randint(-1, i, (1,), generator=g)) if i else -1
                if parent >= 0:
                    sees[s, i] = sees[s, parent]
                sees[s, i, i] = True
    return sees


def _words(sees):
    T = sees.shape[-1]
    bits = torch.tensor([1 << j if j < 63 else -(1 << 63) for j in range(T)], dtype=torch.int64)
    return (sees.long() * bits).sum(-1)


def _case(seed, lens, counts, T, Hk, G, D, B, dtype, shared, kind="tree", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    c = Cache(seed + 1, lens, Hk, D, B, dtype, shared, scale=scale)
    S = len(lens)
    q = torch.randn((S, T, Hk * G, D), generator=g).to(dtype)
    kd, vd = (torch.randn((S, T, Hk, D), generator=g).to(dtype) for _ in range(2))
    sees = _trees(S, T, g, kind)
    words = _words(sees)
    for s, n in enumerate(counts):   # junk behind the last draft: in its key, its value, its query and as bits of the words before
        kd[s, n:], vd[s, n:], q[s, n:] = NAN, NAN, NAN
        for j in range(n, T):
            words[s] |= 1 << j if j < 63 else -(1 << 63)
    return c, q, kd, vd, sees, words


def _want(c, q, kd, vd, sees, counts, G, scale=None):
    S, T, Hq, D = q.shape
    want, bound = torch.zeros((S, T, Hq, D), dtype=torch.float64), torch.zeros((S, T, Hq, D), dtype=torch.float64)
    for s, n in enumerate(counts):
        for h in range(Hq):
            k = torch.cat((c.k[s][h // G], kd[s, :n, h // G].double()))
            v = torch.cat((c.v[s][h // G], vd[s, :n, h // G].double()))
            m = torch.cat((torch.ones((n, c.lens[s]), dtype=torch.bool), sees[s, :n, :n]), 1)
            o, _, b = attend(q[s, :n, h].double(), k, v, m, scale)
            want[s, :n, h], bound[s, :n, h] = o, b
    return want, bound


def _run(c, q, kd, vd, words, counts, T, splits=0, out=None, ws=None, scale=None):
    desc = c.desc(pe, q.shape[2], decode_splits=splits)
    kp, vp, table, lens = c.to(DEV)
    if out is None:
        out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    if ws is None:
        ws = pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T)
        if ws is not None:
            ws.fill_(0xff)   # NaN wherever nothing is written
    dl = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
    pe.pe_tree_decode(desc, T, q.to(DEV), kd.to(DEV), vd.to(DEV), dl, words.to(DEV), kp, vp, table, lens,
                      q.shape[3] ** -0.5 if scale is None else scale, out, ws)
    return out


def _check(out, want, bound, counts, dtype):
    for s, n in enumerate(counts):
        assert_close(out[s, :n], want[s, :n], bound[s, :n], dtype)
        assert bool((out[s, n:] == 7.0).all()), "rows behind the last draft of sequence %d were written" % s


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D,B,Hk,G,T,shared", [
    (64, 16, 2, 1, 1, False), (128, 16, 2, 4, 1, True), (64, 32, 3, 4, 4, True), (128, 16, 1, 8, 3, False), (128, 64, 2, 3, 7, False),
    (64, 16, 1, 5, 7, False), (128, 128, 2, 4, 8, True), (64, 128, 2, 7, 9, False), (128, 32, 2, 2, 17, True), (128, 16, 2, 1, 33, False),
    (64, 64, 1, 6, 31, True), (128, 16, 1, 4, 64, False), (64, 16, 2, 8, 64, False), (128, 32, 1, 8, 63, True)])
def test_tree_against_64_bits(dt, D, B, Hk, G, T, shared):
    """Empty caches, one token, pages that end inside a step, ragged trees (one of them without a draft), every split count."""
    print("case tree", dt, D, B, Hk, G, T, shared, flush=True)
    lens = [0, 1, 15, 16, 33, 100, 257, 700]
    counts = [T, max(1, T - 1), T, T, 0, max(1, T // 2), T, T]
    c, q, kd, vd, sees, words = _case(T * 100 + D + B + G, lens, counts, T, Hk, G, D, B, DTYPES[dt], shared)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    for splits in (0, 1, 2, 5):
        _check(_run(c, q, kd, vd, words, counts, T, splits), want, bound, counts, DTYPES[dt])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["chain", "any"])
def test_masks_that_are_no_tree_and_rows_that_see_nothing(dt, kind):
    """A chain, and arbitrary sets of drafts: later ones, and none at all, which over an empty cache gives zeros."""
    print("case masks", dt, kind, flush=True)
    T, G = 20, 4
    lens, counts = [0, 40, 0], [T, T, 13]
    c, q, kd, vd, sees, words = _case(5, lens, counts, T, 2, G, 128, 16, DTYPES[dt], False, kind)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    for splits in (1, 3):
        out = _run(c, q, kd, vd, words, counts, T, splits)
        _check(out, want, bound, counts, DTYPES[dt])
        if kind == "any":
            assert bool((out[0, 4] == 0).all()) and bool((out[2, 9] == 0).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_large_logits(dt):
    """Logits of several hundred: one token takes nearly everything, and the references move often."""
    print("case large", dt, flush=True)
    T, G = 12, 3
    lens, counts = [900, 64], [T, 5]
    c, q, kd, vd, sees, words = _case(6, lens, counts, T, 2, G, 64, 32, DTYPES[dt], True, scale=30.0)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    for splits in (1, 4):
        _check(_run(c, q, kd, vd, words, counts, T, splits), want, bound, counts, DTYPES[dt])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 16, 60])
@pytest.mark.parametrize("scale", [0.0, -0.25, 1.5])
def test_any_finite_scale(dt, T, scale):
    """Zero weighs all alike, a negative one prefers the smallest product."""
    print("case scale", dt, T, scale, flush=True)
    lens, counts, G = [130, 0, 17], [T, T, 2], 4
    c, q, kd, vd, sees, words = _case(7, lens, counts, T, 1, G, 128, 16, DTYPES[dt], False, "any")
    want, bound = _want(c, q, kd, vd, sees, counts, G, scale)
    for splits in (1, 2):
        _check(_run(c, q, kd, vd, words, counts, T, splits, scale=scale), want, bound, counts, DTYPES[dt])


def test_one_draft_is_a_decode_step():
    """One draft that sees itself: what pe_append_paged_decode gives for a new token, without the append."""
    print("case one draft", flush=True)
    lens, G, Hk, D = [0, 5, 300, 1024], 4, 2, 128
    c, q, kd, vd, sees, words = _case(8, lens, [1] * 4, 1, Hk, G, D, 16, torch.bfloat16, False)
    out = _run(c, q, kd, vd, words, None, 1)
    want, bound = _want(c, q, kd, vd, sees, [1] * 4, G)
    kp, vp, table, sl = c.to(DEV)
    spare = torch.arange(c.pages, c.pages + 4 * Hk, dtype=torch.int32, device=DEV).view(4, Hk, 1)
    kp, vp = (torch.cat((x, torch.zeros((4 * Hk, 16, D), dtype=x.dtype, device=DEV))) for x in (kp, vp))
    desc = pe.make_desc(torch.bfloat16, 4, Hk, Hk * G, D, 16, c.max_blocks, kp.shape[0])
    got, after = torch.empty((4, Hk * G, D), dtype=torch.bfloat16, device=DEV), torch.empty_like(sl)
    freed, used = torch.full((4, Hk), -1, dtype=torch.int32, device=DEV), torch.zeros((4, Hk), dtype=torch.int32, device=DEV)
    pe.pe_append_paged_decode(desc, kd[:, 0].contiguous().to(DEV), vd[:, 0].contiguous().to(DEV), q[:, 0].contiguous().to(DEV), kp, vp, table,
                              sl, after, freed, spare, used, D ** -0.5, got, pe.alloc_workspace(pe.PE_OP_APPEND_PAGED_DECODE, desc))
    assert_close(out[:, 0], want[:, 0], bound[:, 0], torch.bfloat16)
    assert_close(got, want[:, 0], bound[:, 0], torch.bfloat16)


def test_tree_is_repeatable_in_place_and_on_a_side_stream():
    print("case repeat", flush=True)
    T, G = 16, 4
    lens, counts = [2000, 77, 0], [T, 9, T]
    c, q, kd, vd, sees, words = _case(9, lens, counts, T, 2, G, 128, 16, torch.bfloat16, False)
    first = _run(c, q, kd, vd, words, counts, T, 3)
    again = _run(c, q, kd, vd, words, counts, T, 3)
    assert torch.equal(first, again)
    desc = c.desc(pe, q.shape[2], decode_splits=3)
    kp, vp, table, sl = c.to(DEV)
    args = [kd.to(DEV), vd.to(DEV), torch.tensor(counts, dtype=torch.int32, device=DEV), words.to(DEV), kp, vp, table, sl]
    qd = q.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T)
        pe.pe_tree_decode(desc, T, qd, *args, 128 ** -0.5, qd, ws)   # the result takes the queries' place
    torch.cuda.current_stream().wait_stream(side)
    for s, n in enumerate(counts):
        assert torch.equal(qd[s, :n], first[s, :n])


def test_tree_in_a_graph():
    """Replays follow the lengths, the masks and the cache as they are at the time."""
    print("case graph", flush=True)
    T, G = 8, 4
    c, q, kd, vd, sees, words = _case(10, [500, 31], [T, T], T, 2, G, 64, 16, torch.bfloat16, False)
    desc = c.desc(pe, q.shape[2])
    kp, vp, table, sl = c.to(DEV)
    dev = [x.to(DEV) for x in (q, kd, vd)]
    dl, wd, out = torch.full((2,), T, dtype=torch.int32, device=DEV), words.to(DEV), torch.zeros(q.shape, dtype=q.dtype, device=DEV)
    ws = pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T)
    call = lambda to: pe.pe_tree_decode(desc, T, *dev, dl, wd, kp, vp, table, sl, 64 ** -0.5, to, ws)   # noqa: E731
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for n, m in ((500, 8), (123, 3), (16, 8), (0, 5)):
        sl[0], dl[0] = n, m
        out.zero_()
        graph.replay()
        want = torch.zeros_like(out)
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool(out[0, :m].abs().sum() > 0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D,B,Hk,T,shared", [(64, 16, 2, 5, False), (128, 16, 3, 40, True), (64, 128, 2, 64, False), (128, 32, 1, 33, False)])
def test_append_path_against_a_plain_copy(dt, D, B, Hk, T, shared):
    """Paths that end in the newest page, fill it, go on into the next, name a draft twice, are empty or end at what is no draft; the
    pools are compared whole."""
    print("case path", dt, D, B, Hk, T, shared, flush=True)
    g = torch.Generator().manual_seed(D + B + T)
    lens = [0, B - 1, B, 3 * B, 2 * B + 5, 7, 5, B]
    S, P = len(lens), 2 * B + 3
    dtype = DTYPES[dt]
    c = Cache(11, lens, Hk, D, B, dtype, shared, extra_blocks=3, extra_pages=0)
    rows, per_row = (1 if shared else Hk), 3
    more = S * rows * per_row
    kp, vp = (torch.cat((x, torch.full((more,) + x.shape[1:], NAN, dtype=dtype))) for x in (c.k_pool, c.v_pool))
    spare = torch.arange(c.pages, c.pages + more, dtype=torch.int32).view(S, rows, per_row)
    freed = torch.full((S, rows), -1, dtype=torch.int32)
    freed[3] = spare[3, :, 2]    # a page that an eviction has just freed goes first
    kd, vd = (torch.randn((S, T, Hk, D), generator=g).to(dtype) for _ in range(2))
    path = torch.randint(0, T, (S, P), generator=g).int()
    path_lens = torch.tensor([P, 1, 2, B + 3, 2 * B, 0, 9, P + 50], dtype=torch.int32)
    path[6, 4] = T               # no draft: the path ends in front of it
    squeeze = (lambda x: x[:, 0].contiguous()) if shared else (lambda x: x.contiguous())
    table, spare, freed = squeeze(c.table.view(S, rows, -1)), squeeze(spare), squeeze(freed)
    used = torch.zeros(freed.shape, dtype=torch.int32)
    want = [x.clone() for x in (kp, vp, table, c.seq_lens, freed, used)]
    done = torch.zeros(S, dtype=torch.int32)
    dev = [x.to(DEV) for x in (kp, vp, table, c.seq_lens, freed, used, done)]
    desc = pe.make_desc(dtype, S, Hk, 2 * Hk, D, B, c.max_blocks, kp.shape[0], pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    ins = [x.to(DEV) for x in (kd, vd, path, path_lens, spare)]
    for call in range(4):
        wk, wv, wt, wl, wf, wu = want
        for s in range(S):
            end = min(int(path_lens[s]), P)
            take = min(end - int(done[s]), B - int(wl[s]) % B)
            bad = [i for i in range(take) if not 0 <= int(path[s, int(done[s]) + i]) < T]
            take = bad[0] if bad else take
            for i in range(take):
                n, d = int(wl[s]), int(path[s, int(done[s])])
                for r in range(rows):
                    at = (s,) if shared else (s, r)
                    if n % B == 0:
                        if wf[at] >= 0:
                            wt[at][n // B], wf[at] = wf[at].clone(), -1
                        else:
                            wt[at][n // B] = spare[at][wu[at]]
                            wu[at] += 1
                    page = int(wt[at][n // B])
                    wk[page, n % B] = kd[s, d] if shared else kd[s, d, r]
                    wv[page, n % B] = vd[s, d] if shared else vd[s, d, r]
                wl[s] += 1
                done[s] += 1
        pe.pe_append_path(desc, ins[0], ins[1], ins[2], ins[3], dev[6], dev[0], dev[1], dev[2], dev[3], dev[4], ins[4], dev[5])
        torch.cuda.synchronize()
        bits = torch.int32 if dtype == torch.float32 else torch.int16
        for name, got, w in zip(("k_pool", "v_pool", "table", "seq_lens", "freed", "used"), dev, want):
            got = got.cpu()
            same = torch.equal(got.view(bits), w.view(bits)) if got.is_floating_point() else torch.equal(got, w)
            assert same, (call, name)
        assert torch.equal(dev[6].cpu(), done), call
    assert int(done[0]) == P and int(done[6]) == 4 and int(done[5]) == 0


def test_append_path_leaves_full_tables_and_negative_lengths_alone():
    print("case path bounds", flush=True)
    B, S, Hk, D, T = 16, 3, 2, 64, 4
    c = Cache(12, [2 * B, 2 * B, 5], Hk, D, B, torch.bfloat16, False, extra_blocks=0)
    kp, vp, table, lens = c.to(DEV)
    lens[1] = -3
    before = [x.clone() for x in (kp, vp, table, lens)]
    g = torch.Generator().manual_seed(1)
    kd, vd = (torch.randn((S, T, Hk, D), generator=g).bfloat16().to(DEV) for _ in range(2))
    path = torch.zeros((S, T), dtype=torch.int32, device=DEV)
    n, done = torch.tensor([2, 2, 0], dtype=torch.int32, device=DEV), torch.zeros(S, dtype=torch.int32, device=DEV)
    freed, used = torch.full((S, Hk), -1, dtype=torch.int32, device=DEV), torch.zeros((S, Hk), dtype=torch.int32, device=DEV)
    spare = torch.zeros((S, Hk, 1), dtype=torch.int32, device=DEV)
    pe.pe_append_path(c.desc(pe, Hk), kd, vd, path, n, done, kp, vp, table, lens, freed, spare, used)
    torch.cuda.synchronize()
    for a, b in zip((kp, vp, table, lens), before):
        assert torch.equal(a.nan_to_num(9.0) if a.is_floating_point() else a, b.nan_to_num(9.0) if b.is_floating_point() else b)
    assert int(done.sum()) == 0 and int(used.sum()) == 0


@pytest.mark.parametrize("splits", [0, 2, 5])
@pytest.mark.parametrize("D,shared", [(128, False), (64, True)])
def test_many_query_rows_of_sequences_of_very_different_lengths(D, shared, splits):
    """Eight query heads and 64 drafts a sequence; one long sequence, short and empty ones, and some without a draft: a sequence's share of
    the splits goes by its length, and none at all to one without a query."""
    print("case shares", D, shared, splits, flush=True)
    lens, counts, T, G = [0, 1, 64, 3000, 5, 700, 63, 65, 2000, 0], [64, 64, 5, 64, 0, 33, 64, 1, 0, 0], 64, 8
    c, q, kd, vd, sees, words = _case(31 + splits, lens, counts, T, 1, G, D, 16, torch.bfloat16, shared)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    _check(_run(c, q, kd, vd, words, counts, T, splits), want, bound, counts, torch.bfloat16)


@pytest.mark.parametrize("S", [2, 64, 65])
def test_many_query_rows_of_many_sequences(S):
    """As many sequences as have their splits shared out, one more, and two."""
    print("case sequences", S, flush=True)
    T, Hk, G = (40, 8, 8) if S == 2 else (33, 1, 4)
    lens, counts = [(37 * s) % 300 for s in range(S)], [T - s % 3 for s in range(S)]
    c, q, kd, vd, sees, words = _case(S, lens, counts, T, Hk, G, 64, 32, torch.bfloat16, False)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    for splits in (0, 3):
        _check(_run(c, q, kd, vd, words, counts, T, splits), want, bound, counts, torch.bfloat16)
