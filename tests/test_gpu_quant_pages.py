"""A cache's way into 8 bits: whole pages (pe_quant_pages) and a step's token (pe_quant_append), number for number."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import DTYPES, Cache, assert_close
from _quant64 import E4M3, page_score, round_page
from _tokens64 import frequencies, rotate

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")


class Held:
    """An 8-bit cache on the GPU, filled with junk."""

    def __init__(self, desc, shared, dtype):
        heads = (desc.num_kv_heads,) if shared else ()
        pool = (desc.num_phys_blocks, desc.block_size) + heads + (desc.head_dim,)
        tail = (desc.num_seqs, desc.num_kv_heads, desc.block_size, desc.head_dim)
        self.shared = shared
        self.k, self.v = (torch.full(pool, 0xee, dtype=torch.uint8, device=DEV) for _ in range(2))
        self.scales = torch.full((desc.num_phys_blocks,) + heads + (2,), 77.0, device=DEV)
        self.k_tail, self.v_tail = (torch.full(tail, 5.0, dtype=dtype, device=DEV) for _ in range(2))
        self.cache = pe.make_quant_cache(desc, self.k, self.v, self.scales, self.k_tail, self.v_tail)

    def page(self, page, h):
        at = (page, slice(None), h) if self.shared else (page,)
        s = self.scales[page, h] if self.shared else self.scales[page]
        return self.k[at].cpu(), self.v[at].cpu(), s.tolist()

    def untouched(self, pages):
        rest = torch.ones(self.k.shape[0], dtype=torch.bool, device=DEV)
        rest[list(pages)] = False
        return bool((self.k[rest] == 0xee).all()) and bool((self.v[rest] == 0xee).all()) and bool((self.scales[rest] == 77.0).all())


def _steps(a, b):
    """How many fp32 numbers lie between."""
    return abs(int(torch.tensor(a).view(torch.int32)) - int(torch.tensor(b, dtype=torch.float32).view(torch.int32)))


def _pages(seed, lens, Hk, D, B, dt, shared, change=None, scores=True, same=False, **kw):
    dtype = DTYPES[dt]
    c = Cache(seed, lens, Hk, D, B, dtype, shared, **kw)
    if change:
        change(c)
    desc = c.desc(pe, Hk)
    kp, vp, src, sl = c.to(DEV)
    moved = torch.randperm(c.pages, generator=torch.Generator().manual_seed(seed)).int()
    dst = c.table if same else torch.where(c.table >= 0, moved[c.table.clamp(min=0).long()], c.table)
    held = Held(desc, shared, dtype)
    sc = torch.full((len(lens), Hk, c.max_blocks), -3.0, device=DEV) if scores else None
    pe.pe_quant_pages(desc, held.cache, kp, vp, src, sl, src if same else dst.to(DEV), sc)
    torch.cuda.synchronize()
    used = set()
    for s, n in enumerate(lens):
        for h in range(Hk):
            for j in range(n // B):
                a = int(c.table[s, j] if shared else c.table[s, h, j])
                b = int(dst[s, j] if shared else dst[s, h, j])
                if a < 0 or b < 0:
                    assert float(sc[s, h, j]) == INF
                    continue
                used.add(b)
                k, v = (p[a, :, h] if shared else p[a] for p in (c.k_pool, c.v_pool))
                got_k, got_v, got_s = held.page(b, h)
                for x, got, scale in ((k, got_k, got_s[0]), (v, got_v, got_s[1])):
                    want, s2 = round_page(x)
                    assert scale == s2 and torch.equal(got, want), (s, h, j)
                if scores:
                    assert _steps(float(sc[s, h, j]), page_score(k, v)) <= (0 if dt == "bf16" and page_score(k, v) < 1e30 else 1) + 1
            if scores:
                assert bool((sc[s, h, n // B:] == INF).all())
            for tail, x in ((held.k_tail, c.k_pool), (held.v_tail, c.v_pool)):
                j = n // B
                if n % B:
                    a = int(c.table[s, j] if shared else c.table[s, h, j])
                    if a >= 0:
                        assert torch.equal(tail[s, h, :n % B].cpu(), (x[a, :, h] if shared else x[a])[:n % B])
                assert bool((tail[s, h, n % B:] == 5.0).all())
    assert held.untouched(used)
    return c, desc, held, sc, kp, vp, src, sl


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B", [16, 32, 64, 128])
def test_pages(B, D, dt, shared):
    c, desc, held, sc, kp, vp, src, sl = _pages(B + D, [0, 1, B - 1, B, B + 1, 3 * B, 5 * B + 7], 3, D, B, dt, shared)
    # the scores that the uncompressed cache has
    want = torch.empty_like(sc)
    pe.pe_score_blocks(desc, kp, vp, src, sl, want)
    same = (sc.view(torch.int32) - want.view(torch.int32)).abs().max()
    assert int(same) <= (0 if dt == "bf16" else 1)


def test_without_scores_and_into_the_same_pages():
    _pages(1, [50, 16, 200], 2, 64, 16, "bf16", False, scores=False)
    _pages(2, [50, 16, 200], 2, 64, 16, "bf16", False, same=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [False, True])
def test_hard_pages(dt, shared):
    """All zeros; one element alone, at the edge of a scale and beside it; halves between two e4m3 numbers; next to the largest and smallest."""
    dtype = DTYPES[dt]

    def change(c):
        for pool in (c.k_pool, c.v_pool):
            view = lambda s, j: (pool[c.table[s, j], :, 0] if shared else pool[c.table[s, 0, j]])   # noqa: E731
            view(0, 0).zero_()
            for j, top in enumerate((448.0, 450.0, 2.0 ** 127, 2.0 ** -120, 2.0 ** -126, 448 * 2.0 ** 20, 446.0, 1.0)):
                p = view(1, j)
                p.zero_()
                p[3, 5] = -top
            p = view(0, 1)
            every = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).float()           # 0 .. 448
            ties = (every[1:] + every[:-1]) / 2
            flat = torch.cat((ties, -ties, every, -every, ties * (1 + 2.0 ** -7), ties * (1 - 2.0 ** -7)))
            p.copy_(flat[:p.numel()].repeat(1 + p.numel() // flat.numel())[:p.numel()].view(p.shape).to(dtype))
            p[0, 0] = 448.0
    _pages(3, [40, 130], 2, 64, 16, dt, shared, change)


def test_missing_pages():
    def change(c):
        c.table[0, 0, 1] = -1
        c.table[1, 1, 2] = -1
    _pages(4, [50, 40], 2, 64, 16, "bf16", False, change)


def test_lengths_behind_the_table():
    """A length that the table does not hold is the caller's mistake: what the table has is rounded."""
    c = Cache(5, [32, 32], 2, 64, 16, torch.bfloat16, False, extra_blocks=0)
    desc = c.desc(pe, 2)
    kp, vp, table, sl = c.to(DEV)
    held = Held(desc, False, torch.bfloat16)
    sl.copy_(torch.tensor([5000, -7], dtype=torch.int32))
    sc = torch.zeros((2, 2, 2), device=DEV)
    pe.pe_quant_pages(desc, held.cache, kp, vp, table, sl, table, sc)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(sc[0]).all()) and bool((sc[1] == INF).all())
    assert held.untouched(c.table[0].flatten().tolist()) and bool((held.k_tail == 5.0).all())


# ---- a step's token ----

def _grow(seed, start, steps, Hk, G, D, B, dt, shared, R=0, inter=False, keep_scores=True, in_place=False, n_spare=6, max_blocks=None):
    """Sequences grow token by token from a rounded cache of `start` tokens; everything is checked behind every step."""
    dtype = DTYPES[dt]
    S = len(start)
    c = Cache(seed, start, Hk, D, B, dtype, shared, extra_blocks=steps // B + 2 if max_blocks is None else 0, extra_pages=S * Hk * (n_spare + 1))
    g = torch.Generator().manual_seed(seed + 5)
    used = set(c.table[c.table >= 0].tolist())
    spares = [i for i in range(c.pages) if i not in used]
    rows = (S,) if shared else (S, Hk)
    n = S * (1 if shared else Hk)
    spare = torch.tensor(spares[:n * n_spare], dtype=torch.int32).view(rows + (n_spare,))
    freed = torch.full(rows, -1, dtype=torch.int32)
    freed.view(-1)[::2] = torch.tensor(spares[n * n_spare:n * n_spare + (n + 1) // 2], dtype=torch.int32)
    desc = c.desc(pe, Hk * G)
    kp, vp, table, sl = c.to(DEV)
    held = Held(desc, shared, dtype)
    sc = torch.zeros((S, Hk, c.max_blocks), device=DEV)
    pe.pe_quant_pages(desc, held.cache, kp, vp, table, sl, table, sc)
    rope = pe.make_rope(R, 10000.0, interleaved=inter, magnitude=1.25) if R else None
    f = frequencies(R, 10000.0) if R else None
    d_spare, d_freed, d_used = spare.to(DEV), freed.to(DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    want_table, want_freed, want_used = c.table.clone(), freed.clone(), torch.zeros(rows, dtype=torch.int32)
    lens, other = list(start), torch.empty_like(sl)
    shadow = [[([], []) for _ in range(Hk)] for _ in range(S)]       # what the tail holds
    for s in range(S):
        for h in range(Hk):
            for i, t in enumerate((held.k_tail, held.v_tail)):
                shadow[s][h][i].extend(t[s, h, :lens[s] % B].cpu())
    for step in range(steps):
        k, v = (torch.randn((S, Hk, D), generator=g).to(dtype) for _ in range(2))
        q = torch.randn((S, Hk * G, D), generator=g).to(dtype)
        pos = torch.randint(0, 100000, (S,), generator=g, dtype=torch.int32)
        qd = q.to(DEV)
        qo = qd if in_place else torch.full_like(qd, 3.0)
        pe.pe_quant_append(desc, held.cache, rope, pos.to(DEV) if R else None, qd, qo, k.to(DEV), v.to(DEV), table, sl, other, d_freed, d_spare, d_used,
                           sc if keep_scores else None)
        sl, other = other, sl
        torch.cuda.synchronize()
        if R:
            assert_close(qo, *rotate(q, pos, f, inter, 1.25), dtype)
            turned = rotate(k, pos, f, inter, 1.25)
        else:
            assert in_place or bool((qo == 3.0).all())
        for s in range(S):
            slot, j = lens[s] % B, lens[s] // B
            if j >= c.max_blocks:
                continue
            for r in range(1 if shared else Hk):
                at = (s,) if shared else (s, r)
                if slot == 0:
                    page = int(want_freed[at])
                    if page >= 0:
                        want_freed[at] = -1
                    else:
                        u = int(want_used[at])
                        page = int(spare[at][u]) if u < n_spare else -1
                        want_used[at] = u + 1
                    want_table[at][j] = page
            for h in range(Hk):
                if slot == 0:
                    shadow[s][h] = ([], [])
                now = held.k_tail[s, h, slot].cpu()
                if R:
                    assert_close(now, turned[0][s, h], turned[1][s, h], dtype)
                else:
                    assert torch.equal(now, k[s, h])
                shadow[s][h][0].append(now)
                shadow[s][h][1].append(v[s, h])
                for i, t in enumerate((held.k_tail, held.v_tail)):
                    assert torch.equal(t[s, h, :slot + 1].cpu(), torch.stack(shadow[s][h][i]))
                if slot == B - 1:
                    page = int(want_table[s, j] if shared else want_table[s, h, j])
                    kt, vt = (torch.stack(x) for x in shadow[s][h])
                    if page >= 0:
                        got_k, got_v, got_s = held.page(page, h)
                        for x, got, scale in ((kt, got_k, got_s[0]), (vt, got_v, got_s[1])):
                            b, s2 = round_page(x)
                            assert scale == s2 and torch.equal(got, b)
                        if keep_scores:
                            assert _steps(float(sc[s, h, j]), page_score(kt, vt)) <= 1
            lens[s] += 1
        assert sl.tolist() == lens
        assert torch.equal(table.cpu(), want_table) and torch.equal(d_freed.cpu(), want_freed) and torch.equal(d_used.cpu(), want_used)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt,D,B", [("bf16", 128, 16), ("bf16", 64, 32), ("f32", 64, 16), ("f32", 128, 128), ("bf16", 128, 64), ("bf16", 64, 128)])
def test_tokens_join(dt, D, B, shared):
    _grow(D + B, [0, B - 1, B, B - 2, 2 * B + 5], 5 if B > 32 else B + 3, 2, 2, D, B, dt, shared)


@pytest.mark.parametrize("R,inter", [(128, False), (128, True), (64, False), (30, True), (2, False)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_tokens_join_turned(dt, R, inter):
    _grow(R, [0, 15, 31, 14], 4, 2, 5, 128, 16, dt, False, R=R, inter=inter, in_place=inter)


def test_without_scores():
    _grow(3, [14, 15], 3, 2, 1, 64, 16, "bf16", True, keep_scores=False)


def test_spare_pages_that_run_out():
    """As with pe_append_kv the page is missing then: nothing is written for it."""
    _grow(4, [0, 16], 50, 2, 1, 64, 16, "bf16", False, n_spare=1)


def test_full_table_rows():
    _grow(5, [32, 30], 5, 2, 1, 64, 16, "bf16", False, max_blocks=2)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_replayed(dt):
    """A captured append, the lengths in two arrays: two graphs that take turns, eager copies of the same steps beside them."""
    dtype, S, Hk, D, B = DTYPES[dt], 3, 2, 64, 16
    start = [13, 30, 0]
    made = []
    for _ in range(2):
        c = Cache(6, start, Hk, D, B, dtype, False, extra_blocks=4, extra_pages=40)
        desc = c.desc(pe, Hk)
        kp, vp, table, sl = c.to(DEV)
        held = Held(desc, False, dtype)
        sc = torch.zeros((S, Hk, c.max_blocks), device=DEV)
        pe.pe_quant_pages(desc, held.cache, kp, vp, table, sl, table, sc)
        used = set(c.table[c.table >= 0].tolist())
        spares = [i for i in range(c.pages) if i not in used]
        spare = torch.tensor(spares[:S * Hk * 4], dtype=torch.int32, device=DEV).view(S, Hk, 4)
        freed, count = torch.full((S, Hk), -1, dtype=torch.int32, device=DEV), torch.zeros((S, Hk), dtype=torch.int32, device=DEV)
        made.append((desc, held, table, [sl, torch.zeros_like(sl)], freed, spare, count, sc))
    k, v = (torch.zeros((S, Hk, D), dtype=dtype, device=DEV) for _ in range(2))
    q, pos = torch.zeros((S, Hk, D), dtype=dtype, device=DEV), torch.zeros(S, dtype=torch.int32, device=DEV)
    rope = pe.make_rope(D, 10000.0)

    def call(m, i, out):
        desc, held, table, lens, freed, spare, count, sc = m
        pe.pe_quant_append(desc, held.cache, rope, pos, q, out, k, v, table, lens[i], lens[1 - i], freed, spare, count, sc)
    outs = [torch.zeros_like(q) for _ in range(2)]
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            call(made[0], i, outs[0])
    g = torch.Generator().manual_seed(2)
    for step in range(21):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g))
        pos.copy_(torch.randint(0, 9999, (S,), generator=g, dtype=torch.int32))
        graphs[step % 2].replay()
        call(made[1], step % 2, outs[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        for a, b in zip(made[0][2:], made[1][2:]):
            assert all(torch.equal(x, y) for x, y in zip(a, b)) if isinstance(a, list) else torch.equal(a, b)
        for name in ("k", "v", "scales", "k_tail", "v_tail"):
            assert torch.equal(getattr(made[0][1], name), getattr(made[1][1], name)), (step, name)
