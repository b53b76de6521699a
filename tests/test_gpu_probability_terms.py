"""How much of a probability goes into the products with V where a bfloat16 cache is attended to for several query rows: values that cancel
leave an output so small that its own rounding does not hide what the probabilities lost."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _two_tokens(S, Hk, rows, D, seed):
    """Caches of two tokens with keys e_0 and -e_0 and queries x e_0 (|x| <= 1): logits x and -x, exact sums.  Value 0 is all ones; element
    d of value 1 is the bfloat16 number next to -exp(2 x) of query row d, whose output there is what is left of two equal parts."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.rand((S, Hk, rows), generator=g) * 2 - 1).bfloat16()
    pages = S * Hk
    kp, vp = (torch.zeros((pages, 16, D), dtype=torch.bfloat16) for _ in range(2))
    kp[:, 0, 0], kp[:, 1, 0] = 1, -1
    vp[:, 0] = 1
    n = min(rows, D)
    vp.view(S, Hk, 16, D)[:, :, 1, :n] = -torch.exp(2 * x[..., :n].double()).bfloat16()
    table = torch.arange(pages, dtype=torch.int32).view(S, Hk, 1)
    return x, [t.to(DEV) for t in (kp, vp, table, torch.full((S,), 2, dtype=torch.int32))]


def _check(got, x, vp):
    """got [S, Hk, rows, D].  A probability p goes in as a bfloat16 number next to it and one next to the rest: off by 2^-9 of 2^-8 p, half
    steps both.  The other 2^-19 are what is done in 32 bits, of arguments up to 4.5 (log2): the logit, its scale and the reference taken off
    (3 times 4.5 2^-24 ln 2), exp2 (2^-23), two sums and a quotient (4 times 2^-24).  All relative to w_0 |v_0| + w_1 |v_1|."""
    S, Hk, rows, D = got.shape
    n = min(rows, D)
    w0 = torch.sigmoid(2 * x[..., :n].double())
    v1 = vp.cpu().double().view(S, Hk, 16, D)[:, :, 1, :n]
    want, size = w0 + (1 - w0) * v1, w0 + (1 - w0) * v1.abs()
    at = got.double().cpu()[:, :, torch.arange(n), torch.arange(n)]
    bound = (2.0 ** -17 + 2.0 ** -19) * size
    off = (at - want).abs()
    assert bool((want.abs() <= 2.0 ** -8 * size).all())   # (so that half a step of the output is no more than 2^-17 of it)
    far = off / (bound + 2.0 ** -9 * (want.abs() + bound))
    assert float(far.max()) <= 1, "%.2f times what is allowed, %d of %d" % (float(far.max()), int((far > 1).sum()), far.numel())


@pytest.mark.parametrize("S,Hk,G,T,D,splits", [(9, 2, 4, 4, 64, 1), (20, 1, 4, 4, 128, 2), (3, 3, 4, 16, 128, 1), (8, 8, 4, 8, 64, 3),
                                               (9, 2, 4, 32, 128, 1), (9, 3, 2, 64, 64, 2), (3, 3, 8, 60, 128, 1)])
def test_trees(S, Hk, G, T, D, splits):
    """Drafts that see the cache alone; sixteen, thirty-two and 256 query rows a workgroup."""
    print("case terms", S, Hk, G, T, D, splits, flush=True)
    x, (kp, vp, table, lens) = _two_tokens(S, Hk, T * G, D, T + D)
    q = torch.zeros((S, T, Hk * G, D), dtype=torch.bfloat16)
    q[..., 0] = x.view(S, Hk, T, G).permute(0, 2, 1, 3).reshape(S, T, Hk * G)
    kd, vd = (torch.zeros((S, T, Hk, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    desc = pe.make_desc(torch.bfloat16, S, Hk, Hk * G, D, 16, 1, S * Hk, decode_splits=splits)
    out = torch.empty(q.shape, dtype=q.dtype, device=DEV)
    pe.pe_tree_decode(desc, T, q.to(DEV), kd, vd, None, torch.zeros((S, T), dtype=torch.int64, device=DEV), kp, vp, table, lens, 1.0, out,
                      pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T))
    _check(out.view(S, T, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(S, Hk, T * G, D), x, vp)


@pytest.mark.parametrize("D,splits", [(64, 1), (128, 2)])
def test_page_weights(D, splits):
    print("case terms of weights", D, splits, flush=True)
    S, Hk, G = 40, 4, 8
    x, (kp, vp, table, lens) = _two_tokens(S, Hk, G, D, D)
    q = torch.zeros((S, Hk * G, D), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = x.view(S, Hk * G)
    desc = pe.make_desc(torch.bfloat16, S, Hk, Hk * G, D, 16, 1, S * Hk, decode_splits=splits)
    out, w = torch.empty_like(q), torch.empty((S, Hk, 1), device=DEV)
    pe.pe_paged_decode_weights(desc, q, kp, vp, table, lens, 1.0, 1.0, None, w, out, pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, desc))
    _check(out.view(S, Hk, G, D), x, vp)
