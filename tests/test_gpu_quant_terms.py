"""How much of a softmax weight goes into the products with V in attention over a cache in 8 bits: values that cancel leave an output so small
that its own rounding does not hide what the weights lost."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn


def _numbers(S, Hk, G, D, seed, rounded):
    """Queries (x0, x, 64) of every head and the values of three tokens: with keys (1, 0, 0), (0, 1, 0), (0, -1, 0) their logits are x0 >= 1.25, the
    largest, x and -x, exact sums.  The first one's value is 0, the second one's 1; element d of the third's is the number next to -exp(2 x) of
    query head d, whose output there is what is left of two equal parts.  rounded: that number is e4m3, and x next to what gives it."""
    g = torch.Generator().manual_seed(seed)
    x0 = (torch.rand((S, Hk, G), generator=g) * 0.75 + 1.25).bfloat16()
    if rounded:
        r = torch.arange(256, dtype=torch.uint8).view(E4M3).float()
        r = r[(r > 0.14) & (r < 7.3)]
        r = r[torch.randint(len(r), (S, Hk, G), generator=g)]
        x = (r.double().log() / 2).bfloat16()
    else:
        x = (torch.rand((S, Hk, G), generator=g) * 2 - 1).bfloat16()
        r = torch.exp(2 * x.double()).bfloat16()
    q = torch.zeros((S, Hk, G, D), dtype=torch.bfloat16)
    q[..., 0], q[..., 1], q[..., 2] = x0, x, 64
    k = torch.zeros((S * Hk, 16, D))
    k[:, 0, 0], k[:, 1, 1], k[:, 2, 1] = 1, 1, -1
    k[:, 3:, 2] = -64          # logits of -4096: no weight
    v = torch.zeros((S * Hk, 16, D))
    v[:, 1] = 1
    v.view(S, Hk, 16, D)[:, :, 2, :G] = -r.float()
    return x0, x, r.double(), q.view(S, Hk * G, D).to(DEV), k, v


def _check(out, x0, x, r):
    """A weight p goes in as a bfloat16 number next to it and one next to the rest: off by 2^-9 of 2^-8 p, half steps both.  The other 2^-19
    are what is done in 32 bits, half steps of 2^-24: the logit's scale and its product, 2.9 each, the reference taken off, 8 (a number up to
    8), ln 2 times; exp2, 2; a sum of three, a quotient, 4.  All relative to w_1 |v_1| + w_2 |v_2|."""
    w = torch.softmax(torch.stack((x0.double(), x.double(), -x.double())), 0)
    want, size = w[1] - w[2] * r, w[1] + w[2] * r
    assert bool((want.abs() <= 2.0 ** -8 * size).all())   # (so that half a step of the output is no more than 2^-16 of it)
    S, Hk, G = x.shape
    got = out.double().cpu().view(S, Hk, G, -1)[:, :, torch.arange(G), torch.arange(G)]
    bound = (2.0 ** -17 + 2.0 ** -19) * size
    far = (got - want).abs() / (bound + 2.0 ** -8 * (want.abs() + bound))
    assert float(far.max()) <= 1, "%.2f times what is allowed, %d of %d" % (float(far.max()), int((far > 1).sum()), far.numel())


@pytest.mark.parametrize("where", ["tail", "page"])
@pytest.mark.parametrize("D,G,splits", [(64, 4, 1), (64, 8, 2), (128, 4, 1), (128, 8, 1), (128, 2, 3)])
def test_terms_of_a_weight(D, G, splits, where):
    """Four and two classes a head; in the unfinished page, in the activations' type, and in a full one."""
    print("case quant terms", D, G, splits, where, flush=True)
    S, Hk = 400, 8
    x0, x, r, q, k, v = _numbers(S, Hk, G, D, D + G, where == "page")
    desc = pe.make_desc(torch.bfloat16, S, Hk, Hk * G, D, 16, 1, S * Hk, decode_splits=splits)
    if where == "page":
        k8, v8 = (t.to(E4M3).to(DEV) for t in (k, v))
        assert torch.equal(k8.float().cpu(), k) and torch.equal(v8.float().cpu(), v)
        tails = [torch.zeros((S, Hk, 16, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    else:
        k8, v8 = (torch.zeros((S * Hk, 16, D), dtype=torch.uint8, device=DEV) for _ in range(2))
        tails = [t.bfloat16().view(S, Hk, 16, D).to(DEV) for t in (k, v)]
    cache = pe.make_quant_cache(desc, k8, v8, torch.ones((S * Hk, 2), device=DEV), *tails)
    table = torch.arange(S * Hk, dtype=torch.int32, device=DEV).view(S, Hk, 1)
    lens = torch.full((S,), 16 if where == "page" else 3, dtype=torch.int32, device=DEV)
    out = torch.empty_like(q)
    pe.pe_quant_decode(desc, cache, q, table, lens, 1.0, out, pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc))
    _check(out, x0, x, r)
