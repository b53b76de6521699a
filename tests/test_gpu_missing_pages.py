"""Rows that lack pages, as a plan leaves them that found too few, stepped all the same: nothing outside the pools is read or written, and the
other rows are what they are."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt,D,B", [(torch.bfloat16, 128, 16), (torch.float32, 64, 32), (torch.bfloat16, 64, 128), (torch.float32, 128, 16)])
def test_scores(dt, D, B, shared):
    """A missing page is read as page 0, by all ways to a score."""
    print("case scores", dt, D, B, shared, flush=True)
    S, Hk, n = 3, 2, 6
    heads, rows = ((Hk,), ()) if shared else ((), (Hk,))
    P = S * (1 if shared else Hk) * n + 1
    g = torch.Generator().manual_seed(D + B)
    kp, vp = (torch.randn((P, B) + heads + (D,), generator=g).to(dt).to(DEV) for _ in range(2))
    whole = (torch.randperm(P - 1, generator=g).int() + 1).view((S,) + rows + (n,)).to(DEV)
    table, zero = whole.clone(), whole.clone()
    for where in ((0,), (1, ...) + (slice(2, 4),), (2, ...) + (n - 1,)):   # all pages of a sequence, two, the last one
        table[where], zero[where] = -1, 0
    desc = pe.make_desc(dt, S, Hk, Hk, D, B, n, P, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    lens = _i32([n * B] * S)

    def all_ways(t):
        got = []
        for call in (lambda o: pe.pe_score_blocks(desc, kp, vp, t, lens, o), lambda o: pe.pe_score_recent_blocks(desc, kp, vp, t, lens, 3, o),
                     lambda o: pe.pe_score_triggered_blocks(desc, kp, vp, t, lens, 2 * B, o)):
            o = torch.full((S, Hk, n), 7.0, device=DEV)
            call(o)
            got.append(o)
        if not shared:   # in one pass with the eviction, whose choice goes by the same scores
            o, at, freed, t2, l2 = torch.full((S, Hk, n), 7.0, device=DEV), *(torch.full((S, Hk), -9, dtype=torch.int32, device=DEV) for _ in range(2)), t.clone(), lens.clone()
            pe.pe_score_evict(desc, kp, vp, t2, l2, 2 * B, o, at, freed)
            got += [o, at, l2]
            assert torch.equal(freed, t.gather(2, at.long()[..., None])[..., 0])
        torch.cuda.synchronize()
        return got

    for a, b in zip(all_ways(table), all_ways(zero)):
        assert torch.equal(a, b)
