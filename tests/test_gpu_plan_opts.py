"""What a plan of tokens does beside the plan (pe_plan_tokens_ex), against a plain loop over the sequences."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _served(lens, new, budget, left, rows, n_spare, width, B):
    """Which sequences get what they need: 0, or 1 (from no token on), 2."""
    answer, at, short = [], 0, False
    for n, m in zip(lens, new):
        m = max(m, 0)
        kept = max(n, min(n + m, budget)) if budget else n + m
        need = rows * (-(-kept // B) - -(-n // B) + (n_spare if n == 0 and m > 0 else 0))
        ok = -(-kept // B) <= width
        if ok and need:
            short = short or at + need > left
            ok = not short
            at += need if ok else 0
        answer.append(0 if not ok or m == 0 else 1 if n == 0 else 2)
    return answer


class _Call:
    def __init__(self, lens, new, rows, B, width, budget=0, n_spare=0, left=10 ** 6, shared=False, seed=0):
        S = len(lens)
        self.lens, self.new, self.rows, self.B, self.width, self.budget, self.n_spare = lens, new, rows, B, width, budget, n_spare
        self.left = min(left, 4 * S * rows * (width + n_spare))
        self.desc = pe.make_desc(torch.bfloat16, S, 2 if shared else rows, 2 if shared else rows, 64, B, width, 1 << 20,
                                 pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
        g = torch.Generator().manual_seed(seed)
        self.free, self.used = torch.randperm(3 + self.left, generator=g).int().to(DEV), _i32([3])
        self.table = torch.arange(S * rows * width, dtype=torch.int32, device=DEV).view(S, rows, width)
        self.spare = torch.full((S, rows, n_spare), -1, dtype=torch.int32, device=DEV) if n_spare else None
        self.total = sum(max(m, 0) for m in new)

    def run(self, **opts):
        S = len(self.lens)
        out = [torch.zeros(n, dtype=torch.int32, device=DEV) for n in (S, 1, S + 1, self.total)]
        slots = torch.zeros((self.total, self.rows), dtype=torch.int64, device=DEV)
        table, spare = self.table.clone(), None if self.spare is None else self.spare.clone()
        pe.pe_plan_tokens(self.desc, _i32(self.lens), _i32(self.new), None, self.total, self.budget, self.free, self.used, table, spare, *out, slots, **opts)
        torch.cuda.synchronize()
        return [t.tolist() for t in out] + [slots.tolist(), table.tolist(), None if spare is None else spare.tolist()]

    def served(self):
        return _served(self.lens, self.new, self.budget, self.left, self.rows, self.n_spare, self.width, self.B)


CASES = [
    dict(lens=[0, 7, 0, 0, 64, 0], new=[33, 2, 0, 16, 1, -3], rows=2, B=16, width=8, n_spare=1),
    dict(lens=[0, 0, 0, 48, 80], new=[200, 64, 63, 30, 5], rows=2, B=16, width=8, budget=64, n_spare=1),
    dict(lens=[0, 0, 20, 30, 0, 0, 0], new=[40, 100, 2, 1, 17, 50, 300], rows=3, B=16, width=8, n_spare=2, left=25),
    dict(lens=[0, 16, 0], new=[17, 0, 1], rows=1, B=16, width=4, shared=True, left=2),
    dict(lens=[0] * 300 + [5] * 300, new=[3, 40, 0] * 200, rows=2, B=16, width=4, n_spare=1, left=900)]


@pytest.mark.parametrize("case", CASES)
def test_who_was_admitted(case):
    """And the plan itself is what it is without the question."""
    c = _Call(**case)
    admitted = torch.full((len(c.lens),), -9, dtype=torch.int32, device=DEV)
    assert c.run(admitted=admitted) == c.run()
    assert admitted.tolist() == c.served()
