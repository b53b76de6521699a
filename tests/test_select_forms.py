"""Scores of many pages: the form with sixteen loads a wave, over rows whose scores are whole numbers (so that every order of a sum gives
the same and many are equal); and that the rule takes these shapes there (on the CPU)."""
import os
import subprocess

import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd import build

from _paged64 import DTYPES, NAN

DEV = "cuda"
SHAPES = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)]
S, HK, PAGES = 16, 4, 2101   # sequences, heads, the longest row's pages
CHECK = r"""
#include <cstdio>
#include <cstdlib>
#include "%s/pe_select.h"
int main(int argc, char** argv) {
  printf("%%d\n", (int)pe::many_scores(atoll(argv[1]), atoi(argv[2]), atoi(argv[3]), atoi(argv[4]) != 0, 256));
}
"""


@pytest.fixture(scope="module")
def many(tmp_path_factory):
    d = tmp_path_factory.mktemp("scores")
    src, exe = d / "scores.hip", d / "scores"
    src.write_text(CHECK % build.CSRC)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc] + build.FLAGS + [str(src), "-o", str(exe)], check=True, stderr=subprocess.DEVNULL)
    return lambda *a: int(subprocess.run([str(exe)] + [str(x) for x in a], check=True, capture_output=True, text=True).stdout)


def test_which_scores_have_sixteen_loads_a_wave(many):
    for dt, D in SHAPES:
        assert many(S * HK, PAGES, D, int(dt == "bf16")) == 1
    for rows, pages, D, bf16, want in ((32, 4096, 128, 1, 1), (8, 4096, 128, 1, 0), (8, 1024, 128, 1, 0), (512, 1, 64, 1, 1), (511, 256, 64, 1, 0)):
        assert many(rows, pages, D, bf16) == want, (rows, pages)


@pytest.mark.gpu
@pytest.mark.parametrize("dt,D", SHAPES)
@pytest.mark.parametrize("k", [2, 300])
def test_selection_of_many_pages(dt, D, k):
    """Ragged rows, a few of them without a choice; what is not to be read has NaN bounds."""
    print("case many scores", dt, D, k, flush=True)
    B, G, dtype = 16, 2, DTYPES[dt]
    g = torch.Generator(device=DEV).manual_seed(D + k)
    lens = [PAGES * B, (PAGES - 1) * B + 1, 0, 1, k * B, k * B + 1, 1025 * B - 3] + [(137 * s % PAGES) * B + s for s in range(9)]
    assert len(lens) == S
    pages = S * HK * PAGES
    table = torch.randperm(pages, generator=g, device=DEV).int().view(S, HK, PAGES)
    used = torch.arange(PAGES, device=DEV) < torch.tensor([-(-n // B) for n in lens], device=DEV)[:, None, None]
    table = torch.where(used, table, torch.full_like(table, -1))
    q = torch.randint(-3, 4, (S, HK * G, D), generator=g, device=DEV).to(dtype)
    bounds = torch.full((pages, 2, D), NAN, dtype=dtype, device=DEV)
    want = torch.full((S, HK, k), -1, dtype=torch.int32)
    want_lens = torch.zeros(S, dtype=torch.int32)
    for s, length in enumerate(lens):
        n = -(-length // B)
        want_lens[s] = length if n <= k else (k - 1) * B + length - (n - 1) * B
        for h in range(HK):
            if n <= k:
                want[s, h, :n] = torch.arange(n)
                continue
            lo = torch.randint(-4, 3, (n - 1, D), generator=g, device=DEV)
            hi = lo + torch.randint(0, 3, (n - 1, D), generator=g, device=DEV)
            at = table[s, h, :n - 1].long()
            bounds[at, 0], bounds[at, 1] = lo.to(dtype), hi.to(dtype)
            x = q[s, h * G:(h + 1) * G].double()
            score = torch.zeros(n - 1, dtype=torch.float64, device=DEV)
            for i in range(G):   # (no product of matrices: the sum of the larger of two products, element by element)
                score += torch.maximum(x[i] * lo, x[i] * hi).sum(1)
            best = torch.sort(score, descending=True, stable=True).indices[:k - 1].sort().values
            want[s, h] = torch.cat((best.cpu(), torch.tensor([n - 1]))).int()
    desc = pe.make_desc(dtype, S, HK, HK * G, D, B, PAGES, pages)
    to, idx = (torch.full((S, HK, k), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    out_lens = torch.full((S,), -9, dtype=torch.int32, device=DEV)
    ws = pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, desc)
    ws.fill_(0x7f)
    pe.pe_select_pages(desc, q, bounds, table, torch.tensor(lens, dtype=torch.int32, device=DEV), k, to, out_lens, idx, ws)
    assert torch.equal(out_lens.cpu(), want_lens)
    assert torch.equal(idx.cpu(), want)
    pick = torch.where(want >= 0, table.cpu().gather(-1, want.clamp(min=0).long()), torch.full_like(want, -1))
    assert torch.equal(to.cpu(), pick)
