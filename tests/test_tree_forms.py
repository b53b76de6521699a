"""Trees with many query rows: the form that 256 query rows a workgroup have of their own (bfloat16), by every kind of mask, scale and
use; and that the rule takes these shapes there (on the CPU), so that another rule does not leave the form without tests."""
import os
import subprocess

import pytest
import torch

from paper_2509_04377_amd import binding as pe
from paper_2509_04377_amd import build

from _paged64 import assert_close
from test_gpu_tree import _case, _check, _run, _want

DEV = "cuda"
WIDE = [(3, 3, 8, 60), (3, 3, 8, 33), (2, 8, 4, 64)]   # sequences, KV heads, query heads of each, drafts
CHECK = r"""
#include <cstdio>
#include <cstdlib>
#include "%s/pe_rows.h"
int main(int argc, char** argv) {
  printf("%%d\n", pe::tree_tile_rows(atoi(argv[1]) != 0, atoll(argv[2]), atoi(argv[3]), 256));
}
"""


@pytest.fixture(scope="module")
def tile_rows(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    src, exe = d / "forms.hip", d / "forms"
    src.write_text(CHECK % build.CSRC)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc] + build.FLAGS + [str(src), "-o", str(exe)], check=True, stderr=subprocess.DEVNULL)
    return lambda *a: int(subprocess.run([str(exe)] + [str(x) for x in a], check=True, capture_output=True, text=True).stdout)


def test_which_trees_have_256_rows_a_workgroup(tile_rows):
    for S, Hk, G, T in WIDE:
        assert tile_rows(1, S * Hk, T * G) == 256 and tile_rows(0, S * Hk, T * G) == 32, (S, Hk, G, T)
    for kv_rows, rows, want in ((1, 16, 16), (64, 17, 32), (1, 512, 16), (9, 64, 32), (17, 128, 256)):
        assert tile_rows(1, kv_rows, rows) == want, (kv_rows, rows)


@pytest.mark.gpu
@pytest.mark.parametrize("D,shared", [(128, False), (64, True)])
@pytest.mark.parametrize("scale", [0.0, -0.25, 1.5])
def test_any_finite_scale(D, shared, scale):
    """Zero weighs all alike, a negative one prefers the smallest product; arbitrary masks, an empty cache, one without a draft."""
    print("case wide scale", D, shared, scale, flush=True)
    S, Hk, G, T = WIDE[0]
    lens, counts = [130, 0, 17], [T, T, 2]
    c, q, kd, vd, sees, words = _case(7, lens, counts, T, Hk, G, D, 16, torch.bfloat16, shared, "any")
    want, bound = _want(c, q, kd, vd, sees, counts, G, scale)
    for splits in (0, 1, 2):
        _check(_run(c, q, kd, vd, words, counts, T, splits, scale=scale), want, bound, counts, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["chain", "any"])
@pytest.mark.parametrize("D,shared", [(64, False), (128, True)])
def test_masks_that_are_no_tree_and_rows_that_see_nothing(D, shared, kind):
    print("case wide masks", D, shared, kind, flush=True)
    S, Hk, G, T = WIDE[1]
    lens, counts = [0, 200, 0], [T, T, 13]
    c, q, kd, vd, sees, words = _case(5, lens, counts, T, Hk, G, D, 32, torch.bfloat16, shared, kind)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    for splits in (0, 1, 3):
        out = _run(c, q, kd, vd, words, counts, T, splits)
        _check(out, want, bound, counts, torch.bfloat16)
        if kind == "any":
            assert bool((out[0, 4] == 0).all()) and bool((out[2, 9] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
def test_large_logits(D):
    """Logits of several hundred: the references move often, and one token takes nearly everything."""
    print("case wide large", D, flush=True)
    S, Hk, G, T = WIDE[1]
    lens, counts = [900, 64, 333], [T, 5, T]
    c, q, kd, vd, sees, words = _case(6, lens, counts, T, Hk, G, D, 32, torch.bfloat16, True, scale=30.0)
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    for splits in (1, 4):
        _check(_run(c, q, kd, vd, words, counts, T, splits), want, bound, counts, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("splits", [1, 3])
def test_in_place_of_the_queries_and_on_a_side_stream(splits):
    print("case wide in place", splits, flush=True)
    S, Hk, G, T = WIDE[0]
    lens, counts = [2000, 77, 0], [T, 9, T]
    c, q, kd, vd, sees, words = _case(9, lens, counts, T, Hk, G, 128, 16, torch.bfloat16, False)
    first = _run(c, q, kd, vd, words, counts, T, splits)
    assert torch.equal(first, _run(c, q, kd, vd, words, counts, T, splits))
    want, bound = _want(c, q, kd, vd, sees, counts, G)
    _check(first, want, bound, counts, torch.bfloat16)
    desc = c.desc(pe, q.shape[2], decode_splits=splits)
    kp, vp, table, sl = c.to(DEV)
    args = [kd.to(DEV), vd.to(DEV), torch.tensor(counts, dtype=torch.int32, device=DEV), words.to(DEV), kp, vp, table, sl]
    qd = q.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ws = pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T)
        pe.pe_tree_decode(desc, T, qd, *args, 128 ** -0.5, qd, ws)
    torch.cuda.current_stream().wait_stream(side)
    for s, n in enumerate(counts):
        assert torch.equal(qd[s, :n], first[s, :n])


@pytest.mark.gpu
def test_replays_follow_lengths_drafts_and_masks():
    """(The splits are shared out by lengths that only the device knows.)"""
    print("case wide graph", flush=True)
    S, Hk, G, T = WIDE[2]
    c, q, kd, vd, sees, words = _case(10, [900, 31], [T, T], T, Hk, G, 64, 16, torch.bfloat16, False)
    desc = c.desc(pe, q.shape[2], decode_splits=4)
    kp, vp, table, sl = c.to(DEV)
    dev = [x.to(DEV) for x in (q, kd, vd)]
    dl, wd, out = torch.full((2,), T, dtype=torch.int32, device=DEV), words.to(DEV), torch.zeros(q.shape, dtype=q.dtype, device=DEV)
    ws = [pe.alloc_workspace(pe.PE_OP_TREE_DECODE, desc, T) for _ in range(2)]
    call = lambda to, w: pe.pe_tree_decode(desc, T, *dev, dl, wd, kp, vp, table, sl, 64 ** -0.5, to, w)   # noqa: E731
    call(out, ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws[0])
    for n, m in ((900, T), (123, 3), (16, 40), (0, 5), (640, 0)):
        sl[0], dl[0] = n, m
        wd[1, 7] = n + 1
        out.zero_()
        graph.replay()
        want = torch.zeros_like(out)
        call(want, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool(out[1].abs().sum() > 0) and (bool(out[0, :m].abs().sum() > 0) or m == 0)
    sees[1, 7] = torch.tensor([641 >> j & 1 for j in range(T)], dtype=torch.bool)
    c.lens[0] = 640
    for rows in (c.k, c.v):
        rows[0] = [x[:640] for x in rows[0]]
    want, bound = _want(c, q, kd, vd, sees, [0, T], G)
    assert_close(out[1], want[1], bound[1], torch.bfloat16)
