"""Pages of an 8-bit cache, and slots, behind 32 bits of bytes and of elements."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import assert_close
from _quant64 import E4M3, attend, page_score, round_page

pytestmark = pytest.mark.gpu
DEV = "cuda"
B, D, HK, G = 16, 128, 2, 4


def test_far_pages():
    """Pages on both sides of 2^32 bytes (and for the unrounded pools of 2^32 elements), through every call."""
    per = B * D
    P = 2 ** 32 // per + 4
    S, lens = 2, [40, 31]
    far = [P - 1, 2 ** 32 // per, 2 ** 32 // per - 1, 0, P - 2, 5, 2 ** 31 // per, 7, P - 3, 9, 11, 13]
    table = torch.full((S, HK, 3), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(lens):
        for h in range(HK):
            for j in range(-(-n // B)):
                table[s, h, j] = far[at]
                at += 1
    desc = pe.make_desc(torch.bfloat16, S, HK, HK * G, D, B, 3, P)
    kp, vp = (torch.empty((P, B, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k8, v8 = (torch.empty((P, B, D), dtype=torch.uint8, device=DEV) for _ in range(2))
    scales = torch.empty((P, 2), device=DEV)
    kt, vt = (torch.zeros((S, HK, B, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cache = pe.make_quant_cache(desc, k8, v8, scales, kt, vt)
    g = torch.Generator().manual_seed(3)
    total = sum(lens)
    k, v = (torch.randn((total, HK, D), generator=g).to(torch.bfloat16) for _ in range(2))
    slots, t = torch.zeros((total, HK), dtype=torch.int64), 0
    for s, n in enumerate(lens):
        for i in range(n):
            slots[t] = table[s, :, i // B].long() * B + i % B
            t += 1
    rope, zero = pe.make_rope(D, 1e4), torch.zeros(total, dtype=torch.int32, device=DEV)   # (position 0: nothing turns)
    pe.pe_rotate(desc, rope, False, zero, None, k.to(DEV), v.to(DEV), None, None, slots.to(DEV), kp, vp)
    td, sl = table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    sc = torch.zeros((S, HK, 3), device=DEV)
    pe.pe_quant_pages(desc, cache, kp, vp, td, sl, td, sc)
    # the second sequence's page fills
    nk, nv = (torch.randn((S, HK, D), generator=g).to(torch.bfloat16) for _ in range(2))
    other, freed = torch.zeros_like(sl), torch.full((S, HK), -1, dtype=torch.int32, device=DEV)
    pe.pe_quant_append(desc, cache, None, None, None, None, nk.to(DEV), nv.to(DEV), td, sl, other, freed, torch.zeros((S, HK, 1), dtype=torch.int32, device=DEV),
                       torch.zeros((S, HK), dtype=torch.int32, device=DEV), sc)
    q = torch.randn((S, HK * G, D), generator=g).to(torch.bfloat16)
    out = torch.empty_like(q, device=DEV)
    pe.pe_quant_decode(desc, cache, q.to(DEV), td, other, D ** -0.5, out, pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, desc))
    torch.cuda.synchronize()
    start = 0
    for s, n in enumerate(lens):
        for h in range(HK):
            rows = []
            for i, (x, new, held) in enumerate(((k, nk, k8), (v, nv, v8))):
                x = torch.cat((x[start:start + n, h], new[s, h][None]))
                for j in range((n + 1) // B):
                    b, scale = round_page(x[j * B:(j + 1) * B])
                    assert torch.equal(held[int(table[s, h, j])].cpu(), b) and float(scales[int(table[s, h, j]), i]) == scale
                    if i:
                        assert abs(float(sc[s, h, j]) - page_score(whole[j * B:(j + 1) * B], x[j * B:(j + 1) * B])) <= 2.0 ** -22
                whole = x
                full = (n + 1) // B * B
                parts = [round_page(x[j * B:(j + 1) * B]) for j in range(full // B)]
                rows.append(torch.cat([b.view(E4M3).float().double() * s2 for b, s2 in parts] + [x[full:].double()]))
            want, bound = attend(q[s, h * G:(h + 1) * G].double(), rows[0], rows[1], torch.bfloat16)
            assert_close(out[s, h * G:(h + 1) * G], want, bound, torch.bfloat16)
        start += n
