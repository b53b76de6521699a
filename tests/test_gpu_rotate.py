"""Rotary positions (pe_rotate) against 64 bits: pairs, parts of a head, scalings, strides, places, and the way into the pages."""
import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _paged64 import DTYPES, assert_close
from _tokens64 import frequencies, rotate

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALES = {"none": {}, "linear": dict(scaling="linear", factor=8.0),
          "parts": dict(scaling="parts", factor=8.0, low=1.0, high=4.0, original=8192.0)}
HOW = {"none": pe.PE_ROPE_PLAIN, "linear": pe.PE_ROPE_LINEAR, "parts": pe.PE_ROPE_BY_PARTS}


def _rope(R, inter=False, scaling="none", base=500000.0, magnitude=1.0):
    more = {k: v for k, v in SCALES[scaling].items() if k != "scaling"}
    return pe.make_rope(R, base, interleaved=inter, scaling=HOW[scaling], magnitude=magnitude, **more), frequencies(R, base, **SCALES[scaling])


def _positions(T, g, far=120000):
    p = torch.randint(0, far, (T,), generator=g, dtype=torch.int32)
    p[0] = 0
    return p


def _case(seed, T, Hk, G, D, R, dt, inter=False, scaling="none", magnitude=1.0, transpose=False, positions=None):
    g = torch.Generator().manual_seed(seed)
    dtype = DTYPES[dt]
    q, k = (torch.randn((T, h, D), generator=g).to(dtype) for h in (Hk * G, Hk))
    pos = _positions(T, g) if positions is None else positions
    rope, f = _rope(R, inter, scaling, magnitude=magnitude)
    desc = pe.make_desc(dtype, 1, Hk, Hk * G, D, 16, 1, 1)
    want = [rotate(x, pos, f, inter, float(torch.tensor(magnitude).float()), transpose) for x in (q, k)]
    return desc, rope, pos.to(DEV), q, k, want


@pytest.mark.parametrize("scaling", ["none", "linear", "parts"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dt,D,R", [("bf16", 128, 128), ("bf16", 64, 64), ("f32", 128, 128), ("f32", 64, 64), ("bf16", 128, 64), ("bf16", 128, 32),
                                    ("f32", 64, 24), ("bf16", 64, 16), ("bf16", 128, 2), ("bf16", 64, 62), ("f32", 128, 126), ("bf16", 128, 40)])
def test_turned(dt, D, R, inter, scaling):
    desc, rope, pos, q, k, want = _case(R + D, 19, 3, 2, D, R, dt, inter, scaling, magnitude=1.25 if scaling == "parts" else 1.0)
    out = [torch.full_like(x, 7.0, device=DEV) for x in (q, k)]
    pe.pe_rotate(desc, rope, False, pos, q.to(DEV), k.to(DEV), None, *out)
    torch.cuda.synchronize()
    for got, (y, bound) in zip(out, want):
        assert_close(got, y, bound, got.dtype)
        if R < D:
            assert torch.equal(got[..., R:].cpu(), (q if got is out[0] else k)[..., R:])


@pytest.mark.parametrize("G", [1, 4, 7, 8])
@pytest.mark.parametrize("Hk", [1, 2, 8])
def test_heads(Hk, G):
    desc, rope, pos, q, k, want = _case(G, 5, Hk, G, 128, 128, "bf16")
    out = [torch.empty_like(x, device=DEV) for x in (q, k)]
    pe.pe_rotate(desc, rope, False, pos, q.to(DEV), k.to(DEV), None, *out)
    for got, (y, bound) in zip(out, want):
        assert_close(got, y, bound, got.dtype)


def test_very_many_heads():
    desc, rope, pos, q, k, want = _case(1, 2, 30000, 2, 64, 64, "bf16")
    out = [torch.empty_like(x, device=DEV) for x in (q, k)]
    pe.pe_rotate(desc, rope, False, pos, q.to(DEV), k.to(DEV), None, *out)
    for got, (y, bound) in zip(out, want):
        assert_close(got, y, bound, got.dtype)


@pytest.mark.parametrize("Hk,G,D,dt", [(2, 3, 64, "f32"), (1, 1, 64, "bf16"), (1, 2, 128, "bf16"), (2, 4, 128, "bf16")])
@pytest.mark.parametrize("T", [1, 2, 63, 300, 2049, 4097, 8195, 16385])
def test_tokens(T, Hk, G, D, dt):
    """One token a workgroup, and up to eight."""
    desc, rope, pos, q, k, want = _case(T, T, Hk, G, D, D, dt)
    out = [torch.empty_like(x, device=DEV) for x in (q, k)]
    pe.pe_rotate(desc, rope, False, pos, q.to(DEV), k.to(DEV), None, *out)
    for got, (y, bound) in zip(out, want):
        assert_close(got, y, bound, got.dtype)
    ko = torch.empty_like(k, device=DEV)   # one kind of heads alone
    pe.pe_rotate(desc, rope, False, pos, None, k.to(DEV), None, None, ko)
    assert torch.equal(ko, out[1])


def test_far_and_negative_positions():
    pos = torch.tensor([0, 1, -1, 2 ** 20 + 1, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1, -2 ** 31, -123457], dtype=torch.int32)
    desc, rope, p, q, k, want = _case(3, len(pos), 2, 2, 64, 64, "f32", positions=pos)
    out = [torch.empty_like(x, device=DEV) for x in (q, k)]
    pe.pe_rotate(desc, rope, False, p, q.to(DEV), k.to(DEV), None, *out)
    for got, (y, bound) in zip(out, want):
        assert_close(got, y, bound, got.dtype)


def test_position_zero_changes_nothing():
    desc, rope, _, q, k, _ = _case(4, 6, 2, 2, 128, 128, "bf16")
    out = [torch.empty_like(x, device=DEV) for x in (q, k)]
    pe.pe_rotate(desc, rope, False, torch.zeros(6, dtype=torch.int32, device=DEV), q.to(DEV), k.to(DEV), None, *out)
    assert torch.equal(out[0].cpu(), q) and torch.equal(out[1].cpu(), k)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("R", [64, 10])
def test_transpose_is_the_gradient(R, inter):
    """The formula's gradient, a difference quotient's, and the way there and back."""
    desc, rope, pos, q, k, want = _case(5, 9, 2, 2, 64, R, "f32", inter, "parts", magnitude=1.5, transpose=True)
    dq, dk = (torch.empty_like(x, device=DEV) for x in (q, k))
    pe.pe_rotate(desc, rope, True, pos, q.to(DEV), k.to(DEV), None, dq, dk)
    for got, (y, bound) in zip((dq, dk), want):
        assert_close(got, y, bound, got.dtype)
    # <w, rotate(x)> as a function of x, along one direction e: linear, so that the difference is exact but for rounding
    g = torch.Generator().manual_seed(6)
    x, e = (torch.randn(q.shape, generator=g) for _ in range(2))
    ys = [torch.empty_like(q, device=DEV) for _ in range(2)]
    kk = [torch.empty_like(k, device=DEV) for _ in range(2)]
    for y, s, z in zip(ys, (1.0, -1.0), kk):
        pe.pe_rotate(desc, rope, False, pos, (x + s * e).to(DEV), k.to(DEV), None, y, z)
    there = (q.double() * (ys[0] - ys[1]).double().cpu()).sum() / 2
    here = (dq.double().cpu() * e.double()).sum()
    # both sums are off by 8 + 2 half steps of each turned pair, and the inputs by one
    scale = 1.5 * (q.abs().double().mean() * (x.abs() + e.abs()).double().mean() * 2 * q.numel())
    assert abs(float(there - here)) <= 24 * 2.0 ** -24 * float(scale)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("R", [128, 44])
def test_in_place_in_one_row_a_token(R, dt):
    """Queries, keys and values side by side, as a projection leaves them; the values stay."""
    desc, rope, pos, q, k, want = _case(7, 33, 2, 4, 128, R, dt)
    row = torch.cat((q, k, torch.randn(k.shape).to(k.dtype)), 1).to(DEV)
    v = row[:, 10:].clone()
    pe.pe_rotate(desc, rope, False, pos, row[:, :8], row[:, 8:10], None, row[:, :8], row[:, 8:10])
    for got, (y, bound) in zip((row[:, :8], row[:, 8:10]), want):
        assert_close(got, y, bound, got.dtype)
    assert torch.equal(row[:, 10:], v)


@pytest.mark.parametrize("offset", [1, 4])
def test_rows_that_begin_anywhere(offset):
    """Neither 16-byte aligned nor a multiple of 16 bytes apart."""
    desc, rope, pos, q, k, want = _case(8, 12, 2, 2, 64, 64, "bf16")
    width = 4 * 64 + offset
    store = torch.zeros(12 * width + offset, dtype=torch.bfloat16, device=DEV)
    rows = store[offset:].as_strided((12, 4, 64), (width, 64, 1))
    rows.copy_(q)
    ko = torch.empty_like(k, device=DEV)
    pe.pe_rotate(desc, rope, False, pos, rows, k.to(DEV), None, rows, ko)
    assert_close(rows, *want[0], torch.bfloat16)
    assert_close(ko, *want[1], torch.bfloat16)


def test_queries_or_keys_alone_and_no_tokens():
    desc, rope, pos, q, k, want = _case(9, 7, 2, 2, 64, 64, "f32")
    qo, ko = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV)
    pe.pe_rotate(desc, rope, False, pos, q.to(DEV), None, None, qo, None)
    pe.pe_rotate(desc, rope, False, pos, None, k.to(DEV), None, None, ko)
    assert_close(qo, *want[0], torch.float32)
    assert_close(ko, *want[1], torch.float32)
    pe.pe_rotate(desc, rope, False, pos[:0], q[:0].to(DEV), k[:0].to(DEV), None, qo[:0], ko[:0])


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("dt,D,R", [("bf16", 128, 128), ("f32", 64, 32), ("bf16", 64, 22)])
def test_into_the_pages(dt, D, R, shared, keep):
    """Keys turned and values as they are, by slots: -1 and what is no slot are left out, other slots untouched."""
    T, Hk, G, B, P = 21, 3, 2, 16, 7
    desc, rope, pos, q, k, want = _case(11, T, Hk, G, D, R, dt)
    g = torch.Generator().manual_seed(12)
    v = torch.randn(k.shape, generator=g).to(k.dtype)
    desc = pe.make_desc(k.dtype, 1, Hk, Hk * G, D, B, 1, P, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    n = T if shared else T * Hk
    slots = torch.randperm(P * B, generator=g)[:n]
    slots[2], slots[5], slots[n - 1] = -1, P * B, -2 ** 40
    slots = slots if shared else slots.view(T, Hk)
    shape = (P, B, Hk, D) if shared else (P, B, D)
    kp, vp = (torch.full(shape, 9.0, dtype=k.dtype, device=DEV) for _ in range(2))
    qo, ko = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV) if keep else None
    pe.pe_rotate(desc, rope, False, pos, q.to(DEV), k.to(DEV), v.to(DEV), qo, ko, slots.to(DEV), kp, vp)
    torch.cuda.synchronize()
    assert_close(qo, *want[0], q.dtype)
    y, bound = want[1]
    flat = lambda x: x.cpu().reshape((P * B,) + ((Hk,) if shared else ()) + (D,))   # noqa: E731
    hit = torch.zeros(P * B, dtype=torch.bool)
    for t in range(T):
        for h in range(1 if shared else Hk):
            at = int(slots[t] if shared else slots[t, h])
            if 0 <= at < P * B:
                hit[at] = True
                part = slice(None) if shared else h
                assert_close(flat(kp)[at], y[t, part], bound[t, part], k.dtype)
                assert torch.equal(flat(vp)[at], v[t, part])
    assert bool((flat(kp)[~hit] == 9.0).all()) and bool((flat(vp)[~hit] == 9.0).all())
    if keep:
        assert_close(ko, y, bound, k.dtype)


def test_non_finite_elements_stay_in_their_pair():
    desc, rope, pos, q, k, want = _case(13, 3, 1, 1, 64, 64, "f32")
    q[1, 0, 5] = float("inf")
    q[2, 0, 40] = float("nan")
    qo, ko = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV)
    pe.pe_rotate(desc, rope, False, pos, q.to(DEV), k.to(DEV), None, qo, ko)
    bad = ~torch.isfinite(qo.cpu())
    assert set(map(tuple, bad.nonzero().tolist())) <= {(1, 0, 5), (1, 0, 37), (2, 0, 8), (2, 0, 40)} and bool(bad[1, 0, 5]) and bool(bad[2, 0, 40])


def test_on_another_stream():
    desc, rope, pos, q, k, want = _case(14, 50, 2, 2, 64, 64, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        qd, kd = q.to(DEV), k.to(DEV)
        pe.pe_rotate(desc, rope, False, pos, qd, kd, None, qd, kd)
    side.synchronize()
    assert_close(qd, *want[0], torch.bfloat16)
    assert_close(kd, *want[1], torch.bfloat16)


@pytest.mark.parametrize("shared", [False, True])
def test_slots_of_other_tokens_are_refused(shared):
    d = pe.make_desc(torch.bfloat16, 1, 2, 4, 64, 16, 4, 8, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
    on = dict(dtype=torch.bfloat16, device=DEV)
    q, k, pool = torch.zeros((5, 4, 64), **on), torch.zeros((5, 2, 64), **on), torch.zeros((2, 8, 16) + (2,) * shared + (64,), **on)
    for n in (0, 4, 6):
        slots = torch.full((n,) if shared else (n, 2), -1, dtype=torch.int64, device=DEV)
        with pytest.raises(ValueError, match="slots must be"):
            pe.pe_rotate(d, pe.make_rope(64, 1e4), False, torch.zeros(5, dtype=torch.int32, device=DEV), q, k, k.clone(), q.clone(), None, slots,
                         pool[0], pool[1])
