"""What the plan of tokens, the frequencies and the rotation refuse, before anything is launched (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from paper_2509_04377_amd import binding as pe

from _tokens64 import frequencies

P = [ctypes.c_void_p(0x10000000000 * (i + 1)) for i in range(14)]   # never dereferenced: validation fails first
BAD = ctypes.c_void_p(0x2000000003)


def _desc(**kw):
    d = dict(dtype=pe.PE_BF16, num_seqs=4, num_kv_heads=8, num_q_heads=32, head_dim=128, block_size=16, max_blocks=128, num_phys_blocks=4096)
    d.update(kw)
    return pe.make_desc(**d)


def _plan(desc, total=100, budget=0, num_free=64, n_spare=2, **at):
    a = dict(zip(("lens", "new", "first", "free", "used", "table", "spare", "lens_out", "used_out", "cu", "pos", "slots"), P))
    a.update(at)
    return pe.lib().pe_plan_tokens(ctypes.byref(desc) if desc else None, a["lens"], a["new"], a["first"], total, budget, a["free"], num_free,
                                   a["used"], a["table"], a["spare"], n_spare, a["lens_out"], a["used_out"], a["cu"], a["pos"], a["slots"], None)


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(block_size=8), dict(dtype=7), dict(num_q_heads=128), dict(layout=5)])
def test_shapes(kw):
    assert _plan(_desc(**kw)) == pe.PE_ERR_UNSUPPORTED
    assert _rotate(_desc(**kw)) == pe.PE_ERR_UNSUPPORTED


def test_plan_arguments():
    d = _desc()
    assert _plan(None) == pe.PE_ERR_INVALID_ARG
    for name in ("lens", "new", "free", "used", "table", "lens_out", "used_out"):
        assert _plan(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    for kw in (dict(total=-1), dict(total=2 ** 31), dict(budget=-16), dict(budget=40), dict(num_free=0), dict(n_spare=-1), dict(n_spare=0),
               dict(spare=None), dict(slots=ctypes.c_void_p(P[11].value + 4))):
        assert _plan(d, **kw) == pe.PE_ERR_INVALID_ARG, kw
    assert _plan(_desc(num_kv_heads=65537, num_q_heads=65537, num_seqs=1)) == pe.PE_ERR_UNSUPPORTED
    assert _plan(_desc(num_kv_heads=65536, num_q_heads=65536, num_seqs=1, max_blocks=32768)) == pe.PE_ERR_UNSUPPORTED


@pytest.mark.parametrize("out", ["table", "spare", "lens_out", "used_out", "cu", "pos", "slots"])
@pytest.mark.parametrize("other", ["lens", "new", "first", "free", "used", "table", "lens_out", "cu"])
def test_plan_outputs_lie_by_themselves(out, other):
    at = dict(zip(("lens", "new", "first", "free", "used", "table", "spare", "lens_out", "used_out", "cu", "pos", "slots"), P))
    if out != other:
        assert _plan(_desc(), **{out: at[other]}) == pe.PE_ERR_INVALID_ARG


def _rope(R=128, **kw):
    r = pe.pe_rope()
    a = dict(pairs=0, base=1e4, scaling=0, factor=1.0, low=1.0, high=4.0, original=8192.0, magnitude=1.0)
    a.update(kw)
    return pe.lib().pe_rope_init(ctypes.byref(r), R, a["pairs"], a["base"], a["scaling"], a["factor"], a["low"], a["high"], a["original"],
                                 a["magnitude"]), r


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("R,kw,want", [
    (0, {}, -1), (3, {}, -1), (-2, {}, -1), (130, {}, -2), (128, dict(pairs=2), -1), (128, dict(scaling=3), -1), (128, dict(base=1.0), -1),
    (128, dict(base=NAN), -1), (128, dict(base=INF), -1), (128, dict(magnitude=0.0), -1), (128, dict(magnitude=INF), -1),
    (128, dict(magnitude=NAN), -1), (128, dict(magnitude=1e-60), -1), (128, dict(magnitude=1e60), -1), (128, dict(scaling=1, factor=0.5), -1),
    (128, dict(scaling=1, factor=NAN), -1), (128, dict(scaling=2, factor=INF), -1), (128, dict(scaling=2, low=4.0), -1),
    (128, dict(scaling=2, low=-1.0), -1), (128, dict(scaling=2, high=INF), -1), (128, dict(scaling=2, original=0.0), -1),
    (128, dict(scaling=2, original=NAN), -1), (128, dict(factor=NAN, low=9.0, original=-1.0), 0)])
def test_frequencies_that_are_none(R, kw, want):
    status, r = _rope(R, **kw)
    assert status == want and r.filled == (1 if want == 0 else 0)
    assert pe.lib().pe_rope_init(None, 128, 0, 1e4, 0, 1.0, 1.0, 4.0, 8192.0, 1.0) == pe.PE_ERR_INVALID_ARG


@pytest.mark.parametrize("scaling,kw", [(0, {}), (1, dict(factor=8.0)), (2, dict(factor=8.0)), (2, dict(factor=32.0, low=0.5, high=32.0, original=4096.0))])
@pytest.mark.parametrize("R", [2, 30, 64, 128])
def test_frequencies(R, scaling, kw):
    """In turns, to the last bits of 64."""
    for base in (1e4, 5e5):
        status, r = _rope(R, base=base, scaling=scaling, **kw)
        assert status == pe.PE_OK
        want = frequencies(R, base, ("none", "linear", "parts")[scaling], **kw)
        for i, f in enumerate(want):
            # a power, a few products and a quotient in 64 bits; the number is a whole one of 2^-64 turns, rounded: half of one
            assert abs(r.turns[i] / 2.0 ** 64 - f / (2 * math.pi)) <= 2.0 ** -49 * f / (2 * math.pi) + 2.0 ** -65


def _rotate(desc, rope=None, tokens=50, transpose=0, qs=32 * 128, ks=8 * 128, vs=8 * 128, qos=32 * 128, kos=8 * 128, **at):
    a = dict(zip(("pos", "q", "k", "v", "q_out", "k_out", "slots", "k_pool", "v_pool"), P))
    a.update(at)
    rope = _rope()[1] if rope is None else rope
    return pe.lib().pe_rotate(ctypes.byref(desc) if desc else None, ctypes.byref(rope) if rope else None, transpose, tokens, a["pos"], a["q"], qs,
                              a["k"], ks, a["v"], vs, a["q_out"], qos, a["k_out"], kos, a["slots"], a["k_pool"], a["v_pool"], None)


def test_rotate_arguments():
    d = _desc()
    assert _rotate(None) == pe.PE_ERR_INVALID_ARG
    assert _rotate(d, rope=pe.pe_rope()) == pe.PE_ERR_INVALID_ARG          # not filled
    assert _rotate(_desc(head_dim=64)) == pe.PE_ERR_INVALID_ARG            # 128 elements of 64
    assert _rotate(d, tokens=-1) == pe.PE_ERR_INVALID_ARG
    assert _rotate(d, tokens=2 ** 31) == pe.PE_ERR_UNSUPPORTED
    for kw in (dict(pos=None), dict(q=None), dict(q_out=None), dict(k=None), dict(k=None, k_out=None), dict(v=None), dict(k_pool=None),
               dict(v_pool=None), dict(slots=None, k_out=None), dict(qs=32 * 128 - 1), dict(ks=0), dict(vs=-8), dict(qos=1), dict(kos=1023),
               dict(q=BAD), dict(k_out=BAD), dict(k_pool=ctypes.c_void_p(P[7].value + 8)), dict(slots=ctypes.c_void_p(P[6].value + 4)),
               dict(qs=2 ** 45)):
        assert _rotate(d, **kw) == pe.PE_ERR_INVALID_ARG, kw
    assert _rotate(_desc(num_kv_heads=65537, num_q_heads=65537, num_seqs=1), qs=1 << 24, ks=1 << 24, vs=1 << 24, qos=1 << 24, kos=1 << 24) == \
        pe.PE_ERR_UNSUPPORTED
    assert _rotate(d, tokens=0) == pe.PE_OK


def test_rotate_outputs_that_lie_on_something():
    d, near = _desc(), lambda i, n=16: ctypes.c_void_p(P[i].value + n)   # noqa: E731
    for kw in (dict(q_out=near(1)), dict(k_out=near(2)), dict(q_out=P[2]), dict(k_out=P[1]), dict(k_out=P[3]), dict(q_out=P[5]), dict(k_out=P[4]),
               dict(v_pool=P[7]), dict(k_pool=P[1]), dict(v_pool=P[3]), dict(k_pool=P[5]), dict(q_out=P[1], qos=32 * 128 + 8)):
        assert _rotate(d, **kw) == pe.PE_ERR_INVALID_ARG, kw
    for kw in (dict(q_out=P[0]), dict(k_out=near(0, 128)), dict(q_out=P[6]), dict(k_out=near(6, 64))):   # positions, slots
        assert _rotate(d, **kw) == pe.PE_ERR_INVALID_ARG, kw
    # parts of one row a token: in place is fine (the check behind it is reached), the neighbour's place is not
    row = 48 * 128
    side = dict(qs=row, ks=row, vs=row, qos=row, kos=row, q=P[1], k=near(1, 2 * 32 * 128), v=near(1, 2 * 40 * 128))
    assert _rotate(d, **side, q_out=P[1], k_out=near(1, 2 * 40 * 128)) == pe.PE_ERR_INVALID_ARG
    assert _rotate(d, **side, q_out=near(1, 2 * 16 * 128), k_out=P[5]) == pe.PE_ERR_INVALID_ARG


def test_tensors_are_checked_before_the_call():
    x, p = torch.zeros((3, 8, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    d, rope = _desc(num_q_heads=8, head_dim=64), pe.make_rope(64, 1e4)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        pe.pe_rotate(d, rope, False, p, x, x, None, x, x)
    with pytest.raises(ValueError, match="seq_lens must be a GPU tensor"):
        pe.pe_plan_tokens(d, p, p, None, 1, 0, p, p, p, None, p, p, None, None, None)
    with pytest.raises(pe.PeError):
        pe.make_rope(63, 1e4)
