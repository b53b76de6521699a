"""What a plan of tokens with options, and a prune of its sequences, refuse before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2509_04377_amd import binding as pe

P = [ctypes.c_void_p(0x10000000000 * (i + 1)) for i in range(20)]   # never dereferenced: validation fails first
NAMES = ("lens", "new", "first", "free", "used", "table", "spare", "lens_out", "used_out", "cu", "pos", "slots")
AT = dict(zip(NAMES, P))


def _desc(**kw):
    d = dict(dtype=pe.PE_BF16, num_seqs=4, num_kv_heads=8, num_q_heads=32, head_dim=128, block_size=16, max_blocks=128, num_phys_blocks=4096)
    d.update(kw)
    return pe.make_desc(**d)


def _plan(n_spare=2, **opts):
    o = pe.pe_plan_opts()
    for name, x in opts.items():
        setattr(o, name, x.value if isinstance(x, ctypes.c_void_p) else x)
    a = AT
    return pe.lib().pe_plan_tokens_ex(ctypes.byref(_desc()), ctypes.byref(o), a["lens"], a["new"], a["first"], 100, 0, a["free"], 64,
                                      a["used"], a["table"], a["spare"], n_spare, a["lens_out"], a["used_out"], a["cu"], a["pos"], a["slots"], None)


@pytest.mark.parametrize("out", ["admitted", "spare_used", "freed_phys"])
@pytest.mark.parametrize("other", NAMES)
def test_what_is_written_lies_by_itself(out, other):
    assert _plan(**{out: AT[other]}) == pe.PE_ERR_INVALID_ARG
    assert _plan(admitted=P[15], spare_used=P[15]) == _plan(freed_phys=ctypes.c_void_p(P[15].value + 4 * 31), spare_used=P[15]) == pe.PE_ERR_INVALID_ARG


def test_options():
    assert _plan(copies=-1) == pe.PE_ERR_INVALID_ARG
    for out in ("lens_out", "table", "spare", "cu", "pos", "slots", "used_out"):
        assert _plan(only=AT[out]) == pe.PE_ERR_INVALID_ARG, out
    assert _plan(only=P[15], admitted=P[15]) == _plan(only=P[15], spare_used=P[15]) == _plan(only=P[15], freed_phys=P[15]) == pe.PE_ERR_INVALID_ARG


def test_the_prune_s_answer_and_lengths_are_apart():
    for shared in (pe.PE_LAYOUT_PER_HEAD, pe.PE_LAYOUT_SHARED):
        d = _desc(layout=shared)
        call = lambda admitted: pe.lib().pe_prefill_prune_admitted(   # noqa: E731
            ctypes.byref(d), P[0], P[1], P[2], admitted, 100, 50, 64, P[3], P[4], P[5], P[6], None, None, 0, None)
        assert call(P[6]) == call(ctypes.c_void_p(P[6].value + 12)) == pe.PE_ERR_INVALID_ARG
        assert call(P[7]) == call(None) == pe.PE_ERR_WORKSPACE      # (the check behind it)


def test_the_pages_answer_lies_by_itself():
    cache = pe.pe_quant_cache(*(p.value for p in P[:5]))
    call = lambda admitted: pe.lib().pe_quant_pages_admitted(   # noqa: E731
        ctypes.byref(_desc()), ctypes.byref(cache), admitted, P[5], P[6], P[7], P[8], P[9], P[10], None)
    for p in P[:5] + [P[10], ctypes.c_void_p(P[10].value - 12)]:
        assert call(p) == pe.PE_ERR_INVALID_ARG
