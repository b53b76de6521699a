"""What the calls of the cache in 8 bits refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2509_04377_amd import binding as pe

P = [ctypes.c_void_p(0x10000000000 * (i + 1)) for i in range(20)]   # never dereferenced: validation fails first


def _at(i, n):
    return ctypes.c_void_p(P[i].value + n)


def _desc(**kw):
    d = dict(dtype=pe.PE_BF16, num_seqs=4, num_kv_heads=8, num_q_heads=32, head_dim=128, block_size=16, max_blocks=128, num_phys_blocks=4096,
             decode_splits=2)
    d.update(kw)
    return pe.make_desc(**d)


def _cache(**at):
    a = dict(zip(("k", "v", "scales", "k_tail", "v_tail"), (p.value for p in P[:5])))
    a.update(at)
    return pe.pe_quant_cache(a["k"], a["v"], a["scales"], a["k_tail"], a["v_tail"])


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _pages(desc, cache="", **at):
    a = dict(zip(("k_pool", "v_pool", "src", "lens", "table", "scores"), P[5:]))
    a.update(at)
    return pe.lib().pe_quant_pages(_ref(desc), _ref(_cache() if cache == "" else cache), a["k_pool"], a["v_pool"], a["src"], a["lens"], a["table"],
                                   a["scores"], None)


def _append(desc, cache="", rope="", n_spare=2, **at):
    a = dict(zip(("pos", "q", "q_out", "k", "v", "table", "lens", "lens_out", "freed", "spare", "used", "scores"), P[5:]))
    a.update(at)
    return pe.lib().pe_quant_append(_ref(desc), _ref(_cache() if cache == "" else cache), _ref(pe.make_rope(64, 1e4) if rope == "" else rope),
                                    a["pos"], a["q"], a["q_out"], a["k"], a["v"], a["table"], a["lens"], a["lens_out"], a["freed"], a["spare"],
                                    a["used"], n_spare, a["scores"], None)


def _decode(desc, cache="", scale=0.1, ws=P[10], n=1 << 30, **at):
    a = dict(zip(("q", "table", "lens", "out"), P[5:]))
    a.update(at)
    return pe.lib().pe_quant_decode(_ref(desc), _ref(_cache() if cache == "" else cache), a["q"], a["table"], a["lens"], ctypes.c_float(scale),
                                    a["out"], ws, n, None)


CALLS = (_pages, _append, _decode)


@pytest.mark.parametrize("call", CALLS)
def test_descriptors_and_caches(call):
    for kw in (dict(head_dim=96), dict(block_size=8), dict(dtype=7), dict(num_q_heads=128), dict(layout=5)):
        assert call(_desc(**kw)) == pe.PE_ERR_UNSUPPORTED
        assert pe.pe_workspace_bytes(pe.PE_OP_QUANT_DECODE, _desc(**kw)) == 0
    assert call(None) == pe.PE_ERR_INVALID_ARG
    assert call(_desc(), cache=None) == pe.PE_ERR_INVALID_ARG
    for name, off in (("k", 8), ("v", 8), ("scales", 4), ("k_tail", 8), ("v_tail", 8)):
        for bad in (None, 0x9900000000 + off):
            assert call(_desc(), cache=_cache(**{name: bad})) == pe.PE_ERR_INVALID_ARG, name


def test_pages():
    d = _desc()
    for name in ("k_pool", "v_pool", "src", "lens", "table"):
        assert _pages(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    assert _pages(d, k_pool=_at(5, 8)) == pe.PE_ERR_INVALID_ARG
    assert _pages(d, v_pool=_at(6, 8)) == pe.PE_ERR_INVALID_ARG
    assert _pages(d, scores=_at(10, 2)) == pe.PE_ERR_INVALID_ARG
    assert _pages(_desc(num_seqs=1 << 20, max_blocks=2)) == pe.PE_ERR_UNSUPPORTED      # more workgroups than a launch has


def test_append():
    d = _desc()
    for name in ("k", "v", "table", "lens", "lens_out", "freed", "spare", "used", "pos", "q", "q_out"):
        assert _append(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    for i, name in ((6, "q"), (7, "q_out"), (8, "k"), (9, "v")):
        assert _append(d, **{name: _at(i, 8)}) == pe.PE_ERR_INVALID_ARG, name
    assert _append(d, n_spare=0) == pe.PE_ERR_INVALID_ARG
    assert _append(d, rope=pe.pe_rope()) == pe.PE_ERR_INVALID_ARG
    assert _append(_desc(head_dim=64), rope=pe.make_rope(128, 1e4)) == pe.PE_ERR_INVALID_ARG
    assert _append(d, lens_out=P[11]) == pe.PE_ERR_INVALID_ARG                         # the lengths themselves
    assert _append(d, lens_out=_at(11, 4)) == pe.PE_ERR_INVALID_ARG
    for kw in (dict(q_out=_at(6, 16)), dict(q_out=P[8]), dict(q_out=P[9])):
        assert _append(d, **kw) == pe.PE_ERR_INVALID_ARG, kw
    assert _append(_desc(num_kv_heads=65537, num_q_heads=65537, num_seqs=1)) == pe.PE_ERR_UNSUPPORTED
    assert _append(_desc(num_seqs=1 << 20)) == pe.PE_ERR_UNSUPPORTED


def test_decode():
    d = _desc()
    for name in ("q", "table", "lens", "out"):
        assert _decode(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    assert _decode(d, q=_at(5, 8)) == pe.PE_ERR_INVALID_ARG
    assert _decode(d, out=_at(8, 1)) == pe.PE_ERR_INVALID_ARG
    assert _decode(_desc(dtype=pe.PE_F32), out=_at(8, 2)) == pe.PE_ERR_INVALID_ARG
    for scale in (float("nan"), float("inf")):
        assert _decode(d, scale=scale) == pe.PE_ERR_INVALID_ARG
    for kw in (dict(out=_at(5, 16)), dict(out=P[3]), dict(out=P[4])):
        assert _decode(d, **kw) == pe.PE_ERR_INVALID_ARG, kw
    need = pe.pe_workspace_bytes(pe.PE_OP_QUANT_DECODE, d)
    assert need == 2 * 4 * 32 * (128 + 2) * 4
    assert _decode(d, ws=None, n=0) == pe.PE_ERR_WORKSPACE
    assert _decode(d, n=need - 1) == pe.PE_ERR_WORKSPACE
    assert _decode(d, ws=_at(10, 16), n=need) == pe.PE_ERR_WORKSPACE
    assert pe.pe_workspace_bytes(pe.PE_OP_QUANT_DECODE, _desc(decode_splits=1)) == 0


PARTS = ("k", "v", "scales", "k_tail", "v_tail")


@pytest.mark.parametrize("call", CALLS)
def test_caches_whose_tensors_meet(call):
    for shared in (False, True):
        d = _desc(layout=pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD)
        rows = 4096 * (8 if shared else 1)
        size = dict(zip(PARTS, (rows * 16 * 128, rows * 16 * 128, rows * 8, 4 * 8 * 16 * 128 * 2, 4 * 8 * 16 * 128 * 2)))
        for i, one in enumerate(PARTS):
            for j, other in enumerate(PARTS):
                if i != j:   # `one` begins in the last 16 bytes of `other`
                    assert call(d, cache=_cache(**{one: P[j].value + size[other] - 16})) == pe.PE_ERR_INVALID_ARG, (one, other)


def test_tensors_on_the_cache():
    d = _desc()
    for i in range(5):
        for name in ("k_pool", "v_pool"):
            assert _pages(d, **{name: _at(i, 64)}) == pe.PE_ERR_INVALID_ARG, (name, i)
        for name in ("k", "v", "q_out"):
            assert _append(d, **{name: _at(i, 64)}) == pe.PE_ERR_INVALID_ARG, (name, i)
        assert _decode(d, out=_at(i, 64)) == pe.PE_ERR_INVALID_ARG, i
    assert _append(d, q_out=P[5]) == pe.PE_ERR_INVALID_ARG   # the positions


@pytest.mark.parametrize("kw,want", [
    # few splits of very many rows, four waves each; what fits lacks its workspace
    (dict(num_seqs=(1 << 23) - 8, decode_splits=2), pe.PE_ERR_WORKSPACE), (dict(num_seqs=1 << 23, decode_splits=2), pe.PE_ERR_UNSUPPORTED),
    # whole rows, eight waves each
    (dict(num_seqs=1 << 23, decode_splits=1), pe.PE_ERR_UNSUPPORTED), (dict(num_seqs=1 << 23, decode_splits=0), pe.PE_ERR_UNSUPPORTED),
    # the merge, with eight query rows to a row
    (dict(num_seqs=(1 << 20) - 8, num_q_heads=8, decode_splits=2), pe.PE_ERR_WORKSPACE),
    (dict(num_seqs=1 << 20, num_q_heads=8, decode_splits=2), pe.PE_ERR_UNSUPPORTED)])
def test_launches_of_too_many_threads(kw, want):
    base = dict(num_kv_heads=1, num_q_heads=1, head_dim=64, max_blocks=1, num_phys_blocks=1 << 24)
    far = dict(out=ctypes.c_void_p(1 << 60))
    cache = _cache(**{n: (i + 1) << 50 for i, n in enumerate(PARTS)})
    assert _decode(_desc(**dict(base, **kw)), cache=cache, ws=None, n=0, **far) == want


def test_too_many_heads():
    for call in CALLS:
        assert call(_desc(num_kv_heads=65537, num_q_heads=65537, num_seqs=1, max_blocks=2)) == pe.PE_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,want", [
    (dict(num_seqs=1, max_blocks=16), 1), (dict(num_seqs=1, max_blocks=17), 2), (dict(num_seqs=1, head_dim=64, max_blocks=32), 1),
    (dict(num_seqs=1, head_dim=64, max_blocks=33), 4), (dict(num_seqs=1, max_blocks=96), 12), (dict(num_seqs=1, max_blocks=104), 12),
    (dict(num_seqs=1, max_blocks=128), 12), (dict(num_seqs=1, max_blocks=136), 17), (dict(num_seqs=1, num_q_heads=64, max_blocks=96), 8),
    (dict(num_seqs=1, num_q_heads=64, max_blocks=104), 13), (dict(num_seqs=1, max_blocks=4096), 32),
    (dict(num_seqs=1, num_kv_heads=1, num_q_heads=4, max_blocks=4096), 64), (dict(num_seqs=8, max_blocks=64), 4), (dict(num_seqs=10, max_blocks=64), 3),
    (dict(num_seqs=11, max_blocks=63), 1), (dict(num_seqs=16, max_blocks=64), 2), (dict(num_seqs=17, max_blocks=127), 1),
    (dict(num_seqs=17, max_blocks=128), 3), (dict(num_seqs=20, max_blocks=128), 3), (dict(num_seqs=21, max_blocks=128), 4),
    (dict(num_seqs=24, max_blocks=128), 4), (dict(num_seqs=25, max_blocks=128), 1), (dict(num_seqs=32, max_blocks=4096), 1),
    (dict(num_seqs=33, max_blocks=128), 4), (dict(num_seqs=33, max_blocks=127), 1), (dict(num_seqs=41, max_blocks=128), 4),
    (dict(num_seqs=42, max_blocks=128), 1)])
@pytest.mark.parametrize("dtype", [pe.PE_BF16, pe.PE_F32])
def test_split_rule(kw, want, dtype):
    """At the edges, on a device of 256 compute units (what the library assumes without one)."""
    if torch.cuda.is_available() and torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("a device with another number of compute units")
    d = _desc(**dict(dict(decode_splits=0, dtype=dtype), **kw))
    assert pe.pe_workspace_bytes(pe.PE_OP_QUANT_DECODE, d) == (0 if want == 1 else want * d.num_seqs * d.num_q_heads * (d.head_dim + 2) * 4)


def test_tensors_are_checked_before_the_call():
    x, i = torch.zeros((1, 8, 64)), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        pe.make_quant_cache(_desc(), x, x, x, x, x)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        pe.pe_quant_pages(_desc(), _cache(), x, x, i, i, i)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        pe.pe_quant_decode(_desc(), _cache(), x, i, i, 0.1, x)
    with pytest.raises(ValueError, match="must be a GPU tensor"):
        pe.pe_quant_append(_desc(), _cache(), None, None, None, None, x, x, i, i, i, i, i, i)
