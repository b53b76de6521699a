"""What the calls for selected pages refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2509_04377_amd import binding as pe

P = [ctypes.c_void_p(0x1000000 * (i + 1)) for i in range(16)]   # never dereferenced: validation fails first


def _desc(**kw):
    d = dict(dtype=pe.PE_BF16, num_seqs=4, num_kv_heads=8, num_q_heads=32, head_dim=128, block_size=16, max_blocks=128,
             num_phys_blocks=4096)
    d.update(kw)
    return pe.make_desc(**d)


def _bounds(desc, recent=0, **at):
    a = dict(zip(("k_pool", "table", "lens", "bounds"), P))
    a.update(at)
    return pe.lib().pe_page_bounds(ctypes.byref(desc) if desc else None, a["k_pool"], a["table"], a["lens"], recent, a["bounds"], None)


def _select(desc, k=8, ws=P[15], n=1 << 30, **at):
    a = dict(zip(("q", "bounds", "table", "lens", "to", "lens_out", "idx"), P))
    a.update(at)
    return pe.lib().pe_select_pages(ctypes.byref(desc) if desc else None, a["q"], a["bounds"], a["table"], a["lens"], k, a["to"], a["lens_out"],
                                    a["idx"], ws, n, None)


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(block_size=8), dict(dtype=7), dict(num_q_heads=128), dict(layout=5)])
def test_shapes(kw):
    assert _bounds(_desc(**kw)) == pe.PE_ERR_UNSUPPORTED and _select(_desc(**kw)) == pe.PE_ERR_UNSUPPORTED
    assert pe.pe_workspace_bytes(pe.PE_OP_SELECT_PAGES, _desc(**kw)) == 0


def test_arguments():
    d = _desc()
    assert _bounds(None) == pe.PE_ERR_INVALID_ARG and _select(None) == pe.PE_ERR_INVALID_ARG
    assert _bounds(d, -1) == pe.PE_ERR_INVALID_ARG
    for name in ("k_pool", "table", "lens", "bounds"):
        assert _bounds(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    for name in ("k_pool", "bounds"):
        assert _bounds(d, **{name: ctypes.c_void_p(0x9000008)}) == pe.PE_ERR_INVALID_ARG, name
    for name in ("q", "bounds", "table", "lens", "to", "lens_out"):
        assert _select(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    for name in ("q", "bounds"):
        assert _select(d, **{name: ctypes.c_void_p(0x9000008)}) == pe.PE_ERR_INVALID_ARG, name
    for k in (0, -1):
        assert _select(d, k) == pe.PE_ERR_INVALID_ARG
    # an output in what the other rows still read
    table = ctypes.c_void_p(P[2].value + 4 * 8 * 128 * 4 - 4)
    for name in ("to", "idx", "lens_out"):
        assert _select(d, **{name: table}) == pe.PE_ERR_INVALID_ARG, name
        assert _select(d, **{name: P[3]}) == pe.PE_ERR_INVALID_ARG, name


def test_workspace():
    d = _desc()
    need = pe.pe_workspace_bytes(pe.PE_OP_SELECT_PAGES, d)
    assert need >= 4 * 8 * 128 * 4
    assert _select(d, ws=None, n=0) == pe.PE_ERR_WORKSPACE
    assert _select(d, n=need - 1) == pe.PE_ERR_WORKSPACE
    assert _select(d, ws=ctypes.c_void_p(0x9000080), n=need) == pe.PE_ERR_WORKSPACE


def test_tensors_are_checked_before_the_call():
    x = torch.zeros((1, 8, 64))
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        pe.pe_select_pages(_desc(), x, x, x, x, 4, x, x, None, None)
    with pytest.raises(ValueError, match="k_pool must be a GPU tensor"):
        pe.pe_page_bounds(_desc(), x, x, x, 0, x)
