"""What the calls for trees of drafts refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2509_04377_amd import binding as pe

P = [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(16)]   # never dereferenced: validation fails first
F = ctypes.c_float


def _desc(**kw):
    d = dict(dtype=pe.PE_BF16, num_seqs=4, num_kv_heads=8, num_q_heads=32, head_dim=128, block_size=16, max_blocks=128,
             num_phys_blocks=4096)
    d.update(kw)
    return pe.make_desc(**d)


def _tree(desc, T=8, scale=0.1, ws=P[15], n=1 << 30, **at):
    a = dict(q=P[0], k_draft=P[1], v_draft=P[2], draft_lens=None, mask=P[3], k_pool=P[4], v_pool=P[5], table=P[6], lens=P[7], out=P[8])
    a.update(at)
    return pe.lib().pe_tree_decode(ctypes.byref(desc) if desc else None, T, a["q"], a["k_draft"], a["v_draft"], a["draft_lens"], a["mask"],
                                   a["k_pool"], a["v_pool"], a["table"], a["lens"], F(scale), a["out"], ws, n, None)


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(block_size=8), dict(dtype=7), dict(num_q_heads=128), dict(layout=5)])
def test_tree_refuses_shapes_it_is_not_built_for(kw):
    assert _tree(_desc(**kw)) == pe.PE_ERR_UNSUPPORTED
    assert pe.pe_workspace_bytes(pe.PE_OP_TREE_DECODE, _desc(**kw), 8) == 0


def test_tree_refuses_arguments():
    d = _desc()
    assert _tree(None) == pe.PE_ERR_INVALID_ARG
    assert _tree(d, 0) == pe.PE_ERR_INVALID_ARG and _tree(d, -1) == pe.PE_ERR_INVALID_ARG
    assert _tree(d, pe.PE_MAX_DRAFTS + 1) == pe.PE_ERR_UNSUPPORTED
    for name in ("q", "k_draft", "v_draft", "mask", "k_pool", "v_pool", "table", "lens", "out"):
        assert _tree(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    for name in ("q", "k_draft", "v_draft", "k_pool", "v_pool", "mask"):
        assert _tree(d, **{name: ctypes.c_void_p(0x900004)}) == pe.PE_ERR_INVALID_ARG, name
    assert _tree(d, out=ctypes.c_void_p(0x900001)) == pe.PE_ERR_INVALID_ARG
    for scale in (float("nan"), float("inf")):
        assert _tree(d, scale=scale) == pe.PE_ERR_INVALID_ARG
    for name in ("k_draft", "v_draft", "q"):   # (out may be q itself, nothing else)
        assert _tree(d, **{name: ctypes.c_void_p(P[8].value + 16)}) == pe.PE_ERR_INVALID_ARG, name
    assert _tree(_desc(num_seqs=1 << 20, num_kv_heads=8), 64) == pe.PE_ERR_UNSUPPORTED


def test_tree_workspace():
    d = _desc(decode_splits=3)
    need = pe.pe_workspace_bytes(pe.PE_OP_TREE_DECODE, d, 8)
    assert need == 4 * 32 * 8 * 3 * (128 + 2) * 4
    assert _tree(d, ws=None, n=0) == pe.PE_ERR_WORKSPACE
    assert _tree(d, n=need - 1) == pe.PE_ERR_WORKSPACE
    assert _tree(d, ws=ctypes.c_void_p(0x1010), n=need) == pe.PE_ERR_WORKSPACE
    assert pe.pe_workspace_bytes(pe.PE_OP_TREE_DECODE, _desc(decode_splits=1), 8) == 0
    for T in (0, -1, 65):
        assert pe.pe_workspace_bytes(pe.PE_OP_TREE_DECODE, d, T) == 0


def test_path_refuses_arguments():
    L = pe.lib()

    def path(desc, T=8, most=4, slots=2, **at):
        names = ("k_draft", "v_draft", "path", "path_lens", "path_done", "k_pool", "v_pool", "table", "lens", "freed", "spare", "used")
        a = dict(zip(names, P))
        a.update(at)
        return L.pe_append_path(ctypes.byref(desc) if desc else None, T, a["k_draft"], a["v_draft"], a["path"], most, a["path_lens"],
                                a["path_done"], a["k_pool"], a["v_pool"], a["table"], a["lens"], a["freed"], a["spare"], a["used"], slots, None)

    d = _desc()
    assert path(None) == pe.PE_ERR_INVALID_ARG
    for kw in (dict(T=0), dict(most=0), dict(slots=0)):
        assert path(d, **kw) == pe.PE_ERR_INVALID_ARG
    for name in ("k_draft", "v_draft", "path", "path_lens", "path_done", "k_pool", "v_pool", "table", "lens", "freed", "spare", "used"):
        assert path(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    for name in ("k_draft", "v_draft", "k_pool", "v_pool"):
        assert path(d, **{name: ctypes.c_void_p(0x900008)}) == pe.PE_ERR_INVALID_ARG, name
    assert path(_desc(num_seqs=1, num_kv_heads=65537, num_q_heads=65537)) == pe.PE_ERR_UNSUPPORTED
    assert path(_desc(block_size=24)) == pe.PE_ERR_UNSUPPORTED


def test_tensors_are_checked_before_the_call():
    x = torch.zeros((1, 8, 4, 64))
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        pe.pe_tree_decode(_desc(), 8, x, x, x, None, x, x, x, x, x, 0.1, x)
    with pytest.raises(ValueError, match="k_draft must be a GPU tensor"):
        pe.pe_append_path(_desc(), x, x, x, x, x, x, x, x, x, x, x, x)
