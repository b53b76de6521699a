"""What the attention with page weights refuses, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2509_04377_amd import binding as pe

P = [ctypes.c_void_p(0x10000000 * (i + 1)) for i in range(12)]   # never dereferenced: validation fails first
F = ctypes.c_float


def _desc(**kw):
    d = dict(dtype=pe.PE_BF16, num_seqs=4, num_kv_heads=8, num_q_heads=32, head_dim=128, block_size=16, max_blocks=128,
             num_phys_blocks=4096, decode_splits=2)
    d.update(kw)
    return pe.make_desc(**d)


def _call(desc, scale=0.1, decay=1.0, ws=P[11], n=1 << 30, **at):
    a = dict(zip(("q", "k_pool", "v_pool", "table", "lens", "w_in", "w_out", "out"), P))
    a.update(at)
    return pe.lib().pe_paged_decode_weights(ctypes.byref(desc) if desc else None, a["q"], a["k_pool"], a["v_pool"], a["table"], a["lens"],
                                            F(scale), F(decay), a["w_in"], a["w_out"], a["out"], ws, n, None)


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(block_size=8), dict(dtype=7), dict(num_q_heads=128), dict(layout=5)])
def test_shapes(kw):
    assert _call(_desc(**kw)) == pe.PE_ERR_UNSUPPORTED
    assert pe.pe_workspace_bytes(pe.PE_OP_DECODE_WEIGHTS, _desc(**kw)) == 0


def test_table_rows_that_256_splits_do_not_cover():
    most = 256 * (61440 // 8) // 128   # pages of 128 tokens, eight query heads a KV head
    fits, over = (_desc(num_q_heads=64, block_size=128, max_blocks=most + i) for i in (0, 1))
    assert pe.pe_workspace_bytes(pe.PE_OP_DECODE_WEIGHTS, fits) > 0
    assert pe.pe_workspace_bytes(pe.PE_OP_DECODE_WEIGHTS, over) == 0
    assert _call(over) == pe.PE_ERR_UNSUPPORTED


def test_arguments():
    d = _desc()
    assert _call(None) == pe.PE_ERR_INVALID_ARG
    for name in ("q", "k_pool", "v_pool", "table", "lens", "w_out", "out"):
        assert _call(d, **{name: None}) == pe.PE_ERR_INVALID_ARG, name
    for name in ("q", "k_pool", "v_pool"):
        assert _call(d, **{name: ctypes.c_void_p(0x98000008)}) == pe.PE_ERR_INVALID_ARG, name
    for name in ("w_in", "w_out"):
        assert _call(d, **{name: ctypes.c_void_p(0x98000002)}) == pe.PE_ERR_INVALID_ARG, name
    for scale in (float("nan"), float("inf")):
        assert _call(d, scale=scale) == pe.PE_ERR_INVALID_ARG
    for decay in (float("nan"), float("inf"), -0.1, 1.5):
        assert _call(d, decay=decay) == pe.PE_ERR_INVALID_ARG
    beside = lambda i: ctypes.c_void_p(P[i].value + 16)   # noqa: E731
    for kw in (dict(w_in=beside(6)), dict(w_out=beside(0)), dict(w_out=beside(7)), dict(w_in=beside(7)), dict(out=beside(0))):
        assert _call(d, **kw) == pe.PE_ERR_INVALID_ARG, kw
    assert _call(_desc(num_kv_heads=65537, num_q_heads=65537, num_seqs=1)) == pe.PE_ERR_UNSUPPORTED


def test_workspace():
    d = _desc()
    need = pe.pe_workspace_bytes(pe.PE_OP_DECODE_WEIGHTS, d)
    assert need >= 4 * 32 * (2 * (128 + 2) + 128) * 4
    assert _call(d, ws=None, n=0) == pe.PE_ERR_WORKSPACE
    assert _call(d, n=need - 1) == pe.PE_ERR_WORKSPACE
    assert _call(d, ws=ctypes.c_void_p(0xb8000010), n=need) == pe.PE_ERR_WORKSPACE
    assert pe.pe_workspace_bytes(pe.PE_OP_DECODE_WEIGHTS, _desc(decode_splits=1)) == 0


def test_tensors_are_checked_before_the_call():
    x = torch.zeros((1, 8, 64))
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        pe.pe_paged_decode_weights(_desc(), x, x, x, x, x, 0.1, 1.0, None, x, x)
