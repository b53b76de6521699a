"""Shapes whose launches would have 2^32 threads in a row of workgroups are refused on the host, before anything is launched (no GPU needed: what
fits is shown by the workspace that is missing then, not by a launch)."""
import ctypes

import pytest

from paper_2509_04377_amd import binding as pe

P = [ctypes.c_void_p((i + 1) << 42) for i in range(16)]   # never dereferenced: validation fails first
F = ctypes.c_float


def _desc(**kw):
    d = dict(dtype=pe.PE_BF16, num_seqs=4, num_kv_heads=1, num_q_heads=1, head_dim=64, block_size=16, max_blocks=1, num_phys_blocks=1 << 24)
    d.update(kw)
    return pe.make_desc(**d)


def _tree(T=1, **kw):
    return pe.lib().pe_tree_decode(ctypes.byref(_desc(**kw)), T, P[0], P[1], P[2], None, P[3], P[4], P[5], P[6], P[7], F(0.1), P[8], None, 0, None)


def _weights(**kw):
    return pe.lib().pe_paged_decode_weights(ctypes.byref(_desc(**kw)), P[0], P[1], P[2], P[3], P[4], F(0.1), F(1.0), None, P[5], P[6], None, 0, None)


@pytest.mark.parametrize("kw,T,want", [
    # 16 query rows a workgroup, two splits: 2^23 rows are too many, as are 2^24 with one
    (dict(num_seqs=(1 << 23) - 8, decode_splits=2), 1, pe.PE_ERR_WORKSPACE), (dict(num_seqs=1 << 23, decode_splits=2), 1, pe.PE_ERR_UNSUPPORTED),
    (dict(num_seqs=1 << 24, decode_splits=1), 1, pe.PE_ERR_UNSUPPORTED), (dict(num_seqs=1 << 24), 1, pe.PE_ERR_UNSUPPORTED),
    # few sequences and many heads, whose splits are in a grid's other dimension: the merge, a workgroup for four query rows, is what is too many
    (dict(num_seqs=8, num_kv_heads=32768, num_q_heads=8 * 32768, decode_splits=2), 31, pe.PE_ERR_WORKSPACE),
    (dict(num_seqs=8, num_kv_heads=32768, num_q_heads=8 * 32768, decode_splits=2), 32, pe.PE_ERR_UNSUPPORTED),
    # 256 query rows a workgroup, 64 workgroups that merge them
    (dict(num_seqs=1 << 17, num_q_heads=8, decode_splits=2), 32, pe.PE_ERR_WORKSPACE),
    (dict(num_seqs=1 << 18, num_q_heads=8, decode_splits=2), 32, pe.PE_ERR_UNSUPPORTED)])
def test_trees(kw, T, want):
    assert _tree(T, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(num_seqs=(1 << 23) - 8, decode_splits=2), pe.PE_ERR_WORKSPACE), (dict(num_seqs=1 << 23, decode_splits=2), pe.PE_ERR_UNSUPPORTED),
    (dict(num_seqs=512, num_kv_heads=65536, num_q_heads=65536), pe.PE_ERR_UNSUPPORTED)])
def test_weights(kw, want):
    assert _weights(**kw) == want


def test_paths():
    d = _desc(num_seqs=1 << 23)
    assert pe.lib().pe_append_path(ctypes.byref(d), 1, *P[:3], 1, *P[3:12], 1, None) == pe.PE_ERR_UNSUPPORTED


def test_pages():
    d = _desc(layout=pe.PE_LAYOUT_SHARED, num_kv_heads=8, num_q_heads=8, head_dim=128, max_blocks=1 << 27)
    for recent in (0, 1 << 27):
        assert pe.lib().pe_page_bounds(ctypes.byref(d), P[0], P[1], P[2], recent, P[3], None) == pe.PE_ERR_UNSUPPORTED
    for blocks, want in ((1 << 27, pe.PE_ERR_UNSUPPORTED), ((1 << 27) - 8, pe.PE_ERR_WORKSPACE)):
        d = _desc(max_blocks=blocks)
        assert pe.lib().pe_select_pages(ctypes.byref(d), *P[:4], 4, *P[4:7], None, 0, None) == want
