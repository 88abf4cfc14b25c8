"""Host side of the 4-bit cache attention's plan: workspaces and refusals (no pointer is read)."""

import ctypes

import numpy as np
import pytest

from paper_2606_04446_amd import d2sd

FAKE = 1 << 20


def args(**kw):
    return d2sd.AttnArgs(**{**dict(
        batch=1, num_qo_heads=32, num_kv_heads=8, head_dim=128, page_size=16, dtype=d2sd.BF16, stage=d2sd.STAGE_CASCADE,
        total_nodes=16, max_nodes=16, max_ctx_len=4096, num_pages=1 << 20, max_pages=1 << 18, mask_words=65, q=FAKE,
        page_table=FAKE, ctx_len=FAKE, k_tree=FAKE, v_tree=FAKE, node_indptr=FAKE, anc_mask=FAKE, out=FAKE, lse=None), **kw})


def need(**kw):
    n = ctypes.c_size_t(7)
    st = d2sd._ws_size_kv4(ctypes.byref(args(**kw)), ctypes.byref(n))
    return n.value if st == d2sd.OK else st


def test_workspace_only_where_streams_are_cut():
    assert need() > 0
    assert need(max_ctx_len=0) == 0 and need(stage=d2sd.STAGE_TREE) == 0
    assert need(max_ctx_len=100) == 0
    assert need(max_ctx_len=100, kv_split=64) > 0          # an explicit share is kept to
    # many short contexts are one workgroup each, ragged long ones are shared out
    many = dict(batch=64, total_nodes=64, max_nodes=1)
    assert need(max_ctx_len=1000, **many) == 0 and need(max_ctx_len=16000, **many) > 0
    # no more than two states per workgroup of 128 rows, whatever the contexts are
    most = 2 * 512 * 128 * 130 * 4 + 512 * 32
    for ctx in (5000, 100000, 1 << 20):
        assert 0 < need(max_ctx_len=ctx, total_nodes=600, max_nodes=600) <= most


@pytest.mark.parametrize("dtype", [d2sd.F32, d2sd.BF16])
def test_host_offsets_count_the_rows(dtype):
    """With the request's offsets the plan counts rows exactly; the need does not fail for empty ones."""
    ip = np.array([0, 0, 70, 70, 71], np.int32)
    a = dict(batch=4, total_nodes=71, max_nodes=70, max_ctx_len=30000, dtype=dtype)
    assert need(node_indptr_host=ip.ctypes.data, **a) > 0
    assert need(**a) > 0


def test_refusals():
    big = dict(total_nodes=2080, max_nodes=2080, num_qo_heads=64)
    assert need(max_ctx_len=200000, **big) > 1
    got = []
    for ctx in (200000, 280000, 1 << 20):
        n = ctypes.c_size_t(7)
        got.append(d2sd._ws_size_kv4(ctypes.byref(args(max_ctx_len=ctx, **big)), ctypes.byref(n)))
    assert got == [d2sd.OK, d2sd.ERR_UNSUPPORTED, d2sd.ERR_UNSUPPORTED]
    n = ctypes.c_size_t(7)
    for bad in (dict(kv_split=32), dict(kv_split=-64), dict(k_cache=FAKE), dict(row_group=128), dict(packed=1), dict(max_nodes=0)):
        assert d2sd._ws_size_kv4(ctypes.byref(args(**bad)), ctypes.byref(n)) != d2sd.OK, bad
